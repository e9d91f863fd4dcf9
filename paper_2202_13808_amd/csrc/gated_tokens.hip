// The gated projection's forward pass for few tokens (decoding): one pass over the weights.
//
// Bound by reading the weights: 16 tokens 4096 -> 10240 in bf16 35 us, 4.8 TB/s of them.  A workgroup of eight wavefronts takes
// 16 hidden columns, 16 gate rows and the 16 up rows of the same columns, each wavefront an eighth of the sum, so that even a
// small layer has enough loads in flight.  Both operands go from memory straight into the registers of the 16 x 16 matrix
// instructions, with no LDS between; the eighths meet in LDS, in ascending order.
//
// Lane l of an operand holds slot l % 16, so sixteen neighbouring lanes that were sixteen rows would touch sixteen cache
// lines a quarter of a load.  Instead the slots are 16 / P rows in P parts each: neighbouring lanes hold neighbouring 16 bytes
// of a row, and the instruction's result is the wanted product where a row's part meets the same part of a token; the rest of
// it is not used.  Matrix instructions are not what such a call waits for.
#include "common.hpp"
#include "dropit_layers.h"
#include "gated_act.hpp"
#include "gated_internal.hpp"

namespace dropit {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;

constexpr int TOK_THREADS = 512, TOK_WAVES = TOK_THREADS / WAVE, TOK_COLS = 16;

template <bool BF16, int P, int TG>
__global__ void __launch_bounds__(TOK_THREADS)
gated_tokens_kernel(const void *__restrict__ w, const void *__restrict__ x, const void *__restrict__ bias, int tokens, int c_in,
                    int hidden, int act, void *__restrict__ h, void *__restrict__ pre)
{
    constexpr int ES = BF16 ? 2 : 4, PER = 16 / ES;                 // elements of a lane's load,
    constexpr int DEPTH = 4 * P * PER;                              // and of a row's
    constexpr int ROWS = 16 / P, RG = 2 * P;                        // rows (or tokens) of a load; loads for 16 gate and 16 up rows
    constexpr int BATCH = RG + TG > 5 ? 3 : RG + TG > 3 ? 4 : 6;    // depths whose loads are in flight together
    __shared__ __attribute__((aligned(16))) float part[TOK_WAVES][RG * TG][64][4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r = (lane & 15) / P, k_lane = ((lane >> 4) * P + (lane & 15) % P) * PER;
    const int n0 = int(blockIdx.x) * TOK_COLS;
    const char *wr[RG], *xt[TG];
#pragma unroll
    for (int i = 0; i < RG; ++i)                       // gate rows, then the up rows of the same columns
        wr[i] = static_cast<const char *>(w) + (int64_t(min(n0 + (i % P) * ROWS + r, hidden - 1)) + (i >= P ? hidden : 0)) * c_in * ES;
#pragma unroll
    for (int j = 0; j < TG; ++j) xt[j] = static_cast<const char *>(x) + int64_t(min(ROWS * j + r, tokens - 1)) * c_in * ES;
    const int depths = (c_in + DEPTH - 1) / DEPTH;
    const int d0 = depths * wave / TOK_WAVES, d1 = depths * (wave + 1) / TOK_WAVES;

    f32x4 acc[RG][TG];
#pragma unroll
    for (int i = 0; i < RG; ++i)
#pragma unroll
        for (int j = 0; j < TG; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int d = d0; d < d1; d += BATCH) {
        u32x4 a[BATCH][RG], b[BATCH][TG];
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            const int k = (d + u) * DEPTH + k_lane;
            const bool in = d + u < d1 && k < c_in;                 // (rows are whole in 16-byte units)
            const u32x4 zero = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int i = 0; i < RG; ++i) a[u][i] = in ? *reinterpret_cast<const u32x4 *>(wr[i] + int64_t(k) * ES) : zero;
#pragma unroll
            for (int j = 0; j < TG; ++j) b[u][j] = in ? *reinterpret_cast<const u32x4 *>(xt[j] + int64_t(k) * ES) : zero;
        }
#pragma unroll
        for (int u = 0; u < BATCH; ++u)
#pragma unroll
            for (int i = 0; i < RG; ++i)
#pragma unroll
                for (int j = 0; j < TG; ++j) {
                    if constexpr (BF16) {
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[u][i]),
                                                                            __builtin_bit_cast(bf16x8, b[u][j]), acc[i][j], 0, 0, 0);
                    } else {
                        // an instruction takes one element of each lane group: four of them the lanes' sixteen bytes
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[u][i][e]), __uint_as_float(b[u][j][e]), acc[i][j], 0, 0, 0);
                    }
                }
    }
#pragma unroll
    for (int i = 0; i < RG; ++i)
#pragma unroll
        for (int j = 0; j < TG; ++j) *reinterpret_cast<f32x4 *>(part[wave][i * TG + j][lane]) = acc[i][j];
    __syncthreads();
    // lane l held token slot l % 16 and, in register e, row slot 4 (l / 16) + e
    for (int o = threadIdx.x; o < TOK_COLS * ROWS * TG; o += TOK_THREADS) {
        const int col = o % TOK_COLS, t = o / TOK_COLS, i = col / ROWS, j = t / ROWS;
        float g = 0.f, u = 0.f;
#pragma unroll
        for (int v = 0; v < TOK_WAVES; ++v)
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const int slot = (col % ROWS) * P + p, src = (slot >> 2) * 16 + (t % ROWS) * P + p;
                g += part[v][i * TG + j][src][slot & 3];
                u += part[v][(P + i) * TG + j][src][slot & 3];
            }
        const int c = n0 + col;
        if (t >= tokens || c >= hidden) continue;
        auto load = [&](int64_t at) {
            if constexpr (BF16) return __uint_as_float(uint32_t(static_cast<const uint16_t *>(bias)[at]) << 16);
            else return static_cast<const float *>(bias)[at];
        };
        if (bias != nullptr) {
            g += load(c);
            u += load(int64_t(hidden) + c);
        }
        auto store = [&](void *to, int64_t at, float v) {
            if constexpr (BF16) static_cast<__bf16 *>(to)[at] = static_cast<__bf16>(v);
            else static_cast<float *>(to)[at] = v;
        };
        store(h, int64_t(t) * hidden + c, activation<BF16>(g, act) * u);
        if (pre != nullptr) {
            store(pre, int64_t(t) * 2 * hidden + c, g);
            store(pre, int64_t(t) * 2 * hidden + hidden + c, u);
        }
    }
}

}  // namespace

bool gated_tokens_takes(int64_t tokens, int64_t c_in, int64_t hidden, dropit_dtype dt)
{
    const int64_t size = dt == DROPIT_BF16 ? 2 : 4;
    if (c_in % (16 / size) != 0) return false;         // rows in 16-byte units
    if (hidden > 1 << 26) return false;                // a launch has fewer than 2^32 threads
    // Every workgroup reads all tokens.  Up to 16 that is always worth it, beyond while the weights are small (us, calls in a row
    // in a graph, here and in the product that takes the call otherwise).  bf16, 32 tokens: 256 -> 704 3.4 and 4.8, 768 -> 2048
    // 5.2 and 6.1, 2048 -> 4096 12.3 and 13.1; 64 tokens: 4.6 and 7.6, 7.2 and 12.2, 16.9 and 17.8; with more than 32 MB of
    // weights, 2048 -> 5632 at 32 tokens 18.6 and 14.3, at 64 26.4 and 18.5, 4096 -> 10240 58 and 45.5, 80 and 42.6.  fp32, 32
    // tokens: 256 -> 704 5.4 and 7.6, 768 -> 2048 10.8 and 9.9, 1024 -> 2688 12.9 and 16.2; 64 tokens: 7.7 and 8.3, 15.8 and
    // 10.5, 21.4 and 17.8, so that its limit is 32.
    return tokens <= 16 || (tokens <= (dt == DROPIT_BF16 ? 64 : 32) && 2 * hidden * c_in * size <= int64_t(32) << 20);
}

dropit_status launch_gated_tokens(const void *x, int64_t tokens, int c_in, dropit_dtype dt, const void *w, const void *bias,
                                  int hidden, int act, void *h, void *pre, hipStream_t stream)
{
    const uint32_t grid = static_cast<uint32_t>((int64_t(hidden) + TOK_COLS - 1) / TOK_COLS);
    auto launch = [&](auto kernel) {
        kernel<<<grid, TOK_THREADS, 0, stream>>>(w, x, bias, int(tokens), c_in, hidden, act, h, pre);
    };
    // P = 2 where a load of eight tokens' halves serves (us at 4096 -> 10240, 1 and 16 tokens: bf16 38.8 and 48.2 with whole rows,
    // 30.7 and 35.4 in halves, 31.3 in quarters; fp32 84.0, 66.9, 63.3, and at 16 tokens 99.1 against 100.9 in halves)
    if (dt == DROPIT_BF16) {
        if (tokens <= 8) launch(gated_tokens_kernel<true, 2, 1>);
        else if (tokens <= 16) launch(gated_tokens_kernel<true, 2, 2>);
        else if (tokens <= 32) launch(gated_tokens_kernel<true, 1, 2>);
        else launch(gated_tokens_kernel<true, 1, 4>);
    } else {
        if (tokens <= 8) launch(gated_tokens_kernel<false, 2, 1>);
        else if (tokens <= 16) launch(gated_tokens_kernel<false, 1, 1>);
        else launch(gated_tokens_kernel<false, 1, 2>);
    }
    return launch_status();
}

}  // namespace dropit
