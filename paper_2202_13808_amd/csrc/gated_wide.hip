// The gated projection's products on wide tiles: bf16, many tokens (gated.hip takes every other size and type).
//
// A workgroup of eight wavefronts computes 256 rows of the weight operand by 64 * FN tokens, the sum in blocks of 32.
// Both operands of the forward pass have their sum contiguous: tile rows of 64 bytes, read as whole matrix operands by
// ds_read_b128.  The input gradient's weights have it as the slow axis: tile rows of 512 bytes, through the transposing LDS
// read.  Tiles go from global memory straight into LDS, four stages deep.  A direct load fills consecutive bytes, so rows
// cannot be padded; instead the 16-byte unit u of a 64-byte row r lies at unit u ^ (r / 4 % 4), which keeps the 16 lanes of
// an LDS access on different banks, and is paid for by the address a lane asks for, not by instructions.
//
// The two wavefronts of a SIMD alternate: while one multiplies a block (its matrix instructions back to back), the other
// reads the fragments of its next block and issues its share of the direct loads; a workgroup barrier ends each phase.  The
// second group of wavefronts enters the sequence one barrier late and leaves one out at the end.
//   - The stage of block s is read in phases 2s (first group) and 2s + 1 (second); each read phase ends with the wait for
//     its own reads, so behind the barrier of phase 2s + 1 nobody reads it.
//   - The loads of block s + 3 are issued in phases 2s and 2s + 1, into the stage that block s - 1 left in phase 2s - 1.
//   - At the end of its read phase a wavefront waits until only the loads of its two newest blocks are in flight: block
//     s + 1 is then complete before phase 2s + 2 reads it.
// Loads behind the last block repeat it, so that the counts are the same in every step; they fill stages nobody reads.
// Reads, waits and the barrier are asm because the compiler, which cannot tell the stages apart, would drain all loads in
// front of every LDS read that it knows of.
#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "dropit_layers.h"
#include "gated_act.hpp"
#include "gated_internal.hpp"

namespace dropit {

// sixteen bytes that the lanes behind the end of a sum read
__device__ __attribute__((aligned(16))) uint32_t gated_zeros[4];

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(16))) float f32x16;

constexpr int WIDE_THREADS = 512, WIDE_ROWS = 256, WIDE_K = 32, STAGES = 4, AHEAD = STAGES - 1;
constexpr int W_BYTES = WIDE_ROWS * WIDE_K * 2, W_LOADS = W_BYTES / 1024 / 8;
constexpr int TOKEN_GROUP = 8;                         // token tiles that the workgroups of an XCD go through together

template <bool FORWARD, int FN> struct Wide {
    static constexpr int TOKENS = 64 * FN;
    static constexpr int X_BYTES = TOKENS * WIDE_K * 2, X_LOADS = X_BYTES / 1024 / 8, LOADS = W_LOADS + X_LOADS;
    static constexpr int STAGE_BYTES = W_BYTES + X_BYTES;
    // the epilogue's staging areas, in the same bytes: COLS columns (and a pad that spreads rows over the banks) of 64 tokens,
    // of h and both halves of pre or of dx, twice
    static constexpr int COLS = FORWARD ? 128 : 256, PITCH = COLS + 8, PART = 64 * PITCH * 2, OUTS = FORWARD ? 3 : 1;
    static constexpr int LDS_BYTES = STAGES * STAGE_BYTES > 2 * OUTS * PART ? STAGES * STAGE_BYTES : 2 * OUTS * PART;
    static_assert(LDS_BYTES <= 160 * 1024, "LDS of one compute unit");
    static_assert(X_BYTES % 8192 == 0, "the direct loads divide over eight wavefronts");
};

template <int N> __device__ inline void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
__device__ inline void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ inline void workgroup_barrier() { asm volatile("s_barrier" ::: "memory"); }

template <int OFFSET> __device__ inline u32x4 read16(uint32_t at)
{
    u32x4 r;
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(r) : "v"(at), "n"(OFFSET) : "memory");
    return r;
}
// lane i of each 16-lane group receives column i of the 4 x 16 block whose lane p supplied row p / 4, columns 4 (p % 4) ..
template <int OFFSET> __device__ inline u32x2 read_turned(uint32_t at)
{
    u32x2 r;
    asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(r) : "v"(at), "n"(OFFSET) : "memory");
    return r;
}

template <int I, int N, typename F> __device__ inline void static_for(F &&f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        static_for<I + 1, N>(f);
    }
}

template <bool FORWARD, int FN>
__global__ void __launch_bounds__(WIDE_THREADS) __attribute__((amdgpu_waves_per_eu(2, 2)))
gated_wide_kernel(const WideArgs a)
{
    using C = Wide<FORWARD, FN>;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1;           // 64 weight rows, 32 FN tokens

    // Workgroups are dealt to the 8 XCDs in turn: re-number so that those of one XCD are consecutive, and go through the
    // weight tiles with TOKEN_GROUP token tiles at a time, whose operands then stay in that XCD's L2.
    const int per_xcd = gridDim.x / 8;
    const int v = int(blockIdx.x % 8) * per_xcd + int(blockIdx.x / 8);
    if (v >= a.row_tiles * a.token_tiles) return;
    const int group = v / (TOKEN_GROUP * a.row_tiles), within = v - group * TOKEN_GROUP * a.row_tiles;
    const int size = min(TOKEN_GROUP, a.token_tiles - group * TOKEN_GROUP);
    const int rt = within / size;
    const int64_t t0 = int64_t(group * TOKEN_GROUP + within - rt * size) * C::TOKENS;
    const int r0 = rt * (FORWARD ? WIDE_ROWS / 2 : WIDE_ROWS);      // first output column
    const int steps = (a.K + WIDE_K - 1) / WIDE_K;
    const int tail = a.K - (steps - 1) * WIDE_K;       // of the last block: 8, 16, 24 or 32

    // ---- global -> LDS: load q of a wavefront fills 1 KB of a tile, lane l the 16 bytes at l * 16
    const char *src[C::LOADS];
    bool in_tail[C::LOADS];
    const int64_t w_step = FORWARD ? WIDE_K * 2 : int64_t(WIDE_K) * a.c_in * 2;
#pragma unroll
    for (int q = 0; q < W_LOADS; ++q) {
        const int o = (wave * W_LOADS + q) * 1024 + lane * 16;
        if constexpr (FORWARD) {
            const int R = o / 64, unit = (o / 16 & 3) ^ (R >> 2 & 3);
            // rows R of a wavefront's 64: 32 gate rows, then the up rows of the same columns
            const int n = min(r0 + (R >> 6) * 32 + (R & 31), a.hidden - 1);
            src[q] = static_cast<const char *>(a.w) + ((R & 32 ? int64_t(a.hidden) : 0) + n) * a.c_in * 2 + unit * 16;
            in_tail[q] = unit * 8 < tail;
        } else {
            const int k = o / 512, c = min(r0 + ((o & 511) ^ ((k & 3) << 6)) / 2, a.c_in - 8);
            src[q] = static_cast<const char *>(a.w) + (int64_t(k) * a.c_in + c) * 2;
            in_tail[q] = k < tail;
        }
    }
#pragma unroll
    for (int q = 0; q < C::X_LOADS; ++q) {
        const int o = (wave * C::X_LOADS + q) * 1024 + lane * 16;
        const int r = o / 64, unit = (o / 16 & 3) ^ (r >> 2 & 3);
        src[W_LOADS + q] = static_cast<const char *>(a.x) + min<int64_t>(t0 + r, a.tokens - 1) * a.K * 2 + unit * 16;
        in_tail[W_LOADS + q] = unit * 8 < tail;
    }
    auto issue_load = [&](auto q_, int stage, int s) {
        constexpr int q = decltype(q_)::value;
        const char *p = src[q] + s * (q < W_LOADS ? w_step : int64_t(WIDE_K * 2));
        if (s == steps - 1) p = in_tail[q] ? p : reinterpret_cast<const char *>(gated_zeros);
        char *to = lds + stage * C::STAGE_BYTES + (q < W_LOADS ? (wave * W_LOADS + q) * 1024 : W_BYTES + (wave * C::X_LOADS + q - W_LOADS) * 1024);
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)p,
                                         (__attribute__((address_space(3))) void *)to, 16, 0, 0);
    };

    // ---- LDS -> fragments: operand lane l takes row l % 32 and the sum's elements 8 (l / 32) .. + 7 of 16
    const uint32_t base = uint32_t(size_t((__attribute__((address_space(3))) void *)lds));
    const int row = lane & 31, half = lane >> 5;
    const uint32_t unit0 = uint32_t(half ^ (row >> 2 & 3)) * 16;    // (32 rows further on the same: 32 / 4 is a multiple of 4)
    const uint32_t x_at = W_BYTES + uint32_t(wn * 32 * FN + row) * 64 + unit0;
    uint32_t w_at[2];
    if constexpr (FORWARD) {
        w_at[0] = uint32_t(wm * 64 + row) * 64 + unit0;
        w_at[1] = 0;
    } else {
        const int g = lane >> 4, p16 = lane & 15, krow = (g >> 1) * 8 + (p16 >> 2);
#pragma unroll
        for (int i = 0; i < 2; ++i)
            w_at[i] = uint32_t(krow * 512 + (((wm * 64 + i * 32 + (g & 1) * 16 + (p16 & 3) * 4) * 2) ^ ((p16 >> 2) << 6)));
    }
    u32x4 fw[2][2], fx[2][FN];                         // of both 16-deep halves of a block
    u32x2 ft[2][2][2];                                 // (transposing reads bring half an operand each)
    auto read_half = [&](auto kk_, uint32_t stage_base) {
        constexpr int kk = decltype(kk_)::value;
        if constexpr (FORWARD) {
            const uint32_t at = stage_base + (w_at[0] ^ (kk * 32));
            fw[kk][0] = read16<0>(at);
            fw[kk][1] = read16<32 * 64>(at);
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                ft[kk][i][0] = read_turned<kk * 16 * 512>(stage_base + w_at[i]);
                ft[kk][i][1] = read_turned<(kk * 16 + 4) * 512>(stage_base + w_at[i]);
            }
        }
        const uint32_t at = stage_base + (x_at ^ (kk * 32));
        static_for<0, FN>([&](auto j_) { fx[kk][decltype(j_)::value] = read16<decltype(j_)::value * 32 * 64>(at); });
    };

    f32x16 acc[2][FN];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

    const bool late = wave >= 4;
#pragma unroll
    for (int d = 0; d < AHEAD; ++d) static_for<0, C::LOADS>([&](auto q_) { issue_load(q_, d, min(d, steps - 1)); });
    wait_loads<(AHEAD - 1) * C::LOADS>();
    workgroup_barrier();
    if (late) workgroup_barrier();
    int stage = 0, fill = AHEAD;
    for (int s = 0; s < steps; ++s) {
        const uint32_t stage_base = base + stage * C::STAGE_BYTES;
        const int next = min(s + AHEAD, steps - 1);
        static_for<0, 2>([&](auto kk_) {
            constexpr int kk = decltype(kk_)::value;
            read_half(kk_, stage_base);
            static_for<kk * C::LOADS / 2, (kk + 1) * C::LOADS / 2>([&](auto q_) { issue_load(q_, fill, next); });
        });
        wait_lds();
        wait_loads<(AHEAD - 1) * C::LOADS>();
        __builtin_amdgcn_sched_barrier(0);
        workgroup_barrier();
        __builtin_amdgcn_sched_barrier(0);
        static_for<0, 2>([&](auto kk_) {
            constexpr int kk = decltype(kk_)::value;
#pragma unroll
            for (int i = 0; i < 2; ++i) {              // (nothing may move a fragment before the wait above)
                if constexpr (FORWARD) {
                    asm volatile("" : "+v"(fw[kk][i]));
                } else {
                    asm volatile("" : "+v"(ft[kk][i][0]), "+v"(ft[kk][i][1]));
                    fw[kk][i] = __builtin_shufflevector(ft[kk][i][0], ft[kk][i][1], 0, 1, 2, 3);
                }
            }
#pragma unroll
            for (int j = 0; j < FN; ++j) asm volatile("" : "+v"(fx[kk][j]));
            static_for<0, 2 * FN>([&](auto m_) {
                constexpr int m = decltype(m_)::value, i = m / FN, j = m % FN;
                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fw[kk][i]),
                                                                    __builtin_bit_cast(bf16x8, fx[kk][j]), acc[i][j], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            });
        });
        if (!(late && s + 1 == steps)) workgroup_barrier();
        __builtin_amdgcn_sched_barrier(0);
        stage = stage + 1 == STAGES ? 0 : stage + 1;
        fill = fill + 1 == STAGES ? 0 : fill + 1;
    }
    wait_loads<0>();                                   // nothing may still be writing LDS
    __syncthreads();

    // ---- out, 64 tokens at a time (32 of each half of the tile) by way of LDS, in rows of 16-byte units.  Lane l holds token
    // l % 32 and, in register 4 q + e, row 8 q + 4 (l / 32) + e of each 32 x 32 block.
    constexpr int COLS = C::COLS, PITCH = C::PITCH, PART = C::PART, OUTS = C::OUTS;
    const int width = FORWARD ? a.hidden : a.c_in;
    float bias[2][16];
    if constexpr (FORWARD) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int n = min(r0 + wm * 32 + q * 8 + half * 4 + e, a.hidden - 1) + i * a.hidden;
                    bias[i][q * 4 + e] = a.bias != nullptr ? __uint_as_float(uint32_t(static_cast<const uint16_t *>(a.bias)[n]) << 16) : 0.f;
                }
    }
    auto put = [&](char *area, int col, float v0, float v1, float v2, float v3) {
        *reinterpret_cast<bf16x4 *>(area + ((wn * 32 + row) * PITCH + col) * 2) =
            bf16x4{static_cast<__bf16>(v0), static_cast<__bf16>(v1), static_cast<__bf16>(v2), static_cast<__bf16>(v3)};
    };
    auto copy_out = [&](const char *area, void *out, int64_t pitch, int64_t at, int j) {
        constexpr int UNITS = COLS / 8;
#pragma unroll
        for (int r = 0; r < 64 * UNITS / WIDE_THREADS; ++r) {
            const int u = r * WIDE_THREADS + int(threadIdx.x), token = u / UNITS, c = u % UNITS * 8;
            const int64_t t = t0 + (token >> 5) * 32 * FN + j * 32 + (token & 31);
            const int n = r0 + c;
            if (t >= a.tokens || n >= width) continue;
            uint16_t *to = static_cast<uint16_t *>(out) + t * pitch + at + n;
            const u32x4 w = *reinterpret_cast<const u32x4 *>(area + (token * PITCH + c) * 2);
            if (width % 8 == 0) {                      // (then every row starts on 16 bytes)
                *reinterpret_cast<u32x4 *>(to) = w;
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (n + e < width) to[e] = uint16_t(w[e >> 1] >> (16 * (e & 1)));
            }
        }
    };
    static_for<0, FN>([&](auto j_) {
        constexpr int j = decltype(j_)::value;
        char *area = lds + (j & 1) * OUTS * PART;      // (the pass before reads the other one)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if constexpr (FORWARD) {
                float g[4], u[4], h[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    g[e] = acc[0][j][q * 4 + e] + bias[0][q * 4 + e];
                    u[e] = acc[1][j][q * 4 + e] + bias[1][q * 4 + e];
                    h[e] = activation<true>(g[e], a.act) * u[e];
                }
                const int col = wm * 32 + q * 8 + half * 4;
                put(area, col, h[0], h[1], h[2], h[3]);
                if (a.pre != nullptr) {
                    put(area + PART, col, g[0], g[1], g[2], g[3]);
                    put(area + 2 * PART, col, u[0], u[1], u[2], u[3]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    put(area, wm * 64 + i * 32 + q * 8 + half * 4, acc[i][j][q * 4], acc[i][j][q * 4 + 1], acc[i][j][q * 4 + 2], acc[i][j][q * 4 + 3]);
            }
        }
        __syncthreads();
        copy_out(area, a.out, width, 0, j);
        if constexpr (FORWARD) {
            if (a.pre != nullptr) {
                copy_out(area + PART, a.pre, 2 * int64_t(width), 0, j);
                copy_out(area + 2 * PART, a.pre, 2 * int64_t(width), width, j);
            }
        }
    });
}

template <bool FORWARD, int FN>
dropit_status launch(WideArgs a, hipStream_t stream)
{
    using C = Wide<FORWARD, FN>;
    constexpr int per_tile = FORWARD ? WIDE_ROWS / 2 : WIDE_ROWS;
    static std::atomic<uint64_t> done{0};
    if (!once_per_device(done, [] {
            return hipFuncSetAttribute(reinterpret_cast<const void *>(gated_wide_kernel<FORWARD, FN>),
                                       hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS_BYTES) == hipSuccess;
        }))
        return DROPIT_EHIP;
    a.row_tiles = ((FORWARD ? a.hidden : a.c_in) + per_tile - 1) / per_tile;
    a.token_tiles = int((a.tokens + C::TOKENS - 1) / C::TOKENS);
    const int64_t tiles = int64_t(a.row_tiles) * a.token_tiles;
    gated_wide_kernel<FORWARD, FN><<<static_cast<uint32_t>((tiles + 7) / 8 * 8), WIDE_THREADS, C::LDS_BYTES, stream>>>(a);
    return launch_status();
}

}  // namespace

bool gated_wide_takes(int64_t tokens, int c_in, int hidden, bool forward)
{
    return tokens >= 128 && c_in % 8 == 0 && (forward || hidden % 4 == 0);
}

dropit_status launch_gated_wide(const WideArgs &a, bool forward, hipStream_t stream)
{
    return forward ? launch<true, 4>(a, stream) : launch<false, 4>(a, stream);
}

}  // namespace dropit
