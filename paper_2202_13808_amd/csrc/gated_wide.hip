// The gated projection's products on wide tiles: bf16, many tokens (gated.hip takes every other size and type).  Bound by the matrix
// instructions and, in large products, by the clock that the chip's power leaves them: 8192 tokens 4096 -> 10240 990 to 1045 us by
// the card, 1315 to 1390 TFLOP/s, where a plain library product of these sizes takes 947 without activation and product.
//
// A workgroup of eight wavefronts computes 256 rows of the weight operand by 64 * FN tokens, the sum in blocks of 64: 128
// bytes of a row, a whole cache line.  (A load of 16 half lines takes the cache twice as long as one of 8 whole ones; blocks
// of 32 took 1171 us instead of 1066 for 8192 tokens 4096 -> 10240.)  Tiles go from global memory straight into LDS: two
// stages of weights, three of tokens, for FN = 4 all of a compute unit's 160 KB.  Both operands of the forward pass have
// their sum contiguous: tile rows of 128 bytes, read as whole matrix operands by ds_read_b128.  The input gradient's weights
// have it as the slow axis: tile rows of 512 bytes, through the transposing LDS read.  A direct load fills consecutive bytes,
// so rows cannot be padded; instead the 16-byte unit u of a 128-byte row r lies at unit u ^ (r / 2 % 8), which keeps the
// lanes of an LDS access on different banks and is paid for by the address a lane asks for, not by instructions.
//
// The two wavefronts of a SIMD alternate: while one multiplies a block (its matrix instructions back to back), the other
// reads the fragments of its next block and issues direct loads; a workgroup barrier ends each phase.  The second group of
// four wavefronts enters the sequence one barrier late and leaves one out at the end.
//     phase           2s       2s + 1    2s + 2         (R reads, M multiplies)
//     first group     R(s)     M(s)      R(s + 1)
//     second group    M(s-1)   R(s)      M(s)
// Block s is read in phases 2s and 2s + 1; every R ends with the wait for its own reads, so behind that barrier its stages
// are free.  The first group loads the weights: those of block s + 1, in R(s), into the stage that block s - 1 left in phase
// 2s - 1; it waits for them at the end of M(s).  The second group loads the tokens: those of block s + 2, in R(s), into the
// stage that block s - 1 left; it waits for those of block s + 1, issued one R earlier, at the end of R(s).  Both are
// complete before phase 2s + 2 reads them.
//
// A workgroup goes through several tiles, one per compute unit at a time, as one sequence of blocks: the loads run ahead into
// the next tile, and a tile's results leave from registers in front of its group's next R, while the other group multiplies.
// (A workgroup per tile started each with the latency of memory and ended with all of them storing at once: ViT-B's forward
// pass took 122 us, 77 of it the sums.)  Loads behind the last tile's last block repeat it, so that the counts are the same in
// every step; they fill stages nobody reads.
//
// Reads, waits and the barrier are asm because the compiler, which cannot tell the stages apart, would drain all loads in
// front of every LDS read that it knows of.
#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "dropit_layers.h"
#include "gated_act.hpp"
#include "gated_internal.hpp"

namespace dropit {

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef u32x4 u32x4_any __attribute__((aligned(2)));       // at any element's address
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;

constexpr int WIDE_THREADS = 512, WIDE_ROWS = 256, WIDE_K = 64;
constexpr int W_BYTES = WIDE_ROWS * WIDE_K * 2, W_STAGES = 2, X_STAGES = 3, X_AT = W_STAGES * W_BYTES;
constexpr int W_LOADS = W_BYTES / 1024 / 4;            // of a wavefront of the first group and block
constexpr int TOKEN_GROUP = 8;                         // token tiles that the workgroups of an XCD go through together

template <int FN> struct Wide {
    static constexpr int TOKENS = 64 * FN, X_BYTES = TOKENS * WIDE_K * 2, X_LOADS = X_BYTES / 1024 / 4;
    static constexpr int LDS_BYTES = X_AT + X_STAGES * X_BYTES;
    static_assert(FN >= 2 && FN <= 4 && LDS_BYTES <= 160 * 1024, "LDS of one compute unit");
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

// SLICED: the sum in a.splits slices, partial sums out
template <bool FORWARD, int FN, bool SLICED>
__global__ void __launch_bounds__(WIDE_THREADS) __attribute__((amdgpu_waves_per_eu(2, 2)))
gated_wide_kernel(const WideArgs a)
{
    using C = Wide<FN>;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1;           // 64 weight rows, 32 FN tokens
    const bool late = wave >= 4;

    // Workgroups are dealt to the 8 XCDs in turn.  An XCD's share of the tiles is consecutive, and its workgroups take them in
    // turn; the order goes through the weight tiles with TOKEN_GROUP token tiles at a time, whose operands then stay in that
    // XCD's L2.
    const int slice_tiles = a.row_tiles * a.token_tiles, tiles = SLICED ? slice_tiles * a.splits : slice_tiles, per_xcd = (tiles + 7) / 8, stride = int(gridDim.x / 8);
    const int v0 = int(blockIdx.x % 8) * per_xcd + int(blockIdx.x / 8);
    const int v_end = min(int(blockIdx.x % 8 + 1) * per_xcd, tiles);
    if (v0 >= v_end) return;
    auto place = [&](int v, int &rt, int &tt, int &slice) {
        slice = SLICED ? __builtin_amdgcn_readfirstlane(v / slice_tiles) : 0;
        v -= slice * slice_tiles;
        const int group = v / (TOKEN_GROUP * a.row_tiles), within = v - group * TOKEN_GROUP * a.row_tiles;
        const int size = min(TOKEN_GROUP, a.token_tiles - group * TOKEN_GROUP);
        rt = __builtin_amdgcn_readfirstlane(within / size);
        tt = __builtin_amdgcn_readfirstlane(group * TOKEN_GROUP + within - rt * size);
    };
    const int steps = (a.K + WIDE_K - 1) / WIDE_K;
    const int tail = a.K - (steps - 1) * WIDE_K;       // of the last block: 8, 16, .. 64
    auto slice_begin = [&](int slice) { return SLICED ? __builtin_amdgcn_readfirstlane(int(int64_t(steps) * slice / a.splits)) : slice * steps; };

    // ---- global -> LDS: load q of a wavefront fills 1 KB of a tile, lane l the 16 bytes at l * 16.  Through buffer descriptors:
    // a lane gives 32 bits of address, the step is a scalar (64-bit addresses per lane cost the address unit 5 %), and what
    // lies outside arrives as zeros: tokens and weight rows behind the last ones by their offset, which is a lane's own, and
    // columns behind the last one and the last block's elements behind the end of the sum by an offset beyond every range.
    // The descriptors' parts have to be scalars for the compiler too, or it puts a loop around every load.
    constexpr uint32_t OUTSIDE = 0x80000000u;          // (gated_wide_takes: ranges are smaller)
    constexpr int per_tile = FORWARD ? WIDE_ROWS / 2 : WIDE_ROWS;   // output columns
    const int part = wave & 3;                         // of the group's tile
    const uint32_t w_pitch = uint32_t(a.w_pitch) * 2u, x_pitch = uint32_t(a.x_pitch) * 2u;
    // tile rows of 128 bytes: load q holds rows 8 (L part + q) + lane / 8 for L loads of a wavefront, whose units are turned by
    // (row / 2) % 8, that is by lane / 16 and, for odd q (L is even), by 4 more.  Forward weights: row R of a wavefront's 64
    // is gate row R for R < 32, then up rows of the same columns.  Tile rows of 512 bytes: load q holds k = 16 part + 2 q +
    // lane / 32, turned by (k % 4) * 64 bytes.
    const bool turned_tile = !FORWARD && !late;
    const int first = late ? C::X_LOADS * part : W_LOADS * part;    // the wavefront's first load of the tile
    const int unit = (lane & 7) ^ (lane >> 4);
    uint32_t lane_off[2];                              // of even and odd q
    int first_k[2];                                    // the sum's element in a block that a lane's even / odd loads start at
    uint32_t q_step;                                   // from a load to the next but one
    uint32_t column[2] = {0, 0};                       // (turned tile) byte of the row, within the tile's columns
    if (turned_tile) {
#pragma unroll
        for (int o = 0; o < 2; ++o) {
            first_k[o] = 16 * part + 2 * o + (lane >> 5);
            column[o] = uint32_t(((lane & 31) * 16) ^ ((first_k[o] & 3) << 6));
            lane_off[o] = uint32_t(first_k[o]) * w_pitch + column[o];
        }
        q_step = 4u * w_pitch;
    } else {
        const uint32_t pitch = late ? x_pitch : w_pitch;
        const uint32_t row = uint32_t((late ? 8 * first : 32 * part) + (lane >> 3));
#pragma unroll
        for (int o = 0; o < 2; ++o) {
            first_k[o] = (unit ^ (4 * o)) * 8;
            lane_off[o] = (row + 8u * o) * pitch + uint32_t(first_k[o]) * 2u;
        }
        q_step = 16u * pitch;
    }
    const uint32_t up_step = FORWARD && !late ? uint32_t(a.hidden - 32) * w_pitch : 0u;     // loads 4 .. 7 of forward weights
    const int s_step = turned_tile ? WIDE_K * int(w_pitch) : WIDE_K * 2;
    // the loads' own place in the sequence of blocks, and their tile's descriptor
    int lv = v0, ls, l_end;
    const char *l_base;
    int l_range;
    uint32_t l_outside[2];                             // OUTSIDE for lanes behind the last column
    auto load_tile = [&]() {
        int rt, tt, slice;
        place(lv, rt, tt, slice);
        ls = slice_begin(slice);
        l_end = slice_begin(slice + 1);
        l_outside[0] = l_outside[1] = 0u;
        if (late) {
            l_base = static_cast<const char *>(a.x) + int64_t(tt) * C::TOKENS * a.x_pitch * 2;
            l_range = min(int(a.tokens) - tt * C::TOKENS, C::TOKENS) * a.x_pitch * 2;
        } else if constexpr (FORWARD) {
            l_base = static_cast<const char *>(a.w) + int64_t(rt) * per_tile * a.w_pitch * 2;
            l_range = (2 * a.hidden - rt * per_tile) * a.w_pitch * 2;
        } else {
            l_base = static_cast<const char *>(a.w) + int64_t(rt) * per_tile * 2;
            l_range = 2 * a.hidden * a.w_pitch * 2 - rt * per_tile * 2;
#pragma unroll
            for (int o = 0; o < 2; ++o) l_outside[o] = uint32_t(rt * per_tile) * 2u + column[o] < w_pitch ? 0u : OUTSIDE;
        }
    };
    load_tile();
    auto advance = [&]() {
        if (ls + 1 < l_end) {
            ++ls;
        } else if (lv + stride < v_end) {
            lv += stride;
            load_tile();
        }
    };
    auto issue_load = [&](auto q_, char *tile) {
        constexpr int q = decltype(q_)::value;
        if (q >= C::X_LOADS && late) return;
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(l_base), 0, l_range, 0x00020000);
        uint32_t at = lane_off[q & 1] + (q >> 1) * q_step + (q >= 4 ? up_step : 0u);
        if constexpr (!FORWARD) at |= l_outside[q & 1];
        const int k = first_k[q & 1] + (turned_tile ? (q >> 1) * 4 : 0);
        if (ls == steps - 1) at = k < tail ? at : OUTSIDE;
        const int scalar = ls * s_step;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void *)(tile + (first + q) * 1024), 16, int(at),
                                                 scalar, 0, 0);
    };

    // ---- LDS -> fragments: operand lane l takes row l % 32 and the sum's elements 8 (l / 32) .. + 7 of 16
    const uint32_t base = uint32_t(size_t((__attribute__((address_space(3))) void *)lds));
    const int row = lane & 31, half = lane >> 5;
    const uint32_t unit0 = uint32_t(half ^ (row >> 1 & 7)) * 16;    // (32 rows further on the same: 32 / 2 is a multiple of 8)
    const uint32_t x_at = X_AT + uint32_t(wn * 32 * FN + row) * 128 + unit0;
    uint32_t w_at[2];
    if constexpr (FORWARD) {
        w_at[0] = uint32_t(wm * 64 + row) * 128 + unit0;
        w_at[1] = 0;
    } else {
        const int g = lane >> 4, p16 = lane & 15, krow = (g >> 1) * 8 + (p16 >> 2);
#pragma unroll
        for (int i = 0; i < 2; ++i)
            w_at[i] = uint32_t(krow * 512 + (((wm * 64 + i * 32 + (g & 1) * 16 + (p16 & 3) * 4) * 2) ^ ((p16 >> 2) << 6)));
    }
    constexpr int KK = WIDE_K / 16;                    // depths of one matrix instruction
    u32x4 fw[KK][2], fx[KK][FN];
    u32x2 ft[KK][2][2];                                // (transposing reads bring half an operand each)
    auto read_depth = [&](auto kk_, uint32_t w_base, uint32_t x_base) {
        constexpr int kk = decltype(kk_)::value;
        if constexpr (FORWARD) {
            const uint32_t at = w_base + (w_at[0] ^ (kk * 32));
            fw[kk][0] = read16<0>(at);
            fw[kk][1] = read16<32 * 128>(at);
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                ft[kk][i][0] = read_turned<kk * 16 * 512>(w_base + w_at[i]);
                ft[kk][i][1] = read_turned<(kk * 16 + 4) * 512>(w_base + w_at[i]);
            }
        }
        const uint32_t at = x_base + (x_at ^ (kk * 32));
        static_for<0, FN>([&](auto j_) { fx[kk][decltype(j_)::value] = read16<decltype(j_)::value * 32 * 128>(at); });
    };

    // the first block's weights, the first two blocks' tokens
    static_for<0, W_LOADS>([&](auto q_) { issue_load(q_, lds + (late ? X_AT : 0)); });
    if (late) {
        advance();
        static_for<0, W_LOADS>([&](auto q_) { issue_load(q_, lds + X_AT + C::X_BYTES); });
        wait_loads<C::X_LOADS>();
    } else {
        wait_loads<0>();
    }
    workgroup_barrier();
    if (late) workgroup_barrier();
    int w_stage = 0, x_stage = 0;
    for (int v = v0; v < v_end; v += stride) {
        int blocks = steps;
        if constexpr (SLICED) {
            const int slice = __builtin_amdgcn_readfirstlane(v / slice_tiles);
            blocks = slice_begin(slice + 1) - slice_begin(slice);
        }
        f32x16 acc[2][FN];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
        for (int s = 0; s < blocks; ++s) {
            const uint32_t w_base = base + w_stage * W_BYTES, x_base = base + x_stage * C::X_BYTES;
            w_stage ^= 1;                              // the next block's weights
            const int x_fill = x_stage == 0 ? X_STAGES - 1 : x_stage - 1;       // the next but one's tokens
            x_stage = x_stage == X_STAGES - 1 ? 0 : x_stage + 1;
            char *const fill = lds + (late ? X_AT + x_fill * C::X_BYTES : w_stage * W_BYTES);
            advance();
            static_for<0, KK>([&](auto kk_) {
                constexpr int kk = decltype(kk_)::value;
                read_depth(kk_, w_base, x_base);
                static_for<kk * W_LOADS / KK, (kk + 1) * W_LOADS / KK>([&](auto q_) { issue_load(q_, fill); });
            });
            wait_lds();
            if (late) wait_loads<C::X_LOADS>();
            __builtin_amdgcn_sched_barrier(0);
            workgroup_barrier();
            __builtin_amdgcn_sched_barrier(0);
            static_for<0, KK>([&](auto kk_) {
                constexpr int kk = decltype(kk_)::value;
#pragma unroll
                for (int i = 0; i < 2; ++i) {          // (nothing may move a fragment before the wait above)
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
            if (!late) wait_loads<0>();
            __builtin_amdgcn_sched_barrier(0);
            if (!(late && s + 1 == blocks && v + stride >= v_end)) workgroup_barrier();
            __builtin_amdgcn_sched_barrier(0);
        }

        // ---- out: lane l holds token l % 32 and, in register 4 q + e, row 8 q + 4 (l / 32) + e of each 32 x 32 block.  The
        // halves of the wavefront trade their columns of every other eight, so that a lane stores 16 bytes of a row and two
        // lanes 32.
        int rt, tt, slice;
        place(v, rt, tt, slice);
        const int64_t t0 = int64_t(tt) * C::TOKENS;
        const int width = FORWARD ? a.hidden : a.c_in;
        const int n0 = rt * per_tile + wm * (FORWARD ? 32 : 64);
        if constexpr (SLICED) {                        // partial sums, as they are
            const int64_t pitch = FORWARD ? 2 * int64_t(width) : width;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    const int64_t t = t0 + wn * 32 * FN + j * 32 + row;
                    if (t >= a.tokens) continue;
                    float *to = a.partial + (int64_t(slice) * a.tokens + t) * pitch + (FORWARD ? i * width : 0);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int c = n0 + (FORWARD ? 0 : i * 32) + q * 8 + half * 4;
                        if (width % 4 == 0) {
                            if (c < width)
                                *reinterpret_cast<f32x4 *>(to + c) = f32x4{acc[i][j][q * 4], acc[i][j][q * 4 + 1], acc[i][j][q * 4 + 2], acc[i][j][q * 4 + 3]};
                        } else {
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (c + e < width) to[c + e] = acc[i][j][q * 4 + e];
                        }
                    }
                }
            continue;
        }
        auto store_block = [&](const float (&x)[16], void *out, int64_t pitch, int64_t at, int n, int j) {
            const int64_t t = t0 + wn * 32 * FN + j * 32 + row;
            uint16_t *to = static_cast<uint16_t *>(out) + t * pitch + at;
#pragma unroll
            for (int q = 0; q < 4; q += 2) {
                uint32_t d[2][2];
#pragma unroll
                for (int p = 0; p < 2; ++p)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const bf16x2 pair = {static_cast<__bf16>(x[(q + p) * 4 + 2 * e]), static_cast<__bf16>(x[(q + p) * 4 + 2 * e + 1])};
                        d[p][e] = __builtin_bit_cast(uint32_t, pair);
                    }
                u32x4 w;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const auto r = __builtin_amdgcn_permlane32_swap(d[0][e], d[1][e], false, false);
                    w[e] = r[0];
                    w[2 + e] = r[1];
                }
                const int c = n + (q + half) * 8;
                if (t >= a.tokens || c >= width) continue;
                if (c + 8 <= width) {
                    *reinterpret_cast<u32x4_any *>(to + c) = w;
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (c + e < width) to[c + e] = uint16_t(w[e >> 1] >> (16 * (e & 1)));
                }
            }
        };
        if constexpr (FORWARD) {
            float bias[2][16];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int n = min(n0 + (r >> 2) * 8 + half * 4 + (r & 3), a.hidden - 1) + i * a.hidden;
                    bias[i][r] = a.bias != nullptr ? __uint_as_float(uint32_t(static_cast<const uint16_t *>(a.bias)[n]) << 16) : 0.f;
                }
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                float x[16], u[16];
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    x[r] = acc[0][j][r] + bias[0][r];
                    u[r] = acc[1][j][r] + bias[1][r];
                }
                if (a.pre != nullptr) {
                    store_block(x, a.pre, 2 * int64_t(width), 0, n0, j);
                    store_block(u, a.pre, 2 * int64_t(width), width, n0, j);
                }
                activations<true>(x, a.act);
#pragma unroll
                for (int r = 0; r < 16; ++r) x[r] *= u[r];
                store_block(x, a.out, width, 0, n0, j);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    float x[16];
#pragma unroll
                    for (int r = 0; r < 16; ++r) x[r] = acc[i][j][r];
                    store_block(x, a.out, width, 0, n0 + i * 32, j);
                }
        }
    }
    wait_loads<0>();                                   // nothing may still be writing LDS
}

template <bool FORWARD, int FN, bool SLICED>
dropit_status launch(WideArgs a, hipStream_t stream)
{
    using C = Wide<FN>;
    constexpr int per_tile = FORWARD ? WIDE_ROWS / 2 : WIDE_ROWS;
    static std::atomic<uint64_t> done{0};
    if (!once_per_device(done, [] {
            return hipFuncSetAttribute(reinterpret_cast<const void *>(gated_wide_kernel<FORWARD, FN, SLICED>),
                                       hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS_BYTES) == hipSuccess;
        }))
        return DROPIT_EHIP;
    a.row_tiles = ((FORWARD ? a.hidden : a.c_in) + per_tile - 1) / per_tile;
    a.token_tiles = int((a.tokens + C::TOKENS - 1) / C::TOKENS);
    const int64_t tiles = int64_t(a.row_tiles) * a.token_tiles * a.splits;
    const uint32_t grid = static_cast<uint32_t>(std::min<int64_t>((tiles + 7) / 8 * 8, 256));       // one per compute unit
    gated_wide_kernel<FORWARD, FN, SLICED><<<grid, WIDE_THREADS, C::LDS_BYTES, stream>>>(a);
    return launch_status();
}

template <bool FORWARD, int FN>
dropit_status launch(const WideArgs &a, hipStream_t stream)
{
    return a.splits > 1 ? launch<FORWARD, FN, true>(a, stream) : launch<FORWARD, FN, false>(a, stream);
}

}  // namespace

WidePlan gated_wide_plan(int64_t tokens, int64_t c_in, int64_t hidden, bool forward)
{
    // the weights, and 256 tokens, below 2^31 bytes.  Few tokens leave most of a tile empty, but in the gradients its slices fill
    // the chip (us for 16 tokens, here and in gated.hip's product: 384 -> 1024 15 and 19, 2048 -> 5632 23 and 46, 4096 -> 10240 45
    // and 115).  The forward pass's pay from 33 tokens on (32 tokens: 2048 -> 5632 16.4 and 14.3, 4096 -> 7168 30.0 and 32.0, 8192
    // -> 4096 35.1 and 36.1, 4096 -> 10240 38.9 and 45.5, the largest difference; 17 tokens: 16.0 and 14.1, 29.2 and 28.8, 35.8 and
    // 34.3, 38.3 and 42.8)
    WidePlan plan{(!forward || tokens > 32) && 4 * hidden * c_in < int64_t(1) << 31 && std::max(c_in, 2 * hidden) < (1 << 22) - 8, 2, 1, 0.0};
    if (!plan.takes) return plan;
    // How many tokens to a tile, and how many slices of the sum: what the compute unit with the most tiles takes, a block of
    // the sum and a tile's start and end at what they were measured to cost (us; whole chip busy: blocks of 8192 tokens 4096 ->
    // 10240 both ways, ends of ViT-B's and DeiT-S's forward passes, which keep the pre-activations: without them an end stores a
    // third, and the gradients' half or less, so that there a wide end is counted for more than it takes).  Fewer tokens cost more LDS reads per matrix instruction:
    // 64 of them as much as 128 per block, so there is no such tile.  us for 256, 192 and 128 tokens: 12608 tokens 768 -> 2048
    // forward 109, 105, 123, backward 81, 74, 108; 25216 tokens 384 -> 1024 75, 73, 77 and 50, 67, 59; 2048 tokens 2048 ->
    // 5632 93, 84, 93 and 169, 137, 128; 8192 tokens 4096 -> 10240 1004, 1095, 1365.  Slices cost a launch and their partial
    // sums' way to memory and back.
    constexpr double block_us[3] = {1.07, 1.22, 1.57}, end_us[3] = {4.7, 6.3, 8.0};
    const int64_t rows = forward ? (hidden + WIDE_ROWS / 2 - 1) / (WIDE_ROWS / 2) : (c_in + WIDE_ROWS - 1) / WIDE_ROWS;
    const int64_t blocks = ((forward ? c_in : 2 * hidden) + WIDE_K - 1) / WIDE_K;
    const double slice_us = double(tokens) * double(forward ? 2 * hidden : c_in) * 8 / 4e6;         // 4 bytes out and in at 4 TB/s
    double best_us = 0.0;
    for (int f = 0; f < 3; ++f) {
        const int64_t tiles = rows * ((tokens + 64 * (f + 2) - 1) / (64 * (f + 2)));
        for (int splits = 1; splits <= 16 && (splits == 1 || (tiles * splits <= 512 && blocks / splits >= 8)); ++splits) {
            const int64_t rounds = ((tiles * splits + 7) / 8 + 31) / 32;        // of 32 compute units on each of 8 XCDs
            const double us = double(rounds) * (double((blocks + splits - 1) / splits) * block_us[f] + end_us[f]) +
                              (splits > 1 ? 5.0 + splits * slice_us : 0.0);
            if (best_us == 0.0 || us < best_us || (us == best_us && splits == 1)) {
                plan.fn = f + 2;
                plan.splits = splits;
                best_us = us;
            }
        }
    }
    plan.us = best_us;
    return plan;
}

dropit_status launch_gated_wide(const WideArgs &a, const WidePlan &plan, bool forward, hipStream_t stream)
{
    if (plan.fn == 4) return forward ? launch<true, 4>(a, stream) : launch<false, 4>(a, stream);
    if (plan.fn == 3) return forward ? launch<true, 3>(a, stream) : launch<false, 3>(a, stream);
    return forward ? launch<true, 2>(a, stream) : launch<false, 2>(a, stream);
}

}  // namespace dropit
