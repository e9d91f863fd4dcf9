// The gated projection of a feed-forward block and its backward pass (the formulas stand in dropit_layers.h): entry
// points, the product that takes every size and type, and the element-wise part of the backward pass.
//
// Both products sum over a row of the token operand: the forward pass multiplies x [tokens, c_in] by W's gate and up rows,
// the input gradient dpre [tokens, 2 * hidden] by W's columns.  The weights are the matrix instruction's row operand, so a
// lane holds four consecutive output columns of one token.  In the forward pass a wavefront's row blocks come in pairs, a
// gate block and the up block of the same columns, so the activation and the product happen in the accumulators.
#include <algorithm>

#include "common.hpp"
#include "dropit_layers.h"
#include "gated_act.hpp"
#include "gated_internal.hpp"

namespace dropit {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
// sixteen bytes at any element's address: a row of odd length moves in wide accesses too
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));

template <bool BF16> struct Elem { using type = float; static constexpr int PER16 = 4; };
template <> struct Elem<true> { using type = uint16_t; static constexpr int PER16 = 8; };

template <bool BF16> __device__ inline float load_one(const void *p, int64_t i)
{
    if constexpr (BF16) return __uint_as_float(uint32_t(static_cast<const uint16_t *>(p)[i]) << 16);
    else return static_cast<const float *>(p)[i];
}
template <bool BF16> __device__ inline void store_one(void *p, int64_t i, float v)
{
    if constexpr (BF16) static_cast<__bf16 *>(p)[i] = static_cast<__bf16>(v);
    else static_cast<float *>(p)[i] = v;
}

// the first `some` (four, where there are more) of four consecutive elements
template <bool BF16> __device__ inline void store_four(void *p, int64_t i, const f32x4 &v, int some)
{
    if (some < 4) {
        for (int e = 0; e < some; ++e) store_one<BF16>(p, i + e, v[e]);
        return;
    }
    if constexpr (BF16) {
        bf16x4 b;
#pragma unroll
        for (int e = 0; e < 4; ++e) b[e] = static_cast<__bf16>(v[e]);
        *reinterpret_cast<u32x2_any *>(static_cast<uint16_t *>(p) + i) = __builtin_bit_cast(u32x2, b);
    } else {
        *reinterpret_cast<u32x4_any *>(static_cast<float *>(p) + i) = __builtin_bit_cast(u32x4, v);
    }
}

// ---------------------------------------------------------------------------
// The product for every size and type: tiles of 64 tokens by 64 rows of the weight operand, four wavefronts of 32 x 32, in the
// forward pass 16 gate and 16 up rows each.  fp32 runs on the fp32 matrix instructions and is bound by them: 4096 tokens 768 ->
// 2048 209 us, 124 TFLOP/s where a large library product reaches 140.  Small products are bound by how many steps' loads are on
// their way at once: two steps ahead and three or four workgroups to a compute unit, which tiles of 128 rows would leave one
// (1003 tokens 387 -> 515 in fp32 31 us with those, 22 so).
// Few tiles: the sum is cut into slices, whose partial sums finish_kernel adds in ascending order.
constexpr int GEN_THREADS = 256, GEN_ROWS = 64, GEN_TOKENS = 64, GEN_K = 32;

struct GenArgs {
    const void *w, *x;          // weight operand; token operand [tokens][K]
    int64_t tokens;
    int hidden, c_in;
    int K;                      // forward: c_in, backward: 2 * hidden
    int act;
    const void *bias;
    void *out, *pre;            // forward: h and pre; backward: dx
    float *partial;             // [splits][tokens][width], or null: width = 2 * hidden (forward) or c_in (backward)
    int splits, row_tiles, tiles, group;
};

// sixteen bytes of a row from element k on, zeros from `end` on (which may be 0): element by element and without a branch
template <bool BF16>
__device__ inline u32x4 load_elements(const typename Elem<BF16>::type *row, int k, int end)
{
    u32x4 r = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int e = 0; e < Elem<BF16>::PER16; ++e) {
        const auto v = row[max(min(k + e, end - 1), 0)];
        if constexpr (BF16) r[e >> 1] |= (k + e < end ? uint32_t(v) : 0u) << (16 * (e & 1));
        else r[e] = k + e < end ? __float_as_uint(v) : 0u;
    }
    return r;
}

template <bool BF16, bool FORWARD>
__global__ void __launch_bounds__(GEN_THREADS)
gated_product_kernel(const GenArgs a)
{
    constexpr int ES = BF16 ? 2 : 4, PER = Elem<BF16>::PER16;
    constexpr int UNITS = GEN_K / PER;                              // 16-byte units of a tile row
    constexpr int PITCH = GEN_K * ES + 16;                          // bytes of an LDS row: the pad spreads the rows over the banks
    constexpr int A_LOADS = GEN_ROWS * UNITS / GEN_THREADS, B_LOADS = GEN_TOKENS * UNITS / GEN_THREADS;
    // The input gradient's weights arrive along the columns, [k][column].  In fp32 a matrix instruction takes one k at a time
    // and reads them as they lie; in bf16 it takes eight, and they are turned on the way into LDS.
    constexpr bool AS_IT_LIES = !FORWARD && !BF16;
    constexpr int K_PITCH = GEN_ROWS * ES + 16;
    constexpr int A_BYTES = AS_IT_LIES ? GEN_K * K_PITCH : GEN_ROWS * PITCH;
    __shared__ __attribute__((aligned(16))) char tile[2][A_BYTES + GEN_TOKENS * PITCH];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wm = wave >> 1, wn = wave & 1;
    // Workgroups are dealt to the 8 XCDs in turn, each with a cache of its own: an XCD takes consecutive tiles, and the order goes
    // through the weight tiles with a.group token tiles at a time.
    const uint32_t v = blockIdx.x % 8 * (gridDim.x / 8) + blockIdx.x / 8;
    if (v >= uint32_t(a.tiles)) return;
    const uint32_t span = unsigned(a.group * a.row_tiles), first = v / span * unsigned(a.group), within = v % span;
    const uint32_t size = min(unsigned(a.group), unsigned(a.tiles / a.row_tiles) - first);
    const int rt = int(within / size);
    const int64_t t0 = int64_t(first + within % size) * GEN_TOKENS;
    const int split = blockIdx.y;
    const int r0 = rt * (FORWARD ? GEN_ROWS / 2 : GEN_ROWS);        // first output column of the tile
    const int steps_all = (a.K + GEN_K - 1) / GEN_K;
    const int s0 = int(int64_t(steps_all) * split / a.splits), s1 = int(int64_t(steps_all) * (split + 1) / a.splits);

    // weight row of the tile's row R: forward, a wavefront's rows are HALF gate rows and the HALF up rows of the same columns
    constexpr int HALF = GEN_ROWS / 4;
    auto weight_row = [&](int R) -> int64_t {
        const int n = min(r0 + R / (2 * HALF) * HALF + R % HALF, a.hidden - 1);
        return (R & HALF) ? int64_t(a.hidden) + n : n;
    };
    // where a thread's units start; from one step to the next they move by 32 elements, or by 32 rows of W
    using T = typename Elem<BF16>::type;
    const T *wp[A_LOADS], *xp[B_LOADS];
    const int64_t w_step = FORWARD ? GEN_K : int64_t(GEN_K) * a.c_in;
#pragma unroll
    for (int i = 0; i < A_LOADS; ++i) {
        const int unit = i * GEN_THREADS + tid;
        if constexpr (FORWARD) {
            wp[i] = static_cast<const T *>(a.w) + weight_row(unit / UNITS) * a.c_in + unit % UNITS * PER;
        } else {
            const int c = r0 + unit % (GEN_ROWS / PER) * PER;
            wp[i] = static_cast<const T *>(a.w) + int64_t(unit / (GEN_ROWS / PER)) * a.c_in + (c < a.c_in ? c : 0);
        }
    }
#pragma unroll
    for (int i = 0; i < B_LOADS; ++i) {
        const int unit = i * GEN_THREADS + tid;
        xp[i] = static_cast<const T *>(a.x) + min<int64_t>(t0 + unit / UNITS, a.tokens - 1) * a.K + unit % UNITS * PER;
    }
    // Steps whose units pass no end: the input gradient's units that pass the end of a row of W take what follows there, for columns
    // that are not stored, so that step has to end a unit before the end of W.
    const int whole = FORWARD || a.c_in % PER == 0 ? a.K / GEN_K : (a.K - (PER + a.c_in - 1) / a.c_in) / GEN_K;
    struct Units {
        u32x4 a[A_LOADS], b[B_LOADS];
    };
    auto load = [&](int s, Units &r) {
#pragma unroll
        for (int i = 0; i < A_LOADS; ++i) r.a[i] = *reinterpret_cast<const u32x4_any *>(wp[i] + s * w_step);
#pragma unroll
        for (int i = 0; i < B_LOADS; ++i) r.b[i] = *reinterpret_cast<const u32x4_any *>(xp[i] + s * GEN_K);
    };
    // any step, element by element: nothing past the end of a row is read, and zeros stand there
    auto load_last = [&](int s, Units &r) {
        const int k0 = s * GEN_K;
#pragma unroll
        for (int i = 0; i < A_LOADS; ++i) {
            const int unit = i * GEN_THREADS + tid, k = k0 + (FORWARD ? unit % UNITS * PER : unit / (GEN_ROWS / PER));
            if constexpr (FORWARD) r.a[i] = load_elements<BF16>(wp[i] - unit % UNITS * PER, k, a.K);
            else {                                                  // W [K][c_in]: a unit is PER columns of one k
                const int c = r0 + unit % (GEN_ROWS / PER) * PER;
                r.a[i] = load_elements<BF16>(static_cast<const T *>(a.w) + int64_t(min(k, a.K - 1)) * a.c_in, c, k < a.K ? a.c_in : 0);
            }
        }
#pragma unroll
        for (int i = 0; i < B_LOADS; ++i) {
            const int at = (i * GEN_THREADS + tid) % UNITS * PER;
            r.b[i] = load_elements<BF16>(xp[i] - at, k0 + at, a.K);
        }
    };
    auto put = [&](char *to, const Units &r) {
#pragma unroll
        for (int i = 0; i < A_LOADS; ++i) {
            const int unit = i * GEN_THREADS + tid;
            if constexpr (FORWARD) {
                *reinterpret_cast<u32x4 *>(to + unit / UNITS * PITCH + unit % UNITS * 16) = r.a[i];
            } else {
                const int k = unit / (GEN_ROWS / PER), c = unit % (GEN_ROWS / PER) * PER;
                if constexpr (AS_IT_LIES) *reinterpret_cast<u32x4 *>(to + k * K_PITCH + c * ES) = r.a[i];
                else
#pragma unroll
                for (int e = 0; e < PER; ++e) {
                    char *at = to + (c + e) * PITCH + k * ES;
                    *reinterpret_cast<uint16_t *>(at) = uint16_t(r.a[i][e >> 1] >> (16 * (e & 1)));
                }
            }
        }
#pragma unroll
        for (int i = 0; i < B_LOADS; ++i) {
            const int unit = i * GEN_THREADS + tid;
            *reinterpret_cast<u32x4 *>(to + A_BYTES + unit / UNITS * PITCH + unit % UNITS * 16) = r.b[i];
        }
    };

    f32x16 acc;
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = 0.f;
    int turn = 0;
    auto put_and_wait = [&](const Units &r) {
        put(tile[turn], r);
        __syncthreads();                                            // (the other tile's readers passed the barrier before)
    };
    auto multiply = [&]() {
        const char *cur = tile[turn];
        turn ^= 1;
        const char *wa = cur + (wm * 32 + (lane & 31)) * PITCH, *xb = cur + A_BYTES + (wn * 32 + (lane & 31)) * PITCH;
        if constexpr (BF16) {
#pragma unroll
            for (int kk = 0; kk < GEN_K / 16; ++kk) {
                const int at = kk * 32 + (lane >> 5) * 16;
                const bf16x8 b = *reinterpret_cast<const bf16x8 *>(xb + at);
                acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8 *>(wa + at), b, acc, 0, 0, 0);
            }
        } else {
            // an instruction takes one k from each half of the wavefront: k = 8 kk + e and 8 kk + 4 + e
#pragma unroll
            for (int kk = 0; kk < GEN_K / 8; ++kk) {
                const int at = kk * 32 + (lane >> 5) * 16;
                const f32x4 b = *reinterpret_cast<const f32x4 *>(xb + at);
                f32x4 w;
                if constexpr (AS_IT_LIES) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        w[e] = *reinterpret_cast<const float *>(cur + (kk * 8 + (lane >> 5) * 4 + e) * K_PITCH + (wm * 32 + (lane & 31)) * ES);
                } else {
                    w = *reinterpret_cast<const f32x4 *>(wa + at);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(w[e], b[e], acc, 0, 0, 0);
            }
        }
    };
    // Two steps are on their way while one is multiplied; loads behind the last whole step repeat it, so that no branch stands
    // between a load and its wait.  What is no whole step comes first, under the others' first loads.
    Units even, odd;
    const int end = min(s1, whole);
    if (s0 < end) {
        load(s0, even);
        load(min(s0 + 1, end - 1), odd);
    }
    for (int s = max(s0, whole); s < s1; ++s) {
        Units last;
        load_last(s, last);
        put_and_wait(last);
        multiply();
    }
    for (int s = s0; s < end;) {
        put_and_wait(even);
        load(min(s + 2, end - 1), even);
        multiply();
        if (++s >= end) break;
        put_and_wait(odd);
        load(min(s + 2, end - 1), odd);
        multiply();
        ++s;
    }
    // lane l holds token l % 32 and, in register 4 q + e, row 8 q + 4 (l / 32) + e of each 32 x 32 block: four consecutive output
    // columns, stored in one access (one store an element made the stores, 64 rows each, longer than the product)
    const int64_t t = t0 + wn * 32 + (lane & 31);
    if (t >= a.tokens) return;
    if constexpr (FORWARD) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {                               // the up row of gate row m is row m + 16, register 4 (q + 2) + e
            const int n = r0 + wm * HALF + q * 8 + (lane >> 5) * 4, some = a.hidden - n;
            if (some <= 0) continue;
            f32x4 g, u, h;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                g[e] = acc[q * 4 + e];
                u[e] = acc[q * 4 + 8 + e];
            }
            if (a.partial != nullptr) {
                float *to = a.partial + (int64_t(split) * a.tokens + t) * 2 * a.hidden + n;
                store_four<false>(to, 0, g, some);
                store_four<false>(to, a.hidden, u, some);
                continue;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (a.bias != nullptr && e < some) {
                    g[e] += load_one<BF16>(a.bias, n + e);
                    u[e] += load_one<BF16>(a.bias, int64_t(a.hidden) + n + e);
                }
                h[e] = activation<BF16>(g[e], a.act) * u[e];
            }
            store_four<BF16>(a.out, t * a.hidden + n, h, some);
            if (a.pre != nullptr) {
                store_four<BF16>(a.pre, t * 2 * a.hidden + n, g, some);
                store_four<BF16>(a.pre, t * 2 * a.hidden + a.hidden + n, u, some);
            }
        }
    } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int c = r0 + wm * 32 + q * 8 + (lane >> 5) * 4, some = a.c_in - c;
            if (some <= 0) continue;
            f32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = acc[q * 4 + e];
            if (a.partial != nullptr) store_four<false>(a.partial, (int64_t(split) * a.tokens + t) * a.c_in + c, v, some);
            else store_four<BF16>(a.out, t * a.c_in + c, v, some);
        }
    }
}

// Adds the slices' partial sums in ascending order and finishes: bias, activation and product, or the rounding of dx.
template <bool BF16, bool FORWARD>
__global__ void __launch_bounds__(256)
gated_finish_kernel(const GenArgs a)
{
    const int width = FORWARD ? a.hidden : a.c_in;
    const int64_t total = a.tokens * width;
    const int64_t slice = a.tokens * (FORWARD ? 2 * int64_t(a.hidden) : a.c_in);
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < total; i += int64_t(gridDim.x) * 256) {
        const int64_t t = i / width, n = i - t * width;
        if constexpr (FORWARD) {
            const float *p = a.partial + t * 2 * a.hidden + n;
            float g = 0.f, u = 0.f;
            for (int s = 0; s < a.splits; ++s) {
                g += p[s * slice];
                u += p[s * slice + a.hidden];
            }
            if (a.bias != nullptr) {
                g += load_one<BF16>(a.bias, n);
                u += load_one<BF16>(a.bias, int64_t(a.hidden) + n);
            }
            store_one<BF16>(a.out, i, activation<BF16>(g, a.act) * u);
            if (a.pre != nullptr) {
                store_one<BF16>(a.pre, t * 2 * a.hidden + n, g);
                store_one<BF16>(a.pre, t * 2 * a.hidden + a.hidden + n, u);
            }
        } else {
            const float *p = a.partial + i;
            float v = 0.f;
            for (int s = 0; s < a.splits; ++s) v += p[s * slice];
            store_one<BF16>(a.out, i, v);
        }
    }
}

// Slices of the sum, at least eight steps of 32 in each (below that a slice is mostly its own start and end): enough workgroups for
// three on each of 256 compute units, as two leave a third of the time in waits where there is room for more (fp32, us, two and
// three: the gradient of 4000 tokens 384 -> 1024 84 and 74, of 1576 tokens 38.4 and 37.4, four 74 and 39.7).  fp32 products whose
// tiles leave compute units empty take slices of four steps (70 tokens 384 -> 1024 12.2 and 9.4 us; bf16 7.2 and 8.5 at 200 tokens
// 387 -> 515: its steps are shorter than what the second kernel costs).
struct GenPlan {
    int row_tiles, splits;
};
GenPlan gen_plan(int64_t tokens, int64_t c_in, int64_t hidden, dropit_dtype dt, bool forward)
{
    const int64_t across = forward ? 2 * hidden : c_in, K = forward ? c_in : 2 * hidden;
    const int64_t row_tiles = (across + GEN_ROWS - 1) / GEN_ROWS, steps = (K + GEN_K - 1) / GEN_K;
    const int64_t tiles = (tokens + GEN_TOKENS - 1) / GEN_TOKENS * row_tiles;
    int64_t splits = std::max<int64_t>(1, std::min(768 / tiles, steps / 8));
    if (dt == DROPIT_F32) splits = std::max(splits, std::min(256 / tiles, steps / 4));
    return GenPlan{int(row_tiles), int(splits)};
}

template <bool BF16, bool FORWARD>
void launch_finish(const GenArgs &a, hipStream_t stream)
{
    const int64_t blocks = (a.tokens * (FORWARD ? a.hidden : a.c_in) + 255) / 256;
    gated_finish_kernel<BF16, FORWARD><<<static_cast<uint32_t>(std::min<int64_t>(blocks, 1 << 16)), 256, 0, stream>>>(a);
}

template <bool BF16, bool FORWARD>
dropit_status launch_generic(GenArgs a, hipStream_t stream)
{
    const GenPlan plan = gen_plan(a.tokens, a.c_in, a.hidden, BF16 ? DROPIT_BF16 : DROPIT_F32, FORWARD);
    a.row_tiles = plan.row_tiles;
    a.splits = plan.splits;
    if (a.splits == 1) a.partial = nullptr;
    a.tiles = int((a.tokens + GEN_TOKENS - 1) / GEN_TOKENS * plan.row_tiles);
    // Token tiles that share a way through the weights: one while an XCD's cache holds all of those (us for one and for eight: bf16
    // gradients of 1003 tokens 387 -> 515 14.7 and 16.6, fp32 23.6 and 25.5), else eight (bf16 300 tokens 1111 -> 2777 23.2 and
    // 18.3, fp32 4096 tokens 768 -> 2048 223 and 213)
    a.group = 2 * int64_t(a.hidden) * a.c_in * (BF16 ? 2 : 4) <= int64_t(4) << 20 ? 1 : 8;
    const dim3 grid(static_cast<uint32_t>((a.tiles + 7) / 8 * 8), a.splits);
    gated_product_kernel<BF16, FORWARD><<<grid, GEN_THREADS, 0, stream>>>(a);
    if (a.splits > 1) launch_finish<BF16, FORWARD>(a, stream);
    return launch_status();
}

// Rows of any length into rows of whole 16-byte units, zeros behind the end: a copy, for the wide tiles' loads.
__global__ void __launch_bounds__(256)
gated_pad_kernel(const uint16_t *__restrict__ from, int64_t rows, int length, int pitch, uint16_t *__restrict__ to)
{
    const int units = pitch / 8;
    const int64_t total = rows * units;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < total; i += int64_t(gridDim.x) * 256) {
        const int64_t r = i / units;
        const int k = int(i - r * units) * 8;
        *reinterpret_cast<u32x4 *>(to + r * pitch + k) =
            k + 8 <= length ? *reinterpret_cast<const u32x4_any *>(from + r * length + k) : load_elements<true>(from + r * length, k, length);
    }
}

void launch_pad(const void *from, int64_t rows, int length, int pitch, void *to, hipStream_t stream)
{
    const int64_t blocks = (rows * (pitch / 8) + 255) / 256;
    gated_pad_kernel<<<static_cast<uint32_t>(std::min<int64_t>(blocks, 1 << 16)), 256, 0, stream>>>(static_cast<const uint16_t *>(from), rows, length, pitch, static_cast<uint16_t *>(to));
}

// Whether a product runs on wide tiles, and what it keeps in the workspace: the slices' partial sums, and copies of the operands
// whose rows are no whole 16-byte units.
struct WideLayout {
    bool takes;
    WidePlan plan;
    int w_pitch, x_pitch;
    bool pad_w, pad_x;
    size_t partial, w_at, x_at, bytes;                 // bytes of the partial sums, offsets of the copies, all
};

WideLayout wide_layout(int64_t tokens, int64_t c_in, int64_t hidden, bool forward)
{
    WideLayout l{};
    const int64_t k = forward ? c_in : 2 * hidden, c_pad = int64_t(round_up(c_in, 8)), k_pad = int64_t(round_up(k, 8));
    l.w_pitch = int(c_pad);
    l.x_pitch = int(k_pad);
    l.pad_w = c_pad != c_in;
    l.pad_x = k_pad != k;
    l.plan = gated_wide_plan(tokens, c_pad, hidden, forward);
    // Copies pay where the product is long: 2 bytes an element in and out at 4 TB/s and a launch each, against the product of this
    // file, which took 6 us and 230 TFLOP/s forward, 12 us and 180 backward, where it turns the weights element by element.  Both,
    // us: 8192 tokens 1111 -> 2777 122 and 431 forward, 126 and 452 backward; 300 tokens 34 and 22, 42 and 31.
    const double copies = (l.pad_w ? 4.0 + double(2 * hidden) * c_pad * 4 / 4e6 : 0.0) + (l.pad_x ? 4.0 + double(tokens) * k_pad * 4 / 4e6 : 0.0);
    const double work = 4.0 * double(tokens) * double(c_in) * double(hidden), here = forward ? 6.0 + work / 2.3e8 : 12.0 + work / 1.8e8;
    l.takes = l.plan.takes && (copies == 0.0 || l.plan.us + copies < here);
    if (!l.takes) return l;
    l.partial = l.plan.splits == 1 ? 0 : round_up(size_t(l.plan.splits) * tokens * (forward ? 2 * hidden : c_in) * sizeof(float), 256);
    l.w_at = l.partial;
    l.x_at = l.w_at + (l.pad_w ? round_up(size_t(2 * hidden) * c_pad * 2, 256) : 0);
    l.bytes = l.x_at + (l.pad_x ? round_up(size_t(tokens) * k_pad * 2, 256) : 0);
    return l;
}

template <bool FORWARD>
dropit_status launch_wide(GenArgs a, const WideLayout &l, void *workspace, hipStream_t stream)
{
    char *const ws = static_cast<char *>(workspace);
    WideArgs w{};
    w.w = a.w;
    w.x = a.x;
    if (l.pad_w) {
        launch_pad(a.w, 2 * int64_t(a.hidden), a.c_in, l.w_pitch, ws + l.w_at, stream);
        w.w = ws + l.w_at;
    }
    if (l.pad_x) {
        launch_pad(a.x, a.tokens, a.K, l.x_pitch, ws + l.x_at, stream);
        w.x = ws + l.x_at;
    }
    w.w_pitch = l.w_pitch;
    w.x_pitch = l.x_pitch;
    w.tokens = a.tokens;
    w.hidden = a.hidden;
    w.c_in = a.c_in;
    w.K = FORWARD ? l.x_pitch : a.K;
    w.act = a.act;
    w.bias = a.bias;
    w.out = a.out;
    w.pre = a.pre;
    w.partial = a.partial = static_cast<float *>(workspace);
    w.splits = a.splits = l.plan.splits;
    const dropit_status st = launch_gated_wide(w, l.plan, FORWARD, stream);
    if (st != DROPIT_OK || l.plan.splits == 1) return st;
    launch_finish<true, FORWARD>(a, stream);
    return launch_status();
}

// ---------------------------------------------------------------------------
// dpre from dh and pre, and the partial column sums for dbias.  A thread takes 8 (bf16) or 4 (fp32) gate columns, the up
// columns beside them and every fourth row of a block of rows; the four row groups' sums meet in LDS.  Bound by the bytes of dh,
// pre and dpre: 12608 tokens of 2048 columns in bf16 (258 MB) 54.6 us, 4.7 TB/s, where a copy reaches 5.1.
//
// In bf16 the input gradient is a product of dpre as it is rounded here, the dpre that the caller gets and that the weight
// gradient reads: all of them are gradients of one dpre, of the type that the matrix instructions take.  dx is 2.35e-3 off so,
// relative to the whole of it, of which its own rounding is 1.66e-3; dpre in two bf16 parts would leave only that, for a
// product of twice the work.  dbias is summed before the rounding.
constexpr int SLOPE_LANES = 64, SLOPE_GROUPS = 4, SLOPE_ROWS_MOST = 64;

template <bool BF16>
__global__ void __launch_bounds__(SLOPE_LANES * SLOPE_GROUPS)
gated_slope_kernel(const void *__restrict__ dh, const void *__restrict__ pre, int64_t tokens, int hidden, int rows, int act,
                   void *__restrict__ dpre, float *__restrict__ partial /* [row blocks][2 * hidden] or null */)
{
    constexpr int PER = Elem<BF16>::PER16;
    using T = typename Elem<BF16>::type;
    __shared__ float red[SLOPE_GROUPS][SLOPE_LANES * PER * 2];
    const int lane = threadIdx.x % SLOPE_LANES, group = threadIdx.x / SLOPE_LANES;
    const int n = int(blockIdx.x * SLOPE_LANES + lane) * PER;
    const int64_t t0 = int64_t(blockIdx.y) * rows, t1 = min<int64_t>(t0 + rows, tokens);
    float sg[PER], su[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) sg[e] = su[e] = 0.f;
    auto widen = [](const u32x4 &r, float (&x)[PER]) {
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            if constexpr (BF16) x[e] = __uint_as_float((e & 1) ? r[e >> 1] & 0xffff0000u : r[e >> 1] << 16);
            else x[e] = __uint_as_float(r[e]);
        }
    };
    auto narrow = [](const float (&x)[PER]) {
        u32x4 r;
        if constexpr (BF16) {
            bf16x8 b;
#pragma unroll
            for (int e = 0; e < PER; ++e) b[e] = static_cast<__bf16>(x[e]);
            r = __builtin_bit_cast(u32x4, b);
        } else {
#pragma unroll
            for (int e = 0; e < PER; ++e) r[e] = __float_as_uint(x[e]);
        }
        return r;
    };
    if (n < hidden) {
        const bool whole = n + PER <= hidden;
#pragma unroll 2
        for (int64_t t = t0 + group; t < t1; t += SLOPE_GROUPS) {
            const T *pd = static_cast<const T *>(dh) + t * hidden + n, *pg = static_cast<const T *>(pre) + t * 2 * hidden + n;
            T *og = static_cast<T *>(dpre) + t * 2 * hidden + n;
            float d[PER], g[PER], u[PER];
            if (whole) {
                const u32x4 rd = *reinterpret_cast<const u32x4_any *>(pd), rg = *reinterpret_cast<const u32x4_any *>(pg),
                            ru = *reinterpret_cast<const u32x4_any *>(pg + hidden);
                widen(rd, d);
                widen(rg, g);
                widen(ru, u);
            } else {
#pragma unroll
                for (int e = 0; e < PER; ++e) {
                    d[e] = g[e] = u[e] = 0.f;
                    if (n + e < hidden) {
                        d[e] = load_one<BF16>(pd, e);
                        g[e] = load_one<BF16>(pg, e);
                        u[e] = load_one<BF16>(pg + hidden, e);
                    }
                }
            }
            float slope[PER];
            activation_slopes<BF16>(g, act, slope);    // g becomes act(g)
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                u[e] = d[e] * u[e] * slope[e];
                g[e] = d[e] * g[e];
                sg[e] += u[e];
                su[e] += g[e];
            }
            if (whole) {
                *reinterpret_cast<u32x4_any *>(og) = narrow(u);
                *reinterpret_cast<u32x4_any *>(og + hidden) = narrow(g);
            } else {
#pragma unroll
                for (int e = 0; e < PER; ++e)
                    if (n + e < hidden) {
                        store_one<BF16>(og, e, u[e]);
                        store_one<BF16>(og + hidden, e, g[e]);
                    }
            }
        }
    }
    if (partial == nullptr) return;                    // (the same for every thread)
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        red[group][lane * PER + e] = sg[e];
        red[group][SLOPE_LANES * PER + lane * PER + e] = su[e];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < SLOPE_LANES * PER * 2; i += SLOPE_LANES * SLOPE_GROUPS) {
        const bool up = i >= SLOPE_LANES * PER;
        const int col = int(blockIdx.x) * SLOPE_LANES * PER + (up ? i - SLOPE_LANES * PER : i);
        if (col < hidden)
            partial[int64_t(blockIdx.y) * 2 * hidden + (up ? hidden : 0) + col] = (red[0][i] + red[1][i]) + (red[2][i] + red[3][i]);
    }
}

// dbias: the row blocks' partial sums of a column, 16 threads a column, in a fixed order.  Bound by the latency of its loads (197
// row blocks of 4096 columns: 4.5 us with eight of them at a time, 5.9 one by one).
__global__ void __launch_bounds__(256)
gated_bias_kernel(const float *__restrict__ partial, int64_t blocks, int64_t width, float *__restrict__ dbias)
{
    __shared__ float red[16][17];
    const int col = threadIdx.x & 15, part = threadIdx.x >> 4;
    const int64_t n = int64_t(blockIdx.x) * 16 + col;
    float s = 0.f;
    if (n < width)
#pragma unroll 8
        for (int64_t b = part; b < blocks; b += 16) s += partial[b * width + n];
    red[part][col] = s;
    __syncthreads();
    if (part != 0 || n >= width) return;
#pragma unroll
    for (int q = 1; q < 16; ++q) s += red[q][col];
    dbias[n] = s;
}

// columns of the slope kernel's workgroups, and the rows of each: 64 where that still leaves four workgroups to a compute unit,
// fewer for fewer tokens (64 tokens of 1024 columns took 16 us as one block of rows, one row after the other)
int64_t slope_strips(int64_t hidden, dropit_dtype dt)
{
    const int64_t per = dt == DROPIT_BF16 ? 8 : 4;
    return ((hidden + per - 1) / per + SLOPE_LANES - 1) / SLOPE_LANES;
}
int64_t slope_rows(int64_t tokens, int64_t hidden, dropit_dtype dt)
{
    const int64_t wanted = tokens * slope_strips(hidden, dt) / 1024;
    return std::min<int64_t>(SLOPE_ROWS_MOST, std::max<int64_t>(SLOPE_GROUPS, wanted / SLOPE_GROUPS * SLOPE_GROUPS));
}
int64_t row_blocks(int64_t tokens, int64_t rows) { return (tokens + rows - 1) / rows; }

bool valid_sizes(int64_t tokens, int64_t c_in, int64_t hidden, dropit_dtype dt)
{
    if (tokens < 0 || tokens > INT32_MAX || c_in < 1 || c_in > 1 << 28 || hidden < 1 || hidden > 1 << 27) return false;
    if (dt != DROPIT_F32 && dt != DROPIT_BF16) return false;
    // a launch has fewer than 2^32 threads
    const int64_t across = std::max((2 * hidden + GEN_ROWS - 1) / GEN_ROWS, (c_in + GEN_ROWS - 1) / GEN_ROWS);
    return (tokens + GEN_TOKENS - 1) / GEN_TOKENS * across <= (1 << 24) - 8;
}

size_t forward_bytes(int64_t tokens, int64_t c_in, int64_t hidden, dropit_dtype dt)
{
    if (tokens == 0 || gated_tokens_takes(tokens, c_in, hidden, dt)) return 0;
    if (dt == DROPIT_BF16) {
        const WideLayout l = wide_layout(tokens, c_in, hidden, true);
        if (l.takes) return l.bytes;
    }
    const int splits = gen_plan(tokens, c_in, hidden, dt, true).splits;
    return splits == 1 ? 0 : size_t(splits) * tokens * 2 * hidden * sizeof(float);
}

size_t dx_bytes(int64_t tokens, int64_t c_in, int64_t hidden, dropit_dtype dt)
{
    if (tokens == 0) return 0;
    if (dt == DROPIT_BF16) {
        const WideLayout l = wide_layout(tokens, c_in, hidden, false);
        if (l.takes) return l.bytes;
    }
    const int splits = gen_plan(tokens, c_in, hidden, dt, false).splits;
    return splits == 1 ? 0 : size_t(splits) * tokens * c_in * sizeof(float);
}

}  // namespace
}  // namespace dropit

using namespace dropit;

extern "C" size_t dropit_gated_forward_workspace_bytes(int64_t tokens, int64_t c_in, int64_t hidden, dropit_dtype dt)
{
    if (!valid_sizes(tokens, c_in, hidden, dt)) return 0;
    return forward_bytes(tokens, c_in, hidden, dt);
}

extern "C" dropit_status dropit_gated_forward(const void *x, int64_t tokens, int64_t c_in, dropit_dtype dt, const void *w,
                                              const void *bias, int64_t hidden, dropit_act act, void *h, void *pre,
                                              void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (!valid_sizes(tokens, c_in, hidden, dt) || act < DROPIT_ACT_SILU || act > DROPIT_ACT_SIGMOID) return DROPIT_EINVAL;
    if (tokens == 0) return DROPIT_OK;
    if (!x || !w || !h || !aligned(x, 16) || !aligned(w, 16) || !aligned(h, 16) || !aligned(bias, 16) || !aligned(pre, 16))
        return DROPIT_EINVAL;
    const size_t need = forward_bytes(tokens, c_in, hidden, dt);
    if (need > 0 && (workspace == nullptr || !aligned(workspace, 256))) return DROPIT_EINVAL;
    if (workspace_bytes < need) return DROPIT_EWORKSPACE;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    GenArgs a{};
    a.w = w;
    a.x = x;
    a.tokens = tokens;
    a.hidden = int(hidden);
    a.c_in = int(c_in);
    a.K = int(c_in);
    a.act = act;
    a.bias = bias;
    a.out = h;
    a.pre = pre;
    a.partial = static_cast<float *>(workspace);
    if (gated_tokens_takes(tokens, c_in, hidden, dt)) return launch_gated_tokens(x, tokens, a.c_in, dt, w, bias, a.hidden, act, h, pre, stream);
    if (dt == DROPIT_BF16) {
        const WideLayout l = wide_layout(tokens, c_in, hidden, true);
        if (l.takes) return launch_wide<true>(a, l, workspace, stream);
    }
    return dt == DROPIT_BF16 ? launch_generic<true, true>(a, stream) : launch_generic<false, true>(a, stream);
}

extern "C" size_t dropit_gated_backward_workspace_bytes(int64_t tokens, int64_t c_in, int64_t hidden, dropit_dtype dt, int need_dx,
                                                        int need_dbias)
{
    if (!valid_sizes(tokens, c_in, hidden, dt)) return 0;
    size_t need = need_dx ? dx_bytes(tokens, c_in, hidden, dt) : 0;
    if (need_dbias) need = std::max(need, size_t(row_blocks(tokens, slope_rows(tokens, hidden, dt))) * 2 * hidden * sizeof(float));
    return need;
}

extern "C" dropit_status dropit_gated_backward(const void *dh, const void *pre, int64_t tokens, int64_t c_in, dropit_dtype dt,
                                               const void *w, int64_t hidden, dropit_act act, void *dpre, void *dx, float *dbias,
                                               void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (!valid_sizes(tokens, c_in, hidden, dt) || act < DROPIT_ACT_SILU || act > DROPIT_ACT_SIGMOID) return DROPIT_EINVAL;
    if (!aligned(dbias, 16)) return DROPIT_EINVAL;
    if (tokens > 0 && (!dh || !pre || !dpre || (dx && !w) || !aligned(dh, 16) || !aligned(pre, 16) || !aligned(dpre, 16) ||
                       !aligned(w, 16) || !aligned(dx, 16)))
        return DROPIT_EINVAL;
    const size_t need = dropit_gated_backward_workspace_bytes(tokens, c_in, hidden, dt, dx != nullptr, dbias != nullptr);
    if (need > 0 && (workspace == nullptr || !aligned(workspace, 256))) return DROPIT_EINVAL;
    if (workspace_bytes < need) return DROPIT_EWORKSPACE;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const bool bf16 = dt == DROPIT_BF16;
    // the partial column sums and, when those are added, dx's slices share the workspace, one after the other
    float *partial = dbias != nullptr ? static_cast<float *>(workspace) : nullptr;
    const int64_t rows = slope_rows(tokens, hidden, dt), blocks = row_blocks(tokens, rows);
    // the grid's second dimension holds 65535 row blocks: more tokens go in several launches
    for (int64_t b0 = 0; b0 < blocks; b0 += 65535) {
        const int64_t first = b0 * rows, some = std::min<int64_t>(tokens - first, int64_t(65535) * rows);
        const dim3 grid(static_cast<uint32_t>(slope_strips(hidden, dt)), static_cast<uint32_t>(row_blocks(some, rows)));
        const size_t es = bf16 ? 2 : 4;
        const char *d = static_cast<const char *>(dh) + first * hidden * es;
        const char *p = static_cast<const char *>(pre) + first * 2 * hidden * es;
        char *o = static_cast<char *>(dpre) + first * 2 * hidden * es;
        float *part = partial != nullptr ? partial + b0 * 2 * hidden : nullptr;
        if (bf16) gated_slope_kernel<true><<<grid, SLOPE_LANES * SLOPE_GROUPS, 0, stream>>>(d, p, some, int(hidden), int(rows), act, o, part);
        else gated_slope_kernel<false><<<grid, SLOPE_LANES * SLOPE_GROUPS, 0, stream>>>(d, p, some, int(hidden), int(rows), act, o, part);
    }
    if (dbias != nullptr)
        gated_bias_kernel<<<static_cast<uint32_t>((2 * hidden + 15) / 16), 256, 0, stream>>>(partial, blocks, 2 * hidden, dbias);
    if (dx == nullptr || tokens == 0) return launch_status();
    GenArgs a{};
    a.w = w;
    a.x = dpre;
    a.tokens = tokens;
    a.hidden = int(hidden);
    a.c_in = int(c_in);
    a.K = int(2 * hidden);
    a.act = act;
    a.out = dx;
    a.partial = static_cast<float *>(workspace);
    if (bf16) {
        const WideLayout l = wide_layout(tokens, c_in, hidden, false);
        if (l.takes) return launch_wide<false>(a, l, workspace, stream);
    }
    return bf16 ? launch_generic<true, false>(a, stream) : launch_generic<false, false>(a, stream);
}
