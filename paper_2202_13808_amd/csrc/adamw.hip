// AdamW over many tensors at once, with states in fp32 or in 8 bits (the formulas stand in dropit_layers.h).
//
// A streaming operator: 28 bytes an element with everything in fp32, 10 in bf16 with 8-bit states.  What it must not do
// is start a kernel per tensor or keep a table of pointers in device memory that gradients allocated anew each step
// would outdate: the table of 58 to 90 tensors, by how many pointers each needs, travels in the kernel's arguments, and a
// workgroup finds its tensor by a search over the tensors' first chunks.
//
// A thread takes 8 consecutive elements, so that bf16 moves 16 bytes an access and 8-bit codes 8; 32 lanes share a block of
// 256 elements and find its largest pattern by five lane exchanges, without LDS or a second pass over the data.
//
// The arithmetic is that of single fp32 operations, correctly rounded division and square root included: the codes and the
// residual's 16 bits are exact functions of the inputs, which any other implementation of the formulas reproduces.
//
// Measured: 21.8 M fp32 parameters in 150 tensors 134 us, 4.5 TB/s of the 5.1 that a large copy reaches; 269 M bf16 parameters in
// 16 tensors with 8-bit states 620 us, 4.3 TB/s.
#include <cmath>
#include <type_traits>

#include "common.hpp"
#include "dropit_layers.h"

namespace dropit {
namespace {

constexpr int ADAMW_THREADS = 256;
constexpr int ADAMW_PER_THREAD = 8;
constexpr int ADAMW_ROUNDS = 2;                                             // rounds of 2048 elements a workgroup makes
constexpr int ADAMW_CHUNK = ADAMW_THREADS * ADAMW_PER_THREAD * ADAMW_ROUNDS;
constexpr uint32_t WEYL_I = 0x6a09e667u, WEYL_T = 0x9e3779b9u;              // odd: every residue mod 2^32 once a period
constexpr uint32_t LAST_FINITE = 0x7f7u, NAN_OFFSET = 0x7f9u, NAN_CODE = 0x7ffu;

constexpr int64_t ADAMW_MAX_NUMEL = int64_t(1) << 34;                       // a launch has fewer than 2^32 threads
constexpr uint32_t MAX_CHUNKS = 1u << 23;
static_assert(ADAMW_MAX_NUMEL / ADAMW_CHUNK <= MAX_CHUNKS && ADAMW_MAX_NUMEL / (ADAMW_THREADS * ADAMW_PER_THREAD) <= MAX_CHUNKS, "");

// p, g, m, v, then the offsets of 8-bit states, then the residual: what a kind of step needs of each tensor.  As many tensors as
// keep the arguments under 4 KB (48 of them took 4 launches for the 150 tensors of a 12-block encoder, 147 us for 140)
template <bool RESIDUAL, bool BITS8> struct AdamwTable {
    static constexpr int POINTERS = 4 + (BITS8 ? 2 : 0) + (RESIDUAL ? 1 : 0);
    static constexpr int MOST = (4096 - 128) / (POINTERS * 8 + 12);
    void *pointer[POINTERS][MOST];
    int64_t numel[MOST];
    uint32_t first[MOST];                              // first chunk of each tensor
    int count;
};

struct AdamwScalars {
    float beta1, rest1, beta2, rest2, eps, decay;      // rest = 1 - beta, decay = 1 - lr * weight_decay
    float root2, rate;                                 // 1 / sqrt(1 - beta2^t), lr / (1 - beta1^t): host step only
    uint32_t weyl;                                     // t * WEYL_T
    const float *grad_scale;
    const int32_t *step;                               // device step, or null
    double lr, beta1d, beta2d;
};
static_assert(sizeof(AdamwScalars) <= 112, "kernel arguments");

typedef __attribute__((ext_vector_type(4))) float af32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t au32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t au32x2;

// beta^t for t >= 1 by repeated squaring: at most 62 roundings of 2^-53, far below the fp32 that the result is used in
__device__ inline double int_power(double b, uint32_t t)
{
    double r = 1.0;
    for (; t; t >>= 1, b *= b)
        if (t & 1u) r *= b;
    return r;
}

__device__ inline float widen(uint32_t bf16_bits) { return __uint_as_float(bf16_bits << 16); }

__device__ inline uint32_t to_bf16(float f)            // nearest even; a NaN stays one
{
    const uint32_t b = __float_as_uint(f);
    return f != f ? 0x7fc0u : (b + 0x7fffu + ((b >> 16) & 1u)) >> 16;
}

// the largest of 32 lanes' values, in every one of them
__device__ inline uint32_t half_wave_max(uint32_t v)
{
#define DROPIT_DPP_MAX(ctrl) v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), ctrl, 0xf, 0xf, true)))
    DROPIT_DPP_MAX(0xb1);      // quad_perm 1,0,3,2
    DROPIT_DPP_MAX(0x4e);      // quad_perm 2,3,0,1
    DROPIT_DPP_MAX(0x141);     // row_half_mirror
    DROPIT_DPP_MAX(0x140);     // row_mirror        -> the largest of each row of 16
#undef DROPIT_DPP_MAX
    return max(v, uint32_t(__shfl_xor(int(v), 16, WAVE)));
}

// 8 consecutive elements from element i, in registers as fp32; VEC: 16-byte accesses
template <bool BF16, bool VEC>
__device__ inline void load8(const void *base, int64_t i, int n, float (&x)[8])
{
    if constexpr (VEC && BF16) {
        const au32x4 w = *reinterpret_cast<const au32x4 *>(static_cast<const uint16_t *>(base) + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[2 * e] = __uint_as_float(w[e] << 16);
            x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
        }
    } else if constexpr (VEC) {
        const af32x4 *q = reinterpret_cast<const af32x4 *>(static_cast<const float *>(base) + i);
        const af32x4 a = q[0], b = q[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] = a[e];
            x[4 + e] = b[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = 0.f;
            if (e < n) x[e] = BF16 ? widen(static_cast<const uint16_t *>(base)[i + e]) : static_cast<const float *>(base)[i + e];
        }
    }
}

template <bool VEC>
__device__ inline void store8_f32(void *base, int64_t i, int n, const float (&x)[8])
{
    if constexpr (VEC) {
        af32x4 *q = reinterpret_cast<af32x4 *>(static_cast<float *>(base) + i);
        q[0] = af32x4{x[0], x[1], x[2], x[3]};
        q[1] = af32x4{x[4], x[5], x[6], x[7]};
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) static_cast<float *>(base)[i + e] = x[e];
    }
}

template <bool VEC>
__device__ inline void store8_u16(void *base, int64_t i, int n, const uint32_t (&x)[8])
{
    if constexpr (VEC) {
        *reinterpret_cast<au32x4 *>(static_cast<uint16_t *>(base) + i) =
            au32x4{x[0] | (x[1] << 16), x[2] | (x[3] << 16), x[4] | (x[5] << 16), x[6] | (x[7] << 16)};
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) static_cast<uint16_t *>(base)[i + e] = uint16_t(x[e]);
    }
}

template <bool VEC>
__device__ inline au32x2 load8_codes(const void *base, int64_t i, int n)
{
    if constexpr (VEC) {
        return *reinterpret_cast<const au32x2 *>(static_cast<const uint8_t *>(base) + i);
    } else {
        au32x2 c = {0u, 0u};
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) c[e >> 2] |= uint32_t(static_cast<const uint8_t *>(base)[i + e]) << (8 * (e & 3));
        return c;
    }
}

template <bool VEC>
__device__ inline void store8_codes(void *base, int64_t i, int n, au32x2 c)
{
    if constexpr (VEC) {
        *reinterpret_cast<au32x2 *>(static_cast<uint8_t *>(base) + i) = c;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) static_cast<uint8_t *>(base)[i + e] = uint8_t(c[e >> 2] >> (8 * (e & 3)));
    }
}

// the fp32 pattern (no sign) of a magnitude code
__device__ inline uint32_t decode_bits(uint32_t code, uint32_t offset)
{
    return code == 0u ? 0u : min(code + offset, NAN_CODE) << 20;
}

template <bool SIGNED>
__device__ inline void decode8(au32x2 c, uint32_t offset, float (&x)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t code = (c[e >> 2] >> (8 * (e & 3))) & 0xffu;
        if constexpr (SIGNED) x[e] = __uint_as_float(decode_bits(code & 127u, offset) | ((code & 128u) << 24));
        else x[e] = __uint_as_float(decode_bits(code, offset));
    }
}

// the codes of 8 of a block's values (32 lanes hold the block), and the block's offset
template <bool SIGNED>
__device__ inline au32x2 encode8(const float (&x)[8], uint32_t weyl, uint32_t &offset)
{
    constexpr uint32_t TOP = SIGNED ? 127u : 255u;
    uint32_t b[8], largest = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        b[e] = __float_as_uint(x[e]) & 0x7fffffffu;
        largest = max(largest, b[e]);
    }
    largest = half_wave_max(largest);
    if (largest >= 0x7f800000u) {                      // an infinity or a NaN: the whole block decodes to NaN
        offset = NAN_OFFSET;
        return SIGNED ? au32x2{0x7f7f7f7fu, 0x7f7f7f7fu} : au32x2{0xffffffffu, 0xffffffffu};
    }
    offset = uint32_t(max(int(min((largest + 0xfffffu) >> 20, LAST_FINITE)) - int(TOP), 0));
    au32x2 c = {0u, 0u};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t h = (weyl + uint32_t(e) * WEYL_I) >> 12;
        const uint32_t d = SIGNED ? h : h ^ 0xfffffu;
        int code = max(int(min((b[e] + d) >> 20, LAST_FINITE)) - int(offset), 0);
        if constexpr (SIGNED) code |= x[e] < 0.f ? 128 : 0;
        else code = b[e] != 0u ? max(code, 1) : 0;
        c[e >> 2] |= uint32_t(code) << (8 * (e & 3));
    }
    return c;
}

// the same with the width decided per lane
template <bool BF16, bool VEC>
__device__ inline void load8(const void *base, int64_t i, int n, bool wide, float (&x)[8])
{
    if (VEC || wide) load8<BF16, true>(base, i, n, x);
    else load8<BF16, false>(base, i, n, x);
}
template <bool VEC>
__device__ inline void store8_f32(void *base, int64_t i, int n, bool wide, const float (&x)[8])
{
    if (VEC || wide) store8_f32<true>(base, i, n, x);
    else store8_f32<false>(base, i, n, x);
}
template <bool VEC>
__device__ inline void store8_u16(void *base, int64_t i, int n, bool wide, const uint32_t (&x)[8])
{
    if (VEC || wide) store8_u16<true>(base, i, n, x);
    else store8_u16<false>(base, i, n, x);
}
template <bool VEC>
__device__ inline au32x2 load8_codes(const void *base, int64_t i, int n, bool wide)
{
    if (VEC || wide) return load8_codes<true>(base, i, n);
    return load8_codes<false>(base, i, n);
}
template <bool VEC>
__device__ inline void store8_codes(void *base, int64_t i, int n, bool wide, au32x2 c)
{
    if (VEC || wide) store8_codes<true>(base, i, n, c);
    else store8_codes<false>(base, i, n, c);
}

// One round of a thread: 8 elements from element i of the tensor, n of them inside it.  VEC: all of the workgroup's are and
// move in wide accesses; otherwise `wide` says so of this thread's.
template <bool P_BF16, bool RESIDUAL, bool G_BF16, bool BITS8, bool VEC>
__device__ inline void adamw_elements(const dropit_adamw_tensor &t, const AdamwScalars &s, float root2, float rate, float scale,
                                      uint32_t weyl_t, int64_t i, int n, bool wide)
{
#pragma clang fp contract(off)
    float p[8], g[8], m[8], v[8];
    au32x2 mc, vc;
    uint32_t mo = 0, vo = 0, low[8];
    const int64_t block = i / DROPIT_ADAMW_BLOCK;
    load8<G_BF16, VEC>(t.g, i, n, wide, g);
    load8<P_BF16, VEC>(t.p, i, n, wide, p);
    if constexpr (RESIDUAL) {
        float raw[8];                                  // (the 16 bits in the upper half of a register, as bf16 arrive)
        load8<true, VEC>(t.residual, i, n, wide, raw);
#pragma unroll
        for (int e = 0; e < 8; ++e) low[e] = __float_as_uint(raw[e]);
    }
    if constexpr (BITS8) {
        mc = load8_codes<VEC>(t.m, i, n, wide);
        vc = load8_codes<VEC>(t.v, i, n, wide);
        if (n > 0) {
            mo = uint16_t(t.m_offset[block]);
            vo = uint16_t(t.v_offset[block]);
        }
        decode8<true>(mc, mo, m);
        decode8<false>(vc, vo, v);
    } else {
        load8<false, VEC>(t.m, i, n, wide, m);
        load8<false, VEC>(t.v, i, n, wide, v);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if constexpr (RESIDUAL) p[e] = __uint_as_float(__float_as_uint(p[e]) + uint32_t(int32_t(low[e]) >> 16));
        const float ge = g[e] * scale;
        m[e] = m[e] * s.beta1 + ge * s.rest1;
        v[e] = v[e] * s.beta2 + (ge * ge) * s.rest2;
        const float step = m[e] / (sqrtf(v[e]) * root2 + s.eps);
        p[e] = p[e] * s.decay - step * rate;
    }
    if constexpr (!P_BF16) {
        store8_f32<VEC>(t.p, i, n, wide, p);
    } else {
        uint32_t hi[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (RESIDUAL) {
                const uint32_t b = p[e] != p[e] ? 0x7fc00000u : __float_as_uint(p[e]);
                hi[e] = (b + 0x8000u) >> 16;
                low[e] = (b - (hi[e] << 16)) & 0xffffu;
            } else {
                hi[e] = to_bf16(p[e]);
            }
        }
        store8_u16<VEC>(t.p, i, n, wide, hi);
        if constexpr (RESIDUAL) store8_u16<VEC>(t.residual, i, n, wide, low);
    }
    if constexpr (BITS8) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {                  // elements past the end: zeros, whatever the arithmetic made of them
            m[e] = e < n ? m[e] : 0.f;
            v[e] = e < n ? v[e] : 0.f;
        }
        const uint32_t weyl = uint32_t(i) * WEYL_I + weyl_t;
        mc = encode8<true>(m, weyl, mo);
        vc = encode8<false>(v, weyl, vo);
        store8_codes<VEC>(t.m, i, n, wide, mc);
        store8_codes<VEC>(t.v, i, n, wide, vc);
        if ((threadIdx.x & 31) == 0 && n > 0) {
            t.m_offset[block] = int16_t(mo);
            t.v_offset[block] = int16_t(vo);
        }
    } else {
        store8_f32<VEC>(t.m, i, n, wide, m);
        store8_f32<VEC>(t.v, i, n, wide, v);
    }
}

template <bool P_BF16, bool RESIDUAL, bool G_BF16, bool BITS8>
__global__ void __launch_bounds__(ADAMW_THREADS)
adamw_kernel(const AdamwTable<RESIDUAL, BITS8> table, const AdamwScalars s)
{
    __shared__ float shared[2];
    // the last tensor whose first chunk is not behind this one
    int lo = 0, hi = table.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (table.first[mid] <= blockIdx.x) lo = mid; else hi = mid - 1;
    }
    dropit_adamw_tensor t = {};
    t.p = table.pointer[0][lo];
    t.g = table.pointer[1][lo];
    t.m = table.pointer[2][lo];
    t.v = table.pointer[3][lo];
    if constexpr (BITS8) {
        t.m_offset = static_cast<int16_t *>(table.pointer[4][lo]);
        t.v_offset = static_cast<int16_t *>(table.pointer[5][lo]);
    }
    if constexpr (RESIDUAL) t.residual = static_cast<int16_t *>(table.pointer[table.POINTERS - 1][lo]);
    t.numel = table.numel[lo];
    float root2 = s.root2, rate = s.rate;
    uint32_t weyl_t = s.weyl;
    if (s.step != nullptr) {
        const uint32_t step = uint32_t(max(*s.step, 1));
        if (threadIdx.x < WAVE) {
            shared[0] = float(1.0 / sqrt(1.0 - int_power(s.beta2d, step)));
            shared[1] = float(s.lr / (1.0 - int_power(s.beta1d, step)));
        }
        __syncthreads();
        root2 = shared[0];
        rate = shared[1];
        weyl_t = step * WEYL_T;
    }
    const float scale = s.grad_scale != nullptr ? *s.grad_scale : 1.f;
    uintptr_t bits = reinterpret_cast<uintptr_t>(t.p) | reinterpret_cast<uintptr_t>(t.g);
    if (RESIDUAL) bits |= reinterpret_cast<uintptr_t>(t.residual);
    if (BITS8) bits |= (reinterpret_cast<uintptr_t>(t.m) | reinterpret_cast<uintptr_t>(t.v)) << 1;
    else bits |= reinterpret_cast<uintptr_t>(t.m) | reinterpret_cast<uintptr_t>(t.v);
    const int64_t chunk0 = int64_t(blockIdx.x - table.first[lo]) * ADAMW_CHUNK;
    const bool wide = (bits & 15u) == 0, whole = wide && chunk0 + ADAMW_CHUNK <= t.numel;
#pragma unroll
    for (int r = 0; r < ADAMW_ROUNDS; ++r) {
        const int64_t i = chunk0 + (r * ADAMW_THREADS + int(threadIdx.x)) * ADAMW_PER_THREAD;
        if (whole) {
            adamw_elements<P_BF16, RESIDUAL, G_BF16, BITS8, true>(t, s, root2, rate, scale, weyl_t, i, ADAMW_PER_THREAD, true);
        } else {
            // (the lanes past the end go through the block's exchanges too, with no elements)
            const int n = int(max<int64_t>(min<int64_t>(t.numel - i, ADAMW_PER_THREAD), 0));
            adamw_elements<P_BF16, RESIDUAL, G_BF16, BITS8, false>(t, s, root2, rate, scale, weyl_t, i, n, wide && n == ADAMW_PER_THREAD);
        }
    }
}

template <bool SIGNED>
__global__ void __launch_bounds__(ADAMW_THREADS)
adamw_unpack_kernel(const uint8_t *__restrict__ codes, const int16_t *__restrict__ offsets, int64_t numel, bool wide,
                    uint16_t *__restrict__ values)
{
    const int64_t i = (int64_t(blockIdx.x) * ADAMW_THREADS + threadIdx.x) * ADAMW_PER_THREAD;
    if (i >= numel) return;
    const int n = int(min<int64_t>(numel - i, ADAMW_PER_THREAD));
    const uint32_t offset = uint16_t(offsets[i / DROPIT_ADAMW_BLOCK]);
    float x[8];
    uint32_t out[8];
    wide = wide && n == ADAMW_PER_THREAD;
    decode8<SIGNED>(load8_codes<false>(codes, i, n, wide), offset, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] = __float_as_uint(x[e]) >> 16;       // exact: the lower half is zero
    store8_u16<false>(values, i, n, wide, out);
}

template <bool P_BF16, bool RESIDUAL, bool G_BF16, bool BITS8>
void launch_adamw(const dropit_adamw_tensor *tensors, int64_t count, const AdamwScalars &s, hipStream_t stream)
{
    using Table = AdamwTable<RESIDUAL, BITS8>;
    static_assert(sizeof(Table) + sizeof(AdamwScalars) <= 4096, "kernel arguments");
    Table table;
    table.count = 0;
    uint32_t chunks = 0;
    auto flush = [&]() {
        if (table.count == 0) return;
        adamw_kernel<P_BF16, RESIDUAL, G_BF16, BITS8><<<chunks, ADAMW_THREADS, 0, stream>>>(table, s);
        table.count = 0;
        chunks = 0;
    };
    for (int64_t j = 0; j < count; ++j) {
        const dropit_adamw_tensor &t = tensors[j];
        if (t.numel == 0) continue;
        const uint32_t need = uint32_t((t.numel + ADAMW_CHUNK - 1) / ADAMW_CHUNK);
        if (table.count == Table::MOST || chunks + need > MAX_CHUNKS) flush();
        const int at = table.count++;
        table.pointer[0][at] = t.p;
        table.pointer[1][at] = const_cast<void *>(t.g);
        table.pointer[2][at] = t.m;
        table.pointer[3][at] = t.v;
        if constexpr (BITS8) {
            table.pointer[4][at] = t.m_offset;
            table.pointer[5][at] = t.v_offset;
        }
        if constexpr (RESIDUAL) table.pointer[Table::POINTERS - 1][at] = t.residual;
        table.numel[at] = t.numel;
        table.first[at] = chunks;
        chunks += need;
    }
    flush();
}

bool valid_dtype(dropit_dtype dt) { return dt == DROPIT_F32 || dt == DROPIT_BF16; }

}  // namespace
}  // namespace dropit

using namespace dropit;

extern "C" dropit_status dropit_adamw(const dropit_adamw_tensor *tensors, int64_t count, dropit_dtype p_dtype,
                                      dropit_dtype g_dtype, int state_bits, const dropit_adamw_hyper *hyper, void *hip_stream)
{
    if (count < 0 || (count > 0 && tensors == nullptr) || hyper == nullptr || !valid_dtype(p_dtype) || !valid_dtype(g_dtype) ||
        (state_bits != 8 && state_bits != 32))
        return DROPIT_EINVAL;
    const dropit_adamw_hyper &h = *hyper;
    if (!std::isfinite(h.lr) || !std::isfinite(h.weight_decay) || !std::isfinite(h.eps) || !(h.eps >= 0.0) ||
        !(h.beta1 >= 0.0 && h.beta1 < 1.0) || !(h.beta2 >= 0.0 && h.beta2 < 1.0))
        return DROPIT_EINVAL;
    if (h.step_device == nullptr && h.step < 1) return DROPIT_EINVAL;
    if (!aligned(h.step_device, 4) || !aligned(h.grad_scale, 4)) return DROPIT_EINVAL;
    const bool bits8 = state_bits == 8, pbf = p_dtype == DROPIT_BF16, gbf = g_dtype == DROPIT_BF16;
    bool residual = false, any = false;
    for (int64_t j = 0; j < count; ++j) {
        const dropit_adamw_tensor &t = tensors[j];
        if (t.numel < 0 || t.numel > ADAMW_MAX_NUMEL) return DROPIT_EINVAL;
        if (t.numel == 0) continue;
        if (!t.p || !t.g || !t.m || !t.v) return DROPIT_EINVAL;
        if (!aligned(t.p, pbf ? 2 : 4) || !aligned(t.g, gbf ? 2 : 4)) return DROPIT_EINVAL;
        if (bits8) {
            if (!t.m_offset || !t.v_offset || !aligned(t.m_offset, 2) || !aligned(t.v_offset, 2)) return DROPIT_EINVAL;
        } else if (t.m_offset || t.v_offset || !aligned(t.m, 4) || !aligned(t.v, 4)) {
            return DROPIT_EINVAL;
        }
        if (t.residual && (!pbf || !aligned(t.residual, 2))) return DROPIT_EINVAL;
        if (any && residual != (t.residual != nullptr)) return DROPIT_EINVAL;
        residual = t.residual != nullptr;
        any = true;
    }
    if (!any) return DROPIT_OK;
    AdamwScalars s;
    s.beta1 = float(h.beta1);
    s.rest1 = float(1.0 - h.beta1);
    s.beta2 = float(h.beta2);
    s.rest2 = float(1.0 - h.beta2);
    s.eps = float(h.eps);
    s.decay = float(1.0 - h.lr * h.weight_decay);
    s.root2 = s.rate = 0.f;
    s.weyl = 0;
    if (h.step_device == nullptr) {
        s.root2 = float(1.0 / std::sqrt(1.0 - std::pow(h.beta2, double(h.step))));
        s.rate = float(h.lr / (1.0 - std::pow(h.beta1, double(h.step))));
        s.weyl = uint32_t(h.step) * WEYL_T;
    }
    s.grad_scale = h.grad_scale;
    s.step = h.step_device;
    s.lr = h.lr;
    s.beta1d = h.beta1;
    s.beta2d = h.beta2;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    auto launch = [&](auto p, auto r, auto g) {
        constexpr bool P = decltype(p)::value, R = decltype(r)::value, G = decltype(g)::value;
        if (bits8) launch_adamw<P, R, G, true>(tensors, count, s, stream);
        else launch_adamw<P, R, G, false>(tensors, count, s, stream);
    };
    constexpr std::true_type yes{};
    constexpr std::false_type no{};
    if (!pbf) gbf ? launch(no, no, yes) : launch(no, no, no);
    else if (residual) gbf ? launch(yes, yes, yes) : launch(yes, yes, no);
    else gbf ? launch(yes, no, yes) : launch(yes, no, no);
    return launch_status();
}

extern "C" dropit_status dropit_adamw_unpack(const uint8_t *codes, const int16_t *offsets, int64_t numel, int is_signed,
                                             void *values, void *hip_stream)
{
    if (numel < 0 || numel > ADAMW_MAX_NUMEL || (is_signed != 0 && is_signed != 1)) return DROPIT_EINVAL;
    if (numel == 0) return DROPIT_OK;
    if (!codes || !offsets || !values || !aligned(offsets, 2) || !aligned(values, 2)) return DROPIT_EINVAL;
    const bool wide = aligned(codes, 8) && aligned(values, 16);
    constexpr int PER_WG = ADAMW_THREADS * ADAMW_PER_THREAD;
    const uint32_t blocks = uint32_t((numel + PER_WG - 1) / PER_WG);
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    uint16_t *out = static_cast<uint16_t *>(values);
    if (is_signed) adamw_unpack_kernel<true><<<blocks, ADAMW_THREADS, 0, stream>>>(codes, offsets, numel, wide, out);
    else adamw_unpack_kernel<false><<<blocks, ADAMW_THREADS, 0, stream>>>(codes, offsets, numel, wide, out);
    return launch_status();
}
