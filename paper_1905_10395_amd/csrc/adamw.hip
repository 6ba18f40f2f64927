// One AdamW step over every tensor of a program at once, moments held in 32 or in 8 bits.
//
//   g' = c g;  m <- b1 m + (1-b1) g';  v <- b2 v + (1-b2) g' g'
//   x <- x (1 - lr wd) - lr/(1-b1^t) * m / (sqrt(v)/sqrt(1-b2^t) + eps)
//
// Every product, sum, quotient and root is rounded to fp32 by itself (no fused multiply-add): the stored bits then do
// not depend on which code path or compiler evaluates the expression, and the 8-bit codes, where one last bit can move
// a value to the next code, stay reproducible.  The arithmetic hides behind the memory accesses.
//
// 8-bit moments.  A block of 256 elements of a tensor's row shares an fp32 scale: m = sign(q) q^2 s_m with |q| <= 127 and
// sqrt(v) = q^2 s_v with q <= 255, s = (largest in the block) / q_max^2, so the spacing of stored values is 2/q of the
// value: 1.6 % (0.8 %) near the block's largest, and values down to 1/16129 (1/65025) of it are told from zero.  A moment
// changes by a fraction 1-b of itself a step, less than the spacing: rounded to nearest it would never move.  So the
// point between two neighbouring codes above which the upper one is taken walks through (0,1) with the step number by
// the golden ratio; over any run of steps each code is taken in proportion to how near the value is, and slow drift is
// kept on average.  Between two codes v (not its root) is interpolated, or the second moment would be biased upwards.
//
// Bound by memory: 28 bytes an element (x, m, v read and written, g read) with 32-bit moments, 16 with 8-bit ones.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "common.h"

using namespace lsgd;

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));

constexpr int kBlock = LSGD_ADAMW_BLOCK;             // elements that share a scale: one wavefront, four each
static_assert(kBlock == 4 * kWave, "a wavefront holds one block");
// Elements of one workgroup: short pieces in memory order keep what the chip has open in a few DRAM pages (268 M parameters of 30
// bytes 1.32 ms, with 2048 elements 1.31; before accesses were streaming and lanes short, 1.39 and 1.46, and 1.54 with 4096).
constexpr int kChunk = 1024;
constexpr int kThreads32 = kChunk / 2;               // 8-byte lanes: 1.32 ms, against 1.37 with 16-byte ones
constexpr int kThreads = kChunk / 4;
constexpr float kTopM = 127.0f * 127.0f, kTopV = 255.0f * 255.0f;

// Pointers that come from a table in memory: told to be global memory's, or the compiler's generic accesses go by the LDS
// path as well.
template <class V>
using Global = __attribute__((address_space(1))) V;

// Every byte is touched once a step; accesses that do not stay in the caches are the faster ones only if reads and writes
// both are such (1.32 ms; 1.52 with streaming reads alone, 1.48 with such writes alone).
template <class V>
__device__ __forceinline__ V load_once(const V* p) { return __builtin_nontemporal_load((const Global<V>*)p); }
template <class V>
__device__ __forceinline__ void store_once(V v, V* p) { __builtin_nontemporal_store(v, (Global<V>*)p); }
template <class V>
__device__ __forceinline__ V load(const V* p) { return *(const Global<V>*)p; }
template <class V, class U>
__device__ __forceinline__ void store(U v, V* p) { *(Global<V>*)p = (V)v; }

// A tensor as the kernels see it.
struct Tensor {
    float* x;
    const void* g;
    void *m, *v;
    float *m_scale, *v_scale;
    uint16_t* xb;
    float *m_values, *v_values;
    int64_t ld_x, ld_g, ld_s, ld_scale, ld_b, ld_values;
    int64_t n;
    double wd, lr_mult;
    int32_t wide, wide_values;                       // every row of every array starts on a boundary of four elements (32-bit moments: two)
};

// What one workgroup does: elements [start, min(start + kChunk, n)) of one row.
struct Work {
    int32_t tensor, row;
    int64_t start;
};

struct Step {
    double lr, lr_corrected;                         // lr_corrected = lr / (1 - b1^t)
    float b1, b2, one_b1, one_b2, inv_c2, eps, gscale;
    float um, uv;                                    // where between two codes the upper one begins
};

struct Coef {
    float decay, rate;
};

__device__ __forceinline__ Coef coefficients(const Tensor& t, const Step& p)
{
#pragma clang fp contract(off)
    Coef c;
    c.decay = (float)(1.0 - p.lr * t.lr_mult * t.wd);
    c.rate = (float)(p.lr_corrected * t.lr_mult);
    return c;
}

// One element; m and v are its moments before and after, r the root of the second after.
__device__ __forceinline__ void update(float& x, float g, float& m, float& v, float& r, const Coef& c, const Step& p)
{
#pragma clang fp contract(off)
    const float gs = g * p.gscale;
    m = p.b1 * m + p.one_b1 * gs;
    v = p.b2 * v + p.one_b2 * (gs * gs);
    r = sqrtf(v);
    const float den = r * p.inv_c2 + p.eps;
    x = x * c.decay - (m / den) * c.rate;
}

template <class G>
__device__ __forceinline__ float grad1(const void* g, int64_t i)
{
    if constexpr (sizeof(G) == 4) return load(static_cast<const float*>(g) + i);
    else return bf16_to_f32(load(static_cast<const uint16_t*>(g) + i));
}

template <class G>
__device__ __forceinline__ v2f grad2(const void* g, int64_t i)
{
    if constexpr (sizeof(G) == 4) return load_once(reinterpret_cast<const v2f*>(static_cast<const float*>(g) + i));
    else {
        const uint32_t b = load_once(reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(g) + i));
        return v2f{__uint_as_float(b << 16), __uint_as_float(b & 0xFFFF0000u)};
    }
}

template <class G>
__device__ __forceinline__ v4f grad4(const void* g, int64_t i)
{
    if constexpr (sizeof(G) == 4) return load_once(reinterpret_cast<const v4f*>(static_cast<const float*>(g) + i));
    else {
        const v2u b = load_once(reinterpret_cast<const v2u*>(static_cast<const uint16_t*>(g) + i));
        return v4f{__uint_as_float(b.x << 16), __uint_as_float(b.x & 0xFFFF0000u), __uint_as_float(b.y << 16), __uint_as_float(b.y & 0xFFFF0000u)};
    }
}

// ---- 32-bit moments ----
// Bound by memory: 268 M parameters with a bf16 copy in 1.29 to 1.37 ms, by where their arrays lie, 5.9 to 6.25 TB/s of 8.1 GB; half
// of them off alignment 1.50.  5 us a call for a few hundred.
template <class G>
__global__ __launch_bounds__(kThreads32) void adamw32_kernel(const Tensor* __restrict__ tensors, const Work* __restrict__ works, Step p)
{
    const Work w = works[blockIdx.x];
    const Tensor t = tensors[w.tensor];
    const Coef c = coefficients(t, p);
    const int64_t end = w.start + kChunk < t.n ? w.start + kChunk : t.n;
    float* x = t.x + w.row * t.ld_x;
    float* m = static_cast<float*>(t.m) + w.row * t.ld_s;
    float* v = static_cast<float*>(t.v) + w.row * t.ld_s;
    const void* g = static_cast<const char*>(t.g) + w.row * t.ld_g * (int64_t)sizeof(G);
    uint16_t* xb = t.xb ? t.xb + w.row * t.ld_b : nullptr;
    float r;
    int64_t i = w.start + 2 * threadIdx.x;
    if (t.wide && i + 2 <= end) {
        v2f xv = load_once(reinterpret_cast<const v2f*>(x + i));
        const v2f gv = grad2<G>(g, i);
        v2f mv = load_once(reinterpret_cast<const v2f*>(m + i));
        v2f vv = load_once(reinterpret_cast<const v2f*>(v + i));
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float xe = xv[e], me = mv[e], ve = vv[e];
            update(xe, gv[e], me, ve, r, c, p);
            xv[e] = xe; mv[e] = me; vv[e] = ve;
        }
        store_once(xv, reinterpret_cast<v2f*>(x + i));
        store_once(mv, reinterpret_cast<v2f*>(m + i));
        store_once(vv, reinterpret_cast<v2f*>(v + i));
        if (xb) store_once(f32x2_to_bf16x2(xv.x, xv.y), reinterpret_cast<uint32_t*>(xb + i));
        return;
    }
    // not aligned: one element a lane at a time; aligned: what is left at the row's end is one element, of the lane it fell to
    const int64_t step = t.wide ? 2 : kThreads32;
    for (i = t.wide ? i : w.start + threadIdx.x; i < end; i += step) {
        float xe = load(x + i), me = load(m + i), ve = load(v + i);
        update(xe, grad1<G>(g, i), me, ve, r, c, p);
        store(xe, x + i);
        store(me, m + i);
        store(ve, v + i);
        if (xb) store(f32_to_bf16_rne(xe), xb + i);
    }
}

// ---- 8-bit moments ----
// Largest values over the wavefront, of two lists at once (the one's lane shifts fill the other's wait states), in scalar
// registers.  Magnitudes are compared as bit patterns: NaN lies above infinity there.
template <int CTRL>
__device__ __forceinline__ uint32_t max_lanes(uint32_t a)
{
    const uint32_t b = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, CTRL, 0xF, 0xF, false);
    return a > b ? a : b;
}
__device__ __forceinline__ void wave_max2(uint32_t& a, uint32_t& b)
{
    a = max_lanes<0x111>(a); b = max_lanes<0x111>(b);      // the lane one to the left, in its row of 16
    a = max_lanes<0x112>(a); b = max_lanes<0x112>(b);
    a = max_lanes<0x114>(a); b = max_lanes<0x114>(b);
    a = max_lanes<0x118>(a); b = max_lanes<0x118>(b);      // the row's last lane has the row's largest
    a = max_lanes<0x142>(a); b = max_lanes<0x142>(b);      // to the next row, to the upper half
    a = max_lanes<0x143>(a); b = max_lanes<0x143>(b);
    a = (uint32_t)__builtin_amdgcn_readlane((int)a, kWave - 1);
    b = (uint32_t)__builtin_amdgcn_readlane((int)b, kWave - 1);
}

constexpr uint32_t kInf = 0x7F800000u;
__device__ __forceinline__ uint32_t magnitude(float a) { return __float_as_uint(a) & 0x7FFFFFFFu; }

// The largest finite |m| and r of a block.
__device__ __forceinline__ void largest(const float (&m)[4], const float (&r)[4], float& bm, float& bv)
{
    uint32_t a = 0, b = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        a = max(a, magnitude(m[e]));
        b = max(b, magnitude(r[e]));
    }
    wave_max2(a, b);
    if (a >= kInf || b >= kInf) {                          // something is not: once more without it
        a = b = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            a = max(a, magnitude(m[e]) < kInf ? magnitude(m[e]) : 0);
            b = max(b, magnitude(r[e]) < kInf ? magnitude(r[e]) : 0);
        }
        wave_max2(a, b);
    }
    bm = __uint_as_float(a);
    bv = __uint_as_float(b);
}

struct Scales {
    float m, v, inv_m, inv_v;
};

// Scales of a block whose largest finite moments are bm and bv, and their reciprocals; blocks of next to nothing are held
// as zero.  One quotient for both: half of the wavefront divides for m, half for v.
__device__ __forceinline__ Scales scales_of(float bm, float bv)
{
    const bool low = (threadIdx.x & (kWave - 1)) < kWave / 2;
    float s = (low ? bm : bv) * (low ? 1.0f / kTopM : 1.0f / kTopV);
    if (!(s > 0x1p-100f)) s = 0.0f;
    const float inv = s > 0.0f ? 1.0f / s : 0.0f;
    Scales q;
    q.m = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(s), 0));
    q.v = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(s), kWave - 1));
    q.inv_m = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(inv), 0));
    q.inv_v = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(inv), kWave - 1));
    return q;
}

// Codes.  c = floor(root of y) comes from an approximate root and may be one off where y is next to a square; the
// threshold u lies far enough from 0 and 1 that the code taken is then the same: just below (c+1)^2 both choices end at c+1,
// just above c^2 both at c.  All integers below are exact in fp32.  What is not finite gets the largest code: the gradient was
// not (nor is its parameter then), or its square overflows.
__device__ __forceinline__ int code_m(float m, float inv, float u)
{
#pragma clang fp contract(off)
    const float y = fminf(fabsf(m) * inv, kTopM);
    const float c = floorf(__builtin_amdgcn_sqrtf(y));
    const int q = (int)c + (__builtin_fmaf(-c, c, y) > u * __builtin_fmaf(2.0f, c, 1.0f) ? 1 : 0);
    return m < 0.0f ? -q : q;
}

__device__ __forceinline__ int code_v(float r, float inv, float u, int least)
{
#pragma clang fp contract(off)
    const float y = fminf(r * inv, kTopV);
    const float c = floorf(__builtin_amdgcn_sqrtf(y));
    const float c2 = c * c, odd = __builtin_fmaf(2.0f, c, 1.0f);                 // (c+1)^2 - c^2
    const float both = __builtin_fmaf(c, odd, c + 1.0f);                         // (c+1)^2 + c^2
    const int q = (int)c + ((y - c2) * (y + c2) > u * (odd * both) ? 1 : 0);
    return r > 0.0f && q < least ? least : q;                                    // a second moment that is not zero is not held as zero
}

__device__ __forceinline__ float value_m(int q, float s)
{
    const float c = (float)q;
    return c * fabsf(c) * s;
}
__device__ __forceinline__ float value_r(int q, float s)
{
    const float c = (float)q;
    return c * c * s;
}

// A wavefront takes a block: its lanes hold four elements each, adjacent ones where the arrays allow wide accesses.  103 vector
// instructions an element: 268 M elements 787 us, 5.5 TB/s of 16 bytes each, arithmetic and memory about even; half of them off
// alignment 860.
template <class G>
__global__ __launch_bounds__(kThreads) void adamw8_kernel(const Tensor* __restrict__ tensors, const Work* __restrict__ works, Step p)
{
    const Work w = works[blockIdx.x];
    const Tensor t = tensors[w.tensor];
    const Coef c = coefficients(t, p);
    const int lane = threadIdx.x & (kWave - 1);
    const int64_t b = w.start / kBlock + __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int64_t first = b * kBlock;
    if (first >= t.n) return;
    float* x = t.x + w.row * t.ld_x;
    int8_t* m = static_cast<int8_t*>(t.m) + w.row * t.ld_s;
    uint8_t* v = static_cast<uint8_t*>(t.v) + w.row * t.ld_s;
    float* ms = t.m_scale + w.row * t.ld_scale + b;
    float* vs = t.v_scale + w.row * t.ld_scale + b;
    const void* g = static_cast<const char*>(t.g) + w.row * t.ld_g * (int64_t)sizeof(G);
    uint16_t* xb = t.xb ? t.xb + w.row * t.ld_b : nullptr;
    const float sm = load(ms), sv = load(vs);
    const bool wide = t.wide && first + kBlock <= t.n;
    const int64_t k = first + 4 * lane;
    float xe[4], me[4], re[4];
    if (wide) {
        const v4f xv = load_once(reinterpret_cast<const v4f*>(x + k));
        const v4f gv = grad4<G>(g, k);
        const uint32_t mq = load_once(reinterpret_cast<const uint32_t*>(m + k)), vq = load_once(reinterpret_cast<const uint32_t*>(v + k));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            xe[e] = xv[e];
            me[e] = value_m((int)(int8_t)(mq >> (8 * e)), sm);
            const float rr = value_r((int)(vq >> (8 * e) & 255u), sv);
            float ve = rr * rr;
            update(xe[e], gv[e], me[e], ve, re[e], c, p);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t i = first + lane + e * kWave;
            xe[e] = me[e] = re[e] = 0.0f;
            if (i < t.n) {
                xe[e] = load(x + i);
                me[e] = value_m(load(m + i), sm);
                const float rr = value_r(load(v + i), sv);
                float ve = rr * rr;
                update(xe[e], grad1<G>(g, i), me[e], ve, re[e], c, p);
            }
        }
    }
    float bm, bv;
    largest(me, re, bm, bv);
    const Scales s = scales_of(bm, bv);
    const int least = s.v > 0.0f ? 1 : 0;
    int qm[4], qv[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        qm[e] = code_m(me[e], s.inv_m, p.um);
        qv[e] = code_v(re[e], s.inv_v, p.uv, least);
    }
    if (wide) {
        uint32_t mq = 0, vq = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            mq |= (uint32_t)(qm[e] & 255) << (8 * e);
            vq |= (uint32_t)qv[e] << (8 * e);
        }
        const v4f xv = {xe[0], xe[1], xe[2], xe[3]};
        store_once(xv, reinterpret_cast<v4f*>(x + k));
        store_once(mq, reinterpret_cast<uint32_t*>(m + k));
        store_once(vq, reinterpret_cast<uint32_t*>(v + k));
        if (xb) store_once(v2u{f32x2_to_bf16x2(xv.x, xv.y), f32x2_to_bf16x2(xv.z, xv.w)}, reinterpret_cast<v2u*>(xb + k));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t i = first + lane + e * kWave;
            if (i < t.n) {
                store(xe[e], x + i);
                store(qm[e], m + i);
                store(qv[e], v + i);
                if (xb) store(f32_to_bf16_rne(xe[e]), xb + i);
            }
        }
    }
    if (lane == 0) {
        store(s.m, ms);
        store(s.v, vs);
    }
}

// The values that the codes stand for: 268 M elements 400 us, half of them off alignment 825.
__global__ __launch_bounds__(kThreads) void adamw8_values_kernel(const Tensor* __restrict__ tensors, const Work* __restrict__ works)
{
#pragma clang fp contract(off)
    const Work w = works[blockIdx.x];
    const Tensor t = tensors[w.tensor];
    if (!t.m_values) return;
    const int64_t end = w.start + kChunk < t.n ? w.start + kChunk : t.n;
    const int8_t* m = static_cast<const int8_t*>(t.m) + w.row * t.ld_s;
    const uint8_t* v = static_cast<const uint8_t*>(t.v) + w.row * t.ld_s;
    const float* ms = t.m_scale + w.row * t.ld_scale;
    const float* vs = t.v_scale + w.row * t.ld_scale;
    float* om = t.m_values + w.row * t.ld_values;
    float* ov = t.v_values + w.row * t.ld_values;
    const int64_t k = w.start + 4 * threadIdx.x;
    if (t.wide_values && k + 4 <= end) {
        const uint32_t mq = load_once(reinterpret_cast<const uint32_t*>(m + k)), vq = load_once(reinterpret_cast<const uint32_t*>(v + k));
        const float sm = load(ms + k / kBlock), sv = load(vs + k / kBlock);
        v4f a, b;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            a[e] = value_m((int)(int8_t)(mq >> (8 * e)), sm);
            const float r = value_r((int)(vq >> (8 * e) & 255u), sv);
            b[e] = r * r;
        }
        store_once(a, reinterpret_cast<v4f*>(om + k));
        store_once(b, reinterpret_cast<v4f*>(ov + k));
        return;
    }
    const int64_t step = t.wide_values ? 1 : kThreads;
    for (int64_t i = t.wide_values ? k : w.start + threadIdx.x; i < end; i += step) {
        store(value_m(load(m + i), load(ms + i / kBlock)), om + i);
        const float r = value_r(load(v + i), load(vs + i / kBlock));
        store(r * r, ov + i);
    }
}

constexpr size_t kAlign = 256;
size_t align_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }

bool on(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Checks the list and counts workgroups.
lsgd_status check_tensors(const lsgd_adamw_tensor* t, int32_t count, int32_t bits, int32_t g_is_bf16, int64_t* works)
{
    if (count < 0) return set_error(LSGD_ERR_SHAPE, "adamw: n_tensors=%d is negative", (int)count);
    if (count > 0 && !t) return set_error(LSGD_ERR_INVALID_ARG, "adamw: tensors is NULL");
    if (bits != 32 && bits != 8) return set_error(LSGD_ERR_INVALID_ARG, "adamw: state_bits=%d is neither 32 nor 8", (int)bits);
    if (g_is_bf16 != 0 && g_is_bf16 != 1) return set_error(LSGD_ERR_INVALID_ARG, "adamw: g_is_bf16 must be 0 or 1");
    int64_t total = 0;
    for (int k = 0; k < count; ++k) {
        const lsgd_adamw_tensor& a = t[k];
        if (a.rows < 0 || a.n < 0) return set_error(LSGD_ERR_SHAPE, "adamw: tensor %d: negative rows or n", k);
        if (!std::isfinite(a.weight_decay) || !std::isfinite(a.lr_mult))
            return set_error(LSGD_ERR_INVALID_ARG, "adamw: tensor %d: weight_decay and lr_mult must be finite", k);
        if (a.rows == 0 || a.n == 0) continue;
        if (a.rows > 0x7fffffff) return set_error(LSGD_ERR_SHAPE, "adamw: tensor %d: rows=%lld", k, (long long)a.rows);
        if (!a.x || !a.g || !a.m || !a.v) return set_error(LSGD_ERR_INVALID_ARG, "adamw: tensor %d: x, g, m and v are required", k);
        if (!on(a.x, 4) || !on(a.g, g_is_bf16 ? 2 : 4) || !on(a.x_bf16, 2) || (bits == 32 && (!on(a.m, 4) || !on(a.v, 4))) ||
            !on(a.m_scale, 4) || !on(a.v_scale, 4) || !on(a.m_values, 4) || !on(a.v_values, 4))
            return set_error(LSGD_ERR_INVALID_ARG, "adamw: tensor %d: a pointer is not aligned to its element", k);
        if (a.rows > 1 && (a.ld_x < a.n || a.ld_g < a.n || a.ld_state < a.n || (a.x_bf16 && a.ld_bf16 < a.n)))
            return set_error(LSGD_ERR_SHAPE, "adamw: tensor %d: a row stride is smaller than n=%lld", k, (long long)a.n);
        if (bits == 8) {
            if (!a.m_scale || !a.v_scale) return set_error(LSGD_ERR_INVALID_ARG, "adamw: tensor %d: 8-bit moments need m_scale and v_scale", k);
            if (a.rows > 1 && a.ld_scale < (a.n + kBlock - 1) / kBlock)
                return set_error(LSGD_ERR_SHAPE, "adamw: tensor %d: ld_scale is smaller than the %lld blocks of a row", k, (long long)((a.n + kBlock - 1) / kBlock));
            if (!a.m_values != !a.v_values) return set_error(LSGD_ERR_INVALID_ARG, "adamw: tensor %d: give both m_values and v_values or neither", k);
            if (a.m_values && a.rows > 1 && a.ld_values < a.n) return set_error(LSGD_ERR_SHAPE, "adamw: tensor %d: ld_values is smaller than n", k);
        }
        const int64_t per = (a.n - 1) / kChunk + 1;
        if (per > (int64_t)0x7fffffff / a.rows) return set_error(LSGD_ERR_SHAPE, "adamw: tensor %d is too large for one call", k);
        total += per * a.rows;
        if (total > 0x7fffffff) return set_error(LSGD_ERR_SHAPE, "adamw: the tensors are too large for one call");
    }
    *works = total;
    return LSGD_OK;
}

size_t table_bytes(int32_t count, int64_t works)
{
    return align_up(sizeof(Tensor) * (size_t)count) + align_up(sizeof(Work) * (size_t)works);
}

} // namespace

struct lsgd_adamw {
    const Tensor* tensors;
    const Work* works;
    int64_t n_works;
    int32_t bits, g_is_bf16;
    bool values;             // some tensor has room for its moments' values
    hipStream_t stream;
};

namespace {

// All of a handle's workgroups: one launch, but that a launch has fewer than 2^32 threads (8.6 G parameters with 32-bit moments).
template <class... A, class... B>
void launch_all(const lsgd_adamw& h, int threads, void (*kernel)(const Tensor*, const Work*, A...), B... args)
{
    const int64_t most = 0xFFFFFFFFll / threads;
    for (int64_t first = 0; first < h.n_works; first += most)
        hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(most, h.n_works - first)), dim3((unsigned)threads), 0, h.stream, h.tensors, h.works + first, args...);
}

} // namespace

extern "C" {

size_t lsgd_adamw_workspace_bytes(const lsgd_adamw_tensor* tensors, int32_t n_tensors, int32_t state_bits, int32_t g_is_bf16)
{
    int64_t works = 0;
    if (check_tensors(tensors, n_tensors, state_bits, g_is_bf16, &works) != LSGD_OK) return 0;
    const size_t b = table_bytes(n_tensors, works);
    return b ? b : kAlign;
}

lsgd_status lsgd_adamw_create(const lsgd_adamw_tensor* tensors, int32_t n_tensors, int32_t state_bits, int32_t g_is_bf16, void* workspace,
                              size_t workspace_bytes, void* hip_stream, lsgd_adamw** out)
{
    if (!out) return set_error(LSGD_ERR_INVALID_ARG, "adamw: out is NULL");
    *out = nullptr;
    int64_t n_works = 0;
    lsgd_status st = check_tensors(tensors, n_tensors, state_bits, g_is_bf16, &n_works);
    if (st != LSGD_OK) return st;
    if (!workspace) return set_error(LSGD_ERR_INVALID_ARG, "adamw: workspace is NULL");
    if (!on(workspace, kAlign)) return set_error(LSGD_ERR_INVALID_ARG, "adamw: workspace must be 256-byte aligned");
    if (workspace_bytes < table_bytes(n_tensors, n_works))
        return set_error(LSGD_ERR_NOMEM, "adamw: workspace of %zu bytes < %zu needed", workspace_bytes, table_bytes(n_tensors, n_works));
    hipError_t e = hipSuccess;
    lsgd_adamw* h = nullptr;
    try {
        std::vector<Tensor> ts((size_t)n_tensors);
        std::vector<Work> ws;
        ws.reserve((size_t)n_works);
        bool values = false;
        for (int k = 0; k < n_tensors; ++k) {
            const lsgd_adamw_tensor& a = tensors[k];
            Tensor& t = ts[(size_t)k];
            std::memset(&t, 0, sizeof(t));
            if (a.rows == 0 || a.n == 0) continue;
            t.x = a.x; t.g = a.g; t.m = a.m; t.v = a.v;
            t.xb = a.x_bf16;
            // one row: its stride is never multiplied by anything, so it does not matter to the alignment either
            auto ld = [&](int64_t v) { return a.rows > 1 ? v : (int64_t)0; };
            t.ld_x = ld(a.ld_x); t.ld_g = ld(a.ld_g); t.ld_s = ld(a.ld_state); t.ld_b = a.x_bf16 ? ld(a.ld_bf16) : 0;
            const uintptr_t lanes = state_bits == 32 ? 2 : 4, es = state_bits == 32 ? 8 : 4;
            t.wide = on(t.x, 4 * lanes) && on(t.g, (g_is_bf16 ? 2 : 4) * lanes) && on(t.m, es) && on(t.v, es) && on(t.xb, 2 * lanes) &&
                     (t.ld_x | t.ld_g | t.ld_s | t.ld_b) % (int64_t)lanes == 0;
            if (state_bits == 8) {
                t.m_scale = a.m_scale; t.v_scale = a.v_scale; t.ld_scale = ld(a.ld_scale);
                t.m_values = a.m_values; t.v_values = a.v_values; t.ld_values = ld(a.ld_values);
                t.wide_values = on(t.m, 4) && on(t.v, 4) && on(t.m_values, 16) && on(t.v_values, 16) && (t.ld_s | t.ld_values) % 4 == 0;
                values |= a.m_values != nullptr;
            }
            t.n = a.n;
            t.wd = a.weight_decay;
            t.lr_mult = a.lr_mult;
            for (int64_t row = 0; row < a.rows; ++row)
                for (int64_t s = 0; s < a.n; s += kChunk) ws.push_back(Work{k, (int32_t)row, s});
        }
        h = new (std::nothrow) lsgd_adamw();
        if (!h) return set_error(LSGD_ERR_NOMEM, "adamw: host allocation failed");
        char* base = static_cast<char*>(workspace);
        h->tensors = reinterpret_cast<const Tensor*>(base);
        h->works = reinterpret_cast<const Work*>(base + align_up(sizeof(Tensor) * (size_t)n_tensors));
        h->n_works = n_works;
        h->bits = state_bits;
        h->g_is_bf16 = g_is_bf16;
        h->values = values;
        h->stream = static_cast<hipStream_t>(hip_stream);
        if (!ws.empty()) {
            e = hipMemcpyAsync(base, ts.data(), sizeof(Tensor) * ts.size(), hipMemcpyHostToDevice, h->stream);
            if (e == hipSuccess)
                e = hipMemcpyAsync(const_cast<Work*>(h->works), ws.data(), sizeof(Work) * ws.size(), hipMemcpyHostToDevice, h->stream);
            const hipError_t waited = hipStreamSynchronize(h->stream);      // the host vectors were the copy's source
            if (e == hipSuccess) e = waited;
        }
    } catch (const std::bad_alloc&) {
        delete h;
        return set_error(LSGD_ERR_NOMEM, "adamw: host allocation failed");
    }
    if (e != hipSuccess) {
        delete h;
        return set_error(LSGD_ERR_HIP, "adamw: create: %s", hipGetErrorString(e));
    }
    *out = h;
    return LSGD_OK;
}

lsgd_status lsgd_adamw_destroy(lsgd_adamw* opt)
{
    delete opt;
    return LSGD_OK;
}

lsgd_status lsgd_adamw_set_stream(lsgd_adamw* opt, void* hip_stream)
{
    if (!opt) return set_error(LSGD_ERR_INVALID_ARG, "adamw: handle is NULL");
    opt->stream = static_cast<hipStream_t>(hip_stream);
    return LSGD_OK;
}

lsgd_status lsgd_adamw_step(lsgd_adamw* opt, double lr, double beta1, double beta2, double eps, int64_t step, double grad_scale)
{
    if (!opt) return set_error(LSGD_ERR_INVALID_ARG, "adamw: handle is NULL");
    if (!std::isfinite(lr) || !std::isfinite(grad_scale)) return set_error(LSGD_ERR_INVALID_ARG, "adamw: lr and grad_scale must be finite");
    if (!(beta1 >= 0.0 && beta1 < 1.0 && beta2 >= 0.0 && beta2 < 1.0)) return set_error(LSGD_ERR_INVALID_ARG, "adamw: beta1 and beta2 must lie in [0, 1)");
    if (!std::isfinite(eps) || eps < 0.0) return set_error(LSGD_ERR_INVALID_ARG, "adamw: eps must be finite and >= 0");
    if (step < 1) return set_error(LSGD_ERR_INVALID_ARG, "adamw: step=%lld counts from 1", (long long)step);
    if (opt->n_works == 0) return LSGD_OK;
    Step p;
    p.lr = lr;
    p.lr_corrected = lr / (1.0 - std::pow(beta1, (double)step));
    p.b1 = (float)beta1; p.b2 = (float)beta2;
    p.one_b1 = (float)(1.0 - beta1); p.one_b2 = (float)(1.0 - beta2);
    p.inv_c2 = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step)));
    p.eps = (float)eps;
    p.gscale = (float)grad_scale;
    constexpr double kGolden = 0.6180339887498949;
    // not nearer to 0 and 1 than 2^-12: see the codes
    auto inside = [](double u) { return (float)std::min(std::max(u, 0x1p-12), 1.0 - 0x1p-12); };
    p.uv = inside(std::fmod((double)step * kGolden, 1.0));
    p.um = inside(std::fmod((double)step * kGolden + 0.5, 1.0));
    auto go = [&](auto kernel, int threads) { launch_all(*opt, threads, kernel, p); };
    if (opt->bits == 32) opt->g_is_bf16 ? go(adamw32_kernel<uint16_t>, kThreads32) : go(adamw32_kernel<float>, kThreads32);
    else opt->g_is_bf16 ? go(adamw8_kernel<uint16_t>, kThreads) : go(adamw8_kernel<float>, kThreads);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return set_error(LSGD_ERR_HIP, "adamw: %s", hipGetErrorString(e));
    return LSGD_OK;
}

lsgd_status lsgd_adamw_moments(lsgd_adamw* opt)
{
    if (!opt) return set_error(LSGD_ERR_INVALID_ARG, "adamw: handle is NULL");
    if (opt->bits != 8) return set_error(LSGD_ERR_STATE, "adamw: 32-bit moments are their own values");
    if (!opt->values) return set_error(LSGD_ERR_STATE, "adamw: no tensor was given m_values and v_values");
    launch_all(*opt, kThreads, adamw8_values_kernel);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return set_error(LSGD_ERR_HIP, "adamw: moments: %s", hipGetErrorString(e));
    return LSGD_OK;
}

} // extern "C"
