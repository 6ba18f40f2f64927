// Pieces of a row of fp32 or bf16 values that a lane holds in registers as fp32: E adjacent elements (8 of either type, or 4
// of fp32), or what the row's end leaves of them.  Rows may begin anywhere and be of any width: the chip's wide accesses need
// no alignment.  ONCE: past the caches, for data touched once; only where every piece is whole and 16-byte aligned, or lines
// would go to memory in parts.
#pragma once

#include "common.h"

namespace lsgd {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef v4f v4f_any __attribute__((aligned(4)));
typedef v2f v2f_any __attribute__((aligned(4)));
typedef v4u v4u_any __attribute__((aligned(2)));
typedef v2u v2u_any __attribute__((aligned(2)));
typedef uint32_t u32_any __attribute__((aligned(2)));

__device__ __forceinline__ float get1(const float* p) { return *p; }
__device__ __forceinline__ float get1(const uint16_t* p) { return bf16_to_f32(*p); }
__device__ __forceinline__ void put1(float* p, float v) { *p = v; }
__device__ __forceinline__ void put1(uint16_t* p, float v) { *p = f32_to_bf16_rne(v); }

__device__ __forceinline__ void get2(const float* p, float& a, float& b)
{
    const v2f q = *reinterpret_cast<const v2f_any*>(p);
    a = q.x; b = q.y;
}
__device__ __forceinline__ void get2(const uint16_t* p, float& a, float& b)
{
    const uint32_t q = *reinterpret_cast<const u32_any*>(p);
    a = __uint_as_float(q << 16); b = __uint_as_float(q & 0xFFFF0000u);
}
__device__ __forceinline__ void put2(float* p, float a, float b) { *reinterpret_cast<v2f_any*>(p) = v2f{a, b}; }
__device__ __forceinline__ void put2(uint16_t* p, float a, float b) { *reinterpret_cast<u32_any*>(p) = f32x2_to_bf16x2(a, b); }

__device__ __forceinline__ void get4(const float* p, float* v)
{
    const v4f q = *reinterpret_cast<const v4f_any*>(p);
    v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
}
__device__ __forceinline__ void get4(const uint16_t* p, float* v)
{
    const v2u q = *reinterpret_cast<const v2u_any*>(p);
    v[0] = __uint_as_float(q.x << 16); v[1] = __uint_as_float(q.x & 0xFFFF0000u);
    v[2] = __uint_as_float(q.y << 16); v[3] = __uint_as_float(q.y & 0xFFFF0000u);
}
__device__ __forceinline__ void put4(float* p, const float* v) { *reinterpret_cast<v4f_any*>(p) = v4f{v[0], v[1], v[2], v[3]}; }
__device__ __forceinline__ void put4(uint16_t* p, const float* v)
{
    *reinterpret_cast<v2u_any*>(p) = v2u{f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3])};
}

// Whole pieces.
template <bool ONCE, int E>
__device__ __forceinline__ void load_whole(const float* p, float (&v)[E])
{
#pragma unroll
    for (int e = 0; e < E; e += 4) {
        v4f q;
        if constexpr (ONCE) q = __builtin_nontemporal_load(reinterpret_cast<const v4f*>(p + e));
        else q = *reinterpret_cast<const v4f_any*>(p + e);
        v[e] = q.x; v[e + 1] = q.y; v[e + 2] = q.z; v[e + 3] = q.w;
    }
}
template <bool ONCE>
__device__ __forceinline__ void load_whole(const uint16_t* p, float (&v)[8])
{
    v4u q;
    if constexpr (ONCE) q = __builtin_nontemporal_load(reinterpret_cast<const v4u*>(p));
    else q = *reinterpret_cast<const v4u_any*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[2 * e] = __uint_as_float(q[e] << 16);
        v[2 * e + 1] = __uint_as_float(q[e] & 0xFFFF0000u);
    }
}
template <bool ONCE, int E>
__device__ __forceinline__ void store_whole(float* p, const float (&v)[E])
{
#pragma unroll
    for (int e = 0; e < E; e += 4) {
        const v4f q = {v[e], v[e + 1], v[e + 2], v[e + 3]};
        if constexpr (ONCE) __builtin_nontemporal_store(q, reinterpret_cast<v4f*>(p + e));
        else *reinterpret_cast<v4f_any*>(p + e) = q;
    }
}
template <bool ONCE>
__device__ __forceinline__ void store_whole(uint16_t* p, const float (&v)[8])
{
    const v4u q = {f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]), f32x2_to_bf16x2(v[4], v[5]), f32x2_to_bf16x2(v[6], v[7])};
    if constexpr (ONCE) __builtin_nontemporal_store(q, reinterpret_cast<v4u*>(p));
    else *reinterpret_cast<v4u_any*>(p) = q;
}

// The row's elements [c, c + E) as far as it has them (D in all; those past its end are left as they are), by accesses of four,
// two and one; D % E is the same for all lanes, so these branches are the wavefront's.
template <class T, int E>
__device__ __forceinline__ void load_piece(const T* row, int c, int D, float (&v)[E])
{
    static_assert(E == 4 || E == 8, "four or eight elements");
    const T* p = row + c;
    if (c + E <= D) load_whole<false>(p, v);
    else if (c < D) {
        const int r = D % E;
        if constexpr (E == 8) {
            if (r & 4) {
                get4(p, v);
                if (r & 2) get2(p + 4, v[4], v[5]);
                if ((r & 3) == 3) v[6] = get1(p + 6);
                else if (r & 1) v[4] = get1(p + 4);
                return;
            }
        }
        if (r & 2) get2(p, v[0], v[1]);
        if ((r & 3) == 3) v[2] = get1(p + 2);
        else if (r & 1) v[0] = get1(p);
    }
}
template <class T, int E>
__device__ __forceinline__ void store_piece(T* row, int c, int D, const float (&v)[E])
{
    T* p = row + c;
    if (c + E <= D) store_whole<false>(p, v);
    else if (c < D) {
        const int r = D % E;
        if constexpr (E == 8) {
            if (r & 4) {
                put4(p, v);
                if (r & 2) put2(p + 4, v[4], v[5]);
                if ((r & 3) == 3) put1(p + 6, v[6]);
                else if (r & 1) put1(p + 4, v[4]);
                return;
            }
        }
        if (r & 2) put2(p, v[0], v[1]);
        if ((r & 3) == 3) put1(p + 2, v[2]);
        else if (r & 1) put1(p, v[0]);
    }
}

} // namespace lsgd
