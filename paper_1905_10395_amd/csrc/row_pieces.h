// Pieces of a row of fp32 or bf16 values that a lane holds in registers as fp32: E adjacent elements (8 of either type, or 4
// of fp32), or what the row's end leaves of them.  Rows may begin anywhere and be of any width: the chip's wide accesses need
// no alignment.  ONCE: past the caches, for data touched once; only where every piece is whole and 16-byte aligned, or lines
// would go to memory in parts.
#pragma once

#include <type_traits>

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

__device__ __forceinline__ void put1(float* p, float v) { *p = v; }
__device__ __forceinline__ void put1(uint16_t* p, float v) { *p = f32_to_bf16_rne(v); }
__device__ __forceinline__ void put2(float* p, float a, float b) { *reinterpret_cast<v2f_any*>(p) = v2f{a, b}; }
__device__ __forceinline__ void put2(uint16_t* p, float a, float b) { *reinterpret_cast<u32_any*>(p) = f32x2_to_bf16x2(a, b); }
__device__ __forceinline__ void put4(float* p, const float* v) { *reinterpret_cast<v4f_any*>(p) = v4f{v[0], v[1], v[2], v[3]}; }
__device__ __forceinline__ void put4(uint16_t* p, const float* v)
{
    *reinterpret_cast<v2u_any*>(p) = v2u{f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3])};
}

// Column c's address, in 32 bits beyond the row's, which may stay in scalar registers.
template <class T>
__device__ __forceinline__ T* column(T* row, int c)
{
    using Byte = std::conditional_t<std::is_const_v<T>, const char, char>;
    return reinterpret_cast<T*>(reinterpret_cast<Byte*>(row) + (uint32_t)c * (uint32_t)sizeof(T));
}

// A piece as memory has it.  Loads go here and unpack() stands after the last of them: nothing uses a value in between, so all
// are in flight at a time, though each may be in branches of its own.
template <class T, int E>
struct Raw {
    static_assert(E == 8 || (E == 4 && sizeof(T) == 4), "eight elements, or four of fp32");
    v4u q[E * sizeof(T) / 16];
};
template <class T, int E>
__device__ __forceinline__ void clear(Raw<T, E>& v)
{
#pragma unroll
    for (v4u& q : v.q) q = v4u{0, 0, 0, 0};
}
template <int E>
__device__ __forceinline__ void unpack(const Raw<float, E>& v, float (&f)[E])
{
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = __uint_as_float(v.q[e / 4][e % 4]);
}
__device__ __forceinline__ void unpack(const Raw<uint16_t, 8>& v, float (&f)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(e & 1 ? v.q[0][e / 2] & 0xFFFF0000u : v.q[0][e / 2] << 16);
}

// Whole pieces.
template <bool ONCE, class T, int E>
__device__ __forceinline__ void load_whole(const T* p, Raw<T, E>& v)
{
    constexpr int per = 16 / (int)sizeof(T);
#pragma unroll
    for (int e = 0; e < E; e += per) {
        if constexpr (ONCE) v.q[e / per] = __builtin_nontemporal_load(reinterpret_cast<const v4u*>(p + e));
        else v.q[e / per] = *reinterpret_cast<const v4u_any*>(p + e);
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

// The piece of columns c and on.  A row's last one, if it is not whole, is held from further left, so that it ends with the row
// and is whole all the same: its first elements are then another lane's, are not written by this one, and nothing may depend
// on them (that lane may have written its own already).  By accesses of four, two and one in branches of their own the wavefront
// that holds the end waited for each of them: 6 x 4064 x 4495 bf16 normed in 361 us, 270 so.  A row shorter than a piece is
// held from its beginning; SHORT: there may be such.
template <int E>
__device__ __forceinline__ int piece_start(int c, int D) { return c + E <= D || D < E ? c : D - E; }

template <bool SHORT = true, class T, int E>
__device__ __forceinline__ void load_piece(const T* row, int c, int D, Raw<T, E>& v)
{
    if (!SHORT || D >= E) load_whole<false>(column(row, piece_start<E>(c, D)), v);
    else if (c < D) {
        clear(v);
#pragma unroll
        for (int e = 0; e < E - 1; ++e)
            if (e < D) {
                if constexpr (sizeof(T) == 4) v.q[e / 4][e % 4] = __float_as_uint(row[e]);
                else v.q[0][e / 2] |= (uint32_t)row[e] << (16 * (e & 1));
            }
    }
}
// The same as fp32.
template <bool SHORT = true, class T, int E>
__device__ __forceinline__ void load_piece(const T* row, int c, int D, float (&f)[E])
{
    Raw<T, E> v;
    clear(v);
    load_piece<SHORT>(row, c, D, v);
    unpack(v, f);
}
// Zeros in place of elements that are another lane's.
template <int E>
__device__ __forceinline__ void keep_own(int c, int D, float (&f)[E])
{
    const int start = piece_start<E>(c, D);
#pragma unroll
    for (int e = 0; e < E; ++e)
        f[e] = start + e < c ? 0.0f : f[e];
}
// Writes the lane's own elements of its piece; how many those of the last piece are is the same for all rows and lanes.
template <bool SHORT = true, class T, int E>
__device__ __forceinline__ void store_piece(T* row, int c, int D, const float (&f)[E])
{
    static_assert(E == 4 || E == 8, "four or eight elements");
    if (c + E <= D) store_whole<false>(column(row, c), f);
    else if (c < D && (!SHORT || D >= E)) {
        T* p = row + D - E;
        const int r = D % E;
        if constexpr (E == 8) {
            if (r & 4) {
                put4(p + 4, f + 4);
                if (r & 2) put2(p + 2, f[2], f[3]);
                if ((r & 3) == 3) put1(p + 1, f[1]);
                else if (r & 1) put1(p + 3, f[3]);
                return;
            }
        }
        if (r & 2) put2(p + E - 2, f[E - 2], f[E - 1]);
        if ((r & 3) == 3) put1(p + E - 3, f[E - 3]);
        else if (r & 1) put1(p + E - 1, f[E - 1]);
    } else if (SHORT && c < D) {
#pragma unroll
        for (int e = 0; e < E - 1; ++e)
            if (e < D) put1(row + e, f[e]);
    }
}

} // namespace lsgd
