// What the attention kernels share: fragments of the matrix instructions, tiles of rows in LDS, numbering of rows.
//
// Rows.  The query heads that share a key head see the same keys, so their queries are one list of rows: row r = t G + g is
// query t of the head g of the G = Hq / Hk heads of a key head.  A unit is an entry and a key head.
//
// Matrix instructions take 32 x 32 results: A gives rows, B columns, both 8 elements a lane of a contraction of 16 (lane % 32: the row
// or column; lane / 32 = h: contraction places 8 h .. 8 h + 7).  A lane holds of the result column lane % 32, rows
// 8 (i / 4) + 4 h + i % 4, i = 0 .. 15.  So a product's result, rows becoming the contraction, is the next product's B as it lies in the
// registers, if the other operand's contraction places are taken in the same order: 4 h .. 4 h + 3, then 8 + 4 h .. 8 + 4 h + 3 (of
// 16).  One operand of every product stays in registers that way, the other passes through LDS.
//
// Tiles.  R rows of a tile lie in LDS as slabs of WIDTH columns, [slab][row][WIDTH], in pieces of 16 bytes; loads straight to LDS write
// consecutive pieces, so rows cannot be padded: a row's pieces are stored in another order (exclusive or with bits of the row's
// number), such that the reads along rows and those along columns both spread over all banks.  Slabs of 32 columns, or of 64 bf16
// ones where the rows come from memory once: a load then takes whole lines (but the reads' addresses take more registers).
#pragma once

#include <type_traits>

#include "heads.h"
#include "row_pieces.h"

namespace lsgd {
namespace attention {

constexpr int kPart = 32;                   // columns of a part of a tile
constexpr int kMaxColumns = 128;            // of a head
constexpr int kNonTemporal = 2;             // cache policy of a load
constexpr float kLog2e = 1.44269504088896341f;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void* lds_ptr;
typedef const __attribute__((address_space(1))) void* global_ptr;

// Eight elements of an operand.  fp32: as the sum of three bf16 values, each of which takes the next eight bits of what is left (to
// 2^-24 of the element); of the nine products of two such sums the six largest are made, and what is left out is below 2^-24 of the
// whole.  Six bf16 instructions take 6 / 16 of the time of the fp32 ones of the same products; the parts are made on the way from LDS,
// by every wavefront that reads an element, in about as long as its products.  An infinite element, and one that rounds to an infinity
// of bf16, has NaN for its second part.
template <class T> struct Frag;
template <> struct Frag<uint16_t> { bf16x8 v; };
template <> struct Frag<float> { bf16x8 v[3]; };

__device__ __forceinline__ void multiply(f32x16& c, const Frag<uint16_t>& a, const Frag<uint16_t>& b)
{
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, c, 0, 0, 0);
}
__device__ __forceinline__ void multiply(f32x16& c, const Frag<float>& a, const Frag<float>& b)
{
#pragma unroll
    for (int k = 2; k >= 0; --k)                              // the smallest first
#pragma unroll
        for (int i = 0; i <= k; ++i) c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v[i], b.v[k - i], c, 0, 0, 0);
}
__device__ __forceinline__ void split(const float (&x)[8], Frag<float>& f)
{
    float r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = x[e];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        v4u q;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            q[e] = f32x2_to_bf16x2(r[2 * e], r[2 * e + 1]);
            if (k < 2) {
                r[2 * e] -= __uint_as_float(q[e] << 16);
                r[2 * e + 1] -= __uint_as_float(q[e] & 0xFFFF0000u);
            }
        }
        f.v[k] = __builtin_bit_cast(bf16x8, q);
    }
}

// Half of a result's column as an operand: registers 8 k .. 8 k + 7.
__device__ __forceinline__ void from_result(const f32x16& r, int k, Frag<uint16_t>& f)
{
    v4u q;
#pragma unroll
    for (int e = 0; e < 4; ++e) q[e] = f32x2_to_bf16x2(r[8 * k + 2 * e], r[8 * k + 2 * e + 1]);
    f.v = __builtin_bit_cast(bf16x8, q);
}
__device__ __forceinline__ void from_result(const f32x16& r, int k, Frag<float>& f)
{
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = r[8 * k + e];
    split(x, f);
}

// Rows of any alignment and length, by 16 bytes from column c on, zeros past the row's end.  A piece that the end cuts is read so that it ends
// with the row, and then moved to its place: all pieces are asked for before the first is moved, without a branch between (branches between
// them had every piece wait for the one before: 3 x 5161 x 2 x 89 bf16 gradients 468 us, now 355; 4 queries to 4000 keys of 59 columns 39, 23).
template <class T>
__device__ __forceinline__ v4u fetch16(const T* row, int c, int D)
{
    constexpr int per = 16 / (int)sizeof(T);
    return *reinterpret_cast<const v4u_any*>(row + (c < D - per ? c : D - per));
}
template <class T>
__device__ __forceinline__ v4u place16(v4u q, int c, int D)
{
    constexpr int per = 16 / (int)sizeof(T);
    const int over = c + per - D, halves = over > 0 ? over * (int)sizeof(T) / 2 : 0;
    if constexpr (sizeof(T) == 2) {
        if (halves & 1) q = v4u{q[0] >> 16 | q[1] << 16, q[1] >> 16 | q[2] << 16, q[2] >> 16 | q[3] << 16, q[3] >> 16};
    }
    if (halves & 2) q = v4u{q[1], q[2], q[3], 0};
    if (halves & 4) q = v4u{q[2], q[3], 0, 0};
    return halves < 8 ? q : v4u{0, 0, 0, 0};
}
// Rows shorter than a piece.
template <class T>
__device__ __forceinline__ v4u few16(const T* row, int c, int D)
{
    constexpr int per = 16 / (int)sizeof(T);
    v4u q = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < per - 1; ++e)
        if (c + e < D) {
            if constexpr (sizeof(T) == 4) q[e] = __float_as_uint(row[c + e]);
            else q[e / 2] |= (uint32_t)row[c + e] << (16 * (e & 1));
        }
    return q;
}
__device__ __forceinline__ void split(v4f lo, v4f hi, Frag<float>& f)
{
    const float x[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    split(x, f);
}
// A lane's row in pieces: of every 16 columns those from 8 h on.  Only those of the last part can lie behind the row's end.
template <class T, int PARTS>
struct Pieces {
    static constexpr int kPer = 16 / (int)sizeof(T), kEach = 8 / kPer;
    v4u q[2 * PARTS][kEach];
    __device__ __forceinline__ void load(const T* row, int h, int D)
    {
        if (PARTS == 1 && D < kPer) {
#pragma unroll
            for (int i = 0; i < 2 * PARTS * kEach; ++i) q[i / kEach][i % kEach] = few16(row, column(i, h), D);
            return;
        }
#pragma unroll
        for (int i = 0; i < 2 * PARTS * kEach; ++i) {
            const int c = column(i, h);
            if (i < (2 * PARTS - 2) * kEach) q[i / kEach][i % kEach] = *reinterpret_cast<const v4u_any*>(row + c);
            else q[i / kEach][i % kEach] = fetch16(row, c, D);
        }
#pragma unroll
        for (int i = (2 * PARTS - 2) * kEach; i < 2 * PARTS * kEach; ++i) q[i / kEach][i % kEach] = place16<T>(q[i / kEach][i % kEach], column(i, h), D);
    }
    static __device__ __forceinline__ int column(int i, int h) { return 16 * (i / kEach) + 8 * h + i % kEach * kPer; }
    // the elements of 8 columns
    __device__ __forceinline__ float at(int k, int e) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(q[k][e / 4][e % 4]);
        else return __uint_as_float(e & 1 ? q[k][0][e / 2] & 0xffff0000u : q[k][0][e / 2] << 16);
    }
};
// A lane's row as operands, contraction along its columns.
template <class T, int PARTS>
__device__ __forceinline__ void load_frags(const T* row, int h, int D, Frag<T> (&f)[2 * PARTS])
{
    Pieces<T, PARTS> p;
    p.load(row, h, D);
#pragma unroll
    for (int k = 0; k < 2 * PARTS; ++k) {
        if constexpr (sizeof(T) == 2) f[k].v = __builtin_bit_cast(bf16x8, p.q[k][0]);
        else split(__builtin_bit_cast(v4f, p.q[k][0]), __builtin_bit_cast(v4f, p.q[k][1]), f[k]);
    }
}
template <class T, int PARTS>
__device__ __forceinline__ void clear_frags(Frag<T> (&f)[2 * PARTS])
{
#pragma unroll
    for (int k = 0; k < 2 * PARTS; ++k) __builtin_memset(&f[k], 0, sizeof(f[k]));
}

// ---- tiles in LDS ----
template <class T, int WIDTH>
struct Tile {
    static_assert(WIDTH == kPart || (sizeof(T) == 2 && WIDTH == 2 * kPart), "slabs");
    static constexpr int kPer = 16 / (int)sizeof(T);              // elements a piece
    static constexpr int kPieces = WIDTH / kPer;                  // pieces of a slab's row
    static __device__ __forceinline__ int order(int row)
    {
        if constexpr (sizeof(T) == 4) return (row >> 1) & 7;
        else if constexpr (WIDTH == 64) return (row << 1 & 4) | (row >> 2 & 3);
        else return row >> 2 & 3;
    }
    // piece `piece` of a row of slab `slab`
    static __device__ __forceinline__ int at(int rows, int slab, int row, int piece) { return slab * rows * WIDTH + row * WIDTH + (piece ^ order(row)) * kPer; }
};
template <class T>
constexpr int tile_elements(int rows, int parts) { return rows * parts * kPart; }

// Rows as an operand whose contraction are the columns: columns 16 s + 8 h .. + 7 of row `row`.
template <int WIDTH = kPart>
__device__ __forceinline__ void read_row(const uint16_t* tile, int rows, int row, int h, int s, Frag<uint16_t>& f)
{
    f.v = *reinterpret_cast<const bf16x8*>(tile + Tile<uint16_t, WIDTH>::at(rows, 16 * s / WIDTH, row, 16 * s % WIDTH / 8 + h));
}
template <int WIDTH = kPart>
__device__ __forceinline__ void read_row(const float* tile, int rows, int row, int h, int s, Frag<float>& f)
{
    const v4f lo = *reinterpret_cast<const v4f*>(tile + Tile<float, WIDTH>::at(rows, s >> 1, row, (s & 1) * 4 + h * 2));
    const v4f hi = *reinterpret_cast<const v4f*>(tile + Tile<float, WIDTH>::at(rows, s >> 1, row, (s & 1) * 4 + h * 2 + 1));
    split(lo, hi, f);
}
// Columns as an operand whose contraction are the rows r0 .. r0 + 15 (a multiple of 16), in the order of a result's registers: column
// 32 part + lane % 32.  bf16: the LDS transposing read (in every group of 16 lanes, lanes 4 k .. 4 k + 3 point at 16 elements of row k, and
// lane i receives column i of the four rows).
template <int WIDTH = kPart>
__device__ __forceinline__ void read_column(const uint16_t* tile, int rows, int r0, int lane, int part, Frag<uint16_t>& f)
{
    using L = Tile<uint16_t, WIDTH>;
    const int h = lane >> 5, i = lane & 15, row = 4 * h + (i >> 2), slab = kPart * part / WIDTH;
    const int piece = kPart * part % WIDTH / 8 + ((lane & 16) >> 3) + ((i & 3) >> 1);
    const uint16_t* base = tile + (r0 * WIDTH + (i & 1) * 4);     // (orders repeat after 16 rows)
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(base + L::at(rows, slab, row, piece)));
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(base + L::at(rows, slab, row + 8, piece)));
    const s16x8 v = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    f.v = __builtin_bit_cast(bf16x8, v);
}
template <int WIDTH = kPart>
__device__ __forceinline__ void read_column(const float* tile, int rows, int r0, int lane, int part, Frag<float>& f)
{
    const int h = lane >> 5, c = lane & 31;
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = tile[r0 * kPart + Tile<float, WIDTH>::at(rows, part, (e & 3) + 4 * h + 8 * (e >> 2), c >> 2) + (c & 3)];
    split(x, f);
}

// Where the threads' pieces of a tile of R rows and PARTS parts come from.  A wavefront's load writes 64 consecutive pieces, all of one
// slab; wavefront `wid` of `WAVES` takes every WAVES-th 64, so a thread has the same GROUPS rows and the same piece of them in every slab.
template <class T, int R, int PARTS, int WAVES, int WIDTH = kPart>
struct TileLoad {
    using L = Tile<T, WIDTH>;
    static constexpr int kSlabs = PARTS * kPart / WIDTH, kGroups = R * L::kPieces / (64 * WAVES), kLoads = kGroups * kSlabs;
    static_assert(kGroups * 64 * WAVES == R * L::kPieces && kSlabs * WIDTH == PARTS * kPart, "whole wavefronts' loads, whole slabs");
    static __device__ __forceinline__ int row(int group, int wid, int lane) { return ((group * WAVES + wid) * 64 + lane) / L::kPieces; }
    static __device__ __forceinline__ int column(int group, int wid, int lane) { return ((lane % L::kPieces) ^ L::order(row(group, wid, lane))) * L::kPer; }
    static __device__ __forceinline__ int first(int group, int slab, int wid) { return slab * R * WIDTH + (group * WAVES + wid) * 64 * L::kPer; }
};

// Straight to LDS (16-byte aligned rows, a whole number of pieces: one past the row's end becomes its last one; what that multiplies is
// zero, or is not stored), or through registers, where the loads can be on their way while another tile is passed: fetch() asks for them, put()
// lays them down.  src(row): the row's address.  ONCE: past the caches.
template <class T, int R, int PARTS, int WAVES, bool ALIGNED, int WIDTH = kPart, bool ONCE = false>
struct TileOnItsWay {
    using M = TileLoad<T, R, PARTS, WAVES, WIDTH>;
    using L = Tile<T, WIDTH>;
    v4u q[ALIGNED ? 1 : M::kLoads];
    template <class F>
    __device__ __forceinline__ void fetch(T* tile, int wid, int lane, int D, F src)
    {
        if constexpr (ALIGNED) {
#pragma unroll
            for (int g = 0; g < M::kGroups; ++g) {
                const int c = M::column(g, wid, lane), end = D - L::kPer - (M::kSlabs - 1) * WIDTH;
                const T* p = src(M::row(g, wid, lane)) + c;
#pragma unroll
                for (int s = 0; s < M::kSlabs; ++s) {
                    if (s == M::kSlabs - 1) p -= c > end ? c - end : 0;
                    __builtin_amdgcn_global_load_lds((global_ptr)(p + s * WIDTH), (lds_ptr)(tile + M::first(g, s, wid)), 16, 0, ONCE ? kNonTemporal : 0);
                }
            }
        } else if (PARTS == 1 && D < L::kPer) {
#pragma unroll
            for (int g = 0; g < M::kGroups; ++g) q[g] = few16(src(M::row(g, wid, lane)), M::column(g, wid, lane), D);
        } else {
#pragma unroll
            for (int g = 0; g < M::kGroups; ++g) {
                const T* p = src(M::row(g, wid, lane));
                const int c = M::column(g, wid, lane);
#pragma unroll
                for (int s = 0; s < M::kSlabs; ++s) q[g * M::kSlabs + s] = s < M::kSlabs - 1 ? *reinterpret_cast<const v4u_any*>(p + (s * WIDTH + c)) : fetch16(p, s * WIDTH + c, D);
            }
        }
    }
    __device__ __forceinline__ void put(T* tile, int wid, int lane, int D)
    {
        if constexpr (!ALIGNED) {
            const bool few = PARTS == 1 && D < L::kPer;            // those lie in their places
#pragma unroll
            for (int g = 0; g < M::kGroups; ++g)
#pragma unroll
                for (int s = 0; s < M::kSlabs; ++s) {
                    v4u p = q[g * M::kSlabs + s];
                    if (s == M::kSlabs - 1 && !few) p = place16<T>(p, s * WIDTH + M::column(g, wid, lane), D);
                    *reinterpret_cast<v4u*>(tile + (M::first(g, s, wid) + lane * L::kPer)) = p;
                }
        }
    }
};
template <class T, int R, int PARTS, int WAVES, bool ALIGNED, int WIDTH = kPart, bool ONCE = false, class F>
__device__ __forceinline__ void load_tile(T* tile, int wid, int lane, int D, F src)
{
    TileOnItsWay<T, R, PARTS, WAVES, ALIGNED, WIDTH, ONCE> t;
    t.fetch(tile, wid, lane, D, src);
    t.put(tile, wid, lane, D);
}

// The tile handed over: this wavefront's loads have arrived, everyone's part is there, and nobody reads the buffer that is filled next.
__device__ __forceinline__ void tiles_barrier()
{
    __builtin_amdgcn_s_waitcnt(0x0070);                           // vmcnt 0, lgkmcnt 0
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// N products whose operands read(i, f) gets from LDS, DEPTH of them ahead of multiply(i, f): left to itself the compiler reads each one
// just before its product, into the same registers, and every product waits for LDS.  Instructions of the vector unit may be moved
// between the steps.  start() may come earlier, with other work behind it.
template <class T, int N, int DEPTH>
struct Ahead {
    static constexpr int kDepth = DEPTH < N ? DEPTH : N;
    static constexpr int kMayMove = 0x2 | 0x4 | 0x400;            // vector, scalar, transcendental
    Frag<T> f[kDepth];
    template <class R>
    __device__ __forceinline__ void start(R read)
    {
#pragma unroll
        for (int i = 0; i < kDepth; ++i) read(i, f[i]);
        __builtin_amdgcn_sched_barrier(kMayMove);
    }
    template <class R, class M>
    __device__ __forceinline__ void run(R read, M mul)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            mul(i, f[i % kDepth]);
            if (i + kDepth < N) read(i + kDepth, f[i % kDepth]);
            __builtin_amdgcn_sched_barrier(kMayMove);
        }
    }
};

// ---- rows ----
// x / d for x < 2^31
struct Divide {
    uint32_t mul;
    int shift;
};
inline Divide divide_by(int d)
{
    int l = 0;
    while ((INT64_C(1) << l) < d) ++l;
    return Divide{(uint32_t)(((UINT64_C(1) << (31 + l)) + (uint64_t)d - 1) / (uint64_t)d), 31 + l};
}
__device__ __forceinline__ int over(int x, const Divide& d) { return (int)(((uint64_t)(uint32_t)x * d.mul) >> d.shift); }

// The value that the lane of the other half (lane exclusive or 32) holds.
__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32); }

// Units a die, if all dies get (about) as many.
inline int units_a_die(int units)
{
    const int each = (units + 7) / 8;
    return 8 * each * 9 <= units * 10 ? each : 0;
}
// What a call is about; its entries' lengths are read on the device.
struct Shape {
    const int32_t *q_lens, *k_lens;
    int Tq, Tk, Hq, Hk, D, G, rows;  // rows: Tq G
    int units, causal;               // units: entries x key heads
    int per_die;                     // units a die takes for itself, 0: any takes any
    Divide by_g;
};
template <class A>
void set_shape(Shape& g, const A& p)
{
    g.q_lens = p.q_lens; g.k_lens = p.k_lens;
    g.Tq = p.Tq; g.Tk = p.Tk; g.Hq = p.Hq; g.Hk = p.Hk; g.D = p.D;
    g.G = p.Hq / p.Hk; g.rows = p.Tq * g.G;
    g.units = p.B * p.Hk; g.causal = p.causal;
    g.by_g = divide_by(g.G);
    g.per_die = units_a_die(g.units);
}

// A workgroup's unit, and its number among the unit's.  Workgroups go to the eight dies in turn, and each die has a cache of its own:
// where units come out even, a die takes units of its own, every eighth, so that each has some of every part of the batch.  It goes
// through them a few at a time, as many as fill it, whose keys and values its cache then holds.  (32 x 2048 tokens of 16 heads of 128, 1.1 GB
// of keys and values: 1143 us, 1915 with all units at once; their gradients for 16 entries 1237 and 1350; where all fit the memory-side
// cache no difference, 2 x 8192 of 32 and 8 heads 1055 and 1058.)
struct Place {
    int unit, at;
};
constexpr int kFill = 64;                                         // workgroups at work on a die (16: 16 x 2048 x 8 x 64 101 -> 114 us; 256: the first of the above 1197)
__device__ __forceinline__ Place place_of(const Shape& g, int each)
{
    if (g.per_die == 0) return Place{(int)(blockIdx.x % g.units), (int)(blockIdx.x / g.units)};
    const int few = (kFill - 1) / each + 1, at = blockIdx.x >> 3, first = at / (few * each) * few, rest = at - first * each;
    const int here = g.per_die - first < few ? g.per_die - first : few;
    return Place{(int)(blockIdx.x & 7) + (first + rest % here) * 8, rest / here};
}
inline int64_t workgroups(const Shape& g, int64_t each) { return each * (g.per_die ? 8 * g.per_die : g.units); }
__device__ __forceinline__ int length_of(const int32_t* lens, int b, int most)
{
    const int n = lens ? lens[b] : most;
    return n < 0 ? 0 : n > most ? most : n;
}

// Which queries and keys a tile of rows is about.
struct Rows {
    int b, hk, nq, nk;
    int end;                         // keys from there on are seen by none of its rows
};
__device__ __forceinline__ Rows rows_of(const Shape& g, int unit, int r0, int n)
{
    Rows t;
    t.b = unit / g.Hk;
    t.hk = unit % g.Hk;
    t.nq = length_of(g.q_lens, t.b, g.Tq);
    t.nk = length_of(g.k_lens, t.b, g.Tk);
    const int first = over(r0, g.by_g), r1 = r0 + n - 1 < g.rows ? r0 + n - 1 : g.rows - 1;
    int last = over(r1, g.by_g);
    if (last > t.nq - 1) last = t.nq - 1;
    t.end = t.nk;
    if (g.causal && last + t.nk - t.nq + 1 < t.nk) t.end = last + t.nk - t.nq + 1;
    if (first > last || t.end < 0) t.end = 0;
    return t;
}

// A lane's row: its query and head, and how many keys it sees.
struct Row {
    int t, head, sees;
    bool there;
};
__device__ __forceinline__ Row row_of(const Shape& g, const Rows& rows, int r)
{
    Row q;
    q.there = r < g.rows;
    if (!q.there) r = g.rows - 1;
    q.t = over(r, g.by_g);
    q.head = rows.hk * g.G + r - q.t * g.G;
    q.sees = rows.nk;
    if (g.causal && q.t + rows.nk - rows.nq + 1 < q.sees) q.sees = q.t + rows.nk - rows.nq + 1;
    if (q.t >= rows.nq || q.sees < 0) q.sees = 0;
    return q;
}

__device__ __forceinline__ int wave_min(int x)
{
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) x = min(x, __shfl_xor(x, d));
    return __builtin_amdgcn_readfirstlane(x);
}
__device__ __forceinline__ int wave_max(int x)
{
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) x = max(x, __shfl_xor(x, d));
    return __builtin_amdgcn_readfirstlane(x);
}

// Four columns of a row, as many of them as it has.
template <class T>
__device__ __forceinline__ void store4(T* row, int c, int D, const float (&v)[4])
{
    if (c + 4 <= D) put4(row + c, v);
    else
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (c + e < D) put1(row + c + e, v[e]);
}

// Four sums times a factor, or zeros, whatever the sums are.
__device__ __forceinline__ void scaled(const f32x16& s, int i, float factor, bool live, float (&o)[4])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = live ? s[i + e] * factor : 0.0f;
}
// The lane's columns of its row, times a factor, any alignment.  live: not zeros.
template <class T, int PARTS>
__device__ __forceinline__ void store_sums(T* row, int lane, int D, float factor, const f32x16 (&s)[PARTS], bool live = true)
{
#pragma unroll
    for (int p = 0; p < PARTS; ++p)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            float o[4];
            scaled(s[p], i, factor, live, o);
            store4(row, p * kPart + 2 * i + 4 * (lane >> 5), D, o);
        }
}
// The same of 16-byte aligned rows, a whole number of pieces: through LDS ([32][PARTS 32] of the wavefront's own), so that rows are written
// by 16 bytes a lane, one after the other, and not by 8 of 32 rows at a time.  row(i): the address of row i of the 32, NULL: not stored.
template <class T, int PARTS, class F>
__device__ __forceinline__ void store_rows(T* lds, int lane, int D, float factor, const f32x16 (&s)[PARTS], bool live, F row)
{
    constexpr int kPer = 16 / (int)sizeof(T), kPieces = PARTS * kPart / kPer;
    auto at = [](int r, int piece) { return (r * kPieces + (piece + r) % kPieces) * kPer; };      // rotated: over all banks
#pragma unroll
    for (int p = 0; p < PARTS; ++p)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            float o[4];
            scaled(s[p], i, factor, live, o);
            const int c = p * kPart + 2 * i + 4 * (lane >> 5);
            put4(lds + (at(lane & 31, c / kPer) + c % kPer), o);
        }
    asm volatile("" ::: "memory");                                // (LDS serves a wavefront in order)
#pragma unroll
    for (int k = 0; k < 32 * kPieces / 64; ++k) {
        const int slot = k * 64 + lane, r = slot / kPieces, piece = slot % kPieces;
        T* to = row(r);
        if (to && piece * kPer < D) *reinterpret_cast<v4u*>(to + piece * kPer) = *reinterpret_cast<const v4u*>(lds + at(r, piece));
    }
    asm volatile("" ::: "memory");
}

// ---- host ----
constexpr size_t kAlign = 256;
constexpr int kMaxEntries = 1 << 20, kMaxTokens = 1 << 24, kMaxHeads = 1024;

#define LSGD_TRY(x)                         \
    do {                                    \
        const lsgd_status st_ = (x);        \
        if (st_ != LSGD_OK) return st_;     \
    } while (0)

// A scale whose inverse is a normal value as well, with room for scores.
inline bool scale_ok(float scale) { return scale >= 1e-30f && scale <= 1e30f; }
lsgd_status check_attention_shape(const char* who, int64_t B, int64_t Tq, int64_t Tk, int64_t Hq, int64_t Hk, int64_t D);
inline int parts_of(int D) { return (D + kPart - 1) / kPart; }

template <class F>
void by_type_and_parts(bool bf16, int parts, F f)
{
    auto typed = [&](auto type) {
        if (parts == 1) f(type, std::integral_constant<int, 1>{});
        else if (parts == 2) f(type, std::integral_constant<int, 2>{});
        else if (parts == 3) f(type, std::integral_constant<int, 3>{});
        else f(type, std::integral_constant<int, 4>{});
    };
    if (bf16) typed(uint16_t{});
    else typed(float{});
}

} // namespace attention
} // namespace lsgd
