// Gradients of attention, from what the forward call left: with c = scale log2 e, z = lse log2 e, delta = dout . out of a query,
//
//   p = 2^(c s - z),  s = q . k;   dv = p' dout;   dp = dout . v;   ds = p (dp - delta);   dq = scale ds k;   dk = scale ds' q
//
// z / c and delta are taken off where the products begin: their negatives are what the accumulators hold first.  (fp32's s begins with
// zero: its chain of D / 2 sums would round at the size of z / c each time, which the 8 of bf16 can bear.)
//
// Two passes over the pairs, so that every sum has one owner and an order of its own: no atomics, equal calls give equal bits.  By
// rows: 32 rows a wavefront keep q, dout and the sums for dq in registers while K and V tiles pass through LDS; it makes delta on the way and
// leaves z and delta to the other.  By keys: 32 keys a wavefront keep k, v and the sums for dk and dv while tiles of q and dout
// pass; the rows of all query heads that share the key head are in the list, so their gradients add up by themselves.  s and dp are made
// twice: 7 products where 5 would do, for gradients that go through memory once and need no order between workgroups.
//
// In both, results become operands in registers (attention_common.h): by rows s^T and dp^T, keys becoming the contraction, by
// keys s and dp, rows becoming it.  Where a pass has few workgroups, further ones split its contraction, and a launch adds up their sums.
//
// By rows bound by the products, by keys also by loads that are waited for: 4 x 4096 causal tokens of 16 and 4 heads of 128 bf16 0.95 to 1.02 ms,
// 0.95 to 1.0 PFLOP/s of the seven products, the three by rows in 0.35 to 0.4 ms, the four by keys in 0.6.  By keys z and delta are asked
// for after the next tile and laid down at once, and loads arrive in order, so the wavefronts that bring them wait for that tile before they
// pass the present one.  Registers that do not suffice, in bytes of scratch a lane (aligned, off alignment): by keys bf16 of 97 to 128 columns
// 56 and 64, reloaded between the tile's loads; fp32 of 33 to 64 columns 272 and 288, of 97 to 128 16 and 24, few of them off alignment 84; by
// rows fp32 of 33 to 64 columns 12.  fp32: 4 x 2048 causal tokens of 16 and 4 heads of 128 1.56 ms, 110 TFLOP/s of the five products
// counted, of 16 heads of 64 0.9, 96.  Small ones by the chain of one workgroup's tiles (3 x 100 to 259 keys of 72 columns fp32: 14 + 16 + 4 us).
#include <algorithm>
#include <cmath>

#include "attention_common.h"

namespace lsgd {
namespace attention {
namespace {

struct Args : Shape {
    Heads dout, q, k, v, out, dq, dk, dv;
    const float* lse;                // [B][Hq][Tq]
    float *z, *delta;                // [units][rows]: -z / c (fp32: -z), -inf for rows that see nothing, and -delta
    float *dq_parts, *dkv_parts;     // of splits, NULL: one
    int row_tiles, key_tiles;
    int row_splits, row_chunk;       // by rows: workgroups a tile, and the keys of one
    int key_splits, key_chunk;       // by keys: workgroups a tile, and the rows of one
    float scale, inv_scale, c;
};

// A workgroup owns 32 OWN rows, or keys, and SHARE of its wavefronts share each 32: of every tile that passes, each takes PASS of the rows
// (keys), and their sums are added up in order at the end.  BUFFERS tiles: 2, the next is asked for before one is passed.
template <int OWN_, int SHARE_, int PASS_, int BUFFERS_>
struct Form {
    static constexpr int OWN = OWN_, SHARE = SHARE_, PASS = PASS_, BUFFERS = BUFFERS_;
    static constexpr int WAVES = OWN * SHARE, THREADS = 64 * WAVES, TILE = SHARE * PASS, MINE = 32 * OWN;
};
// Many rows: 128 a workgroup.
template <class T> using RowsMany = Form<4, 1, sizeof(T) == 2 ? 64 : 32, 2>;
// Many keys: with a causal mask the first keys have all rows to pass and the last none, and two halves of a workgroup that take every
// second tile halve the longest one's time (gradients of 4 x 4096 x 16 x 128: 1160 -> 955 us).  The parts of wide fp32 leave registers for
// one wavefront a SIMD, so four in all (4 x 1024 x 8 x 128: 345 us, 475 with eight; but 64 columns 169, 192 with four).
template <class T, int PARTS> constexpr bool kWide = sizeof(T) == 4 && PARTS > 2;
template <class T, int PARTS>
using KeysMany = std::conditional_t<kWide<T, PARTS>, Form<2, 2, 32, 2>, Form<4, 2, sizeof(T) == 2 ? 64 : 32, 2>>;
// Few of either: 32 a workgroup.
template <class T> using Few = Form<1, 4, 32, 1>;

template <class T>
constexpr bool kFromZ = sizeof(T) == 2;                  // s begins with -z / c
constexpr int kChunk = 128;                              // chunks of a split are multiples of it

// An operand's element as it was.
__device__ __forceinline__ float value(const Frag<uint16_t>& a, int e) { return (float)a.v[e]; }
__device__ __forceinline__ float value(const Frag<float>& a, int e) { return (float)a.v[0][e] + ((float)a.v[1][e] + (float)a.v[2][e]); }
// Rows off 16 bytes wait in registers while a tile is passed, if those suffice (3 x 5161 x 2 x 89 354 -> 325 us; but 8 x 1000 x 8 x 125 154, late
// 203, fp32 475 and 496).
template <class T, int PARTS>
constexpr bool kLate = sizeof(T) == 2 && PARTS < 4;
// How far operands are read ahead; by keys registers are short.  (4 x 4096 x 16 x 128: 967 us; two by rows and four by keys 1006.)
template <class T>
constexpr int kAheadRows = sizeof(T) == 2 ? 4 : 2;
template <class T>
constexpr int kAheadKeys = 2;
// Wavefronts a SIMD.
template <class F, class T, int PARTS>
constexpr int kOccupancy = kWide<T, PARTS> || F::BUFFERS == 1 ? 1 : 2;

// c += the product of 32 rows of a tile, from row r0 on, with an operand in registers.
template <int AHEAD, class T, int PARTS>
__device__ __forceinline__ void rows_times(const T* tile, int rows, int r0, int lane, const Frag<T> (&b)[2 * PARTS], f32x16& c)
{
    Ahead<T, 2 * PARTS, AHEAD> ops;
    auto read = [&](int k, Frag<T>& f) { read_row(tile, rows, r0 + (lane & 31), lane >> 5, k, f); };
    ops.start(read);
    ops.run(read, [&](int k, const Frag<T>& f) { multiply(c, f, b[k]); });
}
// sums += the columns of 32 rows of a tile times a result made an operand.
template <int AHEAD, class T, int PARTS>
__device__ __forceinline__ void columns_times(const T* tile, int rows, int r0, int lane, const Frag<T> (&b)[2], f32x16 (&sums)[PARTS])
{
    Ahead<T, 2 * PARTS, AHEAD> ops;
    auto read = [&](int i, Frag<T>& f) { read_column(tile, rows, r0 + 16 * (i / PARTS), lane, i % PARTS, f); };
    ops.start(read);
    ops.run(read, [&](int i, const Frag<T>& f) { multiply(sums[i % PARTS], f, b[i / PARTS]); });
}
template <int PARTS>
__device__ __forceinline__ void clear_sums(f32x16 (&s)[PARTS])
{
#pragma unroll
    for (int p = 0; p < PARTS; ++p)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[p][i] = 0.0f;
}
// The sums of the wavefronts that share rows, in the first one's registers: areas of a wavefront's sums in the two tiles' memory.
template <class F, int PARTS>
__device__ __forceinline__ void join_shared(void* tile0, void* tile1, int own, int share, int lane, f32x16 (&s)[PARTS])
{
    if constexpr (F::SHARE > 1) {
        constexpr int kArea = PARTS * 16 * 64, kPerTile = 2;      // floats
        static_assert((F::SHARE - 1) * F::OWN <= 2 * kPerTile, "areas");
        auto area = [&](int k) {
            const int a = k * F::OWN + own;
            return reinterpret_cast<v4f*>(a < kPerTile ? tile0 : tile1) + a % kPerTile * (kArea / 4) + lane;
        };
        __syncthreads();                                          // the tiles, or the last sums, have been read
        if (share) {
            v4f* to = area(share - 1);
#pragma unroll
            for (int i = 0; i < PARTS * 4; ++i) {
                const f32x16& f = s[i / 4];
                const int e = i % 4 * 4;
                to[i * 64] = v4f{f[e], f[e + 1], f[e + 2], f[e + 3]};
            }
        }
        __syncthreads();
        if (!share) {
#pragma unroll
            for (int k = 0; k < F::SHARE - 1; ++k) {
                const v4f* from = area(k);
#pragma unroll
                for (int i = 0; i < PARTS * 16; ++i) s[i / 16][i % 16] += from[i / 4 * 64][i % 4];
            }
        }
    }
}

template <class F, class T, int PARTS, bool ALIGNED>
__global__ __launch_bounds__(F::THREADS, (kOccupancy<F, T, PARTS>)) void attention_dq_kernel(Args g)
{
    constexpr int KEYS = F::TILE, N = tile_elements<T>(KEYS, PARTS);
    static_assert(sizeof(T) * N >= 2 * 4 * PARTS * 16 * 64 || F::SHARE == 1, "two areas a tile");
    __shared__ __attribute__((aligned(16))) T k0[N], k1[F::BUFFERS > 1 ? N : 8];
    __shared__ __attribute__((aligned(16))) T v0[N], v1[F::BUFFERS > 1 ? N : 8];
    const int own = __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) % F::OWN), share = __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) / F::OWN);
    const int lane = threadIdx.x & 63, h = lane >> 5, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Place at = place_of(g, g.row_tiles * g.row_splits);
    if (at.unit >= g.units) return;
    const int split = at.at % g.row_splits, tile = g.row_tiles - 1 - at.at / g.row_splits;   // late rows see most keys: first
    const Rows rows = rows_of(g, at.unit, tile * F::MINE, F::MINE);
    const int r = tile * F::MINE + own * 32 + (lane & 31);
    const Row row = row_of(g, rows, r);
    const int least = wave_min(row.sees), most = wave_max(row.sees);
    Frag<T> qf[2 * PARTS], df[2 * PARTS];
    float z = -INFINITY, delta = 0.0f;                                     // negative, as the accumulators begin
    {
        const T* q = static_cast<const T*>(g.q.p) + rows.b * g.q.lb + row.t * g.q.lt + row.head * g.q.lh;
        const T* d = static_cast<const T*>(g.dout.p) + rows.b * g.dout.lb + row.t * g.dout.lt + row.head * g.dout.lh;
        const T* o = static_cast<const T*>(g.out.p) + rows.b * g.out.lb + row.t * g.out.lt + row.head * g.out.lh;
        if (row.sees == 0) {
            clear_frags<T, PARTS>(qf);
            clear_frags<T, PARTS>(df);
        } else {
            load_frags<T, PARTS>(q, h, g.D, qf);
            load_frags<T, PARTS>(d, h, g.D, df);
            Pieces<T, PARTS> of;
            of.load(o, h, g.D);
#pragma unroll
            for (int i = 0; i < 16 * PARTS; ++i) delta -= of.at(i / 8, i % 8) * value(df[i / 8], i % 8);
            z = -g.lse[((int64_t)rows.b * g.Hq + row.head) * g.Tq + row.t] * (kFromZ<T> ? g.inv_scale : kLog2e);
        }
        delta += other_half(delta);
        if (split == 0 && share == 0 && h == 0 && row.there) {
            g.z[(int64_t)at.unit * g.rows + r] = z;
            g.delta[(int64_t)at.unit * g.rows + r] = delta;
        }
    }
    f32x16 dq[PARTS];
    clear_sums<PARTS>(dq);
    const T* k = static_cast<const T*>(g.k.p) + rows.b * g.k.lb + rows.hk * g.k.lh;
    const T* v = static_cast<const T*>(g.v.p) + rows.b * g.v.lb + rows.hk * g.v.lh;
    const int begin = split * g.row_chunk, end = min(rows.end, begin + g.row_chunk);
    TileOnItsWay<T, KEYS, PARTS, F::WAVES, ALIGNED> kt, vt;
    auto issue = [&](int key0, T* kb, T* vb) {
        auto key = [&](int i) { return key0 + i < rows.nk ? key0 + i : rows.nk - 1; };
        kt.fetch(kb, wid, lane, g.D, [&](int i) { return k + key(i) * g.k.lt; });
        vt.fetch(vb, wid, lane, g.D, [&](int i) { return v + key(i) * g.v.lt; });
    };
    auto put = [&](T* kb, T* vb) {
        kt.put(kb, wid, lane, g.D);
        vt.put(vb, wid, lane, g.D);
    };
    auto pass = [&](int key0, const T* kb, const T* vb) {
        if (key0 + share * F::PASS >= most) return;
        const bool masked = key0 + (share + 1) * F::PASS > least;
#pragma unroll
        for (int n = 0; n < F::PASS / 32; ++n) {
            const int k0 = share * F::PASS + 32 * n;
            f32x16 s, dp;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[i] = kFromZ<T> ? z : 0.0f;
                dp[i] = delta;
            }
            rows_times<kAheadRows<T>, T, PARTS>(kb, KEYS, k0, lane, qf, s);
            rows_times<kAheadRows<T>, T, PARTS>(vb, KEYS, k0, lane, df, dp);
#pragma unroll
            for (int i = 0; i < 16; ++i) dp[i] *= __builtin_amdgcn_exp2f(kFromZ<T> ? s[i] * g.c : fmaf(s[i], g.c, z));
            if (masked) {
#pragma unroll
                for (int i = 0; i < 16; ++i) dp[i] = key0 + k0 + 8 * (i >> 2) + 4 * h + (i & 3) < row.sees ? dp[i] : 0.0f;
            }
            Frag<T> ef[2];
            from_result(dp, 0, ef[0]);
            from_result(dp, 1, ef[1]);
            columns_times<kAheadRows<T>, T, PARTS>(kb, KEYS, k0, lane, ef, dq);
        }
    };
    if constexpr (F::BUFFERS > 1) {
        auto step = [&](int key0, T* kb, T* vb, T* next_k, T* next_v) {
            tiles_barrier();
            if (key0 + KEYS < end) {
                issue(key0 + KEYS, next_k, next_v);
                if (!kLate<T, PARTS>) put(next_k, next_v);
            }
            pass(key0, kb, vb);
            if (kLate<T, PARTS> && key0 + KEYS < end) put(next_k, next_v);
        };
        if (begin < end) {
            issue(begin, k0, v0);
            put(k0, v0);
        }
        for (int key0 = begin; key0 < end; key0 += 2 * KEYS) {
            step(key0, k0, v0, k1, v1);
            if (key0 + KEYS < end) step(key0 + KEYS, k1, v1, k0, v0);
        }
    } else {
        for (int key0 = begin; key0 < end; key0 += KEYS) {
            if (key0 > begin) tiles_barrier();                     // the last tiles have been read
            issue(key0, k0, v0);
            put(k0, v0);
            tiles_barrier();
            pass(key0, k0, v0);
        }
    }
    join_shared<F, PARTS>(k0, v0, own, share, lane, dq);
    if (!row.there || share) return;
    // (a row that sees nothing: zeros, not 0 x infinity of keys that rows beside it see)
    if (g.dq_parts)
        store_sums<float, PARTS>(g.dq_parts + (((int64_t)at.unit * g.rows + r) * g.row_splits + split) * (PARTS * kPart), lane, PARTS * kPart, g.scale, dq, row.sees > 0);
    else
        store_sums<T, PARTS>(static_cast<T*>(g.dq.p) + rows.b * g.dq.lb + row.t * g.dq.lt + row.head * g.dq.lh, lane, g.D, g.scale, dq, row.sees > 0);
}

// The first row that sees a key.
__device__ __forceinline__ int first_row(const Args& g, int nq, int nk, int key)
{
    const int t = key - (nk - nq);
    return g.causal && t > 0 ? (t < nq ? t : nq) * g.G : 0;
}

template <class F, class T, int PARTS, bool ALIGNED>
__global__ __launch_bounds__(F::THREADS, (kOccupancy<F, T, PARTS>)) void attention_dkv_kernel(Args g)
{
    constexpr int ROWS = F::TILE, N = tile_elements<T>(ROWS, PARTS);
    static_assert(sizeof(T) * N >= 2 * 4 * PARTS * 16 * 64 || F::SHARE == 1, "two areas a tile");
    __shared__ __attribute__((aligned(16))) T q0[N], q1[F::BUFFERS > 1 ? N : 8];
    __shared__ __attribute__((aligned(16))) T d0[N], d1[F::BUFFERS > 1 ? N : 8];
    __shared__ __attribute__((aligned(16))) float z0[ROWS], z1[ROWS], e0[ROWS], e1[ROWS];
    const int own = __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) % F::OWN), share = __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) / F::OWN);
    const int lane = threadIdx.x & 63, h = lane >> 5, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Place at = place_of(g, g.key_tiles * g.key_splits);
    if (at.unit >= g.units) return;
    const int split = at.at % g.key_splits, tile = at.at / g.key_splits;
    const int b = at.unit / g.Hk, hk = at.unit % g.Hk;
    const int nq = length_of(g.q_lens, b, g.Tq), nk = length_of(g.k_lens, b, g.Tk);
    const int key0 = tile * F::MINE, key = key0 + own * 32 + (lane & 31);
    const bool live = key < nk;
    Frag<T> kf[2 * PARTS], vf[2 * PARTS];
    if (live) {
        load_frags<T, PARTS>(static_cast<const T*>(g.k.p) + b * g.k.lb + key * g.k.lt + hk * g.k.lh, h, g.D, kf);
        load_frags<T, PARTS>(static_cast<const T*>(g.v.p) + b * g.v.lb + key * g.v.lt + hk * g.v.lh, h, g.D, vf);
    } else {
        clear_frags<T, PARTS>(kf);
        clear_frags<T, PARTS>(vf);
    }
    // a key behind the last has zeros for k and v; what its lane adds up is not stored
    const int from = live ? first_row(g, nq, nk, key) : 0, least = first_row(g, nq, nk, key0 + own * 32), most = wave_max(from);
    // rows that see no key, causal ones before the first that does among them, and places behind the last: p = 0, times what a row that
    // sees some holds, so that NaN in theirs is not passed
    const int rows_live = nq * g.G, row_first = first_row(g, nq, nk, 0);
    int begin = first_row(g, nq, nk, key0) / ROWS * ROWS, end = key0 < nk ? rows_live : 0;
    begin = max(begin, split * g.key_chunk);
    end = min(end, (split + 1) * g.key_chunk);
    f32x16 dk[PARTS], dv[PARTS];
    clear_sums<PARTS>(dk);
    clear_sums<PARTS>(dv);
    const T* q = static_cast<const T*>(g.q.p) + b * g.q.lb + (int64_t)hk * g.G * g.q.lh;
    const T* d = static_cast<const T*>(g.dout.p) + b * g.dout.lb + (int64_t)hk * g.G * g.dout.lh;
    const float* z = g.z + (int64_t)at.unit * g.rows;
    const float* delta = g.delta + (int64_t)at.unit * g.rows;
    TileOnItsWay<T, ROWS, PARTS, F::WAVES, ALIGNED> qt, dt;
    auto put = [&](T* qb, T* db) {
        qt.put(qb, wid, lane, g.D);
        dt.put(db, wid, lane, g.D);
    };
    auto issue = [&](int r0, T* qb, T* db, float* zb, float* eb) {
        auto place = [&](int i, const Heads& a) {
            const int r = min(max(r0 + i, row_first), rows_live - 1), t = over(r, g.by_g);
            return t * a.lt + (r - t * g.G) * a.lh;
        };
        qt.fetch(qb, wid, lane, g.D, [&](int i) { return q + place(i, g.q); });
        dt.fetch(db, wid, lane, g.D, [&](int i) { return d + place(i, g.dout); });
        static_assert(ROWS <= F::THREADS && kChunk % ROWS == 0, "a value a thread, whole tiles a chunk");
        if ((int)threadIdx.x < ROWS) {
            const int r = r0 + (int)threadIdx.x;
            zb[threadIdx.x] = r < rows_live ? z[r] : -INFINITY;
            eb[threadIdx.x] = r < rows_live ? delta[r] : 0.0f;
        }
    };
    auto pass = [&](int r0, const T* qb, const T* db, const float* zb, const float* eb) {
        if (r0 + (share + 1) * F::PASS <= least) return;
        const bool masked = r0 + share * F::PASS < most;
#pragma unroll 1
        for (int n = 0; n < F::PASS / 32; ++n) {
            const int i0 = share * F::PASS + 32 * n;
            f32x16 s, dp;
            auto begin_with = [&](const float* first, f32x16& c) {
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const v4f x = *reinterpret_cast<const v4f*>(first + i0 + 2 * i + 4 * h);
#pragma unroll
                    for (int e = 0; e < 4; ++e) c[i + e] = x[e];
                }
            };
            if constexpr (kFromZ<T>) {
                begin_with(zb, s);
                rows_times<kAheadKeys<T>, T, PARTS>(qb, ROWS, i0, lane, kf, s);
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(s[i] * g.c);
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = 0.0f;
                rows_times<kAheadKeys<T>, T, PARTS>(qb, ROWS, i0, lane, kf, s);
                begin_with(zb, dp);
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], g.c, dp[i]));
            }
            if (masked) {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = r0 + i0 + 8 * (i >> 2) + 4 * h + (i & 3) >= from ? s[i] : 0.0f;
            }
            begin_with(eb, dp);
            rows_times<kAheadKeys<T>, T, PARTS>(db, ROWS, i0, lane, vf, dp);
            // both become operands before either is passed on, so that the products' registers are free
            Frag<T> pf[2], ef[2];
            from_result(s, 0, pf[0]);
            from_result(s, 1, pf[1]);
#pragma unroll
            for (int i = 0; i < 16; ++i) dp[i] *= s[i];
            from_result(dp, 0, ef[0]);
            from_result(dp, 1, ef[1]);
            columns_times<kAheadKeys<T>, T, PARTS>(db, ROWS, i0, lane, pf, dv);
            columns_times<kAheadKeys<T>, T, PARTS>(qb, ROWS, i0, lane, ef, dk);
        }
    };
    if constexpr (F::BUFFERS > 1) {
        auto step = [&](int r0, T* qb, T* db, float* zb, float* eb, T* next_q, T* next_d, float* next_z, float* next_e) {
            tiles_barrier();
            if (r0 + ROWS < end) {
                issue(r0 + ROWS, next_q, next_d, next_z, next_e);
                if (!kLate<T, PARTS>) put(next_q, next_d);
            }
            pass(r0, qb, db, zb, eb);
            if (kLate<T, PARTS> && r0 + ROWS < end) put(next_q, next_d);
        };
        if (begin < end) {
            issue(begin, q0, d0, z0, e0);
            put(q0, d0);
        }
        for (int r0 = begin; r0 < end; r0 += 2 * ROWS) {
            step(r0, q0, d0, z0, e0, q1, d1, z1, e1);
            if (r0 + ROWS < end) step(r0 + ROWS, q1, d1, z1, e1, q0, d0, z0, e0);
        }
    } else {
        for (int r0 = begin; r0 < end; r0 += ROWS) {
            if (r0 > begin) tiles_barrier();                       // the last tiles have been read
            issue(r0, q0, d0, z0, e0);
            put(q0, d0);
            tiles_barrier();
            pass(r0, q0, d0, z0, e0);
        }
    }
    join_shared<F, PARTS>(q0, d0, own, share, lane, dk);
    join_shared<F, PARTS>(q0, d0, own, share, lane, dv);
    if (key >= g.Tk || share) return;
    if (!live) {
        clear_sums<PARTS>(dk);
        clear_sums<PARTS>(dv);
    }
    if (g.dkv_parts) {
        float* part = g.dkv_parts + (((int64_t)at.unit * g.Tk + key) * g.key_splits + split) * (2 * PARTS * kPart);
        store_sums<float, PARTS>(part, lane, PARTS * kPart, g.scale, dk);
        store_sums<float, PARTS>(part + PARTS * kPart, lane, PARTS * kPart, 1.0f, dv);
    } else {
        store_sums<T, PARTS>(static_cast<T*>(g.dk.p) + b * g.dk.lb + key * g.dk.lt + hk * g.dk.lh, lane, g.D, g.scale, dk);
        store_sums<T, PARTS>(static_cast<T*>(g.dv.p) + b * g.dv.lb + key * g.dv.lt + hk * g.dv.lh, lane, g.D, 1.0f, dv);
    }
}

// The sums of the splits' parts, in order: of dq, and of dk and dv.
constexpr int kJoinThreads = 256;
template <class T, int PARTS, bool KV>
__device__ __forceinline__ void join_parts(const Args& g)
{
    constexpr int COLS = PARTS * kPart, LISTS = KV ? 2 : 1;
    const int splits = KV ? g.key_splits : g.row_splits, many = KV ? g.Tk : g.rows;
    const int64_t id = (int64_t)blockIdx.x * kJoinThreads + threadIdx.x, row = id / COLS;
    const int c = (int)(id % COLS), r = (int)(row % many);
    if (row >= (int64_t)g.units * many || c >= g.D) return;
    const int unit = (int)(row / many), b = unit / g.Hk, hk = unit % g.Hk;
    const float* p = (KV ? g.dkv_parts : g.dq_parts) + row * splits * LISTS * COLS + c;
#pragma unroll
    for (int list = 0; list < LISTS; ++list) {
        float s = 0.0f;
        for (int k = 0; k < splits; ++k) s += p[(k * LISTS + list) * COLS];
        const Heads& a = KV ? (list ? g.dv : g.dk) : g.dq;
        const int t = KV ? r : over(r, g.by_g), head = KV ? hk : hk * g.G + r - t * g.G;
        put1(static_cast<T*>(a.p) + b * a.lb + t * a.lt + head * a.lh + c, s);
    }
}
template <class T, int PARTS>
__global__ __launch_bounds__(kJoinThreads) void attention_grad_join_kernel(Args g)
{
    if (blockIdx.y) {
        if (g.dkv_parts) join_parts<T, PARTS, true>(g);
    } else {
        if (g.dq_parts) join_parts<T, PARTS, false>(g);
    }
}

// ---- host ----
constexpr int kComputeUnits = 256;
struct Plan {
    bool few_rows, few_keys;
    int row_tiles, key_tiles, row_splits, row_chunk, key_splits, key_chunk;
    size_t stat, dq, dkv, bytes;     // bytes of z (and of delta), of the parts, of all
};
constexpr size_t padded(size_t n) { return (n + kAlign - 1) / kAlign * kAlign; }

// Splits of `many` into chunks, so that there is a workgroup a compute unit, but chunks of at least `least`: 512 of bf16 (4096 queries of 4
// heads to 64 keys: 35 us, 53 with 128, 67 unsplit; 1 x 512 x 4 x 64 causal 26.4 and 29.0), 128 of fp32, whose products take five times as
// long (the latter 37.7, 53 with 512, 68 unsplit).
void split(int64_t groups, int64_t many, int64_t least, int& splits, int& chunk)
{
    const int64_t step = kChunk;
    const int64_t n = std::max<int64_t>(1, std::min<int64_t>(kComputeUnits / std::max<int64_t>(1, groups), (many + least - 1) / least));
    chunk = (int)std::max<int64_t>(step, ((many + n - 1) / n + step - 1) / step * step);
    splits = (int)std::max<int64_t>(1, (many + chunk - 1) / chunk);
}
Plan plan_of(int B, int Tq, int Tk, int Hq, int Hk, int D, int is_bf16)
{
    Plan p{};
    const int64_t rows = (int64_t)Tq * (Hq / Hk), units = (int64_t)B * Hk;
    const size_t cols = (size_t)parts_of(D) * kPart;
    // Few where 128 a workgroup would leave compute units without one (8 causal heads, us of few and of many: 128 columns bf16, 1024 tokens 48
    // and 66, 2048 91 and 96, 4096, 256 workgroups, 241 and 223; fp32, 2048 tokens, 254 and 338; 64 columns bf16, 2048 tokens, 53 and 61).
    auto tiles = [&](int64_t many, int each, bool& few) {
        few = units * ((many + each - 1) / each) < kComputeUnits;
        const int mine = few ? Few<float>::MINE : each;
        return (int)((many + mine - 1) / mine);
    };
    p.row_tiles = tiles(rows, RowsMany<float>::MINE, p.few_rows);
    p.key_tiles = tiles(Tk, !is_bf16 && parts_of(D) > 2 ? KeysMany<float, 4>::MINE : KeysMany<uint16_t, 4>::MINE, p.few_keys);
    const int64_t least = is_bf16 ? 512 : 128;
    split(units * p.row_tiles, Tk, least, p.row_splits, p.row_chunk);
    split(units * p.key_tiles, rows, least, p.key_splits, p.key_chunk);
    p.stat = padded(sizeof(float) * (size_t)(units * rows));
    p.dq = p.row_splits > 1 ? padded(sizeof(float) * (size_t)(units * rows * p.row_splits) * cols) : 0;
    p.dkv = p.key_splits > 1 ? padded(sizeof(float) * (size_t)(units * Tk * p.key_splits * 2) * cols) : 0;
    p.bytes = std::max(kAlign, 2 * p.stat + p.dq + p.dkv);
    return p;
}

template <class T, int PARTS, bool ALIGNED>
void launch_rows(const Args& g, bool few, hipStream_t s)
{
    const dim3 grid((unsigned)workgroups(g, (int64_t)g.row_tiles * g.row_splits));
    if (few) hipLaunchKernelGGL((attention_dq_kernel<Few<T>, T, PARTS, ALIGNED>), grid, dim3(Few<T>::THREADS), 0, s, g);
    else hipLaunchKernelGGL((attention_dq_kernel<RowsMany<T>, T, PARTS, ALIGNED>), grid, dim3(RowsMany<T>::THREADS), 0, s, g);
}
template <class T, int PARTS, bool ALIGNED>
void launch_keys(const Args& g, bool few, hipStream_t s)
{
    const dim3 grid((unsigned)workgroups(g, (int64_t)g.key_tiles * g.key_splits));
    if (few) hipLaunchKernelGGL((attention_dkv_kernel<Few<T>, T, PARTS, ALIGNED>), grid, dim3(Few<T>::THREADS), 0, s, g);
    else hipLaunchKernelGGL((attention_dkv_kernel<KeysMany<T, PARTS>, T, PARTS, ALIGNED>), grid, dim3(KeysMany<T, PARTS>::THREADS), 0, s, g);
}
template <class T, int PARTS>
void launch(const Args& g, const Plan& p, bool aligned_rows, bool aligned_keys, hipStream_t s)
{
    if (g.rows) {
        if (aligned_keys) launch_rows<T, PARTS, true>(g, p.few_rows, s);
        else launch_rows<T, PARTS, false>(g, p.few_rows, s);
    }
    if (g.Tk) {
        if (aligned_rows) launch_keys<T, PARTS, true>(g, p.few_keys, s);
        else launch_keys<T, PARTS, false>(g, p.few_keys, s);
    }
    if (g.dq_parts || g.dkv_parts) {
        const int64_t many = std::max<int64_t>(g.dq_parts ? g.rows : 0, g.dkv_parts ? g.Tk : 0);
        const dim3 grid((unsigned)((g.units * many * PARTS * kPart + kJoinThreads - 1) / kJoinThreads), 2);
        hipLaunchKernelGGL((attention_grad_join_kernel<T, PARTS>), grid, dim3(kJoinThreads), 0, s, g);
    }
}

// Launches of fewer than 2^32 threads.
bool fits(const Plan& p, int64_t B, int64_t Tk, int64_t rows, int64_t Hk, int D)
{
    const double units = (double)(B * Hk + 7) * 1.2 * 512;
    return units * p.row_tiles * p.row_splits < 4294967296.0 && units * p.key_tiles * p.key_splits < 4294967296.0 &&
           (double)(B * Hk) * (double)std::max(p.row_splits > 1 ? rows : 0, p.key_splits > 1 ? Tk : 0) * (parts_of(D) * kPart) < 4294967040.0;
}

} // namespace
} // namespace attention
} // namespace lsgd

using namespace lsgd;
using namespace lsgd::attention;

extern "C" {

size_t lsgd_attention_grad_workspace_bytes(int32_t B, int32_t Tq, int32_t Tk, int32_t Hq, int32_t Hk, int32_t D, int32_t is_bf16)
{
    if (check_attention_shape("attention_grad", B, Tq, Tk, Hq, Hk, D) != LSGD_OK) return 0;
    return plan_of(B, Tq, Tk, Hq, Hk, D, is_bf16).bytes;
}

lsgd_status lsgd_attention_grad(const lsgd_attention_grad_args* p, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    const char* who = "attention_grad";
    if (!p) return set_error(LSGD_ERR_INVALID_ARG, "%s: arguments are NULL", who);
    const int B = p->B, Tq = p->Tq, Tk = p->Tk, Hq = p->Hq, Hk = p->Hk, D = p->D, es = p->is_bf16 ? 2 : 4;
    LSGD_TRY(check_attention_shape(who, B, Tq, Tk, Hq, Hk, D));
    if (p->is_bf16 & ~1 || p->causal & ~1) return set_error(LSGD_ERR_INVALID_ARG, "%s: is_bf16 and causal must be 0 or 1", who);
    if (!scale_ok(p->scale)) return set_error(LSGD_ERR_INVALID_ARG, "%s: scale must be within [1e-30, 1e30]", who);
    if (Tq == 0 && Tk == 0) return LSGD_OK;
    if ((int64_t)B * Hk > INT64_C(1) << 30) return set_error(LSGD_ERR_SHAPE, "%s: B=%d, Hk=%d are too large for one launch", who, B, Hk);
    const Plan plan = plan_of(B, Tq, Tk, Hq, Hk, D, p->is_bf16);
    if ( !fits(plan, B, Tk, (int64_t)Tq * (Hq / Hk), Hk, D)) return set_error(LSGD_ERR_SHAPE, "%s: B=%d, Tq=%d, Tk=%d, Hk=%d are too large for one launch", who, B, Tq, Tk, Hk);
    const bool q = Tq > 0, k = Tk > 0;
    LSGD_TRY(check_heads(who, "dout", p->dout, B, Tq, Hq, D, es, q || p->dout.data, false));
    LSGD_TRY(check_heads(who, "q", p->q, B, Tq, Hq, D, es, q || p->q.data, false));
    LSGD_TRY(check_heads(who, "k", p->k, B, Tk, Hk, D, es, k || p->k.data, false));
    LSGD_TRY(check_heads(who, "v", p->v, B, Tk, Hk, D, es, k || p->v.data, false));
    LSGD_TRY(check_heads(who, "out", p->out, B, Tq, Hq, D, es, q || p->out.data, false));
    LSGD_TRY(check_heads(who, "dq", p->dq, B, Tq, Hq, D, es, q || p->dq.data, true));
    LSGD_TRY(check_heads(who, "dk", p->dk, B, Tk, Hk, D, es, k || p->dk.data, true));
    LSGD_TRY(check_heads(who, "dv", p->dv, B, Tk, Hk, D, es, k || p->dv.data, true));
    if (q && !p->lse) return set_error(LSGD_ERR_INVALID_ARG, "%s: lse is required", who);
    if (!on(p->q_lens, 4) || !on(p->k_lens, 4) || !on(p->lse, 4)) return set_error(LSGD_ERR_INVALID_ARG, "%s: q_lens, k_lens or lse is not aligned to its element", who);
    if (!workspace) return set_error(LSGD_ERR_INVALID_ARG, "%s: workspace is NULL", who);
    if (!on(workspace, kAlign)) return set_error(LSGD_ERR_INVALID_ARG, "%s: workspace must be 256-byte aligned", who);
    if (workspace_bytes < plan.bytes) return set_error(LSGD_ERR_NOMEM, "%s: workspace of %zu bytes < %zu needed", who, workspace_bytes, plan.bytes);
    Args g{};
    set_shape(g, *p);
    g.dout = heads(p->dout); g.q = heads(p->q); g.k = heads(p->k); g.v = heads(p->v); g.out = heads(p->out);
    g.dq = heads(p->dq); g.dk = heads(p->dk); g.dv = heads(p->dv);
    g.lse = p->lse;
    char* w = static_cast<char*>(workspace);
    g.z = reinterpret_cast<float*>(w);
    g.delta = reinterpret_cast<float*>(w + plan.stat);
    g.dq_parts = plan.dq ? reinterpret_cast<float*>(w + 2 * plan.stat) : nullptr;
    g.dkv_parts = plan.dkv ? reinterpret_cast<float*>(w + 2 * plan.stat + plan.dq) : nullptr;
    g.row_tiles = plan.row_tiles; g.key_tiles = plan.key_tiles;
    g.row_splits = plan.row_splits; g.row_chunk = plan.row_chunk;
    g.key_splits = plan.key_splits; g.key_chunk = plan.key_chunk;
    g.scale = p->scale; g.inv_scale = 1.0f / p->scale; g.c = p->scale * kLog2e;
    // what is read by 16 bytes straight to LDS has to lie on them
    const bool whole = D % (16 / es) == 0;
    const bool aligned_rows = whole && wide_heads(p->q, B, Tq, Hq, es) && wide_heads(p->dout, B, Tq, Hq, es);
    const bool aligned_keys = whole && wide_heads(p->k, B, Tk, Hk, es) && wide_heads(p->v, B, Tk, Hk, es);
    by_type_and_parts(p->is_bf16, parts_of(D), [&](auto type, auto parts) {
        launch<decltype(type), decltype(parts)::value>(g, plan, aligned_rows, aligned_keys, static_cast<hipStream_t>(hip_stream));
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return set_error(LSGD_ERR_HIP, "%s: %s", who, hipGetErrorString(e));
    return LSGD_OK;
}

} // extern "C"
