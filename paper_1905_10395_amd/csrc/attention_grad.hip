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
#include <algorithm>
#include <cmath>

#include "attention_common.h"

namespace lsgd {
namespace attention {
namespace {

struct Args : Shape {
    Heads dout, q, k, v, out, dq, dk, dv;
    const float* lse;                // [B][Hq][Tq]
    float *z, *delta;                // [units][row_tiles 128]: -z / c (fp32: -z), -inf for rows that see nothing, and -delta
    float *dq_parts, *dkv_parts;     // of splits, NULL: one
    int row_tiles, key_tiles;
    int row_splits, row_chunk;       // by rows: workgroups a tile, and the keys of one
    int key_splits, key_chunk;       // by keys: workgroups a tile, and the rows of one
    float scale, inv_scale, c;
};

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kMine = 32 * kWaves;                       // rows, or keys, that a workgroup owns
template <class T>
constexpr int kPass = sizeof(T) == 2 ? 64 : 32;          // keys, or rows, of the tiles that pass
template <class T>
constexpr bool kFromZ = sizeof(T) == 2;                  // s begins with -z / c

__device__ __forceinline__ float dot(const Frag<uint16_t>& a, const Frag<uint16_t>& b)
{
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s += (float)a.v[e] * (float)b.v[e];
    return s;
}
__device__ __forceinline__ float dot(const Frag<float>& a, const Frag<float>& b)
{
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) s += a.lo[e] * b.lo[e] + a.hi[e] * b.hi[e];
    return s;
}
// c += the product of 32 rows of a tile, from row r0 on, with an operand in registers.
template <class T, int PARTS>
__device__ __forceinline__ void rows_times(const T* tile, int rows, int r0, int lane, const Frag<T> (&b)[2 * PARTS], f32x16& c)
{
#pragma unroll
    for (int k = 0; k < 2 * PARTS; ++k) {
        Frag<T> f;
        read_row(tile, rows, r0 + (lane & 31), lane >> 5, k, f);
        multiply(c, f, b[k]);
    }
}
// sums += the columns of 32 rows of a tile times a result.
template <class T, int PARTS>
__device__ __forceinline__ void columns_times(const T* tile, int rows, int r0, int lane, const f32x16& r, f32x16 (&sums)[PARTS])
{
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        Frag<T> b;
        from_result(r, k, b);
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            Frag<T> f;
            read_column(tile, rows, r0 + 16 * k, lane, p, f);
            multiply(sums[p], f, b);
        }
    }
}
template <int PARTS>
__device__ __forceinline__ void clear_sums(f32x16 (&s)[PARTS])
{
#pragma unroll
    for (int p = 0; p < PARTS; ++p)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[p][i] = 0.0f;
}
// The lane's columns of its row, times a factor, in the tensor's type or, for a part, fp32.
template <class T, int PARTS>
__device__ __forceinline__ void store_sums(T* row, int lane, int D, float factor, const f32x16 (&s)[PARTS])
{
#pragma unroll
    for (int p = 0; p < PARTS; ++p)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const float o[4] = {s[p][i] * factor, s[p][i + 1] * factor, s[p][i + 2] * factor, s[p][i + 3] * factor};
            store4(row, p * kPart + 2 * i + 4 * (lane >> 5), D, o);
        }
}

template <class T, int PARTS, bool ALIGNED>
__global__ __launch_bounds__(kThreads, 2) void attention_dq_kernel(Args g)
{
    constexpr int KEYS = kPass<T>, N = tile_elements<T>(KEYS, PARTS);
    __shared__ __attribute__((aligned(16))) T k0[N], k1[N];
    __shared__ __attribute__((aligned(16))) T v0[N], v1[N];
    const int lane = threadIdx.x & 63, h = lane >> 5, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Place at = place_of(g, g.row_tiles * g.row_splits);
    if (at.unit >= g.units) return;
    const int split = at.at % g.row_splits, tile = g.row_tiles - 1 - at.at / g.row_splits;   // late rows see most keys: first
    const Rows rows = rows_of(g, at.unit, tile * kMine, kMine);
    const int r = tile * kMine + wid * 32 + (lane & 31);
    const Row row = row_of(g, rows, r);
    const int least = wave_min(row.sees), most = wave_max(row.sees);
    Frag<T> qf[2 * PARTS], df[2 * PARTS];
    float z = -INFINITY, delta = 0.0f;                                     // negative, as the accumulators begin
    {
        const T* q = static_cast<const T*>(g.q.p) + rows.b * g.q.lb + row.t * g.q.lt + row.head * g.q.lh;
        const T* d = static_cast<const T*>(g.dout.p) + rows.b * g.dout.lb + row.t * g.dout.lt + row.head * g.dout.lh;
        const T* o = static_cast<const T*>(g.out.p) + rows.b * g.out.lb + row.t * g.out.lt + row.head * g.out.lh;
        Frag<T> of[2 * PARTS];
        if (row.sees == 0) {
            clear_frags<T, PARTS>(qf);
            clear_frags<T, PARTS>(df);
        } else {
            load_frags<T, PARTS>(q, h, g.D, qf);
            load_frags<T, PARTS>(d, h, g.D, df);
            load_frags<T, PARTS>(o, h, g.D, of);
#pragma unroll
            for (int k = 0; k < 2 * PARTS; ++k) delta -= dot(of[k], df[k]);
            z = -g.lse[((int64_t)rows.b * g.Hq + row.head) * g.Tq + row.t] * (kFromZ<T> ? g.inv_scale : kLog2e);
        }
        delta += other_half(delta);
        if (split == 0 && h == 0) {
            const int64_t to = (int64_t)at.unit * g.row_tiles * kMine + r;
            g.z[to] = row.there ? z : -INFINITY;
            g.delta[to] = row.there ? delta : 0.0f;
        }
    }
    f32x16 dq[PARTS];
    clear_sums<PARTS>(dq);
    const T* k = static_cast<const T*>(g.k.p) + rows.b * g.k.lb + rows.hk * g.k.lh;
    const T* v = static_cast<const T*>(g.v.p) + rows.b * g.v.lb + rows.hk * g.v.lh;
    const int begin = split * g.row_chunk, end = min(rows.end, begin + g.row_chunk);
    auto issue = [&](int key0, T* kb, T* vb) {
        auto key = [&](int i) { return key0 + i < rows.nk ? key0 + i : rows.nk - 1; };
        load_tile<T, KEYS, PARTS, kWaves, ALIGNED>(kb, wid, lane, g.D, [&](int i) { return k + key(i) * g.k.lt; });
        load_tile<T, KEYS, PARTS, kWaves, ALIGNED>(vb, wid, lane, g.D, [&](int i) { return v + key(i) * g.v.lt; });
    };
    auto step = [&](int key0, T* kb, T* vb, T* next_k, T* next_v) {
        tiles_barrier();
        if (key0 + KEYS < end) issue(key0 + KEYS, next_k, next_v);
        if (key0 >= most) return;
        const bool masked = key0 + KEYS > least;
#pragma unroll
        for (int n = 0; n < KEYS / 32; ++n) {
            f32x16 s, dp;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[i] = kFromZ<T> ? z : 0.0f;
                dp[i] = delta;
            }
            rows_times<T, PARTS>(kb, KEYS, 32 * n, lane, qf, s);
            rows_times<T, PARTS>(vb, KEYS, 32 * n, lane, df, dp);
#pragma unroll
            for (int i = 0; i < 16; ++i) dp[i] *= __builtin_amdgcn_exp2f(kFromZ<T> ? s[i] * g.c : fmaf(s[i], g.c, z));
            if (masked) {
#pragma unroll
                for (int i = 0; i < 16; ++i) dp[i] = key0 + 32 * n + 8 * (i >> 2) + 4 * h + (i & 3) < row.sees ? dp[i] : 0.0f;
            }
            columns_times<T, PARTS>(kb, KEYS, 32 * n, lane, dp, dq);
        }
    };
    if (begin < end) issue(begin, k0, v0);
    for (int key0 = begin; key0 < end; key0 += 2 * KEYS) {
        step(key0, k0, v0, k1, v1);
        if (key0 + KEYS < end) step(key0 + KEYS, k1, v1, k0, v0);
    }
    if (!row.there) return;
    if (g.dq_parts)
        store_sums<float, PARTS>(g.dq_parts + ((((int64_t)at.unit * g.row_tiles + tile) * g.row_splits + split) * kMine + r - tile * kMine) * (PARTS * kPart),
                                 lane, PARTS * kPart, g.scale, dq);
    else
        store_sums<T, PARTS>(static_cast<T*>(g.dq.p) + rows.b * g.dq.lb + row.t * g.dq.lt + row.head * g.dq.lh, lane, g.D, g.scale, dq);
}

// The first row that sees a key.
__device__ __forceinline__ int first_row(const Args& g, int nq, int nk, int key)
{
    const int t = key - (nk - nq);
    return g.causal && t > 0 ? (t < nq ? t : nq) * g.G : 0;
}

template <class T, int PARTS, bool ALIGNED>
__global__ __launch_bounds__(kThreads, 2) void attention_dkv_kernel(Args g)
{
    constexpr int ROWS = kPass<T>, N = tile_elements<T>(ROWS, PARTS);
    __shared__ __attribute__((aligned(16))) T q0[N], q1[N];
    __shared__ __attribute__((aligned(16))) T d0[N], d1[N];
    __shared__ __attribute__((aligned(16))) float z0[ROWS], z1[ROWS], e0[ROWS], e1[ROWS];
    const int lane = threadIdx.x & 63, h = lane >> 5, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Place at = place_of(g, g.key_tiles * g.key_splits);
    if (at.unit >= g.units) return;
    const int split = at.at % g.key_splits, tile = at.at / g.key_splits;
    const int b = at.unit / g.Hk, hk = at.unit % g.Hk;
    const int nq = length_of(g.q_lens, b, g.Tq), nk = length_of(g.k_lens, b, g.Tk);
    const int key0 = tile * kMine, key = key0 + wid * 32 + (lane & 31);
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
    const int from = live ? first_row(g, nq, nk, key) : 0, least = first_row(g, nq, nk, key0 + wid * 32), most = wave_max(from);
    const int rows_live = nq * g.G;
    int begin = first_row(g, nq, nk, key0) / ROWS * ROWS, end = key0 < nk ? rows_live : 0;
    begin = max(begin, split * g.key_chunk);
    end = min(end, (split + 1) * g.key_chunk);
    f32x16 dk[PARTS], dv[PARTS];
    clear_sums<PARTS>(dk);
    clear_sums<PARTS>(dv);
    const T* q = static_cast<const T*>(g.q.p) + b * g.q.lb + (int64_t)hk * g.G * g.q.lh;
    const T* d = static_cast<const T*>(g.dout.p) + b * g.dout.lb + (int64_t)hk * g.G * g.dout.lh;
    const float* z = g.z + (int64_t)at.unit * g.row_tiles * kMine;
    const float* delta = g.delta + (int64_t)at.unit * g.row_tiles * kMine;
    auto issue = [&](int r0, T* qb, T* db, float* zb, float* eb) {
        auto place = [&](int i, const Heads& a) {
            const int r = r0 + i < rows_live ? r0 + i : rows_live - 1, t = over(r, g.by_g);
            return t * a.lt + (r - t * g.G) * a.lh;
        };
        load_tile<T, ROWS, PARTS, kWaves, ALIGNED>(qb, wid, lane, g.D, [&](int i) { return q + place(i, g.q); });
        load_tile<T, ROWS, PARTS, kWaves, ALIGNED>(db, wid, lane, g.D, [&](int i) { return d + place(i, g.dout); });
        // (z and delta have whole tiles of rows)
        if (lane < ROWS && wid == 0) zb[lane] = z[r0 + lane];
        if (lane < ROWS && wid == 1) eb[lane] = delta[r0 + lane];
    };
    auto step = [&](int r0, T* qb, T* db, float* zb, float* eb, T* next_q, T* next_d, float* next_z, float* next_e) {
        tiles_barrier();
        if (r0 + ROWS < end) issue(r0 + ROWS, next_q, next_d, next_z, next_e);
        if (r0 + ROWS <= least) return;
        const bool masked = r0 < most;
#pragma unroll 1
        for (int n = 0; n < ROWS / 32; ++n) {
            f32x16 s, dp;
            auto begin_with = [&](const float* first, f32x16& c) {
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const v4f x = *reinterpret_cast<const v4f*>(first + 32 * n + 2 * i + 4 * h);
#pragma unroll
                    for (int e = 0; e < 4; ++e) c[i + e] = x[e];
                }
            };
            if constexpr (kFromZ<T>) {
                begin_with(zb, s);
                rows_times<T, PARTS>(qb, ROWS, 32 * n, lane, kf, s);
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(s[i] * g.c);
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = 0.0f;
                rows_times<T, PARTS>(qb, ROWS, 32 * n, lane, kf, s);
                begin_with(zb, dp);
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], g.c, dp[i]));
            }
            if (masked) {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = r0 + 32 * n + 8 * (i >> 2) + 4 * h + (i & 3) >= from ? s[i] : 0.0f;
            }
            columns_times<T, PARTS>(db, ROWS, 32 * n, lane, s, dv);
            begin_with(eb, dp);
            rows_times<T, PARTS>(db, ROWS, 32 * n, lane, vf, dp);
#pragma unroll
            for (int i = 0; i < 16; ++i) dp[i] *= s[i];
            columns_times<T, PARTS>(qb, ROWS, 32 * n, lane, dp, dk);
        }
    };
    if (begin < end) issue(begin, q0, d0, z0, e0);
    for (int r0 = begin; r0 < end; r0 += 2 * ROWS) {
        step(r0, q0, d0, z0, e0, q1, d1, z1, e1);
        if (r0 + ROWS < end) step(r0 + ROWS, q1, d1, z1, e1, q0, d0, z0, e0);
    }
    if (key >= g.Tk) return;
    if (!live) {
        clear_sums<PARTS>(dk);
        clear_sums<PARTS>(dv);
    }
    if (g.dkv_parts) {
        float* part = g.dkv_parts + ((((int64_t)at.unit * g.key_tiles + tile) * g.key_splits + split) * 2 * kMine + key - key0) * (PARTS * kPart);
        store_sums<float, PARTS>(part, lane, PARTS * kPart, g.scale, dk);
        store_sums<float, PARTS>(part + kMine * PARTS * kPart, lane, PARTS * kPart, 1.0f, dv);
    } else {
        store_sums<T, PARTS>(static_cast<T*>(g.dk.p) + b * g.dk.lb + key * g.dk.lt + hk * g.dk.lh, lane, g.D, g.scale, dk);
        store_sums<T, PARTS>(static_cast<T*>(g.dv.p) + b * g.dv.lb + key * g.dv.lt + hk * g.dv.lh, lane, g.D, 1.0f, dv);
    }
}

// The sums of the splits' parts, in order.  KV: of dk and dv, else of dq.
template <class T, int PARTS, bool KV>
__global__ __launch_bounds__(kThreads) void attention_grad_join_kernel(Args g)
{
    constexpr int COLS = PARTS * kPart, LISTS = KV ? 2 : 1;
    const int tiles = KV ? g.key_tiles : g.row_tiles, splits = KV ? g.key_splits : g.row_splits, many = KV ? g.Tk : g.rows;
    const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x, row = id / COLS;
    const int c = (int)(id % COLS), unit = (int)(row / many), r = (int)(row % many);
    if (unit >= g.units || c >= g.D) return;
    const float* p = (KV ? g.dkv_parts : g.dq_parts) + (((int64_t)unit * tiles + r / kMine) * splits * LISTS * kMine + r % kMine) * COLS + c;
    const int b = unit / g.Hk, hk = unit % g.Hk;
#pragma unroll
    for (int list = 0; list < LISTS; ++list) {
        float s = 0.0f;
        for (int k = 0; k < splits; ++k) s += p[((int64_t)k * LISTS + list) * kMine * COLS];
        const Heads& a = KV ? (list ? g.dv : g.dk) : g.dq;
        const int t = KV ? r : over(r, g.by_g), head = KV ? hk : hk * g.G + r - t * g.G;
        put1(static_cast<T*>(a.p) + b * a.lb + t * a.lt + head * a.lh + c, s);
    }
}

// ---- host ----
constexpr int kComputeUnits = 256;
struct Plan {
    int row_tiles, key_tiles, row_splits, row_chunk, key_splits, key_chunk;
    size_t stat, dq, dkv, bytes;     // bytes of z (and of delta), of the parts, of all
};
constexpr size_t padded(size_t n) { return (n + kAlign - 1) / kAlign * kAlign; }

// Splits of `many` into chunks, so that there are two workgroups a compute unit, but chunks of at least 512.
void split(int64_t groups, int64_t many, int& splits, int& chunk)
{
    const int64_t least = 512, step = 128;
    const int64_t n = std::max<int64_t>(1, std::min<int64_t>(2 * kComputeUnits / std::max<int64_t>(1, groups), (many + least - 1) / least));
    chunk = (int)std::max<int64_t>(step, ((many + n - 1) / n + step - 1) / step * step);
    splits = (int)std::max<int64_t>(1, (many + chunk - 1) / chunk);
}
Plan plan_of(int B, int Tq, int Tk, int Hq, int Hk, int D)
{
    Plan p{};
    const int64_t rows = (int64_t)Tq * (Hq / Hk), units = (int64_t)B * Hk;
    const size_t cols = (size_t)parts_of(D) * kPart;
    p.row_tiles = (int)((rows + kMine - 1) / kMine);
    p.key_tiles = (Tk + kMine - 1) / kMine;
    split(units * p.row_tiles, Tk, p.row_splits, p.row_chunk);
    split(units * p.key_tiles, rows, p.key_splits, p.key_chunk);
    p.stat = padded(sizeof(float) * (size_t)units * p.row_tiles * kMine);
    p.dq = p.row_splits > 1 ? padded(sizeof(float) * (size_t)units * p.row_tiles * p.row_splits * kMine * cols) : 0;
    p.dkv = p.key_splits > 1 ? padded(sizeof(float) * (size_t)units * p.key_tiles * p.key_splits * 2 * kMine * cols) : 0;
    p.bytes = std::max(kAlign, 2 * p.stat + p.dq + p.dkv);
    return p;
}

template <class T, int PARTS>
void launch(const Args& g, bool aligned_rows, bool aligned_keys, hipStream_t s)
{
    const dim3 threads(kThreads);
    if (g.rows) {
        const dim3 grid((unsigned)workgroups(g, (int64_t)g.row_tiles * g.row_splits));
        if (aligned_keys) hipLaunchKernelGGL((attention_dq_kernel<T, PARTS, true>), grid, threads, 0, s, g);
        else hipLaunchKernelGGL((attention_dq_kernel<T, PARTS, false>), grid, threads, 0, s, g);
        if (g.row_splits > 1)
            hipLaunchKernelGGL((attention_grad_join_kernel<T, PARTS, false>), dim3((unsigned)(((int64_t)g.units * g.rows * PARTS * kPart + kThreads - 1) / kThreads)),
                               threads, 0, s, g);
    }
    if (g.Tk) {
        const dim3 grid((unsigned)workgroups(g, (int64_t)g.key_tiles * g.key_splits));
        if (aligned_rows) hipLaunchKernelGGL((attention_dkv_kernel<T, PARTS, true>), grid, threads, 0, s, g);
        else hipLaunchKernelGGL((attention_dkv_kernel<T, PARTS, false>), grid, threads, 0, s, g);
        if (g.key_splits > 1)
            hipLaunchKernelGGL((attention_grad_join_kernel<T, PARTS, true>), dim3((unsigned)(((int64_t)g.units * g.Tk * PARTS * kPart + kThreads - 1) / kThreads)),
                               threads, 0, s, g);
    }
}

// Launches of fewer than 2^32 threads.
bool fits(const Plan& p, int64_t B, int64_t Tk, int64_t rows, int64_t Hk, int D)
{
    const double units = (double)(B * Hk + 7) * 1.2 * kThreads;
    return units * p.row_tiles * p.row_splits < 4294967296.0 && units * p.key_tiles * p.key_splits < 4294967296.0 &&
           (double)(B * Hk) * (double)std::max(rows, Tk) * (parts_of(D) * kPart) < 4294967040.0;
}

} // namespace
} // namespace attention
} // namespace lsgd

using namespace lsgd;
using namespace lsgd::attention;

extern "C" {

size_t lsgd_attention_grad_workspace_bytes(int32_t B, int32_t Tq, int32_t Tk, int32_t Hq, int32_t Hk, int32_t D, int32_t is_bf16)
{
    (void)is_bf16;
    if (check_attention_shape("attention_grad", B, Tq, Tk, Hq, Hk, D) != LSGD_OK) return 0;
    return plan_of(B, Tq, Tk, Hq, Hk, D).bytes;
}

lsgd_status lsgd_attention_grad(const lsgd_attention_grad_args* p, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    const char* who = "attention_grad";
    if (!p) return set_error(LSGD_ERR_INVALID_ARG, "%s: arguments are NULL", who);
    const int B = p->B, Tq = p->Tq, Tk = p->Tk, Hq = p->Hq, Hk = p->Hk, D = p->D, es = p->is_bf16 ? 2 : 4;
    LSGD_TRY(check_attention_shape(who, B, Tq, Tk, Hq, Hk, D));
    if (p->is_bf16 & ~1 || p->causal & ~1) return set_error(LSGD_ERR_INVALID_ARG, "%s: is_bf16 and causal must be 0 or 1", who);
    if (!std::isfinite(p->scale) || p->scale <= 0.0f) return set_error(LSGD_ERR_INVALID_ARG, "%s: scale must be finite and positive", who);
    if (Tq == 0 && Tk == 0) return LSGD_OK;
    const Plan plan = plan_of(B, Tq, Tk, Hq, Hk, D);
    if ((int64_t)B * Hk > INT64_C(1) << 30 || !fits(plan, B, Tk, (int64_t)Tq * (Hq / Hk), Hk, D)) return set_error(LSGD_ERR_SHAPE, "%s: B=%d, Tq=%d, Tk=%d, Hk=%d are too large for one launch", who, B, Tq, Tk, Hk);
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
        launch<decltype(type), decltype(parts)::value>(g, aligned_rows, aligned_keys, static_cast<hipStream_t>(hip_stream));
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return set_error(LSGD_ERR_HIP, "%s: %s", who, hipGetErrorString(e));
    return LSGD_OK;
}

} // extern "C"
