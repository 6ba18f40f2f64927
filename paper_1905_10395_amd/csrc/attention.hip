// Attention forward: softmax(scale q k') v of the keys that each query sees.
//
//   s = q . k,  c = scale log2 e,  p = 2^(c (s - m)),  l = sum p,  out = (sum p v) / l,  lse = scale m + log l
//
// A row that sees nothing has zeros by its mask, not by its sums: those may hold 0 x infinity from keys that rows beside it see.  A row
// with NaN among its scores has l = NaN, and so its results; one whose scores are all -inf has l = 0, and 0 / 0.
//
// One pass over the keys.  m is a running reference of the scores, not always their maximum: sums are rescaled only when a score
// exceeds it by 8 or more powers of two, so most tiles need no rescaling, and p stays below 2^8.  s^T = K Q^T and out^T = V^T P^T:
// a lane's result column is one query, so its maximum and sum need one exchange between two lanes, and p goes from result to operand
// without leaving the registers (attention_common.h).
//
// Two kernels.  By rows: a workgroup takes 128 rows (query, head of the key head's), 32 a wavefront, and all pass over the keys
// together; K and V tiles are read by all four from LDS, the next ones are on their way meanwhile.  By keys: where there are few rows,
// a workgroup takes 32 of them, and its wavefronts and further workgroups split the keys; each wavefront has tiles of its own and waits
// for nobody, and the parts are joined at the end.
//
// By rows is bound by the products (2 x 8192 causal tokens of 32 and 8 heads of 128 bf16 1.02 to 1.11 ms, 0.99 to 1.08 PFLOP/s where a large
// product alone reaches 1.22), short rows by loading, computing and storing one after the other (64 x 512 of 16 heads of 64 with lengths of
// all kinds 52 to 57 us: its bytes take 31, its exponentials and products some 20); fp32 by splitting operands beside the products, and of 97
// to 128 columns by registers that do not suffice, 108 to 124 bytes of scratch a lane (4 x 2048 causal tokens of 16 and 4 heads of 128 472 us, 146
// TFLOP/s, of 16 heads of 64 249, 138); a single query to a cache by memory (32 entries of up to 16384 keys, 8 heads of 128, 205 to 225 us, 4.9
// to 5.4 TB/s).
#include <algorithm>
#include <cmath>

#include "attention_common.h"

namespace lsgd {
namespace attention {
namespace {

struct Args : Shape {
    Heads q, k, v, out;
    float* lse;                      // [B][Hq][Tq], or NULL
    float* parts;                    // by keys: parts of splits, NULL: one split
    int tiles;                       // of rows
    int splits, chunk;               // by keys: workgroups a tile of rows, and the keys of one
    float scale, c;                  // c: scale log2 e
    int wide_out;                    // rows of out are whole 16-byte pieces
};

// What a wavefront holds of 32 rows: their sums so far, relative to m.
template <int PARTS>
struct State {
    f32x16 o[PARTS];
    float m, l;                      // l: of this lane's keys
    __device__ __forceinline__ State() : m(-INFINITY), l(0.0f)
    {
#pragma unroll
        for (int p = 0; p < PARTS; ++p)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[p][i] = 0.0f;
    }
};

constexpr float kSlack = 8.0f;       // powers of two

// How far operands are read ahead; fp32's parts take the registers.  (Two of bf16 or four of fp32 are as fast here: 64 x 512 x 16 x 64 57.4 and
// 57.1 us; the gradients gain from four, see there.)
template <class T>
constexpr int kAhead = sizeof(T) == 2 ? 4 : 2;

// KEYS keys of a tile: their p of the lane's row, and the state's reference moved if need be.  masked: some row does not see some of
// them.  then() is called when the products are on their way.
template <int WIDTH, class T, int PARTS, int KEYS, class F>
__device__ __forceinline__ void pass_keys(const T* kt, int lane, int key0, int sees, bool masked, float c, const Frag<T> (&qf)[2 * PARTS], State<PARTS>& st,
                                          f32x16 (&s)[KEYS / 32], F then)
{
    constexpr int NS = KEYS / 32;
    const int h = lane >> 5;
#pragma unroll
    for (int n = 0; n < NS; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[n][i] = 0.0f;
    Ahead<T, NS * 2 * PARTS, kAhead<T>> ops;
    auto read = [&](int i, Frag<T>& f) { read_row<WIDTH>(kt, KEYS, 32 * (i % NS) + (lane & 31), h, i / NS, f); };
    ops.start(read);
    ops.run(read, [&](int i, const Frag<T>& f) { multiply(s[i % NS], f, qf[i / NS]); });
    then();
    if (masked) {
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[n][i] = key0 + 32 * n + 8 * (i >> 2) + 4 * h + (i & 3) < sees ? s[n][i] : -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int n = 0; n < NS; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, s[n][i]);
    top = fmaxf(top, other_half(top));
    if (__any((top - st.m) * c > kSlack)) {
        const float m = fmaxf(st.m, top), a = m == st.m ? 1.0f : __builtin_amdgcn_exp2f((st.m - m) * c);
        st.m = m;
        st.l *= a;
#pragma unroll
        for (int p = 0; p < PARTS; ++p)
#pragma unroll
            for (int i = 0; i < 16; ++i) st.o[p][i] *= a;
    }
    const float mc = st.m == -INFINITY ? 0.0f : st.m * c;
#pragma unroll
    for (int n = 0; n < NS; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[n][i] = __builtin_amdgcn_exp2f(fmaf(s[n][i], c, -mc));
            st.l += s[n][i];
        }
}
// Their values, times p.
template <int WIDTH, class T, int PARTS, int KEYS>
struct Values {
    Ahead<T, KEYS / 16 * PARTS, kAhead<T>> ops;
    const T* vt;
    const int lane;
    __device__ __forceinline__ Values(const T* tile, int l) : vt(tile), lane(l) {}
    __device__ __forceinline__ void start()
    {
        ops.start([&](int i, Frag<T>& f) { read_column<WIDTH>(vt, KEYS, 16 * (i / PARTS), lane, i % PARTS, f); });
    }
    __device__ __forceinline__ void pass(const f32x16 (&s)[KEYS / 32], State<PARTS>& st)
    {
        Frag<T> p[KEYS / 16];
#pragma unroll
        for (int k = 0; k < KEYS / 16; ++k) from_result(s[k / 2], k % 2, p[k]);
        ops.run([&](int i, Frag<T>& f) { read_column<WIDTH>(vt, KEYS, 16 * (i / PARTS), lane, i % PARTS, f); },
                [&](int i, const Frag<T>& f) { multiply(st.o[i % PARTS], f, p[i / PARTS]); });
    }
};

template <class T, int PARTS>
__device__ __forceinline__ void load_queries(const Args& g, const Rows& rows, const Row& row, int h, Frag<T> (&qf)[2 * PARTS])
{
    const T* q = static_cast<const T*>(g.q.p) + rows.b * g.q.lb + row.t * g.q.lt + row.head * g.q.lh;
    if (row.sees) load_frags<T, PARTS>(q, h, g.D, qf);
    else clear_frags<T, PARTS>(qf);
}

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kRowsByRows = 32 * kWaves;
template <class T>
constexpr bool kLate = sizeof(T) == 2;                    // rows off 16 bytes wait in registers while a tile is passed (16 x 700 x 8 x 59 32 -> 29 us; fp32 83, late 88)
template <class T>
constexpr int kKeysByRows = sizeof(T) == 2 ? 64 : 32;     // 64 rows of 32 bf16 are a load of each wavefront; two buffers of K and V leave two workgroups a compute unit

template <class T, int PARTS, bool ALIGNED>
__global__ __launch_bounds__(kThreads, 2) void attention_rows_kernel(Args g)
{
    constexpr int KEYS = kKeysByRows<T>;
    // separate objects, so that the compiler sees that a read of one does not wait for loads into another
    __shared__ __attribute__((aligned(16))) T k0[tile_elements<T>(KEYS, PARTS)], k1[tile_elements<T>(KEYS, PARTS)];
    __shared__ __attribute__((aligned(16))) T v0[tile_elements<T>(KEYS, PARTS)], v1[tile_elements<T>(KEYS, PARTS)];
    const int lane = threadIdx.x & 63, h = lane >> 5, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Place at = place_of(g, g.tiles);
    const int unit = at.unit, tile = g.tiles - 1 - at.at;            // late rows see most keys: first
    if (unit >= g.units) return;
    const Rows rows = rows_of(g, unit, tile * kRowsByRows, kRowsByRows);
    const Row row = row_of(g, rows, tile * kRowsByRows + wid * 32 + (lane & 31));
    const int least = wave_min(row.sees), most = wave_max(row.sees);
    Frag<T> qf[2 * PARTS];
    load_queries<T, PARTS>(g, rows, row, h, qf);
    State<PARTS> st;
    const T* k = static_cast<const T*>(g.k.p) + rows.b * g.k.lb + rows.hk * g.k.lh;
    const T* v = static_cast<const T*>(g.v.p) + rows.b * g.v.lb + rows.hk * g.v.lh;
    TileOnItsWay<T, KEYS, PARTS, kWaves, ALIGNED> kt, vt;
    auto issue = [&](int key0, T* kb, T* vb) {
        auto key = [&](int r) { return key0 + r < rows.nk ? key0 + r : rows.nk - 1; };
        kt.fetch(kb, wid, lane, g.D, [&](int r) { return k + key(r) * g.k.lt; });
        vt.fetch(vb, wid, lane, g.D, [&](int r) { return v + key(r) * g.v.lt; });
    };
    auto put = [&](T* kb, T* vb) {
        kt.put(kb, wid, lane, g.D);
        vt.put(vb, wid, lane, g.D);
    };
    auto step = [&](int key0, T* kb, T* vb, T* next_k, T* next_v) {
        tiles_barrier();
        if (key0 + KEYS < rows.end) {
            issue(key0 + KEYS, next_k, next_v);
            if (!kLate<T>) put(next_k, next_v);
        }
        if (key0 < most) {
            f32x16 p[KEYS / 32];
            Values<kPart, T, PARTS, KEYS> values(vb, lane);
            pass_keys<kPart, T, PARTS, KEYS>(kb, lane, key0, row.sees, key0 + KEYS > least, g.c, qf, st, p, [&] { values.start(); });
            values.pass(p, st);
        }
        if (kLate<T> && key0 + KEYS < rows.end) put(next_k, next_v);
    };
    if (rows.end > 0) {
        issue(0, k0, v0);
        put(k0, v0);
    }
    for (int key0 = 0; key0 < rows.end; key0 += 2 * KEYS) {
        step(key0, k0, v0, k1, v1);
        if (key0 + KEYS < rows.end) step(key0 + KEYS, k1, v1, k0, v0);
    }
    const float l = st.l + other_half(st.l), inv = 1.0f / l;
    if (g.lse && row.there && h == 0) g.lse[((int64_t)rows.b * g.Hq + row.head) * g.Tq + row.t] = l != 0.0f ? st.m * g.scale + logf(l) : -INFINITY;
    T* const out = static_cast<T*>(g.out.p) + rows.b * g.out.lb + (int64_t)rows.hk * g.G * g.out.lh;
    auto place = [&](int r) {
        const int t = over(r, g.by_g);
        return out + t * g.out.lt + (r - t * g.G) * g.out.lh;
    };
    const int r0 = tile * kRowsByRows + wid * 32;
    if (g.wide_out) {
        __syncthreads();                                           // the tiles have been read
        constexpr int kMine = PARTS * kPart * 32, kFit = KEYS / 32;    // elements of a wavefront; how many a tile holds
        const int tile_of = wid / kFit;
        T* const mine = (tile_of == 0 ? k0 : tile_of == 1 ? k1 : tile_of == 2 ? v0 : v1) + wid % kFit * kMine;
        store_rows<T, PARTS>(mine, lane, g.D, inv, st.o, row.sees > 0, [&](int i) { return r0 + i < g.rows ? place(r0 + i) : nullptr; });
    } else if (row.there) {
        store_sums<T, PARTS>(place(r0 + (lane & 31)), lane, g.D, inv, st.o, row.sees > 0);
    }
}

// ---- by keys ----
constexpr int kRowsByKeys = 32, kKeysByKeys = 32;

// A split's part: sums relative to m, [32][parts of 32], then m and l of each row.
__host__ __device__ constexpr int part_floats(int parts) { return kRowsByKeys * (parts * kPart + 2); }

// All but the N youngest loads of the wavefront have arrived, and all reads of LDS.
template <int N>
__device__ __forceinline__ void wait_loads()
{
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x0070);
    asm volatile("" ::: "memory");
}

// Each wavefront has one K tile and one V tile: the next K tile is on its way while the values are passed, the next V tile while the keys
// are, so that two workgroups' wavefronts fit a compute unit (eight wavefronts a workgroup gained nothing).
// ONCE: all rows of a unit are one tile, and its keys and values are read by nobody else (32 x 16384 cached keys 213 us, 237 through the
// caches).
template <class T, int PARTS, bool ALIGNED, bool ONCE>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 ? 2 : 1) void attention_keys_kernel(Args g)
{
    constexpr int W = kWaves, KEYS = kKeysByKeys, N = tile_elements<T>(KEYS, PARTS), COLS = PARTS * kPart;
    constexpr int WIDTH = sizeof(T) == 2 && PARTS % 2 == 0 ? 2 * kPart : kPart;
    __shared__ __attribute__((aligned(16))) T kt[W][N];
    __shared__ __attribute__((aligned(16))) T vt[W][N];
    __shared__ float tops[W][kRowsByKeys], ls[W][kRowsByKeys];
    const int lane = threadIdx.x & 63, h = lane >> 5, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // units in turn: were it splits, those that only long entries have would all go to the same dies; those first
    const int unit = (int)(blockIdx.x % g.units), at = (int)(blockIdx.x / g.units);
    const int tile = g.tiles - 1 - at % g.tiles, split = g.splits - 1 - at / g.tiles;
    const Rows rows = rows_of(g, unit, tile * kRowsByKeys, kRowsByKeys);
    const Row row = row_of(g, rows, tile * kRowsByKeys + (lane & 31));
    const int begin = split * g.chunk, end = min(begin + g.chunk, rows.end);
    const int least = wave_min(row.sees);
    State<PARTS> st;
    if (begin + wid * KEYS < end) {
        const T* k = static_cast<const T*>(g.k.p) + rows.b * g.k.lb + rows.hk * g.k.lh;
        const T* v = static_cast<const T*>(g.v.p) + rows.b * g.v.lb + rows.hk * g.v.lh;
        // (behind the last tile too, the last key again and again: under a condition the compiler waits for all loads before it reads)
        auto load = [&](const T* from, int64_t lt, int key0, T* to) {
            load_tile<T, KEYS, PARTS, 1, ALIGNED, WIDTH, ONCE>(to, 0, lane, g.D, [&](int r) { return from + (key0 + r < rows.nk ? key0 + r : rows.nk - 1) * lt; });
        };
        constexpr int later = ALIGNED ? TileLoad<T, KEYS, PARTS, 1, WIDTH>::kLoads : 0;
        Frag<T> qf[2 * PARTS];
        load_queries<T, PARTS>(g, rows, row, h, qf);
        // every wait below counts on the order K, V, K, V, ...: the tiles are objects of their own, which the compiler may load in either order
        load(k, g.k.lt, begin + wid * KEYS, kt[wid]);
        asm volatile("" ::: "memory");
        load(v, g.v.lt, begin + wid * KEYS, vt[wid]);
        for (int key0 = begin + wid * KEYS; key0 < end; key0 += W * KEYS) {
            f32x16 p[1];
            Values<WIDTH, T, PARTS, KEYS> values(vt[wid], lane);
            wait_loads<later>();
            pass_keys<WIDTH, T, PARTS, KEYS>(kt[wid], lane, key0, row.sees, key0 + KEYS > least, g.c, qf, st, p, [] {});
            wait_loads<later>();
            load(k, g.k.lt, key0 + W * KEYS, kt[wid]);
            wait_loads<later>();
            values.start();
            values.pass(p, st);
            wait_loads<later>();
            load(v, g.v.lt, key0 + W * KEYS, vt[wid]);
        }
    }
    // the wavefronts' sums, through the tiles' memory: each wavefront adds up every fourth of the groups of four columns
    constexpr int HELD = N * sizeof(T) / (64 * sizeof(float));     // registers of the sums that a tile holds
    static_assert(2 * HELD >= PARTS * 16, "both hold all");
    float* const in_k = reinterpret_cast<float*>(kt[wid]) + lane;
    float* const in_v = reinterpret_cast<float*>(vt[wid]) + lane;
    const float l = st.l + other_half(st.l);
    wait_loads<0>();
#pragma unroll
    for (int i = 0; i < PARTS * 16; ++i) (i < HELD ? in_k : in_v - HELD * 64)[i * 64] = st.o[i / 16][i % 16];
    if (h == 0) {
        tops[wid][lane] = st.m;
        ls[wid][lane] = l;
    }
    __syncthreads();
    if (!row.there) return;
    float m = tops[0][lane & 31], n = 0.0f, a[W];
#pragma unroll
    for (int w = 1; w < W; ++w) m = fmaxf(m, tops[w][lane & 31]);
#pragma unroll
    for (int w = 0; w < W; ++w) {
        const float mw = tops[w][lane & 31];
        a[w] = mw == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((mw - m) * g.c);
        n += a[w] * ls[w][lane & 31];
    }
    float* const part = g.parts ? g.parts + (((int64_t)unit * g.tiles + tile) * g.splits + split) * part_floats(PARTS) : nullptr;
    T* const out = static_cast<T*>(g.out.p) + rows.b * g.out.lb + row.t * g.out.lt + row.head * g.out.lh;
    const float inv = 1.0f / n;
#pragma unroll
    for (int k = 0; k < PARTS; ++k) {
        const int i0 = 4 * (k * W + wid), c = 8 * (k * W + wid) + 4 * h;
        float o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float* from = (i0 < HELD ? reinterpret_cast<const float*>(kt[w]) : reinterpret_cast<const float*>(vt[w]) - HELD * 64) + lane;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] += a[w] * from[(i0 + e) * 64];
        }
        if (part) {
            if (n != 0.0f) put4(part + (lane & 31) * COLS + c, o);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = row.sees ? o[e] * inv : 0.0f;
            store4(out, c, g.D, o);
        }
    }
    if (wid || h) return;
    if (part) {
        part[kRowsByKeys * COLS + 2 * lane] = m;
        part[kRowsByKeys * COLS + 2 * lane + 1] = n;
    } else if (g.lse) {
        g.lse[((int64_t)rows.b * g.Hq + row.head) * g.Tq + row.t] = n != 0.0f ? m * g.scale + logf(n) : -INFINITY;
    }
}

// The splits' parts of a tile of rows, a wavefront a row.
template <class T, int PARTS>
__global__ __launch_bounds__(kThreads) void attention_join_kernel(Args g)
{
    const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
    const int64_t id = blockIdx.x;
    const int tile = (int)(id % g.tiles), unit = (int)(id / g.tiles);
    const Rows rows = rows_of(g, unit, tile * kRowsByKeys, kRowsByKeys);
    const float* parts = g.parts + id * g.splits * part_floats(PARTS);
    constexpr int COLS = (PARTS * kPart + 63) / 64;
    for (int r = wid; r < kRowsByKeys; r += kWaves) {
        const Row to = row_of(g, rows, tile * kRowsByKeys + r);
        if (!to.there) break;
        const float* ml = parts + kRowsByKeys * PARTS * kPart + 2 * r;
        float m = -INFINITY;
        for (int s = 0; s < g.splits; ++s) m = fmaxf(m, ml[(int64_t)s * part_floats(PARTS)]);
        float o[COLS], n = 0.0f;
#pragma unroll
        for (int k = 0; k < COLS; ++k) o[k] = 0.0f;
        for (int s = 0; s < g.splits; ++s) {
            const float* p = parts + (int64_t)s * part_floats(PARTS);
            const float ms = p[kRowsByKeys * PARTS * kPart + 2 * r], l = p[kRowsByKeys * PARTS * kPart + 2 * r + 1];
            if (l == 0.0f) continue;
            const float a = __builtin_amdgcn_exp2f((ms - m) * g.c);
            n += a * l;
#pragma unroll
            for (int k = 0; k < COLS; ++k)
                if (lane + 64 * k < PARTS * kPart) o[k] += a * p[r * (PARTS * kPart) + lane + 64 * k];
        }
        T* out = static_cast<T*>(g.out.p) + rows.b * g.out.lb + to.t * g.out.lt + to.head * g.out.lh;
#pragma unroll
        for (int k = 0; k < COLS; ++k)
            if (lane + 64 * k < g.D) put1(out + lane + 64 * k, to.sees ? o[k] / n : 0.0f);
        if (g.lse && lane == 0) g.lse[((int64_t)rows.b * g.Hq + to.head) * g.Tq + to.t] = n != 0.0f ? m * g.scale + logf(n) : -INFINITY;
    }
}

// ---- host ----
struct Plan {
    bool by_keys;
    int tiles, splits, chunk;
    size_t bytes;
};
constexpr int kComputeUnits = 256;
// By keys where by rows would leave compute units without a workgroup (heads of 128, 16 query and 4 key heads; us by rows, by keys):
// 1024 causal tokens, 128 workgroups, bf16 24.4, 18.2, fp32 114, 47; 1536, 192 workgroups, bf16 33, 29, fp32 163, 89; but 2048, 256
// workgroups, 42, 40 and 216, 138, and 8 x 512 x 8 x 8, as many, 17, 23 and 65, 62.  The limit is bf16's: fp32's two lie beyond it, and how far was
// not measured.  Without a causal mask rows' workgroups all have as
// much to do, and bf16, bound by the products, gains up to half as many: 1024 tokens 23.5, 21.3; 1152, 144 workgroups, 26.7, 33.5.
//
// Splits of the keys cost their parts' way through memory.  Tiles of many rows: as many splits as compute units take (1152 causal
// tokens in 576 workgroups: 20 us, in two splits 45; 64 x 16 rows to 16384 keys, 128 workgroups: unsplit 142, two splits 93, eight 128).
// One tile, where reading the keys is all there is, and lengths differ: six a compute unit (32 x 8 key heads to up to 16384 keys: 267 us
// with one, 212 with four, 209 with six, 207 with eight; 128 x 4 heads to 4096 keys each: 185, 210, 218, 226).  None of fewer
// than 1024 keys (2 x 4 key heads, one query, 2048 keys: 15.9 us, unsplit 19.2; 16384: 27.5, splits of 2048 35).
Plan plan_of(int B, int Tq, int Tk, int Hq, int Hk, int D, int is_bf16, int causal)
{
    Plan p{};
    const int64_t rows = (int64_t)Tq * (Hq / Hk), units = (int64_t)B * Hk;
    const int64_t by_rows = units * ((rows + kRowsByRows - 1) / kRowsByRows);
    p.by_keys = rows <= kRowsByKeys || by_rows < (is_bf16 && !causal ? kComputeUnits / 2 + 1 : kComputeUnits);
    p.splits = 1;
    p.chunk = std::max(Tk, 1);
    p.bytes = kAlign;
    if (!p.by_keys) {
        p.tiles = (int)((rows + kRowsByRows - 1) / kRowsByRows);
        return p;
    }
    p.tiles = (int)((rows + kRowsByKeys - 1) / kRowsByKeys);
    const int64_t groups = units * p.tiles, wanted = std::max<int64_t>(1, (p.tiles == 1 ? 6 : 1) * kComputeUnits / std::max<int64_t>(1, groups));
    const int least = LSGD_ATTENTION_ONE_LAUNCH, step = 128;
    const int64_t splits = std::min<int64_t>(wanted, (Tk + least - 1) / least);
    if (splits > 1) {
        p.chunk = (int)(((Tk + splits - 1) / splits + step - 1) / step * step);
        p.splits = (Tk + p.chunk - 1) / p.chunk;
        p.bytes = std::max(kAlign, sizeof(float) * (size_t)groups * (size_t)p.splits * (size_t)part_floats(parts_of(D)));   // (groups 0: no queries)
    }
    return p;
}

template <class T, int PARTS>
void launch(const Args& g, const Plan& p, bool aligned, hipStream_t s)
{
    if (!p.by_keys) {
        const dim3 grid((unsigned)workgroups(g, g.tiles));
        if (aligned) hipLaunchKernelGGL((attention_rows_kernel<T, PARTS, true>), grid, dim3(kThreads), 0, s, g);
        else hipLaunchKernelGGL((attention_rows_kernel<T, PARTS, false>), grid, dim3(kThreads), 0, s, g);
        return;
    }
    const dim3 grid((unsigned)((int64_t)g.units * g.tiles * g.splits)), threads(kThreads);
    if (aligned && g.tiles == 1) hipLaunchKernelGGL((attention_keys_kernel<T, PARTS, true, true>), grid, threads, 0, s, g);
    else if (aligned) hipLaunchKernelGGL((attention_keys_kernel<T, PARTS, true, false>), grid, threads, 0, s, g);
    else hipLaunchKernelGGL((attention_keys_kernel<T, PARTS, false, false>), grid, threads, 0, s, g);
    if (g.splits > 1) hipLaunchKernelGGL((attention_join_kernel<T, PARTS>), dim3((unsigned)((int64_t)g.units * g.tiles)), dim3(kThreads), 0, s, g);
}

// Launches of at most 2^31 workgroups and fewer than 2^32 threads.
bool fits(const Plan& p, int B, int Hk)
{
    return (double)((int64_t)B * Hk + 7) * 1.2 * p.tiles * p.splits * kThreads < 4294967296.0;
}

} // namespace

lsgd_status check_attention_shape(const char* who, int64_t B, int64_t Tq, int64_t Tk, int64_t Hq, int64_t Hk, int64_t D)
{
    if (B <= 0 || B > kMaxEntries) return set_error(LSGD_ERR_SHAPE, "%s: B=%lld outside [1,%d]", who, (long long)B, kMaxEntries);
    if (Tq < 0 || Tk < 0 || Tq > kMaxTokens || Tk > kMaxTokens)
        return set_error(LSGD_ERR_SHAPE, "%s: Tq=%lld or Tk=%lld outside [0,%d]", who, (long long)Tq, (long long)Tk, kMaxTokens);
    if (Hk <= 0 || Hq <= 0 || Hq > kMaxHeads || Hq % Hk) return set_error(LSGD_ERR_SHAPE, "%s: Hq=%lld must be a multiple of Hk=%lld and within [1,%d]", who, (long long)Hq, (long long)Hk, kMaxHeads);
    if (D <= 0) return set_error(LSGD_ERR_SHAPE, "%s: D=%lld must be positive", who, (long long)D);
    if (D > kMaxColumns) return set_error(LSGD_ERR_UNSUPPORTED, "%s: D=%lld beyond %d columns", who, (long long)D, kMaxColumns);
    if (Tq * (Hq / Hk) >= INT64_C(1) << 30) return set_error(LSGD_ERR_SHAPE, "%s: Tq * (Hq / Hk) = %lld is too large", who, (long long)(Tq * (Hq / Hk)));
    return LSGD_OK;
}

} // namespace attention
} // namespace lsgd

using namespace lsgd;
using namespace lsgd::attention;

extern "C" {

size_t lsgd_attention_workspace_bytes(int32_t B, int32_t Tq, int32_t Tk, int32_t Hq, int32_t Hk, int32_t D, int32_t is_bf16)
{
    if (check_attention_shape("attention", B, Tq, Tk, Hq, Hk, D) != LSGD_OK) return 0;
    return plan_of(B, Tq, Tk, Hq, Hk, D, is_bf16, 1).bytes;  // where keys are split, they are with either mask
}

lsgd_status lsgd_attention(const lsgd_attention_args* p, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    const char* who = "attention";
    if (!p) return set_error(LSGD_ERR_INVALID_ARG, "%s: arguments are NULL", who);
    const int B = p->B, Tq = p->Tq, Tk = p->Tk, Hq = p->Hq, Hk = p->Hk, D = p->D, es = p->is_bf16 ? 2 : 4;
    LSGD_TRY(check_attention_shape(who, B, Tq, Tk, Hq, Hk, D));
    if (p->is_bf16 & ~1 || p->causal & ~1) return set_error(LSGD_ERR_INVALID_ARG, "%s: is_bf16 and causal must be 0 or 1", who);
    if (!scale_ok(p->scale)) return set_error(LSGD_ERR_INVALID_ARG, "%s: scale must be within [1e-30, 1e30]", who);
    if (Tq == 0) return LSGD_OK;
    const Plan plan = plan_of(B, Tq, Tk, Hq, Hk, D, p->is_bf16, p->causal);
    if ((int64_t)B * Hk > INT64_C(1) << 30 || !fits(plan, B, Hk)) return set_error(LSGD_ERR_SHAPE, "%s: B=%d, Tq=%d, Hk=%d are too large for one launch", who, B, Tq, Hk);
    LSGD_TRY(check_heads(who, "q", p->q, B, Tq, Hq, D, es, true, false));
    LSGD_TRY(check_heads(who, "k", p->k, B, Tk, Hk, D, es, Tk > 0 || p->k.data, false));
    LSGD_TRY(check_heads(who, "v", p->v, B, Tk, Hk, D, es, Tk > 0 || p->v.data, false));
    LSGD_TRY(check_heads(who, "out", p->out, B, Tq, Hq, D, es, true, true));
    if (!on(p->q_lens, 4) || !on(p->k_lens, 4) || !on(p->lse, 4)) return set_error(LSGD_ERR_INVALID_ARG, "%s: q_lens, k_lens or lse is not aligned to its element", who);
    if (plan.splits > 1) {
        if (!workspace) return set_error(LSGD_ERR_INVALID_ARG, "%s: workspace is NULL", who);
        if (!on(workspace, kAlign)) return set_error(LSGD_ERR_INVALID_ARG, "%s: workspace must be 256-byte aligned", who);
        if (workspace_bytes < plan.bytes) return set_error(LSGD_ERR_NOMEM, "%s: workspace of %zu bytes < %zu needed", who, workspace_bytes, plan.bytes);
    }
    Args g{};
    g.q = heads(p->q); g.k = heads(p->k); g.v = heads(p->v); g.out = heads(p->out);
    set_shape(g, *p);
    g.lse = p->lse;
    g.parts = plan.splits > 1 ? static_cast<float*>(workspace) : nullptr;
    g.tiles = plan.tiles;
    g.splits = plan.splits; g.chunk = plan.chunk;
    g.scale = p->scale; g.c = p->scale * kLog2e;
    // what is read by 16 bytes straight to LDS has to lie on them
    const bool aligned = D % (16 / es) == 0 && wide_heads(p->k, B, Tk, Hk, es) && wide_heads(p->v, B, Tk, Hk, es);
    g.wide_out = D % (16 / es) == 0 && wide_heads(p->out, B, Tq, Hq, es);
    by_type_and_parts(p->is_bf16, parts_of(D), [&](auto type, auto parts) {
        launch<decltype(type), decltype(parts)::value>(g, plan, aligned, static_cast<hipStream_t>(hip_stream));
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return set_error(LSGD_ERR_HIP, "%s: %s", who, hipGetErrorString(e));
    return LSGD_OK;
}

} // extern "C"
