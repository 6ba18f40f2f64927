// Embedding lookup with scaling for a population, and the tables' gradient by sorted tokens.
//
//   out[w,t,:] = scale E_w[tok[w,t],:]         dE_w[v,:] (+)= scale sum_{t: tok[w,t] = v} dout[w,t,:]
//
// A token outside [0, V) is padding: zeros forward, nothing backward.
//
// The gradient.  Each worker's tokens are sorted (stable radix sort: equal tokens keep their order), so that the places
// of a table row form one run, and the sorted list is cut into spans of equal length, whatever the runs: a token that
// fills a tenth of the batch costs no team of lanes more than another.  A run inside a span is summed in registers and
// written; of a run that crosses spans each span leaves a partial sum, and a second launch adds those up in order.  No
// atomics touch a floating-point value: the order of every sum depends on the tokens alone, so equal calls give equal bits.
#include <algorithm>
#include <cmath>

#include "common.h"

using namespace lsgd;

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;

// ---- element access: E adjacent elements (E * size is 4, 8, 16 or 32 bytes), or one ----
template <class T> struct Elem;
template <> struct Elem<float> {
    static __device__ __forceinline__ float get(const float* p) { return *p; }
    static __device__ __forceinline__ void put(float* p, float v) { *p = v; }
};
template <> struct Elem<uint16_t> {
    static __device__ __forceinline__ float get(const uint16_t* p) { return bf16_to_f32(*p); }
    static __device__ __forceinline__ void put(uint16_t* p, float v) { *p = f32_to_bf16_rne(v); }
};

template <int E>
__device__ __forceinline__ void load_adjacent(const float* p, float (&v)[E])
{
#pragma unroll
    for (int e = 0; e < E; e += 4) {
        const v4f a = *reinterpret_cast<const v4f*>(p + e);
        v[e] = a.x; v[e + 1] = a.y; v[e + 2] = a.z; v[e + 3] = a.w;
    }
}
template <int E>
__device__ __forceinline__ void load_adjacent(const uint16_t* p, float (&v)[E])
{
    uint32_t q[E / 2];
    if constexpr (E == 8) {
        const v4u a = *reinterpret_cast<const v4u*>(p);
        q[0] = a.x; q[1] = a.y; q[2] = a.z; q[3] = a.w;
    } else {
        const v2u a = *reinterpret_cast<const v2u*>(p);
        q[0] = a.x; q[1] = a.y;
    }
#pragma unroll
    for (int e = 0; e < E / 2; ++e) {
        v[2 * e] = __uint_as_float(q[e] << 16);
        v[2 * e + 1] = __uint_as_float(q[e] & 0xFFFF0000u);
    }
}
template <int E>
__device__ __forceinline__ void store_adjacent(float* p, const float (&v)[E])
{
#pragma unroll
    for (int e = 0; e < E; e += 4) *reinterpret_cast<v4f*>(p + e) = v4f{v[e], v[e + 1], v[e + 2], v[e + 3]};
}
template <int E>
__device__ __forceinline__ void store_adjacent(uint16_t* p, const float (&v)[E])
{
    if constexpr (E == 8)
        *reinterpret_cast<v4u*>(p) = v4u{f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]), f32x2_to_bf16x2(v[4], v[5]), f32x2_to_bf16x2(v[6], v[7])};
    else
        *reinterpret_cast<v2u*>(p) = v2u{f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3])};
}

// ---- lookup ----
constexpr int kLookupEach = 4;      // independent pieces of E elements a thread has in flight

// A workgroup's pieces are adjacent in the output; which token and column a piece is follows from its number.
template <class TI, class TO, int E>
__global__ __launch_bounds__(kThreads) void lookup_kernel(const TI* __restrict__ table, int64_t ld_table, int V, int D,
                                                          const int32_t* __restrict__ tokens, int64_t ld_tokens, int T,
                                                          float scale, TO* __restrict__ out, int64_t ld_out)
{
    const int per = D / E;                                             // pieces of a token
    const int64_t base = (int64_t)blockIdx.x * (kThreads * kLookupEach);
    const int64_t t0 = base / per;
    const uint32_t c0 = (uint32_t)(base - t0 * per) + threadIdx.x;
    table += blockIdx.y * ld_table;
    tokens += blockIdx.y * ld_tokens;
    out += blockIdx.y * ld_out;
    int64_t t[kLookupEach];
    uint32_t c[kLookupEach];
    int tok[kLookupEach];
#pragma unroll
    for (int k = 0; k < kLookupEach; ++k) {
        const uint32_t q = c0 + k * kThreads;
        const uint32_t r = q / (uint32_t)per;
        t[k] = t0 + r;
        c[k] = (q - r * (uint32_t)per) * E;
        tok[k] = t[k] < T ? tokens[t[k]] : -1;
    }
    float v[kLookupEach][E];
#pragma unroll
    for (int k = 0; k < kLookupEach; ++k) {
#pragma unroll
        for (int e = 0; e < E; ++e) v[k][e] = 0.0f;
        if ((uint32_t)tok[k] < (uint32_t)V) {
            const TI* p = table + (int64_t)tok[k] * D + c[k];
            if constexpr (E == 1) v[k][0] = Elem<TI>::get(p);
            else load_adjacent<E>(p, v[k]);
        }
    }
#pragma unroll
    for (int k = 0; k < kLookupEach; ++k) {
        if (t[k] >= T) continue;
        TO* p = out + t[k] * D + c[k];
#pragma unroll
        for (int e = 0; e < E; ++e) v[k][e] *= scale;
        if constexpr (E == 1) Elem<TO>::put(p, v[k][0]);
        else store_adjacent<E>(p, v[k]);
    }
}

// ---- stable radix sort of each worker's tokens ----
constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / kWave;
constexpr int kSortEach = 8;
constexpr int kSortTile = kSortThreads * kSortEach;                    // tokens of one workgroup
constexpr int kMaxBits = 10;                                           // of a digit

struct SortLds {
    uint32_t key[kSortTile];
    int32_t pos[kSortTile];
    uint16_t count[kSortWaves][1 << kMaxBits];                         // of a wavefront's 512 tokens
    uint32_t base[1 << kMaxBits];
    uint32_t wave_sum[kSortWaves];
};

__device__ __forceinline__ uint32_t key_of(int tok, int V) { return (uint32_t)tok < (uint32_t)V ? (uint32_t)tok : (uint32_t)V; }

// Rank of every token of the workgroup among those of its digit: in its wavefront (rank), the wavefronts before it
// (count, turned into a sum over the earlier ones), and over the digits before it (base), which it returns in LDS.  `total`
// adds where the workgroup's tokens of a digit begin, if that is not its own list's start.
template <class F>
__device__ __forceinline__ void rank_digits(SortLds& s, const uint32_t (&digit)[kSortEach], uint32_t (&rank)[kSortEach], int bits, F digit_base)
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, bins = 1 << bits;
    for (int i = threadIdx.x; i < kSortWaves * bins; i += kSortThreads) s.count[i >> bits][i & (bins - 1)] = 0;
    __syncthreads();
    const uint64_t below = (1ull << lane) - 1;
#pragma unroll
    for (int k = 0; k < kSortEach; ++k) {
        uint64_t same = ~0ull;
        for (int b = 0; b < bits; ++b) {
            const uint64_t set = __ballot((digit[k] >> b) & 1u);
            same &= (digit[k] >> b) & 1u ? set : ~set;
        }
        volatile uint16_t* cell = &s.count[wave][digit[k]];
        const uint32_t before = *cell;
        rank[k] = before + (uint32_t)__popcll(same & below);
        __builtin_amdgcn_wave_barrier();
        if ((same & below) == 0) *cell = (uint16_t)(before + (uint32_t)__popcll(same));     // its first lane
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    // thread d: digit d's tokens of each wavefront to a sum over the wavefronts before it; then a scan over the digits
    uint32_t mine = 0;
    if ((int)threadIdx.x < bins) {
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t c = s.count[w][threadIdx.x];
            s.count[w][threadIdx.x] = (uint16_t)mine;
            mine += c;
        }
    }
    digit_base(s, mine);
    __syncthreads();
}

// Exclusive sum of v over the workgroup's threads.
__device__ __forceinline__ uint32_t exclusive_scan(SortLds& s, uint32_t v)
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    uint32_t x = v;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const uint32_t y = __shfl_up(x, o);
        if (lane >= o) x += y;
    }
    if (lane == kWave - 1) s.wave_sum[wave] = x;
    __syncthreads();
    uint32_t before = 0;
    for (int w = 0; w < wave; ++w) before += s.wave_sum[w];
    return before + x - v;
}

// A worker's whole list in one workgroup, all digits: no more than kSortTile tokens.
__global__ __launch_bounds__(kSortThreads) void sort_small_kernel(const int32_t* __restrict__ tokens, int64_t ld_tokens, int T, int V,
                                                                  int bits, int passes, uint32_t* __restrict__ keys, int32_t* __restrict__ pos)
{
    __shared__ SortLds s;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    tokens += blockIdx.x * ld_tokens;
    keys += (int64_t)blockIdx.x * T;
    pos += (int64_t)blockIdx.x * T;
    const int first = wave * (kWave * kSortEach) + lane;
    uint32_t key[kSortEach], digit[kSortEach], rank[kSortEach];
    int32_t at[kSortEach];
#pragma unroll
    for (int k = 0; k < kSortEach; ++k) {
        at[k] = first + k * kWave;
        key[k] = at[k] < T ? key_of(tokens[at[k]], V) : 0xFFFFFFFFu;   // past the end: last in every digit's order
    }
    for (int p = 0; p < passes; ++p) {
        const uint32_t mask = (1u << bits) - 1;
#pragma unroll
        for (int k = 0; k < kSortEach; ++k) digit[k] = (key[k] >> (p * bits)) & mask;
        rank_digits(s, digit, rank, bits, [&](SortLds& l, uint32_t mine) {
            const uint32_t b = exclusive_scan(l, mine);
            if ((int)threadIdx.x < (1 << bits)) l.base[threadIdx.x] = b;
        });
        const bool last = p + 1 == passes;
#pragma unroll
        for (int k = 0; k < kSortEach; ++k) {
            const uint32_t to = s.base[digit[k]] + s.count[wave][digit[k]] + rank[k];
            if (last) {
                if ((int)to < T) { keys[to] = key[k]; pos[to] = at[k]; }
            } else {
                s.key[to] = key[k];
                s.pos[to] = at[k];
            }
        }
        __syncthreads();
        if (!last) {
#pragma unroll
            for (int k = 0; k < kSortEach; ++k) {
                key[k] = s.key[first + k * kWave];
                at[k] = s.pos[first + k * kWave];
            }
            __syncthreads();
        }
    }
}

// Longer lists: how many tokens of each digit every tile has ...
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const int32_t* __restrict__ tokens, int64_t ld_tokens,
                                                                  const uint32_t* __restrict__ keys_in, int T, int V, int bits, int shift,
                                                                  uint32_t* __restrict__ counts)
{
    __shared__ uint32_t bin[1 << kMaxBits];
    const int bins = 1 << bits;
    for (int i = threadIdx.x; i < bins; i += kSortThreads) bin[i] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * kSortTile;
#pragma unroll
    for (int k = 0; k < kSortEach; ++k) {
        const int64_t i = first + k * kSortThreads + threadIdx.x;
        if (i < T) {
            const uint32_t key = keys_in ? keys_in[(int64_t)blockIdx.y * T + i] : key_of(tokens[blockIdx.y * ld_tokens + i], V);
            atomicAdd(&bin[(key >> shift) & (uint32_t)(bins - 1)], 1u);
        }
    }
    __syncthreads();
    uint32_t* to = counts + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * bins;
    for (int i = threadIdx.x; i < bins; i += kSortThreads) to[i] = bin[i];
}

// ... and every tile's tokens to their places: after all smaller digits, and after the same digit's in earlier tiles.
__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(const int32_t* __restrict__ tokens, int64_t ld_tokens,
                                                                  const uint32_t* __restrict__ keys_in, const int32_t* __restrict__ pos_in,
                                                                  int T, int V, int bits, int shift, const uint32_t* __restrict__ counts,
                                                                  uint32_t* __restrict__ keys, int32_t* __restrict__ pos)
{
    __shared__ SortLds s;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, bins = 1 << bits;
    const int64_t off = (int64_t)blockIdx.y * T;
    const int64_t first = (int64_t)blockIdx.x * kSortTile + wave * (kWave * kSortEach) + lane;
    uint32_t key[kSortEach], digit[kSortEach], rank[kSortEach];
    int32_t at[kSortEach];
#pragma unroll
    for (int k = 0; k < kSortEach; ++k) {
        const int64_t i = first + k * kWave;
        key[k] = 0xFFFFFFFFu;
        at[k] = -1;
        if (i < T) {
            key[k] = keys_in ? keys_in[off + i] : key_of(tokens[blockIdx.y * ld_tokens + i], V);
            at[k] = keys_in ? pos_in[off + i] : (int32_t)i;
        }
        digit[k] = (key[k] >> shift) & (uint32_t)(bins - 1);
    }
    rank_digits(s, digit, rank, bits, [&](SortLds& l, uint32_t) {
        uint32_t all = 0, before = 0;
        if ((int)threadIdx.x < bins) {
            const uint32_t* c = counts + (int64_t)blockIdx.y * gridDim.x * bins + threadIdx.x;
            for (unsigned b = 0; b < gridDim.x; ++b) {
                const uint32_t n = c[(int64_t)b * bins];
                if (b < blockIdx.x) before += n;
                all += n;
            }
        }
        const uint32_t b = exclusive_scan(l, all);
        if ((int)threadIdx.x < bins) l.base[threadIdx.x] = b + before;
    });
#pragma unroll
    for (int k = 0; k < kSortEach; ++k) {
        if (at[k] < 0) continue;                                       // past the end of the list
        const int64_t to = off + s.base[digit[k]] + s.count[wave][digit[k]] + rank[k];
        keys[to] = key[k];
        pos[to] = at[k];
    }
}

// First index of a sorted list whose key is >= target; a whole wavefront asks, 64 probes a round.
__device__ __forceinline__ int lower_bound(const uint32_t* __restrict__ keys, int n, uint32_t target)
{
    const int lane = threadIdx.x & (kWave - 1);
    int lo = 0, len = n;
    while (len > 0) {
        const int step = (len + kWave - 1) / kWave;
        const int64_t i = (int64_t)lane * step;
        const bool less = i < len && keys[lo + i] < target;
        const int c = __popcll(__ballot(less));
        if (c == 0) break;                                             // keys[lo] >= target
        const int skip = (c - 1) * step + 1;                           // keys[lo + (c-1) step] < target
        const int upto = c * step < len ? c * step : len;              // keys[lo + c step] >= target, if it exists
        lo += skip;
        len = upto - skip;
    }
    return lo;
}

// ---- the gradient ----
struct GradArgs {
    const void* dout;
    int64_t ld_dout;
    const uint32_t* keys;
    const int32_t* pos;
    float* parts;            // [W][spans][2][Dp]: of the run that came into a span, of the one that began there and goes on
    float* table;
    int64_t ld_table;
    int T, V, D, Dp, L, spans, slices;
    int run_blocks;          // workgroups that sum runs; those after them write zeros to rows without tokens
    int zero_rows;           // table rows of such a workgroup
    float scale;
    int accumulate;
};

// E elements of columns [col, D): adjacent ones, or one every TL columns where rows are not aligned for that.
template <class T, int E, int TL, bool WIDE>
__device__ __forceinline__ void load_row(const T* p, int col, int D, float (&v)[E])
{
    if constexpr (WIDE) {
        if (col < D) load_adjacent<E>(p + col, v);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (col + e * TL < D) v[e] = Elem<T>::get(p + col + e * TL);
    }
}

// TL lanes make a team: they own TL * E columns of one span.
template <class T, int E, int TL, bool WIDE>
__device__ __forceinline__ void sum_runs(const GradArgs& a, int64_t task)
{
    constexpr int U = 4;                                               // rows in flight
    const int w = blockIdx.y;
    const int span = (int)(task / a.slices), slice = (int)(task - (int64_t)span * a.slices);
    if (span >= a.spans) return;
    const int lane = threadIdx.x % TL;
    const int col = WIDE ? (slice * TL + lane) * E : slice * TL * E + lane;
    const uint32_t* keys = a.keys + (int64_t)w * a.T;
    const int32_t* pos = a.pos + (int64_t)w * a.T;
    const T* dout = static_cast<const T*>(a.dout) + w * a.ld_dout;
    float* table = a.table + w * a.ld_table;
    const int s0 = span * a.L, s1 = s0 + a.L < a.T ? s0 + a.L : a.T;
    uint32_t cur = keys[s0];
    bool head = s0 > 0 && keys[s0 - 1] == cur;
    float acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.0f;

    auto flush = [&](bool tail) {
        if (cur >= (uint32_t)a.V) return;                              // padding
        if (head || tail) {
            float* p = a.parts + (((int64_t)w * a.spans + span) * 2 + (head ? 0 : 1)) * a.Dp;
            if constexpr (WIDE) {
                if (col < a.D) store_adjacent<E>(p + col, acc);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (col + e * TL < a.D) p[col + e * TL] = acc[e];
            }
        } else {
            float* p = table + (int64_t)cur * a.D;
            float old[E];
#pragma unroll
            for (int e = 0; e < E; ++e) old[e] = 0.0f;
            if (a.accumulate) load_row<float, E, TL, WIDE>(p, col, a.D, old);
#pragma unroll
            for (int e = 0; e < E; ++e) old[e] += a.scale * acc[e];
            if constexpr (WIDE) {
                if (col < a.D) store_adjacent<E>(p + col, old);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (col + e * TL < a.D) p[col + e * TL] = old[e];
            }
        }
    };

    for (int i = s0; i < s1; i += U) {
        uint32_t key[U];
        int32_t at[U];
        float row[U][E];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            key[u] = i + u < s1 ? keys[i + u] : (uint32_t)a.V;
            at[u] = i + u < s1 ? pos[i + u] : 0;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int e = 0; e < E; ++e) row[u][e] = 0.0f;
            if (key[u] < (uint32_t)a.V) load_row<T, E, TL, WIDE>(dout + (int64_t)at[u] * a.D, col, a.D, row[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i + u < s1 && key[u] != cur) {
                flush(false);
                cur = key[u];
                head = false;
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] = 0.0f;
            }
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] += row[u][e];
        }
    }
    flush(s1 < a.T && keys[s1] == cur);
}

// Zeros to the rows of [v0, v0 + zero_rows) that no token names.
template <bool WIDE>
__device__ __forceinline__ void zero_rows(const GradArgs& a, int64_t v0, uint32_t* present)
{
    const int w = blockIdx.y;
    const uint32_t* keys = a.keys + (int64_t)w * a.T;
    const int n = (int)(a.V - v0 < a.zero_rows ? a.V - v0 : a.zero_rows);
    for (int i = threadIdx.x; i < (a.zero_rows + 31) / 32; i += kThreads) present[i] = 0;
    __syncthreads();
    const int lo = lower_bound(keys, a.T, (uint32_t)v0);
    const int hi = lo + lower_bound(keys + lo, a.T - lo, (uint32_t)(v0 + n));
    for (int i = lo + (int)threadIdx.x; i < hi; i += kThreads) {
        const uint32_t r = keys[i] - (uint32_t)v0;
        atomicOr(&present[r >> 5], 1u << (r & 31));
    }
    __syncthreads();
    float* table = a.table + w * a.ld_table;
    const int lane = threadIdx.x & (kWave - 1);
    for (int r = threadIdx.x / kWave; r < n; r += kThreads / kWave) {
        if (present[r >> 5] >> (r & 31) & 1u) continue;
        float* p = table + (v0 + r) * a.D;
        if constexpr (WIDE) {
            for (int c = 4 * lane; c < a.D; c += 4 * kWave) *reinterpret_cast<v4f*>(p + c) = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        } else {
            for (int c = lane; c < a.D; c += kWave) p[c] = 0.0f;
        }
    }
}

constexpr int kZeroRows = 64;

template <class T, int E, int TL, bool WIDE>
__global__ __launch_bounds__(kThreads) void grad_runs_kernel(GradArgs a)
{
    __shared__ uint32_t present[(kZeroRows + 31) / 32];
    if ((int)blockIdx.x < a.run_blocks) sum_runs<T, E, TL, WIDE>(a, (int64_t)blockIdx.x * (kThreads / TL) + threadIdx.x / TL);
    else zero_rows<WIDE>(a, (int64_t)((int)blockIdx.x - a.run_blocks) * a.zero_rows, present);
}

// Runs that cross spans: the workgroup of the span where one begins adds up its parts, each wavefront a stretch of them.
constexpr int kJoinCols = 4 * kWave;
__global__ __launch_bounds__(kThreads) void grad_join_kernel(GradArgs a)
{
    __shared__ float sum[kThreads / kWave][kJoinCols];
    const int w = blockIdx.y, span = blockIdx.x;
    const uint32_t* keys = a.keys + (int64_t)w * a.T;
    const int s0 = span * a.L, s1 = s0 + a.L;
    if (s1 >= a.T) return;
    const uint32_t cur = keys[s1 - 1];
    if (cur >= (uint32_t)a.V || keys[s1] != cur) return;               // nothing goes on into the next span
    if (keys[s0] == cur && s0 > 0 && keys[s0 - 1] == cur) return;      // it began earlier
    const int end = s1 + lower_bound(keys + s1, a.T - s1, cur + 1);
    const int parts = (end - 1) / a.L - span + 1;                      // the tail of this span, then heads
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, waves = kThreads / kWave;
    const int col0 = blockIdx.z * kJoinCols, col = col0 + 4 * lane;
    const float* first = a.parts + ((int64_t)w * a.spans + span) * 2 * a.Dp;
    const int per = (parts + waves - 1) / waves, p0 = wave * per, p1 = p0 + per < parts ? p0 + per : parts;
    v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
    if (col < a.Dp) {
#pragma unroll 8
        for (int p = p0; p < p1; ++p) {
            const float* q = first + ((int64_t)p * 2 + (p == 0 ? 1 : 0)) * a.Dp + col;
            acc += *reinterpret_cast<const v4f*>(q);
        }
    }
    *reinterpret_cast<v4f*>(&sum[wave][4 * lane]) = acc;
    __syncthreads();
    const int c = col0 + (int)threadIdx.x;
    if (c < a.D) {
        float s = 0.0f;
#pragma unroll
        for (int v = 0; v < waves; ++v) s += sum[v][threadIdx.x];
        float* p = a.table + w * a.ld_table + (int64_t)cur * a.D + c;
        *p = (a.accumulate ? *p : 0.0f) + a.scale * s;
    }
}

// All rows to zero: there is no token.
__global__ __launch_bounds__(kThreads) void zero_table_kernel(float* __restrict__ table, int64_t ld, int64_t n)
{
    table += blockIdx.y * ld;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads) table[i] = 0.0f;
}

// ---- host ----
constexpr size_t kAlign = 256;
size_t align_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }
bool on(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

constexpr int kMaxTokens = 1 << 24, kMaxRows = (1 << 30) - 1;

lsgd_status check_shape(const char* who, int32_t W, int32_t T, int32_t V, int32_t D)
{
    if (W <= 0 || W > LSGD_MAX_WORKERS) return set_error(LSGD_ERR_SHAPE, "%s: W=%d outside [1,%d]", who, (int)W, LSGD_MAX_WORKERS);
    if (T < 0) return set_error(LSGD_ERR_SHAPE, "%s: T=%d is negative", who, (int)T);
    if (V <= 0 || D <= 0) return set_error(LSGD_ERR_SHAPE, "%s: V=%d and D=%d must be positive", who, (int)V, (int)D);
    if (T > kMaxTokens || V > kMaxRows)
        return set_error(LSGD_ERR_UNSUPPORTED, "%s: T=%d or V=%d beyond the %d tokens and %d rows a worker may have", who, (int)T, (int)V, kMaxTokens, kMaxRows);
    return LSGD_OK;
}

struct Plan {
    int bits, passes, tiles;     // of the sort
    int L, spans, Dp;
    size_t keys[2], pos[2], counts, parts, total;
};

// Spans of 32 places once those fill the chip; shorter batches are cut finer.
Plan make_plan(int W, int T, int V, int D)
{
    Plan p;
    int nb = 1;
    while (V >> nb) ++nb;                                              // keys are 0 .. V
    p.passes = (nb + kMaxBits - 1) / kMaxBits;
    p.bits = (nb + p.passes - 1) / p.passes;
    p.tiles = T ? (T - 1) / kSortTile + 1 : 0;
    p.L = 32;
    while (p.L > 8 && (int64_t)W * T / p.L < 2048) p.L /= 2;
    p.spans = T ? (T - 1) / p.L + 1 : 0;
    p.Dp = (D + 7) / 8 * 8;
    const size_t list = align_up(sizeof(uint32_t) * (size_t)W * (size_t)T);
    size_t o = 0;
    for (int k = 0; k < 2; ++k) {
        const bool used = k == 0 || (p.tiles > 1 && p.passes > 1);
        p.keys[k] = o; o += used ? list : 0;
        p.pos[k] = o;  o += used ? list : 0;
    }
    p.counts = o; o += p.tiles > 1 ? align_up(sizeof(uint32_t) * (size_t)W * (size_t)p.tiles << p.bits) : 0;
    p.parts = o;  o += p.spans > 1 ? align_up(sizeof(float) * (size_t)W * (size_t)p.spans * 2 * (size_t)p.Dp) : 0;
    p.total = o ? o : kAlign;
    return p;
}

template <class TI, class TO>
void launch_lookup(int W, int T, int V, int D, const void* table, int64_t ld_table, const int32_t* tokens, int64_t ld_tokens, float scale,
                   void* out, int64_t ld_out, hipStream_t s)
{
    const TI* in = static_cast<const TI*>(table);
    TO* to = static_cast<TO*>(out);
    auto ok = [&](int E) {
        auto fits = [&](const void* p, int64_t ld, size_t es) {
            const size_t a = std::min<size_t>(16, es * (size_t)E);
            return on(p, a) && (W == 1 || (ld * (int64_t)es) % (int64_t)a == 0);
        };
        return D % E == 0 && fits(in, ld_table, sizeof(TI)) && fits(to, ld_out, sizeof(TO));
    };
    auto go = [&](auto kernel, int E) {
        const int64_t pieces = (int64_t)T * (D / E);
        const dim3 grid((unsigned)((pieces - 1) / (kThreads * kLookupEach) + 1), (unsigned)W);
        hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, in, ld_table, V, D, tokens, ld_tokens, T, scale, to, ld_out);
    };
    if (ok(8)) go(lookup_kernel<TI, TO, 8>, 8);
    else if (ok(4)) go(lookup_kernel<TI, TO, 4>, 4);
    else go(lookup_kernel<TI, TO, 1>, 1);
}

template <class T, int E, int TL, bool WIDE>
void launch_grad(GradArgs a, int W, hipStream_t s)
{
    a.slices = (a.D - 1) / (TL * E) + 1;
    const int teams = kThreads / TL;
    a.run_blocks = (int)(((int64_t)a.spans * a.slices - 1) / teams + 1);
    a.zero_rows = kZeroRows;
    const int zero_blocks = a.accumulate ? 0 : (a.V - 1) / kZeroRows + 1;
    hipLaunchKernelGGL((grad_runs_kernel<T, E, TL, WIDE>), dim3((unsigned)(a.run_blocks + zero_blocks), (unsigned)W), dim3(kThreads), 0, s, a);
    if (a.spans > 1)
        hipLaunchKernelGGL(grad_join_kernel, dim3((unsigned)(a.spans - 1), (unsigned)W, (unsigned)((a.D - 1) / kJoinCols + 1)), dim3(kThreads), 0, s, a);
}

template <class T, int E>
void launch_grad_team(const GradArgs& a, int W, bool wide, hipStream_t s)
{
    const int lanes = (a.D - 1) / E + 1;
    if (wide) {
        if (lanes <= 16) launch_grad<T, E, 16, true>(a, W, s);
        else if (lanes <= 32) launch_grad<T, E, 32, true>(a, W, s);
        else launch_grad<T, E, 64, true>(a, W, s);
    } else {
        if (lanes <= 16) launch_grad<T, E, 16, false>(a, W, s);
        else if (lanes <= 32) launch_grad<T, E, 32, false>(a, W, s);
        else launch_grad<T, E, 64, false>(a, W, s);
    }
}

} // namespace

extern "C" {

lsgd_status lsgd_embed_lookup(int32_t W, int32_t T, int32_t V, int32_t D, const void* table, int64_t ld_table, int32_t table_is_bf16,
                              const int32_t* tokens, int64_t ld_tokens, float scale, void* out, int64_t ld_out, int32_t out_is_bf16,
                              void* hip_stream)
{
    const lsgd_status st = check_shape("embed_lookup", W, T, V, D);
    if (st != LSGD_OK) return st;
    if ((table_is_bf16 | out_is_bf16) & ~1) return set_error(LSGD_ERR_INVALID_ARG, "embed_lookup: table_is_bf16 and out_is_bf16 must be 0 or 1");
    if (!std::isfinite(scale)) return set_error(LSGD_ERR_INVALID_ARG, "embed_lookup: scale must be finite");
    if (T == 0) return LSGD_OK;
    if (!table || !tokens || !out) return set_error(LSGD_ERR_INVALID_ARG, "embed_lookup: table, tokens and out are required");
    if (!on(table, table_is_bf16 ? 2 : 4) || !on(out, out_is_bf16 ? 2 : 4) || !on(tokens, 4))
        return set_error(LSGD_ERR_INVALID_ARG, "embed_lookup: a pointer is not aligned to its element");
    if (W > 1 && (ld_table < 0 || ld_tokens < T || ld_out < (int64_t)T * D))
        return set_error(LSGD_ERR_SHAPE, "embed_lookup: a worker stride is smaller than what a worker has (ld_tokens=%lld, ld_out=%lld)",
                         (long long)ld_tokens, (long long)ld_out);
    const int64_t pieces = (int64_t)T * D;
    if (pieces / (kThreads * kLookupEach) >= 0x7fffffff) return set_error(LSGD_ERR_SHAPE, "embed_lookup: T*D=%lld is too large for one launch", (long long)pieces);
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (table_is_bf16) {
        if (out_is_bf16) launch_lookup<uint16_t, uint16_t>(W, T, V, D, table, ld_table, tokens, ld_tokens, scale, out, ld_out, s);
        else launch_lookup<uint16_t, float>(W, T, V, D, table, ld_table, tokens, ld_tokens, scale, out, ld_out, s);
    } else {
        if (out_is_bf16) launch_lookup<float, uint16_t>(W, T, V, D, table, ld_table, tokens, ld_tokens, scale, out, ld_out, s);
        else launch_lookup<float, float>(W, T, V, D, table, ld_table, tokens, ld_tokens, scale, out, ld_out, s);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return set_error(LSGD_ERR_HIP, "embed_lookup: %s", hipGetErrorString(e));
    return LSGD_OK;
}

size_t lsgd_embed_grad_workspace_bytes(int32_t W, int32_t T, int32_t V, int32_t D)
{
    if (check_shape("embed_grad", W, T, V, D) != LSGD_OK) return 0;
    return make_plan(W, T, V, D).total;
}

lsgd_status lsgd_embed_grad(int32_t W, int32_t T, int32_t V, int32_t D, const void* dout, int64_t ld_dout, int32_t dout_is_bf16,
                            const int32_t* tokens, int64_t ld_tokens, float scale, int32_t accumulate, float* dtable, int64_t ld_dtable,
                            void* workspace, size_t workspace_bytes, void* hip_stream)
{
    const lsgd_status st = check_shape("embed_grad", W, T, V, D);
    if (st != LSGD_OK) return st;
    if ((dout_is_bf16 | accumulate) & ~1) return set_error(LSGD_ERR_INVALID_ARG, "embed_grad: dout_is_bf16 and accumulate must be 0 or 1");
    if (!std::isfinite(scale)) return set_error(LSGD_ERR_INVALID_ARG, "embed_grad: scale must be finite");
    if (!dtable || !on(dtable, 4)) return set_error(LSGD_ERR_INVALID_ARG, "embed_grad: dtable is NULL or not aligned to its element");
    if (W > 1 && ld_dtable < (int64_t)V * D)
        return set_error(LSGD_ERR_SHAPE, "embed_grad: ld_dtable=%lld < V*D=%lld: workers' gradients would overlap", (long long)ld_dtable, (long long)V * D);
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    hipError_t e;
    if (T == 0) {
        if (!accumulate) {
            const int64_t n = (int64_t)V * D;
            hipLaunchKernelGGL(zero_table_kernel, dim3((unsigned)std::min<int64_t>((n - 1) / kThreads + 1, 4096), (unsigned)W), dim3(kThreads), 0, s, dtable,
                               ld_dtable, n);
            e = hipGetLastError();
            if (e != hipSuccess) return set_error(LSGD_ERR_HIP, "embed_grad: %s", hipGetErrorString(e));
        }
        return LSGD_OK;
    }
    if (!dout || !tokens) return set_error(LSGD_ERR_INVALID_ARG, "embed_grad: dout and tokens are required");
    if (!on(dout, dout_is_bf16 ? 2 : 4) || !on(tokens, 4)) return set_error(LSGD_ERR_INVALID_ARG, "embed_grad: a pointer is not aligned to its element");
    if (W > 1 && (ld_tokens < T || ld_dout < (int64_t)T * D))
        return set_error(LSGD_ERR_SHAPE, "embed_grad: a worker stride is smaller than what a worker has (ld_tokens=%lld, ld_dout=%lld)",
                         (long long)ld_tokens, (long long)ld_dout);
    if (!workspace) return set_error(LSGD_ERR_INVALID_ARG, "embed_grad: workspace is NULL");
    if (!on(workspace, kAlign)) return set_error(LSGD_ERR_INVALID_ARG, "embed_grad: workspace must be 256-byte aligned");
    const Plan p = make_plan(W, T, V, D);
    if (workspace_bytes < p.total) return set_error(LSGD_ERR_NOMEM, "embed_grad: workspace of %zu bytes < %zu needed", workspace_bytes, p.total);
    if ((int64_t)p.spans * ((D - 1) / 64 + 1) + V / kZeroRows >= 0x7fffffff)
        return set_error(LSGD_ERR_SHAPE, "embed_grad: T=%d of D=%d is too large for one launch", (int)T, (int)D);

    char* base = static_cast<char*>(workspace);
    uint32_t* keys[2] = {reinterpret_cast<uint32_t*>(base + p.keys[0]), reinterpret_cast<uint32_t*>(base + p.keys[1])};
    int32_t* pos[2] = {reinterpret_cast<int32_t*>(base + p.pos[0]), reinterpret_cast<int32_t*>(base + p.pos[1])};
    int at = 0;
    if (p.tiles == 1) {
        hipLaunchKernelGGL(sort_small_kernel, dim3((unsigned)W), dim3(kSortThreads), 0, s, tokens, ld_tokens, (int)T, (int)V, p.bits, p.passes, keys[0], pos[0]);
    } else {
        uint32_t* counts = reinterpret_cast<uint32_t*>(base + p.counts);
        const dim3 grid((unsigned)p.tiles, (unsigned)W);
        for (int k = 0; k < p.passes; ++k) {
            const uint32_t* kin = k ? keys[at ^ 1] : nullptr;
            const int32_t* pin = k ? pos[at ^ 1] : nullptr;
            hipLaunchKernelGGL(sort_count_kernel, grid, dim3(kSortThreads), 0, s, tokens, ld_tokens, kin, (int)T, (int)V, p.bits, k * p.bits, counts);
            hipLaunchKernelGGL(sort_place_kernel, grid, dim3(kSortThreads), 0, s, tokens, ld_tokens, kin, pin, (int)T, (int)V, p.bits, k * p.bits,
                               counts, keys[at], pos[at]);
            if (k + 1 < p.passes) at ^= 1;
        }
    }
    GradArgs a{};
    a.dout = dout; a.ld_dout = ld_dout;
    a.keys = keys[at]; a.pos = pos[at];
    a.parts = reinterpret_cast<float*>(base + p.parts);
    a.table = dtable; a.ld_table = ld_dtable;
    a.T = T; a.V = V; a.D = D; a.Dp = p.Dp; a.L = p.L; a.spans = p.spans;
    a.scale = scale; a.accumulate = accumulate;
    const int E = dout_is_bf16 ? 8 : 4;
    const bool wide = D % E == 0 && on(dout, 16) && on(dtable, 16) && (W == 1 || (ld_dout % E == 0 && ld_dtable % 4 == 0));
    if (dout_is_bf16) launch_grad_team<uint16_t, 8>(a, W, wide, s);
    else launch_grad_team<float, 4>(a, W, wide, s);
    e = hipGetLastError();
    if (e != hipSuccess) return set_error(LSGD_ERR_HIP, "embed_grad: %s", hipGetErrorString(e));
    return LSGD_OK;
}

} // extern "C"
