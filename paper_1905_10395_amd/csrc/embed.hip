// Embedding lookup with scaling for a population, and the tables' gradient by sorted tokens.
//
//   out[w,t,:] = scale E_w[tok[w,t],:]         dE_w[v,:] (+)= scale sum_{t: tok[w,t] = v} dout[w,t,:]
//
// A token outside [0, V) is padding: zeros forward, nothing backward.
//
// The gradient.  Each worker's tokens are sorted (stable radix sort: equal tokens keep their order), so that the places of
// a table row form one run, and the sorted list is cut into spans of equal length, whatever the runs: a token that fills a
// tenth of the batch costs no team of lanes more than another.  Frequencies that fall as 1/rank put two fifths of a batch
// into the first 64 rows of a table; workgroups that own rows instead took seven times as long (2048 tokens, 65536 rows).
//
// Long lists: sorted in memory.  A run is summed in registers and written by the team of the span it begins in, also if
// it ends in the next one; of a longer run each span leaves a partial sum, and another launch adds those up in order.
//
// Short ones take one launch: every workgroup sorts the whole list in LDS for itself, sums the runs that begin in its span
// and writes zeros to its share of the rows without tokens; a run of many places is shared by its wavefronts.
//
// No atomics touch a floating-point value: the order of every sum depends on the tokens alone, so equal calls give equal bits.
#include <algorithm>
#include <cmath>

#include "row_pieces.h"

using namespace lsgd;

namespace {

constexpr int kThreads = 256;

// ---- lookup ----
constexpr int kLookupEach = 4;      // independent pieces a thread has in flight
// Elements of a piece: 16 bytes of it are adjacent to the next lane's, so that streaming stores fill lines (16 x 8192 x 1024 fp32
// 131 us, 159 with 32).
template <class TI, class TO>
constexpr int kLookupPiece = sizeof(TI) == 4 && sizeof(TO) == 4 ? 4 : 8;

// A workgroup's pieces are adjacent in the output; which token and column a piece is follows from its number.  Bound by memory:
// 16 x 8192 x 1024 bf16 from 32768 rows 70 to 72 us, 5.3 TB/s of the 375 MB that have to move (75 us with stores that stay in the
// caches; 76 and 72 us with 2 and 8 pieces in flight).  Rows that are not aligned take up to twice as long as their bytes:
// 8 x 32768 x 1023 195 us bf16, 321 fp32.
template <class TI, class TO, bool ONCE>
__global__ __launch_bounds__(kThreads) void lookup_kernel(const TI* __restrict__ table, int64_t ld_table, int V, int D,
                                                          const int32_t* __restrict__ tokens, int64_t ld_tokens, int T,
                                                          float scale, TO* __restrict__ out, int64_t ld_out)
{
    constexpr int E = kLookupPiece<TI, TO>;
    const int per = (D - 1) / E + 1;                                   // pieces of a token
    const int64_t base = (int64_t)blockIdx.x * (kThreads * kLookupEach);
    const int64_t t0 = base / per;
    const uint32_t c0 = (uint32_t)(base - t0 * per) + threadIdx.x;
    table += blockIdx.y * ld_table;
    tokens += blockIdx.y * ld_tokens;
    out += blockIdx.y * ld_out;
    int64_t t[kLookupEach];
    int c[kLookupEach], tok[kLookupEach];
#pragma unroll
    for (int k = 0; k < kLookupEach; ++k) {
        const uint32_t q = c0 + k * kThreads;
        const uint32_t r = q / (uint32_t)per;
        t[k] = t0 + r;
        c[k] = (int)(q - r * (uint32_t)per) * E;
        tok[k] = t[k] < T ? tokens[t[k]] : -1;
    }
    Raw<TI, E> row[kLookupEach];
#pragma unroll
    for (int k = 0; k < kLookupEach; ++k) {
        clear(row[k]);
        if ((uint32_t)tok[k] >= (uint32_t)V) continue;
        if constexpr (ONCE) load_whole<false>(table + (int64_t)tok[k] * D + c[k], row[k]);
        else load_piece(table + (int64_t)tok[k] * D, c[k], D, row[k]);
    }
#pragma unroll
    for (int k = 0; k < kLookupEach; ++k) {
        if (t[k] >= T) continue;
        float v[E];
        unpack(row[k], v);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] *= scale;
        if constexpr (ONCE) store_whole<true>(out + t[k] * D + c[k], v);
        else store_piece(out + t[k] * D, c[k], D, v);
    }
}

// ---- stable radix sort of each worker's tokens ----
constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / kWave;
constexpr int kMaxBits = 10;                                           // of a digit

struct SortLds {
    alignas(16) uint16_t count[kSortWaves << kMaxBits];                // [wavefront][digit] of the wavefronts' tokens (at most 512)
    uint32_t base[1 << kMaxBits];
    uint32_t wave_sum[kSortWaves];
};

__device__ __forceinline__ uint32_t key_of(int tok, int V) { return (uint32_t)tok < (uint32_t)V ? (uint32_t)tok : (uint32_t)V; }

// Exclusive sum of v over the workgroup's threads (by lane shifts in the vector unit; LDS only between wavefronts).
__device__ __forceinline__ uint32_t exclusive_scan(SortLds& s, uint32_t v)
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    int x = (int)v;
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, true);     // from the lane one to the left, in rows of 16
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);    // the row before's last lane, into rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);    // lane 31, into the upper half
    if (lane == kWave - 1) s.wave_sum[wave] = (uint32_t)x;
    __syncthreads();
    uint32_t before = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
        const uint32_t n = s.wave_sum[w];
        before += w < wave ? n : 0;
    }
    return before + (uint32_t)x - v;
}

// Rank of every token of the workgroup among those of its digit: in its wavefront (rank) and over the wavefronts before it
// (left in count); equal digits keep their order: wavefronts, rounds of a wavefront, lanes.  Thread d gets the number of
// tokens of digit d.  The caller's next barrier makes count whole.
template <int EACH>
__device__ __forceinline__ uint32_t rank_tile(SortLds& s, const uint32_t (&digit)[EACH], uint32_t (&rank)[EACH], int bits)
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, bins = 1 << bits;
    for (int i = threadIdx.x; i < (kSortWaves << bits) / 2; i += kSortThreads) reinterpret_cast<uint32_t*>(s.count)[i] = 0;
    __syncthreads();
    const uint64_t below = (1ull << lane) - 1;
    uint16_t* count = s.count + (wave << bits);
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        uint32_t lo = ~0u, hi = ~0u;                                   // lanes of the same digit
#pragma unroll
        for (int b = 0; b < kMaxBits; ++b) {
            if (b < bits) {
                const uint32_t mine = (uint32_t)((int32_t)(digit[k] << (31 - b)) >> 31);
                const uint64_t set = __ballot(mine != 0);
                lo &= ~((uint32_t)set ^ mine);
                hi &= ~((uint32_t)(set >> 32) ^ mine);
            }
        }
        const uint64_t same = (uint64_t)hi << 32 | lo;
        const uint32_t seen = count[digit[k]];
        rank[k] = seen + (uint32_t)__popcll(same & below);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if ((same & below) == 0) count[digit[k]] = (uint16_t)(seen + (uint32_t)__popcll(same));       // its first lane
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    __syncthreads();
    uint32_t sum = 0;
    if ((int)threadIdx.x < bins) {
        uint32_t c[kSortWaves];
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) c[w] = s.count[(w << bits) + threadIdx.x];
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            s.count[(w << bits) + threadIdx.x] = (uint16_t)sum;
            sum += c[w];
        }
    }
    return sum;
}

// A digit's turn: how many tokens of each digit every tile of EACH * kSortThreads has ...
template <int EACH>
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const int32_t* __restrict__ tokens, int64_t ld_tokens,
                                                                  const uint32_t* __restrict__ keys_in, int T, int V, int bits, int shift,
                                                                  uint32_t* __restrict__ counts)
{
    __shared__ uint32_t bin[1 << kMaxBits];
    const int bins = 1 << bits;
    for (int i = threadIdx.x; i < bins; i += kSortThreads) bin[i] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * (EACH * kSortThreads);
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
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
template <int EACH>
__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(const int32_t* __restrict__ tokens, int64_t ld_tokens,
                                                                  const uint32_t* __restrict__ keys_in, const int32_t* __restrict__ pos_in,
                                                                  int T, int V, int bits, int shift, const uint32_t* __restrict__ counts,
                                                                  uint32_t* __restrict__ keys, int32_t* __restrict__ pos)
{
    __shared__ SortLds s;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, bins = 1 << bits;
    const int64_t off = (int64_t)blockIdx.y * T;
    const int64_t first = (int64_t)blockIdx.x * (EACH * kSortThreads) + wave * (kWave * EACH) + lane;
    uint32_t key[EACH], digit[EACH], rank[EACH];
    int32_t at[EACH];
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        const int64_t i = first + k * kWave;
        key[k] = 0xFFFFFFFFu;                                          // past the end of the list: behind all others of its digit
        at[k] = -1;
        if (i < T) {
            key[k] = keys_in ? keys_in[off + i] : key_of(tokens[blockIdx.y * ld_tokens + i], V);
            at[k] = keys_in ? pos_in[off + i] : (int32_t)i;
        }
        digit[k] = (key[k] >> shift) & (uint32_t)(bins - 1);
    }
    // where the tile's tokens of each digit begin (thread d: digit d)
    uint32_t all = 0, before = 0;
    if ((int)threadIdx.x < bins) {
        const uint32_t* c = counts + (int64_t)blockIdx.y * gridDim.x * bins + threadIdx.x;
#pragma unroll 8
        for (unsigned b = 0; b < gridDim.x; ++b) {
            const uint32_t n = c[(int64_t)b * bins];
            before += b < blockIdx.x ? n : 0;
            all += n;
        }
    }
    const uint32_t smaller = exclusive_scan(s, all);
    if ((int)threadIdx.x < bins) s.base[threadIdx.x] = smaller + before;
    rank_tile<EACH>(s, digit, rank, bits);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        if (at[k] < 0) continue;
        const int64_t to = off + s.base[digit[k]] + s.count[(wave << bits) + digit[k]] + rank[k];
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
    float* parts;            // [W][spans][2][Dp]: of the split run that came into a span, of the one that began there
    float* table;
    int64_t ld_table;
    int T, V, D, Dp, spans, slices;
    int run_blocks;          // workgroups that sum runs; those after them write zeros to rows without tokens
    int zero_rows;           // table rows of such a workgroup
    float scale;
    int accumulate;
};

constexpr int kSpan = 16;              // sorted places of a team, and how far into the next span it may finish a run
constexpr uint32_t kNone = 0xFFFFFFFFu;

// Lane i's value to all lanes of a team of TL (i the same for all of a wavefront's teams).
template <int TL>
__device__ __forceinline__ uint32_t from_lane(uint32_t v, int i)
{
    if constexpr (TL == kWave) return (uint32_t)__builtin_amdgcn_readlane((int)v, i);
    else return (uint32_t)__shfl((int)v, i, TL);
}

// TL lanes make a team: they own TL * E columns of one span.  All it goes by - the keys and places of its span and of the next
// one, a lane each, and four keys around - is on its way at once.  With the zeros, 8 x 32768 x 1024 bf16 into 50000 rows 430 us:
// 5.0 TB/s of the 2.2 GB that have to move (the launches before and after it: 48 us).
template <class T, int E, int TL>
__device__ __forceinline__ void sum_runs(const GradArgs& a, int64_t task)
{
    constexpr int U = 8;                                               // rows in flight (8 x 32768 x 1023: 530 us, 554 with four; x 1024: 478 both)
    static_assert(TL >= kSpan && kSpan % U == 0, "a lane a place, whole batches");
    const int w = blockIdx.y;
    int span = (int)(task / a.slices), slice = (int)(task - (int64_t)span * a.slices);
    if (span >= a.spans) return;
    if constexpr (TL == kWave) {
        span = __builtin_amdgcn_readfirstlane(span);
        slice = __builtin_amdgcn_readfirstlane(slice);
    }
    const int lane = threadIdx.x % TL;
    const int col = (slice * TL + lane) * E;
    const uint32_t* keys = a.keys + (int64_t)w * a.T;
    const int32_t* pos = a.pos + (int64_t)w * a.T;
    const T* dout = static_cast<const T*>(a.dout) + w * a.ld_dout;
    float* table = a.table + w * a.ld_table;
    const int s0 = span * kSpan, m = a.T - s0 < kSpan ? a.T - s0 : kSpan;
    auto key_at = [&](int i) { return i >= 0 && i < a.T ? keys[i] : kNone; };
    const int mine = s0 + lane % kSpan;
    const uint32_t own_keys = key_at(mine), next_keys = key_at(mine + kSpan);
    const uint32_t own_places = mine < a.T ? (uint32_t)pos[mine] : 0, next_places = mine + kSpan < a.T ? (uint32_t)pos[mine + kSpan] : 0;
    const uint32_t before = key_at(s0 - 1), start_before = key_at(s0 - kSpan), long_before = key_at(s0 - kSpan - 1), after = key_at(s0 + m + kSpan);
    // A run is split if it goes on past the span after the one it begins in.  Of the run that comes into this span: it is if
    // it goes on past this one, or if it came into the span before as well.  Else the team before has summed it.
    const uint32_t k0 = from_lane<TL>(own_keys, 0), end = from_lane<TL>(own_keys, m - 1), next = m == kSpan ? from_lane<TL>(next_keys, 0) : kNone;
    const bool came_in = before == k0;
    const bool head_split = came_in && ((end == k0 && next == k0) || (start_before == k0 && long_before == k0));
    const bool tail_split = next == end && after == end;
    const uint32_t skip = came_in && !head_split ? k0 : kNone;         // a run that is not this team's
    uint32_t cur = k0;
    bool head = head_split;
    float acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.0f;

    auto flush = [&](bool tail) {
        if (cur >= (uint32_t)a.V || cur == skip) return;               // padding
        if (head || tail) {
            store_piece(a.parts + (((int64_t)w * a.spans + span) * 2 + (head ? 0 : 1)) * a.Dp, col, a.D, acc);
        } else {
            float* p = table + (int64_t)cur * a.D;
            float old[E] = {};
            if (a.accumulate) load_piece(p, col, a.D, old);
#pragma unroll
            for (int e = 0; e < E; ++e) old[e] += a.scale * acc[e];
            store_piece(p, col, a.D, old);
        }
    };
    // a batch of places of this span (first = 0 .. kSpan - U) or, where only `end` counts, of the next one
    auto batch = [&](uint32_t lane_keys, uint32_t lane_places, int first, bool own) {
        uint32_t key[U];
        Raw<T, E> row[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = (int)from_lane<TL>(lane_places, first + u);
            key[u] = from_lane<TL>(lane_keys, first + u);
            const bool mine = own ? first + u < m : key[u] == end;
            if (!mine) key[u] = (uint32_t)a.V;
            clear(row[u]);
            if (key[u] < (uint32_t)a.V && key[u] != skip) load_piece(dout + (int64_t)at * a.D, col, a.D, row[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (own && first + u < m && key[u] != cur) {
                flush(false);
                cur = key[u];
                head = false;
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] = 0.0f;
            }
            float v[E];
            unpack(row[u], v);
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] += v[e];
        }
    };
    for (int i = 0; i < m; i += U) batch(own_keys, own_places, i, true);
    // on into the next span as long as the last run goes on there, if it began here and is not split
    const bool finish = next == end && !tail_split && end != skip && !(head && end == k0);
    if (finish)
        for (int i = 0; i < kSpan && from_lane<TL>(next_keys, i) == end; i += U) batch(next_keys, next_places, i, false);
    flush(tail_split);
}

// Zeros to a wavefront's columns [c0, c1) of a row.
template <bool ALIGNED>
__device__ __forceinline__ void zero_columns(float* row, int c0, int c1)
{
    for (int c = c0 + 4 * (int)(threadIdx.x & (kWave - 1)); c < c1; c += 4 * kWave) {
        const v4f zero = {0.0f, 0.0f, 0.0f, 0.0f};
        if constexpr (ALIGNED) __builtin_nontemporal_store(zero, reinterpret_cast<v4f*>(row + c));
        else if (c + 4 <= c1) *reinterpret_cast<v4f_any*>(row + c) = zero;
        else {
            for (int e = c; e < c1; ++e) row[e] = 0.0f;
        }
    }
}

// Zeros to the rows of [v0, v0 + zero_rows) that no token names.
template <bool ALIGNED>
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
    for (int r = threadIdx.x / kWave; r < n; r += kThreads / kWave) {
        if (present[r >> 5] >> (r & 31) & 1u) continue;
        zero_columns<ALIGNED>(table + (v0 + r) * a.D, 0, a.D);
    }
}

// Rows to a workgroup; of tables from 2^28 rows on more, so that their workgroups fit one launch (2^28 rows of 16 columns 7.4 ms,
// 10.7 with 64 a workgroup).
constexpr int kZeroRows = 64, kMoreZeroRows = 1024;
constexpr int kManyRows = 1 << 28;

template <class T, int E, int TL, bool ALIGNED>
__global__ __launch_bounds__(kThreads) void grad_runs_kernel(GradArgs a)
{
    __shared__ uint32_t present[kMoreZeroRows / 32];
    if ((int)blockIdx.x < a.run_blocks) sum_runs<T, E, TL>(a, (int64_t)blockIdx.x * (kThreads / TL) + threadIdx.x / TL);
    else zero_rows<ALIGNED>(a, (int64_t)((int)blockIdx.x - a.run_blocks) * a.zero_rows, present);
}

// Split runs.  A workgroup looks at the ends of kJoinSpans spans, a lane each, for such runs that began there (few are), for
// kJoinCols columns; its wavefronts take those in turn and add up a run's parts, or share it if the parts are many.  26 us after
// 8 lists of 32768 tokens drawn as 1/rank: dependent loads of keys, and the most frequent token's parts one after the other.
constexpr int kJoinSpans = 16, kJoinShared = 32, kJoinCols = 4 * kWave;
static_assert(kJoinSpans <= kWave, "one wavefront looks");
__global__ __launch_bounds__(kThreads) void grad_join_kernel(GradArgs a)
{
    constexpr int waves = kThreads / kWave;
    __shared__ float sum[waves][kJoinCols];
    __shared__ int begun[kJoinSpans], shared_parts[kJoinSpans], runs;
    const int w = blockIdx.y;
    const uint32_t* keys = a.keys + (int64_t)w * a.T;
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int col0 = blockIdx.z * kJoinCols, col = col0 + 4 * lane;
    float* table = a.table + w * a.ld_table;
    if (wave == 0) {
        const int span = blockIdx.x * kJoinSpans + lane;
        const int64_t s0 = (int64_t)span * kSpan, s1 = s0 + kSpan;
        bool split = false;
        if (lane < kJoinSpans && s1 + kSpan < a.T) {
            const uint32_t cur = keys[s1 - 1], next = keys[s1], after = keys[s1 + kSpan], start = keys[s0], before = s0 > 0 ? keys[s0 - 1] : ~0u;
            split = next == cur && after == cur && cur < (uint32_t)a.V && !(start == cur && before == cur);
        }
        const uint64_t mask = __ballot(split);
        if (split) begun[__popcll(mask & ((1ull << lane) - 1))] = span;
        if (lane == 0) runs = __popcll(mask);
    }
    __syncthreads();
    const int n_runs = runs;
    auto add = [&](int span, int p0, int p1) {                         // part 0 began in the span, the others came into theirs
        v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
        const float* first = a.parts + ((int64_t)w * a.spans + span) * 2 * a.Dp + col;
        if (col < a.Dp) {
#pragma unroll 8
            for (int p = p0; p < p1; ++p) acc += *reinterpret_cast<const v4f*>(first + (int64_t)(2 * p + (p == 0 ? 1 : 0)) * a.Dp);
        }
        return acc;
    };
    for (int k = wave; k < n_runs; k += waves) {
        const int span = begun[k], s1 = (span + 1) * kSpan;
        const uint32_t cur = keys[s1];
        int n = 3;                                                     // parts: the spans after it that begin with its key
        for (;;) {
            const int64_t i = s1 + (int64_t)(n - 1 + lane) * kSpan;
            const uint64_t goes_on = __ballot(i < a.T && keys[i] == cur);
            if (goes_on != ~0ull) {
                n += __builtin_ctzll(~goes_on);
                break;
            }
            n += kWave;
        }
        if (lane == 0) shared_parts[k] = n > kJoinShared ? n : 0;
        if (n > kJoinShared) continue;
        float* row = table + (int64_t)cur * a.D;
        const v4f acc = add(span, 0, n);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (col + e < a.D) row[col + e] = (a.accumulate ? row[col + e] : 0.0f) + a.scale * acc[e];
    }
    __syncthreads();
    for (int k = 0; k < n_runs; ++k) {                                 // long ones, together
        const int n = shared_parts[k];
        if (n == 0) continue;
        const int span = begun[k];
        const int per = (n + waves - 1) / waves, p0 = wave * per, p1 = p0 + per < n ? p0 + per : n;
        *reinterpret_cast<v4f*>(&sum[wave][4 * lane]) = add(span, p0, p1);
        __syncthreads();
        const int c = col0 + (int)threadIdx.x;
        if (c < a.D) {
            float t = 0.0f;
#pragma unroll
            for (int v = 0; v < waves; ++v) t += sum[v][threadIdx.x];
            float* to = table + (int64_t)keys[(span + 1) * kSpan] * a.D + c;
            *to = (a.accumulate ? *to : 0.0f) + a.scale * t;
        }
        __syncthreads();
    }
}

// ---- the gradient in one launch ----
constexpr int kSmallTokens = LSGD_EMBED_GRAD_ONE_LAUNCH;
static_assert(kSmallTokens == 8 * kSortThreads, "a workgroup sorts them, eight a thread");
constexpr int kSmallRows = 1 << 14;                // table rows whose zeros a workgroup may write
constexpr int kSmallShared = 16;                   // places of a run from which on a workgroup's wavefronts share it

struct SmallArgs {
    const int32_t* tokens;
    int64_t ld_tokens;
    int bits, passes;
    int span;                                      // sorted places whose runs a workgroup sums
    int rows;                                      // table rows whose zeros it writes
    int slices;                                    // of 64 * E columns, that it takes
};

// 4 x 2048 x 512 bf16, added to tables of 65536 rows, 14 us; 3 x 517 x 101 fp32 7: the passes of the sort one after the other,
// then a round of loads.  Where tables are large their zeros take the time (16 x 8192 x 1024 into 32768 rows 566 us, 4.3 TB/s).
template <class T, int E, bool ALIGNED, int EACH>
__global__ __launch_bounds__(kSortThreads) void grad_small_kernel(GradArgs a, SmallArgs q)
{
    constexpr int U = 8, cols = kWave * E;
    __shared__ uint32_t key[EACH * kSortThreads];
    __shared__ uint16_t pos[EACH * kSortThreads];
    __shared__ union {
        SortLds sort;
        uint32_t present[kSmallRows / 32];
        float sum[kSortWaves][cols];
    } s;
    __shared__ int shared_run[EACH * kSortThreads / kSmallShared], shared_places[EACH * kSortThreads / kSmallShared], shared_runs;
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), w = blockIdx.y;
    const int32_t* tokens = q.tokens + w * q.ld_tokens;
    const int first = wave * (kWave * EACH) + lane;
    {
        uint32_t k0[EACH], digit[EACH], rank[EACH], p0[EACH];
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            p0[k] = first + k * kWave;
            k0[k] = (int)p0[k] < a.T ? key_of(tokens[p0[k]], a.V) : 0xFFFFFFFFu;       // past the end: stays behind all others
        }
        for (int p = 0; p < q.passes; ++p) {
#pragma unroll
            for (int k = 0; k < EACH; ++k) digit[k] = (k0[k] >> (p * q.bits)) & ((1u << q.bits) - 1);
            const uint32_t mine = rank_tile<EACH>(s.sort, digit, rank, q.bits);
            const uint32_t smaller = exclusive_scan(s.sort, mine);
            if ((int)threadIdx.x < 1 << q.bits) s.sort.base[threadIdx.x] = smaller;
            __syncthreads();
#pragma unroll
            for (int k = 0; k < EACH; ++k) {
                const uint32_t to = s.sort.base[digit[k]] + s.sort.count[(wave << q.bits) + digit[k]] + rank[k];
                key[to] = k0[k];
                pos[to] = (uint16_t)p0[k];
            }
            __syncthreads();
            if (p + 1 < q.passes) {
#pragma unroll
                for (int k = 0; k < EACH; ++k) {
                    k0[k] = key[first + k * kWave];
                    p0[k] = pos[first + k * kWave];
                }
                __syncthreads();
            }
        }
    }
    const int slice0 = blockIdx.z * q.slices, col_end = (slice0 + q.slices) * cols < a.D ? (slice0 + q.slices) * cols : a.D;
    const T* dout = static_cast<const T*>(a.dout) + w * a.ld_dout;
    float* table = a.table + w * a.ld_table;
    if (threadIdx.x == 0) shared_runs = 0;
    if (!a.accumulate) {
        const int64_t v0 = (int64_t)blockIdx.x * q.rows;
        const int n = (int)(a.V - v0 < q.rows ? (a.V - v0 < 0 ? 0 : a.V - v0) : q.rows);
        for (int i = threadIdx.x; i < (n + 31) / 32; i += kSortThreads) s.present[i] = 0;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            const uint32_t v = key[k * kSortThreads + threadIdx.x] - (uint32_t)v0;      // what is no row here wraps past n
            if (v < (uint32_t)n) atomicOr(&s.present[v >> 5], 1u << (v & 31));
        }
        __syncthreads();
        for (int r = wave; r < n; r += kSortWaves) {
            if (s.present[r >> 5] >> (r & 31) & 1u) continue;
            zero_columns<ALIGNED>(table + (v0 + r) * a.D, slice0 * cols, col_end);
        }
    }
    __syncthreads();

    float acc[E];
    auto add_places = [&](int p0, int p1, int col) {
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = 0.0f;
        for (int b = p0; b < p1; b += U) {
            Raw<T, E> row[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                clear(row[u]);
                if (b + u < p1) {
                    const int at = __builtin_amdgcn_readfirstlane((int)pos[b + u]);
                    load_piece(dout + (int64_t)at * a.D, col, a.D, row[u]);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float v[E];
                unpack(row[u], v);
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] += v[e];
            }
        }
    };
    const int lo = blockIdx.x * q.span, hi = lo + q.span < a.T ? lo + q.span : a.T;
    const int each = (q.span + kSortWaves - 1) / kSortWaves;
    const int j1 = lo + (wave + 1) * each < hi ? lo + (wave + 1) * each : hi;
    for (int j = lo + wave * each; j < j1; ++j) {
        const uint32_t v = __builtin_amdgcn_readfirstlane(key[j]);
        if (v >= (uint32_t)a.V) break;                                 // padding, behind all rows
        if (j > 0 && __builtin_amdgcn_readfirstlane(key[j - 1]) == (int)v) continue;
        int n = 0;
        for (;;) {
            const int i = j + n + lane;
            const uint64_t same = __ballot(i < a.T && key[i] == v);
            if (same != ~0ull) {
                n += __builtin_ctzll(~same);
                break;
            }
            n += kWave;
        }
        if (n > kSmallShared) {
            if (lane == 0) {
                const int k = atomicAdd(&shared_runs, 1);
                shared_run[k] = j;
                shared_places[k] = n;
            }
            continue;
        }
        for (int c = 0; c < q.slices; ++c) {
            const int col0 = (slice0 + c) * cols, col = col0 + lane * E;
            if (col0 >= a.D) break;
            float* p = table + (int64_t)v * a.D;
            float old[E] = {};
            if (a.accumulate) load_piece(p, col, a.D, old);
            add_places(j, j + n, col);
#pragma unroll
            for (int e = 0; e < E; ++e) old[e] += a.scale * acc[e];
            store_piece(p, col, a.D, old);
        }
    }
    __syncthreads();
    for (int k = 0; k < shared_runs; ++k) {
        const int j = shared_run[k], n = shared_places[k];
        float* p = table + (int64_t)key[j] * a.D;
        for (int c = 0; c < q.slices; ++c) {
            const int col0 = (slice0 + c) * cols, col = col0 + lane * E;
            if (col0 >= a.D) break;
            add_places(j + n * wave / kSortWaves, j + n * (wave + 1) / kSortWaves, col);
            const int at = piece_start<E>(col, a.D) - col0;
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (at + e >= lane * E) s.sum[wave][at + e] = acc[e];
            __syncthreads();
            if ((int)threadIdx.x < cols && col0 + (int)threadIdx.x < a.D) {
                float t = 0.0f;
#pragma unroll
                for (int v = 0; v < kSortWaves; ++v) t += s.sum[v][threadIdx.x];
                float* to = p + col0 + threadIdx.x;
                *to = (a.accumulate ? *to : 0.0f) + a.scale * t;
            }
            __syncthreads();
        }
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

constexpr int kMaxTokens = 1 << 24, kMaxRows = (1 << 30) - 1, kMaxWidth = 1 << 20;

lsgd_status check_shape(const char* who, int32_t W, int32_t T, int32_t V, int32_t D)
{
    if (W <= 0 || W > LSGD_MAX_WORKERS) return set_error(LSGD_ERR_SHAPE, "%s: W=%d outside [1,%d]", who, (int)W, LSGD_MAX_WORKERS);
    if (T < 0) return set_error(LSGD_ERR_SHAPE, "%s: T=%d is negative", who, (int)T);
    if (V <= 0 || D <= 0) return set_error(LSGD_ERR_SHAPE, "%s: V=%d and D=%d must be positive", who, (int)V, (int)D);
    if (T > kMaxTokens || V > kMaxRows || D > kMaxWidth)
        return set_error(LSGD_ERR_UNSUPPORTED, "%s: T=%d, V=%d or D=%d beyond the %d tokens, %d rows and %d columns a worker may have", who, (int)T, (int)V, (int)D,
                         kMaxTokens, kMaxRows, kMaxWidth);
    return LSGD_OK;
}

struct Plan {
    int bits, passes, each, tiles;     // of the sort
    int spans, Dp;
    size_t keys[2], pos[2], counts, parts, total;
};

// No memory for what takes one launch.  Sort tiles of 2048 tokens while a list has few of them (a tile adds up the counts of all
// others), of 8192 then.
Plan make_plan(int W, int T, int V, int D)
{
    Plan p{};
    p.total = kAlign;
    int nb = 1;
    while (V >> nb) ++nb;                                              // keys are 0 .. V
    p.passes = (nb + kMaxBits - 1) / kMaxBits;
    p.bits = (nb + p.passes - 1) / p.passes;
    if (T <= kSmallTokens) return p;
    p.each = T <= 64 * 2 * kSortThreads ? 2 : 8;
    p.tiles = (T - 1) / (p.each * kSortThreads) + 1;
    p.spans = (T - 1) / kSpan + 1;
    p.Dp = (D + 7) / 8 * 8;
    const size_t list = align_up(sizeof(uint32_t) * (size_t)W * (size_t)T);
    size_t o = 0;
    for (int k = 0; k < 2; ++k) {
        p.keys[k] = o; o += k == 0 || p.passes > 1 ? list : 0;
        p.pos[k] = o;  o += k == 0 || p.passes > 1 ? list : 0;
    }
    p.counts = o; o += align_up(sizeof(uint32_t) * ((size_t)W * (size_t)p.tiles << p.bits));
    p.parts = o;  o += align_up(sizeof(float) * (size_t)W * (size_t)p.spans * 2 * (size_t)p.Dp);
    p.total = o;
    return p;
}

constexpr int64_t kLaunchThreads = 1ll << 32;                          // a launch has fewer

// Workgroups that sum runs, of teams of `lanes`, and that write zeros.
struct RunPlan {
    int lanes, slices, zero_rows;
    int64_t run_blocks, zero_blocks;
};
RunPlan run_plan(const Plan& p, int V, int D, int elements, int accumulate)
{
    RunPlan r;
    const int lanes = (D - 1) / elements + 1;
    r.lanes = lanes <= 16 ? 16 : lanes <= 32 ? 32 : 64;
    r.slices = (D - 1) / (r.lanes * elements) + 1;
    r.zero_rows = V < kManyRows ? kZeroRows : kMoreZeroRows;
    r.run_blocks = ((int64_t)p.spans * r.slices - 1) / (kThreads / r.lanes) + 1;
    r.zero_blocks = accumulate ? 0 : (V - 1) / r.zero_rows + 1;
    return r;
}

template <class TI, class TO>
void launch_lookup(int W, int T, int V, int D, const void* table, int64_t ld_table, const int32_t* tokens, int64_t ld_tokens, float scale,
                   void* out, int64_t ld_out, hipStream_t s)
{
    TO* to = static_cast<TO*>(out);
    constexpr int E = kLookupPiece<TI, TO>;
    const int64_t pieces = (int64_t)T * ((D - 1) / E + 1);
    const dim3 grid((unsigned)((pieces - 1) / (kThreads * kLookupEach) + 1), (unsigned)W);
    const bool aligned = D % E == 0 && on(to, 16) && (W == 1 || ld_out % E == 0);
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, static_cast<const TI*>(table), ld_table, V, D, tokens, ld_tokens, T, scale, to, ld_out);
    };
    if (aligned) go(lookup_kernel<TI, TO, true>);
    else go(lookup_kernel<TI, TO, false>);
}

template <class T, int E, int TL, bool ALIGNED>
hipError_t launch_grad(GradArgs a, int W, const RunPlan& p, hipStream_t s)
{
    a.slices = p.slices;
    a.run_blocks = (int)p.run_blocks;
    a.zero_rows = p.zero_rows;
    hipLaunchKernelGGL((grad_runs_kernel<T, E, TL, ALIGNED>), dim3((unsigned)(p.run_blocks + p.zero_blocks), (unsigned)W), dim3(kThreads), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;                                     // there are no partial sums to join
    hipLaunchKernelGGL(grad_join_kernel, dim3((unsigned)((a.spans - 1) / kJoinSpans + 1), (unsigned)W, (unsigned)((a.D - 1) / kJoinCols + 1)),
                       dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

// A workgroup a compute unit (each sorts the list again; with two 517 tokens take 10.2 us instead of 7.4, 2048 20.6 instead of
// 13.8), fewer columns each rather than fewer places; two where the zeros of large tables are what takes the time (1000 tokens,
// 4 x 65536 x 1024: 216 us instead of 234; of 8192 tokens the second sort weighs more, 16 x 32768 x 1024: 566 and 534).
constexpr int kSmallGroups = 256;
constexpr int64_t kManyZeros = 128ll << 20;        // bytes of all tables
template <class T, int E, bool ALIGNED>
void launch_grad_small(const GradArgs& a, int W, SmallArgs q, hipStream_t s)
{
    const int slices = (a.D - 1) / (kWave * E) + 1;
    int z = 1;
    while (z < slices && (int64_t)W * z * a.T < 256 * 16) ++z;
    q.slices = (slices - 1) / z + 1;
    z = (slices - 1) / q.slices + 1;
    const bool zeros = !a.accumulate && 4ll * W * a.V * a.D >= kManyZeros;
    int n = std::max(1, (zeros ? 2 : 1) * kSmallGroups / (W * z));
    if (a.accumulate) n = std::min(n, a.T);
    else n = std::max(n, (a.V - 1) / kSmallRows + 1);
    q.span = (a.T - 1) / n + 1;
    q.rows = (a.V - 1) / n + 1;
    const dim3 grid((unsigned)n, (unsigned)W, (unsigned)z), block(kSortThreads);
    if (a.T <= kSortThreads) hipLaunchKernelGGL((grad_small_kernel<T, E, ALIGNED, 1>), grid, block, 0, s, a, q);
    else if (a.T <= 2 * kSortThreads) hipLaunchKernelGGL((grad_small_kernel<T, E, ALIGNED, 2>), grid, block, 0, s, a, q);
    else if (a.T <= 4 * kSortThreads) hipLaunchKernelGGL((grad_small_kernel<T, E, ALIGNED, 4>), grid, block, 0, s, a, q);
    else hipLaunchKernelGGL((grad_small_kernel<T, E, ALIGNED, 8>), grid, block, 0, s, a, q);
}

template <class T, int E>
hipError_t launch_grad_team(const GradArgs& a, int W, const RunPlan& p, bool aligned, hipStream_t s)
{
    if (aligned) {
        if (p.lanes == 16) return launch_grad<T, E, 16, true>(a, W, p, s);
        if (p.lanes == 32) return launch_grad<T, E, 32, true>(a, W, p, s);
        return launch_grad<T, E, 64, true>(a, W, p, s);
    }
    if (p.lanes == 16) return launch_grad<T, E, 16, false>(a, W, p, s);
    if (p.lanes == 32) return launch_grad<T, E, 32, false>(a, W, p, s);
    return launch_grad<T, E, 64, false>(a, W, p, s);
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
    if (W > 1 && (ld_table < 0 || (ld_tokens < T && ld_tokens != 0) || ld_out < (int64_t)T * D))
        return set_error(LSGD_ERR_SHAPE, "embed_lookup: a worker stride is smaller than what a worker has (ld_tokens=%lld, ld_out=%lld)",
                         (long long)ld_tokens, (long long)ld_out);
    const int64_t pieces = (int64_t)T * ((D - 1) / (table_is_bf16 | out_is_bf16 ? kLookupPiece<uint16_t, uint16_t> : kLookupPiece<float, float>) + 1);
    if (((pieces - 1) / (kThreads * kLookupEach) + 1) * kThreads >= kLaunchThreads)
        return set_error(LSGD_ERR_SHAPE, "embed_lookup: T=%d of D=%d is too large for one launch", (int)T, (int)D);
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
    if (W > 1 && ((ld_tokens < T && ld_tokens != 0) || (ld_dout < (int64_t)T * D && ld_dout != 0)))
        return set_error(LSGD_ERR_SHAPE, "embed_grad: a worker stride is smaller than what a worker has (ld_tokens=%lld, ld_dout=%lld)",
                         (long long)ld_tokens, (long long)ld_dout);
    const Plan p = make_plan(W, T, V, D);
    if (!workspace && T > kSmallTokens) return set_error(LSGD_ERR_INVALID_ARG, "embed_grad: workspace is NULL");
    if (!on(workspace, kAlign)) return set_error(LSGD_ERR_INVALID_ARG, "embed_grad: workspace must be 256-byte aligned");
    if (workspace && workspace_bytes < p.total) return set_error(LSGD_ERR_NOMEM, "embed_grad: workspace of %zu bytes < %zu needed", workspace_bytes, p.total);

    GradArgs a{};
    a.dout = dout; a.ld_dout = ld_dout;
    a.table = dtable; a.ld_table = ld_dtable;
    a.T = T; a.V = V; a.D = D;
    a.scale = scale; a.accumulate = accumulate;
    const bool aligned = D % 4 == 0 && on(dtable, 16) && (W == 1 || ld_dtable % 4 == 0);       // of the table's rows
    if (T <= kSmallTokens) {
        SmallArgs q{};
        q.tokens = tokens; q.ld_tokens = ld_tokens;
        q.bits = p.bits; q.passes = p.passes;
        if (dout_is_bf16) aligned ? launch_grad_small<uint16_t, 8, true>(a, W, q, s) : launch_grad_small<uint16_t, 8, false>(a, W, q, s);
        else aligned ? launch_grad_small<float, 4, true>(a, W, q, s) : launch_grad_small<float, 4, false>(a, W, q, s);
        e = hipGetLastError();
        if (e != hipSuccess) return set_error(LSGD_ERR_HIP, "embed_grad: %s", hipGetErrorString(e));
        return LSGD_OK;
    }
    const RunPlan runs = run_plan(p, V, D, dout_is_bf16 ? 8 : 4, accumulate);
    if ((runs.run_blocks + runs.zero_blocks) * kThreads >= kLaunchThreads)
        return set_error(LSGD_ERR_SHAPE, "embed_grad: T=%d of D=%d is too large for one launch", (int)T, (int)D);
    char* base = static_cast<char*>(workspace);
    uint32_t* keys[2] = {reinterpret_cast<uint32_t*>(base + p.keys[0]), reinterpret_cast<uint32_t*>(base + p.keys[1])};
    int32_t* pos[2] = {reinterpret_cast<int32_t*>(base + p.pos[0]), reinterpret_cast<int32_t*>(base + p.pos[1])};
    uint32_t* counts = reinterpret_cast<uint32_t*>(base + p.counts);
    const dim3 grid((unsigned)p.tiles, (unsigned)W);
    int at = 0;
    for (int k = 0; k < p.passes; ++k) {
        const uint32_t* kin = k ? keys[at] : nullptr;
        const int32_t* pin = k ? pos[at] : nullptr;
        if (k) at ^= 1;
        auto go = [&](auto count, auto place) {
            hipLaunchKernelGGL(count, grid, dim3(kSortThreads), 0, s, tokens, ld_tokens, kin, (int)T, (int)V, p.bits, k * p.bits, counts);
            hipLaunchKernelGGL(place, grid, dim3(kSortThreads), 0, s, tokens, ld_tokens, kin, pin, (int)T, (int)V, p.bits, k * p.bits, counts, keys[at], pos[at]);
        };
        if (p.each == 2) go(sort_count_kernel<2>, sort_place_kernel<2>);
        else go(sort_count_kernel<8>, sort_place_kernel<8>);
    }
    a.keys = keys[at]; a.pos = pos[at];
    a.parts = reinterpret_cast<float*>(base + p.parts);
    a.Dp = p.Dp; a.spans = p.spans;
    e = hipGetLastError();
    if (e == hipSuccess)
        e = dout_is_bf16 ? launch_grad_team<uint16_t, 8>(a, W, runs, aligned, s) : launch_grad_team<float, 4>(a, W, runs, aligned, s);
    if (e != hipSuccess) return set_error(LSGD_ERR_HIP, "embed_grad: %s", hipGetErrorString(e));
    return LSGD_OK;
}

} // extern "C"
