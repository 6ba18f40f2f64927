// Queries and keys before attention: each head's norm and the rotation by its token's position in one pass, and the gradients.
//
//   z = q x o w       q = (mean x^2 + eps)^-1/2  (or 1)
//   y = R z           pairs (a, b) of the first 2 n columns turned by the angle 2 pi pos f_i of pair i, times the magnitude:
//                     a' = m (a cos - b sin),  b' = m (a sin + b cos);  the other columns as they are
//
//   backward, from dy, with h = q x:  dz = R' dy;  dx = q (dz o w - h mean(dz o w o h));  dw = sum over tokens and heads dz o h
//
// Bound by memory: 8 x 8192 tokens of 32 and 8 heads of 128 bf16 in 236 to 260 us, 5.2 to 5.7 TB/s, as a copy of the same bytes (245); gradients of
// 8 x 4096 182 us in all, 5.6 TB/s.  Angles: a position far into a text times a frequency is thousands of turns, of which fp32 keeps too few
// bits; the product is made in 64 bits, whole turns are taken off, and the rest goes through sincospi in fp32.  All heads of a
// token turn alike, so a workgroup makes the table of its tokens once, in LDS, and its rows read it there.
//
// A team of lanes holds a head's row, two pieces of E columns a lane, a half of the rotated columns apart: either the partners
// of its pairs or, where neighbours are pairs, whole pairs.  Either way adjacent lanes' accesses are adjacent, and no value
// crosses lanes but the norm's sum.  E is the widest that divides both the half and the rest.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "heads.h"
#include "row_pieces.h"

using namespace lsgd;

namespace {

constexpr int kThreads = 256;
constexpr int kMaxColumns = 256;            // of a head

struct Args {
    Heads x[2], y[2], dx[2];                // queries, keys; forward: x -> y; backward: x, y = dy -> dx
    int H[2];
    const float* w[2];                      // NULL: ones
    int64_t ld_w[2];
    const int32_t* pos;                     // NULL: 0, 1, 2, ...
    int64_t ld_pos;
    const double* turns;                    // [half]
    float* stats;                           // [W][T][Hq + Hk]; forward: may be NULL
    float* parts;                           // backward: [W][workgroups][2][Dp] sums for dw, or NULL
    int T, D, Dp, half, lanes, tokens, norm;
    float eps, inv_d, magnitude;
};

// E elements as memory has them, and as fp32.  ONCE: past the caches, 16-byte aligned.
template <int BYTES> struct Word;
template <> struct Word<16> { using type = v4u_any; };
template <> struct Word<8> { using type = v2u_any; };
template <> struct Word<4> { using type = u32_any; };
template <> struct Word<2> { using type = uint16_t; };
template <class T, int E>
using Packed = typename Word<E * (int)sizeof(T)>::type;

template <bool ONCE, class T, int E>
__device__ __forceinline__ Packed<T, E> get(const T* p)
{
    if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const v4u*>(p));
    else return *reinterpret_cast<const Packed<T, E>*>(p);
}
template <class T, int E>
__device__ __forceinline__ void expand(const Packed<T, E>& v, float (&f)[E])
{
    T t[E];
    __builtin_memcpy(t, &v, sizeof(t));
#pragma unroll
    for (int e = 0; e < E; ++e) {
        if constexpr (sizeof(T) == 4) f[e] = t[e];
        else f[e] = bf16_to_f32(t[e]);
    }
}
template <bool ONCE, class T, int E>
__device__ __forceinline__ void put(T* p, const float (&f)[E])
{
    T t[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        if constexpr (sizeof(T) == 4) t[e] = f[e];
        else t[e] = f32_to_bf16_rne(f[e]);
    }
    Packed<T, E> v;
    __builtin_memcpy(&v, t, sizeof(t));
    if constexpr (ONCE) __builtin_nontemporal_store(static_cast<v4u>(v), reinterpret_cast<v4u*>(p));
    else *reinterpret_cast<Packed<T, E>*>(p) = v;
}

// Sum over a team of `lanes` adjacent lanes (a power of two), the same in all of them.
template <int CTRL>
__device__ __forceinline__ float add_lanes(float a)
{
    return a + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(a), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float team_sum(float a, int lanes)
{
    if (lanes >= 2) a = add_lanes<0xB1>(a);                // the other lane of a pair, the other pair, the other four, eight
    if (lanes >= 4) a = add_lanes<0x4E>(a);
    if (lanes >= 8) a = add_lanes<0x141>(a);
    if (lanes >= 16) a = add_lanes<0x140>(a);
    if (lanes >= 32) a += __shfl_xor(a, 16);
    if (lanes >= 64) a += __shfl_xor(a, 32);
    return a;
}

// x^-1/2 to a last bit (of what is below the normal values: of the smallest of those; NaN stays).
__device__ __forceinline__ float inverse_root(float x) { return __builtin_amdgcn_rsqf(x < 0x1p-126f ? 0x1p-126f : x); }

// Where a lane's N units of two pieces lie in a row.
template <int E, int N, bool NEIGHBOURS>
struct Unit {
    int a[N], b[N], angle[N];               // first columns; angle: first pair of piece a, or -1: not rotated
    bool has_a[N], has_b[N];
    __device__ __forceinline__ Unit(const Args& g, int lane)
    {
        const int turned = g.half / E, rest = (g.D - 2 * g.half) / E, left = (rest + 1) / 2;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int u = lane + n * g.lanes, j = u - turned;
            has_a[n] = j < left;
            angle[n] = j < 0 ? u * E : -1;
            if (E == 1 && NEIGHBOURS) {
                a[n] = 2 * u;
                b[n] = 2 * u + 1;
            } else {
                a[n] = u * E;
                b[n] = g.half + u * E;
                if (NEIGHBOURS && j < 0) angle[n] = u * E / 2;
            }
            if (j >= 0) {
                a[n] = 2 * g.half + j * E;
                b[n] = a[n] + left * E;
            }
            has_b[n] = has_a[n] && b[n] < g.D;
        }
    }
};

// cos and sin, times the magnitude, of the tokens t0 .. t0 + n of worker w: table[token][pair].
__device__ __forceinline__ void make_table(const Args& g, int w, int t0, int n, v2f* table)
{
    for (int i = threadIdx.x; i < n * g.half; i += kThreads) {
        const int k = i / g.half, p = i - k * g.half, t = t0 + k;
        const double a = (double)(g.pos ? g.pos[w * g.ld_pos + t] : t) * g.turns[p];
        float s, c;
        sincospif(2.0f * (float)(a - rint(a)), &s, &c);
        table[i] = v2f{c * g.magnitude, s * g.magnitude};
    }
}

// Turns the pairs of a unit, BACK: the other way.
template <int E, bool NEIGHBOURS, bool BACK>
__device__ __forceinline__ void turn(const v2f* cs, int half, float (&a)[E], float (&b)[E])
{
    auto one = [](v2f r, float& x, float& y) {
        const float c = r[0], s = BACK ? -r[1] : r[1], u = x * c - y * s;
        y = x * s + y * c;
        x = u;
    };
    if constexpr (NEIGHBOURS && E > 1) {
#pragma unroll
        for (int e = 0; e < E; e += 2) {
            one(cs[e / 2], a[e], a[e + 1]);
            one(cs[half / 2 + e / 2], b[e], b[e + 1]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) one(cs[e], a[e], b[e]);
    }
}

template <class T, int E, int N, class U>
__device__ __forceinline__ void weights(const Args& g, int which, int w, const U& at, float (&a)[N][E], float (&b)[N][E])
{
    const float* p = g.w[which] ? g.w[which] + w * g.ld_w[which] : nullptr;
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            a[n][e] = !at.has_a[n] ? 0.0f : p ? p[at.a[n] + e] : 1.0f;
            b[n][e] = !at.has_b[n] ? 0.0f : p ? p[at.b[n] + e] : 1.0f;
        }
}

// A team's rows of a workgroup's tokens: tokens outermost, adjacent teams adjacent heads.
struct RowWalk {
    int token, head;
    const int H, step;
    __device__ __forceinline__ RowWalk(int team, int teams, int heads) : token(team / heads), head(team % heads), H(heads), step(teams) {}
    __device__ __forceinline__ void next()
    {
        for (head += step; head >= H; head -= H) ++token;
    }
};

template <class T>
__device__ __forceinline__ T* row_of(const Heads& a, int w, int t, int h)
{
    return static_cast<T*>(a.p) + w * a.lb + t * a.lt + h * a.lh;
}

template <class T, int E, bool NEIGHBOURS, bool ONCE>
__global__ __launch_bounds__(kThreads) void qk_rotary_kernel(Args g)
{
    constexpr int N = E == 1 ? kMaxColumns / 128 : 1;
    extern __shared__ v2f table[];
    const int lane = threadIdx.x & (g.lanes - 1), team = threadIdx.x / g.lanes, teams = kThreads / g.lanes, w = blockIdx.y;
    const Unit<E, N, NEIGHBOURS> at(g, lane);
    const int t0 = blockIdx.x * g.tokens, tokens = g.T - t0 < g.tokens ? g.T - t0 : g.tokens;
    make_table(g, w, t0, tokens, table);
    __syncthreads();
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        const int H = g.H[which];
        if (H == 0) continue;
        float wa[N][E], wb[N][E];
        weights<T, E, N>(g, which, w, at, wa, wb);
        for (RowWalk r(team, teams, H); r.token < tokens; r.next()) {
            const T* x = row_of<const T>(g.x[which], w, t0 + r.token, r.head);
            Packed<T, E> pa[N], pb[N];
            float a[N][E], b[N][E], s = 0.0f;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if (at.has_a[n]) pa[n] = get<ONCE, T, E>(x + at.a[n]); else pa[n] = Packed<T, E>{};
                if (at.has_b[n]) pb[n] = get<ONCE, T, E>(x + at.b[n]); else pb[n] = Packed<T, E>{};
            }
#pragma unroll
            for (int n = 0; n < N; ++n) {
                expand<T, E>(pa[n], a[n]);
                expand<T, E>(pb[n], b[n]);
#pragma unroll
                for (int e = 0; e < E; ++e) s += a[n][e] * a[n][e] + b[n][e] * b[n][e];
            }
            float q = 1.0f;
            if (g.norm) {
                q = inverse_root(team_sum(s, g.lanes) * g.inv_d + g.eps);
                if (g.stats && lane == 0) g.stats[((int64_t)w * g.T + t0 + r.token) * (g.H[0] + g.H[1]) + (which ? g.H[0] : 0) + r.head] = q;
            }
            T* y = row_of<T>(g.y[which], w, t0 + r.token, r.head);
#pragma unroll
            for (int n = 0; n < N; ++n) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    a[n][e] *= q * wa[n][e];
                    b[n][e] *= q * wb[n][e];
                }
                if (at.angle[n] >= 0 && at.has_a[n]) turn<E, NEIGHBOURS, false>(table + r.token * g.half + at.angle[n], g.half, a[n], b[n]);
                if (at.has_a[n]) put<ONCE, T, E>(y + at.a[n], a[n]);
                if (at.has_b[n]) put<ONCE, T, E>(y + at.b[n], b[n]);
            }
        }
    }
}

template <class T, int E, bool NEIGHBOURS, bool ONCE>
__global__ __launch_bounds__(kThreads) void qk_rotary_grad_kernel(Args g)
{
    constexpr int N = E == 1 ? kMaxColumns / 128 : 1;
    extern __shared__ v2f table[];
    const int lane = threadIdx.x & (g.lanes - 1), team = threadIdx.x / g.lanes, teams = kThreads / g.lanes, w = blockIdx.y;
    const Unit<E, N, NEIGHBOURS> at(g, lane);
    const int which = blockIdx.z, H = g.H[which];          // queries, or keys
    if (H == 0) return;
    float da[N][E], db[N][E];                              // the lane's part of the weight's gradient, over its rows
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int e = 0; e < E; ++e) da[n][e] = db[n][e] = 0.0f;
    const bool whole = g.x[which].p != nullptr;            // absent: neither a norm nor a weight's gradient needs it
    float wa[N][E], wb[N][E];
    weights<T, E, N>(g, which, w, at, wa, wb);
    for (int64_t t64 = (int64_t)blockIdx.x * g.tokens; t64 < g.T; t64 += (int64_t)gridDim.x * g.tokens) {
        const int t0 = (int)t64, tokens = g.T - t0 < g.tokens ? g.T - t0 : g.tokens;
        __syncthreads();                                   // the last tokens' table has been read
        make_table(g, w, t0, tokens, table);
        __syncthreads();
        {
            for (RowWalk r(team, teams, H); r.token < tokens; r.next()) {
                const T* dy = row_of<const T>(g.y[which], w, t0 + r.token, r.head);
                const T* x = whole ? row_of<const T>(g.x[which], w, t0 + r.token, r.head) : nullptr;
                Packed<T, E> pa[N], pb[N], xa[N], xb[N];
                float a[N][E], b[N][E], ha[N][E], hb[N][E], s = 0.0f, q = 1.0f;
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    pa[n] = pb[n] = xa[n] = xb[n] = Packed<T, E>{};
                    if (at.has_a[n]) pa[n] = get<ONCE, T, E>(dy + at.a[n]);
                    if (at.has_b[n]) pb[n] = get<ONCE, T, E>(dy + at.b[n]);
                    if (whole && at.has_a[n]) xa[n] = get<ONCE, T, E>(x + at.a[n]);
                    if (whole && at.has_b[n]) xb[n] = get<ONCE, T, E>(x + at.b[n]);
                }
                if (g.norm) q = g.stats[((int64_t)w * g.T + t0 + r.token) * (g.H[0] + g.H[1]) + (which ? g.H[0] : 0) + r.head];
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    expand<T, E>(pa[n], a[n]);
                    expand<T, E>(pb[n], b[n]);
                    expand<T, E>(xa[n], ha[n]);
                    expand<T, E>(xb[n], hb[n]);
                    if (at.angle[n] >= 0 && at.has_a[n]) turn<E, NEIGHBOURS, true>(table + r.token * g.half + at.angle[n], g.half, a[n], b[n]);
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        ha[n][e] *= q;
                        hb[n][e] *= q;
                        da[n][e] += a[n][e] * ha[n][e];
                        db[n][e] += b[n][e] * hb[n][e];
                        a[n][e] *= wa[n][e];
                        b[n][e] *= wb[n][e];
                        s += a[n][e] * ha[n][e] + b[n][e] * hb[n][e];
                    }
                }
                if (g.norm) {
                    s = team_sum(s, g.lanes) * g.inv_d;
#pragma unroll
                    for (int n = 0; n < N; ++n)
#pragma unroll
                        for (int e = 0; e < E; ++e) {
                            a[n][e] = q * (a[n][e] - ha[n][e] * s);
                            b[n][e] = q * (b[n][e] - hb[n][e] * s);
                        }
                }
                T* dx = row_of<T>(g.dx[which], w, t0 + r.token, r.head);
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    if (at.has_a[n]) put<ONCE, T, E>(dx + at.a[n], a[n]);
                    if (at.has_b[n]) put<ONCE, T, E>(dx + at.b[n], b[n]);
                }
            }
        }
    }
    if (!g.parts) return;
    // the workgroup's teams add up theirs in order
    __shared__ float sum[kThreads * 2 * E * N];
    float* part = g.parts + ((int64_t)w * gridDim.x + blockIdx.x) * 2 * g.Dp;
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (at.has_a[n]) sum[team * g.D + at.a[n] + e] = da[n][e];
            if (at.has_b[n]) sum[team * g.D + at.b[n] + e] = db[n][e];
        }
    __syncthreads();
    for (int c = threadIdx.x; c < g.D; c += kThreads) {
        float s = 0.0f;
        for (int k = 0; k < teams; ++k) s += sum[k * g.D + c];
        part[which * g.Dp + c] = s;
    }
}

// dw[w, :] (+)= the sum over a worker's parts, each wavefront a stretch of them.
constexpr int kJoinThreads = 1024;
struct Join {
    float* dw[2];
    int64_t ld[2];
};
__global__ __launch_bounds__(kJoinThreads) void qk_join_kernel(const float* __restrict__ parts, int chunks, int D, int Dp, Join j, int accumulate)
{
    constexpr int waves = kJoinThreads / kWave;
    __shared__ float sum[waves][kWave];
    float* dw = j.dw[blockIdx.z];
    if (!dw) return;
    dw += blockIdx.y * j.ld[blockIdx.z];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, c = blockIdx.x * kWave + lane;
    const float* p = parts + ((int64_t)blockIdx.y * chunks * 2 + blockIdx.z) * Dp + c;
    const int per = (chunks + waves - 1) / waves, p0 = wave * per, p1 = p0 + per < chunks ? p0 + per : chunks;
    float acc = 0.0f;
    if (c < D) {
#pragma unroll 8
        for (int k = p0; k < p1; ++k) acc += p[(int64_t)k * 2 * Dp];
    }
    sum[wave][lane] = acc;
    __syncthreads();
    if (wave == 0 && c < D) {
        float s = 0.0f;
#pragma unroll
        for (int k = 0; k < waves; ++k) s += sum[k][lane];
        dw[c] = (accumulate ? dw[c] : 0.0f) + s;
    }
}

// ---- host ----
constexpr size_t kAlign = 256;
constexpr int kMaxHeads = 1024, kMaxTokens = 1 << 24;

#define LSGD_TRY(x)                         \
    do {                                    \
        const lsgd_status st_ = (x);        \
        if (st_ != LSGD_OK) return st_;     \
    } while (0)

lsgd_status check_shape(const char* who, int W, int T, int Hq, int Hk, int D, int R)
{
    if (W <= 0 || W > LSGD_MAX_WORKERS) return set_error(LSGD_ERR_SHAPE, "%s: W=%d outside [1,%d]", who, W, LSGD_MAX_WORKERS);
    if (T < 0 || T > kMaxTokens) return set_error(LSGD_ERR_SHAPE, "%s: T=%d outside [0,%d]", who, T, kMaxTokens);
    if (Hq <= 0 || Hk < 0 || Hq > kMaxHeads || Hk > kMaxHeads) return set_error(LSGD_ERR_SHAPE, "%s: Hq=%d outside [1,%d] or Hk=%d outside [0,%d]", who, Hq, kMaxHeads, Hk, kMaxHeads);
    if (D <= 0) return set_error(LSGD_ERR_SHAPE, "%s: D=%d must be positive", who, D);
    if (D > kMaxColumns) return set_error(LSGD_ERR_UNSUPPORTED, "%s: D=%d beyond %d columns", who, D, kMaxColumns);
    if (R < 0 || R > D || R % 2) return set_error(LSGD_ERR_SHAPE, "%s: R=%d must be even and within [0,%d]", who, R, D);
    return LSGD_OK;
}

// Columns a piece: what half the rotated columns and the rest can be divided into, at most 16 bytes.
int piece_of(int D, int R, int es)
{
    int E = 16 / es;
    while ((R / 2) % E || (D - R) % E) E /= 2;
    return E;
}
int lanes_of(int D, int R, int E)
{
    const int units = R / 2 / E + ((D - R) / E + 1) / 2;
    int lanes = 1;
    while (lanes < units && lanes < kWave) lanes *= 2;
    return lanes;
}
// Tokens whose table a workgroup makes at a time: about four rows a team, or one table entry a thread, but no more than leave two workgroups a
// compute unit.  (8 x 8192 tokens, 32 and 8 heads of 128: two rows 321 us, four 255, eight 257, 16 269; gradients of 8 x 4096: 205,
// 191, 201, 208.)
constexpr int kRowsPerTeam = 4, kComputeUnits = 256;
int tokens_of(int W, int T, int H, int R, int lanes)
{
    const int teams = kThreads / lanes;
    const int64_t most = std::max<int64_t>(1, (int64_t)W * T / (2 * kComputeUnits));
    return (int)std::min<int64_t>({most, (kRowsPerTeam * teams + H - 1) / H, std::max(1, 4096 / std::max(R, 1)), std::max(T, 1)});
}

struct GradPlan {
    int groups, Dp;
    size_t bytes;
};
constexpr int kGroupsGrad = 8 * kComputeUnits;      // workgroups in all, each a part of dw's sums (three, six or sixteen a compute unit: within 1 %)
GradPlan grad_plan(int W, int T, int Hq, int Hk, int D, int R, int es)
{
    GradPlan p;
    const int tokens = tokens_of(W, T, Hq + Hk, R, lanes_of(D, R, piece_of(D, R, es)));
    p.groups = (int)std::min<int64_t>((T + tokens - 1) / tokens, std::max(1, kGroupsGrad / W));
    p.Dp = (D + 7) / 8 * 8;
    p.bytes = std::max<size_t>(kAlign, sizeof(float) * (size_t)W * (size_t)p.groups * 2 * (size_t)p.Dp);
    return p;
}

lsgd_status check_weights(const char* who, const char* name, const float* w, int64_t ld, int W, int D, bool written)
{
    if (!w) return LSGD_OK;
    if (!on(w, 4)) return set_error(LSGD_ERR_INVALID_ARG, "%s: %s is not aligned to its element", who, name);
    if (W > 1 && (ld < 0 || (written && ld < D))) return set_error(LSGD_ERR_SHAPE, "%s: %s: worker stride %lld for D=%d", who, name, (long long)ld, D);
    return LSGD_OK;
}

lsgd_status check_positions(const char* who, const int32_t* pos, int64_t ld, const double* turns, int W, int T, int R)
{
    if (!on(pos, 4)) return set_error(LSGD_ERR_INVALID_ARG, "%s: positions are not aligned to their element", who);
    if (pos && W > 1 && ld != 0 && ld < T) return set_error(LSGD_ERR_SHAPE, "%s: ld_positions=%lld for T=%d", who, (long long)ld, T);
    if (R && !turns) return set_error(LSGD_ERR_INVALID_ARG, "%s: turns are required", who);
    if (!on(turns, 8)) return set_error(LSGD_ERR_INVALID_ARG, "%s: turns are not aligned to their element", who);
    return LSGD_OK;
}

// Calls launch(type, E, neighbours, once) for what is at hand.
template <class F>
void dispatch(bool bf16, int E, bool neighbours, bool once, F launch)
{
    auto paired = [&](auto type, auto e, auto streamed) {
        if (neighbours) launch(type, e, std::true_type{}, streamed);
        else launch(type, e, std::false_type{}, streamed);
    };
    auto typed = [&](auto type) {
        constexpr int widest = 16 / (int)sizeof(decltype(type));
        if (E == widest) {
            const std::integral_constant<int, widest> e{};
            if (once) paired(type, e, std::true_type{});
            else paired(type, e, std::false_type{});
        } else if (E == 4) {
            paired(type, std::integral_constant<int, 4>{}, std::false_type{});
        } else if (E == 2) {
            paired(type, std::integral_constant<int, 2>{}, std::false_type{});
        } else {
            paired(type, std::integral_constant<int, 1>{}, std::false_type{});
        }
    };
    if (bf16) typed(uint16_t{});
    else typed(float{});
}

} // namespace

extern "C" {

lsgd_status lsgd_qk_rotary(const lsgd_qk_rotary_args* p, void* hip_stream)
{
    const char* who = "qk_rotary";
    if (!p) return set_error(LSGD_ERR_INVALID_ARG, "%s: arguments are NULL", who);
    const int W = p->W, T = p->T, D = p->D, R = p->R, es = p->is_bf16 ? 2 : 4;
    LSGD_TRY(check_shape(who, W, T, p->Hq, p->Hk, D, R));
    if (p->is_bf16 & ~1 || p->norm & ~1 || p->interleaved & ~1) return set_error(LSGD_ERR_INVALID_ARG, "%s: is_bf16, norm and interleaved must be 0 or 1", who);
    if (!std::isfinite(p->magnitude)) return set_error(LSGD_ERR_INVALID_ARG, "%s: magnitude must be finite", who);
    if (p->norm && (!std::isfinite(p->eps) || p->eps <= 0.0f)) return set_error(LSGD_ERR_INVALID_ARG, "%s: eps must be finite and positive", who);
    if (T == 0) return LSGD_OK;
    LSGD_TRY(check_heads(who, "q", p->q, W, T, p->Hq, D, es, true, false));
    LSGD_TRY(check_heads(who, "q_out", p->q_out, W, T, p->Hq, D, es, true, true));
    LSGD_TRY(check_heads(who, "k", p->k, W, T, p->Hk, D, es, p->Hk > 0, false));
    LSGD_TRY(check_heads(who, "k_out", p->k_out, W, T, p->Hk, D, es, p->Hk > 0, true));
    LSGD_TRY(check_positions(who, p->positions, p->ld_positions, p->turns, W, T, R));
    LSGD_TRY(check_weights(who, "w_q", p->w_q, p->ld_w_q, W, D, false));
    LSGD_TRY(check_weights(who, "w_k", p->w_k, p->ld_w_k, W, D, false));
    if (!on(p->stats, 4)) return set_error(LSGD_ERR_INVALID_ARG, "%s: stats are not aligned to their element", who);
    const int E = piece_of(D, R, es);
    Args g{};
    g.x[0] = heads(p->q); g.x[1] = heads(p->k);
    g.y[0] = heads(p->q_out); g.y[1] = heads(p->k_out);
    g.H[0] = p->Hq; g.H[1] = p->Hk;
    g.w[0] = p->w_q; g.w[1] = p->w_k;
    g.ld_w[0] = W > 1 ? p->ld_w_q : 0; g.ld_w[1] = W > 1 ? p->ld_w_k : 0;
    g.pos = p->positions; g.ld_pos = W > 1 ? p->ld_positions : 0;
    g.turns = p->turns;
    g.stats = p->stats;
    g.T = T; g.D = D; g.half = R / 2; g.norm = p->norm;
    g.lanes = lanes_of(D, R, E);
    g.tokens = tokens_of(W, T, p->Hq + p->Hk, R, g.lanes);
    g.eps = p->eps; g.inv_d = 1.0f / (float)D; g.magnitude = p->magnitude;
    bool once = true;
    for (const lsgd_heads* a : {&p->q, &p->q_out}) once = once && wide_heads(*a, W, T, p->Hq, es);
    for (const lsgd_heads* a : {&p->k, &p->k_out}) once = once && wide_heads(*a, W, T, p->Hk, es);
    const dim3 grid((unsigned)((T + g.tokens - 1) / g.tokens), (unsigned)W);
    if ((double)grid.x * W * kThreads >= 4294967296.0) return set_error(LSGD_ERR_SHAPE, "%s: W=%d, T=%d are too large for one launch", who, W, T);
    dispatch(p->is_bf16, E, p->interleaved, once, [&](auto type, auto e, auto neighbours, auto streamed) {
        hipLaunchKernelGGL((qk_rotary_kernel<decltype(type), decltype(e)::value, decltype(neighbours)::value, decltype(streamed)::value>), grid,
                           dim3(kThreads), sizeof(v2f) * (size_t)std::max(1, g.tokens * g.half), static_cast<hipStream_t>(hip_stream), g);
    });
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return set_error(LSGD_ERR_HIP, "%s: %s", who, hipGetErrorString(err));
    return LSGD_OK;
}

size_t lsgd_qk_rotary_grad_workspace_bytes(int32_t W, int32_t T, int32_t Hq, int32_t Hk, int32_t D, int32_t R, int32_t is_bf16)
{
    if (check_shape("qk_rotary_grad", W, T, Hq, Hk, D, R) != LSGD_OK) return 0;
    return grad_plan(W, T, Hq, Hk, D, R, is_bf16 ? 2 : 4).bytes;
}

lsgd_status lsgd_qk_rotary_grad(const lsgd_qk_rotary_grad_args* p, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    const char* who = "qk_rotary_grad";
    if (!p) return set_error(LSGD_ERR_INVALID_ARG, "%s: arguments are NULL", who);
    const int W = p->W, T = p->T, D = p->D, R = p->R, es = p->is_bf16 ? 2 : 4;
    LSGD_TRY(check_shape(who, W, T, p->Hq, p->Hk, D, R));
    if (p->is_bf16 & ~1 || p->norm & ~1 || p->interleaved & ~1 || p->accumulate & ~1)
        return set_error(LSGD_ERR_INVALID_ARG, "%s: is_bf16, norm, interleaved and accumulate must be 0 or 1", who);
    if (!std::isfinite(p->magnitude)) return set_error(LSGD_ERR_INVALID_ARG, "%s: magnitude must be finite", who);
    LSGD_TRY(check_weights(who, "w_q", p->w_q, p->ld_w_q, W, D, false));
    LSGD_TRY(check_weights(who, "w_k", p->w_k, p->ld_w_k, W, D, false));
    LSGD_TRY(check_weights(who, "dw_q", p->dw_q, p->ld_dw_q, W, D, true));
    LSGD_TRY(check_weights(who, "dw_k", p->dw_k, p->ld_dw_k, W, D, true));
    if (p->Hk == 0 && p->dw_k) return set_error(LSGD_ERR_INVALID_ARG, "%s: dw_k has no meaning without keys", who);
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    const GradPlan plan = grad_plan(W, T, p->Hq, p->Hk, D, R, es);
    const Join join = {{p->dw_q, p->dw_k}, {p->ld_dw_q, p->ld_dw_k}};
    const bool sums = p->dw_q || p->dw_k;
    if (T > 0) {
        const int E = piece_of(D, R, es);
        const bool need_q = p->norm || p->dw_q, need_k = p->Hk > 0 && (p->norm || p->dw_k);
        LSGD_TRY(check_heads(who, "dq_out", p->dq_out, W, T, p->Hq, D, es, true, false));
        LSGD_TRY(check_heads(who, "dk_out", p->dk_out, W, T, p->Hk, D, es, p->Hk > 0, false));
        LSGD_TRY(check_heads(who, "q", p->q, W, T, p->Hq, D, es, need_q || p->q.data, false));
        LSGD_TRY(check_heads(who, "k", p->k, W, T, p->Hk, D, es, need_k || (p->Hk > 0 && p->k.data), false));
        LSGD_TRY(check_heads(who, "dq", p->dq, W, T, p->Hq, D, es, true, true));
        LSGD_TRY(check_heads(who, "dk", p->dk, W, T, p->Hk, D, es, p->Hk > 0, true));
        LSGD_TRY(check_positions(who, p->positions, p->ld_positions, p->turns, W, T, R));
        if (p->norm && !p->stats) return set_error(LSGD_ERR_INVALID_ARG, "%s: stats are required", who);
        if (!on(p->stats, 4)) return set_error(LSGD_ERR_INVALID_ARG, "%s: stats are not aligned to their element", who);
        if (sums) {
            if (!workspace) return set_error(LSGD_ERR_INVALID_ARG, "%s: workspace is NULL", who);
            if (!on(workspace, kAlign)) return set_error(LSGD_ERR_INVALID_ARG, "%s: workspace must be 256-byte aligned", who);
            if (workspace_bytes < plan.bytes) return set_error(LSGD_ERR_NOMEM, "%s: workspace of %zu bytes < %zu needed", who, workspace_bytes, plan.bytes);
        }
        Args g{};
        if (need_q) g.x[0] = heads(p->q);
        if (need_k) g.x[1] = heads(p->k);
        g.y[0] = heads(p->dq_out); g.y[1] = heads(p->dk_out);
        g.dx[0] = heads(p->dq); g.dx[1] = heads(p->dk);
        g.H[0] = p->Hq; g.H[1] = p->Hk;
        g.w[0] = p->w_q; g.w[1] = p->w_k;
        g.ld_w[0] = W > 1 ? p->ld_w_q : 0; g.ld_w[1] = W > 1 ? p->ld_w_k : 0;
        g.pos = p->positions; g.ld_pos = W > 1 ? p->ld_positions : 0;
        g.turns = p->turns;
        g.stats = const_cast<float*>(p->stats);
        g.parts = sums ? static_cast<float*>(workspace) : nullptr;
        g.T = T; g.D = D; g.Dp = plan.Dp; g.half = R / 2; g.norm = p->norm;
        g.lanes = lanes_of(D, R, E);
        g.tokens = tokens_of(W, T, p->Hq + p->Hk, R, g.lanes);
        g.inv_d = 1.0f / (float)D; g.magnitude = p->magnitude;
        bool once = true;
        for (const lsgd_heads* a : {&p->dq_out, &p->q, &p->dq}) once = once && wide_heads(*a, W, T, p->Hq, es);
        for (const lsgd_heads* a : {&p->dk_out, &p->k, &p->dk}) once = once && wide_heads(*a, W, T, p->Hk, es);
        dispatch(p->is_bf16, E, p->interleaved, once, [&](auto type, auto e, auto neighbours, auto streamed) {
            hipLaunchKernelGGL((qk_rotary_grad_kernel<decltype(type), decltype(e)::value, decltype(neighbours)::value, decltype(streamed)::value>),
                               dim3((unsigned)plan.groups, (unsigned)W, p->Hk ? 2 : 1), dim3(kThreads), sizeof(v2f) * (size_t)std::max(1, g.tokens * g.half), s, g);
        });
    }
    // (no tokens: the sums of nothing)
    if (sums && (T > 0 || !p->accumulate))
        hipLaunchKernelGGL(qk_join_kernel, dim3((unsigned)((D - 1) / kWave + 1), (unsigned)W, 2), dim3(kJoinThreads), 0, s, static_cast<const float*>(workspace),
                           T > 0 ? plan.groups : 0, D, plan.Dp, join, p->accumulate);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return set_error(LSGD_ERR_HIP, "%s: %s", who, hipGetErrorString(err));
    return LSGD_OK;
}

} // extern "C"
