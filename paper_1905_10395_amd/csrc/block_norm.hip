// The norms around a block of a model, fused with the block's gate and its scaled residual sum, and their gradients.
//
//   after the block      r' = r + s a o (q_y y o w)       q_y = (mean y^2 + eps)^-1/2, a = sigmoid(u)
//   before the next one  n  = q_r r' o v                  q_r = (mean r'^2 + eps)^-1/2
//
// One pass: a team of lanes holds a token's whole row in registers between the sums and the stores, so r, y and u are
// read once and r' and n written once; between the two norms r' stays fp32 (it is rounded only where it is stored).
//
//   backward, from dn and the gradient dR of r' that comes past the next block; h = q_r r', z = q_y y
//   dr = dR + q_r (v o dn - h mean(v o dn o h))           dv = sum_t dn o h
//   e  = s dr o a;  dy = q_y (e o w - z mean(e o w o z))  dw = sum_t e o z     du = s dr o z o w a (1-a)
//
// Bound by memory.  Workers' weights are columns of fp32 rows; a team keeps them in registers over the tokens it takes,
// as it does its part of the sums over tokens, which go to the workspace once a workgroup and are added up in order by a
// second launch: no atomics, equal calls give equal bits.  Forward 8 x 8192 x 4096 bf16 465 us, 5.8 TB/s of the 2.7 GB that have to
// move; backward 8 x 4096 x 2048 205 us, 5.2 TB/s of 1.07 GB, with the join.
//
// A lane holds eight columns, so a team is as wide as its row.  16 columns a lane and half the lanes: backward 221 instead of 203 us at
// 4 x 4096 x 4096 bf16, forward 155 instead of 139 at 4 x 2048 x 8192, but 452 instead of 466 at 8 x 8192 x 4096.  Teams take every
// grid-th token, so that those at work at a time are neighbours in memory.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "row_pieces.h"

using namespace lsgd;

namespace {

constexpr int kColumns = 8;       // of a row that a lane holds, or twice as many
constexpr int kTeamThreads = 256, kMaxThreads = 1024;

// [W, T, D] with dense rows
struct Rows {
    void* p;
    int64_t lw, lt;
};

struct NormArgs {
    Rows r, y, u, r_out, n;                  // y, u, r_out, n may be absent
    const float *w_post, *w_pre;             // NULL: ones
    int64_t ld_w_post, ld_w_pre;
    float *q_post, *q_pre;                   // [W, T]; may be NULL
    int T, D;
    float scale, eps, inv_d;
    int post;                                // the block's output is normed
};

struct NormGradArgs {
    Rows dn, dr_out, r, y, u, dr, dy, du;    // dn, dr_out, y, u, dy, du may be absent
    const float *w_post, *w_pre;
    int64_t ld_w_post, ld_w_pre;
    const float *q_post, *q_pre;
    float* parts;                            // [W][workgroups][2][Dp]: dw_post, dw_pre of a workgroup's tokens; NULL: not wanted
    int T, D, Dp;
    float scale, inv_d;
    int post;
};

// A lane's columns of a row: pieces of 16 bytes, adjacent lanes' adjacent, so that an access of a wavefront covers whole lines
// (of fp32, 32 bytes a lane took 271 instead of 218 us forward at 8 x 4096 x 2048).  WIDE: all pieces whole and 16-byte aligned; these are
// read once and written once, and streaming accesses in both directions took 466 us where plain ones took 500 (8 x 8192 x 4096
// bf16).  Elements past the row's end read zero and are not written.  SHORT: rows may be shorter than
// a piece.
template <class T, int N, bool WIDE, bool SHORT>
struct Piece {
    static constexpr int E = 16 / (int)sizeof(T), PIECES = N * kColumns / E;
    using Row = Raw<T, E>[PIECES];                                     // as in memory
    using Values = float[PIECES][E];

    static __device__ __forceinline__ int col(int lane, int ts, int n) { return (n * ts + lane) * E; }
    static __device__ __forceinline__ void load(const T* p, int lane, int ts, int D, Row& v)
    {
#pragma unroll
        for (int n = 0; n < PIECES; ++n) {
            const int c = col(lane, ts, n);
            clear(v[n]);
            if constexpr (!WIDE) load_piece<SHORT>(p, c, D, v[n]);
            else if (c < D) load_whole<true>(column(p, c), v[n]);
        }
    }
    static __device__ __forceinline__ void none(Row& v)
    {
#pragma unroll
        for (int n = 0; n < PIECES; ++n) clear(v[n]);
    }
    static __device__ __forceinline__ void get(const Row& v, int lane, int ts, int D, Values& f)
    {
#pragma unroll
        for (int n = 0; n < PIECES; ++n) {
            unpack(v[n], f[n]);
            if constexpr (!WIDE) keep_own(col(lane, ts, n), D, f[n]);
        }
    }
    template <class TO>
    static __device__ __forceinline__ void store(TO* p, int lane, int ts, int D, const Values& v)
    {
#pragma unroll
        for (int n = 0; n < PIECES; ++n) {
            const int c = col(lane, ts, n);
            if constexpr (!WIDE) store_piece<SHORT>(p, c, D, v[n]);
            else if (c < D) store_whole<true>(column(p, c), v[n]);
        }
    }
    // per-column weights of a worker (a team reads them again and again: not streamed); absent: ones.  Past the row's end
    // zero, so that nothing there enters a sum.
    static __device__ __forceinline__ void weights(const float* p, int lane, int ts, int D, Values& v)
    {
#pragma unroll
        for (int n = 0; n < PIECES; ++n) {
            const int c = col(lane, ts, n);
#pragma unroll
            for (int e = 0; e < E; ++e) v[n][e] = c < D ? 1.0f : 0.0f;
            if (p) load_piece<SHORT>(p, c, D, v[n]);
            keep_own(c, D, v[n]);
        }
    }
};

// Whether a team holds the weights and its sums for their gradients in registers over its tokens.  With twice the columns a lane
// they do not fit, and it reads the weights again for each token and keeps the sums in LDS (2 x 2048 x 16384 bf16 backward 229 us,
// 487 with registers spilled; fp32 466 and 841).
template <int N>
constexpr bool kHold = N == 1;

// A lane's part of a weight's gradient, over its tokens: in registers, or where those are short in the lane's own LDS.
template <int N, bool LDS>
struct Grad {
    v4f v[N * kColumns / 4];
    __device__ __forceinline__ v4f& at(int k) { return v[k]; }
};
template <int N>
struct Grad<N, true> {
    v4f* v;
    __device__ __forceinline__ v4f& at(int k) { return v[k * kMaxThreads]; }
};

// Teams: LANES of a wavefront (8 to 64, as many as rows of at most 512 columns need) in workgroups of 256; or, LANES = 0, the
// workgroup, of any whole number of wavefronts.
constexpr int threads_limit(int lanes) { return lanes ? kTeamThreads : kMaxThreads; }

// Sums over rows of 16 lanes and over a wavefront by lane shifts in the vector unit.
template <int CTRL>
__device__ __forceinline__ float add_lanes(float a)
{
    return a + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(a), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float row_sum(float a)          // in all lanes of the row: rotations by 8, 4, 2, 1
{
    return add_lanes<0x121>(add_lanes<0x122>(add_lanes<0x124>(add_lanes<0x128>(a))));
}
__device__ __forceinline__ float wave_sum(float a)
{
    a = row_sum(a);
    const int b = __float_as_int(a);
    return (__int_as_float(__builtin_amdgcn_readlane(b, 0)) + __int_as_float(__builtin_amdgcn_readlane(b, 16))) +
           (__int_as_float(__builtin_amdgcn_readlane(b, 32)) + __int_as_float(__builtin_amdgcn_readlane(b, 48)));
}

// Sum over a team, the same value in all its lanes.  The wavefronts of a workgroup meet in LDS; two buffers in turn, so that
// one barrier a sum is enough (a buffer is written again only after the barrier that follows its last read).
struct TeamSum {
    float (*buf)[16];
    int turn;
};
template <int LANES>
__device__ __forceinline__ float team_sum(float a, TeamSum& s)
{
    if constexpr (LANES == 8 || LANES == 16 || LANES == 32) {
        a = add_lanes<0xB1>(a);                            // the other lane of a pair, the other pair, the other four, ...
        a = add_lanes<0x4E>(a);
        a = add_lanes<0x141>(a);
        if constexpr (LANES >= 16) a = add_lanes<0x140>(a);
        if constexpr (LANES == 32) a += __shfl_xor(a, 16);
    } else {
        a = wave_sum(a);
        if constexpr (LANES == 0) {
            const int lane = threadIdx.x & (kWave - 1), waves = blockDim.x / kWave;
            if (lane == 0) s.buf[s.turn][threadIdx.x / kWave] = a;
            __syncthreads();
            a = row_sum((lane & 15) < waves ? s.buf[s.turn][lane & 15] : 0.0f);
            s.turn ^= 1;
        }
    }
    return a;
}

// The gate, to 2 |u| + 5 roundings: the quick exponential takes a rounded multiple of u, the quick reciprocal is one last bit off.
__device__ __forceinline__ float sigmoid(float u) { return __builtin_amdgcn_rcpf(1.0f + __expf(-u)); }
// The same value, and 1 - a as exp(-u) a: the difference itself would keep only a's absolute error, and nothing from u = 17 on.
// Where the exponential overflows a is zero, and so is the product of the two.
__device__ __forceinline__ float sigmoid(float u, float& rest)
{
    const float t = __expf(-u), a = __builtin_amdgcn_rcpf(1.0f + t);
    rest = fminf(t, 0x1.fffffep127f) * a;
    return a;
}

template <class T>
__device__ __forceinline__ T* row_of(const Rows& a, int w, int64_t t) { return static_cast<T*>(a.p) + w * a.lw + t * a.lt; }

template <class T, int N, bool WIDE, int LANES>
__global__ __launch_bounds__(threads_limit(LANES)) void block_norm_kernel(NormArgs a)
{
    using P = Piece<T, N, WIDE, LANES == 8>;
    constexpr int E = P::E, PIECES = P::PIECES;
    __shared__ float buf[2][16];
    TeamSum sums{buf, 0};
    constexpr int teams = LANES ? kTeamThreads / (LANES ? LANES : 1) : 1;
    const int ts = LANES ? LANES : (int)blockDim.x, lane = threadIdx.x % (unsigned)ts, w = blockIdx.y;
    int team = LANES ? (int)threadIdx.x / ts : 0;
    if constexpr (LANES == kWave) team = __builtin_amdgcn_readfirstlane(team);
    typename P::Values wp, wn;
    auto post_weights = [&] { P::weights(a.w_post ? a.w_post + w * a.ld_w_post : nullptr, lane, ts, a.D, wp); };
    auto pre_weights = [&] { P::weights(a.w_pre ? a.w_pre + w * a.ld_w_pre : nullptr, lane, ts, a.D, wn); };
    if (kHold<N> && a.y.p) post_weights();
    if (kHold<N> && a.n.p) pre_weights();
    for (int64_t t = (int64_t)blockIdx.x * teams + team; t < a.T; t += (int64_t)gridDim.x * teams) {
        typename P::Row rr, ry, ru;
        typename P::Values r;
        // y is waited for first (8 x 8192 x 4096 bf16 466 us, 480 with r's load first; but 6 x 4064 x 4495 283 and 265)
        if (!WIDE || !a.y.p) P::load(row_of<T>(a.r, w, t), lane, ts, a.D, rr);
        if (a.y.p) {
            typename P::Values y, u;
            P::load(row_of<T>(a.y, w, t), lane, ts, a.D, ry);
            if (WIDE) P::load(row_of<T>(a.r, w, t), lane, ts, a.D, rr);
            if (a.u.p) P::load(row_of<T>(a.u, w, t), lane, ts, a.D, ru);
            P::get(ry, lane, ts, a.D, y);
            float q = 1.0f;
            if (a.post) {
                float s = 0.0f;
#pragma unroll
                for (int n = 0; n < PIECES; ++n)
#pragma unroll
                    for (int e = 0; e < E; ++e) s += y[n][e] * y[n][e];
                q = 1.0f / sqrtf(team_sum<LANES>(s, sums) * a.inv_d + a.eps);
                if (a.q_post && lane == 0) a.q_post[(int64_t)w * a.T + t] = q;
            }
            const float sq = a.scale * q;
            if (!kHold<N>) post_weights();
            P::get(rr, lane, ts, a.D, r);
            if (a.u.p) P::get(ru, lane, ts, a.D, u);
#pragma unroll
            for (int n = 0; n < PIECES; ++n)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    float b = y[n][e] * sq * wp[n][e];
                    if (a.u.p) b *= sigmoid(u[n][e]);
                    r[n][e] += b;
                }
            P::store(row_of<T>(a.r_out, w, t), lane, ts, a.D, r);
        } else {
            P::get(rr, lane, ts, a.D, r);
        }
        if (a.n.p) {
            float s = 0.0f;
#pragma unroll
            for (int n = 0; n < PIECES; ++n)
#pragma unroll
                for (int e = 0; e < E; ++e) s += r[n][e] * r[n][e];
            const float q = 1.0f / sqrtf(team_sum<LANES>(s, sums) * a.inv_d + a.eps);
            if (a.q_pre && lane == 0) a.q_pre[(int64_t)w * a.T + t] = q;
            if (!kHold<N>) pre_weights();
#pragma unroll
            for (int n = 0; n < PIECES; ++n)
#pragma unroll
                for (int e = 0; e < E; ++e) r[n][e] *= q * wn[n][e];
            P::store(row_of<T>(a.n, w, t), lane, ts, a.D, r);
        }
    }
}

// Four wavefronts a SIMD have to fit (12 x 11864 x 64 bf16 34 us, 36 where registers decide; 8 x 16000 x 128 54 and 55; the other way
// round for some odd rows, 8 x 16384 x 201 122 and 114), but for fp32 in unaligned pieces, which would spill (201: 173 us so, 266).
template <class T, int N, bool WIDE, int LANES>
__global__ __launch_bounds__(threads_limit(LANES), sizeof(T) == 2 || WIDE ? 4 : 1) void block_norm_grad_kernel(NormGradArgs a)
{
    using P = Piece<T, N, WIDE, LANES == 8>;
    constexpr int E = P::E, PIECES = P::PIECES;
    __shared__ float buf[2][16];
    TeamSum sums{buf, 0};
    constexpr int teams = LANES ? kTeamThreads / (LANES ? LANES : 1) : 1;
    const int ts = LANES ? LANES : (int)blockDim.x, lane = threadIdx.x % (unsigned)ts, w = blockIdx.y;
    int team = LANES ? (int)threadIdx.x / ts : 0;
    if constexpr (LANES == kWave) team = __builtin_amdgcn_readfirstlane(team);
    typename P::Values wp, wn;
    Grad<N, !kHold<N>> dwp, dwn;
    if constexpr (!kHold<N>) {
        __shared__ v4f held[2 * N * kColumns / 4 * kMaxThreads];
        dwp.v = held + threadIdx.x;
        dwn.v = dwp.v + N * kColumns / 4 * kMaxThreads;
    }
    auto post_weights = [&] { P::weights(a.w_post ? a.w_post + w * a.ld_w_post : nullptr, lane, ts, a.D, wp); };
    auto pre_weights = [&] { P::weights(a.w_pre ? a.w_pre + w * a.ld_w_pre : nullptr, lane, ts, a.D, wn); };
    if (kHold<N> && a.y.p) post_weights();
    if (kHold<N> && a.dn.p) pre_weights();
#pragma unroll
    for (int k = 0; k < N * kColumns / 4; ++k) dwp.at(k) = dwn.at(k) = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    for (int64_t t = (int64_t)blockIdx.x * teams + team; t < a.T; t += (int64_t)gridDim.x * teams) {
        typename P::Row rz, ru, rdr, rdn, rh;
        typename P::Values dr, z, u;
        constexpr bool kEarly = N == 1;                                 // in flight while the first sum is made, if registers are left
        if (kEarly && a.y.p) {                                          // (two pieces a lane: 229 us late, 256 early, 2 x 2048 x 16384 bf16)
            P::load(row_of<T>(a.y, w, t), lane, ts, a.D, rz);
            if (a.u.p) P::load(row_of<T>(a.u, w, t), lane, ts, a.D, ru);
        }
        if (a.dn.p) {
            P::load(row_of<T>(a.dn, w, t), lane, ts, a.D, rdn);
            P::load(row_of<T>(a.r, w, t), lane, ts, a.D, rh);
        }
        auto load_dr = [&] {
            if (a.dr_out.p) P::load(row_of<T>(a.dr_out, w, t), lane, ts, a.D, rdr);
            else P::none(rdr);
        };
        if (kEarly) load_dr();
        if (a.dn.p) {
            typename P::Values dn, h;
            P::get(rdn, lane, ts, a.D, dn);
            P::get(rh, lane, ts, a.D, h);
            if (!kHold<N>) pre_weights();
            const float q = a.q_pre[(int64_t)w * a.T + t];
            float s = 0.0f;
#pragma unroll
            for (int n = 0; n < PIECES; ++n)
#pragma unroll
                for (int e = 0; e < E; e += 4) {
                    v4f dw = dwn.at((n * E + e) / 4);
#pragma unroll
                    for (int k = e; k < e + 4; ++k) {
                        h[n][k] *= q;
                        dw[k - e] += dn[n][k] * h[n][k];
                        dn[n][k] *= wn[n][k];
                        s += dn[n][k] * h[n][k];
                    }
                    dwn.at((n * E + e) / 4) = dw;
                }
            s = team_sum<LANES>(s, sums) * a.inv_d;
            if (!kEarly) load_dr();
            P::get(rdr, lane, ts, a.D, dr);
#pragma unroll
            for (int n = 0; n < PIECES; ++n)
#pragma unroll
                for (int e = 0; e < E; ++e) dr[n][e] += q * (dn[n][e] - h[n][e] * s);
        } else {
            if (!kEarly) load_dr();
            P::get(rdr, lane, ts, a.D, dr);
        }
        P::store(row_of<T>(a.dr, w, t), lane, ts, a.D, dr);
        if (a.y.p) {
            if (!kEarly) {
                P::load(row_of<T>(a.y, w, t), lane, ts, a.D, rz);
                if (a.u.p) P::load(row_of<T>(a.u, w, t), lane, ts, a.D, ru);
            }
            P::get(rz, lane, ts, a.D, z);
            if (a.u.p) P::get(ru, lane, ts, a.D, u);
            if (!kHold<N>) post_weights();
            const float q = a.post ? a.q_post[(int64_t)w * a.T + t] : 1.0f;
            float s = 0.0f;
#pragma unroll
            for (int n = 0; n < PIECES; ++n)
#pragma unroll
                for (int e = 0; e < E; e += 4) {
                    v4f dw = dwp.at((n * E + e) / 4);
#pragma unroll
                    for (int k = e; k < e + 4; ++k) {
                        z[n][k] *= q;
                        float d = a.scale * dr[n][k];                   // e of the formula, gate still missing
                        if (a.u.p) {
                            float rest;
                            const float g = sigmoid(u[n][k], rest);
                            u[n][k] = d * z[n][k] * wp[n][k] * (g * rest);
                            d *= g;
                        }
                        dw[k - e] += d * z[n][k];
                        dr[n][k] = d * wp[n][k];
                        s += dr[n][k] * z[n][k];
                    }
                    dwp.at((n * E + e) / 4) = dw;
                }
            if (a.u.p) P::store(row_of<T>(a.du, w, t), lane, ts, a.D, u);
            if (a.post) {
                s = team_sum<LANES>(s, sums) * a.inv_d;
#pragma unroll
                for (int n = 0; n < PIECES; ++n)
#pragma unroll
                    for (int e = 0; e < E; ++e) dr[n][e] = q * (dr[n][e] - z[n][e] * s);
            }
            P::store(row_of<T>(a.dy, w, t), lane, ts, a.D, dr);
        }
    }
    if (!a.parts) return;
    float* part = a.parts + ((int64_t)w * gridDim.x + blockIdx.x) * 2 * a.Dp;
    if constexpr (LANES == 0) {
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            typename P::Values f;
#pragma unroll
            for (int k = 0; k < PIECES * E; ++k) f[k / E][k % E] = (which ? dwn : dwp).at(k / 4)[k % 4];
            P::store(part + which * a.Dp, lane, ts, a.D, f);
        }
    } else {
        // the workgroup's teams add up theirs in order
        __shared__ float sum[teams][LANES * kColumns];
#pragma unroll
        for (int which = 0; which < 2; ++which) {
#pragma unroll
            for (int k = 0; k < PIECES * E; ++k) {
                const int first = P::col(lane, ts, k / E), c = (WIDE ? first : piece_start<E>(first, a.D)) + k % E;
                if (c >= first) sum[team][c] = (which ? dwn : dwp).at(k / 4)[k % 4];
            }
            __syncthreads();
            for (int i = threadIdx.x; i < LANES * kColumns && i < a.D; i += kTeamThreads) {
                float s = 0.0f;
#pragma unroll
                for (int k = 0; k < teams; ++k) s += sum[k][i];
                part[which * a.Dp + i] = s;
            }
            __syncthreads();
        }
    }
}

// dw[w, :] (+)= the sum over a worker's parts, each wavefront a stretch of them.
constexpr int kJoinThreads = 1024;
__global__ __launch_bounds__(kJoinThreads) void norm_join_kernel(const float* __restrict__ parts, int chunks, int D, int Dp, float* dw_post,
                                                                 int64_t ld_post, float* dw_pre, int64_t ld_pre, int accumulate)
{
    constexpr int waves = kJoinThreads / kWave;
    __shared__ float sum[waves][kWave];
    float* dw = blockIdx.z ? dw_pre : dw_post;
    if (!dw) return;
    dw += (int64_t)blockIdx.y * (blockIdx.z ? ld_pre : ld_post);
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

__global__ __launch_bounds__(256) void norm_zero_kernel(float* dw, int64_t ld, int D)
{
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c < D) dw[blockIdx.y * ld + c] = 0.0f;
}

// ---- host ----
constexpr size_t kAlign = 256;
constexpr int kMaxWidth = kMaxThreads * 2 * kColumns;
bool on(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

lsgd_status check_shape(const char* who, int32_t W, int32_t T, int32_t D)
{
    if (W <= 0 || W > LSGD_MAX_WORKERS) return set_error(LSGD_ERR_SHAPE, "%s: W=%d outside [1,%d]", who, (int)W, LSGD_MAX_WORKERS);
    if (T < 0 || D <= 0) return set_error(LSGD_ERR_SHAPE, "%s: T=%d must not be negative, D=%d must be positive", who, (int)T, (int)D);
    if (D > kMaxWidth) return set_error(LSGD_ERR_UNSUPPORTED, "%s: D=%d beyond the %d columns a workgroup holds", who, (int)D, kMaxWidth);
    return LSGD_OK;
}

// One activation tensor: there or not, aligned to its elements, rows that do not overlap.
lsgd_status check_rows(const char* who, const char* name, const lsgd_rows& a, int W, int T, int D, int es, bool wanted, bool written)
{
    if (wanted && !a.data) return set_error(LSGD_ERR_INVALID_ARG, "%s: %s is required", who, name);
    if (!wanted && a.data) return set_error(LSGD_ERR_INVALID_ARG, "%s: %s has no meaning here and must be NULL", who, name);
    if (!a.data) return LSGD_OK;
    if (!on(a.data, es)) return set_error(LSGD_ERR_INVALID_ARG, "%s: %s is not aligned to its element", who, name);
    const int64_t lt = T > 1 ? a.token_stride : D, lw = a.worker_stride;
    if (lt < 0 || (W > 1 && lw < 0)) return set_error(LSGD_ERR_SHAPE, "%s: %s has a negative stride", who, name);
    // what is written must not overlap itself, whichever of the two strides is the larger
    if (written && ((T > 1 && lt < D) || (W > 1 && lw < D) ||
                    (T > 1 && W > 1 && lw < (int64_t)(T - 1) * lt + D && lt < (int64_t)(W - 1) * lw + D)))
        return set_error(LSGD_ERR_SHAPE, "%s: rows of %s overlap", who, name);
    return LSGD_OK;
}

bool wide_rows(const lsgd_rows& a, int W, int T, int es)
{
    const int64_t per = 16 / es;
    return !a.data || (on(a.data, 16) && (W == 1 || a.worker_stride % per == 0) && (T <= 1 || a.token_stride % per == 0));
}

Rows rows(const lsgd_rows& a) { return Rows{a.data, a.worker_stride, a.token_stride}; }

// Lanes of a team within a wavefront for rows of at most 512 columns; whole wavefronts for all of those took 72 us instead of
// 19 for 12 x 11864 x 64 bf16.
int lanes_of(int D)
{
    int lanes = 8;
    while (lanes * kColumns < D) lanes *= 2;
    return lanes;
}

// Lanes and pieces for rows of D columns.
struct Shape {
    int n, teams, threads;
};
Shape shape_of(int D)
{
    if (D <= kWave * kColumns) return {1, kTeamThreads / lanes_of(D), kTeamThreads};
    if (D <= kMaxThreads * kColumns) return {1, 1, (D - 1) / (kWave * kColumns) * kWave + kWave};
    return {2, 1, kMaxThreads};
}

// Workgroups of a worker.  Forward many, by lanes in all: a team's only gain from further tokens is the weights it holds
// (8 x 8192 x 4096: 466 us with 2^22 lanes, 491 with 2^20; x 1024: 111 and 120).  Backward each leaves partial sums; twice what
// the chip holds at a time, which is 1024 lanes a compute unit by their registers: enough to even out (8 x 4096 x 2048 bf16 205 us,
// 215 with once as many, 212 with four times), and whole rounds (6 x 4064 x 4496, nine wavefronts a team: 402 us, 430 with 2^19
// lanes in all, 391 with once as many; 12 x 990 x 7384 300, 370 with 2^19 lanes).
constexpr int kLanes = 1 << 22, kRoundsGrad = 2, kComputeUnits = 256;
int groups_of(int W, int T, const Shape& s, int all)
{
    return (int)std::min<int64_t>((T - 1) / s.teams + 1, std::max(1, all / W));
}

struct GradPlan {
    int groups, Dp;
    size_t bytes;
};
GradPlan grad_plan(int W, int T, int D)
{
    GradPlan p;
    const Shape sh = shape_of(D);
    p.groups = T ? groups_of(W, T, sh, kRoundsGrad * kComputeUnits * (kMaxThreads / sh.threads)) : 0;
    p.Dp = (D + kColumns - 1) / kColumns * kColumns;
    p.bytes = std::max<size_t>(kAlign, sizeof(float) * (size_t)W * (size_t)p.groups * 2 * (size_t)p.Dp);
    return p;
}

// Calls launch(kernel's template arguments) for the type, alignment and width at hand.
template <class F>
void dispatch(int D, bool bf16, bool wide, F launch)
{
    auto shaped = [&](auto type, auto wide_rows) {
        const std::integral_constant<int, 1> one{};
        if (D <= 8 * kColumns) launch(type, one, wide_rows, std::integral_constant<int, 8>{});
        else if (D <= 16 * kColumns) launch(type, one, wide_rows, std::integral_constant<int, 16>{});
        else if (D <= 32 * kColumns) launch(type, one, wide_rows, std::integral_constant<int, 32>{});
        else if (D <= 64 * kColumns) launch(type, one, wide_rows, std::integral_constant<int, 64>{});
        else if (D <= kMaxThreads * kColumns) launch(type, one, wide_rows, std::integral_constant<int, 0>{});
        else launch(type, std::integral_constant<int, 2>{}, wide_rows, std::integral_constant<int, 0>{});
    };
    if (bf16) wide ? shaped(uint16_t{}, std::true_type{}) : shaped(uint16_t{}, std::false_type{});
    else wide ? shaped(float{}, std::true_type{}) : shaped(float{}, std::false_type{});
}

#define LSGD_TRY(x)                         \
    do {                                    \
        const lsgd_status st_ = (x);        \
        if (st_ != LSGD_OK) return st_;     \
    } while (0)

lsgd_status check_weights(const char* who, const char* name, const float* w, int64_t ld, int W, int D, bool written)
{
    if (!w) return LSGD_OK;
    if (!on(w, 4)) return set_error(LSGD_ERR_INVALID_ARG, "%s: %s is not aligned to its element", who, name);
    if (W > 1 && (ld < 0 || (written && ld < D))) return set_error(LSGD_ERR_SHAPE, "%s: %s: worker stride %lld for D=%d", who, name, (long long)ld, D);
    return LSGD_OK;
}

} // namespace

extern "C" {

lsgd_status lsgd_block_norm(const lsgd_block_norm_args* p, void* hip_stream)
{
    const char* who = "block_norm";
    if (!p) return set_error(LSGD_ERR_INVALID_ARG, "%s: arguments are NULL", who);
    const int W = p->W, T = p->T, D = p->D, es = p->is_bf16 ? 2 : 4;
    LSGD_TRY(check_shape(who, W, T, D));
    if (p->is_bf16 & ~1 || p->post_norm & ~1) return set_error(LSGD_ERR_INVALID_ARG, "%s: is_bf16 and post_norm must be 0 or 1", who);
    if (!std::isfinite(p->scale)) return set_error(LSGD_ERR_INVALID_ARG, "%s: scale must be finite", who);
    if (!std::isfinite(p->eps) || p->eps <= 0.0f) return set_error(LSGD_ERR_INVALID_ARG, "%s: eps must be finite and positive", who);
    if (T == 0) return LSGD_OK;
    const bool sum = p->y.data != nullptr;
    LSGD_TRY(check_rows(who, "r", p->r, W, T, D, es, true, false));
    LSGD_TRY(check_rows(who, "y", p->y, W, T, D, es, sum, false));
    LSGD_TRY(check_rows(who, "gate", p->gate, W, T, D, es, sum && p->gate.data, false));
    LSGD_TRY(check_rows(who, "r_out", p->r_out, W, T, D, es, sum, true));
    LSGD_TRY(check_rows(who, "n", p->n, W, T, D, es, !sum || p->n.data, true));
    LSGD_TRY(check_weights(who, "w_post", p->w_post, p->ld_w_post, W, D, false));
    LSGD_TRY(check_weights(who, "w_pre", p->w_pre, p->ld_w_pre, W, D, false));
    if (!on(p->q_post, 4) || !on(p->q_pre, 4)) return set_error(LSGD_ERR_INVALID_ARG, "%s: q_post or q_pre is not aligned to its element", who);

    NormArgs a{};
    a.r = rows(p->r); a.y = rows(p->y); a.u = rows(p->gate); a.r_out = rows(p->r_out); a.n = rows(p->n);
    a.w_post = p->w_post; a.ld_w_post = p->ld_w_post;
    a.w_pre = p->w_pre; a.ld_w_pre = p->ld_w_pre;
    a.q_post = p->q_post; a.q_pre = p->q_pre;
    a.T = T; a.D = D;
    a.scale = p->scale; a.eps = p->eps; a.inv_d = 1.0f / (float)D;
    a.post = p->post_norm;
    bool wide = D % (16 / es) == 0;
    for (const lsgd_rows* q : {&p->r, &p->y, &p->gate, &p->r_out, &p->n}) wide = wide && wide_rows(*q, W, T, es);
    const Shape sh = shape_of(D);
    const dim3 grid((unsigned)groups_of(W, T, sh, kLanes / sh.threads), (unsigned)W);
    dispatch(D, p->is_bf16, wide, [&](auto type, auto n, auto wide_rows, auto lanes) {
        hipLaunchKernelGGL((block_norm_kernel<decltype(type), decltype(n)::value, decltype(wide_rows)::value, decltype(lanes)::value>), grid,
                           dim3((unsigned)sh.threads), 0, static_cast<hipStream_t>(hip_stream), a);
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return set_error(LSGD_ERR_HIP, "%s: %s", who, hipGetErrorString(e));
    return LSGD_OK;
}

size_t lsgd_block_norm_grad_workspace_bytes(int32_t W, int32_t T, int32_t D)
{
    if (check_shape("block_norm_grad", W, T, D) != LSGD_OK) return 0;
    return grad_plan(W, T, D).bytes;
}

lsgd_status lsgd_block_norm_grad(const lsgd_block_norm_grad_args* p, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    const char* who = "block_norm_grad";
    if (!p) return set_error(LSGD_ERR_INVALID_ARG, "%s: arguments are NULL", who);
    const int W = p->W, T = p->T, D = p->D, es = p->is_bf16 ? 2 : 4;
    LSGD_TRY(check_shape(who, W, T, D));
    if (p->is_bf16 & ~1 || p->post_norm & ~1 || p->accumulate & ~1) return set_error(LSGD_ERR_INVALID_ARG, "%s: is_bf16, post_norm and accumulate must be 0 or 1", who);
    if (!std::isfinite(p->scale)) return set_error(LSGD_ERR_INVALID_ARG, "%s: scale must be finite", who);
    LSGD_TRY(check_weights(who, "w_post", p->w_post, p->ld_w_post, W, D, false));
    LSGD_TRY(check_weights(who, "w_pre", p->w_pre, p->ld_w_pre, W, D, false));
    LSGD_TRY(check_weights(who, "dw_post", p->dw_post, p->ld_dw_post, W, D, true));
    LSGD_TRY(check_weights(who, "dw_pre", p->dw_pre, p->ld_dw_pre, W, D, true));
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    hipError_t e;
    if (T == 0) {
        if (!p->accumulate)
            for (int k = 0; k < 2; ++k)
                if (float* dw = k ? p->dw_pre : p->dw_post)
                    hipLaunchKernelGGL(norm_zero_kernel, dim3((unsigned)((D - 1) / 256 + 1), (unsigned)W), dim3(256), 0, s, dw,
                                       k ? p->ld_dw_pre : p->ld_dw_post, D);
        e = hipGetLastError();
        if (e != hipSuccess) return set_error(LSGD_ERR_HIP, "%s: %s", who, hipGetErrorString(e));
        return LSGD_OK;
    }
    const bool sum = p->y.data != nullptr, norm = p->dn.data != nullptr;
    if (!norm && !p->dr_out.data) return set_error(LSGD_ERR_INVALID_ARG, "%s: neither dn nor dr_out is given", who);
    LSGD_TRY(check_rows(who, "dn", p->dn, W, T, D, es, norm, false));
    LSGD_TRY(check_rows(who, "dr_out", p->dr_out, W, T, D, es, p->dr_out.data, false));
    LSGD_TRY(check_rows(who, "r_out", p->r_out, W, T, D, es, norm || p->r_out.data, false));
    LSGD_TRY(check_rows(who, "y", p->y, W, T, D, es, sum, false));
    LSGD_TRY(check_rows(who, "gate", p->gate, W, T, D, es, sum && p->gate.data, false));
    LSGD_TRY(check_rows(who, "dr", p->dr, W, T, D, es, true, true));
    LSGD_TRY(check_rows(who, "dy", p->dy, W, T, D, es, sum, true));
    LSGD_TRY(check_rows(who, "dgate", p->dgate, W, T, D, es, sum && p->gate.data, true));
    if (norm && !p->q_pre) return set_error(LSGD_ERR_INVALID_ARG, "%s: q_pre is required", who);
    if (sum && p->post_norm && !p->q_post) return set_error(LSGD_ERR_INVALID_ARG, "%s: q_post is required", who);
    if (!on(p->q_post, 4) || !on(p->q_pre, 4)) return set_error(LSGD_ERR_INVALID_ARG, "%s: q_post or q_pre is not aligned to its element", who);
    if (p->dw_post && !sum) return set_error(LSGD_ERR_INVALID_ARG, "%s: dw_post needs y", who);
    if (p->dw_pre && !norm) return set_error(LSGD_ERR_INVALID_ARG, "%s: dw_pre needs dn", who);
    const GradPlan plan = grad_plan(W, T, D);
    const bool sums = p->dw_post || p->dw_pre;
    if (sums) {
        if (!workspace) return set_error(LSGD_ERR_INVALID_ARG, "%s: workspace is NULL", who);
        if (!on(workspace, kAlign)) return set_error(LSGD_ERR_INVALID_ARG, "%s: workspace must be 256-byte aligned", who);
        if (workspace_bytes < plan.bytes) return set_error(LSGD_ERR_NOMEM, "%s: workspace of %zu bytes < %zu needed", who, workspace_bytes, plan.bytes);
    }
    NormGradArgs a{};
    a.dn = rows(p->dn); a.dr_out = rows(p->dr_out); a.r = rows(p->r_out); a.y = rows(p->y); a.u = rows(p->gate);
    a.dr = rows(p->dr); a.dy = rows(p->dy); a.du = rows(p->dgate);
    a.w_post = p->w_post; a.ld_w_post = p->ld_w_post;
    a.w_pre = p->w_pre; a.ld_w_pre = p->ld_w_pre;
    a.q_post = p->q_post; a.q_pre = p->q_pre;
    a.parts = sums ? static_cast<float*>(workspace) : nullptr;
    a.T = T; a.D = D; a.Dp = plan.Dp;
    a.scale = p->scale; a.inv_d = 1.0f / (float)D;
    a.post = p->post_norm;
    bool wide = D % (16 / es) == 0;
    for (const lsgd_rows* q : {&p->dn, &p->dr_out, &p->r_out, &p->y, &p->gate, &p->dr, &p->dy, &p->dgate}) wide = wide && wide_rows(*q, W, T, es);
    dispatch(D, p->is_bf16, wide, [&](auto type, auto n, auto wide_rows, auto lanes) {
        hipLaunchKernelGGL((block_norm_grad_kernel<decltype(type), decltype(n)::value, decltype(wide_rows)::value, decltype(lanes)::value>),
                           dim3((unsigned)plan.groups, (unsigned)W), dim3((unsigned)shape_of(D).threads), 0, s, a);
    });
    if (sums)
        hipLaunchKernelGGL(norm_join_kernel, dim3((unsigned)((D - 1) / kWave + 1), (unsigned)W, 2), dim3(kJoinThreads), 0, s, a.parts, plan.groups, D,
                           plan.Dp, p->dw_post, p->ld_dw_post, p->dw_pre, p->ld_dw_pre, p->accumulate);
    e = hipGetLastError();
    if (e != hipSuccess) return set_error(LSGD_ERR_HIP, "%s: %s", who, hipGetErrorString(e));
    return LSGD_OK;
}

} // extern "C"
