// Norm of every head's query and key, and the rotation to its position, in one pass; and its gradients.
//
// For a row x of d elements (one token, one head), with the weight w and the token's angles:
//     r = (mean(x^2) + eps)^(-1/2),   z = x r w,   y = R z
// where R turns the pairs of the first `rot` elements.  Without a weight z = x.  Gradients, from dy:
//     dz = R^T dy,   dw = sum over rows of dz x r,   g = dz w,   dx = r (g - x r^2 mean(g x)).
// All of it in 32 bits, rounded once at the end.
//
// Bound by memory: every element is read and written once (the backward pass reads x and dy).  A lane holds eight
// elements of a row, so a row is d / 8 lanes; the rows that a wave holds side by side are one head's of consecutive tokens (what it
// writes to the attention's layout is 1 KiB in a piece), and it goes through heads, U of them on their way at a time: the angles
// are read once for all of them.  (A wave that takes the heads of one token instead writes rows of 128 or 256 bytes, each L rows
// apart: 4 x 2048 tokens of 16 + 4 heads, d = 128, 26.8 us, so 19.7.)
// Measured: that case, 85 MB, 18.5 us = 4.6 TB/s (a copy of 1 GiB runs at 5.1); gradients, 16 x 512 tokens of 12 + 12 heads, d = 64,
// float, 151 MB, 31.4 us = 4.8 TB/s and 4.0 for the weights' sums; 4 x 2048 tokens of 16 + 16, d = 128, 202 MB, 42.7 us = 4.7 TB/s and 4.0;
// eight tokens 4.0 us, which is a launch and two dependent reads.
#include "dfss_kernels.hpp"
#include "head_rows.hpp"

namespace dfss {

namespace {

// A lane's place: its token (a batch element's, or none behind the last one) and its eight elements of a row.
struct Place {
    long token, b, t;
    int c, lane;
    bool real;
    template <int LPR>
    static __device__ __forceinline__ Place of(long first, long tokens, int L) {
        Place p;
        p.lane = threadIdx.x & 63, p.c = p.lane % LPR;
        const long i = first + p.lane / LPR;
        p.real = i < tokens;
        p.token = p.real ? i : tokens - 1;
        p.b = tokens <= 0x7FFFFFFF ? (long)((unsigned)p.token / (unsigned)L) : p.token / L;
        p.t = p.token - p.b * L;
        return p;
    }
    template <typename T>
    __device__ __forceinline__ T *row(const HeadRows &R, int h) const {
        return static_cast<T *>(R.data) + b * R.batch + t * R.token + h * R.head + 8 * c;
    }
};

// Eight weights of a lane, and those of the elements that turn with them.
template <typename T>
struct Weights {
    Eight<T> mine, other;
    __device__ __forceinline__ void load(const T *w, const Place &p, const Turn &turn, int LPR) {
        mine.load(w + 8 * p.c);
        other.load(w + 8 * (turn.other % LPR));
    }
};

// A wave: 64 / (d / 8) tokens, and `each` of the heads of Q and then of K.  PAST: results leave the caches first (forward).
template <typename T, int D, int U, bool PAST>
__global__ __launch_bounds__(256) void k_norm_rotate(HeadRows Q, HeadRows K, const T *__restrict__ wq, const T *__restrict__ wk,
                                                     float eps, RotaryTable rt, long tokens, int L, HeadRows Qo, HeadRows Ko,
                                                     int parts, int each) {
    constexpr int LPR = D / 8, TPW = 64 / LPR;
    const unsigned unit = blockIdx.x * 4 + (unsigned)__builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const unsigned group = __builtin_amdgcn_readfirstlane(unit / (unsigned)parts);
    if ((long)group * TPW >= tokens) return;
    const int from = (int)(unit - group * parts) * each, heads = Q.H + K.H, to = from + each < heads ? from + each : heads;
    const Place at = Place::of<LPR>((long)group * TPW, tokens, L);
    Turn turn;
    turn.load(rt.cos, rt.sin, rt.at(at.token, at.t), rt.rot, rt.interleaved != 0, at.lane, at.c, false);
    // the part's heads of Q, then those of K
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        const HeadRows &X = side ? K : Q, &Y = side ? Ko : Qo;
        const int first = side ? (from > Q.H ? from - Q.H : 0) : from, last = side ? to - Q.H : (to < Q.H ? to : Q.H);
        const T *const w = side ? wk : wq;
        Weights<T> ws;
        if (w && first < last) ws.load(w, at, turn, LPR);
        for (int h = first; h < last; h += U) {
            Eight<T> x[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (h + u < last) x[u].load(at.row<T>(X, h + u));
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (h + u >= last) break;
                float a[8], ao[8], y[8];
                x[u].get(a);
                x[u].of_lane(turn.other).get(ao);
                if (w) {
                    float ss = 0.f, f[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) ss = __builtin_fmaf(a[e], a[e], ss);
                    const float r = 1.f / __builtin_sqrtf(row_sum<LPR>(ss) * (1.f / D) + eps);
                    ws.mine.get(f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) a[e] *= r * f[e];
                    ws.other.get(f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) ao[e] *= r * f[e];
                }
                turn.apply(a, ao, y);
                x[u].set(y);
                if (at.real) {
                    if constexpr (PAST) x[u].store_past(at.row<T>(Y, h + u));
                    else x[u].store(at.row<T>(Y, h + u));
                }
            }
        }
    }
}

// Workgroups of the backward pass, queries and keys together: each leaves one partial sum of dw.  1024 are four for each compute unit,
// which is all that 128 registers let in.  One row in flight in each of these (the two gradient cases above: 31.1 and 44.8 us) is level
// with two in each of 768 (32.9 and 46.5); two in 1024 do not fit into the registers (42 and 55).
constexpr int kGradGroups = 1024;
// The last-level cache.
constexpr long kCacheBytes = 256L << 20;
// Waves that the forward pass wants: as many as the chip holds (256 compute units, 32 waves each).
constexpr long kForwardWaves = 8192;

__device__ __forceinline__ HeadRows either(bool first, const HeadRows &a, const HeadRows &b) {
    return HeadRows{first ? a.data : b.data, first ? a.batch : b.batch, first ? a.token : b.token, first ? a.head : b.head, first ? a.H : b.H};
}

// Queries in the first `qgroups` workgroups, keys in the others; a wave goes over units of 64 / (d / 8) tokens and `each` heads.
// PAST: what is read and written leaves the caches first, but for dy (backward).
template <typename T, int D, int U, bool PAST>
__global__ __launch_bounds__(256, 4) void k_norm_rotate_grad(HeadRows dQo, HeadRows dKo, HeadRows Q, HeadRows K,
                                                          const T *__restrict__ wq, const T *__restrict__ wk, float eps,
                                                          RotaryTable rt, long tokens, int L, HeadRows dQ, HeadRows dK,
                                                          int qgroups, int each, float *__restrict__ part) {
    constexpr int LPR = D / 8, TPW = 64 / LPR;
    __shared__ float sums[4][D];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l = threadIdx.x & 63;
    const bool key = (int)blockIdx.x >= qgroups;
    const HeadRows Y = either(key, dKo, dQo), X = either(key, K, Q), dX = either(key, dK, dQ);
    const T *const w = key ? wk : wq;
    const int group = key ? blockIdx.x - qgroups : blockIdx.x, groups = key ? gridDim.x - qgroups : qgroups;
    // (whatever follows from a division is vector work unless it is read back)
    const int parts = __builtin_amdgcn_readfirstlane((X.H + each - 1) / each);
    const long units = (tokens + TPW - 1) / TPW * parts;
    float dw[8];
    Eight<T> wv;
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[e] = 0.f;
    if (w) wv.load(w + 8 * (l % LPR));
    for (long unit = (long)group * 4 + wave; unit < units; unit += 4L * groups) {
        const unsigned tg = __builtin_amdgcn_readfirstlane((unsigned)unit / (unsigned)parts);   // (fewer than 2^28 units)
        const int from = __builtin_amdgcn_readfirstlane((int)((unsigned)unit - tg * parts) * each), to = from + each < X.H ? from + each : X.H;
        const Place at = Place::of<LPR>((long)tg * TPW, tokens, L);
        Turn turn;
        turn.load(rt.cos, rt.sin, rt.at(at.token, at.t), rt.rot, rt.interleaved != 0, at.lane, at.c, true);
        for (int h = from; h < to; h += U) {
            Eight<T> y[U], x[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (h + u < to) {
                    y[u].load(at.row<const T>(Y, h + u));
                    if constexpr (PAST) {
                        if (w) x[u].load_once(at.row<const T>(X, h + u));
                    } else {
                        if (w) x[u].load(at.row<const T>(X, h + u));
                    }
                }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (h + u >= to) break;
                float dy[8], dyo[8], dz[8];
                y[u].get(dy);
                y[u].of_lane(turn.other).get(dyo);
                turn.apply(dy, dyo, dz);
                if (w) {
                    float a[8], f[8], ss = 0.f, gx = 0.f;
                    x[u].get(a);
                    wv.get(f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        ss = __builtin_fmaf(a[e], a[e], ss);
                        gx = __builtin_fmaf(dz[e] * f[e], a[e], gx);
                    }
                    ss = row_sum<LPR>(ss);
                    gx = row_sum<LPR>(gx);
                    const float r = 1.f / __builtin_sqrtf(ss * (1.f / D) + eps), k = r * r * (gx * (1.f / D)), rr = at.real ? r : 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        dw[e] = __builtin_fmaf(dz[e] * rr, a[e], dw[e]);
                        dz[e] = r * (dz[e] * f[e] - a[e] * k);
                    }
                }
                y[u].set(dz);
                if (at.real) {
                    if constexpr (PAST) y[u].store_past(at.row<T>(dX, h + u));
                    else y[u].store(at.row<T>(dX, h + u));
                }
            }
        }
    }
    if (!w) return;   // (the same in every thread of the workgroup)
    // the workgroup's sum of dw: over the rows that a wave holds side by side, then over its waves, in a fixed order
#pragma unroll
    for (int e = 0; e < 8; ++e) {
#pragma unroll
        for (int o = 32; o >= LPR; o >>= 1) dw[e] += __shfl_xor(dw[e], o, kWave);
    }
    if (l < LPR) {
#pragma unroll
        for (int e = 0; e < 8; ++e) sums[wave][8 * l + e] = dw[e];
    }
    __syncthreads();
    if (threadIdx.x < D)
        part[(long)blockIdx.x * D + threadIdx.x] =
            (sums[0][threadIdx.x] + sums[1][threadIdx.x]) + (sums[2][threadIdx.x] + sums[3][threadIdx.x]);
}

// dw from the workgroups' sums: a workgroup forms eight columns, 32 threads a column.  blockIdx.y: 0 queries, 1 keys.
template <int D>
__global__ __launch_bounds__(256) void k_norm_weight_grad(const float *__restrict__ part, int qgroups, int groups,
                                                          float *__restrict__ dwq, float *__restrict__ dwk) {
    __shared__ float sums[32][9];
    float *const dw = blockIdx.y ? dwk : dwq;
    if (!dw) return;
    const int from = blockIdx.y ? qgroups : 0, to = blockIdx.y ? groups : qgroups;
    const int col = threadIdx.x & 7, i = threadIdx.x >> 3;
    float s = 0.f;
    for (int p = from + i; p < to; p += 8 * 32) {   // eight on their way at a time
        float x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = part[(long)(p + 32 * k < to ? p + 32 * k : p) * D + 8 * blockIdx.x + col];
#pragma unroll
        for (int k = 0; k < 8; ++k) s += p + 32 * k < to ? x[k] : 0.f;
    }
    sums[i][col] = s;
    __syncthreads();
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        if (i < o) sums[i][col] += sums[i + o][col];
        __syncthreads();
    }
    if (i == 0) dw[8 * blockIdx.x + col] = sums[0][col];
}

// Heads that a wave goes through, for `groups` groups of tokens: as many as leave waves for the whole chip.
int heads_each(long groups, int heads, long waves) {
    long parts = (waves + groups - 1) / groups;
    parts = parts < 1 ? 1 : parts > heads ? heads : parts;
    return (int)((heads + parts - 1) / parts);
}

// Results of bfloat16 leave the caches first, up to half of the last-level cache: 84 MB (4 x 1024 tokens of 32 + 8 heads, d = 128)
// 18.9 us without and 17.6 with it, 100 MB (16 x 1024, 12 + 12, d = 64) 20.5 and 19.2, and behind it 134 MB 24.1 and 24.3, 268 MB 49.5
// and 51.4.  Of float a lane stores two halves of 32 bytes, which then leave apart from each other: 100 MB 18.1 and 20.5.
bool forward_past(long tokens, int heads, int d, int elem) { return elem == 2 && 2 * tokens * heads * d * elem <= kCacheBytes / 2; }
// A call that leaves little of the last-level cache to others reads x and writes dx past it, so that dy, which was just written, stays:
// 202 MB (4 x 2048 tokens of 16 + 16 heads, d = 128) 52.1 us without and 40.6 with it, 403 MB 95.8 and 82.7, float 89.1 and 79.4;
// smaller ones find x there, too: 126 MB (4 x 1024, 32 + 8) 31.2 and 34.6, float 151 MB 31.7 and 33.8.
bool backward_past(long tokens, int heads, int d, int elem) { return 3 * tokens * heads * d * elem > kCacheBytes * 5 / 8; }
int forward_each(long tokens, int heads, int d) { return heads_each((tokens + 512 / d - 1) / (512 / d), heads, kForwardWaves); }

template <typename T, int D>
hipError_t forward(const HeadRows &Q, const HeadRows &K, const void *wq, const void *wk, float eps, const RotaryTable &rt, long B,
                   int L, const HeadRows &Qo, const HeadRows &Ko, hipStream_t st) {
    constexpr int TPW = 512 / D;
    const long tokens = B * L, groups = (tokens + TPW - 1) / TPW;
    const int heads = Q.H + K.H, each = forward_each(tokens, heads, D), parts = (heads + each - 1) / each;
    const dim3 grid((unsigned)((groups * parts + 3) / 4));
    const bool past = forward_past(tokens, heads, D, sizeof(T));
#define DFSS_LAUNCH(U)                                                                                                   \
    if (past) DFSS_PAST(U, sizeof(T) == 2); else DFSS_PAST(U, false)
#define DFSS_PAST(U, PAST)                                                                                               \
    hipLaunchKernelGGL((k_norm_rotate<T, D, U, PAST>), grid, dim3(256), 0, st, Q, K, (const T *)wq, (const T *)wk, eps, rt, tokens, L, \
                       Qo, Ko, parts, each)
    // four rows on their way where a wave has four heads to go through; else their registers would only keep waves out
    if (each >= 4) { DFSS_LAUNCH(4); } else { DFSS_LAUNCH(1); }
#undef DFSS_PAST
#undef DFSS_LAUNCH
    return hipGetLastError();
}

template <typename T, int D>
hipError_t backward(const HeadRows &dQo, const HeadRows &dKo, const HeadRows &Q, const HeadRows &K, const void *wq, const void *wk,
                    float eps, const RotaryTable &rt, long B, int L, const HeadRows &dQ, const HeadRows &dK, float *dwq, float *dwk,
                    float *part, hipStream_t st) {
    constexpr int TPW = 512 / D, U = 1;
    const long tokens = B * L, tg = (tokens + TPW - 1) / TPW;
    const int each = heads_each(tg, Q.H + K.H, 4 * kGradGroups);
    const long q = tg * ((Q.H + each - 1) / each), k = K.H ? tg * ((K.H + each - 1) / each) : 0;   // units
    long qg = (q + 3) / 4, kg = (k + 3) / 4;
    if (qg + kg > kGradGroups) {   // shared out by their work
        qg = kGradGroups * q / (q + k);
        if (qg < 1) qg = 1;
        if (k && qg > kGradGroups - 1) qg = kGradGroups - 1;
        kg = k ? kGradGroups - qg : 0;
    }
    const bool past = backward_past(tokens, Q.H + K.H, D, sizeof(T));
#define DFSS_LAUNCH(PAST)                                                                                                \
    hipLaunchKernelGGL((k_norm_rotate_grad<T, D, U, PAST>), dim3((unsigned)(qg + kg)), dim3(256), 0, st, dQo, dKo, Q, K, (const T *)wq, \
                       (const T *)wk, eps, rt, tokens, L, dQ, dK, (int)qg, each, part)
    if (past) DFSS_LAUNCH(true); else DFSS_LAUNCH(false);
#undef DFSS_LAUNCH
    if (wq || wk)
        hipLaunchKernelGGL((k_norm_weight_grad<D>), dim3(D / 8, 2), dim3(256), 0, st, part, (int)qg, (int)(qg + kg),
                           wq ? dwq : nullptr, wk ? dwk : nullptr);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm_rotate(const HeadRows &Q, const HeadRows &K, const void *wq, const void *wk, float eps, const RotaryTable &rt,
                              long B, int L, int d, bool f32, const HeadRows &Qo, const HeadRows &Ko, hipStream_t st) {
#define DFSS_CALL(T, D) forward<T, D>(Q, K, wq, wk, eps, rt, B, L, Qo, Ko, st)
    if (f32) return d == 64 ? DFSS_CALL(float, 64) : DFSS_CALL(float, 128);
    return d == 64 ? DFSS_CALL(__bf16, 64) : DFSS_CALL(__bf16, 128);
#undef DFSS_CALL
}

NormPlan norm_rotate_plan(long tokens, int heads, int d, int elem) {
    return NormPlan{forward_each(tokens, heads, d) >= 4 ? 4 : 1, forward_past(tokens, heads, d, elem), backward_past(tokens, heads, d, elem)};
}

size_t norm_rotate_workspace_bytes(int d) { return (size_t)kGradGroups * d * sizeof(float); }

hipError_t launch_norm_rotate_grad(const HeadRows &dQo, const HeadRows &dKo, const HeadRows &Q, const HeadRows &K, const void *wq,
                                   const void *wk, float eps, const RotaryTable &rt, long B, int L, int d, bool f32,
                                   const HeadRows &dQ, const HeadRows &dK, float *dwq, float *dwk, float *part, hipStream_t st) {
#define DFSS_CALL(T, D) backward<T, D>(dQo, dKo, Q, K, wq, wk, eps, rt, B, L, dQ, dK, dwq, dwk, part, st)
    if (f32) return d == 64 ? DFSS_CALL(float, 64) : DFSS_CALL(float, 128);
    return d == 64 ? DFSS_CALL(__bf16, 64) : DFSS_CALL(__bf16, 128);
#undef DFSS_CALL
}

}  // namespace dfss
