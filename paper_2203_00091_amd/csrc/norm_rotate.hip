// Norm of every head's query and key, and the rotation to its position, in one pass; and its gradients.
//
// For a row x of d elements (one token, one head), with the weight w and the token's angles:
//     r = (mean(x^2) + eps)^(-1/2),   z = x r w,   y = R z
// where R turns the pairs of the first `rot` elements.  Without a weight z = x.  Gradients, from dy:
//     dz = R^T dy,   dw = sum over rows of dz x r,   g = dz w,   dx = r (g - x r^2 mean(g x)).
// All of it in 32 bits, rounded once at the end.
//
// Bound by memory: every element is read and written once (the backward pass reads x and dy).  A lane holds eight
// elements of a row, so a row is d / 8 lanes; a wave takes one token and HPW x U heads of it, so that the angles are read
// once for all of them, and all its loads are on their way before the first is used.
#include "dfss_kernels.hpp"
#include "head_rows.hpp"

namespace dfss {

namespace {

// Row of head h, counted through those of Q and then of K.
template <typename T>
__device__ __forceinline__ T *row(const HeadRows &Q, const HeadRows &K, int h, long b, long t) {
    const bool q = h < Q.H;
    return static_cast<T *>(q ? Q.data : K.data) + b * (q ? Q.batch : K.batch) + t * (q ? Q.token : K.token) +
           (q ? h : h - Q.H) * (q ? Q.head : K.head);
}

template <typename T, int D, int U>
__global__ __launch_bounds__(256) void k_norm_rotate(HeadRows Q, HeadRows K, const T *__restrict__ wq, const T *__restrict__ wk,
                                                     float eps, RotaryTable rt, long tokens, int L, HeadRows Qo, HeadRows Ko) {
    constexpr int LPR = D / 8, HPW = 64 / LPR;
    const int l = threadIdx.x & 63, c = l % LPR, g = l / LPR;
    const int heads = Q.H + K.H, parts = (heads + HPW * U - 1) / (HPW * U);
    const long unit = (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const long token = unit / parts;
    if (token >= tokens) return;
    const int h0 = (int)(unit - token * parts) * HPW * U + g;
    const long b = token / L, t = token - b * L;

    Eight<T> x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int h = h0 + u * HPW;
        x[u].clear();
        if (h < heads) {
            x[u].load(row<T>(Q, K, h, b, t) + 8 * c);
        }
    }
    Turn turn;
    turn.load(rt.cos, rt.sin, rt.at(token, t), rt.rot, rt.interleaved != 0, l, c, false);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int h = h0 + u * HPW;
        const T *const w = h < Q.H ? wq : wk;
        float a[8], ao[8], y[8], r = 1.f;
        x[u].get(a);
        x[u].of_lane(turn.other).get(ao);
        if (wq || wk) {
            float ss = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) ss = __builtin_fmaf(a[e], a[e], ss);
            ss = row_sum<LPR>(ss);
            if (w) {
                r = 1.f / __builtin_sqrtf(ss * (1.f / D) + eps);
                Eight<T> v;
                float f[8];
                v.load(w + 8 * c);
                v.get(f);
#pragma unroll
                for (int e = 0; e < 8; ++e) a[e] *= r * f[e];
                v.load(w + 8 * (turn.other % LPR));
                v.get(f);
#pragma unroll
                for (int e = 0; e < 8; ++e) ao[e] *= r * f[e];
            }
        }
        turn.apply(a, ao, y);
        if (h < heads) {
            x[u].set(y);
            x[u].store(row<T>(Qo, Ko, h, b, t) + 8 * c);
        }
    }
}

// Workgroups of the backward pass, queries and keys together: each leaves one partial sum of dw.
constexpr int kGradGroups = 512;

// Queries in the first `qgroups` workgroups, keys in the others; a wave goes over units of one token and HPW x U heads.
template <typename T, int D, int U>
__global__ __launch_bounds__(256) void k_norm_rotate_grad(HeadRows dQo, HeadRows dKo, HeadRows Q, HeadRows K,
                                                          const T *__restrict__ wq, const T *__restrict__ wk, float eps,
                                                          RotaryTable rt, long tokens, int L, HeadRows dQ, HeadRows dK,
                                                          int qgroups, float *__restrict__ part) {
    constexpr int LPR = D / 8, HPW = 64 / LPR;
    __shared__ float sums[4][D];
    const int l = threadIdx.x & 63, c = l % LPR, g = l / LPR, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const bool key = (int)blockIdx.x >= qgroups;
    const HeadRows &Y = key ? dKo : dQo, &X = key ? K : Q, &dX = key ? dK : dQ;
    const T *const w = key ? wk : wq;
    const int group = key ? blockIdx.x - qgroups : blockIdx.x, groups = key ? gridDim.x - qgroups : qgroups;
    const int parts = (X.H + HPW * U - 1) / (HPW * U);
    const long units = tokens * parts;
    float f[8], dw[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = 1.f, dw[e] = 0.f;
    if (w) {
        Eight<T> v;
        v.load(w + 8 * c);
        v.get(f);
    }
    for (long unit = (long)group * 4 + wave; unit < units; unit += 4L * groups) {
        const long token = unit / parts, b = token / L, t = token - b * L;
        const int h0 = (int)(unit - token * parts) * HPW * U + g;
        Eight<T> y[U], x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = h0 + u * HPW;
            y[u].clear();
            x[u].clear();
            if (h < X.H) {
                y[u].load(static_cast<const T *>(Y.data) + b * Y.batch + t * Y.token + h * Y.head + 8 * c);
                if (w) x[u].load(static_cast<const T *>(X.data) + b * X.batch + t * X.token + h * X.head + 8 * c);
            }
        }
        Turn turn;
        turn.load(rt.cos, rt.sin, rt.at(token, t), rt.rot, rt.interleaved != 0, l, c, true);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = h0 + u * HPW;
            float dy[8], dyo[8], dz[8];
            y[u].get(dy);
            y[u].of_lane(turn.other).get(dyo);
            turn.apply(dy, dyo, dz);
            if (w) {
                float a[8], ss = 0.f, gx = 0.f;
                x[u].get(a);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    ss = __builtin_fmaf(a[e], a[e], ss);
                    gx = __builtin_fmaf(dz[e] * f[e], a[e], gx);
                }
                ss = row_sum<LPR>(ss);
                gx = row_sum<LPR>(gx);
                const float r = 1.f / __builtin_sqrtf(ss * (1.f / D) + eps), k = r * r * (gx * (1.f / D));
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    dw[e] = __builtin_fmaf(dz[e] * r, a[e], dw[e]);
                    dz[e] = r * (dz[e] * f[e] - a[e] * k);
                }
            }
            if (h < X.H) {
                y[u].set(dz);
                y[u].store(static_cast<T *>(dX.data) + b * dX.batch + t * dX.token + h * dX.head + 8 * c);
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
    if (g == 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) sums[wave][8 * c + e] = dw[e];
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
    for (int p = from + i; p < to; p += 32) s += part[(long)p * D + 8 * blockIdx.x + col];
    sums[i][col] = s;
    __syncthreads();
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        if (i < o) sums[i][col] += sums[i + o][col];
        __syncthreads();
    }
    if (i == 0) dw[8 * blockIdx.x + col] = sums[0][col];
}

template <typename T, int D>
hipError_t forward(const HeadRows &Q, const HeadRows &K, const void *wq, const void *wk, float eps, const RotaryTable &rt, long B,
                   int L, const HeadRows &Qo, const HeadRows &Ko, hipStream_t st) {
    constexpr int HPW = 512 / D;
    const long tokens = B * L;
    const int heads = Q.H + K.H;
    const int u = heads > 2 * HPW && tokens >= 512 ? 4 : heads > HPW && tokens >= 512 ? 2 : 1;
    const long units = tokens * ((heads + HPW * u - 1) / (HPW * u));
    const dim3 grid((unsigned)((units + 3) / 4));
#define DFSS_LAUNCH(U)                                                                                                   \
    hipLaunchKernelGGL((k_norm_rotate<T, D, U>), grid, dim3(256), 0, st, Q, K, (const T *)wq, (const T *)wk, eps, rt, tokens, L, Qo, Ko)
    if (u == 4) DFSS_LAUNCH(4); else if (u == 2) DFSS_LAUNCH(2); else DFSS_LAUNCH(1);
#undef DFSS_LAUNCH
    return hipGetLastError();
}

template <typename T, int D>
hipError_t backward(const HeadRows &dQo, const HeadRows &dKo, const HeadRows &Q, const HeadRows &K, const void *wq, const void *wk,
                    float eps, const RotaryTable &rt, long B, int L, const HeadRows &dQ, const HeadRows &dK, float *dwq, float *dwk,
                    float *part, hipStream_t st) {
    constexpr int HPW = 512 / D, U = 2;
    const long tokens = B * L;
    auto units = [&](int H) { return tokens * ((H + HPW * U - 1) / (HPW * U)); };
    const long q = units(Q.H), k = K.H ? units(K.H) : 0;
    long qg = (q + 3) / 4, kg = (k + 3) / 4;
    if (qg + kg > kGradGroups) {   // shared out by their work
        long part_q = kGradGroups * q / (q + k);
        if (part_q < 1) part_q = 1;
        if (k && part_q > kGradGroups - 1) part_q = kGradGroups - 1;
        qg = part_q;
        kg = k ? kGradGroups - part_q : 0;
    }
    hipLaunchKernelGGL((k_norm_rotate_grad<T, D, U>), dim3((unsigned)(qg + kg)), dim3(256), 0, st, dQo, dKo, Q, K, (const T *)wq,
                       (const T *)wk, eps, rt, tokens, L, dQ, dK, (int)qg, part);
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
