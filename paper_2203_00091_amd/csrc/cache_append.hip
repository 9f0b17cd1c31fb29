// New keys and values into a paged cache of 8 bits; the keys are normed and rotated on the way.
//
// A page holds 16 to 128 tokens of one sequence; for every page and key head the cache keeps the e4m3 codes of K and V,
// [page, d], and one scale each, s = 2^ceil(log2(amax / 448)) over what the page holds (448 is the largest e4m3 value, so
// |x| / s <= 448 and nothing saturates; at least 2^-64).  Powers of two, because the reader then gets its bfloat16
// operands from one conversion instruction, exactly, and because codes that a larger scale replaces keep their three bits
// of fraction (only those that become subnormal are rounded again).
//
// Bound by memory (2 bytes read and 1 written for each value), and by latency where a sequence gets one token.  A
// workgroup owns what a call adds to one page of one head, of K or of V, so that nobody else touches the page's scale:
// it holds the new rows in registers, finds their amax, and with the old scale, where the page holds earlier tokens, the
// new one; the earlier codes are read and written only if it grew.
#include "dfss_kernels.hpp"
#include "head_rows.hpp"

namespace dfss {

namespace {

// 2^ceil(log2(amax / 448)), at least 2^-64; amax >= 0.  448 = 1.75 * 2^8.
__device__ __forceinline__ int scale_exponent(float amax) {
    const uint32_t u = __builtin_bit_cast(uint32_t, amax);
    const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return e < -64 ? -64 : e;
}
__device__ __forceinline__ float exp2_int(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }

__device__ __forceinline__ u32x2 encode(const float *x, float inv) {   // eight values, nearest-even
    u32x2 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i] * inv, x[4 * i + 1] * inv, 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2] * inv, x[4 * i + 3] * inv, w, true);
        r[i] = (uint32_t)w;
    }
    return r;
}
__device__ __forceinline__ void decode(u32x2 c, float *x) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i], true);
        x[4 * i] = a[0], x[4 * i + 1] = a[1], x[4 * i + 2] = b[0], x[4 * i + 3] = b[1];
    }
}

// Grid: x = slots, y = head, z = 0 for K and 1 for V.  Sequence b has the slots from cu[b] / page + 2 b on: more than the
// pages that its tokens lie in ((n - 1) / page + 2 at most), and sequence and page follow from the slot by one look at cu.
// NP passes of 2048 / D rows make up a page.
template <int D, int NP>
__global__ __launch_bounds__(256) void k_cache_append(HeadRows K, HeadRows V, int T, const int *__restrict__ cu, int B, int most,
                                                      int max_len, const __bf16 *__restrict__ w, float eps, RotaryTable rt,
                                                      PagedCache cache) {
    constexpr int LPR = D / 8, RPP = 256 / LPR;
    __shared__ float amax4[4];
    const int l = threadIdx.x & 63, c = threadIdx.x % LPR, row = threadIdx.x / LPR;
    const int page = 1 << cache.page_shift, head = blockIdx.y;
    const bool is_v = blockIdx.z != 0;

    int b, lo, n, slot;
    if (cu) {
        int before = 0;   // sequences whose slots begin at or before this one
        for (int i = 0; i < B; i += 64) {
            const int at = i + l < B ? i + l : B - 1;
            int first = cu[at];
            first = first < 0 ? 0 : first < T ? first : T;
            before += __popcll(__ballot(i + l < B && (first >> cache.page_shift) + 2 * at <= (int)blockIdx.x));
        }
        if (before == 0) return;
        b = before - 1;
        lo = cu[b], n = cu[b + 1];
        lo = lo < 0 ? 0 : lo < T ? lo : T;
        n = n < lo ? lo : n < T ? n : T;
        n -= lo;
        slot = (int)blockIdx.x - (lo >> cache.page_shift) - 2 * b;
    } else {
        const int per = (most - 1) / page + 2;
        b = (int)blockIdx.x / per;
        slot = (int)blockIdx.x - b * per;
        lo = b * most;
        n = most;
    }
    if (n <= 0) return;
    const int len = cache.len[b] < 0 ? 0 : cache.len[b];
    const long capacity = (long)cache.width << cache.page_shift;
    const int limit = max_len < capacity ? max_len : (int)capacity;   // tokens from here on are not kept
    const int start = len - n;
    const int from = start < 0 ? 0 : start, to = len < limit ? len : limit;
    const int p = (from >> cache.page_shift) + slot;
    const int first = from > p * page ? from : p * page, end = to < (p + 1) * page ? to : (p + 1) * page;
    if (p >= cache.width || first >= end) return;
    const int id = cache.table[(long)b * cache.width + p];
    if ((unsigned)id >= (unsigned)cache.n_pages) return;   // no such page: its tokens are not kept
    const int s0 = first - p * page, s1 = end - p * page;  // the page's rows that are written
    const HeadRows &X = is_v ? V : K;
    const __bf16 *const src = static_cast<const __bf16 *>(X.data) + head * X.head + 8 * c;
    const long token0 = (long)lo + (p * (long)page - start);   // the token of the page's row 0 (may lie before the first)

    Eight<__bf16> raw[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int r = i * RPP + row;
        raw[i].clear();
        if (r >= s0 && r < s1) raw[i].load(src + (token0 + r) * X.token);
    }
    float x[NP][8], amax = 0.f;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int r = i * RPP + row;
        raw[i].get(x[i]);
        if (!is_v && (i * RPP < s1 && (i + 1) * RPP > s0)) {   // (the same in every lane)
            const long token = token0 + r;
            const bool real = r >= s0 && r < s1;
            Turn turn;
            turn.load(rt.cos, rt.sin, real ? rt.at(token, start + (token - lo)) : 0, rt.rot, rt.interleaved != 0, l, c, false);
            float xo[8];
            raw[i].of_lane(turn.other).get(xo);
            // In 64 bits: a code has a border every 16th of its value, and each 32-bit rounding on the way would put a few of a
            // million values on the wrong side of theirs.  (Free here: 24 operations for three bytes that pass the memory.)
            double f[8], fo[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = x[i][e], fo[e] = xo[e];
            if (w) {
                double ss = 0.;
                float wf[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) ss += f[e] * f[e];
#pragma unroll
                for (int o = LPR / 2; o > 0; o >>= 1) ss += __shfl_xor(ss, o, kWave);
                const double rn = 1. / __builtin_sqrt(ss * (1. / D) + eps);
                Eight<__bf16> v;
                v.load(w + 8 * c);
                v.get(wf);
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] *= rn * wf[e];
                v.load(w + 8 * (turn.other % LPR));
                v.get(wf);
#pragma unroll
                for (int e = 0; e < 8; ++e) fo[e] *= rn * wf[e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] = (float)(f[e] * turn.cos[e] + (turn.interleaved ? f[e ^ 1] : fo[e]) * turn.sin[e]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = fmaxf(amax, __builtin_fabsf(x[i][e]));
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor(amax, o, kWave));
    if (l == 0) amax4[threadIdx.x >> 6] = amax;
    float *const scale = (is_v ? cache.v_scale : cache.k_scale) + (long)id * cache.Hk + head;
    uint8_t *const codes = (is_v ? cache.v : cache.k) + (((long)id * cache.Hk + head) << cache.page_shift) * D + 8 * c;
    const float old = s0 > 0 ? *scale : 0.f;
    __syncthreads();   // (also: everybody has read the old scale)
    const int e = scale_exponent(fmaxf(fmaxf(amax4[0], amax4[1]), fmaxf(amax4[2], amax4[3])));
    float now = exp2_int(e);
    if (old >= now) {
        now = old;
    } else if (s0 > 0) {
        const float ratio = old / now;   // (both powers of two)
        for (int r = row; r < s0; r += RPP) {
            u32x2 *const at = reinterpret_cast<u32x2 *>(codes + (long)r * D);
            float v[8];
            decode(*at, v);
            *at = encode(v, ratio);
        }
    }
    if (threadIdx.x == 0) *scale = now;
    const float inv = 1.f / now;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int r = i * RPP + row;
        if (r >= s0 && r < s1) *reinterpret_cast<u32x2 *>(codes + (long)r * D) = encode(x[i], inv);
    }
}

}  // namespace

hipError_t launch_cache_append(const HeadRows &K, const HeadRows &V, int T, const int *cu, int B, int most, int max_len, int d,
                               const void *w, float eps, const RotaryTable &rt, const PagedCache &c, hipStream_t st) {
    const int page = 1 << c.page_shift, passes = page * d / 2048;
    const unsigned slots = cu ? (unsigned)(T / page + 2 * B) : (unsigned)B * (unsigned)((most - 1) / page + 2);
    const dim3 grid(slots, (unsigned)c.Hk, 2);
#define DFSS_LAUNCH(D, NP)                                                                                              \
    hipLaunchKernelGGL((k_cache_append<D, NP>), grid, dim3(256), 0, st, K, V, T, cu, B, most, max_len, (const __bf16 *)w, eps, rt, c)
    if (d == 64) {
        if (passes <= 1) DFSS_LAUNCH(64, 1); else if (passes == 2) DFSS_LAUNCH(64, 2); else DFSS_LAUNCH(64, 4);
    } else {
        if (passes <= 1) DFSS_LAUNCH(128, 1); else if (passes == 2) DFSS_LAUNCH(128, 2); else if (passes == 4) DFSS_LAUNCH(128, 4); else DFSS_LAUNCH(128, 8);
    }
#undef DFSS_LAUNCH
    return hipGetLastError();
}

}  // namespace dfss
