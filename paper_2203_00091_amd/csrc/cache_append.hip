// New keys and values into a paged cache of 8 bits; the keys are normed and rotated on the way.
//
// A page holds 16 to 128 tokens of one sequence; for every page and key head the cache keeps the e4m3 codes of K and V,
// [page, d], and one scale each, s = 2^ceil(log2(amax / 448)) over what the page holds (448 is the largest e4m3 value, so
// |x| / s <= 448 and nothing saturates; at least 2^-64).  Powers of two, because the reader then gets its bfloat16
// operands from one conversion instruction, exactly, and because codes that a larger scale replaces keep their three bits
// of fraction (only those that become subnormal are rounded again).
//
// Bound by memory (2 bytes read and 1 written for each value), and by latency where a sequence gets one token.  What a call
// adds to one page of one head, of K or of V, is a unit's, so that nobody else touches the page's scale: it holds the new rows
// in registers, finds their amax, and with the old scale, where the page holds earlier tokens, the new one; the earlier codes are
// read and written only if it grew.  A unit is a wave where four of its passes (8 elements in each lane) hold the rows, else a
// workgroup.
//
// Measured: 8 sequences of up to 2048 tokens (12k in all) x 16 heads, d = 64, pages of 16, 79 MB, 22.6 us = 3.5 TB/s (1 of them to round to odd); one token each
// of 64 sequences, 8 heads, d = 128, pages of 64, 5.4 us: a chain of reads (offsets, length, page, scale, codes of the page if the
// scale grew), 0.4 MB.
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

// y in 32 bits, cut, the lowest bit set where something was cut off (rounded to odd): rounding that to the nearest of fewer bits, or
// comparing it with a number of fewer, has the outcome that y would have had.
__device__ __forceinline__ float to_odd(double y) {
    const uint64_t u = __builtin_bit_cast(uint64_t, y);
    uint32_t lo = (uint32_t)u;
    lo = (lo | ((lo & 0x1FFFFFFFu) + 0x1FFFFFFFu)) & 0xE0000000u;
    return (float)__builtin_bit_cast(double, (u & 0xFFFFFFFF00000000u) | lo);
}

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

// Grid: x = slots, y = K and V of the heads: a unit takes `each` of them, one after the other.  Sequence b has the slots from cu[b] / page + 2 b
// on: more than the pages that its tokens lie in ((n - 1) / page + 2 at most), and sequence and page follow from the slot by a look
// at cu, two from 65 sequences on, three from 4097 on.  (A look at every 64 sequences, one token each of 1024, 4096 and 16384: 23, 201 and
// 1612 us, so 12, 38 and 100.)
template <int D, int WU, int NP>
__global__ __launch_bounds__(256) void k_cache_append(HeadRows K, HeadRows V, int T, const int *__restrict__ cu, int B, int most,
                                                      int max_len, const __bf16 *__restrict__ w, float eps, RotaryTable rt,
                                                      PagedCache cache, int each) {
    constexpr int LPR = D / 8, RPP = 64 * WU / LPR;   // lanes of a row; rows of a pass
    __shared__ float amax4[4];
    const int l = threadIdx.x & 63, c = threadIdx.x % LPR, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int row = (WU == 1 ? l : (int)threadIdx.x) / LPR;
    const int page = 1 << cache.page_shift;
    // (the four waves of a workgroup take neighbouring heads, whose rows are one piece of the token's)
    constexpr int STEP = WU == 1 ? 4 : 1;
    const bool is_v = blockIdx.y & 1;
    const int group = ((int)blockIdx.y >> 1) * each * STEP, head0 = group + (WU == 1 ? wave : 0);
    const int heads = group + each * STEP < cache.Hk ? group + each * STEP : cache.Hk;
    if (head0 >= heads) return;

    int b = -1, lo = 0, n = 0, slot = 0, len = 0;
    if (cu) {
        // the last sequence whose slots begin at or before this one: 64 places of the range at a time, until it is 64 sequences
        int base = 0, span = B;
        auto first_of = [&](int from, int at) { return ((from < 0 ? 0 : from < T ? from : T) >> cache.page_shift) + 2 * at; };
        while (span > 64) {
            const int step = (span + 63) / 64, at = base + l * step;
            const bool in = l * step < span;
            const uint64_t before = __ballot(in && first_of(cu[in ? at : base], at) <= (int)blockIdx.x);
            if (!before) return;
            const int skip = (63 - __builtin_clzll(before)) * step;
            base += skip;
            span = span - skip < step ? span - skip : step;
        }
        const int at = l < span ? base + l : base, length = cache.len[at];
        int from = cu[at], to = cu[at + 1];
        const int first = first_of(from, at);
        from = from < 0 ? 0 : from < T ? from : T;
        to = to < from ? from : to < T ? to : T;
        const uint64_t before = __ballot(l < span && first <= (int)blockIdx.x);
        if (!before) return;
        const int lane = 63 - __builtin_clzll(before);
        b = base + lane;
        lo = __builtin_amdgcn_readlane(from, lane);
        n = __builtin_amdgcn_readlane(to, lane) - lo;
        slot = (int)blockIdx.x - __builtin_amdgcn_readlane(first, lane);
        len = __builtin_amdgcn_readlane(length, lane);
    } else {
        const int per = (most - 1) / page + 2;
        b = __builtin_amdgcn_readfirstlane((int)blockIdx.x / per);
        slot = (int)blockIdx.x - b * per;
        lo = b * most;
        n = most;
        len = cache.len[b];
    }
    if (n <= 0) return;
    len = len < 0 ? 0 : len;
    const long capacity = (long)cache.width << cache.page_shift;
    const int limit = max_len < capacity ? max_len : (int)capacity;   // tokens from here on are not kept
    const int start = len - n;
    const int from = start < 0 ? 0 : start, to = len < limit ? len : limit;
    const int p = (from >> cache.page_shift) + slot;
    const int first = from > p * page ? from : p * page, end = to < (p + 1) * page ? to : (p + 1) * page;
    if (p >= cache.width || first >= end) return;
    const int id = cache.table[(long)b * cache.width + p];
    if ((unsigned)id >= (unsigned)cache.n_pages) return;   // no such page: its tokens are not kept
    const int s0 = first - p * page, rows = end - first;   // the page's rows that are written
    const HeadRows &X = is_v ? V : K;
    const long token0 = (long)lo + (first - start);         // token of row s0
    const __bf16 *const src = static_cast<const __bf16 *>(X.data) + token0 * X.token + 8 * c;

    Eight<__bf16> w_mine, w_other, raw[NP];
    if (w) w_mine.load(w + 8 * c);
    float x[NP][8], old = 0.f;
    float *const scales = static_cast<float *>(is_v ? cache.v_scale : cache.k_scale) + (long)id * cache.Hk;
    auto load = [&](int head, int g0) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int r = g0 + i * RPP + row;
            raw[i].clear();
            if (r < rows) raw[i].load(src + r * X.token + head * X.head);
        }
    };
    // x = the values of the new rows g0 .. g0 + NP RPP - 1 (0 where there are fewer), from raw
    auto values = [&](int g0) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            raw[i].get(x[i]);
            if (is_v || g0 + i * RPP >= rows) continue;
            const int r = g0 + i * RPP + row;
            const long token = token0 + r;
            Turn turn;
            turn.load(rt.cos, rt.sin, r < rows ? rt.at(token, start + (token - lo)) : 0, rt.rot, rt.interleaved != 0, l, c, false);
            float xo[8];
            raw[i].of_lane(turn.other).get(xo);
            // y = r (x w cos + x' w' sin) in 64 bits (x w is exact in 32) and from there to odd, so that the code is the one rounding: a code
            // has a border every 16th of its value, and each 32-bit rounding on the way would put some of a million values on the wrong
            // side of theirs.
            double rn = 1.;
            if (w) {
                double ss = 0.;
                float f[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) ss += (double)(x[i][e] * x[i][e]);
#pragma unroll
                for (int o = LPR / 2; o > 0; o >>= 1) ss += __shfl_xor(ss, o, kWave);
                ss = r < rows ? ss * (1. / D) + eps : 1.;   // (no infinity of a row that is none, where eps is 0)
                rn = __builtin_amdgcn_rsqf((float)ss);   // 1 / sqrt to 2^-22, and a step of Newton's: to 2^-43
                rn = rn * (1.5 - 0.5 * ss * rn * rn);
                w_mine.get(f);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[i][e] *= f[e];
                if (i == 0) w_other.load(w + 8 * (turn.other % LPR));   // (the same chunk in every pass)
                w_other.get(f);
#pragma unroll
                for (int e = 0; e < 8; ++e) xo[e] *= f[e];
            }
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                y[e] = to_odd(rn * __builtin_fma((double)x[i][e], (double)turn.cos[e], (double)(turn.interleaved ? x[i][e ^ 1] : xo[e]) * (double)turn.sin[e]));
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] = y[e];
        }
    };
    // Rows that the registers hold.  Of more of them (launch_cache_append: only with NP = 1) the values are formed twice.
    constexpr int GROUP = NP * RPP;
    const bool held = NP > 1 || rows <= GROUP;
    load(head0, 0);
    if (s0 > 0) old = scales[head0];
    for (int head = head0; head < heads; head += STEP) {
        uint8_t *const codes = (is_v ? cache.v : cache.k) + (((long)id * cache.Hk + head) << cache.page_shift) * D + 8 * c;
        auto store = [&](int g0, float inv) {
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int r = g0 + i * RPP + row;
                // (written once, to be read by another call: they leave the caches first; 16 x 512 tokens of 8 heads, d = 128, 19.7 us, so 18.9)
                if (r < rows) __builtin_nontemporal_store(encode(x[i], inv), reinterpret_cast<u32x2 *>(codes + (long)(s0 + r) * D));
            }
        };
        float amax = 0.f;
        const float before = old;
        for (int g0 = 0; g0 < (held ? 1 : rows); g0 += GROUP) {
            if (g0 > 0) load(head, g0);
            values(g0);
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) amax = fmaxf(amax, __builtin_fabsf(x[i][e]));
        }
        if (held && head + STEP < heads) {   // the next head's are on their way
            load(head + STEP, 0);
            if (s0 > 0) old = scales[head + STEP];
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor(amax, o, kWave));
        if constexpr (WU == 4) {
            __syncthreads();   // (the last head's have been read)
            if (l == 0) amax4[wave] = amax;
            __syncthreads();   // (also: everybody has read the old scale)
            amax = fmaxf(fmaxf(amax4[0], amax4[1]), fmaxf(amax4[2], amax4[3]));
        }
        float now = exp2_int(scale_exponent(amax));
        if (before >= now) {
            now = before;
        } else if (s0 > 0) {
            const float ratio = before / now;   // (both powers of two)
            for (int r = row; r < s0; r += RPP) {
                u32x2 *const at = reinterpret_cast<u32x2 *>(codes + (long)r * D);
                float v[8];
                decode(*at, v);
                *at = encode(v, ratio);
            }
        }
        if ((WU == 1 ? l : (int)threadIdx.x) == 0) scales[head] = now;
        const float inv = 1.f / now;
        if (held) {
            store(0, inv);
            continue;
        }
        for (int g0 = 0; g0 < rows; g0 += GROUP) {
            load(head, g0);
            values(g0);
            store(g0, inv);
        }
        if (head + STEP < heads) {
            load(head + STEP, 0);
            if (s0 > 0) old = scales[head + STEP];
        }
    }
}

// Waves that fill the chip, at 2 to 4 for each SIMD unit.  The case above has 24k units of a wave: four heads in turn 26.3 us, two 31.1,
// one 36.2 (22.6 with four since the instances that never need a second pass have none and codes leave the caches first).
constexpr long kFullWaves = 4096;

}  // namespace

AppendPlan append_plan(int T, bool ragged, int B, int most, int page, int Hk, int d) {
    AppendPlan p;
    p.slots = ragged ? (unsigned)(T / page + 2 * B) : (unsigned)B * (unsigned)((most - 1) / page + 2);
    // Rows that a call adds to a page, at most -- or, where the calls are those of a step of generation (about a token for each
    // sequence), most likely.  As few registers as those rows need: of many short units waves wait for memory one after the other.
    const int added = ragged ? (T <= 2 * B ? 2 : T) : most, rows = page < added ? page : added;
    p.passes = (rows * (d / 8) + 63) / 64;
    p.wave = p.passes <= 4;
    // heads that a unit takes one after the other, its next rows on their way: as many as leave the chip full
    const long waves = (long)p.slots * 2 * Hk * (p.wave ? 1 : 4);
    p.each = waves >= 4 * kFullWaves ? 4 : waves >= 2 * kFullWaves ? 2 : 1;
    return p;
}

hipError_t launch_cache_append(const HeadRows &K, const HeadRows &V, int T, const int *cu, int B, int most, int max_len, int d,
                               const void *w, float eps, const RotaryTable &rt, const PagedCache &c, hipStream_t st) {
    const AppendPlan p = append_plan(T, cu != nullptr, B, most, 1 << c.page_shift, c.Hk, d);
    const int passes = p.passes, heads = p.each * (p.wave ? 4 : 1);
    const dim3 grid(p.slots, 2 * (unsigned)((c.Hk + heads - 1) / heads));
#define DFSS_LAUNCH(D, WU, NP)                                                                                          \
    hipLaunchKernelGGL((k_cache_append<D, WU, NP>), grid, dim3(256), 0, st, K, V, T, cu, B, most, max_len, (const __bf16 *)w, eps, rt, c, p.each)
    // 12k tokens x 1024 elements, us: one wave of eight passes 30.5 (d = 128, pages of 32) and 31.6 (64, 64), four of two 27.4 and
    // 27.5; four waves of eight 33.5 (128, 64), of four 28.8.
#define DFSS_PASSES(D)                                                                                                  \
    if (passes <= 1) DFSS_LAUNCH(D, 1, 1); else if (passes <= 2) DFSS_LAUNCH(D, 1, 2); else if (passes <= 4) DFSS_LAUNCH(D, 1, 4); \
    else if (passes <= 8) DFSS_LAUNCH(D, 4, 2); else DFSS_LAUNCH(D, 4, 4)
    if (d == 64) {
        DFSS_PASSES(64);   // (128 rows are 16 passes)
    } else if (passes <= 16) {
        DFSS_PASSES(128);
    } else {
        DFSS_LAUNCH(128, 4, 8);
    }
#undef DFSS_PASSES
#undef DFSS_LAUNCH
    return hipGetLastError();
}

}  // namespace dfss
