// Attention over a paged cache of 8 bits (cache_append.hip), N:M pruned or full, for one query a sequence or many.
//
// The queries of a sequence that share a key head -- its G = Hq / Hk heads times its query tokens -- are rows of one
// product, 16 to a tile of the matrix instruction.  With codes k, v and the page's scales (powers of two):
//     s_j = q . (k_j ks),   kept = the N largest of each aligned run of M (hidden keys: -inf),   O = sum p_j (v_j vs) / sum p_j
// where p = exp(scale (s - reference)) over the kept ones, with a running reference as in k_few.
//
// One token a sequence reads every code once for a handful of operations each, so memory bounds it, and the kernel is
// made of bytes in flight: a wave takes 64-key blocks of its own, K and V straight into registers one block ahead, no
// LDS and no barrier before the merge.
//   K   a lane holds 16 bytes of a key, which serve two steps of 32 elements (Q is read in the same order of elements)
//   V   a lane holds the same d / 16 columns of eight consecutive keys per step; bytes of two keys are put side by side
//       (v_perm_b32), which makes the operand's pairs of keys, and column d / 16 li + t goes to tile t
// v_cvt_scalef32_pk_bf16_fp8 turns a pair of codes into bfloat16 times the scale, exactly: a code has 4 significant bits
// and the scale is a power of two.  The weights are rounded to bfloat16 for the second product, and summed as rounded.
//
// K and V of one block only: with registers for two, half as many waves fit, and 64 sequences of up to 4096 keys took 127 us, so 83.
//
// The keys of a row tile go to the NW waves of a workgroup, and to several workgroups where the tiles are few or the
// sequences long; partial results (reference, sum, unnormalised O, fp32) are merged in a fixed order.
//
// Measured, one query a sequence (bytes of the codes that the lengths reach; a copy of 1 GiB, half of it writes, runs at 5.1 TB/s):
//   64 sequences of up to 4096 keys, 32 heads on 8, d = 128, pages of 16, 2:4      404 MB   74 us   5.5 TB/s
//   128 of up to 2048, 16 heads on 16, d = 64, pages of 32, full                   404 MB   71 us   5.7 TB/s
//   4 of up to 32768, 32 heads on 8, d = 128, pages of 128, full                   201 MB   40 + 5 (merge) us   5.0 TB/s
//   24 of up to 2500, four queries, 12 heads on 4, d = 64, pages of 32, 1:2         23 MB   12.4 us: five blocks a wave, one after the other
//   1 of 4096, 12 heads on 12, d = 64, pages of 64, 2:4                              6 MB   13.2 us: the same, four blocks a wave
#include <math.h>

#include <type_traits>

#include "cached_rows.hpp"

namespace dfss {

using namespace cached;

namespace {

template <bool ONCE, typename T>
__device__ __forceinline__ T load(const T *p) {
    if constexpr (ONCE) return __builtin_nontemporal_load(p);
    else return *p;
}

constexpr float kTau = 8.0f * 1.4426950408889634f;   // how far (in exponents of two) scores may exceed the reference
// From a block's scores of 16 queries (query l % 16, the lane's 16 keys) to the kept ones' weights as operand of the second
// product: selection, the reference raised where the block outgrew it (accumulators with it: rows 4 (l / 16) + r), exponentials, row
// sums of the weights as rounded.
template <int MODE, int DT>
__device__ __forceinline__ void weigh(const f32x4 (&s)[4], float c, int kb, bf16x8 ones8, float &m_ref, f32x4 (&acc_o)[DT], f32x4 &acc_l,
                                      bf16x8 (&p)[MODE == MODE_DENSE ? 2 : 1], uint32_t &idx) {
    constexpr int NP = MODE == MODE_DENSE ? 16 : 8;   // weights of the lane
    float x[NP], m_blk = -3.0e38f;
    idx = 0;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        if constexpr (MODE == MODE_DENSE) {
#pragma unroll
            for (int r = 0; r < 4; ++r) x[4 * t + r] = s[t][r], m_blk = fmaxf(m_blk, s[t][r]);
        } else {
            uint32_t code;
            if constexpr (MODE == MODE_2TO4) select_2of4(s[t][0], s[t][1], s[t][2], s[t][3], 4 * t, x[2 * t], x[2 * t + 1], code);
            else select_1of2(s[t][0], s[t][1], s[t][2], s[t][3], 4 * t, x[2 * t], x[2 * t + 1], code);
            idx |= code;
            m_blk = fmaxf(fmaxf(m_blk, x[2 * t]), x[2 * t + 1]);
        }
    }
    if (__any((m_blk - m_ref) * c > kTau)) {
        m_blk = fmaxf(m_blk, __shfl_xor(m_blk, 16, 64));
        m_blk = fmaxf(m_blk, __shfl_xor(m_blk, 32, 64));
        const float m_new = (m_blk - m_ref) * c > kTau ? m_blk : m_ref;
        const float alpha = __builtin_amdgcn_exp2f((m_ref - m_new) * c);
        m_ref = m_new;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float a_r = __shfl(alpha, 4 * kb + r, 64);
            acc_l[r] *= a_r;
#pragma unroll
            for (int t = 0; t < DT; ++t) acc_o[t][r] *= a_r;
        }
    }
    const float mb = fmaxf(m_ref * c, -1.0e37f);   // (no infinity while there is no reference: -inf + inf is no weight)
#pragma unroll
    for (int y = 0; y < NP / 8; ++y) {
        u32x4 pk;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            pk[e] = pack_bf16x2(__builtin_amdgcn_exp2f(__builtin_fmaf(x[8 * y + 2 * e], c, -mb)),
                                __builtin_amdgcn_exp2f(__builtin_fmaf(x[8 * y + 2 * e + 1], c, -mb)));
        p[y] = __builtin_bit_cast(bf16x8, pk);
        acc_l = mfma16(p[y], ones8, acc_l);
    }
}

// Codes that are read once (ONCE) leave the caches first: V at d = 128, K at d = 64, whose loads take whole rows (the others take half of
// one each, and the second half is then no longer there: 64 sequences of up to 4096 keys, 8 key heads, d = 128, 85 us, V 74, K 81 to 86,
// both 83; 128 of 2048, 16 heads, d = 64, full, 81, V 79, K 74, both 75).
// BIG: pages of 64 tokens or more, a block lies in one.
template <int D, int MODE, int NW, int RT, bool BIG, bool ONCE>
__global__ __launch_bounds__(64 * NW, NW == 16 ? 4 : RT == 1 && D == 64 ? 3 : RT <= 2 ? 2 : 1) void k_cached(const __bf16 *__restrict__ Q, const int *__restrict__ cu, PagedCache cache,
                                                    const uint8_t *__restrict__ Kc, const uint8_t *__restrict__ Vc,
                                                    const float *__restrict__ Ks, const float *__restrict__ Vs,
                                                    const int *__restrict__ table, Sizes sz, uint16_t *__restrict__ O,
                                                    float *__restrict__ part) {
    constexpr int SS = D / 64;          // 16-byte pieces of a key's row that a lane holds
    constexpr int STEPS = D / 32;       // MFMA k-steps of Q K^T
    constexpr int DT = D / 16;          // 16-column tiles of O
    constexpr int VW = D / 64;          // dwords of V that a lane holds of a key
    constexpr int NF = 4 * DT + 5;      // floats per lane of a partial result
    constexpr bool DENSE = MODE == MODE_DENSE;
    __shared__ float slots[NW * NF * 64];

    const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l = threadIdx.x & 63, li = l & 15, kb = l >> 4;
    // workgroups: [sequence][head][tile], or [share][head][tile] where keys are shared
    const unsigned id = xcd_contiguous(blockIdx.x, gridDim.x);
    const int x = scalar(id / (unsigned)sz.tiles), tile = id - x * sz.tiles, number = scalar(x / (unsigned)cache.Hk), head = x - number * cache.Hk;
    int seq = number, begin = 0, end, first = 0;
    Shares sh;
    if (sz.target) {
        sh.init(sz, cache, l);
        seq = sh.find(sz, cache, l, number, -1, &first);
        if (seq < 0) return;
    }
    Rows R;
    if (!R.init(sz, cu, cache, seq, head, tile, 16 * RT)) return;
    const int nblocks = R.blocks();
    end = nblocks;
    if (sz.target) {
        begin = (number - first) * sh.per;
        if (begin >= nblocks) return;
        end = begin + sh.per < nblocks ? begin + sh.per : nblocks;
    }
    const bool alone = begin == 0 && end == nblocks;   // nobody else has keys of these rows: no second kernel
    const int page_mask = (1 << cache.page_shift) - 1, last_entry = (R.keys > 0 ? R.keys - 1 : 0) >> cache.page_shift;
    const int *const my_table = table + (long)R.b * cache.width;
    const int seen_by_all = scalar(R.limit(sz, R.r0));

    // Q operand of step s: lane (column li, chunk kb) holds the elements 64 (s / 2) + 16 kb + 8 (s % 2) .. +7
    bf16x8 bq[RT][STEPS];
    int limit[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        int r = R.r0 + 16 * rt + li;
        r = r < R.rows ? r : R.rows - 1;
        limit[rt] = R.limit(sz, r);
        const int i = r / sz.G, g = r - i * sz.G;
        const __bf16 *const q = Q + (R.lo + i) * sz.q_token + (R.h * sz.G + g) * sz.q_head;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) bq[rt][s] = *reinterpret_cast<const bf16x8 *>(q + 64 * (s >> 1) + 16 * kb + 8 * (s & 1));
    }

    // Key of MFMA row i of tile t, so that a lane (query li, kb) ends up with whole runs and, for the second product,
    //   pruned  keys 16 kb .. +15                 row i: key 16 (i / 4) + 4 t + i % 4
    //   full    keys 8 kb .. +7 and 32 + the same  row i: key 32 (t / 2) + 8 (i / 4) + 4 (t % 2) + i % 4
    // A block is NG groups of keys, each in one page (16 keys, or all 64).  Pages and scales are the same for the whole wave
    // (scalar loads): the pages two blocks ahead, the scales one.
    constexpr int NG = BIG ? 1 : 4;
    struct Pages {
        long at[NG];          // page of each group (0 where there is none) * Hk + head
        int bad;              // a bit for each 16 keys without one
    };
    struct Scales {
        float k[NG], v[NG];
    };
    auto pages = [&](int jb) {
        Pages p;
        p.bad = 0;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            const int entry = (jb * KB + 16 * g) >> cache.page_shift;
            const int id = scalar_load(my_table, entry < last_entry ? entry : last_entry);
            const bool none = (unsigned)id >= (unsigned)cache.n_pages;
            p.at[g] = (long)(none ? 0 : id) * cache.Hk + R.h;
            p.bad |= none ? (BIG ? 15 : 1 << g) : 0;
        }
        return p;
    };
    auto scales = [&](const Pages &p) {
        Scales s;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            s.k[g] = scalar_load(Ks, p.at[g]);
            s.v[g] = scalar_load(Vs, p.at[g]);
        }
        return s;
    };
    const int place_shift = cache.page_shift + (D == 64 ? 6 : 7);
    auto place = [&](const Pages &p, int jb, int g) {   // bytes before a group's first key
        return (p.at[g] << place_shift) + ((jb * KB + 16 * g) & page_mask) * D;
    };
    auto pick = [](bool second, auto x, auto y) { return second ? y : x; };   // (by value: of an array it would be a load)
    constexpr int G1 = BIG ? 0 : 1, G2 = BIG ? 0 : 2, G3 = BIG ? 0 : 3;
    // first key that the lane loads, within its group: of K, and of V
    const int k_group = DENSE ? li >> 3 : li >> 2, v_group = kb >> 1;
    const uint32_t k_lane = (uint32_t)(((BIG ? 16 * k_group : 0) + (DENSE ? 8 * ((li >> 2) & 1) + (li & 3) : li & 3)) * D + 16 * kb);
    const uint32_t v_lane = (uint32_t)(((BIG ? 16 * v_group : 0) + 8 * (kb & 1)) * D + li * (4 * VW));

    u32x4 kr[4][SS];             // the block's K and V, as they lie in memory
    uint32_t vr[2][8][VW];
    auto load_k = [&](const Pages &p, int jb) {
        long at[NG], half[2];
#pragma unroll
        for (int g = 0; g < NG; ++g) at[g] = place(p, jb, g);
        half[0] = half[1] = at[0];
        if constexpr (!BIG) {
            half[0] = pick(k_group & 1, at[0], at[G1]), half[1] = pick(k_group & 1, at[G2], at[G3]);
            if constexpr (!DENSE) half[0] = half[1] = pick(k_group & 2, half[0], half[1]);
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            // (DENSE: the last two tiles are those of keys 32 .. 63)
            const uint8_t *const q = Kc + half[t >> 1] + (k_lane + (DENSE ? 4 * (t & 1) + (BIG ? 32 * (t >> 1) : 0) : 4 * t) * D);
#pragma unroll
            for (int x = 0; x < SS; ++x) kr[t][x] = load<ONCE && D == 64>(reinterpret_cast<const u32x4 *>(q + 64 * x));
        }
    };
    auto load_v = [&](const Pages &p, int jb) {
        long at[NG];
#pragma unroll
        for (int g = 0; g < NG; ++g) at[g] = place(p, jb, g);
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            const long from = BIG ? at[0] : st ? pick(v_group, at[G2], at[G3]) : pick(v_group, at[0], at[G1]);
            const uint8_t *const q = Vc + from + (v_lane + (BIG ? 32 * st * D : 0));
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if constexpr (VW == 2) {
                    const u32x2 x = load<ONCE>(reinterpret_cast<const u32x2 *>(q + e * D));
                    vr[st][e][0] = x[0], vr[st][e][VW - 1] = x[1];
                } else {
                    vr[st][e][0] = *reinterpret_cast<const uint32_t *>(q + e * D);
                }
            }
        }
    };

    float m_ref[RT];
    f32x4 acc_o[RT][DT], acc_l[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m_ref[rt] = kNoReference;
        acc_l[rt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t = 0; t < DT; ++t) acc_o[rt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const uint32_t one2 = 0x3F803F80u;  // two bfloat16 ones
    const bf16x8 ones8 = __builtin_bit_cast(bf16x8, u32x4{one2, one2, one2, one2});
    auto pair = [](uint32_t codes, float scale, auto high) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, decltype(high)::value));
    };
    constexpr std::false_type lo16{};
    constexpr std::true_type hi16{};

    // A block: the scores take K out of its registers, which the next block's K then goes into; the second product takes V.
    // So one or the other is on its way all the time, with registers for one block.
    Pages p_now, p_next;
    Scales sc;
    int jb = begin + w;
    if (jb < end) {
        p_now = pages(jb);
        sc = scales(p_now);
        load_k(p_now, jb);
        load_v(p_now, jb);
        p_next = pages(jb + NW);
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int s = 0; s < STEPS; ++s) arrived(bq[rt][s]);
    for (; jb < end; jb += NW) {
        const bool more = jb + NW < end;
        const bool masked = jb * KB + KB > seen_by_all || p_now.bad;   // (the same in every lane)
        float k_s[2] = {sc.k[0], sc.k[0]}, v_s[2] = {sc.v[0], sc.v[0]};
        if constexpr (!BIG) {
            k_s[0] = pick(k_group & 1, sc.k[0], sc.k[G1]), k_s[1] = pick(k_group & 1, sc.k[G2], sc.k[G3]);
            if constexpr (!DENSE) k_s[0] = k_s[1] = pick(k_group & 2, k_s[0], k_s[1]);
            v_s[0] = pick(v_group, sc.v[0], sc.v[G1]), v_s[1] = pick(v_group, sc.v[G2], sc.v[G3]);
        }
        const int bad = p_now.bad;
        if (more) sc = scales(p_next);
        // s[rt][t][r] = q . k of query li of tile rt and the lane's key r of tile t
        f32x4 s[RT][4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            bf16x8 a[STEPS];
            const float ks = k_s[t >> 1];
#pragma unroll
            for (int x = 0; x < SS; ++x)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const uint32_t c0 = kr[t][x][2 * y], c1 = kr[t][x][2 * y + 1];
                    a[2 * x + y] = __builtin_bit_cast(bf16x8, u32x4{pair(c0, ks, lo16), pair(c0, ks, hi16), pair(c1, ks, lo16), pair(c1, ks, hi16)});
                }
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                s[rt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int x = 0; x < STEPS; ++x) s[rt][t] = mfma16(a[x], bq[rt][x], s[rt][t]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (more) load_k(p_next, jb + NW);
        __builtin_amdgcn_sched_barrier(0);
        if (masked) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const int left = limit[rt] - jb * KB;
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int key = DENSE ? 32 * (t >> 1) + 8 * kb + 4 * (t & 1) + r : 16 * kb + 4 * t + r;
                        if (key >= left || (bad >> (key >> 4) & 1)) s[rt][t][r] = -INFINITY;
                    }
            }
            // what lies behind the last key is no value at all (0 x NaN is not 0)
#pragma unroll
            for (int st = 0; st < 2; ++st)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int key = 32 * st + 8 * kb + e;
                    if (jb * KB + key >= R.keys || (bad >> (key >> 4) & 1))
#pragma unroll
                        for (int x = 0; x < VW; ++x) vr[st][e][x] = 0u;
                }
            // (nor is the scale of the page that was read in place of none)
#pragma unroll
            for (int st = 0; st < 2; ++st)
                if (bad >> (2 * st + v_group) & 1) v_s[st] = 1.f;
        }
        bf16x8 p[RT][DENSE ? 2 : 1];
        uint32_t idx[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) weigh<MODE, DT>(s[rt], sz.c, kb, ones8, m_ref[rt], acc_o[rt], acc_l[rt], p[rt], idx[rt]);
        // O: four column tiles at a time, from one dword of each of the lane's 16 keys
#pragma unroll
        for (int x = 0; x < VW; ++x) {
            uint32_t two[2][4][2];   // bytes of keys (2y, 2y + 1): columns 0, 1 and columns 2, 3
#pragma unroll
            for (int st = 0; st < 2; ++st)
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const uint32_t e0 = vr[st][2 * y][x], e1 = vr[st][2 * y + 1][x];
                    two[st][y][0] = __builtin_amdgcn_perm(e1, e0, 0x05010400u);
                    two[st][y][1] = __builtin_amdgcn_perm(e1, e0, 0x07030602u);
                }
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                u32x4 bv[2];
#pragma unroll
                for (int st = 0; st < 2; ++st)
#pragma unroll
                    for (int y = 0; y < 4; ++y)
                        bv[st][y] = t & 1 ? pair(two[st][y][t >> 1], v_s[st], hi16) : pair(two[st][y][t >> 1], v_s[st], lo16);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    f32x4 &o = acc_o[rt][4 * x + t];
                    if constexpr (DENSE) {
                        o = mfma16(p[rt][0], __builtin_bit_cast(bf16x8, bv[0]), o);
                        o = mfma16(p[rt][1], __builtin_bit_cast(bf16x8, bv[1]), o);
                    } else {
                        typedef uint32_t u32x8 __attribute__((ext_vector_type(8)));
                        const u32x8 both = __builtin_shufflevector(bv[0], bv[1], 0, 1, 2, 3, 4, 5, 6, 7);
                        o = __builtin_amdgcn_smfmac_f32_16x16x64_bf16(p[rt][0], __builtin_bit_cast(bf16x16, both), o, (int)idx[rt], 0, 0);
                    }
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (more) {
            load_v(p_next, jb + NW);
            p_now = p_next;
            p_next = pages(jb + 2 * NW);
        }
        __builtin_amdgcn_sched_barrier(0);
    }

    // Merge: value f of lane l of wave g at float f * 64 + l of the wave's slot; a wave forms every NW-th of the four rows
    // that a lane holds, all D / 16 columns of it.
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        if (rt) __syncthreads();
        float *const mine = slots + w * (NF * 64) + l;
        mine[0] = m_ref[rt];
#pragma unroll
        for (int r = 0; r < 4; ++r) mine[(1 + r) * 64] = acc_l[rt][r];
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) mine[(5 + 4 * t + r) * 64] = acc_o[rt][t][r];
        __syncthreads();
        for (int r = w; r < 4; r += NW) {
            const int row = 4 * kb + r, at = R.r0 + 16 * rt + row;
            if (at >= R.rows) continue;
            float m = kNoReference;
#pragma unroll
            for (int g = 0; g < NW; ++g) m = fmaxf(m, slots[g * (NF * 64) + row]);
            float sum = 0.f, o[DT];
#pragma unroll
            for (int t = 0; t < DT; ++t) o[t] = 0.f;
#pragma unroll
            for (int g = 0; g < NW; ++g) {
                const float *const from = slots + g * (NF * 64);
                const float f = __builtin_amdgcn_exp2f((from[row] - m) * sz.c);
                sum += f * from[(1 + r) * 64 + l];
#pragma unroll
                for (int t = 0; t < DT; ++t) o[t] += f * from[(5 + 4 * t + r) * 64 + l];
            }
            if (!alone) {
                float *const P = part + ((long)id * RT + rt) * partial_floats<D>();
                if (li == 0) P[row] = m, P[16 + row] = sum;
#pragma unroll
                for (int t = 0; t < DT; t += 4) *reinterpret_cast<f32x4 *>(P + 32 + row * D + DT * li + t) = f32x4{o[t], o[t + 1], o[t + 2], o[t + 3]};
            } else {
                const float inv = sum > 0.f ? 1.f / sum : 0.f;   // (a row that sees no key: 0)
                const int i = at / sz.G, g = at - i * sz.G;
                uint32_t *const out = reinterpret_cast<uint32_t *>(O + ((long)(R.lo + i) * sz.Hq + R.h * sz.G + g) * D + DT * li);
                if constexpr (DT == 8)
                    *reinterpret_cast<u32x4 *>(out) = u32x4{pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv),
                                                           pack_bf16x2(o[4] * inv, o[5] * inv), pack_bf16x2(o[6] * inv, o[7] * inv)};
                else
                    *reinterpret_cast<u32x2 *>(out) = u32x2{pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv)};
            }
        }
    }
}

// O of the row tiles whose keys several workgroups shared (or nobody: 0), in a fixed order.  One workgroup per 16 rows; a
// thread forms 8 columns of a row.  RT as in the kernel before.  Eight partial results are on their way at a time.
template <int D>
__global__ __launch_bounds__(2 * D) void k_cached_merge(const float *__restrict__ part, const int *__restrict__ cu, PagedCache cache,
                                                        Sizes sz, int RT, uint16_t *__restrict__ O) {
    constexpr int AT_ONCE = 8;
    const int l = threadIdx.x & 63;
    const int x = scalar(blockIdx.x / (unsigned)RT), rt = blockIdx.x - x * RT, y = scalar(x / (unsigned)sz.tiles), tile = x - y * sz.tiles, seq = scalar(y / (unsigned)cache.Hk),
              head = y - seq * cache.Hk;
    Rows R;
    if (!R.init(sz, cu, cache, seq, head, tile, 16 * RT)) return;
    Shares sh;
    sh.init(sz, cache, l);
    const int nblocks = R.blocks(), shares = (nblocks + sh.per - 1) / sh.per;
    if (shares == 1) return;
    const int first = sh.find(sz, cache, l, 0, seq, nullptr);
    const int row = threadIdx.x / (D / 8), c = (threadIdx.x % (D / 8)) * 8, at = R.r0 + 16 * rt + row;
    if (at >= R.rows) return;
    const long step = (long)cache.Hk * sz.tiles * RT * partial_floats<D>();   // from a share to the next one
    const float *P = part + (((long)first * cache.Hk + head) * sz.tiles + tile) * RT * partial_floats<D>() + rt * partial_floats<D>();
    float m = kNoReference, sum = 0.f;
    f32x4 a0 = {0.f, 0.f, 0.f, 0.f}, a1 = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < shares; s0 += AT_ONCE, P += AT_ONCE * step) {
        float ms[AT_ONCE], ls[AT_ONCE], top = m;
        f32x4 o0[AT_ONCE], o1[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const float *const S = P + (s0 + i < shares ? i : 0) * step;
            const f32x4 *const src = reinterpret_cast<const f32x4 *>(S + 32 + row * D + c);
            ms[i] = S[row], ls[i] = S[16 + row], o0[i] = src[0], o1[i] = src[1];
        }
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) top = fmaxf(top, ms[i]);
        const float f = __builtin_amdgcn_exp2f((m - top) * sz.c);
        m = top;
        sum *= f, a0 *= f, a1 *= f;
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const float g = s0 + i < shares ? __builtin_amdgcn_exp2f((ms[i] - m) * sz.c) : 0.f;
            sum += g * ls[i];
            a0 += o0[i] * g;
            a1 += o1[i] * g;
        }
    }
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    a0 *= inv, a1 *= inv;
    const int i = at / sz.G, g = at - i * sz.G;
    *reinterpret_cast<u32x4 *>(O + ((long)(R.lo + i) * sz.Hq + R.h * sz.G + g) * D + c) = u32x4{
        pack_bf16x2(a0[0], a0[1]), pack_bf16x2(a0[2], a0[3]), pack_bf16x2(a1[0], a1[1]), pack_bf16x2(a1[2], a1[3])};
}

// 16-row tiles of a workgroup: 1, 2, or 8 (cached_wide.hip; for its 128 rows a block is converted once, whether they are there or not).
// Us in tiles of 32 rows and of 128:
//   d = 128: 64 rows.  32 sequences of up to 4096 keys, 8 key heads, pages of 64
//     2:4   48 rows 61 and 77, 64 rows 61 and 77, 96 rows 92 and 79, 128 rows 97 and 81
//     1:2   64 rows 61 and 68, 96 rows 88 and 71;   full  64 rows 59 and 73, 96 rows 84 and 77
//   d = 64: 192 rows with up to 4096 keys, 128 with more.  16 sequences of up to 4096 keys, 16 key heads, pages of 64, then of 32
//     2:4   160 rows 82 and 105, 192 rows 90 and 104, 256 rows 117 and 105;   97 and 110, 107 and 110, 140 and 111
//     1:2   160 rows 73 and 89, 192 rows 77 and 88, 256 rows 102 and 90;   78 and 97, 87 and 98, 114 and 100
//     full  160 rows 63 and 93, 192 rows 69 and 93, 256 rows 89 and 94;   81 and 97, 90 and 98, 119 and 100
//     one sequence of 1024, 8 key heads, 192 rows, 2:4: 9.9 and 19.5; in pages of 16 tiles of 32 lose at the end (8 sequences x 12 key heads,
//     160 rows, 2:4 78 and 64, full 58 and 58)
//     192 rows of 4 sequences of 6000 x 8 key heads, pages of 64: 2:4 56 and 32, full 49 and 30; of 16 of 8192, 137 and 112, 106 and 102
//     at 128 rows tiles of 128 win on a full chip (32 x 16 key heads, pages of 32, 2:4 145 and 117) and lose on one in part (one sequence, 9.8 and 19.5)
int row_tiles(long rows, int max_len, int d) {
    const long most = d == 128 ? 64 : max_len <= 4096 ? 192 : 128;
    return rows <= 16 ? 1 : rows <= most ? 2 : kWide;
}

struct Plan {
    int RT, NW, tiles, target, least, fill;   // fill: `per` is the least possible; NW: waves of a workgroup; target 0: nobody shares
};
Plan plan(int B, int Hk, int G, int most, int max_len, int d) {
    Plan p;
    const long rows = (long)most * G;
    p.RT = row_tiles(rows, max_len, d);
    p.tiles = (int)((rows + 16 * p.RT - 1) / (16 * p.RT));
    const long per_share = (long)Hk * p.tiles, items = B * per_share;   // workgroups of a share, and without shares
    const int blocks = (max_len + KB - 1) / KB;
    // Eight waves where that is still one workgroup for each compute unit at most: the wave's own chain of blocks sets the time there
    // (4 sequences of 32768 keys, 8 key heads, d = 128, shared: 42 + 5 us, with four waves 48 + 8).  Four where workgroups follow each
    // other, since a new one then starts sooner (128 sequences of 2048 keys, 16 heads, d = 64: 77, with eight 87, both with all codes through the caches).
    // (Also of shares of few blocks: eight waves and four, us, 1 sequence of 6000 keys, 8 key heads, d = 64 10.9 and 11.6, of 16384 15.6 and 18.9,
    // d = 128 13.7 and 13.6, 18.8 and 21.8; 4 of 8192 14.8 and 15.4, 19.4 and 19.9; 1 of 32768, 2 heads 18.1 and 26.4, 20.3 and 28.1.)
    p.NW = items <= 256 || p.RT == kWide ? 8 : 4;
    p.target = 0;
    p.least = p.NW;
    p.fill = 0;
    // d = 64: sixteen waves walk 80 blocks before a second kernel pays.  Us of sixteen waves and of eight that share, merge included, 2600 and
    // 4096 keys, in a graph: 12 workgroups 9.8 and 9.8, 12.5 and 9.9; 48 10.8 and 11.6, 13.9 and 13.2; 64 10.8 and 13.0, 13.6 and 14.6; 96 11.0 and
    // 14.9, 13.8 and 16.8; 240 (4096) 21.2 and 30.8.  Called one by one, two kernels and their workspace are 4 us more of the host's time
    // (12 workgroups, 4096 keys: 12.3 and 15.7 a call), which few workgroups would gain back in graphs alone.  Eight waves are enough up to 40
    // blocks (2000 keys, 12 workgroups 8.9 and 8.9, 96 10.1 and 10.3).  (At d = 128 they would have to spill 142 to 174 registers.)
    if (d == 64 && p.RT == 1 && items <= 256 && blocks > 40 && blocks <= 80) p.NW = 16;
    // Five blocks a wave cost less than a second kernel, 5 us, unless a block is long (d = 128, tiles of 128 rows) and so much of the chip
    // idle that sharing makes one of them of the five.  Us alone and shared, merge included, in a graph; shared calls one by one are 16 us
    // of the host's time, so that no border stands where alone is less:
    //   d = 64, one query                  2500 keys, 8 workgroups 10.1 and 10.3, 96 11.5 and 13.9, 128 11.9 and 15.5
    //   d = 128, one query                 2100 and 2500 keys, 8 workgroups 15.7 and 12.1, 18.4 and 12.3; 64 16.6 and 14.8, 19.1 and 15.9; 96 16.8
    //                                      and 17.3, 19.3 and 19.2; 128 17.0 and 19.3, 19.5 and 20.9
    //   d = 128, 8 queries x 4 heads       1600 and 2500 keys, 8 workgroups 17.3 and 16.2, 22.2 and 16.8; 64 18.1 and 18.5, 23.2 and 20.6
    //   tiles of 128 rows, d = 64, 128     1600 keys, 16 workgroups 25.9 and 17.5, 32.8 and 22.3; 64 25.9 and 21.4, 32.8 and 29.5; 128 26.0
    //                                      and 26.9, 34.1 and 36.7
    // (Behind 2^30 the sum of blocks that the shares are counted in would pass 32 bits.)
    const int walk = items > 64 ? 5 : p.RT == kWide ? 3 : d == 128 ? 4 : 5;
    if (blocks <= walk * p.NW || (long)B * blocks > 1 << 30) return p;
    // Workgroups that the chip holds at a time, by their registers and LDS.  Where the sequences alone are that many, sharing only
    // evens their lengths out, which is worth the merge for long ones alone (64 sequences of up to 4096 keys, 8 key heads, d = 128:
    // 81 us alone, 96 + 6 shared, likewise), and with four rounds of them lengths even out by themselves.
    const long slots = p.NW == 8 ? 256 : 512;
    if (items >= 4 * slots || (items >= slots && blocks < 128)) return p;
    p.least = p.NW;
    const long fit = slots / per_share - B;       // (the last share of a sequence is cut short)
    long t = fit > B / 2 ? fit : B / 2 > 0 ? B / 2 : 1;
    const long most_shares = (long)B * ((blocks + p.least - 1) / p.least);
    p.target = (int)(t < most_shares ? t : most_shares);
    // All shares have a place on the chip at once, and a sequence has four at most: 16 sequences of 6000 keys, 8 key heads, d = 128, 42.5 us
    // and 37.0 with the least `per`, 8 of 8192, 8 heads, 26.3 and 25.4, 2 of 8192 with 100 queries of 4 heads to a key head 57.9 and 52.2; with
    // more shares than that the search costs what it gains (7 of 10000, 4 heads, d = 64, 14.9 and 15.5, 4 of 32768 44.8 and 45.0).
    p.fill = p.target <= fit && B <= 64 && p.target + B <= 4L * B;
    return p;
}
// Shares of all sequences, at most (of a valid plan that shares)
long shares_of(const Plan &p, int B) { return (long)p.target + B; }

template <int D, int MODE>
hipError_t launch(const HeadRows &Q, int T, const int *cu, int B, int most, int max_len, float scale, bool causal,
                  const PagedCache &c, void *O, float *part, const Plan &p, hipStream_t st) {
    const Sizes sz = {T, B, Q.H, Q.H / c.Hk, most, max_len, p.tiles, p.target, p.least, Q.token, Q.head, p.target ? 1. / p.target : 0., p.fill ? 1. / (p.target + B) : 0.,
                      scale * 1.4426950408889634f, causal ? 1 : 0};
    const unsigned items = (unsigned)((long)B * c.Hk * p.tiles), shares = (unsigned)(shares_of(p, B) * c.Hk * p.tiles);
#define DFSS_LAUNCH(KERNEL)                                                                                             \
    hipLaunchKernelGGL((KERNEL), dim3(p.target ? shares : items), dim3(64 * p.NW), 0, st, (const __bf16 *)Q.data, cu, c, c.k, c.v,  \
                       c.k_scale, c.v_scale, c.table, sz, (uint16_t *)O, part)
#define DFSS_PAGES(NW, RT, ONCE)                                                                                        \
    if (c.page_shift >= 6) DFSS_LAUNCH(DFSS_K(NW, RT, true, ONCE)); else DFSS_LAUNCH(DFSS_K(NW, RT, false, ONCE))
#define DFSS_K(NW, RT, BIG, ONCE) k_cached<D, MODE, NW, RT, BIG, ONCE>
#define DFSS_ROWS(NW, RT)                                                                                               \
    if (once) { DFSS_PAGES(NW, RT, true); } else { DFSS_PAGES(NW, RT, false); }
    // Codes leave the caches first where nobody else of the call reads them and they are more than three quarters of the last-level
    // cache of 256 MB, so far as the host knows: 32 sequences of up to 4096 keys, 8 key heads, four queries, d = 128, 44.3 us and 38.8; 4 of
    // 32768 keys 48.6 and 45.1; in smaller calls the next one finds them there (16 of 4096 keys, one query, 30.7 and 31.9).
    const long tokens = (long)B * max_len, room = (long)c.n_pages << c.page_shift;
    const bool once = p.tiles == 1 && (tokens < room ? tokens : room) * c.Hk * (2 * D) >= 192L << 20;
    if (p.RT == kWide) {
        if (const hipError_t e = launch_wide((const __bf16 *)Q.data, cu, c, D, MODE, sz, p.target ? shares : items, (uint16_t *)O, part, st)) return e;
    } else if (p.RT == 1) {
        // (sixteen waves: 256 workgroups of 80 blocks, 168 MB, at most)
        if (p.NW == 16) { if constexpr (D == 64) { DFSS_PAGES(16, 1, false); } } else if (p.NW == 8) { DFSS_ROWS(8, 1); } else { DFSS_ROWS(4, 1); }
    } else {
        if (p.NW == 8) { DFSS_ROWS(8, 2); } else { DFSS_ROWS(4, 2); }
    }
#undef DFSS_ROWS
#undef DFSS_K
#undef DFSS_PAGES
#undef DFSS_LAUNCH
    if (p.target)
        hipLaunchKernelGGL(k_cached_merge<D>, dim3(items * p.RT), dim3(2 * D), 0, st, part, cu, c, sz, p.RT, (uint16_t *)O);
    return hipGetLastError();
}

}  // namespace

CachedPlan cached_plan(int B, int Hq, int Hk, int most, int max_len, int d) {
    const Plan p = plan(B, Hk, Hq / Hk, most, max_len, d);
    return CachedPlan{p.RT, p.NW, p.target, p.fill};
}

size_t cached_workspace_bytes(int B, int Hq, int Hk, int most, int max_len, int d) {
    const Plan p = plan(B, Hk, Hq / Hk, most, max_len, d);
    return p.target ? (size_t)shares_of(p, B) * Hk * p.tiles * p.RT * 16 * (d + 2) * sizeof(float) : 0;
}

hipError_t launch_attention_cached(const HeadRows &Q, int T, const int *cu, int B, int most, int max_len, int d, int mode,
                                   float scale, bool causal, const PagedCache &c, void *O, void *part, hipStream_t st) {
    const Plan p = plan(B, c.Hk, Q.H / c.Hk, most, max_len, d);
#define DFSS_CALL(D, M) launch<D, M>(Q, T, cu, B, most, max_len, scale, causal, c, O, (float *)part, p, st)
    if (d == 64) return mode == 0 ? DFSS_CALL(64, MODE_2TO4) : mode == 1 ? DFSS_CALL(64, MODE_1TO2) : DFSS_CALL(64, MODE_DENSE);
    return mode == 0 ? DFSS_CALL(128, MODE_2TO4) : mode == 1 ? DFSS_CALL(128, MODE_1TO2) : DFSS_CALL(128, MODE_DENSE);
#undef DFSS_CALL
}

}  // namespace dfss
