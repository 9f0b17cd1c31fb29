// Attention over the paged cache of 8 bits (cached_attention.hip) for many rows: a prompt's queries, or a part of them.
//
// Here the matrix unit, the exponentials and the selection bound it, and what a code costs on the way to an operand.  A
// workgroup takes 128 rows, 32 to a wave, and its waves share the keys as bfloat16 in LDS, so that a block is read and
// converted once for all of them (a wave of k_cached with 32 rows does both for itself: 4 x 512 queries x 4 heads to a key head, 4096
// keys, d = 128, 120 us; with 64 rows 130).  Two teams of four waves take every other block, each out of LDS of its own: two waves to a
// SIMD unit, without partial results in memory (two workgroups that share the keys: 111 us, and 12 for the merge).  The next
// block's codes are in registers while this one is worked on, those after it on their way; one barrier a block.
//
// Tiles and products are those of k_fused32 (fused_attention32.hip): 32 x 32.  Scores and selection are those of k_cached: whole 32-bit
// scores are compared, and the reference comes in behind that, so a query keeps the same keys whatever else is in the call (but for
// the order of a 32-bit sum).  (With scores relative to the reference from the accumulator on and the position in the two lowest bits, as
// k_fused32 has it, small scores are lost at the reference's magnitude, and it is no faster here: 4 x 512 queries of 16 heads on 4, up to 4096 keys, d = 128, 2:4 75.8 us, so
// 71.1; 1:2 74.5 and 68.3; full 78.0 and 71.7; d = 64 56.6 and 54.1, 55.3 and 47.1, 59.8 and 50.1; d = 128, 2:4, pages of 16 78.9 and
// 78.7.)
// What bounds it is the rate at which two waves of a SIMD unit issue: about 450 instructions a block and wave.  (Level: the tiles
// of the first product in turn, more operands ahead, the teams in step.)
#include <math.h>

#include "cached_rows.hpp"

namespace dfss {

using namespace cached;

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kTau = 8.0f * 1.4426950408889634f;   // how far (in exponents of two) scores may exceed the reference

// BIG: pages of 64 tokens or more, a block lies in one.
template <int D, int MODE, bool BIG>
__global__ __launch_bounds__(512, 2) void k_cached_wide(const __bf16 *__restrict__ Q, const int *__restrict__ cu, PagedCache cache,
                                                        const uint8_t *__restrict__ Kc, const uint8_t *__restrict__ Vc,
                                                        const float *__restrict__ Ks, const float *__restrict__ Vs,
                                                        const int *__restrict__ table, Sizes sz, uint16_t *__restrict__ O,
                                                        float *__restrict__ part) {
    constexpr int CPR = D / 8;          // 16-byte chunks of a row of K or V in LDS
    constexpr int TILE = KB * CPR;
    constexpr int STEPS = D / 16, DT = D / 32;
    constexpr int PIECES = D / 64;      // 16-byte pieces of K (and of V) that a thread fetches of a block, 64 / PIECES keys apart
    constexpr bool DENSE = MODE == MODE_DENSE;
    constexpr int NP = DENSE ? 8 : 4;   // packed weights of a lane and 32 keys
    constexpr int NF = 16 * (DT + 1) + 1;      // floats of a lane's result
    __shared__ u32x4 lds_all[2][2][2][TILE];   // [team][buffer][K, V]
    static_assert(4 * NF * 64 * 4 <= (int)sizeof(lds_all), "a team's results fit into LDS");

    const int w8 = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), team = w8 >> 2, w = w8 & 3, tid = threadIdx.x & 255;
    const int l = threadIdx.x & 63, lj = l & 31, h = l >> 5;
    // The tiles of a head read the same keys, so they go to one XCD (workgroups go to the 8 of them in turn), and the heads to the
    // XCDs in turn, since sequences differ in length and in rows.
    const unsigned pairs = gridDim.x / (unsigned)sz.tiles, whole = pairs / 8 * 8 * (unsigned)sz.tiles;
    const unsigned in8 = blockIdx.x / 8;
    const int x = scalar(blockIdx.x < whole ? in8 / (unsigned)sz.tiles * 8 + blockIdx.x % 8 : blockIdx.x / (unsigned)sz.tiles);
    const int tile = scalar(blockIdx.x < whole ? in8 % (unsigned)sz.tiles : blockIdx.x % (unsigned)sz.tiles);
    const int number = scalar((unsigned)x / (unsigned)cache.Hk), head = x - number * cache.Hk;
    const unsigned id = (unsigned)x * sz.tiles + tile;
    int seq = number, begin = 0, end, first = 0;
    Shares sh;
    if (sz.target) {
        sh.init(sz, cache, l);
        seq = sh.find(sz, cache, l, number, -1, &first);
        if (seq < 0) return;
    }
    Rows R;
    if (!R.init(sz, cu, cache, seq, head, tile, 16 * kWide)) return;
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
    u32x4(*const lds)[2][TILE] = lds_all[team];

    // this wave's rows; the keys that the first of them sees are seen by all, those that the last one does not by none
    const int wr0 = R.r0 + 32 * w, wr1 = wr0 + 31 < R.rows ? wr0 + 31 : R.rows - 1;
    const int seen_by_all = wr0 < R.rows ? scalar(R.limit(sz, wr0)) : 0, seen = wr0 < R.rows ? scalar(R.limit(sz, wr1)) : 0;
    const int my_row = wr0 + lj < R.rows ? wr0 + lj : R.rows - 1, limit = R.limit(sz, my_row);
    bf16x8 bq[STEPS];   // lane (column lj, half h) of step s holds Q[q][16 s + 8 h .. +7]
    {
        const int i = my_row / sz.G, g = my_row - i * sz.G;
        const __bf16 *const q = Q + (R.lo + i) * sz.q_token + (R.h * sz.G + g) * sz.q_head;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) bq[s] = *reinterpret_cast<const bf16x8 *>(q + 16 * s + 8 * h);
    }

    // Fetching: thread t of a team has the 16 codes from element 16 (t % (D / 16)) on of key t / (D / 16) (+ 64 / PIECES): a wave's
    // keys lie in one group of 16, and so in one page.
    constexpr int LPK = D / 16;         // threads of a key
    const int f_key = tid / LPK, f_el = 16 * (tid % LPK);
    constexpr int NG = BIG ? 1 : 4;     // groups of a block's keys that lie in one page each
    struct Pages {
        int id[NG];
        // groups of 16 keys without a page, a bit each
        __device__ __forceinline__ int bad(int n_pages) const {
            int b = 0;
#pragma unroll
            for (int g = 0; g < NG; ++g) b |= (unsigned)id[g] >= (unsigned)n_pages ? (BIG ? 15 : 1 << g) : 0;
            return b;
        }
    };
    auto pages = [&](int jb) {
        Pages p;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            const int entry = (jb * KB + 16 * g) >> cache.page_shift;
            p.id[g] = scalar_load(my_table, entry < last_entry ? entry : last_entry);
        }
        return p;
    };
    struct Fetched {
        u32x4 k[PIECES], v[PIECES];
        float ks[PIECES], vs[PIECES];
        int bad;             // of the block
    };
    const uint32_t f_lane = (uint32_t)((BIG ? f_key : f_key & 15) * D + f_el);   // within the block, or within the group
    auto fetch = [&](int jb, const Pages &p, Fetched &f) {
        f.bad = p.bad(cache.n_pages);
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int group = BIG ? 0 : (64 / LPK * w + 64 / PIECES * i) >> 4;   // of the wave's keys
            int id = p.id[0];
            if constexpr (!BIG) {   // (by value: of an array it would be a load)
                const int i1 = p.id[1], i2 = p.id[2], i3 = p.id[3], lo = group & 1 ? i1 : id, hi = group & 1 ? i3 : i2;
                id = group & 2 ? hi : lo;
            }
            id = (unsigned)id >= (unsigned)cache.n_pages ? 0 : id;
            const long at = (long)id * cache.Hk + R.h;
            if (!BIG || i == 0) f.ks[i] = scalar_load(Ks, at), f.vs[i] = scalar_load(Vs, at);
            else f.ks[i] = f.ks[0], f.vs[i] = f.vs[0];
            const long from = ((at << cache.page_shift) + ((jb * KB + 16 * group) & page_mask)) * D + (BIG ? 64 / PIECES * i * D : 0);
            f.k[i] = *reinterpret_cast<const u32x4 *>(Kc + from + f_lane);
            f.v[i] = *reinterpret_cast<const u32x4 *>(Vc + from + f_lane);
        }
    };
    // K: the key 32 t + 16 h' + 4 g + x at slot 32 t + 8 g + 4 h' + x (k_fused32), V: row by key; both as bfloat16
    auto put = [&](int jb, int buf, Fetched &f) {
        if (jb * KB + KB > R.keys || f.bad) {   // what lies behind the last key is no value at all (0 x NaN is not 0)
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const int key = (64 / PIECES) * i + f_key;
                if (jb * KB + key >= R.keys || (f.bad >> (key >> 4) & 1)) f.v[i] = u32x4{0u, 0u, 0u, 0u};
                // (nor is the scale of the page that was read in place of none; the group of the wave's keys, as in fetch)
                if (f.bad >> ((64 / LPK * w + 64 / PIECES * i) >> 4) & 1) f.vs[i] = 1.f;
            }
        }
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int key = (64 / PIECES) * i + f_key;
            const int slot = (key & 32) | ((key >> 2) & 3) << 3 | ((key >> 4) & 1) << 2 | (key & 3);
            const int chunk = f_el / 8;
            u32x4 *const kd = &lds[buf][0][slot * CPR], *const vd = &lds[buf][1][key * CPR];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                u32x4 a, b;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t k = f.k[i][2 * y + e], v = f.v[i][2 * y + e];
                    a[2 * e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(k, f.ks[i], false));
                    a[2 * e + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(k, f.ks[i], true));
                    b[2 * e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, f.vs[i], false));
                    b[2 * e + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, f.vs[i], true));
                }
                kd[(chunk + y) ^ operand_row_swizzle<CPR, 32>(slot)] = a;
                vd[(chunk + y) ^ tr32_swizzle<CPR>(key)] = b;
            }
        }
    };
    const float k2 = sz.c;                                   // weight = exp2((s - reference) k2)
    float m_ref = kNoReference;                              // reference of query lj (raw dot product)
    f32x16 acc_o[DT], acc_l;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        acc_l[r] = 0.f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) acc_o[dt][r] = 0.f;
    }
    const uint32_t one2 = 0x3F803F80u;  // two bfloat16 ones
    const bf16x8 ones8 = __builtin_bit_cast(bf16x8, u32x4{one2, one2, one2, one2});
    const int s16 = l & 15, tr_row = s16 >> 2, tr_sub = (s16 >> 1) & 1, tr_byte = 8 * (s16 & 1), tr_xor = tr32_swizzle<CPR>(tr_row);
    const int tr_colgrp = (l >> 4) & 1;   // which 16 of the 32 columns of a tile this lane group reads

    Fetched f;
    f.bad = 0;
    Pages ahead;                 // of the block that is fetched next (asked for a step ahead)
    int bad = 0;                 // groups without a page of this block
    const int mine = begin + team;
    if (mine < end) {
        fetch(mine, pages(mine), f);
        bad = f.bad;
        ahead = pages(mine + 2);
        put(mine, 0, f);
        if (mine + 2 < end) fetch(mine + 2, ahead, f);
        ahead = pages(mine + 4);
    }
#pragma unroll
    for (int s = 0; s < STEPS; ++s) arrived(bq[s]);
    // The next block goes where the last one was, and the one after it is asked for: by the second team before its work on this
    // block, by the first one after it, so that one of the two is at its products while the other is not.
    int buf = 0;
    for (int jb = mine; jb < end + team; jb += 2, buf ^= 1) {   // (as many steps in both teams)
        auto next = [&]() {
            if (jb + 2 >= end) return;
            put(jb + 2, buf ^ 1, f);
            if (jb + 4 < end) {
                fetch(jb + 4, ahead, f);
                ahead = pages(jb + 6);
            }
        };
        __syncthreads();   // this block is in LDS, and nobody reads the one before it any more
        const int bad_after = f.bad;   // (of the block jb + 2, which f still holds)
        if (team == 1) next();
        if (jb < end && jb * KB < seen) {   // (the same in every lane)
            const u32x4 *const kt = lds[buf][0];
            const char *const vt = reinterpret_cast<const char *>(lds[buf][1]);
            // acc[t][4 g + x] = q . k for query lj, key 64 jb + 32 t + 16 h + 4 g + x
            constexpr f32x16 zero = {};
            f32x16 acc[2];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int s = 0; s < STEPS; ++s) {
                    const int slot = 32 * t + lj;
                    const bf16x8 a = __builtin_bit_cast(bf16x8, kt[slot * CPR + ((2 * s + h) ^ operand_row_swizzle<CPR, 32>(slot))]);
                    acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, bq[s], s == 0 ? zero : acc[t], 0, 0, 0);
                }
            read_ahead<2 * STEPS, 1, 2, 1>();
            if (jb * KB + KB > seen_by_all || bad) {
                const int left = limit - (jb * KB + 16 * h);   // keys of the lane that the query sees
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const bool none = bad >> (2 * t + h) & 1;
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (32 * t + r >= left || none) acc[t][r] = -INFINITY;
                }
            }
            float kept[2][2 * NP], m_blk = -3.0e38f;
            uint32_t idx = 0;       // positions: tile 0 in the low half
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const float a0 = acc[t][4 * g], a1 = acc[t][4 * g + 1], a2 = acc[t][4 * g + 2], a3 = acc[t][4 * g + 3];
                    if constexpr (DENSE) {
                        kept[t][4 * g] = a0, kept[t][4 * g + 1] = a1, kept[t][4 * g + 2] = a2, kept[t][4 * g + 3] = a3;
                        m_blk = fmaxf(m_blk, fmaxf(fmaxf(a0, a1), fmaxf(a2, a3)));
                    } else {
                        float &lo = kept[t][2 * g], &hi = kept[t][2 * g + 1];
                        uint32_t code;
                        if constexpr (MODE == MODE_2TO4) select_2of4(a0, a1, a2, a3, 16 * t + 4 * g, lo, hi, code);
                        else select_1of2(a0, a1, a2, a3, 16 * t + 4 * g, lo, hi, code);
                        idx |= code;
                        m_blk = fmaxf(fmaxf(m_blk, lo), hi);
                    }
                }
            if constexpr (!DENSE) arrived(idx);   // (formed here: its lane masks are more than there are scalar registers for behind the branch)
            if (__any((m_blk - m_ref) * k2 > kTau)) {
                m_blk = fmaxf(m_blk, __shfl_xor(m_blk, 32, 64));   // lanes lj and lj + 32 hold different keys of the same query
                const float m_new = (m_blk - m_ref) * k2 > kTau ? m_blk : m_ref;
                const float alpha = __builtin_amdgcn_exp2f((m_ref - m_new) * k2);
                m_ref = m_new;
                // accumulator rows are queries 8 (r/4) + 4 h + r%4: their factors from those columns' lanes
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float a_r = __shfl(alpha, 8 * (r >> 2) + 4 * h + (r & 3), 64);
                    acc_l[r] *= a_r;
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) acc_o[dt][r] *= a_r;
                }
            }
            const float mb = fmaxf(m_ref * k2, -1.0e37f);   // (no infinity while there is no reference: -inf + inf is no weight)
            uint32_t pk[2][NP];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < NP; ++e)
                    pk[t][e] = pack_bf16x2(__builtin_amdgcn_exp2f(__builtin_fmaf(kept[t][2 * e], k2, -mb)),
                                           __builtin_amdgcn_exp2f(__builtin_fmaf(kept[t][2 * e + 1], k2, -mb)));
            auto tr = [&](int key0, int dt) {
                const int chunk = (4 * dt + 2 * tr_colgrp + tr_sub) ^ tr_xor;
                return lds_read_tr16(vt + ((key0 + tr_row) * CPR + chunk) * 16 + tr_byte);
            };
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                if constexpr (!DENSE) {
                    const bf16x8 a = __builtin_bit_cast(bf16x8, u32x4{pk[t][0], pk[t][1], pk[t][2], pk[t][3]});
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) {
                        const int k0 = 32 * t + 8 * h;
                        const s16x4 t0 = tr(k0, dt), t1 = tr(k0 + 4, dt), t2 = tr(k0 + 16, dt), t3 = tr(k0 + 20, dt);
                        const s16x8 lo = __builtin_shufflevector(t0, t1, 0, 1, 2, 3, 4, 5, 6, 7), hi = __builtin_shufflevector(t2, t3, 0, 1, 2, 3, 4, 5, 6, 7);
                        const bf16x16 b = __builtin_bit_cast(bf16x16, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 14, 15));
                        if (t == 0) acc_o[dt] = __builtin_amdgcn_smfmac_f32_32x32x32_bf16(a, b, acc_o[dt], (int)idx, 0, 0);
                        else acc_o[dt] = __builtin_amdgcn_smfmac_f32_32x32x32_bf16(a, b, acc_o[dt], (int)idx, 0, 1);
                    }
                    acc_l = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, ones8, acc_l, 0, 0, 0);   // (against ones the positions do not matter)
                } else {
                    // m (0, 1): the lanes' keys 16 h + 8 m .. +7
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
                        const bf16x8 a = __builtin_bit_cast(bf16x8, u32x4{pk[t][4 * m], pk[t][4 * m + 1], pk[t][4 * m + 2], pk[t][4 * m + 3]});
#pragma unroll
                        for (int dt = 0; dt < DT; ++dt) {
                            const int k0 = 32 * t + 16 * h + 8 * m;
                            const s16x4 t0 = tr(k0, dt), t1 = tr(k0 + 4, dt);
                            const bf16x8 b = __builtin_bit_cast(bf16x8, __builtin_shufflevector(t0, t1, 0, 1, 2, 3, 4, 5, 6, 7));
                            acc_o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, acc_o[dt], 0, 0, 0);
                        }
                        acc_l = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, ones8, acc_l, 0, 0, 0);
                    }
                }
            }
            if constexpr (DENSE) read_ahead<4 * DT, 2, 2, 2, 4>();
            else read_ahead<2 * DT, 4, 2, 2, 2>();
        }
        if (team == 0) next();
        bad = bad_after;
    }

    // The second team's results join the first one's: value f of lane l of wave w at float w NF 64 + f 64 + l.
    __syncthreads();
    float *const slot = reinterpret_cast<float *>(lds_all) + w * (NF * 64) + l;
    if (team == 1) {
        slot[0] = m_ref;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            slot[(1 + r) * 64] = acc_l[r];
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) slot[(17 + 16 * dt + r) * 64] = acc_o[dt][r];
        }
    }
    __syncthreads();
    if (team == 1) return;
    {
        const float other = slot[0], m = fmaxf(m_ref, other);
        const float fa = __builtin_amdgcn_exp2f((m_ref - m) * k2), fb = __builtin_amdgcn_exp2f((other - m) * k2);
        m_ref = m;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int from = 8 * (r >> 2) + 4 * h + (r & 3);
            const float a_r = __shfl(fa, from, 64), b_r = __shfl(fb, from, 64);
            acc_l[r] = a_r * acc_l[r] + b_r * slot[(1 + r) * 64];
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) acc_o[dt][r] = a_r * acc_o[dt][r] + b_r * slot[(17 + 16 * dt + r) * 64];
        }
    }

    // O: rows 8 (r / 4) + 4 h + r % 4 of the wave's 32, columns 32 dt + lj
    float *const P = part + ((long)id * kWide + 2 * w) * partial_floats<D>();   // two 16-row tiles, one behind the other
    if (!alone && h == 0 && wr0 + lj < R.rows) P[(lj >> 4) * partial_floats<D>() + (lj & 15)] = m_ref;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int row = 8 * (r >> 2) + 4 * h + (r & 3), at = wr0 + row;
        if (at >= R.rows) continue;
        if (!alone) {
            float *const p = P + (row >> 4) * partial_floats<D>();
            if (lj == 0) p[16 + (row & 15)] = acc_l[r];
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) p[32 + (row & 15) * D + 32 * dt + lj] = acc_o[dt][r];
            continue;
        }
        const float inv = acc_l[r] > 0.f ? 1.f / acc_l[r] : 0.f;   // (a row that sees no key: 0)
        const int i = at / sz.G, g = at - i * sz.G;
        uint16_t *const out = O + ((long)(R.lo + i) * sz.Hq + R.h * sz.G + g) * D + lj;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) out[32 * dt] = (uint16_t)(pack_bf16x2(acc_o[dt][r] * inv, 0.f) & 0xFFFFu);
    }
}

}  // namespace

namespace cached {

hipError_t launch_wide(const __bf16 *Q, const int *cu, const PagedCache &c, int d, int mode, const Sizes &sz, unsigned workgroups,
                       uint16_t *O, float *part, hipStream_t st) {
#define DFSS_PAGES(D, MODE, BIG)                                                                                        \
    hipLaunchKernelGGL((k_cached_wide<D, MODE, BIG>), dim3(workgroups), dim3(512), 0, st, Q, cu, c, c.k, c.v, c.k_scale, c.v_scale,  \
                       c.table, sz, O, part)
#define DFSS_LAUNCH(D, MODE)                                                                                            \
    if (c.page_shift >= 6) DFSS_PAGES(D, MODE, true); else DFSS_PAGES(D, MODE, false)
    if (d == 64) {
        if (mode == MODE_2TO4) { DFSS_LAUNCH(64, MODE_2TO4); } else if (mode == MODE_1TO2) { DFSS_LAUNCH(64, MODE_1TO2); } else { DFSS_LAUNCH(64, MODE_DENSE); }
    } else {
        if (mode == MODE_2TO4) { DFSS_LAUNCH(128, MODE_2TO4); } else if (mode == MODE_1TO2) { DFSS_LAUNCH(128, MODE_1TO2); } else { DFSS_LAUNCH(128, MODE_DENSE); }
    }
#undef DFSS_PAGES
#undef DFSS_LAUNCH
    return hipGetLastError();
}

}  // namespace cached

}  // namespace dfss
