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
// The keys of a row tile go to the NW waves of a workgroup, and to several workgroups where the tiles are few or the
// sequences long; partial results (reference, sum, unnormalised O, fp32) are merged in a fixed order.
#include <math.h>

#include <type_traits>

#include "dfss_device.hpp"
#include "dfss_kernels.hpp"

namespace dfss {

namespace {

constexpr int KB = 64;    // keys per block
constexpr float kTau = 8.0f * 1.4426950408889634f;   // how far (in exponents of two) scores may exceed the reference
enum { MODE_2TO4 = 0, MODE_1TO2 = 1, MODE_DENSE = 2 };

struct Sizes {
    int T, B, Hq, G, most, max_len, tiles, splits, least;   // tiles: row tiles (of 16 RT rows) of a sequence and key head
    long q_token, q_head;
    float c;          // scale * log2(e)
    int causal;
};

// What a row tile needs to know of its sequence.
struct Rows {
    int b, h, lo, n, len, first;   // first: position of query 0
    int r0, rows;                  // first row of the tile, rows of the sequence
    int keys;                      // keys that any row of the tile sees
    __device__ __forceinline__ bool init(const Sizes &s, const int *cu, const PagedCache &c, int item, int tile_rows) {
        const int tile = item % s.tiles, bh = item / s.tiles;
        b = bh / c.Hk, h = bh - b * c.Hk;
        lo = b * s.most, n = s.most;
        if (cu) {
            lo = cu[b], n = cu[b + 1];
            lo = lo < 0 ? 0 : lo < s.T ? lo : s.T;
            n = n < lo ? 0 : (n < s.T ? n : s.T) - lo;
        }
        const int queries = n < s.most ? n : s.most;
        r0 = tile * tile_rows, rows = queries * s.G;
        if (r0 >= rows) return false;
        const long capacity = (long)c.width << c.page_shift;
        len = c.len[b] < 0 ? 0 : c.len[b];
        first = len - n;           // (by the length given: a longer one than the call allows is cut, positions stay)
        const int most_keys = s.max_len < capacity ? s.max_len : (int)capacity;
        len = len < most_keys ? len : most_keys;
        const int last = r0 + tile_rows < rows ? r0 + tile_rows - 1 : rows - 1;
        keys = limit(s, last);
        return true;
    }
    // keys that row r sees: those before it
    __device__ __forceinline__ int limit(const Sizes &s, int r) const {
        if (!s.causal) return len;
        const int x = first + r / s.G + 1;
        return x < 0 ? 0 : x < len ? x : len;
    }
    __device__ __forceinline__ int blocks() const { return (keys + KB - 1) / KB; }
    // blocks of one of the workgroups that share the keys: the more the fewer of them there are
    __device__ __forceinline__ int per_split(const Sizes &s) const {
        const int per = (blocks() + s.splits - 1) / s.splits;
        return per < s.least ? s.least : per;
    }
};

template <int D>
constexpr int partial_floats() { return 16 * (D + 2); }   // of a 16-row tile: references, sums, O

template <int D, int MODE, int NW, int RT, bool SPLIT>
__global__ __launch_bounds__(64 * NW) void k_cached(const __bf16 *__restrict__ Q, const int *__restrict__ cu, PagedCache cache,
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
    constexpr int KG = DENSE ? 2 : 1;   // 16-key groups that the lane's K rows lie in
    __shared__ float slots[NW * NF * 64];

    const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l = threadIdx.x & 63, li = l & 15, kb = l >> 4;
    const unsigned share = xcd_contiguous(blockIdx.x, gridDim.x);
    const unsigned item = SPLIT ? share / (unsigned)sz.splits : share;
    const int sp = SPLIT ? share % (unsigned)sz.splits : 0;
    Rows R;
    if (!R.init(sz, cu, cache, item, 16 * RT)) return;
    const int nblocks = R.blocks();
    const int per = SPLIT ? R.per_split(sz) : nblocks;
    const int begin = sp * per, end = begin + per < nblocks ? begin + per : nblocks;
    if (SPLIT && begin >= nblocks) return;
    const int page_mask = (1 << cache.page_shift) - 1, last_entry = (R.keys > 0 ? R.keys - 1 : 0) >> cache.page_shift;
    const int *const my_table = table + (long)R.b * cache.width;
    const int seen_by_all = R.limit(sz, R.r0);

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
    struct Block {
        u32x4 k[4][SS];
        uint32_t v[2][8][VW];
        float ks[KG], vs[2];
        int bad;          // groups of 16 keys whose page is none (a bit each)
    };
    const uint32_t k_lane = (uint32_t)((DENSE ? 8 * ((li >> 2) & 1) + (li & 3) : li & 3) * D + 16 * kb);
    const uint32_t v_lane = (uint32_t)(8 * (kb & 1) * D + li * (4 * VW));
    auto load_block = [&](int jb, Block &b) {
        long at[4];
        float ks[4], vs[4];
        b.bad = 0;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int key = jb * KB + 16 * g;
            int entry = key >> cache.page_shift;
            entry = __builtin_amdgcn_readfirstlane(entry < last_entry ? entry : last_entry);
            int id = my_table[entry];
            if ((unsigned)id >= (unsigned)cache.n_pages) id = 0, b.bad |= 1 << g;
            const long head = (long)id * cache.Hk + R.h;
            at[g] = ((head << cache.page_shift) + (key & page_mask)) * D;
            ks[g] = Ks[head];
            vs[g] = Vs[head];
        }
        const int kg = li >> 2, vg = kb >> 1;
        long ka[KG];
        if constexpr (DENSE) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                ka[x] = li & 8 ? at[2 * x + 1] : at[2 * x];
                b.ks[x] = li & 8 ? ks[2 * x + 1] : ks[2 * x];
            }
        } else {
            const long a0 = kg & 1 ? at[1] : at[0], a1 = kg & 1 ? at[3] : at[2];
            const float s0 = kg & 1 ? ks[1] : ks[0], s1 = kg & 1 ? ks[3] : ks[2];
            ka[0] = kg & 2 ? a1 : a0;
            b.ks[0] = kg & 2 ? s1 : s0;
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const uint8_t *const p = Kc + ka[DENSE ? t >> 1 : 0] + k_lane + (DENSE ? 4 * (t & 1) : 4 * t) * D;
#pragma unroll
            for (int x = 0; x < SS; ++x) b.k[t][x] = *reinterpret_cast<const u32x4 *>(p + 64 * x);
        }
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            const uint8_t *const p = Vc + (vg ? at[2 * st + 1] : at[2 * st]) + v_lane;
            b.vs[st] = vg ? vs[2 * st + 1] : vs[2 * st];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if constexpr (VW == 2) {
                    const u32x2 x = *reinterpret_cast<const u32x2 *>(p + e * D);
                    b.v[st][e][0] = x[0], b.v[st][e][VW - 1] = x[1];
                } else {
                    b.v[st][e][0] = *reinterpret_cast<const uint32_t *>(p + e * D);
                }
            }
        }
    };

    float m_ref[RT];
    f32x4 acc_o[RT][DT], acc_l[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m_ref[rt] = -1.0e30f;
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

    auto block = [&](int jb, Block &b) {
        const bool masked = jb * KB + KB > seen_by_all || b.bad;   // (the same in every lane)
        // s[rt][t][r] = q . k of query li of tile rt and the lane's key r of tile t
        f32x4 s[RT][4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            bf16x8 a[STEPS];
            const float ks = b.ks[DENSE ? t >> 1 : 0];
#pragma unroll
            for (int x = 0; x < SS; ++x)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const uint32_t c0 = b.k[t][x][2 * y], c1 = b.k[t][x][2 * y + 1];
                    a[2 * x + y] = __builtin_bit_cast(bf16x8, u32x4{pair(c0, ks, lo16), pair(c0, ks, hi16), pair(c1, ks, lo16), pair(c1, ks, hi16)});
                }
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                s[rt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int x = 0; x < STEPS; ++x) s[rt][t] = mfma16(a[x], bq[rt][x], s[rt][t]);
            }
        }
        if (masked) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const int left = limit[rt] - jb * KB;
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int key = DENSE ? 32 * (t >> 1) + 8 * kb + 4 * (t & 1) + r : 16 * kb + 4 * t + r;
                        if (key >= left || (b.bad >> (key >> 4) & 1)) s[rt][t][r] = -INFINITY;
                    }
            }
            // what lies behind the last key is no value at all (0 x NaN is not 0)
#pragma unroll
            for (int st = 0; st < 2; ++st)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int key = 32 * st + 8 * kb + e;
                    if (jb * KB + key >= R.keys || (b.bad >> (key >> 4) & 1))
#pragma unroll
                        for (int x = 0; x < VW; ++x) b.v[st][e][x] = 0u;
                }
        }
        bf16x8 p[RT][DENSE ? 2 : 1];
        uint32_t idx[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            constexpr int NP = DENSE ? 16 : 8;   // weights of the lane
            float x[NP], m_blk = -3.0e38f;
            idx[rt] = 0;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                if constexpr (DENSE) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[4 * t + r] = s[rt][t][r], m_blk = fmaxf(m_blk, s[rt][t][r]);
                } else {
                    uint32_t code;
                    if constexpr (MODE == MODE_2TO4) select_2of4(s[rt][t][0], s[rt][t][1], s[rt][t][2], s[rt][t][3], 4 * t, x[2 * t], x[2 * t + 1], code);
                    else select_1of2(s[rt][t][0], s[rt][t][1], s[rt][t][2], s[rt][t][3], 4 * t, x[2 * t], x[2 * t + 1], code);
                    idx[rt] |= code;
                    m_blk = fmaxf(fmaxf(m_blk, x[2 * t]), x[2 * t + 1]);
                }
            }
            if (__any((m_blk - m_ref[rt]) * sz.c > kTau)) {   // raise the reference where the block outgrew it
                m_blk = fmaxf(m_blk, __shfl_xor(m_blk, 16, 64));
                m_blk = fmaxf(m_blk, __shfl_xor(m_blk, 32, 64));
                const float m_new = (m_blk - m_ref[rt]) * sz.c > kTau ? m_blk : m_ref[rt];
                const float alpha = __builtin_amdgcn_exp2f((m_ref[rt] - m_new) * sz.c);
                m_ref[rt] = m_new;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float a_r = __shfl(alpha, 4 * kb + r, 64);
                    acc_l[rt][r] *= a_r;
#pragma unroll
                    for (int t = 0; t < DT; ++t) acc_o[rt][t][r] *= a_r;
                }
            }
            const float mb = m_ref[rt] * sz.c;
#pragma unroll
            for (int y = 0; y < NP / 8; ++y) {
                u32x4 pk;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    pk[e] = pack_bf16x2(__builtin_amdgcn_exp2f(__builtin_fmaf(x[8 * y + 2 * e], sz.c, -mb)),
                                        __builtin_amdgcn_exp2f(__builtin_fmaf(x[8 * y + 2 * e + 1], sz.c, -mb)));
                p[rt][y] = __builtin_bit_cast(bf16x8, pk);
                acc_l[rt] = mfma16(p[rt][y], ones8, acc_l[rt]);
            }
        }
        // O: four column tiles at a time, from one dword of each of the lane's 16 keys
#pragma unroll
        for (int x = 0; x < VW; ++x) {
            uint32_t two[2][4][2];   // bytes of keys (2y, 2y + 1): columns 0, 1 and columns 2, 3
#pragma unroll
            for (int st = 0; st < 2; ++st)
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const uint32_t e0 = b.v[st][2 * y][x], e1 = b.v[st][2 * y + 1][x];
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
                        bv[st][y] = t & 1 ? pair(two[st][y][t >> 1], b.vs[st], hi16) : pair(two[st][y][t >> 1], b.vs[st], lo16);
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
    };

    {
        Block b0, b1;
        int jb = begin + w;
        if (jb < end) load_block(jb, b0);
        while (jb < end) {
            int jn = jb + NW;
            if (jn < end) load_block(jn, b1);
            block(jb, b0);
            if (jn >= end) break;
            jb = jn + NW;
            if (jb < end) load_block(jb, b0);
            block(jn, b1);
        }
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
            float m = -1.0e30f;
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
            if constexpr (SPLIT) {
                float *const P = part + (((long)item * RT + rt) * sz.splits + sp) * partial_floats<D>();
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

// O of the row tiles whose keys several workgroups shared, in a fixed order.  One workgroup per 16 rows; a thread forms 8
// columns of a row.  RT as in the kernel before.
template <int D>
__global__ __launch_bounds__(2 * D) void k_cached_merge(const float *__restrict__ part, const int *__restrict__ cu, PagedCache cache,
                                                        Sizes sz, int RT, uint16_t *__restrict__ O) {
    Rows R;
    const int item = blockIdx.x / RT, rt = blockIdx.x - item * RT;
    if (!R.init(sz, cu, cache, item, 16 * RT)) return;
    const int row = threadIdx.x / (D / 8), c = (threadIdx.x % (D / 8)) * 8, at = R.r0 + 16 * rt + row;
    if (at >= R.rows) return;
    const int per = R.per_split(sz), shares = (R.blocks() + per - 1) / per;
    const float *const P = part + (long)blockIdx.x * sz.splits * partial_floats<D>();
    float m = -1.0e30f;
    for (int sp = 0; sp < shares; ++sp) m = fmaxf(m, P[sp * partial_floats<D>() + row]);
    float sum = 0.f;
    f32x4 a0 = {0.f, 0.f, 0.f, 0.f}, a1 = {0.f, 0.f, 0.f, 0.f};
    for (int sp = 0; sp < shares; ++sp) {
        const float *const S = P + sp * partial_floats<D>();
        const float f = __builtin_amdgcn_exp2f((S[row] - m) * sz.c);
        const f32x4 *const src = reinterpret_cast<const f32x4 *>(S + 32 + row * D + c);
        sum += f * S[16 + row];
        a0 += src[0] * f;
        a1 += src[1] * f;
    }
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    a0 *= inv, a1 *= inv;
    const int i = at / sz.G, g = at - i * sz.G;
    *reinterpret_cast<u32x4 *>(O + ((long)(R.lo + i) * sz.Hq + R.h * sz.G + g) * D + c) = u32x4{
        pack_bf16x2(a0[0], a0[1]), pack_bf16x2(a0[2], a0[3]), pack_bf16x2(a1[0], a1[1]), pack_bf16x2(a1[2], a1[3])};
}

constexpr int waves_of(int d) { return d == 64 ? 8 : 4; }
// 16-row tiles of a workgroup
int row_tiles(long rows) { return rows <= 16 ? 1 : 2; }

struct Plan {
    int RT, tiles, splits, least;
};
Plan plan(int B, int Hk, int G, int most, int max_len, int d) {
    Plan p;
    const long rows = (long)most * G;
    p.RT = row_tiles(rows);
    p.tiles = (int)((rows + 16 * p.RT - 1) / (16 * p.RT));
    const long items = (long)B * Hk * p.tiles;
    const int blocks = (max_len + KB - 1) / KB, nw = waves_of(d);
    p.least = nw;                                 // at least a block for each wave
    long n = 512 / items;                         // two workgroups to a compute unit
    const long by_length = blocks / 64;           // and none of more than 4096 keys: sequences differ in length
    n = n > by_length ? n : by_length;
    const long most_splits = (blocks + p.least - 1) / p.least;
    n = n < most_splits ? n : most_splits;
    n = n < (1 << 22) / items ? n : (1 << 22) / items;   // (a launch has fewer than 2^32 threads)
    p.splits = n < 1 ? 1 : (int)n;
    return p;
}

template <int D, int MODE, int RT>
hipError_t launch(const HeadRows &Q, int T, const int *cu, int B, int most, int max_len, float scale, bool causal,
                  const PagedCache &c, void *O, float *part, const Plan &p, hipStream_t st) {
    constexpr int NW = waves_of(D);
    const Sizes sz = {T, B, Q.H, Q.H / c.Hk, most, max_len, p.tiles, p.splits, p.least, Q.token, Q.head,
                      scale * 1.4426950408889634f, causal ? 1 : 0};
    const unsigned items = (unsigned)((long)B * c.Hk * p.tiles);
#define DFSS_LAUNCH(SPLIT)                                                                                              \
    hipLaunchKernelGGL((k_cached<D, MODE, NW, RT, SPLIT>), dim3(items * p.splits), dim3(64 * NW), 0, st,               \
                       (const __bf16 *)Q.data, cu, c, c.k, c.v, c.k_scale, c.v_scale, c.table, sz, (uint16_t *)O, part)
    if (p.splits > 1) {
        DFSS_LAUNCH(true);
        hipLaunchKernelGGL(k_cached_merge<D>, dim3(items * RT), dim3(2 * D), 0, st, part, cu, c, sz, RT, (uint16_t *)O);
    } else {
        DFSS_LAUNCH(false);
    }
#undef DFSS_LAUNCH
    return hipGetLastError();
}

}  // namespace

size_t cached_workspace_bytes(int B, int Hq, int Hk, int most, int max_len, int d) {
    const Plan p = plan(B, Hk, Hq / Hk, most, max_len, d);
    return p.splits == 1 ? 0 : (size_t)B * Hk * p.tiles * p.RT * p.splits * 16 * (d + 2) * sizeof(float);
}

hipError_t launch_attention_cached(const HeadRows &Q, int T, const int *cu, int B, int most, int max_len, int d, int mode,
                                   float scale, bool causal, const PagedCache &c, void *O, void *part, hipStream_t st) {
    const Plan p = plan(B, c.Hk, Q.H / c.Hk, most, max_len, d);
#define DFSS_CALL(D, M, RT) launch<D, M, RT>(Q, T, cu, B, most, max_len, scale, causal, c, O, (float *)part, p, st)
#define DFSS_MODE(D, M) (p.RT == 1 ? DFSS_CALL(D, M, 1) : DFSS_CALL(D, M, 2))
    if (d == 64) return mode == 0 ? DFSS_MODE(64, MODE_2TO4) : mode == 1 ? DFSS_MODE(64, MODE_1TO2) : DFSS_MODE(64, MODE_DENSE);
    return mode == 0 ? DFSS_MODE(128, MODE_2TO4) : mode == 1 ? DFSS_MODE(128, MODE_1TO2) : DFSS_MODE(128, MODE_DENSE);
#undef DFSS_MODE
#undef DFSS_CALL
}

}  // namespace dfss
