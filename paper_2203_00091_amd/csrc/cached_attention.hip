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

// A load at an address that is the same in every lane, of memory that no kernel of the call writes, by the scalar unit: what
// follows from it (pages, addresses) stays off the vector unit.
template <typename T>
__device__ __forceinline__ T scalar_load(const T *p, long i) {
    typedef const T __attribute__((address_space(4))) *constant;
    return ((constant)(uintptr_t)p)[i];
}

// Integer division is vector work, and so would be all that follows from its result.
__device__ __forceinline__ int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }

struct Sizes {
    int T, B, Hq, G, most, max_len, tiles, target, least;   // tiles: row tiles (of 16 RT rows) of a sequence and key head
    long q_token, q_head;
    double per_target;   // 1 / target
    float c;          // scale * log2(e)
    int causal;
};

// Where keys are shared: sequences are cut into shares of `per` blocks, the same for all of them, so that each of `target`
// workgroups for every key head and row tile gets about one, whatever the lengths are: per = ceil(all blocks / target), so that all
// sequences together have at most target + B shares.  They are numbered through the sequences.
struct Shares {
    int per;
    // Blocks of a sequence by its length (its row tiles may see fewer under the causal mask).
    static __device__ __forceinline__ int blocks(const Sizes &s, const PagedCache &c, int b) {
        const long capacity = (long)c.width << c.page_shift;
        const int most = s.max_len < capacity ? s.max_len : (int)capacity, len = c.len[b];
        return ((len < 0 ? 0 : len < most ? len : most) + KB - 1) / KB;
    }
    // Sum over the lanes up to this one.
    static __device__ __forceinline__ int scan(int x) {
#define DFSS_STEP(ctrl, rows) x += __builtin_amdgcn_update_dpp(0, x, ctrl, rows, 0xF, true)
        DFSS_STEP(0x111, 0xF);   // from 1, 2, 4 and 8 lanes before, within rows of 16
        DFSS_STEP(0x112, 0xF);
        DFSS_STEP(0x114, 0xF);
        DFSS_STEP(0x118, 0xF);
        DFSS_STEP(0x142, 0xA);   // the last lane of the row before into rows 1 and 3
        DFSS_STEP(0x143, 0xC);   // lane 31 into rows 2 and 3
#undef DFSS_STEP
        return x;
    }
    __device__ __forceinline__ void init(const Sizes &s, const PagedCache &c, int l) {
        int total = 0;   // (plan: at most 2^30 blocks)
        for (int i = 0; i < s.B; i += 64) total += i + l < s.B ? blocks(s, c, i + l) : 0;
        total = __builtin_amdgcn_readlane(scan(total), 63);
        int p = (int)((double)total * s.per_target);
        p += (long)p * s.target < total;   // rounded up (a division would take ten times the instructions)
        per = scalar(p < s.least ? s.least : p);
    }
    // Number of the first share of sequence `upto`, or (upto < 0) the sequence that share `at` belongs to, and the number of
    // its first one.  Returns -1 if there is no such share.
    __device__ __forceinline__ int find(const Sizes &s, const PagedCache &c, int l, int at, int upto, int *first) const {
        int before = 0;
        for (int i = 0; i < s.B; i += 64) {
            const int n = i + l < s.B ? (blocks(s, c, i + l) + per - 1) / per : 0, sum = scan(n);
            if (upto >= 0) {
                if (upto < i + 64) return before + __builtin_amdgcn_readlane(sum - n, upto - i);
            } else {
                const uint64_t after = __ballot(at < before + sum);
                if (after) {
                    const int lane = __builtin_ctzll(after);
                    *first = before + __builtin_amdgcn_readlane(sum - n, lane);
                    return i + lane;
                }
            }
            before += __builtin_amdgcn_readlane(sum, 63);
        }
        return upto >= 0 ? before : -1;
    }
};

// What a row tile needs to know of its sequence.
struct Rows {
    int b, h, lo, n, len, first;   // first: position of query 0
    int r0, rows;                  // first row of the tile, rows of the sequence
    int keys;                      // keys that any row of the tile sees
    __device__ __forceinline__ bool init(const Sizes &s, const int *cu, const PagedCache &c, int seq, int head, int tile, int tile_rows) {
        b = seq, h = head;
        lo = b * s.most, n = s.most;
        if (cu) {
            lo = scalar_load(cu, b), n = scalar_load(cu, b + 1);
            lo = lo < 0 ? 0 : lo < s.T ? lo : s.T;
            n = n < lo ? 0 : (n < s.T ? n : s.T) - lo;
        }
        const int queries = n < s.most ? n : s.most;
        r0 = tile * tile_rows, rows = queries * s.G;
        if (r0 >= rows) return false;
        const long capacity = (long)c.width << c.page_shift;
        len = scalar_load(c.len, b);
        len = len < 0 ? 0 : len;
        first = len - n;           // (by the length given: a longer one than the call allows is cut, positions stay)
        const int most_keys = s.max_len < capacity ? s.max_len : (int)capacity;
        len = len < most_keys ? len : most_keys;
        const int last = r0 + tile_rows < rows ? r0 + tile_rows - 1 : rows - 1;
        keys = scalar(limit(s, last));
        return true;
    }
    // keys that row r sees: those before it
    __device__ __forceinline__ int limit(const Sizes &s, int r) const {
        if (!s.causal) return len;
        const int x = first + r / s.G + 1;
        return x < 0 ? 0 : x < len ? x : len;
    }
    __device__ __forceinline__ int blocks() const { return (keys + KB - 1) / KB; }
};

template <int D>
constexpr int partial_floats() { return 16 * (D + 2); }   // of a 16-row tile: references, sums, O

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
    const float mb = m_ref * c;
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

// BIG: pages of 64 tokens or more, a block lies in one.
template <int D, int MODE, int NW, int RT, bool BIG>
__global__ __launch_bounds__(64 * NW, RT == 1 && D == 64 ? 3 : RT <= 2 ? 2 : 1) void k_cached(const __bf16 *__restrict__ Q, const int *__restrict__ cu, PagedCache cache,
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
        int id[NG], bad;      // page of each group (0 where there is none), and a bit for each 16 keys without one
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
            p.id[g] = none ? 0 : id;
            p.bad |= none ? (BIG ? 15 : 1 << g) : 0;
        }
        return p;
    };
    auto scales = [&](const Pages &p) {
        Scales s;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            const long at = (long)p.id[g] * cache.Hk + R.h;
            s.k[g] = scalar_load(Ks, at);
            s.v[g] = scalar_load(Vs, at);
        }
        return s;
    };
    auto place = [&](const Pages &p, int jb, int g) {   // bytes before a group's first key
        return ((((long)p.id[g] * cache.Hk + R.h) << cache.page_shift) + ((jb * KB + 16 * g) & page_mask)) * D;
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
            for (int x = 0; x < SS; ++x) kr[t][x] = *reinterpret_cast<const u32x4 *>(q + 64 * x);
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
                    const u32x2 x = *reinterpret_cast<const u32x2 *>(q + e * D);
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

// The same for many rows: a prompt's queries, or a part of them.  Here the matrix unit and the exponentials bound it, and
// what a code costs on the way to an operand: a workgroup takes 128 rows, 32 to a wave, and its waves share the keys as bfloat16 in
// LDS, so that a block is read and converted once for all of them (a wave of k_cached with 32 rows did both for itself: 4 x 512 queries
// x 4 heads to a key head, 4096 keys, d = 128, 120 us, with 64 rows 130).  Two teams of four waves take every other block, each
// out of LDS of its own: two waves to a SIMD unit, of which one computes while the other waits, without partial results in memory
// (two workgroups that share the keys: 111 us, and 12 for the merge).  The next block's codes are in registers while this one is
// worked on, those after it on their way; one barrier a block.
//   K   row of MFMA row i of tile t (k_cached's keys) at slot 16 t + i, chunks of 16 bytes by the slot's low bits
//   V   row by key, read with the transposing LDS read as in k_few: column li of tile ds is d = 16 ds + li
template <int D, int MODE>
__global__ __launch_bounds__(512, 2) void k_cached_wide(const __bf16 *__restrict__ Q, const int *__restrict__ cu, PagedCache cache,
                                                        const uint8_t *__restrict__ Kc, const uint8_t *__restrict__ Vc,
                                                        const float *__restrict__ Ks, const float *__restrict__ Vs,
                                                        const int *__restrict__ table, Sizes sz, uint16_t *__restrict__ O,
                                                        float *__restrict__ part) {
    constexpr int RT = 2;               // 16-row tiles of a wave
    constexpr int CPR = D / 8;          // 16-byte chunks of a row of K or V in LDS
    constexpr int TILE = KB * CPR;
    constexpr int STEPS = D / 32, DT = D / 16;
    constexpr int PIECES = D / 64;      // 16-byte pieces of K (and of V) that a thread fetches of a block, 64 / PIECES keys apart
    constexpr bool DENSE = MODE == MODE_DENSE;
    constexpr int NF = 4 * DT + 5;      // floats per lane and row tile of a team's result
    __shared__ u32x4 lds_all[2][2][2][TILE];   // [team][buffer][K, V]
    static_assert(4 * RT * NF * 64 * 4 <= (int)sizeof(lds_all), "a team's results fit into LDS");

    const int w8 = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), team = w8 >> 2, w = w8 & 3, tid = threadIdx.x & 255, l = threadIdx.x & 63, li = l & 15, kb = l >> 4;
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
    if (!R.init(sz, cu, cache, seq, head, tile, 128)) return;
    const int nblocks = R.blocks();
    end = nblocks;
    if (sz.target) {
        begin = (number - first) * sh.per;
        if (begin >= nblocks) return;
        end = begin + sh.per < nblocks ? begin + sh.per : nblocks;
    }
    const bool alone = begin == 0 && end == nblocks;
    const int page_mask = (1 << cache.page_shift) - 1, last_entry = (R.keys > 0 ? R.keys - 1 : 0) >> cache.page_shift;
    const int *const my_table = table + (long)R.b * cache.width;

    u32x4(*const lds)[2][TILE] = lds_all[team];

    // this wave's rows; the keys that the first of them sees are seen by all, those that the last one does not by none
    const int wr0 = R.r0 + 32 * w, wr1 = wr0 + 31 < R.rows ? wr0 + 31 : R.rows - 1;
    const int seen_by_all = wr0 < R.rows ? scalar(R.limit(sz, wr0)) : 0, seen = wr0 < R.rows ? scalar(R.limit(sz, wr1)) : 0;
    bf16x8 bq[RT][STEPS];
    int limit[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        int r = wr0 + 16 * rt + li;
        r = r < R.rows ? r : R.rows - 1;
        limit[rt] = R.limit(sz, r);
        const int i = r / sz.G, g = r - i * sz.G;
        const __bf16 *const q = Q + (R.lo + i) * sz.q_token + (R.h * sz.G + g) * sz.q_head;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) bq[rt][s] = *reinterpret_cast<const bf16x8 *>(q + 32 * s + 8 * kb);
    }

    // Fetching: thread t has the 16 codes from element 16 (t % (D / 16)) on of key t / (D / 16) (+ 64 / PIECES): a wave's keys lie
    // in one group of 16, and so in one page.
    constexpr int LPK = D / 16;         // threads of a key
    const int f_key = tid / LPK, f_el = 16 * (tid % LPK);
    struct Fetched {
        u32x4 k[PIECES], v[PIECES];
        float ks[PIECES], vs[PIECES];
        bool none[PIECES];   // the page is none
    };
    auto fetch = [&](int jb, Fetched &f) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int key0 = jb * KB + (64 / LPK) * w + (64 / PIECES) * i;     // the wave's first key
            const int entry = key0 >> cache.page_shift;
            int page = scalar_load(my_table, entry < last_entry ? entry : last_entry);
            f.none[i] = (unsigned)page >= (unsigned)cache.n_pages;
            page = f.none[i] ? 0 : page;
            const long at = (long)page * cache.Hk + R.h;
            f.ks[i] = scalar_load(Ks, at);
            f.vs[i] = scalar_load(Vs, at);
            const long row = ((at << cache.page_shift) + ((jb * KB + (64 / PIECES) * i + f_key) & page_mask)) * D + f_el;
            f.k[i] = *reinterpret_cast<const u32x4 *>(Kc + row);
            f.v[i] = *reinterpret_cast<const u32x4 *>(Vc + row);
        }
    };
    auto put = [&](int jb, int buf, const Fetched &f) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int key = (64 / PIECES) * i + f_key;
            const int slot = DENSE ? 16 * (2 * (key >> 5) + ((key >> 2) & 1)) + 4 * ((key >> 3) & 3) + (key & 3)
                                   : 16 * ((key >> 2) & 3) + 4 * (key >> 4) + (key & 3);
            const int chunk = f_el / 8;
            u32x4 *const kd = &lds[buf][0][slot * CPR], *const vd = &lds[buf][1][key * CPR];
            // what lies behind the last key is no value at all (0 x NaN is not 0)
            const bool real = jb * KB + key < R.keys && !f.none[i];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                u32x4 a, b;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t k = f.k[i][2 * y + e], v = real ? f.v[i][2 * y + e] : 0u;
                    a[2 * e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(k, f.ks[i], false));
                    a[2 * e + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(k, f.ks[i], true));
                    b[2 * e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, f.vs[i], false));
                    b[2 * e + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, f.vs[i], true));
                }
                kd[(chunk + y) ^ operand_row_swizzle<CPR, 16>(slot)] = a;
                vd[(chunk + y) ^ tr_row_swizzle<CPR>(key)] = b;
            }
        }
    };
    // groups of 16 keys of a block without a page, a bit each
    auto without_page = [&](int jb) {
        int bad = 0;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int entry = (jb * KB + 16 * g) >> cache.page_shift;
            bad |= (unsigned)scalar_load(my_table, entry < last_entry ? entry : last_entry) >= (unsigned)cache.n_pages ? 1 << g : 0;
        }
        return bad;
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
    const int tr_row = li >> 2, tr_sub = (li >> 1) & 1, tr_byte = 8 * (li & 1);

    Fetched f;
    int bad = 0, bad_next = 0;   // of this block, and of the next one (asked for a block ahead)
    const int mine = begin + team;
    if (mine < end) {
        fetch(mine, f);
        bad = without_page(mine);
        put(mine, 0, f);
        if (mine + 2 < end) fetch(mine + 2, f);
        bad_next = without_page(mine + 2);
    }
    int buf = 0;
    for (int jb = mine; jb < end + team; jb += 2, buf ^= 1) {   // (as many steps in both teams)
        __syncthreads();   // this block is in LDS, and nobody reads the one before it any more
        const u32x4 *const kt = lds[buf][0];
        const char *const vt = reinterpret_cast<const char *>(lds[buf][1]);
        if (jb < end && jb * KB < seen) {   // (the same in every lane)
            // s[rt][t][r] = q . k of query li of tile rt and the lane's key r of tile t
            f32x4 s[RT][4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) s[rt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int y = 0; y < STEPS; ++y) {
                    const int slot = 16 * t + li;
                    const bf16x8 a = __builtin_bit_cast(bf16x8, kt[slot * CPR + ((4 * y + kb) ^ operand_row_swizzle<CPR, 16>(slot))]);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) s[rt][t] = mfma16(a, bq[rt][y], s[rt][t]);
                }
            }
            read_ahead<4 * STEPS, 1, 4, 1, 0, RT>();
            if (jb * KB + KB > seen_by_all || bad) {
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
            }
            bf16x8 p[RT][DENSE ? 2 : 1];
            uint32_t idx[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) weigh<MODE, DT>(s[rt], sz.c, kb, ones8, m_ref[rt], acc_o[rt], acc_l[rt], p[rt], idx[rt]);
#pragma unroll
            for (int ds = 0; ds < DT; ++ds) {
                auto tr = [&](int key0) {
                    const int row = key0 + tr_row, chunk = (2 * ds + tr_sub) ^ tr_row_swizzle<CPR>(row);
                    return lds_read_tr16(vt + (row * CPR + chunk) * 16 + tr_byte);
                };
                const s16x4 t0 = tr(8 * kb), t1 = tr(8 * kb + 4), t2 = tr(32 + 8 * kb), t3 = tr(36 + 8 * kb);
                const s16x8 lo = __builtin_shufflevector(t0, t1, 0, 1, 2, 3, 4, 5, 6, 7);
                const s16x8 hi = __builtin_shufflevector(t2, t3, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    if constexpr (DENSE) {
                        acc_o[rt][ds] = mfma16(p[rt][0], __builtin_bit_cast(bf16x8, lo), acc_o[rt][ds]);
                        acc_o[rt][ds] = mfma16(p[rt][1], __builtin_bit_cast(bf16x8, hi), acc_o[rt][ds]);
                    } else {
                        const s16x16 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 14, 15);
                        acc_o[rt][ds] = __builtin_amdgcn_smfmac_f32_16x16x64_bf16(p[rt][0], __builtin_bit_cast(bf16x16, both), acc_o[rt][ds], (int)idx[rt], 0, 0);
                    }
                }
            }
            read_ahead<DT, 4, 2, 2, 0, DENSE ? 2 * RT : RT>();
        }
        if (jb + 2 < end) {
            put(jb + 2, buf ^ 1, f);
            if (jb + 4 < end) fetch(jb + 4, f);
            bad = bad_next;
            bad_next = without_page(jb + 4);
        }
    }

    // The second team's results join the first one's: value f of lane l of wave w and row tile rt at float (w RT + rt) NF 64 + f 64 + l.
    __syncthreads();
    float *const slots = reinterpret_cast<float *>(lds_all) + w * (RT * NF * 64) + l;
    if (team == 1) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float *const to = slots + rt * (NF * 64);
            to[0] = m_ref[rt];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                to[(1 + r) * 64] = acc_l[rt][r];
#pragma unroll
                for (int t = 0; t < DT; ++t) to[(5 + 4 * t + r) * 64] = acc_o[rt][t][r];
            }
        }
    }
    __syncthreads();
    if (team == 1) return;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const float *const from = slots + rt * (NF * 64);
        const float other = from[0], m = fmaxf(m_ref[rt], other);
        const float fa = __builtin_amdgcn_exp2f((m_ref[rt] - m) * sz.c), fb = __builtin_amdgcn_exp2f((other - m) * sz.c);
        m_ref[rt] = m;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float a_r = __shfl(fa, 4 * kb + r, 64), b_r = __shfl(fb, 4 * kb + r, 64);
            acc_l[rt][r] = a_r * acc_l[rt][r] + b_r * from[(1 + r) * 64];
#pragma unroll
            for (int t = 0; t < DT; ++t) acc_o[rt][t][r] = a_r * acc_o[rt][t][r] + b_r * from[(5 + 4 * t + r) * 64];
        }
    }

    // O: rows 4 kb + r of each tile, columns 16 ds + li
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int t16 = 2 * w + rt;   // the 16-row tile within the workgroup's
        float *const P = part + ((long)id * 8 + t16) * partial_floats<D>();
        if (!alone && kb == 0 && R.r0 + 16 * t16 + li < R.rows) P[li] = m_ref[rt];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = 4 * kb + r, at = R.r0 + 16 * t16 + row;
            if (at >= R.rows) continue;
            const float sum = acc_l[rt][r];
            if (!alone) {
                if (li == 0) P[16 + row] = sum;
#pragma unroll
                for (int ds = 0; ds < DT; ++ds) P[32 + row * D + 16 * ds + li] = acc_o[rt][ds][r];
                continue;
            }
            const float inv = sum > 0.f ? 1.f / sum : 0.f;   // (a row that sees no key: 0)
            const int i = at / sz.G, g = at - i * sz.G;
            uint16_t *const out = O + ((long)(R.lo + i) * sz.Hq + R.h * sz.G + g) * D + li;
#pragma unroll
            for (int ds = 0; ds < DT; ++ds) out[16 * ds] = (uint16_t)(pack_bf16x2(acc_o[rt][ds][r] * inv, 0.f) & 0xFFFFu);
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
    float m = -1.0e30f, sum = 0.f;
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

constexpr int kWide = 8;   // k_cached_wide
// 16-row tiles of a workgroup
int row_tiles(long rows) { return rows <= 16 ? 1 : rows <= 32 ? 2 : kWide; }

struct Plan {
    int RT, NW, tiles, target, least;   // NW: waves of a workgroup; target 0: nobody shares
};
Plan plan(int B, int Hk, int G, int most, int max_len, int d) {
    Plan p;
    const long rows = (long)most * G;
    p.RT = row_tiles(rows);
    p.tiles = (int)((rows + 16 * p.RT - 1) / (16 * p.RT));
    const long per_share = (long)Hk * p.tiles, items = B * per_share;   // workgroups of a share, and without shares
    const int blocks = (max_len + KB - 1) / KB;
    p.NW = items <= 256 || p.RT == kWide ? 8 : 4;
    p.target = 0;
    p.least = p.NW;
    if (blocks <= 5 * p.NW || (long)B * blocks > 1 << 30) return p;
    if (items * blocks <= 4096 && p.RT != kWide) p.NW = 4;
    const long slots = p.NW == 8 ? 256 : 512;
    if (items >= 4 * slots || (items >= slots && blocks < 128)) return p;
    p.least = p.NW;
    const long fit = slots / per_share - B;       // (the last share of a sequence is cut short)
    long t = fit > B / 2 ? fit : B / 2 > 0 ? B / 2 : 1;
    const long most_shares = (long)B * ((blocks + p.least - 1) / p.least);
    p.target = (int)(t < most_shares ? t : most_shares);
    return p;
}
// Shares of all sequences, at most (of a valid plan that shares)
long shares_of(const Plan &p, int B) { return (long)p.target + B; }

template <int D, int MODE>
hipError_t launch(const HeadRows &Q, int T, const int *cu, int B, int most, int max_len, float scale, bool causal,
                  const PagedCache &c, void *O, float *part, const Plan &p, hipStream_t st) {
    const Sizes sz = {T, B, Q.H, Q.H / c.Hk, most, max_len, p.tiles, p.target, p.least, Q.token, Q.head, p.target ? 1. / p.target : 0.,
                      scale * 1.4426950408889634f, causal ? 1 : 0};
    const unsigned items = (unsigned)((long)B * c.Hk * p.tiles), shares = (unsigned)(shares_of(p, B) * c.Hk * p.tiles);
#define DFSS_LAUNCH(KERNEL)                                                                                             \
    hipLaunchKernelGGL((KERNEL), dim3(p.target ? shares : items), dim3(64 * p.NW), 0, st, (const __bf16 *)Q.data, cu, c, c.k, c.v,  \
                       c.k_scale, c.v_scale, c.table, sz, (uint16_t *)O, part)
#define DFSS_PAGES(NW, RT)                                                                                              \
    if (c.page_shift >= 6) DFSS_LAUNCH(DFSS_K(NW, RT, true)); else DFSS_LAUNCH(DFSS_K(NW, RT, false))
#define DFSS_K(NW, RT, BIG) k_cached<D, MODE, NW, RT, BIG>
#define DFSS_WIDE k_cached_wide<D, MODE>
    if (p.RT == kWide) {
        DFSS_LAUNCH(DFSS_WIDE);
    } else if (p.RT == 1) {
        if (p.NW == 8) { DFSS_PAGES(8, 1); } else { DFSS_PAGES(4, 1); }
    } else {
        if (p.NW == 8) { DFSS_PAGES(8, 2); } else { DFSS_PAGES(4, 2); }
    }
#undef DFSS_K
#undef DFSS_WIDE
#undef DFSS_PAGES
#undef DFSS_LAUNCH
    if (p.target)
        hipLaunchKernelGGL(k_cached_merge<D>, dim3(items * p.RT), dim3(2 * D), 0, st, part, cu, c, sz, p.RT, (uint16_t *)O);
    return hipGetLastError();
}

}  // namespace

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
