// What the kernels over the paged cache share: sizes of a call, rows and keys of a workgroup, keys shared between workgroups.
#pragma once
#include "dfss_device.hpp"
#include "dfss_kernels.hpp"

namespace dfss {
namespace cached {

constexpr int KB = 64;    // keys per block
enum { MODE_2TO4 = 0, MODE_1TO2 = 1, MODE_DENSE = 2 };

// The softmax reference (in raw scores) of a query that has seen no key yet: below all that the calls allow (scaled scores to 2^24 under
// a scale of 2^-100: 2^124 = 2.1e37) by so much that the first one seen replaces it (7.9e37 x 2^-100 is 6e7).
constexpr float kNoReference = -1.0e38f;

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
    double per_target, per_place;   // 1 / target; 1 / (target + B) where `per` is to be the least possible, else 0
    float c;          // scale * log2(e)
    int causal;
};

// Where keys are shared: sequences are cut into shares of `per` blocks, the same for all of them, so that each of `target`
// workgroups for every key head and row tile gets about one, whatever the lengths are: per = ceil(all blocks / target), so that all
// sequences together have at most target + B shares.  With few shares to a sequence (per_place), the last one of each, which is cut short,
// leaves much of the chip idle: there `per` is the least that makes no more than target + B shares.  They are numbered through the sequences.
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
        if (s.per_place == 0.) return;
        // (a smaller `per` never makes fewer shares, so halving finds it; up to 64 sequences, one to a lane)
        const int n = l < s.B ? blocks(s, c, l) : 0;
        int lo = scalar((int)((double)total * s.per_place)), hi = per;
        lo = lo < s.least ? s.least : lo;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (__builtin_amdgcn_readlane(scan((n + mid - 1) / mid), 63) <= s.target + s.B) hi = mid;
            else lo = mid + 1;
        }
        per = hi;
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

// Waits for an operand that was loaded before a loop, there.  (Left to the compiler, the wait stands in the loop, where it waits
// for all that the loop has asked for in the meantime.)
template <typename T>
__device__ __forceinline__ void arrived(T &x) {
    asm volatile("" : "+v"(x));
}

// A call of many rows (cached_wide.hip): row tiles of 16 kWide queries, workgroups of 512 threads.
constexpr int kWide = 8;
hipError_t launch_wide(const __bf16 *Q, const int *cu, const PagedCache &c, int d, int mode, const Sizes &sz, unsigned workgroups,
                       uint16_t *O, float *part, hipStream_t st);

}  // namespace cached
}  // namespace dfss
