// What the kernels share that take rows of single heads as a projection leaves them: element types, the rotation's table.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dfss_device.hpp"

namespace dfss {

// Eight consecutive elements of a head's row, which one lane holds: 16 bytes of bfloat16, 32 of float.  load_once and store_past: what
// nobody is expected to read again soon goes from the caches first (non-temporal).
template <typename T>
struct Eight;
template <>
struct Eight<__bf16> {
    u32x4 w;
    __device__ __forceinline__ void load(const __bf16 *p) { w = *reinterpret_cast<const u32x4 *>(p); }
    __device__ __forceinline__ void store(__bf16 *p) const { *reinterpret_cast<u32x4 *>(p) = w; }
    __device__ __forceinline__ void load_once(const __bf16 *p) { w = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p)); }
    __device__ __forceinline__ void store_past(__bf16 *p) const { __builtin_nontemporal_store(w, reinterpret_cast<u32x4 *>(p)); }
    __device__ __forceinline__ void get(float *x) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[2 * e] = bf16_lo_to_f32(w[e]), x[2 * e + 1] = bf16_hi_to_f32(w[e]);
    }
    __device__ __forceinline__ void set(const float *x) {
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2(x[2 * e], x[2 * e + 1]);
    }
    __device__ __forceinline__ Eight of_lane(int l) const {
        Eight r;
#pragma unroll
        for (int e = 0; e < 4; ++e) r.w[e] = (uint32_t)__shfl((int)w[e], l, kWave);
        return r;
    }
    __device__ __forceinline__ void clear() { w = u32x4{0u, 0u, 0u, 0u}; }
};
template <>
struct Eight<float> {
    f32x4 a, b;
    __device__ __forceinline__ void load(const float *p) {
        a = reinterpret_cast<const f32x4 *>(p)[0];
        b = reinterpret_cast<const f32x4 *>(p)[1];
    }
    __device__ __forceinline__ void store(float *p) const {
        reinterpret_cast<f32x4 *>(p)[0] = a;
        reinterpret_cast<f32x4 *>(p)[1] = b;
    }
    __device__ __forceinline__ void load_once(const float *p) {
        a = __builtin_nontemporal_load(reinterpret_cast<const f32x4 *>(p));
        b = __builtin_nontemporal_load(reinterpret_cast<const f32x4 *>(p) + 1);
    }
    __device__ __forceinline__ void store_past(float *p) const {
        __builtin_nontemporal_store(a, reinterpret_cast<f32x4 *>(p));
        __builtin_nontemporal_store(b, reinterpret_cast<f32x4 *>(p) + 1);
    }
    __device__ __forceinline__ void get(float *x) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = a[e], x[4 + e] = b[e];
    }
    __device__ __forceinline__ void set(const float *x) {
#pragma unroll
        for (int e = 0; e < 4; ++e) a[e] = x[e], b[e] = x[4 + e];
    }
    __device__ __forceinline__ Eight of_lane(int l) const {
        Eight r;
#pragma unroll
        for (int e = 0; e < 4; ++e) r.a[e] = __shfl(a[e], l, kWave), r.b[e] = __shfl(b[e], l, kWave);
        return r;
    }
    __device__ __forceinline__ void clear() { a = b = f32x4{0.f, 0.f, 0.f, 0.f}; }
};

// The rotation of a token, as the lane with chunk c (elements 8c .. 8c+7) of a row needs it.
//   halves       pairs (i, i + rot/2): the lane's other elements are those of the lane `other`, chunk c +- rot/16
//   interleaved  pairs (2i, 2i + 1): all in the lane
// y_e = x_e cos_e + x'_e sin_e with x' the other element of the pair and sin_e negative at the first one; elements from
// `rot` on stay (cos 1, sin 0).  The inverse (the gradient's way) has the signs of sin exchanged.
struct Turn {
    float cos[8], sin[8];
    int other;
    bool interleaved;

    __device__ __forceinline__ void load(const float *__restrict__ cos_t, const float *__restrict__ sin_t, long pos, int rot,
                                         bool inter, int lane, int c, bool inverse) {
        interleaved = inter;
        other = lane;
        if (8 * c >= rot) {
#pragma unroll
            for (int e = 0; e < 8; ++e) cos[e] = 1.f, sin[e] = 0.f;
            return;
        }
        const int half = rot >> 1;
        const long row = pos * half;
        if (inter) {
            const f32x4 a = *reinterpret_cast<const f32x4 *>(cos_t + row + 4 * c), b = *reinterpret_cast<const f32x4 *>(sin_t + row + 4 * c);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                cos[e] = a[e >> 1];
                sin[e] = (e & 1) != (int)inverse ? b[e >> 1] : -b[e >> 1];
            }
            return;
        }
        const bool first = 8 * c < half;
        const int at = first ? 8 * c : 8 * c - half;
        other = lane + (first ? rot >> 4 : -(rot >> 4));
        const f32x4 *const pc = reinterpret_cast<const f32x4 *>(cos_t + row + at), *const ps = reinterpret_cast<const f32x4 *>(sin_t + row + at);
        const f32x4 c0 = pc[0], c1 = pc[1], s0 = ps[0], s1 = ps[1];
        const bool neg = first != inverse;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            cos[e] = c0[e], cos[4 + e] = c1[e];
            sin[e] = neg ? -s0[e] : s0[e], sin[4 + e] = neg ? -s1[e] : s1[e];
        }
    }
    // y = the rotated x; xo: the elements of the lane `other` (halves only)
    __device__ __forceinline__ void apply(const float *x, const float *xo, float *y) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = x[e] * cos[e] + (interleaved ? x[e ^ 1] : xo[e]) * sin[e];
    }
};

// Sum over the LPR lanes that hold a row.
template <int LPR>
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
    return v;
}

}  // namespace dfss
