// Activation functions of the feed-forward operators and their slopes, in fp32, and the 8-column step the GEMM's epilogues
// share: bias, activation and residual forwards, the activation's slope backwards.
#ifndef CCL_ACT_CUH_
#define CCL_ACT_CUH_

#include <cuda_bf16.h>

#include "ccl_common.h"

namespace ccl {

// What is computed and how exactly.  The logistic function s(t) = 1 / (1 + exp(-t)) is taken with the hardware's exponential and
// reciprocal (a few units of 2^-22): every result below is rounded to bf16 (2^-9) or summed in fp32.
//   relu       max(z, 0), NaN kept           slope 1 for z > 0, 0 for z <= 0
//   gelu_tanh  z/2 (1 + tanh(t/2)) = z s(t), t = 2 sqrt(2/pi) (z + 0.044715 z^3)    slope s + z s (1 - s) dt/dz
//   gelu_erf   z/2 (1 + erf(z/sqrt 2))       slope of that: 1/2 (1 + erf(z/sqrt 2)) + z exp(-z^2/2) / sqrt(2 pi)
//   silu       z s(z)                        slope s (1 + z (1 - s))
// The product form z s(t) costs one exponential and one reciprocal where tanh takes several steps.
__device__ __forceinline__ float logistic(float t) { return __fdividef(1.0f, 1.0f + __expf(-t)); }

constexpr float kGeluA = 1.5957691216057308f;            // 2 sqrt(2 / pi)
constexpr float kGeluB = 0.044715f;

template <int ACT>
__device__ __forceinline__ float act_value(float z) {
    if (ACT == CCL_ACT_RELU) return z < 0.0f ? 0.0f : z;
    if (ACT == CCL_ACT_GELU_TANH) return z * logistic(kGeluA * z * fmaf(kGeluB * z, z, 1.0f));
    if (ACT == CCL_ACT_GELU_ERF) return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
    if (ACT == CCL_ACT_SILU) return z * logistic(z);
    return z;
}
template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
    if (ACT == CCL_ACT_RELU) return z <= 0.0f ? 0.0f : 1.0f;
    if (ACT == CCL_ACT_GELU_TANH) {
        const float s = logistic(kGeluA * z * fmaf(kGeluB * z, z, 1.0f));
        const float c = fminf(fmaxf(z, -12.0f), 12.0f);  // s (1 - s) is 0 in fp32 beyond that, and z^2 must not reach infinity: 0 * inf
        return fmaf(c * s * (1.0f - s), kGeluA * fmaf(3.0f * kGeluB * c, c, 1.0f), s);
    }
    if (ACT == CCL_ACT_GELU_ERF)
        return fmaf(z * 0.39894228040143268f, __expf(-0.5f * z * z), 0.5f * (1.0f + erff(z * 0.70710678118654752f)));
    if (ACT == CCL_ACT_SILU) {
        const float s = logistic(z);
        return s * fmaf(z, 1.0f - s, 1.0f);
    }
    return 1.0f;
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t bf16_pack(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void bf16x8_unpack(const uint4& w, float (&v)[8]) {
    v[0] = bf16_lo(w.x); v[1] = bf16_hi(w.x); v[2] = bf16_lo(w.y); v[3] = bf16_hi(w.y);
    v[4] = bf16_lo(w.z); v[5] = bf16_hi(w.z); v[6] = bf16_lo(w.w); v[7] = bf16_hi(w.w);
}
__device__ __forceinline__ uint4 bf16x8_pack(const float (&v)[8]) {
    return make_uint4(bf16_pack(v[0], v[1]), bf16_pack(v[2], v[3]), bf16_pack(v[4], v[5]), bf16_pack(v[6], v[7]));
}

// v <- act(v); the branch is the same for the whole launch
__device__ __forceinline__ void act8(int act, float (&v)[8]) {
#define CCL_ACT8(A) case A: _Pragma("unroll") for (int i = 0; i < 8; ++i) v[i] = act_value<A>(v[i]); break
    switch (act) { CCL_ACT8(CCL_ACT_RELU); CCL_ACT8(CCL_ACT_GELU_TANH); CCL_ACT8(CCL_ACT_GELU_ERF); CCL_ACT8(CCL_ACT_SILU); default: break; }
#undef CCL_ACT8
}
// v <- v * act'(z)
__device__ __forceinline__ void slope8(int act, float (&v)[8], const float (&z)[8]) {
#define CCL_ACT8(A) case A: _Pragma("unroll") for (int i = 0; i < 8; ++i) v[i] *= act_slope<A>(z[i]); break
    switch (act) { CCL_ACT8(CCL_ACT_RELU); CCL_ACT8(CCL_ACT_GELU_TANH); CCL_ACT8(CCL_ACT_GELU_ERF); CCL_ACT8(CCL_ACT_SILU); default: break; }
#undef CCL_ACT8
}

// Column sums of a warp's 32 rows (one per lane) over 2 W columns: halves are exchanged with the lane across and added, W
// steps in all instead of 5 for each column.  Afterwards lane L holds the sums of columns (2 W / 32) L ... of the 2 W, for
// 2 W = 64: columns 2 L and 2 L + 1, in v[0] and v[1].  The order of the additions is fixed.
__device__ __forceinline__ void column_sums64(float (&v)[64], int lane) {
#pragma unroll
    for (int w = 32; w >= 2; w >>= 1) {
        const bool up = lane & (w >> 1);
#pragma unroll
        for (int i = 0; i < w; ++i) {
            const float send = up ? v[i] : v[i + w], keep = up ? v[i + w] : v[i];
            v[i] = keep + __shfl_xor_sync(0xffffffffu, send, w >> 1);
        }
    }
}
// The same for 8 columns: every lane ends up with the sum of column lane / 4.
__device__ __forceinline__ float column_sums8(float (&v)[8], int lane) {
#pragma unroll
    for (int w = 4; w >= 1; w >>= 1) {
        const bool up = lane & (w << 2);
#pragma unroll
        for (int i = 0; i < w; ++i) {
            const float send = up ? v[i] : v[i + w], keep = up ? v[i + w] : v[i];
            v[i] = keep + __shfl_xor_sync(0xffffffffu, send, w << 2);
        }
    }
    v[0] += __shfl_xor_sync(0xffffffffu, v[0], 2);
    v[0] += __shfl_xor_sync(0xffffffffu, v[0], 1);
    return v[0];
}

}  // namespace ccl

#endif  // CCL_ACT_CUH_
