// Activation functions of the feed-forward operators and their slopes, in fp32, and the 8-column step the GEMM's epilogues
// share: bias, activation and residual forwards, the activation's slope backwards.
#ifndef CCL_ACT_CUH_
#define CCL_ACT_CUH_

#include <cuda_bf16.h>

#include "ccl_common.h"

namespace ccl {

// Two fp32 values in one 64-bit register: sm_100 multiplies and adds such pairs in one instruction.  Under a GEMM that runs at the
// power limit an epilogue costs what its instructions cost in energy, whether or not there is time for them (measured,
// 4096 x 8192 x 2048: the clock falls from 1.5 to 1.25 GHz behind gelu's slope): about 0.8 us an instruction a value there.
struct f32x2 { uint64_t v; };
__device__ __forceinline__ f32x2 pair(float lo, float hi) {
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ f32x2 both(float x) { return pair(x, x); }
__device__ __forceinline__ void split(f32x2 a, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(a.v)); }
__device__ __forceinline__ f32x2 operator*(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ f32x2 operator+(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
__device__ __forceinline__ float exp2_fast(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ float rcp_fast(float x) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ f32x2 exp2_fast(f32x2 a) { float x, y; split(a, x, y); return pair(exp2_fast(x), exp2_fast(y)); }
__device__ __forceinline__ f32x2 rcp_fast(f32x2 a) { float x, y; split(a, x, y); return pair(rcp_fast(x), rcp_fast(y)); }

// What is computed and how exactly.  The logistic function s(t) = 1 / (1 + 2^(-t log2 e)) is taken with the hardware's exponential and
// reciprocal (a few units of 2^-22): every result below is rounded to bf16 (2^-9) or summed in fp32.
//   relu       max(z, 0), NaN kept           slope 1 for z > 0, 0 for z <= 0
//   gelu_tanh  z/2 (1 + tanh(t/2)) = z s(t), t = 2 sqrt(2/pi) (z + 0.044715 z^3)    slope s + z s (1 - s) dt/dz
//   gelu_erf   z P(z), P(z) = 1/2 (1 + erf(z/sqrt 2))                                slope P + z exp(-z^2/2) / sqrt(2 pi)
//   silu       z s(z)                        slope s (1 + z (1 - s))
// The product form z s(t) costs one exponential and one reciprocal where tanh takes several steps.  P(z) comes from its tail, which has to
// be right relative to itself: left of 0 it is the result.  P(-x) = exp(-x^2 / 2) k g(k), k = 1 / (1 + 0.3 x), x >= 0, where g is the
// polynomial of degree 7 with the least relative error for 0 <= x <= 14 (fitted by Lawson's reweighted least squares to the scaled
// complementary error function in 64 bits): 1.5e-7.  With the roundings in fp32 the tail is off by less than 1e-6 of itself, and the
// exponential's by 2^-23 x^2 / 2 more.  (Formula 7.1.26 of Abramowitz and Stegun, three terms shorter, keeps 1.5e-7 of erf but not of the
// tail: 5e-4 of it at x = 4, 2 % at x = 10.)  The exponential is the slope's as well.
__device__ __forceinline__ float logistic(float t) { return rcp_fast(1.0f + exp2_fast(t * -1.4426950408889634f)); }

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kGeluA = 1.5957691216057308f;            // 2 sqrt(2 / pi)
constexpr float kGeluB = 0.044715f;

// 1 - P(|z|) and exp(-z^2 / 2)
__device__ __forceinline__ f32x2 normal_tail(f32x2 z, f32x2& density) {
    float x, y;
    split(z, x, y);
    const f32x2 k = rcp_fast(fma2(pair(fabsf(x), fabsf(y)), both(0.3f), both(1.0f)));
    density = exp2_fast(z * (z * both(-0.5f * kLog2e)));
    f32x2 g = fma2(k, both(0.035674781f), both(-0.157203093f));
    g = fma2(k, g, both(0.206353486f));
    g = fma2(k, g, both(-0.0536836348f));
    g = fma2(k, g, both(0.128561616f));
    g = fma2(k, g, both(0.0999135002f));
    g = fma2(k, g, both(0.120753959f));
    g = fma2(k, g, both(0.119629301f));
    return k * g * density;
}
// P(z) from the tail on z's side
__device__ __forceinline__ f32x2 normal_cdf(f32x2 z, f32x2 tail) {
    float x, y, a, b;
    split(z, x, y);
    split(tail, a, b);
    return pair(x < 0.0f ? a : 1.0f - a, y < 0.0f ? b : 1.0f - b);
}

template <int ACT>
__device__ __forceinline__ f32x2 act_value(f32x2 z) {
    if (ACT == CCL_ACT_RELU) {
        float x, y;
        split(z, x, y);
        return pair(x < 0.0f ? 0.0f : x, y < 0.0f ? 0.0f : y);
    }
    if (ACT == CCL_ACT_GELU_TANH) {                      // (z^2 = infinity leaves s at 0 or 1)
        const f32x2 e = exp2_fast(z * fma2(z * z, both(-kLog2e * kGeluA * kGeluB), both(-kLog2e * kGeluA)));
        return z * rcp_fast(e + both(1.0f));
    }
    if (ACT == CCL_ACT_GELU_ERF) {
        f32x2 d;
        const f32x2 tail = normal_tail(z, d);
        return z * normal_cdf(z, tail);
    }
    if (ACT == CCL_ACT_SILU) return z * rcp_fast(exp2_fast(z * both(-kLog2e)) + both(1.0f));
    return z;
}
// The slope at two values of z given as a bf16 pair
template <int ACT>
__device__ __forceinline__ f32x2 act_slope(uint32_t zz) {
    if (ACT == CCL_ACT_GELU_TANH) {
        // beyond 12 the slope is 0 or 1 in fp32, and z^2 must not reach infinity: 0 * inf (NaN passes both limits)
        asm("min.NaN.bf16x2 %0, %0, %1;" : "+r"(zz) : "r"(0x41404140u));
        asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(zz) : "r"(0xC140C140u));
    }
    const float x = __uint_as_float(zz << 16), y = __uint_as_float(zz & 0xFFFF0000u);
    const f32x2 z = pair(x, y);
    if (ACT == CCL_ACT_RELU) return pair(x <= 0.0f ? 0.0f : 1.0f, y <= 0.0f ? 0.0f : 1.0f);
    if (ACT == CCL_ACT_GELU_TANH) {
        const f32x2 q = z * z, e = exp2_fast(z * fma2(q, both(-kLog2e * kGeluA * kGeluB), both(-kLog2e * kGeluA)));
        const f32x2 s = rcp_fast(e + both(1.0f)), dt = fma2(q, both(3.0f * kGeluA * kGeluB), both(kGeluA));
        return fma2(fma2(s * both(-1.0f), s, s), z * dt, s);
    }
    if (ACT == CCL_ACT_GELU_ERF) {
        f32x2 d;
        const f32x2 tail = normal_tail(z, d);
        return fma2(z * both(0.39894228040143268f), d, normal_cdf(z, tail));
    }
    if (ACT == CCL_ACT_SILU) {
        const f32x2 s = rcp_fast(exp2_fast(z * both(-kLog2e)) + both(1.0f));
        return s * fma2(z, fma2(s, both(-1.0f), both(1.0f)), both(1.0f));
    }
    return both(1.0f);
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t bf16_pack(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t bf16_pack(f32x2 a) {
    float x, y;
    split(a, x, y);
    return bf16_pack(x, y);
}
__device__ __forceinline__ f32x2 bf16_unpack(uint32_t w) { return pair(bf16_lo(w), bf16_hi(w)); }
__device__ __forceinline__ uint4 bf16x8_pack(const f32x2* v) { return make_uint4(bf16_pack(v[0]), bf16_pack(v[1]), bf16_pack(v[2]), bf16_pack(v[3])); }

// v <- act(v), v <- v * act'(z) for 2 N values; the branch is the same for the whole launch
template <int N>
__device__ __forceinline__ void act_pairs(int act, f32x2 (&v)[N]) {
#define CCL_ACT_N(A) case A: _Pragma("unroll") for (int i = 0; i < N; ++i) v[i] = act_value<A>(v[i]); break
    switch (act) { CCL_ACT_N(CCL_ACT_RELU); CCL_ACT_N(CCL_ACT_GELU_TANH); CCL_ACT_N(CCL_ACT_GELU_ERF); CCL_ACT_N(CCL_ACT_SILU); default: break; }
#undef CCL_ACT_N
}
template <int N>
__device__ __forceinline__ void slope_pairs(int act, f32x2 (&v)[N], const uint32_t (&z)[N]) {
#define CCL_ACT_N(A) case A: _Pragma("unroll") for (int i = 0; i < N; ++i) v[i] = v[i] * act_slope<A>(z[i]); break
    switch (act) { CCL_ACT_N(CCL_ACT_RELU); CCL_ACT_N(CCL_ACT_GELU_TANH); CCL_ACT_N(CCL_ACT_GELU_ERF); CCL_ACT_N(CCL_ACT_SILU); default: break; }
#undef CCL_ACT_N
}

// Sums of 16 columns over a warp's 32 rows (one per lane): halves are exchanged with the lane across and added, 16 exchanges in
// all instead of 5 for each column.  Every lane ends up with the sum of column lane / 2.  The order of the additions is fixed.
__device__ __forceinline__ float column_sums16(float (&v)[16], int lane) {
#pragma unroll
    for (int w = 8; w >= 1; w >>= 1) {
        const bool up = lane & (w << 1);
#pragma unroll
        for (int i = 0; i < w; ++i) {
            const float send = up ? v[i] : v[i + w], keep = up ? v[i + w] : v[i];
            v[i] = keep + __shfl_xor_sync(0xffffffffu, send, w << 1);
        }
    }
    return v[0] + __shfl_xor_sync(0xffffffffu, v[0], 1);
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
