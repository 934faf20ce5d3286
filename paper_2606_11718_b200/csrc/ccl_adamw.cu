// ccl_adamw: one step of AdamW over a list of tensors, optimiser states in 32 bits or in 8.
//
// Every operation is rounded to nearest in fp32, one by one, in the order the header states (no contraction into fused
// multiply-adds), so a step gives the same bits as the same operations done one after the other.
//
// Bound by memory: parameters, gradient and states are read once and written once.  The list travels in the kernel's parameters
// (no table on the device, nothing to copy, a captured call keeps its own), kMost tensors a launch at most; each tensor is cut into
// pieces of kPiece elements, the pieces of all tensors are numbered through, and persistent CTAs take them in turn, so that one large
// tensor and hundreds of small ones fill the GPU alike.  235M parameters in 32 bits, bf16 gradients and copies: 1.10-1.12 ms, 5.9 TB/s.
//
// 8 bits: 256 consecutive elements of a tensor share a scale.  The first moment m is kept as e4m3 times (largest |m| / 448); the
// second as the e4m3 of its square root, so that its range is that of the gradients and not of their squares, and never rounded
// down to zero (a zero there would turn the next step of a parameter into one of size m / eps).  A warp has a block of 256: eight
// elements a lane, the largest found by one reduction instruction.  204M parameters: 692 us, 5.0 TB/s, 65 % of the issue slots.
#include <algorithm>
#include <cmath>

#include <cuda_fp8.h>

#include "ccl_act.cuh"
#include "ccl_launch.cuh"
#include "ccl_tma.h"

namespace ccl {

bool device_units(int* sms, int* pairs);                 // ccl_gemm.cu

constexpr int kAdamThreads = 256;
constexpr int kPiece = 4096;                             // elements of a piece: 16 a thread, 16 blocks of 256
constexpr int kBlock = 256;                              // elements that share a scale
constexpr float kF8Max = 448.0f;
constexpr float kDropped = 1e-30f;                       // a block whose largest state is smaller is kept as zeros (its scale's reciprocal could overflow)
constexpr int kFew = 40, kMost = 400;                    // tensors of a launch: parameter blocks of 3 KB and of 29 KB (32764 bytes is the limit)

struct AdamTensor {
    float* p;
    uint16_t* copy;
    const void* g;
    void *m, *v;
    float *ms, *vs;
    int64_t n;
};
struct AdamScalars {                                     // (see the header's formulas)
    float b1, b1c, b2, b2c, decay, step, root, eps;
};
template <int N>
struct AdamParams {
    AdamTensor t[N];
    int32_t first[N + 1];                                // number of a tensor's first piece
    uint8_t wide[N];                                     // gradient in fp32
    uint8_t vec[N];                                      // all of its buffers allow 16-byte accesses
    int32_t count;
    AdamScalars s;
    const float *grad_scale, *lr_dev;
    const int64_t* step_dev;
    double lr, beta1, beta2, weight_decay;
};

// What depends on the rate and on the number of the step, in 64 bits, rounded once
__host__ __device__ inline void adam_scalars(double lr, double beta1, double beta2, double weight_decay, double t, AdamScalars* s) {
    s->decay = (float)(1.0 - lr * weight_decay);
    s->step = (float)(lr / (1.0 - pow(beta1, t)));
    s->root = (float)(1.0 / sqrt(1.0 - pow(beta2, t)));
}

// m and v (its root r) of the last step become this one's, p is updated
__device__ __forceinline__ void adam_element(const AdamScalars& s, float g, float& p, float& m, float& v, float& r) {
    m = __fadd_rn(__fmul_rn(m, s.b1), __fmul_rn(g, s.b1c));
    v = __fadd_rn(__fmul_rn(v, s.b2), __fmul_rn(__fmul_rn(g, s.b2c), g));
    r = __fsqrt_rn(v);
    const float d = __fdiv_rn(m, __fadd_rn(__fmul_rn(r, s.root), s.eps));
    p = __fadd_rn(__fmul_rn(p, s.decay), -__fmul_rn(d, s.step));
}

__device__ __forceinline__ float grad_at(const void* g, bool wide, int64_t i) {
    return wide ? static_cast<const float*>(g)[i] : bf16_lo(static_cast<const uint16_t*>(g)[i]);
}
// Four consecutive gradients from an aligned place on
__device__ __forceinline__ void grads4(const void* g, bool wide, int64_t i, float (&f)[4]) {
    if (wide) {
        const float4 w = *reinterpret_cast<const float4*>(static_cast<const float*>(g) + i);
        f[0] = w.x; f[1] = w.y; f[2] = w.z; f[3] = w.w;
    } else {
        const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(g) + i);
        f[0] = bf16_lo(w.x); f[1] = bf16_hi(w.x); f[2] = bf16_lo(w.y); f[3] = bf16_hi(w.y);
    }
}
__device__ __forceinline__ uint16_t bf16_of(float x) { return (uint16_t)bf16_pack(x, 0.0f); }

__device__ __forceinline__ void piece32(const AdamTensor& t, bool wide, bool vec, const AdamScalars& s, bool scaled, float scale, int64_t lo, int64_t hi) {
    float *m = static_cast<float*>(t.m), *v = static_cast<float*>(t.v);
    int64_t done = lo;
    if (vec) {
        constexpr int U = 2;                             // groups of four a thread has in flight
        done = lo + (hi - lo) / 4 * 4;
        for (int64_t i = lo + threadIdx.x * 4; i < done; i += kAdamThreads * 4 * U) {
            float4 P[U], M[U], V[U];
            float g[U][4];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t k = i + u * kAdamThreads * 4;
                if (k < done) {
                    P[u] = *reinterpret_cast<const float4*>(t.p + k);
                    M[u] = *reinterpret_cast<const float4*>(m + k);
                    V[u] = *reinterpret_cast<const float4*>(v + k);
                    grads4(t.g, wide, k, g[u]);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t k = i + u * kAdamThreads * 4;
                if (k < done) {
                    float r;
                    if (scaled)
#pragma unroll
                        for (int j = 0; j < 4; ++j) g[u][j] = __fmul_rn(g[u][j], scale);
                    adam_element(s, g[u][0], P[u].x, M[u].x, V[u].x, r);
                    adam_element(s, g[u][1], P[u].y, M[u].y, V[u].y, r);
                    adam_element(s, g[u][2], P[u].z, M[u].z, V[u].z, r);
                    adam_element(s, g[u][3], P[u].w, M[u].w, V[u].w, r);
                    *reinterpret_cast<float4*>(t.p + k) = P[u];
                    *reinterpret_cast<float4*>(m + k) = M[u];
                    *reinterpret_cast<float4*>(v + k) = V[u];
                    if (t.copy) *reinterpret_cast<uint2*>(t.copy + k) = make_uint2(bf16_pack(P[u].x, P[u].y), bf16_pack(P[u].z, P[u].w));
                }
            }
        }
    }
    for (int64_t k = done + threadIdx.x; k < hi; k += kAdamThreads) {
        float g = grad_at(t.g, wide, k), p = t.p[k], mm = m[k], vv = v[k], r;
        if (scaled) g = __fmul_rn(g, scale);
        adam_element(s, g, p, mm, vv, r);
        t.p[k] = p; m[k] = mm; v[k] = vv;
        if (t.copy) t.copy[k] = bf16_of(p);
    }
}

__device__ __forceinline__ float f8_value(uint8_t q) { return (float)*reinterpret_cast<const __nv_fp8_e4m3*>(&q); }
// Two values of 448 at most (or NaN) to e4m3, to nearest even
__device__ __forceinline__ uint32_t f8_pair(float lo, float hi) {
    uint16_t q;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %2, %1;" : "=h"(q) : "f"(lo), "f"(hi));
    return q;
}
// Largest of non-negative values over a warp (their bits are ordered as their values are, NaN above all)
__device__ __forceinline__ float warp_max(float x) { return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(x))); }
__device__ __forceinline__ float larger(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
// (an infinite top makes the whole block NaN, as a NaN does: with an infinite scale the roots kept at the least value would decode to
// infinities, and their parameters stand still without a sign of it)
__device__ __forceinline__ void f8_scale(float top, float& scale, float& inverse) {
    const bool kept = !(top < kDropped);
    scale = kept ? (top < INFINITY ? __fmul_rn(top, 1.0f / kF8Max) : __int_as_float(0x7FFFFFFF)) : 0.0f;
    inverse = kept ? __fdiv_rn(kF8Max, top) : 0.0f;
}

__device__ __forceinline__ void piece8(const AdamTensor& t, bool wide, bool vec, const AdamScalars& s, bool scaled, float scale, int64_t lo, int64_t hi) {
    uint8_t *mq = static_cast<uint8_t*>(t.m), *vq = static_cast<uint8_t*>(t.v);
    const int lane = threadIdx.x & 31;
    for (int64_t b0 = lo + (threadIdx.x >> 5) * kBlock; b0 < hi; b0 += kAdamThreads / 32 * kBlock) {
        // a lane's eight: two groups of four, 128 elements apart (a warp then reads 512 contiguous bytes of fp32 at a time)
        const bool whole = vec && b0 + kBlock <= hi;
        const int64_t block = b0 / kBlock;
        float p[8], g[8];
        uint32_t mw[2], vw[2];
        if (whole) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int64_t k = b0 + u * 128 + lane * 4;
                const float4 w = *reinterpret_cast<const float4*>(t.p + k);
                p[4 * u] = w.x; p[4 * u + 1] = w.y; p[4 * u + 2] = w.z; p[4 * u + 3] = w.w;
                float h[4];
                grads4(t.g, wide, k, h);
#pragma unroll
                for (int j = 0; j < 4; ++j) g[4 * u + j] = h[j];
                mw[u] = *reinterpret_cast<const uint32_t*>(mq + k);
                vw[u] = *reinterpret_cast<const uint32_t*>(vq + k);
            }
        } else {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                mw[u] = vw[u] = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int64_t k = b0 + u * 128 + lane * 4 + j;
                    const bool in = k < hi;
                    p[4 * u + j] = in ? t.p[k] : 0.0f;
                    g[4 * u + j] = in ? grad_at(t.g, wide, k) : 0.0f;
                    mw[u] |= (uint32_t)(in ? mq[k] : 0) << (8 * j);
                    vw[u] |= (uint32_t)(in ? vq[k] : 0) << (8 * j);
                }
            }
        }
        const float ms = t.ms[block], vs = t.vs[block];
        float m[8], r[8], top_m = 0.0f, top_r = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            m[i] = __fmul_rn(f8_value((uint8_t)(mw[i >> 2] >> (8 * (i & 3)))), ms);
            const float old = __fmul_rn(f8_value((uint8_t)(vw[i >> 2] >> (8 * (i & 3)))), vs);
            float v = __fmul_rn(old, old);
            if (scaled) g[i] = __fmul_rn(g[i], scale);
            adam_element(s, g[i], p[i], m[i], v, r[i]);
            top_m = larger(top_m, fabsf(m[i]));
            top_r = larger(top_r, r[i]);
        }
        float m_scale, m_inv, v_scale, v_inv;
        f8_scale(warp_max(top_m), m_scale, m_inv);
        f8_scale(warp_max(top_r), v_scale, v_inv);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            uint32_t q[4];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int i = 4 * u + 2 * j;
                q[j] = f8_pair(__fmul_rn(m[i], m_inv), __fmul_rn(m[i + 1], m_inv));
                q[2 + j] = f8_pair(__fmul_rn(r[i], v_inv), __fmul_rn(r[i + 1], v_inv));
                if ((q[2 + j] & 0xffu) == 0 && r[i] > 0.0f) q[2 + j] |= 1u;              // the least value there is, not zero
                if ((q[2 + j] & 0xff00u) == 0 && r[i + 1] > 0.0f) q[2 + j] |= 0x100u;
            }
            mw[u] = q[0] | q[1] << 16;
            vw[u] = q[2] | q[3] << 16;
        }
        if (whole) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int64_t k = b0 + u * 128 + lane * 4;
                *reinterpret_cast<float4*>(t.p + k) = make_float4(p[4 * u], p[4 * u + 1], p[4 * u + 2], p[4 * u + 3]);
                *reinterpret_cast<uint32_t*>(mq + k) = mw[u];
                *reinterpret_cast<uint32_t*>(vq + k) = vw[u];
                if (t.copy) *reinterpret_cast<uint2*>(t.copy + k) = make_uint2(bf16_pack(p[4 * u], p[4 * u + 1]), bf16_pack(p[4 * u + 2], p[4 * u + 3]));
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int64_t k = b0 + (i >> 2) * 128 + lane * 4 + (i & 3);
                if (k < hi) {
                    t.p[k] = p[i];
                    mq[k] = (uint8_t)(mw[i >> 2] >> (8 * (i & 3)));
                    vq[k] = (uint8_t)(vw[i >> 2] >> (8 * (i & 3)));
                    if (t.copy) t.copy[k] = bf16_of(p[i]);
                }
            }
        }
        if (lane == 0) { t.ms[block] = m_scale; t.vs[block] = v_scale; }
    }
}

template <int N, bool EIGHT>
__global__ void __launch_bounds__(kAdamThreads, 4) adamw_kernel(const __grid_constant__ AdamParams<N> a) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ int first[N + 1];
    __shared__ AdamScalars shared_scalars;
    for (int i = threadIdx.x; i <= a.count; i += kAdamThreads) first[i] = a.first[i];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (threadIdx.x == 0) {
        AdamScalars s = a.s;
        if (a.step_dev || a.lr_dev)                      // the rate or the step's number as they are when the kernel runs (a captured step)
            adam_scalars(a.lr_dev ? (double)*a.lr_dev : a.lr, a.beta1, a.beta2, a.weight_decay, (double)*a.step_dev, &s);
        shared_scalars = s;
    }
    __syncthreads();
    const AdamScalars s = shared_scalars;
    const bool scaled = a.grad_scale != nullptr;
    const float scale = scaled ? *a.grad_scale : 1.0f;
    for (int piece = blockIdx.x; piece < first[a.count]; piece += gridDim.x) {
        int lo = 0, hi = a.count;                        // the last tensor whose first piece is not behind this one (none is empty)
        while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (first[mid] <= piece) lo = mid; else hi = mid; }
        const AdamTensor& t = a.t[lo];
        const int64_t from = (int64_t)(piece - first[lo]) * kPiece, to = min(t.n, from + kPiece);
        if (EIGHT) piece8(t, a.wide[lo], a.vec[lo], s, scaled, scale, from, to);
        else piece32(t, a.wide[lo], a.vec[lo], s, scaled, scale, from, to);
    }
}

namespace {

uintptr_t bits(const void* p) { return reinterpret_cast<uintptr_t>(p); }

template <int N>
ccl_status run_adamw(const ccl_adamw_desc* d, const ccl_adamw_tensor* tensors, int count, cudaStream_t st) {
    int sms, pairs;
    device_units(&sms, &pairs);
    static thread_local AdamParams<N> a;                 // (29 KB: not on a caller's stack)
    a.s = AdamScalars{(float)d->beta1, (float)(1.0 - d->beta1), (float)d->beta2, (float)(1.0 - d->beta2), 0.0f, 0.0f, 0.0f, (float)d->eps};
    a.grad_scale = d->grad_scale_dev; a.lr_dev = d->lr_dev; a.step_dev = d->step_dev;
    a.lr = d->lr; a.beta1 = d->beta1; a.beta2 = d->beta2; a.weight_decay = d->weight_decay;
    if (!d->step_dev) adam_scalars(d->lr, d->beta1, d->beta2, d->weight_decay, (double)d->step, &a.s);
    const bool eight = d->state_bits == 8;
    for (int i = 0; i < count;) {
        int64_t pieces = 0;
        a.count = 0;
        for (; i < count && a.count < N; ++i) {
            const ccl_adamw_tensor& t = tensors[i];
            if (t.n == 0) continue;
            const int64_t mine = (t.n + kPiece - 1) / kPiece;
            if (a.count && pieces + mine > (INT64_C(1) << 30)) break;        // (the numbers of a launch's pieces are 32 bits)
            AdamTensor& o = a.t[a.count];
            o = AdamTensor{t.param, static_cast<uint16_t*>(t.param_bf16), t.grad, t.m, t.v, t.m_scale, t.v_scale, t.n};
            a.first[a.count] = (int32_t)pieces;
            a.wide[a.count] = t.grad_fp32 != 0;
            uintptr_t align = bits(t.param) | bits(t.param_bf16) << 1 | bits(t.grad) << (t.grad_fp32 ? 0 : 1);
            align |= eight ? (bits(t.m) | bits(t.v)) << 2 : bits(t.m) | bits(t.v);
            a.vec[a.count] = (align & 15) == 0;
            pieces += mine;
            ++a.count;
        }
        if (!a.count) break;
        a.first[a.count] = (int32_t)pieces;
        ccl_status s = launch_early(eight ? adamw_kernel<N, true> : adamw_kernel<N, false>, dim3((unsigned)std::min(a.first[a.count], sms * 4)), kAdamThreads, 0, st, a);
        if (s) return s;
    }
    return CCL_OK;
}

}  // namespace
}  // namespace ccl

using namespace ccl;

extern "C" ccl_status ccl_adamw(const ccl_adamw_desc* d, const ccl_adamw_tensor* tensors, int32_t count, void* cuda_stream) {
    if (!d || count < 0 || (count && !tensors)) return fail(CCL_ERR_INVALID_ARG, "ccl_adamw: NULL argument or negative count");
    if (d->state_bits != 32 && d->state_bits != 8) return fail(CCL_ERR_UNSUPPORTED, "ccl_adamw: states of %d bits (32 or 8 are taken)", d->state_bits);
    const double big = 1e30;
    if (!(d->lr >= 0 && d->lr < big) || !(d->beta1 >= 0 && d->beta1 < 1) || !(d->beta2 >= 0 && d->beta2 < 1) || !(d->eps > 0 && (float)d->eps > 0.0f && d->eps < big) ||
        !(d->weight_decay >= 0 && d->weight_decay < big))
        return fail(CCL_ERR_INVALID_ARG, "ccl_adamw: lr and weight_decay must be numbers >= 0, beta1 and beta2 in [0, 1), eps > 0");
    if (!d->step_dev && (d->step < 1 || d->lr_dev)) return fail(CCL_ERR_INVALID_ARG, "ccl_adamw: step must be at least 1 (lr_dev goes with step_dev)");
    if ((bits(d->grad_scale_dev) | bits(d->lr_dev)) & 3 || bits(d->step_dev) & 7) return fail(CCL_ERR_ALIGN, "ccl_adamw: a scalar's pointer is not aligned to its type");
    for (int i = 0; i < count; ++i) {
        const ccl_adamw_tensor& t = tensors[i];
        if (t.n < 0) return fail(CCL_ERR_INVALID_ARG, "ccl_adamw: tensor %d: negative size", i);
        if (t.n == 0) continue;
        if (t.n > (INT64_C(1) << 40)) return fail(CCL_ERR_UNSUPPORTED, "ccl_adamw: tensor %d is too large", i);
        if (!t.param || !t.grad || !t.m || !t.v) return fail(CCL_ERR_INVALID_ARG, "ccl_adamw: tensor %d: NULL buffer", i);
        if (d->state_bits == 8 && (!t.m_scale || !t.v_scale)) return fail(CCL_ERR_INVALID_ARG, "ccl_adamw: tensor %d: 8-bit states need their scales", i);
        uintptr_t four = bits(t.param) | (t.grad_fp32 ? bits(t.grad) : 0);
        four |= d->state_bits == 8 ? bits(t.m_scale) | bits(t.v_scale) : bits(t.m) | bits(t.v);
        if (four & 3 || (bits(t.grad) | bits(t.param_bf16)) & 1) return fail(CCL_ERR_ALIGN, "ccl_adamw: tensor %d: a buffer is not aligned to its type", i);
    }
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    return count <= kFew ? run_adamw<kFew>(d, tensors, count, st) : run_adamw<kMost>(d, tensors, count, st);
}
