// ccl_bias_act_grad: dZ = dY * act'(Z) and dbias[n] = sum over the rows of dZ, in one pass and one launch.
//
// Bound by memory: dY and Z are read once, dZ is written once, the sums never leave the chip.  A cluster of up to eight CTAs
// owns a strip of columns and shares its rows; every thread keeps the fp32 sums of its (eight) columns in registers, the CTA's
// row lanes meet in shared memory and the CTAs of the cluster in distributed shared memory, in a fixed order: the same bits on
// every run, no workspace, no second launch, no atomics.
#include <algorithm>

#include "ccl_act.cuh"
#include "ccl_tma.h"

namespace ccl {

constexpr int kBiasThreads = 256;

struct BiasGradParams {
    MatView v;
    const uint16_t *dy, *z;
    uint16_t *dz, *dbias;
    int32_t lanes;              // threads side by side along a row (a power of two); the others take other rows
    int64_t rows_per_cta;
};

// A thread's columns of a row as bf16 pairs (VEC = 1: one value, the other zero)
template <int VEC>
__device__ __forceinline__ void load_cols(const uint16_t* p, uint32_t (&v)[(VEC + 1) / 2]) {
    if constexpr (VEC == 8) {
        const uint4 w = *reinterpret_cast<const uint4*>(p);
        v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w;
    } else v[0] = *p;
}

// VEC: columns of a thread: 8 (16-byte accesses) or 1.  LINEAR: a column strip's rows follow each other at one pitch (row-major
// and CCL split along the columns); otherwise every element is looked up in the address map.
template <int ACT, int VEC, bool LINEAR>
__global__ void __launch_bounds__(kBiasThreads, 4) bias_act_grad_kernel(const BiasGradParams p) {
    __shared__ float part[kBiasThreads * VEC];
    uint32_t rank, ctas;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(ctas));
    const int L = p.lanes, R = kBiasThreads / L, lx = threadIdx.x & (L - 1), ly = threadIdx.x / L;
    const int64_t tile = blockIdx.x / ctas, col = (tile * L + lx) * VEC;
    const bool col_ok = col < p.v.cols;
    constexpr int PR = (VEC + 1) / 2;
    f32x2 sum2[PR];
#pragma unroll
    for (int i = 0; i < PR; ++i) sum2[i] = both(0.0f);
    if (col_ok) {
        const int64_t r1 = min(p.v.rows, (int64_t)(rank + 1) * p.rows_per_cta);
        int64_t r = (int64_t)rank * p.rows_per_cta + ly;
        const int64_t base = LINEAR ? map(p.v, 0, col) : 0, pitch = p.v.split == 2 ? strip_w_of(p.v, col / p.v.w) : p.v.cols;
        auto at = [&](int64_t row) { return LINEAR ? base + row * pitch : map(p.v, row, col); };
        // U rows at a time: their loads are all in flight before the first is used
        constexpr int U = 4;
        for (; r < r1; r += (int64_t)U * R) {
            uint32_t g[U][PR], z[U][PR];
            int64_t off[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t row = min(r + (int64_t)u * R, r1 - 1);
                off[u] = at(row);
                load_cols<VEC>(p.dy + off[u], g[u]);
                if (ACT != CCL_ACT_NONE) load_cols<VEC>(p.z + off[u], z[u]);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (r + (int64_t)u * R >= r1) break;
                f32x2 d[PR];
#pragma unroll
                for (int i = 0; i < PR; ++i) {
                    d[i] = bf16_unpack(g[u][i]);
                    if (ACT != CCL_ACT_NONE) d[i] = d[i] * act_slope<ACT>(z[u][i]);
                    sum2[i] = sum2[i] + d[i];
                }
                if (p.dz) {
                    if constexpr (VEC == 8) *reinterpret_cast<uint4*>(p.dz + off[u]) = bf16x8_pack(d);
                    else p.dz[off[u]] = (uint16_t)bf16_pack(d[0]);
                }
            }
        }
    }
    if (!p.dbias) return;                                // (the same for every CTA)
    const int cols = L * VEC;
    float sum[2 * PR];
#pragma unroll
    for (int i = 0; i < PR; ++i) split(sum2[i], sum[2 * i], sum[2 * i + 1]);
#pragma unroll
    for (int i = 0; i < VEC; ++i) part[ly * cols + lx * VEC + i] = sum[i];
    __syncthreads();
    float s = 0.0f;
    if ((int)threadIdx.x < cols)
        for (int y = 0; y < R; ++y) s += part[y * cols + threadIdx.x];
    __syncthreads();
    if ((int)threadIdx.x < cols) part[threadIdx.x] = s;
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (rank == 0 && (int)threadIdx.x < cols) {
        for (uint32_t k = 1; k < ctas; ++k) {
            uint32_t remote;
            float x;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(smem_u32(&part[threadIdx.x])), "r"(k));
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(remote) : "memory");
            s += x;
        }
        const int64_t n = tile * cols + threadIdx.x;
        if (n < p.v.cols) reinterpret_cast<__nv_bfloat16*>(p.dbias)[n] = __float2bfloat16_rn(s);
    }
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");   // the sums of a CTA stay until CTA 0 has read them
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

template <int ACT>
static ccl_status launch_bias_grad(const BiasGradParams& p, bool vec, bool linear, unsigned grid, int ctas, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid, 1, 1);
    cfg.blockDim = dim3(kBiasThreads, 1, 1);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)ctas; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    auto kernel = vec ? (linear ? bias_act_grad_kernel<ACT, 8, true> : bias_act_grad_kernel<ACT, 8, false>)
                      : (linear ? bias_act_grad_kernel<ACT, 1, true> : bias_act_grad_kernel<ACT, 1, false>);
    CCL_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, p));
    count_launch();
    return CCL_OK;
}

}  // namespace ccl

using namespace ccl;

extern "C" ccl_status ccl_bias_act_grad(const ccl_mat* m, int32_t act, const void* dY_dev, const void* Z_dev, void* dZ_dev, void* dbias_dev,
                                        void* cuda_stream) {
    BiasGradParams p;
    ccl_status s = make_view(m, "ccl_bias_act_grad", &p.v);
    if (s) return s;
    if (act < CCL_ACT_NONE || act > CCL_ACT_SILU) return fail(CCL_ERR_INVALID_ARG, "ccl_bias_act_grad: unknown activation %d", act);
    if (!dY_dev || (act != CCL_ACT_NONE && !Z_dev)) return fail(CCL_ERR_INVALID_ARG, "ccl_bias_act_grad: NULL operand");
    if (!dZ_dev && !dbias_dev) return fail(CCL_ERR_INVALID_ARG, "ccl_bias_act_grad: neither dZ nor dbias is wanted");
    if (p.v.e != 2) return fail(CCL_ERR_UNSUPPORTED, "ccl_bias_act_grad: only 2-byte (bf16) elements are supported");
    const uintptr_t any = reinterpret_cast<uintptr_t>(dY_dev) | reinterpret_cast<uintptr_t>(act != CCL_ACT_NONE ? Z_dev : nullptr) | reinterpret_cast<uintptr_t>(dZ_dev);
    if ((any | reinterpret_cast<uintptr_t>(dbias_dev)) & 1) return fail(CCL_ERR_ALIGN, "ccl_bias_act_grad: a base pointer is not 2-byte aligned");
    p.dy = static_cast<const uint16_t*>(dY_dev); p.z = static_cast<const uint16_t*>(Z_dev);
    p.dz = static_cast<uint16_t*>(dZ_dev); p.dbias = static_cast<uint16_t*>(dbias_dev);
    const MatView& v = p.v;
    // eight columns at a time where every group of eight is one aligned 16-byte piece of the buffer
    const bool vec = (any & 15) == 0 && v.cols % 8 == 0 && (v.split != 2 || (v.w % 8 == 0 && v.wlast % 8 == 0)) && v.stride % 8 == 0 && v.ichunk % 8 == 0;
    const bool linear = !v.ichunk && v.split != 1;
    const int64_t groups = vec ? v.cols / 8 : v.cols;    // threads needed for one row
    // As many threads along a row as leave every SM three CTAs or more (four fit at a time): 16 of them read 256 contiguous bytes
    int lanes = 32, ctas = 8;
    while (ctas > 1 && v.rows < (int64_t)ctas * 32) ctas /= 2;
    while (lanes > 2 && (groups + lanes - 1) / lanes * ctas < 148 * 3) lanes /= 2;
    const int64_t tiles = (groups + lanes - 1) / lanes;
    if (tiles * ctas >= (INT64_C(1) << 31)) return fail(CCL_ERR_UNSUPPORTED, "ccl_bias_act_grad: too many columns");
    p.lanes = lanes;
    p.rows_per_cta = (v.rows + ctas - 1) / ctas;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    const unsigned grid = (unsigned)(tiles * ctas);
    switch (act) {
        case CCL_ACT_NONE: return launch_bias_grad<CCL_ACT_NONE>(p, vec, linear, grid, ctas, st);
        case CCL_ACT_RELU: return launch_bias_grad<CCL_ACT_RELU>(p, vec, linear, grid, ctas, st);
        case CCL_ACT_GELU_TANH: return launch_bias_grad<CCL_ACT_GELU_TANH>(p, vec, linear, grid, ctas, st);
        case CCL_ACT_GELU_ERF: return launch_bias_grad<CCL_ACT_GELU_ERF>(p, vec, linear, grid, ctas, st);
        default: return launch_bias_grad<CCL_ACT_SILU>(p, vec, linear, grid, ctas, st);
    }
}
