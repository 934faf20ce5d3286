// ccl_norm: y = (x - mean) / sqrt(var + eps) * gamma + beta of every row (or x / sqrt(mean of squares + eps) * gamma), and
// ccl_norm_grad: the gradients of x, gamma and beta.
//
// Bound by memory: a row is read once into registers, its statistics are taken from there and the result is written from there.  The
// variance is the mean square about a mean: about the warp's own one first, and the warps' moments are then joined with
//   var = sum of var_w + n_w / H (mean_w - mean)^2          (var_w: a warp's share of the mean square about its own mean)
// so that one meeting of a row's warps is enough and a mean far from zero costs no digits (a difference of E x^2 and (E x)^2 would).
// The gradients of gamma and beta are sums over the rows, in a fixed order, without atomics: the same bits on every run.
//
// Three ways, by size and alignment (plan_norm).  Many rows in aligned 16-byte pieces: bulk copies into shared memory keep the loads under way
// (norm_rows_kernel, norm_grad_stream_kernel).  Few rows, odd widths, other layouts: rows through registers.  Rows longer than a CTA's
// registers hold: read again from the L2.
#include <algorithm>
#include <atomic>

#include "ccl_act.cuh"
#include "ccl_launch.cuh"
#include "ccl_tma.h"

namespace ccl {

bool device_units(int* sms, int* pairs);                 // ccl_gemm.cu

struct NormParams {
    MatView v;
    const uint16_t *x, *dy, *addend, *gamma, *beta;
    uint16_t* out;                  // y or dx (may be one of the inputs: an element is written by the thread that has read it)
    float *mean, *rstd;             // written by ccl_norm, read by ccl_norm_grad
    float* partial;                 // norm_grad_stream_kernel: [CTAs][2][cols] sums for gamma and beta, or NULL
    int32_t layer;                  // 1: about the row's mean, 0: about zero
    float eps, inv_cols;
    int32_t lanes;                  // threads of a row
};

template <int VEC>
__device__ __forceinline__ void load_vec(const uint16_t* p, uint32_t (&v)[(VEC + 1) / 2]) {
    if constexpr (VEC == 8) {
        const uint4 w = *reinterpret_cast<const uint4*>(p);
        v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w;
    } else v[0] = *p;
}
template <int VEC>
__device__ __forceinline__ void load_weights(const uint16_t* p, int64_t col, float none, float (&f)[VEC]) {
    if (!p) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) f[i] = none;
        return;
    }
    if constexpr (VEC == 8) {
        const uint4 w = __ldg(reinterpret_cast<const uint4*>(p + col));
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[2 * i] = bf16_lo(u[i]); f[2 * i + 1] = bf16_hi(u[i]); }
    } else f[0] = bf16_lo(__ldg(p + col));
}
template <int VEC>
__device__ __forceinline__ void unpack(const uint32_t (&v)[(VEC + 1) / 2], float (&f)[VEC]) {
#pragma unroll
    for (int i = 0; i < (VEC + 1) / 2; ++i) {
        f[2 * i] = bf16_lo(v[i]);
        if (VEC > 1) f[2 * i + (VEC > 1)] = bf16_hi(v[i]);
    }
}
template <int VEC>
__device__ __forceinline__ void store_vec(uint16_t* p, const float (&f)[VEC]) {
    if constexpr (VEC == 8) *reinterpret_cast<uint4*>(p) = make_uint4(bf16_pack(f[0], f[1]), bf16_pack(f[2], f[3]), bf16_pack(f[4], f[5]), bf16_pack(f[6], f[7]));
    else *p = (uint16_t)bf16_pack(f[0], 0.0f);
}
// Sum over the `lanes` (a power of two, 32 at most) threads of a row that share a warp
__device__ __forceinline__ float lanes_sum(float s, int lanes) {
    for (int w = lanes >> 1; w >= 1; w >>= 1) s += __shfl_xor_sync(0xffffffffu, s, w);
    return s;
}

// A thread's NV groups of VEC columns: where they are in the row it works on and how far the next row is.  LINEAR: a column strip's rows
// follow each other at one pitch (row-major and CCL split along the columns); otherwise every group is looked up in the address map.
template <int VEC, int NV, bool LINEAR>
struct RowCursor {
    int64_t off[NV], step[NV];
    int64_t row;
    __device__ RowCursor(const NormParams& p, int lane, int64_t row0, int64_t stride) : row(row0) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int64_t col = min(column(p, lane, i), p.v.cols - VEC);
            off[i] = 0; step[i] = stride;
            if (LINEAR) {
                const int64_t pitch = p.v.split == 2 ? strip_w_of(p.v, col / p.v.w) : p.v.cols;
                off[i] = map(p.v, 0, col) + row0 * pitch;
                step[i] = stride * pitch;
            }
        }
    }
    __device__ static int64_t column(const NormParams& p, int lane, int i) { return ((int64_t)i * p.lanes + lane) * VEC; }
    __device__ int64_t at(const NormParams& p, int lane, int i) const { return LINEAR ? off[i] : map(p.v, row, column(p, lane, i)); }
    __device__ void next(int64_t stride) {
        row += stride;
        if (LINEAR)
#pragma unroll
            for (int i = 0; i < NV; ++i) off[i] += step[i];
    }
};

// ONE: a row's threads lie in one warp (several rows in a CTA side by side); otherwise the CTA has one row at a time
template <int VEC, int NV, bool LINEAR, bool ONE>
__global__ void __launch_bounds__(ONE ? 256 : 1024) norm_kernel(const __grid_constant__ NormParams p) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ float2 moments[2][32];
    __shared__ float counts[32];
    const int lanes = p.lanes, lane = ONE ? threadIdx.x & (lanes - 1) : threadIdx.x, warp = threadIdx.x >> 5, wl = threadIdx.x & 31, warps = blockDim.x >> 5;
    const int64_t rows_at_once = ONE ? blockDim.x / lanes : 1, stride = gridDim.x * rows_at_once;
    RowCursor<VEC, NV, LINEAR> cur(p, lane, blockIdx.x * rows_at_once + (ONE ? threadIdx.x / lanes : 0), stride);
    bool mine[NV];
    float n_warp = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        mine[i] = cur.column(p, lane, i) < p.v.cols;
        n_warp += mine[i] ? (float)VEC : 0.0f;
    }
    if (!ONE) {
        n_warp = lanes_sum(n_warp, 32);
        if ((threadIdx.x & 31) == 0) counts[warp] = n_warp;
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    uint32_t nx[NV][(VEC + 1) / 2];
    auto fetch = [&]() {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int j = 0; j < (VEC + 1) / 2; ++j) nx[i][j] = 0;
            if (mine[i] && cur.row < p.v.rows) load_vec<VEC>(p.x + cur.at(p, lane, i), nx[i]);
        }
    };
    fetch();
    int turn = 0;
    // (ONE: the rows of a warp end together, so that its shuffles stay whole)
    for (int64_t first = blockIdx.x * rows_at_once; first < p.v.rows; first += stride, turn ^= 1) {
        const int64_t row = cur.row;
        int64_t to[NV];
        float f[NV][VEC];
#pragma unroll
        for (int i = 0; i < NV; ++i) { to[i] = row < p.v.rows && mine[i] ? cur.at(p, lane, i) : 0; unpack<VEC>(nx[i], f[i]); }
        cur.next(stride);
        fetch();
        float s = 0.0f, mean = 0.0f, m2 = 0.0f;
        if (p.layer) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < VEC; ++j) s += f[i][j];
            s = lanes_sum(s, ONE ? lanes : 32);
            mean = ONE ? s * p.inv_cols : (n_warp > 0.0f ? s / n_warp : 0.0f);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float d = mine[i] ? f[i][j] - mean : 0.0f;
                m2 = fmaf(d * p.inv_cols, d, m2);        // (a mean as it grows: a sum of H squares could leave fp32 where their mean does not)
            }
        m2 = lanes_sum(m2, ONE ? lanes : 32);
        if (!ONE) {                                      // (a lane a warp: its mean, its share of the variance, its share of the values)
            if (wl == 0) moments[turn][warp] = make_float2(mean, m2);
            __syncthreads();
            const float2 o = wl < warps ? moments[turn][wl] : make_float2(0.0f, 0.0f);
            const float n = wl < warps ? counts[wl] * p.inv_cols : 0.0f;
            mean = p.layer ? lanes_sum(n * o.x, 32) : 0.0f;
            m2 = lanes_sum(fmaf(n * (o.x - mean), o.x - mean, o.y), 32);
        }
        const float rstd = rsqrtf(m2 + p.eps);
        if (row < p.v.rows) {
            if (lane == 0) {
                if (p.mean) p.mean[row] = mean;
                if (p.rstd) p.rstd[row] = rstd;
            }
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (mine[i]) {
                    float g[VEC], b[VEC];
                    load_weights<VEC>(p.gamma, cur.column(p, lane, i), 1.0f, g);
                    load_weights<VEC>(p.beta, cur.column(p, lane, i), 0.0f, b);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) f[i][j] = fmaf((f[i][j] - mean) * rstd, g[j], b[j]);
                    store_vec<VEC>(p.out + to[i], f[i]);
                }
        }
    }
}

template <int VEC, int NV, bool LINEAR, bool ONE>
__global__ void __launch_bounds__(ONE ? 256 : 1024) norm_grad_kernel(const __grid_constant__ NormParams p) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ float2 sums[2][32];
    const int lanes = p.lanes, lane = ONE ? threadIdx.x & (lanes - 1) : threadIdx.x, warp = threadIdx.x >> 5, wl = threadIdx.x & 31, warps = blockDim.x >> 5;
    const int64_t rows_at_once = ONE ? blockDim.x / lanes : 1, stride = gridDim.x * rows_at_once;
    RowCursor<VEC, NV, LINEAR> cur(p, lane, blockIdx.x * rows_at_once + (ONE ? threadIdx.x / lanes : 0), stride);
    bool mine[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) mine[i] = cur.column(p, lane, i) < p.v.cols;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    constexpr int PR = (VEC + 1) / 2;
    int turn = 0;
    for (int64_t first = blockIdx.x * rows_at_once; first < p.v.rows; first += stride, turn ^= 1) {
        const int64_t row = cur.row;
        const bool live = row < p.v.rows;
        const float rstd = live ? p.rstd[row] : 0.0f, mean = live && p.layer ? p.mean[row] : 0.0f;
        int64_t to[NV];
        uint32_t ad[NV][PR], x[NV][PR], y[NV][PR];
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            to[i] = live && mine[i] ? cur.at(p, lane, i) : 0;
#pragma unroll
            for (int j = 0; j < PR; ++j) x[i][j] = y[i][j] = ad[i][j] = 0;
            if (live && mine[i]) {
                load_vec<VEC>(p.x + to[i], x[i]);
                load_vec<VEC>(p.dy + to[i], y[i]);
                if (p.addend) load_vec<VEC>(p.addend + to[i], ad[i]);
            }
        }
        cur.next(stride);
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (mine[i]) {
                float f[VEC], d[VEC], g[VEC];
                unpack<VEC>(x[i], f);
                unpack<VEC>(y[i], d);
                load_weights<VEC>(p.gamma, cur.column(p, lane, i), 1.0f, g);
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    s1 = fmaf(d[j], g[j], s1);
                    s2 = fmaf(d[j] * g[j], (f[j] - mean) * rstd, s2);
                }
            }
        s1 = lanes_sum(s1, ONE ? lanes : 32);
        s2 = lanes_sum(s2, ONE ? lanes : 32);
        if (!ONE) {
            if (wl == 0) sums[turn][warp] = make_float2(s1, s2);
            __syncthreads();
            const float2 o = wl < warps ? sums[turn][wl] : make_float2(0.0f, 0.0f);
            s1 = lanes_sum(o.x, 32);
            s2 = lanes_sum(o.y, 32);
        }
        s1 = p.layer ? s1 * p.inv_cols : 0.0f;
        s2 *= p.inv_cols;
        if (live)
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (mine[i]) {
                    float f[VEC], d[VEC], g[VEC], a[VEC];
                    unpack<VEC>(x[i], f);
                    unpack<VEC>(y[i], d);
                    unpack<VEC>(ad[i], a);
                    load_weights<VEC>(p.gamma, cur.column(p, lane, i), 1.0f, g);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const float h = (f[j] - mean) * rstd;
                        f[j] = fmaf(rstd, fmaf(-h, s2, fmaf(d[j], g[j], -s1)), a[j]);
                    }
                    store_vec<VEC>(p.out + to[i], f);
                }
    }
}

// dgamma and dbeta where the rows' kernel leaves them (few rows, rows of odd widths or layouts): a cluster of up to eight CTAs owns a strip of
// columns and shares its rows; a thread keeps the sums of its (eight) columns, the CTA's row lanes meet in shared memory and the cluster's
// CTAs in distributed shared memory, in a fixed order.  x and dy are read once more, from the L2 where they fit it.
template <int VEC, bool LINEAR>
__global__ void __launch_bounds__(256) norm_sums_kernel(const __grid_constant__ NormParams p, uint16_t* dgamma, uint16_t* dbeta, int64_t rows_per_cta) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ float part[2][256 * VEC];                 // [warp][column]
    uint32_t rank, ctas;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(ctas));
    const int L = p.lanes, R = 256 / L, lx = threadIdx.x & (L - 1), ly = threadIdx.x / L;
    const int64_t tile = blockIdx.x / ctas, col = (tile * L + lx) * VEC;
    const bool col_ok = col < p.v.cols;
    float dg[VEC], db[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) dg[i] = db[i] = 0.0f;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (col_ok) {
        const int64_t r1 = min(p.v.rows, (int64_t)(rank + 1) * rows_per_cta);
        const int64_t base = LINEAR ? map(p.v, 0, col) : 0, pitch = p.v.split == 2 ? strip_w_of(p.v, col / p.v.w) : p.v.cols;
        constexpr int U = VEC == 8 ? 2 : 8;              // rows whose loads are all in flight before the first is used
        for (int64_t r = (int64_t)rank * rows_per_cta + ly; r < r1; r += (int64_t)U * R) {
            uint32_t x[U][(VEC + 1) / 2], y[U][(VEC + 1) / 2];
            float mean[U], rstd[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t row = min(r + (int64_t)u * R, r1 - 1), at = LINEAR ? base + row * pitch : map(p.v, row, col);
                load_vec<VEC>(p.x + at, x[u]);
                load_vec<VEC>(p.dy + at, y[u]);
                rstd[u] = p.rstd[row];
                mean[u] = p.layer ? p.mean[row] : 0.0f;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (r + (int64_t)u * R >= r1) break;
                float f[VEC], d[VEC];
                unpack<VEC>(x[u], f);
                unpack<VEC>(y[u], d);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    dg[i] = fmaf(d[i], (f[i] - mean[u]) * rstd[u], dg[i]);
                    db[i] += d[i];
                }
            }
        }
    }
    // the row lanes of a warp by exchanges, the eight warps in shared memory, the cluster's CTAs in distributed shared memory
    for (int w = L; w < 32; w <<= 1)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            dg[i] += __shfl_xor_sync(0xffffffffu, dg[i], w);
            db[i] += __shfl_xor_sync(0xffffffffu, db[i], w);
        }
    const int cols = L * VEC, warp = threadIdx.x >> 5;
    if ((int)(threadIdx.x & 31) < L)
#pragma unroll
        for (int i = 0; i < VEC; ++i) { part[0][warp * cols + lx * VEC + i] = dg[i]; part[1][warp * cols + lx * VEC + i] = db[i]; }
    __syncthreads();
    float s[2] = {0.0f, 0.0f};
    if ((int)threadIdx.x < cols)
#pragma unroll
        for (int y = 0; y < 8; ++y) { s[0] += part[0][y * cols + threadIdx.x]; s[1] += part[1][y * cols + threadIdx.x]; }
    __syncthreads();
    if ((int)threadIdx.x < cols) { part[0][threadIdx.x] = s[0]; part[1][threadIdx.x] = s[1]; }
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (rank == 0 && (int)threadIdx.x < cols) {
        const int64_t n = tile * cols + threadIdx.x;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            uint16_t* out = k ? dbeta : dgamma;
            float x[7];
#pragma unroll
            for (uint32_t c = 1; c < 8; ++c) {           // (all on their way before the first is added)
                uint32_t remote;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(smem_u32(&part[k][threadIdx.x])), "r"(c < ctas ? c : 0u));
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x[c - 1]) : "r"(remote));
            }
#pragma unroll
            for (uint32_t c = 1; c < 8; ++c) s[k] += c < ctas ? x[c - 1] : 0.0f;
            if (out && n < p.v.cols) reinterpret_cast<__nv_bfloat16*>(out)[n] = __float2bfloat16_rn(s[k]);
        }
    }
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");   // the sums of a CTA stay until CTA 0 has read them
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// ---- many rows whose column groups are aligned 16-byte pieces (row-major and CCL split along the columns) -------------------
//
// Loads are bulk copies into shared memory, under way whatever the warps are doing, one copy for each strip of a set of rows.

static __device__ int g_norm_status = 0;

__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(smem_u32(dst)), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void group_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ uint4 shared16(const void* p) { return *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ void parts(const uint4& w, f32x2 (&f)[4]) { f[0] = bf16_unpack(w.x); f[1] = bf16_unpack(w.y); f[2] = bf16_unpack(w.z); f[3] = bf16_unpack(w.w); }
__device__ __forceinline__ float warp_total(f32x2 a) { float lo, hi; split(a, lo, hi); return lanes_sum(lo + hi, 32); }

constexpr uint16_t kOne = 0x3F80;                        // 1 in bf16

// PHASED: rows of a row-major matrix whose width is no multiple of 8.  A row then starts anywhere in a 16-byte piece, but rows `period` apart start
// at the same place, and a CTA takes only such rows (blockIdx mod period, and every period-th from there on): with its `phase` as a constant every
// thread keeps its columns, whole 16-byte pieces are moved, and only a row's first and last piece are looked at element by element.
struct StreamParams {
    NormParams n;
    int32_t groups, slots, arrays, set_rows, period, pieces;        // pieces: of 8 elements, room for a row
    uint32_t slot_bytes, array_bytes;
};

// A row of a PHASED set: its pieces to shared memory; what lies in the buffer's last, incomplete piece element by element.  Returns the bytes of
// the bulk copy (the caller announces them; the single elements are written before it does).
__device__ __forceinline__ uint32_t phased_bytes(const MatView& v, int64_t row, int phase, int pieces) {
    const int64_t whole = (v.rows * v.cols >> 3) - ((row * v.cols - phase) >> 3);
    return (uint32_t)min((int64_t)pieces, whole) * 16;
}
__device__ __forceinline__ void phased_tail(const MatView& v, const uint16_t* src, int64_t row, int phase, int pieces, uint16_t* to) {
    const int64_t at = row * v.cols - phase, total = v.rows * v.cols;
    for (int64_t k = total & ~INT64_C(7); k < total && k < at + pieces * 8; ++k) to[k - at] = src[k];
}
// Elements of piece i that belong to a row of `cols` columns: [first, last) of 0..8
__device__ __forceinline__ bool phased_edge(int i, int phase, int cols, int& first, int& last) {
    first = phase - i * 8;
    last = phase + cols - i * 8;
    return first > 0 || last < 8;
}
// Eight results to an aligned place; of a row's first and last piece the row's own elements alone
__device__ __forceinline__ void store_piece(uint16_t* to, const uint4& w, bool edge, int i, int phase, int cols) {
    int first, last;
    if (!edge || !phased_edge(i, phase, cols, first, last)) { *reinterpret_cast<uint4*>(to) = w; return; }
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j >= first && j < last) to[j] = (uint16_t)(u[j >> 1] >> (16 * (j & 1)));
}
// gamma or beta behind the slots, from `phase` on
__device__ __forceinline__ void stage_weights(uint16_t* to, const uint16_t* w, uint16_t none, int phase, int cols, int pieces) {
    const bool wide = w && !(reinterpret_cast<uintptr_t>(w) & 15);
    if (wide)
        for (int c = threadIdx.x * 8; c + 8 <= cols; c += blockDim.x * 8) {
            const uint4 v = __ldg(reinterpret_cast<const uint4*>(w + c));
            if (phase == 0) { *reinterpret_cast<uint4*>(to + c) = v; continue; }
            const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int j = 0; j < 8; ++j) to[phase + c + j] = (uint16_t)(u[j >> 1] >> (16 * (j & 1)));
        }
    // what is left: all of them where they are not aligned, else the last few; and the places that no column has
    const int begin = wide ? cols & ~7 : 0;
    for (int c = begin + threadIdx.x; c < cols; c += blockDim.x) to[phase + c] = w ? __ldg(w + c) : none;
    if ((int)threadIdx.x < phase) to[threadIdx.x] = none;
    const int end = phase + cols + threadIdx.x;
    if (end < pieces * 8) to[end] = none;                // (fewer than eight)
}

// Forward.  A warp has a row to itself and nothing to wait for but its own loads: no CTA-wide meeting, eight to sixteen rows in different
// phases side by side.  A warp owns `slots` slots of `set_rows` consecutive rows and refills one as soon as it is done with it.  The row is
// read from its slot twice: first and second moment, then the result; gamma and beta lie behind the slots.  8192 x 8192: 53-54 us, 5.0 TB/s (with a
// row to a CTA and its loads in registers 88-90; over a ring of bulk copies 63).
//   The moments are taken about the mean of the row's first 256 values, and the variance is E d^2 - a^2 with a = E d.  Where those values lie
// elsewhere than the rest (a few channels about 30, the others about 0), a^2 is nearly all of E d^2, up to H / 256 - 1 times the variance, and the
// difference loses as many bits (rstd off by 6e-6 at 8192 columns and by 1.4e-5 at 16384; 2e-7 and 4e-7 as it is done here).  A row whose a^2 is over a quarter of E d^2 is read a third
// time, about its mean; of the others the difference loses less than half a bit.
template <bool LAYER, bool PHASED>
__global__ void __launch_bounds__(512, 1) norm_rows_kernel(const __grid_constant__ StreamParams q) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ uint64_t full[64];
    const NormParams& p = q.n;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5, cols = (int)p.v.cols;
    const int period = PHASED ? q.period : 1, first_row = PHASED ? blockIdx.x % period : 0, phase = PHASED ? (int)((int64_t)first_row * cols & 7) : 0;
    const int pieces = PHASED ? (phase + cols + 7) >> 3 : cols >> 3;
    uint16_t *weights = reinterpret_cast<uint16_t*>(smem + (size_t)warps * q.slots * q.slot_bytes), *shifts = weights + q.pieces * 8;
    if ((int)threadIdx.x < warps * q.slots) { mbar_init(&full[threadIdx.x], 1); fence_barrier_init(); }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    // sets of `set_rows` rows (one where PHASED), the next one of this warp `stride` further
    const int64_t rows = p.v.rows, step = (int64_t)warps * q.set_rows * period, stride = step * (PHASED ? (gridDim.x - first_row + period - 1) / period : gridDim.x);
    const int64_t begin = first_row + (int64_t)(blockIdx.x / period) * step + (int64_t)warp * q.set_rows * period;
    unsigned char* mine = smem + (size_t)warp * q.slots * q.slot_bytes;
    uint64_t* bars = full + warp * q.slots;
    int64_t next = begin;                                // (of lane 0: the first row of the next set to be loaded)
    auto fill = [&](int slot) {
        if (next >= rows) return;
        unsigned char* to = mine + (size_t)slot * q.slot_bytes;
        if (PHASED) {
            const uint32_t bytes = phased_bytes(p.v, next, phase, pieces);
            phased_tail(p.v, p.x, next, phase, pieces, reinterpret_cast<uint16_t*>(to));
            mbar_expect_tx(&bars[slot], bytes);
            if (bytes) bulk_load(to, p.x + next * cols - phase, bytes, &bars[slot]);
        } else {
            const int64_t n = min((int64_t)q.set_rows, rows - next);
            mbar_expect_tx(&bars[slot], (uint32_t)(n * cols * 2));
            for (int64_t s = 0; s < p.v.nstrips; ++s) {
                const int64_t w = strip_w_of(p.v, s);
                bulk_load(to + s * q.set_rows * p.v.w * 2, p.x + s * p.v.stride + next * w, (uint32_t)(n * w * 2), &bars[slot]);
            }
        }
        next += stride;
    };
    // (gamma and beta first: behind a CTA's slots full of rows they would wait for those)
    stage_weights(weights, p.gamma, kOne, phase, cols, pieces);
    if (LAYER) stage_weights(shifts, p.beta, 0, phase, cols, pieces);
    __syncthreads();
    if (lane == 0)
        for (int s = 0; s < q.slots; ++s) fill(s);
    const int n_first = min(cols, 256 - phase);
    const float inv_first = 1.0f / (float)n_first;
    int slot = 0;
    uint32_t parity = 0;
    for (int64_t r0 = begin; r0 < rows; r0 += stride) {
        const bool ok = __all_sync(0xffffffffu, mbar_wait_bounded(&bars[slot], parity));
        if (!ok) {                                       // (the copies under way land before the CTA ends)
            if (lane == 0) {
                atomicExch(&g_norm_status, 11);
                for (int s = 0; s < q.slots; ++s)
                    if (r0 + s * stride < next) mbar_wait_bounded(&bars[(slot + s) % q.slots], slot + s < q.slots ? parity : parity ^ 1);
            }
            break;
        }
        const uint16_t* set = reinterpret_cast<const uint16_t*>(mine + (size_t)slot * q.slot_bytes);
        const int n = PHASED ? 1 : (int)min((int64_t)q.set_rows, rows - r0);
        for (int r = 0; r < n; ++r) {
            const int64_t row = r0 + r;
            // every strip's columns of the row: f(place in the slot, first column, pieces, place in the output)
            auto strips = [&](auto f) {
                if (PHASED) f(set, 0, pieces, p.out + row * cols - phase);
                else
                    for (int64_t s = 0; s < p.v.nstrips; ++s) {
                        const int w = (int)strip_w_of(p.v, s);
                        f(set + s * q.set_rows * p.v.w + r * w, (int)(s * p.v.w), w >> 3, p.out + s * p.v.stride + row * w);
                    }
            };
            // elements of a row's first or last piece that are not the row's: `instead`
            auto mask = [&](int i, f32x2 (&f)[4], float instead) {
                int first, last;
                if (PHASED && (i == 0 || i == pieces - 1) && phased_edge(i, phase, cols, first, last))
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float lo, hi;
                        split(f[j], lo, hi);
                        f[j] = pair(2 * j >= first && 2 * j < last ? lo : instead, 2 * j + 1 >= first && 2 * j + 1 < last ? hi : instead);
                    }
            };
            f32x2 f[4];
            float pivot = 0.0f;
            if (LAYER) {
                const int c = lane * 8;
                const int64_t s = PHASED ? 0 : c / p.v.w;            // (strips may be narrower than the first 256 columns)
                parts(lane < pieces ? shared16(PHASED ? set + c : set + s * q.set_rows * p.v.w + r * strip_w_of(p.v, s) + (c - s * p.v.w)) : make_uint4(0u, 0u, 0u, 0u), f);
                mask(lane, f, 0.0f);
                pivot = warp_total((f[0] + f[1]) + (f[2] + f[3])) * inv_first;
            }
            // sums of the differences from `about` and of their squares (times `by`), over H
            auto moments = [&](float about, float by, float& a, float& var) {
                f32x2 m1[2] = {both(0.0f), both(0.0f)}, m2[2] = {both(0.0f), both(0.0f)};
                strips([&](const uint16_t* x, int, int groups, uint16_t*) {
#pragma unroll 4
                    for (int i = lane; i < groups; i += 32) {
                        parts(shared16(x + i * 8), f);
                        mask(i, f, about);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const f32x2 d = LAYER ? f[j] + both(-about) : f[j];
                            if (LAYER) m1[j & 1] = m1[j & 1] + d;
                            m2[j & 1] = fma2(by == 1.0f ? d : d * both(by), d, m2[j & 1]);
                        }
                    }
                });
                a = LAYER ? warp_total(m1[0] + m1[1]) * p.inv_cols : 0.0f;
                var = warp_total((m2[0] + m2[1]) * both(p.inv_cols));
            };
            float a, var;
            moments(pivot, 1.0f, a, var);
            float mean = pivot + a;
            // Once more about the mean where the pivot was no good (see above), and where a lane's squares have left fp32, which the mean of all need
            // not (a lane has 512 values at most: times 2^-16 their squares' sum is below the mean over the row)
            if ((LAYER && a * a > 0.25f * var) || !(var < INFINITY)) {
                const float by = var < INFINITY ? 1.0f : 0x1p-16f;
                moments(mean, by, a, var);
                if (fabsf(a) < INFINITY) mean += a;      // (what the mean's rounding has left; a row with an infinite value keeps its mean)
                if (LAYER) var = fmaf(-a * by, a, var);
                var *= 1.0f / by;
            } else if (LAYER) var = fmaf(-a, a, var);
            var = var < 0.0f ? 0.0f : var;
            const float rstd = rsqrtf(var + p.eps);
            if (lane == 0) {
                if (p.mean) p.mean[row] = mean;
                if (p.rstd) p.rstd[row] = rstd;
            }
            strips([&](const uint16_t* x, int col, int groups, uint16_t* to) {
#pragma unroll 4
                for (int i = lane; i < groups; i += 32) {
                    f32x2 g[4], b[4];
                    parts(shared16(x + i * 8), f);
                    parts(shared16(weights + col + i * 8), g);
                    if (LAYER) parts(shared16(shifts + col + i * 8), b);
#pragma unroll
                    for (int j = 0; j < 4; ++j) f[j] = LAYER ? fma2(f[j] + both(-mean), g[j] * both(rstd), b[j]) : f[j] * (g[j] * both(rstd));
                    store_piece(to + i * 8, bf16x8_pack(f), PHASED && (i == 0 || i == pieces - 1), i, phase, cols);
                }
            });
        }
        __syncwarp();
        if (lane == 0) fill(slot);
        if (++slot == q.slots) { slot = 0; parity ^= 1; }
    }
}

// Back.  The sums for gamma and beta want a thread to keep its columns, so a row is spread over a group of `lanes` threads, R rows at a time
// (two chains of sums that do not wait for each other, gamma unpacked once for both); `groups` groups side by side have the next rows.  A
// stage of the ring is set_rows = groups x R rows of all inputs; warp 0 refills it when all warps are done with it.  One CTA an SM.  8192 x 8192 with
// an addend: 102-110 us with the sums' kernel, 5.1 TB/s, half of the issue slots (one row at a time 143, loads to registers 161).
constexpr int kGradThreads = 512;

template <int NV, int R, bool PHASED>
__global__ void __launch_bounds__(kGradThreads, 1) norm_grad_stream_kernel(const __grid_constant__ StreamParams q) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ uint64_t full[8], empty[8];
    __shared__ float2 sums[2][R][kGradThreads / 32];
    __shared__ int gone[2][kGradThreads / 32];           // a wait of a group ran out
    const NormParams& p = q.n;
    const int L = p.lanes, G = q.groups, warp = threadIdx.x >> 5, wl = threadIdx.x & 31, cols = (int)p.v.cols;
    const int period = PHASED ? q.period : 1, first_row = PHASED ? blockIdx.x % period : 0, phase = PHASED ? (int)((int64_t)first_row * cols & 7) : 0;
    const int pieces = PHASED ? (phase + cols + 7) >> 3 : cols >> 3;
    // sets of set_rows rows, `period` apart; the next one of this CTA `stride` further
    const int64_t rows = p.v.rows, set_rows = q.set_rows, step = set_rows * period;
    const int64_t stride = step * (PHASED ? (gridDim.x - first_row + period - 1) / period : gridDim.x), begin = first_row + (int64_t)(blockIdx.x / period) * step;
    if (threadIdx.x == 0) {
        for (int s = 0; s < q.slots; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], L * G / 32); }
        fence_barrier_init();
    }
    if (threadIdx.x < kGradThreads / 32) gone[0][threadIdx.x] = gone[1][threadIdx.x] = 0;
    uint16_t* weights = reinterpret_cast<uint16_t*>(ring + (size_t)q.slots * q.slot_bytes);
    const uint4 zeros = make_uint4(0u, 0u, 0u, 0u);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    int64_t next = begin;                                // (of warp 0: the first row of the next set to be loaded)
    auto fill = [&](int slot) {                          // (a lane for each row or strip)
        if (next >= rows) return;
        unsigned char* to = ring + (size_t)slot * q.slot_bytes;
        if (PHASED) {
            const int64_t row = next + wl * period;
            uint32_t bytes = 0;
            if (wl < q.set_rows && row < rows) {
                bytes = phased_bytes(p.v, row, phase, pieces);
                const int64_t from = row * cols - phase;
                unsigned char* at = to + wl * q.pieces * 16;
                const uint16_t* src[3] = {p.x, p.dy, p.addend};
#pragma unroll
                for (int a = 0; a < 3; ++a)
                    if (a < q.arrays) {
                        phased_tail(p.v, src[a], row, phase, pieces, reinterpret_cast<uint16_t*>(at + a * q.array_bytes));
                        if (bytes) bulk_load(at + a * q.array_bytes, src[a] + from, bytes, &full[slot]);
                    }
            }
            bytes = __reduce_add_sync(0xffffffffu, bytes) * q.arrays;
            __syncwarp();                                // (the single elements are written before lane 0 arrives; it may announce the bytes after they have landed)
            if (wl == 0) mbar_expect_tx(&full[slot], bytes);
        } else {
            const int64_t n = min(set_rows, rows - next);
            if (wl == 0) mbar_expect_tx(&full[slot], (uint32_t)(n * cols * 2) * q.arrays);
            if (wl < p.v.nstrips) {
                const int64_t w = strip_w_of(p.v, wl), from = wl * p.v.stride + next * w, at = wl * set_rows * p.v.w * 2;
                bulk_load(to + at, p.x + from, (uint32_t)(n * w * 2), &full[slot]);
                bulk_load(to + q.array_bytes + at, p.dy + from, (uint32_t)(n * w * 2), &full[slot]);
                if (q.arrays == 3) bulk_load(to + 2 * q.array_bytes + at, p.addend + from, (uint32_t)(n * w * 2), &full[slot]);
            }
        }
        next += stride;
    };
    stage_weights(weights, p.gamma, kOne, phase, cols, pieces);      // (first, as in norm_rows_kernel)
    __syncthreads();
    if (warp == 0)
        for (int s = 0; s < q.slots; ++s) fill(s);
    const int group = threadIdx.x / L, lane = threadIdx.x - group * L, warp0 = group * (L / 32), warps = L / 32;
    bool mine[NV], edge[NV];
    int col[NV], spot[NV], pitch[NV];                    // column (of a piece's first element), its place among a stage's elements, elements to the next row there
    uint16_t* out[NV];                                   // this thread's columns in the output's row 0
    f32x2 dgamma[NV][4], dbeta[NV][4];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        col[i] = (i * L + lane) * 8;
        mine[i] = col[i] < pieces * 8;
        edge[i] = col[i] == 0 || col[i] == (pieces - 1) * 8;
        const int64_t c = mine[i] ? col[i] : 0, s = PHASED ? 0 : c / p.v.w;
        pitch[i] = PHASED ? q.pieces * 8 : (int)strip_w_of(p.v, s);
        spot[i] = (int)(s * set_rows * p.v.w + group * R * pitch[i] + (c - s * p.v.w));
        out[i] = p.out + s * p.v.stride + (c - s * p.v.w) - phase;
#pragma unroll
        for (int j = 0; j < 4; ++j) dgamma[i][j] = dbeta[i][j] = both(0.0f);
    }
    // how far apart a thread's rows are in the output
    auto out_pitch = [&](int i) { return PHASED ? (int64_t)cols : (int64_t)pitch[i]; };
    int slot = 0, turn = 0;
    uint32_t parity = 0;
    float n_mean[R], n_rstd[R];
    auto statistics = [&](int64_t row) {                 // (of the rows after these, ahead)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t at = row + r * period;
            n_rstd[r] = at < rows ? p.rstd[at] : 0.0f;
            n_mean[r] = at < rows && p.layer ? p.mean[at] : 0.0f;
        }
    };
    auto weight = [&](int i, f32x2 (&w)[4]) { parts(shared16(weights + col[i]), w); };
    statistics(begin + group * R * period);
    for (int64_t r0 = begin; r0 < rows; r0 += stride, turn ^= 1) {
        const int64_t row = r0 + group * R * period;
        bool lost = !mbar_wait_bounded(&full[slot], parity);
        const unsigned char* st = ring + (size_t)slot * q.slot_bytes;
        // (elements of a row's first or last piece that are not the row's read as zeros)
        auto at = [&](int array, int r, int i) {
            uint4 w = shared16(st + array * q.array_bytes + (spot[i] + r * pitch[i]) * 2);
            int first, last;
            if (PHASED && edge[i] && phased_edge(col[i] >> 3, phase, cols, first, last)) {
                uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < first || j >= last) u[j >> 1] &= j & 1 ? 0xFFFFu : 0xFFFF0000u;
                w = make_uint4(u[0], u[1], u[2], u[3]);
            }
            return w;
        };
        if (warp == 0 && r0 != begin && next < rows) {
            // refill the stage of the rows before these once all warps are done with it
            const int before = slot ? slot - 1 : q.slots - 1;
            if (__all_sync(0xffffffffu, mbar_wait_bounded(&empty[before], slot ? parity : parity ^ 1))) fill(before); else lost = true;
        }
        if (lost) { atomicExch(&g_norm_status, 11); *(volatile int*)&gone[turn][group] = 1; }
        float mean[R], rstd[R], s1[R], s2[R];
        f32x2 a[R], b[R];
#pragma unroll
        for (int r = 0; r < R; ++r) { mean[r] = n_mean[r]; rstd[r] = n_rstd[r]; a[r] = b[r] = both(0.0f); }
        statistics(row + stride);
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (mine[i]) {
                f32x2 w[4];
                weight(i, w);
#pragma unroll
                for (int r = 0; r < R; ++r)
                    if (row + r * period < rows) {
                        f32x2 f[4], d[4];
                        parts(at(0, r, i), f); parts(at(1, r, i), d);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const f32x2 h = (f[j] + both(-mean[r])) * both(rstd[r]), g = d[j] * w[j];
                            a[r] = a[r] + g;
                            b[r] = fma2(g, h, b[r]);
                            dgamma[i][j] = fma2(d[j], h, dgamma[i][j]);
                            dbeta[i][j] = dbeta[i][j] + d[j];
                        }
                    }
            }
#pragma unroll
        for (int r = 0; r < R; ++r) { s1[r] = warp_total(a[r]); s2[r] = warp_total(b[r]); }
        if (warps > 1) {                                 // (at most eight groups of two warps or more: named barriers 1 to 8)
            if (wl == 0)
#pragma unroll
                for (int r = 0; r < R; ++r) sums[turn][r][warp] = make_float2(s1[r], s2[r]);
            group_sync(1 + group, L);
#pragma unroll
            for (int r = 0; r < R; ++r) {                // a lane a warp, 16 warps at most
                const float2 o = wl < warps ? sums[turn][r][warp0 + wl] : make_float2(0.0f, 0.0f);
                s1[r] = __shfl_sync(0xffffffffu, lanes_sum(o.x, 16), 0);
                s2[r] = __shfl_sync(0xffffffffu, lanes_sum(o.y, 16), 0);
            }
        } else __syncwarp();
        // (the same for every thread of the group: written before its meeting, and the other one of the two is written before the next)
        if (*(volatile int*)&gone[turn][group]) break;
#pragma unroll
        for (int r = 0; r < R; ++r) { s1[r] = p.layer ? s1[r] * p.inv_cols : 0.0f; s2[r] *= p.inv_cols; }
        if (p.out)
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (mine[i]) {
                    f32x2 w[4];
                    weight(i, w);
                    uint16_t* to = out[i] + row * out_pitch(i);
#pragma unroll
                    for (int r = 0; r < R; ++r)
                        if (row + r * period < rows) {
                            f32x2 f[4], d[4], o[4];
                            parts(at(0, r, i), f); parts(at(1, r, i), d); parts(q.arrays == 3 ? at(2, r, i) : zeros, o);
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const f32x2 h = (f[j] + both(-mean[r])) * both(rstd[r]);
                                o[j] = fma2(both(rstd[r]), fma2(h, both(-s2[r]), fma2(d[j], w[j], both(-s1[r]))), o[j]);
                            }
                            store_piece(to + r * period * out_pitch(i), bf16x8_pack(o), PHASED && edge[i], col[i] >> 3, phase, cols);
                        }
                }
        __syncwarp();
        if (wl == 0) mbar_arrive(&empty[slot]);
        if (++slot == q.slots) { slot = 0; parity ^= 1; }
    }
    // (left early: the copies under way land before the CTA ends)
    if (threadIdx.x == 0 && (gone[0][0] || gone[1][0])) {
        const int64_t fills = (next - begin) / stride;
        for (int s = 0; s < q.slots && s < fills; ++s) mbar_wait_bounded(&full[s], (uint32_t)((fills - 1 - s) / q.slots) & 1);
    }
    __syncthreads();
    if (!p.partial) return;
    // the groups' sums one after the other, by way of the ring's memory (where PHASED the line begins with `phase` idle columns)
    const int width = q.pieces * 8;
    float* line = p.partial + (int64_t)blockIdx.x * 2 * width;
    float* lines = reinterpret_cast<float*>(ring);
    for (int g = 0; g < G; ++g) {
        if (group == g)
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (mine[i])
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        float f[8];
#pragma unroll
                        for (int j = 0; j < 4; ++j) split(k ? dbeta[i][j] : dgamma[i][j], f[2 * j], f[2 * j + 1]);
                        float4* t = reinterpret_cast<float4*>(lines + k * width + col[i]);
                        float4 u = make_float4(f[0], f[1], f[2], f[3]), v = make_float4(f[4], f[5], f[6], f[7]);
                        if (g) {
                            const float4 a = t[0], b = t[1];
                            u.x += a.x; u.y += a.y; u.z += a.z; u.w += a.w;
                            v.x += b.x; v.y += b.y; v.z += b.z; v.w += b.w;
                        }
                        if (g == G - 1) t = reinterpret_cast<float4*>(line + k * width + col[i]);
                        t[0] = u; t[1] = v;
                    }
        if (g < G - 1) __syncthreads();
    }
}

// Rows longer than the registers of a CTA: the row is read once for every sum and once more for the result (from the L2, where it still
// is), by any layout's address map.
template <int VEC, bool GRAD>
__global__ void __launch_bounds__(512) norm_long_kernel(const __grid_constant__ NormParams p) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    __shared__ float2 part[2][16];
    const int warp = threadIdx.x >> 5;
    constexpr int PR = (VEC + 1) / 2;
    int turn = 0;
    auto meet = [&](float& a, float& b) {                // sums over the CTA
        a = lanes_sum(a, 32); b = lanes_sum(b, 32);
        if ((threadIdx.x & 31) == 0) part[turn][warp] = make_float2(a, b);
        __syncthreads();
        a = b = 0.0f;
        for (int w = 0; w < 16; ++w) { a += part[turn][w].x; b += part[turn][w].y; }
        turn ^= 1;
    };
    for (int64_t row = blockIdx.x; row < p.v.rows; row += gridDim.x) {
        float mean = 0.0f, rstd = 0.0f, s1 = 0.0f, s2 = 0.0f;
        uint32_t u[PR];
        if (!GRAD) {
            if (p.layer) {
                float none = 0.0f;
                for (int64_t c = (int64_t)threadIdx.x * VEC; c < p.v.cols; c += 512 * VEC) {
                    float f[VEC];
                    load_vec<VEC>(p.x + map(p.v, row, c), u);
                    unpack<VEC>(u, f);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) mean += f[j];
                }
                meet(mean, none);
                mean *= p.inv_cols;
            }
            for (int64_t c = (int64_t)threadIdx.x * VEC; c < p.v.cols; c += 512 * VEC) {
                float f[VEC];
                load_vec<VEC>(p.x + map(p.v, row, c), u);
                unpack<VEC>(u, f);
#pragma unroll
                for (int j = 0; j < VEC; ++j) { s1 += f[j] - mean; s2 = fmaf((f[j] - mean) * p.inv_cols, f[j] - mean, s2); }
            }
            meet(s1, s2);
            // (s1 is zero but for the mean's own rounding, which it takes out of the variance)
            if (p.layer) s2 -= (s1 * p.inv_cols) * (s1 * p.inv_cols);
            rstd = rsqrtf((s2 < 0.0f ? 0.0f : s2) + p.eps);
            if (threadIdx.x == 0) {
                if (p.mean) p.mean[row] = mean;
                if (p.rstd) p.rstd[row] = rstd;
            }
        } else {
            mean = p.layer ? p.mean[row] : 0.0f;
            rstd = p.rstd[row];
            for (int64_t c = (int64_t)threadIdx.x * VEC; c < p.v.cols; c += 512 * VEC) {
                float f[VEC], d[VEC], g[VEC];
                const int64_t at = map(p.v, row, c);
                load_vec<VEC>(p.x + at, u);
                unpack<VEC>(u, f);
                load_vec<VEC>(p.dy + at, u);
                unpack<VEC>(u, d);
                load_weights<VEC>(p.gamma, c, 1.0f, g);
#pragma unroll
                for (int j = 0; j < VEC; ++j) { s1 += d[j] * g[j]; s2 = fmaf(d[j] * g[j], (f[j] - mean) * rstd, s2); }
            }
            meet(s1, s2);
            s1 = p.layer ? s1 * p.inv_cols : 0.0f;
            s2 *= p.inv_cols;
        }
        for (int64_t c = (int64_t)threadIdx.x * VEC; c < p.v.cols; c += 512 * VEC) {
            const int64_t at = map(p.v, row, c);
            float f[VEC], g[VEC], o[VEC];
            load_vec<VEC>(p.x + at, u);
            unpack<VEC>(u, f);
            load_weights<VEC>(p.gamma, c, 1.0f, g);
            if (!GRAD) {
                float b[VEC];
                load_weights<VEC>(p.beta, c, 0.0f, b);
#pragma unroll
                for (int j = 0; j < VEC; ++j) o[j] = fmaf((f[j] - mean) * rstd, g[j], b[j]);
                store_vec<VEC>(p.out + at, o);
            } else {
                float d[VEC], a[VEC];
                load_vec<VEC>(p.dy + at, u);
                unpack<VEC>(u, d);
#pragma unroll
                for (int j = 0; j < PR; ++j) u[j] = 0;
                if (p.addend) load_vec<VEC>(p.addend + at, u);
                unpack<VEC>(u, a);
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float h = (f[j] - mean) * rstd;
                    o[j] = fmaf(rstd, fmaf(-h, s2, fmaf(d[j], g[j], -s1)), a[j]);
                }
                store_vec<VEC>(p.out + at, o);
            }
        }
    }
}

// dgamma and dbeta (blockIdx.y) from the CTAs' lines: 32 columns a block, eight warps over the lines, their sums added in a fixed order
__global__ void __launch_bounds__(256) norm_grad_finish_kernel(const float* partial, int ctas, int64_t cols, int width, int phases, uint16_t* dgamma, uint16_t* dbeta) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    __shared__ float part[8][32];
    uint16_t* out = blockIdx.y ? dbeta : dgamma;
    if (!out) return;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int64_t n = (int64_t)blockIdx.x * 32 + lane;
    float s = 0.0f;
    if (n < cols)
        for (int b0 = w; b0 < ctas; b0 += 8 * 20) {      // (twenty loads in flight: all of a line's, one line an SM)
            float x[20];
#pragma unroll
            for (int u = 0; u < 20; ++u) {
                const int b = b0 + 8 * u;
                x[u] = b < ctas ? partial[((int64_t)b * 2 + blockIdx.y) * width + ((b & phases) * (int)(cols & 7) & 7) + n] : 0.0f;
            }
#pragma unroll
            for (int u = 0; u < 20; ++u) s += x[u];
        }
    part[w][lane] = s;
    __syncthreads();
    if (w == 0 && n < cols) {
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += part[i][lane];
        reinterpret_cast<__nv_bfloat16*>(out)[n] = __float2bfloat16_rn(s);
    }
}

namespace {

constexpr int64_t kRing = 192 * 1024;                    // bytes of the gradient's ring: two stages of the longest rows (32 KB) with three inputs
constexpr int64_t kSlots = 216 * 1024;                   // bytes of the forward pass's slots with gamma and beta
constexpr int64_t kStreamCols = 16384;

// How a problem is laid over threads
struct NormPlan {
    int vec, nv, lanes, threads;    // nv 0: the kernel for long rows
    bool linear, one;
    int64_t groups;                 // CTAs that would each have one row (or one set of rows side by side)
    int stream, slots, arrays;      // norm_rows_kernel: warps, norm_grad_stream_kernel: groups side by side (0: neither is taken)
    int period, pieces;             // (see StreamParams)
    int64_t set_rows;
};

bool vectors(const MatView& v) {    // every group of eight columns is one aligned 16-byte piece of the buffer
    return v.cols % 8 == 0 && (v.split != 2 || (v.w % 8 == 0 && v.wlast % 8 == 0)) && v.stride % 8 == 0 && v.ichunk % 8 == 0;
}

// aligned: all matrices are 16-byte aligned, weights: gamma and beta are; arrays: inputs of the shape of a row (1 forward; 2 or 3 back)
NormPlan plan_norm(const MatView& v, bool aligned, bool weights, bool grad, int arrays, int sms) {
    NormPlan q = {};
    const bool whole = aligned && vectors(v);
    q.linear = !v.ichunk && v.split != 1;
    q.period = 1;
    if (!whole) while ((q.period * v.cols) % 8) q.period *= 2;
    q.pieces = (int)std::min<int64_t>((v.cols + (whole ? 7 : 14)) / 8, INT32_MAX / 16);
    if (aligned && q.linear && v.cols >= 256 && q.pieces <= kStreamCols / 8 && (whole ? v.nstrips <= 16 : v.split == 0)) {
        const int64_t row = (int64_t)q.pieces * 16;                  // bytes
        q.arrays = arrays;
        if (grad) {
            q.nv = q.pieces < 64 ? 1 : (q.pieces <= 2 * kGradThreads ? 2 : 4);
            q.lanes = ((q.pieces + q.nv - 1) / q.nv + 31) / 32 * 32;
            q.stream = kGradThreads / q.lanes;
            q.threads = q.stream * q.lanes;
            q.set_rows = q.stream * (q.nv == 4 ? 1 : 2);
            q.slots = (int)std::min<int64_t>(8, kRing / (q.set_rows * row * arrays));        // (two at least)
            q.groups = (v.rows + q.set_rows - 1) / q.set_rows;
        } else {
            const int64_t room = kSlots - 2 * row;                   // (gamma and beta)
            q.set_rows = whole ? std::max<int64_t>(1, 4096 / row) : 1;
            const int64_t all = room / (q.set_rows * row);           // slots of a CTA
            // a warp each; no more warps than leave every SM its rows
            const int64_t sets = (v.rows + q.set_rows - 1) / q.set_rows;
            q.stream = (int)std::min<int64_t>(std::min<int64_t>(16, all), std::max<int64_t>(4, (sets + sms - 1) / sms));
            q.slots = (int)std::min<int64_t>(4, all / q.stream);
            q.threads = q.stream * 32;
            q.groups = (v.rows + q.stream * q.set_rows - 1) / (q.stream * q.set_rows);
        }
        // (few rows: the register kernels have more threads for each; of odd widths they know single elements only)
        if (!whole || v.rows >= (grad ? sms * q.set_rows : 8 * sms)) {
            q.groups = std::max<int64_t>(q.groups, q.period);        // (a CTA for every phase)
            return q;
        }
        q.stream = 0;
    }
    q.vec = whole && weights ? 8 : 1;
    const int64_t groups = (v.cols + q.vec - 1) / q.vec;            // column groups of a row
    const int64_t most = 1024;
    if (q.vec == 8) q.nv = groups <= 32 ? 1 : (groups <= 2 * most ? 2 : 4);
    else q.nv = groups <= 64 ? 2 : 8;
    const int64_t need = (groups + q.nv - 1) / q.nv;
    if (need > most) { q.nv = 0; q.threads = 512; q.lanes = 512; q.groups = v.rows; return q; }
    q.one = need <= 32;
    if (q.one) {
        q.lanes = 8;
        while (q.lanes < need) q.lanes *= 2;
        q.threads = 256;
        q.groups = (v.rows + q.threads / q.lanes - 1) / (q.threads / q.lanes);
    } else {
        q.lanes = q.threads = (int)((need + 31) / 32 * 32);
        q.groups = v.rows;
    }
    return q;
}

unsigned grid_of(const NormPlan& q, int sms) { return (unsigned)std::min<int64_t>(q.groups, (int64_t)sms * (q.stream ? 1 : std::max(1, 2048 / q.threads))); }

template <bool GRAD, int VEC, int NV, bool ONE>
ccl_status launch_shape(const NormParams& p, const NormPlan& q, unsigned grid, cudaStream_t st) {
    if constexpr (GRAD) return launch_early(q.linear ? norm_grad_kernel<VEC, NV, true, ONE> : norm_grad_kernel<VEC, NV, false, ONE>, dim3(grid), q.threads, 0, st, p);
    else return launch_early(q.linear ? norm_kernel<VEC, NV, true, ONE> : norm_kernel<VEC, NV, false, ONE>, dim3(grid), q.threads, 0, st, p);
}
template <int WHICH>
ccl_status launch_stream(void (*kernel)(const StreamParams), const NormParams& p, const NormPlan& q, unsigned grid, cudaStream_t st) {
    static std::atomic<uint64_t> configured{0};          // bit per device: the shared-memory limit has been raised
    int dev = 0;
    CCL_CUDA_TRY(cudaGetDevice(&dev));
    if (dev >= 64 || !(configured.load() >> dev & 1)) {
        CCL_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(WHICH < 4 ? kSlots : kRing + kStreamCols * 2)));
        if (dev < 64) configured.fetch_or(1ull << dev);
    }
    StreamParams sp;
    sp.n = p;
    sp.groups = q.stream; sp.slots = q.slots; sp.arrays = q.arrays; sp.set_rows = (int32_t)q.set_rows; sp.period = q.period; sp.pieces = q.pieces;
    sp.array_bytes = (uint32_t)(q.set_rows * q.pieces * 16);
    sp.slot_bytes = sp.array_bytes * (uint32_t)q.arrays;
    const size_t smem = (size_t)sp.slot_bytes * q.slots * (WHICH < 4 ? q.stream : 1) + (size_t)q.pieces * (WHICH < 4 ? 32 : 16);
    return launch_early(kernel, dim3(grid), q.threads, smem, st, sp);
}
template <bool GRAD>
ccl_status launch_plan(const NormParams& p, const NormPlan& q, unsigned grid, cudaStream_t st) {
    if (q.stream && !GRAD) {
        if (q.period > 1) return p.layer ? launch_stream<0>(norm_rows_kernel<true, true>, p, q, grid, st) : launch_stream<1>(norm_rows_kernel<false, true>, p, q, grid, st);
        return p.layer ? launch_stream<2>(norm_rows_kernel<true, false>, p, q, grid, st) : launch_stream<3>(norm_rows_kernel<false, false>, p, q, grid, st);
    }
    if (q.stream && q.period > 1)
        return q.nv == 1 ? launch_stream<4>(norm_grad_stream_kernel<1, 2, true>, p, q, grid, st)
                         : (q.nv == 2 ? launch_stream<5>(norm_grad_stream_kernel<2, 2, true>, p, q, grid, st) : launch_stream<6>(norm_grad_stream_kernel<4, 1, true>, p, q, grid, st));
    if (q.stream)
        return q.nv == 1 ? launch_stream<7>(norm_grad_stream_kernel<1, 2, false>, p, q, grid, st)
                         : (q.nv == 2 ? launch_stream<8>(norm_grad_stream_kernel<2, 2, false>, p, q, grid, st) : launch_stream<9>(norm_grad_stream_kernel<4, 1, false>, p, q, grid, st));
    if (q.nv == 0) return launch_early(q.vec == 8 ? norm_long_kernel<8, GRAD> : norm_long_kernel<1, GRAD>, dim3(grid), q.threads, 0, st, p);
    if (q.vec == 8) {
        if (q.one) return q.nv == 1 ? launch_shape<GRAD, 8, 1, true>(p, q, grid, st) : launch_shape<GRAD, 8, 2, true>(p, q, grid, st);
        return q.nv == 2 ? launch_shape<GRAD, 8, 2, false>(p, q, grid, st) : launch_shape<GRAD, 8, 4, false>(p, q, grid, st);
    }
    if (q.one) return q.nv == 2 ? launch_shape<GRAD, 1, 2, true>(p, q, grid, st) : launch_shape<GRAD, 1, 8, true>(p, q, grid, st);
    return launch_shape<GRAD, 1, 8, false>(p, q, grid, st);
}

ccl_status norm_view(const char* who, const ccl_mat* m, int32_t kind, MatView* v) {
    ccl_status s = make_view(m, who, v);
    if (s) return s;
    if (kind != CCL_NORM_LAYER && kind != CCL_NORM_RMS) return fail(CCL_ERR_INVALID_ARG, "%s: unknown kind %d", who, kind);
    if (v->e != 2) return fail(CCL_ERR_UNSUPPORTED, "%s: only 2-byte (bf16) elements are supported", who);
    if (v->cols >= (INT64_C(1) << 31)) return fail(CCL_ERR_UNSUPPORTED, "%s: rows of %lld columns are too long", who, (long long)v->cols);
    return CCL_OK;
}
uintptr_t bits(const void* p) { return reinterpret_cast<uintptr_t>(p); }
const uint16_t* bf16(const void* p) { return static_cast<const uint16_t*>(p); }

// Lines of sums that the gradient's kernel leaves (0: it leaves them to norm_sums_kernel), whatever the buffers' alignment and the addend
size_t grad_workspace(const MatView& v, int sms) {
    size_t lines = 0;
    for (int arrays : {2, 3}) {
        const NormPlan q = plan_norm(v, true, true, true, arrays, sms);
        if (q.stream) lines = std::max<size_t>(lines, (size_t)grid_of(q, sms) * q.pieces);
    }
    return lines * 2 * 8 * 4;
}

ccl_status launch_sums(NormParams p, const NormPlan& q, int sms, uint16_t* dgamma, uint16_t* dbeta, cudaStream_t st) {
    // as many threads along a row as leave every SM a few CTAs; eight CTAs at most share the rows
    const int64_t groups = (p.v.cols + q.vec - 1) / q.vec;
    int lanes = 32, ctas = 8;
    while (ctas > 1 && p.v.rows < (int64_t)ctas * 32) ctas /= 2;
    while (lanes > 2 && (groups + lanes - 1) / lanes * ctas < sms * 3) lanes /= 2;
    const int64_t tiles = (groups + lanes - 1) / lanes;
    if (tiles * ctas >= (INT64_C(1) << 31)) return fail(CCL_ERR_UNSUPPORTED, "ccl_norm_grad: too many columns");
    p.lanes = lanes;
    auto kernel = q.vec == 8 ? (q.linear ? norm_sums_kernel<8, true> : norm_sums_kernel<8, false>) : (q.linear ? norm_sums_kernel<1, true> : norm_sums_kernel<1, false>);
    return launch_early_clusters(kernel, dim3((unsigned)(tiles * ctas)), 256, ctas, st, p, dgamma, dbeta, (p.v.rows + ctas - 1) / ctas);
}

}  // namespace

// The status word of this file's kernels, read and cleared (ccl_gemm_status)
ccl_status norm_status_take(int* code) {
    int zero = 0;
    CCL_CUDA_TRY(cudaMemcpyFromSymbol(code, g_norm_status, sizeof(int)));
    if (*code) CCL_CUDA_TRY(cudaMemcpyToSymbol(g_norm_status, &zero, sizeof(int)));
    return CCL_OK;
}

}  // namespace ccl

using namespace ccl;

extern "C" ccl_status ccl_norm(const ccl_mat* m, int32_t kind, float eps, const void* X_dev, const void* gamma_dev, const void* beta_dev, void* Y_dev,
                               float* mean_dev, float* rstd_dev, void* cuda_stream) {
    NormParams p = {};
    ccl_status s = norm_view("ccl_norm", m, kind, &p.v);
    if (s) return s;
    if (!(eps >= 0.0f && eps < 1e30f)) return fail(CCL_ERR_INVALID_ARG, "ccl_norm: eps must be a number >= 0");
    if (!X_dev || !Y_dev) return fail(CCL_ERR_INVALID_ARG, "ccl_norm: NULL operand");
    if (kind == CCL_NORM_RMS && (beta_dev || mean_dev)) return fail(CCL_ERR_INVALID_ARG, "ccl_norm: the root-mean-square form has neither beta nor means");
    const uintptr_t any = bits(X_dev) | bits(Y_dev), weights = bits(gamma_dev) | bits(beta_dev);
    if ((any | weights) & 1) return fail(CCL_ERR_ALIGN, "ccl_norm: a base pointer is not 2-byte aligned");
    if ((bits(mean_dev) | bits(rstd_dev)) & 3) return fail(CCL_ERR_ALIGN, "ccl_norm: mean / rstd is not 4-byte aligned");
    p.x = bf16(X_dev); p.out = static_cast<uint16_t*>(Y_dev); p.gamma = bf16(gamma_dev); p.beta = bf16(beta_dev);
    p.mean = mean_dev; p.rstd = rstd_dev;
    p.layer = kind == CCL_NORM_LAYER; p.eps = eps; p.inv_cols = (float)(1.0 / (double)p.v.cols);
    const uint64_t whole = (uint64_t)buffer_elems(p.v) * 2, row = (uint64_t)p.v.cols * 2, column = (uint64_t)p.v.rows * 4;
    const Span all[6] = {{Y_dev, whole}, {mean_dev, column}, {rstd_dev, column}, {X_dev == Y_dev ? nullptr : X_dev, whole}, {gamma_dev, row}, {beta_dev, row}};
    for (int i = 0; i < 3; ++i)
        if (overlaps_any(all[i], all) || (i && overlap(all[i], {X_dev, whole})))
            return fail(CCL_ERR_INVALID_ARG, "ccl_norm: Y, mean or rstd lies over another buffer (Y may be X)");
    int sms, pairs;
    device_units(&sms, &pairs);
    const NormPlan q = plan_norm(p.v, (any & 15) == 0, (weights & 15) == 0, false, 1, sms);
    p.lanes = q.lanes;
    return launch_plan<false>(p, q, grid_of(q, sms), reinterpret_cast<cudaStream_t>(cuda_stream));
}

extern "C" ccl_status ccl_norm_grad_workspace(const ccl_mat* m, size_t* bytes) {
    MatView v;
    ccl_status s = norm_view("ccl_norm_grad_workspace", m, CCL_NORM_LAYER, &v);
    if (s) return s;
    if (!bytes) return fail(CCL_ERR_INVALID_ARG, "ccl_norm_grad_workspace: NULL output");
    int sms, pairs;
    device_units(&sms, &pairs);
    *bytes = grad_workspace(v, sms);
    return CCL_OK;
}

extern "C" ccl_status ccl_norm_grad(const ccl_mat* m, int32_t kind, const void* X_dev, const void* gamma_dev, const float* mean_dev, const float* rstd_dev,
                                    const void* dY_dev, const void* addend_dev, void* dX_dev, void* dgamma_dev, void* dbeta_dev, void* ws_dev,
                                    size_t ws_bytes, void* cuda_stream) {
    NormParams p = {};
    ccl_status s = norm_view("ccl_norm_grad", m, kind, &p.v);
    if (s) return s;
    const bool layer = kind == CCL_NORM_LAYER;
    if (!X_dev || !dY_dev || !rstd_dev || (layer && !mean_dev)) return fail(CCL_ERR_INVALID_ARG, "ccl_norm_grad: NULL operand");
    if (!dX_dev && !dgamma_dev && !dbeta_dev) return fail(CCL_ERR_INVALID_ARG, "ccl_norm_grad: no output is wanted");
    if (!layer && dbeta_dev) return fail(CCL_ERR_INVALID_ARG, "ccl_norm_grad: the root-mean-square form has no beta");
    // (with few rows dgamma and dbeta are written before gamma is read for dX)
    const void* outs[3] = {dX_dev, dgamma_dev, dbeta_dev};
    for (int i = 0; i < 3; ++i)
        if (outs[i] && (outs[i] == gamma_dev || outs[i] == outs[(i + 1) % 3]))
            return fail(CCL_ERR_INVALID_ARG, "ccl_norm_grad: dX, dgamma and dbeta need buffers of their own, and not gamma's");
    const uintptr_t any = bits(X_dev) | bits(dY_dev) | bits(addend_dev) | bits(dX_dev);
    if ((any | bits(gamma_dev) | bits(dgamma_dev) | bits(dbeta_dev)) & 1) return fail(CCL_ERR_ALIGN, "ccl_norm_grad: a base pointer is not 2-byte aligned");
    if ((bits(mean_dev) | bits(rstd_dev)) & 3) return fail(CCL_ERR_ALIGN, "ccl_norm_grad: mean / rstd is not 4-byte aligned");
    int sms, pairs;
    device_units(&sms, &pairs);
    p.x = bf16(X_dev); p.dy = bf16(dY_dev); p.addend = dX_dev ? bf16(addend_dev) : nullptr; p.out = static_cast<uint16_t*>(dX_dev); p.gamma = bf16(gamma_dev);
    p.mean = const_cast<float*>(mean_dev); p.rstd = const_cast<float*>(rstd_dev);
    p.layer = layer; p.inv_cols = (float)(1.0 / (double)p.v.cols);
    uint16_t *dgamma = static_cast<uint16_t*>(dgamma_dev), *dbeta = static_cast<uint16_t*>(dbeta_dev);
    const bool sums = dgamma || dbeta;
    const size_t need = sums ? grad_workspace(p.v, sms) : 0;
    if (sums) {
        if (need && (!ws_dev || ws_bytes < need)) return fail(CCL_ERR_WORKSPACE, "ccl_norm_grad: needs %zu bytes of workspace (got %zu)", need, ws_dev ? ws_bytes : (size_t)0);
        if (bits(ws_dev) & 15) return fail(CCL_ERR_ALIGN, "ccl_norm_grad: workspace is not 16-byte aligned");
    }
    const uint64_t whole = (uint64_t)buffer_elems(p.v) * 2, row = (uint64_t)p.v.cols * 2, column = (uint64_t)p.v.rows * 4;
    const Span written[4] = {{dX_dev, whole}, {dgamma_dev, row}, {dbeta_dev, row}, {need ? ws_dev : nullptr, need}};
    const Span read[6] = {{X_dev, whole}, {dY_dev, whole}, {p.addend, whole}, {gamma_dev, row}, {layer ? mean_dev : nullptr, column}, {rstd_dev, column}};
    for (const Span& o : written) {
        bool bad = overlaps_any(o, written);
        for (const Span& r : read) bad = bad || (overlap(o, r) && !(o.p == dX_dev && r.p == dX_dev && &r < read + 3));
        if (bad) return fail(CCL_ERR_INVALID_ARG, "ccl_norm_grad: dX, dgamma, dbeta or the workspace lies over another buffer (dX may be X, dY or the addend)");
    }
    const NormPlan q = plan_norm(p.v, (any & 15) == 0, (bits(gamma_dev) & 15) == 0, true, p.addend ? 3 : 2, sms);
    p.lanes = q.lanes;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    const unsigned grid = grid_of(q, sms);
    if (q.stream && sums) {
        p.partial = static_cast<float*>(ws_dev);
        if ((s = launch_plan<true>(p, q, grid, st))) return s;
        return launch_early(norm_grad_finish_kernel, dim3((unsigned)((p.v.cols + 31) / 32), 2), 256, 0, st, (const float*)p.partial, (int)grid, p.v.cols, q.pieces * 8,
                            q.period - 1, dgamma, dbeta);
    }
    if (sums && (s = launch_sums(p, q, sms, dgamma, dbeta, st))) return s;        // (first: dX may take the place of X or dY)
    return p.out ? launch_plan<true>(p, q, grid, st) : CCL_OK;
}
