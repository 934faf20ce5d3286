// ccl_linear_xent: the cross entropy of z = X W^T over a large vocabulary, and ccl_linear_xent_grad: its gradients with respect to X and W.
// The logits z are never stored.
//
// Forward.  The GEMM of ccl_gemm (ccl_gemm_kernel.cuh, EPI = 3) with another drain: a lane has a row of 64 of the tile's columns, adds their
// logits up in fp32 from accumulators of 1024 of K each (256 with up to 128 tokens), and leaves the largest and the sum of exponentials about it (the target's logit
// where it passes by), and a second kernel joins a row's numbers:  lse = max + log(sum of s_i exp(m_i - max)).  Powers of two throughout: one
// multiply-add and one hardware exponential a logit, behind the next tile's product.
//
// Gradient.  dz = dloss / s (exp(z - lse) - [target]), piece by piece of the vocabulary: the logits' product again, its drain turning z into dz
// (EPI = 4), rounded to bf16 because it is the operand of the two products that follow; dW of the piece = s dz^T X, a whole sum over the
// tokens, and dX += s dz W, which is kept in fp32 from piece to piece (EPI = 5) and rounded once at the end.  s is the largest |dloss|, so
// that where all are alike (a mean over the tokens) the rounding is that of p - 1 and p themselves: a target that has little of the
// probability is -1 then, exact or nearly so, where -dloss would be off by 2^-9 of itself (777 tokens: errors of dX and dW against 64 bits
// 0.0025 -> 0.0019 of their norms, of which 0.0017 are the outputs' own rounding).  Where tokens weigh differently it is 0.0023 (weights
// uniform from 0 to 2) to 0.0025 (e to a normal deviate).
//   Up to 16 tokens, whose roundings little averages (0.0036 to 0.0038 with one), have two rows of dz each: the rounded values and, 16 rows further at most, what is left of them, rounded too.  X lies in the workspace twice, one below the
// other, so that the products need not know; dX comes from fp32 sums of both rows.  The outputs' own rounding is then all there is
// (0.0016 to 0.0017; of 1662 drawn gradients of 2 to 16 tokens 115 were off by over 1.5 times the plain form's error, 6 are, where p - 1 itself
// cancels), for some us: 1 x 131072 x 4096 553 / 555, 8 x 64000 x 8192 533 / 538, 1 x 5000 x 512 27 / 32; four strips, whose products are then
// added one by one, 1 x 32000 x 2048 97 / 118.
//   A piece's dz is at most kPieceBytes unless 256 columns (or a strip) are more.  Recomputing the logits costs a quarter of the gradient's
// products; keeping them would cost T x V x 4 bytes.
//
// Bound by the tensor cores: 2 T V H and 6 T V H operations.
#include "ccl_gemm_epi.cuh"

namespace ccl {

ccl_status gemm_cut(const ccl_gemm_desc* d, int64_t rows_c, int64_t rows_b, const float* alpha_dev, const void* A, const void* B, void* C, void* ws, size_t ws_bytes,
                    void* stream);                       // ccl_gemm.cu

constexpr int64_t kPieceBytes = INT64_C(1) << 29;

template <int EPI, int BN, int CTAS>
static ccl_status launch_logits_warps(const GemmPlan& plan, const CUtensorMap* maps, const EpiMaps<EPI>& em, cudaStream_t st) {
    if constexpr (EPI == 3) return launch_epi_warps<BN, CTAS, false, 0, EPI, 16>(plan, maps, em, st);
    if constexpr (EPI == 4)
        if (plan.opw == 16) return launch_epi_warps<BN, CTAS, false, 0, EPI, 16>(plan, maps, em, st);
    if constexpr (EPI != 3) return launch_epi_warps<BN, CTAS, false, 0, EPI, 8>(plan, maps, em, st);
}

// A product over part of the vocabulary.  rows_b: rows of B that exist (0: all that the descriptor says), the rest reads as zeros; rows_c: rows
// of C likewise, the rest is not written.
template <int EPI>
static ccl_status run_logits(GemmPlan& plan, const EpiMaps<EPI>& em, int64_t rows_b, const void* A, const void* B, void* C, cudaStream_t st, int64_t rows_c = 0) {
    if (!plan.lean) return fail(CCL_ERR_UNSUPPORTED, "ccl_linear_xent: this layout of W is not supported");
    if (rows_b) plan.vb.rows = rows_b;
    if (rows_c) { plan.p.M = plan.p.Wm = (int32_t)rows_c; plan.vc.rows = rows_c; }
    CUtensorMap maps[6];
    ccl_status s = encode_maps(plan, A, B, C, maps);
    if (s) return s;
    plan.p.C = static_cast<uint16_t*>(C);
    plan.p.alpha = 1.0f;
    if ((s = wave_barrier(plan, true, st))) return s;
    switch (plan.bn * 10 + plan.ctas) {
        case 2562: return launch_logits_warps<EPI, 256, 2>(plan, maps, em, st);
        case 1282: return launch_logits_warps<EPI, 128, 2>(plan, maps, em, st);
        case 2561: return launch_logits_warps<EPI, 256, 1>(plan, maps, em, st);
        default: return launch_logits_warps<EPI, 128, 1>(plan, maps, em, st);
    }
}

// Joins `lines` pairs (log2 of a scale, sum about it) of each row: `lanes` rows side by side in a block, the other threads along the lines,
// always in the same order.  The last steps, a few per row, are taken in 64 bits.
__global__ void __launch_bounds__(256) xent_finish_kernel(const float2* part, int lines, int M, int lanes, const int32_t* targets, int32_t ignore, int32_t classes,
                                                          const float* at_target, float* loss, float* lse) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    __shared__ float2 both_[256];
    const int across = 256 / lanes, lx = threadIdx.x & (lanes - 1), ly = threadIdx.x / lanes;
    const int64_t row = (int64_t)blockIdx.x * lanes + lx;
    float t = -1e30f, s = 0.0f;
    auto join = [&](float2 o) {
        const float top = fmaxf(t, o.x);
        s = fmaf(s, exp2_fast(t - top), o.y * exp2_fast(o.x - top));
        t = top;
    };
    if (row < M) {
        int b = ly;
        for (; b + 7 * across < lines; b += 8 * across) {            // (eight loads in flight)
            float2 v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = part[(int64_t)(b + i * across) * M + row];
#pragma unroll
            for (int i = 0; i < 8; ++i) join(v[i]);
        }
        for (; b < lines; b += across) join(part[(int64_t)b * M + row]);
    }
    both_[threadIdx.x] = make_float2(t, s);
    for (int w = across >> 1; w >= 1; w >>= 1) {
        __syncthreads();
        if (ly < w) {
            join(both_[threadIdx.x + w * lanes]);
            both_[threadIdx.x] = make_float2(t, s);
        }
    }
    if (ly != 0 || row >= M) return;
    const double l = ((double)t + log2((double)s)) * 0.6931471805599453;
    if (lse) lse[row] = (float)l;
    const int cls = targets[row];
    const bool live = cls != ignore && (unsigned)cls < (unsigned)classes;
    if (!live && cls != ignore) report_input(10);
    if (loss) loss[row] = live ? (float)(l - (double)at_target[row]) : 0.0f;
}

// scale = the largest finite |dloss| of the rows that take part (1 where all are zero or there is none; 2^-126 at least, whose reciprocal
// is finite: below it, 1 / scale would be infinite and a row with dloss = 0 beside it NaN).  The blocks behind the first write x
// (n8 pieces of 16 bytes) twice, one below the other, to x2.
__global__ void __launch_bounds__(1024) xent_scale_kernel(const float* dloss, const int32_t* targets, int M, int32_t ignore, int32_t classes, float* scale,
                                                          const uint4* x, uint4* x2, int64_t n8) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    __shared__ float tops[32];
    if (blockIdx.x) {
        for (int64_t i = (int64_t)(blockIdx.x - 1) * 1024 + threadIdx.x; i < n8; i += (int64_t)(gridDim.x - 1) * 1024) {
            const uint4 w = x[i];
            x2[i] = w;
            x2[n8 + i] = w;
        }
        return;
    }
    float top = 0.0f;
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < M; i += 1024) {
        const int cls = targets[i];
        const float d = fabsf(dloss[i]);
        if (cls != ignore && (unsigned)cls < (unsigned)classes && d < INFINITY) top = fmaxf(top, d);
    }
    top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));         // (ordered as their bits are)
    if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
    __syncthreads();
    if (threadIdx.x < 32) {
        top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(tops[threadIdx.x])));
        if (threadIdx.x == 0) *scale = top > 0.0f ? fmaxf(top, 0x1p-126f) : 1.0f;
    }
}

// dX = bf16(scale x sum of the `parts` fp32 sums), eight values a thread
__global__ void __launch_bounds__(256) xent_dx_kernel(const float* acc, int parts, int64_t n, const float* scale, uint16_t* dx) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const f32x2 by = both(*scale);
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8; i < n; i += (int64_t)gridDim.x * 256 * 8) {
        f32x2 v[4] = {both(0.0f), both(0.0f), both(0.0f), both(0.0f)};
#pragma unroll 8
        for (int k = 0; k < parts; ++k) {
            const float4 a = *reinterpret_cast<const float4*>(acc + k * n + i), b = *reinterpret_cast<const float4*>(acc + k * n + i + 4);
            v[0] = v[0] + pair(a.x, a.y); v[1] = v[1] + pair(a.z, a.w);
            v[2] = v[2] + pair(b.x, b.y); v[3] = v[3] + pair(b.z, b.w);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = v[j] * by;
        *reinterpret_cast<uint4*>(dx + i) = bf16x8_pack(v);
    }
}

namespace {

ccl_mat matrix(int64_t rows, int64_t cols) { return ccl_mat{rows, cols, 2, 1, CCL_PART_NONE, CCL_ROWMAJOR, 0}; }
ccl_gemm_desc product(int64_t M, int64_t N, int64_t K, const ccl_mat& A, int a_trans, const ccl_mat& B, int b_trans, const ccl_mat& C) {
    ccl_gemm_desc d = {};
    d.M = M; d.N = N; d.K = K; d.A = A; d.B = B; d.C = C;
    d.a_trans = a_trans; d.b_trans = b_trans; d.out_part = CCL_PART_NONE; d.P = 1;
    return d;
}
int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

struct Vocabulary {
    int64_t T, V, H;
    int64_t M;                      // rows of the gradient's dz
    bool trans;                     // W stored [V x H]; otherwise [H x V] in strips
    ccl_mat W;
    int64_t strip, strips, stride;  // columns of a strip, their number, elements between them
    uint64_t bytes;                 // of W
};

ccl_status check_vocabulary(const char* who, const ccl_xent_desc* d, Vocabulary* v) {
    if (!d) return fail(CCL_ERR_INVALID_ARG, "%s: NULL descriptor", who);
    if (d->T <= 0 || d->V <= 0 || d->H <= 0) return fail(CCL_ERR_INVALID_ARG, "%s: T, V and H must be positive", who);
    if (d->T >= (INT64_C(1) << 31) - 256 || d->V >= (INT64_C(1) << 31) - 256 || d->H >= (INT64_C(1) << 31) - 256) return fail(CCL_ERR_UNSUPPORTED, "%s: dimension too large", who);
    if (d->H % 8) return fail(CCL_ERR_UNSUPPORTED, "%s: H (%lld) is not a multiple of 8", who, (long long)d->H);
    MatView w;
    ccl_status s = make_view(&d->W, who, &w);
    if (s) return s;
    if (w.rows != (d->w_trans ? d->V : d->H) || w.cols != (d->w_trans ? d->H : d->V)) return fail(CCL_ERR_SHAPE, "%s: W is not %s", who, d->w_trans ? "[V x H]" : "[H x V]");
    if (w.e != 2) return fail(CCL_ERR_UNSUPPORTED, "%s: only 2-byte (bf16) elements are supported", who);
    if (d->w_trans ? w.split != 0 : (w.split == 1 || w.ichunk || ragged(w) || w.w % 8 || w.stride % 8))
        return fail(CCL_ERR_UNSUPPORTED, "%s: W must be [V x H] row-major, or [H x V] in equal strips of a multiple of 8 columns", who);
    v->T = d->T; v->V = d->V; v->H = d->H; v->M = 2 * d->T <= kTwofoldRows ? 2 * d->T : d->T; v->trans = d->w_trans != 0; v->W = d->W;
    v->strip = w.w; v->strips = w.nstrips; v->stride = w.stride; v->bytes = (uint64_t)buffer_elems(w) * 2;
    return CCL_OK;
}

// `rows` rows over the whole vocabulary (logits, dz), kept in the strips that W has
ccl_mat strips_of(const Vocabulary& v, int64_t rows) {
    return v.strips > 1 ? ccl_mat{rows, v.V, 2, (int32_t)v.strips, CCL_PART_COLS, CCL_CCL, 0} : matrix(rows, v.V);
}
// The logits of `real` classes from one piece (all: of the whole of W); a row-major W is padded to whole 64s with classes that read as zeros
ccl_gemm_desc logits(const Vocabulary& v, int64_t rows, int64_t real, bool all) {
    const int64_t n = v.trans ? up(real, 64) : real;
    if (!v.trans && all) return product(rows, n, v.H, matrix(rows, v.H), 0, v.W, 0, strips_of(v, rows));
    return product(rows, n, v.H, matrix(rows, v.H), 0, v.trans ? matrix(n, v.H) : matrix(v.H, n), v.trans, matrix(rows, n));
}

int forward_lines(const GemmPlan& plan) { return plan.p.tiles_n * (plan.opw / 4); }

// The gradient's pieces of the vocabulary and the layout of its workspace
struct GradPlan {
    int64_t pieces, width;          // classes of a piece but the last
    bool all;                       // one piece that is the whole of W
    int64_t sums, sum_width;        // products that dX is the sum of, classes of each (1: one a piece, where there is one piece)
    bool direct;                    // dX is one product; otherwise it comes from
    int parts;                      //   as many fp32 sums
    size_t acc_at, x2_at, gemm_at, gemm_bytes, scale_at, bytes;
};

int64_t piece_real(const Vocabulary& v, const GradPlan& g, int64_t i) { return std::min(g.width, v.V - i * g.width); }
ccl_gemm_desc dx_product(const Vocabulary& v, const GradPlan& g, int64_t real) {
    const int64_t n = v.trans ? up(real, 64) : real;
    if (!v.trans && g.sums == 1) return product(v.M, v.H, n, strips_of(v, v.M), 0, v.W, 1, matrix(v.M, v.H));
    return product(v.M, v.H, n, matrix(v.M, n), 0, v.trans ? matrix(n, v.H) : matrix(v.H, n), v.trans ? 0 : 1, matrix(v.M, v.H));
}
ccl_gemm_desc dw_product(const Vocabulary& v, const GradPlan& g, int64_t real) {
    if (v.trans) {
        const int64_t n = up(real, 64);
        return product(n, v.H, v.M, matrix(v.M, n), 1, matrix(v.M, v.H), 0, matrix(n, v.H));
    }
    return product(v.H, real, v.M, matrix(v.M, v.H), 1, g.all ? strips_of(v, v.M) : matrix(v.M, real), 0, g.all ? v.W : matrix(v.H, real));
}

ccl_status make_grad_plan(const Vocabulary& v, GradPlan* g) {
    if (v.trans) {
        const int64_t most = std::max<int64_t>(256, kPieceBytes / (2 * v.M) / 256 * 256);
        g->pieces = (v.V + most - 1) / most;
        g->width = g->pieces == 1 ? v.V : up((v.V + g->pieces - 1) / g->pieces, 256);
        g->pieces = (v.V + g->width - 1) / g->width;
        g->all = g->pieces == 1;
        g->sums = g->pieces;
        g->sum_width = g->width;
    } else {
        g->all = v.strips == 1 || 2 * v.M * v.V <= kPieceBytes;
        g->pieces = g->all ? 1 : v.strips;
        g->width = g->all ? v.V : v.strip;
        // (strips along the K of dX's product have to be whole blocks of it; others are added up one by one, and so are all where dX comes from
        // fp32 sums anyway)
        g->sums = g->all && (v.strips == 1 || (v.strip % BK == 0 && v.M == v.T)) ? 1 : v.strips;
        g->sum_width = g->sums == 1 ? v.V : v.strip;
    }
    g->direct = g->sums == 1 && v.M == v.T;
    g->parts = 0;
    g->gemm_bytes = 0;
    ccl_status s;
    size_t n;
    const int64_t ends[2] = {piece_real(v, *g, 0), piece_real(v, *g, g->pieces - 1)};
    for (int64_t real : ends) {
        ccl_gemm_desc d = dw_product(v, *g, real);
        if ((s = ccl_gemm_workspace(&d, &n))) return s;
        g->gemm_bytes = std::max(g->gemm_bytes, n);
        d = dx_product(v, *g, std::min(real, g->sum_width));
        if (g->direct) {
            if ((s = ccl_gemm_workspace(&d, &n))) return s;
            g->gemm_bytes = std::max(g->gemm_bytes, n);
        } else {
            GemmPlan plan;
            if ((s = shape_plan(&d, 5, &plan))) return s;
            g->parts = std::max(g->parts, (int)plan.p.splits);
        }
    }
    const size_t dz = up256((size_t)v.M * (size_t)(v.trans ? up(g->width, 64) : g->width) * 2);
    g->acc_at = dz;
    g->x2_at = up256(dz + (size_t)g->parts * (size_t)v.M * (size_t)v.H * 4);
    g->gemm_at = up256(g->x2_at + (v.M == v.T ? 0 : (size_t)v.M * (size_t)v.H * 2));
    g->scale_at = up256(g->gemm_at + g->gemm_bytes);
    g->bytes = g->scale_at + 4;
    return CCL_OK;
}

// Plans of the gradient, by shape (four products planned cost 20 us)
struct GradKey {
    int64_t f[9];
    int dev;
    char env[60];
};
struct GradSlot {
    GradKey key;
    GradPlan plan;
    bool valid = false;
};
GradSlot g_grads[16];
int g_grads_next = 0;
std::mutex g_grads_mutex;

ccl_status plan_grad(const Vocabulary& v, GradPlan* g) {
    GradKey key;
    std::memset(&key, 0, sizeof(key));
    const int64_t f[9] = {v.T, v.V, v.H, v.trans, v.W.P, v.W.part, v.W.layout, v.W.strip_align_bytes, v.strips};
    std::memcpy(key.f, f, sizeof(f));
    key_surroundings(&key.dev, key.env, sizeof(key.env));
    {
        std::lock_guard<std::mutex> lock(g_grads_mutex);
        for (const GradSlot& s : g_grads)
            if (s.valid && std::memcmp(&s.key, &key, sizeof(key)) == 0) { *g = s.plan; return CCL_OK; }
    }
    ccl_status s = make_grad_plan(v, g);
    if (s) return s;
    std::lock_guard<std::mutex> lock(g_grads_mutex);
    g_grads[g_grads_next].key = key;
    g_grads[g_grads_next].plan = *g;
    g_grads[g_grads_next].valid = true;
    g_grads_next = (g_grads_next + 1) % 16;
    return CCL_OK;
}

ccl_status check_common(const char* who, const ccl_xent_desc* d, Vocabulary* v, const void* X, const void* W, const int32_t* targets) {
    ccl_status s = check_vocabulary(who, d, v);
    if (s) return s;
    if (!X || !W || !targets) return fail(CCL_ERR_INVALID_ARG, "%s: NULL operand", who);
    if (misaligned(X) || misaligned(W)) return fail(CCL_ERR_ALIGN, "%s: X / W is not 16-byte aligned", who);
    if (reinterpret_cast<uintptr_t>(targets) & 3) return fail(CCL_ERR_ALIGN, "%s: targets are not 4-byte aligned", who);
    return CCL_OK;
}
ccl_status check_workspace(const char* who, size_t need, const void* ws, size_t ws_bytes) {
    if (!ws || ws_bytes < need) return fail(CCL_ERR_WORKSPACE, "%s: needs %zu bytes of workspace (got %zu)", who, need, ws ? ws_bytes : (size_t)0);
    return misaligned(ws) ? fail(CCL_ERR_ALIGN, "%s: workspace is not 16-byte aligned", who) : CCL_OK;
}

}  // namespace

// The status word of this file's kernels, read and cleared (ccl_gemm_status)
ccl_status xent_status_take(int* code) {
    int zero = 0;
    CCL_CUDA_TRY(cudaMemcpyFromSymbol(code, g_gemm_status, sizeof(int)));
    if (*code) CCL_CUDA_TRY(cudaMemcpyToSymbol(g_gemm_status, &zero, sizeof(int)));
    return CCL_OK;
}

}  // namespace ccl

using namespace ccl;

static size_t forward_bytes(const GemmPlan& plan, int64_t T) { return up256((size_t)forward_lines(plan) * (size_t)T * 8) + (size_t)T * 4; }

extern "C" ccl_status ccl_linear_xent_workspace(const ccl_xent_desc* d, size_t* bytes) {
    Vocabulary v = {};
    ccl_status s = check_vocabulary("ccl_linear_xent_workspace", d, &v);
    if (s) return s;
    if (!bytes) return fail(CCL_ERR_INVALID_ARG, "ccl_linear_xent_workspace: NULL output");
    const ccl_gemm_desc g = logits(v, v.T, v.V, true);
    GemmPlan plan;
    if ((s = shape_plan(&g, 3, &plan))) return s;
    *bytes = forward_bytes(plan, v.T);
    return CCL_OK;
}

extern "C" ccl_status ccl_linear_xent(const ccl_xent_desc* d, const void* X_dev, const void* W_dev, const int32_t* targets_dev, float* loss_dev, float* lse_dev,
                                      void* ws_dev, size_t ws_bytes, void* cuda_stream) {
    const char* who = "ccl_linear_xent";
    Vocabulary v = {};
    ccl_status s = check_common(who, d, &v, X_dev, W_dev, targets_dev);
    if (s) return s;
    if (!loss_dev && !lse_dev) return fail(CCL_ERR_INVALID_ARG, "%s: no output is wanted", who);
    if ((reinterpret_cast<uintptr_t>(loss_dev) | reinterpret_cast<uintptr_t>(lse_dev)) & 3) return fail(CCL_ERR_ALIGN, "%s: loss / lse is not 4-byte aligned", who);
    const ccl_gemm_desc g = logits(v, v.T, v.V, true);
    GemmPlan plan;
    if ((s = shape_plan(&g, 3, &plan))) return s;
    if ((s = check_workspace(who, forward_bytes(plan, v.T), ws_dev, ws_bytes))) return s;
    const Span x = {X_dev, (uint64_t)v.T * v.H * 2}, w = {W_dev, v.bytes}, row = {targets_dev, (uint64_t)v.T * 4};
    const Span all[6] = {{ws_dev, forward_bytes(plan, v.T)}, {loss_dev, row.bytes}, {lse_dev, row.bytes}, x, w, row};
    for (int i = 0; i < 3; ++i)
        if (overlaps_any(all[i], all)) return fail(CCL_ERR_INVALID_ARG, "%s: loss, lse or the workspace lies over another buffer", who);
    EpiMaps<3> em = {};
    LogitArgs& la = em.logits;
    const int lines = forward_lines(plan);
    la.targets = targets_dev; la.ignore = d->ignore_index; la.classes = la.all = (int32_t)v.V;
    la.blocks = v.T <= BM ? kLogitBlocksFew : kLogitBlocks;
    la.part = static_cast<float2*>(ws_dev);
    la.at_target = reinterpret_cast<float*>(static_cast<char*>(ws_dev) + up256((size_t)lines * (size_t)v.T * 8));
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    if ((s = run_logits<3>(plan, em, v.trans ? v.V : 0, X_dev, W_dev, nullptr, st))) return s;
    // few rows side by side where there are few, and the more threads along the lines (1024 rows of 2048 lines: 80 us with 32 a block, on
    // 32 SMs; four are a whole sector of memory)
    int sms, pairs, lanes = 1;
    device_units(&sms, &pairs);
    while (lanes < 32 && lanes < v.T && (lanes < 4 || v.T > (int64_t)lanes * sms * 2)) lanes *= 2;
    return launch_early(xent_finish_kernel, dim3((unsigned)((v.T + lanes - 1) / lanes)), 256, 0, st, (const float2*)la.part, lines, (int)v.T, lanes, targets_dev,
                        la.ignore, la.classes, (const float*)la.at_target, loss_dev, lse_dev);
}

extern "C" ccl_status ccl_linear_xent_grad_workspace(const ccl_xent_desc* d, size_t* bytes) {
    Vocabulary v = {};
    ccl_status s = check_vocabulary("ccl_linear_xent_grad_workspace", d, &v);
    if (s) return s;
    if (!bytes) return fail(CCL_ERR_INVALID_ARG, "ccl_linear_xent_grad_workspace: NULL output");
    GradPlan g;
    if ((s = plan_grad(v, &g))) return s;
    *bytes = g.bytes;
    return CCL_OK;
}

extern "C" ccl_status ccl_linear_xent_grad(const ccl_xent_desc* d, const void* X_dev, const void* W_dev, const int32_t* targets_dev, const float* lse_dev,
                                           const float* dloss_dev, void* dX_dev, void* dW_dev, void* ws_dev, size_t ws_bytes, void* cuda_stream) {
    const char* who = "ccl_linear_xent_grad";
    Vocabulary v = {};
    ccl_status s = check_common(who, d, &v, X_dev, W_dev, targets_dev);
    if (s) return s;
    if (!lse_dev || !dloss_dev) return fail(CCL_ERR_INVALID_ARG, "%s: NULL operand", who);
    if (!dX_dev && !dW_dev) return fail(CCL_ERR_INVALID_ARG, "%s: no output is wanted", who);
    if (dX_dev == X_dev || dW_dev == W_dev) return fail(CCL_ERR_INVALID_ARG, "%s: a gradient needs a buffer of its own", who);
    if (misaligned(dX_dev) || misaligned(dW_dev)) return fail(CCL_ERR_ALIGN, "%s: dX / dW is not 16-byte aligned", who);
    if ((reinterpret_cast<uintptr_t>(lse_dev) | reinterpret_cast<uintptr_t>(dloss_dev)) & 3) return fail(CCL_ERR_ALIGN, "%s: lse / dloss is not 4-byte aligned", who);
    GradPlan g;
    if ((s = plan_grad(v, &g))) return s;
    if ((s = check_workspace(who, g.bytes, ws_dev, ws_bytes))) return s;
    const uint64_t x_bytes = (uint64_t)v.T * v.H * 2, row = (uint64_t)v.T * 4;
    const Span all[8] = {{ws_dev, g.bytes}, {dX_dev, x_bytes}, {dW_dev, v.bytes}, {X_dev, x_bytes}, {W_dev, v.bytes}, {targets_dev, row}, {lse_dev, row}, {dloss_dev, row}};
    for (int i = 0; i < 3; ++i)
        if (overlaps_any(all[i], all)) return fail(CCL_ERR_INVALID_ARG, "%s: dX, dW or the workspace lies over another buffer", who);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    char* ws = static_cast<char*>(ws_dev);
    void *dz = ws, *gemm_ws = g.gemm_bytes ? ws + g.gemm_at : nullptr;
    float *acc = reinterpret_cast<float*>(ws + g.acc_at), *scale = reinterpret_cast<float*>(ws + g.scale_at);
    int sms, pairs;
    device_units(&sms, &pairs);
    const bool twofold = v.M != v.T;
    const int64_t x8 = twofold ? v.T * v.H / 8 : 0;
    uint4* x2 = reinterpret_cast<uint4*>(ws + g.x2_at);
    if ((s = launch_early(xent_scale_kernel, dim3((unsigned)(1 + std::min<int64_t>((x8 + 1023) / 1024, sms))), 1024, 0, st, dloss_dev, targets_dev, (int)v.T, d->ignore_index,
                          (int32_t)v.V, scale, static_cast<const uint4*>(X_dev), x2, x8))) return s;
    const void* X = twofold ? static_cast<const void*>(x2) : X_dev;
    int have = 0;                                            // sums of dX that earlier pieces have begun
    for (int64_t i = 0; i < g.pieces; ++i) {
        const int64_t real = piece_real(v, g, i), rows = v.trans ? real : 0;
        const int64_t at = v.trans ? i * g.width * v.H : i * v.stride;
        const uint16_t* W = static_cast<const uint16_t*>(W_dev) + at;
        GemmPlan plan;
        ccl_gemm_desc p = logits(v, v.M, real, g.all);
        if ((s = shape_plan(&p, 4, &plan))) return s;
        EpiMaps<4> em = {};
        LogitArgs& la = em.logits;
        la.targets = targets_dev; la.ignore = d->ignore_index; la.v0 = (int32_t)(i * g.width); la.classes = (int32_t)real; la.all = (int32_t)v.V;
        la.lse = lse_dev; la.dloss = dloss_dev; la.scale = scale;
        la.half = twofold ? (int32_t)v.T : INT32_MAX;
        if ((s = run_logits<4>(plan, em, rows, X, W, dz, st))) return s;
        if (dX_dev) {
            p = dx_product(v, g, std::min(real, g.sum_width));
            if (g.direct) {
                if ((s = gemm_cut(&p, 0, rows, scale, dz, W, dX_dev, gemm_ws, g.gemm_bytes, cuda_stream))) return s;
            } else {
                // (the piece's dz and W; or one of their strips after the other)
                for (int64_t k = 0; k < (g.all ? g.sums : 1); ++k) {
                    if ((s = shape_plan(&p, 5, &plan))) return s;
                    EpiMaps<5> sums = {acc, have};
                    if ((s = run_logits<5>(plan, sums, rows, static_cast<uint16_t*>(dz) + k * v.M * v.strip, W + k * v.stride, nullptr, st))) return s;
                    have = std::max(have, (int)plan.p.splits);
                }
            }
        }
        if (dW_dev) {
            p = dw_product(v, g, real);
            const void *A = v.trans ? dz : X, *B = v.trans ? X : dz;
            uint16_t* C = static_cast<uint16_t*>(dW_dev) + at;
            // Enough tiles for every SM: 256 columns, drained behind the next tile's product (131072 x 512 x 1024: 105 us, by ccl_gemm with
            // alpha 114; 32768 x 4096 x 1024: 196 and 215).  Few tiles and a long K are split along K.
            if (((p.M + BM - 1) / BM) * ((p.N + 255) / 256) >= sms) {
                if ((s = shape_plan(&p, 6, &plan))) return s;
                EpiMaps<6> by = {scale};
                if ((s = run_logits<6>(plan, by, 0, A, B, C, st, rows))) return s;
            } else if ((s = gemm_cut(&p, rows, 0, scale, A, B, C, gemm_ws, g.gemm_bytes, cuda_stream))) return s;
        }
    }
    if (!dX_dev || g.direct) return CCL_OK;
    if (twofold) have *= 2;                                  // (a sum's second half of rows is a sum more)
    const int64_t n = v.T * v.H;
    return launch_early(xent_dx_kernel, dim3((unsigned)std::min<int64_t>((n / 8 + 255) / 256, sms * 8)), 256, 0, st, (const float*)acc, have, n, (const float*)scale, static_cast<uint16_t*>(dX_dev));
}
