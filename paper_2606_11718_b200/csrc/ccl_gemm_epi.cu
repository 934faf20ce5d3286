// ccl_gemm_epilogue: C = act(A B + bias) + residual, and ccl_gemm_act_grad: dZ = (A B) * act'(Z) with the column sums of dZ --
// the GEMM of ccl_gemm with more in its epilogue.  The kernel, its tile shapes, K splits and layouts are those of ccl_gemm
// (ccl_gemm_kernel.cuh, EPI = 1 and 2); this file instantiates, plans and launches them.
//
// A plan is kept per problem shape and layout, never by a buffer's address: the tensor maps, which hold addresses, are
// encoded for every call (three to six of them, ~0.2 us each on the host).
#include "ccl_gemm_kernel.cuh"
#include "ccl_gemm_plan.cuh"

namespace ccl {

template <int BN, int CTAS, bool FULL, int KS, int EPI, int OPW>
static ccl_status launch_epi_warps(const GemmPlan& plan, const CUtensorMap* maps, const EpiMaps<EPI>& em, cudaStream_t st) {
    auto kernel = ccl_gemm_kernel<BN, CTAS, false, 0, FULL, KS, EPI, OPW>;
    static std::atomic<uint64_t> configured{0};                 // bit per device: the shared-memory limit has been raised
    int dev = 0;
    CCL_CUDA_TRY(cudaGetDevice(&dev));
    if (dev >= 64 || !(configured.load() >> dev & 1)) {
        CCL_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(smem_budget_op(KS, OPW) + staging_bytes<EPI, KS, OPW> + 2048)));
        if (dev < 64) configured.fetch_or(1ull << dev);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(plan.grid, 1, 1);
    cfg.blockDim = dim3(gemm_threads<EPI, OPW>, 1, 1);
    cfg.dynamicSmemBytes = plan.smem_bytes;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = KS ? KS : CTAS; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    static const bool pdl = []() { const char* f = std::getenv("CCL_GEMM_PDL"); return !f || atoi(f) != 0; }();
    if (pdl) {                                                  // as for ccl_gemm: set-up overlaps the previous kernel's tail
        attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[1].val.programmaticStreamSerializationAllowed = 1;
        cfg.numAttrs = 2;
    }
    CCL_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, maps[0], maps[1], maps[2], maps[3], maps[4], maps[5], plan.p, em));
    count_launch();
    return CCL_OK;
}

template <int BN, int CTAS, bool FULL, int KS, int EPI>
static ccl_status launch_epi(const GemmPlan& plan, const CUtensorMap* maps, const EpiMaps<EPI>& em, cudaStream_t st) {
    if constexpr (KS != 0) return launch_epi_warps<BN, CTAS, FULL, KS, EPI, 16>(plan, maps, em, st);
    else if constexpr (FULL) return launch_epi_warps<BN, CTAS, FULL, KS, EPI, 8>(plan, maps, em, st);
    else return plan.opw == 16 ? launch_epi_warps<BN, CTAS, FULL, KS, EPI, 16>(plan, maps, em, st) : launch_epi_warps<BN, CTAS, FULL, KS, EPI, 8>(plan, maps, em, st);
}

template <int EPI>
static ccl_status launch_variant(const GemmPlan& plan, const CUtensorMap* maps, const EpiMaps<EPI>& em, cudaStream_t st) {
    if (plan.ks) {
        switch (plan.bn * 10 + plan.ks) {
            case 2562: return launch_epi<256, 1, false, 2, EPI>(plan, maps, em, st);
            case 2564: return launch_epi<256, 1, false, 4, EPI>(plan, maps, em, st);
            case 2568: return launch_epi<256, 1, false, 8, EPI>(plan, maps, em, st);
            case 1922: return launch_epi<192, 1, false, 2, EPI>(plan, maps, em, st);
            case 1924: return launch_epi<192, 1, false, 4, EPI>(plan, maps, em, st);
            case 1928: return launch_epi<192, 1, false, 8, EPI>(plan, maps, em, st);
            case 1282: return launch_epi<128, 1, false, 2, EPI>(plan, maps, em, st);
            case 1284: return launch_epi<128, 1, false, 4, EPI>(plan, maps, em, st);
            default: return launch_epi<128, 1, false, 8, EPI>(plan, maps, em, st);
        }
    }
    if (!plan.lean) {                                           // (make_plan offers these two widths only)
        if (plan.ctas == 2) return plan.bn == 256 ? launch_epi<256, 2, true, 0, EPI>(plan, maps, em, st) : launch_epi<128, 2, true, 0, EPI>(plan, maps, em, st);
        return plan.bn == 256 ? launch_epi<256, 1, true, 0, EPI>(plan, maps, em, st) : launch_epi<128, 1, true, 0, EPI>(plan, maps, em, st);
    }
    switch (plan.bn * 10 + plan.ctas) {
        case 2562: return launch_epi<256, 2, false, 0, EPI>(plan, maps, em, st);
        case 1922: return launch_epi<192, 2, false, 0, EPI>(plan, maps, em, st);
        case 1282: return launch_epi<128, 2, false, 0, EPI>(plan, maps, em, st);
        case 2561: return launch_epi<256, 1, false, 0, EPI>(plan, maps, em, st);
        case 1921: return launch_epi<192, 1, false, 0, EPI>(plan, maps, em, st);
        default: return launch_epi<128, 1, false, 0, EPI>(plan, maps, em, st);
    }
}

// Sum of the K splits' partial sums (in the order of k), then the epilogue: a block takes 32 rows x 64 columns, a thread 8
// columns of a row.  Column sums of the block go to its line of the partial sums, as in the GEMM kernel.
template <int EPI>
static __global__ void __launch_bounds__(256) splitk_epilogue_kernel(const GemmParams p) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");            // the GEMM has completed
    const int row = blockIdx.y * 32 + (threadIdx.x >> 3), n = blockIdx.x * 64 + (threadIdx.x & 7) * 8;
    const bool ok = row < p.M && n < p.N;
    const int r = min(row, p.M - 1), c = min(n, p.N - 8);
    const int64_t off = c_offset(p, r, c);
    const uint4 x8 = ld_global_v4_if(p.addend + off, ok && p.addend), b8 = ld_global_v4_if(p.bias + c, EPI == 1 && ok && p.bias);
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.0f;
    for (int sp = 0; sp < p.splits; ++sp) {
        const float4* src = reinterpret_cast<const float4*>(p.ws + ((int64_t)sp * p.M + r) * p.N + c);
        const float4 x = src[0], y = src[1];
        v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
        v[4] += y.x; v[5] += y.y; v[6] += y.z; v[7] += y.w;
    }
    epilogue8<EPI>(p, v, off, ok, x8, b8);
    st_global_v4_if(p.C + off, bf16x8_pack(v), ok);
    if (EPI == 2 && p.colsum) {
        __shared__ float part[32][64 + 4];
#pragma unroll
        for (int i = 0; i < 8; ++i) part[threadIdx.x >> 3][(threadIdx.x & 7) * 8 + i] = v[i];
        __syncthreads();
        const int col = blockIdx.x * 64 + threadIdx.x;
        if (threadIdx.x < 64 && col < p.N) {
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < 32; ++i) s += part[i][threadIdx.x];
            p.colsum[(int64_t)blockIdx.y * p.N + col] = s;
        }
    }
}

// dbias[n] = bf16(sum over the row blocks of partial[block][n]): 32 columns a block, eight warps over the row blocks, their
// sums added in a fixed order.  Reads blocks x N floats once (4 bytes for every 64 of dZ).
__global__ void __launch_bounds__(256) column_sum_finish_kernel(const float* partial, int blocks, int N, uint16_t* dbias) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");            // the kernel that writes the partial sums has completed
    __shared__ float part[8][32];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, n = blockIdx.x * 32 + lane;
    float s = 0.0f;
    if (n < N)
#pragma unroll 16                                        // (sixteen loads in flight: the time is a trip or two to the L2)
        for (int b = w; b < blocks; b += 8) s += partial[(int64_t)b * N + n];
    part[w][lane] = s;
    __syncthreads();
    if (w == 0 && n < N) {
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += part[i][lane];
        reinterpret_cast<__nv_bfloat16*>(dbias)[n] = __float2bfloat16_rn(s);
    }
}

// A kernel of this file behind the GEMM: placed early (its CTAs wait for the GEMM's completion themselves)
template <typename... Params, typename... Args>
static ccl_status launch_behind(void (*kernel)(Params...), dim3 grid, cudaStream_t st, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(256, 1, 1);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    CCL_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, args...));
    count_launch();
    return CCL_OK;
}

// ---- plans, by shape ---------------------------------------------------------------------------------------------
namespace {
struct ShapeKey {
    int64_t f[30];
    int dev, epi;
    char env[60];
};
struct ShapePlan {
    ShapeKey key;
    GemmPlan plan;
    bool valid = false;
};
constexpr int kShapeSlots = 64;
ShapePlan g_shapes[kShapeSlots];
int g_shapes_next = 0;
std::mutex g_shapes_mutex;

void shape_key(const ccl_gemm_desc* d, int epi, ShapeKey* k) {
    std::memset(k, 0, sizeof(*k));
    int64_t* f = k->f;
    f[0] = d->M; f[1] = d->N; f[2] = d->K;
    const ccl_mat* ms[3] = {&d->A, &d->B, &d->C};
    for (int X = 0; X < 3; ++X) {
        int64_t* g = f + 3 + 7 * X;
        g[0] = ms[X]->rows; g[1] = ms[X]->cols; g[2] = ms[X]->elem_bytes; g[3] = ms[X]->P; g[4] = ms[X]->part; g[5] = ms[X]->layout; g[6] = ms[X]->strip_align_bytes;
    }
    f[24] = d->a_trans; f[25] = d->b_trans; f[26] = d->out_part; f[27] = d->P; f[28] = d->grouped_raster;
    f[29] = d->out_part == CCL_PART_2D ? d->part_m : 0;
    k->epi = epi;
    k->dev = -1;
    if (cudaGetDevice(&k->dev) != cudaSuccess) (void)cudaGetLastError();
    size_t pos = 0;
    for (const char* name : {"CCL_GEMM_CTAS", "CCL_GEMM_BN", "CCL_GEMM_SPLITK", "CCL_GEMM_CLUSTERK"}) {
        const char* v = std::getenv(name);
        for (const char* c = v ? v : ""; *c && pos + 2 < sizeof(k->env); ++c) k->env[pos++] = *c;
        if (pos + 1 < sizeof(k->env)) k->env[pos++] = ';';
    }
}

// Validates the descriptor and finds or makes its plan (a B200's unit counts when no device can be asked).
ccl_status shape_plan(const ccl_gemm_desc* d, int epi, GemmPlan* out) {
    if (!d) return fail(CCL_ERR_INVALID_ARG, "ccl_gemm: NULL descriptor");
    ShapeKey key;
    shape_key(d, epi, &key);
    {
        std::lock_guard<std::mutex> lock(g_shapes_mutex);
        for (const ShapePlan& s : g_shapes)
            if (s.valid && std::memcmp(&s.key, &key, sizeof(key)) == 0) { *out = s.plan; return CCL_OK; }
    }
    ShapePlan made;
    ccl_status s = make_plan(d, 1, false, nullptr, nullptr, nullptr, 148, 74, &made.plan, 0, false, 0, false, epi);   // validation: no CUDA call on bad input
    if (s) return s;
    int sms, pairs;
    const bool have_device = device_units(&sms, &pairs);
    if ((s = make_plan(d, 1, false, nullptr, nullptr, nullptr, sms, pairs, &made.plan, 0, false, 0, have_device, epi))) return s;
    const GemmParams& q = made.plan.p;
    const bool ks = (q.a_mn ? q.a.split == 1 : q.a.split == 2) || (q.b_mn ? q.b.split == 1 : q.b.split == 2);
    made.plan.lean = q.group_dim != 2 && !q.a.il_mode && !q.b.il_mode && !q.c.il_mode && !ks && !q.a.rag && !q.b.rag && !q.c.rag;
    made.key = key; made.valid = true;
    *out = made.plan;
    std::lock_guard<std::mutex> lock(g_shapes_mutex);
    g_shapes[g_shapes_next] = made;
    g_shapes_next = (g_shapes_next + 1) % kShapeSlots;
    return CCL_OK;
}

// Row blocks of the partial column sums: 32 rows each, of every tile row that has rows (whole tiles) or of the matrix (K split).
// Tile rows are numbered strip by strip, tps_m to a strip; a last strip that is lower than the others may have fewer, and the places
// behind its last one, which are the last of all, are skipped by the kernel: their sums are never written.
int64_t row_blocks(const GemmPlan& plan) {
    const GemmParams& p = plan.p;
    if (p.splits > 1) return ((int64_t)p.M + 31) / 32;
    const int64_t strips = ((int64_t)p.M + p.Wm - 1) / p.Wm, tile = (int64_t)BM * plan.ctas, last = (int64_t)p.M - (strips - 1) * p.Wm;
    return ((strips - 1) * p.tps_m + (last + tile - 1) / tile) * 4 * plan.ctas;
}
size_t partial_sums_at(const GemmPlan& plan) { return (plan.ws_bytes + 255) & ~(size_t)255; }

// A matrix laid out like C, in C's boxes: its map, and that of its last strip
ccl_status encode_like_c(const GemmPlan& plan, const void* base, CUtensorMap* m, CUtensorMap* m2) {
    ccl_status s = operand_tmap(m, plan.vc, base, 64, 32, 1, 0);
    if (s) return s;
    *m2 = *m;
    return ragged(plan.vc) ? operand_tmap(m2, plan.vc, base, 64, 32, 1, 0, true) : CCL_OK;
}

template <int EPI>
ccl_status launch_with_maps(const GemmPlan& plan, const CUtensorMap* maps, cudaStream_t st) {
    EpiMaps<EPI> em;
    ccl_status s;
    std::memset(&em, 0, sizeof(em));
    if (plan.p.addend && (s = encode_like_c(plan, plan.p.addend, &em.addend, &em.addend2))) return s;
    return launch_variant<EPI>(plan, maps, em, st);
}

ccl_status encode_maps(const GemmPlan& plan, const void* A, const void* B, void* C, CUtensorMap* m) {
    const GemmParams& p = plan.p;
    const uint32_t bnh = (uint32_t)(plan.subn / plan.ctas);   // B rows of one K-major box
    struct { const MatView* v; const void* base; uint32_t inner, rows; } op[3] = {
        {&plan.va, A, p.a_mn ? 64u : (uint32_t)BK, p.a_mn ? (uint32_t)BK : (uint32_t)plan.a_box_rows},
        {&plan.vb, B, p.b_mn ? 64u : (uint32_t)BK, p.b_mn ? (uint32_t)BK : bnh},
        {&plan.vc, C, 64u, 32u}};
    for (int X = 0; X < 3; ++X) {
        ccl_status s = operand_tmap(&m[X], *op[X].v, op[X].base, op[X].inner, op[X].rows, 1, 0);
        if (s) return s;
        m[3 + X] = m[X];
        if (ragged(*op[X].v) && (s = operand_tmap(&m[3 + X], *op[X].v, op[X].base, op[X].inner, op[X].rows, 1, 0, true))) return s;
    }
    return CCL_OK;
}

bool misaligned(const void* p) { return reinterpret_cast<uintptr_t>(p) & 15; }

// `epi` 1: bias / residual / preact; 2: addend = Z, dbias
ccl_status run_epi(const char* who, int epi, const ccl_gemm_desc* d, int act, const void* bias, const void* addend, void* preact, void* dbias,
                   const void* A, const void* B, void* C, void* ws, size_t ws_bytes, void* cuda_stream) {
    if (!A || !B || !C) return fail(CCL_ERR_INVALID_ARG, "%s: NULL operand", who);
    if (act < CCL_ACT_NONE || act > CCL_ACT_SILU) return fail(CCL_ERR_INVALID_ARG, "%s: unknown activation %d", who, act);
    if (epi == 2 && act != CCL_ACT_NONE && !addend) return fail(CCL_ERR_INVALID_ARG, "%s: NULL pre-activation", who);
    GemmPlan plan;
    ccl_status s = shape_plan(d, epi, &plan);
    if (s) return s;
    if (misaligned(A) || misaligned(B) || misaligned(C) || misaligned(bias) || misaligned(addend) || misaligned(preact))
        return fail(CCL_ERR_ALIGN, "%s: a base pointer is not 16-byte aligned", who);
    if (reinterpret_cast<uintptr_t>(dbias) & 1) return fail(CCL_ERR_ALIGN, "%s: dbias is not 2-byte aligned", who);
    if (preact && (preact == C || preact == addend)) return fail(CCL_ERR_INVALID_ARG, "%s: the pre-activation needs a buffer of its own", who);
    GemmParams& p = plan.p;
    const size_t sums_at = partial_sums_at(plan), need = dbias ? sums_at + (size_t)row_blocks(plan) * (size_t)p.N * 4 : plan.ws_bytes;
    if (need) {
        if (!ws || ws_bytes < need) return fail(CCL_ERR_WORKSPACE, "%s: needs %zu bytes of workspace (got %zu)", who, need, ws ? ws_bytes : (size_t)0);
        if (misaligned(ws)) return fail(CCL_ERR_ALIGN, "%s: workspace is not 16-byte aligned", who);
    }
    CUtensorMap maps[6];
    if ((s = encode_maps(plan, A, B, C, maps))) return s;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    p.C = static_cast<uint16_t*>(C);
    p.alpha = 1.0f;
    p.ws = static_cast<float*>(ws);
    p.act = act;
    p.bias = static_cast<const uint16_t*>(bias);
    p.addend = epi == 2 && act == CCL_ACT_NONE ? nullptr : static_cast<const uint16_t*>(addend);
    p.preact = static_cast<uint16_t*>(preact);
    p.addend_tma = p.c.il_mode != 3;
    p.colsum = dbias ? reinterpret_cast<float*>(static_cast<char*>(ws) + sums_at) : nullptr;
    if ((s = wave_barrier(plan, true, st))) return s;
    if ((s = epi == 1 ? launch_with_maps<1>(plan, maps, st) : launch_with_maps<2>(plan, maps, st))) return s;
    if (p.splits > 1) {
        const dim3 grid((unsigned)((p.N + 63) / 64), (unsigned)((p.M + 31) / 32));
        if ((s = epi == 1 ? launch_behind(splitk_epilogue_kernel<1>, grid, st, p) : launch_behind(splitk_epilogue_kernel<2>, grid, st, p))) return s;
    }
    if (!dbias) return CCL_OK;
    return launch_behind(column_sum_finish_kernel, dim3((unsigned)((p.N + 31) / 32)), st, (const float*)p.colsum, (int)row_blocks(plan), (int)p.N, static_cast<uint16_t*>(dbias));
}
}  // namespace

// The status word of this file's kernels, read and cleared (ccl_gemm_status)
ccl_status epi_status_take(int* code) {
    int zero = 0;
    CCL_CUDA_TRY(cudaMemcpyFromSymbol(code, g_gemm_status, sizeof(int)));
    if (*code) CCL_CUDA_TRY(cudaMemcpyToSymbol(g_gemm_status, &zero, sizeof(int)));
    return CCL_OK;
}

}  // namespace ccl

using namespace ccl;

extern "C" ccl_status ccl_gemm_epilogue_workspace(const ccl_gemm_desc* d, size_t* bytes) {
    GemmPlan plan;
    ccl_status s = shape_plan(d, 1, &plan);
    if (s) return s;
    if (!bytes) return fail(CCL_ERR_INVALID_ARG, "ccl_gemm_epilogue_workspace: NULL output");
    *bytes = plan.ws_bytes;
    return CCL_OK;
}

extern "C" ccl_status ccl_gemm_epilogue(const ccl_gemm_desc* d, const ccl_epilogue* e, const void* A_dev, const void* B_dev, void* C_dev, void* ws_dev,
                                        size_t ws_bytes, void* cuda_stream) {
    if (!e) return fail(CCL_ERR_INVALID_ARG, "ccl_gemm_epilogue: NULL epilogue");
    return run_epi("ccl_gemm_epilogue", 1, d, e->act, e->bias_dev, e->residual_dev, e->preact_dev, nullptr, A_dev, B_dev, C_dev, ws_dev, ws_bytes, cuda_stream);
}

extern "C" ccl_status ccl_gemm_act_grad_workspace(const ccl_gemm_desc* d, size_t* bytes) {
    GemmPlan plan;
    ccl_status s = shape_plan(d, 2, &plan);
    if (s) return s;
    if (!bytes) return fail(CCL_ERR_INVALID_ARG, "ccl_gemm_act_grad_workspace: NULL output");
    *bytes = partial_sums_at(plan) + (size_t)row_blocks(plan) * (size_t)plan.p.N * 4;
    return CCL_OK;
}

extern "C" ccl_status ccl_gemm_act_grad(const ccl_gemm_desc* d, int32_t act, const void* A_dev, const void* B_dev, const void* Z_dev, void* dZ_dev,
                                        void* dbias_dev, void* ws_dev, size_t ws_bytes, void* cuda_stream) {
    return run_epi("ccl_gemm_act_grad", 2, d, act, nullptr, Z_dev, nullptr, dbias_dev, A_dev, B_dev, dZ_dev, ws_dev, ws_bytes, cuda_stream);
}
