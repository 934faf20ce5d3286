// Launching the GEMM kernels with an operator in their epilogue: shared by ccl_gemm_epi.cu and ccl_xent.cu.
#ifndef CCL_GEMM_EPI_CUH_
#define CCL_GEMM_EPI_CUH_

#include "ccl_gemm_kernel.cuh"
#include "ccl_gemm_plan.cuh"
#include "ccl_launch.cuh"

namespace ccl {

template <int BN, int CTAS, bool FULL, int KS, int EPI, int OPW>
static ccl_status launch_epi_warps(const GemmPlan& plan, const CUtensorMap* maps, const EpiMaps<EPI>& em, cudaStream_t st) {
    auto kernel = ccl_gemm_kernel<BN, CTAS, false, 0, FULL, KS, EPI, OPW>;
    static std::atomic<uint64_t> configured{0};                 // bit per device: the shared-memory limit has been raised
    int dev = 0;
    CCL_CUDA_TRY(cudaGetDevice(&dev));
    if (dev >= 64 || !(configured.load() >> dev & 1)) {
        CCL_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(smem_budget_op(KS, OPW, EPI) + staging_bytes<EPI, KS, OPW> + 2048)));
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

static ccl_status encode_maps(const GemmPlan& plan, const void* A, const void* B, void* C, CUtensorMap* m) {
    const GemmParams& p = plan.p;
    const uint32_t bnh = (uint32_t)(plan.subn / plan.ctas);   // B rows of one K-major box
    struct { const MatView* v; const void* base; uint32_t inner, rows; } op[3] = {
        {&plan.va, A, p.a_mn ? 64u : (uint32_t)BK, p.a_mn ? (uint32_t)BK : (uint32_t)plan.a_box_rows},
        {&plan.vb, B, p.b_mn ? 64u : (uint32_t)BK, p.b_mn ? (uint32_t)BK : bnh},
        {&plan.vc, C, 64u, 32u}};
    for (int X = 0; X < 3; ++X) {
        if (!op[X].base) { m[X] = m[3 + X] = m[0]; continue; }   // (no C: what the drain leaves goes elsewhere)
        ccl_status s = operand_tmap(&m[X], *op[X].v, op[X].base, op[X].inner, op[X].rows, 1, 0);
        if (s) return s;
        m[3 + X] = m[X];
        if (ragged(*op[X].v) && (s = operand_tmap(&m[3 + X], *op[X].v, op[X].base, op[X].inner, op[X].rows, 1, 0, true))) return s;
    }
    return CCL_OK;
}

static bool misaligned(const void* p) { return reinterpret_cast<uintptr_t>(p) & 15; }

// ---- plans, by shape ---------------------------------------------------------------------------------------------
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
static ShapePlan g_shapes[kShapeSlots];
static int g_shapes_next = 0;
static std::mutex g_shapes_mutex;

// What else a plan depends on: the device and the planner's switches (`env` comes cleared)
static void key_surroundings(int* dev, char* env, size_t size) {
    *dev = -1;
    if (cudaGetDevice(dev) != cudaSuccess) (void)cudaGetLastError();
    size_t pos = 0;
    for (const char* name : {"CCL_GEMM_CTAS", "CCL_GEMM_BN", "CCL_GEMM_SPLITK", "CCL_GEMM_BALANCED", "CCL_GEMM_CLUSTERK"}) {
        const char* v = std::getenv(name);
        for (const char* c = v ? v : ""; *c && pos + 2 < size; ++c) env[pos++] = *c;
        if (pos + 1 < size) env[pos++] = ';';
    }
}
static void shape_key(const ccl_gemm_desc* d, int epi, ShapeKey* k) {
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
    key_surroundings(&k->dev, k->env, sizeof(k->env));
}

// Validates the descriptor and finds or makes its plan (a B200's unit counts when no device can be asked).
static ccl_status shape_plan(const ccl_gemm_desc* d, int epi, GemmPlan* out) {
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

}  // namespace ccl

#endif  // CCL_GEMM_EPI_CUH_
