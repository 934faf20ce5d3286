// ccl_moe_tokens: a mixture-of-experts feed-forward layer for a few tokens -- router, top-k, gated expert products and the
// weighted sum -- in one cooperative launch of one CTA per SM.
//
// Bound by memory: every chosen expert's weights are read once (3 H I elements each) and nothing else is of that order; with
// m tokens an expert the arithmetic is 2 m flops per 2-byte weight, far below what the tensor cores take.  So the kernel is a
// stream of weight rows through a shared-memory ring, filled by bulk copies that never wait for anything but a free slot:
//   1. router: the CTAs share the E x T dot products; first meeting of the grid; every CTA then works out the same top-k and the
//      same lists of tokens per expert by itself
//   2. gate and up: the (expert, 8 features) units are shared out evenly.  A unit is 16 weight rows -- 8 gate, 8 up -- times
//      its expert's tokens (n = 8 columns): one m16n8k16 accumulator then holds the gate and the up value of a
//      feature in the same lane, and silu(gate) * up needs no exchange.  h goes to the workspace; second meeting
//   3. down: a CTA owns a few rows of Wd (H / #SMs of them, at most 16) and takes every chosen expert's: the sum over a token's
//      experts stays inside the CTA, in a fixed order, and Y is written once.  The ring is filled with phase 3's
//      weights while phase 2's last units and the meeting are still going on: the stream does not stop there.
// Warp roles: 8 consumer warps split every slot's k range between them; warp 8 fills the weight ring; warp 9 waits for the
// second meeting and fills the (small) ring of h rows.
//
// The matrix instructions are mma.sync: with n = 8 columns a tcgen05 tile would be 128 rows high and leave most SMs without
// work for one token; they are nowhere near their limit here.  Weights and tokens are both K-contiguous, so a lane may take any 8
// consecutive k as its share of two k steps as long as both operands do: 16-byte shared-memory loads, no ldmatrix, and a
// row pitch of 64 bytes more than a multiple of 128 keeps them free of bank conflicts.
#include <algorithm>
#include <atomic>
#include <chrono>

#include "ccl_act.cuh"
#include "ccl_tma.h"

namespace ccl {

constexpr int kMoeConsumers = 8;                         // warps
constexpr int kMoeThreads = (kMoeConsumers + 2) * 32;
constexpr int kMoeK = 512;                               // k elements of a slot
constexpr int kMoePitch = kMoeK * 2 + 64;                // bytes between the rows of a slot
constexpr int kMoeSlot = 16 * kMoePitch;
constexpr int kMoeMaxSlots = 12, kMoeMaxHSlots = 8;
constexpr int64_t kMoeMaxT = 64, kMoeMaxE = 512, kMoeMaxK = 16;

static __device__ int g_moe_status = 0;

struct MoeParams {
    int32_t T, H, I, E, topk, norm;
    int32_t gu_half, gu_strip;              // gate rows of a strip; rows of a strip
    int64_t gu_stride, d_stride;            // bytes from one expert to the next
    const uint16_t *x, *wr, *residual;
    const unsigned char *wgu, *wd;
    uint16_t* y;
    int32_t* ids;
    float* weights;
    float* logits;                          // workspace: [T][E]
    unsigned long long* flags;              // workspace: [2 meetings][CTAs]
    unsigned char* h;                       // workspace: [pairs][h_pitch bytes] bf16
    int64_t h_pitch;
    unsigned long long mark;                // this launch's mark in the flags
    int32_t group;                          // tokens of an expert taken together (8, 16 or 32 columns)
    int32_t slots, h_slots;
    int32_t x_pitch;                        // bytes between the token rows in shared memory
    int32_t rows_per_block, blocks;         // phase 3: rows of Wd a CTA takes at a time, such blocks in all
    // byte offsets in shared memory
    int32_t at_region, at_hring, at_red, at_mask, at_off, at_ent, at_tok, at_wt, at_sel, at_selw, at_bars;
};

__device__ __forceinline__ void bar_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void mma_16x8x16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void st_release_u64(unsigned long long* p, unsigned long long v) {
    asm volatile("st.release.gpu.global.u64 [%0], %1;" ::"l"(p), "l"(v) : "memory");
}
__device__ __forceinline__ unsigned long long ld_acquire_flag(const unsigned long long* p) {
    unsigned long long v;
    asm volatile("ld.acquire.gpu.global.u64 %0, [%1];" : "=l"(v) : "l"(p) : "memory");
    return v;
}
// One warp waits (bounded) until every CTA has set its flag to `mark`.
__device__ __forceinline__ bool meet(const unsigned long long* flags, int ctas, unsigned long long mark, int lane) {
    bool ok = true;
    const uint64_t t0 = global_timer_ns();
    for (int i = lane; ok && i < ctas; i += 32)
        for (uint32_t n = 1; ld_acquire_flag(flags + i) != mark; ++n)
            if ((n & 255u) == 0 && global_timer_ns() - t0 > kWaitLimitNs) { ok = false; break; }
    return __all_sync(0xffffffffu, ok);
}

// Order-preserving integer image of a float; NaN below every number, 0 is left for "taken".
__device__ __forceinline__ uint32_t order_key(float f) {
    if (f != f) return 1u;
    const uint32_t u = __float_as_uint(f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// The 32-element k steps of a slot that belong to this warp: acc += W[16 rows] * B[columns], both in shared memory at `w` (row
// pitch kMoePitch) and `b`.  kc: valid k elements of the slot (a multiple of 8; both operands read as zero behind it); cols:
// columns that exist (zero behind them; nothing is read there).
template <int NT>
__device__ __forceinline__ void slot_product(float (&acc)[NT][4], uint32_t w, uint32_t b, int b_pitch, int kc, int cols, int warp, int lane) {
    const int g = lane >> 2, q = lane & 3;
#pragma unroll
    for (int st = 0; st < kMoeK / 32 / kMoeConsumers; ++st) {
        const int k = (st * kMoeConsumers + warp) * 32;
        if (k >= kc) break;
        const int kq = k + q * 8;
        const bool ok = kq < kc;
        const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
        const uint4 lo = ok ? lds128(w + g * kMoePitch + kq * 2) : zero, hi = ok ? lds128(w + (g + 8) * kMoePitch + kq * 2) : zero;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            if (n * 8 >= cols) break;
            const uint4 t = ok && n * 8 + g < cols ? lds128(b + (n * 8 + g) * b_pitch + kq * 2) : zero;
            mma_16x8x16(acc[n], lo.x, hi.x, lo.y, hi.y, t.x, t.y);
            mma_16x8x16(acc[n], lo.z, hi.z, lo.w, hi.w, t.z, t.w);
        }
    }
}

// NT: most column groups of 8 an expert's tokens are taken in
template <int NT>
__global__ void __launch_bounds__(kMoeThreads, 1) moe_tokens_kernel(const __grid_constant__ MoeParams p) {
    extern __shared__ __align__(128) unsigned char smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, cta = blockIdx.x, ctas = gridDim.x;
    constexpr int kConsumerThreads = kMoeConsumers * 32;
    unsigned long long* mask = reinterpret_cast<unsigned long long*>(smem + p.at_mask);      // per expert: the tokens that chose it
    uint16_t* off = reinterpret_cast<uint16_t*>(smem + p.at_off);                            // per expert: its first pair
    uint32_t* ent = reinterpret_cast<uint32_t*>(smem + p.at_ent);                            // entries: expert | first pair << 9 | columns << 20
    uint8_t* tok = smem + p.at_tok;                                                          // per pair (by expert): token
    float* wt = reinterpret_cast<float*>(smem + p.at_wt);                                    // ... and its weight
    uint16_t* sel = reinterpret_cast<uint16_t*>(smem + p.at_sel);                            // per (token, choice): expert
    float* selw = reinterpret_cast<float*>(smem + p.at_selw);
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + p.at_bars);
    uint64_t *wfull = bars, *wempty = wfull + p.slots, *hfull = wempty + p.slots, *hempty = hfull + p.h_slots, *rfull = hempty + p.h_slots, *rempty = rfull + 2;
    int* shared = reinterpret_cast<int*>(rempty + 2);                                        // [0] entries, [1] gave up
    const uint32_t ring0 = smem_u32(smem), x0 = smem_u32(smem + p.at_region), hring0 = smem_u32(smem + p.at_hring);
    float* yacc = reinterpret_cast<float*>(smem + p.at_region);                              // phase 3, where x was: [warp][token][16]

    if (threadIdx.x == 0) {
        for (int i = 0; i < p.slots; ++i) { mbar_init(&wfull[i], 1); mbar_init(&wempty[i], kMoeConsumers); }
        for (int i = 0; i < p.h_slots; ++i) { mbar_init(&hfull[i], 1); mbar_init(&hempty[i], kMoeConsumers); }
        for (int i = 0; i < 2; ++i) { mbar_init(&rfull[i], kMoeConsumers); mbar_init(&rempty[i], 1); }
        shared[1] = 0;
        fence_barrier_init();
        p.flags[ctas + cta] = 0;                          // the second meeting's flag; seen by all once the first meeting is over
    }
    for (int e = threadIdx.x; e < p.E; e += kMoeThreads) mask[e] = 0;
    __syncthreads();
    const int nch1 = (p.H + kMoeK - 1) / kMoeK, nch2 = (p.I + kMoeK - 1) / kMoeK, nfb = p.I / 8;
    const bool fixed_x = p.T <= 8;                        // column = token for every expert: x is staged once

    // ---- 1. router --------------------------------------------------------------------------------------------------
    if (warp < kMoeConsumers) {
        if (fixed_x)
            for (int i = threadIdx.x; i < p.T * (p.H / 8); i += kConsumerThreads) {
                const int t = i / (p.H / 8), c = i - t * (p.H / 8);
                *reinterpret_cast<uint4*>(smem + p.at_region + t * p.x_pitch + c * 16) = __ldg(reinterpret_cast<const uint4*>(p.x + (int64_t)t * p.H) + c);
            }
        // an item is one expert's row times up to 8 tokens; with fewer tokens the warps split the row as well
        float* part = reinterpret_cast<float*>(smem + p.at_red);
        const int ntb = (p.T + 7) / 8;
        int flip = 0;
        for (int item = cta; item < p.E * ntb; item += ctas) {
            const int tb = item / p.E, e = item - tb * p.E, nt = min(8, p.T - tb * 8);
            const int np = nt > 4 ? 8 : (nt > 2 ? 4 : nt), nsl = kMoeConsumers / np, t = warp & (np - 1), sl = warp / np;
            float s = 0.0f;
            if (t < nt) {
                const int pieces = p.H / 8, lo = pieces * sl / nsl, hi = pieces * (sl + 1) / nsl;
                const uint4 *xr = reinterpret_cast<const uint4*>(p.x + (int64_t)(tb * 8 + t) * p.H), *wr = reinterpret_cast<const uint4*>(p.wr + (int64_t)e * p.H);
#pragma unroll 4
                for (int i = lo + lane; i < hi; i += 32) {
                    float a[8], b[8];
                    bf16x8_unpack(__ldg(xr + i), a);
                    bf16x8_unpack(__ldg(wr + i), b);
#pragma unroll
                    for (int j = 0; j < 8; ++j) s = fmaf(a[j], b[j], s);
                }
#pragma unroll
                for (int m = 16; m >= 1; m >>= 1) s += __shfl_xor_sync(0xffffffffu, s, m);
            }
            if (nsl == 1) {
                if (lane == 0 && t < nt) p.logits[(int64_t)(tb * 8 + t) * p.E + e] = s;
            } else {
                if (lane == 0) part[flip + warp] = s;
                bar_sync(1, kConsumerThreads);
                if ((int)threadIdx.x < nt) {
                    s = 0.0f;
                    for (int i = 0; i < nsl; ++i) s += part[flip + i * np + threadIdx.x];
                    p.logits[(int64_t)(tb * 8 + threadIdx.x) * p.E + e] = s;
                }
                flip ^= 8;
            }
        }
        bar_sync(1, kConsumerThreads);
        if (warp == 0) {
            if (lane == 0) { __threadfence(); st_release_u64(p.flags + cta, p.mark); }
            if (!meet(p.flags, ctas, p.mark, lane) && lane == 0) { shared[1] = 1; atomicExch(&g_moe_status, 8); }
        }
        bar_sync(1, kConsumerThreads);
        // top-k, a warp per token
        for (int t = warp; t < p.T; t += kMoeConsumers) {
            constexpr int V = (int)(kMoeMaxE / 32);
            float l[V];
            uint32_t key[V];
            bool nan = false;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int e = lane + 32 * j;
                if (32 * j < p.E && e < p.E) { l[j] = __ldcg(p.logits + (int64_t)t * p.E + e); key[j] = order_key(l[j]); nan |= l[j] != l[j]; }
                else { l[j] = 0.0f; key[j] = 0u; }
            }
            nan = __any_sync(0xffffffffu, nan);
            float first = 0.0f, mine = 0.0f, sum = 0.0f;  // the largest logit; the chosen one this lane keeps; sum of exponentials
            int mine_e = 0;
            for (int k = 0; k < p.topk; ++k) {
                uint32_t best = 0u;
#pragma unroll
                for (int j = 0; j < V; ++j) if (32 * j < p.E) best = max(best, key[j]);
                best = __reduce_max_sync(0xffffffffu, best);
                uint32_t at = 0xffffffffu;
                float val = 0.0f;
#pragma unroll
                for (int j = V - 1; j >= 0; --j) if (32 * j < p.E && key[j] == best) { at = (uint32_t)(lane + 32 * j); val = l[j]; }
                const uint32_t e = __reduce_min_sync(0xffffffffu, at);
                val = __shfl_sync(0xffffffffu, val, (int)(e & 31u));
#pragma unroll
                for (int j = 0; j < V; ++j) if (32 * j < p.E && (uint32_t)(lane + 32 * j) == e) key[j] = 0u;
                if (k == 0) first = val;
                if (lane == k) { mine = val; mine_e = (int)e; }
            }
            if (p.norm) { if (lane < p.topk) sum = expf(mine - first); }
            else {
#pragma unroll
                for (int j = 0; j < V; ++j) if (32 * j < p.E && lane + 32 * j < p.E) sum += expf(l[j] - first);
            }
#pragma unroll
            for (int m = 16; m >= 1; m >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, m);
            if (lane < p.topk) {
                const float w = nan ? __int_as_float(0x7fffffff) : expf(mine - first) / sum;
                sel[t * p.topk + lane] = (uint16_t)mine_e;
                selw[t * p.topk + lane] = w;
                atomicOr(&mask[mine_e], 1ull << t);       // (the order of the bits' arrival does not matter)
                if (cta == 0) {
                    if (p.ids) p.ids[t * p.topk + lane] = mine_e;
                    if (p.weights) p.weights[t * p.topk + lane] = w;
                }
            }
        }
        bar_sync(1, kConsumerThreads);
        // pairs sorted by expert, then token; entries of at most `group` pairs of one expert
        if (warp == 0) {
            int pairs = 0, ents = 0;
            for (int e0 = 0; e0 < p.E; e0 += 32) {
                const int e = e0 + lane, cnt = e < p.E ? __popcll(mask[e]) : 0, ne = (cnt + p.group - 1) / p.group;
                int sc = cnt, se = ne;
#pragma unroll
                for (int m = 1; m < 32; m <<= 1) {
                    const int a = __shfl_up_sync(0xffffffffu, sc, m), b = __shfl_up_sync(0xffffffffu, se, m);
                    if (lane >= m) { sc += a; se += b; }
                }
                const int o = pairs + sc - cnt, i0 = ents + se - ne;
                if (e < p.E) off[e] = (uint16_t)o;
                for (int i = 0; i < ne; ++i) ent[i0 + i] = (uint32_t)e | (uint32_t)(o + i * p.group) << 9 | (uint32_t)min(p.group, cnt - i * p.group) << 20;
                pairs += __shfl_sync(0xffffffffu, sc, 31);
                ents += __shfl_sync(0xffffffffu, se, 31);
            }
            if (lane == 0) shared[0] = ents;
        }
        bar_sync(1, kConsumerThreads);
        for (int i = threadIdx.x; i < p.T * p.topk; i += kConsumerThreads) {
            const int t = i / p.topk, e = sel[i], s = off[e] + __popcll(mask[e] & ((1ull << t) - 1ull));
            tok[s] = (uint8_t)t;
            wt[s] = selw[i];
        }
    }
    __syncthreads();
    if (shared[1]) return;                                // the first meeting did not come about: nothing is in flight yet
    const int ents = shared[0], units = ents * nfb;
    const int u0 = (int)((int64_t)units * cta / ctas), u1 = (int)((int64_t)units * (cta + 1) / ctas);

    if (warp == kMoeConsumers) {
        // ---- weight ring --------------------------------------------------------------------------------------------
        int slot = 0, issued = 0;
        uint32_t phase = 0;
        bool ok = true;
        auto fill = [&](const unsigned char* row, bool active, int rows, int kc) {      // this lane's row, if it has one
            ok = __all_sync(0xffffffffu, mbar_wait_bounded(&wempty[slot], phase ^ 1));
            if (!ok) { if (lane == 0) atomicExch(&g_moe_status, 8); return; }
            if (lane == 0) mbar_expect_tx(&wfull[slot], (uint32_t)(rows * kc * 2));
            if (active) bulk_load(ring0 + (uint32_t)(slot * kMoeSlot + lane * kMoePitch), row, (uint32_t)(kc * 2), smem_u32(&wfull[slot]));
            ++issued;
            if (++slot == p.slots) { slot = 0; phase ^= 1; }
        };
        for (int u = u0; ok && u < u1; ++u) {
            const int i = u / nfb, f = (u - i * nfb) * 8 + (lane & 7), g = f / p.gu_half;          // feature, and its strip
            const unsigned char* row = p.wgu + (int64_t)(ent[i] & 511u) * p.gu_stride +
                                       (int64_t)(g * p.gu_strip + (f - g * p.gu_half) + (lane >= 8 ? p.gu_half : 0)) * p.H * 2;
            for (int c = 0; ok && c < nch1; ++c) fill(row + c * kMoeK * 2, lane < 16, 16, min(kMoeK, p.H - c * kMoeK));
        }
        for (int b = cta; ok && b < p.blocks; b += ctas) {
            const int r0 = b * p.rows_per_block, rows = min(p.rows_per_block, p.H - r0);
            for (int i = 0; ok && i < ents; ++i) {
                const unsigned char* row = p.wd + (int64_t)(ent[i] & 511u) * p.d_stride + (int64_t)(r0 + lane) * p.I * 2;
                for (int c = 0; ok && c < nch2; ++c) fill(row + c * kMoeK * 2, lane < rows, rows, min(kMoeK, p.I - c * kMoeK));
            }
        }
        if (!ok)                                          // given up: the copies in flight land before the CTA may leave
            for (int i = max(0, issued - p.slots); i < issued; ++i) mbar_wait_bounded(&wfull[i % p.slots], (uint32_t)(i / p.slots) & 1u);
    } else if (warp == kMoeConsumers + 1) {
        // ---- h ring -------------------------------------------------------------------------------------------------
        bool ok = meet(p.flags + ctas, ctas, p.mark, lane);
        if (!ok && lane == 0) atomicExch(&g_moe_status, 8);
        if (ok && lane == 0) p.flags[cta] = 0;            // everyone is past the first meeting: its flag is cleared for the next launch
        asm volatile("fence.proxy.async;" ::: "memory");  // h was written by ordinary stores and is fetched by the copy engine; x was read by ordinary loads
        __syncwarp();
        int slot = 0, issued = 0;
        uint32_t phase = 0;
        for (int b = cta; ok && b < p.blocks; b += ctas)
            for (int i = 0; ok && i < ents; ++i) {
                const uint32_t en = ent[i];
                const int first = (int)(en >> 9 & 2047u), cnt = (int)(en >> 20);
                for (int c = 0; ok && c < nch2; ++c) {
                    ok = __all_sync(0xffffffffu, mbar_wait_bounded(&hempty[slot], phase ^ 1));
                    if (!ok) { if (lane == 0) atomicExch(&g_moe_status, 8); break; }
                    const int kc = min(kMoeK, p.I - c * kMoeK);
                    if (lane == 0) mbar_expect_tx(&hfull[slot], (uint32_t)(cnt * kc * 2));
                    if (lane < cnt)
                        bulk_load(hring0 + (uint32_t)((slot * p.group + lane) * kMoePitch), p.h + (int64_t)(first + lane) * p.h_pitch + c * kMoeK * 2, (uint32_t)(kc * 2),
                                  smem_u32(&hfull[slot]));
                    ++issued;
                    if (++slot == p.h_slots) { slot = 0; phase ^= 1; }
                }
            }
        if (!ok)
            for (int i = max(0, issued - p.h_slots); i < issued; ++i) mbar_wait_bounded(&hfull[i % p.h_slots], (uint32_t)(i / p.h_slots) & 1u);
    } else {
        const int g = lane >> 2, q = lane & 3;
        int slot = 0, cur = -1, cols = p.T, nt = (p.T + 7) / 8;      // columns staged (with more than 8 tokens: the entry's)
        uint32_t phase = 0;
        bool ok = true;
        // ---- 2. gate and up -------------------------------------------------------------------------------------------
        float* red = reinterpret_cast<float*>(smem + p.at_red);                  // [buffer][column group][warp][lane] float4
        for (int u = u0; ok && u < u1; ++u) {
            const int i = u / nfb, fb = u - i * nfb, n = u - u0, buf = n & 1;
            const uint32_t en = ent[i];
            const int first = (int)(en >> 9 & 2047u), cnt = (int)(en >> 20);
            if (!fixed_x && i != cur) {                                          // another expert: its tokens' rows of x
                bar_sync(1, kConsumerThreads);
                for (int j = threadIdx.x; j < cnt * (p.H / 8); j += kConsumerThreads) {
                    const int t = j / (p.H / 8), c = j - t * (p.H / 8);
                    *reinterpret_cast<uint4*>(smem + p.at_region + t * p.x_pitch + c * 16) = __ldg(reinterpret_cast<const uint4*>(p.x + (int64_t)tok[first + t] * p.H) + c);
                }
                bar_sync(1, kConsumerThreads);
                cur = i;
                cols = cnt;
                nt = (cnt + 7) / 8;
            }
            float acc[NT][4];
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.0f;
            for (int c = 0; ok && c < nch1; ++c) {
                ok = __all_sync(0xffffffffu, mbar_wait_bounded(&wfull[slot], phase));
                if (!ok) break;
                slot_product<NT>(acc, ring0 + (uint32_t)(slot * kMoeSlot), x0 + (uint32_t)(c * kMoeK * 2), p.x_pitch, min(kMoeK, p.H - c * kMoeK), cols, warp, lane);
                __syncwarp();
                if (lane == 0) mbar_arrive(&wempty[slot]);
                if (++slot == p.slots) { slot = 0; phase ^= 1; }
            }
            // the warps' partial sums meet in shared memory; the warps take turns in finishing a unit
            const uint32_t rphase = (uint32_t)(n >> 1) & 1u;
            ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(&rempty[buf], rphase ^ 1));
            if (!ok) break;
            float4* out = reinterpret_cast<float4*>(red) + (size_t)buf * NT * kConsumerThreads;
#pragma unroll
            for (int j = 0; j < NT; ++j)
                if (j < nt) out[j * kConsumerThreads + warp * 32 + lane] = make_float4(acc[j][0], acc[j][1], acc[j][2], acc[j][3]);
            __syncwarp();
            if (lane == 0) mbar_arrive(&rfull[buf]);
            if (warp == (n & (kMoeConsumers - 1))) {
                ok = __all_sync(0xffffffffu, mbar_wait_bounded(&rfull[buf], rphase));
                if (!ok) break;
                const unsigned long long em = mask[en & 511u];
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    if (j >= nt) break;
                    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                    for (int w = 0; w < kMoeConsumers; ++w) {
                        const float4 v = out[j * kConsumerThreads + w * 32 + lane];
                        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
                    }
                    const float h2[2] = {s.x * logistic(s.x) * s.z, s.y * logistic(s.y) * s.w};
#pragma unroll
                    for (int c = 0; c < 2; ++c) {                                // gate | up of feature g, columns 2q and 2q + 1
                        const int col = j * 8 + 2 * q + c;
                        const bool has = fixed_x ? (col < p.T && (em >> col & 1)) : col < cnt;
                        const int pair = fixed_x ? first + __popcll(em & ((1ull << col) - 1ull)) : first + col;
                        if (has) reinterpret_cast<__nv_bfloat16*>(p.h + (int64_t)pair * p.h_pitch)[fb * 8 + g] = __float2bfloat16_rn(h2[c]);
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&rempty[buf]);
            }
        }
        if (!ok && lane == 0) atomicExch(&g_moe_status, 8);
        asm volatile("fence.proxy.async;" ::: "memory");
        bar_sync(1, kConsumerThreads);
        if (threadIdx.x == 0) { __threadfence(); st_release_u64(p.flags + ctas + cta, p.mark); }
        // ---- 3. down --------------------------------------------------------------------------------------------------
        for (int i = threadIdx.x; i < kMoeConsumers * p.T * 16; i += kConsumerThreads) yacc[i] = 0.0f;     // (x is no longer read)
        bar_sync(1, kConsumerThreads);
        float* ya = yacc + (size_t)warp * p.T * 16;
        int hslot = 0;
        uint32_t hphase = 0;
        for (int b = cta; b < p.blocks; b += ctas) {
            const int r0 = b * p.rows_per_block, rows = min(p.rows_per_block, p.H - r0);
            for (int i = 0; ok && i < ents; ++i) {
                const uint32_t en = ent[i];
                const int first = (int)(en >> 9 & 2047u), cnt = (int)(en >> 20), n8 = (cnt + 7) / 8;
                float acc[NT][4];
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.0f;
                for (int c = 0; ok && c < nch2; ++c) {
                    ok = __all_sync(0xffffffffu, mbar_wait_bounded(&wfull[slot], phase) && mbar_wait_bounded(&hfull[hslot], hphase));
                    if (!ok) break;
                    slot_product<NT>(acc, ring0 + (uint32_t)(slot * kMoeSlot), hring0 + (uint32_t)(hslot * p.group * kMoePitch), kMoePitch, min(kMoeK, p.I - c * kMoeK), cnt, warp, lane);
                    __syncwarp();
                    if (lane == 0) { mbar_arrive(&wempty[slot]); mbar_arrive(&hempty[hslot]); }
                    if (++slot == p.slots) { slot = 0; phase ^= 1; }
                    if (++hslot == p.h_slots) { hslot = 0; hphase ^= 1; }
                }
                // this warp's share of w * (Wd h), into its own sums: a token is in one column of an entry only
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    if (j >= n8) break;
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int col = j * 8 + 2 * q + c;
                        if (col < cnt) {
                            float* a = ya + tok[first + col] * 16 + g;
                            const float w = wt[first + col];
                            a[0] = fmaf(w, acc[j][c], a[0]);
                            a[8] = fmaf(w, acc[j][c + 2], a[8]);
                        }
                    }
                }
                __syncwarp();                             // (the next entry may hold the same token in another lane's column)
            }
            if (!ok && lane == 0) atomicExch(&g_moe_status, 8);
            bar_sync(1, kConsumerThreads);
            for (int i = threadIdx.x; i < p.T * 16; i += kConsumerThreads) {
                const int t = i >> 4, r = i & 15;
                float s = 0.0f;
#pragma unroll
                for (int w = 0; w < kMoeConsumers; ++w) { s += yacc[(w * p.T) * 16 + i]; yacc[(w * p.T) * 16 + i] = 0.0f; }
                if (r < rows) {
                    const int64_t at = (int64_t)t * p.H + r0 + r;
                    if (p.residual) s += bf16_lo(p.residual[at]);
                    reinterpret_cast<__nv_bfloat16*>(p.y)[at] = __float2bfloat16_rn(s);
                }
            }
            bar_sync(1, kConsumerThreads);
        }
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------
struct MoePlan {
    MoeParams p;
    int nt, ctas;
    size_t smem, ws;
};

static size_t up128(size_t n) { return (n + 127) & ~(size_t)127; }

static ccl_status plan_moe(const ccl_moe_desc* d, int sms, MoePlan* plan) {
    if (!d) return fail(CCL_ERR_INVALID_ARG, "ccl_moe_tokens: NULL descriptor");
    if (d->T < 1 || d->H < 1 || d->I < 1 || d->E < 1 || d->topk < 1) return fail(CCL_ERR_INVALID_ARG, "ccl_moe_tokens: T, H, I, E and topk must be positive");
    if (d->topk > d->E) return fail(CCL_ERR_SHAPE, "ccl_moe_tokens: topk (%d) is larger than E (%d)", d->topk, d->E);
    if (d->T > kMoeMaxT || d->E > kMoeMaxE || d->topk > kMoeMaxK || d->H > 8192 || d->I > 32768)
        return fail(CCL_ERR_UNSUPPORTED, "ccl_moe_tokens: takes at most 64 tokens, 512 experts, 16 experts a token, H = 8192 and I = 32768");
    if (d->H % 8 || d->I % 8) return fail(CCL_ERR_UNSUPPORTED, "ccl_moe_tokens: H and I must be multiples of 8");
    if (d->gu_strips < 1) return fail(CCL_ERR_INVALID_ARG, "ccl_moe_tokens: gu_strips must be at least 1");
    if (d->I / 8 % d->gu_strips) return fail(CCL_ERR_SHAPE, "ccl_moe_tokens: gu_strips (%d) must divide I / 8", d->gu_strips);
    const int64_t gu = 4 * d->I * d->H, dn = 2 * d->I * d->H;
    if (d->gu_stride_bytes < 0 || d->d_stride_bytes < 0 || (d->gu_stride_bytes && d->gu_stride_bytes < gu) || (d->d_stride_bytes && d->d_stride_bytes < dn))
        return fail(CCL_ERR_INVALID_ARG, "ccl_moe_tokens: an expert stride is smaller than an expert's weights");
    if (d->gu_stride_bytes % 16 || d->d_stride_bytes % 16) return fail(CCL_ERR_ALIGN, "ccl_moe_tokens: expert strides must be multiples of 16 bytes");
    MoeParams& p = plan->p;
    p = MoeParams{};
    p.T = (int32_t)d->T; p.H = (int32_t)d->H; p.I = (int32_t)d->I; p.E = d->E; p.topk = d->topk; p.norm = d->norm_topk != 0;
    p.gu_half = (int32_t)(d->I / d->gu_strips); p.gu_strip = 2 * p.gu_half;
    p.gu_stride = d->gu_stride_bytes ? d->gu_stride_bytes : gu; p.d_stride = d->d_stride_bytes ? d->d_stride_bytes : dn;
    plan->ctas = sms;
    const int64_t per = (d->H + (int64_t)sms * 16 - 1) / ((int64_t)sms * 16);              // row blocks a CTA takes
    p.rows_per_block = (int32_t)((d->H + sms * per - 1) / (sms * per));
    p.blocks = (int32_t)((d->H + p.rows_per_block - 1) / p.rows_per_block);
    p.x_pitch = (int32_t)(up128((size_t)d->H * 2) + 64);
    const int pairs = (int)(d->T * d->topk);
    // Tokens of an expert taken together.  An expert with more is taken several times, its weights re-read (from the L2, they
    // were just used); more columns cost shared memory that the ring of weights in flight would have.
    const int64_t mean = (pairs + d->E - 1) / d->E;
    for (p.group = d->T <= 8 ? 8 : (mean <= 8 ? 16 : 32);; p.group /= 2) {
        const size_t yacc = up128((size_t)kMoeConsumers * (size_t)d->T * 16 * 4), hslot = (size_t)p.group * kMoePitch, xs = (size_t)std::min<int64_t>(p.group, d->T) * (size_t)p.x_pitch;
        const int most = std::min(pairs, d->E) + pairs / p.group;                            // entries
        size_t at = 0;
        auto take = [&](size_t bytes) { const size_t a = at; at += up128(bytes); return (int32_t)a; };
        // (the ring comes first; its size is what the rest leaves)
        for (p.h_slots = kMoeMaxHSlots; p.h_slots > 2 && yacc + p.h_slots * hslot > xs; --p.h_slots) {}
        p.at_region = take(std::max(xs, yacc + p.h_slots * hslot));
        p.at_hring = p.at_region + (int32_t)yacc;
        p.at_red = take((size_t)2 * (p.group / 8) * kMoeConsumers * 32 * 16);
        p.at_mask = take((size_t)d->E * 8);
        p.at_off = take((size_t)d->E * 2);
        p.at_ent = take((size_t)most * 4);
        p.at_tok = take((size_t)pairs);
        p.at_wt = take((size_t)pairs * 4);
        p.at_sel = take((size_t)pairs * 2);
        p.at_selw = take((size_t)pairs * 4);
        p.at_bars = take((size_t)(2 * kMoeMaxSlots + 2 * kMoeMaxHSlots + 4) * 8 + 16);
        const size_t room = 227 * 1024;
        p.slots = at < room ? (int32_t)std::min<size_t>(kMoeMaxSlots, (room - at) / kMoeSlot) : 0;
        if (p.slots < 4 && p.group > 8) continue;
        if (p.slots < 2) return fail(CCL_ERR_UNSUPPORTED, "ccl_moe_tokens: this problem does not fit shared memory");
        const int32_t ring = p.slots * kMoeSlot;
        for (int32_t* a : {&p.at_region, &p.at_hring, &p.at_red, &p.at_mask, &p.at_off, &p.at_ent, &p.at_tok, &p.at_wt, &p.at_sel, &p.at_selw, &p.at_bars}) *a += ring;
        plan->smem = at + (size_t)ring;
        break;
    }
    plan->nt = p.group / 8;
    p.h_pitch = (int64_t)up128((size_t)d->I * 2);
    plan->ws = up128((size_t)(d->T * d->E) * 4) + up128((size_t)sms * 2 * 8) + (size_t)pairs * (size_t)p.h_pitch;
    return CCL_OK;
}

static int moe_sms() {
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) == cudaSuccess && cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess && n > 0) return n;
    (void)cudaGetLastError();
    return 148;
}

template <int NT>
static ccl_status launch_moe(const MoePlan& plan, cudaStream_t st) {
    static std::atomic<uint64_t> configured{0};
    int dev = 0;
    CCL_CUDA_TRY(cudaGetDevice(&dev));
    if (dev >= 64 || !(configured.load() >> dev & 1)) {
        CCL_CUDA_TRY(cudaFuncSetAttribute(moe_tokens_kernel<NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024));
        if (dev < 64) configured.fetch_or(1ull << dev);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)plan.ctas, 1, 1);
    cfg.blockDim = dim3(kMoeThreads, 1, 1);
    cfg.dynamicSmemBytes = plan.smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeCooperative;         // all CTAs resident at once, or the launch fails
    attr[0].val.cooperative = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    CCL_CUDA_TRY(cudaLaunchKernelEx(&cfg, moe_tokens_kernel<NT>, plan.p));
    count_launch();
    return CCL_OK;
}

// The status word of this file's kernel, read and cleared (ccl_gemm_status)
ccl_status moe_status_take(int* code) {
    int zero = 0;
    CCL_CUDA_TRY(cudaMemcpyFromSymbol(code, g_moe_status, sizeof(int)));
    if (*code) CCL_CUDA_TRY(cudaMemcpyToSymbol(g_moe_status, &zero, sizeof(int)));
    return CCL_OK;
}

}  // namespace ccl

using namespace ccl;

extern "C" ccl_status ccl_moe_tokens_workspace(const ccl_moe_desc* d, size_t* bytes) {
    MoePlan plan;
    ccl_status s = plan_moe(d, 148, &plan);
    if (s) return s;
    if (!bytes) return fail(CCL_ERR_INVALID_ARG, "ccl_moe_tokens_workspace: NULL output");
    if ((s = plan_moe(d, moe_sms(), &plan))) return s;
    *bytes = plan.ws;
    return CCL_OK;
}

extern "C" ccl_status ccl_moe_tokens(const ccl_moe_desc* d, const void* X_dev, const void* Wr_dev, const void* Wgu_dev, const void* Wd_dev,
                                     const void* residual_dev, void* Y_dev, int32_t* ids_dev, float* weights_dev, void* ws_dev, size_t ws_bytes,
                                     void* cuda_stream) {
    if (!X_dev || !Wr_dev || !Wgu_dev || !Wd_dev || !Y_dev) return fail(CCL_ERR_INVALID_ARG, "ccl_moe_tokens: NULL operand");
    MoePlan plan;
    ccl_status s = plan_moe(d, 148, &plan);              // validation first: no CUDA call on bad input
    if (s) return s;
    uintptr_t all = 0;
    for (const void* q : {X_dev, Wr_dev, Wgu_dev, Wd_dev, residual_dev, static_cast<const void*>(Y_dev), static_cast<const void*>(ws_dev)}) all |= reinterpret_cast<uintptr_t>(q);
    if (all & 15) return fail(CCL_ERR_ALIGN, "ccl_moe_tokens: a base pointer is not 16-byte aligned");
    if ((reinterpret_cast<uintptr_t>(ids_dev) | reinterpret_cast<uintptr_t>(weights_dev)) & 3) return fail(CCL_ERR_ALIGN, "ccl_moe_tokens: ids or weights are not 4-byte aligned");
    if (!ws_dev || ws_bytes < plan.ws) return fail(CCL_ERR_WORKSPACE, "ccl_moe_tokens: needs %zu bytes of workspace (got %zu)", plan.ws, ws_dev ? ws_bytes : (size_t)0);
    const int sms = moe_sms();
    if (sms != 148 && (s = plan_moe(d, sms, &plan))) return s;
    if (ws_bytes < plan.ws) return fail(CCL_ERR_WORKSPACE, "ccl_moe_tokens: needs %zu bytes of workspace (got %zu)", plan.ws, ws_bytes);
    MoeParams& p = plan.p;
    p.x = static_cast<const uint16_t*>(X_dev); p.wr = static_cast<const uint16_t*>(Wr_dev); p.residual = static_cast<const uint16_t*>(residual_dev);
    p.wgu = static_cast<const unsigned char*>(Wgu_dev); p.wd = static_cast<const unsigned char*>(Wd_dev);
    p.y = static_cast<uint16_t*>(Y_dev); p.ids = ids_dev; p.weights = weights_dev;
    unsigned char* ws = static_cast<unsigned char*>(ws_dev);
    p.logits = reinterpret_cast<float*>(ws);
    p.flags = reinterpret_cast<unsigned long long*>(ws + up128((size_t)p.T * p.E * 4));
    p.h = ws + up128((size_t)p.T * p.E * 4) + up128((size_t)plan.ctas * 2 * 8);
    // A mark that no workspace holds yet, whatever its contents.  A launch leaves the first meeting's flags cleared and clears the
    // second's before the first meeting, so that a replayed CUDA graph may use its mark again.
    static std::atomic<unsigned long long> next{(unsigned long long)std::chrono::steady_clock::now().time_since_epoch().count() * 0x9E3779B97F4A7C15ull};
    do p.mark = next.fetch_add(0x9E3779B97F4A7C15ull); while (p.mark == 0);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    switch (plan.nt) {
        case 1: return launch_moe<1>(plan, st);
        case 2: return launch_moe<2>(plan, st);
        default: return launch_moe<4>(plan, st);
    }
}
