// ccl_moe_tokens: a mixture-of-experts feed-forward layer for a few tokens -- router, top-k, gated expert products and the
// weighted sum -- in one cooperative launch of one CTA per SM.
//
// Bound by memory: every chosen expert's weights are read once (3 H I elements each) and nothing else is of that order; with
// m tokens an expert the arithmetic is 2 m flops per 2-byte weight, far below what the tensor cores take.  So the kernel is a
// stream of weights through shared memory that stops for nothing it can avoid:
//   1. router: the CTAs share the E x T dot products (16 experts x 8 tokens a matrix product); first meeting of the grid; top-k, by
//      every CTA for itself for up to 8 tokens, by a CTA a token and with one more meeting for more; every CTA works out the same lists
//      of tokens per expert
//   2. gate and up: the (expert, 16 features) units are shared out evenly.  A unit is 32 weight rows -- 16 gate, 16 up -- times
//      its expert's tokens (n = 8 columns): two m16n8k16 accumulators then hold the gate and the up value of a
//      feature in the same lane, and silu(gate) * up needs no exchange.  h goes to the workspace; second meeting
//   3. down: a pair of CTAs (a cluster) owns a few rows of Wd (2 H / #SMs of them, at most 32) and takes every chosen expert's:
//      the sum over a token's experts stays inside the pair, in a fixed order, and Y is written once.
// The k range of a unit is dealt out in blocks of 64 (32 rows x 128 bytes) to the 8 consumer warps of the CTA in turn (phase 3: to
// the 16 of the pair).  A ninth warp fetches the blocks, one TMA copy each, up to 32 of them ahead: it stops for nothing but a
// full ring, runs ahead across units and from phase 2 into phase 3, so the weights of phase 3 arrive during the second meeting.
// Four more fetch the h that goes with phase 3's blocks, by cp.async: the TMA takes ~60 ns a block as it is (a 128-byte row every four
// cycles), and h by TMA as well had the products wait.  (Consumers that issued their own copies, or read h themselves, made loops
// that were slower to run than the weights to come: phase 3 of 64 tokens x 128 experts of 2048 x 768 took 118 and 86 us, 66 now.)
//
// Measured (B200, 128 experts of 2048 x 768, 8 a token): 64 tokens 215-226 us, 5.3-5.5 TB/s over everything and above 6 while weights
// stream; 16 tokens 134-136 us; one token 29.5-30.7 us, of which the weights take 12 and the rest is launch, router, top-k and two meetings.
//
// The matrix instructions are mma.sync: with n = 8 columns a tcgen05 tile would be 128 rows high and leave most SMs without
// work for one token; they are nowhere near their limit here.  Weights and tokens are both K-contiguous, so a lane may take any 8
// consecutive k as its share of two k steps as long as both operands do: 16-byte loads, no ldmatrix.
// h keeps 16 significant bits: it is stored as two bf16 rows (the rounded value and what the rounding left), two columns of the same
// product, which the n = 8 columns have room for.
#include <algorithm>
#include <atomic>
#include <chrono>

#include "ccl_act.cuh"
#include "ccl_tma.h"

namespace ccl {

constexpr int kMoeWarps = 8;                             // consumers
constexpr int kMoeThreads = kMoeWarps * 32;
constexpr int kMoeHWarps = 4;                            // warps that fetch h, for two consumers each
constexpr int kMoeBlockThreads = kMoeThreads + 32 + 32 * kMoeHWarps;         // and the one that fetches weights
constexpr int kMoeRows = 32;                             // rows of a block,
constexpr int kMoeBlockK = 64;                           // its k elements (128 bytes of a row)
constexpr int kMoeBlock = kMoeRows * kMoeBlockK * 2;
constexpr int kMoeDepth = 4;                             // most blocks in a warp's ring
constexpr int kMoeGroup = 8;                             // most tokens of an expert taken together: two groups of 4, each 8 columns of phase 3
constexpr int kMoeHBlock = 2 * 8 * kMoeBlockK * 2;       // h for a block
constexpr size_t kMoeSmem = 227 * 1024;
constexpr int64_t kMoeMaxT = 64, kMoeMaxE = 512, kMoeMaxK = 16;

static __device__ int g_moe_status = 0;

struct MoeParams {
    int32_t T, H, I, E, topk, norm;
    int32_t gu_half, strip_units;           // gate rows of a strip; units of a strip
    const uint16_t *x, *wr, *residual;
    uint16_t* y;
    int32_t* ids;
    float* weights;
    float* logits;                          // workspace: [T][E]
    unsigned long long* flags;              // workspace: a flag per CTA (first meeting)
    unsigned long long* gate;               // workspace: the word that ends the first meeting, the counters of the others
    int2* choice;                           // workspace: [T][topk] expert, weight (more than 8 tokens)
    unsigned char* h;                       // workspace: [groups of 4 pairs][value, remainder][4][h_pitch bytes] bf16
    int64_t h_pitch;
    unsigned long long mark;                // this launch's mark in the flags
    int32_t writers;                        // CTAs the first meeting waits for: the first of the grid, those with logits to write
    int32_t quorum;                         // CTAs the others wait for: all
    uint64_t wait_ns;                       // how long a CTA waits at a meeting
    int32_t group;                          // most tokens of an expert taken together (8 or 4)
    int32_t depth;                          // blocks in a warp's ring
    int32_t all_x;                          // 1: the rows of all tokens are staged once; 0: those of an expert's tokens when it comes up
    int32_t x_pitch;                        // bytes between the token rows in shared memory
    int32_t rows_per_block, blocks;         // phase 3: rows of Wd a pair of CTAs takes at a time, such blocks in all
    // byte offsets in shared memory
    int32_t at_bars, at_region, at_hring, at_red, at_mask, at_off, at_ent, at_hgroup, at_sel, at_selw, at_pair;
};

__device__ __forceinline__ uint4 lds128(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
// 16 bytes, or zeros where `ok` is off (nothing is read then)
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src, bool ok) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}
__device__ __forceinline__ void mma_16x8x16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// All consumer threads
__device__ __forceinline__ void bar_consumers() { asm volatile("bar.sync 1, %0;" ::"n"(kMoeThreads) : "memory"); }
__device__ __forceinline__ bool bar_consumers_and(bool v) {
    uint32_t r;
    asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n barrier.cta.red.and.pred q, 1, %2, p;\n selp.u32 %0, 1, 0, q;\n}" : "=r"(r) : "r"((uint32_t)v), "n"(kMoeThreads) : "memory");
    return r != 0;
}
// (out of line: the loops that wait must stay small)
__device__ __noinline__ bool wait_long(uint32_t bar, uint32_t parity) { return mbar_wait_bounded_addr(bar, parity); }
__device__ __forceinline__ bool wait_for(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    if (!__all_sync(0xffffffffu, done)) done = __all_sync(0xffffffffu, wait_long(bar, parity));
    return done;
}
// One thread waits (bounded) until the word is `mark` (exact) or at least that.
__device__ __noinline__ bool wait_word(const unsigned long long* word, unsigned long long mark, bool exact, uint64_t limit_ns) {
    const uint64_t t0 = global_timer_ns();
    for (;;) {
        unsigned long long v;
        asm volatile("ld.acquire.gpu.global.u64 %0, [%1];" : "=l"(v) : "l"(word) : "memory");
        if (exact ? v == mark : v >= mark) return true;
        if (global_timer_ns() - t0 > limit_ns) return false;
    }
}
__device__ __forceinline__ void st_release(unsigned long long* p, unsigned long long v) { asm volatile("st.release.gpu.global.u64 [%0], %1;" ::"l"(p), "l"(v) : "memory"); }
// The grid's meetings (all consumer threads call; what a CTA wrote before is seen by all behind it).  Measured, 148 CTAs: 1.3 us
// when every CTA adds to one counter and one thread of each reads it; 4.9 us when 148 threads of every CTA read a flag of each.
// The counter needs a start, so the first meeting -- which ends when the `writers`, the first CTAs of the grid, have their logits out
// -- has flags (any contents but this launch's mark mean "not yet").  Up to 16 of them are read by every CTA (one token, 8 writers:
// 1.2 us less than the other way); of more, CTA 0 alone reads them and lets the others go by a word.  CTA 0 clears the counters of
// the later meetings on the way.  `meanwhile` is done between a CTA's arrival and its wait.  A CTA that leaves the kernel, on whatever
// way, clears its flag (leave_meetings): a replayed CUDA graph uses the same mark again, and must not take an old flag for a new one.
constexpr int kMoeReaders = 16;
template <typename F>
__device__ __forceinline__ bool meet_first(const MoeParams& p, F meanwhile) {
    const int writers = p.writers;
    bar_consumers();
    bool ok = true;
    if (threadIdx.x == 0 && (int)blockIdx.x < writers) {
        if (blockIdx.x == 0) p.gate[1] = p.gate[2] = 0;
        st_release(p.flags + blockIdx.x, p.mark);
    }
    meanwhile();
    const bool all = writers <= kMoeReaders;
    if (all || blockIdx.x == 0) {
#pragma unroll 1
        for (int i = threadIdx.x; i < writers; i += kMoeThreads) ok = wait_word(p.flags + i, p.mark, true, p.wait_ns) && ok;
        ok = bar_consumers_and(ok);
        if (threadIdx.x == 0 && ok && !all) st_release(p.gate, p.mark);
    } else {
        if (threadIdx.x == 0) ok = wait_word(p.gate, p.mark, true, p.wait_ns);
        ok = bar_consumers_and(ok);
    }
    if (!ok && threadIdx.x == 0) atomicExch(&g_moe_status, 8);
    return ok;
}
__device__ __forceinline__ bool meet_counted(const MoeParams& p, unsigned long long* counter) {
    bar_consumers();
    bool ok = true;
    if (threadIdx.x == 0) {
        asm volatile("red.release.gpu.global.add.u64 [%0], 1;" ::"l"(counter) : "memory");
        ok = wait_word(counter, (unsigned long long)p.quorum, false, p.wait_ns);
        if (!ok) atomicExch(&g_moe_status, 8);
    }
    return bar_consumers_and(ok);
}
// One thread of a CTA that goes to no meeting any more.  (Where all came about, everyone is past the first; where one did not, a CTA that
// still waits for this flag runs into its limit as well.)
__device__ __forceinline__ void leave_meetings(const MoeParams& p) {
    p.flags[blockIdx.x] = 0;
    if (blockIdx.x == 0) p.gate[0] = 0;
}
// All threads of the CTA pair
__device__ __forceinline__ void pair_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// The consumers of a CTA pair meet at a barrier of each CTA's that one thread of the other CTA arrives at (the warps that fetch are
// not to stop for it): what either wrote to its shared memory before is seen by the other behind the wait.
__device__ __forceinline__ void tell_other(uint64_t* bar, uint32_t other) {
    uint32_t remote;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(smem_u32(bar)), "r"(other));
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(remote) : "memory");
}
__device__ __noinline__ bool wait_other(uint64_t* bar, uint32_t parity) {
    const uint64_t t0 = global_timer_ns();
    for (;;) {
        uint32_t done;
        asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(done) : "r"(smem_u32(bar)), "r"(parity) : "memory");
        if (done) return true;
        if (global_timer_ns() - t0 > kWaitLimitNs) return false;
    }
}

// Order-preserving integer image of a float; NaN below every number, 0 for no number at all.
__device__ __forceinline__ uint32_t order_key(float f) {
    if (f != f) return 1u;
    const uint32_t u = __float_as_uint(f == 0.0f ? 0.0f : f);        // (-0 and 0 are equal)
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k); }

// d = A B for a block's 16 rows (m) of one of its two halves of 32 k: two k steps
__device__ __forceinline__ void mma_half(float (&d)[4], const uint4& lo, const uint4& hi, const uint4& b) {
    mma_16x8x16(d, lo.x, hi.x, lo.y, hi.y, b.x, b.y);
    mma_16x8x16(d, lo.z, hi.z, lo.w, hi.w, b.z, b.w);
}

// Byte offset of the 16 bytes that row r, piece c (of 8) of a block are kept at (the TMA's 128-byte swizzle), and the row a lane
// with g = lane / 4 takes as row g of a matrix fragment: consecutive g lie four rows apart, so that the 8 lanes of a 16-byte
// load's phase (two g, four pieces each) hit different banks.
__device__ __forceinline__ uint32_t block_at(int r, int c) { return (uint32_t)(r * 128 + ((c ^ (r & 7)) << 4)); }
__device__ __forceinline__ int fragment_row(int g) { return (g & 1) << 2 | g >> 1; }

// Sums of a token's rows r, r + 8, r + 16 and r + 24 (r < 8) lie side by side, turned by the token so that the tokens of a
// product's columns meet in different banks.  Offset of the four, and the row of place `at` of a token's 32.
__device__ __forceinline__ int sum_at(int t, int r) { return t * kMoeRows + ((r ^ (t & 7)) << 2); }
__device__ __forceinline__ int sum_row(int t, int at) { return ((at >> 2) ^ (t & 7)) + (at & 3) * 8; }

__global__ void __launch_bounds__(kMoeBlockThreads, 1) moe_tokens_kernel(const __grid_constant__ CUtensorMap map_gu, const __grid_constant__ CUtensorMap map_d,
                                                                        const __grid_constant__ MoeParams p) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, cta = blockIdx.x, ctas = gridDim.x;
    unsigned long long* mask = reinterpret_cast<unsigned long long*>(smem + p.at_mask);      // per expert: the tokens that chose it
    uint16_t* off = reinterpret_cast<uint16_t*>(smem + p.at_off);                            // per expert: its first pair
    uint16_t* hgroup = reinterpret_cast<uint16_t*>(smem + p.at_hgroup);                      // per entry: its first group of h
    uint32_t* ent = reinterpret_cast<uint32_t*>(smem + p.at_ent);                            // entries: expert | first pair << 9 | pairs << 19
    uint16_t* sel = reinterpret_cast<uint16_t*>(smem + p.at_sel);                            // per (token, choice): expert
    float* selw = reinterpret_cast<float*>(smem + p.at_selw);                                // ... and weight
    int2* pair = reinterpret_cast<int2*>(smem + p.at_pair);                                  // per pair, sorted by expert, then token: token, weight
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + p.at_bars);                          // [warp][slot]: a block has arrived; then: ... has been used; its h has
    uint64_t *used = bars + kMoeWarps * kMoeDepth, *h_bars = used + kMoeWarps * kMoeDepth;
    uint64_t* pair_bars = h_bars + kMoeWarps * kMoeDepth;                                    // the other CTA's sums are there; it has read this one's
    uint64_t* met_bar = pair_bars + 2;                                                       // the second meeting is over
    int* shared = reinterpret_cast<int*>(met_bar + 1);                                       // [0] entries, [1] the first meeting came about, [2] the second
    const int warp2 = (cta & 1) * kMoeWarps + warp;       // this warp's number in the CTA pair
    const int pairs = p.T * p.topk, nb1 = (p.H + kMoeBlockK - 1) / kMoeBlockK, nb2 = (p.I + kMoeBlockK - 1) / kMoeBlockK, nfb = p.I / p.gu_half * p.strip_units;
    const uint32_t x0 = smem_u32(smem + p.at_region);
    float* yacc = reinterpret_cast<float*>(smem + p.at_region);                              // phase 3, where x was: [warp][token][32], see sum_at

    if (threadIdx.x == 0) { prefetch_tmap(&map_gu); prefetch_tmap(&map_d); }
    if ((int)threadIdx.x < 3 * kMoeWarps * kMoeDepth + 3) { mbar_init(&bars[threadIdx.x], (int)threadIdx.x >= 2 * kMoeWarps * kMoeDepth && (int)threadIdx.x < 3 * kMoeWarps * kMoeDepth ? 32 : 1); fence_barrier_init(); }
    if (warp < kMoeWarps)
        for (int e = threadIdx.x; e < p.E; e += kMoeThreads) mask[e] = 0;
    // rows of x (zeros behind H) in shared memory; row t is token `of(t)`
    auto stage_x = [&](int rows, auto of) {
        const int pieces = nb1 * (kMoeBlockK / 8);
        for (int c = threadIdx.x; c < pieces; c += kMoeThreads)
#pragma unroll 4
            for (int t = 0; t < rows; ++t) {
                uint4 v = make_uint4(0u, 0u, 0u, 0u);
                if (c * 8 < p.H) v = __ldg(reinterpret_cast<const uint4*>(p.x + (int64_t)of(t) * p.H) + c);
                *reinterpret_cast<uint4*>(smem + p.at_region + t * p.x_pitch + c * 16) = v;
            }
    };

    // ---- 1. router --------------------------------------------------------------------------------------------------
    // an item is 16 experts' rows times up to 8 tokens, one matrix product; the warps split its k range
    if (warp < kMoeWarps) {
        float4* part = reinterpret_cast<float4*>(smem + p.at_red);
        const int g = lane >> 2, q = lane & 3, ne = (p.E + 15) / 16, ntb = (p.T + 7) / 8, steps = (p.H + 31) / 32;
#pragma unroll 1
        for (int item = cta; item < ne * ntb; item += ctas) {
            const int tb = item / ne, e0 = (item - tb * ne) * 16, t0 = tb * 8;
            const uint4 *wlo = reinterpret_cast<const uint4*>(p.wr + (int64_t)min(e0 + g, p.E - 1) * p.H) + q, *whi = reinterpret_cast<const uint4*>(p.wr + (int64_t)min(e0 + g + 8, p.E - 1) * p.H) + q;
            const uint4* xr = reinterpret_cast<const uint4*>(p.x + (int64_t)min(t0 + g, p.T - 1) * p.H) + q;
            float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
            for (int s0 = warp; s0 < steps; s0 += 8 * kMoeWarps) {       // eight steps' loads in flight together
                uint4 a[8], b[8], c[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int s = s0 + j * kMoeWarps;
                    a[j] = b[j] = c[j] = make_uint4(0u, 0u, 0u, 0u);
                    if (s * 32 + q * 8 < p.H) { a[j] = __ldg(wlo + s * 4); b[j] = __ldg(whi + s * 4); c[j] = __ldg(xr + s * 4); }
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    mma_16x8x16(acc, a[j].x, b[j].x, a[j].y, b[j].y, c[j].x, c[j].y);
                    mma_16x8x16(acc, a[j].z, b[j].z, a[j].w, b[j].w, c[j].z, c[j].w);
                }
            }
            part[threadIdx.x] = make_float4(acc[0], acc[1], acc[2], acc[3]);
            bar_consumers();
            if (warp == 0) {
                float4 v = part[lane];
#pragma unroll
                for (int w = 1; w < kMoeWarps; ++w) {
                    const float4 z = part[w * 32 + lane];
                    v.x += z.x; v.y += z.y; v.z += z.z; v.w += z.w;
                }
                const float l[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int t = t0 + 2 * q + (c & 1), e = e0 + g + (c >> 1) * 8;
                    if (t < p.T && e < p.E) p.logits[(int64_t)t * p.E + e] = l[c];
                }
            }
            bar_consumers();
        }
    bool met1 = meet_first(p, [&]() { if (p.all_x) stage_x(p.T, [](int t) { return t; }); });
    if (threadIdx.x == 0) shared[1] = met1;
    // top-k of a token: an expert's place is the number of those before it (a larger logit, or an equal one of a lower expert), a
    // thread an expert against all of them in shared memory.  Up to 8 tokens are worked out by every CTA for itself; of more, each
    // by one CTA, and the grid meets once more: 64 tokens x 128 experts took 10 us the first way, a warp a token.
    {
        const bool every = p.T <= 8;
        const int first = every ? 0 : cta, nt = !met1 ? 0 : (every ? p.T : (cta < p.T ? 1 : 0)), ep = (p.E + 3) / 4 * 4;     // tokens at hand
        uint32_t* keys = reinterpret_cast<uint32_t*>(smem + p.at_red);           // [token][ep]
        float* vals = reinterpret_cast<float*>(keys + nt * ep);                  // [token][16]: the chosen logits, best first
        int* who = reinterpret_cast<int*>(vals + nt * kMoeMaxK);                 // ... and their experts
#pragma unroll 4
        for (int i = threadIdx.x; i < nt * ep; i += kMoeThreads) {
            const int t = i / ep, e = i - t * ep;
            keys[i] = e < p.E ? order_key(__ldcg(p.logits + (int64_t)(first + t) * p.E + e)) : 0u;
        }
        bar_consumers();
        for (int i = threadIdx.x; i < nt * p.E; i += kMoeThreads) {
            const int t = i / p.E, e = i - t * p.E;
            const uint32_t* kt = keys + t * ep;
            const uint32_t k = kt[e];
            int place[4] = {0, 0, 0, 0};
#pragma unroll 4
            for (int o = 0; o < p.E; o += 4) {
                const uint4 v = *reinterpret_cast<const uint4*>(kt + o);
                place[0] += v.x >= (o < e ? k : k + 1u); place[1] += v.y >= (o + 1 < e ? k : k + 1u);
                place[2] += v.z >= (o + 2 < e ? k : k + 1u); place[3] += v.w >= (o + 3 < e ? k : k + 1u);
            }
            const int at = place[0] + place[1] + place[2] + place[3];
            if (at < p.topk) { vals[t * kMoeMaxK + at] = key_value(k); who[t * kMoeMaxK + at] = e; }
        }
        bar_consumers();
        if (warp < nt) {
            const int t = first + warp;
            keys += warp * ep; vals += warp * kMoeMaxK; who += warp * kMoeMaxK;
            const float top = vals[0];
            float sum = 0.0f, w = 0.0f;
            bool nan = false;
            if (lane < p.topk) w = __expf(vals[lane] - top);
            for (int e = lane; e < p.E; e += 32) {
                nan |= keys[e] == 1u;
                if (!p.norm) sum += __expf(key_value(keys[e]) - top);
            }
            if (p.norm) sum = w;
#pragma unroll
            for (int m = 16; m >= 1; m >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, m);
            nan = __any_sync(0xffffffffu, nan);
            if (lane < p.topk) {
                const int at = t * p.topk + lane, e = who[lane];
                w = nan ? __int_as_float(0x7fffffff) : w / sum;
                if (every) {
                    sel[at] = (uint16_t)e;
                    selw[at] = w;
                    atomicOr(reinterpret_cast<uint32_t*>(mask + e), 1u << t);    // (in whatever order the bits arrive; 64-bit ones are emulated)
                } else p.choice[at] = make_int2(e, __float_as_int(w));
                if (!every || cta == 0) {
                    if (p.ids) p.ids[at] = e;
                    if (p.weights) p.weights[at] = w;
                }
            }
        }
        if (!every) {
            met1 = met1 && meet_counted(p, p.gate + 2);
            if (threadIdx.x == 0) shared[1] = met1;
            for (int i = threadIdx.x; met1 && i < pairs; i += kMoeThreads) {
                const int2 c = __ldcg(p.choice + i);
                const int t = i / p.topk;
                sel[i] = (uint16_t)c.x;
                selw[i] = __int_as_float(c.y);
                atomicOr(reinterpret_cast<uint32_t*>(mask + c.x) + (t >> 5), 1u << (t & 31));
            }
        }
    }
    bar_consumers();
    // pairs sorted by expert, then token: every expert's first one; entries of at most `group` pairs of one expert
    if (warp == 0) {
        int np = 0, ne = 0, nh = 0;                       // pairs, entries and groups of h so far
#pragma unroll 1
        for (int e = lane; e - lane < p.E; e += 32) {
            const int cnt = e < p.E ? __popcll(mask[e]) : 0, gr = (cnt + 3) / 4;
            const int n = cnt <= p.group ? (cnt > 0) : (cnt + p.group - 1) / p.group;
            int sum = cnt << 16 | n, sumh = gr;           // the prefix sums (two at once)
#pragma unroll
            for (int m = 1; m < 32; m <<= 1) {
                const int a = __shfl_up_sync(0xffffffffu, sum, m), b = __shfl_up_sync(0xffffffffu, sumh, m);
                if (lane >= m) { sum += a; sumh += b; }
            }
            const int o = np + (sum >> 16) - cnt, i0 = ne + (sum & 0xffff) - n, h0 = nh + sumh - gr;
            if (e < p.E) off[e] = (uint16_t)o;
            for (int i = 0; i < n; ++i) {
                ent[i0 + i] = (uint32_t)e | (uint32_t)(o + i * p.group) << 9 | (uint32_t)min(p.group, cnt - i * p.group) << 19;
                hgroup[i0 + i] = (uint16_t)(h0 + i * (p.group / 4));
            }
            sum = __shfl_sync(0xffffffffu, sum, 31);
            np += sum >> 16; ne += sum & 0xffff; nh += __shfl_sync(0xffffffffu, sumh, 31);
        }
        if (lane == 0) shared[0] = ne;
    }
    bar_consumers();
    for (int i = threadIdx.x; i < pairs; i += kMoeThreads) {
        const int t = i / p.topk, e = sel[i], s = off[e] + __popcll(mask[e] & ((1ull << t) - 1ull));
        pair[s] = make_int2(t, __float_as_int(selw[i]));
    }
    }
    __syncthreads();
    if (!shared[1]) {                                     // a meeting did not come about; nothing is in flight
        if (threadIdx.x == 0) leave_meetings(p);
        pair_sync();
        return;
    }
    const int ents = shared[0], units = ents * nfb;
    const int u0 = (int)((int64_t)units * cta / ctas), u1 = (int)((int64_t)units * (cta + 1) / ctas);

    const int per_row_block = ents * nb2;                // blocks of a row block in phase 3: number j goes to warp j % 16 of the pair

    if (warp >= kMoeWarps) {
        // ---- the streams of weights and of h ---------------------------------------------------------------------------
        // Lane w < 8 follows the blocks of consumer warp w: eight places are waited for, and eight copies started, at a time (one
        // after the other they took 330 cycles a block, 170 ns, where the memory delivers one in 95 ns).
        const bool weights = warp == kMoeWarps;
        constexpr int kPer = kMoeWarps / kMoeHWarps;      // consumers a warp fetches h for, from number v0 on
        const int v0 = weights ? 0 : (warp - kMoeWarps - 1) * kPer, v1 = weights ? kMoeWarps : v0 + kPer;
        const int w = lane & (kMoeWarps - 1), in_phase2 = ((u1 - u0) * nb1 + kMoeWarps - 1 - w) / kMoeWarps;       // the warp's blocks there
        uint64_t* full = bars + w * kMoeDepth;
        unsigned char* ring = smem + w * p.depth * kMoeBlock;
        bool ok = true;
        int count = 0;                                    // copies started for the warp
        int at = weights ? 0 : in_phase2 % p.depth;       // the place of the next one; how often it has been around, mod 2
        uint32_t turn = weights ? 0u : (uint32_t)(in_phase2 / p.depth) & 1u;
        const uint32_t used0 = smem_u32(used + w * kMoeDepth);
        // Waits for the place of the next block of every lane that `has` one; false: a wait ran out
        auto places = [&](bool has) {
            uint32_t done = !has;
            if (has) asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(done) : "r"(used0 + at * 8), "r"(turn ^ 1u) : "memory");
            if (!__all_sync(0xffffffffu, done)) {
                if (has) done = wait_long(used0 + at * 8, turn ^ 1u);
                ok = __all_sync(0xffffffffu, done);
            }
            return ok;
        };
        auto next_place = [&](bool has) {
            if (!has) return;
            ++count;
            if (++at == p.depth) { at = 0; turn ^= 1u; }
        };
        if (weights) {
            int u = u0, kb = lane, i = u0 / nfb, f = u0 - i * nfb, strip = f / p.strip_units, in_strip = f - strip * p.strip_units;
#pragma unroll 1
            while (ok) {
                while (kb >= nb1 && u < u1) {
                    kb -= nb1; ++u;
                    if (++in_strip == p.strip_units) { in_strip = 0; ++strip; }
                    if (++f == nfb) { f = 0; strip = 0; ++i; }
                }
                const bool has = lane < kMoeWarps && u < u1;
                if (!__any_sync(0xffffffffu, has)) break;
                if (places(has) && has) {
                    mbar_expect_tx(full + at, kMoeBlock);
                    tma_load_4d(ring + at * kMoeBlock, &map_gu, full + at, kb * kMoeBlockK, in_strip * 16, 2 * strip, (int)(ent[i] & 511u));
                    next_place(has);
                }
                kb += kMoeWarps;
            }
        } else {
            ok = wait_long(smem_u32(met_bar), 0u) && shared[2];      // h is complete when the second meeting is over
        }
#pragma unroll 1
        for (int b = cta >> 1; ok && b < p.blocks; b += ctas >> 1) {
            int j = (cta & 1) * kMoeWarps + lane, kb = j, i = 0;
#pragma unroll 1
            while (ok) {
                const bool has = lane >= v0 && lane < v1 && j < per_row_block;
                if (!__any_sync(0xffffffffu, has)) break;
                while (kb >= nb2) { kb -= nb2; ++i; }
                if (!places(has)) break;
                if (weights) {
                    if (has) {
                        mbar_expect_tx(full + at, (uint32_t)(p.rows_per_block * 128));
                        tma_load_3d(ring + at * kMoeBlock, &map_d, full + at, kb * kMoeBlockK, b * p.rows_per_block, (int)(ent[i] & 511u));
                    }
                } else {
                    // Lane v describes consumer v's block -- where its h starts, how many rows and pieces of 8 there are, the place in the
                    // ring -- and the whole warp copies one after the other; nothing waits, so they overlap.
                    const int ii = min(i, ents - 1), cnt = (int)(ent[ii] >> 19);
                    const uint32_t from = (uint32_t)((int64_t)hgroup[ii] * 8 * p.h_pitch / 16) + (uint32_t)kb * 8u;       // in 16-byte units
                    const uint32_t what = has ? (uint32_t)cnt | (uint32_t)min(8, (p.I - kb * kMoeBlockK) / 8) << 8 | (uint32_t)at << 16 : 0u;
                    const int c = lane & 7, r = lane >> 3;
#pragma unroll
                    for (int vv = 0; vv < kPer; ++vv) {
                        const int v = v0 + vv;
                        const uint32_t fv = __shfl_sync(0xffffffffu, from, v), wv = __shfl_sync(0xffffffffu, what, v);
                        const int n = (int)(wv & 255u), pieces = (int)(wv >> 8 & 255u), slot = v * p.depth + (int)(wv >> 16);
                        const unsigned char* src = p.h + ((int64_t)fv + c) * 16 + (int64_t)r * p.h_pitch;
                        const uint32_t dst = smem_u32(smem + p.at_hring) + (uint32_t)(slot * kMoeHBlock);
#pragma unroll
                        for (int t = 0; t < 4; ++t)                  // rows 4 t ... 4 t + 3: values (t even) or remainders of group t / 2
                            if ((t >> 1) * 4 + r < n) copy_async(dst + block_at(t * 4 + r, c), c < pieces ? src + (int64_t)(t * 4) * p.h_pitch : p.h, c < pieces);
                        if (n) asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(h_bars + v * kMoeDepth + (int)(wv >> 16))) : "memory");
                    }
                }
                next_place(has);
                j += 2 * kMoeWarps; kb += 2 * kMoeWarps;
            }
        }
        if (!ok && lane == 0) atomicExch(&g_moe_status, 9);
        // whatever became of the consumers, every copy has landed before the CTA leaves
        if (!weights) asm volatile("cp.async.wait_all;" ::: "memory");
        else if (lane < kMoeWarps)
            for (int m = max(0, count - p.depth); m < count; ++m) wait_long(smem_u32(full + m % p.depth), (uint32_t)(m / p.depth) & 1u);
        pair_sync();
        return;
    }

    const int g = lane >> 2, q = lane & 3, fr = fragment_row(g);
    const uint32_t ring = smem_u32(smem) + (uint32_t)(warp * p.depth * kMoeBlock), hring = smem_u32(smem) + (uint32_t)(p.at_hring + warp * p.depth * kMoeHBlock), full0 = smem_u32(bars + warp * kMoeDepth);
    uint32_t slot = 0, parity = 0;
    bool ok = true;                                       // no wait of this warp has run out
    // The next block of the ring: wait for it, and give its place back.
    auto block = [&]() {
        ok = ok && wait_for(full0 + slot * 8, parity);
        return ring + slot * kMoeBlock;
    };
    auto done_with_block = [&]() {
        __syncwarp();                                     // every lane has read the block
        if (lane == 0) mbar_arrive(&used[warp * kMoeDepth + slot]);
        if (++slot == (uint32_t)p.depth) { slot = 0; parity ^= 1; }
    };

    // A block's weights as matrix fragments: [half of its k][16 rows of its 32], rows fr and fr + 8.  All eight loads are under way
    // before the first product waits for one; the two halves have sums of their own, so that no product waits for more than one other.
    // (With loads and products in turn a block took 1350 cycles.)
    struct Fragments { uint4 lo[2][2], hi[2][2]; };
    auto fragments = [&](uint32_t w) {
        Fragments a;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                a.lo[s][m] = lds128(w + block_at(m * 16 + fr, s * 4 + q));
                a.hi[s][m] = lds128(w + block_at(m * 16 + fr + 8, s * 4 + q));
            }
        return a;
    };

    // ---- 2. gate and up ------------------------------------------------------------------------------------------------
    {
        float4* red = reinterpret_cast<float4*>(smem + p.at_red);                // [buffer][column group][warp][lane]
        int i = u0 / nfb, f = u0 - i * nfb, cur = -1, first = 0, cnt = 0, kb = warp;     // kb: this warp's next block of the unit
        uint32_t xrow = 0;                                // this lane's column: its row of x
#pragma unroll 1
        for (int u = u0; u < u1; ++u) {
            if (i != cur) {
                first = (int)(ent[i] >> 9 & 1023u); cnt = (int)(ent[i] >> 19); cur = i;
                if (!p.all_x) {
                    bar_consumers();
                    stage_x(cnt, [&](int t) { return pair[first + t].x; });
                    bar_consumers();
                }
                const int col = min(g, cnt - 1);                                 // (columns behind the last repeat it; nobody looks at them)
                xrow = x0 + (uint32_t)((p.all_x ? pair[first + col].x : col) * p.x_pitch);
            }
            float acc[2][2][4];                           // [half of k][gate, up]
#pragma unroll
            for (int j = 0; j < 16; ++j) acc[j >> 3][j >> 2 & 1][j & 3] = 0.0f;
#pragma unroll 1
            for (; kb < nb1; kb += kMoeWarps) {
                const Fragments a = fragments(block());
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const uint4 b = lds128(xrow + (uint32_t)(kb * 128 + s * 64 + q * 16));
                    mma_half(acc[s][0], a.lo[s][0], a.hi[s][0], b);
                    mma_half(acc[s][1], a.lo[s][1], a.hi[s][1], b);
                }
                done_with_block();
            }
            kb -= nb1;
            // the warps' partial sums meet in shared memory (two buffers, one barrier a unit) and the warps take turns in
            // finishing a unit: a buffer is written again only behind the next barrier, which its reader has reached by then
            const int turn = u - u0;
            float4* out = red + (size_t)(turn & 1) * 2 * kMoeThreads;
#pragma unroll
            for (int m = 0; m < 2; ++m)
                out[m * kMoeThreads + threadIdx.x] = make_float4(acc[0][m][0] + acc[1][m][0], acc[0][m][1] + acc[1][m][1], acc[0][m][2] + acc[1][m][2], acc[0][m][3] + acc[1][m][3]);
            bar_consumers();
            if (warp == (turn & (kMoeWarps - 1))) {
                float4 a = make_float4(0.0f, 0.0f, 0.0f, 0.0f), b = a;
#pragma unroll
                for (int w = 0; w < kMoeWarps; ++w) {
                    const float4 v = out[w * 32 + lane], z = out[kMoeThreads + w * 32 + lane];
                    a.x += v.x; a.y += v.y; a.z += v.z; a.w += v.w;
                    b.x += z.x; b.y += z.y; b.z += z.z; b.w += z.w;
                }
                // gate and up of features fr (columns 2q and 2q + 1) and fr + 8 (the same columns) of the unit
                const int su = f / p.strip_units, in_strip = (f - su * p.strip_units) * 16 + fr;        // (strip, row in its half)
                const float h[4] = {a.x * logistic(a.x) * b.x, a.y * logistic(a.y) * b.y, a.z * logistic(a.z) * b.z, a.w * logistic(a.w) * b.w};
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int col = 2 * q + (c & 1), feat = su * p.gu_half + in_strip + (c >> 1) * 8;
                    if (col < cnt && in_strip + (c >> 1) * 8 < p.gu_half) {
                        __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(p.h + (int64_t)((hgroup[i] + (col >> 2)) * 8 + (col & 3)) * p.h_pitch) + feat;
                        const __nv_bfloat16 v = __float2bfloat16_rn(h[c]);
                        const float rest = h[c] - __bfloat162float(v);
                        dst[0] = v;
                        dst[2 * p.h_pitch] = __float2bfloat16_rn(rest == rest ? rest : 0.0f);     // (four rows on; inf - inf: the value says it all)
                    }
                }
            }
            if (++f == nfb) { f = 0; ++i; }
        }
    }
    const bool met = meet_counted(p, p.gate + 1);
    if (threadIdx.x == 0) { shared[2] = met; mbar_arrive(met_bar); leave_meetings(p); }

    // ---- 3. down -------------------------------------------------------------------------------------------------------
    {
        for (int i = threadIdx.x; i < kMoeWarps * p.T * kMoeRows; i += kMoeThreads) yacc[i] = 0.0f;   // (x is no longer read)
        bar_consumers();
        float* ya = yacc + (size_t)warp * p.T * kMoeRows;
        int turn = 0;                                     // row blocks done
        uint32_t hphase = 0, hcount = 0;                  // of the ring of h
#pragma unroll 1
        for (int b = met ? cta >> 1 : p.blocks; b < p.blocks; b += ctas >> 1) {
            const int r0 = b * p.rows_per_block, rows = min(p.rows_per_block, p.H - r0);
            int i = 0, kb = warp2;
#pragma unroll 1
            for (int j = warp2; j < per_row_block; j += 2 * kMoeWarps, kb += 2 * kMoeWarps) {
                while (kb >= nb2) { kb -= nb2; ++i; }
                const uint32_t en = ent[i];
                const int first = (int)(en >> 9 & 1023u), cnt = (int)(en >> 19);
                const int2 p0 = pair[first + min(q, cnt - 1)], p1 = pair[first + min(4 + q, cnt - 1)];      // token and weight of this lane's columns
                const uint32_t wb = block();
                ok = ok && wait_for(smem_u32(h_bars + warp * kMoeDepth + slot), hphase);
                const Fragments a = fragments(wb);
                const uint32_t hb = hring + slot * kMoeHBlock;
                auto product = [&](int n, const int2& pr) {
                    const uint4 h0 = lds128(hb + block_at(n * 8 + fr, q)), h1 = lds128(hb + block_at(n * 8 + fr, 4 + q));
                    float4* to = reinterpret_cast<float4*>(ya + sum_at(pr.x, fr));
                    float4 v = *to;
                    float acc[2][2][4];
#pragma unroll
                    for (int c = 0; c < 16; ++c) acc[c >> 3][c >> 2 & 1][c & 3] = 0.0f;
                    mma_half(acc[0][0], a.lo[0][0], a.hi[0][0], h0);
                    mma_half(acc[0][1], a.lo[0][1], a.hi[0][1], h0);
                    mma_half(acc[1][0], a.lo[1][0], a.hi[1][0], h1);
                    mma_half(acc[1][1], a.lo[1][1], a.hi[1][1], h1);
                    // weight * (this block's share of Wd h) into the warp's own sums: a token is in one column of an entry only.  (Columns
                    // 2 q and 2 q + 1 are h's rows fragment_row(2 q) = q and fragment_row(2 q + 1) = q + 4: a pair's value and remainder.)
                    if (n * 4 + q < cnt) {
                        const float wj = __int_as_float(pr.y);
                        v.x = fmaf(wj, acc[0][0][0] + acc[0][0][1] + (acc[1][0][0] + acc[1][0][1]), v.x);
                        v.y = fmaf(wj, acc[0][0][2] + acc[0][0][3] + (acc[1][0][2] + acc[1][0][3]), v.y);
                        v.z = fmaf(wj, acc[0][1][0] + acc[0][1][1] + (acc[1][1][0] + acc[1][1][1]), v.z);
                        v.w = fmaf(wj, acc[0][1][2] + acc[0][1][3] + (acc[1][1][2] + acc[1][1][3]), v.w);
                        *to = v;
                    }
                };
                product(0, p0);
                if (cnt > 4) product(1, p1);
                done_with_block();
                if (++hcount == (uint32_t)p.depth) { hcount = 0; hphase ^= 1; }
            }
            // the warps' sums, then the pair's, in this order; CTA 0 of the pair finishes the even tokens, CTA 1 the odd ones
            bar_consumers();
            for (int j = threadIdx.x; j < p.T * kMoeRows; j += kMoeThreads) {
                float s = 0.0f;
#pragma unroll
                for (int w = 0; w < kMoeWarps; ++w) s += yacc[w * p.T * kMoeRows + j];
                yacc[j] = s;
            }
            bar_consumers();
            if (threadIdx.x == 0) tell_other(&pair_bars[0], ~cta & 1);
            const bool there = wait_other(&pair_bars[0], turn & 1);
            ok = ok && there;
            for (int j = threadIdx.x; j < p.T * kMoeRows; j += kMoeThreads) {
                const int t = j / kMoeRows, r = sum_row(t, j & (kMoeRows - 1));
                if ((p.T > 1 && (t & 1) != (cta & 1)) || (p.T == 1 && (r & 1) != (cta & 1)) || r >= rows || !there) continue;
                uint32_t remote;
                float other;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(smem_u32(&yacc[j])), "r"(~cta & 1));
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(other) : "r"(remote) : "memory");
                float s = cta & 1 ? other + yacc[j] : yacc[j] + other;
                const int64_t at = (int64_t)t * p.H + r0 + r;
                if (p.residual) s += bf16_lo(p.residual[at]);
                reinterpret_cast<__nv_bfloat16*>(p.y)[at] = __float2bfloat16_rn(s);
            }
            ++turn;
            if (b + (ctas >> 1) < p.blocks) {              // another row block: the sums stay until the other CTA has read them
                bar_consumers();
                if (threadIdx.x == 0) tell_other(&pair_bars[1], ~cta & 1);
                ok = wait_other(&pair_bars[1], (turn - 1) & 1) && ok;
                for (int j = threadIdx.x; j < kMoeWarps * p.T * kMoeRows; j += kMoeThreads) yacc[j] = 0.0f;
                bar_consumers();
            }
        }
    }
    if (!ok && lane == 0) atomicExch(&g_moe_status, 9);
    pair_sync();                                          // (neither CTA leaves while the other may still read its sums)
}

// ---- host ------------------------------------------------------------------------------------------------------------
struct MoePlan {
    MoeParams p;
    int ctas, h_groups;
    int64_t gu_stride, d_stride;            // bytes from one expert to the next
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
    p.gu_half = (int32_t)(d->I / d->gu_strips); p.strip_units = (p.gu_half + 15) / 16;
    plan->gu_stride = d->gu_stride_bytes ? d->gu_stride_bytes : gu; plan->d_stride = d->d_stride_bytes ? d->d_stride_bytes : dn;
    if (plan->gu_stride >= (INT64_C(1) << 40) || plan->d_stride >= (INT64_C(1) << 40)) return fail(CCL_ERR_UNSUPPORTED, "ccl_moe_tokens: an expert stride is too large for a tensor map");
    plan->ctas = sms & ~1;                               // CTA pairs
    if (plan->ctas < d->T) return fail(CCL_ERR_UNSUPPORTED, "ccl_moe_tokens: %lld tokens need as many SMs (the device has %d)", (long long)d->T, sms);
    const int64_t pr = sms / 2, per = (d->H + pr * kMoeRows - 1) / (pr * kMoeRows);          // row blocks a pair takes
    p.rows_per_block = (int32_t)((d->H + pr * per - 1) / (pr * per));
    p.blocks = (int32_t)((d->H + p.rows_per_block - 1) / p.rows_per_block);
    const int64_t nb1 = (d->H + kMoeBlockK - 1) / kMoeBlockK;
    p.x_pitch = (int32_t)(nb1 * 128 + 64);               // (not a multiple of 128: neighbouring rows start in different banks)
    const int pairs = (int)(d->T * d->topk);
    // Groups of 4 of an expert's tokens, at most
    plan->h_groups = (pairs + 3 * std::min(pairs, d->E)) / 4;
    for (p.depth = kMoeDepth;; --p.depth) {
        if (p.depth < 2) return fail(CCL_ERR_UNSUPPORTED, "ccl_moe_tokens: this problem does not fit shared memory");
        const size_t room = kMoeSmem - 1024, ring = (size_t)kMoeWarps * p.depth * kMoeBlock;       // (the rings start at multiples of 1024)
        size_t at = ring;
        auto take = [&](size_t bytes) { const size_t a = at; at += up128(bytes); return (int32_t)a; };
        p.at_bars = take((size_t)(3 * kMoeWarps * kMoeDepth + 3) * 8 + 16);
        p.at_mask = take((size_t)d->E * 8);
        p.at_off = take((size_t)d->E * 2);
        p.at_sel = take((size_t)pairs * 2);
        p.at_selw = take((size_t)pairs * 4);
        p.at_pair = take((size_t)pairs * 8);
        const int most = std::min(pairs, d->E) + pairs / 4;                                        // entries
        p.at_ent = take((size_t)most * 4);
        p.at_hgroup = take((size_t)most * 2);
        at = (at + 1023) & ~(size_t)1023;
        // x and the units' partial sums (before them the top-k's keys); in phase 3 its own sums and h where both were
        const size_t keys = (size_t)(d->T <= 8 ? d->T : 1) * (size_t)((d->E + 3) / 4 * 16 + kMoeMaxK * 8);
        const size_t red = std::max((size_t)2 * 2 * kMoeThreads * 16, up128(keys)), yacc = ((size_t)kMoeWarps * (size_t)d->T * kMoeRows * 4 + 1023) & ~(size_t)1023;
        if (at + red > room) continue;
        const int64_t rows = (int64_t)((room - at - red) / (size_t)p.x_pitch);                     // of x that there is room for
        p.all_x = d->T <= rows;
        p.group = rows >= kMoeGroup || p.all_x ? kMoeGroup : 4;
        if (rows < std::min<int64_t>(4, d->T)) continue;
        p.at_region = (int32_t)at;
        p.at_hring = (int32_t)(at + yacc);
        p.at_red = take((size_t)(p.all_x ? d->T : p.group) * (size_t)p.x_pitch);                   // (x)
        p.at_red = take(red);
        plan->smem = std::max(at, (size_t)p.at_hring + (size_t)kMoeWarps * p.depth * kMoeHBlock) + 1024;
        if (plan->smem <= kMoeSmem) break;
    }
    p.h_pitch = (int64_t)up128((size_t)d->I * 2);
    plan->ws = up128((size_t)(d->T * d->E) * 4) + up128((size_t)(plan->ctas + 32 + pairs) * 8) + (size_t)plan->h_groups * 8 * (size_t)p.h_pitch;
    return CCL_OK;
}

static int moe_sms() {
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) == cudaSuccess && cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess && n > 0) return n;
    (void)cudaGetLastError();
    return 148;
}

static ccl_status launch_moe(const MoePlan& plan, const CUtensorMap& map_gu, const CUtensorMap& map_d, cudaStream_t st) {
    static std::atomic<uint64_t> configured{0};
    int dev = 0;
    CCL_CUDA_TRY(cudaGetDevice(&dev));
    if (dev >= 64 || !(configured.load() >> dev & 1)) {
        CCL_CUDA_TRY(cudaFuncSetAttribute(moe_tokens_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMoeSmem));
        if (dev < 64) configured.fetch_or(1ull << dev);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)plan.ctas, 1, 1);
    cfg.blockDim = dim3(kMoeBlockThreads, 1, 1);
    cfg.dynamicSmemBytes = plan.smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeCooperative;         // all CTAs resident at once, or the launch fails
    attr[0].val.cooperative = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    CCL_CUDA_TRY(cudaLaunchKernelEx(&cfg, moe_tokens_kernel, map_gu, map_d, plan.p));
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

// `absent`: 0, or the number of the meeting (1, 2) that waits for a CTA more than there are, for `wait_ns` at most
static ccl_status moe_impl(const ccl_moe_desc* d, const void* X_dev, const void* Wr_dev, const void* Wgu_dev, const void* Wd_dev, const void* residual_dev,
                           void* Y_dev, int32_t* ids_dev, float* weights_dev, void* ws_dev, size_t ws_bytes, void* cuda_stream, int absent, uint64_t wait_ns) {
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
    p.y = static_cast<uint16_t*>(Y_dev); p.ids = ids_dev; p.weights = weights_dev;
    unsigned char* ws = static_cast<unsigned char*>(ws_dev);
    p.logits = reinterpret_cast<float*>(ws);
    p.flags = reinterpret_cast<unsigned long long*>(ws + up128((size_t)p.T * p.E * 4));
    p.gate = p.flags + plan.ctas + 16;                   // (in another line than the flags)
    p.choice = reinterpret_cast<int2*>(p.gate + 16);
    p.h = ws + up128((size_t)p.T * p.E * 4) + up128((size_t)(plan.ctas + 32 + p.T * p.topk) * 8);
    // A mark that no workspace holds yet, whatever its contents.  A launch leaves the first meeting's flags and word cleared, whatever
    // became of it, so that a replayed CUDA graph may use its mark again.
    static std::atomic<unsigned long long> next{(unsigned long long)std::chrono::steady_clock::now().time_since_epoch().count() * 0x9E3779B97F4A7C15ull};
    do p.mark = next.fetch_add(0x9E3779B97F4A7C15ull); while (p.mark == 0);
    p.writers = absent == 1 ? plan.ctas + 1 : std::min(plan.ctas, (p.E + 15) / 16 * ((p.T + 7) / 8));
    p.quorum = absent == 2 ? plan.ctas + 1 : plan.ctas;
    p.wait_ns = wait_ns;
    // gate | up weights as {k, row of a strip's half, half of a strip, expert}: a block is the same 16 rows of a strip's gate and up
    // half.  Down weights as {k, row, expert}.  Rows and k past the end read as zero.
    CUtensorMap map_gu, map_d;
    {
        const uint64_t H = (uint64_t)p.H, I = (uint64_t)p.I, E = (uint64_t)p.E, half = (uint64_t)p.gu_half;
        const uint64_t dims[4] = {H, half, 2 * (I / half), E}, strides[3] = {H * 2, half * H * 2, (uint64_t)plan.gu_stride};
        const uint32_t box[4] = {kMoeBlockK, kMoeRows / 2, 2, 1};
        if ((s = encode_tmap(&map_gu, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, Wgu_dev, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B))) return s;
        const uint64_t ddims[3] = {I, H, E}, dstrides[2] = {I * 2, (uint64_t)plan.d_stride};
        const uint32_t dbox[3] = {kMoeBlockK, (uint32_t)p.rows_per_block, 1};
        if ((s = encode_tmap(&map_d, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, Wd_dev, ddims, dstrides, dbox, CU_TENSOR_MAP_SWIZZLE_128B))) return s;
    }
    return launch_moe(plan, map_gu, map_d, reinterpret_cast<cudaStream_t>(cuda_stream));
}

extern "C" ccl_status ccl_moe_tokens(const ccl_moe_desc* d, const void* X_dev, const void* Wr_dev, const void* Wgu_dev, const void* Wd_dev,
                                     const void* residual_dev, void* Y_dev, int32_t* ids_dev, float* weights_dev, void* ws_dev, size_t ws_bytes,
                                     void* cuda_stream) {
    return moe_impl(d, X_dev, Wr_dev, Wgu_dev, Wd_dev, residual_dev, Y_dev, ids_dev, weights_dev, ws_dev, ws_bytes, cuda_stream, 0, kWaitLimitNs);
}

extern "C" ccl_status ccl_selftest_moe_timeout(const ccl_moe_desc* d, const void* X_dev, const void* Wr_dev, const void* Wgu_dev, const void* Wd_dev,
                                               void* Y_dev, void* ws_dev, size_t ws_bytes, int32_t meeting, uint32_t limit_us, void* cuda_stream) {
    if (meeting != 1 && meeting != 2) return fail(CCL_ERR_INVALID_ARG, "ccl_selftest_moe_timeout: meeting must be 1 or 2");
    if (limit_us < 1 || limit_us > 100000) return fail(CCL_ERR_INVALID_ARG, "ccl_selftest_moe_timeout: limit_us must be in [1, 100000]");
    return moe_impl(d, X_dev, Wr_dev, Wgu_dev, Wd_dev, nullptr, Y_dev, nullptr, nullptr, ws_dev, ws_bytes, cuda_stream, meeting, (uint64_t)limit_us * 1000ull);
}
