// linear.cu -- the bf16 matrix product with its epilogue
//   out[m, n] = residual[m, n] + act(sum_k x[m, k] w[n, k] + bias[n])
// for x [M, K], w [N, K] bf16, fp32 sums, one rounding to the output type.  The sums
// are the tensor core's, whose additions truncate: with normal operands a dot product is
// 1e-9 of itself too small for each element of K that it adds up in one go (1.6e-5 at
// K = 16384, a quarter of that split in four), as a library's bf16 product is.
//
// This kernel, for few rows of x: D = w x^T on tcgen05 (kind::f16), 128 weight rows
// the MMA's M (TMEM lanes), NT rows of x its N, so that hardly a lane is idle and w
// is read once.  The sums of a tile stay in TMEM over all of K; two tiles' worth of
// columns let the next tile's products run under the epilogue of the last.
//
// Roles (192 threads): warp 0 TMA producer (two K blocks of 128 rows of w and of
// NT rows of x per copy), warp 1 TMEM allocator and MMA issuer, warps 2-5 epilogue:
// one TMEM lane quarter each to shared memory, and from there four columns of four
// rows to a thread, so that a warp stores 128 consecutive outputs of a row.  What it
// reads of the residual for the first of them is asked for before the sums are waited
// for.
//
// Where tiles are few, the CTAs of a cluster of S split K; each sends every CTA its
// sums of that CTA's share of the rows (asynchronous stores that the receiver's
// mbarrier counts), which adds them in rank order: the result does not depend on
// timing.
#include <type_traits>

#include "linear.h"

namespace xp {

namespace {

constexpr int LF_BN = 128;                             // weight rows per tile
constexpr int LF_EPI = 4;                              // epilogue warps
constexpr int LF_THREADS = 32 * (2 + LF_EPI);
constexpr uint32_t LF_W = LF_BN * 128;                 // 16 KB: a K block of w
constexpr int LF_SKB = 2;                              // K blocks of a stage
constexpr int LF_MAX_STAGES = 6;

template <int NT>
struct FewShape {
    static constexpr uint32_t X = NT * 128;            // a K block of x
    static constexpr uint32_t STAGE = LF_SKB * (LF_W + X);       // w's K blocks, then x's
    static constexpr uint32_t TMEM_COLS = 2 * NT < 32 ? 32 : 2 * NT;
    static constexpr uint32_t IDESC = idesc_bf16(LF_BN, NT);
    // Sums, of a K split those of this CTA's rows from each of the CTAs: by 4 rows of x
    // (2 where a split leaves no more to a CTA), 4 x 33 places of the weight rows n % 4, n / 4.
    static constexpr int PLACES = 132;
    static constexpr size_t PART = (size_t)NT * PLACES * 4;
};

__device__ __forceinline__ int place_of(int n) { return n % 4 * 33 + n / 4; }

struct FewBars {
    uint64_t full[LF_MAX_STAGES], empty[LF_MAX_STAGES];
    uint64_t tfull[2], tempty[2];
    uint64_t drain, joined;
    long long since;
    uint32_t tmem_base;
    int abort;
};

__device__ __forceinline__ void lf_epi_bar() { asm volatile("bar.sync 1, %0;" ::"n"(LF_EPI * 32) : "memory"); }

// grid: clusters of S CTAs; LF_THREADS threads; stages of STAGE bytes, then the sums.
template <int NT, bool BF16>
__global__ void __launch_bounds__(LF_THREADS, NT <= 32 ? 2 : 1)
    k_linear_few(const __grid_constant__ LinArgs g, const __grid_constant__ CUtensorMap tmap_w,
                 const __grid_constant__ CUtensorMap tmap_x)
{
    using Sh = FewShape<NT>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *base = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int stages = g.stages;
    float *part = reinterpret_cast<float *>(base + stages * Sh::STAGE);
    __shared__ FewBars sh;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int S = g.S, rank = S > 1 ? (int)cluster_rank() : 0;
    const int KB = (g.K + LK - 1) / LK;
    const int KP = (KB + LF_SKB - 1) / LF_SKB;             // stages of K, split over the cluster
    const int kb0 = (int)((int64_t)KP * rank / S) * LF_SKB, kb1 = min(KB, (int)((int64_t)KP * (rank + 1) / S) * LF_SKB);
    const bool whole = g.K % LK == 0;                      // the maps: (64 columns, rows, K blocks), else (K, rows)
    const int NRB = (g.N + LF_BN - 1) / LF_BN, NC = (g.M + NT - 1) / NT;
    const int64_t items = (int64_t)NRB * NC;               // item i: weight rows 128 (i / NC), rows of x NT (i % NC)
    const int64_t first = blockIdx.x / S, step = gridDim.x / S;

    if (threadIdx.x == 0) {
        for (int i = 0; i < stages; ++i) { mbar_init(&sh.full[i], 1); mbar_init(&sh.empty[i], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&sh.tfull[i], 1); mbar_init(&sh.tempty[i], LF_EPI); }
        mbar_init(&sh.drain, 1);
        mbar_init(&sh.joined, 1);
        sh.abort = 0;
        sh.since = 0;
        fence_barrier_init();
        tma_prefetch_desc(&tmap_w);
        tma_prefetch_desc(&tmap_x);
    }
    if (warp == 1) { tmem_alloc(&sh.tmem_base, Sh::TMEM_COLS); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem_base;
    volatile int *abort = &sh.abort;
    if (S > 1) cluster_arrive();                            // waited for before the first access to another CTA
    pdl_wait();

    if (warp == 0) {
        // ------------------------------------------------------- producer
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0, pending = 0, pend_par = 0;
            bool ok = true;
            for (int64_t it = first; it < items && ok; it += step) {
                const int rb = (int)(it / NC), mc = (int)(it % NC);
                for (int kb = kb0; kb < kb1; kb += LF_SKB) {
                    if (!mm_wait(&sh.empty[stage], phase ^ 1, abort)) { ok = false; break; }
                    uint8_t *dw = base + stage * Sh::STAGE, *dx = dw + LF_SKB * LF_W;
                    if (whole) {
                        // one copy per operand; a K block past the end reads as zero
                        mbar_expect_tx(&sh.full[stage], Sh::STAGE);
                        tma_load_3d(dw, &tmap_w, &sh.full[stage], 0, rb * LF_BN, kb);
                        tma_load_3d(dx, &tmap_x, &sh.full[stage], 0, mc * NT, kb);
                    } else {
                        const int n = min(LF_SKB, kb1 - kb);
                        mbar_expect_tx(&sh.full[stage], n * (LF_W + Sh::X));
                        for (int i = 0; i < n; ++i) {
                            tma_load_2d(dw + i * LF_W, &tmap_w, &sh.full[stage], (kb + i) * 128, rb * LF_BN);
                            tma_load_2d(dx + i * Sh::X, &tmap_x, &sh.full[stage], (kb + i) * 128, mc * NT);
                        }
                    }
                    pending |= 1u << stage;
                    pend_par = (pend_par & ~(1u << stage)) | (phase << stage);
                    if (++stage == stages) { stage = 0; phase ^= 1; }
                }
            }
            // no copy may still be landing when the CTA leaves
            int dummy = 0;
            for (int st = 0; st < stages; ++st)
                if (pending & (1u << st)) mm_wait(&sh.full[st], (pend_par >> st) & 1, &dummy, MM_WAIT_CYCLES / 20);
        }
    } else if (warp == 1) {
        // ---------------------------------------------------- MMA issuer
        // the whole warp runs the loop, so that the descriptors stay in uniform
        // registers, and one elected lane issues
        const uint32_t base_u = __shfl_sync(0xffffffffu, smem_u32(base), 0);
        const uint32_t tmem_u = __shfl_sync(0xffffffffu, tmem, 0);
        const uint32_t lo0 = (uint32_t)smem_desc_sw128(base_u), hi = (uint32_t)(smem_desc_sw128(base_u) >> 32);
        int stage = 0, buf = 0;
        uint32_t phase = 0, tphase = 0;
        bool ok = true;
        for (int64_t it = first; it < items && ok; it += step) {
            ok = __all_sync(0xffffffffu, mm_wait(&sh.tempty[buf], tphase ^ 1, abort));
            for (int kb = kb0; kb < kb1 && ok; kb += LF_SKB) {
                ok = __all_sync(0xffffffffu, mm_wait(&sh.full[stage], phase, abort));
                if (!ok) break;
                tc_fence_after();
                const uint32_t w_lo = lo0 + stage * (Sh::STAGE >> 4), x_lo = w_lo + (LF_SKB * LF_W >> 4);
                if (elect_one()) {
                    for (int i = 0; i < LF_SKB && kb + i < kb1; ++i)
                        tc_mma_bf16_kblock<1>(tmem_u + buf * NT, w_lo + i * (LF_W >> 4), x_lo + i * (Sh::X >> 4), hi, Sh::IDESC,
                                              kb + i > kb0);
                    tc_commit(&sh.empty[stage]);
                    if (kb + LF_SKB >= kb1) tc_commit(&sh.tfull[buf]);
                }
                __syncwarp();
                if (++stage == stages) { stage = 0; phase ^= 1; }
            }
            buf ^= 1;
            if (buf == 0) tphase ^= 1;
        }
        if (elect_one()) tc_commit(&sh.drain);
        __syncwarp();
        int dummy = 0;
        mm_wait(&sh.drain, 0, &dummy, MM_WAIT_CYCLES / 20);
        __syncwarp();
    } else {
        // ------------------------------------------------------ epilogue
        const int q = warp & 3, row = q * 32 + lane, w0 = warp - 2;
        const uint32_t lane_base = (uint32_t)(q * 32) << 16;
        const int share = NT / S, vw = share >= 4 ? 4 : 2;         // rows of x that end here, and travel together
        int buf = 0;
        uint32_t tphase = 0;
        bool ok = true;
        for (int64_t it = first; it < items; it += step) {
            const int rb = (int)(it / NC), mc = (int)(it % NC), n0 = rb * LF_BN + 4 * lane;
            const int rows = min(NT, g.M - mc * NT);                // of the item
            const int m0 = mc * NT + rank * share, mine = max(0, min(share, g.M - m0));      // of this CTA
            Quad<true> bias;
            lin_bias4(g, n0, bias);
            Quad<BF16> next[4];
            auto fetch = [&](int j0) {
                if (g.res && n0 < g.N)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (j0 + j < mine) lin_res4(g, m0 + j0 + j, n0, next[j]);
            };
            fetch(4 * w0);
            if (ok) ok = mm_wait(&sh.tfull[buf], tphase, abort, MM_WAIT_CYCLES, S > 1 ? &sh.since : nullptr);
            ok = __all_sync(0xffffffffu, ok);
            tc_fence_after();
            if (S > 1) { __syncwarp(); cluster_wait(); }            // one item per cluster (the host's grid)
            const int place = place_of(row);
#pragma unroll 1
            for (int j0 = 0; j0 < NT && j0 < rows; j0 += 16) {
                float d[16];
                if (ok) tmem_ld16(tmem + lane_base + buf * NT + j0, d);
                else
#pragma unroll
                    for (int j = 0; j < 16; ++j) d[j] = 0.0f;
                if (S == 1) {
#pragma unroll
                    for (int j = 0; j < 16; j += 4)
                        *reinterpret_cast<float4 *>(part + ((j0 + j) * Sh::PLACES + place * 4)) = make_float4(d[j], d[j + 1], d[j + 2], d[j + 3]);
                } else if (share >= 4) {
#pragma unroll
                    for (int j = 0; j < 16; j += 4) {
                        const int jj = j0 + j;
                        if (jj < rows)
                            st_async4(cluster_addr(part + ((rank * share + jj % share) * Sh::PLACES + place * 4), jj / share),
                                      cluster_addr(&sh.joined, jj / share), d + j);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 16; j += 2) {
                        const int jj = j0 + j;
                        if (jj < rows)
                            st_async2(cluster_addr(part + (rank * share * Sh::PLACES + place * 2), jj / share),
                                      cluster_addr(&sh.joined, jj / share), d + j);
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.tempty[buf]);
            if (S == 1) {
                lf_epi_bar();
            } else if (mine > 0) {
                if (threadIdx.x == 64) mbar_expect_tx(&sh.joined, S * ((mine + vw - 1) / vw * vw) * LF_BN * 4);
                ok = __all_sync(0xffffffffu, mm_wait_joined(&sh.joined, abort)) && ok;
            }
#pragma unroll 1
            for (int j0 = 4 * w0; j0 < mine; j0 += 4 * LF_EPI) {
                float v[4][4];                                       // [row][column]
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j][c] = 0.0f;
                for (int s = 0; s < S; ++s)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const int at = c * 33 + lane;
                        if (vw == 4) {
                            const float4 p = *reinterpret_cast<const float4 *>(part + ((s * share + j0) * Sh::PLACES + at * 4));
                            v[0][c] += p.x; v[1][c] += p.y; v[2][c] += p.z; v[3][c] += p.w;
                        } else {
                            const float2 p = *reinterpret_cast<const float2 *>(part + (s * share * Sh::PLACES + at * 2));
                            v[0][c] += p.x; v[1][c] += p.y;
                        }
                    }
                Quad<BF16> r[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) r[j] = next[j];
                fetch(j0 + 4 * LF_EPI);
#pragma unroll
                for (int j = 0; j < 4; ++j) lin_add4(v[j], bias);
                lin_act<BF16, 16>(g.act, v[0]);
                if (ok && n0 < g.N)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (j0 + j < mine) lin_store4(g, m0 + j0 + j, n0, v[j], r[j]);
            }
            if (S == 1) lf_epi_bar();                               // the sums have been read
            buf ^= 1;
            if (buf == 0) tphase ^= 1;
        }
    }
    if (S > 1 && warp < 2) { __syncwarp(); cluster_wait(); }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, Sh::TMEM_COLS);
    }
    if (threadIdx.x == 0 && sh.abort) set_status(g.status, ST_TIMEOUT);
}

struct LinPlan {
    int NT, S;             // NT = 0: the kernel for many rows, S pairs of CTAs to a tile's K
};

// Clusters of S CTAs with an SM each that the current device runs at a time (0, so
// no split, where it cannot tell).
int resident(int S)
{
    static std::atomic<int> known[MAX_DEVICES][3];       // plus 1
    static OncePerDevice once;
    const int i = S == 2 ? 0 : S == 4 ? 1 : 2;
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) { (void)cudaGetLastError(); return 0; }
    if (dev < MAX_DEVICES && (n = known[dev][i].load(std::memory_order_relaxed)) > 0) return n - 1;
    cudaLaunchAttribute a[1];
    a[0].id = cudaLaunchAttributeClusterDimension;
    a[0].val.clusterDim.x = S;
    a[0].val.clusterDim.y = a[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(S);
    cfg.blockDim = dim3(LF_THREADS);
    cfg.dynamicSmemBytes = MM_SMEM_LIMIT - 1024;
    cfg.attrs = a;
    cfg.numAttrs = 1;
    if (allow_smem(once, k_linear_few<16, true>, MM_SMEM_LIMIT - 1024) != cudaSuccess) return 0;
    if (cudaOccupancyMaxActiveClusters(&n, k_linear_few<16, true>, &cfg) != cudaSuccess) { (void)cudaGetLastError(); return 0; }
    if (dev < MAX_DEVICES) known[dev][i].store(n + 1, std::memory_order_relaxed);
    return n;
}

// The launch's shape by its estimated time in us, from times measured on GB300 with
// bias, SiLU and residual, all from HBM:
//   few rows   a stage (two K blocks) takes a CTA 0.30 us (NT = 16), 0.33 (32) or 0.42
//              (64) (1 x 4096 x 4096 without a split 14.3, 64 x 4096 x 16384 52), an item
//              1.5 more, with two CTAs on an SM 1.43 times as long; joining a split 1;
//              the weights stream at 6.3 TB/s (64 x 16384 x 4096: 28)
//   many rows  0.59 for a stage of a 256 x 256 tile, 12 to start and for the last tile's
//              epilogue (500 x 500 x 64: 11.9, 2048 x 4096 x 4096 in two rounds: 51), 7 at
//              least from tile to tile, the weights' stream at 5 TB/s
// At 128 x 4096 x 16384 the choice is NT = 64 with S = 2 (34; many rows with S = 2:
// 52), at 512 x 4096 x 4096 many rows with S = 2 (24; without a split 30, NT = 64: 31).
// Of 28 shapes timed with every plan, 25 get their fastest to 5 %, the worst 1.12 of it.
LinPlan plan_linear(int M, int N, int KB, int sms)
{
    const int KP = (KB + LF_SKB - 1) / LF_SKB;
    const float bytes = 2.0f * N * KB * LK;
    LinPlan best{16, 1};
    float least = INFINITY;
    const auto offer = [&](int NT, int S, float us) {
        if (us < least) { least = us; best = {NT, S}; }
    };
    const float stage[3] = {0.30f, 0.33f, 0.42f};
    for (int i = 0, NT = 16; i < 3; ++i, NT *= 2) {
        const int64_t items = (int64_t)((N + LF_BN - 1) / LF_BN) * ((M + NT - 1) / NT);
        const int per_sm = NT <= 32 && items >= 2 * sms ? 2 : 1;
        const float stream = bytes / 6.3e6f, rounds = (float)((items + per_sm * sms - 1) / (per_sm * sms));
        for (int S = 1; S <= 8 && 2 * S <= KP + 1; S *= 2) {
            if (S > 1 && items > resident(S)) break;
            const float work = rounds * ((KP + S - 1) / S * stage[i] + 1.5f) * (per_sm == 2 ? 1.43f : 1.0f);
            offer(NT, S, 3.5f + 0.02f * NT + (S > 1 ? 1.0f : 0.0f) + (work > stream ? work : stream));
        }
        if (M <= NT) break;
    }
    if (M > 64) {
        const int64_t tiles = (int64_t)((M + 255) / 256) * ((N + 255) / 256), pairs = sms / 2;
        const float stream = bytes / 5e6f;
        for (int S = 1; S <= 4 && S <= KP; S *= 2) {
            if (S > 1 && tiles > resident(2 * S)) break;
            const float tile = 0.59f * ((KP + S - 1) / S), rounds = S > 1 ? 1.0f : (float)((tiles + pairs - 1) / pairs);
            const float work = tile + (rounds - 1.0f) * (tile > 7.0f ? tile : 7.0f);
            offer(0, S, 12.0f + (work > stream ? work : stream));
        }
    }
    return best;
}

template <int NT, bool BF16>
int launch_few(LinArgs g, int S, const void *x, int64_t ldx, const void *w, int64_t ldw, int sms, cudaStream_t st)
{
    using Sh = FewShape<NT>;
    const int KB = (g.K + LK - 1) / LK, KP = (KB + LF_SKB - 1) / LF_SKB, want = (KP + S - 1) / S;
    const int64_t items = (int64_t)((g.N + LF_BN - 1) / LF_BN) * ((g.M + NT - 1) / NT);
    g.S = S;
    // two CTAs per SM where there are many items, so that one streams while the other
    // starts, drains or stores
    const int per_sm = NT <= 32 && items >= 2 * sms ? 2 : 1;
    const size_t fixed = 1024 + Sh::PART + 1024;
    g.stages = (int)((MM_SMEM_LIMIT / per_sm - fixed) / Sh::STAGE);
    if (g.stages > LF_MAX_STAGES) g.stages = LF_MAX_STAGES;
    if (S > 1 && g.stages > want) g.stages = want;          // a cluster has one item
    const size_t smem = fixed - 1024 + (size_t)g.stages * Sh::STAGE;
    static OncePerDevice once;
    XH_CUDA(allow_smem(once, k_linear_few<NT, BF16>, MM_SMEM_LIMIT - 1024));
    // by K blocks only where they are whole: past the last one the rows' padding
    // would be read
    CUtensorMap tw{}, tx{};
    const bool ok = g.K % LK == 0
                        ? tmap_bytes_kblocks(&tw, w, (uint64_t)KB, (uint64_t)g.N, (uint64_t)ldw * 2, LF_BN, LF_SKB) &&
                              tmap_bytes_kblocks(&tx, x, (uint64_t)KB, (uint64_t)g.M, (uint64_t)ldx * 2, NT, LF_SKB)
                        : tmap_bytes(&tw, w, (uint64_t)g.K * 2, (uint64_t)g.N, (uint64_t)ldw * 2, 128, LF_BN) &&
                              tmap_bytes(&tx, x, (uint64_t)g.K * 2, (uint64_t)g.M, (uint64_t)ldx * 2, 128, NT);
    if (!ok) return XPRESS_ERR_CUDA;
    const int64_t grid = S > 1 ? items * S : items < per_sm * sms ? items : per_sm * sms;
    XH_CUDA(launch_head(k_linear_few<NT, BF16>, dim3((unsigned)grid), LF_THREADS, smem, st, (unsigned)S, g, tw, tx));
    return XPRESS_OK;
}

}  // namespace
}  // namespace xp

using namespace xp;

extern "C" size_t xpress_linear_workspace_size(void) { return 256; }

extern "C" int xpress_linear(const xpress_linear_args *in, void *ws, size_t ws_bytes, void *stream)
{
    if (!in || in->M < 0 || in->N < 1 || in->K < 1 || !in->x || !in->w || !in->out) return XPRESS_ERR_INVALID_ARG;
    if ((in->out_dtype != XPRESS_F32 && in->out_dtype != XPRESS_BF16) || in->act < XPRESS_ACT_NONE || in->act > XPRESS_ACT_RELU)
        return XPRESS_ERR_UNSUPPORTED;
    const bool bf16 = in->out_dtype == XPRESS_BF16;
    const uintptr_t es = bf16 ? 2 : 4;
    if (in->ldx < in->K || in->ldw < in->K || in->ldx % 8 || in->ldw % 8 || !aligned(in->x, 16) || !aligned(in->w, 16) ||
        in->ldo < in->N || !aligned(in->out, es) || !aligned(in->bias, 2) ||
        (in->residual && (in->ldr < in->N || !aligned(in->residual, es) ||
                          (in->residual == in->out && in->ldr != in->ldo && in->M > 1))))
        return XPRESS_ERR_INVALID_ARG;
    if (in->K > MAX_DIM / 64 || in->M > MAX_DIM || in->N > MAX_DIM) return XPRESS_ERR_UNSUPPORTED;
    if (!ws || !aligned(ws, 256) || ws_bytes < xpress_linear_workspace_size()) return XPRESS_ERR_WORKSPACE;
    if (in->M == 0) return XPRESS_OK;
    const int sms = current_sms();
    if (sms < 1) return XPRESS_ERR_CUDA;
    LinArgs g{};
    g.M = in->M; g.N = in->N; g.K = in->K;
    g.bias = static_cast<const uint16_t *>(in->bias);
    g.res = in->residual; g.ldr = in->ldr;
    g.out = in->out; g.ldo = in->ldo;
    g.act = in->act;
    g.bf16 = bf16;
    g.quads = aligned(g.out, 4 * es) && g.ldo % 4 == 0 && aligned(g.bias, 8) && (!g.res || (aligned(g.res, 4 * es) && g.ldr % 4 == 0));
    g.status = static_cast<int32_t *>(ws);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const LinPlan p = plan_linear(in->M, in->N, (in->K + LK - 1) / LK, sms);
    const auto few = [&](auto nt) {
        constexpr int NT = decltype(nt)::value;
        return bf16 ? launch_few<NT, true>(g, p.S, in->x, in->ldx, in->w, in->ldw, sms, st)
                    : launch_few<NT, false>(g, p.S, in->x, in->ldx, in->w, in->ldw, sms, st);
    };
    if (p.NT == 16) return few(std::integral_constant<int, 16>());
    if (p.NT == 32) return few(std::integral_constant<int, 32>());
    if (p.NT == 64) return few(std::integral_constant<int, 64>());
    g.S = p.S;
    return launch_lin_wide(g, in->x, in->ldx, in->w, in->ldw, sms, st);
}
