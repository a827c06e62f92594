// matmul_fp8.cu -- the block-scaled 8-bit matrix product
//   out[m, n] = sum_kb sa[m, kb] sw[n / 128, kb] sum_{k in kb} a[m, k] w[n, k]
// of e4m3 activations a [M, K] (one scale per row and 128 elements of K) and
// e4m3 weights w [N, K] (one scale per 128 x 128 block), fp32 sums, one
// rounding to the output type.
//
// D = w a^T on tcgen05 (kind::f8f6f4): 128 weight rows are the MMA's M (TMEM
// lanes), NT rows of a its N.  The tensor core sums one 128-wide K block (4
// MMAs) into a TMEM buffer; the epilogue adds it to the running sums in
// registers with its scales, sum[n, m] += (sa sw) d[n, m], while the MMAs of
// the next K blocks fill the other buffers.
//
// Roles (192 threads): warp 0 TMA producer (two K blocks of 128 rows of w and of
// NT rows of a at a time into a ring), warp 1 TMEM allocator and MMA issuer,
// warps 2-5 epilogue (one TMEM lane quarter each).  The scales of the
// NT rows of a over the CTA's K range stay in shared memory; those of w
// travel through a lane each, 32 K blocks at a time.
//
// Work items are (128 weight rows, NT rows of a), dealt round-robin to
// clusters of S CTAs.  The CTAs of a cluster split K; each sends every CTA its
// sums of that CTA's share of the rows of a (asynchronous stores into the
// other's shared memory, which its mbarrier counts: no cluster barrier, and a
// sender may leave), which adds them in rank order, so that the result does not
// depend on timing.
//
// Bound by the weights' stream for large w (16 x 151936 x 4096: 96 us, 6.5 TB/s
// of w alone), by the chain first copy - MMAs - join - store for small ones
// (1 x 4096 x 4096: 5.9 us).
#include "matmul_fp8.h"

namespace xp {

namespace {

constexpr int MM_BN = 128;                             // weight rows per tile
constexpr int MM_EPI = 4;                              // epilogue warps
constexpr int MM_THREADS = 32 * (2 + MM_EPI);
constexpr uint32_t MM_W_STAGE = MM_BN * QBLOCK;        // 16 KB
constexpr int MM_SKB = 2;                              // K blocks of a stage
constexpr int MM_MAX_STAGES = 6;

template <int NT>
struct MmShape {
    static constexpr uint32_t A_STAGE = NT * QBLOCK;
    static constexpr uint32_t STAGE = MM_SKB * (MM_W_STAGE + A_STAGE);   // w's K blocks, then a's
    static constexpr int NBUF = 4;
    static constexpr uint32_t TMEM_COLS = NBUF * NT;   // a power of two from 64 to 256
    static constexpr uint32_t IDESC = idesc_e4m3(MM_BN, NT);
    static constexpr size_t PART = (size_t)NT * MM_BN * 4;    // sums of a K split
};

struct MmBars {
    uint64_t full[MM_MAX_STAGES], empty[MM_MAX_STAGES];
    uint64_t tfull[4], tempty[4];
    uint64_t drain, joined;
    long long since;
    uint32_t tmem_base;
    int abort;
};

__device__ __forceinline__ void tma_load_3d(void *dst, const CUtensorMap *map, uint64_t *bar, int x, int y, int z)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
        : "memory");
}

__device__ __forceinline__ void mm_epi_bar() { asm volatile("bar.sync 1, %0;" ::"n"(MM_EPI * 32) : "memory"); }

__device__ __forceinline__ void mm_store(const MmArgs &g, int m, int n, float v)
{
    const int64_t at = (int64_t)m * g.ldo + n;
    if (g.bf16) static_cast<uint16_t *>(g.out)[at] = f2bf(v);
    else static_cast<float *>(g.out)[at] = v;
}

// grid: clusters of S CTAs; MM_THREADS threads.
template <int NT>
__global__ void __launch_bounds__(MM_THREADS, 2)
    k_matmul_fp8(const __grid_constant__ MmArgs g, const __grid_constant__ CUtensorMap tmap_w,
                 const __grid_constant__ CUtensorMap tmap_a)
{
    using Sh = MmShape<NT>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *base = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int stages = g.stages;
    uint8_t *after = base + stages * Sh::STAGE;
    float *table = reinterpret_cast<float *>(after);                       // [K blocks of this CTA][NT]
    float *part = reinterpret_cast<float *>(after + g.table_bytes);        // [S][groups of vw rows of a][128][vw] (S > 1)
    __shared__ MmBars sh;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int S = g.S, rank = S > 1 ? (int)cluster_rank() : 0;
    const int KB = (g.K + QBLOCK - 1) / QBLOCK;
    const int KP = (KB + MM_SKB - 1) / MM_SKB;             // stages of K, split over the cluster
    const int kb0 = KP * rank / S * MM_SKB, kb1 = min(KB, KP * (rank + 1) / S * MM_SKB);
    const bool whole = g.K % QBLOCK == 0;                  // the maps: (128 columns, rows, K blocks), else (K, rows)
    const int NRB = (g.N + MM_BN - 1) / MM_BN, NC = (g.M + NT - 1) / NT;
    const int64_t items = (int64_t)NRB * NC;               // item i: weight rows 128 (i / NC), rows of a NT (i % NC)
    const int64_t first = blockIdx.x / S, step = gridDim.x / S;

    if (threadIdx.x == 0) {
        for (int i = 0; i < stages; ++i) { mbar_init(&sh.full[i], 1); mbar_init(&sh.empty[i], 1); }
        for (int i = 0; i < Sh::NBUF; ++i) { mbar_init(&sh.tfull[i], 1); mbar_init(&sh.tempty[i], MM_EPI); }
        mbar_init(&sh.drain, 1);
        mbar_init(&sh.joined, 1);
        sh.abort = 0;
        sh.since = 0;
        fence_barrier_init();
        tma_prefetch_desc(&tmap_w);
        tma_prefetch_desc(&tmap_a);
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
                for (int kb = kb0; kb < kb1; kb += MM_SKB) {
                    if (!mm_wait(&sh.empty[stage], phase ^ 1, abort)) { ok = false; break; }
                    uint8_t *dw = base + stage * Sh::STAGE, *da = dw + MM_SKB * MM_W_STAGE;
                    if (whole) {
                        // one copy per operand (a copy takes the same time at 16 and
                        // at 32 KB); a K block past the end reads as zero
                        mbar_expect_tx(&sh.full[stage], Sh::STAGE);
                        tma_load_3d(dw, &tmap_w, &sh.full[stage], 0, rb * MM_BN, kb);
                        tma_load_3d(da, &tmap_a, &sh.full[stage], 0, mc * NT, kb);
                    } else {
                        const int n = min(MM_SKB, kb1 - kb);
                        mbar_expect_tx(&sh.full[stage], n * (MM_W_STAGE + Sh::A_STAGE));
                        for (int i = 0; i < n; ++i) {
                            tma_load_2d(dw + i * MM_W_STAGE, &tmap_w, &sh.full[stage], (kb + i) * QBLOCK, rb * MM_BN);
                            tma_load_2d(da + i * Sh::A_STAGE, &tmap_a, &sh.full[stage], (kb + i) * QBLOCK, mc * NT);
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
            for (int kb = kb0; kb < kb1 && ok; kb += MM_SKB) {
                ok = __all_sync(0xffffffffu, mm_wait(&sh.full[stage], phase, abort));
                const uint32_t w_lo = lo0 + stage * (Sh::STAGE >> 4), a_lo = w_lo + (MM_SKB * MM_W_STAGE >> 4);
                for (int i = 0; i < MM_SKB && kb + i < kb1 && ok; ++i) {
                    ok = __all_sync(0xffffffffu, mm_wait(&sh.tempty[buf], tphase ^ 1, abort));
                    if (!ok) break;
                    tc_fence_after();
                    if (elect_one()) {
                        tc_mma_fp8_kblock(tmem_u + buf * NT, w_lo + i * (MM_W_STAGE >> 4), a_lo + i * (Sh::A_STAGE >> 4), hi,
                                          Sh::IDESC);
                        tc_commit(&sh.tfull[buf]);
                        if (i + 1 == MM_SKB || kb + i + 1 == kb1) tc_commit(&sh.empty[stage]);
                    }
                    __syncwarp();
                    if (++buf == Sh::NBUF) { buf = 0; tphase ^= 1; }
                }
                if (++stage == stages) { stage = 0; phase ^= 1; }
            }
        }
        if (elect_one()) tc_commit(&sh.drain);
        __syncwarp();
        int dummy = 0;
        mm_wait(&sh.drain, 0, &dummy, MM_WAIT_CYCLES / 20);
        __syncwarp();
    } else {
        // ------------------------------------------------------ epilogue
        const int et = threadIdx.x - 64, q = warp & 3;
        const uint32_t lane_base = (uint32_t)(q * 32) << 16;
        int buf = 0, cur = -1;
        uint32_t tphase = 0;
        bool ok = true;
        for (int64_t it = first; it < items; it += step) {
            const int rb = (int)(it / NC), mc = (int)(it % NC);
            if (mc != cur) {
                // the scales of this chunk's rows of a, [K block][row]
                mm_epi_bar();
                const int n = kb1 - kb0;
                for (int i = et; i < n * NT; i += MM_EPI * 32) {
                    const int m = mc * NT + i / n, kb = i % n;
                    table[kb * NT + i / n] = m < g.M ? g.sa[(int64_t)m * g.ldsa + kb0 + kb] : 0.0f;
                }
                mm_epi_bar();
                cur = mc;
            }
            float acc[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[j] = 0.0f;
            const float *swr = g.sw + (int64_t)rb * g.ldsw;
            float sw32 = 0.0f;
            for (int kb = kb0; kb < kb1; ++kb) {
                const int i = kb - kb0;
                if ((i & 31) == 0) sw32 = kb + lane < kb1 ? swr[kb + lane] : 0.0f;
                const float sw = __shfl_sync(0xffffffffu, sw32, i & 31);
                if (ok) ok = mm_wait(&sh.tfull[buf], tphase, abort, MM_WAIT_CYCLES, S > 1 ? &sh.since : nullptr);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                float d[NT];
#pragma unroll
                for (int j = 0; j < NT; j += 16) tmem_ld16(tmem + lane_base + buf * NT + j, d + j);
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.tempty[buf]);
                if (++buf == Sh::NBUF) { buf = 0; tphase ^= 1; }
                const float4 *tr = reinterpret_cast<const float4 *>(table + i * NT);
#pragma unroll
                for (int j = 0; j < NT; j += 4) {
                    const float4 s = tr[j / 4];
                    acc[j] = fmaf(d[j], s.x * sw, acc[j]);
                    acc[j + 1] = fmaf(d[j + 1], s.y * sw, acc[j + 1]);
                    acc[j + 2] = fmaf(d[j + 2], s.z * sw, acc[j + 2]);
                    acc[j + 3] = fmaf(d[j + 3], s.w * sw, acc[j + 3]);
                }
            }
            const int row = q * 32 + lane, n = rb * MM_BN + row;
            if (S == 1) {
                if (ok && n < g.N)
#pragma unroll
                    for (int j = 0; j < NT; ++j)
                        if (mc * NT + j < g.M) mm_store(g, mc * NT + j, n, acc[j]);
            } else {
                // S > 1: one item per cluster (the host's grid), joined below; rows
                // of a travel in groups of 4 (2 where a share has no more)
                const int share = NT / S;
                __syncwarp();
                cluster_wait();
                if (share >= 4) {
#pragma unroll
                    for (int j = 0; j < NT; j += 4)
                        if (mc * NT + j < g.M)
                            st_async4(cluster_addr(part + ((rank * share + j % share) * MM_BN + row * 4), j / share),
                                      cluster_addr(&sh.joined, j / share), acc + j);
                } else {
#pragma unroll
                    for (int j = 0; j < NT; j += 2)
                        if (mc * NT + j < g.M)
                            st_async2(cluster_addr(part + (rank * share * MM_BN + row * 2), j / share),
                                      cluster_addr(&sh.joined, j / share), acc + j);
                }
            }
        }
    }
    if (S > 1) {
        __syncwarp();
        if (warp < 2) cluster_wait();
        const int rb = (int)(first / NC), mc = (int)(first % NC), share = NT / S, vw = share >= 4 ? 4 : 2;
        const int m0 = mc * NT + rank * share;                 // this CTA's rows of a: m0 .. m0 + rows - 1
        const int rows = max(0, min(share, g.M - m0)), sent = (rows + vw - 1) / vw * vw;
        if (sent > 0) {
            if (threadIdx.x == 0) mbar_expect_tx(&sh.joined, S * sent * MM_BN * 4);
            if (mm_wait_joined(&sh.joined, abort))
                for (int i = threadIdx.x; i < rows * MM_BN; i += MM_THREADS) {
                    const int j = i / MM_BN, row = i % MM_BN, n = rb * MM_BN + row;
                    float v = 0.0f;
                    for (int s = 0; s < S; ++s) v += part[(s * share + j / vw * vw) * MM_BN + row * vw + j % vw];
                    if (n < g.N) mm_store(g, m0 + j, n, v);
                }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, Sh::TMEM_COLS);
    }
    if (threadIdx.x == 0 && sh.abort) set_status(g.status, ST_TIMEOUT);
}

// A launch's shape and its estimated time in us beyond what every launch costs
// (about 3), from times measured on GB300:
//   few rows   a stage (two K blocks) takes a CTA 0.58 us (NT = 16) or 0.66 (32)
//              (16 x 4096 x 4096 without a split: 12.4 us, with S = 4: 6.0);
//              joining a split costs about 0.6 us and 0.075 for each row of a
//              (16 x 4096 x 512 with S = 2: 5.3 us, 4.1 without); with two CTAs
//              on an SM a stage takes 1.43 times as long and an item 1.5 stages
//              more, and so it has where a CTA takes several; the weights stream
//              at 6.3 TB/s
//   many rows  0.41 us for a K block of a 128 x 256 tile, 0.6 to start and 2 for
//              the epilogue of 128 rows (512 x 1024 x 1024: 9.2 us, 300 x 4096 x
//              4096: 19), with K split over 2, 4 and 8 CTAs 1.7 and 1.9, 2.7, 3.1
//              (300 x 600 x 8192: 33 us, 18.4, 13.8, 11.4), 1.5 and 0.7 more where
//              out's rows start anywhere, two fifths of the weights' stream at
//              5.9 TB/s (512 x 4096 x 4096 with S = 2: 14.9).  Where a CTA takes
//              several tiles, 0.5 us for a K block, 1 to start, 2 between tiles,
//              or the stream (64 x 151936 x 256: 15.9)
// At 24 x 151936 x 4096 the choice is NT = 32 (96 us; 16: 102, many rows: 118),
// at 64 x 151936 x 4096 many rows (103; 126 and 177), at 300 x 2048 x 1024
// NT = 16 (6.1; 32: 10.3, many rows: 9.1), at 512 x 4096 x 4096 many rows with
// S = 2 (14.9; without a split 19.7, few rows 31.6).
struct MmPlan {
    int NT, S;
    float us;
};

// Clusters of 2, 4 or 8 CTAs with an SM each that the current device runs at a time
// (0, so no split, where it cannot tell).
int resident_clusters(int S)
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
    cfg.blockDim = dim3(MM_THREADS);
    cfg.dynamicSmemBytes = MM_SMEM_LIMIT - 1024;
    cfg.attrs = a;
    cfg.numAttrs = 1;
    if (allow_smem(once, k_matmul_fp8<16>, MM_SMEM_LIMIT - 1024) != cudaSuccess) return 0;
    if (cudaOccupancyMaxActiveClusters(&n, k_matmul_fp8<16>, &cfg) != cudaSuccess) { (void)cudaGetLastError(); return 0; }
    if (dev < MAX_DEVICES) known[dev][i].store(n + 1, std::memory_order_relaxed);
    return n;
}

MmPlan plan_few(int M, int N, int KB, int NT, int sms)
{
    const int KP = (KB + MM_SKB - 1) / MM_SKB;
    const int64_t items = (int64_t)((N + MM_BN - 1) / MM_BN) * ((M + NT - 1) / NT);
    const float stage = NT == 16 ? 0.58f : 0.66f, join = 0.6f + 0.075f * (M < NT ? M : NT);
    if (items >= 2 * sms) {
        const int slots = 2 * sms;
        const float rounds = 0.5f * ((float)items / slots + (float)((items + slots - 1) / slots));
        const float stream = (float)N * KB * QBLOCK / 6.3e6f, work = rounds * (KP + 1.5f) * stage * 1.43f;
        return {NT, 1, stream > work ? stream : work};
    }
    MmPlan best{NT, 1, items <= sms ? KP * stage : (float)((items + sms - 1) / sms) * (KP + 1.5f) * stage};
    for (int S = 2; S <= 8 && S <= KP && items <= resident_clusters(S); S *= 2) {
        const float us = (KP + S - 1) / S * stage + join;
        if (us < best.us) best = {NT, S, us};
    }
    return best;
}

// ragged: out's rows do not all start on 32 bytes.
MmPlan plan_mm(int M, int N, int KB, bool ragged, int sms)
{
    MmPlan best = plan_few(M, N, KB, 16, sms);
    if (M > 16) {
        const MmPlan b = plan_few(M, N, KB, 32, sms);
        if (b.us < best.us) best = b;
        // NT = 0: the kernel for many rows
        const int64_t tiles = (int64_t)((M + 127) / 128) * ((N + 255) / 256);
        const float stream = (float)N * KB * QBLOCK / 5.9e6f;
        if (tiles > sms) {
            const float work = 1.0f + 0.5f * KB + (0.5f * KB + 2.0f) * ((tiles - 1) / sms);
            const float us = stream > work ? stream : work;
            if (us < best.us) best = {0, 1, us};
        }
        const float full = M < 128 ? (M + 31) / 32 / 4.0f : 1.0f;                   // part of the epilogue that has rows
        const float epilogue[4] = {2.0f, 1.9f, 2.7f, 3.1f};
        for (int i = 0, S = 1; S <= 8 && S <= KB && tiles <= (S == 1 ? sms : resident_clusters(S)); ++i, S *= 2) {
            const float us = (S == 1 ? 0.6f : 1.7f) + epilogue[i] * full + 0.41f * ((KB + S - 1) / S) + 0.4f * stream +
                             (ragged ? S == 1 ? 1.5f : 0.7f : 0.0f);
            if (us < best.us) best = {0, S, us};
        }
    }
    return best;
}

template <int NT>
int launch_mm(MmArgs g, int S, const void *a, int64_t lda, const void *w, int64_t ldw, int sms, cudaStream_t st)
{
    using Sh = MmShape<NT>;
    const int KB = (g.K + QBLOCK - 1) / QBLOCK, KP = (KB + MM_SKB - 1) / MM_SKB;
    const int64_t items = (int64_t)((g.N + MM_BN - 1) / MM_BN) * ((g.M + NT - 1) / NT);
    g.S = S;
    // many items: two CTAs per SM, so that one streams while the other starts,
    // drains or stores (1 x 151936 x 256: 11.2 -> 7.8 us, 16 x 151936 x 4096: 98
    // -> 96); a cluster has one item and takes as many stages as it has K blocks
    // for
    const size_t table = (size_t)((KP + S - 1) / S) * MM_SKB * NT * 4;        // a multiple of 128
    const size_t fixed = 1024 + table + (S > 1 ? Sh::PART : 0) + 1024;
    const int want = (KP + S - 1) / S;
    int per_sm = items >= 2 * sms ? 2 : 1;
    size_t limit = MM_SMEM_LIMIT / per_sm;
    if (fixed + 2 * Sh::STAGE > limit) { limit = MM_SMEM_LIMIT; per_sm = 1; }
    if (fixed + 2 * Sh::STAGE > limit) return XPRESS_ERR_UNSUPPORTED;
    g.stages = (int)((limit - fixed) / Sh::STAGE);
    if (g.stages > MM_MAX_STAGES) g.stages = MM_MAX_STAGES;
    if (S > 1 && g.stages > want) g.stages = want;
    g.table_bytes = (uint32_t)table;
    const size_t smem = fixed - 1024 + (size_t)g.stages * Sh::STAGE;
    static OncePerDevice once;
    XH_CUDA(allow_smem(once, k_matmul_fp8<NT>, MM_SMEM_LIMIT - 1024));
    // by K blocks only where they are whole: past the last one the rows'
    // padding would be read
    CUtensorMap tw{}, ta{};
    const bool ok = g.K % QBLOCK == 0
                        ? tmap_bytes_kblocks(&tw, w, (uint64_t)KB, (uint64_t)g.N, (uint64_t)ldw, MM_BN, MM_SKB) &&
                              tmap_bytes_kblocks(&ta, a, (uint64_t)KB, (uint64_t)g.M, (uint64_t)lda, NT, MM_SKB)
                        : tmap_bytes(&tw, w, (uint64_t)g.K, (uint64_t)g.N, (uint64_t)ldw, QBLOCK, MM_BN) &&
                              tmap_bytes(&ta, a, (uint64_t)g.K, (uint64_t)g.M, (uint64_t)lda, QBLOCK, NT);
    if (!ok) return XPRESS_ERR_CUDA;
    const int64_t grid = S > 1 ? items * S : items < per_sm * sms ? items : per_sm * sms;
    XH_CUDA(launch_head(k_matmul_fp8<NT>, dim3((unsigned)grid), MM_THREADS, smem, st, (unsigned)S, g, tw, ta));
    return XPRESS_OK;
}

}  // namespace
}  // namespace xp

using namespace xp;

extern "C" size_t xpress_matmul_fp8_workspace_size(void) { return 256; }

extern "C" int xpress_matmul_fp8(const xpress_matmul_args *in, void *ws, size_t ws_bytes, void *stream)
{
    if (!in || in->M < 0 || in->N < 1 || in->K < 1 || !in->a || !in->a_scale || !in->w || !in->w_scale || !in->out)
        return XPRESS_ERR_INVALID_ARG;
    if (in->out_dtype != XPRESS_F32 && in->out_dtype != XPRESS_BF16) return XPRESS_ERR_UNSUPPORTED;
    const int KB = (in->K - 1) / QBLOCK + 1;
    if (in->lda < in->K || in->ldw < in->K || in->lda % 16 || in->ldw % 16 || !aligned(in->a, 16) ||
        !aligned(in->w, 16) || in->ldo < in->N || in->ld_a_scale < KB || in->ld_w_scale < KB ||
        !aligned(in->a_scale, 4) || !aligned(in->w_scale, 4) ||
        !aligned(in->out, in->out_dtype == XPRESS_BF16 ? 2 : 4))
        return XPRESS_ERR_INVALID_ARG;
    if (in->K > 65536 || in->M > MAX_DIM || in->N > MAX_DIM) return XPRESS_ERR_UNSUPPORTED;
    if (!ws || !aligned(ws, 256) || ws_bytes < xpress_matmul_fp8_workspace_size()) return XPRESS_ERR_WORKSPACE;
    if (in->M == 0) return XPRESS_OK;
    const int sms = current_sms();
    if (sms < 1) return XPRESS_ERR_CUDA;
    MmArgs g{};
    g.M = in->M; g.N = in->N; g.K = in->K;
    g.sa = in->a_scale; g.sw = in->w_scale;
    g.ldsa = in->ld_a_scale; g.ldsw = in->ld_w_scale;
    g.out = in->out; g.ldo = in->ldo;
    g.bf16 = in->out_dtype == XPRESS_BF16;
    g.status = static_cast<int32_t *>(ws);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const MmPlan p = plan_mm(in->M, in->N, KB, !mm_out_vec(g), sms);
    if (p.NT == 16) return launch_mm<16>(g, p.S, in->a, in->lda, in->w, in->ldw, sms, st);
    if (p.NT == 32) return launch_mm<32>(g, p.S, in->a, in->lda, in->w, in->ldw, sms, st);
    g.S = p.S;
    return launch_mm_wide(g, in->a, in->lda, in->w, in->ldw, sms, st);
}
