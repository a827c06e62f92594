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
// Roles (192 threads): warp 0 TMA producer (a 128 x 128 box of w and an
// NT x 128 box of a per K block into a ring), warp 1 TMEM allocator and MMA
// issuer, warps 2-5 epilogue (one TMEM lane quarter each).  The scales of the
// NT rows of a over the CTA's K range stay in shared memory; those of w
// travel through a lane each, 32 K blocks at a time.
//
// Work items are (128 weight rows, NT rows of a), dealt round-robin to
// clusters of S CTAs.  The CTAs of a cluster split K; each leaves its sums in
// its shared memory, and every CTA adds a share of the rows of a over the
// cluster in rank order, so that the result does not depend on timing.
#include <mutex>

#include "matmul_fp8.h"

namespace xp {

namespace {

constexpr int MM_BN = 128;                             // weight rows per tile
constexpr int MM_EPI = 4;                              // epilogue warps
constexpr int MM_THREADS = 32 * (2 + MM_EPI);
constexpr uint32_t MM_W_STAGE = MM_BN * QBLOCK;        // 16 KB
constexpr int MM_MAX_STAGES = 12;

template <int NT>
struct MmShape {
    static constexpr uint32_t A_STAGE = NT * QBLOCK;
    static constexpr uint32_t STAGE = MM_W_STAGE + A_STAGE;
    static constexpr int NBUF = 4;
    static constexpr uint32_t TMEM_COLS = NBUF * NT;   // a power of two from 64 to 256
    static constexpr uint32_t IDESC = idesc_e4m3(MM_BN, NT);
    static constexpr size_t PART = (size_t)NT * MM_BN * 4;    // sums of a K split
};

struct MmBars {
    uint64_t full[MM_MAX_STAGES], empty[MM_MAX_STAGES];
    uint64_t tfull[4], tempty[4];
    uint64_t drain;
    uint32_t tmem_base;
    int abort;
};

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float *v)
{
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, "
        "%14, %15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}

// A float of CTA `rank`'s shared memory at this CTA's address `p`.
__device__ __forceinline__ float ld_cluster(const float *p, uint32_t rank)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(cluster_addr(p, rank)) : "memory");
    return v;
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
__global__ void __launch_bounds__(MM_THREADS, 1)
    k_matmul_fp8(const __grid_constant__ MmArgs g, const __grid_constant__ CUtensorMap tmap_w,
                 const __grid_constant__ CUtensorMap tmap_a)
{
    using Sh = MmShape<NT>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *base = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int stages = g.stages;
    uint8_t *after = base + stages * Sh::STAGE;
    float *table = reinterpret_cast<float *>(after);                       // [K blocks of this CTA][NT]
    float *part = reinterpret_cast<float *>(after + g.table_bytes);        // [NT][128] (S > 1)
    __shared__ MmBars sh;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int S = g.S, rank = S > 1 ? (int)cluster_rank() : 0;
    const int KB = (g.K + QBLOCK - 1) / QBLOCK;
    const int kb0 = (int)((int64_t)KB * rank / S), kb1 = (int)((int64_t)KB * (rank + 1) / S);
    const int NRB = (g.N + MM_BN - 1) / MM_BN, NC = (g.M + NT - 1) / NT;
    const int64_t items = (int64_t)NRB * NC;               // item i: weight rows 128 (i / NC), rows of a NT (i % NC)
    const int64_t first = blockIdx.x / S, step = gridDim.x / S;

    if (threadIdx.x == 0) {
        for (int i = 0; i < stages; ++i) { mbar_init(&sh.full[i], 1); mbar_init(&sh.empty[i], 1); }
        for (int i = 0; i < Sh::NBUF; ++i) { mbar_init(&sh.tfull[i], 1); mbar_init(&sh.tempty[i], MM_EPI); }
        mbar_init(&sh.drain, 1);
        sh.abort = 0;
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
    pdl_trigger();
    pdl_wait();

    if (warp == 0) {
        // ------------------------------------------------------- producer
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0, pending = 0, pend_par = 0;
            bool ok = true;
            for (int64_t it = first; it < items && ok; it += step) {
                const int rb = (int)(it / NC), mc = (int)(it % NC);
                for (int kb = kb0; kb < kb1; ++kb) {
                    if (!mm_wait(&sh.empty[stage], phase ^ 1, abort)) { ok = false; break; }
                    uint8_t *dst = base + stage * Sh::STAGE;
                    mbar_expect_tx(&sh.full[stage], Sh::STAGE);
                    tma_load_2d(dst, &tmap_w, &sh.full[stage], kb * QBLOCK, rb * MM_BN);
                    tma_load_2d(dst + MM_W_STAGE, &tmap_a, &sh.full[stage], kb * QBLOCK, mc * NT);
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
            for (int kb = kb0; kb < kb1; ++kb) {
                ok = mm_wait(&sh.tempty[buf], tphase ^ 1, abort) && mm_wait(&sh.full[stage], phase, abort);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    const uint32_t w_lo = lo0 + stage * (Sh::STAGE >> 4);
                    tc_mma_fp8_kblock(tmem_u + buf * NT, w_lo, w_lo + (MM_W_STAGE >> 4), hi, Sh::IDESC);
                    tc_commit(&sh.empty[stage]);
                    tc_commit(&sh.tfull[buf]);
                }
                __syncwarp();
                if (++stage == stages) { stage = 0; phase ^= 1; }
                if (++buf == Sh::NBUF) { buf = 0; tphase ^= 1; }
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
                if (ok) ok = mm_wait(&sh.tfull[buf], tphase, abort);
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
                // S > 1: one item per cluster (the host's grid), joined below
#pragma unroll
                for (int j = 0; j < NT; ++j) part[j * MM_BN + row] = acc[j];
            }
        }
    }
    if (S > 1) {
        // every thread of every CTA of the cluster comes here, whatever its role saw
        __syncwarp();
        cluster_arrive();
        cluster_wait();
        const int rb = (int)(first / NC), mc = (int)(first % NC);
        for (int i = threadIdx.x; i < (NT / S) * MM_BN; i += MM_THREADS) {
            const int j = rank * (NT / S) + i / MM_BN, row = i % MM_BN;
            const int m = mc * NT + j, n = rb * MM_BN + row;
            if (m < g.M && n < g.N) {
                float v = 0.0f;
                for (int s = 0; s < S; ++s) v += ld_cluster(part + j * MM_BN + row, s);
                mm_store(g, m, n, v);
            }
        }
        __syncwarp();
        cluster_arrive();
        cluster_wait();
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, Sh::TMEM_COLS);
    }
    if (threadIdx.x == 0 && sh.abort) set_status(g.status, ST_TIMEOUT);
}

template <int NT>
int launch_mm(MmArgs g, const void *a, int64_t lda, const void *w, int64_t ldw, int sms, cudaStream_t st)
{
    using Sh = MmShape<NT>;
    const int KB = (g.K + QBLOCK - 1) / QBLOCK;
    const int64_t items = (int64_t)((g.N + MM_BN - 1) / MM_BN) * ((g.M + NT - 1) / NT);
    // few tiles: split K over the CTAs of a cluster, at least two K blocks each
    int S = 1;
    while (S < 8 && items * S * 2 <= sms && KB >= S * 4) S *= 2;
    g.S = S;
    const size_t table = (((size_t)((KB + S - 1) / S + 1) * NT * 4) + 127) & ~size_t(127);
    const size_t fixed = 1024 + table + (S > 1 ? Sh::PART : 0) + 1024;
    if (fixed + 3 * Sh::STAGE > MM_SMEM_LIMIT) return XPRESS_ERR_UNSUPPORTED;
    g.stages = (int)((MM_SMEM_LIMIT - fixed) / Sh::STAGE);
    if (g.stages > MM_MAX_STAGES) g.stages = MM_MAX_STAGES;
    g.table_bytes = (uint32_t)table;
    const size_t smem = fixed - 1024 + (size_t)g.stages * Sh::STAGE;
    static std::once_flag once;
    static cudaError_t attr;
    std::call_once(once, [] {
        attr = cudaFuncSetAttribute(k_matmul_fp8<NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)MM_SMEM_LIMIT - 1024);
    });
    if (attr != cudaSuccess) { (void)cudaGetLastError(); return XPRESS_ERR_CUDA; }
    CUtensorMap tw{}, ta{};
    if (!tmap_bytes(&tw, w, (uint64_t)g.K, (uint64_t)g.N, (uint64_t)ldw, QBLOCK, MM_BN) ||
        !tmap_bytes(&ta, a, (uint64_t)g.K, (uint64_t)g.M, (uint64_t)lda, QBLOCK, NT))
        return XPRESS_ERR_CUDA;
    const int64_t grid = S > 1 ? items * S : items < sms ? items : sms;
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
    if (in->M > 64) return launch_mm_wide(g, in->a, in->lda, in->w, in->ldw, sms, st);
    if (in->M <= 16) return launch_mm<16>(g, in->a, in->lda, in->w, in->ldw, sms, st);
    return launch_mm<32>(g, in->a, in->lda, in->w, in->ldw, sms, st);
}
