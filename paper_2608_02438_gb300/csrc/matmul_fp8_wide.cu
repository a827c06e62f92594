// matmul_fp8_wide.cu -- the block-scaled 8-bit product (see matmul_fp8.cu for
// the definition) for many rows of a: bound by the tensor cores and by what
// feeds them, not by the weights' stream.
//
// A pair of CTAs (tcgen05 cta_group::2) takes a tile of 256 rows of a (the
// MMA's M, 128 in each CTA's TMEM) by 256 weight rows (N; each CTA stages half
// of them, and the pair's MMA reads both halves), so that every byte brought
// from L2 feeds twice the products of a single CTA's tile.  One 128-wide K
// block is 4 MMAs into one of two TMEM buffers of 256 columns; the epilogue
// adds the other to the running sums with its scale.  With a's rows on the
// lanes a thread has one scale per K block (its row's, times that of the
// weight block its 128 columns are), and the addition is 64 packed FMAs.
//
// Roles (384 threads): warp 0 TMA producer (both CTAs load their own halves;
// the copies complete on the leader's barrier), warp 1 TMEM allocator and, in
// the leader, MMA issuer; warps 4-11 epilogue (lane quarter warp % 4, column
// half (warp - 4) / 4) with the 128 sums of a thread in registers: the first
// warpgroup hands its registers to theirs.
#include <mutex>

#include "matmul_fp8.h"

namespace xp {

namespace {

constexpr int WD_BM = 256, WD_BN = 256;                 // tile of a pair
constexpr int WD_EPI = 8;
constexpr int WD_THREADS = 32 * (4 + WD_EPI);
// registers per thread: the kernel is launched with 168 x 384 (the most that
// 65,536 allow); 80 x 128 + 208 x 256 = 63,488 of those 64,512
constexpr int WD_REGS_FEW = 80, WD_REGS_MANY = 208;
constexpr uint32_t WD_HALF = 128 * QBLOCK;              // 16 KB: 128 rows of one operand
constexpr uint32_t WD_STAGE = 2 * WD_HALF;
constexpr int WD_STAGES = 6;
constexpr uint32_t WD_IDESC = idesc_e4m3(WD_BM, WD_BN);
constexpr size_t WD_TILE = 32 * 33 * 4;                 // a warp's transpose
constexpr size_t WD_SMEM = 1024 + WD_STAGES * WD_STAGE + WD_EPI * WD_TILE;
constexpr int WD_BAND = 16;                             // row tiles that share the weights while they are in L2

struct WideBars {
    uint64_t full[WD_STAGES], empty[WD_STAGES];
    uint64_t tfull[2], tempty[2];
    uint64_t drain;
    uint32_t tmem_base;
    int abort;
};

__device__ __forceinline__ void tma_load_pair(void *dst, const CUtensorMap *map, uint32_t bar, int x, int y)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], "
        "[%4];" ::"r"(smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar)
        : "memory");
}

__device__ __forceinline__ void tc_mma_fp8_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc,
                                                uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}

// Arrive on `bar` of both CTAs once every MMA issued so far by this thread is done.
__device__ __forceinline__ void tc_commit_pair(uint64_t *bar)
{
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
        ::"r"(smem_u32(bar)), "h"((uint16_t)3)
        : "memory");
}

// mbar_wait for a barrier that the other CTA of the pair arrives on.
__device__ __forceinline__ bool mbar_wait_cluster(uint64_t *bar, uint32_t parity, volatile int *abort)
{
    unsigned long long t0 = 0;
    for (uint32_t it = 0;; ++it) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(smem_u32(bar)), "r"(parity), "r"(20000u)
            : "memory");
        if (ok) return true;
        if ((it & 7u) == 0) {
            if (*abort) return false;
            if (t0 == 0) t0 = globaltimer();
            else if (globaltimer() - t0 > 2000000000ull) { *abort = 1; return false; }
        }
    }
}

__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// 32 TMEM columns of this warp's lane quarter.
__device__ __forceinline__ void tmem_ld32w(uint32_t taddr, uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, "
        "%14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]),
          "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]),
          "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}

// (a0, a1) += (d0, d1) * (f0, f1)
__device__ __forceinline__ void fma2(uint64_t &a, uint32_t d0, uint32_t d1, uint64_t f)
{
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(d0), "r"(d1));
    asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(a) : "l"(d), "l"(f));
}
__device__ __forceinline__ void halves(uint64_t a, float &lo, float &hi)
{
    uint32_t l, h;
    asm("mov.b64 {%0, %1}, %2;" : "=r"(l), "=r"(h) : "l"(a));
    lo = __uint_as_float(l);
    hi = __uint_as_float(h);
}

__device__ __forceinline__ void store32(void *p, const uint32_t (&w)[8])
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]),
                 "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
}

// Tile t in the order of bands of WD_BAND row tiles, within a band the row
// tiles of one column tile after another.
__device__ __forceinline__ void tile_at(int64_t t, int MT, int NT, int &mt, int &nt)
{
    const int64_t band = t / ((int64_t)WD_BAND * NT);
    const int m0 = (int)band * WD_BAND, rows = min(WD_BAND, MT - m0);
    const int64_t in = t - band * WD_BAND * NT;
    mt = m0 + (int)(in % rows);
    nt = (int)(in / rows);
}

// grid: pairs of CTAs, WD_THREADS threads, WD_SMEM bytes; vec: out's rows start on 32 bytes.
__global__ void __launch_bounds__(WD_THREADS, 1)
    k_matmul_fp8_wide(const __grid_constant__ MmArgs g, const __grid_constant__ CUtensorMap tmap_a,
                      const __grid_constant__ CUtensorMap tmap_w, int vec)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t *base = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ WideBars sh;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = cluster_rank();
    const int KB = (g.K + QBLOCK - 1) / QBLOCK;
    const int MT = (g.M + WD_BM - 1) / WD_BM, NT = (g.N + WD_BN - 1) / WD_BN;
    const int64_t tiles = (int64_t)MT * NT, first = blockIdx.x / 2, step = gridDim.x / 2;

    if (threadIdx.x == 0) {
        for (int i = 0; i < WD_STAGES; ++i) { mbar_init(&sh.full[i], 1); mbar_init(&sh.empty[i], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&sh.tfull[i], 1); mbar_init(&sh.tempty[i], 2 * WD_EPI); }
        mbar_init(&sh.drain, 1);
        sh.abort = 0;
        fence_barrier_init();
        tma_prefetch_desc(&tmap_w);
        tma_prefetch_desc(&tmap_a);
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem_base)),
                     "r"(512u)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_arrive();                                    // both CTAs' barriers exist before either signals the other
    cluster_wait();
    tc_fence_after();
    const uint32_t tmem = sh.tmem_base;
    volatile int *abort = &sh.abort;
    pdl_trigger();
    pdl_wait();

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(WD_REGS_FEW));
    if (warp == 0) {
        // ------------------------------------------------------- producer
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0, pending = 0, pend_par = 0;
            bool ok = true;
            for (int64_t t = first; t < tiles && ok; t += step) {
                int mt, nt;
                tile_at(t, MT, NT, mt, nt);
                const int row = mt * WD_BM + (int)rank * 128, col = nt * WD_BN + (int)rank * 128;
                for (int kb = 0; kb < KB; ++kb) {
                    if (!mbar_wait(&sh.empty[stage], phase ^ 1, abort)) { ok = false; break; }
                    uint8_t *dst = base + stage * WD_STAGE;
                    const uint32_t bar = cluster_addr(&sh.full[stage], 0);
                    if (rank == 0) mbar_expect_tx(&sh.full[stage], 2 * WD_STAGE);
                    tma_load_pair(dst, &tmap_a, bar, kb * QBLOCK, row);
                    tma_load_pair(dst + WD_HALF, &tmap_w, bar, kb * QBLOCK, col);
                    pending |= 1u << stage;
                    pend_par = (pend_par & ~(1u << stage)) | (phase << stage);
                    if (++stage == WD_STAGES) { stage = 0; phase ^= 1; }
                }
            }
            // no copy of the pair may still be landing when it leaves
            int dummy = 0;
            if (rank == 0)
                for (int st = 0; st < WD_STAGES; ++st)
                    if (pending & (1u << st)) mbar_wait(&sh.full[st], (pend_par >> st) & 1, &dummy, 100000000ull);
        }
    } else if (warp == 1) {
        // ---------------------------------------------------- MMA issuer
        if (lane == 0 && rank == 0) {
            int stage = 0, buf = 0;
            uint32_t phase = 0, tphase = 0;
            bool ok = true;
            for (int64_t t = first; t < tiles && ok; t += step) {
                for (int kb = 0; kb < KB; ++kb) {
                    if (!mbar_wait_cluster(&sh.tempty[buf], tphase ^ 1, abort) || !mbar_wait(&sh.full[stage], phase, abort)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t d = tmem + buf * WD_BN;
                    const uint64_t ad = smem_desc_sw128(smem_u32(base + stage * WD_STAGE));
                    const uint64_t wd = smem_desc_sw128(smem_u32(base + stage * WD_STAGE + WD_HALF));
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk) tc_mma_fp8_pair(d, ad + 2 * kk, wd + 2 * kk, WD_IDESC, kk != 0);
                    tc_commit_pair(&sh.empty[stage]);
                    tc_commit_pair(&sh.tfull[buf]);
                    if (++stage == WD_STAGES) { stage = 0; phase ^= 1; }
                    buf ^= 1;
                    if (buf == 0) tphase ^= 1;
                }
            }
            tc_commit_pair(&sh.drain);
            int dummy = 0;
            mbar_wait(&sh.drain, 0, &dummy, 100000000ull);
        }
    }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(WD_REGS_MANY));
        // ------------------------------------------------------ epilogue
        const int q = warp & 3, half = (warp - 4) / 4;
        const uint32_t taddr = tmem + ((uint32_t)(q * 32) << 16) + half * 128;
        float (*tp)[33] = reinterpret_cast<float (*)[33]>(base + WD_STAGES * WD_STAGE + (warp - 4) * WD_TILE);
        int buf = 0;
        uint32_t tphase = 0;
        bool ok = true;
        for (int64_t t = first; t < tiles && ok; t += step) {
            int mt, nt;
            tile_at(t, MT, NT, mt, nt);
            const int m0 = mt * WD_BM + (int)rank * 128 + q * 32, n0 = nt * WD_BN + half * 128;
            const float *sar = g.sa + (int64_t)min(m0 + lane, g.M - 1) * g.ldsa;
            const float *swr = g.sw + (int64_t)(min(n0, g.N - 1) / QBLOCK) * g.ldsw;
            uint64_t acc[64];
#pragma unroll
            for (int j = 0; j < 64; ++j) acc[j] = 0;
            float f_next = sar[0] * swr[0];
            for (int kb = 0; kb < KB; ++kb) {
                const float f = f_next;
                uint64_t f2;
                asm("mov.b64 %0, {%1, %1};" : "=l"(f2) : "r"(__float_as_uint(f)));
                if (kb + 1 < KB) f_next = sar[kb + 1] * swr[kb + 1];
                if (ok) ok = mbar_wait(&sh.tfull[buf], tphase, abort);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t d[32];
                    tmem_ld32w(taddr + buf * WD_BN + c * 32, d);
                    if (c == 3) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_cluster(cluster_addr(&sh.tempty[buf], 0));
                    }
#pragma unroll
                    for (int j = 0; j < 16; ++j) fma2(acc[c * 16 + j], d[2 * j], d[2 * j + 1], f2);
                }
                buf ^= 1;
                if (buf == 0) tphase ^= 1;
            }
            if (!ok || m0 >= g.M || n0 >= g.N) continue;
            if (vec && n0 + 128 <= g.N) {
                if (m0 + lane < g.M) {
                    if (g.bf16) {
                        uint16_t *p = static_cast<uint16_t *>(g.out) + (int64_t)(m0 + lane) * g.ldo + n0;
#pragma unroll
                        for (int c = 0; c < 8; ++c) {
                            uint32_t w[8];
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                float lo, hi;
                                halves(acc[c * 8 + j], lo, hi);
                                w[j] = pack_bf16(lo, hi);
                            }
                            store32(p + c * 16, w);
                        }
                    } else {
                        float *p = static_cast<float *>(g.out) + (int64_t)(m0 + lane) * g.ldo + n0;
#pragma unroll
                        for (int c = 0; c < 16; ++c) {
                            uint32_t w[8];
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                float lo, hi;
                                halves(acc[c * 4 + j], lo, hi);
                                w[2 * j] = __float_as_uint(lo);
                                w[2 * j + 1] = __float_as_uint(hi);
                            }
                            store32(p + c * 8, w);
                        }
                    }
                }
            } else {
                // rows of out that start anywhere, or a partial tile: transpose
                // 32 columns at a time, so that a warp stores consecutive elements
                const int rows = min(32, g.M - m0);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int n = n0 + c * 32 + lane;
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        float lo, hi;
                        halves(acc[c * 16 + j], lo, hi);
                        tp[lane][2 * j] = lo;
                        tp[lane][2 * j + 1] = hi;
                    }
                    __syncwarp();
                    if (n < g.N)
                        for (int r = 0; r < rows; ++r) {
                            const int64_t at = (int64_t)(m0 + r) * g.ldo + n;
                            if (g.bf16) static_cast<uint16_t *>(g.out)[at] = f2bf(tp[r][lane]);
                            else static_cast<float *>(g.out)[at] = tp[r][lane];
                        }
                    __syncwarp();
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    cluster_arrive();                                    // neither CTA leaves while the other may signal it
    cluster_wait();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
    if (threadIdx.x == 0 && sh.abort) set_status(g.status, ST_TIMEOUT);
}

}  // namespace

int launch_mm_wide(const MmArgs &g, const void *a, int64_t lda, const void *w, int64_t ldw, int sms, cudaStream_t st)
{
    static std::once_flag once;
    static cudaError_t attr;
    std::call_once(once, [] {
        attr = cudaFuncSetAttribute(k_matmul_fp8_wide, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)WD_SMEM);
    });
    if (attr != cudaSuccess) { (void)cudaGetLastError(); return XPRESS_ERR_CUDA; }
    CUtensorMap ta{}, tw{};
    if (!tmap_bytes(&ta, a, (uint64_t)g.K, (uint64_t)g.M, (uint64_t)lda, QBLOCK, 128) ||
        !tmap_bytes(&tw, w, (uint64_t)g.K, (uint64_t)g.N, (uint64_t)ldw, QBLOCK, 128))
        return XPRESS_ERR_CUDA;
    const int64_t tiles = (int64_t)((g.M + WD_BM - 1) / WD_BM) * ((g.N + WD_BN - 1) / WD_BN);
    const int64_t pairs = tiles < sms / 2 ? tiles : sms / 2;
    const int es = g.bf16 ? 2 : 4;
    const int vec = aligned(g.out, 32) && g.ldo * es % 32 == 0;
    XH_CUDA(launch_head(k_matmul_fp8_wide, dim3((unsigned)(2 * pairs)), WD_THREADS, WD_SMEM, st, 2, g, ta, tw, vec));
    return XPRESS_OK;
}

}  // namespace xp
