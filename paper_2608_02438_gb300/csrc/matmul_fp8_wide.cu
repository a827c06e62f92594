// matmul_fp8_wide.cu -- the block-scaled 8-bit product (see matmul_fp8.cu for
// the definition) for many rows of a: bound by the tensor cores and by what
// feeds them, not by the weights' stream.
//
// A CTA takes a tile of 128 rows of a (the MMA's M) by 256 weight rows (two
// MMAs' N of 128).  One 128-wide K block of a half tile is 4 MMAs into one of
// four TMEM buffers of 128 columns; the epilogue adds the others to the running
// sums with their scales.  With a's rows on the lanes a thread has one scale
// per K block (its row's, times that of the weight block its columns are in).
// The running sums (128 KB) are what limits the tile; four small buffers
// instead of two large ones cover the way from a finished MMA over the epilogue
// back to the MMA that reuses its buffer.
//
// Roles (640 threads): warp 0 TMA producer; warps 1 and 2 MMA issuers, one for
// each half tile (warp 1 also allocates TMEM): waiting, issuing 4 MMAs and
// committing takes a warp longer than the tensor core takes for them; warp 3
// stages the products of the scales (128 rows by the tile's 2 weight blocks,
// four K blocks at a time) in shared memory; warps 4-19 epilogue (lane quarter
// warp % 4, 64 columns of a half tile) with the 64 sums of a thread in
// registers: the first warpgroup hands registers to the others.
//
// Measured at 2048 x 38912 x 4096: 279 us, 2.3 PFLOP/s; the MMAs and their
// hand-offs alone take 191 us, with the operands' copies 224, with the TMEM loads
// 210.  What binds is the epilogue: 64 FMAs (32 packed) and 4 TMEM loads per
// thread and K block on 16 warps.  One issuer warp took 379 us, unpacked FMAs
// 321, a pair of CTAs on a 256 x 256 tile with two TMEM buffers 568 (each K block
// waited for the other CTA's epilogue); sharing copies in clusters of 2 or 4 CTAs
// by multicast gained nothing.
#include <mutex>

#include "matmul_fp8.h"

namespace xp {

namespace {

constexpr int WD_BM = 128, WD_BN = 256;                 // tile of a CTA
constexpr int WD_EPI = 16;
constexpr int WD_COLS = 64;                             // columns of an epilogue warp
constexpr int WD_THREADS = 32 * (4 + WD_EPI);
// registers per thread: the kernel is launched with 96 x 640 (the most that
// five warps of a sub-partition's 16,384 allow); 64 x 128 + 104 x 512 = 61,440
// are all of them
constexpr int WD_REGS_FEW = 64, WD_REGS_MANY = 104;
constexpr uint32_t WD_HALF = 128 * QBLOCK;              // 16 KB: 128 rows of an operand's K block
constexpr uint32_t WD_STAGE = 3 * WD_HALF;              // a, then the two halves of w
constexpr int WD_STAGES = 4;
constexpr uint32_t WD_IDESC = idesc_e4m3(128, 128);
constexpr int WD_BUFS = 4;                              // TMEM buffers: K block parity, half
constexpr int WD_TCOLS = 8;                             // columns of a transpose
constexpr size_t WD_TILE = 32 * (WD_TCOLS + 1) * 4;     // a warp's transpose
constexpr int WD_GROUP = 4;                             // K blocks whose scales are staged together
constexpr size_t WD_SCALES = WD_GROUP * 2 * 128 * 4;    // [K block][weight block][row]
constexpr size_t WD_SMEM = 1024 + WD_STAGES * WD_STAGE + WD_EPI * WD_TILE + 2 * WD_SCALES;
constexpr int WD_BAND = 32;                             // row tiles that share the weights while they are in L2

struct WideBars {
    uint64_t full[WD_STAGES], empty[WD_STAGES];
    uint64_t tfull[WD_BUFS], tempty[WD_BUFS];
    uint64_t sfull[2], sempty[2];
    uint64_t drain[2];
    uint32_t tmem_base;
    int abort;
};

// (x[0], x[1]) += (d[0], d[1]) * f, as one packed FMA.
__device__ __forceinline__ void fma2(float *x, const float *d, float f)
{
    asm("{\n\t.reg .b64 a, b, c;\n\t"
        "mov.b64 a, {%2, %3};\n\t"
        "mov.b64 b, {%4, %4};\n\t"
        "mov.b64 c, {%0, %1};\n\t"
        "fma.rn.f32x2 c, a, b, c;\n\t"
        "mov.b64 {%0, %1}, c;\n\t}"
        : "+f"(x[0]), "+f"(x[1])
        : "f"(d[0]), "f"(d[1]), "f"(f));
}

__device__ __forceinline__ void store32(void *p, const uint32_t (&w)[8])
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]),
                 "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
}

__device__ __forceinline__ bool aligned_dev(const void *p, uintptr_t a)
{
    return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0;
}

// First row and column of tile t, in the order of bands of WD_BAND row tiles,
// within a band the row tiles of one column tile after another.
__device__ __forceinline__ void tile_at(int64_t t, int MT, int NT, int &row, int &col)
{
    const int64_t band = t / ((int64_t)WD_BAND * NT);
    const int m0 = (int)band * WD_BAND, rows = min(WD_BAND, MT - m0);
    const int64_t in = t - band * WD_BAND * NT;
    row = (m0 + (int)(in % rows)) * WD_BM;
    col = (int)(in / rows) * WD_BN;
}

// grid: any; WD_THREADS threads, WD_SMEM bytes; vec: out's rows start on 32 bytes.
__global__ void __launch_bounds__(WD_THREADS, 1)
    k_matmul_fp8_wide(const __grid_constant__ MmArgs g, const __grid_constant__ CUtensorMap tmap_a,
                      const __grid_constant__ CUtensorMap tmap_w, int vec)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t *base = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ WideBars sh;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int KB = (g.K + QBLOCK - 1) / QBLOCK;
    const int MT = (g.M + WD_BM - 1) / WD_BM, NT = (g.N + WD_BN - 1) / WD_BN;
    const int64_t tiles = (int64_t)MT * NT, first = blockIdx.x, step = gridDim.x;

    if (threadIdx.x == 0) {
        for (int i = 0; i < WD_STAGES; ++i) { mbar_init(&sh.full[i], 1); mbar_init(&sh.empty[i], 2); }
        for (int i = 0; i < WD_BUFS; ++i) { mbar_init(&sh.tfull[i], 1); mbar_init(&sh.tempty[i], WD_EPI / 2); }
        for (int i = 0; i < 2; ++i) { mbar_init(&sh.sfull[i], 1); mbar_init(&sh.sempty[i], WD_EPI); }
        for (int i = 0; i < 2; ++i) mbar_init(&sh.drain[i], 1);
        sh.abort = 0;
        fence_barrier_init();
        tma_prefetch_desc(&tmap_w);
        tma_prefetch_desc(&tmap_a);
    }
    if (warp == 1) { tmem_alloc(&sh.tmem_base, WD_BUFS * 128); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem_base;
    volatile int *abort = &sh.abort;
    float *scales = reinterpret_cast<float *>(base + WD_STAGES * WD_STAGE + WD_EPI * WD_TILE);
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
                    int row, col;
                    tile_at(t, MT, NT, row, col);
                    for (int kb = 0; kb < KB; ++kb) {
                        if (!mm_wait(&sh.empty[stage], phase ^ 1, abort)) { ok = false; break; }
                        uint8_t *dst = base + stage * WD_STAGE;
                        mbar_expect_tx(&sh.full[stage], WD_STAGE);
                        tma_load_2d(dst, &tmap_a, &sh.full[stage], kb * QBLOCK, row);
                        tma_load_2d(dst + WD_HALF, &tmap_w, &sh.full[stage], kb * QBLOCK, col);
                        pending |= 1u << stage;
                        pend_par = (pend_par & ~(1u << stage)) | (phase << stage);
                        if (++stage == WD_STAGES) { stage = 0; phase ^= 1; }
                    }
                }
                // no copy may still be landing when the CTA leaves
                int dummy = 0;
                for (int st = 0; st < WD_STAGES; ++st)
                    if (pending & (1u << st)) mm_wait(&sh.full[st], (pend_par >> st) & 1, &dummy, MM_WAIT_CYCLES / 20);
            }
        } else if (warp <= 2) {
            // --------------------------------------------------- MMA issuers
            // the whole warp runs the loop, so that the descriptors stay in uniform
            // registers, and one elected lane issues
            const int h = warp - 1;
            const uint32_t base_u = __shfl_sync(0xffffffffu, smem_u32(base), 0);
            const uint32_t d0 = __shfl_sync(0xffffffffu, tmem + h * 128, 0);
            const uint32_t lo0 = (uint32_t)smem_desc_sw128(base_u), hi = (uint32_t)(smem_desc_sw128(base_u) >> 32);
            const uint32_t w0 = __shfl_sync(0xffffffffu, lo0 + (1 + h) * (WD_HALF >> 4), 0);
            int stage = 0;
            uint32_t phase = 0, par = 0, tphase = 0;               // par: K block parity, which names the TMEM buffer
            bool ok = true;
            for (int64_t t = first; t < tiles && ok; t += step) {
                for (int kb = 0; kb < KB; ++kb) {
                    ok = mm_wait(&sh.full[stage], phase, abort) && mm_wait(&sh.tempty[par * 2 + h], tphase ^ 1, abort);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    tc_fence_after();
                    if (elect_one()) {
                        const uint32_t off = stage * (WD_STAGE >> 4);
                        tc_mma_fp8_kblock(d0 + par * 256, lo0 + off, w0 + off, hi, WD_IDESC);
                        tc_commit(&sh.tfull[par * 2 + h]);
                        tc_commit(&sh.empty[stage]);
                    }
                    __syncwarp();
                    if (++stage == WD_STAGES) { stage = 0; phase ^= 1; }
                    par ^= 1;
                    if (par == 0) tphase ^= 1;
                }
            }
            if (elect_one()) tc_commit(&sh.drain[h]);
            __syncwarp();
            int dummy = 0;
            mm_wait(&sh.drain[h], 0, &dummy, MM_WAIT_CYCLES / 20);
            __syncwarp();
        } else {
            // -------------------------------------------------- scale products
            const bool vec4 = aligned_dev(g.sa, 16) && g.ldsa % 4 == 0;
            int slot = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int64_t t = first; t < tiles && ok; t += step) {
                int row, col;
                tile_at(t, MT, NT, row, col);
                const int wb = col / QBLOCK, wl = (g.N - 1) / QBLOCK;
                const float *w0 = g.sw + (int64_t)min(wb, wl) * g.ldsw, *w1 = g.sw + (int64_t)min(wb + 1, wl) * g.ldsw;
                const float *s[4];                                  // rows lane, lane + 32, ...
#pragma unroll
                for (int r = 0; r < 4; ++r) s[r] = g.sa + (int64_t)min(row + r * 32 + lane, g.M - 1) * g.ldsa;
                for (int kb = 0; kb < KB; kb += WD_GROUP) {
                    float a[4][WD_GROUP], b[2][WD_GROUP];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        if (vec4 && kb + WD_GROUP <= KB) {
                            const float4 x = *reinterpret_cast<const float4 *>(s[r] + kb);
                            a[r][0] = x.x; a[r][1] = x.y; a[r][2] = x.z; a[r][3] = x.w;
                        } else
#pragma unroll
                            for (int i = 0; i < WD_GROUP; ++i) a[r][i] = kb + i < KB ? s[r][kb + i] : 0.0f;
                    }
#pragma unroll
                    for (int i = 0; i < WD_GROUP; ++i) {
                        b[0][i] = kb + i < KB ? w0[kb + i] : 0.0f;
                        b[1][i] = kb + i < KB ? w1[kb + i] : 0.0f;
                    }
                    ok = __all_sync(0xffffffffu, mm_wait(&sh.sempty[slot], phase ^ 1, abort));
                    if (!ok) break;
                    float *f = scales + slot * (WD_SCALES / 4) + lane;
#pragma unroll
                    for (int i = 0; i < WD_GROUP; ++i)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            f[(2 * i) * 128 + r * 32] = a[r][i] * b[0][i];
                            f[(2 * i + 1) * 128 + r * 32] = a[r][i] * b[1][i];
                        }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.sfull[slot]);
                    slot ^= 1;
                    if (slot == 0) phase ^= 1;
                }
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(WD_REGS_MANY));
        // ------------------------------------------------------ epilogue
        const int q = warp & 3, part = (warp - 4) / 4, half = part / 2;
        const uint32_t taddr = tmem + ((uint32_t)(q * 32) << 16) + part * WD_COLS;
        float (*tp)[WD_TCOLS + 1] = reinterpret_cast<float (*)[WD_TCOLS + 1]>(base + WD_STAGES * WD_STAGE + (warp - 4) * WD_TILE);
        int slot = 0;
        uint32_t par = 0, tphase = 0, sphase = 0;
        bool ok = true;
        for (int64_t t = first; t < tiles && ok; t += step) {
            int row, col;
            tile_at(t, MT, NT, row, col);
            const int m0 = row + q * 32, n0 = col + part * WD_COLS;
            float acc[WD_COLS];
#pragma unroll
            for (int j = 0; j < WD_COLS; ++j) acc[j] = 0.0f;
#pragma unroll 4
            for (int kb = 0; kb < KB; ++kb) {
                const int i = kb % WD_GROUP;
                if (i == 0) ok = mm_wait(&sh.sfull[slot], sphase, abort);
                ok = __all_sync(0xffffffffu, ok && mm_wait(&sh.tfull[par * 2 + half], tphase, abort));
                if (!ok) break;
                tc_fence_after();
                const float f = scales[slot * (WD_SCALES / 4) + (2 * i + half) * 128 + q * 32 + lane];
#pragma unroll
                for (int c = 0; c < WD_COLS; c += 16) {
                    float d[16];
                    tmem_ld16(taddr + par * 256 + c, d);
                    if (c + 16 == WD_COLS) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&sh.tempty[par * 2 + half]);
                    }
#pragma unroll
                    for (int j = 0; j < 16; j += 2) fma2(acc + c + j, d + j, f);
                }
                par ^= 1;
                if (par == 0) tphase ^= 1;
                if (i == WD_GROUP - 1 || kb == KB - 1) {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.sempty[slot]);
                    slot ^= 1;
                    if (slot == 0) sphase ^= 1;
                }
            }
            if (!ok || m0 >= g.M || n0 >= g.N) continue;
            if (vec && n0 + WD_COLS <= g.N) {
                if (m0 + lane < g.M) {
                    const int64_t at = (int64_t)(m0 + lane) * g.ldo + n0;
                    if (g.bf16) {
#pragma unroll
                        for (int c = 0; c < WD_COLS; c += 16) {
                            uint32_t w[8];
#pragma unroll
                            for (int j = 0; j < 8; ++j) w[j] = pack_bf16(acc[c + 2 * j], acc[c + 2 * j + 1]);
                            store32(static_cast<uint16_t *>(g.out) + at + c, w);
                        }
                    } else {
#pragma unroll
                        for (int c = 0; c < WD_COLS; c += 8) {
                            uint32_t w[8];
#pragma unroll
                            for (int j = 0; j < 8; ++j) w[j] = __float_as_uint(acc[c + j]);
                            store32(static_cast<float *>(g.out) + at + c, w);
                        }
                    }
                }
            } else {
                // rows of out that start anywhere, or a partial tile: transpose 8
                // columns at a time, so that 8 lanes store consecutive elements
                const int rows = min(32, g.M - m0), cl = lane % WD_TCOLS;
#pragma unroll
                for (int c = 0; c < WD_COLS; c += WD_TCOLS) {
                    const int n = n0 + c + cl;
#pragma unroll
                    for (int j = 0; j < WD_TCOLS; ++j) tp[lane][j] = acc[c + j];
                    __syncwarp();
                    if (n < g.N)
                        for (int r = lane / WD_TCOLS; r < rows; r += 32 / WD_TCOLS) {
                            const int64_t at = (int64_t)(m0 + r) * g.ldo + n;
                            if (g.bf16) static_cast<uint16_t *>(g.out)[at] = f2bf(tp[r][cl]);
                            else static_cast<float *>(g.out)[at] = tp[r][cl];
                        }
                    __syncwarp();
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, WD_BUFS * 128);
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
    if (!tmap_bytes(&ta, a, (uint64_t)g.K, (uint64_t)g.M, (uint64_t)lda, QBLOCK, WD_BM) ||
        !tmap_bytes(&tw, w, (uint64_t)g.K, (uint64_t)g.N, (uint64_t)ldw, QBLOCK, WD_BN))
        return XPRESS_ERR_CUDA;
    const int64_t tiles = (int64_t)((g.M + WD_BM - 1) / WD_BM) * ((g.N + WD_BN - 1) / WD_BN);
    const int es = g.bf16 ? 2 : 4;
    const int vec = aligned(g.out, 32) && g.ldo * es % 32 == 0;
    XH_CUDA(launch_head(k_matmul_fp8_wide, dim3((unsigned)(tiles < sms ? tiles : sms)), WD_THREADS, WD_SMEM, st, 1, g, ta,
                        tw, vec));
    return XPRESS_OK;
}

}  // namespace xp
