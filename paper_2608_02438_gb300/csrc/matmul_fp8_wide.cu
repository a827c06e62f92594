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
// Where the tiles are fewer than the SMs, the CTAs of a cluster of S split K.
// Every thread of the epilogue sends its sums to its counterparts, each of which
// gets 64 / S columns and adds them in rank order, so that the result does not
// depend on timing.  The sums land where the operands' stages were, so all
// CTAs of the cluster meet once before them.  Each CTA starts with the next one
// in rank: with all of them sending to the same CTA first, joining 4 took 1.5 us
// longer.  From there a warp stores whole rows of its columns, which is also
// how a single tile goes out whose rows start anywhere (700 x 3000 x 256: 9.1 ->
// 7.3 us; rows on 32 bytes leave from the registers, 0.6 us faster than through
// shared memory).  512 x 4096 x 4096: 19.8 us, 14.9 with S = 2; 300 x 600 x 8192:
// 33 us, 11.4 with S = 8.
//
// Roles (640 threads): warp 0 TMA producer; warps 1 and 2 MMA issuers, one for
// each half tile (warp 1 also allocates TMEM): waiting, issuing 4 MMAs and
// committing takes a warp longer than the tensor core takes for them; warp 3
// stages the products of the scales (128 rows by the tile's 2 weight blocks,
// four K blocks at a time) in shared memory; warps 4-19 epilogue (lane quarter
// warp % 4, 64 columns of a half tile) with the 64 sums of a thread in
// registers: the first warpgroup hands registers to the others.
//
// Measured at 2048 x 38912 x 4096: 271 to 279 us, 2.4 PFLOP/s; the MMAs and their
// hand-offs alone take 191 us, with the operands' copies 224, with the TMEM loads
// 210.  No unit is saturated (2048 x 19456 x 4096): the tensor cores work 49 % of
// the cycles, their operands' reads take shared memory's port in as many, the
// other accesses in 25 %, and the warps issue in 54 %; the rest is what copies,
// MMAs and the epilogue (32 packed FMAs and 4 TMEM loads per thread and K block on
// 16 warps) wait for one another.  One issuer warp took 379 us, unpacked FMAs
// 321, a pair of CTAs on a 256 x 256 tile with two TMEM buffers 568 (each K block
// waited for the other CTA's epilogue); sharing copies in clusters of 2 or 4 CTAs
// by multicast gained nothing.
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
// Sums of a CTA's only tile: 4 columns of each of the 512 threads, then the next
// 4, four banks on.
constexpr int WD_GROUP4 = WD_EPI * 32 * 4 + 4;
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
    uint64_t joined[WD_EPI];
    long long since;
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

// 32 bytes to an address that is a multiple of 32 (wide) or of 16.
__device__ __forceinline__ void store32(void *p, const uint32_t (&w)[8], bool wide)
{
    if (!wide) {
        static_cast<uint4 *>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        static_cast<uint4 *>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
        return;
    }
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]),
                 "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
}

__device__ __forceinline__ bool aligned_dev(const void *p, uintptr_t a)
{
    return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0;
}

// Eight columns of the warp's 32 rows, v of row `lane`, to rows m0 .. and columns
// n .. of out through a transpose, so that 8 lanes store consecutive elements.
__device__ __forceinline__ void store_cols8(const MmArgs &g, int m0, int n, const float *v, float (*tp)[WD_TCOLS + 1])
{
    const int lane = threadIdx.x % 32;
    const int rows = min(32, g.M - m0), cl = lane % WD_TCOLS;
#pragma unroll
    for (int j = 0; j < WD_TCOLS; ++j) tp[lane][j] = v[j];
    __syncwarp();
    if (n + cl < g.N)
        for (int r = lane / WD_TCOLS; r < rows; r += 32 / WD_TCOLS) {
            const int64_t at = (int64_t)(m0 + r) * g.ldo + n + cl;
            if (g.bf16) static_cast<uint16_t *>(g.out)[at] = f2bf(tp[r][cl]);
            else static_cast<float *>(g.out)[at] = tp[r][cl];
        }
    __syncwarp();
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

// grid: a cluster of S CTAs for each tile, or with S = 0 any number of CTAs that
// take tile after tile; WD_THREADS threads, WD_SMEM bytes; vec: out's rows start
// on this many bytes (32, 16 or 0: any), pairs: on two elements.
template <int S>
__global__ void __launch_bounds__(WD_THREADS, 1)
    k_matmul_fp8_wide(const __grid_constant__ MmArgs g, const __grid_constant__ CUtensorMap tmap_a,
                      const __grid_constant__ CUtensorMap tmap_w, int vec, int pairs)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t *base = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ WideBars sh;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int KB = (g.K + QBLOCK - 1) / QBLOCK;
    const int MT = (g.M + WD_BM - 1) / WD_BM, NT = (g.N + WD_BN - 1) / WD_BN;
    constexpr int CS = S ? S : 1;
    const int rank = S > 1 ? (int)cluster_rank() : 0;
    const int kb0 = S > 1 ? KB * rank / CS : 0, kb1 = S > 1 ? KB * (rank + 1) / CS : KB;
    const int64_t first = blockIdx.x / CS, tiles = S ? first + 1 : (int64_t)MT * NT, step = S ? 1 : gridDim.x;

    if (threadIdx.x == 0) {
        for (int i = 0; i < WD_STAGES; ++i) { mbar_init(&sh.full[i], 1); mbar_init(&sh.empty[i], 2); }
        for (int i = 0; i < WD_BUFS; ++i) { mbar_init(&sh.tfull[i], 1); mbar_init(&sh.tempty[i], WD_EPI / 2); }
        for (int i = 0; i < 2; ++i) { mbar_init(&sh.sfull[i], 1); mbar_init(&sh.sempty[i], WD_EPI); }
        for (int i = 0; i < 2; ++i) mbar_init(&sh.drain[i], 1);
        for (int i = 0; i < WD_EPI; ++i) mbar_init(&sh.joined[i], 1);
        sh.abort = 0;
        sh.since = 0;
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
                    for (int kb = kb0; kb < kb1; ++kb) {
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
                for (int kb = kb0; kb < kb1; ++kb) {
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
            const bool vec4 = aligned_dev(g.sa + kb0, 16) && g.ldsa % 4 == 0;
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
                for (int kb = kb0; kb < kb1; kb += WD_GROUP) {
                    float a[4][WD_GROUP], b[2][WD_GROUP];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        if (vec4 && kb + WD_GROUP <= kb1) {
                            const float4 x = *reinterpret_cast<const float4 *>(s[r] + kb);
                            a[r][0] = x.x; a[r][1] = x.y; a[r][2] = x.z; a[r][3] = x.w;
                        } else
#pragma unroll
                            for (int i = 0; i < WD_GROUP; ++i) a[r][i] = kb + i < kb1 ? s[r][kb + i] : 0.0f;
                    }
#pragma unroll
                    for (int i = 0; i < WD_GROUP; ++i) {
                        b[0][i] = kb + i < kb1 ? w0[kb + i] : 0.0f;
                        b[1][i] = kb + i < kb1 ? w1[kb + i] : 0.0f;
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
        __syncwarp();
        if (S > 1) { cluster_arrive(); cluster_wait(); }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(WD_REGS_MANY));
        // ------------------------------------------------------ epilogue
        const int q = warp & 3, part = (warp - 4) / 4, half = part / 2;
        const uint32_t taddr = tmem + ((uint32_t)(q * 32) << 16) + part * WD_COLS;
        float (*tp)[WD_TCOLS + 1] = reinterpret_cast<float (*)[WD_TCOLS + 1]>(base + WD_STAGES * WD_STAGE + (warp - 4) * WD_TILE);
        int slot = 0;
        uint32_t par = 0, tphase = 0, sphase = 0;
        bool ok = true;
        int m0 = g.M, n0 = g.N;
        volatile long long *since = S > 1 ? &sh.since : nullptr;    // one limit before the sums go to other CTAs
        float acc[WD_COLS];
        for (int64_t t = first; t < tiles; t += step) {
            int row, col;
            tile_at(t, MT, NT, row, col);
            m0 = row + q * 32;
            n0 = col + part * WD_COLS;
#pragma unroll
            for (int j = 0; j < WD_COLS; ++j) acc[j] = 0.0f;
#pragma unroll 4
            for (int kb = 0; kb < kb1 - kb0; ++kb) {
                const int i = kb % WD_GROUP;
                if (i == 0) ok = mm_wait(&sh.sfull[slot], sphase, abort, MM_WAIT_CYCLES, since);
                ok = __all_sync(0xffffffffu, ok && mm_wait(&sh.tfull[par * 2 + half], tphase, abort, MM_WAIT_CYCLES, since));
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
                if (i == WD_GROUP - 1 || kb == kb1 - kb0 - 1) {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.sempty[slot]);
                    slot ^= 1;
                    if (slot == 0) sphase ^= 1;
                }
            }
            if (!ok || S) break;
            if (m0 >= g.M || n0 >= g.N) continue;
            if (vec && n0 + WD_COLS <= g.N) {
                if (m0 + lane < g.M) {
                    const int64_t at = (int64_t)(m0 + lane) * g.ldo + n0;
                    if (g.bf16) {
#pragma unroll
                        for (int c = 0; c < WD_COLS; c += 16) {
                            uint32_t w[8];
#pragma unroll
                            for (int j = 0; j < 8; ++j) w[j] = pack_bf16(acc[c + 2 * j], acc[c + 2 * j + 1]);
                            store32(static_cast<uint16_t *>(g.out) + at + c, w, vec == 32);
                        }
                    } else {
#pragma unroll
                        for (int c = 0; c < WD_COLS; c += 8) {
                            uint32_t w[8];
#pragma unroll
                            for (int j = 0; j < 8; ++j) w[j] = __float_as_uint(acc[c + j]);
                            store32(static_cast<float *>(g.out) + at + c, w, vec == 32);
                        }
                    }
                }
            } else {
#pragma unroll
                for (int c = 0; c < WD_COLS; c += WD_TCOLS) store_cols8(g, m0, n0 + c, acc + c, tp);
            }
        }
        // the only tile, when the MMAs have read their operands for good (of all CTAs
        // of the cluster); a warp outside out neither sends nor waits
        if (S > 1) { __syncwarp(); cluster_arrive(); cluster_wait(); }
        else if (S == 1) asm volatile("bar.sync 1, %0;" ::"n"(WD_EPI * 32) : "memory");
        if (S && m0 < g.M && n0 < g.N && (S > 1 || ok)) {
            constexpr int share = WD_COLS / CS, LPR = share / 2;     // columns that stay here, lanes of a row
            const int et = threadIdx.x - 128;
            float *sums = reinterpret_cast<float *>(base);
            uint64_t *joined = &sh.joined[warp - 4];
            if (S > 1 && lane == 0) mbar_expect_tx(joined, (WD_COLS - share) * 32 * 4);
#pragma unroll
            for (int r = 0; r < CS; ++r)
                if (r == rank)
#pragma unroll
                    for (int k = 1; k <= CS; ++k) {
                        const int d = (r + k) % CS;
                        const uint32_t there = cluster_addr(sums, d), bar = cluster_addr(joined, d);
#pragma unroll
                        for (int c = 0; c < share; c += 4) {
                            const int at = (r * share + c) / 4 * WD_GROUP4 + et * 4;
                            const float *v = acc + d * share + c;
                            if (k < CS) st_async4(there + at * 4, bar, v);
                            else *reinterpret_cast<float4 *>(sums + at) = make_float4(v[0], v[1], v[2], v[3]);
                        }
                    }
            __syncwarp();
            if (S > 1) ok = __all_sync(0xffffffffu, mm_wait_joined(joined, abort)) && ok;
            const int c = lane % LPR * 2, n = n0 + rank * share + c;
            const float *from = sums + c / 4 * WD_GROUP4 + (et - lane) * 4 + c % 4;
#pragma unroll 2
            for (int i = lane / LPR; i < 32 && ok; i += 32 / LPR) {
                float2 v = make_float2(0.0f, 0.0f);
#pragma unroll
                for (int k = 0; k < S; ++k) {
                    const float2 x = *reinterpret_cast<const float2 *>(from + k * (share / 4) * WD_GROUP4 + i * 4);
                    v.x += x.x;
                    v.y += x.y;
                }
                const int64_t at = (int64_t)(m0 + i) * g.ldo + n;
                if (m0 + i >= g.M || n >= g.N) continue;
                if (pairs && n + 1 < g.N) {
                    if (g.bf16) *reinterpret_cast<uint32_t *>(static_cast<uint16_t *>(g.out) + at) = pack_bf16(v.x, v.y);
                    else *reinterpret_cast<float2 *>(static_cast<float *>(g.out) + at) = v;
                } else if (g.bf16) {
                    static_cast<uint16_t *>(g.out)[at] = f2bf(v.x);
                    if (n + 1 < g.N) static_cast<uint16_t *>(g.out)[at + 1] = f2bf(v.y);
                } else {
                    static_cast<float *>(g.out)[at] = v.x;
                    if (n + 1 < g.N) static_cast<float *>(g.out)[at + 1] = v.y;
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

template <int S>
int launch_wide(const MmArgs &g, const CUtensorMap &ta, const CUtensorMap &tw, int64_t grid, cudaStream_t st)
{
    static OncePerDevice once;
    XH_CUDA(allow_smem(once, k_matmul_fp8_wide<S>, WD_SMEM));
    const int vec = mm_out_vec(g) ? 32 : aligned(g.out, 16) && g.ldo * (g.bf16 ? 2 : 4) % 16 == 0 ? 16 : 0;
    const int pairs = aligned(g.out, g.bf16 ? 4 : 8) && g.ldo % 2 == 0;
    XH_CUDA(launch_head(k_matmul_fp8_wide<S>, dim3((unsigned)grid), WD_THREADS, WD_SMEM, st, S ? S : 1u, g, ta, tw, vec,
                        pairs));
    return XPRESS_OK;
}

}  // namespace

int launch_mm_wide(const MmArgs &g, const void *a, int64_t lda, const void *w, int64_t ldw, int sms, cudaStream_t st)
{
    CUtensorMap ta{}, tw{};
    if (!tmap_bytes(&ta, a, (uint64_t)g.K, (uint64_t)g.M, (uint64_t)lda, QBLOCK, WD_BM) ||
        !tmap_bytes(&tw, w, (uint64_t)g.K, (uint64_t)g.N, (uint64_t)ldw, QBLOCK, WD_BN))
        return XPRESS_ERR_CUDA;
    const int64_t tiles = (int64_t)((g.M + WD_BM - 1) / WD_BM) * ((g.N + WD_BN - 1) / WD_BN);
    return g.S == 1 && tiles <= sms && !mm_out_vec(g) ? launch_wide<1>(g, ta, tw, tiles, st)
         : g.S == 8     ? launch_wide<8>(g, ta, tw, tiles * 8, st)
         : g.S == 4     ? launch_wide<4>(g, ta, tw, tiles * 4, st)
         : g.S == 2     ? launch_wide<2>(g, ta, tw, tiles * 2, st)
                        : launch_wide<0>(g, ta, tw, tiles < sms ? tiles : sms, st);
}

}  // namespace xp
