// linear_wide.cu -- the bf16 product with bias, activation and residual (see
// linear.cu for the definition) for many rows of x: bound by the tensor cores.
//
// A pair of CTAs (tcgen05 cta_group::2) takes a tile of 256 rows of x (the MMA's M,
// 128 in each CTA's TMEM) by 256 weight rows (N; each CTA stages half of them, and
// the pair's MMA reads both halves): what a CTA reads from its shared memory for a
// K block feeds twice the products of a single CTA's tile, without which that port
// and not the tensor core would set the pace.  A tile's sums stay in TMEM over all
// of K; two buffers of 256 columns let the next tile's products run under the
// epilogue of the last.
//
// Where tiles are few, S pairs of a cluster split a tile's K.  Each sends every
// pair its sums of that pair's columns (asynchronous stores into the stages' shared
// memory, which the receiver's mbarrier counts), which adds them in rank order, so
// that the result does not depend on timing.
//
// Roles (384 threads): warp 0 TMA producer (two K blocks of 128 rows per copy; both
// CTAs load their own halves, the copies complete on the pair leader's barrier),
// warp 1 TMEM allocator and, in the leader, MMA issuer; warps 4-11 epilogue (lane
// quarter warp % 4, column half (warp - 4) / 4).
#include "linear.h"

namespace xp {

namespace {

constexpr int LW_BM = 256, LW_BN = 256;                 // tile of a pair
constexpr int LW_EPI = 8;
constexpr int LW_THREADS = 32 * (4 + LW_EPI);
constexpr uint32_t LW_HALF = 128 * 128;                 // 16 KB: a K block of 128 rows of an operand
constexpr int LW_SKB = 2;                               // K blocks of a stage
constexpr uint32_t LW_OPND = LW_SKB * LW_HALF;
constexpr uint32_t LW_STAGE = 2 * LW_OPND;              // x's K blocks, then w's
constexpr int LW_STAGES = 3;
constexpr uint32_t LW_IDESC = idesc_bf16(LW_BM, LW_BN);
constexpr size_t LW_TILE = 32 * 33 * 4;                 // a warp's transpose
constexpr size_t LW_SMEM = 1024 + LW_STAGES * LW_STAGE + LW_EPI * LW_TILE;
constexpr int LW_BAND = 16;                             // row tiles that share the weights while they are in L2
// Sums of a split tile: 4 columns of the CTA's 128 rows, then the next 4, four banks on.
constexpr int LW_GROUP4 = 128 * 4 + 4;
static_assert(64 * LW_GROUP4 * 4 <= LW_STAGES * LW_STAGE, "the sums of a split fit the stages");

struct LinBars {
    uint64_t full[LW_STAGES], empty[LW_STAGES];
    uint64_t tfull[2], tempty[2];
    uint64_t drain, joined;
    long long since;
    uint32_t tmem_base;
    int abort;
};

__device__ __forceinline__ void tma_pair_2d(void *dst, const CUtensorMap *map, uint32_t bar, int x, int y)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], "
        "[%4];" ::"r"(smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void tma_pair_3d(void *dst, const CUtensorMap *map, uint32_t bar, int x, int y, int z)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], "
        "[%5];" ::"r"(smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
}

// Arrive on `bar` of the pair's CTAs (mask) once every MMA issued so far by this thread is done.
__device__ __forceinline__ void tc_commit_pair(uint64_t *bar, uint32_t mask)
{
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
        ::"r"(smem_u32(bar)), "h"((uint16_t)mask)
        : "memory");
}

// mm_wait for a barrier that other CTAs of the cluster arrive on.
__device__ __forceinline__ bool wait_cluster(uint64_t *bar, uint32_t parity, volatile int *abort)
{
    long long t0 = 0;
    for (uint32_t it = 1;; ++it) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(smem_u32(bar)), "r"(parity)
            : "memory");
        if (ok) return true;
        if ((it & 63u) == 0) {
            if (*abort) return false;
            const long long t = clock64();
            if (t0 == 0) t0 = t;
            if (t - t0 > MM_WAIT_CYCLES) { *abort = 1; return false; }
        }
    }
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// First row and column of tile t, in the order of bands of LW_BAND row tiles,
// within a band the row tiles of one column tile after another.
__device__ __forceinline__ void tile_at(int64_t t, int MT, int NT, int &row, int &col)
{
    const int64_t band = t / ((int64_t)LW_BAND * NT);
    const int m0 = (int)band * LW_BAND, rows = min(LW_BAND, MT - m0);
    const int64_t in = t - band * LW_BAND * NT;
    row = (m0 + (int)(in % rows)) * LW_BM;
    col = (int)(in / rows) * LW_BN;
}

// 8 consecutive elements of a row in 16-byte accesses.
__device__ __forceinline__ void load_res8(const LinArgs &g, int64_t at, float (&v)[8])
{
    if (g.bf16) load8(static_cast<const uint16_t *>(g.res) + at, v);
    else load8(static_cast<const float *>(g.res) + at, v);
}
__device__ __forceinline__ void store_out8(const LinArgs &g, int64_t at, const float (&v)[8])
{
    if (g.bf16) store8(static_cast<uint16_t *>(g.out) + at, v);
    else store8(static_cast<float *>(g.out) + at, v);
}

// The warp's 32 rows by 32 columns of sums, d of row `lane`, through the epilogue to
// rows m0 .. and columns n0 .. of out.
__device__ __forceinline__ void emit32(const LinArgs &g, int m0, int n0, const float (&d)[32], float (*tp)[33])
{
    const int lane = threadIdx.x % 32, rows = min(32, g.M - m0);
    if (rows <= 0 || n0 >= g.N) return;
    if (g.vec && n0 + 32 <= g.N) {
        if (lane >= rows) return;
#pragma unroll
        for (int c = 0; c < 32; c += 8) {
            float v[8], r[8];
            if (g.res) load_res8(g, (int64_t)(m0 + lane) * g.ldr + n0 + c, r);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = lin_act(g.act, g.bf16, d[c + j] + (g.bias ? bf2f(g.bias[n0 + c + j]) : 0.0f));
                if (g.res) v[j] += r[j];
            }
            store_out8(g, (int64_t)(m0 + lane) * g.ldo + n0 + c, v);
        }
        return;
    }
    // rows that start anywhere, or a partial tile: transposed, so that a warp stores
    // consecutive elements
#pragma unroll
    for (int j = 0; j < 32; ++j) tp[lane][j] = d[j];
    __syncwarp();
    const int n = n0 + lane;
    if (n < g.N) {
        const float b = lin_bias(g, n);
        for (int r = 0; r < rows; ++r) {
            float v = lin_act(g.act, g.bf16, tp[r][lane] + b);
            if (g.res) v += lin_res(g, m0 + r, n);
            lin_store(g, m0 + r, n, v);
        }
    }
    __syncwarp();
}

// grid: pairs of CTAs that take tile after tile (S = 1), or a cluster of S pairs for
// each tile; LW_THREADS threads, LW_SMEM bytes.
template <int S>
__global__ void __launch_bounds__(LW_THREADS, 1)
    k_linear_wide(const __grid_constant__ LinArgs g, const __grid_constant__ CUtensorMap tmap_x,
                  const __grid_constant__ CUtensorMap tmap_w)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t *base = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ LinBars sh;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int crank = (int)cluster_rank(), rank = crank & 1, split = crank >> 1;
    const int KB = (g.K + LK - 1) / LK, KP = (KB + LW_SKB - 1) / LW_SKB;
    const int kb0 = (int)((int64_t)KP * split / S) * LW_SKB, kb1 = min(KB, (int)((int64_t)KP * (split + 1) / S) * LW_SKB);
    const bool whole = g.K % LK == 0;                       // the maps: (64 columns, rows, K blocks), else (K, rows)
    const int MT = (g.M + LW_BM - 1) / LW_BM, NT = (g.N + LW_BN - 1) / LW_BN;
    const int64_t first = blockIdx.x / (2 * S), tiles = S > 1 ? first + 1 : (int64_t)MT * NT, step = S > 1 ? 1 : gridDim.x / 2;
    const uint32_t both = 3u << (crank & ~1);

    if (threadIdx.x == 0) {
        for (int i = 0; i < LW_STAGES; ++i) { mbar_init(&sh.full[i], 1); mbar_init(&sh.empty[i], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&sh.tfull[i], 1); mbar_init(&sh.tempty[i], 2 * LW_EPI); }
        mbar_init(&sh.drain, 1);
        mbar_init(&sh.joined, 1);
        sh.abort = 0;
        sh.since = 0;
        fence_barrier_init();
        tma_prefetch_desc(&tmap_w);
        tma_prefetch_desc(&tmap_x);
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem_base)),
                     "r"(512u)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_arrive();                                    // the CTAs' barriers exist before any signals another
    cluster_wait();
    tc_fence_after();
    const uint32_t tmem = sh.tmem_base;
    volatile int *abort = &sh.abort;
    pdl_wait();

    if (warp == 0) {
        // ------------------------------------------------------- producer
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0, pending = 0, pend_par = 0;
            bool ok = true;
            for (int64_t t = first; t < tiles && ok; t += step) {
                int row, col;
                tile_at(t, MT, NT, row, col);
                row += rank * 128;
                col += rank * 128;
                for (int kb = kb0; kb < kb1; kb += LW_SKB) {
                    if (!wait_cluster(&sh.empty[stage], phase ^ 1, abort)) { ok = false; break; }
                    uint8_t *dx = base + stage * LW_STAGE, *dw = dx + LW_OPND;
                    const uint32_t bar = cluster_addr(&sh.full[stage], crank & ~1);
                    if (whole) {
                        // one copy per operand; a K block past the end reads as zero
                        if (rank == 0) mbar_expect_tx(&sh.full[stage], 2 * LW_STAGE);
                        tma_pair_3d(dx, &tmap_x, bar, 0, row, kb);
                        tma_pair_3d(dw, &tmap_w, bar, 0, col, kb);
                    } else {
                        const int n = min(LW_SKB, kb1 - kb);
                        if (rank == 0) mbar_expect_tx(&sh.full[stage], n * 4 * LW_HALF);
                        for (int i = 0; i < n; ++i) {
                            tma_pair_2d(dx + i * LW_HALF, &tmap_x, bar, (kb + i) * 128, row);
                            tma_pair_2d(dw + i * LW_HALF, &tmap_w, bar, (kb + i) * 128, col);
                        }
                    }
                    pending |= 1u << stage;
                    pend_par = (pend_par & ~(1u << stage)) | (phase << stage);
                    if (++stage == LW_STAGES) { stage = 0; phase ^= 1; }
                }
            }
            // no copy of the pair may still be landing when it leaves
            int dummy = 0;
            if (rank == 0)
                for (int st = 0; st < LW_STAGES; ++st)
                    if (pending & (1u << st)) mm_wait(&sh.full[st], (pend_par >> st) & 1, &dummy, MM_WAIT_CYCLES / 20);
        }
    } else if (warp == 1 && rank == 0) {
        // ---------------------------------------------------- MMA issuer
        // the whole warp runs the loop, so that the descriptors stay in uniform
        // registers, and one elected lane issues
        const uint32_t base_u = __shfl_sync(0xffffffffu, smem_u32(base), 0);
        const uint32_t tmem_u = __shfl_sync(0xffffffffu, tmem, 0);
        const uint32_t lo0 = (uint32_t)smem_desc_sw128(base_u), hi = (uint32_t)(smem_desc_sw128(base_u) >> 32);
        int stage = 0, buf = 0;
        uint32_t phase = 0, tphase = 0;
        bool ok = true;
        for (int64_t t = first; t < tiles && ok; t += step) {
            ok = __all_sync(0xffffffffu, wait_cluster(&sh.tempty[buf], tphase ^ 1, abort));
            for (int kb = kb0; kb < kb1 && ok; kb += LW_SKB) {
                ok = __all_sync(0xffffffffu, wait_cluster(&sh.full[stage], phase, abort));
                if (!ok) break;
                tc_fence_after();
                const uint32_t x_lo = lo0 + stage * (LW_STAGE >> 4), w_lo = x_lo + (LW_OPND >> 4);
                if (elect_one()) {
#pragma unroll
                    for (int i = 0; i < LW_SKB; ++i)
                        if (kb + i < kb1)
                            tc_mma_bf16_kblock<2>(tmem_u + buf * LW_BN, x_lo + i * (LW_HALF >> 4), w_lo + i * (LW_HALF >> 4), hi,
                                                  LW_IDESC, kb + i > kb0);
                    tc_commit_pair(&sh.empty[stage], both);
                    if (kb + LW_SKB >= kb1) tc_commit_pair(&sh.tfull[buf], both);
                }
                __syncwarp();
                if (++stage == LW_STAGES) { stage = 0; phase ^= 1; }
            }
            buf ^= 1;
            if (buf == 0) tphase ^= 1;
        }
        if (elect_one()) tc_commit_pair(&sh.drain, both);
        __syncwarp();
        int dummy = 0;
        mm_wait(&sh.drain, 0, &dummy, MM_WAIT_CYCLES / 20);
        __syncwarp();
    } else if (warp >= 4) {
        // ------------------------------------------------------ epilogue
        const int q = warp & 3, half = (warp - 4) / 4;
        const uint32_t taddr = tmem + ((uint32_t)(q * 32) << 16) + half * 128;
        const uint32_t tempty0 = cluster_addr(&sh.tempty[0], crank & ~1);
        float (*tp)[33] = reinterpret_cast<float (*)[33]>(base + LW_STAGES * LW_STAGE + (warp - 4) * LW_TILE);
        int buf = 0;
        uint32_t tphase = 0;
        bool ok = true;
        for (int64_t t = first; t < tiles; t += step) {
            int row, col;
            tile_at(t, MT, NT, row, col);
            const int m0 = row + rank * 128 + q * 32, n0 = col + half * 128;
            if (ok) ok = wait_cluster(&sh.tfull[buf], tphase, abort);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok && S == 1) break;
            tc_fence_after();
            if (S > 1) { cluster_arrive(); cluster_wait(); }        // no CTA reads its stages any more
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
                float d[32];
                if (ok) tmem_ld32(taddr + buf * LW_BN + c * 32, d);
                else
#pragma unroll
                    for (int j = 0; j < 32; ++j) d[j] = 0.0f;
                if (c == 3 && S == 1) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(tempty0 + buf * 8);
                }
                if (S == 1) {
                    emit32(g, m0, n0 + c * 32, d, tp);
                } else {
                    constexpr int share = LW_BN / S;                 // columns of a pair
                    const int cc = half * 128 + c * 32, dst = cc / share * 2 + rank;
                    const uint32_t there = cluster_addr(base, dst), bar = cluster_addr(&sh.joined, dst);
#pragma unroll
                    for (int j = 0; j < 32; j += 4)
                        st_async4(there + (((split * share + cc % share + j) / 4) * LW_GROUP4 + (q * 32 + lane) * 4) * 4, bar, d + j);
                }
            }
            buf ^= 1;
            if (buf == 0) tphase ^= 1;
        }
        if (S > 1) {
            // the pair's columns, added in rank order: 8 lanes to 32 columns of a row
            constexpr int share = LW_BN / S;
            int row, col;
            tile_at(first, MT, NT, row, col);
            row += rank * 128;
            col += split * share;
            if (threadIdx.x == 128) mbar_expect_tx(&sh.joined, LW_BN * 128 * 4);
            const bool got = __all_sync(0xffffffffu, mm_wait_joined(&sh.joined, abort));
            const float *sums = reinterpret_cast<const float *>(base);
            const int w8 = warp - 4;
            for (int c = 0; c < share && got; c += 32) {
                const int cl = c + lane % 8 * 4, n = col + cl;
                float b[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) b[j] = lin_bias(g, n + j);
#pragma unroll 1
                for (int i = lane / 8; i < 16; i += 4) {
                    const int r = w8 * 16 + i, m = row + r;
                    if (m >= g.M || n >= g.N) continue;
                    const bool quad = g.pairs && n + 4 <= g.N;
                    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f}, x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                    if (g.res) {
                        const int64_t at = (int64_t)m * g.ldr + n;
                        if (quad && g.bf16) {
                            const uint2 p = *reinterpret_cast<const uint2 *>(static_cast<const uint16_t *>(g.res) + at);
                            x[0] = __uint_as_float(p.x << 16); x[1] = __uint_as_float(p.x & 0xffff0000u);
                            x[2] = __uint_as_float(p.y << 16); x[3] = __uint_as_float(p.y & 0xffff0000u);
                        } else if (quad) {
                            const float4 p = *reinterpret_cast<const float4 *>(static_cast<const float *>(g.res) + at);
                            x[0] = p.x; x[1] = p.y; x[2] = p.z; x[3] = p.w;
                        } else {
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                if (n + j < g.N) x[j] = lin_res(g, m, n + j);
                        }
                    }
#pragma unroll
                    for (int k = 0; k < S; ++k) {
                        const float4 p = *reinterpret_cast<const float4 *>(sums + ((k * share + cl) / 4) * LW_GROUP4 + r * 4);
                        v[0] += p.x; v[1] += p.y; v[2] += p.z; v[3] += p.w;
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = lin_act(g.act, g.bf16, v[j] + b[j]) + x[j];
                    const int64_t at = (int64_t)m * g.ldo + n;
                    if (quad && g.bf16)
                        *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(g.out) + at) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
                    else if (quad)
                        *reinterpret_cast<float4 *>(static_cast<float *>(g.out) + at) = make_float4(v[0], v[1], v[2], v[3]);
                    else
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (n + j < g.N) lin_store(g, m, n + j, v[j]);
                }
            }
        }
    }
    if (S > 1 && warp < 4) { __syncwarp(); cluster_arrive(); cluster_wait(); }
    tc_fence_before();
    __syncthreads();
    cluster_arrive();                                    // no CTA leaves while another may signal it
    cluster_wait();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
    if (threadIdx.x == 0 && sh.abort) set_status(g.status, ST_TIMEOUT);
}

template <int S>
int launch(const LinArgs &g, const CUtensorMap &tx, const CUtensorMap &tw, int64_t pairs, cudaStream_t st)
{
    static OncePerDevice once;
    XH_CUDA(allow_smem(once, k_linear_wide<S>, LW_SMEM));
    XH_CUDA(launch_head(k_linear_wide<S>, dim3((unsigned)(2 * pairs)), LW_THREADS, LW_SMEM, st, 2u * S, g, tx, tw));
    return XPRESS_OK;
}

}  // namespace

int launch_lin_wide(const LinArgs &g, const void *x, int64_t ldx, const void *w, int64_t ldw, int sms, cudaStream_t st)
{
    CUtensorMap tx{}, tw{};
    const uint64_t KB = (uint64_t)(g.K / LK);
    const bool ok = g.K % LK == 0 ? tmap_bytes_kblocks(&tx, x, KB, (uint64_t)g.M, (uint64_t)ldx * 2, 128, LW_SKB) &&
                                        tmap_bytes_kblocks(&tw, w, KB, (uint64_t)g.N, (uint64_t)ldw * 2, 128, LW_SKB)
                                  : tmap_bytes(&tx, x, (uint64_t)g.K * 2, (uint64_t)g.M, (uint64_t)ldx * 2, 128, 128) &&
                                        tmap_bytes(&tw, w, (uint64_t)g.K * 2, (uint64_t)g.N, (uint64_t)ldw * 2, 128, 128);
    if (!ok) return XPRESS_ERR_CUDA;
    const int64_t tiles = (int64_t)((g.M + LW_BM - 1) / LW_BM) * ((g.N + LW_BN - 1) / LW_BN);
    return g.S == 4   ? launch<4>(g, tx, tw, tiles * 4, st)
           : g.S == 2 ? launch<2>(g, tx, tw, tiles * 2, st)
                      : launch<1>(g, tx, tw, tiles < sms / 2 ? tiles : sms / 2, st);
}

}  // namespace xp
