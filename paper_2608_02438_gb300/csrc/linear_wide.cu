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
// warp 1 TMEM allocator and, in the leader, MMA issuer, warp 2 passes "accumulators
// read" on to the leader, so that no epilogue warp waits for it; warps 4-11 epilogue:
// lane quarter warp % 4, 128 columns (warp - 4) / 4, 32 (fp32: 16) at a time by way of
// shared memory, so that four lanes store consecutive outputs of a row.  The residual
// is read the same way, a step ahead, and asked into L2 a tile ahead.  (Sixteen such
// warps have 96 registers each and spill; with eight 168.)
//
// 16384 x 16384 x 4096 with SiLU and bias 1117 us at the full clock, without them 1108,
// 1.98 PFLOP/s (a library product 1100), and 1283, 1276 and 1272 one after another for
// half a second, when the power limit takes the clock to 1450 to 1570 MHz; 8192 x 8192 x
// 4096 with residual: tensor pipe 84 % of the cycles, 1.3 times the operands and outputs
// from and to HBM.  Short K is bound by the epilogue: 4096 x 8192 x 64 with residual
// 53 us, 2.5 TB/s.  Smaller ones by the rounds: 2048 x 4096 x 4096 46 to 49 us, 128 tiles
// for 76 pairs.  What it took with four columns to a lane stored from TMEM, without
// shared memory: 1498 us (1250 to 1320 now, under the power limit as then).
#include <type_traits>

#include "linear.h"

namespace xp {

namespace {

constexpr int LW_BM = 256, LW_BN = 256;                 // tile of a pair
constexpr int LW_EPI = 8;
constexpr int LW_COLS = 128;                            // columns of an epilogue warp
constexpr int LW_THREADS = 32 * (4 + LW_EPI);
constexpr uint32_t LW_HALF = 128 * 128;                 // 16 KB: a K block of 128 rows of an operand
constexpr int LW_SKB = 2;                               // K blocks of a stage
constexpr uint32_t LW_OPND = LW_SKB * LW_HALF;
constexpr uint32_t LW_STAGE = 2 * LW_OPND;              // x's K blocks, then w's
constexpr int LW_STAGES = 3;
constexpr uint32_t LW_IDESC = idesc_bf16(LW_BM, LW_BN);
constexpr size_t LW_TILE = 2 * 32 * 16 * 4;             // a warp's transposes
constexpr size_t LW_SMEM = 1024 + LW_STAGES * LW_STAGE + LW_EPI * LW_TILE;
constexpr int LW_BAND = 16;                             // row tiles that share the weights while they are in L2
// Sums of a split tile: 4 columns of the CTA's 128 rows, then the next 4, four banks on.
constexpr int LW_GROUP4 = 128 * 4 + 4;
static_assert(64 * LW_GROUP4 * 4 <= LW_STAGES * LW_STAGE, "the sums of a split fit the stages");

struct LinBars {
    uint64_t full[LW_STAGES], empty[LW_STAGES];
    uint64_t tfull[2], tread[2], tempty[2];    // tread: by this CTA's epilogue; tempty (leader): by both CTAs'
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

// Where a warp's transpose keeps the four columns 4 c .. of a row: so that eight lanes'
// accesses by rows as well as by columns hit different banks.
__device__ __forceinline__ float4 *quad_of(float4 *tp, int row, int c) { return tp + row * 4 + (c ^ (row >> 1 & 3)); }

// grid: pairs of CTAs that take tile after tile (S = 1), or a cluster of S pairs for
// each tile; LW_THREADS threads, LW_SMEM bytes.
template <int S, bool BF16>
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
        for (int i = 0; i < 2; ++i) { mbar_init(&sh.tfull[i], 1); mbar_init(&sh.tread[i], LW_EPI); mbar_init(&sh.tempty[i], 2); }
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
    } else if (warp == 2 && S == 1) {
        // ------------------------------------ accumulators read, to the leader
        // (an arrival on another CTA's barrier waits for the thread's stores: the
        // epilogue's warps would stand still for theirs)
        if (lane == 0) {
            int buf = 0;
            uint32_t tphase = 0;
            for (int64_t t = first; t < tiles; t += step) {
                if (!mm_wait(&sh.tread[buf], tphase, abort)) break;
                tc_fence_after();
                tc_fence_before();
                mbar_arrive_cluster(cluster_addr(&sh.tempty[buf], crank & ~1));
                buf ^= 1;
                if (buf == 0) tphase ^= 1;
            }
        }
        __syncwarp();
    } else if (warp >= 4) {
        // ------------------------------------------------------ epilogue
        const int q = warp & 3, part = (warp - 4) / 4, cl = lane % 4, rl = lane / 4;
        const uint32_t taddr = tmem + ((uint32_t)(q * 32) << 16) + part * LW_COLS;
        float4 *tp = reinterpret_cast<float4 *>(base + LW_STAGES * LW_STAGE + (warp - 4) * LW_TILE);
        // of a split tile: this thread's quads of the pair's columns, 8 lanes to 32 columns of a row
        constexpr int share = LW_BN / S, QPT = share / 4 * 128 / (LW_EPI * 32), JOIN = S == 1 ? 1 : QPT;
        Quad<true> jbias[JOIN];
        Quad<BF16> jres[JOIN];
        auto quad_at = [&](int k, int &r, int &c) {
            const int i = k * LW_EPI * 32 + (int)threadIdx.x - 128;
            c = i % 8 * 4 + i / (8 * 128) * 32;
            r = i / 8 % 128;
        };
        if (S > 1) {
            int row, col;
            tile_at(first, MT, NT, row, col);
#pragma unroll
            for (int k = 0; k < JOIN; ++k) {
                int r, c;
                quad_at(k, r, c);
                const int m = row + rank * 128 + r, n = col + split * share + c;
                lin_bias4(g, n, jbias[k]);
                if (g.res && m < g.M && n < g.N) lin_res4(g, m, n, jres[k]);
            }
        }
        // The residual of this warp's part of a tile on its way to L2, a tile ahead.
        auto to_l2 = [&](int row, int col) {
            const int m = row + rank * 128 + q * 32 + lane;
            if (!g.res || m >= g.M) return;
#pragma unroll
            for (int c = 0; c < LW_COLS; c += BF16 ? 64 : 32) {
                const int n = min(col + part * LW_COLS + c, g.N - 1);
                const uint8_t *p = static_cast<const uint8_t *>(g.res) + ((int64_t)m * g.ldr + n) * (BF16 ? 2 : 4);
                asm volatile("prefetch.global.L2 [%0];" ::"l"(p));
            }
        };
        int buf = 0;
        uint32_t tphase = 0;
        bool ok = true;
        for (int64_t t = first; t < tiles; t += step) {
            int row, col;
            tile_at(t, MT, NT, row, col);
            const int m0 = row + rank * 128 + q * 32, n0 = col + part * LW_COLS;
            if (S == 1) {
                if (t == first) to_l2(row, col);
                if (t + step < tiles) {
                    tile_at(t + step, MT, NT, row, col);
                    to_l2(row, col);
                }
            }
            const auto wait = [&] {
                if (ok) ok = wait_cluster(&sh.tfull[buf], tphase, abort);
                ok = __all_sync(0xffffffffu, ok);
                tc_fence_after();
            };
            if (S == 1) {
                // A tile's part, 32 columns at a time by way of shared memory, what is read for
                // the next ones ahead: rows m0 + rl + 8 i, columns 4 cl .. of each 16.  `whole`:
                // all of it is inside out, by quads, so that nothing needs a check.
                const auto part_of_tile = [&](auto whole) {
                    constexpr bool WHOLE = decltype(whole)::value;
                    constexpr int ES = BF16 ? 2 : 4;
                    const int64_t at = (int64_t)(m0 + rl) * g.ldo + n0 + 4 * cl, rat = (int64_t)(m0 + rl) * g.ldr + n0 + 4 * cl;
                    uint8_t *out = static_cast<uint8_t *>(g.out) + at * ES;
                    const uint8_t *res = static_cast<const uint8_t *>(g.res) + rat * ES;
                    const int64_t ostep = 8 * g.ldo * ES, rstep = 8 * g.ldr * ES;
                    Quad<true> bias[2];
                    Quad<BF16> next[2][4];
                    bias[0].w[0] = bias[0].w[1] = bias[1].w[0] = bias[1].w[1] = 0;
                    const auto fetch = [&](int c, int h) {
                        const int n = n0 + c + 16 * h + 4 * cl;
                        if (WHOLE) {
                            if (g.bias) bias[h].load(g.bias + n, true, 4);
                        } else {
                            lin_bias4(g, n, bias[h]);
                        }
                        if (g.res)
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                if (WHOLE) next[h][i].load(res + i * rstep + (c + 16 * h) * ES, true, 4);
                                else if (n < g.N && m0 + rl + 8 * i < g.M) lin_res4(g, m0 + rl + 8 * i, n, next[h][i]);
                            }
                    };
                    fetch(0, 0);
                    fetch(0, 1);
                    wait();
                    if (!ok) return;
                    constexpr int H = BF16 ? 2 : 1;          // 16 columns each, as many as registers allow
#pragma unroll 1
                    for (int c = 0; c < LW_COLS; c += 32)
#pragma unroll
                        for (int h0 = 0; h0 < 2; h0 += H) {
                            float d[16 * H];
                            if constexpr (H == 2) tmem_ld32(taddr + buf * LW_BN + c, d);
                            else tmem_ld16(taddr + buf * LW_BN + c + 16 * h0, d);
                            if (h0 + H == 2 && c + 32 == LW_COLS) {
                                tc_fence_before();
                                __syncwarp();
                                if (lane == 0) mbar_arrive(&sh.tread[buf]);
                            }
#pragma unroll
                            for (int j = 0; j < 4 * H; ++j)
                                *quad_of(tp + (h0 + j / 4) * 128, lane, j % 4) = make_float4(d[4 * j], d[4 * j + 1], d[4 * j + 2], d[4 * j + 3]);
                            __syncwarp();
                            float v[4 * H][4];
#pragma unroll
                            for (int k = 0; k < 4 * H; ++k) {
                                const float4 p = *quad_of(tp + (h0 + k / 4) * 128, rl + 8 * (k % 4), cl);
                                v[k][0] = p.x; v[k][1] = p.y; v[k][2] = p.z; v[k][3] = p.w;
                                lin_add4(v[k], bias[h0 + k / 4]);
                            }
                            __syncwarp();
                            lin_act<BF16, 16 * H>(g.act, v[0]);
#pragma unroll
                            for (int k = 0; k < 4 * H; ++k) {
                                const int h = h0 + k / 4, i = k % 4, n = n0 + c + 16 * h + 4 * cl;
                                if (!WHOLE) {
                                    if (m0 + rl + 8 * i < g.M && n < g.N) lin_store4(g, m0 + rl + 8 * i, n, v[k], next[h][i]);
                                    continue;
                                }
                                if (g.res)
#pragma unroll
                                    for (int j = 0; j < 4; ++j) v[k][j] += next[h][i][j];
                                uint8_t *p = out + i * ostep + (c + 16 * h) * ES;
                                if (BF16) *reinterpret_cast<uint2 *>(p) = make_uint2(pack_bf16(v[k][0], v[k][1]), pack_bf16(v[k][2], v[k][3]));
                                else *reinterpret_cast<float4 *>(p) = make_float4(v[k][0], v[k][1], v[k][2], v[k][3]);
                            }
                            if (c + 32 < LW_COLS)
#pragma unroll
                                for (int h = h0; h < h0 + H; ++h) fetch(c + 32, h);
                        }
                };
                if (g.quads && m0 + 32 <= g.M && n0 + LW_COLS <= g.N) part_of_tile(std::true_type());
                else part_of_tile(std::false_type());
                if (!ok) break;
            } else {
                wait();
                cluster_arrive();                                    // no CTA reads its stages any more
                cluster_wait();
#pragma unroll 1
                for (int c = 0; c < LW_COLS; c += 16) {
                    float d[16];
                    if (ok) tmem_ld16(taddr + buf * LW_BN + c, d);
                    else
#pragma unroll
                        for (int j = 0; j < 16; ++j) d[j] = 0.0f;
                    const int cc = part * LW_COLS + c, dst = cc / share * 2 + rank;
                    const uint32_t there = cluster_addr(base, dst), bar = cluster_addr(&sh.joined, dst);
#pragma unroll
                    for (int j = 0; j < 16; j += 4)
                        st_async4(there + (((split * share + cc % share + j) / 4) * LW_GROUP4 + (q * 32 + lane) * 4) * 4, bar, d + j);
                }
            }
            buf ^= 1;
            if (buf == 0) tphase ^= 1;
        }
        if (S > 1) {
            // the pair's columns, added in rank order
            int row, col;
            tile_at(first, MT, NT, row, col);
            if (threadIdx.x == 128) mbar_expect_tx(&sh.joined, LW_BN * 128 * 4);
            const bool got = __all_sync(0xffffffffu, mm_wait_joined(&sh.joined, abort));
            const float *sums = reinterpret_cast<const float *>(base);
            // four at a time
            float v[4][4];
#pragma unroll
            for (int k = 0; k < JOIN; ++k) {
                int r, c;
                quad_at(k, r, c);
                float4 a = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    const float4 p = *reinterpret_cast<const float4 *>(sums + ((s * share + c) / 4) * LW_GROUP4 + r * 4);
                    a.x += p.x; a.y += p.y; a.z += p.z; a.w += p.w;
                }
                v[k % 4][0] = a.x; v[k % 4][1] = a.y; v[k % 4][2] = a.z; v[k % 4][3] = a.w;
                lin_add4(v[k % 4], jbias[k]);
                if (k % 4 != 3) continue;
                lin_act<BF16, 16>(g.act, v[0]);
#pragma unroll
                for (int i = k - 3; i <= k; ++i) {
                    quad_at(i, r, c);
                    const int m = row + rank * 128 + r, n = col + split * share + c;
                    if (got && m < g.M && n < g.N) lin_store4(g, m, n, v[i % 4], jres[i]);
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

template <int S, bool BF16>
int launch(const LinArgs &g, const CUtensorMap &tx, const CUtensorMap &tw, int64_t pairs, cudaStream_t st)
{
    static OncePerDevice once;
    XH_CUDA(allow_smem(once, k_linear_wide<S, BF16>, LW_SMEM));
    XH_CUDA(launch_head(k_linear_wide<S, BF16>, dim3((unsigned)(2 * pairs)), LW_THREADS, LW_SMEM, st, 2u * S, g, tx, tw));
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
    const auto go = [&](auto bf16) {
        constexpr bool BF16 = decltype(bf16)::value;
        return g.S == 4   ? launch<4, BF16>(g, tx, tw, tiles * 4, st)
               : g.S == 2 ? launch<2, BF16>(g, tx, tw, tiles * 2, st)
                          : launch<1, BF16>(g, tx, tw, tiles < sms / 2 ? tiles : sms / 2, st);
    };
    return g.bf16 ? go(std::true_type()) : go(std::false_type());
}

}  // namespace xp
