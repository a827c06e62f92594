// rmsnorm.cu -- the drafter's final norm with the residual's addition and an
// 8-bit output for the block-scaled product (matmul_fp8.cu):
//   t = x + residual                     (32 bits; stored rounded once)
//   y = t / sqrt(mean_i t_i^2 + eps) * w (stored rounded once)
//   scale_g = max(max_{i in g} |y_i| / 448, 2^-126),  q_i = e4m3(y_i / scale_g)
// for groups g of 128 consecutive elements.  The norm is of the 32-bit sum,
// not of its stored rounding, and q is of the 32-bit y: each output is rounded
// once.
//
// One CTA per row.  A thread keeps its share of the row in registers (V slots
// of 8 elements), so x is read once; the only exchange is the sum of squares.
// A warp owns segments of 256 elements: lane l holds 8 consecutive ones (a
// 16-byte load; a group of 128 is half a warp) or, where a row does not start
// on 16 bytes, the elements l, l + 32, ... (loads of consecutive elements
// across the warp; a group is 4 of a lane's elements).  Rows longer than the
// registers hold (V = 0) are read twice, the second time from L2.
#include "head.h"

namespace xp {

namespace {

struct NormArgs {
    const void *x, *residual, *weight;
    void *sum, *y;
    uint8_t *q;
    float *scale;
    int64_t ldx, ldr, lds, ldy, ldq, ldscale;   // row pitches in elements
    int H;
    float eps;
};

constexpr int SEG = 256;                        // elements a warp takes at a time

__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// Element j of this lane in a segment.
template <bool VEC> __device__ __forceinline__ int elem(int lane, int j) { return VEC ? lane * 8 + j : j * 32 + lane; }

// 8 elements of a segment starting at e0 (zero past H).
template <typename T, bool VEC>
__device__ __forceinline__ void load_seg(const T *row, int e0, int H, int lane, float (&v)[8])
{
    if (VEC && e0 + lane * 8 + 8 <= H) { load8(row + e0 + lane * 8, v); return; }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int e = e0 + elem<VEC>(lane, j);
        v[j] = e < H ? load1(row + e) : 0.0f;
    }
}

template <typename T, bool VEC>
__device__ __forceinline__ void store_seg(T *row, int e0, int H, int lane, const float (&v)[8])
{
    if (VEC && e0 + lane * 8 + 8 <= H) { store8(row + e0 + lane * 8, v); return; }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int e = e0 + elem<VEC>(lane, j);
        if (e < H) store1(row + e, v[j]);
    }
}

// q and the scales of a segment (two groups) of y.
template <bool VEC>
__device__ __forceinline__ void quant_seg(uint8_t *qrow, float *srow, int e0, int H, int lane, const float (&y)[8])
{
    if (VEC) {
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = max(m, abs_bits(y[j]));
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
        const float s = group_scale(m);
        const ScaleDiv div(s);
        const int e = e0 + lane * 8;
        if ((lane & 15) == 0 && e < H) srow[e / QBLOCK] = s;
        if (e + 8 <= H) store8_e4m3(qrow + e, y, div);
        else
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (e + j < H) qrow[e + j] = to_e4m3(div(y[j]));
    } else {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            uint32_t m = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) m = max(m, abs_bits(y[4 * g + j]));
            m = __reduce_max_sync(0xffffffffu, m);
            const float s = group_scale(m);
            const ScaleDiv div(s);
            if (lane == 0 && e0 + g * QBLOCK < H) srow[e0 / QBLOCK + g] = s;
#pragma unroll
            for (int j = 4 * g; j < 4 * g + 4; ++j) {
                const int e = e0 + j * 32 + lane;
                if (e < H) qrow[e] = to_e4m3(div(y[j]));
            }
        }
    }
}

// grid: rows; V > 0: 32 ceil(H / 256 / V) threads or more; V = 0: any.
// FEW: the weights are read before the sum of squares is known, which saves
// their latency; else after it (from L1), and registers are kept for 2048
// threads on an SM (16384 x 4096 bf16 with a residual and all outputs: 102 us,
// 5.9 TB/s; 113 with 1536 threads, 163 with the weights held).
template <typename T, bool VEC, int V, int THREADS, bool FEW>
__global__ void __launch_bounds__(THREADS, FEW ? 1 : 2048 / THREADS) k_rmsnorm(const __grid_constant__ NormArgs a)
{
    __shared__ float part[THREADS / 32];
    constexpr int WARPS = THREADS / 32;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, H = a.H;
    const int64_t r = blockIdx.x;
    pdl_wait();
    const T *x = static_cast<const T *>(a.x) + r * a.ldx;
    const T *res = a.residual ? static_cast<const T *>(a.residual) + r * a.ldr : nullptr;
    const T *w = static_cast<const T *>(a.weight);
    T *sum = a.sum ? static_cast<T *>(a.sum) + r * a.lds : nullptr;
    T *y = a.y ? static_cast<T *>(a.y) + r * a.ldy : nullptr;
    uint8_t *q = a.q ? a.q + r * a.ldq : nullptr;
    float *scale = a.q ? a.scale + r * a.ldscale : nullptr;

    auto load_t = [&](int e0, float (&t)[8]) {
        load_seg<T, VEC>(x, e0, H, lane, t);
        if (res) {
            float u[8];
            load_seg<T, VEC>(res, e0, H, lane, u);
#pragma unroll
            for (int j = 0; j < 8; ++j) t[j] += u[j];
        }
    };
    auto finish = [&](int e0, const float (&t)[8], const float (&wv)[8], float inv) {
        float o[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = t[j] * inv * wv[j];
        if (y) store_seg<T, VEC>(y, e0, H, lane, o);
        if (q) quant_seg<VEC>(q, scale, e0, H, lane, o);
    };

    float ss = 0.0f;
    float t[V ? V : 1][8], wv[V && FEW ? V : 1][8];
    if (V) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int e0 = (i * WARPS + warp) * SEG;
            if (e0 < H) load_t(e0, t[i]);
            if (FEW && e0 < H) load_seg<T, VEC>(w, e0, H, lane, wv[i]);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int e0 = (i * WARPS + warp) * SEG;
            if (e0 < H) {
#pragma unroll
                for (int j = 0; j < 8; ++j) ss = fmaf(t[i][j], t[i][j], ss);
                if (sum) store_seg<T, VEC>(sum, e0, H, lane, t[i]);
            }
        }
    } else {
        for (int e0 = warp * SEG; e0 < H; e0 += WARPS * SEG) {
            float s8 = 0.0f;                     // one partial per segment: short sums of many
            load_t(e0, t[0]);
#pragma unroll
            for (int j = 0; j < 8; ++j) s8 = fmaf(t[0][j], t[0][j], s8);
            ss += s8;
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    if (lane == 0) part[warp] = ss;
    __syncthreads();
    ss = lane < WARPS ? part[lane] : 0.0f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    const float inv = 1.0f / sqrtf(ss / (float)H + a.eps);
    if (V) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int e0 = (i * WARPS + warp) * SEG;
            if (e0 >= H) continue;
            if (!FEW) load_seg<T, VEC>(w, e0, H, lane, wv[0]);
            finish(e0, t[i], wv[FEW ? i : 0], inv);
        }
    } else {
        // a row is read by its own CTA alone and a segment by the same warp
        // both times, so sum may be x's or the residual's own memory
        for (int e0 = warp * SEG; e0 < H; e0 += WARPS * SEG) {
            load_t(e0, t[0]);
            if (sum) store_seg<T, VEC>(sum, e0, H, lane, t[0]);
            load_seg<T, VEC>(w, e0, H, lane, wv[0]);
            finish(e0, t[0], wv[0], inv);
        }
    }
}

template <typename T, bool VEC, int V, int THREADS>
cudaError_t launch_norm(const NormArgs &a, int rows, bool few, cudaStream_t st)
{
    auto *k = few ? k_rmsnorm<T, VEC, V, THREADS, true> : k_rmsnorm<T, VEC, V, THREADS, false>;
    return launch_head(k, dim3(rows), THREADS, 0, st, 1, a);
}

template <typename T, bool VEC>
cudaError_t launch_norm_h(const NormArgs &a, int rows, bool few, cudaStream_t st)
{
    const int segs = (a.H + SEG - 1) / SEG;
    if (segs <= 4) return launch_norm<T, VEC, 1, 128>(a, rows, few, st);
    if (segs <= 8) return launch_norm<T, VEC, 1, 256>(a, rows, few, st);
    if (segs <= 16 && !few) return launch_norm<T, VEC, 2, 256>(a, rows, few, st);
    if (segs <= 16) return launch_norm<T, VEC, 1, 512>(a, rows, few, st);
    if (segs <= 32) return launch_norm<T, VEC, 2, 512>(a, rows, few, st);
    if (segs <= 64) return launch_norm<T, VEC, 2, 1024>(a, rows, true, st);
    return launch_norm<T, VEC, 0, 1024>(a, rows, true, st);
}

template <typename T>
cudaError_t launch_norm_t(const NormArgs &a, int rows, cudaStream_t st)
{
    // 16-byte loads need every row of every tensor on 16 bytes (q: 8)
    const int es = sizeof(T);
    auto on16 = [&](const void *p, int64_t ld) { return !p || (aligned(p, 16) && ld * es % 16 == 0); };
    const bool vec = on16(a.x, a.ldx) && on16(a.residual, a.ldr) && on16(a.weight, 0) && on16(a.sum, a.lds) &&
                     on16(a.y, a.ldy) && (!a.q || (aligned(a.q, 8) && a.ldq % 8 == 0));
    const bool few = rows <= current_sms();      // a CTA per SM at most: latency counts
    return vec ? launch_norm_h<T, true>(a, rows, few, st) : launch_norm_h<T, false>(a, rows, few, st);
}

}  // namespace
}  // namespace xp

using namespace xp;

extern "C" int xpress_rmsnorm(const xpress_norm_args *in, void *stream)
{
    if (!in || in->rows < 0 || in->H < 1 || !in->x || !in->weight || (!in->sum && !in->y && !in->q))
        return XPRESS_ERR_INVALID_ARG;
    if ((in->dtype != XPRESS_F32 && in->dtype != XPRESS_BF16) || in->H > MAX_DIM) return XPRESS_ERR_UNSUPPORTED;
    if (in->ldx < in->H || (in->residual && in->ldr < in->H) || (in->sum && in->lds < in->H) ||
        (in->y && in->ldy < in->H) || (in->q && (in->ldq < in->H || !in->scale ||
                                                 in->ldscale < (in->H + QBLOCK - 1) / QBLOCK)) ||
        !(in->eps >= 0.0f))
        return XPRESS_ERR_INVALID_ARG;
    const uintptr_t es = in->dtype == XPRESS_BF16 ? 2 : 4;
    if (!aligned(in->x, es) || !aligned(in->residual, es) || !aligned(in->weight, es) || !aligned(in->sum, es) ||
        !aligned(in->y, es) || !aligned(in->scale, 4))
        return XPRESS_ERR_INVALID_ARG;
    if (in->rows == 0) return XPRESS_OK;
    NormArgs a{in->x, in->residual, in->weight, in->sum, in->y, static_cast<uint8_t *>(in->q), in->scale,
               in->ldx, in->ldr, in->lds, in->ldy, in->ldq, in->ldscale, in->H, in->eps};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    XH_CUDA(in->dtype == XPRESS_BF16 ? launch_norm_t<uint16_t>(a, in->rows, st) : launch_norm_t<float>(a, in->rows, st));
    return XPRESS_OK;
}
