// rmsnorm.cu -- the drafter's final norm with the residual's addition and an
// 8-bit output for the block-scaled product (matmul_fp8.cu):
//   t = x + residual                     (32 bits; stored rounded once)
//   y = t / sqrt(mean_i t_i^2 + eps) * w (stored rounded once)
//   scale_g = max(max_{i in g} |y_i| / 448, 2^-126),  q_i = e4m3(y_i / scale_g)
// for groups g of 128 consecutive elements.  The norm is of the 32-bit sum,
// not of its stored rounding, and q is of the 32-bit y: each output is rounded
// once.  Rows whose squares leave the range of 32 bits are scaled by a power of two
// first, so that any finite row has the norm of the formula.
//
// One CTA per row.  A thread keeps its share of the row in registers (V slots
// of 8 elements), so x is read once; the only exchange is the sum of squares.
// A warp owns segments of 256 elements: lane l holds 8 consecutive ones (a
// 16-byte load; a group of 128 is half a warp) or, where a row does not start
// on 16 bytes, the pairs at 2 l, 2 l + 64, ..., or where it starts on no pair
// either the elements l, l + 32, ... (loads of consecutive elements across the
// warp; a group is 4 of a lane's elements).  11853 x 5202 bf16 with rows on 4
// bytes: 159 us by elements, 112 by pairs.  Rows longer than the registers hold
// (V = 0) are read twice, the second time from L2.
#include <type_traits>

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
constexpr float MIN_MEAN = 7.52316385e-37f;     // 2^-120: what the squares' underflow adds to a mean, 2^-150, is below 2^-29 of it

__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// Element j of this lane in a segment; VEC: its consecutive elements (8, 2 or 1).
template <int VEC> __device__ __forceinline__ int elem(int lane, int j)
{
    return VEC == 8 ? lane * 8 + j : VEC == 2 ? j / 2 * 64 + lane * 2 + j % 2 : j * 32 + lane;
}
// One or two elements, aligned to their number.
template <int N> __device__ __forceinline__ void load_n(const uint16_t *p, float *v)
{
    if (N == 1) { v[0] = bf2f(*p); return; }
    const uint32_t w = *reinterpret_cast<const uint32_t *>(p);
    v[0] = __uint_as_float(w << 16);
    v[1] = __uint_as_float(w & 0xffff0000u);
}
template <int N> __device__ __forceinline__ void load_n(const float *p, float *v)
{
    if (N == 1) { v[0] = *p; return; }
    const float2 w = *reinterpret_cast<const float2 *>(p);
    v[0] = w.x;
    v[1] = w.y;
}
template <int N> __device__ __forceinline__ void store_n(uint16_t *p, const float *v)
{
    if (N == 1) *p = f2bf(v[0]);
    else *reinterpret_cast<uint32_t *>(p) = pack_bf16(v[0], v[1]);
}
template <int N> __device__ __forceinline__ void store_n(float *p, const float *v)
{
    if (N == 1) *p = v[0];
    else *reinterpret_cast<float2 *>(p) = make_float2(v[0], v[1]);
}

// 8 elements of a segment starting at e0 (zero past H).
template <typename T, int VEC>
__device__ __forceinline__ void load_seg(const T *row, int e0, int H, int lane, float (&v)[8])
{
    if (VEC == 8 && e0 + lane * 8 + 8 <= H) { load8(row + e0 + lane * 8, v); return; }
    // (one branch for the whole warp: with one for each piece it would wait for the
    // piece before)
    if (VEC < 8 && e0 + SEG <= H) {
#pragma unroll
        for (int j = 0; j < 8; j += VEC) load_n<VEC>(row + e0 + elem<VEC>(lane, j), v + j);
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int e = e0 + elem<VEC>(lane, j);
        v[j] = e < H ? load1(row + e) : 0.0f;
    }
}

template <typename T, int VEC>
__device__ __forceinline__ void store_seg(T *row, int e0, int H, int lane, const float (&v)[8])
{
    if (VEC == 8 && e0 + lane * 8 + 8 <= H) { store8(row + e0 + lane * 8, v); return; }
    if (VEC < 8 && e0 + SEG <= H) {
#pragma unroll
        for (int j = 0; j < 8; j += VEC) store_n<VEC>(row + e0 + elem<VEC>(lane, j), v + j);
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int e = e0 + elem<VEC>(lane, j);
        if (e < H) store1(row + e, v[j]);
    }
}

// q and the scales of a segment (two groups) of y, which it may scale.
template <int VEC>
__device__ __forceinline__ void quant_seg(uint8_t *qrow, float *srow, int e0, int H, int lane, float (&y)[8])
{
    if (VEC == 8) {
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = max(m, abs_bits(y[j]));
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
        const float s = group_scale(m);
        const ScaleDiv div(s);
        div.raise<8>(y);
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
            div.raise<4>(y + 4 * g);
            if (lane == 0 && e0 + g * QBLOCK < H) srow[e0 / QBLOCK + g] = s;
            if (VEC == 2 && e0 + SEG <= H) {
#pragma unroll
                for (int j = 4 * g; j < 4 * g + 4; j += 2)
                    *reinterpret_cast<uint16_t *>(qrow + e0 + elem<VEC>(lane, j)) = to_e4m3x2(div(y[j]), div(y[j + 1]));
                continue;
            }
#pragma unroll
            for (int j = 4 * g; j < 4 * g + 4; ++j) {
                const int e = e0 + elem<VEC>(lane, j);
                if (e < H) qrow[e] = to_e4m3(div(y[j]));
            }
        }
    }
}

// grid: rows; V > 0: 32 ceil(H / 256 / V) threads or more (of THREADS at most);
// V = 0: any.
// FEW: the weights are read before the sum of squares is known, which saves
// their latency; else after it (from L1), and registers are kept for 2048
// threads on an SM (16384 x 4096 bf16 with a residual and all outputs: 102 us,
// 5.9 TB/s; 113 with 1536 threads, 163 with the weights held, 100 to 110 with CTAs
// that stay and copy 2 to 4 rows ahead into shared memory).
template <typename T, int VEC, int V, int THREADS, bool FEW>
__global__ void __launch_bounds__(THREADS, FEW ? 1 : 2048 / THREADS) k_rmsnorm(const __grid_constant__ NormArgs a)
{
    __shared__ float part[THREADS / 32];
    const int WARPS = blockDim.x / 32;
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
    auto over_block = [&](float v) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if (lane == 0) part[warp] = v;
        __syncthreads();
        v = lane < WARPS ? part[lane] : 0.0f;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        return v;
    };
    float mean = over_block(ss) / (float)H + a.eps, up = 1.0f;
    if (mean == INFINITY || mean < MIN_MEAN) {
        // out of the squares' range (magnitudes above 1.8e19, or so small that eps
        // does not cover what underflows): the row once more, times the power of two
        // `up` that brings its largest magnitude, or the root of eps, to 2^40 (2^30
        // squares still add up, and what underflows there does so in y as well)
        auto all = [&](auto f) {                   // f(t of a segment)
            if (V) {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if ((i * WARPS + warp) * SEG < H) f(t[i]);
            } else {
                for (int e0 = warp * SEG; e0 < H; e0 += WARPS * SEG) {
                    load_t(e0, t[0]);
                    f(t[0]);
                }
            }
        };
        uint32_t m = __float_as_uint(sqrtf(a.eps));
        all([&](float (&v)[8]) {
#pragma unroll
            for (int j = 0; j < 8; ++j) m = max(m, abs_bits(v[j]));
        });
        m = __reduce_max_sync(0xffffffffu, m);
        __syncthreads();                           // all have read part
        if (lane == 0) part[warp] = __uint_as_float(m);
        __syncthreads();
        m = __reduce_max_sync(0xffffffffu, lane < WARPS ? __float_as_uint(part[lane]) : 0u);
        up = __uint_as_float((uint32_t)min(294 - (int)(m >> 23), 253) << 23);
        ss = 0.0f;
        all([&](float (&v)[8]) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] *= up;
                ss = fmaf(v[j], v[j], ss);
            }
        });
        __syncthreads();
        mean = over_block(ss) / (float)H + a.eps * up * up;
    }
    const float inv = 1.0f / sqrtf(mean);
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
#pragma unroll
            for (int j = 0; j < 8; ++j) t[0][j] *= up;
            finish(e0, t[0], wv[0], inv);
        }
    }
}

template <typename T, int VEC, int V, int THREADS, bool FEW>
cudaError_t launch_norm(const NormArgs &a, int rows, cudaStream_t st)
{
    // as many warps as have a segment (12779 x 2301 bf16, 9 segments: 64 us with
    // 8 warps of two slots, 51 with 5)
    const int segs = (a.H + SEG - 1) / SEG;
    return launch_head(k_rmsnorm<T, VEC, V, THREADS, FEW>, dim3(rows), V ? 32 * ((segs + V - 1) / V) : THREADS, 0, st, 1, a);
}

// (few rows hold twice the warps at 4096 elements; rows past the registers have one form)
template <typename T, int VEC, bool FEW>
cudaError_t launch_norm_h(const NormArgs &a, int rows, cudaStream_t st)
{
    constexpr int V16 = FEW ? 1 : 2;
    const int segs = (a.H + SEG - 1) / SEG;
    if (segs <= 4) return launch_norm<T, VEC, 1, 128, FEW>(a, rows, st);
    if (segs <= 8) return launch_norm<T, VEC, 1, 256, FEW>(a, rows, st);
    if (segs <= 16) return launch_norm<T, VEC, V16, 512 / V16, FEW>(a, rows, st);
    if (segs <= 32) return launch_norm<T, VEC, 2, 512, FEW>(a, rows, st);
    if (segs <= 64) return launch_norm<T, VEC, 2, 1024, FEW>(a, rows, st);
    return launch_norm<T, VEC, 0, 1024, true>(a, rows, st);
}

template <typename T>
cudaError_t launch_norm_t(const NormArgs &a, int rows, cudaStream_t st)
{
    // n elements at a time need every row of every tensor on n elements
    const int es = sizeof(T);
    auto on = [&](int bytes, int q_bytes) {
        auto rows_on = [&](const void *p, int64_t ld) { return !p || (aligned(p, bytes) && ld * es % bytes == 0); };
        return rows_on(a.x, a.ldx) && rows_on(a.residual, a.ldr) && rows_on(a.weight, 0) && rows_on(a.sum, a.lds) &&
               rows_on(a.y, a.ldy) && (!a.q || (aligned(a.q, q_bytes) && a.ldq % q_bytes == 0));
    };
    const bool few = rows <= current_sms();      // a CTA per SM at most: latency counts
    auto launch = [&](auto vec) {
        constexpr int VEC = decltype(vec)::value;
        return few ? launch_norm_h<T, VEC, true>(a, rows, st) : launch_norm_h<T, VEC, false>(a, rows, st);
    };
    return on(16, 8)       ? launch(std::integral_constant<int, 8>())
         : on(2 * es, 2) ? launch(std::integral_constant<int, 2>())
                         : launch(std::integral_constant<int, 1>());
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
