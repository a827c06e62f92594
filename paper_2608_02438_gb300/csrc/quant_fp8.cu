// quant_fp8.cu -- weights for the block-scaled 8-bit product: every 128 x 128
// block of W gets the scale max(max |W| / 448, 2^-126) and its elements become
// e4m3(W / scale).
//
// One CTA per block, which it holds in registers as it is stored (32 elements
// per thread), so W is read once; the only exchange is the block's largest
// magnitude.  HBM bound: what counts is loads in flight, so registers are kept
// for four CTAs of 512 threads on an SM (two for fp32): 151936 x 4096 bf16 takes
// 274 us, 6.8 TB/s (782 with 256 threads and the elements held as fp32), 32768 x 4096
// fp32 97 us, 6.9 TB/s.
// Threads take 8 consecutive elements (16 lanes span a row of the block) where
// rows start on 16 bytes, else single elements that are consecutive across the
// warp.
#include "head.h"

namespace xp {

namespace {

constexpr int QT = 512;                  // threads: 16 warps
constexpr int QS = QBLOCK * QBLOCK / 8 / QT;     // slots of 8 elements of a thread

template <typename T, bool VEC>
__global__ void __launch_bounds__(QT, sizeof(T) == 2 ? 4 : 2)
    k_quant_weight(const T *W, int64_t ldw, int rows, int cols, uint8_t *q, int64_t ldq, float *scale, int ncb)
{
    __shared__ uint32_t part[QT / 32];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int rb = blockIdx.x / ncb, c0 = blockIdx.x % ncb * QBLOCK;
    pdl_wait();
    // VEC: slot i is row 32 i + thread / 16, columns 8 (thread % 16) + j;
    // else slot i holds rows 32 i + 2 warp + (j / 4), columns 32 (j % 4) + lane
    Raw8<T> raw[QS];
#pragma unroll
    for (int i = 0; i < QS; ++i) {
        if (VEC) {
            const int r = rb * QBLOCK + i * 32 + threadIdx.x / 16, c = c0 + threadIdx.x % 16 * 8;
            raw[i] = load_raw<true>(W + (int64_t)r * ldw + c, r < rows ? cols - c : 0);
        } else {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int r = rb * QBLOCK + i * 32 + 2 * warp + j / 4, c = c0 + (j % 4) * 32 + lane;
                v[j] = r < rows && c < cols ? load1(W + (int64_t)r * ldw + c) : 0.0f;
            }
            pack(v, raw[i]);
        }
    }
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < QS; ++i) m = max(m, amax8(raw[i]));
    m = __reduce_max_sync(0xffffffffu, m);
    if (lane == 0) part[warp] = m;
    __syncthreads();
    m = __reduce_max_sync(0xffffffffu, part[lane % (QT / 32)]);
    const float s = group_scale(m);
    const ScaleDiv div(s);
    if (threadIdx.x == 0) scale[blockIdx.x] = s;
    if (div.small)
#pragma unroll
        for (int i = 0; i < QS; ++i) {
            float v[8];
            unpack(raw[i], v);
            div.raise<8>(v);
            pack(v, raw[i]);                       // exact
        }
#pragma unroll
    for (int i = 0; i < QS; ++i) {
        float v[8];
        unpack(raw[i], v);
        if (VEC) {
            const int r = rb * QBLOCK + i * 32 + threadIdx.x / 16, c = c0 + threadIdx.x % 16 * 8;
            uint8_t *p = q + (int64_t)r * ldq + c;
            if (r < rows && c + 8 <= cols) store8_e4m3(p, v, div);
            else
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (r < rows && c + j < cols) p[j] = to_e4m3(div(v[j]));
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int r = rb * QBLOCK + i * 32 + 2 * warp + j / 4, c = c0 + (j % 4) * 32 + lane;
                if (r < rows && c < cols) q[(int64_t)r * ldq + c] = to_e4m3(div(v[j]));
            }
        }
    }
}

template <typename T>
cudaError_t launch_quant(const void *W, int64_t ldw, int rows, int cols, uint8_t *q, int64_t ldq, float *scale,
                         cudaStream_t st)
{
    const int nrb = (rows + QBLOCK - 1) / QBLOCK, ncb = (cols + QBLOCK - 1) / QBLOCK;
    const bool vec = aligned(W, 16) && ldw * sizeof(T) % 16 == 0 && aligned(q, 8) && ldq % 8 == 0;
    auto *k = vec ? k_quant_weight<T, true> : k_quant_weight<T, false>;
    return launch_head(k, dim3((unsigned)((int64_t)nrb * ncb)), QT, 0, st, 1, static_cast<const T *>(W), ldw, rows, cols,
                       q, ldq, scale, ncb);
}

}  // namespace
}  // namespace xp

using namespace xp;

extern "C" int xpress_quantize_weight(const void *W, int dtype, int rows, int cols, int64_t ldw, void *q, int64_t ldq,
                                      float *scale, void *stream)
{
    if (!W || !q || !scale || rows < 0 || cols < 1 || ldw < cols || ldq < cols) return XPRESS_ERR_INVALID_ARG;
    if (dtype != XPRESS_F32 && dtype != XPRESS_BF16) return XPRESS_ERR_UNSUPPORTED;
    const uintptr_t es = dtype == XPRESS_BF16 ? 2 : 4;
    if (!aligned(W, es) || !aligned(scale, 4)) return XPRESS_ERR_INVALID_ARG;
    if (rows == 0) return XPRESS_OK;
    if (rows > MAX_DIM || cols > MAX_DIM ||
        (int64_t)((rows + QBLOCK - 1) / QBLOCK) * ((cols + QBLOCK - 1) / QBLOCK) > 0x7fffffff)
        return XPRESS_ERR_UNSUPPORTED;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    uint8_t *qb = static_cast<uint8_t *>(q);
    XH_CUDA(dtype == XPRESS_BF16 ? launch_quant<uint16_t>(W, ldw, rows, cols, qb, ldq, scale, st)
                                 : launch_quant<float>(W, ldw, rows, cols, qb, ldq, scale, st));
    return XPRESS_OK;
}
