// head.h -- what the kernels of the 8-bit drafter head share (rmsnorm.cu,
// quant_fp8.cu, matmul_fp8.cu, logits.cu): the 8-bit conversion, 8-wide loads
// and stores, and the host helpers of their entry points.
#pragma once

#include <atomic>

#include "common.cuh"
#include "xpress.h"

namespace xp {

constexpr int MAX_DIM = 1 << 30;         // largest row or column count (index arithmetic in 32 bits)
constexpr int QBLOCK = 128;              // elements along K (and weight rows) that share a scale
constexpr float FP8_MAX = 448.0f;        // largest e4m3 value
constexpr float MIN_SCALE = 1.17549435e-38f;   // 2^-126: the scale of an all-zero group

// The scale of a group whose largest magnitude has the bits `amax_bits`
// (magnitudes compare as unsigned words, and a NaN's word is above every
// other's, so that a NaN in the group shows in its scale).
__device__ __forceinline__ float group_scale(uint32_t amax_bits)
{
    const float s = __uint_as_float(amax_bits) / FP8_MAX;
    return s < MIN_SCALE ? MIN_SCALE : s;
}

// Two values as e4m3 (nearest even, magnitudes above 448 become 448, NaN stays NaN).
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint8_t to_e4m3(float x) { return (uint8_t)to_e4m3x2(x, 0.0f); }

// 8 consecutive elements at p (16-byte aligned) as fp32.
__device__ __forceinline__ void load8(const uint16_t *p, float (&v)[8])
{
    const uint4 a = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load8(const float *p, float (&v)[8])
{
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    return (uint32_t)f2bf(lo) | ((uint32_t)f2bf(hi) << 16);
}
__device__ __forceinline__ void store8(uint16_t *p, const float (&v)[8])
{
    *reinterpret_cast<uint4 *>(p) =
        make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}
__device__ __forceinline__ void store8(float *p, const float (&v)[8])
{
    *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4 *>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store1(uint16_t *p, float v) { *p = f2bf(v); }
__device__ __forceinline__ void store1(float *p, float v) { *p = v; }
__device__ __forceinline__ float load1(const uint16_t *p) { return bf2f(*p); }
__device__ __forceinline__ float load1(const float *p) { return *p; }

// 8 elements as they are stored.
template <typename T> struct Raw8;
template <> struct Raw8<uint16_t> { uint4 a; };
template <> struct Raw8<float> { float4 a, b; };

__device__ __forceinline__ void unpack(const Raw8<uint16_t> &r, float (&v)[8])
{
    const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void unpack(const Raw8<float> &r, float (&v)[8])
{
    v[0] = r.a.x; v[1] = r.a.y; v[2] = r.a.z; v[3] = r.a.w;
    v[4] = r.b.x; v[5] = r.b.y; v[6] = r.b.z; v[7] = r.b.w;
}
// 8 elements from p (`n` of them exist); VEC: p is 16-byte aligned.
template <bool VEC>
__device__ __forceinline__ Raw8<uint16_t> load_raw(const uint16_t *p, int n)
{
    if (VEC && n >= 8) return {*reinterpret_cast<const uint4 *>(p)};
    uint32_t e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = j < n ? p[j] : 0u;
    return {make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16)};
}
template <bool VEC>
__device__ __forceinline__ Raw8<float> load_raw(const float *p, int n)
{
    if (VEC && n >= 8) return {*reinterpret_cast<const float4 *>(p), *reinterpret_cast<const float4 *>(p + 4)};
    float e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = j < n ? p[j] : 0.0f;
    return {make_float4(e[0], e[1], e[2], e[3]), make_float4(e[4], e[5], e[6], e[7])};
}
__device__ __forceinline__ void pack(const float (&v)[8], Raw8<uint16_t> &r)
{
    r.a = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}
__device__ __forceinline__ void pack(const float (&v)[8], Raw8<float> &r)
{
    r.a = make_float4(v[0], v[1], v[2], v[3]);
    r.b = make_float4(v[4], v[5], v[6], v[7]);
}
// The bits of the largest magnitude as fp32 (a NaN's are above all others).
__device__ __forceinline__ uint32_t amax8(const Raw8<uint16_t> &r)
{
    // two bf16 magnitudes per word, compared as 16-bit unsigned integers
    const uint32_t m = __vmaxu2(__vmaxu2(r.a.x & 0x7fff7fffu, r.a.y & 0x7fff7fffu),
                                __vmaxu2(r.a.z & 0x7fff7fffu, r.a.w & 0x7fff7fffu));
    return max(m << 16, m & 0xffff0000u);
}
__device__ __forceinline__ uint32_t amax8(const Raw8<float> &r)
{
    float v[8];
    unpack(r, v);
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(v[j]) & 0x7fffffffu);
    return m;
}

// Division by a group's scale, rounded as x / s is (ties between e4m3 values are
// common: inputs of few bits over a scale made of one of them) at a fraction of a
// division's instructions.  The method is Markstein's (Computation of elementary
// functions on the IBM RISC System/6000 processor, IBM J. Res. Dev. 34, 1990): with
// the correctly rounded inv = 1 / s and q = x inv, the remainder x - q s is exact in
// one FMA and q + (x - q s) inv rounds as the quotient.  An infinite scale takes no
// remainder: finite elements become 0 and infinite ones NaN, as x / s.  Where s is so
// small that the remainder would underflow, x has to come times `up` (raise(); as a
// factor in operator() it costs 5 % of the weights' quantisation).
struct ScaleDiv {
    float inv, s;
    bool small;
    static constexpr float UP = 1.84467441e19f;                     // 2^64
    __device__ __forceinline__ explicit ScaleDiv(float scale) : small(scale < 7.88860905e-31f)   // 2^-100
    {
        s = small ? scale * UP : scale;
        inv = 1.0f / s;
        if (s == INFINITY) s = 0.0f;
    }
    template <int N> __device__ __forceinline__ void raise(float *x) const
    {
        if (__builtin_expect(small, 0))
#pragma unroll
            for (int j = 0; j < N; ++j) x[j] *= UP;
    }
    __device__ __forceinline__ float operator()(float x) const
    {
        const float q = x * inv;
        return fmaf(fmaf(-q, s, x), inv, q);
    }
};

// 8 values over their scale as e4m3 at p (8-byte aligned).
__device__ __forceinline__ void store8_e4m3(uint8_t *p, const float (&v)[8], const ScaleDiv &d)
{
    const uint32_t lo = to_e4m3x2(d(v[0]), d(v[1])) | (to_e4m3x2(d(v[2]), d(v[3])) << 16);
    const uint32_t hi = to_e4m3x2(d(v[4]), d(v[5])) | (to_e4m3x2(d(v[6]), d(v[7])) << 16);
    *reinterpret_cast<uint2 *>(p) = make_uint2(lo, hi);
}

// ------------------------------------------------------------------- host

#define XH_CUDA(call)                                                                                          \
    do {                                                                                                       \
        if ((call) != cudaSuccess) {                                                                           \
            (void)cudaGetLastError();                                                                          \
            return XPRESS_ERR_CUDA;                                                                            \
        }                                                                                                      \
    } while (0)

inline bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Launch with programmatic stream serialization, optionally in clusters: every
// kernel here waits with griddepcontrol.wait before it touches global memory, so
// that its set-up overlaps the end of a predecessor that lets it.  None lets a
// kernel of another call start early: the acceptance's row kernel reads the
// target's logits without waiting (it runs beside the refinement, which does not
// write them), and these calls may have written them.  Starting early would gain
// 0.5 us at most (xpress_matmul_fp8, 1 x 4096 x 4096).
template <typename... KArgs, typename... Args>
cudaError_t launch_head(void (*kernel)(KArgs...), dim3 grid, unsigned block, size_t smem, cudaStream_t st,
                        unsigned cluster, Args... args)
{
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
    if (e != cudaSuccess) (void)cudaGetLastError();
    return e;
}

// SMs of the current device (0 on an error).
int current_sms();

constexpr int MAX_DEVICES = 64;          // that what is known of a device is kept for

// What holds for the current device only, a kernel's attributes above all, set by
// the first call on each device.  A failure is not kept: the next call tries again.
class OncePerDevice {
    std::atomic<bool> done_[MAX_DEVICES] = {};

public:
    template <typename Set> cudaError_t operator()(Set set)
    {
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e == cudaSuccess) {
            if (dev < MAX_DEVICES && done_[dev].load(std::memory_order_acquire)) return cudaSuccess;
            e = set();
        }
        if (e != cudaSuccess) (void)cudaGetLastError();
        else if (dev < MAX_DEVICES) done_[dev].store(true, std::memory_order_release);
        return e;
    }
};
// The kernel's limit of dynamic shared memory on the current device.
template <typename K> cudaError_t allow_smem(OncePerDevice &once, K kernel, size_t bytes)
{
    return once([&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes); });
}

// 2-D byte tensor [rows][inner] with a row pitch of `pitch` bytes, 128-byte
// swizzle, zero fill out of bounds (base 16-byte aligned, pitch a multiple of 16).
bool tmap_bytes(CUtensorMap *m, const void *base, uint64_t inner, uint64_t rows, uint64_t pitch, uint32_t box_inner,
                uint32_t box_rows);
// Byte matrix [rows][128 kblocks] as (128 columns, rows, K blocks): a box of
// 128 x box_rows x box_kblocks lands as the K blocks' tiles of 2-D boxes, back
// to back, with the same 128-byte swizzle.
bool tmap_bytes_kblocks(CUtensorMap *m, const void *base, uint64_t kblocks, uint64_t rows, uint64_t pitch,
                        uint32_t box_rows, uint32_t box_kblocks);

}  // namespace xp
