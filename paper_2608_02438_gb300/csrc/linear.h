// linear.h -- what the two kernels of the bf16 product with bias, activation and
// residual share (linear.cu: few rows of x; linear_wide.cu: many).
#pragma once

#include "head.h"
#include "matmul_fp8.h"

namespace xp {

struct LinArgs {
    int M, N, K, S;                // S: clusters' split of K
    const uint16_t *bias;          // [N] bf16 or NULL
    const void *res;               // [M, N] like out, or NULL
    int64_t ldr;
    void *out;
    int64_t ldo;
    int act;                       // xpress_act
    int bf16;                      // type of out and res
    int vec;                       // out's and res's rows start on 16 bytes
    int pairs;                     // ... on 4 elements
    int stages;
    int32_t *status;
};

constexpr int LK = 64;             // elements of a K block: 128 bytes, a row of the swizzle

// D[tmem] (+)= A[smem] B[smem]^T over one K block of 64, bf16 operands (K = 16 per
// instruction), fp32 sums: the descriptors' low words step by 32 bytes.
template <int GROUP>
__device__ __forceinline__ void tc_mma_bf16_kblock(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc,
                                                   uint32_t accumulate)
{
    if (GROUP == 1)
        asm volatile(
            "{\n\t.reg .pred f, t;\n\t.reg .b64 a, b;\n\t"
            "setp.ne.b32 f, %11, 0;\n\tsetp.eq.b32 t, 0, 0;\n\t"
            "mov.b64 a, {%1, %9};\n\tmov.b64 b, {%5, %9};\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %10, f;\n\t"
            "mov.b64 a, {%2, %9};\n\tmov.b64 b, {%6, %9};\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %10, t;\n\t"
            "mov.b64 a, {%3, %9};\n\tmov.b64 b, {%7, %9};\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %10, t;\n\t"
            "mov.b64 a, {%4, %9};\n\tmov.b64 b, {%8, %9};\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %10, t;}"
            ::"r"(d_tmem), "r"(a_lo), "r"(a_lo + 2), "r"(a_lo + 4), "r"(a_lo + 6), "r"(b_lo), "r"(b_lo + 2), "r"(b_lo + 4),
            "r"(b_lo + 6), "r"(hi), "r"(idesc), "r"(accumulate)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred f, t;\n\t.reg .b64 a, b;\n\t"
            "setp.ne.b32 f, %11, 0;\n\tsetp.eq.b32 t, 0, 0;\n\t"
            "mov.b64 a, {%1, %9};\n\tmov.b64 b, {%5, %9};\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %10, f;\n\t"
            "mov.b64 a, {%2, %9};\n\tmov.b64 b, {%6, %9};\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %10, t;\n\t"
            "mov.b64 a, {%3, %9};\n\tmov.b64 b, {%7, %9};\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %10, t;\n\t"
            "mov.b64 a, {%4, %9};\n\tmov.b64 b, {%8, %9};\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %10, t;}"
            ::"r"(d_tmem), "r"(a_lo), "r"(a_lo + 2), "r"(a_lo + 4), "r"(a_lo + 6), "r"(b_lo), "r"(b_lo + 2), "r"(b_lo + 4),
            "r"(b_lo + 6), "r"(hi), "r"(idesc), "r"(accumulate)
            : "memory");
}

// act(t).  Outputs in bf16 take the fast exponential and division (about 2^-21 off,
// under a tenth of their rounding); the tail of GELU needs erfc, not 1 + erf.
__device__ __forceinline__ float lin_act(int act, bool bf16, float t)
{
    if (act == XPRESS_ACT_SILU) return bf16 ? __fdividef(t, 1.0f + __expf(-t)) : t / (1.0f + expf(-t));
    if (act == XPRESS_ACT_GELU) return 0.5f * t * erfcf(-0.70710678118654752f * t);
    if (act == XPRESS_ACT_RELU) return t < 0.0f ? 0.0f : t;      // a NaN stays
    return t;
}

__device__ __forceinline__ float lin_bias(const LinArgs &g, int n) { return g.bias && n < g.N ? bf2f(g.bias[n]) : 0.0f; }
__device__ __forceinline__ float lin_res(const LinArgs &g, int m, int n)
{
    return ld_any(g.res, g.bf16, (size_t)((int64_t)m * g.ldr + n));
}
__device__ __forceinline__ void lin_store(const LinArgs &g, int m, int n, float v)
{
    const int64_t at = (int64_t)m * g.ldo + n;
    if (g.bf16) static_cast<uint16_t *>(g.out)[at] = f2bf(v);
    else static_cast<float *>(g.out)[at] = v;
}

__device__ __forceinline__ void tma_load_3d(void *dst, const CUtensorMap *map, uint64_t *bar, int x, int y, int z)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
        : "memory");
}

// many rows of x (linear_wide.cu)
int launch_lin_wide(const LinArgs &g, const void *x, int64_t ldx, const void *w, int64_t ldw, int sms, cudaStream_t st);

}  // namespace xp
