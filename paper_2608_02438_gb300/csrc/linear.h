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
    int quads;                     // bias, and out's and res's rows, start on 4 elements
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
// (One branch for all N values, 16 or 32: with one for each, and the way through
// unrolled, the epilogue's code was fetched from L2 in every tile, 10 us of it for
// 256 x 256.)
template <bool BF16, int N> __device__ __forceinline__ void lin_act(int act, float *t)
{
    // a few values at a time: the others keep their registers to themselves
    const auto hold = [&](float *h) {
        asm volatile("" : "+f"(h[0]), "+f"(h[1]), "+f"(h[2]), "+f"(h[3]), "+f"(h[4]), "+f"(h[5]), "+f"(h[6]), "+f"(h[7]),
                     "+f"(h[8]), "+f"(h[9]), "+f"(h[10]), "+f"(h[11]), "+f"(h[12]), "+f"(h[13]), "+f"(h[14]), "+f"(h[15]));
    };
    if (act == XPRESS_ACT_SILU) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            t[j] = BF16 ? __fdividef(t[j], 1.0f + __expf(-t[j])) : t[j] / (1.0f + expf(-t[j]));
            if (!BF16 && j % 4 == 3) hold(t + j / 16 * 16);
        }
    } else if (act == XPRESS_ACT_GELU) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            t[j] = 0.5f * t[j] * erfcf(-0.70710678118654752f * t[j]);
            if (j % 2 == 1) hold(t + j / 16 * 16);
        }
    } else if (act == XPRESS_ACT_RELU) {
#pragma unroll
        for (int j = 0; j < N; ++j) t[j] = t[j] < 0.0f ? 0.0f : t[j];        // a NaN stays
    }
}

// Four consecutive columns n .. of a row: what is read of them ahead of time (out's
// type: two or four words; bias: two), and the way through the epilogue.
template <bool BF16> struct Quad {
    uint32_t w[BF16 ? 2 : 4];

    __device__ __forceinline__ float operator[](int j) const
    {
        return BF16 ? __uint_as_float(j % 2 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16) : __uint_as_float(w[BF16 ? 0 : j]);
    }
    // From p; `whole`: 16 (8) bytes at once, else the first `n` of the four.
    __device__ __forceinline__ void load(const void *p, bool whole, int n)
    {
        if (whole) {
            if (BF16) {
                const uint2 x = *static_cast<const uint2 *>(p);
                w[0] = x.x;
                w[1] = x.y;
            } else {
                const uint4 x = *static_cast<const uint4 *>(p);
                w[0] = x.x; w[1] = x.y; w[BF16 ? 0 : 2] = x.z; w[BF16 ? 0 : 3] = x.w;
            }
            return;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (BF16) {
                const uint32_t v = j < n ? static_cast<const uint16_t *>(p)[j] : 0u;
                w[j / 2] = j % 2 ? w[j / 2] | v << 16 : v;
            } else {
                w[BF16 ? 0 : j] = j < n ? static_cast<const uint32_t *>(p)[j] : 0u;
            }
        }
    }
};
template <bool BF16> __device__ __forceinline__ void lin_res4(const LinArgs &g, int m, int n, Quad<BF16> &r)
{
    r.load(static_cast<const uint8_t *>(g.res) + ((int64_t)m * g.ldr + n) * (BF16 ? 2 : 4), g.quads && n + 4 <= g.N, g.N - n);
}
__device__ __forceinline__ void lin_bias4(const LinArgs &g, int n, Quad<true> &b)
{
    b.w[0] = b.w[1] = 0;
    if (g.bias && n < g.N) b.load(g.bias + n, g.quads && n + 4 <= g.N, g.N - n);
}
template <bool BF16>
__device__ __forceinline__ void lin_store4(const LinArgs &g, int m, int n, float (&v)[4], const Quad<BF16> &r)
{
    if (g.res)
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] += r[j];
    const int64_t at = (int64_t)m * g.ldo + n;
    if (g.quads && n + 4 <= g.N) {
        if (BF16) *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(g.out) + at) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
        else *reinterpret_cast<float4 *>(static_cast<float *>(g.out) + at) = make_float4(v[0], v[1], v[2], v[3]);
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (n + j < g.N) {
            if (BF16) static_cast<uint16_t *>(g.out)[at + j] = f2bf(v[j]);
            else static_cast<float *>(g.out)[at + j] = v[j];
        }
}
__device__ __forceinline__ void lin_add4(float (&v)[4], const Quad<true> &b)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] += b[j];
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
