// matmul_fp8.h -- what the two kernels of the block-scaled 8-bit product share
// (matmul_fp8.cu: few rows of a; matmul_fp8_wide.cu: many).
#pragma once

#include "head.h"
#include "matmul_wait.h"

namespace xp {

struct MmArgs {
    int M, N, K, S;
    const float *sa, *sw;
    int64_t ldsa, ldsw, ldo;
    void *out;
    int bf16;
    int stages;
    uint32_t table_bytes;
    int32_t *status;
};

constexpr size_t MM_SMEM_LIMIT = 227 * 1024;

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// The address at which CTA `rank` of the cluster keeps what this CTA has at p.
__device__ __forceinline__ uint32_t cluster_addr(const void *p, uint32_t rank)
{
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
    return a;
}

// Floats to a shared::cluster address (aligned to their size), counted in bytes
// by the mbarrier `bar` of the same CTA once they are there.
__device__ __forceinline__ void st_async2(uint32_t addr, uint32_t bar, const float *v)
{
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%2, %3}, [%1];" ::"r"(addr), "r"(bar),
                 "f"(v[0]), "f"(v[1])
                 : "memory");
}
__device__ __forceinline__ void st_async4(uint32_t addr, uint32_t bar, const float *v)
{
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%2, %3, %4, %5}, [%1];" ::"r"(addr),
                 "r"(bar), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3])
                 : "memory");
}

// Instruction descriptor, kind::f8f6f4: fp32 sums, e4m3 A and B, both K-major.
constexpr uint32_t idesc_e4m3(int M, int N)
{
    return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// One lane of a converged warp.
__device__ __forceinline__ bool elect_one()
{
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "elect.sync _|p, 0xffffffff;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(r));
    return r != 0;
}

// D[tmem] = A[smem] B[smem]^T over one 128-wide K block, e4m3 operands (K = 32
// per instruction), fp32 sums: the descriptors' low words step by 32 bytes, the
// high word (the layout) is the same for both operands.
__device__ __forceinline__ void tc_mma_fp8_kblock(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t hi,
                                                  uint32_t idesc)
{
    asm volatile(
        "{\n\t.reg .pred f, t;\n\t.reg .b64 a, b;\n\t"
        "setp.ne.b32 f, 0, 0;\n\tsetp.eq.b32 t, 0, 0;\n\t"
        "mov.b64 a, {%1, %9};\n\tmov.b64 b, {%5, %9};\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b, %10, f;\n\t"
        "mov.b64 a, {%2, %9};\n\tmov.b64 b, {%6, %9};\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b, %10, t;\n\t"
        "mov.b64 a, {%3, %9};\n\tmov.b64 b, {%7, %9};\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b, %10, t;\n\t"
        "mov.b64 a, {%4, %9};\n\tmov.b64 b, {%8, %9};\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b, %10, t;}"
        ::"r"(d_tmem), "r"(a_lo), "r"(a_lo + 2), "r"(a_lo + 4), "r"(a_lo + 6), "r"(b_lo), "r"(b_lo + 2), "r"(b_lo + 4),
        "r"(b_lo + 6), "r"(hi), "r"(idesc)
        : "memory");
}

// 16 TMEM columns of this warp's lane quarter.
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float *v)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, "
        "%14, %15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
          "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
        : "r"(taddr)
        : "memory");
}

// out's rows start on 32 bytes
inline bool mm_out_vec(const MmArgs &g) { return aligned(g.out, 32) && g.ldo * (g.bf16 ? 2 : 4) % 32 == 0; }

// many rows of a (matmul_fp8_wide.cu)
int launch_mm_wide(const MmArgs &g, const void *a, int64_t lda, const void *w, int64_t ldw, int sms, cudaStream_t st);

}  // namespace xp
