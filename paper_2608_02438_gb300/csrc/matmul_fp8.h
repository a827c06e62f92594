// matmul_fp8.h -- what the two kernels of the block-scaled 8-bit product share
// (matmul_fp8.cu: few rows of a; matmul_fp8_wide.cu: many).
#pragma once

#include "head.h"

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

// Instruction descriptor, kind::f8f6f4: fp32 sums, e4m3 A and B, both K-major.
constexpr uint32_t idesc_e4m3(int M, int N)
{
    return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// many rows of a (matmul_fp8_wide.cu)
int launch_mm_wide(const MmArgs &g, const void *a, int64_t lda, const void *w, int64_t ldw, int sms, cudaStream_t st);

}  // namespace xp
