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

// Bounded wait for a phase of `bar` (CLUSTER: the other CTA of a pair arrives
// on it).  It polls (a wait with a sleep hint wakes up later: 2048 x 38912 x
// 4096 took 739 us against 683) and bounds itself by the SM's cycle counter,
// read once in 64 polls: the global timer's latency would sit in every
// hand-off of a K block.
constexpr long long MM_WAIT_CYCLES = 4000000000ll;       // about 2 s
template <bool CLUSTER = false>
__device__ __forceinline__ bool mm_wait(uint64_t *bar, uint32_t parity, volatile int *abort,
                                        long long cycles = MM_WAIT_CYCLES)
{
    long long t0 = 0;
    for (uint32_t it = 1;; ++it) {
        uint32_t ok;
        if (CLUSTER)
            asm volatile(
                "{\n\t.reg .pred p;\n\t"
                "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
                "selp.u32 %0, 1, 0, p;\n\t}"
                : "=r"(ok)
                : "r"(smem_u32(bar)), "r"(parity)
                : "memory");
        else
            ok = mbar_try_wait(bar, parity);
        if (ok) return true;
        if ((it & 63u) == 0) {
            if (*abort) return false;
            const long long t = clock64();
            if (t0 == 0) t0 = t;
            else if (t - t0 > cycles) { *abort = 1; return false; }
        }
    }
}

// Instruction descriptor, kind::f8f6f4: fp32 sums, e4m3 A and B, both K-major.
constexpr uint32_t idesc_e4m3(int M, int N)
{
    return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// many rows of a (matmul_fp8_wide.cu)
int launch_mm_wide(const MmArgs &g, const void *a, int64_t lda, const void *w, int64_t ldw, int sms, cudaStream_t st);

}  // namespace xp
