// sample.cu -- draws tokens from logits rows under a request's temperature, top-k,
// top-p and min-p, from given random numbers, and truncates rows for the acceptance.
// For a row l at temperature T > 0, with its maximum m:
//   w_v = exp((l_v - m) / T), the order: l falling, equal ones by id
//   kept by min-p and top-k: w_v >= min_p and one of the first k
//   kept by top-p: what stands before v in the order has less than top_p of the
//     mass of those (the first one is always kept)
//   token: the first id v at which the kept mass up to v exceeds u times all of it
// T <= 0 keeps the first maximum alone.  All filters keep a prefix of the order, so
// what is kept is a threshold t, with q of the elements equal to t (the first ones).
//
// A cluster of C CTAs takes a row.  The row is read once, into the CTAs' shared
// memory; every further pass over it stays there.  A thread owns consecutive
// 16-byte pieces, an odd number of them: the lanes' accesses then hit different
// banks, and sums per thread, warp and CTA are in the order of the ids.
//   maximum    with the load; with it the smallest of the maxima of as many groups
//              of lanes as k needs, a bound below the k-th largest
//   thresholds by histograms of the order-preserving bits between a lower bound and
//              the maximum, 2048 bins: one level where these are bf16 values of two
//              or three octaves, up to three levels for fp32
//   draw       sums per warp, exchanged through the cluster; the warp whose range
//              contains u Z looks for the element
//
// Every decision compares masses.  They are 64-bit fixed-point sums, so that no
// order of additions matters, of weights to 2^-31 (weight_exact).  Those take about
// 40 instructions, so passes over a whole row first use the hardware's exponential;
// where a decision falls within what that may be off, it is taken again with the
// exact weights.
#include "matmul_fp8.h"

namespace xp {

namespace {

// 2^(j / 64) as 33-bit integers, from the exponential's series.
struct ExpTable {
    uint64_t v[64];
};
constexpr ExpTable make_exp_table()
{
    ExpTable t{};
    for (int j = 0; j < 64; ++j) {
        const double x = j * 0.693147180559945309417232 / 64;
        double term = 1.0, sum = 1.0;
        for (int i = 1; i < 24; ++i) { term *= x / i; sum += term; }
        t.v[j] = (uint64_t)(sum * 4294967296.0 + 0.5);
    }
    return t;
}
struct SampleArgs {
    const void *in;
    void *out;
    int64_t ld, ldo;
    int rows, V;                   // rows of a sequence
    const float *T, *top_p, *min_p, *u;
    const int32_t *top_k;
    int32_t *tokens;
    float mask_value;
    int per;                       // pieces of a thread (odd)
    int scale;                     // a weight of 1 is 2^scale
    float slack;                   // what a sum of fast weights may be off, relative
    ExpTable table;
};

constexpr int ST = 512, SWARPS = ST / 32;
constexpr int BINS = 2048;
constexpr int MAX_CLUSTER = 8;
constexpr int ALL = 0x7fffffff;
constexpr size_t HIST_BYTES = BINS * 12;         // counts, then masses (64 bits)
constexpr size_t SAMPLE_SMEM = 219 * 1024, SAMPLE_HALF = 107 * 1024;      // pieces and histogram of one, of two CTAs on an SM

template <typename T> struct Piece;
template <> struct Piece<uint16_t> {
    static constexpr int E = 8, KEY_SHIFT = 16;
    static __device__ __forceinline__ void unpack(const uint4 &r, float (&v)[8])
    {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ uint32_t no_nan2(uint32_t w)
    {
        const __nv_bfloat162 low = __floats2bfloat162_rn(-INFINITY, -INFINITY);
        const __nv_bfloat162 r = __hmax2(*reinterpret_cast<const __nv_bfloat162 *>(&w), low);
        return *reinterpret_cast<const uint32_t *>(&r);
    }
    // NaNs become -inf.
    static __device__ __forceinline__ uint4 no_nan(const uint4 &r)
    {
        return make_uint4(no_nan2(r.x), no_nan2(r.y), no_nan2(r.z), no_nan2(r.w));
    }
    static __device__ __forceinline__ float max_of(const uint4 &r)
    {
        const __nv_bfloat162 *p = reinterpret_cast<const __nv_bfloat162 *>(&r);
        const __nv_bfloat162 m = __hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3]));
        return fmaxf(__low2float(m), __high2float(m));
    }
    static __device__ __forceinline__ uint4 pack_raw(const uint16_t (&e)[8])
    {
        return make_uint4(e[0] | (uint32_t)e[1] << 16, e[2] | (uint32_t)e[3] << 16, e[4] | (uint32_t)e[5] << 16,
                          e[6] | (uint32_t)e[7] << 16);
    }
    static constexpr uint16_t NEG_INF = 0xff80;
    static __device__ __forceinline__ uint16_t raw(float v) { return f2bf(v); }
    static __device__ __forceinline__ float value(uint32_t key)      // of a key
    {
        return __uint_as_float((key & 0x8000u ? key & 0x7fffu : ~key & 0xffffu) << 16);
    }
};
template <> struct Piece<float> {
    static constexpr int E = 4, KEY_SHIFT = 0;
    static __device__ __forceinline__ void unpack(const uint4 &r, float (&v)[4])
    {
        v[0] = __uint_as_float(r.x); v[1] = __uint_as_float(r.y);
        v[2] = __uint_as_float(r.z); v[3] = __uint_as_float(r.w);
    }
    static __device__ __forceinline__ uint32_t no_nan1(uint32_t w) { return __float_as_uint(fmaxf(__uint_as_float(w), -INFINITY)); }
    static __device__ __forceinline__ uint4 no_nan(const uint4 &r)
    {
        return make_uint4(no_nan1(r.x), no_nan1(r.y), no_nan1(r.z), no_nan1(r.w));
    }
    static __device__ __forceinline__ float max_of(const uint4 &r)
    {
        float v[4];
        unpack(r, v);
        return fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3]));
    }
    static __device__ __forceinline__ uint4 pack_raw(const float (&e)[4])
    {
        return make_uint4(__float_as_uint(e[0]), __float_as_uint(e[1]), __float_as_uint(e[2]), __float_as_uint(e[3]));
    }
    static constexpr float NEG_INF = -INFINITY;
    static __device__ __forceinline__ float raw(float v) { return v; }
    static __device__ __forceinline__ float value(uint32_t key)
    {
        return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
    }
};

// The order-preserving word of a value, -0 as 0.
__device__ __forceinline__ uint32_t order_of(float v)
{
    const uint32_t b = __float_as_uint(v + 0.0f);
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
constexpr uint32_t LOWEST = 0x00800000u;         // of the lowest finite value

// A row's temperature: K = log2(e) / T in two parts.
struct Scale {
    float m, kh, kl;
    int bits;                                    // a weight of 1 is 2^bits
};

// w = 2^(K (l - m)) as a 64-bit fixed-point number, to 2^-31 of its value (and half a
// unit).  The difference and its product with K are kept in two parts; of the
// exponent, the steps of 1/64 come from a table, the rest g (|g| <= 1/128) from the
// series of 2^g - 1, whose fifth term is below 2^-42.
__device__ __forceinline__ unsigned long long weight_exact(float l, const Scale &s, const unsigned long long *table)
{
    if (l == s.m) return 1ull << s.bits;
    const float dh = __fsub_rn(l, s.m), bb = __fsub_rn(dh, l);
    const float dl = __fadd_rn(__fsub_rn(l, __fsub_rn(dh, bb)), __fsub_rn(-s.m, bb));
    const float ph = __fmul_rn(dh, s.kh);
    if (!(ph > -63.0f)) return 0;
    const float pl = fmaf(dh, s.kh, -ph) + fmaf(dh, s.kl, dl * s.kh);
    const float steps = rintf(ph * 64.0f);
    const float g = fmaf(steps, -0.015625f, ph) + pl;
    const float e = g * fmaf(g, fmaf(g, fmaf(g, 9.61812910e-3f, 5.55041087e-2f), 2.40226507e-1f), 6.93147181e-1f);
    const int i = (int)steps, down = -(i >> 6);
    const unsigned long long t = table[i & 63];
    const unsigned long long w = t + (unsigned long long)(((long long)t * __float2int_rn(e * 4294967296.0f)) >> 32);
    // w has 32 bits behind the point
    const int up = s.bits - 32 - down;
    return up >= 0 ? w << up : up > -34 ? (w + (1ull << (-up - 1))) >> -up : 0;
}
// The same with the hardware's exponential: 2^-22 off, and 2^-24 of the exponent
// from each of three roundings (the difference, K, the product).
__device__ __forceinline__ float weight_fast(float l, const Scale &s) { return ex2_approx(fminf(l - s.m, 0.0f) * s.kh); }

__device__ __forceinline__ unsigned long long warp_sum(unsigned long long v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
template <typename U> __device__ __forceinline__ U warp_scan(U v)      // inclusive
{
    const int lane = threadIdx.x % 32;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const U x = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += x;
    }
    return v;
}

__device__ __forceinline__ void st_cluster(uint32_t addr, unsigned long long v)
{
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(v) : "memory");
}
__device__ __forceinline__ uint4 ld_cluster4(uint32_t addr)
{
    uint4 v;
    asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void ld_cluster2(uint32_t addr, unsigned long long &a, unsigned long long &b)
{
    asm volatile("ld.shared::cluster.v2.u64 {%0, %1}, [%2];" : "=l"(a), "=l"(b) : "r"(addr) : "memory");
}
__device__ __forceinline__ void cluster_sync() { cluster_arrive(); cluster_wait(); }

struct SampleShared {
    unsigned long long table[64];                                    // 2^(j / 64)
    unsigned long long slot[2][2][MAX_CLUSTER * SWARPS];             // what the cluster's warps exchange: [turn][value][warp]
    unsigned long long scan[2][SWARPS];
    unsigned long long note[4];                                      // written by one thread of the cluster: the id cut, a draw to repeat
    double k, shift;                                                 // log2(e) / T and T ln(min_p)
    unsigned long long before, mass;                                 // of the bin that was looked for
    uint32_t bin, count, above;
};

// What a kernel's passes share.
template <typename T, bool RES>
struct Sampler {
    using P = Piece<T>;
    static constexpr int E = P::E;
    const SampleArgs &a;
    SampleShared &sh;
    uint4 *pieces;                 // [per * ST] of this CTA (RES)
    uint32_t *cnt;                 // [BINS]
    unsigned long long *mass;      // [BINS]
    const T *row;                  // the row's first element
    int shift;                     // elements from a 16-byte boundary to it
    int C, rank, turn;
    Scale s;

    __device__ __forceinline__ int64_t position(int p) const { return ((int64_t)rank * a.per * ST + p) * E; }
    __device__ uint4 fetch(int p) const                              // piece p of this CTA from the row, NaNs and what is outside as -inf
    {
        const int64_t at = position(p) - shift;
        if (at >= 0 && at + E <= a.V) return P::no_nan(*reinterpret_cast<const uint4 *>(row + at));
        T e[E];
#pragma unroll
        for (int j = 0; j < E; ++j) e[j] = at + j >= 0 && at + j < a.V ? row[at + j] : P::NEG_INF;
        return P::no_nan(P::pack_raw(e));
    }
    __device__ __forceinline__ uint4 piece(int p) const
    {
        if (RES) return pieces[p];
        return fetch(p);
    }
    // Every warp's two values to all CTAs of the cluster.
    __device__ void exchange(unsigned long long v0, unsigned long long v1)
    {
        const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
        turn ^= 1;
        if (lane < C) {
            const uint32_t to = cluster_addr(&sh.slot[turn][0][rank * SWARPS + warp], lane);
            st_cluster(to, v0);
            st_cluster(to + sizeof(sh.slot[0][0]), v1);
        }
        cluster_sync();
    }
    __device__ unsigned long long slot_of(int which, int i) const { return i < C * SWARPS ? sh.slot[turn][which][i] : 0; }
    // The sum of what the warps exchanged.
    __device__ unsigned long long exchanged_sum(int which) const
    {
        unsigned long long v = 0;
#pragma unroll
        for (int i = 0; i < MAX_CLUSTER * SWARPS / 32; ++i) v += slot_of(which, threadIdx.x % 32 + 32 * i);
        return warp_sum(v);
    }
    // Exclusive sum over the CTA's threads; total of all.
    __device__ unsigned long long block_scan(unsigned long long v, int which, unsigned long long &total)
    {
        const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
        const unsigned long long in = warp_scan(v);
        if (lane == 31) sh.scan[which][warp] = in;
        __syncthreads();
        const unsigned long long w = warp_scan(lane < SWARPS ? sh.scan[which][lane] : 0ull);
        total = __shfl_sync(0xffffffffu, w, SWARPS - 1);
        const unsigned long long base = __shfl_sync(0xffffffffu, w, (warp + 31) % 32);
        return (warp ? base : 0) + in - v;
    }

    // Sum of the weights of l > t and number of l == t in `count` pieces from p of this CTA.
    template <bool EXACT>
    __device__ void sums(int p, int count, float t, unsigned long long &sum, uint32_t &ties) const
    {
        unsigned long long fixed = 0;
        float hi = 0.0f, lo = 0.0f;
        ties = 0;
        for (int i = 0; i < count; ++i) {
            const uint4 r = piece(p + i);
            if (EXACT && P::max_of(r) < t) continue;
            float v[E];
            P::unpack(r, v);
            if (EXACT) {
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    if (v[j] > t) fixed += weight_exact(v[j], s, sh.table);
                    ties += v[j] == t;
                }
            } else {
                float w[E];
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    w[j] = weight_fast(v[j], s);
                    if (!(v[j] > t)) w[j] = 0.0f;
                    ties += v[j] == t;
                }
#pragma unroll
                for (int o = E / 2; o > 0; o >>= 1)
#pragma unroll
                    for (int j = 0; j < o; ++j) w[j] += w[j + o];
                // hi + lo keeps what the addition rounds away
                const float n = __fadd_rn(hi, w[0]), b = __fsub_rn(n, hi);
                lo += __fadd_rn(__fsub_rn(hi, __fsub_rn(n, b)), __fsub_rn(w[0], b));
                hi = n;
            }
        }
        const float one = __uint_as_float((uint32_t)(127 + s.bits) << 23);
        sum = EXACT ? fixed : __float2ull_rn(hi * one) + (unsigned long long)__float2ll_rn(lo * one);
    }

    // Counts (and masses) of the elements from lo up whose keys are at most khi, by
    // bins of 2^bits keys from the largest down; each thread gets four of the bins,
    // summed over the cluster.
    template <bool MASS>
    __device__ void histogram(float lo, uint32_t khi, int bits, uint32_t (&c)[4], unsigned long long (&w)[4])
    {
        const int tid = threadIdx.x;
        reinterpret_cast<uint4 *>(cnt)[tid] = make_uint4(0, 0, 0, 0);
        if (MASS) {
            reinterpret_cast<uint4 *>(mass)[tid] = make_uint4(0, 0, 0, 0);
            reinterpret_cast<uint4 *>(mass)[tid + ST] = make_uint4(0, 0, 0, 0);
        }
        __syncthreads();
        for (int i = 0; i < a.per; ++i) {
            const uint4 r = piece(tid * a.per + i);
            if (!(P::max_of(r) >= lo)) continue;
            float v[E];
            P::unpack(r, v);
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (v[j] >= lo) {
                    const uint32_t key = order_of(v[j]) >> P::KEY_SHIFT;
                    if (key > khi) continue;
                    const uint32_t b = (khi - key) >> bits;            // below BINS: key is at least lo's
                    atomicAdd(cnt + b, 1u);
                    if (MASS) atomicAdd(mass + b, weight_exact(v[j], s, sh.table));
                }
        }
        cluster_sync();
#pragma unroll
        for (int k = 0; k < 4; ++k) { c[k] = 0; w[k] = 0; }
#pragma unroll
        for (int r = 0; r < MAX_CLUSTER; ++r)
            if (r < C) {
                const uint4 x = ld_cluster4(cluster_addr(cnt + 4 * tid, r));
                c[0] += x.x; c[1] += x.y; c[2] += x.z; c[3] += x.w;
            }
        if (MASS)
#pragma unroll
            for (int r = 0; r < MAX_CLUSTER; ++r)
                if (r < C) {
                    unsigned long long x[4];
                    ld_cluster2(cluster_addr(mass + 4 * tid, r), x[0], x[1]);
                    ld_cluster2(cluster_addr(mass + 4 * tid + 2, r), x[2], x[3]);
#pragma unroll
                    for (int k = 0; k < 4; ++k) w[k] += x[k];
                }
        cluster_arrive();                          // others may read on; waited for before the bins are used again
    }
    static __device__ __forceinline__ int level_bits(uint32_t klo, uint32_t khi)
    {
        const int n = 32 - __clz(khi - klo);       // bits of the largest difference
        return n > 11 ? n - 11 : 0;
    }
    // The first of the CTA's bins (four of each thread) at which the sum of x reaches
    // `target`; before and count as there.  False: none does.
    __device__ bool find_bin(const unsigned long long (&x)[4], const uint32_t (&c)[4], unsigned long long target, int which)
    {
        const int tid = threadIdx.x;
        if (tid == 0) sh.bin = BINS;
        unsigned long long total, at = block_scan(x[0] + x[1] + x[2] + x[3], which, total);    // its barrier comes before the writing
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (at < target && target <= at + x[k]) {
                sh.bin = 4 * tid + k;
                sh.before = at;
                sh.mass = x[k];
                sh.count = c[k];
            }
            at += x[k];
        }
        __syncthreads();
        return sh.bin < BINS;
    }
};

// grid: a cluster of C CTAs for each row; ST threads; pieces, then the histogram.
template <typename T, bool RES>
__global__ void __launch_bounds__(ST, 2) k_sample(const __grid_constant__ SampleArgs a)
{
    using S = Sampler<T, RES>;
    using P = Piece<T>;
    constexpr int E = P::E, KS = P::KEY_SHIFT;
    extern __shared__ __align__(16) uint8_t dyn[];
    __shared__ SampleShared sh;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    uint32_t C;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(C));
    const int64_t n = blockIdx.x / C;
    const int q_seq = (int)(n / a.rows);
    uint8_t *after = dyn + (RES ? (size_t)a.per * ST * 16 : 0);
    const T *row = static_cast<const T *>(a.in) + n * a.ld;
    S x{a, sh, reinterpret_cast<uint4 *>(dyn), reinterpret_cast<uint32_t *>(after + BINS * 8),
        reinterpret_cast<unsigned long long *>(after), row, (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T)), (int)C,
        (int)cluster_rank(), 0, Scale{}};
    if (tid < 64) sh.table[tid] = a.table.v[tid];
    if (tid < 4) sh.note[tid] = ~0ull;
    cluster_arrive();                              // waited for before the first access to another CTA
    pdl_wait();
    const float temp = a.T[q_seq];
    const int top_k = a.top_k ? a.top_k[q_seq] : 0;
    const float top_p = a.top_p ? a.top_p[q_seq] : 1.0f, min_p = a.min_p ? a.min_p[q_seq] : 0.0f;
    const float u = a.tokens ? fminf(fmaxf(a.u[n], 0.0f), 1.0f) : 0.0f;
    const bool greedy = !(temp > 0.0f);
    if (tid == 0) {
        sh.k = 1.4426950408889634 / (double)temp;
        sh.shift = min_p > 0.0f ? (double)temp * log(fmin((double)min_p, 1.0)) : 0.0;
    }

    // ---------------------------------------------------- the row, and its maximum
    float mx = -INFINITY;
    {
        constexpr int UN = 4;
        for (int j0 = 0; j0 < a.per; j0 += UN) {
            uint4 r[UN];
#pragma unroll
            for (int j = 0; j < UN; ++j)
                if (j0 + j < a.per) r[j] = x.fetch((j0 + j) * ST + tid);
#pragma unroll
            for (int j = 0; j < UN; ++j)
                if (j0 + j < a.per) {
                    mx = fmaxf(mx, P::max_of(r[j]));
                    if (RES) x.pieces[(j0 + j) * ST + tid] = r[j];
                }
        }
    }
    // the maxima of groups of 2^g lanes, at least top_k of them: the smallest bounds
    // the top_k-th largest element from below
    uint32_t key = order_of(mx), group = 0;
    {
        int g = -1;
        if (top_k > 0 && top_k <= (int)C * ST) g = min(5, 31 - __clz((int)C * ST / top_k));
#pragma unroll
        for (int i = 0; i <= 5; ++i) {
            if (i == g) group = __reduce_min_sync(0xffffffffu, key);
            if (i < 5) key = max(key, __shfl_xor_sync(0xffffffffu, key, 1 << i));
        }
    }
    cluster_wait();
    x.exchange(key, group);
    uint32_t kmax = 0, kgroup = 0xffffffffu;
#pragma unroll
    for (int i = 0; i < MAX_CLUSTER * SWARPS / 32; ++i) {
        const int at = lane + 32 * i;
        if (at < (int)C * SWARPS) {
            kmax = max(kmax, (uint32_t)sh.slot[x.turn][0][at]);
            kgroup = min(kgroup, (uint32_t)sh.slot[x.turn][1][at]);
        }
    }
    kmax = __reduce_max_sync(0xffffffffu, kmax);
    kgroup = __reduce_min_sync(0xffffffffu, kgroup);

    float t = -INFINITY;                           // kept: l > t, and the first q with l == t
    int q = 0, kept_at_most = ALL;
    const bool empty = kmax < LOWEST;
    if (!empty) {
        const float m = Piece<float>::value(kmax);
        const double k = fmin(fmax(sh.k, 1e-38), 3e38);
        x.s = Scale{m, (float)k, 0.0f, a.scale};
        x.s.kl = (float)(k - (double)x.s.kh);
        const uint32_t top = kmax >> KS;
        float low = -3.402823466e38f;              // the lowest value that may be kept
        if (m == INFINITY) low = INFINITY;         // the limit: the infinities share all the mass
        else if (min_p > 0.0f) low = fmaxf(__double2float_ru((double)m + sh.shift), low);
        if (low > -3.402823466e38f) { t = low; q = ALL; }
        if (greedy || top_k == 1 || (top_p <= 0.0f)) {
            t = m;
            q = kept_at_most = 1;
        } else {
            bool k_on = top_k > 0 && top_k < a.V && m < INFINITY, p_on = top_p < 1.0f && m < INFINITY;
            uint32_t c[4];
            unsigned long long w[4], wide[4];
            // -------------------------------------------------------- top-k
            if (k_on) {
                float lo = fmaxf(low, kgroup >= LOWEST ? Piece<float>::value(kgroup) : low);
                uint32_t klo = order_of(lo) >> KS, khi = top, left = top_k;
                for (int level = 0;; ++level) {
                    const int bits = S::level_bits(klo, khi);
                    x.template histogram<false>(lo, khi, bits, c, w);
#pragma unroll
                    for (int i = 0; i < 4; ++i) wide[i] = c[i];
                    const bool found = x.find_bin(wide, c, left, level & 1);
                    cluster_wait();
                    if (!found) { k_on = false; break; }              // fewer than k
                    left -= (uint32_t)sh.before;
                    khi -= sh.bin << bits;
                    if (bits == 0) {
                        t = P::value(khi);
                        q = (int)left;
                        kept_at_most = top_k;
                        if (p_on && level == 0) {
                            // the bins are single values: top-p from the same counts
                            const uint32_t last = sh.bin;
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const uint32_t b = 4 * tid + i;
                                if (b > last) c[i] = 0;
                                if (b == last) c[i] = left;
                                w[i] = c[i] ? c[i] * weight_exact(P::value(top - b), x.s, sh.table) : 0;
                            }
                            unsigned long long z;
                            x.block_scan(w[0] + w[1] + w[2] + w[3], 1, z);
                            const unsigned long long target = (unsigned long long)fmax(ceil((double)top_p * (double)z), 1.0);
                            if (x.find_bin(w, c, target, 0)) {
                                t = P::value(top - sh.bin);
                                q = (int)((target - sh.before + sh.mass / sh.count - 1) / (sh.mass / sh.count));
                            }
                            p_on = false;
                            __syncthreads();                          // before what was found is written again
                        }
                        break;
                    }
                    klo = max(klo, khi - ((1u << bits) - 1));
                    lo = fmaxf(lo, P::value(klo));
                    __syncthreads();
                }
            }
            // -------------------------------------------------------- top-p
            const float t0 = t;
            const int q0 = q;
            for (int attempt = kept_at_most <= 4096 * (int)C ? 1 : 0; p_on; ++attempt) {
                unsigned long long sum;
                uint32_t ties;
                if (attempt) x.template sums<true>(tid * a.per, a.per, t, sum, ties);
                else x.template sums<false>(tid * a.per, a.per, t, sum, ties);
                x.exchange(warp_sum(sum), warp_sum(ties));
                unsigned long long z = x.exchanged_sum(0);
                const unsigned long long nt = min(x.exchanged_sum(1), (unsigned long long)q);
                if (nt) z += nt * weight_exact(t, x.s, sh.table);
                const unsigned long long target = (unsigned long long)fmax(ceil((double)top_p * (double)z), 1.0);
                const unsigned long long slack = attempt ? 0 : (unsigned long long)((double)z * a.slack) + 64;
                // what may be left out has at most 1 - top_p of the mass
                float lo = fmaxf(low, t);
                {
                    const float share = (1.0f - top_p) * ((float)z * __uint_as_float((uint32_t)(127 - a.scale) << 23)) / (float)a.V;
                    const float d = (logf(share) - 0.01f) * temp;
                    lo = fmaxf(lo, m + d * (d < 0.0f ? 1.001f : 0.999f) - 1e-5f * fabsf(m));
                    lo = fminf(lo, m);
                }
                uint32_t klo = order_of(lo) >> KS, khi = top;
                unsigned long long left = target;
                bool sure = true, found;
                for (int level = 0;; ++level) {
                    const int bits = S::level_bits(klo, khi);
                    if (bits == 0) {                                  // single values: their masses from the counts
                        x.template histogram<false>(lo, khi, bits, c, w);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            w[i] = c[i] ? c[i] * weight_exact(P::value(khi - (4 * tid + i)), x.s, sh.table) : 0;
                    } else {
                        x.template histogram<true>(lo, khi, bits, c, w);
                    }
                    found = x.find_bin(w, c, left, level & 1);
                    cluster_wait();
                    if (!found) { sure = false; break; }
                    left -= sh.before;
                    khi -= sh.bin << bits;
                    if (bits == 0) {
                        const unsigned long long each = sh.mass / sh.count, need = (left + each - 1) / each;
                        sure = left > (need - 1) * each + slack && need * each >= left + slack;
                        t = P::value(khi);
                        q = (int)need;
                        kept_at_most = ALL;
                        break;
                    }
                    klo = max(klo, khi - ((1u << bits) - 1));
                    lo = fmaxf(lo, P::value(klo));
                    __syncthreads();
                }
                __syncthreads();
                if (sure || attempt) break;
                t = t0;                            // once more, with the exact mass
                q = q0;
            }
        }
    }

    // ------------------------------------------------------------------- the draw
    int cut = ALL;                                 // the last id with l == t that is kept
    if (empty) {
        if (tid == 0 && x.rank == 0 && a.tokens) a.tokens[n] = -1;
        t = INFINITY;
        q = 0;
    } else if (a.tokens || (a.out && q < ALL)) {
        const unsigned long long wt = q ? weight_exact(t, x.s, sh.table) : 0;
        for (int attempt = kept_at_most <= 4096 * (int)C ? 1 : 0;; ++attempt) {
            unsigned long long sum;
            uint32_t ties;
            if (attempt) x.template sums<true>(tid * a.per, a.per, t, sum, ties);
            else x.template sums<false>(tid * a.per, a.per, t, sum, ties);
            x.exchange(warp_sum(sum), warp_sum(ties));
            // each lane takes four consecutive warps: their ties, then their kept mass
            unsigned long long wm[4];
            uint32_t wn[4], n4 = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) n4 += wn[i] = (uint32_t)x.slot_of(1, 4 * lane + i);
            const uint32_t n_in = warp_scan(n4), n_ex = n_in - n4;
            uint32_t at_n = n_ex;
            unsigned long long m4 = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t b = min(at_n, (uint32_t)q), e = min(at_n + wn[i], (uint32_t)q);
                m4 += wm[i] = x.slot_of(0, 4 * lane + i) + (e - b) * wt;
                at_n += wn[i];
            }
            const unsigned long long m_in = warp_scan(m4);
            const unsigned long long z = __shfl_sync(0xffffffffu, m_in, 31);
            const uint32_t all_ties = __shfl_sync(0xffffffffu, n_in, 31);
            const bool cuts = q && (uint32_t)q < all_ties;
            if (cuts && a.out && attempt <= 1) {
                // the q-th of the ties
                int who = 4 * MAX_CLUSTER * SWARPS;
                uint32_t base = n_ex, there = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (base < (uint32_t)q && (uint32_t)q <= base + wn[i]) { who = 4 * lane + i; there = base; }
                    base += wn[i];
                }
                const unsigned found = __ballot_sync(0xffffffffu, who < MAX_CLUSTER * SWARPS);
                const int src = __ffs(found) - 1;
                who = __shfl_sync(0xffffffffu, who, src);
                there = __shfl_sync(0xffffffffu, there, src);
                if (who == x.rank * SWARPS + warp) {
                    const uint32_t in = warp_scan(ties);
                    uint32_t seen = there + in - ties;
                    if (seen < (uint32_t)q && (uint32_t)q <= seen + ties) {
                        for (int i = 0; i < a.per; ++i) {
                            float v[E];
                            P::unpack(x.piece(tid * a.per + i), v);
#pragma unroll
                            for (int j = 0; j < E; ++j)
                                if (v[j] == t && ++seen == (uint32_t)q)
                                    for (int r = 0; r < (int)C; ++r)
                                        st_cluster(cluster_addr(&sh.note[0], r),
                                                   (unsigned long long)(x.position(tid * a.per + i) + j - x.shift));
                        }
                    }
                }
            }
            if (a.tokens) {
                unsigned long long goal = (unsigned long long)((double)u * (double)z);
                if (goal >= z) goal = z - 1;
                const unsigned long long slack = attempt ? 0 : (unsigned long long)((double)z * a.slack) + 64;
                int who = MAX_CLUSTER * SWARPS;
                unsigned long long base = m_in - m4, there = 0;
                uint32_t base_n = n_ex, there_n = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (base <= goal && goal < base + wm[i]) { who = 4 * lane + i; there = base; there_n = base_n; }
                    base += wm[i];
                    base_n += wn[i];
                }
                const unsigned found = __ballot_sync(0xffffffffu, who < MAX_CLUSTER * SWARPS);
                const int src = __ffs(found) - 1;
                who = __shfl_sync(0xffffffffu, who, src);
                there = __shfl_sync(0xffffffffu, there, src);
                there_n = __shfl_sync(0xffffffffu, there_n, src);
                if (who == x.rank * SWARPS + warp) {
                    // the lane, then the piece, then the element
                    int token = -1;
                    bool sure = true;
                    unsigned long long mine = sum;
                    uint32_t my_ties = ties;
                    int p = tid * a.per, count = a.per;
                    bool ok = true;
                    for (int step = 0; step < 2 && ok; ++step) {
                        for (int p0 = 0;; p0 += 32) {
                            // step 0: the lanes' own ranges; step 1: 32 pieces of the range found
                            if (step == 1) {
                                mine = 0;
                                my_ties = 0;
                                if (p0 + lane < count) {
                                    if (attempt) x.template sums<true>(p + p0 + lane, 1, t, mine, my_ties);
                                    else x.template sums<false>(p + p0 + lane, 1, t, mine, my_ties);
                                }
                            }
                            const uint32_t in_n = warp_scan(my_ties), ex_n = there_n + in_n - my_ties;
                            const uint32_t b = min(ex_n, (uint32_t)q), e = min(ex_n + my_ties, (uint32_t)q);
                            const unsigned long long kept = mine + (e - b) * wt;
                            const unsigned long long in_m = warp_scan(kept), ex_m = there + in_m - kept;
                            const unsigned hit = __ballot_sync(0xffffffffu, ex_m <= goal && goal < ex_m + kept);
                            if (hit) {
                                const int l = __ffs(hit) - 1;
                                there = __shfl_sync(0xffffffffu, ex_m, l);
                                there_n = __shfl_sync(0xffffffffu, ex_n, l);
                                p = step == 0 ? __shfl_sync(0xffffffffu, p, l) : p + p0 + l;
                                break;
                            }
                            there += __shfl_sync(0xffffffffu, in_m, 31);
                            there_n += __shfl_sync(0xffffffffu, in_n, 31);
                            if (step == 0 || p0 + 32 >= count) { ok = false; break; }
                        }
                    }
                    if (ok) {
                        float v[E];
                        P::unpack(x.piece(p), v);
                        unsigned long long at = there;
                        uint32_t at_tie = there_n;
                        sure = false;
#pragma unroll
                        for (int j = 0; j < E; ++j) {
                            unsigned long long w = 0;
                            if (v[j] > t) w = weight_exact(v[j], x.s, sh.table);
                            else if (v[j] == t) { if (at_tie < (uint32_t)q) w = wt; ++at_tie; }
                            if (token < 0 && goal < at + w) {
                                token = (int)(x.position(p) + j - x.shift);
                                sure = attempt || (goal >= at + slack && goal + slack < at + w);
                            }
                            at += w;
                        }
                    }
                    if (token < 0) sure = false;
                    if (lane == 0) {
                        if (token >= 0) a.tokens[n] = token;
                        if (!sure && !attempt)
                            for (int r = 0; r < (int)C; ++r) st_cluster(cluster_addr(&sh.note[1], r), 1ull);
                    }
                }
            }
            if (attempt && !(cuts && a.out)) break;
            cluster_sync();
            if (cuts && a.out) cut = (int)sh.note[0];
            if (attempt || sh.note[1] != 1ull) break;
        }
    }

    // -------------------------------------------------------------- the truncated row
    if (a.out) {
        if (!RES) cluster_sync();                  // nobody reads the row any more: out may be it
        T *out = static_cast<T *>(a.out) + n * a.ldo;
        const bool same = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(row)) & 15) == 0;
        const T dropped = P::raw(a.mask_value);
        for (int i = 0; i < a.per; ++i) {
            const int p = i * ST + tid;
            const int64_t at = x.position(p) - x.shift;
            if (at <= -E || at >= a.V) continue;
            const uint4 r = x.piece(p);
            float v[E];
            P::unpack(r, v);
            T e[E];
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const bool keep = v[j] > t || (v[j] == t && q && at + j <= cut);
                e[j] = keep ? P::raw(v[j]) : dropped;
            }
            if (same && at >= 0 && at + E <= a.V) {
                *reinterpret_cast<uint4 *>(out + at) = P::pack_raw(e);
            } else {
#pragma unroll
                for (int j = 0; j < E; ++j)
                    if (at + j >= 0 && at + j < a.V) out[at + j] = e[j];
            }
        }
    }
}

struct SamplePlan {
    int C, per;
    bool resident;
};

// CTAs of a row's cluster and pieces of a thread: the fewest CTAs that leave two on
// an SM, more while SMs would be idle.
SamplePlan sample_plan(int64_t n, int V, int E, int sms)
{
    auto per_of = [&](int C) {
        const int64_t pieces = ((int64_t)V + E - 1 + E - 1) / E;
        const int64_t per = (pieces + (int64_t)C * ST - 1) / ((int64_t)C * ST);
        return (int)(per | 1);
    };
    auto bytes = [&](int C) { return (size_t)per_of(C) * ST * 16 + HIST_BYTES; };
    int C = 1;
    while (C < MAX_CLUSTER && (bytes(C) > SAMPLE_HALF || (n * C * 2 <= sms && per_of(C) > 1))) C *= 2;
    return {C, per_of(C), bytes(C) <= SAMPLE_SMEM};
}

template <typename T, bool RES>
int launch_sample(const SampleArgs &a, int64_t n, int C, cudaStream_t st)
{
    static OncePerDevice once;
    XH_CUDA(allow_smem(once, k_sample<T, RES>, SAMPLE_SMEM));
    const size_t smem = (RES ? (size_t)a.per * ST * 16 : 0) + HIST_BYTES;
    XH_CUDA(launch_head(k_sample<T, RES>, dim3((unsigned)(n * C)), ST, smem, st, (unsigned)C, a));
    return XPRESS_OK;
}

constexpr int SAMPLE_MAX_V = 1 << 24;

}  // namespace
}  // namespace xp

using namespace xp;

extern "C" int xpress_sample(const xpress_sample_args *in, void *stream)
{
    if (!in || in->n_seq < 0 || in->rows < 1 || in->V < 1 || !in->logits || (!in->out && !in->tokens) || !in->temperature ||
        (in->tokens && !in->u) || in->ld < in->V || (in->out && in->ldo < in->V))
        return XPRESS_ERR_INVALID_ARG;
    if ((in->dtype != XPRESS_F32 && in->dtype != XPRESS_BF16) || in->V > SAMPLE_MAX_V ||
        (int64_t)in->n_seq * in->rows > 0x7fffffff / MAX_CLUSTER)
        return XPRESS_ERR_UNSUPPORTED;
    const uintptr_t es = in->dtype == XPRESS_BF16 ? 2 : 4;
    if (!aligned(in->logits, es) || !aligned(in->out, es) || !aligned(in->tokens, 4) || !aligned(in->u, 4) ||
        !aligned(in->temperature, 4) || !aligned(in->top_k, 4) || !aligned(in->top_p, 4) || !aligned(in->min_p, 4))
        return XPRESS_ERR_INVALID_ARG;
    const int64_t n = (int64_t)in->n_seq * in->rows;
    if (n == 0) return XPRESS_OK;
    const int sms = current_sms();
    if (sms < 1) return XPRESS_ERR_CUDA;
    SampleArgs a{};
    a.in = in->logits; a.out = in->out; a.ld = in->ld; a.ldo = in->ldo;
    a.rows = in->rows; a.V = in->V;
    a.T = in->temperature; a.top_k = in->top_k; a.top_p = in->top_p; a.min_p = in->min_p; a.u = in->u;
    a.tokens = in->tokens;
    a.mask_value = in->mask_value;
    static constexpr ExpTable table = make_exp_table();
    a.table = table;
    int log2v = 0;
    while ((1 << log2v) < in->V) ++log2v;
    a.scale = 61 - log2v;
    // the exponential, three roundings of the exponent (whose mean over the mass is
    // below log2 V + 5: an element at -x has at most 2^-x of it), the sums
    a.slack = 1.1f * (1.0f / (1 << 21) + 3.0f * 0.6932f * (log2v + 5) / (1 << 24));
    const SamplePlan p = sample_plan(n, in->V, (int)(16 / es), sms);
    a.per = p.per;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (in->dtype == XPRESS_BF16)
        return p.resident ? launch_sample<uint16_t, true>(a, n, p.C, st) : launch_sample<uint16_t, false>(a, n, p.C, st);
    return p.resident ? launch_sample<float, true>(a, n, p.C, st) : launch_sample<float, false>(a, n, p.C, st);
}
