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
    int slice;                     // 16-byte pieces of a CTA
    int per;                       // ... of a thread (odd)
    int scale;                     // a weight of 1 is 2^scale
    float slack;                   // what a sum of fast weights may be off, relative
    ExpTable table;
};

constexpr int ST = 256, SWARPS = ST / 32;
constexpr int BINS = 4 * ST;                     // of a histogram: four to a thread
constexpr int MAX_CLUSTER = 8;
constexpr int ALL = 0x7fffffff;
constexpr size_t HIST_BYTES = BINS * 16;         // counts, masses, largest and smallest key
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
    const float dh = __fsub_rn(l, s.m), bb = __fsub_rn(dh, l);
    const float dl = __fadd_rn(__fsub_rn(l, __fsub_rn(dh, bb)), __fsub_rn(-s.m, bb));
    const float ph = fmaxf(__fmul_rn(dh, s.kh), -70.0f);            // 2^-70 is below half a unit
    const float pl = fmaf(dh, s.kh, -ph) + fmaf(dh, s.kl, dl * s.kh);
    const float steps = rintf(ph * 64.0f);
    const float g = fmaf(steps, -0.015625f, ph) + pl;
    const float e = g * fmaf(g, fmaf(g, fmaf(g, 9.61812910e-3f, 5.55041087e-2f), 2.40226507e-1f), 6.93147181e-1f);
    const int i = (int)steps;
    const unsigned long long t = table[i & 63];
    const unsigned long long w = t + (unsigned long long)(((long long)t * __float2int_rn(e * 4294967296.0f)) >> 32);
    // w has 32 bits behind the point, and 2^(i >> 6) to come
    const int up = s.bits - 32 + (i >> 6), down = min(max(-up, 1), 63);
    const unsigned long long r = up >= 0 ? w << max(up, 0) : (w + (1ull << (down - 1))) >> down;
    return l == s.m ? 1ull << s.bits : r;                            // (both may be infinite)
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
__device__ __forceinline__ void cluster_sync() { cluster_arrive(); cluster_wait(); }

struct SampleShared {
    unsigned long long table[64];                                    // 2^(j / 64)
    unsigned long long slot[2][3][MAX_CLUSTER * SWARPS];             // what the cluster's warps exchange: [turn][value][warp]
    unsigned long long scan[2][SWARPS];
    unsigned long long note[4];                                      // written by one thread of the cluster: the id cut, a draw to repeat
    double shift;                                                    // T ln(min_p)
    unsigned long long before, mass;                                 // of the bin that was looked for
    uint32_t bin, count, largest, smallest;
};

// Four bins of each thread, summed over the cluster.
struct Bins {
    uint32_t count[4], mass[4], largest[4], smallest[4];
};

// What a kernel's passes share.
template <typename T, bool RES>
struct Sampler {
    using P = Piece<T>;
    static constexpr int E = P::E;
    const SampleArgs &a;
    SampleShared &sh;
    uint4 *pieces;                 // [slice] of this CTA (RES)
    uint32_t *hist;                // [4][BINS]: counts, masses, largest and smallest key
    const T *row;                  // the row's first element
    int shift;                     // elements from a 16-byte boundary to it
    int C, rank, turn;
    Scale s;

    __device__ __forceinline__ int64_t position(int p) const { return ((int64_t)rank * a.slice + p) * E; }
    // This thread's pieces, in the order of the ids.
    __device__ __forceinline__ int first() const { return threadIdx.x * a.per; }
    __device__ __forceinline__ int count(int from) const { return max(0, min(a.per, a.slice - from)); }
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
    // Every warp's values to all CTAs of the cluster.
    __device__ void exchange(unsigned long long v0, unsigned long long v1, unsigned long long v2 = 0)
    {
        const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
        turn ^= 1;
        if (lane < C) {
            const uint32_t to = cluster_addr(&sh.slot[turn][0][rank * SWARPS + warp], lane);
            st_cluster(to, v0);
            st_cluster(to + (uint32_t)sizeof(sh.slot[0][0]), v1);
            st_cluster(to + 2 * (uint32_t)sizeof(sh.slot[0][0]), v2);
        }
        cluster_sync();
    }
    // What the warp 2 lane + i exchanged (0 past the last one).
    __device__ __forceinline__ unsigned long long slot_of(int which, int i) const
    {
        const int w = 2 * (threadIdx.x % 32) + i;
        return w < C * SWARPS ? sh.slot[turn][which][w] : 0;
    }
    // The sum of what the warps exchanged.
    __device__ unsigned long long exchanged_sum(int which) const { return warp_sum(slot_of(which, 0) + slot_of(which, 1)); }
    // The smallest key above `key` (or the largest below it) of any element; ~0 (0) if there is none.
    __device__ uint32_t next_key(uint32_t key, bool above)
    {
        uint32_t best = above ? ~0u : 0u;
        for (int i = 0; i < count(first()); ++i) {
            float v[E];
            P::unpack(piece(first() + i), v);
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const uint32_t k = order_of(v[j]) >> P::KEY_SHIFT;
                if (above && k > key) best = min(best, k);
                if (!above && k < key) best = max(best, k);
            }
        }
        best = above ? __reduce_min_sync(0xffffffffu, best) : __reduce_max_sync(0xffffffffu, best);
        exchange(above ? (uint32_t)~best : best, 0);
        best = __reduce_max_sync(0xffffffffu, max((uint32_t)slot_of(0, 0), (uint32_t)slot_of(0, 1)));
        return above ? ~best : best;
    }
    // Exclusive sum over the CTA's threads.
    __device__ unsigned long long block_scan(unsigned long long v, int which)
    {
        const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
        const unsigned long long in = warp_scan(v);
        if (lane == 31) sh.scan[which][warp] = in;
        __syncthreads();
        unsigned long long base = 0;
#pragma unroll
        for (int i = 0; i < SWARPS; ++i) base += i < warp ? sh.scan[which][i] : 0ull;
        return base + in - v;
    }

    // Sum of the weights of l > t and number of l == t in n pieces from p of this CTA
    // (ROW: of every element, none of which is limited by t).
    template <bool EXACT, bool ROW>
    __device__ void sums(int p, int n, float t, unsigned long long &sum, uint32_t &ties) const
    {
        unsigned long long fixed = 0;
        float hi = 0.0f, lo = 0.0f;
        ties = 0;
#pragma unroll 2
        for (int i = 0; i < n; ++i) {
            const uint4 r = piece(p + i);
            if (!ROW && P::max_of(r) < t) continue;
            float v[E];
            P::unpack(r, v);
            if (EXACT) {
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    const unsigned long long w = weight_exact(v[j], s, sh.table);
                    fixed += v[j] > t ? w : 0ull;
                    ties += v[j] == t;
                }
            } else {
                float w[E];
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    w[j] = weight_fast(v[j], s);
                    if (!ROW) {
                        if (!(v[j] > t)) w[j] = 0.0f;
                        ties += v[j] == t;
                    }
                }
#pragma unroll
                for (int o = E / 2; o > 0; o >>= 1)
#pragma unroll
                    for (int j = 0; j < o; ++j) w[j] += w[j + o];
                // hi + lo keeps what the addition rounds away
                const float x = __fadd_rn(hi, w[0]), b = __fsub_rn(x, hi);
                lo += __fadd_rn(__fsub_rn(hi, __fsub_rn(x, b)), __fsub_rn(w[0], b));
                hi = x;
            }
        }
        const float one = __uint_as_float((uint32_t)(127 + s.bits) << 23);
        sum = EXACT ? fixed : __float2ull_rn(hi * one) + (unsigned long long)__float2ll_rn(lo * one);
    }
    __device__ void sums(bool exact, int p, int n, float t, unsigned long long &sum, uint32_t &ties) const
    {
        if (exact) sums<true, false>(p, n, t, sum, ties);
        else if (t == -INFINITY) sums<false, true>(p, n, t, sum, ties);
        else sums<false, false>(p, n, t, sum, ties);
    }
    // sums() of this thread's pieces with exact weights for t, and for a lower t0 beside it.
    __device__ void sums_two(float t, float t0, unsigned long long &sum, uint32_t &ties, unsigned long long &sum0, uint32_t &ties0) const
    {
        sum = sum0 = 0;
        ties = ties0 = 0;
        const int n = count(first());
        for (int i = 0; i < n; ++i) {
            const uint4 r = piece(first() + i);
            if (P::max_of(r) < t0) continue;
            float v[E];
            P::unpack(r, v);
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const unsigned long long w = weight_exact(v[j], s, sh.table);
                sum += v[j] > t ? w : 0ull;
                sum0 += v[j] > t0 ? w : 0ull;
                ties += v[j] == t;
                ties0 += v[j] == t0;
            }
        }
    }

    // Histogram of the elements from lo up whose keys are at most khi, from the largest
    // down, by bins of equal width 1 / inv (inv > 0) or of 2^bits keys: their number, and
    // where a bin may have several keys (bits > 0) the largest and the smallest, and
    // (MASS) their mass times `unit`, rounded.
    template <bool MASS>
    __device__ void histogram(float lo, uint32_t khi, int bits, float inv, float unit, Bins &b)
    {
        const int tid = threadIdx.x, n = count(first());
        const bool keys = bits > 0;
        reinterpret_cast<uint4 *>(hist)[tid] = make_uint4(0, 0, 0, 0);
        if (keys) {
            if (MASS) reinterpret_cast<uint4 *>(hist + BINS)[tid] = make_uint4(0, 0, 0, 0);
            reinterpret_cast<uint4 *>(hist + 2 * BINS)[tid] = make_uint4(0, 0, 0, 0);
            reinterpret_cast<uint4 *>(hist + 3 * BINS)[tid] = make_uint4(~0u, ~0u, ~0u, ~0u);
        }
        __syncthreads();
#pragma unroll 2
        for (int i = 0; i < n; ++i) {
            const uint4 r = piece(first() + i);
            if (!(P::max_of(r) >= lo)) continue;
            float v[E];
            P::unpack(r, v);
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (v[j] >= lo) {
                    const uint32_t key = order_of(v[j]) >> P::KEY_SHIFT;
                    if (key > khi) continue;
                    // (below BINS also by keys: key is at least lo's)
                    const uint32_t at = inv > 0.0f ? min((uint32_t)((s.m - v[j]) * inv), (uint32_t)BINS - 1) : (khi - key) >> bits;
                    atomicAdd(hist + at, 1u);
                    if (keys) {
                        if (MASS) atomicAdd(hist + BINS + at, __float2uint_rn(weight_fast(v[j], s) * unit));
                        atomicMax(hist + 2 * BINS + at, key);
                        atomicMin(hist + 3 * BINS + at, key);
                    }
                }
        }
        cluster_sync();
#pragma unroll
        for (int k = 0; k < 4; ++k) { b.count[k] = b.mass[k] = b.largest[k] = 0; b.smallest[k] = ~0u; }
#pragma unroll
        for (int r = 0; r < MAX_CLUSTER; ++r)
            if (r < C) {
                const uint4 x = ld_cluster4(cluster_addr(hist + 4 * tid, r));
                b.count[0] += x.x; b.count[1] += x.y; b.count[2] += x.z; b.count[3] += x.w;
            }
        if (keys)
#pragma unroll 2
            for (int r = 0; r < C; ++r) {
                if (MASS) {
                    const uint4 x = ld_cluster4(cluster_addr(hist + BINS + 4 * tid, r));
                    b.mass[0] += x.x; b.mass[1] += x.y; b.mass[2] += x.z; b.mass[3] += x.w;
                }
                const uint4 y = ld_cluster4(cluster_addr(hist + 2 * BINS + 4 * tid, r));
                b.largest[0] = max(b.largest[0], y.x); b.largest[1] = max(b.largest[1], y.y);
                b.largest[2] = max(b.largest[2], y.z); b.largest[3] = max(b.largest[3], y.w);
                const uint4 z = ld_cluster4(cluster_addr(hist + 3 * BINS + 4 * tid, r));
                b.smallest[0] = min(b.smallest[0], z.x); b.smallest[1] = min(b.smallest[1], z.y);
                b.smallest[2] = min(b.smallest[2], z.z); b.smallest[3] = min(b.smallest[3], z.w);
            }
        cluster_arrive();                          // others may read on; waited for before the bins are used again
    }
    // Bins of equal width from m down to lo, for the first level (0 where the width has no use).
    __device__ __forceinline__ float bins_per(float lo) const
    {
        const float d = s.m - lo;
        return d > 1e-30f && d < 1e30f ? (BINS - 0.5f) / d : 0.0f;
    }
    static __device__ __forceinline__ int level_bits(uint32_t klo, uint32_t khi)
    {
        constexpr int LOG = 10;
        static_assert(1 << LOG == BINS, "bins by bits of the keys");
        const int n = 32 - __clz(khi - klo);       // bits of the largest difference
        return n > LOG ? n - LOG : 0;
    }
    // The first of the CTA's bins at which the sum of x reaches `target`; what is known
    // of it.  False: none does.
    __device__ bool find_bin(const unsigned long long (&x)[4], const Bins &b, unsigned long long target, int which)
    {
        const int tid = threadIdx.x;
        if (tid == 0) sh.bin = BINS;
        unsigned long long at = block_scan(x[0] + x[1] + x[2] + x[3], which);    // its barrier comes before the writing
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (at < target && target <= at + x[k]) {
                sh.bin = 4 * tid + k;
                sh.before = at;
                sh.mass = x[k];
                sh.count = b.count[k];
                sh.largest = b.largest[k];
                sh.smallest = b.smallest[k];
            }
            at += x[k];
        }
        __syncthreads();
        return sh.bin < BINS;
    }
};

// What a row keeps: l > t, and the first q with l == t.
struct Kept {
    float t;
    int q;
};

// grid: a cluster of C CTAs for each row; ST threads; pieces, then the histogram.
template <typename T, bool RES>
__global__ void __launch_bounds__(ST, 4) k_sample(const __grid_constant__ SampleArgs a)
{
    using S = Sampler<T, RES>;
    using P = Piece<T>;
    using F = Piece<float>;
    constexpr int E = P::E, KS = P::KEY_SHIFT;
    extern __shared__ __align__(16) uint8_t dyn[];
    __shared__ SampleShared sh;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    uint32_t C;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(C));
    const int64_t n = blockIdx.x / C;
    const int q_seq = (int)(n / a.rows);
    const T *row = static_cast<const T *>(a.in) + n * a.ld;
    S x{a, sh, reinterpret_cast<uint4 *>(dyn), reinterpret_cast<uint32_t *>(dyn + (RES ? (size_t)a.slice * 16 : 0)), row,
        (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T)), (int)C, (int)cluster_rank(), 0, Scale{}};
    if (tid < 64) sh.table[tid] = a.table.v[tid];
    if (tid < 4) sh.note[tid] = ~0ull;
    cluster_arrive();                              // waited for before the first access to another CTA
    pdl_wait();
    const float temp = a.T[q_seq];
    const int top_k = a.top_k ? a.top_k[q_seq] : 0;
    const float top_p = a.top_p ? a.top_p[q_seq] : 1.0f, min_p = a.min_p ? a.min_p[q_seq] : 0.0f;
    const float u = a.tokens ? fminf(fmaxf(a.u[n], 0.0f), 1.0f) : 0.0f;

    // ---------------------------------------------------- the row, and its maximum
    float mx = -INFINITY;
    const int64_t ids0 = (int64_t)x.rank * a.slice * E - x.shift;              // the id of this CTA's position 0
    if (RES) {
        // what lies inside the row comes by asynchronous copies, all under way at once
        const int p0 = ids0 < 0 ? 1 : 0, p1 = (int)min((int64_t)a.slice, max((a.V - ids0) / E, (int64_t)0));
        const uint64_t policy = policy_evict_first();
        const int half = (a.slice / 2 + ST - 1) / ST * ST;
        for (int p = tid; p < a.slice; p += ST) {
            if (p >= p0 && p < p1) cp_async16(x.pieces + p, row + ids0 + (int64_t)p * E, 16, policy);
            if (p < half && p + ST >= half) cp_async_commit();                  // (each thread has one such p, or none)
        }
        cp_async_commit();
        if (tid == 0) sh.shift = min_p > 0.0f ? (double)temp * log(fmin((double)min_p, 1.0)) : 0.0;
        auto take = [&](int from, int to) {
#pragma unroll 4
            for (int p = from; p < to; p += ST) {
                const bool inside = p >= p0 && p < p1;
                const uint4 got = inside ? x.pieces[p] : make_uint4(0, 0, 0, 0), r = inside ? P::no_nan(got) : x.fetch(p);
                if (!inside || r.x != got.x || r.y != got.y || r.z != got.z || r.w != got.w) x.pieces[p] = r;
                mx = fmaxf(mx, P::max_of(r));
            }
        };
        if (tid < half) {
            cp_async_wait<1>();
            take(tid, min(half, a.slice));
        }
        cp_async_wait<0>();
        take(half + tid, a.slice);
    } else {
        if (tid == 0) sh.shift = min_p > 0.0f ? (double)temp * log(fmin((double)min_p, 1.0)) : 0.0;
#pragma unroll 4
        for (int p = tid; p < a.slice; p += ST) mx = fmaxf(mx, P::max_of(x.fetch(p)));
    }
    // the maxima of groups of 2^g lanes, at least top_k of them: the smallest bounds
    // the top_k-th largest element from below
    uint32_t key = order_of(mx), group = ~0u, groups = 0;
    {
        int g = -1;
        if (top_k > 0) {
            const int64_t pieces = ((int64_t)a.V + x.shift + E - 1) / E, full = pieces / a.slice;
            const int64_t threads = full * min(ST, a.slice) + min((int64_t)ST, pieces - full * a.slice);    // that have elements
            if (threads >= top_k) g = min(5, 31 - __clz((int)threads / top_k));
        }
#pragma unroll
        for (int i = 0; i <= 5; ++i) {
            if (i == g) {
                groups = __popc(__ballot_sync(0xffffffffu, key >= LOWEST)) >> g;
                group = __reduce_min_sync(0xffffffffu, key >= LOWEST ? key : ~0u);
            }
            if (i < 5) key = max(key, __shfl_xor_sync(0xffffffffu, key, 1 << i));
        }
    }
    cluster_wait();
    x.exchange(key, (unsigned long long)groups << 32 | (uint32_t)~group);
    const uint32_t kmax = __reduce_max_sync(0xffffffffu, max((uint32_t)x.slot_of(0, 0), (uint32_t)x.slot_of(0, 1)));
    uint32_t kgroup = ~__reduce_max_sync(0xffffffffu, max((uint32_t)x.slot_of(1, 0), (uint32_t)x.slot_of(1, 1)));
    if ((int)__reduce_add_sync(0xffffffffu, (uint32_t)(x.slot_of(1, 0) >> 32) + (uint32_t)(x.slot_of(1, 1) >> 32)) < top_k) kgroup = 0;

    Kept kept{-INFINITY, 0};
    const bool empty = kmax < LOWEST;
    bool k_on = false, p_on = false, check_p = false;
    int few = ALL;                                 // at most so many are kept
    unsigned long long z1 = 0;                     // mass of what min-p and top-k keep
    bool z1_exact = false;
    Kept first{-INFINITY, 0};                      // ... as a threshold
    if (!empty) {
        const float m = F::value(kmax);
        {
            // log2(e) / T to 48 bits: the quotient's rounding comes back through the remainder
            const float tc = fminf(fmaxf(temp, 1e-37f), 1e37f), kh = 1.44269502f / tc;
            x.s = Scale{m, kh, (fmaf(-kh, tc, 1.44269502f) + 1.92596303e-8f) / tc, a.scale};
        }
        const uint32_t top = kmax >> KS;
        float low = -3.402823466e38f;              // the lowest value that may be kept
        if (m == INFINITY) low = INFINITY;         // the limit: the infinities share all the mass
        else if (min_p > 0.0f) low = fmaxf(__double2float_ru((double)m + sh.shift), low);
        if (low > -3.402823466e38f) kept = {low, ALL};
        if (!(temp > 0.0f) || top_k == 1 || top_p <= 0.0f) {
            kept = {m, 1};
            few = 1;
        } else {
            k_on = top_k > 0 && top_k < a.V && m < INFINITY;
            p_on = top_p < 1.0f && m < INFINITY;
        }
        Bins b;
        unsigned long long wide[4];
        // ------------------------------------------------------------ top-k
        if (k_on) {
            float lo = kgroup >= LOWEST ? fmaxf(low, F::value(kgroup)) : low;
            uint32_t klo = order_of(lo) >> KS, khi = top, left = top_k;
            for (int level = 0;; ++level) {
                const int bits = S::level_bits(klo, khi);
                x.template histogram<false>(lo, khi, bits, level == 0 && bits ? x.bins_per(lo) : 0.0f, 0.0f, b);
#pragma unroll
                for (int i = 0; i < 4; ++i) wide[i] = b.count[i];
                const bool found = x.find_bin(wide, b, left, level & 1);
                cluster_wait();
                if (!found) break;                                    // fewer than k
                few = top_k;
                left -= (uint32_t)sh.before;
                if (bits == 0) {
                    kept = {P::value(khi - sh.bin), (int)left};
                    if (p_on && level == 0) {
                        // the bins are single values: top-p from the same counts
                        const uint32_t last = sh.bin;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t at = 4 * tid + i;
                            if (at > last) b.count[i] = 0;
                            if (at == last) b.count[i] = left;
                            wide[i] = b.count[i] ? b.count[i] * weight_exact(P::value(top - at), x.s, sh.table) : 0;
                        }
                        const unsigned long long mine = wide[0] + wide[1] + wide[2] + wide[3];
                        const unsigned long long z = warp_sum(mine);
                        __syncthreads();                              // what was found has been read
                        if (lane == 0) sh.scan[1][warp] = z;
                        __syncthreads();
                        for (int i = 0; i < SWARPS; ++i) z1 += sh.scan[1][i];
                        const unsigned long long target = (unsigned long long)fmax(ceil((double)top_p * (double)z1), 1.0);
                        if (x.find_bin(wide, b, target, 0)) {
                            const unsigned long long each = sh.mass / sh.count;
                            kept = {P::value(top - sh.bin), (int)((target - sh.before + each - 1) / each)};
                        }
                        p_on = false;
                    }
                    break;
                }
                if (left == 1) { kept = {P::value(sh.largest), 1}; break; }
                if (left == sh.count) { kept = {P::value(sh.smallest), ALL}; break; }
                klo = sh.smallest;
                khi = sh.largest;
                lo = P::value(klo);
                __syncthreads();
            }
        }
        // ------------------------------------------------------------ top-p
        first = kept;
        if (p_on) {
            unsigned long long sum;
            uint32_t ties;
            z1_exact = few <= 4096 * (int)C;
            x.sums(z1_exact, x.first(), x.count(x.first()), kept.t, sum, ties);
            x.exchange(warp_sum(sum), warp_sum(ties));
            z1 = x.exchanged_sum(0);
            const unsigned long long nt = min(x.exchanged_sum(1), (unsigned long long)kept.q);
            if (nt) z1 += nt * weight_exact(kept.t, x.s, sh.table);
            const unsigned long long target = (unsigned long long)fmax(ceil((double)top_p * (double)z1), 1.0);
            const unsigned long long slack = z1_exact ? 0 : (unsigned long long)((double)z1 * a.slack) + 64;
            const int down = max(0, 33 - __clzll(z1));                // z1 >> down has 31 bits
            const float unit = __uint_as_float((uint32_t)(127 + a.scale - down) << 23);
            // what may be left out has at most 1 - top_p of the mass
            float lo = fmaxf(low, kept.t);
            {
                const float share = (1.0f - top_p) * ((float)z1 * __uint_as_float((uint32_t)(127 - a.scale) << 23)) / (float)a.V;
                const float d = (logf(share) - 0.01f) * temp;
                lo = fminf(fmaxf(lo, m + d * (d < 0.0f ? 1.001f : 0.999f) - 1e-5f * fabsf(m)), m);
            }
            uint32_t klo = order_of(lo) >> KS, khi = top;
            unsigned long long left = 0;
            bool sure = true;                                         // no bin was taken by rounded masses
            for (int level = 0;; ++level) {
                const int bits = S::level_bits(klo, khi);
                x.template histogram<true>(lo, khi, bits, level == 0 && bits ? x.bins_per(lo) : 0.0f, unit, b);
                if (level == 0) left = bits ? target >> down : target;
                bool found;
                if (bits == 0) {
                    // single values: their masses from the counts
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        wide[i] = b.count[i] ? b.count[i] * weight_exact(P::value(khi - (4 * tid + i)), x.s, sh.table) : 0;
                    found = x.find_bin(wide, b, sure ? left : max(left, 1ull) << down, level & 1);
                } else {
                    sure = false;
#pragma unroll
                    for (int i = 0; i < 4; ++i) wide[i] = b.mass[i];
                    found = x.find_bin(wide, b, max(left, 1ull), level & 1);
                }
                cluster_wait();
                if (!found) {
                    // by rounding: the smallest that was counted, or what the bound left out
                    check_p = true;
                    kept.t = P::value(klo);
                    break;
                }
                left -= min(left, sh.before);
                if (bits == 0) {
                    kept.t = P::value(khi - sh.bin);
                    if (sure) {
                        const unsigned long long each = sh.mass / sh.count, need = (left + each - 1) / each;
                        kept.q = (int)need;
                        check_p = !(left > (need - 1) * each + slack && need * each >= left + slack);
                    } else {
                        check_p = true;
                    }
                    break;
                }
                check_p = true;
                // one of two, or the largest of several, by its mass
                const uint32_t big = sh.largest, small = sh.smallest;
                const bool take = left <= (weight_exact(P::value(big), x.s, sh.table) >> down);
                if (take || sh.count <= 2) { kept.t = P::value(take ? big : small); break; }
                klo = small;
                khi = big;
                lo = P::value(klo);
                __syncthreads();
            }
        }
    }

    // ------------------------------------------------------------------- the draw
    int cut = ALL;                                 // the last id with l == t that is kept
    if (empty) {
        if (tid == 0 && x.rank == 0 && a.tokens) a.tokens[n] = -1;
        kept = {INFINITY, 0};
    } else if (a.tokens || check_p || (a.out && kept.q < ALL && kept.q > 0)) {
        // a check that the fast weights could hardly decide starts with exact ones
        bool exact = few <= 4096 * (int)C || (check_p && (double)weight_exact(kept.t, x.s, sh.table) < 20.0 * a.slack * (double)z1);
        // while t is not sure: what is known of its key, from below and above
        uint32_t known_lo = max(order_of(first.t), LOWEST) >> KS, known_hi = kmax >> KS;
        int moves = 0;
        for (;;) {
            const float t = kept.t;
            unsigned long long sum;
            uint32_t ties;
            if (check_p && exact && !z1_exact) {
                unsigned long long sum0;
                uint32_t ties0;
                x.sums_two(t, first.t, sum, ties, sum0, ties0);
                x.exchange(warp_sum(sum), warp_sum((unsigned long long)ties0 << 32 | ties), warp_sum(sum0));
                z1 = x.exchanged_sum(2);
                const unsigned long long nt = min(x.exchanged_sum(1) >> 32, (unsigned long long)first.q);
                if (nt) z1 += nt * weight_exact(first.t, x.s, sh.table);
                z1_exact = true;
            } else {
                x.sums(exact, x.first(), x.count(x.first()), t, sum, ties);
                x.exchange(warp_sum(sum), warp_sum(ties));
            }
            // each lane takes two consecutive warps: their ties, then their kept mass
            const uint32_t wn0 = (uint32_t)x.slot_of(1, 0), wn1 = (uint32_t)x.slot_of(1, 1);
            const unsigned long long ws0 = x.slot_of(0, 0), ws1 = x.slot_of(0, 1);
            const uint32_t n_in = warp_scan(wn0 + wn1), n0 = n_in - wn0 - wn1, n1 = n_in - wn1;
            const uint32_t all_ties = __shfl_sync(0xffffffffu, n_in, 31);
            const unsigned long long wt = all_ties ? weight_exact(t, x.s, sh.table) : 0;
            if (check_p) {
                // is t where the mass before reaches the target?  How many of its ties?
                const unsigned long long above = warp_sum(ws0 + ws1);
                const uint32_t may = t == first.t ? min(all_ties, (uint32_t)first.q) : all_ties;
                const unsigned long long target = (unsigned long long)fmax(ceil((double)top_p * (double)z1), 1.0);
                const unsigned long long slack = (exact ? 0 : (unsigned long long)((double)above * a.slack) + 64) +
                                                 (z1_exact ? 0 : (unsigned long long)((double)z1 * a.slack) + 64);
                const bool small = above >= target + slack, large = above + may * wt + slack < target && t > first.t;
                if ((small || large) && moves < 40) {                 // 33 halve any range of keys to one
                    // the next value first (rounded masses put t off by one), then the middle
                    const uint32_t at = order_of(t) >> KS;
                    if (small) known_lo = max(known_lo, at + 1);
                    else known_hi = min(known_hi, at - 1);
                    uint32_t to = known_lo + (known_hi - known_lo) / 2;
                    if (moves++ == 0) to = min(max(x.next_key(at, small), known_lo), known_hi);
                    kept.t = P::value(to);
                    continue;
                }
                const unsigned long long over = target > above ? target - above : 1;
                const unsigned long long need = wt ? min((over + wt - 1) / wt, (unsigned long long)max(may, 1u)) : 1;
                const bool sure = target > above + (need - 1) * wt + slack && (above + need * wt >= target + slack);
                if (!sure && !(exact && z1_exact)) {
                    exact = true;                                     // once more, with exact masses
                    continue;
                }
                kept.q = (int)need;
                check_p = false;
            }
            const uint32_t q = (uint32_t)kept.q;
            const unsigned long long wm0 = ws0 + (min(n0 + wn0, q) - min(n0, q)) * wt, wm1 = ws1 + (min(n1 + wn1, q) - min(n1, q)) * wt;
            const unsigned long long m_in = warp_scan(wm0 + wm1);
            const unsigned long long z = __shfl_sync(0xffffffffu, m_in, 31);
            const bool cuts = a.out && q && q < all_ties;
            const int me = x.rank * SWARPS + warp;
            if (cuts) {
                // the q-th of the ties
                const unsigned f0 = __ballot_sync(0xffffffffu, n0 < q && q <= n0 + wn0), f1 = __ballot_sync(0xffffffffu, n1 < q && q <= n1 + wn1);
                const int who = f0 ? 2 * (__ffs(f0) - 1) : 2 * (__ffs(f1) - 1) + 1;
                if (who == me) {
                    const uint32_t there = __shfl_sync(0xffffffffu, f0 ? n0 : n1, who / 2);
                    const uint32_t in = warp_scan(ties);
                    uint32_t seen = there + in - ties;
                    if (seen < q && q <= seen + ties) {
                        for (int i = 0; i < x.count(x.first()); ++i) {
                            float v[E];
                            P::unpack(x.piece(x.first() + i), v);
#pragma unroll
                            for (int j = 0; j < E; ++j)
                                if (v[j] == t && ++seen == q)
                                    for (int r = 0; r < (int)C; ++r)
                                        st_cluster(cluster_addr(&sh.note[0], r),
                                                   (unsigned long long)(x.position(x.first() + i) + j - x.shift));
                        }
                    }
                }
            }
            if (a.tokens) {
                unsigned long long goal = (unsigned long long)((double)u * (double)z);
                if (goal >= z) goal = z - 1;
                const unsigned long long slack = exact ? 0 : (unsigned long long)((double)z * a.slack) + 64;
                const unsigned long long m0 = m_in - wm0 - wm1, m1 = m_in - wm1;
                const unsigned f0 = __ballot_sync(0xffffffffu, m0 <= goal && goal < m0 + wm0), f1 = __ballot_sync(0xffffffffu, m1 <= goal && goal < m1 + wm1);
                const int who = f0 ? 2 * (__ffs(f0) - 1) : 2 * (__ffs(f1) - 1) + 1;
                if (who == me) {
                    // the lane, then the piece, then the element
                    unsigned long long there = __shfl_sync(0xffffffffu, f0 ? m0 : m1, who / 2), mine = sum;
                    uint32_t there_n = __shfl_sync(0xffffffffu, f0 ? n0 : n1, who / 2), my_ties = ties;
                    int p = 0;
                    bool ok = true;
                    for (int step = 0; step < 3 && ok; ++step) {
                        for (int p0 = 0;; p0 += 32) {
                            // step 0: the lanes' own ranges; 1: 32 pieces of the range found; 2: the elements of the piece found
                            if (step == 1) {
                                mine = 0;
                                my_ties = 0;
                                if (p0 + lane < x.count(p)) x.sums(exact, p + p0 + lane, 1, t, mine, my_ties);
                            }
                            if (step == 2) {
                                mine = 0;
                                my_ties = 0;
                                if (lane < E) {
                                    float v[E];
                                    P::unpack(x.piece(p), v);
                                    float l = v[0];
#pragma unroll
                                    for (int j = 1; j < E; ++j) l = lane == j ? v[j] : l;
                                    if (l > t) mine = weight_exact(l, x.s, sh.table);
                                    my_ties = l == t;
                                }
                            }
                            const uint32_t in_n = warp_scan(my_ties), ex_n = there_n + in_n - my_ties;
                            const unsigned long long own = mine + (min(ex_n + my_ties, q) - min(ex_n, q)) * wt;
                            const unsigned long long in_m = warp_scan(own), ex_m = there + in_m - own;
                            const unsigned hit = __ballot_sync(0xffffffffu, ex_m <= goal && goal < ex_m + own);
                            if (hit) {
                                const int l = __ffs(hit) - 1;
                                if (step == 2) {
                                    const bool sure = ex_m + slack <= goal && goal + slack < ex_m + own;
                                    if (lane == l) {
                                        a.tokens[n] = (int)(x.position(p) + l - x.shift);
                                        if (!exact && !sure)
                                            for (int r = 0; r < (int)C; ++r) st_cluster(cluster_addr(&sh.note[1], r), 1ull);
                                    }
                                    p = -1;
                                } else {
                                    there = __shfl_sync(0xffffffffu, ex_m, l);
                                    there_n = __shfl_sync(0xffffffffu, ex_n, l);
                                    p = step == 0 ? (warp * 32 + l) * a.per : p + p0 + l;
                                }
                                break;
                            }
                            there += __shfl_sync(0xffffffffu, in_m, 31);
                            there_n += __shfl_sync(0xffffffffu, in_n, 31);
                            if (step != 1 || p0 + 32 >= x.count(p)) { ok = false; break; }
                        }
                    }
                    if (!exact && p >= 0 && lane < (int)C) st_cluster(cluster_addr(&sh.note[1], lane), 1ull);   // lost in rounding
                }
            }
            if (exact && !cuts) break;
            cluster_sync();
            if (cuts) cut = (int)sh.note[0];
            if (exact || sh.note[1] != 1ull) break;
            exact = true;
        }
    }

    // -------------------------------------------------------------- the truncated row
    if (a.out) {
        if (!RES) cluster_sync();                  // nobody reads the row any more: out may be it
        T *out = static_cast<T *>(a.out) + n * a.ldo;
        const bool same = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(row)) & 15) == 0;
        const T dropped = P::raw(a.mask_value);
#pragma unroll 2
        for (int p = tid; p < a.slice; p += ST) {
            const int64_t at = x.position(p) - x.shift;
            if (at >= a.V) break;
            const uint4 r = x.piece(p);
            T e[E];
#pragma unroll
            for (int j = 0; j < E; ++j) e[j] = dropped;
            if (P::max_of(r) >= kept.t) {
                float v[E];
                P::unpack(r, v);
#pragma unroll
                for (int j = 0; j < E; ++j)
                    if (v[j] > kept.t || (v[j] == kept.t && kept.q && at + j <= cut)) e[j] = P::raw(v[j]);
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
    int C, slice, per;
    bool resident;
};

// CTAs of a row's cluster: the fewest that leave two on an SM, more while SMs would be
// idle; the pieces of a CTA and of a thread.
SamplePlan sample_plan(int64_t n, int V, int E, int sms)
{
    const int64_t pieces = ((int64_t)V + E - 1 + E - 1) / E;          // wherever the row starts
    auto slice_of = [&](int C) { return (pieces + C - 1) / C; };
    auto bytes = [&](int C) { return (size_t)slice_of(C) * 16 + HIST_BYTES; };
    int C = 1;
    while (C < MAX_CLUSTER && (bytes(C) > SAMPLE_HALF || (n * C < 2 * sms && slice_of(C) > 2 * ST))) C *= 2;
    const int slice = (int)slice_of(C);
    return {C, slice, ((slice + ST - 1) / ST) | 1, bytes(C) <= SAMPLE_SMEM};
}

template <typename T, bool RES>
int launch_sample(const SampleArgs &a, int64_t n, int C, cudaStream_t st)
{
    static OncePerDevice once;
    XH_CUDA(allow_smem(once, k_sample<T, RES>, SAMPLE_SMEM));
    const size_t smem = (RES ? (size_t)a.slice * 16 : 0) + HIST_BYTES;
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
    a.slice = p.slice;
    a.per = p.per;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (in->dtype == XPRESS_BF16)
        return p.resident ? launch_sample<uint16_t, true>(a, n, p.C, st) : launch_sample<uint16_t, false>(a, n, p.C, st);
    return p.resident ? launch_sample<float, true>(a, n, p.C, st) : launch_sample<float, false>(a, n, p.C, st);
}
