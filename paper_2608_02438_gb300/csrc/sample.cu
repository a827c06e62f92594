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
// A cluster of C CTAs takes a row.  The row is read once, by asynchronous copies into
// the CTAs' shared memory; every further pass over it stays there.  A thread owns
// consecutive 16-byte pieces, an odd number of them: the lanes' accesses then hit
// different banks, and sums per thread, warp and CTA are in the order of the ids.
//   maximum    with it, by bisection, the k/C-th largest of the threads' maxima of
//              each CTA: the smallest is a bound below the k-th largest element
//   the few    where at most 1024 elements are above it, or above min-p's limit, they
//              are gathered in every CTA, which finds the thresholds and draws alone:
//              128 or fewer by comparing each with all (three barriers), more by
//              histograms of them
//   thresholds else by histograms between a lower bound and the maximum: 1024 bins of
//              single bf16 values, or of equal width first and of keys after that,
//              until a bin's largest and smallest elements decide.  By numbers for
//              top-k; by rounded masses for top-p, which the draw's sums confirm or
//              move on from
//   draw       sums per warp, exchanged through the cluster; the warp whose range
//              contains u Z looks for the element
//
// Every decision compares masses: 64-bit fixed-point sums, in which no order of
// additions matters, of weights to 2^-29.8 (weight_exact2).  Their scale first leaves
// room for V weights of 1, and is refined to what the row's mass leaves: a flat tail of
// V weights that each fall below a unit may hold 2^-14 of it.  Sums of a whole row first
// use the hardware's exponential (weight_fast2, a third of the instructions); where a
// decision falls within what that may be off, 2^-21 of the mass, it is taken again with
// exact weights: one row in 200 of a softmax over 15000 likely tokens.
//
// Bound by latency: a row is a chain of some ten passes, barriers and scans.  One row
// of 151936 bf16, top-k 50 and top-p 0.9: 11.2 us (load 1.3, bound 1.0, exchange 1.3,
// the few 5.6, the rest 2.0).  32 x 17 truncated rows of it under mixed filters: 155 us,
// 2.1 TB/s; shared memory holds 76 rows at a time, for 16 us (median) each: with top-k 20
// 126 us for all, 300 178, top-p alone 328.  64 rows without filters: 22.5 to 27 us; 5 of a row's
// 15 are the weights, at the issue limit, and a row that has to be taken again needs 13
// more.  What it took before: one row 19 and 544 rows 443 us with CTAs of two passes per
// level, 64-bit atomics on masses and 64-bit floating point at two lanes a cycle; 15 and
// 201 with histograms for all of the few and a bound from the maxima of groups of lanes
// (266 elements above it, not 68); 64 rows 26.6 with weights of 36 bits behind the point
// before their shift, which 64-bit shifts made.  (Of top-p alone the likely few gathered
// first, as for a top-k of 512: 340 us for 343 where they are enough, 41 for 34 where
// not: left out.)
#include "matmul_fp8.h"

namespace xp {

namespace {

// 2^(j / 64) 2^31, from the exponential's series.
struct ExpTable {
    uint32_t v[64];
};
constexpr ExpTable make_exp_table()
{
    ExpTable t{};
    for (int j = 0; j < 64; ++j) {
        const double x = j * 0.693147180559945309417232 / 64;
        double term = 1.0, sum = 1.0;
        for (int i = 1; i < 24; ++i) { term *= x / i; sum += term; }
        t.v[j] = (uint32_t)(sum * 2147483648.0 + 0.5);
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
    int scale;                     // a weight of 1 is 2^scale until a row's mass is known
    ExpTable table;
};

constexpr int BINS = 1024;                       // of a histogram
constexpr int FEW = BINS;                        // elements that are sorted: as many to a thread as bins
constexpr int ROOM = 61;                         // masses stay below 2^ROOM or little above
constexpr int FEW_SCALE = ROOM - 10;             // a weight of 1 in sums of FEW
constexpr int PAIRS = 128;                       // ... by comparing each with all
constexpr int MAX_CLUSTER = 8;
constexpr int ALL = 0x7fffffff;
constexpr size_t HIST_BYTES = BINS * 16 + FEW * 8;        // counts, masses, largest and smallest key; a CTA's part of the few
constexpr size_t SAMPLE_SMEM = 219 * 1024, SAMPLE_HALF = 105 * 1024;      // pieces and histogram of one, of two CTAs on an SM

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
    static __device__ __forceinline__ float pick(const uint4 &r, int j)
    {
        const uint32_t w = j & 4 ? (j & 2 ? r.w : r.z) : (j & 2 ? r.y : r.x);
        return __uint_as_float(j & 1 ? w & 0xffff0000u : w << 16);
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
    static __device__ __forceinline__ float pick(const uint4 &r, int j)
    {
        return __uint_as_float(j & 2 ? (j & 1 ? r.w : r.z) : (j & 1 ? r.y : r.x));
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
    float floor;                                 // below it weights are under 2^-120
    float rest;                                  // K m's fraction
    uint32_t back;                               // K m's integer, negative, at a float's exponent
    bool near;                                   // K m is small enough for weight_fast's exponents
};
constexpr float MAGIC = 12582912.0f;             // 1.5 2^23: added and taken away, it rounds to an integer

__device__ __forceinline__ Scale make_scale(float m, float T, int bits)
{
    // log2(e) / T to 48 bits: the quotient's rounding comes back through the remainder
    const float t = fminf(fmaxf(T, 1e-37f), 1e37f), kh = 1.44269502f / t;
    const float kl = (fmaf(-kh, t, 1.44269502f) + 1.92596303e-8f) / t;
    const float ph = __fmul_rn(m, kh), pl = fmaf(m, kl, fmaf(m, kh, -ph)), i = __fadd_rn(ph, MAGIC);
    const float reach = 120.0f / kh;
    return Scale{m, kh, kl, bits, m - reach, __fsub_rn(ph, __fsub_rn(i, MAGIC)) + pl, 0u - (__float_as_uint(i) << 23),
                 fabsf(ph) < 5e5f && reach < 1e30f};
}

// Two values at a time.
using f32x2 = unsigned long long;
__device__ __forceinline__ f32x2 pack2(float a, float b)
{
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(f32x2 v, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b)
{
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b)
{
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c)
{
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ f32x2 both(float a) { return pack2(a, a); }
__device__ __forceinline__ f32x2 sub2(f32x2 a, f32x2 b) { return fma2(b, both(-1.0f), a); }

// w = 2^(K (l - m)) as a 64-bit fixed-point number, to 2^-29.8 of its value (and half a
// unit).  The difference and its product with K are kept in two parts; of the
// exponent, the steps of 1/64 come from a table, the rest g (|g| <= 1/128) from the
// series of 2^g - 1, whose fifth term is below 2^-42.
__device__ __forceinline__ void weight_exact2(float l0, float l1, const Scale &s, const uint32_t *table, unsigned long long (&w)[2])
{
    const f32x2 l = pack2(l0, l1), nm = both(-s.m), kh = both(s.kh);
    const f32x2 dh = add2(l, nm), bb = sub2(dh, l), dl = add2(sub2(l, sub2(dh, bb)), sub2(nm, bb));
    float p[2], steps[2], e[2];
    unpack2(mul2(dh, kh), p[0], p[1]);
    p[0] = fmaxf(p[0], -70.0f);                                      // 2^-70 is below half a unit
    p[1] = fmaxf(p[1], -70.0f);
    const f32x2 ph = pack2(p[0], p[1]);
    const f32x2 pl = add2(fma2(dh, kh, mul2(ph, both(-1.0f))), fma2(dh, both(s.kl), mul2(dl, kh)));
    const f32x2 t = fma2(ph, both(64.0f), both(MAGIC));              // its low bits: 64 ph as an integer
    const f32x2 g = add2(fma2(add2(t, both(-MAGIC)), both(-0.015625f), ph), pl);
    unpack2(t, steps[0], steps[1]);
    f32x2 q = fma2(g, both(9.61812910e-3f), both(5.55041087e-2f));
    q = fma2(g, q, both(2.40226507e-1f));
    q = fma2(g, q, both(6.93147181e-1f));
    unpack2(mul2(mul2(g, q), both(8589934592.0f)), e[0], e[1]);      // (2^g - 1) 2^33
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int i = (int)(__float_as_uint(steps[k]) - __float_as_uint(MAGIC));
        const uint32_t tj = table[i & 63];                           // 2^(j / 64) 2^31
        const uint32_t y = tj + (uint32_t)__mulhi((int)(tj >> 1), __float2int_rn(e[k]));         // 31 bits behind the point
        const int up = s.bits - 31 + (i >> 6);                       // 30 at most
        w[k] = up >= 0 ? (unsigned long long)y * (1u << max(up, 0))
                       : (unsigned long long)((__funnelshift_rc(y, 0u, (uint32_t)(-up - 1)) + 1u) >> 1);
    }
    // (both may be infinite)
    if (l0 == s.m) w[0] = 1ull << s.bits;
    if (l1 == s.m) w[1] = 1ull << s.bits;
}
__device__ __forceinline__ unsigned long long weight_exact(float l, const Scale &s, const uint32_t *table)
{
    unsigned long long w[2];
    weight_exact2(l, l, s, table, w);
    return w[0];
}
// The same with the hardware's exponential of the exponent's fraction: 2^-22 off, and
// 2^-24 from the fraction's roundings (K l is split into an integer, its fraction and
// the product's remainder).
__device__ __forceinline__ f32x2 weight_fast2(float l0, float l1, const Scale &s)
{
    if (!s.near)                                   // (a guess: such rows are summed exactly)
        return pack2(ex2_approx(fminf(l0 - s.m, 0.0f) * s.kh), ex2_approx(fminf(l1 - s.m, 0.0f) * s.kh));
    const f32x2 l = pack2(fmaxf(l0, s.floor), fmaxf(l1, s.floor)), kh = both(s.kh);
    const f32x2 ph = mul2(l, kh), i = add2(ph, both(MAGIC)), n = add2(i, both(-MAGIC));
    const f32x2 f = add2(sub2(ph, n), add2(fma2(l, kh, mul2(ph, both(-1.0f))), fma2(l, both(s.kl), both(-s.rest))));
    float f0, f1, i0, i1;
    unpack2(f, f0, f1);
    unpack2(i, i0, i1);
    return pack2(__uint_as_float(__float_as_uint(ex2_approx(f0)) + (__float_as_uint(i0) << 23) + s.back),
                 __uint_as_float(__float_as_uint(ex2_approx(f1)) + (__float_as_uint(i1) << 23) + s.back));
}
__device__ __forceinline__ float weight_fast(float l, const Scale &s)
{
    float a, b;
    unpack2(weight_fast2(l, l, s), a, b);
    return a;
}
// What fast weights may be off, and a sum of them by its own roundings (three levels
// of 2^-24 each), in 2^-26 of their size, a tenth added; and by fixed-point roundings.
constexpr float SLACK_W = 24.0f, SLACK_SUM = 14.0f, SLACK = SLACK_W + SLACK_SUM;
constexpr unsigned long long SLACK_UNITS = 8192;
// 2^-26 of z, as a float.
__device__ __forceinline__ float part_of(unsigned long long z) { return (float)(uint32_t)(z >> 32) * 64.0f; }

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
__device__ __forceinline__ void ld_cluster(uint32_t addr, uint32_t (&v)[4])
{
    asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ld_cluster(uint32_t addr, uint32_t (&v)[2])
{
    asm volatile("ld.shared::cluster.v2.u32 {%0, %1}, [%2];" : "=r"(v[0]), "=r"(v[1]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t ld_cluster1(uint32_t addr)
{
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void cluster_sync() { cluster_arrive(); cluster_wait(); }

template <int SWARPS> struct SampleShared {
    uint32_t table[64];                                              // 2^(j / 64) 2^31
    unsigned long long slot[2][3][MAX_CLUSTER * SWARPS];             // what the cluster's warps exchange: [turn][value][warp]
    unsigned long long scan[2][SWARPS];
    unsigned long long note[4];                                      // written by one thread of the cluster: the id cut, a draw to repeat
    float shift_hi, shift_lo;                                        // T ln(min_p)
    unsigned long long before, mass;                                 // of the bin that was looked for
    uint32_t bin, count, largest, smallest;
    int base[MAX_CLUSTER + 1];                                       // where the CTAs' parts of the few begin
};

// z f, rounded down, and whether anything was lost; 0 <= f < 1.
__device__ __forceinline__ unsigned long long scaled(unsigned long long z, float f, bool &more)
{
    const uint32_t bits = __float_as_uint(f), e = bits >> 23;
    const unsigned long long mant = e ? (bits & 0x7fffffu) | 0x800000u : bits & 0x7fffffu;
    const int s = 150 - (int)max(e, 1u);                             // f = mant 2^-s, s >= 24
    const unsigned long long hi = __umul64hi(z, mant), lo = z * mant;
    if (s < 64) {
        more = lo << (64 - s) != 0;
        return hi << (64 - s) | lo >> s;
    }
    const int t = min(s - 64, 63);
    more = lo != 0 || (hi & ((1ull << t) - 1)) != 0;
    return hi >> t;
}
// The mass that top-p's kept tokens have to reach: at least one unit, so that one is kept.
__device__ __forceinline__ unsigned long long goal_of(unsigned long long z, float p)
{
    bool more;
    const unsigned long long g = scaled(z, p, more);
    return max(g + more, 1ull);
}

// What a kernel's passes share.
template <typename T, bool RES, int ST>
struct Sampler {
    using P = Piece<T>;
    using F = Piece<float>;
    static constexpr int E = P::E, SWARPS = ST / 32;
    static constexpr int NB = BINS / ST;         // bins of a thread
    static constexpr int NS = MAX_CLUSTER * SWARPS / 32;             // warps whose exchanged values a lane looks at
    const SampleArgs &a;
    SampleShared<SWARPS> &sh;
    uint4 *pieces;                 // [slice] of this CTA (RES)
    uint32_t *hist;                // [4][BINS]: counts, masses, largest and smallest key
    const T *row;                  // the row's first element
    int shift;                     // elements from a 16-byte boundary to it
    int C, rank, turn;
    bool open;                     // other CTAs may still read this one's histogram
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
        open = false;
    }
    // What the warp NS lane + i exchanged (0 past the last one).
    __device__ __forceinline__ unsigned long long slot_of(int which, int i) const
    {
        const int w = NS * (threadIdx.x % 32) + i;
        return w < C * SWARPS ? sh.slot[turn][which][w] : 0;
    }
    // The sum, and the largest low word, of what the warps exchanged.
    __device__ unsigned long long exchanged_sum(int which) const
    {
        unsigned long long v = 0;
#pragma unroll
        for (int i = 0; i < NS; ++i) v += slot_of(which, i);
        return warp_sum(v);
    }
    __device__ uint32_t exchanged_max(int which) const
    {
        uint32_t v = 0;
#pragma unroll
        for (int i = 0; i < NS; ++i) v = max(v, (uint32_t)slot_of(which, i));
        return __reduce_max_sync(0xffffffffu, v);
    }
    // A finer scale for sums that are no more than z, where z leaves room: by how many bits.
    __device__ __forceinline__ int refine(unsigned long long z)
    {
        const int up = max(0, __clzll(z) - (64 - ROOM));
        s.bits += up;
        return up;
    }
    // ... for sums of elements from t up, from an estimate (2^-12 off).
    __device__ void refine_from(float t)
    {
        float z = 0.0f;
        for (int i = 0; i < count(first()); ++i) {
            const uint4 r = piece(first() + i);
            if (P::max_of(r) < t) continue;
            float v[E];
            P::unpack(r, v);
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (v[j] >= t) z += weight_fast(v[j], s);
        }
        exchange(warp_sum(__float2ull_rn(z * __uint_as_float((uint32_t)(127 + s.bits) << 23))), 0);
        refine(exchanged_sum(0));
    }
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
        best = exchanged_max(0);
        return above ? ~best : best;
    }
    // Exclusive sum over the CTA's threads.
    __device__ unsigned long long block_scan(unsigned long long v, int which)
    {
        const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
        const unsigned long long in = warp_scan(v);
        if (lane == 31) sh.scan[which][warp] = in;
        __syncthreads();
        return warp_sum(lane < warp ? sh.scan[which][lane] : 0ull) + in - v;
    }

    // Sum over the CTA's threads.
    __device__ unsigned long long block_sum(unsigned long long v, int which)
    {
        v = warp_sum(v);
        if (threadIdx.x % 32 == 0) sh.scan[which][threadIdx.x / 32] = v;
        __syncthreads();
        return warp_sum(threadIdx.x % 32 < SWARPS ? sh.scan[which][threadIdx.x % 32] : 0ull);
    }

    // The elements from t up, of the whole row and in the order of the ids, up to NB to
    // each thread of every CTA: their order's word above the id, 0 past the last one.  Their
    // number; above FEW nothing is done.
    __device__ int gather(float t, unsigned long long (&e)[NB])
    {
        const int tid = threadIdx.x, lane = tid % 32, n = count(first());
        uint2 *list = reinterpret_cast<uint2 *>(hist + 4 * BINS);
        uint32_t c = 0, some = 0;                                    // elements, and the pieces that have them
#pragma unroll 2
        for (int i = 0; i < n; ++i) {
            const uint4 r = piece(first() + i);
            if (P::max_of(r) < t) continue;
            some |= 1u << (i & 31);
            float v[E];
            P::unpack(r, v);
#pragma unroll
            for (int j = 0; j < E; ++j) c += v[j] >= t;
        }
        uint32_t at = (uint32_t)block_scan(c, 0);
        for (int i = 0; c && at < FEW && i < n; ++i) {
            if (!(some >> (i & 31) & 1u)) continue;
            float v[E];
            P::unpack(piece(first() + i), v);
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (v[j] >= t) {
                    if (at < FEW) list[at] = make_uint2(order_of(v[j]), (uint32_t)(position(first() + i) + j - shift));
                    ++at;
                }
        }
        exchange(warp_sum(c), 0);
        uint32_t mine = 0;
#pragma unroll
        for (int i = 0; i < NS; ++i) mine += (uint32_t)slot_of(0, i);
        const uint32_t to = warp_scan(mine);                         // (SWARPS / NS = 4 lanes to a CTA)
        const int total = (int)__shfl_sync(0xffffffffu, to, 31);
        if (total > FEW) return total;
        if (tid < 32 && lane % 4 == 0) sh.base[lane / 4] = (int)(to - mine);
        if (tid == 0) sh.base[MAX_CLUSTER] = total;
        __syncthreads();
        const int each = (total + ST - 1) / ST;
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const int k = each * tid + i;
            e[i] = 0;
            if (i < each && k < total) {
                int r = 0;
#pragma unroll
                for (int c = 1; c < MAX_CLUSTER; ++c) r += k >= sh.base[c];
                uint32_t x[2];
                ld_cluster(cluster_addr(list + (k - sh.base[r]), r), x);
                e[i] = (unsigned long long)x[0] << 32 | x[1];
            }
        }
        open = true;
        return total;
    }
    static __device__ __forceinline__ uint32_t word_of(unsigned long long e) { return (uint32_t)(e >> 32); }
    static __device__ __forceinline__ float value_of(unsigned long long e) { return Piece<float>::value((uint32_t)(e >> 32)); }

    // Of gathered elements with words from klo to khi, each worth x (0: out of it), from
    // the largest down: the word at which their sum reaches `target`, and of the elements
    // with it the one that does, counted from 1.  False: none does.  By levels of this
    // CTA's histogram of worths (numbers, where they are 1; so too where a bin has one
    // value, times its weight: 64-bit sums take the place of many), largest and smallest
    // words.
    template <bool MASS>
    __device__ bool select(const unsigned long long (&e)[NB], const unsigned long long (&x)[NB], uint32_t klo, uint32_t khi,
                           unsigned long long target, uint32_t &word, uint32_t &which)
    {
        const int tid = threadIdx.x;
        constexpr bool COUNT = !MASS || P::KEY_SHIFT > 0;
        unsigned long long *worth = reinterpret_cast<unsigned long long *>(hist);
        for (;;) {
            constexpr int LOG = 10;
            const int n = 32 - __clz(khi - klo), bits = n > LOG ? n - LOG : 0;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i * ST + tid < BINS) {
                    if (COUNT) hist[i * ST + tid] = 0;
                    else worth[i * ST + tid] = 0;
                    hist[2 * BINS + i * ST + tid] = 0;
                    hist[3 * BINS + i * ST + tid] = ~0u;
                }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < NB; ++i)
                if (x[i] && word_of(e[i]) >= klo && word_of(e[i]) <= khi) {
                    const uint32_t at = (khi - word_of(e[i])) >> bits;
                    if (COUNT) atomicAdd(hist + at, 1u);
                    else atomicAdd(worth + at, x[i]);
                    atomicMax(hist + 2 * BINS + at, word_of(e[i]));
                    atomicMin(hist + 3 * BINS + at, word_of(e[i]));
                }
            __syncthreads();
            unsigned long long w[NB];
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const int at = NB * tid + i;
                if (!COUNT) w[i] = worth[at];
                else if (!MASS) w[i] = hist[at];
                else if (bits <= P::KEY_SHIFT) w[i] = hist[at] ? hist[at] * weight_exact(F::value(hist[2 * BINS + at]), s, sh.table) : 0;
                else w[i] = 0;
            }
            if (MASS && COUNT && bits > P::KEY_SHIFT) {
                // (a range of more than ten octaves) the sums themselves
                __syncthreads();
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i * ST + tid < BINS) worth[i * ST + tid] = 0;
                __syncthreads();
#pragma unroll
                for (int i = 0; i < NB; ++i)
                    if (x[i] && word_of(e[i]) >= klo && word_of(e[i]) <= khi) atomicAdd(worth + ((khi - word_of(e[i])) >> bits), x[i]);
                __syncthreads();
#pragma unroll
                for (int i = 0; i < NB; ++i) w[i] = worth[NB * tid + i];
            }
            if (!find_bin(w, target, 0, false)) return false;
            const uint32_t bin = sh.bin, big = hist[2 * BINS + bin], small = hist[3 * BINS + bin];
            target -= sh.before;
            if (big == small) {
                word = big;
                // equal elements are worth the same
                unsigned long long each = 0;
#pragma unroll
                for (int i = 0; i < NB; ++i)
                    if (x[i] && word_of(e[i]) == big) each = x[i];
                if (each) sh.mass = each;
                __syncthreads();
                each = sh.mass;
                which = (uint32_t)((target + each - 1) / each);
                return true;
            }
            klo = small;
            khi = big;
            __syncthreads();
        }
    }

    // Exact weights of a piece's elements above t0, two at a time (a warp goes on until
    // its fullest piece is done): what exceeds t to `sum`, all of it to `sum0` (BOTH).
    template <bool BOTH>
    __device__ __forceinline__ void add_exact(const uint4 &r, float t, float t0, unsigned long long &sum, uint32_t &ties,
                                              unsigned long long &sum0, uint32_t &ties0) const
    {
        float v[E];
        P::unpack(r, v);
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            m |= v[j] > (BOTH ? t0 : t) ? 1u << j : 0u;
            ties += v[j] == t;
            if (BOTH) ties0 += v[j] == t0;
        }
        while (m) {
            const int j0 = __ffs(m) - 1;
            m &= m - 1;
            const int j1 = m ? __ffs(m) - 1 : -1;
            m &= m - 1;
            const float a = P::pick(r, j0), b = P::pick(r, j1);
            unsigned long long w[2];
            weight_exact2(a, b, s, sh.table, w);
            if (j1 < 0) w[1] = 0;
            sum += (!BOTH || a > t ? w[0] : 0ull) + (!BOTH || b > t ? w[1] : 0ull);
            if (BOTH) sum0 += w[0] + w[1];
        }
    }
    // Sum of the weights of l > t and number of l == t in n pieces from p of this CTA
    // (fast weights: of every element; t is -inf).
    __device__ void sums(bool exact, int p, int n, float t, unsigned long long &sum, uint32_t &ties) const
    {
        sum = 0;
        ties = 0;
        if (exact) {
            unsigned long long none = 0;
            uint32_t none0 = 0;
#pragma unroll 1
            for (int i = 0; i < n; ++i) {
                const uint4 r = piece(p + i);
                if (t == -INFINITY) {                                // (by pieces' places: 29.4 us for 26.5)
                    float v[E];
                    P::unpack(r, v);
#pragma unroll
                    for (int j = 0; j < E; j += 2) {
                        unsigned long long w[2];
                        weight_exact2(v[j], v[j + 1], s, sh.table, w);
                        sum += w[0] + w[1];
                    }
                } else if (P::max_of(r) >= t) {
                    add_exact<false>(r, t, t, sum, ties, none, none0);
                }
            }
            return;
        }
        float hi = 0.0f, lo = 0.0f;
#pragma unroll 2
        for (int i = 0; i < n; ++i) {
            float v[E];
            P::unpack(piece(p + i), v);
            f32x2 w[E / 2];
#pragma unroll
            for (int j = 0; j < E; j += 2) w[j / 2] = weight_fast2(v[j], v[j + 1], s);
#pragma unroll
            for (int o = E / 4; o > 0; o >>= 1)
#pragma unroll
                for (int j = 0; j < o; ++j) w[j] = add2(w[j], w[j + o]);
            float a, c;
            unpack2(w[0], a, c);
            a += c;
            // hi + lo keeps what the addition rounds away
            const float x = __fadd_rn(hi, a), b = __fsub_rn(x, hi);
            lo += __fadd_rn(__fsub_rn(hi, __fsub_rn(x, b)), __fsub_rn(a, b));
            hi = x;
        }
        const float one = __uint_as_float((uint32_t)(127 + s.bits) << 23);
        sum = __float2ull_rn(hi * one) + (unsigned long long)__float2ll_rn(lo * one);
    }
    // sums() of this thread's pieces with exact weights for t, and for a lower t0 beside it.
    __device__ void sums_two(float t, float t0, unsigned long long &sum, uint32_t &ties, unsigned long long &sum0, uint32_t &ties0) const
    {
        sum = sum0 = 0;
        ties = ties0 = 0;
        const int n = count(first());
#pragma unroll 1
        for (int i = 0; i < n; ++i) {
            const uint4 r = piece(first() + i);
            if (P::max_of(r) >= t0) add_exact<true>(r, t, t0, sum, ties, sum0, ties0);
        }
    }

    // Histogram of the elements from lo up whose keys are at most khi, from the largest
    // down, by bins of equal width 1 / inv (inv > 0) or of 2^bits keys: their number, and
    // where a bin may have several keys (bits > 0) the largest and the smallest, and
    // (MASS) their mass times `unit`, rounded.  Each thread gets NB of the masses, or of
    // the numbers, summed over the cluster.
    template <bool MASS>
    __device__ void histogram(float lo, uint32_t khi, int bits, float inv, float unit, uint32_t (&b)[NB])
    {
        const int tid = threadIdx.x, n = count(first());
        const bool keys = bits > 0;
        if (open) cluster_sync();
        for (int i = tid; i < BINS / 4; i += ST) {
            reinterpret_cast<uint4 *>(hist)[i] = make_uint4(0, 0, 0, 0);
            if (keys) {
                if (MASS) reinterpret_cast<uint4 *>(hist + BINS)[i] = make_uint4(0, 0, 0, 0);
                reinterpret_cast<uint4 *>(hist + 2 * BINS)[i] = make_uint4(0, 0, 0, 0);
                reinterpret_cast<uint4 *>(hist + 3 * BINS)[i] = make_uint4(~0u, ~0u, ~0u, ~0u);
            }
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
        open = true;
        uint32_t x[MAX_CLUSTER][NB];
        const uint32_t *from = hist + (MASS && keys ? BINS : 0) + NB * tid;
#pragma unroll
        for (int r = 0; r < MAX_CLUSTER; ++r)
            if (r < C) ld_cluster(cluster_addr(from, r), x[r]);
#pragma unroll
        for (int k = 0; k < NB; ++k) {
            b[k] = 0;
#pragma unroll
            for (int r = 0; r < MAX_CLUSTER; ++r)
                if (r < C) b[k] += x[r][k];
        }
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
    // The first bin at which the sum of x reaches `target`, and what is known of it
    // (keys: its number of elements, largest and smallest key).  False: none does.
    __device__ bool find_bin(const unsigned long long (&x)[NB], unsigned long long target, int which, bool keys)
    {
        const int tid = threadIdx.x;
        if (tid == 0) sh.bin = BINS;
        unsigned long long mine = 0;
#pragma unroll
        for (int k = 0; k < NB; ++k) mine += x[k];
        unsigned long long at = block_scan(mine, which);             // its barrier comes before the writing
#pragma unroll
        for (int k = 0; k < NB; ++k) {
            if (at < target && target <= at + x[k]) {
                sh.bin = NB * tid + k;
                sh.before = at;
                sh.mass = x[k];
            }
            at += x[k];
        }
        __syncthreads();
        const uint32_t bin = sh.bin;
        if (bin == BINS) return false;
        if (keys) {
            if (tid < 32) {
                uint32_t c = 0, big = 0, small = ~0u;
                if (tid < C) {
                    c = ld_cluster1(cluster_addr(hist + bin, tid));
                    big = ld_cluster1(cluster_addr(hist + 2 * BINS + bin, tid));
                    small = ld_cluster1(cluster_addr(hist + 3 * BINS + bin, tid));
                }
                c = __reduce_add_sync(0xffffffffu, c);
                big = __reduce_max_sync(0xffffffffu, big);
                small = __reduce_min_sync(0xffffffffu, small);
                if (tid == 0) { sh.count = c; sh.largest = big; sh.smallest = small; }
            }
            __syncthreads();
        }
        return true;
    }
};

// What a row keeps: l > t, and the first q with l == t.
struct Kept {
    float t;
    int q;
};

// grid: a cluster of C CTAs for each row; ST threads; pieces, then the histogram.
template <typename T, bool RES, int ST>
__global__ void __launch_bounds__(ST, 1024 / ST) k_sample(const __grid_constant__ SampleArgs a)
{
    using S = Sampler<T, RES, ST>;
    using P = Piece<T>;
    using F = Piece<float>;
    constexpr int E = P::E, KS = P::KEY_SHIFT, SWARPS = ST / 32, NB = S::NB, NS = S::NS;
    extern __shared__ __align__(16) uint8_t dyn[];
    __shared__ SampleShared<SWARPS> sh;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    uint32_t C;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(C));
    const int64_t n = blockIdx.x / C;
    const int q_seq = (int)(n / a.rows);
    const T *row = static_cast<const T *>(a.in) + n * a.ld;
    S x{a, sh, reinterpret_cast<uint4 *>(dyn), reinterpret_cast<uint32_t *>(dyn + (RES ? (size_t)a.slice * 16 : 0)), row,
        (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T)), (int)C, (int)cluster_rank(), 0, false, Scale{}};
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
        if (tid == 0 && min_p > 0.0f) {
            const double d = (double)temp * log(fmin((double)min_p, 1.0));
            sh.shift_hi = (float)d;
            sh.shift_lo = (float)(d - (double)sh.shift_hi);
        }
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
        if (tid == 0 && min_p > 0.0f) {
            const double d = (double)temp * log(fmin((double)min_p, 1.0));
            sh.shift_hi = (float)d;
            sh.shift_lo = (float)(d - (double)sh.shift_hi);
        }
#pragma unroll 4
        for (int p = tid; p < a.slice; p += ST) mx = fmaxf(mx, P::max_of(x.fetch(p)));
    }
    // The r-th largest of the threads' maxima, r of C for top_k: the smallest of the CTAs'
    // bounds the top_k-th largest element from below, with about a third more above it.
    // (To 16 bits; two bits a barrier, counted in shared memory: 12.2 us a row, 11.2 so.)
    const uint32_t key = order_of(mx);
    const int r_k = (top_k + (int)C - 1) / (int)C, of = min(ST, a.slice);
    uint32_t bound = 0;
    if (top_k > 1 && r_k <= of)
        for (int bit = 31; bit >= 16; --bit)
            if (__syncthreads_count(key >= (bound | 1u << bit)) >= r_k) bound |= 1u << bit;
    cluster_wait();
    x.exchange(__reduce_max_sync(0xffffffffu, key), (uint32_t)~bound);
    const uint32_t kmax = x.exchanged_max(0), kbound = ~x.exchanged_max(1);

    Kept kept{-INFINITY, 0};
    // The truncated row; cut: the last id with l == t that is kept.  (Pieces below the
    // first bound written as soon as it is known: 226 us for 544 rows, 209 without.)
    auto write_out = [&](int cut) {
        T *out = static_cast<T *>(a.out) + n * a.ldo;
        const bool same = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(row)) & 15) == 0;
        const T dropped = P::raw(a.mask_value);
#pragma unroll 4
        for (int p = tid; p < a.slice; p += ST) {
            const int64_t at = ids0 + (int64_t)p * E;
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
    };
    const bool empty = kmax < LOWEST;
    bool k_on = false, p_on = false, check_p = false, settled = false;
    int cut = ALL;
    bool one = false;                              // the first maximum alone is kept
    unsigned long long z1 = 0;                     // mass of what min-p and top-k keep
    bool z1_exact = false;
    Kept first{-INFINITY, 0};                      // ... as a threshold
    // Sums are off by half a unit for each of their elements.  Whether the first scale
    // keeps that below 2^-31 of the mass (which is 1 at least, and min_p for each of them);
    // else a pass over them comes first (64 rows of 151936, top-k 20000: 109 us, 96 without).
    const uint32_t many = 1u << (a.scale - 30);
    const bool coarse = kmax == order_of(INFINITY) || (uint32_t)a.V <= many || (top_k > 0 && (uint32_t)top_k <= many) ||
                        min_p * (float)many >= 1.0f;
    if (!empty) {
        const float m = F::value(kmax);
        x.s = make_scale(m, temp, a.scale);
        const uint32_t top = kmax >> KS;
        float low = -3.402823466e38f;              // the lowest value that may be kept
        if (m == INFINITY) low = INFINITY;         // the limit: the infinities share all the mass
        else if (min_p > 0.0f) {
            // the smallest value that is not below m + T ln(min_p)
            const float hi = sh.shift_hi, sum = __fadd_rn(m, hi), bb = __fsub_rn(sum, m);
            const float rest = __fadd_rn(__fsub_rn(m, __fsub_rn(sum, bb)), __fsub_rn(hi, bb)) + sh.shift_lo;
            low = fmaxf(rest > 0.0f ? nextafterf(sum, INFINITY) : sum, low);
        }
        if (low > -3.402823466e38f) kept = {low, ALL};
        if (!(temp > 0.0f) || top_k == 1 || top_p <= 0.0f || min_p > 1.0f) {          // (no weight is above 1)
            kept = {m, 1};
            one = true;
        } else if (m == INFINITY) {
            // equal weights: the first top_k, and top-p's share of their number
            if (top_k > 0) kept.q = top_k;
            check_p = top_p < 1.0f;
        } else {
            k_on = top_k > 0 && top_k < a.V;
            p_on = top_p < 1.0f;
        }
        uint32_t b[NB];
        unsigned long long wide[NB];
        // All of it where few elements, those from t up, can be kept.  False if there are
        // too many.
        auto settle = [&](float t, int k) {
            unsigned long long e[NB];
            const int total = x.gather(t, e);
            if (total > FEW) return false;
            x.s.bits = FEW_SCALE;
            if (total <= PAIRS) {
                // every one against every other: how many stand before it, and their mass
                settled = true;
                if (!a.out && x.rank > 0) return true;
                ulonglong2 *all = reinterpret_cast<ulonglong2 *>(x.hist);
                const unsigned long long mine = e[0] ^ 0xffffffffull, w = tid < total ? weight_exact(S::value_of(e[0]), x.s, sh.table) : 0;
                if (tid < total) all[tid] = make_ulonglong2(mine, w);
                __syncthreads();
                int place = 0;
                unsigned long long before = 0;
                if (tid < total) {
#pragma unroll 4
                    for (int i = 0; i < total; ++i) {
                        const ulonglong2 o = all[i];
                        place += o.x > mine;
                        before += o.x > mine ? o.y : 0ull;
                    }
                }
                const int of_k = min(total, k) - 1;
                if (tid < total && place == of_k) sh.mass = before + w;
                __syncthreads();
                const unsigned long long goal = p_on ? goal_of(sh.mass, top_p) : ~0ull;
                const bool keep = tid < total && place <= of_k && before < goal;
                if (keep && (place == of_k || before + w >= goal)) sh.note[2] = e[0];     // the last one
                const unsigned long long at = x.block_scan(keep ? w : 0ull, 0);
                kept = {S::value_of(sh.note[2]), 1};
                cut = (int)(uint32_t)sh.note[2];
                if (a.tokens && x.rank == 0) {
                    const unsigned long long z = warp_sum(tid % 32 < S::SWARPS ? sh.scan[0][tid % 32] : 0ull);
                    bool more;
                    const unsigned long long draw = u < 1.0f ? min(scaled(z, u, more), z - 1) : z - 1;
                    if (keep && at <= draw && draw < at + w) a.tokens[n] = (int)(uint32_t)e[0];
                }
                return true;
            }
            uint32_t last = max(order_of(low), order_of(t)), q = ALL;  // kept: words above last, and the first q of those equal to it
            if (total > k) {
#pragma unroll
                for (int i = 0; i < NB; ++i) wide[i] = S::word_of(e[i]) >= last;
                x.template select<false>(e, wide, last, kmax, k, last, q);             // (false: fewer than k)
            }
            // the ties' places, as long as only some of them are kept
            uint32_t tie = 0;
            auto worth = [&]() {
                uint32_t at = 0;
                if (q < ALL) {
                    uint32_t ties = 0;
#pragma unroll
                    for (int i = 0; i < NB; ++i) ties += S::word_of(e[i]) == last;
                    __syncthreads();
                    at = tie = (uint32_t)x.block_scan(ties, 1);
                }
#pragma unroll
                for (int i = 0; i < NB; ++i) {
                    const bool equal = S::word_of(e[i]) == last;
                    const bool keep = S::word_of(e[i]) > last || (equal && at < q);
                    at += equal;
                    wide[i] = keep && e[i] ? weight_exact(S::value_of(e[i]), x.s, sh.table) : 0;
                }
            };
            if (p_on) {
                worth();
                unsigned long long mine = 0;
#pragma unroll
                for (int i = 0; i < NB; ++i) mine += wide[i];
                __syncthreads();
                z1 = x.block_sum(mine, 0);
                __syncthreads();
                uint32_t word, which;
                if (x.template select<true>(e, wide, last, kmax, goal_of(z1, top_p), word, which)) { last = word; q = which; }
            }
            kept = {F::value(last), 1};
            settled = true;
            worth();
            if (q < ALL) {
                // the id of the last tie that is kept
                if (tid == 0) sh.note[2] = (unsigned long long)ALL;
                __syncthreads();
#pragma unroll
                for (int i = 0; i < NB; ++i)
                    if (S::word_of(e[i]) == last && ++tie == q) sh.note[2] = (uint32_t)e[i];
                __syncthreads();
                cut = (int)sh.note[2];
            }
            if (a.tokens && x.rank == 0) {
                unsigned long long mine = 0;
#pragma unroll
                for (int i = 0; i < NB; ++i) mine += wide[i];
                const unsigned long long z = x.block_sum(mine, 0);
                bool more;
                const unsigned long long goal = u < 1.0f ? min(scaled(z, u, more), z - 1) : z - 1;
                __syncthreads();
                unsigned long long at = x.block_scan(mine, 1);
#pragma unroll
                for (int i = 0; i < NB; ++i) {
                    if (at <= goal && goal < at + wide[i]) a.tokens[n] = (int)(uint32_t)e[i];
                    at += wide[i];
                }
            }
            return true;
        };
        const float lo_k = kbound >= LOWEST ? fmaxf(low, F::value(kbound)) : low;
        if (one) {
            settle(m, 1);
        } else if (m < INFINITY && (min_p > 0.0f || (k_on && kbound >= LOWEST && top_k <= FEW / 2 && 2 * r_k <= of))) {
            if (settle(k_on ? lo_k : low, k_on ? top_k : ALL)) k_on = p_on = false;
        }
        // ------------------------------------------------------------ top-k
        if (k_on) {
            float lo = lo_k;
            uint32_t klo = order_of(lo) >> KS, khi = top, left = top_k;
            for (int level = 0; k_on; ++level) {
                const int bits = S::level_bits(klo, khi);
                x.template histogram<false>(lo, khi, bits, level == 0 && bits ? x.bins_per(lo) : 0.0f, 0.0f, b);
#pragma unroll
                for (int i = 0; i < NB; ++i) wide[i] = b[i];
                const bool found = x.find_bin(wide, left, level & 1, bits > 0);
                if (!found) break;                                    // fewer than k
                if (level == 0 && (bits ? sh.count : sh.mass) + sh.before <= FEW) {
                    const float t = bits ? P::value(sh.smallest) : P::value(khi - sh.bin);
                    __syncthreads();
                    settle(t, top_k);
                    p_on = false;
                    break;
                }
                left -= (uint32_t)sh.before;
                if (bits == 0) {
                    kept = {P::value(khi - sh.bin), (int)left};
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
            z1_exact = kept.t > -INFINITY || !x.s.near;
            if (z1_exact && !coarse) x.refine_from(kept.t);
            x.sums(z1_exact, x.first(), x.count(x.first()), kept.t, sum, ties);
            x.exchange(warp_sum(sum), warp_sum(ties));
            z1 = x.exchanged_sum(0);
            const unsigned long long nt = min(x.exchanged_sum(1), (unsigned long long)kept.q);
            if (nt) z1 += nt * weight_exact(kept.t, x.s, sh.table);
            unsigned long long units = SLACK_UNITS;
            if (!z1_exact) {
                const int up = x.refine(z1);
                z1 <<= up;
                units <<= up;
            }
            const unsigned long long target = goal_of(z1, top_p);
            // only the target is off: its masses are exact
            const unsigned long long slack = z1_exact ? 0 : (unsigned long long)(part_of(z1) * (SLACK * top_p)) + units;
            const int down = max(0, 33 - __clzll(z1));                // z1 >> down has 31 bits
            const float unit = __uint_as_float((uint32_t)(127 + x.s.bits - down) << 23);
            // what may be left out has at most 1 - top_p of the mass
            float lo = fmaxf(low, kept.t);
            {
                const float share = (1.0f - top_p) * ((float)z1 * __uint_as_float((uint32_t)(127 - x.s.bits) << 23)) / (float)a.V;
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
                    for (int i = 0; i < NB; ++i)
                        wide[i] = b[i] ? b[i] * weight_exact(P::value(khi - (NB * tid + i)), x.s, sh.table) : 0;
                    found = x.find_bin(wide, sure ? left : max(left, 1ull) << down, level & 1, false);
                } else {
                    sure = false;
#pragma unroll
                    for (int i = 0; i < NB; ++i) wide[i] = b[i];
                    found = x.find_bin(wide, max(left, 1ull), level & 1, true);
                }
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
                        const unsigned long long each = weight_exact(kept.t, x.s, sh.table), need = (left + each - 1) / each;
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
    bool written = false;
    if (empty) {
        if (tid == 0 && x.rank == 0 && a.tokens) a.tokens[n] = -1;
        kept = {INFINITY, 0};
    } else if (!settled && (a.tokens || check_p || (a.out && kept.q < ALL && kept.q > 0))) {
        // (fast weights for whole rows only: with the checks by exact ones at once, a third
        // form of the sums and its slack are gone from the code; 5 to 8 % everywhere)
        bool exact = kept.t > -INFINITY || !x.s.near;
        if (exact && !coarse && !one && !p_on) x.refine_from(kept.t);
        // while t is not sure: what is known of its key, from below and above
        uint32_t known_lo = max(order_of(first.t), LOWEST) >> KS, known_hi = kmax >> KS;
        int moves = 0;
        for (;;) {
            const float t = kept.t;
            unsigned long long sum;
            uint32_t ties;
            if (check_p && !z1_exact) {
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
            // each lane takes NS consecutive warps: their ties, then their kept mass
            uint32_t wn[NS], nb[NS], n_sum = 0;
            unsigned long long wm[NS];
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                nb[i] = n_sum;                                       // ties before, from the lane's first warp
                n_sum += wn[i] = (uint32_t)x.slot_of(1, i);
                wm[i] = x.slot_of(0, i);
            }
            const uint32_t n_in = warp_scan(n_sum);
#pragma unroll
            for (int i = 0; i < NS; ++i) nb[i] += n_in - n_sum;
            const uint32_t all_ties = __shfl_sync(0xffffffffu, n_in, 31);
            const unsigned long long wt = all_ties ? weight_exact(t, x.s, sh.table) : 0;
            if (check_p) {
                // is t where the mass before reaches the target?  How many of its ties?
                const unsigned long long above = x.exchanged_sum(0);
                const uint32_t may = t == first.t ? min(all_ties, (uint32_t)first.q) : all_ties;
                const unsigned long long target = goal_of(z1, top_p);
                // above - top_p z1, with the same weights in both where both are fast
                const bool small = above >= target, large = above + may * wt < target && t > first.t;
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
                kept.q = (int)need;
                check_p = false;
            }
            const uint32_t q = (uint32_t)kept.q;
            unsigned long long m_sum = 0, mb[NS];
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                mb[i] = m_sum;
                m_sum += wm[i] += (min(nb[i] + wn[i], q) - min(nb[i], q)) * wt;
            }
            const unsigned long long m_in = warp_scan(m_sum);
            const unsigned long long z = __shfl_sync(0xffffffffu, m_in, 31);
#pragma unroll
            for (int i = 0; i < NS; ++i) mb[i] += m_in - m_sum;
            const bool cuts = a.out && q && q < all_ties;
            const int me = x.rank * SWARPS + warp;
            if (cuts) {
                // the q-th of the ties
                int who = -1;
                uint32_t there = 0;
#pragma unroll
                for (int i = 0; i < NS; ++i)
                    if (nb[i] < q && q <= nb[i] + wn[i]) { who = NS * lane + i; there = nb[i]; }
                const int src = __ffs(__ballot_sync(0xffffffffu, who >= 0)) - 1;
                who = __shfl_sync(0xffffffffu, who, src);
                there = __shfl_sync(0xffffffffu, there, src);
                if (who == me) {
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
                bool more;
                const unsigned long long goal = u < 1.0f ? min(scaled(z, u, more), z - 1) : z - 1;
                int who = -1;
                unsigned long long there = 0, mine = sum;
                uint32_t there_n = 0, my_ties = ties;
#pragma unroll
                for (int i = 0; i < NS; ++i)
                    if (mb[i] <= goal && goal < mb[i] + wm[i]) { who = NS * lane + i; there = mb[i]; there_n = nb[i]; }
                const int src = __ffs(__ballot_sync(0xffffffffu, who >= 0)) - 1;
                who = __shfl_sync(0xffffffffu, who, src);
                if (who == me) {
                    // the lane, then the piece, then the element
                    there = __shfl_sync(0xffffffffu, there, src);
                    there_n = __shfl_sync(0xffffffffu, there_n, src);
                    int p = 0;
                    bool ok = true;
                    unsigned long long slack = 0;
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
                                    // the sums before the lane less u of all, with the same weights in both; and
                                    // the lane's own, which are looked at once more
                                    if (step == 0 && !exact)
                                        slack = (unsigned long long)(SLACK * (part_of(z) * (2.0f * u * (1.0f - u)) +
                                                                              part_of(__shfl_sync(0xffffffffu, own, l)))) + SLACK_UNITS;
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
            cluster_arrive();
            if (RES && a.out && !cuts) {           // while the draw goes on
                write_out(cut);
                written = true;
            }
            cluster_wait();
            if (cuts) cut = (int)sh.note[0];
            if (exact || sh.note[1] != 1ull) break;
            exact = true;
            x.refine(z);
        }
    }
    if (!RES && a.out) cluster_sync();             // nobody reads the row any more: out may be it

    if (a.out && !written) write_out(cut);
    if (x.open) cluster_sync();                    // others may still read the histogram
}

struct SamplePlan {
    int C, threads, slice, per;
    bool resident;
};

// CTAs of a row's cluster: the fewest that leave two on an SM; more while they have
// more than 2048 pieces and all rows' CTAs have a place at the same time (64 rows of
// 151936 bf16: 4 CTAs, 27 us, 31 with 2; 68 rows of 32000: 2 CTAs, 12.4 us, 13.7 with
// one, 11.4 with 4).  8 for a few rows only (one row 11.2 us, 12.1 with 4; 17 rows 14.3
// with 4, 15.9 with 8).  The pieces of a CTA and of a thread.
SamplePlan sample_plan(int64_t n, int V, int E, int sms)
{
    const int64_t pieces = ((int64_t)V + E - 1 + E - 1) / E;          // wherever the row starts
    auto slice_of = [&](int C) { return (pieces + C - 1) / C; };
    auto threads_of = [&](int C) { return slice_of(C) > 1024 ? 512 : 256; };
    auto bytes = [&](int C) { return (size_t)slice_of(C) * 16 + HIST_BYTES; };
    auto fits = [&](int C) { return n * C * threads_of(C) <= (int64_t)sms * 1024 && (C < 8 || n * C <= sms / 2); };
    int C = 1;
    while (C < MAX_CLUSTER && (bytes(C) > SAMPLE_HALF || (fits(2 * C) && slice_of(C) > 2048))) C *= 2;
    const int slice = (int)slice_of(C);
    const bool resident = bytes(C) <= SAMPLE_SMEM;
    const int threads = resident ? threads_of(C) : 512;
    return {C, threads, slice, ((slice + threads - 1) / threads) | 1, resident};
}

template <typename T, bool RES, int ST>
int launch_sample(const SampleArgs &a, int64_t n, int C, cudaStream_t st)
{
    static OncePerDevice once;
    XH_CUDA(allow_smem(once, k_sample<T, RES, ST>, SAMPLE_SMEM));
    const size_t smem = (RES ? (size_t)a.slice * 16 : 0) + HIST_BYTES;
    XH_CUDA(launch_head(k_sample<T, RES, ST>, dim3((unsigned)(n * C)), ST, smem, st, (unsigned)C, a));
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
    if (in->out == in->logits && in->ldo != in->ld && n > 1) return XPRESS_ERR_INVALID_ARG;
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
    const SamplePlan p = sample_plan(n, in->V, (int)(16 / es), sms);
    a.slice = p.slice;
    a.per = p.per;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (in->dtype == XPRESS_BF16)
        return !p.resident ? launch_sample<uint16_t, false, 512>(a, n, p.C, st)
               : p.threads == 512 ? launch_sample<uint16_t, true, 512>(a, n, p.C, st)
                                  : launch_sample<uint16_t, true, 256>(a, n, p.C, st);
    return !p.resident ? launch_sample<float, false, 512>(a, n, p.C, st)
           : p.threads == 512 ? launch_sample<float, true, 512>(a, n, p.C, st)
                              : launch_sample<float, true, 256>(a, n, p.C, st);
}
