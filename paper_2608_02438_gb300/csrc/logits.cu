// logits.cu -- the request's rules on logits rows, in one pass over them, with
// the first maximum of the row that results (Algorithm 1's seed Y^(0) when the
// rows are the base logits).  For row j of sequence q and token v, with c the
// times v was answered (the history after the prompt, and the block's tokens
// 0 .. j - 1) and seen = c > 0 or v in the prompt:
//   l <- l > 0 ? l / rep : l * rep        if seen
//   l <- l - freq c - pres [c > 0]
//   l <- l + bias_v
//   l <- mask_value                       if the row's grammar mask forbids v
// in 32 bits, each operation rounded on its own (no fused multiply-add, so
// that the result does not depend on the compiler), one rounding to the
// storage type at the end.
//
// A CTA takes a share of the vocabulary for the rows of one sequence: every
// G-th segment of 256 ids, so that the frequent tokens, which vocabularies keep
// together, are spread over the CTAs.  Ids with a count or a bias are few, and
// their arithmetic (a division among it) would run in nearly every warp if it
// sat in the stream of the rows, so the work is split:
//   counts  the history's tokens that fall into the share, in shared memory
//           (every CTA of a sequence reads the whole history, from L2), and a
//           list of the ids that have a count, a bias or a place in the block
//   stream  rows in 16-byte pieces, each read while the one before it is worked
//           on: the mask, the copy and the packed maximum of the ids that are
//           not listed; listed ids pass unchanged
//   patch   after every 4 rows, while they are in L2, their listed ids, read
//           once more and rewritten, with their own maximum (after all rows of a
//           large batch they would come from and go to HBM, 32 bytes each)
// Each warp leaves its argmax keys; a second kernel takes the largest of a
// row's.  (The last CTA of a sequence doing that took longer: 8.7 us against 6.8
// for one row of one request, 118 against 113 for the batch below.)
//
// 32 x 17 rows of 151936 bf16 (histories of 3000 to 6000, half of the rows
// masked): 112 us, 3.0 TB/s; without rules 62 us, 5.3 TB/s.  No unit is saturated (53 %
// of the issue slots, 33 % of HBM): with two CTAs of eight warps on an SM the
// latencies of dependent instructions show, 2.1 of the 7.2 cycles from one of a
// warp's instructions to its next, loads 0.9 and shared memory 0.8.  The patch is about a
// third.  One row of one request: 6.9 us, bound by the chain offsets - history -
// counts - row - second kernel.
#include "head.h"

namespace xp {

namespace {

struct LogitsArgs {
    const void *in;
    void *out;
    int64_t ld, ldo;
    int rows, V;
    int rows_each;                 // rows of a CTA
    const float *rep, *freq, *pres;
    const int32_t *hist;
    int64_t n_hist;
    const int64_t *hist_off;
    const int32_t *prompt_len;
    const int32_t *draft;
    int64_t ld_draft;
    const int32_t *bias_ids;
    const float *bias_val;
    int64_t n_bias;
    const int64_t *bias_off;
    const int32_t *mask;
    int64_t ld_mask;
    int mask_rows;
    const int32_t *mask_row;
    float mask_value;
    int patch;                     // a rule on single ids is given
    uint32_t magic;                // ceil(2^32 / gridDim.x)
    unsigned long long *part;      // [n_seq * rows][gridDim.x][8, with patch NT / 32 more] argmax keys (0: none), or NULL
};

constexpr int LT = 256;            // threads: 8 warps
constexpr int64_t MAX_ENTRIES = 1 << 30;     // of history (its counts stay below it) and bias
constexpr int MAX_V = 1 << 24;     // so that Share's division by multiplication is exact ((V / 256) (V / 2048) < 2^32)
constexpr int LWARPS = LT / 32;
constexpr uint32_t IN_PROMPT = 1u << 31, IN_BLOCK = 1u << 30, TIMES = IN_BLOCK - 1;   // of a count

// The first n elements of r to p, 16-byte aligned.
__device__ __forceinline__ void store_raw(uint16_t *p, int n, const Raw8<uint16_t> &r)
{
    if (n >= 8) { *reinterpret_cast<uint4 *>(p) = r.a; return; }
    const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < n) p[j] = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
}
__device__ __forceinline__ void store_raw(float *p, int n, const Raw8<float> &r)
{
    if (n >= 8) {
        *reinterpret_cast<float4 *>(p) = r.a;
        *reinterpret_cast<float4 *>(p + 4) = r.b;
        return;
    }
    float v[8];
    unpack(r, v);
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < n) p[j] = v[j];
}

// The warp's 256 elements, 8 of each lane, to p, where n of them have a place: by
// way of shared memory, so that the lanes store consecutive elements (each its
// own 8, they would write every 32-byte sector 8 times or more).
template <typename T>
__device__ __forceinline__ void store_turned(T *p, int n, const Raw8<T> &r, Raw8<T> *turn)
{
    const int lane = threadIdx.x % 32;
    turn[lane] = r;
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (k * 32 + lane < n) p[k * 32 + lane] = reinterpret_cast<const T *>(turn)[k * 32 + lane];
    __syncwarp();
}

// Word masks of the 8 bf16 elements of a piece for every byte of bits (bit k:
// element k), in shared memory: a byte expands by one load.
__device__ __forceinline__ void fill_masks(uint4 *masks, int b)
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (b >> (2 * i) & 1 ? 0xffffu : 0u) | (b >> (2 * i + 1) & 1 ? 0xffff0000u : 0u);
    masks[b] = make_uint4(w[0], w[1], w[2], w[3]);
}
// The elements of r whose bit in `keep` is clear become `other`.
__device__ __forceinline__ void select8(Raw8<uint16_t> &r, uint32_t keep, float other, const uint4 *masks)
{
    const uint32_t o = f2bf(other), oo = o | o << 16;
    const uint4 m = masks[keep];
    r.a.x = (r.a.x & m.x) | (oo & ~m.x);
    r.a.y = (r.a.y & m.y) | (oo & ~m.y);
    r.a.z = (r.a.z & m.z) | (oo & ~m.z);
    r.a.w = (r.a.w & m.w) | (oo & ~m.w);
}
__device__ __forceinline__ void select8(Raw8<float> &r, uint32_t keep, float other, const uint4 *)
{
    float *v = reinterpret_cast<float *>(&r);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (keep >> i & 1u) ? v[i] : other;
}
// The largest element, NaNs apart.
__device__ __forceinline__ float max8(const Raw8<uint16_t> &r)
{
    const __nv_bfloat162 *p = reinterpret_cast<const __nv_bfloat162 *>(&r.a);
    const __nv_bfloat162 m = __hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3]));
    return fmaxf(__low2float(m), __high2float(m));
}
__device__ __forceinline__ float max8(const Raw8<float> &r)
{
    return fmaxf(fmaxf(fmaxf(r.a.x, r.a.y), fmaxf(r.a.z, r.a.w)), fmaxf(fmaxf(r.b.x, r.b.y), fmaxf(r.b.z, r.b.w)));
}

// The order-preserving word of argmax_key, -0 as 0.
__device__ __forceinline__ uint32_t order_word(float v)
{
    const uint32_t b = __float_as_uint(v + 0.0f);
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
// The warp's argmax key: the lanes' largest `top` words, the smallest id among them.
__device__ __forceinline__ unsigned long long warp_key(uint32_t mine, uint32_t top, uint32_t id)
{
    id = __reduce_min_sync(0xffffffffu, mine == top ? id : 0xffffffffu);
    return id == 0xffffffffu ? 0ull : ((unsigned long long)top << 32) | (0xffffffffu - id);
}

// Sequence q's entries o0 .. o0 + n - 1 of an array of `total` < 2^31 (offsets cut to it).
__device__ __forceinline__ void range_of(const int64_t *off, int q, int64_t total, int64_t &o0, int &n)
{
    o0 = min(max(off[q], (int64_t)0), total);
    n = (int)max(min(off[q + 1], total) - o0, (int64_t)0);
}

// Where a CTA of G keeps its ids: id SEG (G i + blockIdx.x) + r is its element
// SEG i + r.
constexpr int SEG_BITS = 8, SEG = 1 << SEG_BITS;
struct Share {
    uint32_t G, blk, magic;
    __device__ __forceinline__ int id(int at) const
    {
        return (int)((((uint32_t)at >> SEG_BITS) * G + blk) << SEG_BITS | (at & (SEG - 1)));
    }
    // the element of id t, or a number of no element of any share
    __device__ __forceinline__ uint32_t at(int t) const
    {
        // (negative ids end up past every share's elements)
        const uint32_t seg = (uint32_t)t >> SEG_BITS, i = G == 1 ? seg : __umulhi(seg, magic);
        return i * G + blk == seg ? i << SEG_BITS | (t & (SEG - 1)) : 0xffffffffu;
    }
};

// Counts one history token.
__device__ __forceinline__ void count_token(uint32_t *cnt, const Share &sh, int size, int t, bool prompt)
{
    const uint32_t i = sh.at(t);
    if (i < (uint32_t)size) {
        if (prompt) atomicOr(cnt + i, IN_PROMPT);
        else atomicAdd(cnt + i, 1u);
    }
}

// CTAs of LT threads that an SM takes.  The next row's pieces want registers:
// three CTAs for several rows of fp32 by two slots (510 rows of 151936: 154 us with
// four, 135 with three) or element by element (136 rows of 55191: 37 and 24), four
// where these suffice (225 rows of 25984 fp32: 20 us, 26 with three; 340 rows of
// 55192 bf16: 45 and 56).
constexpr int ctas_per_sm(bool f32, bool vec, int U, bool multi)
{
    return !multi ? 4 : U == 4 ? 2 : f32 && (U == 2 || !vec) ? 3 : 4;
}

// grid (shares of 2048 U ids, sequences, parts of the rows); shared memory with
// patch: counts [C], with a bias as many floats, the list [C] (16 bits).
// MULTI: several rows of a CTA.  NT: LT threads, or more, of which those past LT
// count and patch only.
template <typename T, bool VEC, int U, bool MULTI, int NT>
__global__ void __launch_bounds__(NT, NT > LT ? 1 : ctas_per_sm(sizeof(T) == 4, VEC, U, MULTI)) k_logits(const __grid_constant__ LogitsArgs a)
{
    constexpr int C = LT * 8 * U;
    constexpr int PR = MULTI ? 4 : 1;              // rows patched together
    __shared__ int listed;
    __shared__ uint4 masks[sizeof(T) == 2 ? 256 : 1];
    __shared__ Raw8<T> turn[VEC ? 1 : LT];
    extern __shared__ __align__(16) uint32_t cnt[];            // [C]: IN_PROMPT | IN_BLOCK | times answered
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const int q = blockIdx.y, V = a.V, R = a.rows;
    const int jb = blockIdx.z * a.rows_each, je = min(jb + a.rows_each, R);     // this CTA's rows
    const Share sh{gridDim.x, blockIdx.x, a.magic};
    const bool streams = NT == LT || tid < LT;
    const bool has_bias = a.bias_ids != nullptr;
    uint32_t *bias = cnt + C;                      // [C]: the bias as fp32 bits (while being built: entry + 1)
    uint16_t *list = reinterpret_cast<uint16_t *>(has_bias ? bias + C : bias);
    if (a.part) pdl_trigger();                     // k_logits_argmax may start and wait
    if (tid == 0) listed = 0;
    if (sizeof(T) == 2 && tid < 256) fill_masks(masks, tid);
    __syncthreads();
    if (a.patch) {
        for (int i = tid; i < C / 4; i += NT) reinterpret_cast<uint4 *>(cnt)[i] = make_uint4(0, 0, 0, 0);
        if (has_bias)
            for (int i = tid; i < C / 4; i += NT) reinterpret_cast<uint4 *>(bias)[i] = make_uint4(0, 0, 0, 0);
    }
    pdl_wait();

    const int64_t n0 = (int64_t)q * R;
    const T *in = static_cast<const T *>(a.in) + n0 * a.ld;
    T *out = a.out ? static_cast<T *>(a.out) + n0 * a.ldo : nullptr;
    const bool in_place = a.out == a.in && a.ld == a.ldo;
    // slot u of a thread that streams: its elements 2048 u + 8 tid + 0 .. 7, with the ids
    // id0 + u id_step + 0 .. 7; their bits are 8 u + k
    const int id0 = sh.id(tid * 8), id_step = LT * 8 * (int)gridDim.x;
    uint32_t inside = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int n = min(max(V - id0 - u * id_step, 0), 8);
        inside |= ((1u << n) - 1u) << (8 * u);
    }

    float rep = 1.0f, freq = 0.0f, pres = 0.0f;
    int64_t b0 = 0;
    uint32_t special = 0;
    if (a.patch) {
        // all that does not depend on one another is asked for at once
        int64_t o0 = 0;
        int n = 0, bn = 0, plen = 0;
        if (a.hist) range_of(a.hist_off, q, a.n_hist, o0, n);
        if (a.hist && a.prompt_len) plen = a.prompt_len[q];
        if (has_bias) range_of(a.bias_off, q, a.n_bias, b0, bn);
        if (a.rep) rep = a.rep[q];
        if (a.freq) freq = a.freq[q];
        if (a.pres) pres = a.pres[q];
        const int32_t *h = a.hist + o0;
        const int head = min((int)((16 - (reinterpret_cast<uintptr_t>(h) & 15)) & 15) / 4, n);
        const int4 *h4 = reinterpret_cast<const int4 *>(h + head);
        const int n4 = (n - head) / 4;
        constexpr int UN = 4;
        auto fetch = [&](int i0, int4 (&t)[UN]) {
#pragma unroll
            for (int u = 0; u < UN; ++u) t[u] = i0 + u * NT < n4 ? h4[i0 + u * NT] : make_int4(-1, -1, -1, -1);
        };
        int4 nt[UN];
        fetch(tid, nt);
        const bool penal = rep != 1.0f || freq != 0.0f || pres != 0.0f;
        __syncthreads();
        if (penal) {
            if (tid < head) count_token(cnt, sh, C, h[tid], tid < plen);
            for (int i0 = tid; i0 < n4; i0 += UN * NT) {
                int4 t[UN];
#pragma unroll
                for (int u = 0; u < UN; ++u) t[u] = nt[u];
                fetch(i0 + UN * NT, nt);           // under way while this piece is counted
#pragma unroll
                for (int u = 0; u < UN; ++u) {
                    const int p = head + 4 * (i0 + u * NT);
                    count_token(cnt, sh, C, t[u].x, p < plen);
                    count_token(cnt, sh, C, t[u].y, p + 1 < plen);
                    count_token(cnt, sh, C, t[u].z, p + 2 < plen);
                    count_token(cnt, sh, C, t[u].w, p + 3 < plen);
                }
            }
            const int tail = head + 4 * n4 + tid;
            if (tid < 4 && tail < n) count_token(cnt, sh, C, h[tail], tail < plen);
            if (a.draft)
                for (int i = tid; i < R - 1; i += NT) {
                    const uint32_t k = sh.at(a.draft[q * a.ld_draft + i]);
                    if (k < (uint32_t)C) atomicOr(cnt + k, IN_BLOCK);
                }
        }
        // of several bias entries for one id the last one counts
        for (int i = tid; i < bn; i += NT) {
            const uint32_t k = sh.at(a.bias_ids[b0 + i]);
            if (k < (uint32_t)C) atomicMax(bias + k, (uint32_t)i + 1);
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!streams) break;
            const int s = u * LT * 8 + tid * 8;
            const uint4 lo = *reinterpret_cast<const uint4 *>(cnt + s), hi = *reinterpret_cast<const uint4 *>(cnt + s + 4);
            const uint32_t c[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (c[k]) special |= 1u << (8 * u + k);
            if (has_bias) {
                const uint4 bl = *reinterpret_cast<const uint4 *>(bias + s), bh = *reinterpret_cast<const uint4 *>(bias + s + 4);
                const uint32_t e[8] = {bl.x, bl.y, bl.z, bl.w, bh.x, bh.y, bh.z, bh.w};
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (e[k]) {
                        bias[s + k] = __float_as_uint(a.bias_val[b0 + e[k] - 1]);
                        special |= 1u << (8 * u + k);
                    }
            }
        }
        special &= inside;
        if (special) {
            int at = atomicAdd(&listed, __popc(special));
            for (uint32_t b = special; b; b &= b - 1) {
                const int i = __ffs(b) - 1;
                list[at++] = (uint16_t)(i / 8 * LT * 8 + tid * 8 + i % 8);
            }
        }
    }

    const int slots = LWARPS + a.patch * (NT / 32);
    unsigned long long *part = a.part ? a.part + (n0 * gridDim.x + blockIdx.x) * slots + warp : nullptr;
    auto mask_of = [&](int j) -> const uint8_t * {
        if (!a.mask || j >= je) return nullptr;
        const int64_t mr = a.mask_row ? (int64_t)a.mask_row[n0 + j] : n0 + j;
        return mr >= 0 && mr < a.mask_rows ? reinterpret_cast<const uint8_t *>(a.mask + mr * a.ld_mask) : nullptr;
    };
    auto fetch_row = [&](int j, Raw8<T> (&x)[U]) {
        if (j >= je) return;
        const T *row = in + (int64_t)j * a.ld;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int id = id0 + u * id_step;
            if (id < V) x[u] = load_raw<VEC>(row + id, V - id);
        }
    };
    // bytes of a row's mask, as they are stored: arithmetic on them here would
    // wait for them here
    auto fetch_bits = [&](const uint8_t *mask, uint32_t (&bits)[U]) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int id = id0 + u * id_step;
            if (mask && id < V) bits[u] = mask[id / 8];
        }
    };

    Raw8<T> nx[U];
    uint32_t nbits[U];
    const uint8_t *mask = nullptr, *mask1 = mask_of(jb), *mask2 = MULTI ? mask_of(jb + 1) : nullptr;   // of rows j, j + 1, j + 2
    if (streams) {
        fetch_bits(mask1, nbits);
        fetch_row(jb, nx);
    }
    const uint8_t *pmask = nullptr;                // of the row that this thread patches
    for (int j = jb; j < je; ++j) {
        const int in_group = (j - jb) % PR;
        if (a.patch && in_group == 0) pmask = mask_of(j + tid % PR);
        if (streams) {
            struct { Raw8<T> x[U]; } cur;
            uint32_t bits[U];
#pragma unroll
            for (int u = 0; u < U; ++u) { cur.x[u] = nx[u]; bits[u] = nbits[u]; }
            mask = mask1;
            mask1 = mask2;
            if (MULTI) {
                mask2 = mask_of(j + 2);
                fetch_bits(mask1, nbits);
                fetch_row(j + 1, nx);
            }
            T *orow = out + (int64_t)j * a.ldo;
            uint32_t allow = 0xffffffffu;
            if (mask) {
                allow = 0;
#pragma unroll
                for (int u = 0; u < U; ++u) allow |= bits[u] << (8 * u);
            }
            const uint32_t use = allow & inside & ~special;
            float mx[U], m = -INFINITY;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int id = id0 + u * id_step;
                mx[u] = -INFINITY;
                const int seg = id - lane * 8;     // the warp's first id
                if ((VEC ? id : seg) >= V) continue;
                const uint32_t keep = (allow | special) >> (8 * u) & 0xffu;
                if (keep != 0xffu) select8(cur.x[u], keep, a.mask_value, masks);
                const bool moves = out && !(in_place && keep == 0xffu);
                if (VEC) {
                    if (moves) store_raw(orow + id, V - id, cur.x[u]);
                } else if (__any_sync(0xffffffffu, moves)) {
                    store_turned(orow + seg, V - seg, cur.x[u], turn + warp * 32);
                }
                if (part) {
                    const uint32_t us = use >> (8 * u) & 0xffu;
                    Raw8<T> y = cur.x[u];
                    if (us != 0xffu) select8(y, us, -INFINITY, masks);
                    mx[u] = max8(y);
                    m = fmaxf(m, mx[u]);
                }
            }
            if (part) {
                const uint32_t mine = order_word(m), top = __reduce_max_sync(0xffffffffu, mine);
                uint32_t id = 0xffffffffu;
                if (mine == top) {
#pragma unroll
                    for (int u = U - 1; u >= 0; --u)
                        if (mx[u] == m) {
                            float v[8];
                            unpack(cur.x[u], v);
#pragma unroll
                            for (int k = 7; k >= 0; --k)
                                if ((use >> (8 * u + k) & 1u) && v[k] == m) id = id0 + u * id_step + k;
                        }
                }
                const unsigned long long key = warp_key(mine, top, id);
                if (lane == 0) part[(int64_t)j * gridDim.x * slots] = key;
            }
        }
        if (a.patch && (in_group == PR - 1 || j == je - 1)) {
            __syncthreads();                       // the list, and the rows as they were copied
            const int j0 = j - in_group, jr = j0 + tid % PR, n = jr <= j ? listed : 0;
            const T *row = in + (int64_t)jr * a.ld;
            uint32_t word = 0, pid = 0xffffffffu;
            constexpr int EU = 4, ES = NT / PR;    // ids in flight, threads of a row
            for (int e0 = tid / PR; e0 < n; e0 += EU * ES) {
                T raw[EU];
                uint32_t mb[EU];
                int at[EU];
#pragma unroll
                for (int i = 0; i < EU; ++i) {
                    const int e = e0 + i * ES;
                    at[i] = list[e < n ? e : e0];
                    const int v = sh.id(at[i]);
                    raw[i] = row[v];
                    mb[i] = pmask ? pmask[v / 8] : 0xffu;
                }
#pragma unroll
                for (int i = 0; i < EU; ++i) {
                    if (e0 + i * ES >= n) continue;
                    const int v = sh.id(at[i]);
                    const bool ok = mb[i] >> (v % 8) & 1u;
                    const uint32_t c = cnt[at[i]];
                    uint32_t times = c & TIMES;
                    if (c & IN_BLOCK)
                        for (int t = 0; t < jr; ++t) times += a.draft[q * a.ld_draft + t] == v;
                    float y = load1(&raw[i]);
                    if (times || (c & IN_PROMPT)) y = y > 0.0f ? __fdiv_rn(y, rep) : __fmul_rn(y, rep);
                    if (times) y = __fsub_rn(__fsub_rn(y, __fmul_rn(freq, (float)times)), pres);
                    if (has_bias) y = __fadd_rn(y, __uint_as_float(bias[at[i]]));
                    if (!ok) y = a.mask_value;
                    if (sizeof(T) == 2) y = bf2f(f2bf(y));
                    if (out) store1(out + (int64_t)jr * a.ldo + v, y);
                    if (ok && y == y) {
                        const uint32_t w = order_word(y);
                        if (w > word || (w == word && (uint32_t)v < pid)) { word = w; pid = v; }
                    }
                }
            }
            if (part)
#pragma unroll
                for (int r = 0; r < PR; ++r) {
                    const bool mine = tid % PR == r;
                    const uint32_t w = mine ? word : 0, top = __reduce_max_sync(0xffffffffu, w);
                    const unsigned long long key = warp_key(w, top, mine ? pid : 0xffffffffu);
                    if (lane == 0 && j0 + r <= j) part[(int64_t)(j0 + r) * gridDim.x * slots + LWARPS] = key;
                }
        }
        if (!MULTI) break;
    }
}

// grid: rows; 256 threads: the largest of a row's n keys.
__global__ void __launch_bounds__(256) k_logits_argmax(const unsigned long long *part, int n, int32_t *argmax)
{
    __shared__ unsigned long long best_of[8];
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x % 32;
    pdl_wait();
    unsigned long long best = 0;
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += 256) best = max(best, part[row * n + i]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
    if (lane == 0) best_of[threadIdx.x / 32] = best;
    __syncthreads();
    if (threadIdx.x >= 32) return;
    best = best_of[lane % 8];
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
    if (lane == 0) {
        float v;
        int id = -1;
        if (best) argmax_unkey(best, v, id);
        argmax[row] = id;
    }
}

constexpr int LT_FEW = 512;        // threads of a CTA that has an SM for itself and a long history

struct LogitsPlan {
    int U, threads, rows_each;
};

// Slots per thread: shares of 2048, 4096 or 8192 ids, the largest that still
// gives every SM four CTAs.
int logits_slots(int n_seq, int V, int sms)
{
    int U = 4;
    while (U > 1 && (int64_t)n_seq * ((V + LT * 8 * U - 1) / (LT * 8 * U)) < 4 * sms) U /= 2;
    return U;
}

// Few CTAs: a sequence's rows are split over as many as the SMs hold at a time
// (17 rows of 10000 bf16, 3 requests: 11.7 us with parts of 4 rows, 8.8 with one
// row each).  Each part counts the history for itself, so that from 4096 tokens
// on there are two per SM (16 rows of 32000, 4 requests of 8000 tokens: 18 us,
// 22 with four).  Where not even every SM gets one and histories are longer yet,
// a CTA takes 512 threads for the counts and the patch (6 sequences of 30000
// tokens, V = 32003, 5 rows: 32 -> 21 us; a short history gains nothing), and
// there is one per SM (17 rows of 5000, one request of 20000 tokens: 11 us, 43
// with all rows in one CTA).
LogitsPlan logits_plan(const LogitsArgs &a, int n_seq, bool f32, bool vec, int sms)
{
    LogitsPlan p{logits_slots(n_seq, a.V, sms), LT, a.rows};
    const int64_t ctas = (int64_t)n_seq * ((a.V + LT * 8 - 1) / (LT * 8));
    if (p.U != 1) return p;
    const int64_t each = a.patch ? a.n_hist / n_seq : 0;
    if (ctas <= sms && each >= 8192) p.threads = LT_FEW;
    const int64_t room = (int64_t)sms * (p.threads == LT_FEW ? 1 : each >= 4096 ? 2 : ctas_per_sm(f32, vec, 1, true));
    const int64_t parts = room > ctas ? room / ctas : 1;
    p.rows_each = (int)((a.rows + parts - 1) / parts);
    return p;
}

template <typename T, bool VEC, int U, bool MULTI, int NT>
cudaError_t launch_logits_u(LogitsArgs a, int n_seq, cudaStream_t st)
{
    constexpr int C = LT * 8 * U;
    static OncePerDevice once;
    const cudaError_t attr = allow_smem(once, k_logits<T, VEC, U, MULTI, NT>, C * 10);
    if (attr != cudaSuccess) return attr;
    const size_t smem = a.patch ? (size_t)C * (a.bias_ids ? 10 : 6) : 0;
    const unsigned G = (a.V + C - 1) / C;
    a.magic = (uint32_t)(((1ull << 32) + G - 1) / G);
    return launch_head(k_logits<T, VEC, U, MULTI, NT>, dim3(G, n_seq, (a.rows + a.rows_each - 1) / a.rows_each), NT, smem, st, 1, a);
}

template <typename T, bool VEC, bool MULTI>
cudaError_t launch_logits_r(const LogitsArgs &a, int n_seq, const LogitsPlan &p, cudaStream_t st)
{
    return p.threads == LT_FEW ? launch_logits_u<T, VEC, 1, MULTI, LT_FEW>(a, n_seq, st)
         : p.U == 1 ? launch_logits_u<T, VEC, 1, MULTI, LT>(a, n_seq, st)
         : p.U == 2 ? launch_logits_u<T, VEC, 2, MULTI, LT>(a, n_seq, st)
                    : launch_logits_u<T, VEC, 4, MULTI, LT>(a, n_seq, st);
}

template <typename T, bool VEC>
cudaError_t launch_logits(const LogitsArgs &a, int n_seq, const LogitsPlan &p, cudaStream_t st)
{
    return a.rows_each > 1 ? launch_logits_r<T, VEC, true>(a, n_seq, p, st) : launch_logits_r<T, VEC, false>(a, n_seq, p, st);
}

}  // namespace
}  // namespace xp

using namespace xp;

extern "C" size_t xpress_process_logits_workspace_size(int n_seq, int rows, int V)
{
    if (n_seq < 1 || rows < 1 || V < 1) return 0;
    const int sms = current_sms(), C = LT * 8 * (sms > 0 ? logits_slots(n_seq, V, sms) : 1);
    return (size_t)n_seq * rows * ((V - 1) / C + 1) * (LWARPS + LT_FEW / 32) * 8;
}

extern "C" int xpress_process_logits(const xpress_logits_args *in, void *ws, size_t ws_bytes, void *stream)
{
    if (!in || in->n_seq < 0 || in->rows < 1 || in->V < 1 || !in->logits || (!in->out && !in->argmax) ||
        in->ld < in->V || (in->out && in->ldo < in->V))
        return XPRESS_ERR_INVALID_ARG;
    if ((in->dtype != XPRESS_F32 && in->dtype != XPRESS_BF16) || in->n_seq > 65535 || in->V > MAX_V ||
        (int64_t)in->n_seq * in->rows > 0x7fffffff || in->n_history >= MAX_ENTRIES || in->n_bias > MAX_ENTRIES)
        return XPRESS_ERR_UNSUPPORTED;
    if ((in->history && (!in->history_offsets || in->n_history < 0)) ||
        (in->bias_ids && (!in->bias_values || !in->bias_offsets || in->n_bias < 0)) ||
        (in->draft && in->ld_draft < in->rows - 1) ||
        (in->mask && (in->mask_rows < 0 || in->ld_mask < (in->V + 31) / 32)))
        return XPRESS_ERR_INVALID_ARG;
    const uintptr_t es = in->dtype == XPRESS_BF16 ? 2 : 4;
    if (!aligned(in->logits, es) || !aligned(in->out, es) || !aligned(in->argmax, 4) || !aligned(in->repetition, 4) ||
        !aligned(in->frequency, 4) || !aligned(in->presence, 4) || !aligned(in->history, 4) ||
        !aligned(in->history_offsets, 8) || !aligned(in->prompt_len, 4) || !aligned(in->draft, 4) ||
        !aligned(in->bias_ids, 4) || !aligned(in->bias_values, 4) || !aligned(in->bias_offsets, 8) ||
        !aligned(in->mask, 4) || !aligned(in->mask_row, 4))
        return XPRESS_ERR_INVALID_ARG;
    if (in->n_seq == 0) return XPRESS_OK;
    if (in->argmax && (!ws || !aligned(ws, 256) ||
                       ws_bytes < xpress_process_logits_workspace_size(in->n_seq, in->rows, in->V)))
        return XPRESS_ERR_WORKSPACE;
    const int sms = current_sms();
    if (sms < 1) return XPRESS_ERR_CUDA;
    LogitsArgs a{};
    a.in = in->logits; a.out = in->out; a.ld = in->ld; a.ldo = in->ldo;
    a.rows = in->rows; a.V = in->V;
    a.rep = in->repetition; a.freq = in->frequency; a.pres = in->presence;
    a.hist = in->history; a.n_hist = in->n_history; a.hist_off = in->history_offsets; a.prompt_len = in->prompt_len;
    a.draft = in->draft; a.ld_draft = in->ld_draft;
    a.bias_ids = in->bias_ids; a.bias_val = in->bias_values; a.n_bias = in->n_bias; a.bias_off = in->bias_offsets;
    a.mask = in->mask; a.ld_mask = in->ld_mask; a.mask_rows = in->mask_rows; a.mask_row = in->mask_row;
    a.mask_value = in->mask_value;
    a.patch = in->repetition || in->frequency || in->presence || in->bias_ids;
    a.part = in->argmax ? static_cast<unsigned long long *>(ws) : nullptr;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool vec = aligned(in->logits, 16) && in->ld * es % 16 == 0 &&
                     (!in->out || (aligned(in->out, 16) && in->ldo * es % 16 == 0));
    const LogitsPlan plan = logits_plan(a, in->n_seq, in->dtype == XPRESS_F32, vec, sms);
    a.rows_each = plan.rows_each;
    XH_CUDA(in->dtype == XPRESS_BF16
                ? (vec ? launch_logits<uint16_t, true>(a, in->n_seq, plan, st)
                       : launch_logits<uint16_t, false>(a, in->n_seq, plan, st))
                : (vec ? launch_logits<float, true>(a, in->n_seq, plan, st)
                       : launch_logits<float, false>(a, in->n_seq, plan, st)));
    if (in->argmax) {
        const int C = LT * 8 * plan.U, n = (in->V + C - 1) / C * (LWARPS + a.patch * (plan.threads / 32));
        XH_CUDA(launch_head(k_logits_argmax, dim3((unsigned)(in->n_seq * in->rows)), 256, 0, st, 1,
                            (const unsigned long long *)ws, n, in->argmax));
    }
    return XPRESS_OK;
}
