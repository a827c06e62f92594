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
// A CTA takes a range of the vocabulary for all rows of one sequence.  It
// counts the history's tokens that fall into its range in shared memory (every
// CTA of a sequence reads the whole history, from L2), then streams the rows.
// A thread owns the same ids in every row, so the block's tokens are added to
// the counts by their owners without a barrier, and a register holds one bit
// per owned id that has a count or a bias: the others pass through untouched.
// HBM bound for many rows (each logit read and written once); for one row
// bound by the latency of offsets -> history -> counts.
#include "head.h"

namespace xp {

namespace {

struct LogitsArgs {
    const void *in;
    void *out;
    int64_t ld, ldo;
    int rows, V;
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
    unsigned long long *part;      // [n_seq * rows][8 gridDim.x] argmax keys (0: none), or NULL
};

constexpr int LT = 256;            // threads: 8 warps
constexpr int LWARPS = LT / 32;
constexpr uint32_t IN_PROMPT = 1u << 31;

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
__device__ __forceinline__ Raw8<uint16_t> repack(const float (&v)[8], uint16_t)
{
    return {make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]))};
}
__device__ __forceinline__ Raw8<float> repack(const float (&v)[8], float)
{
    return {make_float4(v[0], v[1], v[2], v[3]), make_float4(v[4], v[5], v[6], v[7])};
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
template <bool VEC>
__device__ __forceinline__ void store_raw(uint16_t *p, int n, const Raw8<uint16_t> &r)
{
    if (VEC && n >= 8) { *reinterpret_cast<uint4 *>(p) = r.a; return; }
    const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < n) p[j] = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
}
template <bool VEC>
__device__ __forceinline__ void store_raw(float *p, int n, const Raw8<float> &r)
{
    if (VEC && n >= 8) {
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

// Sequence q's entries o0 .. o0 + n - 1 of an array of `total` (offsets cut to it).
__device__ __forceinline__ void range_of(const int64_t *off, int q, int64_t total, int64_t &o0, int64_t &n)
{
    o0 = min(max(off[q], (int64_t)0), total);
    n = max(min(off[q + 1], total) - o0, (int64_t)0);
}

// Counts one history token of position `pos` that falls into [c0, c0 + C).
template <int C>
__device__ __forceinline__ void count_token(uint32_t *cnt, int c0, int t, bool prompt)
{
    const uint32_t i = (uint32_t)t - (uint32_t)c0;
    if (t >= 0 && i < (uint32_t)C) {
        if (prompt) atomicOr(cnt + i, IN_PROMPT);
        else atomicAdd(cnt + i, 1u);
    }
}

// grid (vocabulary ranges of 2048 U ids, sequences); shared memory: counts and,
// with a bias, as many floats.
template <typename T, bool VEC, int U>
__global__ void __launch_bounds__(LT) k_logits(const __grid_constant__ LogitsArgs a)
{
    constexpr int C = LT * 8 * U;
    extern __shared__ uint32_t cnt[];              // [C]: IN_PROMPT | times answered
    uint32_t *bias = cnt + C;                      // [C]: the bias as fp32 bits (while being built: entry + 1)
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const int q = blockIdx.y, c0 = blockIdx.x * C, V = a.V, R = a.rows;
    const bool has_bias = a.bias_ids != nullptr;
    pdl_trigger();
    for (int i = tid; i < C / 4; i += LT) reinterpret_cast<uint4 *>(cnt)[i] = make_uint4(0, 0, 0, 0);
    if (has_bias)
        for (int i = tid; i < C / 4; i += LT) reinterpret_cast<uint4 *>(bias)[i] = make_uint4(0, 0, 0, 0);
    pdl_wait();

    const float rep = a.rep ? a.rep[q] : 1.0f, freq = a.freq ? a.freq[q] : 0.0f, pres = a.pres ? a.pres[q] : 0.0f;
    const bool penal = rep != 1.0f || freq != 0.0f || pres != 0.0f;
    __syncthreads();
    if (penal && a.hist) {
        int64_t o0, n;
        range_of(a.hist_off, q, a.n_hist, o0, n);
        const int64_t plen = a.prompt_len ? a.prompt_len[q] : 0;
        const int32_t *h = a.hist + o0;
        int64_t head = (int64_t)((16 - (reinterpret_cast<uintptr_t>(h) & 15)) & 15) / 4;
        if (head > n) head = n;
        if (tid < head) count_token<C>(cnt, c0, h[tid], tid < plen);
        const int4 *h4 = reinterpret_cast<const int4 *>(h + head);
        const int64_t n4 = n > head ? (n - head) / 4 : 0;
        constexpr int UN = 4;
        for (int64_t i0 = tid; i0 < n4; i0 += UN * LT) {
            int4 t[UN];
#pragma unroll
            for (int u = 0; u < UN; ++u) t[u] = i0 + u * LT < n4 ? h4[i0 + u * LT] : make_int4(-1, -1, -1, -1);
#pragma unroll
            for (int u = 0; u < UN; ++u) {
                const int64_t p = head + 4 * (i0 + u * LT);
                count_token<C>(cnt, c0, t[u].x, p < plen);
                count_token<C>(cnt, c0, t[u].y, p + 1 < plen);
                count_token<C>(cnt, c0, t[u].z, p + 2 < plen);
                count_token<C>(cnt, c0, t[u].w, p + 3 < plen);
            }
        }
        const int64_t tail = head + 4 * n4 + tid;
        if (tid < 4 && tail < n) count_token<C>(cnt, c0, h[tail], tail < plen);
    }
    int64_t b0 = 0;
    if (has_bias) {
        // of several entries for one id the last one counts
        int64_t n;
        range_of(a.bias_off, q, a.n_bias, b0, n);
        for (int64_t i = tid; i < n; i += LT) {
            const int t = a.bias_ids[b0 + i];
            const uint32_t k = (uint32_t)t - (uint32_t)c0;
            if (t >= 0 && k < (uint32_t)C) atomicMax(bias + k, (uint32_t)i + 1);
        }
    }
    __syncthreads();

    // slot u of this thread: ids c0 + 2048 u + 8 tid + 0 .. 7; bit 8 u + k of
    // `special`: id k of slot u has a count or a bias
    uint32_t special = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int s = u * LT * 8 + tid * 8;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            bool on = cnt[s + k] != 0;
            if (has_bias && bias[s + k]) {
                bias[s + k] = __float_as_uint(a.bias_val[b0 + bias[s + k] - 1]);
                on = true;
            }
            if (on) special |= 1u << (8 * u + k);
        }
    }

    const int64_t n0 = (int64_t)q * R;
    const T *in = static_cast<const T *>(a.in) + n0 * a.ld;
    T *out = a.out ? static_cast<T *>(a.out) + n0 * a.ldo : nullptr;
    const bool in_place = a.out == a.in && a.ld == a.ldo;
    const int id0 = c0 + tid * 8;

    auto load_row = [&](int j, Raw8<T> (&x)[U], uint32_t &allow) {
        allow = 0xffffffffu;
        if (j >= R) return;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int id = id0 + u * LT * 8;
            if (id < V) x[u] = load_raw<VEC>(in + j * a.ld + id, V - id);
        }
        if (a.mask) {
            const int64_t mr = a.mask_row ? (int64_t)a.mask_row[n0 + j] : n0 + j;
            if (mr >= 0 && mr < a.mask_rows) {
                const uint8_t *m = reinterpret_cast<const uint8_t *>(a.mask + mr * a.ld_mask);
                allow = 0;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int id = id0 + u * LT * 8;
                    if (id < V) allow |= (uint32_t)m[id / 8] << (8 * u);
                }
            }
        }
    };

    Raw8<T> nx[U];
    uint32_t nallow = 0;
    load_row(0, nx, nallow);
    for (int j = 0; j < R; ++j) {
        Raw8<T> x[U];
        const uint32_t allow = nallow;
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = nx[u];
        load_row(j + 1, nx, nallow);
        if (j > 0 && a.draft && penal) {
            const int t = a.draft[q * a.ld_draft + j - 1];
            const uint32_t i = (uint32_t)t - (uint32_t)c0;
            if (t >= 0 && i < (uint32_t)C && (i / 8) % LT == (uint32_t)tid) {
                cnt[i] += 1;
                special |= 1u << (8 * (i / (8 * LT)) + i % 8);
            }
        }
        float best = -INFINITY;
        int best_id = -1;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int id = id0 + u * LT * 8;
            if (id >= V) continue;
            const uint32_t al = (allow >> (8 * u)) & 0xffu, sp = (special >> (8 * u)) & 0xffu;
            float v[8];
            unpack(x[u], v);
            const bool touched = sp != 0 || al != 0xffu;
            if (touched) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    if (sp >> k & 1) {
                        const int s = u * LT * 8 + tid * 8 + k;
                        const uint32_t c = cnt[s], times = c & ~IN_PROMPT;
                        if (c) v[k] = v[k] > 0.0f ? __fdiv_rn(v[k], rep) : __fmul_rn(v[k], rep);
                        if (times) {
                            v[k] = __fsub_rn(v[k], __fmul_rn(freq, (float)times));
                            v[k] = __fsub_rn(v[k], pres);
                        }
                        if (has_bias) v[k] = __fadd_rn(v[k], __uint_as_float(bias[s]));
                    }
                    if (!(al >> k & 1)) v[k] = a.mask_value;
                }
                x[u] = repack(v, T{});
                unpack(x[u], v);
            }
            if (out && !(in_place && !touched)) store_raw<VEC>(out + j * a.ldo + id, V - id, x[u]);
            if (a.part) {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if ((al >> k & 1) && id + k < V && (v[k] > best || (best_id < 0 && v[k] == v[k]))) {
                        best = v[k];
                        best_id = id + k;
                    }
            }
        }
        if (a.part) {
            // the warp's first maximum: the largest value, then the smallest id (-0 counts as 0)
            const unsigned long long key = best_id < 0 ? 0ull : argmax_key(best + 0.0f, best_id);
            const uint32_t hi = (uint32_t)(key >> 32), top = __reduce_max_sync(0xffffffffu, hi);
            const uint32_t lo = __reduce_max_sync(0xffffffffu, hi == top ? (uint32_t)key : 0u);
            if (lane == 0)
                a.part[(n0 + j) * (gridDim.x * LWARPS) + blockIdx.x * LWARPS + warp] =
                    ((unsigned long long)top << 32) | lo;
        }
    }
}

// grid ceil(rows / 8), 256 threads: warp w combines the n keys of row 8 blockIdx.x + w.
__global__ void __launch_bounds__(256) k_logits_argmax(const unsigned long long *part, int n, int64_t rows,
                                                        int32_t *argmax)
{
    const int64_t row = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
    const int lane = threadIdx.x % 32;
    pdl_trigger();
    pdl_wait();
    if (row >= rows) return;
    unsigned long long best = 0;
    for (int i = lane; i < n; i += 32) {
        const unsigned long long k = part[row * n + i];
        if (k > best) best = k;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const unsigned long long k = __shfl_xor_sync(0xffffffffu, best, o);
        if (k > best) best = k;
    }
    if (lane == 0) {
        float v;
        int id = -1;
        if (best) argmax_unkey(best, v, id);
        argmax[row] = id;
    }
}

// Slots per thread: ranges of 2048, 4096 or 8192 ids, the largest that still
// gives every SM two CTAs.
int logits_slots(int n_seq, int V, int sms)
{
    int U = 4;
    while (U > 1 && (int64_t)n_seq * ((V + LT * 8 * U - 1) / (LT * 8 * U)) < 2 * sms) U /= 2;
    return U;
}

template <typename T, bool VEC>
cudaError_t launch_logits(const LogitsArgs &a, int n_seq, int U, cudaStream_t st)
{
    const int C = LT * 8 * U;
    const dim3 grid((a.V + C - 1) / C, n_seq);
    const size_t smem = (size_t)C * 4 * (a.bias_ids ? 2 : 1);
    auto *k = U == 1 ? k_logits<T, VEC, 1> : U == 2 ? k_logits<T, VEC, 2> : k_logits<T, VEC, 4>;
    if (smem > 48 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) { (void)cudaGetLastError(); return e; }
    }
    return launch_head(k, grid, LT, smem, st, 1, a);
}

}  // namespace
}  // namespace xp

using namespace xp;

extern "C" size_t xpress_process_logits_workspace_size(int n_seq, int rows, int V)
{
    if (n_seq < 1 || rows < 1 || V < 1) return 0;
    return (size_t)n_seq * rows * ((V + LT * 8 - 1) / (LT * 8)) * LWARPS * 8;
}

extern "C" int xpress_process_logits(const xpress_logits_args *in, void *ws, size_t ws_bytes, void *stream)
{
    if (!in || in->n_seq < 0 || in->rows < 1 || in->V < 1 || !in->logits || (!in->out && !in->argmax) ||
        in->ld < in->V || (in->out && in->ldo < in->V))
        return XPRESS_ERR_INVALID_ARG;
    if ((in->dtype != XPRESS_F32 && in->dtype != XPRESS_BF16) || in->n_seq > 65535 || in->V > MAX_DIM)
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
    a.part = in->argmax ? static_cast<unsigned long long *>(ws) : nullptr;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int U = logits_slots(in->n_seq, in->V, sms);
    const bool vec = aligned(in->logits, 16) && in->ld * es % 16 == 0 &&
                     (!in->out || (aligned(in->out, 16) && in->ldo * es % 16 == 0));
    XH_CUDA(in->dtype == XPRESS_BF16
                ? (vec ? launch_logits<uint16_t, true>(a, in->n_seq, U, st)
                       : launch_logits<uint16_t, false>(a, in->n_seq, U, st))
                : (vec ? launch_logits<float, true>(a, in->n_seq, U, st)
                       : launch_logits<float, false>(a, in->n_seq, U, st)));
    if (in->argmax) {
        const int64_t rows = (int64_t)in->n_seq * in->rows;
        const int n = (in->V + LT * 8 * U - 1) / (LT * 8 * U) * LWARPS;
        XH_CUDA(launch_head(k_logits_argmax, dim3((unsigned)((rows + 7) / 8)), 256, 0, st, 1,
                            (const unsigned long long *)ws, n, rows, in->argmax));
    }
    return XPRESS_OK;
}
