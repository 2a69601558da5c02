// The model-stages' own steps on the LM head's logits for sm_100a: penalties, biases and grammar masks of a generation
// step (nereus_logits_process), a teacher's top logits of an inference stage (nereus_teacher_top) and the distillation
// from them of a training stage (nereus_distill_forward / _backward / _step).
//
// Logits come cut by vocabulary into column shards, one device buffer each.  All three walk rows of some 100,000
// elements with a handful of operations on each, so their floor is HBM bandwidth.
//
// One block works on one row and reads it from memory as often as it needs it.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>

#include "nereus_internal.hpp"

using namespace nereus;

namespace nereus {
namespace {

#define NEREUS_CUDA(call)                                               \
    do {                                                                \
        cudaError_t e_ = (call);                                        \
        if (e_ != cudaSuccess) { set_cuda_error((int)e_); (void)cudaGetLastError(); return NEREUS_ERR_CUDA; } \
    } while (0)

// A view of cut logits as a kernel parameter.
struct LogitsCut {
    char*   shard[NEREUS_VOCAB_MAX_TP];
    int64_t row_bytes;
    int32_t tp, cols, vocab;
};

constexpr int kThreads = 512;
constexpr int kSlice   = 4096;        // vocabulary columns whose history counters are in shared memory at a time

template <class T> __device__ __forceinline__ float to_float(T v);
template <> __device__ __forceinline__ float to_float<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

template <class T> __device__ __forceinline__ T* row_of(const LogitsCut& c, int s, int64_t row) {
    return reinterpret_cast<T*>(c.shard[s] + row * c.row_bytes);
}
__device__ __forceinline__ int width_of(const LogitsCut& c, int s) {
    const int64_t left = (int64_t)c.vocab - (int64_t)s * c.cols;
    return left <= 0 ? 0 : left < c.cols ? (int)left : c.cols;
}

// f(token, element) for every element of the row, the block's threads side by side.
template <class T, class F> __device__ __forceinline__ void for_row(const LogitsCut& c, int64_t row, F f) {
    for (int s = 0; s < c.tp; ++s) {
        const int w = width_of(c, s);
        const T*  p = w ? row_of<T>(c, s, row) : nullptr;
        for (int i = threadIdx.x; i < w; i += kThreads) f(s * c.cols + i, to_float(p[i]));
    }
}

__device__ float block_sum(float v, float* scratch) {
    __syncthreads();
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    float r = 0.f;
    for (int i = 0; i < kThreads / 32; ++i) r += scratch[i];
    return r;
}
__device__ float block_max(float v, float* scratch) {
    __syncthreads();
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    float r = -INFINITY;
    for (int i = 0; i < kThreads / 32; ++i) r = fmaxf(r, scratch[i]);
    return r;
}
__device__ int block_min(int v, int* scratch) {
    __syncthreads();
    for (int o = 16; o; o >>= 1) v = min(v, __shfl_xor_sync(0xffffffffu, v, o));
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    int r = 0x7fffffff;
    for (int i = 0; i < kThreads / 32; ++i) r = min(r, scratch[i]);
    return r;
}
__device__ int block_count(int v, int* scratch) {
    __syncthreads();
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    int r = 0;
    for (int i = 0; i < kThreads / 32; ++i) r += scratch[i];
    return r;
}

// log of a sum of exponentials from its maximum and the sum of exp(x - max)
__device__ __forceinline__ float log_sum(float m, float scaled_m, float sum) {
    if (sum != sum) return sum;
    return m == -INFINITY || m == INFINITY ? m : scaled_m + logf(sum);
}
// exp((x - m) * t) where m is at least x: 1 at the maximum itself, an infinite one included, and 0 at -inf
__device__ __forceinline__ float exp_below(float x, float m, float t) {
    return x == m ? (x == -INFINITY ? 0.f : 1.f) : expf((x - m) * t);
}

// ---- penalties, biases, masks --------------------------------------------------------------------------------

template <class TI, class TO>
__global__ void __launch_bounds__(kThreads) process_kernel(LogitsCut in, LogitsCut out, nereus_penalties_t how, int32_t* token,
                                                           float* lse) {
    // seen: bit 31 in the history, the other bits the entry of the bias list, from 1; made: how often generated
    __shared__ uint32_t seen[kSlice], made[kSlice];
    __shared__ float scratch[32];
    __shared__ int   iscratch[32];
    const int64_t row = blockIdx.x;
    const float rho = how.repetition ? how.repetition[row] : 1.f;
    const float pres = how.presence ? how.presence[row] : 0.f, freq = how.frequency ? how.frequency[row] : 0.f;
    int total = 0, prompt = 0;
    if (how.history) {
        total = how.total_len ? max(0, min((int)how.history_len, how.total_len[row])) : (int)how.history_len;
        prompt = how.prompt_len ? how.prompt_len[row] : 0;
    }
    const int32_t* hist = how.history + (how.history ? row * how.history_stride : 0);
    int64_t mrow = how.mask ? (how.mask_row ? how.mask_row[row] : row) : -1;
    const int32_t* mask = mrow >= 0 && mrow < how.mask_rows ? how.mask + mrow * how.mask_stride : nullptr;

    float best = -INFINITY, m = -INFINITY, sum = 0.f;
    int   at = 0x7fffffff;
    for (int v0 = 0; v0 < in.vocab; v0 += kSlice) {
        const int n = min(kSlice, in.vocab - v0);
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += kThreads) seen[i] = made[i] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < total; i += kThreads) {
            const uint32_t v = (uint32_t)hist[i] - (uint32_t)v0;
            if (hist[i] >= 0 && v < (uint32_t)n) {
                atomicOr(&seen[v], 0x80000000u);
                if (i >= prompt) atomicAdd(&made[v], 1u);
            }
        }
        if (how.bias_ids)
            for (int i = threadIdx.x; i < how.bias_count; i += kThreads) {
                const int     id = how.bias_ids[row * how.bias_count + i];
                const uint32_t v = (uint32_t)id - (uint32_t)v0;
                if (id >= 0 && v < (uint32_t)n) {
                    uint32_t old = seen[v], assumed;
                    do {
                        assumed = old;
                        if ((assumed & 0x7fffffffu) >= (uint32_t)(i + 1)) break;
                        old = atomicCAS(&seen[v], assumed, (assumed & 0x80000000u) | (uint32_t)(i + 1));
                    } while (old != assumed);
                }
            }
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const int v = v0 + i, s = v / in.cols, c = v - s * in.cols;
            float x = to_float(row_of<TI>(in, s, row)[c]);
            const uint32_t w = seen[i];
            if (w >> 31) x = x > 0.f ? __fdiv_rn(x, rho) : __fmul_rn(x, rho);
            if (const uint32_t k = made[i]) x = __fsub_rn(__fsub_rn(x, __fmul_rn(freq, (float)k)), pres);
            if (const uint32_t b = w & 0x7fffffffu) x = __fadd_rn(x, how.bias_values[row * how.bias_count + b - 1]);
            if (mask && !((uint32_t)mask[v >> 5] >> (v & 31) & 1u)) x = -INFINITY;
            const TO y = from_float<TO>(x);
            row_of<TO>(out, s, row)[c] = y;
            x = to_float(y);
            if (x > best) { best = x; at = v; }
            if (x > m) { sum *= exp_below(m, x, 1.f); m = x; }
            sum += exp_below(x, m, 1.f);                    // NaN stays NaN
        }
    }
    const float top = block_max(best, scratch);
    const int   where = block_min(best == top && top > -INFINITY ? at : 0x7fffffff, iscratch);
    const float all = block_sum(sum == 0.f ? 0.f : sum * exp_below(m, top, 1.f), scratch);
    if (threadIdx.x == 0) {
        if (token) token[row] = top > -INFINITY ? where : -1;
        if (lse) lse[row] = log_sum(top, top, all);
    }
}

// ---- a teacher's top logits ----------------------------------------------------------------------------------

// orders as the values do, -0 as +0; NaN below everything
__device__ __forceinline__ uint32_t key_of(float x) {
    if (x != x) return 0u;
    const uint32_t u = __float_as_uint(x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) {
    return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

template <class T>
__global__ void __launch_bounds__(kThreads) top_kernel(LogitsCut in, int k, float inv_t, float* values, int32_t* ids,
                                                       float* lse) {
    __shared__ float scratch[32];
    __shared__ int   iscratch[32];
    __shared__ unsigned long long cand[NEREUS_TOP_MAX_K];
    __shared__ int n_cand;
    const int64_t row = blockIdx.x;
    float m = -INFINITY;
    for_row<T>(in, row, [&](int, float x) { m = fmaxf(m, x); });
    m = block_max(m, scratch);
    float sum = 0.f;
    for_row<T>(in, row, [&](int, float x) { sum += exp_below(x, m, inv_t); });
    sum = block_sum(sum, scratch);
    if (threadIdx.x == 0) { lse[row] = log_sum(m, m * inv_t, sum); n_cand = 0; }

    uint32_t t = 0;                       // the largest key that k elements reach
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t u = t | 1u << bit;
        int n = 0;
        for_row<T>(in, row, [&](int, float x) { n += key_of(x) >= u; });
        if (block_count(n, iscratch) >= k) t = u;
    }
    // among equals of the k-th the lowest ids
    int above = 0;
    for_row<T>(in, row, [&](int, float x) { above += key_of(x) > t; });
    above = block_count(above, iscratch);
    int lo = -1;                          // the largest id so that fewer than k elements lie at or before it
    if (t) {
        for (int bit = 23; bit >= 0; --bit) {
            const int u = lo + (1 << bit);
            int n = 0;
            for_row<T>(in, row, [&](int v, float x) { n += key_of(x) == t && v <= u; });
            if (above + block_count(n, iscratch) < k) lo = u;
        }
    }
    for_row<T>(in, row, [&](int v, float x) {
        const uint32_t key = key_of(x);
        if (key > t || (t && key == t && v <= lo + 1)) cand[atomicAdd(&n_cand, 1)] = (unsigned long long)key << 32 | (0xffffffffu - v);
    });
    __syncthreads();
    const int n = n_cand;
    for (int i = threadIdx.x; i < k; i += kThreads) {
        if (i < n) {
            int rank = 0;
            for (int j = 0; j < n; ++j) rank += cand[j] > cand[i];
            values[row * k + rank] = value_of((uint32_t)(cand[i] >> 32));
            ids[row * k + rank] = (int32_t)(0xffffffffu - (uint32_t)cand[i]);
        } else {
            values[row * k + i] = -INFINITY;
            ids[row * k + i] = -1;
        }
    }
}

// ---- distillation --------------------------------------------------------------------------------------------

enum Pass { kForward, kBackward, kStep };

template <class T, int kPass>
__global__ void __launch_bounds__(kThreads) distill_kernel(LogitsCut in, LogitsCut grad, nereus_distill_t how, float* loss,
                                                           float* saved, const float* grad_loss) {
    __shared__ float scratch[32];
    __shared__ int   iscratch[32];
    const int64_t row = blockIdx.x;
    const int     k = how.k, tid = threadIdx.x;
    float weight = how.weight ? how.weight[row] : 1.f;
    if (weight == 0.f) {
        if (tid == 0 && kPass != kBackward) loss[row] = 0.f;
        if (tid < 4 && kPass == kForward) saved[row * 4 + tid] = 0.f;
        if (kPass != kForward)
            for (int s = 0; s < grad.tp; ++s)
                for (int i = tid; i < width_of(grad, s); i += kThreads) row_of<T>(grad, s, row)[i] = from_float<T>(0.f);
        return;
    }
    const float inv_t = 1.f / how.temperature;
    int   id = tid < k ? how.ids[row * k + tid] : -1;
    if (id < 0 || id >= in.vocab) id = -1;
    const float y = id >= 0 ? how.values[row * k + tid] : 0.f;
    const float x = id >= 0 ? to_float(row_of<T>(in, id / in.cols, row)[id % in.cols]) : 0.f;
    const int   entries = block_count(id >= 0, iscratch);

    float m, total, rest;
    if (kPass == kBackward) {
        m = saved[row * 4]; total = saved[row * 4 + 1]; rest = saved[row * 4 + 2];
    } else {
        m = -INFINITY;
        for_row<T>(in, row, [&](int, float v) { m = fmaxf(m, v); });
        m = block_max(m, scratch);
        // the rest is summed on its own: as a difference it would lose its digits where the entries hold nearly all
        const float mine = id >= 0 ? expf((x - m) * inv_t) : 0.f;
        float r = 0.f;
        __shared__ int taken[NEREUS_TOP_MAX_K];
        if (tid < k) taken[tid] = id;
        __syncthreads();
        for_row<T>(in, row, [&](int v, float e) {
            bool entry = false;
            for (int j = 0; j < k; ++j) entry |= taken[j] == v;
            if (!entry) r += expf((e - m) * inv_t);
        });
        rest = block_sum(r, scratch);
        total = rest + block_sum(mine, scratch);
    }

    // the groups: entry `tid` on its thread, the rest on all
    const bool  has_rest = entries < in.vocab;
    const float log_total = logf(total);
    const float log_q = (x - m) * inv_t - log_total, q = expf(log_q);
    const float log_q_rest = logf(rest) - log_total, q_rest = rest / total;
    float log_p, p, p_rest, mass;
    if (how.lse) {
        log_p = y * inv_t - how.lse[row];
        p = id >= 0 ? expf(log_p) : 0.f;
        p_rest = has_rest ? fmaxf(0.f, 1.f - block_sum(p, scratch)) : 0.f;
        mass = 1.f;
    } else {
        const float top = block_max(id >= 0 ? y : -INFINITY, scratch);
        const float e = id >= 0 ? expf((y - top) * inv_t) : 0.f;
        const float sum = block_sum(e, scratch);
        log_p = (y - top) * inv_t - logf(sum);
        p = entries ? e / sum : 0.f;
        p_rest = 0.f;
        mass = entries ? 1.f : 0.f;
    }
    float term = 0.f, slope = 0.f, term_rest = 0.f, slope_rest = 0.f, mean;
    // of the forward KL the products Q f and Q sum Q f are kept, which stay finite where Q is 0
    if (how.divergence == NEREUS_FORWARD_KL) {
        if (p > 0.f) term = p * (log_p - log_q);
        if (p_rest > 0.f) term_rest = p_rest * (logf(p_rest) - log_q_rest);
        mean = 0.f;
    } else if (how.divergence == NEREUS_REVERSE_KL) {
        p_rest = fmaxf(p_rest, 5.9604644775390625e-8f);
        if (q > 0.f && id >= 0) { slope = log_q - log_p; term = q * slope; }
        if (q_rest > 0.f) { slope_rest = log_q_rest - logf(p_rest); term_rest = q_rest * slope_rest; }
        mean = block_sum(term, scratch) + term_rest;
    } else {
        const float a = how.beta, b = 1.f - how.beta;
        float qf = 0.f, qf_rest = 0.f;
        if (id >= 0) {
            const float log_m = logf(a * p + b * q);
            if (q > 0.f) { slope = b * (log_q - log_m); qf = q * slope; }
            term = qf + (p > 0.f ? a * p * (log_p - log_m) : 0.f);
        }
        const float log_m = logf(a * p_rest + b * q_rest);
        if (q_rest > 0.f) { slope_rest = b * (log_q_rest - log_m); qf_rest = q_rest * slope_rest; }
        term_rest = qf_rest + (p_rest > 0.f ? a * p_rest * (logf(p_rest) - log_m) : 0.f);
        mean = block_sum(qf, scratch) + qf_rest;
    }
    const float d = block_sum(id >= 0 ? term : 0.f, scratch) + term_rest;
    if (tid == 0 && kPass != kBackward) loss[row] = weight * d;
    if (tid == 0 && kPass == kForward) {
        saved[row * 4] = m; saved[row * 4 + 1] = total; saved[row * 4 + 2] = rest; saved[row * 4 + 3] = d;
    }
    if (kPass == kForward) return;
    if (kPass == kBackward && grad_loss) weight *= grad_loss[row];
    const float scale = weight * inv_t;
    float g, c;
    if (how.divergence == NEREUS_FORWARD_KL) {
        g = (mass * q - p) * scale;
        c = (mass - (p_rest > 0.f && rest > 0.f ? p_rest / q_rest : 0.f)) * scale / total;
    } else {
        g = q > 0.f ? q * (slope - mean) * scale : 0.f;
        c = (slope_rest - mean) * scale / total;
    }
    for_row<T>(in, row, [&](int v, float e) {
        const int s = v / in.cols;
        row_of<T>(grad, s, row)[v - s * in.cols] = from_float<T>(expf((e - m) * inv_t) * c);
    });
    __syncthreads();
    if (id >= 0) row_of<T>(grad, id / in.cols, row)[id % in.cols] = from_float<T>(g);
}

// ---- host side: the checks of the arguments ------------------------------------------------------------------

constexpr int64_t kMaxRows  = 1 << 24;
constexpr int64_t kMaxVocab = 1 << 24;

int size_of(int dtype) { return dtype == NEREUS_BF16 ? 2 : 4; }

int64_t held_cols(const nereus_logits_t& v, int s) {
    const int64_t left = v.vocab - (int64_t)s * v.shard_cols;
    return left <= 0 ? 0 : left < v.shard_cols ? left : v.shard_cols;
}

int check_view(const nereus_logits_t* v) {
    if (!v) return NEREUS_ERR_ARG;
    if (v->dtype != NEREUS_BF16 && v->dtype != NEREUS_FP32) return NEREUS_ERR_UNSUPPORTED;
    if (v->tp < 1 || v->tp > NEREUS_VOCAB_MAX_TP || v->rows < 0 || v->vocab < 1 || v->shard_cols < 1) return NEREUS_ERR_ARG;
    if (v->rows > kMaxRows || v->vocab > kMaxVocab || v->shard_cols > kMaxVocab) return NEREUS_ERR_TOO_LARGE;
    if (v->shard_cols * v->tp < v->vocab) return NEREUS_ERR_ARG;
    if (v->row_stride < 0 || v->row_stride > ((int64_t)1 << 40)) return NEREUS_ERR_ARG;
    if (v->rows > 1 && v->row_stride < held_cols(*v, 0)) return NEREUS_ERR_ARG;
    for (int s = 0; s < v->tp; ++s) {
        if (!held_cols(*v, s)) continue;
        if (!v->shard[s] && v->rows > 0) return NEREUS_ERR_ARG;
        if ((uintptr_t)v->shard[s] % size_of(v->dtype)) return NEREUS_ERR_ALIGN;
    }
    return NEREUS_OK;
}

// Whether two shards have no byte in common.  Two column slices of one tensor interleave without touching.
bool apart(const nereus_logits_t& a, int s, const nereus_logits_t& b, int t) {
    const int64_t ea = size_of(a.dtype), eb = size_of(b.dtype), wa = held_cols(a, s) * ea, wb = held_cols(b, t) * eb;
    if (!wa || !wb) return true;
    const int64_t sa = a.row_stride * ea, sb = b.row_stride * eb;
    const int64_t pa = (int64_t)(uintptr_t)a.shard[s], pb = (int64_t)(uintptr_t)b.shard[t];
    const int64_t end_a = pa + (a.rows - 1) * sa + wa, end_b = pb + (b.rows - 1) * sb + wb;
    if (end_a <= pb || end_b <= pa) return true;
    if (a.rows < 2 || sa != sb) return false;
    const int64_t gap = pa <= pb ? (pb - pa) % sa : (pa - pb) % sa;
    return pa <= pb ? gap >= wa && gap + wb <= sa : gap >= wb && gap + wa <= sa;
}

int check_written(const nereus_logits_t& in, const nereus_logits_t* out) {
    if (int rc = check_view(out)) return rc;
    if (out->rows != in.rows || out->vocab != in.vocab || out->tp != in.tp || out->shard_cols != in.shard_cols)
        return NEREUS_ERR_MISMATCH;
    if (in.rows == 0) return NEREUS_OK;
    const bool alike = out->dtype == in.dtype && (out->row_stride == in.row_stride || in.rows == 1);
    for (int s = 0; s < in.tp; ++s)
        for (int t = 0; t < in.tp; ++t) {
            if (!(s == t && alike && in.shard[s] == out->shard[s]) && !apart(in, s, *out, t)) return NEREUS_ERR_ALIAS;
            if (s < t && !apart(*out, s, *out, t)) return NEREUS_ERR_ALIAS;
        }
    return NEREUS_OK;
}

LogitsCut cut_of(const nereus_logits_t& v) {
    LogitsCut c;
    for (int s = 0; s < NEREUS_VOCAB_MAX_TP; ++s) c.shard[s] = s < v.tp ? (char*)v.shard[s] : nullptr;
    c.row_bytes = v.row_stride * size_of(v.dtype);
    c.tp = v.tp; c.cols = (int32_t)v.shard_cols; c.vocab = (int32_t)v.vocab;
    return c;
}

bool misaligned(const void* p) { return (uintptr_t)p & 3; }

int check_penalties(const nereus_logits_t& in, const nereus_penalties_t& h) {
    if (h.history) {
        if (h.history_len < 0 || h.history_stride < h.history_len) return NEREUS_ERR_ARG;
        if (h.history_len > NEREUS_HISTORY_MAX) return NEREUS_ERR_TOO_LARGE;
    } else if (h.prompt_len || h.total_len) {
        return NEREUS_ERR_ARG;
    }
    if (!h.bias_ids != !h.bias_values || h.bias_count < 0) return NEREUS_ERR_ARG;
    if (h.bias_count > NEREUS_BIAS_MAX) return NEREUS_ERR_TOO_LARGE;
    if (h.mask) {
        if (h.mask_stride < (in.vocab + 31) / 32 || h.mask_rows < 0) return NEREUS_ERR_ARG;
        if (!h.mask_row && h.mask_rows < in.rows) return NEREUS_ERR_ARG;
    } else if (h.mask_row) {
        return NEREUS_ERR_ARG;
    }
    if (misaligned(h.history) || misaligned(h.prompt_len) || misaligned(h.total_len) || misaligned(h.repetition) ||
        misaligned(h.presence) || misaligned(h.frequency) || misaligned(h.bias_ids) || misaligned(h.bias_values) ||
        misaligned(h.mask) || misaligned(h.mask_row))
        return NEREUS_ERR_ALIGN;
    return NEREUS_OK;
}

int check_distill(const nereus_logits_t* in, const nereus_distill_t* h) {
    if (int rc = check_view(in)) return rc;
    if (!h || h->k < 1 || h->k > NEREUS_TOP_MAX_K || !h->values || !h->ids) return NEREUS_ERR_ARG;
    if (h->divergence < NEREUS_FORWARD_KL || h->divergence > NEREUS_JENSEN) return NEREUS_ERR_ARG;
    if (h->divergence == NEREUS_JENSEN && !(h->beta > 0.f && h->beta < 1.f)) return NEREUS_ERR_ARG;
    if (!(h->temperature > 0.f) || !std::isfinite(h->temperature)) return NEREUS_ERR_ARG;
    if (!h->lse && h->divergence != NEREUS_FORWARD_KL) return NEREUS_ERR_UNSUPPORTED;
    if (misaligned(h->values) || misaligned(h->ids) || misaligned(h->lse) || misaligned(h->weight)) return NEREUS_ERR_ALIGN;
    return NEREUS_OK;
}

template <int kPass>
int distill(const nereus_logits_t* in, const nereus_distill_t* how, float* loss, float* saved, const float* grad_loss,
            const nereus_logits_t* grad, void* stream) {
    if (int rc = check_distill(in, how)) return rc;
    if (misaligned(loss) || misaligned(saved) || misaligned(grad_loss)) return NEREUS_ERR_ALIGN;
    if (kPass != kForward) {
        if (int rc = check_written(*in, grad)) return rc;
        if (grad->dtype != in->dtype) return NEREUS_ERR_UNSUPPORTED;
    }
    if (in->rows == 0) return NEREUS_OK;
    if ((kPass != kBackward && !loss) || (kPass != kStep && !saved)) return NEREUS_ERR_ARG;
    const LogitsCut ci = cut_of(*in), cg = kPass == kForward ? LogitsCut() : cut_of(*grad);
    cudaStream_t st = (cudaStream_t)stream;
    if (in->dtype == NEREUS_BF16)
        distill_kernel<__nv_bfloat16, kPass><<<(unsigned)in->rows, kThreads, 0, st>>>(ci, cg, *how, loss, saved, grad_loss);
    else
        distill_kernel<float, kPass><<<(unsigned)in->rows, kThreads, 0, st>>>(ci, cg, *how, loss, saved, grad_loss);
    NEREUS_CUDA(cudaGetLastError());
    return NEREUS_OK;
}

}  // namespace
}  // namespace nereus

extern "C" {

int nereus_logits_process(const nereus_logits_t* in, const nereus_logits_t* out, const nereus_penalties_t* how,
                          int32_t* token, float* lse, void* cuda_stream) {
    if (int rc = check_view(in)) return rc;
    if (int rc = check_written(*in, out)) return rc;
    if (!how) return NEREUS_ERR_ARG;
    if (out->dtype != in->dtype && out->dtype != NEREUS_FP32) return NEREUS_ERR_UNSUPPORTED;
    if (int rc = check_penalties(*in, *how)) return rc;
    if (misaligned(token) || misaligned(lse)) return NEREUS_ERR_ALIGN;
    if (in->rows == 0) return NEREUS_OK;
    const LogitsCut ci = cut_of(*in), co = cut_of(*out);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const unsigned grid = (unsigned)in->rows;
    if (in->dtype == NEREUS_FP32) process_kernel<float, float><<<grid, kThreads, 0, st>>>(ci, co, *how, token, lse);
    else if (out->dtype == NEREUS_FP32) process_kernel<__nv_bfloat16, float><<<grid, kThreads, 0, st>>>(ci, co, *how, token, lse);
    else process_kernel<__nv_bfloat16, __nv_bfloat16><<<grid, kThreads, 0, st>>>(ci, co, *how, token, lse);
    NEREUS_CUDA(cudaGetLastError());
    return NEREUS_OK;
}

int nereus_teacher_top(const nereus_logits_t* in, int k, float temperature, float* values, int32_t* ids, float* lse,
                       void* cuda_stream) {
    if (int rc = check_view(in)) return rc;
    if (k < 1 || k > NEREUS_TOP_MAX_K || k > in->vocab) return NEREUS_ERR_ARG;
    if (!(temperature > 0.f) || !std::isfinite(temperature)) return NEREUS_ERR_ARG;
    if (misaligned(values) || misaligned(ids) || misaligned(lse)) return NEREUS_ERR_ALIGN;
    if (in->rows == 0) return NEREUS_OK;
    if (!values || !ids || !lse) return NEREUS_ERR_ARG;
    const LogitsCut ci = cut_of(*in);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const unsigned grid = (unsigned)in->rows;
    if (in->dtype == NEREUS_BF16) top_kernel<__nv_bfloat16><<<grid, kThreads, 0, st>>>(ci, k, 1.f / temperature, values, ids, lse);
    else top_kernel<float><<<grid, kThreads, 0, st>>>(ci, k, 1.f / temperature, values, ids, lse);
    NEREUS_CUDA(cudaGetLastError());
    return NEREUS_OK;
}

int nereus_distill_forward(const nereus_logits_t* in, const nereus_distill_t* how, float* loss, float* saved,
                           void* cuda_stream) {
    return distill<kForward>(in, how, loss, saved, nullptr, nullptr, cuda_stream);
}

int nereus_distill_backward(const nereus_logits_t* in, const nereus_distill_t* how, const float* saved,
                            const float* grad_loss, const nereus_logits_t* grad, void* cuda_stream) {
    return distill<kBackward>(in, how, nullptr, const_cast<float*>(saved), grad_loss, grad, cuda_stream);
}

int nereus_distill_step(const nereus_logits_t* in, const nereus_distill_t* how, float* loss,
                        const nereus_logits_t* grad, void* cuda_stream) {
    return distill<kStep>(in, how, loss, nullptr, nullptr, grad, cuda_stream);
}

}  // extern "C"
