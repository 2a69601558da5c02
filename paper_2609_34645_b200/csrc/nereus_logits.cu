// The model-stages' own steps on the LM head's logits for sm_100a: penalties, biases and grammar masks of a generation
// step (nereus_logits_process), a teacher's top logits of an inference stage (nereus_teacher_top) and the distillation
// from them of a training stage (nereus_distill_forward / _backward / _step).
//
// Logits come cut by vocabulary into column shards, one device buffer each.  All three walk rows of some 100,000
// elements with a handful of operations on each, so their floor is HBM bandwidth: every logit read once, every written
// one stored once.  The common frame:
//   * A row belongs to one thread-block cluster of C = 1, 2, 4 or 8 blocks of 512 threads; its 16-byte vectors are dealt
//     out in layers of 512 (8 KiB), layer l to block l % C.  A layer lies inside one shard, so that everything about it
//     but the thread's own vector is the same for the block: one 32-byte record per layer in shared memory.
//   * A block's share of the row stays in shared memory (cp.async, every thread reads back only the vectors that it
//     copied itself, so arrival needs no barrier and no wait that could hang), because the result needs the row's sums
//     before the first element can be written.  C is the smallest for which three blocks fit on an SM, so that one
//     block loads while another reduces and a third stores; few rows get more blocks each.
//   * The blocks of a cluster exchange a few numbers through distributed shared memory and one cluster barrier.
//   * Rows of any alignment: vectors that a row fills only in part (its ends, where it does not start on a 16-byte
//     boundary) are read and written element by element; what lies outside the row is -inf in shared memory.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
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

// How rows are dealt out: `per_shard` layers in every shard, `layers` in all, 1 << log_c blocks per row, `mine` layers
// (at most) per block.
struct Deal {
    int32_t per_shard, layers, log_c, mine;
    int32_t aligned;      // every row of every shard starts on a 16-byte boundary
};

constexpr int kThreads  = 512;
constexpr int kWarps    = kThreads / 32;
constexpr int kMaxCtas  = 8;                      // portable cluster size
constexpr float kLog2e  = 1.4426950408889634f;

// One layer of the block's share: positions 0 .. 512 * (elements per vector) - 1, of which [lo, hi) are the row's.
struct __align__(16) Layer {
    const char* in;       // address of position 0, 16-byte aligned; may lie before the row where lo > 0
    char*       out;      // ... of the written view, congruent to `in` or not
    int32_t     token;    // token of position 0; negative where lo > 0 in the first shard
    int32_t     lo, hi;
    int32_t     vec_out;  // `out` is 16-byte aligned too
};
static_assert(sizeof(Layer) == 32, "Layer is read as two 16-byte words");

template <class T> constexpr int kPerVec = 16 / (int)sizeof(T);
template <class T> constexpr int kPerLayer = kThreads * kPerVec<T>;

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

// Block `rank`'s i-th layer of a row; hi = 0 where it has none.
template <class TI, class TO>
__device__ __forceinline__ Layer layer_of(const LogitsCut& in, const LogitsCut& out, const Deal& d, int64_t row, int rank, int i) {
    Layer r = {nullptr, nullptr, 0, 0, 0, 0};
    const int l = (i << d.log_c) + rank;
    if (l >= d.layers) return r;
    const int s = l / d.per_shard, first = (l - s * d.per_shard) * kPerLayer<TI>;
    const int w = width_of(in, s);
    if (!w) return r;
    const uintptr_t a = (uintptr_t)row_of<TI>(in, s, row);
    const int       phase = (int)(a & 15) / (int)sizeof(TI);       // the row starts at this position of its first vector
    r.in = (const char*)(a & ~(uintptr_t)15) + (int64_t)first * (int)sizeof(TI);
    r.lo = max(0, phase - first);
    r.hi = max(0, min(kPerLayer<TI>, phase + w - first));
    r.token = s * in.cols + first - phase;
    if (out.tp) {
        r.out = (char*)row_of<TO>(out, s, row) + (int64_t)(first - phase) * (int)sizeof(TO);
        r.vec_out = ((uintptr_t)r.out & 15) == 0;
    }
    return r;
}

// A 16-byte vector as floats, and back (bf16: round to nearest even).
template <class T> struct Vec;
template <> struct Vec<float> {
    static __device__ __forceinline__ void unpack(uint4 v, float (&f)[4]) {
        f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[4]) {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
    static __device__ __forceinline__ float max(uint4 v) {           // NaN is passed over
        float f[4];
        unpack(v, f);
        return fmaxf(fmaxf(f[0], f[1]), fmaxf(f[2], f[3]));
    }
};
template <> struct Vec<__nv_bfloat16> {
    static __device__ __forceinline__ void unpack(uint4 v, float (&f)[8]) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ uint32_t pair(float lo, float hi) {
        uint32_t r;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
        return make_uint4(pair(f[0], f[1]), pair(f[2], f[3]), pair(f[4], f[5]), pair(f[6], f[7]));
    }
    static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
        uint32_t r;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static __device__ __forceinline__ float max(uint4 v) {
        const uint32_t m = max2(max2(v.x, v.y), max2(v.z, v.w));
        return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
    }
};

__device__ __forceinline__ float exp2_approx(float x) {              // relative error 2^-22, 0 at -inf
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ uint32_t smem_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy_async(uint32_t to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int n> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(n) : "memory"); }

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t peer_address(const void* p, int rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_address(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ void peer_store(uint32_t at, float a, float b) {
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(at), "f"(a), "f"(b) : "memory");
}
__device__ __forceinline__ unsigned long long peer_load64(uint32_t at) {
    unsigned long long v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(at) : "memory");
    return v;
}

// Starts the copies of the block's share into slots [layer][thread], in four commit groups of `quarter` layers.
template <class T>
__device__ __forceinline__ void load_share(const Layer* table, uint4* slots, int n, int quarter) {
    const int t = threadIdx.x, p = t * kPerVec<T>;
    int i = 0;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const int end = min(n, (g + 1) * quarter);
        for (; i < end; ++i) {
            const int lo = table[i].lo, hi = table[i].hi;
            if (p >= lo && p + kPerVec<T> <= hi) copy_async(smem_address(&slots[i * kThreads + t]), table[i].in + t * 16);
        }
        copy_commit();
    }
    for (i = 0; i < n; ++i) {                 // vectors that the row fills in part
        const int lo = table[i].lo, hi = table[i].hi;
        if (p < hi && p + kPerVec<T> > lo && (p < lo || p + kPerVec<T> > hi)) {
            T e[kPerVec<T>];
#pragma unroll
            for (int j = 0; j < kPerVec<T>; ++j)
                e[j] = p + j >= lo && p + j < hi ? reinterpret_cast<const T*>(table[i].in)[p + j] : from_float<T>(-INFINITY);
#pragma unroll
            for (int j = 0; j < kPerVec<T>; ++j) reinterpret_cast<T*>(&slots[i * kThreads + t])[j] = e[j];
        }
    }
}

// f(layer index) for every layer in which this thread has a vector of the row, in the order of arrival.
template <class T, class F>
__device__ __forceinline__ void on_arrival(const Layer* table, int n, int quarter, F f) {
    const int p = threadIdx.x * kPerVec<T>;
    auto some = [&](int a, int b) {
        for (int i = a; i < min(b, n); ++i)
            if (p < table[i].hi && p + kPerVec<T> > table[i].lo) f(i);
    };
    copy_wait<3>();
    some(0, quarter);
    copy_wait<2>();
    some(quarter, 2 * quarter);
    copy_wait<1>();
    some(2 * quarter, 3 * quarter);
    copy_wait<0>();
    some(3 * quarter, 4 * quarter);
}

template <class T>
__device__ __forceinline__ void store_vector(const Layer& l, uint4 v) {
    const int p = threadIdx.x * kPerVec<T>;
    if (l.vec_out && p >= l.lo && p + kPerVec<T> <= l.hi) {
        __stcs(reinterpret_cast<uint4*>(l.out + threadIdx.x * 16), v);
    } else {
        T* o = reinterpret_cast<T*>(l.out);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < kPerVec<T>; ++j)
            if (p + j >= l.lo && p + j < l.hi) {
                if (sizeof(T) == 4) reinterpret_cast<uint32_t*>(o)[p + j] = w[j * sizeof(T) / 4];
                else reinterpret_cast<uint16_t*>(o)[p + j] = (uint16_t)(w[j / 2] >> (j % 2 * 16));
            }
    }
}

// Sum of two values over the block, in the same order for every thread.
__device__ __forceinline__ float2 block_sum2(float a, float b, float2* scratch) {
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        a += __shfl_xor_sync(0xffffffffu, a, o);
        b += __shfl_xor_sync(0xffffffffu, b, o);
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = make_float2(a, b);
    __syncthreads();
    float2 r = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < kWarps; ++i) { r.x += scratch[i].x; r.y += scratch[i].y; }
    return r;
}
__device__ __forceinline__ float block_max(float v, float2* scratch) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5].x = v;
    __syncthreads();
    float r = -INFINITY;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) r = fmaxf(r, scratch[i].x);
    return r;
}

// A maximum m and the sum of 2^((x - m) c): two of them joined.  A maximum of -inf goes with a sum of 0 (or NaN).
__device__ __forceinline__ float scale_to(float m, float to, float c) {
    return m == to ? 1.f : exp2_approx((m - to) * c);
}
__device__ __forceinline__ float2 join(float2 a, float2 b, float c) {
    const float m = fmaxf(a.x, b.x);
    // the same whichever comes first: no product is contracted into the sum
    return make_float2(m, __fadd_rn(__fmul_rn(a.y, scale_to(a.x, m, c)), __fmul_rn(b.y, scale_to(b.x, m, c))));
}

// The whole cluster's (maximum, sum), the same on every thread: warp shuffles, the block's 16 warps, and the blocks'
// results through distributed shared memory.  The caller has arrived at the cluster barrier once since the kernel's
// start (so that the peers run) and not waited; nothing touches a peer's memory after the call.
__device__ float2 cluster_join(float2 v, float c, int rank, int log_c, float2* scratch, float2* from_peers) {
#pragma unroll
    for (int o = 16; o; o >>= 1)
        v = join(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, o), __shfl_xor_sync(0xffffffffu, v.y, o)), c);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    __syncthreads();                              // the last reader of scratch is done
    if (lane == 0) scratch[warp] = v;
    __syncthreads();
    v = scratch[lane % kWarps];
#pragma unroll
    for (int o = kWarps / 2; o; o >>= 1)
        v = join(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, o), __shfl_xor_sync(0xffffffffu, v.y, o)), c);
    if (log_c == 0) return v;
    cluster_wait();
    if (threadIdx.x < 1 << log_c) peer_store(peer_address(&from_peers[rank], threadIdx.x), v.x, v.y);
    cluster_arrive();
    cluster_wait();
    v = from_peers[0];
    for (int i = 1; i < 1 << log_c; ++i) v = join(v, from_peers[i], c);
    return v;
}

// log of a sum of exponentials from its maximum, the scaled maximum and the sum of exp(x - max)
__device__ __forceinline__ float log_sum(float m, float scaled_m, float sum) {
    if (sum != sum) return sum;
    return m == -INFINITY || m == INFINITY ? m : scaled_m + logf(sum);
}

// The sum of 2^((x - m) c) over a vector, m >= all of x, m finite; NaN stays NaN.
template <class T> __device__ __forceinline__ float exp_sum(uint4 v, float m, float c) {
    float f[kPerVec<T>];
    Vec<T>::unpack(v, f);
#pragma unroll
    for (int j = 0; j < kPerVec<T>; ++j) f[j] = exp2_approx((f[j] - m) * c);
#pragma unroll
    for (int w = kPerVec<T> / 2; w; w /= 2)
#pragma unroll
        for (int j = 0; j < w; ++j) f[j] += f[j + w];
    return f[0];
}
// ... for a maximum of +inf: the infinite ones count 1
template <class T> __device__ __noinline__ float exp_sum_inf(uint4 v) {
    float f[kPerVec<T>], r = 0.f;
    Vec<T>::unpack(v, f);
    for (int j = 0; j < kPerVec<T>; ++j) r += f[j] == INFINITY ? 1.f : f[j] == f[j] ? 0.f : f[j];
    return r;
}

// Where a token of the row lies: its layer, and its position there.
struct Place {
    int rank, layer, position;
};
template <class T>
__device__ __forceinline__ Place place_of(const LogitsCut& in, const Deal& d, int64_t row, int token) {
    const int s = in.tp == 1 ? 0 : token / in.cols;
    int       q = token - s * in.cols;
    if (!d.aligned) q += (int)((uintptr_t)row_of<T>(in, s, row) & 15) / (int)sizeof(T);
    const int l = s * d.per_shard + q / kPerLayer<T>;
    return {l & ((1 << d.log_c) - 1), l >> d.log_c, q % kPerLayer<T>};
}
__device__ __forceinline__ int layers_of(const Deal& d, int rank) { return max(0, (d.layers - rank + (1 << d.log_c) - 1) >> d.log_c); }

// One bit per element of the block's share, a byte per vector, for the few elements that need more than the others.
__device__ __forceinline__ void set_flag(uint32_t* flags, int layer, int vec, int element) {
    const int byte = layer * kThreads + vec;
    atomicOr(&flags[byte >> 2], 1u << ((byte & 3) * 8 + element));
}

// ---- penalties, biases, masks --------------------------------------------------------------------------------
//
// A sweep over the row with everything that is sparse prepared in shared memory: one counter per column of the block's
// share (the history is read once per block and lands there with shared-memory atomics: sums of whole numbers, so that
// no order shows), and a hash table of the bias entries with one flag per column that has one.  The elements go from
// memory through registers to memory; the running (maximum, its id, sum of exponentials) stays on the thread.

constexpr int kHash = 2048;               // slots of the bias table, over twice NEREUS_BIAS_MAX

// Counter of a column: the top bit "in the history", the others "generated so often".
template <class Count> constexpr uint32_t kSeen = 1u << (sizeof(Count) * 8 - 1);

template <class Count> __device__ __forceinline__ void count_token(uint32_t* words, int column, bool generated) {
    if (sizeof(Count) == 4) {
        atomicOr(&words[column], kSeen<Count>);
        if (generated) atomicAdd(&words[column], 1u);
    } else {
        const int shift = (column & 1) * 16;
        atomicOr(&words[column >> 1], kSeen<Count> << shift);
        if (generated) atomicAdd(&words[column >> 1], 1u << shift);
    }
}

template <class TI, class TO, class Count>
__global__ void __launch_bounds__(kThreads) process_kernel(const __grid_constant__ LogitsCut in,
                                                           const __grid_constant__ LogitsCut out, Deal deal,
                                                           const __grid_constant__ nereus_penalties_t how, int32_t* token,
                                                           float* lse) {
    constexpr int E = kPerVec<TI>;
    extern __shared__ __align__(16) unsigned char dynamic[];
    __shared__ float2 scratch[kWarps], from_peers[kMaxCtas];
    __shared__ int    id_scratch[kWarps], id_peers[kMaxCtas];
    const int     tid = threadIdx.x, rank = blockIdx.x & ((1 << deal.log_c) - 1);
    const int64_t row = blockIdx.x >> deal.log_c;
    if (deal.log_c) cluster_arrive();

    Layer*    table = reinterpret_cast<Layer*>(dynamic);
    uint32_t* flags = reinterpret_cast<uint32_t*>(table + deal.mine);
    uint32_t* hash = flags + (how.bias_ids ? deal.mine * kThreads / 4 : 0);
    uint32_t* counters = hash + (how.bias_ids ? 2 * kHash : 0);
    int32_t*  hash_id = reinterpret_cast<int32_t*>(hash);
    int32_t*  hash_entry = hash_id + kHash;

    const float rho = how.repetition ? how.repetition[row] : 1.f;
    const float pres = how.presence ? how.presence[row] : 0.f, freq = how.frequency ? how.frequency[row] : 0.f;
    int total = 0, prompt = 0;
    if (how.history) {
        total = how.total_len ? max(0, min((int)how.history_len, how.total_len[row])) : (int)how.history_len;
        prompt = how.prompt_len ? how.prompt_len[row] : 0;
    }
    const int32_t* hist = how.history + (how.history ? row * how.history_stride : 0);
    const int64_t  mrow = how.mask ? (how.mask_row ? how.mask_row[row] : row) : -1;
    const int32_t* mask = mrow >= 0 && mrow < how.mask_rows ? how.mask + mrow * how.mask_stride : nullptr;
    const int      mask_last = (in.vocab - 1) >> 5;

    const int n_all = layers_of(deal, rank);
    float m = -INFINITY, sum = 0.f;
    int   at = 0x7fffffff;
    for (int first = 0; first < n_all; first += deal.mine) {       // one round unless the counters do not fit
        const int n = min(deal.mine, n_all - first);
        __syncthreads();
        if (tid < n) table[tid] = layer_of<TI, TO>(in, out, deal, row, rank, first + tid);
        if (total > 0)
            for (int i = tid; i < n * kThreads * E * (int)sizeof(Count) / 16; i += kThreads)
                reinterpret_cast<uint4*>(counters)[i] = make_uint4(0, 0, 0, 0);
        if (how.bias_ids) {
            for (int i = tid; i < n * kThreads / 4; i += kThreads) flags[i] = 0;
            for (int i = tid; i < 2 * kHash; i += kThreads) hash_id[i] = -1;
        }
        __syncthreads();
        for (int i = tid; i < total; i += kThreads) {
            const int id = hist[i];
            if ((uint32_t)id >= (uint32_t)in.vocab) continue;
            const Place p = place_of<TI>(in, deal, row, id);
            const int   l = p.layer - first;
            if (p.rank == rank && (uint32_t)l < (uint32_t)n) count_token<Count>(counters, l * kPerLayer<TI> + p.position, i >= prompt);
        }
        if (how.bias_ids)
            for (int i = tid; i < how.bias_count; i += kThreads) {
                const int id = how.bias_ids[row * how.bias_count + i];
                if ((uint32_t)id >= (uint32_t)in.vocab) continue;
                const Place p = place_of<TI>(in, deal, row, id);
                const int   l = p.layer - first;
                if (p.rank != rank || (uint32_t)l >= (uint32_t)n) continue;
                set_flag(flags, l, p.position / E, p.position % E);
                uint32_t h = (uint32_t)id * 2654435761u % kHash;
                for (int probe = 0; probe < kHash; ++probe, h = (h + 1) % kHash) {
                    const int was = atomicCAS(&hash_id[h], -1, id);
                    if (was == -1 || was == id) { atomicMax(&hash_entry[h], i); break; }
                }
            }
        __syncthreads();
        const int p0 = tid * E;
#pragma unroll 2
        for (int l = 0; l < n; ++l) {
            const Layer L = table[l];
            if (p0 >= L.hi || p0 + E <= L.lo) continue;
            const bool whole = p0 >= L.lo && p0 + E <= L.hi;
            float x[E];
            if (whole) {
                Vec<TI>::unpack(__ldcs(reinterpret_cast<const uint4*>(L.in + tid * 16)), x);
            } else {
#pragma unroll
                for (int j = 0; j < E; ++j)
                    x[j] = p0 + j >= L.lo && p0 + j < L.hi ? to_float(reinterpret_cast<const TI*>(L.in)[p0 + j]) : -INFINITY;
            }
            const int v0 = L.token + p0;
            if (total > 0) {
                uint32_t c[E];
                uint32_t any = 0;
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    c[j] = reinterpret_cast<const Count*>(counters)[l * kPerLayer<TI> + p0 + j];
                    any |= c[j];
                }
                if (any) {
#pragma unroll
                    for (int j = 0; j < E; ++j) {
                        if (!c[j]) continue;
                        x[j] = x[j] > 0.f ? __fdiv_rn(x[j], rho) : __fmul_rn(x[j], rho);
                        if (const uint32_t k = c[j] & (kSeen<Count> - 1))
                            x[j] = __fsub_rn(__fsub_rn(x[j], __fmul_rn(freq, (float)k)), pres);
                    }
                }
            }
            if (how.bias_ids) {
                if (const uint32_t f = reinterpret_cast<const uint8_t*>(flags)[l * kThreads + tid]) {
#pragma unroll
                    for (int j = 0; j < E; ++j) {
                        if (!(f >> j & 1)) continue;
                        uint32_t h = (uint32_t)(v0 + j) * 2654435761u % kHash;
                        for (int probe = 0; probe < kHash && hash_id[h] != v0 + j; ++probe) h = (h + 1) % kHash;
                        x[j] = __fadd_rn(x[j], how.bias_values[row * how.bias_count + hash_entry[h]]);
                    }
                }
            }
            if (mask) {
                const int      w = max(v0, 0) >> 5;
                const uint32_t low = (uint32_t)mask[w], high = (uint32_t)mask[min(w + 1, mask_last)];
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    const int v = v0 + j;
                    const uint32_t word = v >> 5 == w ? low : high;
                    if (!(word >> (v & 31) & 1u)) x[j] = -INFINITY;
                }
            }
            // written, and from here on what was written
            TO y[E];
            float top = -INFINITY;
#pragma unroll
            for (int j = 0; j < E; ++j) {
                y[j] = from_float<TO>(x[j]);
                x[j] = to_float(y[j]);
                top = fmaxf(top, x[j]);
            }
            if (whole && L.vec_out) {
                const uint4* w = reinterpret_cast<const uint4*>(y);
                uint4*       o = reinterpret_cast<uint4*>(L.out + p0 * (int)sizeof(TO));
#pragma unroll
                for (int j = 0; j < E * (int)sizeof(TO) / 16; ++j) __stcs(o + j, w[j]);
            } else {
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    if (p0 + j >= L.lo && p0 + j < L.hi) reinterpret_cast<TO*>(L.out)[p0 + j] = y[j];
                    else x[j] = -INFINITY;
                }
            }
            if (top > m) {
                sum *= scale_to(m, top, kLog2e);
                m = top;
#pragma unroll
                for (int j = E - 1; j >= 0; --j)
                    if (x[j] == top) at = v0 + j;
            }
            if (m == INFINITY) {
                for (int j = 0; j < E; ++j) sum += x[j] == INFINITY ? 1.f : x[j] == x[j] ? 0.f : x[j];
            } else {
                const float base = m == -INFINITY ? 0.f : m;
                float       part = 0.f;
#pragma unroll
                for (int j = 0; j < E; ++j) part += exp2_approx((x[j] - base) * kLog2e);
                sum += part;
            }
        }
    }

    // the block's result, and the cluster's on its first block
    const float mine = m;
    float2 v = make_float2(m, sum);
#pragma unroll
    for (int o = 16; o; o >>= 1)
        v = join(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, o), __shfl_xor_sync(0xffffffffu, v.y, o)), kLog2e);
    const int warp_at = (int)__reduce_min_sync(0xffffffffu, mine == v.x ? (uint32_t)at : 0x7fffffffu);
    if ((tid & 31) == 0) { scratch[tid >> 5] = v; id_scratch[tid >> 5] = warp_at; }
    __syncthreads();
    if (deal.log_c) cluster_wait();
    if (tid == 0) {
        v = scratch[0];
        int id = id_scratch[0];
        for (int i = 1; i < kWarps; ++i) {
            if (scratch[i].x > v.x) id = id_scratch[i];
            else if (scratch[i].x == v.x) id = min(id, id_scratch[i]);
            v = join(v, scratch[i], kLog2e);
        }
        if (deal.log_c) {
            peer_store(peer_address(&from_peers[rank], 0), v.x, v.y);
            asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(peer_address(&id_peers[rank], 0)), "r"(id) : "memory");
        } else {
            from_peers[0] = v;
            id_peers[0] = id;
        }
    }
    if (deal.log_c) { __syncwarp(); cluster_arrive(); cluster_wait(); }
    if (rank == 0 && tid == 0) {
        v = from_peers[0];
        int id = id_peers[0];
        for (int i = 1; i < 1 << deal.log_c; ++i) {
            if (from_peers[i].x > v.x) id = id_peers[i];
            else if (from_peers[i].x == v.x) id = min(id, id_peers[i]);
            v = join(v, from_peers[i], kLog2e);
        }
        if (token) token[row] = v.x > -INFINITY ? id : -1;
        if (lse) lse[row] = log_sum(v.x, v.x, v.y);
    }
}

// ---- a teacher's top logits ----------------------------------------------------------------------------------
//
// Every thread knows the largest of its own elements after the pass that also sums the exponentials.  The k-th largest
// of a block's 512 such maxima bounds the block's k-th largest element from below, whatever the order of the row, and
// few elements reach it (those of the k threads, and what else of theirs does); only the threads whose maximum reaches
// it look through their elements again, in shared memory.  What they find is ranked by counting, (value, lower id)
// as one 64-bit key, and the blocks' lists are joined by binary search.  Rows with so many equal values that the list
// would overflow take an exact search for the k-th key and the id to cut at.

constexpr int kCandidates = 1024;

// orders as the values do, -0 as +0; NaN below everything
__device__ __forceinline__ uint32_t key_of(float x) {
    if (x != x) return 0u;
    const uint32_t u = __float_as_uint(x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) {
    return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}
constexpr uint32_t kKeyMinusInf = 0x007fffffu;

__device__ __forceinline__ int block_count(int v, int* scratch) {
    v = __reduce_add_sync(0xffffffffu, v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    int r = 0;
    for (int i = 0; i < kWarps; ++i) r += scratch[i];
    return r;
}

template <class T>
__global__ void __launch_bounds__(kThreads) top_kernel(const __grid_constant__ LogitsCut in, Deal deal, int k, float inv_t,
                                                       float* values, int32_t* ids, float* lse) {
    constexpr int E = kPerVec<T>;
    extern __shared__ __align__(16) unsigned char dynamic[];
    __shared__ float2 scratch[kWarps];
    __shared__ int    count_scratch[kWarps];
    __shared__ unsigned long long found[kCandidates];
    __shared__ unsigned long long best[NEREUS_TOP_MAX_K];          // the block's own, falling, 0 where there are fewer
    __shared__ float2 stats;                                       // (maximum, sum) of the block
    __shared__ int    n_found;
    const int     tid = threadIdx.x, ctas = 1 << deal.log_c, rank = blockIdx.x & (ctas - 1);
    const int64_t row = blockIdx.x >> deal.log_c;
    const int     n = layers_of(deal, rank), quarter = (n + 3) / 4;
    const float   c = inv_t * kLog2e;

    Layer* table = reinterpret_cast<Layer*>(dynamic);
    uint4* slots = reinterpret_cast<uint4*>(table + deal.mine);
    if (tid < n) table[tid] = layer_of<T, T>(in, LogitsCut(), deal, row, rank, tid);
    if (tid == 0) n_found = 0;
    if (tid < k) best[tid] = 0;
    __syncthreads();
    load_share<T>(table, slots, n, quarter);

    float m = -INFINITY, sum = 0.f;
    on_arrival<T>(table, n, quarter, [&](int i) { m = fmaxf(m, Vec<T>::max(slots[i * kThreads + tid])); });
    const int p0 = tid * E;
    if (m == INFINITY) {
        for (int i = 0; i < n; ++i)
            if (p0 < table[i].hi && p0 + E > table[i].lo) sum += exp_sum_inf<T>(slots[i * kThreads + tid]);
    } else {
        const float base = m == -INFINITY ? 0.f : m;
#pragma unroll 2
        for (int i = 0; i < n; ++i)
            if (p0 < table[i].hi && p0 + E > table[i].lo) sum += exp_sum<T>(slots[i * kThreads + tid], base, c);
    }

    // the k-th largest of the threads' maxima, to 16 bits from below
    uint32_t       t = 0;
    const uint32_t key = key_of(m);
#pragma unroll 1
    for (int bit = 31; bit >= 16; --bit)
        if (__syncthreads_count(key >= (t | 1u << bit)) >= k) t |= 1u << bit;
    t = max(t, kKeyMinusInf);
    const float bound = value_of(t);
    // every element of this thread's share that is not NaN: f(key, token)
    auto each = [&](float least, auto f) {
        for (int i = 0; i < n; ++i) {
            const Layer& L = table[i];
            if (p0 >= L.hi || p0 + E <= L.lo) continue;
            const uint4 v = slots[i * kThreads + tid];
            if (!(Vec<T>::max(v) >= least)) continue;
            float x[E];
            Vec<T>::unpack(v, x);
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (x[j] >= least && p0 + j >= L.lo && p0 + j < L.hi) f(key_of(x[j]), L.token + p0 + j);
        }
    };
    auto push = [&](uint32_t kk, int v) {
        const int i = atomicAdd(&n_found, 1);
        if (i < kCandidates) found[i] = (unsigned long long)kk << 32 | (0xffffffffu - (uint32_t)v);
    };
    if (m >= bound) each(bound, push);

    // meanwhile the block's sum
    float2 v = make_float2(m, sum);
#pragma unroll
    for (int o = 16; o; o >>= 1)
        v = join(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, o), __shfl_xor_sync(0xffffffffu, v.y, o)), c);
    if ((tid & 31) == 0) scratch[tid >> 5] = v;
    __syncthreads();
    if (tid == 0) {
        v = scratch[0];
        for (int i = 1; i < kWarps; ++i) v = join(v, scratch[i], c);
        stats = v;
    }
    if (n_found > kCandidates) {
        uint32_t kth = 0;                      // the largest key that k elements reach, 0 if there are fewer
#pragma unroll 1
        for (int bit = 31; bit >= 0; --bit) {
            int reach = 0;
            each(-INFINITY, [&](uint32_t kk, int) { reach += kk >= (kth | 1u << bit); });
            if (block_count(reach, count_scratch) >= k) kth |= 1u << bit;
        }
        int above = 0;
        each(-INFINITY, [&](uint32_t kk, int) { above += kk > kth; });
        above = block_count(above, count_scratch);
        int before = -1;                       // the largest id up to which fewer than k are taken
#pragma unroll 1
        for (int bit = 23; bit >= 0; --bit) {
            int reach = 0;
            each(-INFINITY, [&](uint32_t kk, int id) { reach += kk == kth && id <= before + (1 << bit); });
            if (above + block_count(reach, count_scratch) < k) before += 1 << bit;
        }
        if (tid == 0) n_found = 0;
        __syncthreads();
        each(-INFINITY, [&](uint32_t kk, int id) { if (kk > kth || (kk == kth && id <= before + 1)) push(kk, id); });
        __syncthreads();
    }
    const int n_list = n_found;
    for (int i = tid; i < n_list; i += kThreads) {
        const unsigned long long mine = found[i];
        int place = 0;
        for (int j = 0; j < n_list; ++j) place += found[j] > mine;
        if (place < k) best[place] = mine;
    }
    __syncthreads();

    unsigned long long mine = tid < k ? best[tid] : 0;
    int  place = tid;
    if (deal.log_c) {
        // the lists of all blocks, side by side where the row was: nothing reads its elements any more
        unsigned long long* lists = reinterpret_cast<unsigned long long*>(slots);
        cluster_arrive();
        cluster_wait();
        for (int i = tid; i < ctas * k; i += kThreads) lists[i] = peer_load64(peer_address(&best[i % k], i / k));
        if (tid < ctas) {
            const unsigned long long w = peer_load64(peer_address(&stats, tid));
            scratch[tid] = make_float2(__uint_as_float((uint32_t)w), __uint_as_float((uint32_t)(w >> 32)));
        }
        cluster_arrive();
        __syncthreads();
        if (mine)
            for (int r = 0; r < ctas; ++r) {
                if (r == rank) continue;
                int lo = 0, hi = k;            // how many of list r are larger
                while (lo < hi) {
                    const int mid = (lo + hi) / 2;
                    if (lists[r * k + mid] > mine) lo = mid + 1; else hi = mid;
                }
                place += lo;
            }
    }
    if (mine && place < k) {
        values[row * k + place] = value_of((uint32_t)(mine >> 32));
        ids[row * k + place] = (int32_t)(0xffffffffu - (uint32_t)mine);
    }
    if (rank == 0) {
        // places that no element takes
        int have = mine != 0;
        if (deal.log_c) {
            have = 0;
            const unsigned long long* lists = reinterpret_cast<const unsigned long long*>(slots);
            for (int i = tid; i < ctas * k; i += kThreads) have += lists[i] != 0;
        }
        have = block_count(have, count_scratch);
        if (tid >= have && tid < k) { values[row * k + tid] = -INFINITY; ids[row * k + tid] = -1; }
        if (tid == 0) {
            v = stats;
            if (deal.log_c) {
                v = scratch[0];
                for (int i = 1; i < ctas; ++i) v = join(v, scratch[i], c);
            }
            lse[row] = log_sum(v.x, v.x * inv_t, v.y);
        }
    }
    if (deal.log_c) cluster_wait();            // the peers have read this block's list
}

// ---- distillation --------------------------------------------------------------------------------------------
//
// The sum over the rest is taken on its own, with the entries' elements left out (one flag bit per element): as the
// difference of the whole sum and the entries' it would lose its digits where the entries hold nearly all of the mass.
// The gradient of a token of the rest is exp((x - m) / T) times one number per row; the entries' gradients are worked out
// by one thread each and left in the elements' places in shared memory, from where they go out with the others.

enum Pass { kForward, kBackward, kStep };

template <class T, int kPass>
__global__ void __launch_bounds__(kThreads) distill_kernel(const __grid_constant__ LogitsCut in,
                                                           const __grid_constant__ LogitsCut grad, Deal deal,
                                                           const __grid_constant__ nereus_distill_t how, float* loss,
                                                           float* saved, const float* grad_loss) {
    constexpr int E = kPerVec<T>;
    extern __shared__ __align__(16) unsigned char dynamic[];
    __shared__ float2 scratch[kWarps], from_peers[kMaxCtas];
    const int     k = how.k, tid = threadIdx.x, rank = blockIdx.x & ((1 << deal.log_c) - 1), p0 = tid * E;
    const int64_t row = blockIdx.x >> deal.log_c;
    const int     n = layers_of(deal, rank), quarter = (n + 3) / 4;
    float         weight = how.weight ? how.weight[row] : 1.f;

    Layer*    table = reinterpret_cast<Layer*>(dynamic);
    uint4*    slots = reinterpret_cast<uint4*>(table + deal.mine);
    uint32_t* flags = reinterpret_cast<uint32_t*>(slots + deal.mine * kThreads);
    if (tid < n) table[tid] = layer_of<T, T>(in, grad, deal, row, rank, tid);
    if (weight == 0.f) {
        if (rank == 0 && tid == 0 && kPass != kBackward) loss[row] = 0.f;
        if (rank == 0 && tid < 4 && kPass == kForward) saved[row * 4 + tid] = 0.f;
        if (kPass != kForward) {
            __syncthreads();
            for (int i = 0; i < n; ++i)
                if (p0 < table[i].hi && p0 + E > table[i].lo) store_vector<T>(table[i], make_uint4(0, 0, 0, 0));
        }
        return;
    }
    if (kPass != kBackward && deal.log_c) cluster_arrive();       // the peers run, for cluster_join
    for (int i = tid; i < n * kThreads / 4; i += kThreads) flags[i] = 0;
    __syncthreads();
    load_share<T>(table, slots, n, quarter);

    // entry `tid`: teacher and student, and its place if the block holds it
    const float t = how.temperature, c = kLog2e / t;
    int id = tid < k ? how.ids[row * k + tid] : -1;
    if ((uint32_t)id >= (uint32_t)in.vocab) id = -1;
    const float y = id >= 0 ? how.values[row * k + tid] : 0.f;
    float x = 0.f;
    T*    slot = nullptr;
    if (id >= 0) {
        const Place p = place_of<T>(in, deal, row, id);
        const int   s = in.tp == 1 ? 0 : id / in.cols;
        x = to_float(row_of<T>(in, s, row)[id - s * in.cols]);
        if (p.rank == rank) {
            slot = reinterpret_cast<T*>(slots + p.layer * kThreads) + p.position;
            set_flag(flags, p.layer, p.position / E, p.position % E);
        }
    }
    // a block may overwrite the logits once all blocks have read the entries' (cluster_join orders the other passes)
    if (kPass == kBackward && deal.log_c) cluster_arrive();
    const float lse = how.lse ? how.lse[row] : block_max(id >= 0 ? y : -INFINITY, scratch);
    float log_p, p, p_rest, mass = 1.f;
    int   entries;
    if (how.lse) {
        log_p = y / t - lse;
        p = id >= 0 ? expf(log_p) : 0.f;
        const float2 s = block_sum2(p, id >= 0 ? 1.f : 0.f, scratch);
        entries = (int)s.y;
        p_rest = entries < in.vocab ? fmaxf(0.f, 1.f - s.x) : 0.f;
    } else {
        const float  e = id >= 0 ? expf((y - lse) / t) : 0.f;
        const float2 s = block_sum2(e, id >= 0 ? 1.f : 0.f, scratch);
        entries = (int)s.y;
        log_p = (y - lse) / t - logf(s.x);
        p = entries ? e / s.x : 0.f;
        p_rest = 0.f;
        if (!entries) mass = 0.f;
    }                                             // (the sums' barriers also publish the flags)

    const uint8_t* flag_of = reinterpret_cast<const uint8_t*>(flags) + tid;
    float m, total, rest;
    if (kPass == kBackward) {
        m = saved[row * 4]; total = saved[row * 4 + 1]; rest = saved[row * 4 + 2];
        copy_wait<0>();
        __syncthreads();
    } else {
        m = -INFINITY;
        on_arrival<T>(table, n, quarter, [&](int i) { m = fmaxf(m, Vec<T>::max(slots[i * kThreads + tid])); });
        const float base = m == -INFINITY ? 0.f : m;
        float       sum = 0.f;
#pragma unroll 2
        for (int i = 0; i < n; ++i) {
            if (p0 >= table[i].hi || p0 + E <= table[i].lo) continue;
            uint4 v = slots[i * kThreads + tid];
            if (const uint32_t f = flag_of[i * kThreads]) {
                float e[E];
                Vec<T>::unpack(v, e);
#pragma unroll
                for (int j = 0; j < E; ++j)
                    if (f >> j & 1) e[j] = -INFINITY;
                v = Vec<T>::pack(e);
            }
            sum += exp_sum<T>(v, base, c);
        }
        const float2 all = cluster_join(make_float2(m, sum), c, rank, deal.log_c, scratch, from_peers);
        m = all.x;
        rest = all.y;
        total = rest + block_sum2(id >= 0 ? expf((x - m) / t) : 0.f, 0.f, scratch).x;
    }

    // the groups: entry `tid` on its thread, the rest on all
    const float log_total = logf(total);
    const float log_q = (x - m) / t - log_total, q = expf(log_q);
    const float log_q_rest = logf(rest) - log_total, q_rest = rest / total;
    float term = 0.f, qf = 0.f, slope = 0.f, term_rest = 0.f, qf_rest = 0.f, slope_rest = 0.f;
    if (how.divergence == NEREUS_FORWARD_KL) {
        if (p > 0.f) term = p * (log_p - log_q);
        if (p_rest > 0.f) term_rest = p_rest * (logf(p_rest) - log_q_rest);
    } else if (how.divergence == NEREUS_REVERSE_KL) {
        p_rest = fmaxf(p_rest, 5.9604644775390625e-8f);
        if (q > 0.f && id >= 0) { slope = log_q - log_p; term = qf = q * slope; }
        if (q_rest > 0.f) { slope_rest = log_q_rest - logf(p_rest); term_rest = qf_rest = q_rest * slope_rest; }
    } else {
        const float a = how.beta, b = 1.f - how.beta;
        if (id >= 0) {
            const float log_m = logf(a * p + b * q);
            if (q > 0.f) { slope = b * (log_q - log_m); qf = q * slope; }
            term = qf + (p > 0.f ? a * p * (log_p - log_m) : 0.f);
        }
        const float log_m = logf(a * p_rest + b * q_rest);
        if (q_rest > 0.f) { slope_rest = b * (log_q_rest - log_m); qf_rest = q_rest * slope_rest; }
        term_rest = qf_rest + (p_rest > 0.f ? a * p_rest * (logf(p_rest) - log_m) : 0.f);
    }
    const float2 sums = block_sum2(id >= 0 ? term : 0.f, qf, scratch);
    const float  d = sums.x + term_rest, mean = sums.y + qf_rest;
    if (rank == 0 && tid == 0) {
        if (kPass != kBackward) loss[row] = weight * d;
        if (kPass == kForward) {
            float* const o = saved + row * 4;
            o[0] = m; o[1] = total; o[2] = rest; o[3] = d;
        }
    }
    if (kPass == kForward) return;
    if (kPass == kBackward && grad_loss) weight *= grad_loss[row];
    const float scale = weight / t;
    float g, rest_scale;
    if (how.divergence == NEREUS_FORWARD_KL) {    // Q f and Q sum Q f, which stay finite where Q is 0
        g = (mass * q - p) * scale;
        rest_scale = (mass - (p_rest > 0.f && rest > 0.f ? p_rest / q_rest : 0.f)) * scale / total;
    } else {
        g = q > 0.f ? q * (slope - mean) * scale : 0.f;
        rest_scale = (slope_rest - mean) * scale / total;
    }
    if (slot) *slot = from_float<T>(g);
    if (kPass == kBackward && deal.log_c) cluster_wait();
    __syncthreads();
#pragma unroll 2
    for (int i = 0; i < n; ++i) {
        if (p0 >= table[i].hi || p0 + E <= table[i].lo) continue;
        const uint4 raw = slots[i * kThreads + tid];
        float       e[E];
        Vec<T>::unpack(raw, e);
#pragma unroll
        for (int j = 0; j < E; ++j) e[j] = exp2_approx((e[j] - m) * c) * rest_scale;
        if (const uint32_t f = flag_of[i * kThreads]) {
            float ready[E];
            Vec<T>::unpack(raw, ready);
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (f >> j & 1) e[j] = ready[j];
        }
        store_vector<T>(table[i], Vec<T>::pack(e));
    }
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

constexpr int kMaxDevices = 64;
constexpr int kSmemShare  = 73 * 1024;      // shared memory per block for which three blocks fit on an SM

struct Device {
    int sms = 0, smem = 0;
};
// The current device's numbers, looked up once.
int device_of(Device* d) {
    static std::atomic<int> sms[kMaxDevices], smem[kMaxDevices];
    int dev = 0, n = 0, m = 0;
    NEREUS_CUDA(cudaGetDevice(&dev));
    if (dev < 0 || dev >= kMaxDevices) return NEREUS_ERR_UNSUPPORTED;
    n = sms[dev].load();
    m = smem[dev].load();
    if (!n || !m) {
        NEREUS_CUDA(cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev));
        NEREUS_CUDA(cudaDeviceGetAttribute(&m, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev));
        sms[dev].store(n);
        smem[dev].store(m);
    }
    d->sms = n;
    d->smem = m;
    return NEREUS_OK;
}

// Deals a row out so that a block's share takes at most kSmemShare bytes at `per_layer` a layer and `fixed` once, and
// further while rows x blocks stay within the SMs.
Deal deal_of(const nereus_logits_t& v, int64_t per_layer, int64_t fixed, int sms) {
    Deal d;
    const int64_t e = 16 / size_of(v.dtype), w = held_cols(v, 0), bytes = v.row_stride * size_of(v.dtype);
    d.aligned = v.rows < 2 || bytes % 16 == 0;
    for (int s = 0; s < v.tp; ++s)
        if (held_cols(v, s) && (uintptr_t)v.shard[s] % 16) d.aligned = 0;
    const int64_t vecs = d.aligned ? (w + e - 1) / e : (w + 2 * e - 2) / e;
    const int64_t used = (v.vocab + v.shard_cols - 1) / v.shard_cols;
    d.per_shard = (int)((vecs + kThreads - 1) / kThreads);
    d.layers = (int)(d.per_shard * used);
    d.log_c = 0;
    auto share = [&] { return (int64_t)(d.layers + (1 << d.log_c) - 1) >> d.log_c; };
    while (d.log_c < 3 && share() * per_layer + fixed > kSmemShare) ++d.log_c;
    while (d.log_c < 3 && (2 << d.log_c) <= d.layers && (v.rows << d.log_c) * 2 <= sms) ++d.log_c;
    d.mine = (int)share();
    return d;
}

// Launches a kernel with a cluster of blocks per row.
template <class... P, class... A>
int launch(void (*kernel)(P...), std::atomic<int>* opted, int64_t rows, const Deal& d, int64_t smem, const Device& dev,
           cudaStream_t stream, A... args) {
    if (smem > dev.smem - 16384) return NEREUS_ERR_TOO_LARGE;          // 16 KiB: the kernels' static part
    if (smem > 32768 && opted->load() < smem) {
        // the largest any call will ask for, so that this happens once
        NEREUS_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, dev.smem - 16384));
        opted->store(dev.smem);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(rows << d.log_c));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr = {};
    if (d.log_c) {
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = 1u << d.log_c;
        attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
    }
    NEREUS_CUDA(cudaLaunchKernelEx(&cfg, kernel, args...));
    return NEREUS_OK;
}

template <class T, int kPass>
int distill_launch(const nereus_logits_t& in, const nereus_distill_t& how, float* loss, float* saved,
                   const float* grad_loss, const nereus_logits_t* grad, cudaStream_t stream) {
    static std::atomic<int> opted[kMaxDevices];
    Device dev;
    if (int rc = device_of(&dev)) return rc;
    int id = 0;
    NEREUS_CUDA(cudaGetDevice(&id));
    const int64_t per_layer = sizeof(Layer) + kThreads * 17;
    const Deal    d = deal_of(in, per_layer, 0, dev.sms);
    return launch(distill_kernel<T, kPass>, &opted[id], in.rows, d, d.mine * per_layer, dev, stream,
                  cut_of(in), kPass == kForward ? LogitsCut() : cut_of(*grad), d, how, loss, saved, grad_loss);
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
    auto go = in->dtype == NEREUS_BF16 ? distill_launch<__nv_bfloat16, kPass> : distill_launch<float, kPass>;
    return go(*in, *how, loss, saved, grad_loss, grad, (cudaStream_t)stream);
}

template <class TI, class TO, class Count>
int process_launch(const nereus_logits_t& in, const nereus_logits_t& out, const nereus_penalties_t& how, int32_t* token,
                   float* lse, cudaStream_t stream) {
    static std::atomic<int> opted[kMaxDevices];
    Device dev;
    if (int rc = device_of(&dev)) return rc;
    int id = 0;
    NEREUS_CUDA(cudaGetDevice(&id));
    const int64_t per_layer = sizeof(Layer) + (how.history ? kPerLayer<TI> * sizeof(Count) : 0) + (how.bias_ids ? kThreads : 0);
    const int64_t fixed = how.bias_ids ? 2 * kHash * 4 : 0;
    Deal d = deal_of(in, per_layer, fixed, dev.sms);
    // what does not fit is done in rounds
    while (d.mine > 1 && (d.mine * per_layer + fixed > dev.smem - 16384 || d.mine > kThreads)) d.mine = (d.mine + 1) / 2;
    return launch(process_kernel<TI, TO, Count>, &opted[id], in.rows, d, d.mine * per_layer + fixed, dev, stream,
                  cut_of(in), cut_of(out), d, how, token, lse);
}

template <class T>
int top_launch(const nereus_logits_t& in, int k, float temperature, float* values, int32_t* ids, float* lse, cudaStream_t stream) {
    static std::atomic<int> opted[kMaxDevices];
    Device dev;
    if (int rc = device_of(&dev)) return rc;
    int id = 0;
    NEREUS_CUDA(cudaGetDevice(&id));
    const int64_t per_layer = sizeof(Layer) + kThreads * 16;
    const Deal    d = deal_of(in, per_layer, 0, dev.sms);
    // the slots also take the lists of all blocks of the cluster
    const int64_t lists = d.log_c ? ((int64_t)k << d.log_c) * 8 + d.mine * (int64_t)sizeof(Layer) : 0;
    return launch(top_kernel<T>, &opted[id], in.rows, d, std::max(d.mine * per_layer, lists), dev, stream, cut_of(in),
                  d, k, 1.f / temperature, values, ids, lse);
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
    // two bytes per column count a history shorter than 2^15
    const bool small = how->history_len < 32768;
    auto go = in->dtype == NEREUS_FP32 ? (small ? process_launch<float, float, uint16_t> : process_launch<float, float, uint32_t>)
              : out->dtype == NEREUS_FP32
                  ? (small ? process_launch<__nv_bfloat16, float, uint16_t> : process_launch<__nv_bfloat16, float, uint32_t>)
                  : (small ? process_launch<__nv_bfloat16, __nv_bfloat16, uint16_t>
                           : process_launch<__nv_bfloat16, __nv_bfloat16, uint32_t>);
    return go(*in, *out, *how, token, lse, (cudaStream_t)cuda_stream);
}

int nereus_teacher_top(const nereus_logits_t* in, int k, float temperature, float* values, int32_t* ids, float* lse,
                       void* cuda_stream) {
    if (int rc = check_view(in)) return rc;
    if (k < 1 || k > NEREUS_TOP_MAX_K || k > in->vocab) return NEREUS_ERR_ARG;
    if (!(temperature > 0.f) || !std::isfinite(temperature)) return NEREUS_ERR_ARG;
    if (misaligned(values) || misaligned(ids) || misaligned(lse)) return NEREUS_ERR_ALIGN;
    if (in->rows == 0) return NEREUS_OK;
    if (!values || !ids || !lse) return NEREUS_ERR_ARG;
    auto go = in->dtype == NEREUS_BF16 ? top_launch<__nv_bfloat16> : top_launch<float>;
    return go(*in, k, temperature, values, ids, lse, (cudaStream_t)cuda_stream);
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
