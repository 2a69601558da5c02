// What the kernels on an LM head's cut logits share (nereus_logits.cu, nereus_beam.cu): views of cut logits, how a row's vectors are
// dealt out to threads and blocks, its way through shared memory, running sums of exponentials, and on the host the checks
// of views and the launch.  Included by these two files alone; everything here is local to them.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "nereus_internal.hpp"

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
    float   per_col;      // 1 / cols
};

// How rows are dealt out: `per_shard` layers in every shard, `layers` in all, 1 << log_c blocks per row, `mine` layers
// (at most) per block.
struct Deal {
    int32_t per_shard, layers, log_c, mine;
    int32_t aligned;      // every row of every shard starts on a 16-byte boundary
};

constexpr int kThreads  = 256;
constexpr int kWide     = 512;                    // ... of the blocks that write a gradient
constexpr int kVecs     = 2 * kThreads;           // vectors of a layer: two a thread, in wide blocks too
constexpr int kWarps    = kThreads / 32;
constexpr int kMaxCtas  = 8;                      // portable cluster size
constexpr float kLog2e  = 1.4426950408889634f;

// One layer of the block's share: positions 0 .. kPerLayer - 1, of which [lo, hi) are the row's.
struct __align__(16) Layer {
    const char* in;       // address of position 0, 16-byte aligned; may lie before the row where lo > 0
    char*       out;      // ... of the written view, congruent to `in` or not
    int32_t     token;    // token of position 0; negative where lo > 0 in the first shard
    int32_t     lo, hi;
    int32_t     vec_out;  // `out` is 16-byte aligned too
};
static_assert(sizeof(Layer) == 32, "Layer is read as two 16-byte words");

template <class T> constexpr int kPerVec = 16 / (int)sizeof(T);
template <class T, int TH = kThreads> constexpr int kPerLayer = 2 * TH * kPerVec<T>;

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

// The layer of shard s that begins at vector position `first`, counted in elements; hi = 0 where the row has none there.
template <class TI, class TO, int TH>
__device__ __forceinline__ Layer layer_in(const LogitsCut& in, const LogitsCut& out, int64_t row, int s, int first) {
    Layer r = {nullptr, nullptr, 0, 0, 0, 0};
    const int w = width_of(in, s);
    if (!w) return r;
    const uintptr_t a = (uintptr_t)row_of<TI>(in, s, row);
    const int       phase = (int)(a & 15) / (int)sizeof(TI);       // the row starts at this position of its first vector
    r.in = (const char*)(a & ~(uintptr_t)15) + (int64_t)first * (int)sizeof(TI);
    r.lo = max(0, phase - first);
    r.hi = max(0, min(kPerLayer<TI, TH>, phase + w - first));
    r.token = s * in.cols + first - phase;
    if (out.tp) {
        r.out = (char*)row_of<TO>(out, s, row) + (int64_t)(first - phase) * (int)sizeof(TO);
        r.vec_out = ((uintptr_t)r.out & 15) == 0;
    }
    return r;
}
// Block `rank`'s i-th layer of a row.
template <class TI, class TO, int TH = kThreads>
__device__ __forceinline__ Layer layer_of(const LogitsCut& in, const LogitsCut& out, const Deal& d, int64_t row, int rank, int i) {
    const int l = (i << d.log_c) + rank;
    if (l >= d.layers) return {nullptr, nullptr, 0, 0, 0, 0};
    const int s = l / d.per_shard;
    return layer_in<TI, TO, TH>(in, out, row, s, (l - s * d.per_shard) * kPerLayer<TI, TH>);
}

// Two fp32 in one 64-bit register: sm_100 has add, mul and fma on pairs, which halves the instructions of the loops.
typedef unsigned long long Pair;
__device__ __forceinline__ Pair pair(float lo, float hi) {
    Pair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 halves(Pair p) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(p));
    return r;
}
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ float exp2_approx(float x) {              // relative error 2^-22, 0 at -inf
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ Pair exp2_pair(Pair p) {
    const float2 f = halves(p);
    return pair(exp2_approx(f.x), exp2_approx(f.y));
}

// A 16-byte vector as pairs of fp32, and back (bf16: round to nearest even).  `Max` accumulates maxima without
// unpacking; NaN is passed over.
template <class T> struct Vec;
template <> struct Vec<float> {
    static constexpr int kPairs = 2;
    typedef float Max;
    static __device__ __forceinline__ Max lowest() { return -INFINITY; }
    static __device__ __forceinline__ uint4 none() { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }
    static __device__ __forceinline__ void unpack(uint4 v, Pair (&p)[2]) {
        p[0] = pair(__uint_as_float(v.x), __uint_as_float(v.y));
        p[1] = pair(__uint_as_float(v.z), __uint_as_float(v.w));
    }
    static __device__ __forceinline__ uint4 pack(const Pair (&p)[2]) {
        const float2 a = halves(p[0]), b = halves(p[1]);
        return make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
    }
    static __device__ __forceinline__ Max join(Max a, Max b) { return fmaxf(a, b); }
    static __device__ __forceinline__ Max max(uint4 v) {
        return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
    }
    static __device__ __forceinline__ float value(Max m) { return m; }
};
template <> struct Vec<__nv_bfloat16> {
    static constexpr int kPairs = 4;
    typedef uint32_t Max;
    static __device__ __forceinline__ Max lowest() { return 0xff80ff80u; }
    static __device__ __forceinline__ uint4 none() { return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }
    static __device__ __forceinline__ Pair open(uint32_t w) { return pair(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
    static __device__ __forceinline__ uint32_t close(Pair p) {
        const float2 f = halves(p);
        uint32_t r;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(f.y), "f"(f.x));
        return r;
    }
    static __device__ __forceinline__ void unpack(uint4 v, Pair (&p)[4]) {
        p[0] = open(v.x); p[1] = open(v.y); p[2] = open(v.z); p[3] = open(v.w);
    }
    static __device__ __forceinline__ uint4 pack(const Pair (&p)[4]) {
        return make_uint4(close(p[0]), close(p[1]), close(p[2]), close(p[3]));
    }
    static __device__ __forceinline__ Max join(Max a, Max b) {
        uint32_t r;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static __device__ __forceinline__ Max max(uint4 v) { return join(join(v.x, v.y), join(v.z, v.w)); }
    static __device__ __forceinline__ float value(Max m) {
        return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
    }
};
template <class T> __device__ __forceinline__ void unpack(uint4 v, float (&f)[kPerVec<T>]) {
    Pair p[Vec<T>::kPairs];
    Vec<T>::unpack(v, p);
#pragma unroll
    for (int i = 0; i < Vec<T>::kPairs; ++i) {
        const float2 h = halves(p[i]);
        f[2 * i] = h.x;
        f[2 * i + 1] = h.y;
    }
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
__device__ __forceinline__ float warp_max(float v) {                 // NaN is passed over
    float r;
    asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Fills the block's table with its layers first .. first + n - 1, n <= 32; bit i of the answer: layer i lies wholly inside
// the row.  Ends in a barrier.
template <class TI, class TO>
__device__ __forceinline__ uint32_t fill_table(Layer* table, uint32_t* mask, const LogitsCut& in, const LogitsCut& out, const Deal& d,
                                            int64_t row, int rank, int first, int n) {
    if (threadIdx.x < 32) {
        Layer l = {nullptr, nullptr, 0, 0, 0, 0};
        if ((int)threadIdx.x < n) table[threadIdx.x] = l = layer_of<TI, TO>(in, out, d, row, rank, first + (int)threadIdx.x);
        const uint32_t whole = __ballot_sync(0xffffffffu, l.hi - l.lo == kPerLayer<TI>);
        if (threadIdx.x == 0) *mask = whole;
    }
    __syncthreads();
    return *mask;
}

// f(layer, vector of the layer) for every vector of this thread in layer i that holds elements of the row.
template <class T, int TH = kThreads, class F> __device__ __forceinline__ void for_edges(const Layer* table, int i, F f) {
    const int lo = table[i].lo, hi = table[i].hi;
#pragma unroll 1
    for (int v = threadIdx.x; v < 2 * TH; v += TH)
        if (v * kPerVec<T> < hi && (v + 1) * kPerVec<T> > lo) f(i, v);
}
template <class T>
__device__ __forceinline__ void store_vector(const Layer& l, int vec, uint4 v) {
    const int p = vec * kPerVec<T>;
    if (l.vec_out && p >= l.lo && p + kPerVec<T> <= l.hi) {
        __stcs(reinterpret_cast<uint4*>(l.out + vec * 16), v);
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

// Sums of exponentials are kept as (m, sum of 2^((x - m) c)), c = log2(e) / T.  An element costs one fma: with
// mc = round(m c), 2^(x c - mc) has no rounding but the fma's own, and the sum of these is put right once by 2^(mc - m c).
// mc - m c is up to half a unit in the last place of mc: from |mc| = 2^31 on these two powers leave the range of fp32 in
// opposite directions, and their product is NaN.  From there on (a mask's -1e10, the type's lowest value, an infinity, a low
// temperature) the elements' differences are taken instead; where neighbouring floats are that far apart they are as exact.
// What counts is the maximum that a thread has seen so far, not the row's: its first vectors may be masked ones.
// A maximum of -inf goes with a sum of 0 (or NaN), one of +inf with the number of such elements.
struct Base {
    Pair  c, minus_mc;
    float m, right;
    bool  far;
};
__device__ __forceinline__ bool is_far(float mc, float from = 0x1p31f) { return !(fabsf(mc) < from); }
__device__ __forceinline__ Base base_of(float m, float c) {
    const float b = m == -INFINITY ? 0.f : m, mc = b * c;
    return {pair(c, c), pair(-mc, -mc), b, exp2_approx(fmaf(-b, c, mc)), is_far(mc)};
}
__device__ __forceinline__ float scale_to(float m, float to, float c) {
    return m == to ? 1.f : exp2_approx((m - to) * c);
}
// The same without the roundings of the exponent, c in 64 bits.
__device__ __forceinline__ float scale_finely(float m, float to, double c) {
    if (m == to) return 1.f;
    const double z = ((double)m - (double)to) * c;
    const float  t = (float)z;
    return t > -150.f ? exp2_approx(t) * fmaf((float)(z - (double)t), 0.693147182f, 1.f) : 0.f;
}
// Sums of 2^(x c - mc), with kFine of 2^(x (c + low) - mc).
template <class T, bool kFine> __device__ __forceinline__ Pair exp_sum(uint4 v, Pair c, Pair low, Pair minus_mc) {
    Pair p[Vec<T>::kPairs], sum = 0;
    Vec<T>::unpack(v, p);
#pragma unroll
    for (int i = 0; i < Vec<T>::kPairs; ++i) {
        Pair z = fma2(p[i], c, minus_mc);
        if (kFine) z = fma2(p[i], low, z);
        sum = add2(sum, exp2_pair(z));
    }
    return sum;
}
// 2^((x - m) c) of elements where m is far.  Beside a maximum of +inf only such elements count.
__device__ __forceinline__ Pair exp_far(Pair x, float m, Pair c) {
    if (m == INFINITY) {
        const float2 f = halves(x);
        return pair(f.x == m ? 1.f : f.x != f.x ? f.x : 0.f, f.y == m ? 1.f : f.y != f.y ? f.y : 0.f);
    }
    return exp2_pair(mul2(add2(x, pair(-m, -m)), c));
}
template <class T> __device__ __noinline__ float exp_sum_far(uint4 a, uint4 b, float m, Pair c) {
    Pair p[Vec<T>::kPairs], q[Vec<T>::kPairs], sum = 0;
    Vec<T>::unpack(a, p);
    Vec<T>::unpack(b, q);
#pragma unroll
    for (int i = 0; i < Vec<T>::kPairs; ++i) sum = add2(add2(sum, exp_far(p[i], m, c)), exp_far(q[i], m, c));
    const float2 h = halves(sum);
    return h.x + h.y;
}
// log of a sum of exponentials from its maximum, the scaled maximum and the sum of exp(x - max)
__device__ __forceinline__ float log_sum(float m, float scaled_m, float sum) {
    if (sum != sum) return sum;
    return m == -INFINITY || m == INFINITY ? m : scaled_m + logf(sum);
}

// Where a token of the row lies: its block, its layer there, and its position in the layer.
struct Place {
    int rank, layer, position;
};
// token / cols: tokens and columns are below 2^24, so that the product's rounding is off by one at most
__device__ __forceinline__ int shard_of(const LogitsCut& in, int token) {
    if (in.tp == 1) return 0;
    const int s = (int)((float)token * in.per_col), r = token - s * in.cols;
    return r < 0 ? s - 1 : r >= in.cols ? s + 1 : s;
}
template <class T, int TH = kThreads>
__device__ __forceinline__ Place place_of(const LogitsCut& in, const Deal& d, int64_t row, int token) {
    const int s = shard_of(in, token);
    int       q = token - s * in.cols;
    if (!d.aligned) q += (int)((uintptr_t)row_of<T>(in, s, row) & 15) / (int)sizeof(T);
    const int l = s * d.per_shard + q / kPerLayer<T, TH>;
    return {l & ((1 << d.log_c) - 1), l >> d.log_c, q % kPerLayer<T, TH>};
}
__device__ __forceinline__ int layers_of(const Deal& d, int rank) { return max(0, (d.layers - rank + (1 << d.log_c) - 1) >> d.log_c); }

// Elements a .. b - 1 of E as bits, where these may lie outside.
__device__ __forceinline__ uint32_t bits_between(int a, int b, int E) {
    const uint32_t below = (1u << min(max(b, 0), E)) - 1;
    return below & ~((1u << min(max(a, 0), E)) - 1);
}
// A vector of a layer that the row fills in part; what is not the row's is -inf.
template <class T> __device__ __noinline__ uint4 edge_vector(const Layer& l, int vec) {
    constexpr int E = kPerVec<T>;
    const int a = l.lo - vec * E, b = l.hi - vec * E;
    if (a <= 0 && b >= E) return __ldcs(reinterpret_cast<const uint4*>(l.in) + vec);
    if (b <= 0 || a >= E) return Vec<T>::none();
    T e[E];
#pragma unroll
    for (int j = 0; j < E; ++j) e[j] = j >= a && j < b ? reinterpret_cast<const T*>(l.in)[vec * E + j] : from_float<T>(-INFINITY);
    return *reinterpret_cast<const uint4*>(e);
}
// ---- rows that are read once ---------------------------------------------------------------------------------
//
// Where nothing is written per element the row need not stay on the chip: one block takes a whole row, its layers through
// a ring in shared memory, several blocks on an SM.

constexpr int kStreamRing = 3;            // layers on their way to a block that needs the row once
constexpr int kStepRing   = 5;            // ... and twice

// Fills a table of any number of layers.  Ends in a barrier.
template <class T, int TH = kThreads>
__device__ __forceinline__ void fill_long_table(Layer* table, const LogitsCut& in, const LogitsCut& out, const Deal& d, int64_t row) {
    for (int i = threadIdx.x; i < d.layers; i += TH) table[i] = layer_of<T, T, TH>(in, out, d, row, 0, i);
    __syncthreads();
}
// Starts the copies of this thread's two vectors of layer l into place `slot` of the ring, one commit group; nothing but the
// group past the last layer.
template <class T, int TH>
__device__ __forceinline__ void load_layer(const Layer* table, uint4* ring, int slot, int l, int n) {
    if (l < n) {
        uint4* const to = ring + slot * 2 * TH + threadIdx.x;
        const Layer& L = table[l];
        const char* from = L.in + threadIdx.x * 16;
        if (L.hi - L.lo == kPerLayer<T, TH>) {
            copy_async(smem_address(to), from);
            copy_async(smem_address(to + TH), from + TH * 16);
        } else {
#pragma unroll 1
            for (int v = 0; v < 2 * TH; v += TH) {
                const int at = ((int)threadIdx.x + v) * kPerVec<T>;
                if (at >= L.lo && at + kPerVec<T> <= L.hi) copy_async(smem_address(to + v), from + v * 16);
                else to[v] = edge_vector<T>(L, threadIdx.x + v);
            }
        }
    }
    copy_commit();
}
// f(layer, first vector, second vector) for this thread's vectors of all layers of the row, in order, through a ring of R
// layers, after start_stream.
template <class T, int TH, int R> __device__ __forceinline__ void start_stream(const Layer* table, uint4* ring, int n) {
#pragma unroll
    for (int l = 0; l < R; ++l) load_layer<T, TH>(table, ring, l, l, n);
}
template <class T, int TH, int R, class F> __device__ __forceinline__ void stream(const Layer* table, uint4* ring, int n, F f) {
    const uint4* mine = ring + threadIdx.x;
#pragma unroll 1
    for (int l = 0; l < n; l += R)
#pragma unroll
        for (int slot = 0; slot < R; ++slot) {
            if (l + slot >= n) break;
            copy_wait<R - 1>();
            const uint4 a = mine[slot * 2 * TH], b = mine[slot * 2 * TH + TH];
            if (l + slot + R < n) load_layer<T, TH>(table, ring, slot, l + slot + R, n);      // the last R layers stay
            else copy_commit();
            f(l + slot, a, b);
        }
}
// The same backwards, after stream: the last R layers are still in the ring, and of the others those come first that L2 has
// seen last.
template <class T, int TH, int R, class F> __device__ __forceinline__ void stream_back(const Layer* table, uint4* ring, int n, F f) {
    const uint4* mine = ring + threadIdx.x;
    int slot = (n - 1) % R;
#pragma unroll 1
    for (int l = n - 1; l >= 0; --l) {
        copy_wait<R - 1>();
        const uint4 a = mine[slot * 2 * TH], b = mine[slot * 2 * TH + TH];
        if (l >= R) load_layer<T, TH>(table, ring, slot, l - R, n);
        else copy_commit();
        f(l, a, b);
        slot = slot ? slot - 1 : R - 1;
    }
}

// 1 / T, and log2(e) / T: rounded, and as the sum of two fp32.  The first of these is cut, not rounded, and the second at
// least 2^-126, so that -inf times either is -inf.
struct Scale {
    double inv_t;
    float  c, high, low;
};

// A running sum of exponentials: (base, sum of 2^((x - base) c)) whose base follows the maximum only when that has gone
// 2^40 ahead: terms stay below 2^41 and most vectors leave it alone.  c = log2(e) / T; see Base for the arithmetic.
// kFine, for sums that a difference of near numbers is made of: c has its second part (alone, the first shifts the whole
// sum by up to 4e-8 |x - base| / T), and the base follows 2^8 behind, since an element ahead of it carries half a unit in
// the last place of the distance in its exponent.  What is left is 1e-7, half of it ex2.approx's.
template <bool kFine> struct Running {
    static constexpr float kAhead = kFine ? 8.f : 40.f;
    static constexpr float kFar = kFine ? 0x1p27f : 0x1p31f;      // the second part of c adds 2^-23 of mc to the exponent
    float base, base_c, right, ahead, sum, low;
    Pair  c, minus;
    __device__ __forceinline__ explicit Running(float scale, float scale_low = 0.f) {
        c = pair(scale, scale);
        low = scale_low;
        base = -INFINITY;
        ahead = -INFINITY;
        base_c = sum = 0.f;
        right = 1.f;
        minus = pair(-0.f, -0.f);
    }
    // before the elements whose maximum is `top` are added
    __device__ __forceinline__ void see(float top) {
        if (top > ahead) {
            const float scale = halves(c).x;
            sum *= scale_to(base, top, scale);
            base = top;
            base_c = top * scale;
            right = exp2_approx(fmaf(-top, scale, base_c) - (kFine ? top * low : 0.f));
            minus = pair(-base_c, -base_c);
            ahead = top + kAhead / scale;
        }
    }
    template <class T> __device__ __forceinline__ void add(uint4 a, uint4 b) {
        if (__any_sync(0xffffffffu, is_far(base_c, kFar))) {     // seldom, and then for the whole warp
            sum += exp_sum_far<T>(a, b, base == -INFINITY ? 0.f : base, c);
        } else {
            const Pair   d = pair(low, low);
            const float2 h = halves(add2(exp_sum<T, kFine>(a, c, d, minus), exp_sum<T, kFine>(b, c, d, minus)));
            sum = fmaf(h.x + h.y, right, sum);
        }
    }
};

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

// A note: the upper half of a float that is not below x, ordered by its value as a float.
__device__ __forceinline__ uint16_t note_of(float x) {
    const uint32_t u = __float_as_uint(x);
    return (uint16_t)((u >> 16) + ((u & 0xffffu) && !(u >> 31) ? 1u : 0u));       // a negative one is cut towards 0: up
}
__device__ __forceinline__ float value_of_note(uint16_t n) { return __uint_as_float((uint32_t)n << 16); }
// ... and the next below it: not above x.
__device__ __forceinline__ float note_below(uint16_t n) {
    return n == 0 || n == 0x8000u ? -__uint_as_float(0x00010000u) : __uint_as_float((uint32_t)(n >> 15 ? n + 1 : n - 1) << 16);
}

// ---- host side ------------------------------------------------------------------------------------------------

constexpr int64_t kMaxRows  = 1 << 24;
constexpr int64_t kMaxVocab = 1 << 24;

inline int size_of(int dtype) { return dtype == NEREUS_BF16 ? 2 : 4; }

inline int64_t held_cols(const nereus_logits_t& v, int s) {
    const int64_t left = v.vocab - (int64_t)s * v.shard_cols;
    return left <= 0 ? 0 : left < v.shard_cols ? left : v.shard_cols;
}

inline int check_view(const nereus_logits_t* v) {
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

inline LogitsCut cut_of(const nereus_logits_t& v) {
    LogitsCut c;
    for (int s = 0; s < NEREUS_VOCAB_MAX_TP; ++s) c.shard[s] = s < v.tp ? (char*)v.shard[s] : nullptr;
    c.row_bytes = v.row_stride * size_of(v.dtype);
    c.per_col = 1.f / (float)v.shard_cols;
    c.tp = v.tp; c.cols = (int32_t)v.shard_cols; c.vocab = (int32_t)v.vocab;
    return c;
}

inline bool misaligned(const void* p) { return (uintptr_t)p & 3; }
constexpr int kMaxDevices = 64;
constexpr int kSmemShare  = 73 * 1024;      // shared memory per block for which three blocks fit on an SM

struct Device {
    int id = 0, smem = 0, sms = 0;      // dynamic shared memory that a block may have
};
// The current device; its shared memory and SMs are looked up once.
inline int device_of(Device* d) {
    static std::atomic<int> smem[kMaxDevices], sms[kMaxDevices];
    NEREUS_CUDA(cudaGetDevice(&d->id));
    if (d->id < 0 || d->id >= kMaxDevices) return NEREUS_ERR_UNSUPPORTED;
    d->sms = sms[d->id].load();
    d->smem = smem[d->id].load();
    if (!d->smem || !d->sms) {
        int most = 0;
        NEREUS_CUDA(cudaDeviceGetAttribute(&most, cudaDevAttrMaxSharedMemoryPerBlockOptin, d->id));
        d->smem = most - 16384;                                   // 16 KiB: the kernels' static part
        NEREUS_CUDA(cudaDeviceGetAttribute(&d->sms, cudaDevAttrMultiProcessorCount, d->id));
        sms[d->id].store(d->sms);
        smem[d->id].store(d->smem);
    }
    return NEREUS_OK;
}

// Layers of a shard of w columns whose rows start on 16-byte boundaries, and of one whose rows start anywhere: a vector more.
inline int layers_aligned(int64_t w, int64_t e, int threads) { return (int)(((w + e - 1) / e + 2 * threads - 1) / (2 * threads)); }
inline int layers_anywhere(int64_t w, int64_t e, int threads) { return (int)(((w + 2 * e - 2) / e + 2 * threads - 1) / (2 * threads)); }

// A row for each block.
inline Deal deal_of(const nereus_logits_t& v, int threads) {
    Deal d;
    const int64_t e = 16 / size_of(v.dtype), w = held_cols(v, 0), bytes = v.row_stride * size_of(v.dtype);
    d.aligned = v.rows < 2 || bytes % 16 == 0;
    for (int s = 0; s < v.tp; ++s)
        if (held_cols(v, s) && (uintptr_t)v.shard[s] % 16) d.aligned = 0;
    d.per_shard = d.aligned ? layers_aligned(w, e, threads) : layers_anywhere(w, e, threads);
    d.layers = d.mine = d.per_shard * (int)((v.vocab + v.shard_cols - 1) / v.shard_cols);
    d.log_c = 0;
    return d;
}

// Deals a row out over the fewest blocks whose share has at most `most` layers and takes at most kSmemShare bytes, at
// `per_layer` a layer and `fixed` once.  Which layer goes to which block, and with it the order of a row's sums, must not
// depend on the other rows: neither their number nor where they start has a part in it.  So a shard has its layers for rows
// that start anywhere, always (one more, and for aligned rows an empty one, only where its vectors fill layers exactly), and
// the number of blocks goes by those of aligned rows.  The last shard's empty one shifts no other and is left out.
inline Deal spread_of(const nereus_logits_t& v, int threads, int64_t per_layer, int64_t fixed, int most) {
    Deal d = deal_of(v, threads);
    const int64_t e = 16 / size_of(v.dtype), w = held_cols(v, 0);
    const int     used = (int)((v.vocab + v.shard_cols - 1) / v.shard_cols), least = layers_aligned(w, e, threads), main = least * used;
    d.per_shard = layers_anywhere(w, e, threads);
    d.layers = d.per_shard * used - (d.aligned ? d.per_shard - least : 0);
    auto share = [&](int layers) { return (int64_t)(layers + (1 << d.log_c) - 1) >> d.log_c; };
    while (d.log_c < 3 && (share(main) > most || share(main) * per_layer + fixed > kSmemShare)) ++d.log_c;
    d.mine = (int)share(d.layers);
    return d;
}

// Launches a kernel with a cluster of blocks for each row.  `opted`: whether the kernel has been given its shared memory,
// per device.
template <class... P, class... A>
int launch(void (*kernel)(P...), std::atomic<bool>* opted, int threads, int64_t rows, const Deal& d, int64_t smem,
           const Device& dev, cudaStream_t stream, A... args) {
    if (smem > dev.smem) return NEREUS_ERR_TOO_LARGE;
    if (!opted[dev.id].load()) {
        NEREUS_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, dev.smem));
        opted[dev.id].store(true);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(rows << d.log_c));
    cfg.blockDim = dim3((unsigned)threads);
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

inline Scale scale_of(double temperature) {
    Scale r;
    r.inv_t = 1.0 / temperature;
    const double c = 1.4426950408889634 * r.inv_t;
    r.c = r.high = (float)c;
    if ((double)r.high > c) r.high = std::nextafter(r.high, 0.f);
    r.low = c < 0x1p127 ? std::max((float)(c - (double)r.high), 0x1p-126f) : 0x1p-126f;
    return r;
}

}  // namespace
}  // namespace nereus
