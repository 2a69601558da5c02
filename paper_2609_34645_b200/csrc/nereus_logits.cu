// The model-stages' own steps on the LM head's logits for sm_100a: penalties, biases and grammar masks of a generation
// step (nereus_logits_process), a teacher's top logits of an inference stage (nereus_teacher_top) and the distillation
// from them of a training stage (nereus_distill_forward / _backward / _step).
//
// Logits come cut by vocabulary into column shards, one device buffer each.  All three walk rows of some 100,000
// elements with a handful of operations on each, so their floor is HBM bandwidth: every logit read once, every written
// one stored once; 2 exponentials an element (16 a clock and SM) come next.  What the kernels share:
//   * A row's 16-byte vectors are dealt out in layers of two vectors a thread.  A layer lies inside one shard, so that
//     everything about it but the thread's own vectors is the same for the block: one 32-byte record in shared memory.
//   * Elements come through a ring of layers in shared memory by cp.async.  Every thread reads back only what it copied
//     itself, so that an arrival needs no barrier, and no wait that could hang: nothing here spins on a flag.
//   * Rows of any alignment: vectors that a row fills only in part (its ends, where it does not start on a 16-byte
//     boundary) are read and written element by element; what lies outside the row is -inf in shared memory.
//   * The number of rows decides nothing but the grid: a row's result is the same, bit for bit, in any batch in which its
//     shards start alike modulo 16 bytes.
//   * One block takes a whole row where that leaves it little to keep (teacher_top, distillation), a cluster of 1 to 8
//     blocks where every column needs a counter (process).
#include "nereus_rows.hpp"

using namespace nereus;

namespace nereus {
namespace {

// ---- penalties, biases, masks --------------------------------------------------------------------------------
//
// A sweep over the row, elements through a ring of three layers in shared memory to registers and from there to memory.
// Everything else waits in shared memory: mask bits, one counter per column of the block's share (the history lands there
// with shared-memory atomics: sums of whole numbers, so that no order shows), a hash table of the bias entries with a flag
// per column.  The running (maximum, where it is, sum of exponentials) stays on the thread.
// Every block reads the whole history (from L2) and keeps what falls into its share: reading it once per cluster and
// counting into the peers' shared memory was no faster (256 rows of up to 16384 tokens: 166 against 170 us) and takes two
// cluster barriers.  A share is at most four layers where counters allow, for as many blocks as a small batch can use.
// Not bound by HBM, which is at 20% for 256 rows of 152064 fp32 with histories up to 16384 (167 us, 1.9-2.0 TB/s): issue slots
// are 63% busy there, and three blocks, 24 warps, an SM (74 registers, 68 KB) are too few to cover one another's phases in
// the rest.  64 x 128256 bf16 to fp32, with 16 biases, 33 us: 86 KB a block, of which the bias table takes 24, leave two
// blocks an SM, and 512 blocks are two waves.  One row of 128256: 9 us of GPU time, a chain of phases on 8 SMs.

constexpr int kHash   = 2048;             // slots of the bias table, over twice NEREUS_BIAS_MAX
constexpr int kRing   = 3;                // layers on their way to a block

// Counter of a column, 0 for a token that is not in the history: the top bit "in the prompt", the others "generated so
// often".
template <class Count> constexpr uint32_t kPrompt = 1u << (sizeof(Count) * 8 - 1);

template <class Count> __device__ __forceinline__ void count_token(uint32_t* words, int column, bool generated) {
    const int shift = sizeof(Count) == 4 ? 0 : (column & 1) * 16;
    uint32_t* word = words + (sizeof(Count) == 4 ? column : column >> 1);
    if (generated) atomicAdd(word, 1u << shift);
    else atomicOr(word, kPrompt<Count> << shift);
}
// The counters of a vector, `column` its first; returns whether one is set.
template <class Count, int E> __device__ __forceinline__ bool counts_of(const uint32_t* words, int column, uint32_t (&c)[E]) {
    constexpr int N = E * (int)sizeof(Count) / 4;          // words of a vector
    const uint32_t* from = words + column * (int)sizeof(Count) / 4;
    uint32_t w[N], any = 0;
#pragma unroll
    for (int i = 0; i < N; i += 2) *reinterpret_cast<uint2*>(w + i) = *reinterpret_cast<const uint2*>(from + i);
#pragma unroll
    for (int i = 0; i < N; ++i) any |= w[i];
#pragma unroll
    for (int j = 0; j < E; ++j) c[j] = sizeof(Count) == 4 ? w[j * N / E] : w[j * N / E] >> (j % 2 * 16) & 0xffffu;
    return any != 0;
}

// Penalties of a vector whose counters are c.  A quotient x / rho has to come out as IEEE division rounds it, for many x
// that share rho: with y = the rounded 1 / rho, q = x y and the remainder r = x - q rho, exact by fma, q + r y by fma is
// the correctly rounded quotient (Markstein, Computation of elementary functions on the IBM RISC System/6000 processor,
// 1990) as long as nothing on the way over- or underflows; a vector or row where that could be is divided.
struct Penalty {
    float rho, inverse, frequency, presence;
    bool  plain;               // rho lies in 2^-60 .. 2^60, as x has to
};
__device__ __forceinline__ Penalty penalty_of(float rho, float frequency, float presence) {
    return {rho, __frcp_rn(rho), frequency, presence, rho >= 0x1p-60f && rho <= 0x1p60f};
}
template <class Count, int E> __device__ __forceinline__ void penalise(float (&x)[E], const uint32_t (&c)[E], const Penalty& p) {
    float q[E];
    bool  odd = !p.plain;
#pragma unroll
    for (int j = 0; j < E; ++j) {
        constexpr uint32_t least = 0x21800000u, most = 0x5d800000u;      // 2^-60, 2^60
        odd |= x[j] > 0.f && __float_as_uint(x[j]) - least > most - least;
        q[j] = x[j] * p.inverse;
        q[j] = fmaf(fmaf(-q[j], p.rho, x[j]), p.inverse, q[j]);
    }
    if (odd) {
#pragma unroll
        for (int j = 0; j < E; ++j) q[j] = __fdiv_rn(x[j], p.rho);
    }
#pragma unroll
    for (int j = 0; j < E; ++j) {
        const float    y = x[j] > 0.f ? q[j] : __fmul_rn(x[j], p.rho);
        const uint32_t made = c[j] & (kPrompt<Count> - 1);
        const float    z = __fsub_rn(__fsub_rn(y, __fmul_rn(p.frequency, (float)made)), p.presence);
        x[j] = !c[j] ? x[j] : made ? z : y;
    }
}

// The bias of a token that has one.
__device__ __forceinline__ uint32_t hash_of(int token) { return (uint32_t)token * 2654435761u >> 16 & (kHash - 1); }
__device__ __noinline__ float bias_of(const int32_t* ids, const float* values, int token) {
    uint32_t h = hash_of(token);
    while (ids[h] != token && ids[h] != -1) h = (h + 1) % kHash;     // the table is never full
    return values[h];
}
template <int E> __device__ __forceinline__ float far_sum(const float (&x)[E], float base) {
    Pair sum = 0;
#pragma unroll
    for (int j = 0; j < E; j += 2) sum = add2(sum, exp_far(pair(x[j], x[j + 1]), base, pair(kLog2e, kLog2e)));
    const float2 h = halves(sum);
    return h.x + h.y;
}

template <class TI, class TO, class Count>
__global__ void __launch_bounds__(kThreads, 3) process_kernel(const __grid_constant__ LogitsCut in,
                                                              const __grid_constant__ LogitsCut out, Deal deal,
                                                              const __grid_constant__ nereus_penalties_t how, int32_t* token,
                                                              float* lse) {
    constexpr int E = kPerVec<TI>;
    extern __shared__ __align__(16) unsigned char dynamic[];
    __shared__ float2 scratch[kWarps], from_peers[kMaxCtas];
    __shared__ int    id_scratch[kWarps], id_peers[kMaxCtas];
    __shared__ uint32_t whole_layers;
    const int     tid = threadIdx.x, rank = blockIdx.x & ((1 << deal.log_c) - 1);
    const int64_t row = blockIdx.x >> deal.log_c;
    if (deal.log_c) cluster_arrive();              // this block runs: its shared memory may be written
    constexpr int kMaskWords = kPerLayer<TI> / 32 + 1;       // of a layer, which may begin anywhere in a word
    Layer*     table = reinterpret_cast<Layer*>(dynamic);
    uint4*     ring = reinterpret_cast<uint4*>(table + deal.mine);
    uint32_t*  words = reinterpret_cast<uint32_t*>(ring + kRing * kVecs);                    // mask words
    uint32_t*  biased = words + (how.mask ? (deal.mine * kMaskWords + 3) / 4 * 4 : 0);        // a byte per vector
    int32_t*   hash_id = reinterpret_cast<int32_t*>(biased + (how.bias_ids ? deal.mine * kVecs / 4 : 0));
    int32_t*   hash_entry = hash_id + kHash;                  // the last entry of the id
    float*     hash_value = reinterpret_cast<float*>(hash_entry + kHash);
    uint32_t*  counters = reinterpret_cast<uint32_t*>(hash_id + (how.bias_ids ? 3 * kHash : 0));

    const Penalty penalty = penalty_of(how.repetition ? how.repetition[row] : 1.f, how.frequency ? how.frequency[row] : 0.f,
                                       how.presence ? how.presence[row] : 0.f);
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
    // The largest value and the first vector that has it.  The sum is kept from a base that follows the maximum only when
    // it has fallen 40 behind: its terms stay below 2^58, and most vectors leave it alone.
    float m = -INFINITY, base = -INFINITY, base_c = 0.f, right = 1.f, sum = 0.f;
    const char* m_vector = nullptr;
    int         m_token = 0;
    uint32_t    m_held = 0;                                  // elements of the vector that are the row's
    auto rebase = [&](float top) {
        sum *= scale_to(base, top, kLog2e);
        base = top;
        base_c = top * kLog2e;
        right = exp2_approx(fmaf(-top, kLog2e, base_c));
    };
    for (int first = 0; first < n_all; first += deal.mine) {      // one round unless the counters do not fit
        const int n = min(deal.mine, n_all - first);
        // what is a memory latency away and needed soon: the first tokens of the history, and the biases
        constexpr int kAhead = 4, kMost = (NEREUS_BIAS_MAX + kThreads - 1) / kThreads;
        int   ahead[kAhead], bias_id[kMost];
        float bias_value[kMost];
        if (how.history) {
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                ahead[j] = tid + j * kThreads < how.history_len ? how.history[row * how.history_stride + tid + j * kThreads] : -1;
        }
        if (how.bias_ids) {
#pragma unroll
            for (int j = 0; j < kMost; ++j) {
                const bool    is = tid + j * kThreads < how.bias_count;
                const int64_t at = row * how.bias_count + tid + j * kThreads;
                bias_id[j] = is ? how.bias_ids[at] : -1;
                bias_value[j] = is ? how.bias_values[at] : 0.f;
            }
        }
        __syncthreads();
        const uint32_t whole = fill_table<TI, TO>(table, &whole_layers, in, out, deal, row, rank, first, n);
        // this thread's two vectors of layer l into their places in the ring
        auto fetch = [&](int l) {
            if (l < n) {
                uint4* const to = ring + l % kRing * kVecs + tid;
                if (whole >> l & 1u) {
                    const char* from = table[l].in + tid * 16;
                    copy_async(smem_address(to), from);
                    copy_async(smem_address(to + kThreads), from + kThreads * 16);
                } else {
#pragma unroll 1
                    for (int v = 0; v < kVecs; v += kThreads) {
                        const int p = (tid + v) * E;
                        if (p >= table[l].lo && p + E <= table[l].hi) copy_async(smem_address(to + v), table[l].in + (tid + v) * 16);
                        else to[v] = edge_vector<TI>(table[l], tid + v);
                    }
                }
            }
            copy_commit();
        };
#pragma unroll 1
        for (int l = 0; l < kRing; ++l) fetch(l);
        if (total > 0)
            for (int i = tid; i < n * kPerLayer<TI> * (int)sizeof(Count) / 16; i += kThreads)
                reinterpret_cast<uint4*>(counters)[i] = make_uint4(0, 0, 0, 0);
        if (how.bias_ids)
            for (int i = tid; i < 2 * kHash / 4; i += kThreads) reinterpret_cast<int4*>(hash_id)[i] = make_int4(-1, -1, -1, -1);
        if (how.bias_ids)
            for (int i = tid; i < n * kVecs / 4; i += kThreads) biased[i] = 0;
        if (mask) {
#pragma unroll 4
            for (int i = tid; i < n * kMaskWords; i += kThreads) {
                const int w = (table[i / kMaskWords].token >> 5) + i % kMaskWords;
                words[i] = w >= 0 && w <= mask_last ? (uint32_t)mask[w] : 0u;
            }
        }
        __syncthreads();
        {
            auto count = [&](int i, int id) {
                if ((uint32_t)id >= (uint32_t)in.vocab) return;
                const Place p = place_of<TI>(in, deal, row, id);
                const int   l = p.layer - first;
                if (p.rank == rank && (uint32_t)l < (uint32_t)n) count_token<Count>(counters, l * kPerLayer<TI> + p.position, i >= prompt);
            };
            // four tokens a thread at a time, the next four on their way
            for (int i = tid; i - tid < total; i += kAhead * kThreads) {
                int id[kAhead];
#pragma unroll
                for (int j = 0; j < kAhead; ++j) {
                    const int next = i + (j + kAhead) * kThreads;
                    id[j] = ahead[j];
                    ahead[j] = next < total ? hist[next] : -1;
                }
#pragma unroll
                for (int j = 0; j < kAhead; ++j)
                    if (i + j * kThreads < total) count(i + j * kThreads, id[j]);
            }
        }
        if (how.bias_ids) {
            // an entry's slot in the hash table, or -1 where another block holds the token
            int slot[kMost];
#pragma unroll
            for (int j = 0; j < kMost; ++j) {
                const int id = bias_id[j];
                slot[j] = -1;
                if (j * kThreads >= how.bias_count) continue;
                if ((uint32_t)id >= (uint32_t)in.vocab) continue;
                const Place p = place_of<TI>(in, deal, row, id);
                const int   l = p.layer - first;
                if (p.rank != rank || (uint32_t)l >= (uint32_t)n) continue;
                const int vec = l * kVecs + p.position / E;
                atomicOr(biased + vec / 4, 1u << (vec % 4 * 8 + p.position % E));
                uint32_t h = hash_of(id);
                for (;; h = (h + 1) % kHash) {             // over twice as many slots as entries: one is free
                    const int was = atomicCAS(&hash_id[h], -1, id);
                    if (was == -1 || was == id) break;
                }
                slot[j] = (int)h;
                atomicMax(&hash_entry[h], tid + j * kThreads);
            }
            __syncthreads();
            // of the entries of one id the last counts
#pragma unroll
            for (int j = 0; j < kMost; ++j)
                if (slot[j] >= 0 && hash_entry[slot[j]] == tid + j * kThreads) hash_value[slot[j]] = bias_value[j];
        }
        __syncthreads();

        // bit j: element j of the vector is allowed
        auto allowed = [&](int l, int vec) {
            const uint32_t* w = words + l * kMaskWords;
            const int       bit = (table[l].token & 31) + vec * E;
            return __funnelshift_r(w[bit >> 5], w[min((bit >> 5) + 1, kMaskWords - 1)], bit & 31);
        };
        // One layer at a time, a thread's two vectors together.
#pragma unroll 1
        for (int l = 0; l < n; ++l) {
            copy_wait<kRing - 1>();
            const Layer& L = table[l];
            float    x[2][E], top[2];
            uint32_t held[2] = {(1u << E) - 1, (1u << E) - 1};     // elements that are the row's
            unpack<TI>(ring[l % kRing * kVecs + tid], x[0]);
            unpack<TI>(ring[l % kRing * kVecs + tid + kThreads], x[1]);
            fetch(l + kRing);
            if (!(whole >> l & 1u)) {
                held[0] = bits_between(L.lo - tid * E, L.hi - tid * E, E);
                held[1] = bits_between(L.lo - (tid + kThreads) * E, L.hi - (tid + kThreads) * E, E);
            }
            if (total > 0) {
                uint32_t   c0[E], c1[E];
                const bool a = counts_of<Count>(counters, l * kPerLayer<TI> + tid * E, c0);
                const bool b = counts_of<Count>(counters, l * kPerLayer<TI> + (tid + kThreads) * E, c1);
                if (a || b) {
                    penalise<Count>(x[0], c0, penalty);
                    penalise<Count>(x[1], c1, penalty);
                }
            }
            if (how.bias_ids) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int      vec = tid + i * kThreads;
                    const uint32_t f = reinterpret_cast<const uint8_t*>(biased)[l * kVecs + vec];
                    if (f) {
#pragma unroll
                        for (int j = 0; j < E; ++j)
                            if (f >> j & 1u) x[i][j] = __fadd_rn(x[i][j], bias_of(hash_id, hash_value, L.token + vec * E + j));
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int vec = tid + i * kThreads;
                if (mask) {
                    const uint32_t f = allowed(l, vec);
#pragma unroll
                    for (int j = 0; j < E; ++j) x[i][j] = f >> j & 1u ? x[i][j] : -INFINITY;
                }
                // written, and from here on what was written
                TO y[E];
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    y[j] = from_float<TO>(x[i][j]);
                    x[i][j] = to_float(y[j]);
                }
                char* const o = L.out + vec * E * (int)sizeof(TO);
                if (L.vec_out && held[i] == (1u << E) - 1) {
                    const uint4* w = reinterpret_cast<const uint4*>(y);
#pragma unroll
                    for (int j = 0; j < E * (int)sizeof(TO) / 16; ++j) __stcs(reinterpret_cast<uint4*>(o) + j, w[j]);
                } else {
#pragma unroll
                    for (int j = 0; j < E; ++j) {
                        if (held[i] >> j & 1u) reinterpret_cast<TO*>(o)[j] = y[j];
                        else x[i][j] = -INFINITY;
                    }
                }
                top[i] = x[i][0];
#pragma unroll
                for (int j = 1; j < E; ++j) top[i] = fmaxf(top[i], x[i][j]);
            }
            const float most = fmaxf(top[0], top[1]);
            if (most > m) {
                m = most;
                const int vec = top[0] == most ? tid : tid + kThreads;
                m_vector = L.out + vec * E * (int)sizeof(TO);
                m_token = L.token + vec * E;
                m_held = top[0] == most ? held[0] : held[1];
            }
            if (most > base + 40.f) rebase(most);
            if (__any_sync(0xffffffffu, is_far(base_c))) {       // seldom, and then for the whole warp
                const float from = base == -INFINITY ? 0.f : base;
                sum += far_sum(x[0], from) + far_sum(x[1], from);
            } else {
                Pair part[2] = {0, 0};
                const Pair c = pair(kLog2e, kLog2e), minus = pair(-base_c, -base_c);
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < E; j += 2) part[i] = add2(part[i], exp2_pair(fma2(pair(x[i][j], x[i][j + 1]), c, minus)));
                const float2 h = halves(add2(part[0], part[1]));
                sum = fmaf(h.x + h.y, right, sum);
            }
        }
    }
    sum *= scale_to(base, m, kLog2e);

    // the warp's result, the block's on its first warp, and the cluster's on its first block
    auto warp_join = [&](float2 v) {
        const float top = warp_max(v.x);
        return make_float2(top, warp_sum(v.y * scale_to(v.x, top, kLog2e)));
    };
    float2 v = warp_join(make_float2(m, sum));
    // the lowest id of the maximum: only the threads that have it read their vector back
    int at = 0x7fffffff;
    if (m == v.x && m_vector) {
#pragma unroll 1
        for (int j = E - 1; j >= 0; --j)
            if ((m_held >> j & 1u) && to_float(reinterpret_cast<const TO*>(m_vector)[j]) == v.x) at = m_token + j;
    }
    at = (int)__reduce_min_sync(0xffffffffu, (uint32_t)at);
    const int lane = tid & 31;
    if (lane == 0) { scratch[tid >> 5] = v; id_scratch[tid >> 5] = at; }
    __syncthreads();
    if (deal.log_c) cluster_wait();
    if (tid < 32) {
        const float2 mine = lane < kWarps ? scratch[lane] : make_float2(-INFINITY, 0.f);
        v = warp_join(mine);
        at = (int)__reduce_min_sync(0xffffffffu, lane < kWarps && mine.x == v.x ? (uint32_t)id_scratch[lane] : 0x7fffffffu);
        if (lane == 0) {
            peer_store(peer_address(&from_peers[rank], 0), v.x, v.y);
            asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(peer_address(&id_peers[rank], 0)), "r"(at) : "memory");
        }
    }
    if (deal.log_c) {
        __syncwarp();
        cluster_arrive();
        if (rank) return;
        cluster_wait();
    }
    if (tid < 32) {
        __syncwarp();
        const int    ctas = 1 << deal.log_c;
        const float2 mine = lane < ctas ? from_peers[lane] : make_float2(-INFINITY, 0.f);
        v = warp_join(mine);
        at = (int)__reduce_min_sync(0xffffffffu, lane < ctas && mine.x == v.x ? (uint32_t)id_peers[lane] : 0x7fffffffu);
        if (lane == 0) {
            if (token) token[row] = v.x > -INFINITY ? at : -1;
            if (lse) lse[row] = log_sum(v.x, v.x, v.y);
        }
    }
}

// A vector with -inf in the elements of `bits`.
template <class T> __device__ __forceinline__ uint4 without(uint4 v, uint32_t bits) {
    Pair p[Vec<T>::kPairs];
    Vec<T>::unpack(v, p);
#pragma unroll
    for (int i = 0; i < Vec<T>::kPairs; ++i) {
        const float2 h = halves(p[i]);
        p[i] = pair(bits >> 2 * i & 1u ? -INFINITY : h.x, bits >> (2 * i + 1) & 1u ? -INFINITY : h.y);
    }
    return Vec<T>::pack(p);
}

// ---- a teacher's top logits ----------------------------------------------------------------------------------
//
// One pass over the row sums the exponentials and notes the largest of every 16 elements, a thread's vectors of one layer
// (fp32: of two), in two bytes (fp32 rounded up).  If each of the 8 warps takes the j-th largest of its threads' maxima, j =
// k / 8 rounded up, at least k elements reach the least of these 8 values, whatever the order of the row: it bounds the
// row's k-th largest from below, and for most rows some 1.4 k elements reach it.  Only the vectors whose note does are read
// again, and what is found in them is ranked by counting, as one 64-bit key of (value, lower id).  Rows of so few distinct
// values that more is found than the list holds are searched for the k-th key and the id to cut at, exactly: some 57 more
// passes over the row, 28 ms for 4096 rows of 128256 that a mask left 20 tokens each, of which the 64 largest were asked.
// 4096 x 128256 bf16, k = 64: 233-244 us, 4.3-4.5 TB/s read, the exponentials at 60% of their rate and four blocks an SM
// short of hiding the selection (a quarter of a row's time); 512 x 152064 fp32, k = 128: 76-80 us, 3.9-4.1 TB/s.

constexpr int kCandidates = 1024;
template <class T> constexpr int kNote = (int)sizeof(T) / 2;          // layers of a note

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
__global__ void __launch_bounds__(kThreads, 4) top_kernel(const __grid_constant__ LogitsCut in, Deal deal, int k, int j,
                                                          float inv_t, float* values, int32_t* ids, float* lse) {
    constexpr int E = kPerVec<T>;
    typedef unsigned long long Key;
    extern __shared__ __align__(16) unsigned char dynamic[];
    __shared__ float2   scratch[kWarps];
    __shared__ uint32_t least[kWarps];
    __shared__ int      count_scratch[kWarps], n_found, n_noted;
    const int     tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = deal.layers;
    const int64_t row = blockIdx.x;
    const float   c = inv_t * kLog2e;

    uint4*    ring = reinterpret_cast<uint4*>(dynamic);
    Layer*    table = reinterpret_cast<Layer*>(ring + kStreamRing * kVecs);
    uint16_t* notes = reinterpret_cast<uint16_t*>(table + n) + tid;          // of this thread
    // once the row has gone through, the ring takes the lists of what is found
    Key*      found = reinterpret_cast<Key*>(ring);
    uint32_t* noted_list = reinterpret_cast<uint32_t*>(found + kCandidates);
    constexpr int kNoted = (kStreamRing * kVecs * 16 - kCandidates * 8) / 4;
    if (tid == 0) n_found = n_noted = 0;
    fill_long_table<T>(table, in, LogitsCut(), deal, row);

    Running<false> running(c);
    typename Vec<T>::Max m0 = Vec<T>::lowest(), m1 = m0;         // of the thread's first and second vectors
    float to_note = -INFINITY;
    start_stream<T, kThreads, kStreamRing>(table, ring, n);
    stream<T, kThreads, kStreamRing>(table, ring, n, [&](int l, uint4 a, uint4 b) {
        const typename Vec<T>::Max ma = Vec<T>::max(a), mb = Vec<T>::max(b);
        const float m = Vec<T>::value(Vec<T>::join(ma, mb));
        m0 = Vec<T>::join(m0, ma);
        m1 = Vec<T>::join(m1, mb);
        to_note = l % kNote<T> ? fmaxf(to_note, m) : m;
        notes[l / kNote<T> * kThreads] = sizeof(T) == 2 ? (uint16_t)(__float_as_uint(to_note) >> 16) : note_of(to_note);
        running.see(m);
        running.template add<T>(a, b);
    });
    const float f0 = Vec<T>::value(m0), f1 = Vec<T>::value(m1);
    bool has0 = false, has1 = false;
    for (int l = 0; l < n; ++l) {
        const int lo = table[l].lo, hi = table[l].hi;
        has0 |= tid * E < hi && (tid + 1) * E > lo;
        has1 |= (tid + kThreads) * E < hi && (tid + kThreads + 1) * E > lo;
        if (hi - lo == kPerLayer<T>) break;
    }

    // the warp's j-th largest maximum (of both vectors' where j is large), to 16 bits from below; a warp in which a lane
    // has no element does not take part
    const float m = fmaxf(f0, f1);
    {
        const bool     full = __all_sync(0xffffffffu, has0 || has1), two = j > 8 && __all_sync(0xffffffffu, has0 && has1);
        const uint32_t key0 = key_of(two ? f0 : m), key1 = two ? key_of(f1) : 0;
        uint32_t       t = 0;
#pragma unroll 1
        for (int bit = 31; bit >= 16; --bit) {
            const uint32_t u = t | 1u << bit;
            int reach = __popc(__ballot_sync(0xffffffffu, key0 >= u));
            if (two) reach += __popc(__ballot_sync(0xffffffffu, key1 >= u));
            if (reach >= j) t = u;
        }
        const float top = warp_max(m), sum = warp_sum(running.sum * scale_to(running.base, top, c));
        if (lane == 0) {
            least[warp] = full ? max(t, kKeyMinusInf) : 0xffffffffu;
            scratch[warp] = make_float2(top, sum);
        }
    }
    __syncthreads();
    uint32_t low = least[0];
#pragma unroll
    for (int i = 1; i < kWarps; ++i) low = min(low, least[i]);
    // no warp is full in rows of less than 32 vectors: everything is a candidate
    const float bound = low == 0xffffffffu || j > 64 ? -INFINITY : value_of(low);

    // every element of this thread's vectors of layer l that is not NaN: f(key, token)
    auto look = [&](int l, auto f) {
        const Layer& L = table[l];
#pragma unroll 1
        for (int vec = tid; vec < kVecs; vec += kThreads) {
            const int a = L.lo - vec * E, b = L.hi - vec * E;
            if (b <= 0 || a >= E) continue;
            float x[E];
            unpack<T>(edge_vector<T>(L, vec), x);
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (x[e] == x[e] && e >= a && e < b) f(key_of(x[e]), L.token + vec * E + e);
        }
    };
    auto push = [&](uint32_t key, int v) {
        const int i = atomicAdd(&n_found, 1);
        if (i < kCandidates) found[i] = (Key)key << 32 | (0xffffffffu - (uint32_t)v);
    };
    // the notes that reach it into a list, then each of their vectors on a thread of its own
    if (m >= bound) {
        const int notes_of = (n + kNote<T> - 1) / kNote<T>;
#pragma unroll 1
        for (int q0 = 0; q0 < notes_of; q0 += 32) {
            uint32_t  reach = 0;
            const int count = min(32, notes_of - q0);
#pragma unroll 8
            for (int q = 0; q < count; ++q) reach |= (value_of_note(notes[(q0 + q) * kThreads]) >= bound ? 1u : 0u) << q;
            for (; reach; reach &= reach - 1) {
                const int i = atomicAdd(&n_noted, 1);
                if (i < kNoted) noted_list[i] = (uint32_t)(q0 + __ffs(reach) - 1) * kThreads + tid;
            }
        }
    }
    __syncthreads();
    const bool crowded = n_noted > kNoted;
    if (!crowded) {
        const int vecs = n_noted * 2 * kNote<T>;
#pragma unroll 1
        for (int i = tid; i < vecs; i += kThreads) {
            const uint32_t note = noted_list[i / (2 * kNote<T>)];
            const int      vec = note % kThreads + i % 2 * kThreads, l = note / kThreads * kNote<T> + i / 2 % kNote<T>;
            if (l >= n) continue;
            const Layer& L = table[l];
            const int    a = L.lo - vec * E, b = L.hi - vec * E;
            if (b <= 0 || a >= E) continue;
            float x[E];
            unpack<T>(edge_vector<T>(L, vec), x);
            uint32_t hits = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) hits |= (x[e] >= bound ? 1u : 0u) << e;
            hits &= bits_between(a, b, E);
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (hits >> e & 1u) push(key_of(x[e]), L.token + vec * E + e);
        }
    }
    __syncthreads();
    if (crowded || n_found > kCandidates) {
        auto each = [&](auto f) {
#pragma unroll 1
            for (int l = 0; l < n; ++l) look(l, f);
        };
        uint32_t kth = 0;                      // the largest key that k elements reach, 0 if there are fewer
#pragma unroll 1
        for (int bit = 31; bit >= 0; --bit) {
            int reach = 0;
            each([&](uint32_t key, int) { reach += key >= (kth | 1u << bit); });
            if (block_count(reach, count_scratch) >= k) kth |= 1u << bit;
        }
        int above = 0;
        each([&](uint32_t key, int) { above += key > kth; });
        above = block_count(above, count_scratch);
        int before = -1;                       // the largest id up to which fewer than k are taken
#pragma unroll 1
        for (int bit = 23; bit >= 0; --bit) {
            int reach = 0;
            each([&](uint32_t key, int id) { reach += key == kth && id <= before + (1 << bit); });
            if (above + block_count(reach, count_scratch) < k) before += 1 << bit;
        }
        if (tid == 0) n_found = 0;
        __syncthreads();
        each([&](uint32_t key, int id) { if (key > kth || (key == kth && id <= before + 1)) push(key, id); });
        __syncthreads();
    }
    const int total = n_found, groups = (total + 3) / 4;         // the list is read four keys at a time
    if (tid < 4 * groups - total) found[total + tid] = 0;
    __syncthreads();
    // a key on `team` neighbouring threads that share the comparing
    const int team = total <= 32 ? 8 : total <= 64 ? 4 : total <= 128 ? 2 : 1, part = tid & (team - 1);
    for (int at = tid / team; at < (total + 31) / 32 * 32; at += kThreads / team) {
        const Key mine = at < total ? found[at] : 0;
        int place = 0;
#pragma unroll 4
        for (int q = part; q < groups; q += team) {
            const ulonglong2 a = reinterpret_cast<const ulonglong2*>(found)[2 * q], b = reinterpret_cast<const ulonglong2*>(found)[2 * q + 1];
            place += (a.x > mine) + (a.y > mine) + (b.x > mine) + (b.y > mine);
        }
        for (int o = 1; o < team; o *= 2) place += __shfl_xor_sync(0xffffffffu, place, o);
        if (mine && part == 0 && place < k) {
            values[row * k + place] = value_of((uint32_t)(mine >> 32));
            ids[row * k + place] = (int32_t)(0xffffffffu - (uint32_t)mine);
        }
    }
    if (tid >= total && tid < k) { values[row * k + tid] = -INFINITY; ids[row * k + tid] = -1; }      // no element is left
    if (warp == 0) {
        const float2 mine = lane < kWarps ? scratch[lane] : make_float2(-INFINITY, 0.f);
        const float  top = warp_max(mine.x), all = warp_sum(mine.y * scale_to(mine.x, top, c));
        if (lane == 0) lse[row] = log_sum(top, top * inv_t, all);
    }
}

// ---- distillation --------------------------------------------------------------------------------------------
//
// The sum over the rest is taken on its own, with the entries left out: as the difference of the whole sum and the
// entries' it would lose its digits where the entries hold nearly all of the mass.  The gradient of a token of the rest is
// exp((x - m) / T) times one number per row.  The entries, k <= 256, are worked out by one thread each on the block's first
// k / 32 warps.

enum Pass { kForward, kBackward, kStep };
// Threads of a block.  A wide block has half as many rows in work for the same warps on an SM: the step's second reading
// finds more of them in L2 (8192 x 128256 bf16: 809-816 against 826-828 us), and a row alone takes less long (131 x 50257:
// 16.4 against 18.4 us); the forward pass reads once and is better off with smaller layers (111 against 117 us).
__host__ __device__ constexpr int threads_of(int pass) { return pass == kForward ? kThreads : kWide; }

// The divergence is a small difference of large terms where the student is near its teacher (terms of order P d, their sum
// of order P d^2), and the teacher's rest a small difference of 1 and a sum near it: in 32 bits neither keeps a digit there.
// So all that is done once per entry is done in 64 bits, from the logits, the teacher's and the sum over the rest on: an
// exponential of the teacher's and one of the student's, and logarithms for the loss.  Q sums to one as exactly, because S is
// the sum over the rest and these exponentials; only the rest's own relative error, 1e-7, is left, and it moves a
// divergence by Q_rest - P_rest times that.

// Sum of two values over the first `warps` warps, the only ones to call it; the same on every thread.
__device__ __forceinline__ double2 entry_sum(double a, double b, int warps, double2* scratch) {
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        a += __shfl_xor_sync(0xffffffffu, a, o);
        b += __shfl_xor_sync(0xffffffffu, b, o);
    }
    if (warps == 1) return make_double2(a, b);
    asm volatile("bar.sync 1, %0;" ::"r"(warps * 32) : "memory");
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = make_double2(a, b);
    asm volatile("bar.sync 1, %0;" ::"r"(warps * 32) : "memory");
    double2 r = scratch[0];
    for (int i = 1; i < warps; ++i) { r.x += scratch[i].x; r.y += scratch[i].y; }
    return r;
}

// Entry `threadIdx.x` of a row: the teacher's and the student's logit; id -1 where there is none.
struct Entry {
    int   id;
    float y, x, lse;
};
template <class T>
__device__ __forceinline__ void fetch_entry(Entry& e, int id, const LogitsCut& in, const nereus_distill_t& how, int64_t row) {
    e = {-1, 0.f, 0.f, 0.f};
    if (how.lse) e.lse = how.lse[row];
    if ((uint32_t)id >= (uint32_t)in.vocab) return;
    e.id = id;
    e.y = how.values[row * how.k + threadIdx.x];
    const int s = shard_of(in, id);
    e.x = to_float(row_of<T>(in, s, row)[id - s * in.cols]);
}

// The entry's probability, log P = y / T - norm; norm, P_rest and the sum of all P are the row's.
struct Teacher {
    double log_p, p, norm, p_rest, mass;
};
__device__ __forceinline__ Teacher teacher_of(const Entry& e, int vocab, const nereus_distill_t& how, double inv_t, int warps,
                                              double2* scratch) {
    Teacher r;
    if (how.lse) {
        r.norm = (double)e.lse;
        r.log_p = (double)e.y * inv_t - r.norm;
        r.p = e.id >= 0 ? exp(r.log_p) : 0.0;
        const double2 s = entry_sum(r.p, e.id >= 0 ? 1.0 : 0.0, warps, scratch);
        r.p_rest = (int)s.y < vocab ? fmax(0.0, 1.0 - s.x) : 0.0;
        r.mass = s.x + r.p_rest;         // 1 unless the entries alone have more than that, or are all tokens
        return r;
    }
    float top = warp_max(e.id >= 0 ? e.y : -INFINITY);
    if (warps > 1) {
        asm volatile("bar.sync 1, %0;" ::"r"(warps * 32) : "memory");
        if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5].x = top;
        asm volatile("bar.sync 1, %0;" ::"r"(warps * 32) : "memory");
        for (int i = 0; i < warps; ++i) top = fmaxf(top, (float)scratch[i].x);
    }
    const double  z = ((double)e.y - (double)top) * inv_t, v = e.id >= 0 ? exp(z) : 0.0;
    const double2 s = entry_sum(v, e.id >= 0 ? 1.0 : 0.0, warps, scratch);
    r.norm = (double)top * inv_t + log(s.x);
    r.log_p = (double)e.y * inv_t - r.norm;
    r.p = s.y > 0.0 ? v / s.x : 0.0;
    r.p_rest = 0.0;
    r.mass = s.y > 0.0 ? 1.0 : 0.0;
    return r;
}

// The student's entry: (x - m) / T, its probability, and the rest's; total and rest in units of exp(m / T).
struct Student {
    double z, q, q_rest, total, rest;
};
// What the forward KL's loss needs of a row.
struct Sums {
    double norm, p_rest, total, rest;
    float  m;
};
// P log(P / Q) of the entry and of the rest.
__device__ __forceinline__ double2 forward_terms(const Entry& e, const Sums& r, double inv_t) {
    const double log_p = (double)e.y * inv_t - r.norm, p = e.id >= 0 ? exp(log_p) : 0.0, log_total = log(r.total);
    return make_double2(p > 0.0 ? p * (log_p - (((double)e.x - (double)r.m) * inv_t - log_total)) : 0.0,
                        r.p_rest > 0.0 ? r.p_rest * (log(r.p_rest) - (log(r.rest) - log_total)) : 0.0);
}
// The divergence's terms of the entry and of the rest, f (its derivative after Q) and Q f of both: reverse KL, Jensen.
struct Groups {
    double term, term_rest, qf, qf_rest, f, f_rest;
};
__device__ __forceinline__ Groups groups_of(bool is, const Teacher& p, const Student& q, const nereus_distill_t& how) {
    Groups g = {0.0, 0.0, 0.0, 0.0, 0.0, 0.0};
    const double log_total = log(q.total), log_q = q.z - log_total, log_q_rest = log(q.rest) - log_total;
    if (how.divergence == NEREUS_REVERSE_KL) {
        if (q.q > 0.0) { g.f = log_q - p.log_p; g.term = g.qf = q.q * g.f; }
        if (q.q_rest > 0.0) {
            g.f_rest = log_q_rest - log(fmax(p.p_rest, 5.9604644775390625e-8));
            g.term_rest = g.qf_rest = q.q_rest * g.f_rest;
        }
        return g;
    }
    const double a = how.beta, b = 1.0 - a;
    if (is) {
        const double log_m = log(a * p.p + b * q.q);
        if (q.q > 0.0) { g.f = b * (log_q - log_m); g.qf = q.q * g.f; }
        g.term = g.qf + (p.p > 0.0 ? a * p.p * (p.log_p - log_m) : 0.0);
    }
    const double log_m = log(a * p.p_rest + b * q.q_rest);
    if (q.q_rest > 0.0) { g.f_rest = b * (log_q_rest - log_m); g.qf_rest = q.q_rest * g.f_rest; }
    g.term_rest = g.qf_rest + (p.p_rest > 0.0 ? a * p.p_rest * (log(p.p_rest) - log_m) : 0.0);
    return g;
}

// A row goes by once for its sums (see above: rows that are read once); which elements are entries stands in shared memory,
// two bytes (fp32: one) for a thread's two vectors of a layer.  The step lets it go by a second time for the gradient,
// backwards: the layers read last are in the ring, and some of the ones before them in L2.  The gradients of the entries are
// stored after the others'.
// Forward, 1024 x 152064 fp32: 106-112 us, 5.6-5.9 TB/s, HBM; the second part of log2(e) / T takes 2% of it, the entries'
// 64 bits 3% (102-106 us without either).  Backward, 2048 x 128256 bf16: 180-186 us, 5.7-5.8 TB/s, HBM with as many bytes
// written as read.  Step, 8192 x 128256 bf16, a quarter of the rows without weight: 806-828 us, 4.5-4.6 TB/s of the bytes that
// have to move; 37% of the second reading come from HBM (2368 rows, 455 MB of them live: 623 MB read, 560 written, 239 us),
// and HBM idles where a block's warps wait for the few that work on the entries.  (Holding the row in a cluster's shared
// memory instead took 930 us: the cluster's exchange left HBM idle.)
template <class T, int kPass>
__global__ void __launch_bounds__(threads_of(kPass), kPass == kForward ? 4 : 2)
    distill_kernel(const __grid_constant__ LogitsCut in, const __grid_constant__ LogitsCut grad, Deal deal,
                   const __grid_constant__ nereus_distill_t how, Scale scale, float* loss, float* saved, const float* grad_loss) {
    constexpr int E = kPerVec<T>, R = kPass == kStep ? kStepRing : kStreamRing;
    constexpr int TH = threads_of(kPass), W = TH / 32;
    typedef std::conditional_t<E == 8, uint16_t, uint8_t> Flags;
    extern __shared__ __align__(16) unsigned char dynamic[];
    __shared__ Sums    sums_of_row;
    __shared__ double2 entry_scratch[W];
    __shared__ float2  scratch[W];
    __shared__ float   m_scratch[W], rest_scale_of_row, near_of_row;
    const int     tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = deal.layers, entry_warps = (how.k + 31) >> 5;
    const int64_t row = blockIdx.x;
    const float   weight = how.weight ? how.weight[row] : 1.f, c = scale.c;
    int           id = -1;
    if (tid < how.k) id = how.ids[row * how.k + tid];
    uint4*    ring = reinterpret_cast<uint4*>(dynamic);
    Layer*    table = reinterpret_cast<Layer*>(ring + R * 2 * TH);
    uint32_t* flags = reinterpret_cast<uint32_t*>(table + n);
    if (weight == 0.f) {
        if (tid == 0 && kPass != kBackward) loss[row] = 0.f;
        if (tid < 4 && kPass == kForward) saved[row * 4 + tid] = 0.f;
        if (kPass != kForward) {
            fill_long_table<T, TH>(table, in, grad, deal, row);
            for (int i = 0; i < n; ++i)
                for_edges<T, TH>(table, i, [&](int l, int vec) { store_vector<T>(table[l], vec, make_uint4(0, 0, 0, 0)); });
        }
        return;
    }
    if (kPass != kBackward)
        for (int i = tid; i < n * TH * (int)sizeof(Flags) / 4; i += TH) flags[i] = 0;
    fill_long_table<T, TH>(table, in, kPass == kForward ? LogitsCut() : grad, deal, row);
    start_stream<T, TH, R>(table, ring, n);

    Entry e = {-1, 0.f, 0.f, 0.f};
    if (warp < entry_warps) {
        fetch_entry<T>(e, id, in, how, row);
        if (kPass != kBackward && e.id >= 0) {
            const Place at = place_of<T, TH>(in, deal, row, e.id);
            const int   vec = at.position / E, slot = at.layer * TH + vec % TH;
            const int   bit = slot * 2 * E + vec / TH * E + at.position % E;
            atomicOr(&flags[bit >> 5], 1u << (bit & 31));
        }
    }
    __syncthreads();

    if (kPass != kBackward) {
        const Flags* mine = reinterpret_cast<const Flags*>(flags) + tid;
        Running<true> running(scale.high, scale.low);
        typename Vec<T>::Max top = Vec<T>::lowest();
        stream<T, TH, R>(table, ring, n, [&](int l, uint4 a, uint4 b) {
            typename Vec<T>::Max v = Vec<T>::join(Vec<T>::max(a), Vec<T>::max(b));
            top = Vec<T>::join(top, v);
            if (const uint32_t f = mine[l * TH]) {
                a = without<T>(a, f);
                b = without<T>(b, f >> E);
                v = Vec<T>::join(Vec<T>::max(a), Vec<T>::max(b));
            }
            running.see(Vec<T>::value(v));
            running.template add<T>(a, b);
        });
        const float m_warp = warp_max(Vec<T>::value(top)), base = warp_max(running.base);
        const float sum = warp_sum(running.sum * scale_finely(running.base, base, (double)scale.high + (double)scale.low));
        if (lane == 0) {
            scratch[warp] = make_float2(base, sum);
            m_scratch[warp] = m_warp;
        }
        __syncthreads();
    }
    double  divergence = 0.0, divergence_rest = 0.0;
    float   g = 0.f;
    if (warp < entry_warps) {
        Student student;
        const Teacher teacher = teacher_of(e, in.vocab, how, scale.inv_t, entry_warps, entry_scratch);
        // the row's largest logit, one near the rest's largest, and the sum over the rest in units of exp(near / T): the rest
        // may lie so far below the entries that in units of exp(m / T) it is no fp32, nor the gradient's factor
        float  m, near;
        double sum;
        if (kPass == kBackward) {
            m = near = saved[row * 4];
            student.rest = sum = saved[row * 4 + 2];
            if (sum > 0.0 && sum < 1.0) {
                near = (float)((double)m + log(sum) / scale.inv_t);
                sum *= exp(((double)m - (double)near) * scale.inv_t);
            }
        } else {
            const float2 part = lane < W ? scratch[lane] : make_float2(-INFINITY, 0.f);
            m = warp_max(lane < W ? m_scratch[lane] : -INFINITY);
            near = warp_max(part.x);
            sum = (double)part.y * (double)scale_finely(part.x, near, (double)scale.high + (double)scale.low);
#pragma unroll
            for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            student.rest = near == m ? sum : sum * exp(((double)near - (double)m) * scale.inv_t);
        }
        student.z = ((double)e.x - (double)m) * scale.inv_t;
        const double mine = e.id >= 0 ? exp(student.z) : 0.0;
        student.total = student.rest + entry_sum(mine, 0.0, entry_warps, entry_scratch).x;
        student.q = mine / student.total;
        student.q_rest = student.rest / student.total;

        const double to_grad = (double)weight * (kPass == kBackward && grad_loss ? (double)grad_loss[row] : 1.0) * scale.inv_t;
        double       to_rest;              // the gradient of the whole rest
        if (how.divergence == NEREUS_FORWARD_KL) {
            // Q f, not f, which need not be finite; a step works out its loss after the gradient has gone out
            g = (float)((teacher.mass * student.q - teacher.p) * to_grad);
            to_rest = (teacher.mass * student.q_rest - teacher.p_rest) * to_grad;
            const Sums sums = {teacher.norm, teacher.p_rest, student.total, student.rest, m};
            if (kPass == kStep && tid == 0) sums_of_row = sums;
            if (kPass == kForward) {
                const double2 d = forward_terms(e, sums, scale.inv_t);
                divergence = entry_sum(d.x, 0.0, entry_warps, entry_scratch).x;
                divergence_rest = d.y;
            }
        } else {
            const Groups  v = groups_of(e.id >= 0, teacher, student, how);
            const double2 sums = entry_sum(v.term, v.qf, entry_warps, entry_scratch);
            const double  mean = sums.y + v.qf_rest;
            divergence = sums.x;
            divergence_rest = v.term_rest;
            g = student.q > 0.0 ? (float)(student.q * (v.f - mean) * to_grad) : 0.f;
            to_rest = student.q_rest * (v.f_rest - mean) * to_grad;
        }
        if (kPass == kForward && tid == 0) {
            const double d = divergence + divergence_rest;
            loss[row] = (float)((double)weight * d);
            float* const o = saved + row * 4;
            o[0] = m; o[1] = (float)student.total; o[2] = (float)student.rest; o[3] = (float)d;
        }
        if (tid == 0) { rest_scale_of_row = sum == 0.0 ? 0.f : (float)(to_rest / sum); near_of_row = near; }
    }
    if (kPass == kForward) return;
    __syncthreads();
    {
        const Base  b = base_of(near_of_row, c);
        const float to_rest = b.far ? rest_scale_of_row : rest_scale_of_row * b.right;
        const Pair  s = pair(to_rest, to_rest);
        auto gradient = [&](uint4 v) {
            Pair p[Vec<T>::kPairs];
            Vec<T>::unpack(v, p);
            if (b.far) {
#pragma unroll
                for (int j = 0; j < Vec<T>::kPairs; ++j) {
                    const float2 x = halves(p[j]);
                    p[j] = mul2(pair(scale_to(x.x, b.m, c), scale_to(x.y, b.m, c)), s);
                }
            } else {
#pragma unroll
                for (int j = 0; j < Vec<T>::kPairs; ++j) p[j] = mul2(exp2_pair(fma2(p[j], b.c, b.minus_mc)), s);
            }
            return Vec<T>::pack(p);
        };
        auto write = [&](int l, uint4 a, uint4 b) {
            const Layer& L = table[l];
            const uint4  ga = gradient(a), gb = gradient(b);
            if (L.vec_out && L.hi - L.lo == kPerLayer<T, TH>) {
                uint4* const to = reinterpret_cast<uint4*>(L.out) + tid;
                __stcs(to, ga);
                __stcs(to + TH, gb);
            } else {
                store_vector<T>(L, tid, ga);
                store_vector<T>(L, tid + TH, gb);
            }
        };
        if constexpr (kPass == kStep) stream_back<T, TH, R>(table, ring, n, write);
        else stream<T, TH, R>(table, ring, n, write);
    }
    __syncthreads();                                  // the entries' places have been written as of the rest
    if (e.id >= 0) {
        const int s = shard_of(in, e.id);
        row_of<T>(grad, s, row)[e.id - s * in.cols] = from_float<T>(g);
    }
    if (kPass == kStep && warp < entry_warps) {
        if (how.divergence == NEREUS_FORWARD_KL) {
            const double2 d = forward_terms(e, sums_of_row, scale.inv_t);
            divergence = entry_sum(d.x, 0.0, entry_warps, entry_scratch).x;
            divergence_rest = d.y;
        }
        if (tid == 0) loss[row] = (float)((double)weight * (divergence + divergence_rest));
    }
}

// ---- host side: the checks of the arguments ------------------------------------------------------------------

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

bool is_temperature(double t) { return (float)t >= 0x1p-126f && std::isfinite((float)t); }

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
    if (h->divergence == NEREUS_JENSEN && !(h->beta > 0.0 && h->beta < 1.0)) return NEREUS_ERR_ARG;
    if (!is_temperature(h->temperature)) return NEREUS_ERR_ARG;
    if (!h->lse && h->divergence != NEREUS_FORWARD_KL) return NEREUS_ERR_UNSUPPORTED;
    if (misaligned(h->values) || misaligned(h->ids) || misaligned(h->lse) || misaligned(h->weight)) return NEREUS_ERR_ALIGN;
    return NEREUS_OK;
}

template <class T, int kPass>
int distill_launch(const nereus_logits_t& in, const nereus_distill_t& how, float* loss, float* saved,
                   const float* grad_loss, const nereus_logits_t* grad, cudaStream_t stream) {
    constexpr int TH = threads_of(kPass);
    static std::atomic<bool> opted[kMaxDevices];
    Device dev;
    if (int rc = device_of(&dev)) return rc;
    const Deal    d = deal_of(in, TH);
    const Scale   scale = scale_of(how.temperature);
    const int64_t smem = (kPass == kStep ? kStepRing : kStreamRing) * 2 * TH * 16 + d.layers * (int64_t)(sizeof(Layer) + (kPass == kBackward ? 0 : TH * kPerVec<T> / 4));
    return launch(distill_kernel<T, kPass>, opted, TH, in.rows, d, smem, dev, stream, cut_of(in),
                  kPass == kForward ? LogitsCut() : cut_of(*grad), d, how, scale, loss, saved, grad_loss);
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
    static std::atomic<bool> opted[kMaxDevices];
    Device dev;
    if (int rc = device_of(&dev)) return rc;
    const int64_t per_layer = sizeof(Layer) + (how.history ? kPerLayer<TI> * sizeof(Count) : 0) +
                              (how.bias_ids ? kVecs : 0) + (how.mask ? (kPerLayer<TI> / 32 + 1) * 4 : 0);
    const int64_t fixed = (how.bias_ids ? 12 * kHash : 0) + 16 + kRing * kVecs * 16;
    Deal d = spread_of(in, kThreads, per_layer, fixed, 4);
    // what does not fit is done in rounds
    while (d.mine > 1 && (d.mine * per_layer + fixed > dev.smem || d.mine > 32)) d.mine = (d.mine + 1) / 2;
    return launch(process_kernel<TI, TO, Count>, opted, kThreads, in.rows, d, d.mine * per_layer + fixed, dev, stream,
                  cut_of(in), cut_of(out), d, how, token, lse);
}

template <class T>
int top_launch(const nereus_logits_t& in, int k, double temperature, float* values, int32_t* ids, float* lse, cudaStream_t stream) {
    static std::atomic<bool> opted[kMaxDevices];
    Device dev;
    if (int rc = device_of(&dev)) return rc;
    Deal d = deal_of(in, kThreads);
    // warps of which every lane has a vector, at least: how many of the k largest each has to vouch for
    const int64_t w = held_cols(in, 0), vecs = (w + kPerVec<T> - 1) / kPerVec<T>;
    const int     full = (int)std::min<int64_t>(vecs / 32, kWarps), j = full ? (k + full - 1) / full : 1;
    const int64_t smem = kStreamRing * kVecs * 16 + d.layers * (int64_t)sizeof(Layer) +
                         (d.layers + kNote<T> - 1) / kNote<T> * (int64_t)kThreads * 2;
    return launch(top_kernel<T>, opted, kThreads, in.rows, d, smem, dev, stream, cut_of(in), d, k, j, (float)(1.0 / temperature), values, ids, lse);
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

int nereus_teacher_top(const nereus_logits_t* in, int k, double temperature, float* values, int32_t* ids, float* lse,
                       void* cuda_stream) {
    if (int rc = check_view(in)) return rc;
    if (k < 1 || k > NEREUS_TOP_MAX_K || k > in->vocab) return NEREUS_ERR_ARG;
    if (!is_temperature(temperature)) return NEREUS_ERR_ARG;
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
