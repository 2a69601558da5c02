// One step of a beam search for sm_100a (nereus_beam_select): of what the beams of a request offer, score + x - log-sum-exp
// over the vocabulary, the k best.
//
// Every logit is read once; the floor is HBM bandwidth, with one exponential an element next (16 a clock and SM, which is what
// bf16 from HBM asks three quarters of).  Two launches:
//   * sum: the layers of all rows are dealt out evenly to as many blocks as the GPU holds, whatever requests they belong to, each
//     block's one after the other.  Of what it has of a row a block leaves the sum of exponentials, and of every part (a layer,
//     or a few) and thread the largest element, in 16 bits rounded up: a note;
//   * pick: a block for a request puts the sums together to log-sum-exps, so that elements of different rows can be compared.
//     The notes are worth something then: of 8 sets of them the j-th largest bounds the k-th best hypothesis from below,
//     whatever the order of the rows.  Only vectors whose note reaches the bound are read again; what is found in them, a
//     few times k hypotheses, is ranked by counting.
// Where more is found than the list holds (rows of few distinct values: a mask's lowest value, say), the bound is made exact
// by counting the keys' bytes, the highest first, a pass over the request for each byte that is needed.
// 128 requests x 8 x 128256 bf16 (32.6 us of HBM): 45 us the sum, 4.8 TB/s, and 12 the pick, a chain of dependent steps.  No unit is
// full while the sum runs: instructions are issued in 61% of the cycles, 8 an element, of which 3.3 are on whole numbers where opening
// a bf16 asks for one; the exponentials' unit is at 56%, DRAM at 59%.  A scheduler has 6.4 warps, 1.7 of them ready; the others wait
// for fixed latencies, for the queue of exponentials and shared memory, and for the next layer, in about equal parts.  One
// request of 4 beams takes 10 us, by the pick's chain.
// Hypotheses are compared in 64 bits, as keys of (total / norm, lower index): within a row these order as the logits do.
#include "nereus_rows.hpp"

using namespace nereus;

namespace nereus {
namespace {

constexpr int kTH       = kThreads;               // of a summing block
constexpr int kV        = 4;                      // vectors of a layer here, a thread's
constexpr int kRoom     = kV * kTH;
constexpr int kHalf     = kRoom / 2;              // a Layer is described as two vectors of so many threads
constexpr int kStages   = 2;                      // layers on their way to a block
constexpr int kBlocks   = 4;                      // on an SM
constexpr int kItems    = 128;                    // layers in its table at a time
constexpr int kListed   = 4096;                   // rows that it lists
constexpr int kParts    = 128;                    // parts of a request's rows, at most: a part is a layer, or several
constexpr int kPick     = 1024;                   // threads of a picking block
constexpr int kPickWarps = kPick / 32;
constexpr int kSets     = 8;
constexpr int kFound    = 1024;                   // hypotheses that its list holds
constexpr int kNoted    = 1024;                   // notes, or groups of 8, that reach the bound
typedef unsigned long long Key;

// Sums of exponentials are kept as (K, sum of 2^(x c - K)) with a whole number K, so that sums go together without another
// rounding.  A thread adds up a layer's 4 vectors in 32 bits, with K next to the largest x c among them, and layers in 64: how
// the layers are dealt out shows in the 53rd bit of a sum at most.  c = log2(e) has 24 bits, kLog2eLow is the rest: it is put
// right for the largest element of a row at the end, and an element at a distance of d from that is off by 2e-8 d of itself.
// K stays within +-2^21: a row whose largest element lies beyond (a mask's lowest value in all of it, say) is summed again, by
// differences from it.
constexpr float  kLargestK = 0x1p21f;
constexpr double kLog2eLow = 1.4426950408889634 - (double)kLog2e, kLn2 = 0.69314718055994531;
struct Sum {
    double  sum;
    int32_t k;
    float   top;                                  // the largest element
};
__device__ __forceinline__ double power_of_two(int k) {          // k not above 0
    return __hiloint2double(max(1023 + k, 0) << 20, 0);
}
// What a block leaves of a part.
struct Record {
    Sum      sum;
    uint16_t notes[kTH];
};
template <int kLanes> __device__ __forceinline__ double sum_of_lanes(double x) {
#pragma unroll
    for (int o = kLanes / 2; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
// log2 of a positive normal number, 1e-7 off
__device__ __forceinline__ double log2_of(double x) {
    const long long u = __double_as_longlong(x);
    return (double)((int)(u >> 52) - 1023) + (double)log2f((float)__longlong_as_double((u & 0xfffffffffffffll) | 1023ll << 52));
}

struct Select {
    int32_t beams, k, settle, rows;
    int32_t parts, of_part;                       // parts of a row, layers of a part (a power of two)
    float   per_shard_1;                          // 1 / layers of a shard
    const float*   score;
    const int32_t* ended;
    const float*   norm;
    Record*  records;                             // [rows, parts]
    float*   out_score;
    int32_t *out_parent, *out_token;
};
// a / b for a below 2^22, one_by = 1 / b rounded: off by one at most before it is put right.
__device__ __forceinline__ int quotient(int a, int b, float one_by) {
    const int q = (int)((float)a * one_by), r = a - q * b;
    return q + (r >= b) - (r < 0);
}
// Whether a beam's row is read: its score and norm are numbers and it has not ended.
__device__ __forceinline__ bool offers(const Select& s, int64_t row, int vocab, float* score, float* norm, int* ended) {
    *score = s.score[row];
    *norm = s.norm ? s.norm[row] : 1.f;
    *ended = s.ended ? s.ended[row] : -1;
    return fabsf(*score) < INFINITY && *norm > 0.f && *norm < INFINITY;
}
template <class T> __device__ __forceinline__ Layer layer_at(const LogitsCut& in, const Deal& deal, const Select& s, int64_t row, int l) {
    if (l >= deal.layers) return {nullptr, nullptr, 0, 0, 0, 0};
    const int shard = quotient(l, deal.per_shard, s.per_shard_1);
    return layer_in<T, T, kHalf>(in, LogitsCut(), row, shard, (l - shard * deal.per_shard) * kPerLayer<T, kHalf>);
}

// ---- sums ----------------------------------------------------------------------------------------------------

// Starts the copies of this thread's vectors of layer l, one commit group; nothing but the group past the last layer.
template <class T> __device__ __forceinline__ void load_layer_of(const Layer* table, uint4* to, int l, int n) {
    if (l < n) {
        const Layer& L = table[l];
        const char*  from = L.in + threadIdx.x * 16;
        if (L.hi - L.lo == kPerLayer<T, kHalf>) {
#pragma unroll
            for (int v = 0; v < kV; ++v) copy_async(smem_address(to + v * kTH), from + v * kTH * 16);
        } else {
#pragma unroll
            for (int v = 0; v < kV; ++v) {
                const int at = ((int)threadIdx.x + v * kTH) * kPerVec<T>;
                if (at >= L.lo && at + kPerVec<T> <= L.hi) copy_async(smem_address(to + v * kTH), from + v * kTH * 16);
                else to[v * kTH] = at + kPerVec<T> <= L.lo || at >= L.hi ? Vec<T>::none() : edge_vector<T>(L, threadIdx.x + v * kTH);
            }
        }
    }
    copy_commit();
}

template <class T>
__global__ void __launch_bounds__(kTH, kBlocks) beam_sum_kernel(const __grid_constant__ LogitsCut in, const Deal deal, const Select s) {
    __shared__ __align__(16) uint4 ring[kStages * kRoom];
    __shared__ Layer    table[kItems];
    __shared__ uint32_t record_of[kItems];
    __shared__ uint16_t listed[kListed];
    __shared__ Sum      of_warps[2][kWarps];
    __shared__ int      of_warp[kWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    // The rows that are read.  They are listed, so that their parts come to all blocks alike; where there are many their
    // number evens out what each block gets, and rows that are not read are passed over.
    int  n = s.rows;
    bool list = s.rows <= kListed;
    auto read = [&](int row) {
        float score, norm;
        int   ended;
        return offers(s, row, in.vocab, &score, &norm, &ended) && (uint32_t)ended >= (uint32_t)in.vocab;
    };
    if (list) {
        n = 0;
        uint32_t flags = 0;                                // of rows tid, tid + kTH, ...
#pragma unroll
        for (int j = 0; j < kListed / kTH; ++j)
            if (j * kTH < s.rows) flags |= (j * kTH + tid < s.rows && read(j * kTH + tid) ? 1u : 0u) << j;
#pragma unroll 1
        for (int j = 0; j * kTH < s.rows; ++j) {
            const uint32_t who = __ballot_sync(0xffffffffu, flags >> j & 1u);
            __syncthreads();
            if (lane == 0) of_warp[warp] = __popc(who);
            __syncthreads();
            int before = n;
            for (int w = 0; w < kWarps; ++w) {
                if (w < warp) before += of_warp[w];
                n += of_warp[w];
            }
            if (flags >> j & 1u) listed[before + __popc(who & ((1u << lane) - 1))] = (uint16_t)(j * kTH + tid);
        }
        __syncthreads();
    }

    constexpr int kNone = -(1 << 21);
    float  top = -INFINITY, row_top = -INFINITY;          // of the part, and of what the block has of the row
    int    k = kNone;
    double sum = 0.0;
    int    odd = 0;
    uint4* const  mine = ring + tid;
    const Pair    c = pair(kLog2e, kLog2e);
    // the block's units, one after the other: parts of a few layers, all of a row and then the next row's
    const int     log_part = __ffs(s.of_part) - 1;
    const int64_t units = (int64_t)n * s.parts, lo = units * blockIdx.x / gridDim.x, hi = units * (blockIdx.x + 1) / gridDim.x;
    auto unit_of = [&](int64_t x, int* part) {
        const uint32_t u = (uint32_t)(lo + x), q = u / (uint32_t)s.parts;
        *part = (int)(u - q * (uint32_t)s.parts);
        return list ? (int)listed[q] : (int)q;
    };
    const int64_t layers = (hi - lo) << log_part;
    for (int64_t first = 0; first < layers; first += kItems) {
        const int items = (int)min((int64_t)kItems, layers - first);
        __syncthreads();
        if (tid < items) {
            int       part;
            const int row = unit_of((first + tid) >> log_part, &part), in_part = (int)(first + tid) & (s.of_part - 1);
            const bool last = in_part + 1 == s.of_part;
            table[tid] = list || read(row) ? layer_at<T>(in, deal, s, row, (part << log_part) + in_part) : Layer{nullptr, nullptr, 0, 0, 0, 0};
            // where its part's record is; whether the part ends with it, and what the block has of the row
            record_of[tid] = ((uint32_t)row * (uint32_t)s.parts + (uint32_t)part) << 2 | (last ? 2u : 0u) |
                             (last && (part + 1 == s.parts || first + tid + 1 == layers) ? 1u : 0u);
        }
        __syncthreads();
#pragma unroll 1
        for (int l = 0; l < kStages; ++l) load_layer_of<T>(table, mine + l * kRoom, l, items);
        int slot = 0;
#pragma unroll 1
        for (int item = 0; item < items; ++item) {
            copy_wait<kStages - 1>();
            uint4* const here = mine + slot * kRoom;
            uint4 x[kV];
#pragma unroll
            for (int j = 0; j < kV; ++j) x[j] = here[j * kTH];
            load_layer_of<T>(table, here, item + kStages, items);
            slot = slot + 1 == kStages ? 0 : slot + 1;
            typename Vec<T>::Max m = Vec<T>::max(x[0]);
#pragma unroll
            for (int j = 1; j < kV; ++j) m = Vec<T>::join(m, Vec<T>::max(x[j]));
            const float v = Vec<T>::value(m);              // NaN is passed over
            top = fmaxf(top, v);
            // rint by the addition of a number whose last place is 1
            constexpr float kWhole = 0x1.8p23f;
            const float  t = fminf(fmaxf(v * kLog2e, -kLargestK), kLargestK) + kWhole, of_k = t - kWhole;
            const int    now = __float_as_int(t) - __float_as_int(kWhole), next = max(k, now);
            const Pair   minus = pair(-of_k, -of_k);
            Pair of_layer = exp_sum<T, false>(x[0], c, c, minus);
#pragma unroll
            for (int j = 1; j < kV; ++j) of_layer = add2(of_layer, exp_sum<T, false>(x[j], c, c, minus));
            const float2 h = halves(of_layer);
            sum = fma((double)(h.x + h.y), power_of_two(now - next), sum * power_of_two(k - next));
            k = next;
            const uint32_t what = record_of[item];
            if (what & 2u) {
                Record* const to = s.records + (what >> 2);
                to->notes[tid] = note_of(top);
                row_top = fmaxf(row_top, top);
                top = -INFINITY;
                if (!(what & 1u)) {
                    if (tid == 0) to->sum = {0.0, kNone, -INFINITY};
                    continue;
                }
                const int   all = __reduce_max_sync(0xffffffffu, k);
                const float most = warp_max(row_top);
                const Sum   mine = {sum_of_lanes<32>(sum * power_of_two(k - all)), all, most};
                if (lane == 0) of_warps[odd][warp] = mine;
                __syncthreads();
                if (warp == 0) {                           // two sets of sums: the others are at the next row's meanwhile
                    Sum u = lane < kWarps ? of_warps[odd][lane] : Sum{0.0, kNone, -INFINITY};
                    const int of_all = __reduce_max_sync(0xffffffffu, u.k);
                    u = {sum_of_lanes<kWarps>(u.sum * power_of_two(u.k - of_all)), of_all, warp_max(u.top)};
                    if (lane == 0) to->sum = u;
                }
                odd ^= 1;
                row_top = -INFINITY;
                k = kNone;
                sum = 0.0;
            }
        }
    }
}

// ---- the pick ------------------------------------------------------------------------------------------------

// orders as the values do, -0 as +0
__device__ __forceinline__ Key key_of_double(double x) {
    const Key u = (Key)__double_as_longlong(x + 0.0);
    return u >> 63 ? ~u : u | (Key)1 << 63;
}
constexpr Key kKeyNone = 0x000fffffffffffffull;   // of -inf

// A beam of the request.
struct Beam {
    double   off, norm;                           // score - log-sum-exp; NaN: the row offers nothing
    float    off_1, inverse;                      // off and 1 / norm in 32 bits
    float    least;                               // elements below are not among the best; NaN: none is
    float    score;
    int32_t  ended;                               // its token, -1: it goes on
    int32_t  pad;
};

// A hypothesis: the element, later the total, of a token of a beam.
struct Hit {
    float   x;
    int32_t beam, token;
};
__device__ __forceinline__ float largest_note(const Record* records, int g) {
    const uint4 v = reinterpret_cast<const uint4*>(records[g / 32].notes)[g % 32];
    return Vec<__nv_bfloat16>::value(Vec<__nv_bfloat16>::max(v));
}
// The log-sum-exp of a row whose largest element lies far from 0, by a warp.
template <class T> __device__ __noinline__ double far_row(const LogitsCut& in, const Deal& deal, const Select& s, int64_t row, float top, double* sum) {
    double all = 0.0;
    for (int l = 0; l < deal.layers; ++l) {
        const Layer L = layer_at<T>(in, deal, s, row, l);
        for (int vec = threadIdx.x & 31; vec < kRoom; vec += 64)
            all += (double)exp_sum_far<T>(edge_vector<T>(L, vec), edge_vector<T>(L, vec + 32), top, pair(kLog2e, kLog2e));
    }
    all = sum_of_lanes<32>(all);
    *sum = all;
    return (double)top + kLn2 * log2_of(all);
}

// What the picking block shares with its search of last resort.
struct Pick {
    __align__(16) Key found[kFound];
    Beam     beams[NEREUS_BEAM_MAX];
    Hit      rest[kFound];
    uint32_t histogram[256], choice[4], of_warp[kPickWarps], all_of[3], any_of[3];
    int      n_found;
};
// whether a beam offers itself alone
__device__ __forceinline__ bool ended(const Beam& r) { return r.ended >= 0 && r.off == r.off; }
__device__ __forceinline__ void push(Pick& pick, int beam, float x, int token) {
    const int at = atomicAdd(&pick.n_found, 1);
    if (at < kFound) pick.rest[at] = {x, beam, token};
}
// what a hypothesis is worth, in 64 bits; 0: it is not offered
__device__ __forceinline__ Key key_of_hit(const Select& s, const Beam& r, float x, float* total) {
    const double sum = r.ended >= 0 ? r.off : r.off + (double)x;
    const Key    key = key_of_double(s.norm ? sum / r.norm : sum);
    *total = r.ended >= 0 ? r.score : (float)sum;
    return key > kKeyNone ? key : 0;
}
// Leaves the hypotheses to rank in the list, where they were too many for it.  On its own, out of the pick's registers: they
// spilled otherwise.  128 requests x 8 x 128256 with 24 tokens allowed each, the others at a mask's lowest value: k 16 in 0.20
// ms, k 64, where the k-th is a masked one, in 2.4.
template <class T> __device__ __noinline__ void search_by_bytes(const LogitsCut& in, const Deal& deal, const Select& s, int64_t first_row, Pick& pick) {
    constexpr int E = kPerVec<T>;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    auto& beams = pick.beams;
    auto& histogram = pick.histogram;
    auto& choice = pick.choice;
    auto& of_warp = pick.of_warp;
    auto& all_of = pick.all_of;
    auto& any_of = pick.any_of;
    auto& n_found = pick.n_found;
    // The k-th key exactly, or as much of it as leaves few enough: byte by byte of (key, ~index), the 12 bytes highest
    // first, by the number of hypotheses that share the bytes found so far.  Bytes that all of these have in common are
    // passed over, and a key is worked out once where neighbours are equal.
    Key      key_is = 0, key_mask = 0;
    uint32_t index_is = 0, index_mask = 0;
    int      left = s.k, above = 0;
    // f(key, beam, x, token, count) for all that may be among the best, a vector a thread of four layers at a time; `count`
    // tokens of one key at once where a vector's elements are equal
    auto each = [&](auto f) {
        auto one = [&](int b, float x, int token) {
            float     unused;
            const Key key = key_of_hit(s, beams[b], x, &unused);
            if (key) f(key, b, x, token, 1);
        };
#pragma unroll 1
        for (int b = 0; b < s.beams; ++b) {
            const float least = beams[b].least;
            if (least != least) continue;
            float last = NAN;
            Key   key = 0;
#pragma unroll 1
            for (int l = 0; l < deal.layers; l += 4) {
                uint4    v[4];
                int      token[4];
                uint32_t inside[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const Layer L = layer_at<T>(in, deal, s, first_row + b, l + j);
                    const int   lo = L.lo - tid * E, hi = L.hi - tid * E;
                    token[j] = L.token + tid * E;
                    inside[j] = bits_between(lo, hi, E);
                    v[j] = lo <= 0 && hi >= E ? __ldg(reinterpret_cast<const uint4*>(L.in) + tid) : inside[j] ? edge_vector<T>(L, tid) : Vec<T>::none();
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float top = Vec<T>::value(Vec<T>::max(v[j]));
                    if (!inside[j] || !(top >= least) || !(top > -INFINITY)) continue;
                    const bool equal = v[j].x == v[j].y && v[j].x == v[j].z && v[j].x == v[j].w && (sizeof(T) == 4 || v[j].x >> 16 == (v[j].x & 0xffffu));
                    const int  step = equal && inside[j] == (1u << E) - 1 ? E : 1;
                    float x[E];
                    unpack<T>(v[j], x);
#pragma unroll 1
                    for (int e = 0; e < E; e += step) {
                        float y = x[0];
#pragma unroll
                        for (int o = 1; o < E; ++o) y = o == e ? x[o] : y;
                        if (!(inside[j] >> e & 1u) || !(y >= least) || !(y > -INFINITY)) continue;
                        if (y != last) {
                            float unused;
                            key = key_of_hit(s, beams[b], y, &unused);
                            last = y;
                        }
                        if (key) f(key, b, y, token[j] + e, step);
                    }
                }
            }
        }
        if (tid < s.beams && ended(beams[tid])) one(tid, 0.f, beams[tid].ended);
    };
    static_assert(kPick == kRoom && kPickWarps == 32, "a vector of a layer for every thread, a lane for every warp");
    int byte = 0;
#pragma unroll 1
    while (byte < 12) {
        if (tid < 256) histogram[tid] = 0;
        if (tid == 0) {
            choice[0] = 256;
            for (int j = 0; j < 3; ++j) { all_of[j] = ~0u; any_of[j] = 0u; }
        }
        __syncthreads();
        int      bin = 0;
        uint32_t run = 0;                              // elements of one bin come one after the other
        Key      all_key = ~(Key)0, any_key = 0;
        uint32_t all_index = ~0u, any_index = 0;
        each([&](Key key, int beam, float, int token, int count) {
            if ((key ^ key_is) & key_mask) return;
            all_key &= key;
            any_key |= key;
            // tokens whose index shares this byte and those above it go together
            const int shift = byte < 8 ? 31 : 88 - 8 * byte;
#pragma unroll 1
            for (int done = 0; done < count;) {
                const uint32_t first = ~(uint32_t)(beam * in.vocab + token + done), last = first - (uint32_t)(count - done - 1);
                const int      n = byte < 8 || first >> shift == last >> shift ? count - done : 1;
                done += n;
                if ((first ^ index_is) & index_mask) continue;
                all_index &= n > 1 ? first & last : first;
                any_index |= n > 1 ? first | last : first;
                const int b = (int)(byte < 8 ? key >> (56 - 8 * byte) : (Key)(first >> shift)) & 255;
                if (b != bin) {
                    if (run) atomicAdd(&histogram[bin], run);
                    bin = b;
                    run = 0;
                }
                run += n;
            }
        });
        if (run) atomicAdd(&histogram[bin], run);
        const uint32_t alls[3] = {(uint32_t)(all_key >> 32), (uint32_t)all_key, all_index}, anys[3] = {(uint32_t)(any_key >> 32), (uint32_t)any_key, any_index};
#pragma unroll
        for (int j = 0; j < 3; ++j) {
            const uint32_t x = __reduce_and_sync(0xffffffffu, alls[j]), y = __reduce_or_sync(0xffffffffu, anys[j]);
            if (lane == 0) { atomicAnd(&all_of[j], x); atomicOr(&any_of[j], y); }
        }
        __syncthreads();
        // the bins from the highest down: how many there are up to this one
        const uint32_t c = tid < 256 ? histogram[255 - tid] : 0;
        uint32_t       upto = c;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const uint32_t u = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += u;
        }
        if (lane == 31) of_warp[warp] = upto;
        __syncthreads();
        for (int w = 0; w < warp; ++w) upto += of_warp[w];
        if (tid < 256 && upto >= (uint32_t)left && upto - c < (uint32_t)left) {
            choice[0] = 255 - tid;
            choice[1] = upto - c;
            choice[2] = c;
        }
        __syncthreads();
        const uint32_t b = choice[0], higher = choice[1], same = choice[2];
        if (b == 256) break;                           // fewer than k in all: everything is taken
        above += (int)higher;
        left -= (int)higher;
        // this byte, and those behind it that all have in common
#pragma unroll 1
        for (bool first = true; byte < 12; first = false) {
            const int      shift = 24 - 8 * (byte & 3);
            const uint32_t all = all_of[byte >> 2] >> shift & 255u, any = any_of[byte >> 2] >> shift & 255u;
            if (!first && all != any) break;
            const uint32_t is = first ? b : all;
            if (byte < 8) { key_is |= (Key)is << (56 - 8 * byte); key_mask |= (Key)255 << (56 - 8 * byte); }
            else { index_is |= is << shift; index_mask |= 255u << shift; }
            ++byte;
        }
        __syncthreads();
        if (above + (int)same <= kFound) break;
    }
    if (tid == 0) n_found = 0;
    __syncthreads();
    // everything from the bytes found on
    each([&](Key key, int beam, float x, int token, int count) {
        const Key top = key & key_mask;
        if (top < key_is) return;
#pragma unroll 1
        for (int j = 0; j < count; ++j)
            if (top > key_is || (~(uint32_t)(beam * in.vocab + token + j) & index_mask) >= index_is) push(pick, beam, x, token + j);
    });
    __syncthreads();
}

template <class T>
__global__ void __launch_bounds__(kPick) beam_pick_kernel(const __grid_constant__ LogitsCut in, const Deal deal, const Select s) {
    constexpr int E = kPerVec<T>;
    extern __shared__ __align__(16) unsigned char dynamic[];
    Record* const records = reinterpret_cast<Record*>(dynamic);
    __shared__ Pick pick;
    auto& beams = pick.beams;
    auto& found = pick.found;
    auto& rest = pick.rest;
    auto& of_warp = pick.of_warp;
    auto& n_found = pick.n_found;
    __shared__ uint32_t noted[kNoted], grouped[kNoted], peak[kPick], at_place[NEREUS_BEAM_MAX_K];
    __shared__ int      n_noted, n_grouped;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t request = blockIdx.x, first_row = request * s.beams;

    for (int b = tid; b < s.beams; b += kPick) {
        Beam  r;
        float norm;
        const bool is = offers(s, first_row + b, in.vocab, &r.score, &norm, &r.ended);
        if ((uint32_t)r.ended >= (uint32_t)in.vocab) r.ended = -1;
        r.norm = (double)norm;
        r.inverse = 1.f / norm;
        if (isinf(r.inverse)) r.inverse = NAN;         // 1 / norm is beyond fp32: its notes are worth nothing for the bound
        r.off = is ? (double)r.score : (double)NAN;
        r.least = NAN;
        beams[b] = r;
    }
    if (tid == 0) n_found = n_noted = n_grouped = 0;
    __syncthreads();
    asm volatile("griddepcontrol.wait;" ::: "memory");                      // the sums and notes are there

    // what the sums' blocks have left of the request
    const int   row_parts = s.beams * s.parts, groups = row_parts * (kTH / 8);
    const float parts_1 = 1.f / (float)s.parts;
    {
        const uint4* const from = reinterpret_cast<const uint4*>(s.records + first_row * s.parts);
#pragma unroll 1
        for (int x = tid; x < row_parts * (int)(sizeof(Record) / 16); x += kPick)
            copy_async(smem_address(reinterpret_cast<uint4*>(records) + x), from + x);
        copy_commit();
        copy_wait<0>();
    }
    __syncthreads();

    // every row's log-sum-exp, a warp for each
#pragma unroll 1
    for (int b = warp; b < s.beams; b += kPickWarps) {
        Beam& r = beams[b];
        if (r.off != r.off || r.ended >= 0) {
            if (lane == 0) r.off_1 = NAN;
            continue;
        }
        int    k = -(1 << 21);
        float  top = -INFINITY;
        double sum = 0.0;
#pragma unroll 1
        for (int e = lane; e < s.parts; e += 32) {
            const Sum u = records[b * s.parts + e].sum;
            const int to = max(k, u.k);
            sum = fma(u.sum, power_of_two(u.k - to), sum * power_of_two(k - to));
            k = to;
            top = fmaxf(top, u.top);
        }
        const int all = __reduce_max_sync(0xffffffffu, k);
        top = warp_max(top);
        sum = sum_of_lanes<32>(sum * power_of_two(k - all));
        double lse = kLn2 * ((double)all + log2_of(sum) + (double)top * kLog2eLow);
        if (fabsf(top * kLog2e) >= kLargestK && fabsf(top) < INFINITY) lse = far_row<T>(in, deal, s, first_row + b, top, &sum);
        if (lane == 0) {
            r.off = fabsf(top) < INFINITY && sum == sum ? r.off - lse : (double)NAN;
            r.off_1 = (float)r.off;
        }
    }
    __syncthreads();

    // The notes, 8 at a time; a warp's are of one row and part.  Of each set of threads the j-th largest of what their notes
    // are worth, off + x, by the norm, in 32 bits and a little less for the roundings: the least of these bounds the k-th
    // best from below.
    auto worth_below = [](const Beam& r, float x) {
        // Not a number (an offset or 1 / norm beyond fp32): it vouches for nothing.  A quotient beyond fp32 counts as the largest
        // number, which it is not below.  1e-38: so that what the smallest floats are rounded by is covered too.
        const float sum = fmaf(-1e-6f, fabsf(r.off_1) + fabsf(x) + 1e-38f, r.off_1 + x);
        const float w = fminf(fmaxf(sum * r.inverse, -INFINITY), 3.402823466e38f);
        return fmaf(-1e-6f, fabsf(w) + 1e-38f, w);
    };
    float most = -INFINITY;
#pragma unroll 1
    for (int g = tid; g < groups; g += kPick) {
        const Beam& r = beams[quotient(g / 32, s.parts, parts_1)];
        if (r.off_1 != r.off_1) continue;
        const float up = largest_note(records, g);
        // a note of a fp32 was rounded up: the next below it is not above the element
        const float x = sizeof(T) == 2 ? up : note_below((uint16_t)(__float_as_uint(up) >> 16));
        if (up > -INFINITY) most = fmaxf(most, worth_below(r, x));
    }
    peak[tid] = key_of(most);
    __syncthreads();
    if (warp < kSets) {
        uint32_t key = 0, t = 0;
        // a row's notes are on neighbouring threads: every set has its share of every row's
#pragma unroll
        for (int x = 0; x < kPick; x += kSets * 32) key = max(key, peak[x + lane * kSets + warp]);
#pragma unroll 1
        for (int i = 0; i < s.k; i += kSets) {
            t = __reduce_max_sync(0xffffffffu, key);
            if (lane == __ffs(__ballot_sync(0xffffffffu, key == t)) - 1) key = 0;
        }
        if (lane == 0) of_warp[warp] = t;
    }
    __syncthreads();
    // of every row the least x whose worth reaches the bound, or a little less; in 64 bits, where nothing overflows
    auto set_least = [&](uint32_t key) {
        if (tid >= s.beams) return;
        Beam&        r = beams[tid];
        const double reach = (double)value_of(key) * r.norm;
        r.least = r.off_1 != r.off_1 ? NAN : key > kKeyMinusInf ? __double2float_rd(fma(-1e-6, fabs(reach) + fabs(r.off), reach - r.off)) : -INFINITY;
    };
    // the groups of notes that reach it, then the notes
    auto list_groups = [&]() {
#pragma unroll 1
        for (int g = tid; g < groups; g += kPick)
            if (const float up = largest_note(records, g); up >= beams[quotient(g / 32, s.parts, parts_1)].least && up > -INFINITY) {
                const int at = atomicAdd(&n_grouped, 1);
                if (at < kNoted) grouped[at] = (uint32_t)g;
            }
    };
    if (tid < s.beams) {
        uint32_t t = 0xffffffffu;
#pragma unroll
        for (int i = 0; i < kSets; ++i) t = min(t, of_warp[i]);
        set_least(t);
    }
    __syncthreads();
    list_groups();
    __syncthreads();
    if (n_grouped > kNoted) {
        // Some set had little to vouch with (what a mask leaves lies on few threads): the k-th largest of all notes, to 16 bits.
        uint32_t t = 0;
#pragma unroll 1
        for (int bit = 31; bit >= 16; --bit) {
            int reach = 0;
#pragma unroll 1
            for (int n = tid; n < groups * 8; n += kPick) {
                const Beam&    r = beams[quotient(n / kTH, s.parts, parts_1)];
                const uint16_t note = records[n / kTH].notes[n % kTH];
                const float    x = sizeof(T) == 2 ? value_of_note(note) : note_below(note);
                if (value_of_note(note) > -INFINITY && r.off_1 == r.off_1) reach += key_of(worth_below(r, x)) >= (t | 1u << bit);
            }
            reach = __reduce_add_sync(0xffffffffu, reach);
            __syncthreads();
            if (lane == 0) of_warp[warp] = (uint32_t)reach;
            __syncthreads();
            if ((int)__reduce_add_sync(0xffffffffu, of_warp[lane]) >= s.k) t |= 1u << bit;
        }
        if (tid == 0) n_grouped = 0;
        set_least(t);
        __syncthreads();
        list_groups();
        __syncthreads();
    }
    const int n_groups = n_grouped;
#pragma unroll 1
    for (int j = tid; j < min(n_groups, kNoted) * 8; j += kPick) {
        const int g = (int)grouped[j / 8], row_part = g / 32, thread = g % 32 * 8 + (j & 7);
        if (value_of_note(records[row_part].notes[thread]) >= beams[quotient(row_part, s.parts, parts_1)].least) {
            const int at = atomicAdd(&n_noted, 1);
            if (at < kNoted) noted[at] = (uint32_t)(row_part * kTH + thread);
        }
    }
    __syncthreads();

    // f(beam, x, token) for every element of vector `vec` of a layer that may be among the best
    auto look = [&](int b, const Layer& L, int vec, auto f) {
        const int lo = L.lo - vec * E, hi = L.hi - vec * E;
        if (hi <= 0 || lo >= E) return;
        const float least = beams[b].least;
        float x[E];
        unpack<T>(edge_vector<T>(L, vec), x);
        uint32_t hits = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) hits |= (x[e] >= least && x[e] > -INFINITY ? 1u : 0u) << e;
        hits &= bits_between(lo, hi, E);
#pragma unroll 1
        for (; hits; hits &= hits - 1) {
            const int e = __ffs(hits) - 1;
            float y = x[0];
#pragma unroll
            for (int o = 1; o < E; ++o) y = o == e ? x[o] : y;
            f(b, y, L.token + vec * E + e);
        }
    };
    const int log_part = __ffs(s.of_part) - 1, noted_all = max(n_noted, n_groups);
    if (noted_all <= kNoted) {
        // every vector of a note on a thread of its own
        const int of_note = kV << log_part, vecs = n_noted * of_note;
#pragma unroll 1
        for (int j = tid; j < vecs; j += kPick) {
            const int which = (int)noted[j / of_note], row_part = which / kTH, b = quotient(row_part, s.parts, parts_1), v = j % of_note;
            const int l = ((row_part - b * s.parts) << log_part) + v / kV;
            look(b, layer_at<T>(in, deal, s, first_row + b, l), which % kTH + v % kV * kTH, [&](int beam, float x, int token) { push(pick, beam, x, token); });
        }
    }
    if (tid < s.beams && ended(beams[tid])) push(pick, tid, 0.f, beams[tid].ended);
    __syncthreads();

    if (noted_all > kNoted || n_found > kFound) search_by_bytes<T>(in, deal, s, first_row, pick);

    // which hypothesis is the j-th, and its beam in the upper half
    const int total = n_found, quads = (total + 3) / 4;    // keys are read four at a time
    if (tid < s.k) at_place[tid] = 0xffffffffu;
#pragma unroll 1
    for (int j = tid; j < 4 * quads; j += kPick) {
        if (j < total) found[j] = key_of_hit(s, beams[rest[j].beam], rest[j].x, &rest[j].x);       // its total takes the element's place
        else found[j] = 0;
    }
    __syncthreads();
    // a key on `team` neighbouring threads that share the comparing
    const int team = total <= 32 ? 16 : total <= 64 ? 8 : total <= 128 ? 4 : total <= 256 ? 2 : 1, sub = tid & (team - 1);
#pragma unroll 1
    for (int j = tid / team; j < (total + 31) / 32 * 32; j += kPick / team) {
        const Key me = j < total ? found[j] : 0;
        int place = 0, equal = 0;
#pragma unroll 1
        for (int o = sub; o < quads; o += team) {
            const ulonglong2 a = reinterpret_cast<const ulonglong2*>(found)[2 * o], b = reinterpret_cast<const ulonglong2*>(found)[2 * o + 1];
            place += (a.x > me) + (a.y > me) + (b.x > me) + (b.y > me);
            equal += (a.x == me) + (a.y == me) + (b.x == me) + (b.y == me);
        }
        int both = place << 16 | equal;                    // of at most 1024 keys
#pragma unroll 1
        for (int o = 1; o < team; o *= 2) both += __shfl_xor_sync(0xffffffffu, both, o);
        place = both >> 16;
        if (!me || sub || place >= s.k) continue;
        if ((both & 0xffff) > 1) {
            const Hit mine = rest[j];
            for (int o = 0; o < total; ++o)
                place += found[o] == me && (rest[o].beam < mine.beam || (rest[o].beam == mine.beam && rest[o].token < mine.token));
        }
        if (place < s.k) at_place[place] = (uint32_t)(j | rest[j].beam << 16);
    }
    __syncthreads();
    if (tid < s.k) {
        const uint32_t at = at_place[tid], j = at & 0xffffu;
        const bool     is = at != 0xffffffffu;
        const int      beam = is ? (int)(at >> 16) : -1;
        int            to = tid;
        if (s.settle) {
            // rows that something goes on from keep their best; the others take the places that are left, in order
            Key  seen = 0;
            int  others = 0;
            bool first = is;
            for (int o = 0; o < s.k; ++o) {
                const uint32_t u = at_place[o];
                const bool     leads = u != 0xffffffffu && !(seen >> (u >> 16) & 1);
                if (o < tid) {
                    others += !leads;
                    if (u != 0xffffffffu && (int)(u >> 16) == beam) first = false;
                }
                if (leads) seen |= (Key)1 << (u >> 16);
            }
            if (first) to = beam;
            else {
                to = 0;
                for (int skip = others;; ++to)
                    if (!(seen >> to & 1) && skip-- == 0) break;
            }
        }
        const int64_t o = request * s.k + to;
        s.out_score[o] = is ? rest[j].x : -INFINITY;
        s.out_parent[o] = is ? (int32_t)(first_row + beam) : -1;
        s.out_token[o] = is ? rest[j].token : -1;
    }
}

// ---- host side -----------------------------------------------------------------------------------------------

int check_beams(const nereus_logits_t* in, const nereus_beams_t* how) {
    if (int rc = check_view(in)) return rc;
    if (!how || how->beams < 1 || how->beams > NEREUS_BEAM_MAX || how->k < 1 || how->k > NEREUS_BEAM_MAX_K || how->reserved) return NEREUS_ERR_ARG;
    if (how->settle < 0 || how->settle > 1 || (how->settle && how->k != how->beams) || in->rows % how->beams) return NEREUS_ERR_ARG;
    return NEREUS_OK;
}

// How the rows are cut, and where the workspace's arrays are; returns its size.
size_t lay_out(const nereus_logits_t& in, const nereus_beams_t& how, Deal* deal, Select* s, char* workspace) {
    *deal = spread_of(in, kHalf, 0, 0, INT32_MAX);
    s->beams = how.beams;
    s->k = how.k;
    s->settle = how.settle;
    s->rows = (int32_t)in.rows;
    s->score = how.score;
    s->ended = how.ended;
    s->norm = how.norm;
    // no more parts of a request than one block looks through in a microsecond
    s->of_part = 1;
    while ((int64_t)((deal->layers + s->of_part - 1) / s->of_part) * how.beams > kParts) s->of_part *= 2;
    s->parts = (deal->layers + s->of_part - 1) / s->of_part;
    s->per_shard_1 = 1.f / (float)deal->per_shard;
    s->records = reinterpret_cast<Record*>(workspace);
    return (size_t)in.rows * s->parts * sizeof(Record);
}

template <class T> int beam_launch(const LogitsCut& cut, const Deal& deal, const Select& s, const Device& dev, cudaStream_t stream) {
    static std::atomic<bool> opted[kMaxDevices];
    constexpr int kMost = kParts * (int)sizeof(Record);
    if (!opted[dev.id].load()) {
        NEREUS_CUDA(cudaFuncSetAttribute(beam_pick_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost));
        opted[dev.id].store(true);
    }
    const int64_t units = (int64_t)s.rows * s.parts;
    beam_sum_kernel<T><<<(unsigned)std::min<int64_t>(units, kBlocks * dev.sms), kTH, 0, stream>>>(cut, deal, s);
    NEREUS_CUDA(cudaGetLastError());
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(s.rows / s.beams));
    cfg.blockDim = dim3(kPick);
    cfg.dynamicSmemBytes = (size_t)s.beams * s.parts * sizeof(Record);
    cfg.stream = stream;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;          // its blocks come while the last sums are made
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    NEREUS_CUDA(cudaLaunchKernelEx(&cfg, beam_pick_kernel<T>, cut, deal, s));
    return NEREUS_OK;
}

}  // namespace
}  // namespace nereus

extern "C" {

int nereus_beam_workspace(const nereus_logits_t* in, const nereus_beams_t* how, size_t* bytes) {
    if (int rc = check_beams(in, how)) return rc;
    if (!bytes) return NEREUS_ERR_ARG;
    if (in->rows == 0) { *bytes = 0; return NEREUS_OK; }
    Device dev;
    if (int rc = device_of(&dev)) return rc;
    Deal   deal;
    Select s;
    *bytes = lay_out(*in, *how, &deal, &s, nullptr);
    return NEREUS_OK;
}

int nereus_beam_select(const nereus_logits_t* in, const nereus_beams_t* how, void* workspace, size_t workspace_bytes, float* out_score,
                       int32_t* out_parent, int32_t* out_token, void* cuda_stream) {
    if (int rc = check_beams(in, how)) return rc;
    if (misaligned(how->score) || misaligned(how->ended) || misaligned(how->norm) || misaligned(out_score) || misaligned(out_parent) || misaligned(out_token))
        return NEREUS_ERR_ALIGN;
    if ((uintptr_t)workspace & 15) return NEREUS_ERR_ALIGN;
    if (in->rows == 0) return NEREUS_OK;
    if (!how->score || !out_score || !out_parent || !out_token || !workspace) return NEREUS_ERR_ARG;
    Device dev;
    if (int rc = device_of(&dev)) return rc;
    Deal   deal;
    Select s;
    if (lay_out(*in, *how, &deal, &s, (char*)workspace) > workspace_bytes) return NEREUS_ERR_TOO_SMALL;
    s.out_score = out_score;
    s.out_parent = out_parent;
    s.out_token = out_token;
    auto go = in->dtype == NEREUS_BF16 ? beam_launch<__nv_bfloat16> : beam_launch<float>;
    return go(cut_of(*in), deal, s, dev, (cudaStream_t)cuda_stream);
}

}  // extern "C"
