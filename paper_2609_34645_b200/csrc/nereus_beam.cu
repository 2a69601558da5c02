// One step of a beam search for sm_100a (nereus_beam_select): of what the beams of a request offer, score + x - log-sum-exp
// over the vocabulary, the k best.
//
// Every logit is read once; the floor is HBM bandwidth, with one exponential an element next (16 a clock and SM, which is what
// bf16 from HBM asks three quarters of).  Two launches:
//   * sum: the rows are cut into parts of a few layers, dealt out evenly to as many blocks as the GPU holds, whatever requests
//     they belong to.  Of its part of a row a block leaves every warp's sum of exponentials, and of every thread the largest
//     element that it has seen, in 16 bits rounded up: its note;
//   * pick: a block for a request puts the sums together to log-sum-exps, so that elements of different rows can be compared.
//     The notes are worth something then: of 8 sets of them the j-th largest bounds the k-th best hypothesis from below,
//     whatever the order of the rows.  Only vectors whose note reaches the bound are read again; what is found in them, a
//     few times k hypotheses, is ranked by counting.
// Where more is found than the list holds (rows of few distinct values: a mask's lowest value, say), the bound is made exact
// by counting the keys' bytes, the highest first, a pass over the request for each byte that is needed.
// Hypotheses are compared in 64 bits, as keys of (total / norm, lower index): within a row these order as the logits do.
#include "nereus_rows.hpp"

using namespace nereus;

namespace nereus {
namespace {

constexpr int kTH       = kThreads;               // of a summing block
constexpr int kItems    = 256;                    // layers in its table at a time
constexpr int kPart     = 16;                     // layers of a part, as a rule at most
constexpr int kParts    = 256;                    // parts of a request's rows, as far as a part's layers fit the table
constexpr int kPick     = 512;                    // threads of a picking block
constexpr int kPickWarps = kPick / 32;
constexpr int kSets     = 8;
constexpr int kFound    = 1024;                   // hypotheses that its list holds
constexpr int kNoted    = 2048;
typedef unsigned long long Key;

// Sums of exponentials are kept as (K, sum of 2^(x c - K)) with a whole number K near the largest x c, so that sums of different
// threads go together without another rounding; a thread adds up 2 vectors in 32 bits and these in 64.  c = log2(e) has 24
// bits, kLog2eLow is the rest: it is put right for the largest element of a row at the end, and an element at a distance of d
// from that is off by 2e-8 d of itself.  K stays within +-2^22: a row whose largest element lies beyond (a mask's lowest value
// in all of it, say) is summed again, by differences from it.
constexpr float  kLargestK = 0x1p22f;
constexpr double kLog2eLow = 1.4426950408889634 - (double)kLog2e, kLn2 = 0.69314718055994531;
struct Sum {
    double sum;
    float  k, top;                                // and the largest element
};
__device__ __forceinline__ double power_of_two(float k) {        // k whole and not above 0
    return !(k >= -1000.f) ? 0.0 : __longlong_as_double((long long)(1023 + (int)k) << 52);
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
    Sum*      sums;                               // [rows, parts, kWarps]
    uint16_t* notes;                              // [rows, parts, kTH]
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
    return layer_in<T, T, kTH>(in, LogitsCut(), row, shard, (l - shard * deal.per_shard) * kPerLayer<T, kTH>);
}

// ---- sums ----------------------------------------------------------------------------------------------------

template <class T>
__global__ void __launch_bounds__(kTH, 4) beam_sum_kernel(const __grid_constant__ LogitsCut in, const Deal deal, const Select s) {
    __shared__ __align__(16) uint4 ring[kStreamRing * kVecs];
    __shared__ Layer    table[kItems];
    __shared__ uint32_t unit_of[kItems];
    __shared__ int      of_warp[kWarps + 1];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    typename Vec<T>::Max top = Vec<T>::lowest();
    float  k = -kLargestK;
    double sum = 0.0;
    int    i = 0;
    const uint4* from = ring + tid;
    const Pair   c = pair(kLog2e, kLog2e);
    const int64_t units = (int64_t)s.rows * s.parts;
    const int     log_part = __ffs(s.of_part) - 1, slots = kItems >> log_part;
    for (int64_t first = blockIdx.x; first < units; first += (int64_t)slots * gridDim.x) {
        // of the next units those whose rows are read, in order
        const int64_t unit = first + (int64_t)tid * gridDim.x;
        bool is = tid < slots && unit < units;
        if (is) {
            float score, norm;
            int   ended;
            is = offers(s, (uint32_t)unit % (uint32_t)s.rows, in.vocab, &score, &norm, &ended) && (uint32_t)ended >= (uint32_t)in.vocab;
        }
        const uint32_t who = __ballot_sync(0xffffffffu, is);
        __syncthreads();
        if (lane == 0) of_warp[warp] = __popc(who);
        __syncthreads();
        int before = 0, n = 0;
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) before += of_warp[w];
            n += of_warp[w];
        }
        if (is) unit_of[before + __popc(who & ((1u << lane) - 1))] = (uint32_t)unit;
        __syncthreads();
        const int items = n << log_part;
        if (tid < items) {
            const uint32_t u = unit_of[tid >> log_part];
            const int      part = (int)(u / (uint32_t)s.rows);
            table[tid] = layer_at<T>(in, deal, s, u - (uint32_t)part * (uint32_t)s.rows, (part << log_part) + (tid & (s.of_part - 1)));
        }
        __syncthreads();
#pragma unroll 1
        for (int l = 0; l < kStreamRing; ++l) load_layer<T, kTH>(table, ring, l, l, items);
        int slot = 0;
#pragma unroll 1
        for (int item = 0; item < items; ++item) {
            copy_wait<kStreamRing - 1>();
            const uint4 a = from[slot * kVecs], b = from[slot * kVecs + kTH];
            if (item + kStreamRing < items) load_layer<T, kTH>(table, ring, slot, item + kStreamRing, items);
            else copy_commit();
            slot = slot + 1 == kStreamRing ? 0 : slot + 1;
            top = Vec<T>::join(top, Vec<T>::join(Vec<T>::max(a), Vec<T>::max(b)));
            const float v = Vec<T>::value(top);
            // an element ahead of K carries the roundings of the distance: 2^4 at most
            if (v * kLog2e > k + 4.f) {
                const float to = fminf(fmaxf(rintf(v * kLog2e), -kLargestK), kLargestK);
                sum *= power_of_two(k - to);
                k = to;
            }
            const Pair   minus = pair(-k, -k);
            const float2 h = halves(add2(exp_sum<T, false>(a, c, c, minus), exp_sum<T, false>(b, c, c, minus)));
            sum += (double)(h.x + h.y);
            if (++i == s.of_part) {
                const uint32_t u = unit_of[item >> log_part];
                const int      part = (int)(u / (uint32_t)s.rows);
                const int64_t  at = (int64_t)(u - (uint32_t)part * (uint32_t)s.rows) * s.parts + part;
                s.notes[at * kTH + tid] = note_of(v);
                const float all = warp_max(k), most = warp_max(v);
                double      of_lanes = sum * power_of_two(k - all);
#pragma unroll
                for (int o = 16; o; o >>= 1) of_lanes += __shfl_xor_sync(0xffffffffu, of_lanes, o);
                if (lane == 0) s.sums[at * kWarps + warp] = {of_lanes, all, most};
                top = Vec<T>::lowest();
                k = -kLargestK;
                sum = 0.0;
                i = 0;
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

template <class T>
__global__ void __launch_bounds__(kPick) beam_pick_kernel(const __grid_constant__ LogitsCut in, const Deal deal, const Select s) {
    constexpr int E = kPerVec<T>;
    __shared__ Beam     beams[NEREUS_BEAM_MAX];
    __shared__ __align__(16) Key found[kFound];
    __shared__ struct { uint32_t index; float total; } rest[kFound];       // index: beam * vocab + token
    __shared__ uint32_t noted[kNoted];
    __shared__ uint32_t peak[kPick], histogram[256], at_place[NEREUS_BEAM_MAX_K], choice[4], of_warp[kPickWarps];
    __shared__ int      n_found, n_noted;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t request = blockIdx.x, first_row = request * s.beams;

    for (int b = tid; b < s.beams; b += kPick) {
        Beam  r;
        float norm;
        const bool is = offers(s, first_row + b, in.vocab, &r.score, &norm, &r.ended);
        if ((uint32_t)r.ended >= (uint32_t)in.vocab) r.ended = -1;
        r.norm = (double)norm;
        r.inverse = 1.f / norm;
        r.off = is ? (double)r.score : (double)NAN;
        r.least = NAN;
        beams[b] = r;
    }
    if (tid == 0) n_found = n_noted = 0;
    __syncthreads();
    asm volatile("griddepcontrol.wait;" ::: "memory");                      // the sums and notes are there

    // every row's log-sum-exp, a warp for each
    const int entries = s.parts * kWarps;
    for (int b = warp; b < s.beams; b += kPickWarps) {
        Beam& r = beams[b];
        if (r.off != r.off || r.ended >= 0) {
            if (lane == 0) r.off_1 = NAN;
            continue;
        }
        const Sum* sums = s.sums + (first_row + b) * entries;
        float  k = -INFINITY, top = -INFINITY;
        double sum = 0.0;
        for (int e = lane; e < entries; e += 32) {
            const uint4 u = __ldcg(reinterpret_cast<const uint4*>(sums + e));
            const float of_k = __uint_as_float(u.z), to = fmaxf(k, of_k);
            sum = fma(__longlong_as_double((long long)((Key)u.y << 32 | u.x)), power_of_two(of_k - to), sum * power_of_two(k - to));
            k = to;
            top = fmaxf(top, __uint_as_float(u.w));
        }
        const float all = warp_max(k);
        top = warp_max(top);
        sum *= power_of_two(k - all);
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        double lse = kLn2 * ((double)all + log2_of(sum) + (double)top * kLog2eLow);
        if (fabsf(top * kLog2e) >= kLargestK && fabsf(top) < INFINITY) {
            sum = 0.0;
            for (int l = 0; l < deal.layers; ++l) {
                const Layer L = layer_at<T>(in, deal, s, first_row + b, l);
                for (int vec = lane; vec < kVecs; vec += 64)
                    sum += (double)exp_sum_far<T>(edge_vector<T>(L, vec), edge_vector<T>(L, vec + 32), top, pair(kLog2e, kLog2e));
            }
            for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            lse = (double)top + kLn2 * log2_of(sum);
        }
        if (lane == 0) {
            r.off = fabsf(top) < INFINITY && sum == sum ? r.off - lse : (double)NAN;
            r.off_1 = (float)r.off;
        }
    }
    __syncthreads();

    // What an element is worth: off + x, by the norm; in 64 bits, and in 32 and a little less for the roundings.
    auto worth = [&](const Beam& r, float x, double* total) {
        *total = r.off + (double)x;
        return s.norm ? *total / r.norm : *total;
    };
    auto worth_below = [](const Beam& r, float x) {
        const float w = fmaf(-1e-6f, fabsf(r.off_1) + fabsf(x), r.off_1 + x) * r.inverse;
        return fmaf(-1e-6f, fabsf(w), w);
    };
    // Notes, 8 at a time: those of one row and part.
    const uint4* const all_notes = reinterpret_cast<const uint4*>(s.notes + first_row * s.parts * kTH);
    constexpr int kEach = kTH / 8;
    const int     groups = s.beams * s.parts * kEach;
    const float   parts_1 = 1.f / (float)(s.parts * kEach);
    {
        float most = -INFINITY;
#pragma unroll 4
        for (int g = tid; g < groups; g += kPick) {
            const Beam& r = beams[quotient(g, s.parts * kEach, parts_1)];
            const uint4 v = __ldcg(all_notes + g);
            // the largest of 8 notes is the largest as bf16; that of a fp32 was rounded up: the next below is not above it
            const float up = Vec<__nv_bfloat16>::value(Vec<__nv_bfloat16>::max(v));
            const float x = sizeof(T) == 2 ? up : note_below((uint16_t)(__float_as_uint(up) >> 16));
            if (up > -INFINITY && r.off_1 == r.off_1) most = fmaxf(most, worth_below(r, x));
        }
        peak[tid] = key_of(most);
    }
    __syncthreads();
    // of each set the j-th largest; the least of these bounds the k-th best from below
    {
        const int j = (s.k + kSets - 1) / kSets;
        uint32_t  t = 0xffffffffu;
        if (warp < kSets) {
            uint32_t key = 0;
            // a row's notes are on neighbouring threads: every set has its share of every row's
            for (int x = lane * kSets + warp; x < kPick; x += kSets * 32) key = max(key, peak[x]);
#pragma unroll 1
            for (int i = 0; i < j; ++i) {
                t = __reduce_max_sync(0xffffffffu, key);
                if (lane == __ffs(__ballot_sync(0xffffffffu, key == t)) - 1) key = 0;
            }
            if (lane == 0) of_warp[warp] = t;
        }
        __syncthreads();
        t = __reduce_min_sync(0xffffffffu, lane < kSets ? of_warp[lane] : 0xffffffffu);
        const float bound = t > kKeyMinusInf ? value_of(t) : -INFINITY;
        for (int b = tid; b < s.beams; b += kPick) {
            Beam& r = beams[b];
            // the least x whose worth reaches the bound, or a little less
            const float norm = (float)r.norm, at = fmaf(bound, norm, -r.off_1);
            r.least = r.off_1 != r.off_1 ? NAN : bound > -INFINITY ? fmaf(-1e-6f, fabsf(bound * norm) + fabsf(r.off_1), at) : -INFINITY;
        }
        __syncthreads();
        // the notes that reach it
#pragma unroll 4
        for (int g = tid; g < groups; g += kPick) {
            const float least = beams[quotient(g, s.parts * kEach, parts_1)].least;
            const uint4 v = __ldcg(all_notes + g);
            const float up = Vec<__nv_bfloat16>::value(Vec<__nv_bfloat16>::max(v));
            if (!(up >= least && up > -INFINITY)) continue;
            float x[8];
            unpack<__nv_bfloat16>(v, x);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (x[e] >= least && x[e] > -INFINITY) {
                    const int at = atomicAdd(&n_noted, 1);
                    if (at < kNoted) noted[at] = (uint32_t)(g * 8 + e);
                }
        }
    }
    __syncthreads();

    // f(key, total, index) for every element of vector `vec` of a layer that may be among the best
    auto look = [&](int b, const Layer& L, int vec, auto f) {
        const Beam& r = beams[b];
        const int   lo = L.lo - vec * E, hi = L.hi - vec * E;
        if (hi <= 0 || lo >= E) return;
        float x[E];
        unpack<T>(edge_vector<T>(L, vec), x);
        uint32_t hits = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) hits |= (x[e] >= r.least && x[e] > -INFINITY ? 1u : 0u) << e;
        hits &= bits_between(lo, hi, E);
#pragma unroll 1
        for (; hits; hits &= hits - 1) {
            const int e = __ffs(hits) - 1;
            float y = x[0];
#pragma unroll
            for (int o = 1; o < E; ++o) y = o == e ? x[o] : y;
            double    total;
            const Key key = key_of_double(worth(r, y, &total));
            if (key > kKeyNone) f(key, (float)total, (uint32_t)(b * in.vocab + L.token + vec * E + e));
        }
    };
    auto push = [&](Key key, float total, uint32_t index) {
        const int at = atomicAdd(&n_found, 1);
        if (at < kFound) {
            found[at] = key;
            rest[at] = {index, total};
        }
    };
    // the beams that have ended offer themselves
    auto each_ended = [&](auto f) {
        if (tid >= s.beams) return;
        const Beam& r = beams[tid];
        if (r.ended >= 0 && r.off == r.off) f(key_of_double(s.norm ? r.off / r.norm : r.off), r.score, (uint32_t)(tid * in.vocab + r.ended));
    };
    const int log_part = __ffs(s.of_part) - 1, noted_all = n_noted;
    if (noted_all <= kNoted) {
        // every vector of a note on a thread of its own
        const int log_vecs = log_part + 1, vecs = noted_all << log_vecs;
        for (int j = tid; j < vecs; j += kPick) {
            const uint32_t which = noted[j >> log_vecs];
            const int      row_part = which / kTH, b = quotient(row_part, s.parts, parts_1 * kEach), part = row_part - b * s.parts;
            const int      l = (part << log_part) + (j >> 1 & (s.of_part - 1));
            look(b, layer_at<T>(in, deal, s, first_row + b, l), which % kTH + (j & 1) * kTH, push);
        }
    }
    each_ended(push);
    __syncthreads();

    if (noted_all > kNoted || n_found > kFound) {
        // The k-th key exactly, or as much of it as leaves few enough: byte by byte of (key, ~index), the 12 bytes highest
        // first, by the number of hypotheses that share the bytes found so far.
        Key      key_is = 0, key_mask = 0;
        uint32_t index_is = 0, index_mask = 0;
        int      left = s.k, above = 0;
        auto each = [&](auto f) {
            for (int b = 0; b < s.beams; ++b) {
                if (beams[b].least != beams[b].least) continue;
                for (int l = 0; l < deal.layers; ++l) {
                    const Layer L = layer_at<T>(in, deal, s, first_row + b, l);
                    for (int vec = tid; vec < kVecs; vec += kPick) look(b, L, vec, f);
                }
            }
            each_ended(f);
        };
#pragma unroll 1
        for (int byte = 0; byte < 12; ++byte) {
            if (tid < 256) histogram[tid] = 0;
            if (tid == 0) choice[0] = 256;
            __syncthreads();
            int      bin = 0;
            uint32_t run = 0;                              // elements of one bin come one after the other
            each([&](Key key, float, uint32_t index) {
                if (((key ^ key_is) & key_mask) || ((~index ^ index_is) & index_mask)) return;
                const int b = (int)(byte < 8 ? key >> (56 - 8 * byte) : ~index >> (88 - 8 * byte)) & 255;
                if (b != bin) {
                    if (run) atomicAdd(&histogram[bin], run);
                    bin = b;
                    run = 0;
                }
                ++run;
            });
            if (run) atomicAdd(&histogram[bin], run);
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
            __syncthreads();
            if (b == 256) break;                           // fewer than k in all: everything is taken
            above += (int)higher;
            left -= (int)higher;
            if (byte < 8) { key_is |= (Key)b << (56 - 8 * byte); key_mask |= (Key)255 << (56 - 8 * byte); }
            else { index_is |= b << (88 - 8 * byte); index_mask |= 255u << (88 - 8 * byte); }
            if (above + (int)same <= kFound) break;
        }
        if (tid == 0) n_found = 0;
        __syncthreads();
        // everything from the bytes found on
        each([&](Key key, float total, uint32_t index) {
            const Key top = key & key_mask;
            if (top > key_is || (top == key_is && (~index & index_mask) >= index_is)) push(key, total, index);
        });
        __syncthreads();
    }

    // which hypothesis is the j-th, and its beam in the upper half
    const int total = n_found, quads = (total + 3) / 4;    // keys are read four at a time
    if (tid < s.k) at_place[tid] = 0xffffffffu;
    if (tid < 4 * quads - total) found[total + tid] = 0;
    __syncthreads();
    // a key on `team` neighbouring threads that share the comparing
    const int team = total <= 32 ? 16 : total <= 64 ? 8 : total <= 128 ? 4 : total <= 256 ? 2 : 1, sub = tid & (team - 1);
    for (int j = tid / team; j < (total + 31) / 32 * 32; j += kPick / team) {
        const Key me = j < total ? found[j] : 0;
        int place = 0, equal = 0;
#pragma unroll 2
        for (int o = sub; o < quads; o += team) {
            const ulonglong2 a = reinterpret_cast<const ulonglong2*>(found)[2 * o], b = reinterpret_cast<const ulonglong2*>(found)[2 * o + 1];
            place += (a.x > me) + (a.y > me) + (b.x > me) + (b.y > me);
            equal += (a.x == me) + (a.y == me) + (b.x == me) + (b.y == me);
        }
        for (int o = 1; o < team; o *= 2) {
            place += __shfl_xor_sync(0xffffffffu, place, o);
            equal += __shfl_xor_sync(0xffffffffu, equal, o);
        }
        if (!me || sub || place >= s.k) continue;
        const uint32_t index = rest[j].index;
        if (equal > 1)
            for (int o = 0; o < total; ++o) place += found[o] == me && rest[o].index < index;
        if (place < s.k) at_place[place] = (uint32_t)j | index / (uint32_t)in.vocab << 16;
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
        s.out_score[o] = is ? rest[j].total : -INFINITY;
        s.out_parent[o] = is ? (int32_t)(first_row + beam) : -1;
        s.out_token[o] = is ? (int32_t)(rest[j].index - (uint32_t)beam * (uint32_t)in.vocab) : -1;
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
size_t lay_out(const nereus_logits_t& in, const nereus_beams_t& how, int sms, Deal* deal, Select* s, char* workspace) {
    *deal = spread_of(in, kTH, 0, 0, INT32_MAX);
    s->beams = how.beams;
    s->k = how.k;
    s->settle = how.settle;
    s->rows = (int32_t)in.rows;
    s->score = how.score;
    s->ended = how.ended;
    s->norm = how.norm;
    // A few parts for every block that the GPU holds (4 on an SM), so that they end together; no more of a request than one
    // block puts together in a microsecond.
    const int64_t all = in.rows * deal->layers;
    s->of_part = 1;
    while ((s->of_part < kPart && all / (2 * s->of_part) >= 16 * sms) || (s->of_part < kItems && (int64_t)((deal->layers + s->of_part - 1) / s->of_part) * how.beams > kParts))
        s->of_part *= 2;
    s->parts = (deal->layers + s->of_part - 1) / s->of_part;
    s->per_shard_1 = 1.f / (float)deal->per_shard;
    const size_t units = (size_t)in.rows * s->parts, sums = units * kWarps * sizeof(Sum);
    s->sums = reinterpret_cast<Sum*>(workspace);
    s->notes = reinterpret_cast<uint16_t*>(workspace + sums);
    return sums + units * kTH * 2;
}

template <class T> int beam_launch(const LogitsCut& cut, const Deal& deal, const Select& s, const Device& dev, cudaStream_t stream) {
    const int64_t units = (int64_t)s.rows * s.parts;
    // an odd number of blocks: beams that offer nothing (all but a request's first on its first step) come to all of them
    const int64_t most = 4 * dev.sms - 1;
    beam_sum_kernel<T><<<(unsigned)std::min<int64_t>(units, most), kTH, 0, stream>>>(cut, deal, s);
    NEREUS_CUDA(cudaGetLastError());
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(s.rows / s.beams));
    cfg.blockDim = dim3(kPick);
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
    *bytes = lay_out(*in, *how, dev.sms, &deal, &s, nullptr);
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
    if (lay_out(*in, *how, dev.sms, &deal, &s, (char*)workspace) > workspace_bytes) return NEREUS_ERR_TOO_SMALL;
    s.out_score = out_score;
    s.out_parent = out_parent;
    s.out_token = out_token;
    auto go = in->dtype == NEREUS_BF16 ? beam_launch<__nv_bfloat16> : beam_launch<float>;
    return go(cut_of(*in), deal, s, dev, (cudaStream_t)cuda_stream);
}

}  // extern "C"
