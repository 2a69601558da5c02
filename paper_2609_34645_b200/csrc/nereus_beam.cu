// One step of a beam search for sm_100a (nereus_beam_select): of what the beams of a request offer, score + x - log-sum-exp
// over the vocabulary, the k best.
//
// Every logit is read once; the floor is HBM bandwidth, with one exponential an element next.  A cluster takes a request:
//   * its blocks share every row of it (a few rows of 128256 are a megabyte, which one SM would read for 10 us), each summing
//     the exponentials of its layers and noting the largest element of every thread's vectors of one or a few layers;
//   * one exchange through distributed shared memory gives every block the log-sum-exp of every row, so that elements of
//     different rows can be compared, and the largest elements that the warps have seen: the k-th largest of these bounds
//     the k-th best hypothesis from below, whatever the order of the rows;
//   * only vectors whose note reaches the bound are read again (from L2); what is found in them, little more than k
//     hypotheses, goes to the first block, which ranks it by counting.
// Where more is found than the lists hold (rows of few distinct values: a mask's lowest value, say), the bound is made exact
// by counting the keys' bytes, the highest first, a pass over the request for each byte that is needed.
// Hypotheses are compared in 64 bits, as keys of (total / norm, lower index): within a row these order as the logits do.
#include "nereus_rows.hpp"

using namespace nereus;

namespace nereus {
namespace {

constexpr int kMaxNotes = 64;                     // of a thread
constexpr int kMaxItems = 512;                    // layers in the block's table at a time
constexpr int kFound    = 1024;                   // hypotheses that a list holds
constexpr int kNoted    = (kStreamRing * kVecs * 16 - kFound * 16) / 4;
typedef unsigned long long Key;

struct Found {
    Key      key;
    uint32_t index;                               // beam * vocab + token
    float    total;
};
static_assert(sizeof(Found) == 16, "Found is moved as 16 bytes");

struct Select {
    int32_t beams, k, settle, per_note, notes;    // layers of a note, notes of a row
    const float*   score;
    const int32_t* ended;
    const float*   norm;
    float*   out_score;
    int32_t *out_parent, *out_token;
};

// orders as the values do, -0 as +0
__device__ __forceinline__ Key key_of_double(double x) {
    const Key u = (Key)__double_as_longlong(x + 0.0);
    return u >> 63 ? ~u : u | (Key)1 << 63;
}
constexpr Key kKeyNone = 0x000fffffffffffffull;   // of -inf

__device__ __forceinline__ uint32_t peer_load(const void* p, int rank) {
    uint32_t r;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(r) : "r"(peer_address(p, rank)) : "memory");
    return r;
}
__device__ __forceinline__ float2 peer_load2(const void* p, int rank) {
    float2 r;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(r.x), "=f"(r.y) : "r"(peer_address(p, rank)) : "memory");
    return r;
}
__device__ __forceinline__ uint4 peer_load4(const void* p, int rank) {
    uint4 r;
    asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(peer_address(p, rank)) : "memory");
    return r;
}

// A row of the request that is read.
struct Live {
    double   off, norm;                           // score - log-sum-exp; NaN: the row offers nothing
    float    least;                               // elements below are not among the best; NaN: none is
    int32_t  beam;
};

template <class T>
__global__ void __launch_bounds__(kThreads, 4) beam_kernel(const __grid_constant__ LogitsCut in, const Deal deal, const Select s, const Scale scale) {
    constexpr int E = kPerVec<T>;
    extern __shared__ __align__(16) unsigned char dynamic[];
    __shared__ float2   part[NEREUS_BEAM_MAX][kWarps];     // of every row and warp: largest element, sum of exponentials
    __shared__ float    quarter[8][kWarps * 4];            // ... of the first rows and every 8 lanes: largest element
    __shared__ Live     live[NEREUS_BEAM_MAX];
    __shared__ uint32_t histogram[2][256];
    __shared__ uint32_t choice[4];
    __shared__ int      n_live, n_found, n_noted, n_exact;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int blocks = 1 << deal.log_c, rank = (int)blockIdx.x & (blocks - 1);
    const int64_t request = blockIdx.x >> deal.log_c, first_row = request * s.beams;

    uint4*    ring = reinterpret_cast<uint4*>(dynamic);
    Layer*    table = reinterpret_cast<Layer*>(ring + kStreamRing * kVecs);
    const int room = min(kMaxItems, s.beams * deal.mine);
    uint16_t* notes = reinterpret_cast<uint16_t*>(table + room) + tid;      // of this thread
    Found*    found = reinterpret_cast<Found*>(ring);                       // once the rows have gone through
    uint32_t* noted = reinterpret_cast<uint32_t*>(found + kFound);

    // the rows that are read, in order
    if (warp < 2) {
        // both halves' counts on both warps: 64 beams at most
        int before = 0;
        for (int half = 0; half <= warp; ++half) {
            const int b = half * 32 + lane;
            bool is = b < s.beams;
            float norm = 1.f;
            if (is) {
                const float score = s.score[first_row + b];
                if (s.norm) norm = s.norm[first_row + b];
                is = fabsf(score) < INFINITY && norm > 0.f && norm < INFINITY && !(s.ended && (uint32_t)s.ended[first_row + b] < (uint32_t)in.vocab);
            }
            const uint32_t who = __ballot_sync(0xffffffffu, is);
            if (half == warp && is) {
                Live& l = live[before + __popc(who & ((1u << lane) - 1))];
                l.beam = b;
                l.norm = norm;
            }
            before += __popc(who);
        }
        if (warp == 1 && lane == 0) n_live = before;
    }
    if (tid == 0) n_found = n_noted = n_exact = 0;
    __syncthreads();
    const int n = n_live, mine = deal.mine;

    // which of a row's shares this block has: rows take turns, so that short rows come to all blocks
    auto share_of = [&](int q) { return (rank + live[q].beam) & (blocks - 1); };
    auto layer_at = [&](int q, int i) {
        return layer_of<T, T>(in, LogitsCut(), deal, first_row + live[q].beam, share_of(q), i);
    };

    {
        Running<true> running(scale.high, scale.low);
        typename Vec<T>::Max top = Vec<T>::lowest();
        float to_note = -INFINITY;
        int   q = 0, i = 0, in_note = 0;
        for (int first = 0; first < n * mine; first += room) {
            const int items = min(room, n * mine - first);
            if (first) __syncthreads();
            for (int j = tid; j < items; j += kThreads) table[j] = layer_at((first + j) / mine, (first + j) % mine);
            __syncthreads();
            start_stream<T, kThreads, kStreamRing>(table, ring, items);
            stream<T, kThreads, kStreamRing>(table, ring, items, [&](int item, uint4 a, uint4 b) {
                const Layer& L = table[item];
                if (L.hi > L.lo) {                         // the same for the block; else the ring holds another layer's vectors
                    const typename Vec<T>::Max m = Vec<T>::join(Vec<T>::max(a), Vec<T>::max(b));
                    const float v = Vec<T>::value(m);
                    top = Vec<T>::join(top, m);
                    to_note = fmaxf(to_note, v);
                    running.see(v);
                    running.template add<T>(a, b);
                }
                const bool end = i + 1 == mine;
                if (++in_note == s.per_note || end) {
                    notes[(q * s.notes + i / s.per_note) * kThreads] = note_of(to_note);
                    to_note = -INFINITY;
                    in_note = 0;
                }
                if (end) {
                    const float m = Vec<T>::value(top), all = warp_max(m);
                    const float sum = warp_sum(running.sum * scale_finely(running.base, all, 1.4426950408889634));
                    if (lane == 0) part[q][warp] = make_float2(all, sum);
                    if (q < 8) {
                        float g = m;
#pragma unroll
                        for (int o = 1; o < 8; o *= 2) g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, o));
                        if ((lane & 7) == 0) quarter[q][warp * 4 + (lane >> 3)] = g;
                    }
                    running = Running<true>(scale.high, scale.low);
                    top = Vec<T>::lowest();
                    i = 0;
                    ++q;
                } else {
                    ++i;
                }
            });
        }
    }
    cluster_arrive();
    cluster_wait();

    // every row's log-sum-exp, the same in every block: its shares in the row's own order
    for (int q = warp; q < n; q += kWarps) {
        float2    v[kMaxCtas * kWarps / 32];
        float     all = -INFINITY;
        const int entries = blocks * kWarps;
#pragma unroll
        for (int j = 0; j < kMaxCtas * kWarps / 32; ++j) {
            const int e = j * 32 + lane;
            v[j] = e < entries ? peer_load2(&part[q][e % kWarps], (e / kWarps - live[q].beam) & (blocks - 1)) : make_float2(-INFINITY, 0.f);
            all = fmaxf(all, v[j].x);
        }
        all = warp_max(all);
        double sum = 0.0;
#pragma unroll
        for (int j = 0; j < kMaxCtas * kWarps / 32; ++j) sum += (double)v[j].y * (double)scale_finely(v[j].x, all, 1.4426950408889634);
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) {
            const bool ok = all > -INFINITY && all < INFINITY && sum > 0.0 && sum < (double)INFINITY;
            live[q].off = ok ? (double)s.score[first_row + live[q].beam] - ((double)all + log(sum)) : NAN;
        }
    }
    __syncthreads();

    // what an element is worth: off + x, by the norm; in 64 bits
    auto worth = [&](const Live& l, float x, double* total) {
        *total = l.off + (double)x;
        return s.norm ? *total / l.norm : *total;
    };

    // the k-th largest of the groups' largest elements; few rows: groups of 8 lanes, else of a warp
    {
        const bool small = n * blocks * kWarps < 4 * s.k && n <= 8;
        const int  of_row = blocks * (small ? kWarps * 4 : kWarps);
        float      v = -INFINITY;
        for (int g = tid; g < n * of_row; g += kThreads) {
            const int q = g / of_row, e = g - q * of_row;
            if (live[q].off != live[q].off) continue;
            const float x = small ? __uint_as_float(peer_load(&quarter[q][e & (kWarps * 4 - 1)], e / (kWarps * 4)))
                                  : __uint_as_float(peer_load(&part[q][e & (kWarps - 1)].x, e / kWarps));
            double total;
            if (x > -INFINITY) v = fmaxf(v, __double2float_rd(worth(live[q], x, &total)));
        }
        const uint32_t key = key_of(v);
        uint32_t       t = 0;
#pragma unroll 1
        for (int bit = 31; bit >= 16; --bit) {
            const uint32_t u = t | 1u << bit;
            if (__syncthreads_count(key >= u) >= s.k) t = u;
        }
        if (tid < n) {
            Live&       l = live[tid];
            const float bound = t > kKeyMinusInf ? value_of(t) : -INFINITY;
            // the least x whose worth reaches the bound, or a little less
            const double at = (double)bound * l.norm - l.off, slack = 1e-14 * (fabs((double)bound * l.norm) + fabs(l.off));
            l.least = l.off != l.off ? NAN : bound > -INFINITY ? __double2float_rd(at - slack) : -INFINITY;
        }
    }
    __syncthreads();

    // f(key, total, index) for every element of this thread's vector `vec` of a layer that may be among the best
    auto look = [&](const Live& l, const Layer& L, int vec, auto f) {
        const int a = L.lo - vec * E, b = L.hi - vec * E;
        if (b <= 0 || a >= E) return;
        float x[E];
        unpack<T>(edge_vector<T>(L, vec), x);
        const uint32_t inside = bits_between(a, b, E);
#pragma unroll
        for (int e = 0; e < E; ++e)
            if ((inside >> e & 1u) && x[e] >= l.least && x[e] > -INFINITY) {
                double    total;
                const Key key = key_of_double(worth(l, x[e], &total));
                if (key > kKeyNone) f(key, (float)total, (uint32_t)(l.beam * in.vocab + L.token + vec * E + e));
            }
    };
    auto push = [&](int* count, Key key, float total, uint32_t index) {
        const int at = atomicAdd(count, 1);
        if (at < kFound) found[at] = {key, index, total};
    };
    // the beams that have ended offer themselves; the first block sees to them
    auto each_ended = [&](auto f) {
        if (rank || !s.ended || tid >= s.beams) return;
        const int   token = s.ended[first_row + tid];
        const float score = s.score[first_row + tid], norm = s.norm ? s.norm[first_row + tid] : 1.f;
        if ((uint32_t)token >= (uint32_t)in.vocab || !(fabsf(score) < INFINITY) || !(norm > 0.f && norm < INFINITY)) return;
        f(key_of_double(s.norm ? (double)score / (double)norm : (double)score), score, (uint32_t)(tid * in.vocab + token));
    };

    for (int q = 0; q < n; ++q) {
        const float least = live[q].least;
        for (int j = 0; j < s.notes; ++j) {
            const float top = value_of_note(notes[(q * s.notes + j) * kThreads]);
            if (top >= least && top > -INFINITY) {
                const int at = atomicAdd(&n_noted, 1);
                if (at < kNoted) noted[at] = (uint32_t)((q * s.notes + j) * kThreads + tid);
            }
        }
    }
    __syncthreads();
    const bool full = n_noted > kNoted;
    if (!full) {
        const int vecs = n_noted * 2 * s.per_note;
        for (int j = tid; j < vecs; j += kThreads) {
            const uint32_t which = noted[j / (2 * s.per_note)], note = which / kThreads;
            const int      q = note / s.notes, i = note % s.notes * s.per_note + j / 2 % s.per_note, vec = which % kThreads + j % 2 * kThreads;
            if (i < mine) look(live[q], layer_at(q, i), vec, [&](Key key, float total, uint32_t index) { push(&n_found, key, total, index); });
        }
    }
    each_ended([&](Key key, float total, uint32_t index) { push(&n_found, key, total, index); });
    __syncthreads();
    if (tid == 0 && full) n_found = kFound + 1;
    cluster_arrive();
    cluster_wait();

    int* count = &n_found;
    int  total = 0;
    bool crowded = false;
    for (int r = 0; r < blocks; ++r) {
        const int c = (int)peer_load(&n_found, r);
        crowded |= c > kFound;
        total += c;
    }
    if (crowded || total > kFound) {
        // The k-th key exactly, or as much of it as leaves few enough: byte by byte of (key, ~index), the 12 bytes highest
        // first, by the number of hypotheses that share the bytes found so far.
        Key      key_is = 0, key_mask = 0;
        uint32_t index_is = 0, index_mask = 0;
        int      left = s.k, above = 0;
        bool     done = false;
        auto each = [&](auto f) {
            for (int q = 0; q < n; ++q) {
                if (live[q].off != live[q].off) continue;
                for (int i = 0; i < mine; ++i) {
                    const Layer L = layer_at(q, i);
                    for (int vec = tid; vec < kVecs; vec += kThreads) look(live[q], L, vec, f);
                }
            }
            each_ended(f);
        };
#pragma unroll 1
        for (int byte = 0; byte < 12 && !done; ++byte) {
            uint32_t* const h = histogram[byte & 1];
            h[tid] = 0;
            __syncthreads();
            int      bin = 0;
            uint32_t run = 0;                              // elements of one bin come one after the other
            each([&](Key key, float, uint32_t index) {
                if (((key ^ key_is) & key_mask) || ((~index ^ index_is) & index_mask)) return;
                const int b = (int)(byte < 8 ? key >> (56 - 8 * byte) : ~index >> (88 - 8 * byte)) & 255;
                if (b != bin) {
                    if (run) atomicAdd(&h[bin], run);
                    bin = b;
                    run = 0;
                }
                ++run;
            });
            if (run) atomicAdd(&h[bin], run);
            cluster_arrive();
            cluster_wait();
            uint32_t c = 0;
            for (int r = 0; r < blocks; ++r) c += peer_load(&h[255 - tid], r);
            // the bins from the highest down: how many there are up to this one
            uint32_t upto = c;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const uint32_t u = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += u;
            }
            __shared__ uint32_t of_warp[kWarps];
            if (lane == 31) of_warp[warp] = upto;
            if (tid == 0) choice[0] = 256;
            __syncthreads();
            for (int w = 0; w < warp; ++w) upto += of_warp[w];
            if (upto >= (uint32_t)left && upto - c < (uint32_t)left) {
                choice[0] = 255 - tid;
                choice[1] = upto - c;
                choice[2] = c;
            }
            __syncthreads();
            const uint32_t b = choice[0];
            if (b == 256) { done = true; break; }          // fewer than k in all: everything is taken
            above += (int)choice[1];
            left -= (int)choice[1];
            if (byte < 8) { key_is |= (Key)b << (56 - 8 * byte); key_mask |= (Key)255 << (56 - 8 * byte); }
            else { index_is |= b << (88 - 8 * byte); index_mask |= 255u << (88 - 8 * byte); }
            done = above + (int)choice[2] <= kFound;
            __syncthreads();
        }
        // everything from the bytes found on; this list's counter is another one, since the others may still read the first
        count = &n_exact;
        each([&](Key key, float total, uint32_t index) {
            const Key k = key & key_mask;
            if (k > key_is || (k == key_is && (~index & index_mask) >= index_is)) push(&n_exact, key, total, index);
        });
        cluster_arrive();
        cluster_wait();
    }

    if (rank == 0) {
        // the other blocks' lists behind this one's
        int at = min(*count, kFound);
        for (int r = 1; r < blocks; ++r) {
            const int c = min((int)peer_load(count, r), kFound - at);
            for (int j = tid; j < c; j += kThreads) *reinterpret_cast<uint4*>(found + at + j) = peer_load4(found + j, r);
            at += c;
        }
        total = at;
    }
    cluster_arrive();                                      // nothing is read from the others from here on
    if (rank == 0) {
        __syncthreads();
        uint32_t* const at_place = noted;                  // which hypothesis is the j-th, and its beam in the upper half
        if (tid < s.k) at_place[tid] = 0xffffffffu;
        __syncthreads();
        const int team = total <= 32 ? 8 : total <= 64 ? 4 : total <= 128 ? 2 : 1, sub = tid & (team - 1);
        for (int j = tid / team; j < (total + 31) / 32 * 32; j += kThreads / team) {
            const Found me = found[min(j, max(total - 1, 0))];
            int place = 0;
            for (int o = sub; o < total; o += team) place += found[o].key > me.key || (found[o].key == me.key && found[o].index < me.index);
            for (int o = 1; o < team; o *= 2) place += __shfl_xor_sync(0xffffffffu, place, o);
            if (j < total && sub == 0 && place < s.k) at_place[place] = (uint32_t)j | me.index / (uint32_t)in.vocab << 16;
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
            s.out_score[o] = is ? found[j].total : -INFINITY;
            s.out_parent[o] = is ? (int32_t)(first_row + beam) : -1;
            s.out_token[o] = is ? (int32_t)(found[j].index - (uint32_t)beam * (uint32_t)in.vocab) : -1;
        }
    }
    cluster_wait();
}

template <class T> int beam_launch(const nereus_logits_t& in, const nereus_beams_t& how, float* score, int32_t* parent, int32_t* token, cudaStream_t stream) {
    static std::atomic<bool> opted[kMaxDevices];
    Device dev;
    if (int rc = device_of(&dev)) return rc;
    // as many blocks as leave each four layers of the request at least; the number of requests has no part in it
    Deal d = spread_of(in, kThreads, 0, 0, INT32_MAX);
    const int64_t e = 16 / size_of(in.dtype), used = (in.vocab + in.shard_cols - 1) / in.shard_cols;
    const int64_t main = layers_aligned(held_cols(in, 0), e, kThreads) * used;
    while (d.log_c < 3 && (main * how.beams) >> (d.log_c + 1) >= 4) ++d.log_c;
    d.mine = (d.layers + (1 << d.log_c) - 1) >> d.log_c;
    Select s = {how.beams, how.k, how.settle, 0, 0, how.score, how.ended, how.norm, score, parent, token};
    s.per_note = (d.mine + kMaxNotes / how.beams - 1) / (kMaxNotes / how.beams);
    s.notes = (d.mine + s.per_note - 1) / s.per_note;
    const int64_t smem = kStreamRing * kVecs * 16 + std::min<int64_t>(kMaxItems, (int64_t)how.beams * d.mine) * (int64_t)sizeof(Layer) +
                         (int64_t)how.beams * s.notes * kThreads * 2;
    return launch(beam_kernel<T>, opted, kThreads, in.rows / how.beams, d, smem, dev, stream, cut_of(in), d, s, scale_of(1.0));
}

}  // namespace
}  // namespace nereus

extern "C" int nereus_beam_select(const nereus_logits_t* in, const nereus_beams_t* how, float* out_score, int32_t* out_parent, int32_t* out_token,
                                  void* cuda_stream) {
    if (int rc = check_view(in)) return rc;
    if (!how || how->beams < 1 || how->beams > NEREUS_BEAM_MAX || how->k < 1 || how->k > NEREUS_BEAM_MAX_K || how->reserved) return NEREUS_ERR_ARG;
    if (how->settle < 0 || how->settle > 1 || (how->settle && how->k != how->beams) || in->rows % how->beams) return NEREUS_ERR_ARG;
    if (misaligned(how->score) || misaligned(how->ended) || misaligned(how->norm) || misaligned(out_score) || misaligned(out_parent) || misaligned(out_token))
        return NEREUS_ERR_ALIGN;
    if (in->rows == 0) return NEREUS_OK;
    if (!how->score || !out_score || !out_parent || !out_token) return NEREUS_ERR_ARG;
    auto go = in->dtype == NEREUS_BF16 ? beam_launch<__nv_bfloat16> : beam_launch<float>;
    return go(*in, *how, out_score, out_parent, out_token, (cudaStream_t)cuda_stream);
}
