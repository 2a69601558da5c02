// A generation stage's states and cache for sm_100a: rows of dense states that follow the beams that go on
// (nereus_states_reorder), and the pages of a cache: forking, freeing and making room (nereus_cache_fork), moving the pages
// in use to the front (nereus_cache_compact), copying pages (nereus_cache_copy).
//
// Two kinds of work.  Bytes that move: their floor is HBM bandwidth, every byte read once and written once.  And books
// (page table, reference counts): whole numbers, a few MB at most, where what counts is the chain of dependent steps.
// Everything is exact, and no result depends on the order in which threads come: counts are sums of whole numbers, and free
// pages are handed out by rank.
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <climits>
#include <cstdint>
#include <cstdlib>
#include <type_traits>

#include "nereus_internal.hpp"

using namespace nereus;

namespace nereus {
namespace {

#define NEREUS_CUDA(call)                                               \
    do {                                                                \
        cudaError_t e_ = (call);                                        \
        if (e_ != cudaSuccess) { set_cuda_error((int)e_); (void)cudaGetLastError(); return NEREUS_ERR_CUDA; } \
    } while (0)

constexpr int kMaxDevices = 64;
constexpr int64_t kMaxBytes = (int64_t)1 << 46;       // of a buffer
constexpr int64_t kMaxPage  = (int64_t)1 << 30;

// ---- copying pages -------------------------------------------------------------------------------------------
//
// A warp takes a tile of up to 4 KiB of one page in one pool, loads all of it and stores it, then goes on by the grid's size.
// HBM bounds it: 700 pages x 64 pools (734 MB read and written) in 116 us, 6.35 TB/s of the 6.56 of a plain copy.  That takes
// blocks that the hardware deals out as others end, a warp for every two tiles; a grid of what the GPU holds took 127 us.
// Forks and compactions, whose pairs only the device counts, have a warp for every four tiles of the most pairs there can be, up
// to 32 times the blocks that the GPU holds.  With nothing to move of 400 thousand pages x 64 pools a compaction takes 59 us
// (8 times: 38, 64 times: 93, no bound: 684), and the 6000 pages below 245 (8 times: 257).

constexpr int kFew = 64;                   // buffers of most calls: a kernel's parameters of 4 KiB take 2 us more to hand over
template <int N> struct Pools {
    char*   from[N];
    char*   to[N];
    int64_t from_stride, to_stride, page_bytes;
    int32_t pools, from_pages, to_pages, chunks;
};
constexpr int kCopyThreads = 256;
constexpr int kTileVecs = 8;               // of a thread
constexpr int kMostWaves = 32;            // of blocks where the device counts the pairs

// The tiles of `n` pairs, from this warp's first on; src, dst: `step` apart.
template <class V, class P>
__device__ __forceinline__ void copy_pages(const P& p, int64_t n, const int32_t* src, const int32_t* dst, int step, int64_t warp, int64_t warps) {
    const int     lane = threadIdx.x & 31;
    const int64_t per_pair = (int64_t)p.pools * p.chunks, vecs = p.page_bytes / (int64_t)sizeof(V);
    // this warp's place as (pair, pool, chunk), and how far it goes on
    int64_t   pair = warp / per_pair;
    int       pool = (int)(warp - pair * per_pair) / p.chunks, chunk = (int)(warp - pair * per_pair) % p.chunks;
    const int64_t by_pair = warps / per_pair;
    const int by_pool = (int)(warps - by_pair * per_pair) / p.chunks, by_chunk = (int)(warps - by_pair * per_pair) % p.chunks;
    int s = 0, d = 0;                                  // of the next tile
    if (pair < n) { s = __ldcg(src + pair * step); d = __ldcg(dst + pair * step); }
#pragma unroll 1
    while (pair < n) {
        const int     from_page = s, to_page = d;
        const int64_t at = (int64_t)chunk * (32 * kTileVecs) + lane;
        const char*   from = p.from[pool];
        char*         to = p.to[pool];
        chunk += by_chunk;
        if (chunk >= p.chunks) { chunk -= p.chunks; ++pool; }
        pool += by_pool;
        if (pool >= p.pools) { pool -= p.pools; ++pair; }
        pair += by_pair;
        if (pair < n) { s = __ldcg(src + pair * step); d = __ldcg(dst + pair * step); }
        if ((unsigned)from_page >= (unsigned)p.from_pages || (unsigned)to_page >= (unsigned)p.to_pages) continue;
        const V* a = reinterpret_cast<const V*>(from + from_page * p.from_stride) + at;
        V*       b = reinterpret_cast<V*>(to + to_page * p.to_stride) + at;
        V v[kTileVecs];
#pragma unroll
        for (int i = 0; i < kTileVecs; ++i)
            if (at + 32 * i < vecs) v[i] = __ldcs(a + 32 * i);
#pragma unroll
        for (int i = 0; i < kTileVecs; ++i)
            if (at + 32 * i < vecs) __stcs(b + 32 * i, v[i]);
    }
}

template <class V, class P>
__global__ void __launch_bounds__(kCopyThreads) copy_kernel(const __grid_constant__ P p, int64_t n, const int32_t* src, const int32_t* dst) {
    copy_pages<V, P>(p, n, src, dst, 1, ((int64_t)blockIdx.x * kCopyThreads + threadIdx.x) >> 5, ((int64_t)gridDim.x * kCopyThreads) >> 5);
}

// ---- what the books' kernels share -----------------------------------------------------------------------------
//
// A call is a chain of launches, each of which is told to come up while the one before it runs and waits for its end only
// where it needs what that has written: what it can work out from the call's arguments is ready by then.  Free pages are ranked
// by one cluster, whose barriers cost a microsecond or so: every block has a slice of the pages, every warp a part of the slice.

constexpr int kBookThreads = 1024;
constexpr int kBookWarps   = kBookThreads / 32;
constexpr int kMaxCluster  = 16;
constexpr int kGroup       = 128;             // pages that a warp looks at at a time, four a lane

__device__ __forceinline__ void let_next_come() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_last() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_sync() {
    cluster_arrive();
    cluster_wait();
}
__device__ __forceinline__ uint32_t peer_address(const void* p, int rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ void peer_store(uint32_t at, unsigned long long v) {
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(at), "l"(v) : "memory");
}
typedef unsigned long long Wide;

__device__ __forceinline__ Wide warp_scan(Wide v) {                  // inclusive
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const Wide u = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += u;
    }
    return v;
}
// Sum over the warps before this one of what their lanes' v is in all, and the block's total.  scratch: kWarps + 1.
template <int kWarps = kBookWarps> __device__ __forceinline__ Wide warps_before(Wide of_warp, Wide* scratch, Wide* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    __syncthreads();
    if (lane == 0) scratch[warp] = of_warp;
    __syncthreads();
    if (warp == 0) {
        const Wide mine = lane < kWarps ? scratch[lane] : 0, upto = warp_scan(mine);
        __syncwarp();
        if (lane < kWarps) scratch[lane] = upto - mine;
        if (lane == kWarps - 1) scratch[kWarps] = upto;
    }
    __syncthreads();
    *total = scratch[kWarps];
    return scratch[warp];
}
// What the blocks before this one have, and all of them, of one number each.  Ends in no barrier: `totals` is written once.
__device__ __forceinline__ Wide blocks_before(Wide mine, Wide* totals, int rank, int blocks, Wide* total) {
    if (blocks == 1) {
        *total = mine;
        return 0;
    }
    if (threadIdx.x < blocks) peer_store(peer_address(totals + rank, threadIdx.x), mine);
    cluster_sync();
    Wide before = 0, all = 0;
    for (int b = 0; b < blocks; ++b) {
        const Wide v = totals[b];
        if (b < rank) before += v;
        all += v;
    }
    *total = all;
    return before;
}
// This warp's part [lo, hi) of the pages, in whole groups; blocks is a power of two.
struct Part {
    int lo, hi;
};
__device__ __forceinline__ Part part_of(int pages, int rank, int blocks) {
    const int64_t groups = (pages + kGroup - 1) / kGroup, parts = (int64_t)blocks * kBookWarps, i = (int64_t)rank * kBookWarps + (threadIdx.x >> 5);
    const int     shift = __ffsll(parts) - 1;
    return {(int)min((int64_t)pages, (groups * i >> shift) * kGroup), (int)min((int64_t)pages, (groups * (i + 1) >> shift) * kGroup)};
}
// Counts of the lane's four pages of the group that begins at p; `none` past hi.
__device__ __forceinline__ int4 counts_of(const int32_t* refs, int p, int hi, bool aligned, int none) {
    const int at = p + 4 * (threadIdx.x & 31);
    if (aligned && at + 4 <= hi) return __ldcg(reinterpret_cast<const int4*>(refs + at));
    int4 v;
    v.x = at < hi ? __ldcg(refs + at) : none;
    v.y = at + 1 < hi ? __ldcg(refs + at + 1) : none;
    v.z = at + 2 < hi ? __ldcg(refs + at + 2) : none;
    v.w = at + 3 < hi ? __ldcg(refs + at + 3) : none;
    return v;
}
__device__ __forceinline__ int live_of(int4 v) { return (v.x > 0) + (v.y > 0) + (v.z > 0) + (v.w > 0); }
// Pages in use of a warp's part, in all its lanes together.
__device__ __forceinline__ int count_live(const int32_t* refs, Part part, bool aligned) {
    int n = 0;
#pragma unroll 4
    for (int p = part.lo; p < part.hi; p += kGroup) n += live_of(counts_of(refs, p, part.hi, aligned, 0));
    return __reduce_add_sync(0xffffffffu, n);
}

// x / d for 0 <= x < 2^52, one_by = 1 / d rounded: off by one at most before it is put right.
struct Divisor {
    double  one_by;
    int32_t d;
};
__device__ __forceinline__ int64_t quotient(int64_t x, const Divisor& by) {
    const int64_t q = __double2ll_rz((double)x * by.one_by), r = x - q * by.d;
    return r < 0 ? q - 1 : r >= by.d ? q + 1 : q;
}

// x / d for 0 <= x < 2^31
__device__ __forceinline__ int64_t quotient64(int x, int64_t d) { return d > x ? 0 : (int64_t)((uint32_t)x / (uint32_t)d); }

struct Books {
    const int32_t *table, *length, *refs;
    int64_t  stride;
    int32_t  rows, columns, pages;
};
struct NewBooks {
    int32_t *table, *length, *refs;
    int64_t  stride;
    int32_t  rows;
};

// ---- forking -------------------------------------------------------------------------------------------------
//
// Four launches: start (counts copied, the table's plain entries), count (what the rows' old and new holders change), assign
// (which pages are free, and which row gets which), apply (page copies).  1024 rows of 2001 columns over 790 thousand pages take
// 23 us, most of it assign (16 us, 3.3 MB read): its steps hang on one another.  All books in one cluster took 117 us.

struct Fork {
    const int32_t *parent, *room_of;
    int32_t *copies, *status;
    Divisor  page_size;
    int32_t  room;
};
// What becomes of a row: its parent (-1: it is empty), the tokens and full pages it starts with, and the columns until which it
// has to have pages.
struct Heir {
    int     parent, n, full;
    bool    begun;
    int64_t until;
};
__device__ __forceinline__ int tokens_of(const Books& b, const Fork& f, int row) {
    return (int)min((int64_t)max(b.length[row], 0), (int64_t)b.columns * f.page_size.d);
}
__device__ __forceinline__ Heir heir_of(const Books& b, const Fork& f, int row) {
    Heir h = {f.parent[row], 0, 0, false, 0};
    if ((unsigned)h.parent >= (unsigned)b.rows) h.parent = -1;
    else {
        h.n = tokens_of(b, f, h.parent);
        h.full = (int)quotient(h.n, f.page_size);
        h.begun = h.n != h.full * f.page_size.d;
        h.until = quotient((int64_t)h.n + max(f.room_of ? f.room_of[row] : f.room, 0) + f.page_size.d - 1, f.page_size);
    }
    return h;
}
__device__ __forceinline__ bool is_page(int e, int pages) { return (unsigned)e < (unsigned)pages; }

constexpr int kStartThreads = 256;
constexpr int kPerThread    = 8;              // entries of a thread
constexpr int kRefsUnit     = kStartThreads * kPerThread * 2;
constexpr int kTableUnit    = kStartThreads * kPerThread;

// Counts and plain entries, dealt out in units to all blocks: HBM is what bounds them where they are many.
__global__ void __launch_bounds__(kStartThreads) fork_start_kernel(const Books from, const NewBooks to, const Fork f, int refs_units, int chunks) {
    const int  tid = threadIdx.x;
    const bool aligned = (((uintptr_t)from.refs | (uintptr_t)to.refs) & 15) == 0;
    let_next_come();
#pragma unroll 1
    for (int64_t u = blockIdx.x; u < refs_units + (int64_t)to.rows * chunks; u += gridDim.x) {
        if (u < refs_units) {
            const int lo = (int)u * kRefsUnit, hi = (int)min((int64_t)lo + kRefsUnit, (int64_t)from.pages);
            if (aligned && hi - lo == kRefsUnit) {
                int4 v[kPerThread / 2];
#pragma unroll
                for (int j = 0; j < kPerThread / 2; ++j) v[j] = __ldcg(reinterpret_cast<const int4*>(from.refs + lo) + tid + j * kStartThreads);
#pragma unroll
                for (int j = 0; j < kPerThread / 2; ++j) __stcg(reinterpret_cast<int4*>(to.refs + lo) + tid + j * kStartThreads, v[j]);
            } else {
                for (int p = lo + tid; p < hi; p += kStartThreads) to.refs[p] = from.refs[p];
            }
            continue;
        }
        const int  i = (int)((u - refs_units) / chunks), first = (int)((u - refs_units) - (int64_t)i * chunks) * kTableUnit;
        const int  end = min(first + kTableUnit, from.columns);
        const Heir h = heir_of(from, f, i);
        int        before = 0;                         // whether a row above names the same parent
        if (h.parent >= 0 && end > h.full)
            for (int j = tid; j < i; j += kStartThreads) before |= f.parent[j] == h.parent;
        const bool     leads = !__syncthreads_or(before);
        const int32_t* row = from.table + max(h.parent, 0) * from.stride;
        int32_t* const out = to.table + i * to.stride;
        int e[kPerThread];
#pragma unroll
        for (int j = 0; j < kPerThread; ++j) {
            const int c = first + tid + j * kStartThreads;
            e[j] = h.parent >= 0 && c < end && (c < h.full || leads) ? __ldcg(row + c) : -1;
        }
#pragma unroll
        for (int j = 0; j < kPerThread; ++j) {
            const int c = first + tid + j * kStartThreads;
            // a column that lacks a page gets its entry later
            if (c < end && !(c >= h.full && c < h.until && !is_page(e[j], from.pages))) __stcg(out + c, e[j]);
        }
        if (first == 0 && tid == 0) {
            to.length[i] = h.n;
            f.copies[2 * i] = f.copies[2 * i + 1] = -1;
        }
    }
}

// A thread goes down a column over a few rows: beams of one request hold the same pages one above the other, whose changes are
// added up before they go out.
constexpr int kCountThreads = 256;
constexpr int kMostRows     = 64;
constexpr int kAtATime      = 8;
__global__ void __launch_bounds__(kCountThreads) fork_count_kernel(const Books from, const NewBooks to, const Fork f, int group) {
    __shared__ int kids[kMostRows], full[kMostRows];
    const int tid = threadIdx.x, first = blockIdx.y * group, n = min(group, from.rows - first), c = blockIdx.x * kCountThreads + tid;
    let_next_come();
    if (tid < n) {
        kids[tid] = 0;
        full[tid] = (int)quotient(tokens_of(from, f, first + tid), f.page_size);
    }
    __syncthreads();
    for (int i = tid; i < to.rows; i += kCountThreads) {
        const int r = f.parent[i] - first;
        if ((unsigned)r < (unsigned)n) atomicAdd(&kids[r], 1);
    }
    __syncthreads();
    wait_for_last();                                   // the old counts are there
    if (c >= from.columns) return;
    int page = -1, sum = 0;
#pragma unroll 1
    for (int first_of = 0; first_of < n; first_of += kAtATime) {
        int e[kAtATime], change[kAtATime];
#pragma unroll
        for (int j = 0; j < kAtATime; ++j) {
            const int r = min(first_of + j, n - 1), k = kids[r];
            change[j] = first_of + j >= n ? 0 : c < full[r] ? k - 1 : k ? 0 : -1;
            e[j] = change[j] ? __ldcg(from.table + (first + r) * from.stride + c) : -1;
        }
#pragma unroll
        for (int j = 0; j < kAtATime; ++j) {
            if (!is_page(e[j], from.pages)) continue;
            if (e[j] != page) {
                if (sum) atomicAdd(&to.refs[page], sum);
                page = e[j];
                sum = 0;
            }
            sum += change[j];
        }
    }
    if (sum) atomicAdd(&to.refs[page], sum);
}

// A row's need of fresh pages, and 1 << 48 where its first is a copy.
constexpr Wide kOneCopy = (Wide)1 << 48;
__device__ __forceinline__ int64_t pages_in(Wide need) { return (int64_t)(need & (kOneCopy - 1)); }

// Of a row that lacks pages: its parent, the columns in which it lacks them, whether it has pages between these.
struct Lack {
    int parent, full, until;
};
constexpr int64_t kWholeEntries = 8192;       // of both tables: 4 x 256 x 2 in the time of the chain, 128 x 129 x 2 26 us instead of 20
constexpr int kSmallThreads = 256;
constexpr int kWindow = 2048;                 // free pages of a block that are handed out at a time
constexpr int kStaticBooks = 10240;           // shared memory that is not dynamic, with room to spare
constexpr int kSelf = 8;                      // columns that a row's own thread looks through; a warp takes rows with more

// One cluster.  Of every new row: what it needs, then the sum of that over the rows before; what it lacks.  first: of every old
// row, the lowest new row that names it.  free_of: free pages of the block's groups, then their sum over the groups before.
// kWhole: small books, whose launches would cost more than one block's work: it does what start and count do, too.
template <bool kWhole>
__global__ void __launch_bounds__(kWhole ? kSmallThreads : kBookThreads, 1) fork_assign_kernel(const Books from, const NewBooks to, const Fork f, int groups_of_block) {
    constexpr int kThreads = kWhole ? kSmallThreads : kBookThreads, kWarps = kThreads / 32;
    extern __shared__ __align__(16) unsigned char dynamic[];
    __shared__ Wide scratch[kWarps + 1], totals[kMaxCluster];
    __shared__ Wide lacking_columns;
    __shared__ int  window[kWindow];
    Wide* need    = reinterpret_cast<Wide*>(dynamic);
    Lack* lack    = reinterpret_cast<Lack*>(need + to.rows);
    int*  first   = reinterpret_cast<int*>(lack + to.rows);
    int*  free_of = first + from.rows;
    int*  kids    = free_of + groups_of_block;         // kWhole: how many rows name an old row
    const int  tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, blocks = gridDim.x, rank = blockIdx.x;
    const bool aligned = ((uintptr_t)to.refs & 15) == 0;

    let_next_come();
    if (tid == 0) lacking_columns = 0;
    cluster_arrive();                                  // this block has begun: the others may write to it
    for (int r = tid; r < from.rows; r += kThreads) {
        first[r] = INT_MAX;
        if (kWhole) kids[r] = 0;
    }
    if (kWhole)
        for (int p = tid; p < from.pages; p += kThreads) to.refs[p] = from.refs[p];
    __syncthreads();
    for (int i = tid; i < to.rows; i += kThreads) {
        const int p = f.parent[i];
        if ((unsigned)p >= (unsigned)from.rows) continue;
        atomicMin(&first[p], i);
        if (kWhole) atomicAdd(&kids[p], 1);
    }
    __syncthreads();
    // what the rows need: every block goes through all of them
    bool long_rows = false;
#pragma unroll 1
    for (int i = tid; i < to.rows; i += kThreads) {
        const Heir h = heir_of(from, f, i);
        const int  until = (int)min(h.until, (int64_t)from.columns);
        Wide       w = 0;
        if (h.parent >= 0) {
            const int32_t* row = from.table + h.parent * from.stride;
            const bool     leads = first[h.parent] == i;
            if (h.until > from.columns) atomicAdd(&lacking_columns, (Wide)(h.until - from.columns));
            if (h.full >= until) {
            } else if (!leads) {
                w = (Wide)(until - h.full) + (h.begun && is_page(row[h.full], from.pages) ? kOneCopy : 0);
            } else if (until - h.full <= kSelf) {
#pragma unroll
                for (int c = 0; c < kSelf; ++c) w += h.full + c < until && !is_page(row[min(h.full + c, from.columns - 1)], from.pages);
            } else {
                long_rows = true;
                w = ~(Wide)0;
            }
        }
        need[i] = w;
        lack[i] = {h.parent, h.full, until};
        if (kWhole) {
            to.length[i] = h.n;
            f.copies[2 * i] = f.copies[2 * i + 1] = -1;
        }
    }
    const bool some_long = __syncthreads_or(long_rows);
    cluster_wait();
    if (kWhole) {
        // a warp for a row: what its holders change, then the plain entries
#pragma unroll 1
        for (int r = warp; r < from.rows; r += kWarps) {
            const int k = kids[r], full = k == 1 ? 0 : (int)quotient(tokens_of(from, f, r), f.page_size), end = k == 1 ? 0 : k ? full : from.columns;
#pragma unroll 4
            for (int c = lane; c < end; c += 32) {
                const int e = from.table[r * from.stride + c];
                if (is_page(e, from.pages)) atomicAdd(&to.refs[e], c < full ? k - 1 : -1);
            }
        }
#pragma unroll 1
        for (int i = warp; i < to.rows; i += kWarps) {
            const Lack     l = lack[i];
            const int      end = l.parent < 0 ? 0 : first[l.parent] == i ? from.columns : l.full;
            const int32_t* row = from.table + max(l.parent, 0) * from.stride;
            int32_t* const out = to.table + i * to.stride;
#pragma unroll 4
            for (int c = lane; c < from.columns; c += 32) {
                const int e = c < end ? row[c] : -1;
                if (!(c >= l.full && c < l.until && !is_page(e, from.pages))) out[c] = e;
            }
        }
        __syncthreads();
    }
    if (some_long) {                                   // in all blocks: their rows are shared out
        cluster_sync();                                // nobody marks them any more
        for (int i = rank * kWarps + warp; i < to.rows; i += blocks * kWarps) {
            if (need[i] != ~(Wide)0) continue;
            const Lack     l = lack[i];
            const int32_t* row = from.table + l.parent * from.stride;
            unsigned       n = 0;
#pragma unroll 4
            for (int c = l.full + lane; c < l.until; c += 32) n += !is_page(__ldcg(row + c), from.pages);
            n = __reduce_add_sync(0xffffffffu, n);
            __syncwarp();
            if (lane < blocks) peer_store(peer_address(need + i, lane), n);
        }
        cluster_sync();
    }
    // need: sum over the rows before
    Wide needed = 0;
    {
        const int per = (to.rows + kThreads - 1) / kThreads, lo = min(tid * per, to.rows), hi = min(lo + per, to.rows);
        Wide sum = 0;
        for (int i = lo; i < hi; ++i) sum += need[i];
        const Wide upto = warp_scan(sum);
        Wide at = warps_before<kWarps>(__shfl_sync(0xffffffffu, upto, 31), scratch, &needed) + upto - sum;
        for (int i = lo; i < hi; ++i) { const Wide w = need[i]; need[i] = at; at += w; }
    }
    const int64_t fresh = pages_in(needed);
    const int     n_copies = (int)(needed >> 48);
    wait_for_last();                                   // all changes are in

    // free pages: of every group, in all, and before the block
    const int first_group = rank * groups_of_block, n_groups = min(groups_of_block, max(0, (from.pages + kGroup - 1) / kGroup - first_group));
#pragma unroll 1
    for (int g0 = warp; g0 < n_groups; g0 += 8 * kWarps) {
        int4 v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = counts_of(to.refs, (first_group + min(g0 + j * kWarps, n_groups - 1)) * kGroup, from.pages, aligned, 1);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int n = __reduce_add_sync(0xffffffffu, 4 - live_of(v[j]));
            if (lane == 0 && g0 + j * kWarps < n_groups) free_of[g0 + j * kWarps] = n;
        }
    }
    __syncthreads();
    Wide of_block, free_pages;
    {
        const int per = (n_groups + kThreads - 1) / kThreads, lo = min(tid * per, n_groups), hi = min(lo + per, n_groups);
        int sum = 0;
        for (int g = lo; g < hi; ++g) sum += free_of[g];
        const int upto = (int)warp_scan((Wide)sum);
        int at = (int)warps_before<kWarps>((Wide)__shfl_sync(0xffffffffu, upto, 31), scratch, &of_block) + upto - sum;
        for (int g = lo; g < hi; ++g) { const int n = free_of[g]; free_of[g] = at; at += n; }
    }
    const int64_t before = (int64_t)blocks_before(of_block, totals, rank, blocks, &free_pages);
    const int64_t missing = max((int64_t)0, fresh - (int64_t)free_pages) + (int64_t)lacking_columns;
    if (missing == 0) {
        // The block's free pages by rank, a window of them at a time, then a thread for each that is handed out, which marks it as
        // taken: a group in which a window ends is read again for the next, and what is left of it begins that one.
        const int mine = (int)max((int64_t)0, min((int64_t)of_block, fresh - before));
#pragma unroll 1
        for (int base = 0; base < mine; base += kWindow) {
#pragma unroll 1
            for (int g = warp; g < n_groups && free_of[g] < min(base + kWindow, mine); g += kWarps) {
                if ((g + 1 < n_groups ? free_of[g + 1] : (int)of_block) <= base) continue;
                const int      p = (first_group + g) * kGroup;
                const int4     v = counts_of(to.refs, p, from.pages, aligned, 1);
                const unsigned below = (1u << lane) - 1;
                int            j = max(free_of[g] - base, 0);      // what the windows before took of the group counts as free no more
#pragma unroll
                for (int e = 0; e < 4; ++e) j += __popc(__ballot_sync(0xffffffffu, (e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w) <= 0) & below);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if ((e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w) > 0) continue;
                    if ((unsigned)j < (unsigned)kWindow) window[j] = p + 4 * lane + e;
                    ++j;
                }
            }
            __syncthreads();
#pragma unroll 1
            for (int x = tid; x < min(kWindow, mine - base); x += kThreads) {
                const int64_t j = before + base + x;
                int lo = 0, hi = to.rows;              // the last row whose sum is not above j
                while (hi - lo > 1) {
                    const int mid = (lo + hi) / 2;
                    if (pages_in(need[mid]) <= j) lo = mid;
                    else hi = mid;
                }
                const Wide here = need[lo], next = lo + 1 < to.rows ? need[lo + 1] : needed;
                const Lack l = lack[lo];
                const int  page = window[x];
                int        k = (int)(j - pages_in(here)), c = l.full + k;
                const int32_t* row = from.table + l.parent * from.stride;
                if (pages_in(next - here) != l.until - l.full)
                    for (c = l.full; c < l.until; ++c)         // the row has pages between those it lacks
                        if (!is_page(row[c], from.pages) && k-- == 0) break;
                to.table[lo * to.stride + c] = page;
                to.refs[page] = 1;
                if (c == l.full && next >> 48 != here >> 48) {
                    const int at = (int)(here >> 48);
                    f.copies[2 * at] = row[c];
                    f.copies[2 * at + 1] = page;
                }
            }
            __syncthreads();
        }
    } else {
        const int lo = first_group * kGroup, hi = (int)min((int64_t)from.pages, (int64_t)(first_group + n_groups) * kGroup);
        for (int p = lo + tid; p < hi; p += kThreads) to.refs[p] = from.refs[p];
    }
    int64_t left = (int64_t)free_pages - fresh;
    if (missing && rank == 0) {
        int n = 0;
        for (int p = tid; p < from.pages; p += kThreads) n += from.refs[p] <= 0;
        Wide all;
        warps_before<kWarps>(__reduce_add_sync(0xffffffffu, n), scratch, &all);
        left = (int64_t)all;
    }
    if (rank == 0 && tid == 0) {
        f.status[0] = (int)left;
        f.status[1] = (int)min(missing, (int64_t)INT_MAX);
        f.status[2] = missing ? 0 : n_copies;
        f.status[3] = 0;
    }
}

// The page copies; where the fork is refused, the old table and lengths.
template <class V, class P>
__global__ void __launch_bounds__(kCopyThreads) fork_apply_kernel(const __grid_constant__ P p, const Books from, const NewBooks to, const Fork f) {
    wait_for_last();
    const int n = __ldcg(f.status + 2);
    if (__ldcg(f.status + 1))
        for (int i = blockIdx.x; i < to.rows; i += gridDim.x) {
            for (int c = threadIdx.x; c < from.columns; c += kCopyThreads) to.table[i * to.stride + c] = i < from.rows ? from.table[i * from.stride + c] : -1;
            if (threadIdx.x == 0) to.length[i] = i < from.rows ? from.length[i] : 0;
        }
    copy_pages<V, P>(p, n, f.copies, f.copies + 1, 2, ((int64_t)blockIdx.x * kCopyThreads + threadIdx.x) >> 5, ((int64_t)gridDim.x * kCopyThreads) >> 5);
}

// ---- compacting ----------------------------------------------------------------------------------------------
//
// Two launches: one cluster ranks the pages in use and writes the books (10 us at 6000 pages, a chain of dependent steps), then
// the page copies, which HBM bounds: 2400 pages x 64 pools in 245 us where their bytes take 230.

struct Compact {
    int64_t  keep;
    int32_t *map, *moves, *status;
};
__global__ void __launch_bounds__(kBookThreads, 1) compact_kernel(const Books from, const NewBooks to, const Compact c) {
    __shared__ Wide scratch[kBookWarps + 1], totals[2][kMaxCluster];
    const int  tid = threadIdx.x, lane = tid & 31, blocks = gridDim.x, rank = blockIdx.x;
    const Part part = part_of(from.pages, rank, blocks);
    const bool aligned = ((uintptr_t)from.refs & 15) == 0, stores = (((uintptr_t)to.refs | (uintptr_t)c.map) & 15) == 0;
    let_next_come();
    cluster_arrive();                                  // this block has begun: the others may write to it
    const int of_part = count_live(from.refs, part, aligned);
    Wide of_block, live;
    warps_before((Wide)of_part, scratch, &of_block);
    cluster_wait();
    blocks_before(of_block, totals[0], rank, blocks, &live);
    const int64_t missing = c.keep < 0 ? 0 : max((int64_t)0, (int64_t)live - c.keep);
    const int     keep = missing ? from.pages : c.keep < 0 ? (int)live : (int)min(c.keep, (int64_t)from.pages);
    // pages that go (in the upper half) and holes that take them, before this warp and in all; one part may lie on both sides
    Wide of_warp = part.hi <= keep ? (Wide)(part.hi - part.lo - of_part) : (Wide)of_part << 32;
    if (part.lo < keep && part.hi > keep) {
        const int low = count_live(from.refs, {part.lo, keep}, aligned);
        of_warp = ((Wide)(of_part - low) << 32) + (Wide)(keep - part.lo - low);
    }
    Wide all, before = warps_before(of_warp, scratch, &of_block);
    before += blocks_before(of_block, totals[1], rank, blocks, &all);
    const int moves = (int)(all >> 32);
    int goes = (int)(before >> 32), hole = (int)before;
#pragma unroll 1
    for (int p = part.lo; p < part.hi; p += kGroup) {
        const int4     v = counts_of(from.refs, p, part.hi, aligned, 0);
        const int      r[4] = {v.x, v.y, v.z, v.w}, at = p + 4 * lane;
        const unsigned below = (1u << lane) - 1;
        int g = goes, h = hole;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool     in = at + e < part.hi, up = at + e >= keep;
            const unsigned who = __ballot_sync(0xffffffffu, in && r[e] > 0 && up), where = __ballot_sync(0xffffffffu, in && r[e] <= 0 && !up);
            g += __popc(who & below);
            h += __popc(where & below);
            goes += __popc(who);
            hole += __popc(where);
        }
        int now[4], counts[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int  page = at + e;
            const bool in = page < part.hi, is = r[e] > 0, up = page >= keep;
            now[e] = is && !up ? page : -1;            // pages that go and holes that take them come right below
            counts[e] = is && !up ? r[e] : 0;
            if (in && is && up) c.moves[2 * g++] = page;
            if (in && !is && !up && h++ < moves) c.moves[2 * h - 1] = page;
        }
        if (stores && at + 4 <= part.hi) {
            *reinterpret_cast<int4*>(c.map + at) = make_int4(now[0], now[1], now[2], now[3]);
            *reinterpret_cast<int4*>(to.refs + at) = make_int4(counts[0], counts[1], counts[2], counts[3]);
        } else {
            for (int e = 0; e < 4 && at + e < part.hi; ++e) {
                c.map[at + e] = e == 0 ? now[0] : e == 1 ? now[1] : e == 2 ? now[2] : now[3];
                to.refs[at + e] = e == 0 ? counts[0] : e == 1 ? counts[1] : e == 2 ? counts[2] : counts[3];
            }
        }
    }
    cluster_sync();
    for (int j = rank * kBookThreads + tid; j < moves; j += blocks * kBookThreads) {
        const int2 m = __ldcg(reinterpret_cast<const int2*>(c.moves) + j);
        c.map[m.x] = m.y;
        to.refs[m.y] = from.refs[m.x];
    }
    if (rank == 0 && tid == 0) {
        c.status[0] = (int)live;
        c.status[1] = (int)missing;
        c.status[2] = moves;
        c.status[3] = keep;
    }
}
template <class V, class P>
__global__ void __launch_bounds__(kCopyThreads) compact_apply_kernel(const __grid_constant__ P p, const Books from, const NewBooks to, const Compact c) {
    wait_for_last();
    for (int i = blockIdx.x; i < to.rows; i += gridDim.x)
#pragma unroll 4
        for (int j = threadIdx.x; j < from.columns; j += kCopyThreads) {
            const int e = __ldcg(from.table + i * from.stride + j);
            __stcg(to.table + i * to.stride + j, is_page(e, from.pages) ? __ldcg(c.map + e) : e);
        }
    copy_pages<V, P>(p, __ldcg(c.status + 2), c.moves, c.moves + 1, 2, ((int64_t)blockIdx.x * kCopyThreads + threadIdx.x) >> 5, ((int64_t)gridDim.x * kCopyThreads) >> 5);
}

// ---- reordering rows -----------------------------------------------------------------------------------------
//
// A thread takes one vector's place in the rows of a group: it loads what moves from every row that something goes on from,
// then stores.  No other thread touches that place, so that parents may cross in place without a barrier.  HBM bounds it: half
// of 64 rows in 32 buffers of 67 MB (1.34 GB read and written) in 207 us, 6.5 TB/s.  Few moves leave few loads in flight, so
// a thread takes several tiles at a time then (one: 228 us), 16 tiles a block (8: 212, 4: 231, 24: 210 us).

template <int N> struct States {
    char*   from[N];
    char*   to[N];
    int64_t from_row, to_row, from_outer, to_outer;        // strides
    int64_t piece;                                         // bytes of a piece: tokens * token_bytes
    int64_t token_bytes, tokens;
    int32_t buffers, from_rows, to_rows, outer, group, in_place;
    int32_t blocks;                                        // of a group
};
constexpr int kMoveThreads = 128;
struct Move {
    int64_t from, to, bytes;
};

template <class V, int N, class S>
__global__ void __launch_bounds__(kMoveThreads) reorder_kernel(const __grid_constant__ S s, const int32_t* parent, const int32_t* length) {
    __shared__ Move moves[N];
    __shared__ int  n_moves;
    __shared__ Wide most_bytes;
    const int group = blockIdx.x / s.blocks, block = blockIdx.x % s.blocks, tid = threadIdx.x;
    if (tid == 0) { n_moves = 0; most_bytes = 0; }
    __syncthreads();
    const int row = group * s.group + tid;
    if (tid < s.group && row < s.to_rows) {
        const int p = parent[row];
        if (s.in_place ? p != row && p >= group * s.group && p < (group + 1) * s.group : (unsigned)p < (unsigned)s.from_rows) {
            const int64_t tokens = length ? min((int64_t)max(length[p], 0), s.tokens) : s.tokens;
            if (tokens) {
                moves[atomicAdd(&n_moves, 1)] = {p * s.from_row, row * s.to_row, tokens * s.token_bytes};
                atomicMax(&most_bytes, (Wide)(tokens * s.token_bytes));
            }
        }
    }
    __syncthreads();
    constexpr int kTile = kMoveThreads * (int)sizeof(V);
    // few moves: a thread takes several places at a time, one tile apart
    const int     n_rows = n_moves, places = n_rows ? N / n_rows : 0, n = n_rows * places;
    const int64_t most = (int64_t)most_bytes, step = (int64_t)places * kTile;
    if (!n) return;
    for (int i = n_rows + tid; i < n; i += kMoveThreads) {
        const Move    m = moves[i % n_rows];
        const int64_t by = (int64_t)(i / n_rows) * kTile;
        moves[i] = {m.from + by, m.to + by, m.bytes - by};
    }
    __syncthreads();
    // this block's items: (buffer, piece, stretch of `places` tiles), and how far it goes on
    const int64_t  tiles = quotient(s.piece + step - 1, Divisor{1.0 / (double)step, (int)step});
    const uint32_t outer = (uint32_t)s.outer;
    const int64_t  line = quotient64(block, tiles), by_line = quotient64(s.blocks, tiles);
    int64_t        tile = block - line * tiles, b = (uint32_t)line / outer;
    uint32_t       o = (uint32_t)line % outer;
    const int64_t  by_tile = s.blocks - by_line * tiles, by_b = (uint32_t)by_line / outer;
    const uint32_t by_o = (uint32_t)by_line % outer;
#pragma unroll 1
    while (b < s.buffers) {
        const int64_t at = tile * step + tid * (int)sizeof(V);
        const char* from = s.from[b] + o * s.from_outer + at;
        char*       to = s.to[b] + o * s.to_outer + at;
        tile += by_tile;
        if (tile >= tiles) { tile -= tiles; ++o; }
        o += by_o;
        if (o >= outer) { o -= outer; ++b; }
        b += by_b;
        if (at >= most) continue;
        V v[N];
        bool edge = false;                                 // the last bytes of a row that are no whole vector
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n) {
                const int64_t left = moves[i].bytes - at;
                if (left >= (int64_t)sizeof(V)) v[i] = __ldcg(reinterpret_cast<const V*>(from + moves[i].from));
                else edge |= left > 0;
            }
        // Before any whole vector is stored: that may be where a shorter row's bytes come from, and none is loaded from where these go.
        if (sizeof(V) > 1 && edge)
            for (int k = 0; k < (int)sizeof(V); ++k) {
                unsigned char c[N];
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (i < n && moves[i].bytes - at < (int64_t)sizeof(V) && moves[i].bytes - at > k) c[i] = from[moves[i].from + k];
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (i < n && moves[i].bytes - at < (int64_t)sizeof(V) && moves[i].bytes - at > k) to[moves[i].to + k] = c[i];
            }
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n && moves[i].bytes - at >= (int64_t)sizeof(V)) __stcg(reinterpret_cast<V*>(to + moves[i].to), v[i]);
    }
}

// ---- host side -----------------------------------------------------------------------------------------------

bool misaligned(const void* p) { return (uintptr_t)p & 3; }

struct Device {
    int id = 0, sms = 0, smem = 0;
};
int device_of(Device* d) {
    static std::atomic<int> sms[kMaxDevices], smem[kMaxDevices];
    NEREUS_CUDA(cudaGetDevice(&d->id));
    if (d->id < 0 || d->id >= kMaxDevices) return NEREUS_ERR_UNSUPPORTED;
    d->sms = sms[d->id].load();
    d->smem = smem[d->id].load();
    if (!d->sms || !d->smem) {
        NEREUS_CUDA(cudaDeviceGetAttribute(&d->smem, cudaDevAttrMaxSharedMemoryPerBlockOptin, d->id));
        NEREUS_CUDA(cudaDeviceGetAttribute(&d->sms, cudaDevAttrMultiProcessorCount, d->id));
        smem[d->id].store(d->smem);
        sms[d->id].store(d->sms);
    }
    return NEREUS_OK;
}
// Blocks of a kernel that an SM holds, looked up once.
template <class K> int resident(K kernel, int threads, std::atomic<int>* known, const Device& d, int* out) {
    int n = known[d.id].load();
    if (!n) {
        NEREUS_CUDA(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, 0));
        if (n < 1) n = 1;
        known[d.id].store(n);
    }
    *out = n;
    return NEREUS_OK;
}

struct Range {
    uintptr_t lo, hi;
};
bool meet(const Range& a, const Range& b) { return a.lo < b.hi && b.lo < a.hi; }
Range ints(const void* p, int64_t n) { return {(uintptr_t)p, (uintptr_t)p + 4 * (uintptr_t)std::max<int64_t>(n, 0)}; }

// Whether two strided sets of pieces share no byte, as far as ranges and one common stride show it.
bool apart(uintptr_t a, int64_t na, int64_t sa, int64_t wa, uintptr_t b, int64_t nb, int64_t sb, int64_t wb) {
    if (na < 1 || nb < 1 || wa < 1 || wb < 1) return true;
    const uintptr_t end_a = a + (na - 1) * sa + wa, end_b = b + (nb - 1) * sb + wb;
    if (end_a <= b || end_b <= a) return true;
    if (sa != sb || sa < 1) return false;
    const int64_t gap = (int64_t)((a <= b ? b - a : a - b) % (uintptr_t)sa);
    return a <= b ? gap >= wa && gap + wb <= sa : gap >= wb && gap + wa <= sa;
}
// Whether no buffer of one side shares a byte with one of the other.
struct Side {
    void* const* base;
    int     n;
    int64_t count, stride, width;
};
bool apart(const Side& a, const Side& b) {
    auto hull = [](const Side& s) {
        Range r = {UINTPTR_MAX, 0};
        for (int i = 0; i < s.n; ++i) {
            const uintptr_t p = (uintptr_t)s.base[i];
            r.lo = std::min(r.lo, p);
            r.hi = std::max(r.hi, p + (s.count - 1) * s.stride + s.width);
        }
        return r;
    };
    if (!meet(hull(a), hull(b))) return true;
    // in the order of their starts, a range meets one of the other side before it or none
    struct Item {
        uintptr_t lo, hi;
        bool second;
    } all[2 * NEREUS_MAX_BUFFERS];
    int n = 0;
    for (const Side* s : {&a, &b})
        for (int i = 0; i < s->n; ++i) {
            const uintptr_t lo = (uintptr_t)s->base[i];
            all[n++] = {lo, lo + (s->count - 1) * s->stride + s->width, s == &b};
        }
    std::sort(all, all + n, [](const Item& x, const Item& y) { return x.lo < y.lo; });
    uintptr_t end[2] = {0, 0};
    bool      met = false;
    for (int i = 0; i < n && !met; ++i) {
        met = all[i].lo < end[!all[i].second];
        end[all[i].second] = std::max(end[all[i].second], all[i].hi);
    }
    if (!met) return true;
    for (int i = 0; i < a.n; ++i)
        for (int j = 0; j < b.n; ++j)
            if (!apart((uintptr_t)a.base[i], a.count, a.stride, a.width, (uintptr_t)b.base[j], b.count, b.stride, b.width)) return false;
    return true;
}

// Pieces of a buffer: n0 times n1 of `width` bytes, s0 and s1 apart, in the order of their addresses.
struct Grid {
    int64_t n0, s0, n1, s1, width;
    int64_t inner() const { return (n1 - 1) * s1 + width; }
    int64_t whole() const { return (n0 - 1) * s0 + inner(); }
};
// Whether a buffer of such pieces and one of the same strides, of n0 times n1, share a byte when the second lies `delta` bytes behind
// the first.  A piece meets those next to its own distance alone.
bool meet(const Grid& g, int64_t delta, int64_t n0, int64_t n1) {
    auto below = [](int64_t x, int64_t step) { return x >= 0 ? x / step : -((step - 1 - x) / step); };
    const int64_t first = g.s0 > 0 ? below(delta, g.s0) : 0;
    for (int64_t i = first; i <= first + 1; ++i) {
        const int64_t rest = delta - i * g.s0;
        if (i <= -n0 || i >= g.n0 || rest >= g.inner() || -rest >= (n1 - 1) * g.s1 + g.width) continue;
        const int64_t second = g.s1 > 0 ? below(rest, g.s1) : 0;
        for (int64_t j = second; j <= second + 1; ++j)
            if (j > -n1 && j < g.n1 && std::abs(rest - j * g.s1) < g.width) return true;
    }
    return false;
}
// Whether the bytes of an array meet a piece of the buffer at `base`.
bool meet(const Grid& g, uintptr_t base, const Range& r) {
    if (r.lo >= r.hi || r.hi <= base || r.lo >= base + g.whole()) return false;
    // the first piece that ends behind r.lo
    const int64_t at = r.lo > base ? (int64_t)(r.lo - base) : 0;
    int64_t       i = g.n0 > 1 ? at / g.s0 : 0, rest = at - i * g.s0, j = g.n1 > 1 ? rest / g.s1 : 0;
    if (rest - j * g.s1 >= g.width) ++j;
    if (j >= g.n1) { ++i; j = 0; }
    return i < g.n0 && base + i * g.s0 + j * g.s1 < r.hi;
}
// Whether n buffers share no byte with any of the arrays.
bool clear_of(const Grid& g, void* const* base, int n, const Range* arrays, int n_arrays) {
    Range hull = {UINTPTR_MAX, 0};
    for (int i = 0; i < n; ++i) hull = {std::min(hull.lo, (uintptr_t)base[i]), std::max(hull.hi, (uintptr_t)base[i] + g.whole())};
    for (int a = 0; a < n_arrays; ++a)
        if (arrays[a].lo < arrays[a].hi && meet(hull, arrays[a]))
            for (int i = 0; i < n; ++i)
                if (meet(g, (uintptr_t)base[i], arrays[a])) return false;
    return true;
}
// Whether n buffers of such pieces share no byte with one another.  Where `other` is given, two that are the same here and there
// count as one.  Buffers one after the other, and such whose pieces or inner stretches lie side by side, are seen at a glance.
bool disjoint(const Grid& g, void* const* base, int n, void* const* other) {
    struct Item {
        uintptr_t lo;
        int       i;
    } all[NEREUS_MAX_BUFFERS];
    for (int i = 0; i < n; ++i) all[i] = {(uintptr_t)base[i], i};
    auto before = [](const Item& a, const Item& b) { return a.lo < b.lo; };
    if (!std::is_sorted(all, all + n, before)) std::sort(all, all + n, before);
    uintptr_t least = UINTPTR_MAX;
    for (int i = 1; i < n; ++i) least = std::min(least, all[i].lo - all[i - 1].lo);
    if (n < 2 || least >= (uintptr_t)g.whole()) return true;
    const uintptr_t span = all[n - 1].lo - all[0].lo;
    if (g.n0 > 1 && least >= (uintptr_t)g.inner() && span + g.inner() <= (uintptr_t)g.s0) return true;
    if (g.n1 > 1 && least >= (uintptr_t)g.width && span + g.width <= (uintptr_t)g.s1 && (g.n0 < 2 || span + g.inner() <= (uintptr_t)g.s0)) return true;
    for (int i = 0; i < n; ++i)
        for (int j = i + 1; j < n && all[j].lo - all[i].lo < (uintptr_t)g.whole(); ++j) {
            if (other && all[i].lo == all[j].lo && other[all[i].i] == other[all[j].i]) continue;
            if (meet(g, (int64_t)(all[j].lo - all[i].lo), g.n0, g.n1)) return false;
        }
    return true;
}

// The largest of 16, 4 and 1 that divides everything.
int unit_of(uint64_t bits) { return bits % 16 == 0 ? 16 : bits % 4 == 0 ? 4 : 1; }

int check_pages(const nereus_pages_t* p) {
    if (!p || p->pools < 0 || p->pools > NEREUS_MAX_BUFFERS || p->pages < 1) return NEREUS_ERR_ARG;
    if (p->pages > NEREUS_CACHE_MAX_PAGES) return NEREUS_ERR_TOO_LARGE;
    if (!p->pools) return NEREUS_OK;
    if (p->page_bytes < 1 || p->page_stride < 0 || (p->pages > 1 && p->page_stride < p->page_bytes)) return NEREUS_ERR_ARG;
    if (p->page_bytes > kMaxPage || p->page_stride > kMaxBytes / p->pages) return NEREUS_ERR_TOO_LARGE;
    for (int i = 0; i < p->pools; ++i)
        if (!p->pool[i]) return NEREUS_ERR_ARG;
    return NEREUS_OK;
}
int check_books(const nereus_page_table_t* t, bool length) {
    if (!t || t->rows < 0 || t->columns < 1 || t->stride < 0 || (t->rows > 1 && t->stride < t->columns)) return NEREUS_ERR_ARG;
    if (t->rows > NEREUS_CACHE_MAX_ROWS || t->columns > 1 << 20 || t->stride > kMaxBytes) return NEREUS_ERR_TOO_LARGE;
    if (!t->refs || (t->rows && (!t->table || (length && !t->length)))) return NEREUS_ERR_ARG;
    if (misaligned(t->refs) || misaligned(t->table) || (length && misaligned(t->length))) return NEREUS_ERR_ALIGN;
    return NEREUS_OK;
}
// The pages of a call's pools.
Grid grid_of(const nereus_pages_t& p) { return {p.pages, p.page_stride, 1, 0, p.page_bytes}; }
// The rows of a page table.
Grid grid_of(const nereus_page_table_t& t) { return {std::max(t.rows, 1), t.rows > 1 ? 4 * t.stride : 0, 1, 0, 4 * (int64_t)t.columns}; }
// The old and new books, arrays of a call and its pools share no byte; two pools are apart, or one.
int check_apart(const nereus_pages_t& pools, const nereus_page_table_t& a, const nereus_page_table_t& b, bool length, const Range* read, int n_read,
                const Range* written, int n_written) {
    Range r[16];                                       // what is read, then what is written; the tables on their own
    int   n = 0;
    auto books = [&](const nereus_page_table_t& t) {
        r[n++] = ints(t.refs, pools.pages);
        r[n++] = t.rows && length ? ints(t.length, t.rows) : Range{0, 0};
    };
    books(a);
    for (int i = 0; i < n_read; ++i) r[n++] = read[i];
    const int first = n;
    books(b);
    for (int i = 0; i < n_written; ++i) r[n++] = written[i];
    for (int i = first; i < n; ++i)
        for (int j = 0; j < i; ++j)
            if (meet(r[i], r[j])) return NEREUS_ERR_ALIAS;
    // tables may be columns of one wider tensor
    const Grid at = grid_of(a), bt = grid_of(b);
    if (a.rows && b.rows && !apart((uintptr_t)a.table, at.n0, at.s0, at.width, (uintptr_t)b.table, bt.n0, bt.s0, bt.width)) return NEREUS_ERR_ALIAS;
    for (int i = 0; i < n; ++i)
        if ((i >= first && a.rows && meet(at, (uintptr_t)a.table, r[i])) || (b.rows && meet(bt, (uintptr_t)b.table, r[i]))) return NEREUS_ERR_ALIAS;
    r[n++] = ints(a.table, a.rows ? (a.rows - 1) * a.stride + a.columns : 0);
    r[n++] = ints(b.table, b.rows ? (b.rows - 1) * b.stride + b.columns : 0);
    const Grid pages = grid_of(pools);
    if (!disjoint(pages, pools.pool, pools.pools, pools.pool) || !clear_of(pages, pools.pool, pools.pools, r, n)) return NEREUS_ERR_ALIAS;
    return NEREUS_OK;
}

// f(a vector of the widest type that divides everything, the parameters), for as many buffers as there are.
template <int N, class F> int with_pools(const nereus_pages_t& a, const nereus_pages_t& b, F f) {
    Pools<N> p;
    uint64_t bits = (uint64_t)a.page_bytes | (a.pages > 1 ? a.page_stride : 0) | (b.pages > 1 ? b.page_stride : 0);
    for (int i = 0; i < a.pools; ++i) {
        p.from[i] = (char*)a.pool[i];
        p.to[i] = (char*)b.pool[i];
        bits |= (uintptr_t)a.pool[i] | (uintptr_t)b.pool[i];
    }
    const int unit = a.pools ? unit_of(bits) : 16;
    p.from_stride = a.page_stride;
    p.to_stride = b.page_stride;
    p.page_bytes = a.pools ? a.page_bytes : 0;
    p.pools = a.pools;
    p.from_pages = a.pages;
    p.to_pages = b.pages;
    const int64_t tile = (int64_t)unit * 32 * kTileVecs;
    p.chunks = a.pools ? (int32_t)((a.page_bytes + tile - 1) / tile) : 1;
    if (!p.pools) { p.pools = 1; p.from_pages = 0; }       // no pair is in range
    return unit == 16 ? f(uint4(), p) : unit == 4 ? f(uint32_t(), p) : f((unsigned char)0, p);
}
template <class F> int with_pools(const nereus_pages_t& a, const nereus_pages_t& b, F f) {
    return a.pools <= kFew ? with_pools<kFew>(a, b, f) : with_pools<NEREUS_MAX_BUFFERS>(a, b, f);
}

// Launches a kernel; cluster: of all its blocks; chained: it comes up while the launch before it runs, and waits for that itself.
template <class... P, class... A>
int launch(void (*kernel)(P...), dim3 grid, int threads, int64_t smem, bool cluster, bool chained, cudaStream_t stream, const A&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2] = {};
    if (cluster) {
        attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
        attr[cfg.numAttrs].val.clusterDim.x = grid.x;
        attr[cfg.numAttrs].val.clusterDim.y = attr[cfg.numAttrs].val.clusterDim.z = 1;
        ++cfg.numAttrs;
    }
    if (chained) {
        attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[cfg.numAttrs].val.programmaticStreamSerializationAllowed = 1;
        ++cfg.numAttrs;
    }
    cfg.attrs = attr;
    NEREUS_CUDA(cudaLaunchKernelEx(&cfg, kernel, args...));
    return NEREUS_OK;
}
// Blocks of the cluster that ranks pages: one where its own pass over them takes no longer than a cluster's barriers.
unsigned cluster_of(int pages) { return pages <= 32768 ? 1 : kMaxCluster; }

Books    books_of(const nereus_page_table_t& t, int pages) { return {t.table, t.length, t.refs, t.stride, t.rows, t.columns, pages}; }
NewBooks new_books_of(const nereus_page_table_t& t) { return {t.table, t.length, t.refs, t.stride, t.rows}; }

// Blocks that copy `all` blocks' tiles.
int64_t copy_blocks(int64_t all, int64_t resident, int64_t each) {
    return std::min<int64_t>(std::max(std::min(all, resident), (all + each - 1) / each), INT_MAX);
}
template <class V, class P> int copy_launch(const P& p, int64_t n, const int32_t* src, const int32_t* dst, const Device& dev, cudaStream_t stream) {
    static std::atomic<int> known[kMaxDevices];
    int per_sm;
    if (int rc = resident(copy_kernel<V, P>, kCopyThreads, known, dev, &per_sm)) return rc;
    const int64_t warps = kCopyThreads / 32, tiles = n * p.pools * p.chunks;
    const int64_t grid = copy_blocks((tiles + warps - 1) / warps, (int64_t)per_sm * dev.sms, 2);
    return launch(copy_kernel<V, P>, dim3((unsigned)grid), kCopyThreads, 0, false, false, stream, p, n, src, dst);
}
// The last launch of a fork or compaction: `most_pairs` page copies at most.
template <class P, class Work>
int apply_launch(void (*kernel)(P, Books, NewBooks, Work), std::atomic<int>* known, const P& p, int64_t most_pairs, const Books& from, const NewBooks& to,
                 const Work& w, const Device& dev, cudaStream_t stream) {
    int per_sm;
    if (int rc = resident(kernel, kCopyThreads, known, dev, &per_sm)) return rc;
    const int64_t warps = kCopyThreads / 32, tiles = p.page_bytes ? most_pairs * p.pools * p.chunks : 0;
    const int64_t held = (int64_t)per_sm * dev.sms;
    const int64_t grid = std::min(std::max(copy_blocks((tiles + warps - 1) / warps, held, 4), std::min<int64_t>(std::max(to.rows, 1), held)), kMostWaves * held);
    return launch(kernel, dim3((unsigned)grid), kCopyThreads, 0, false, true, stream, p, from, to, w);
}
template <class V, class P> int fork_apply(const P& p, const Books& from, const NewBooks& to, const Fork& f, const Device& dev, cudaStream_t stream) {
    static std::atomic<int> known[kMaxDevices];
    return apply_launch(fork_apply_kernel<V, P>, known, p, to.rows, from, to, f, dev, stream);
}
template <class V, class P> int compact_apply(const P& p, const Books& from, const NewBooks& to, const Compact& c, const Device& dev, cudaStream_t stream) {
    static std::atomic<int> known[kMaxDevices];
    return apply_launch(compact_apply_kernel<V, P>, known, p, from.pages / 2, from, to, c, dev, stream);
}

int check_states(const nereus_states_t* s) {
    if (!s || s->buffers < 1 || s->buffers > NEREUS_MAX_BUFFERS || s->rows < 0 || s->outer < 1 || s->tokens < 0 || s->token_bytes < 1) return NEREUS_ERR_ARG;
    if (s->rows > 1 << 24 || s->outer > 1 << 24 || s->tokens > kMaxBytes || s->token_bytes > kMaxBytes / std::max<int64_t>(s->tokens, 1)) return NEREUS_ERR_TOO_LARGE;
    const int64_t piece = s->tokens * s->token_bytes;
    if ((s->outer > 1 && s->outer_stride < piece) || (s->rows > 1 && s->row_stride < piece)) return NEREUS_ERR_ARG;
    if ((s->outer > 1 && s->outer_stride > kMaxBytes / s->outer) || (s->rows > 1 && s->row_stride > kMaxBytes / s->rows)) return NEREUS_ERR_TOO_LARGE;
    // one row's pieces lie before the next row's, or one piece of all rows before the next piece
    if (s->outer > 1 && s->rows > 1 && s->row_stride < (s->outer - 1) * s->outer_stride + piece && s->outer_stride < (s->rows - 1) * s->row_stride + piece)
        return NEREUS_ERR_ARG;
    for (int i = 0; i < s->buffers; ++i)
        if (!s->buffer[i] && s->rows && piece) return NEREUS_ERR_ARG;
    return NEREUS_OK;
}

Grid grid_of(const nereus_states_t& t) {
    const int64_t piece = t.tokens * t.token_bytes, row = t.rows > 1 ? t.row_stride : 0, step = t.outer > 1 ? t.outer_stride : 0;
    return t.rows < 2 || row >= (t.outer - 1) * step + piece ? Grid{t.rows, row, t.outer, step, piece} : Grid{t.outer, step, t.rows, row, piece};
}

// Whether no buffer of one side shares a byte with one of the other.
bool apart(const nereus_states_t& a, const nereus_states_t& b) {
    const int64_t piece = a.tokens * a.token_bytes;
    // rows whose pieces lie between other rows' are looked at piece by piece
    auto side = [&](const nereus_states_t& t) {
        const Grid g = grid_of(t);
        return Side{t.buffer, t.buffers, g.n0, g.s0, g.inner()};
    };
    if (apart(side(a), side(b))) return true;
    if ((a.rows > 1 && b.rows > 1 && a.row_stride != b.row_stride) || (a.outer > 1 && a.outer_stride != b.outer_stride)) return false;
    // buffers that interleave, as keys and values of every head do
    const int64_t row = a.rows > 1 ? a.row_stride : b.rows > 1 ? b.row_stride : 0, step = a.outer > 1 ? a.outer_stride : 0;
    const bool    by_row = std::max(a.rows, b.rows) < 2 || row >= (a.outer - 1) * step + piece;
    const Grid    g = by_row ? Grid{a.rows, row, a.outer, step, piece} : Grid{a.outer, step, a.rows, row, piece};
    for (int i = 0; i < a.buffers; ++i)
        for (int j = 0; j < b.buffers; ++j)
            if (meet(g, (int64_t)((uintptr_t)b.buffer[j] - (uintptr_t)a.buffer[i]), by_row ? b.rows : b.outer, by_row ? b.outer : b.rows)) return false;
    return true;
}

template <class V, int N, class S> int reorder_launch(S& s, const int32_t* parent, const int32_t* length, const Device& dev, cudaStream_t stream) {
    constexpr int64_t kTile = (int64_t)kMoveThreads * sizeof(V);
    const int64_t groups = ((int64_t)s.to_rows + s.group - 1) / s.group, items = (s.piece + kTile - 1) / kTile * s.outer * s.buffers;
    // Blocks that the GPU holds at a time (6 on an SM), as long as each then has 16 tiles at most: few enough that the last ones do
    // not keep it waiting.
    const int64_t each = std::max<int64_t>(1, std::min<int64_t>(16, (items * groups + 6 * dev.sms - 1) / (6 * dev.sms)));
    s.blocks = (int32_t)std::min<int64_t>(std::min<int64_t>((items + each - 1) / each, (((int64_t)1 << 31) - 1) / groups), 1 << 20);
    return launch(reorder_kernel<V, N, S>, dim3((unsigned)(groups * s.blocks)), kMoveThreads, 0, false, false, stream, s, parent, length);
}
template <class V, class S> int reorder_by(S& s, const int32_t* parent, const int32_t* length, const Device& dev, cudaStream_t stream) {
    typedef typename std::conditional<sizeof(V) == 1, unsigned char, uint32_t>::type Small;       // 64 vectors of 16 bytes are no registers
    return s.group <= 4    ? reorder_launch<V, 4>(s, parent, length, dev, stream)
           : s.group <= 8  ? reorder_launch<V, 8>(s, parent, length, dev, stream)
           : s.group <= 16 ? reorder_launch<V, 16>(s, parent, length, dev, stream)
                           : reorder_launch<Small, 64>(s, parent, length, dev, stream);
}
template <int N>
int reorder(const nereus_states_t& from, const nereus_states_t& to, int group, bool in_place, uint64_t bits, const int32_t* parent, const int32_t* length, const Device& dev,
            cudaStream_t stream) {
    States<N> s;
    for (int i = 0; i < to.buffers; ++i) {
        s.from[i] = (char*)from.buffer[i];
        s.to[i] = (char*)to.buffer[i];
    }
    s.from_row = from.rows > 1 ? from.row_stride : 0;
    s.to_row = to.rows > 1 ? to.row_stride : 0;
    s.from_outer = to.outer > 1 ? from.outer_stride : 0;
    s.to_outer = to.outer > 1 ? to.outer_stride : 0;
    s.piece = to.tokens * to.token_bytes;
    s.token_bytes = to.token_bytes;
    s.tokens = to.tokens;
    s.buffers = to.buffers;
    s.from_rows = from.rows;
    s.to_rows = to.rows;
    s.outer = (int32_t)to.outer;
    s.group = group;
    s.in_place = in_place;
    const int unit = unit_of(bits);
    return unit == 16  ? reorder_by<uint4>(s, parent, length, dev, stream)
           : unit == 4 ? reorder_by<uint32_t>(s, parent, length, dev, stream)
                       : reorder_by<unsigned char>(s, parent, length, dev, stream);
}

}  // namespace
}  // namespace nereus

extern "C" {

int nereus_states_reorder(const nereus_states_t* from, const nereus_states_t* to, int beams, const int32_t* parent, const int32_t* length,
                          void* cuda_stream) {
    if (int rc = check_states(from)) return rc;
    if (int rc = check_states(to)) return rc;
    if (from->buffers != to->buffers || from->outer != to->outer || from->tokens != to->tokens || from->token_bytes != to->token_bytes)
        return NEREUS_ERR_MISMATCH;
    if (misaligned(parent) || misaligned(length)) return NEREUS_ERR_ALIGN;
    if (beams < 0 || beams > NEREUS_BEAM_MAX) return NEREUS_ERR_ARG;
    if (to->rows && !parent) return NEREUS_ERR_ARG;
    const int64_t piece = to->tokens * to->token_bytes;
    if (!to->rows || !from->rows || !piece) return NEREUS_OK;
    uint64_t bits = (from->rows > 1 ? from->row_stride : 0) | (to->rows > 1 ? to->row_stride : 0) | (to->outer > 1 ? from->outer_stride | to->outer_stride : 0);
    bool same = true;
    for (int i = 0; i < to->buffers; ++i) {
        bits |= (uintptr_t)from->buffer[i] | (uintptr_t)to->buffer[i];
        same &= from->buffer[i] == to->buffer[i];
    }
    if (same) {
        if (from->rows != to->rows || (to->rows > 1 && from->row_stride != to->row_stride) || (to->outer > 1 && from->outer_stride != to->outer_stride))
            return NEREUS_ERR_MISMATCH;
        if (beams < 1 || to->rows % beams) return NEREUS_ERR_ARG;
        if (!disjoint(grid_of(*to), to->buffer, to->buffers, nullptr)) return NEREUS_ERR_ALIAS;
    } else {
        if (beams) return NEREUS_ERR_ARG;
        if (!apart(*from, *to) || !disjoint(grid_of(*to), to->buffer, to->buffers, from->buffer)) return NEREUS_ERR_ALIAS;
    }
    const Range arrays[] = {ints(parent, to->rows), ints(length, length ? from->rows : 0)};
    if (!clear_of(grid_of(*to), to->buffer, to->buffers, arrays, 2)) return NEREUS_ERR_ALIAS;
    Device dev;
    if (int rc = device_of(&dev)) return rc;
    auto go = to->buffers <= kFew ? reorder<kFew> : reorder<NEREUS_MAX_BUFFERS>;
    return go(*from, *to, same ? beams : 8, same, bits, parent, length, dev, (cudaStream_t)cuda_stream);
}

int nereus_cache_copy(const nereus_pages_t* from, const nereus_pages_t* to, int64_t n, const int32_t* src, const int32_t* dst, void* cuda_stream) {
    if (int rc = check_pages(from)) return rc;
    if (int rc = check_pages(to)) return rc;
    if (n < 0) return NEREUS_ERR_ARG;
    if (n > (int64_t)1 << 32) return NEREUS_ERR_TOO_LARGE;
    if (from->pools != to->pools || (from->pools && from->page_bytes != to->page_bytes)) return NEREUS_ERR_MISMATCH;
    if (misaligned(src) || misaligned(dst)) return NEREUS_ERR_ALIGN;
    if (n && (!src || !dst)) return NEREUS_ERR_ARG;
    bool same = from->page_stride == to->page_stride;
    for (int i = 0; i < from->pools; ++i) same &= from->pool[i] == to->pool[i];
    if (!same && !apart(Side{from->pool, from->pools, from->pages, from->page_stride, from->page_bytes},
                        Side{to->pool, to->pools, to->pages, to->page_stride, to->page_bytes}))
        return NEREUS_ERR_ALIAS;
    if (!n || !from->pools) return NEREUS_OK;
    const Range arrays[] = {ints(src, n), ints(dst, n)};
    if (!disjoint(grid_of(*to), to->pool, to->pools, from->pool) || !clear_of(grid_of(*to), to->pool, to->pools, arrays, 2)) return NEREUS_ERR_ALIAS;
    Device dev;
    if (int rc = device_of(&dev)) return rc;
    return with_pools(*from, *to, [&](auto vector, auto& p) { return copy_launch<decltype(vector)>(p, n, src, dst, dev, (cudaStream_t)cuda_stream); });
}

int nereus_cache_fork(const nereus_pages_t* pools, const nereus_page_table_t* from, const nereus_page_table_t* to, const int32_t* parent,
                      int page_size, int room, const int32_t* room_of, int32_t* copies, int32_t* status, void* cuda_stream) {
    if (int rc = check_pages(pools)) return rc;
    if (int rc = check_books(from, true)) return rc;
    if (int rc = check_books(to, true)) return rc;
    if (from->columns != to->columns) return NEREUS_ERR_MISMATCH;
    if (page_size < 1 || room < 0) return NEREUS_ERR_ARG;
    if ((int64_t)page_size * from->columns > INT_MAX) return NEREUS_ERR_TOO_LARGE;
    if (!status || (to->rows && (!parent || !copies))) return NEREUS_ERR_ARG;
    if (misaligned(parent) || misaligned(room_of) || misaligned(copies) || misaligned(status)) return NEREUS_ERR_ALIGN;
    const Range read[] = {ints(parent, to->rows), ints(room_of, room_of ? to->rows : 0)}, written[] = {ints(copies, 2 * (int64_t)to->rows), ints(status, 4)};
    if (int rc = check_apart(*pools, *from, *to, true, read, 2, written, 2)) return rc;
    Device dev;
    if (int rc = device_of(&dev)) return rc;
    const Books    old = books_of(*from, pools->pages);
    const NewBooks now = new_books_of(*to);
    const Fork     f = {parent, room_of, copies, status, {1.0 / page_size, page_size}, room};
    static std::atomic<bool> opted[kMaxDevices];
    if (!opted[dev.id].load()) {
        NEREUS_CUDA(cudaFuncSetAttribute(fork_assign_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, dev.smem - kStaticBooks));
        NEREUS_CUDA(cudaFuncSetAttribute(fork_assign_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, dev.smem - kStaticBooks));
        NEREUS_CUDA(cudaFuncSetAttribute(fork_assign_kernel<false>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
        opted[dev.id].store(true);
    }
    cudaStream_t   stream = (cudaStream_t)cuda_stream;
    const unsigned blocks = cluster_of(pools->pages);
    const int      groups = ((pools->pages + kGroup - 1) / kGroup + (int)blocks - 1) / (int)blocks;
    const int64_t  smem = (int64_t)to->rows * (int64_t)(8 + sizeof(Lack)) + ((int64_t)from->rows + groups) * 4;
    if (smem > dev.smem - kStaticBooks) return NEREUS_ERR_TOO_LARGE;
    auto apply = [&](auto vector, auto& p) { return fork_apply<decltype(vector)>(p, old, now, f, dev, stream); };
    if (blocks == 1 && ((int64_t)from->rows + to->rows) * from->columns <= kWholeEntries && smem + from->rows * 4 <= dev.smem - kStaticBooks) {
        if (int rc = launch(fork_assign_kernel<true>, dim3(1), kSmallThreads, smem + from->rows * 4, false, false, stream, old, now, f, groups)) return rc;
        return with_pools(*pools, *pools, apply);
    }
    const int     refs_units = (pools->pages + kRefsUnit - 1) / kRefsUnit, chunks = (from->columns + kTableUnit - 1) / kTableUnit;
    const int64_t units = refs_units + (int64_t)to->rows * chunks;
    if (int rc = launch(fork_start_kernel, dim3((unsigned)std::min<int64_t>(units, 8 * dev.sms)), kStartThreads, 0, false, false, stream, old, now, f, refs_units, chunks))
        return rc;
    if (from->rows) {
        // rows enough for beams to stand together, few enough for blocks on all SMs
        const int columns = (from->columns + kCountThreads - 1) / kCountThreads, most = std::max(1, 8 * dev.sms / columns);
        const int group = std::min(kMostRows, std::max(16, (from->rows + most - 1) / most));
        if (int rc = launch(fork_count_kernel, dim3((unsigned)columns, (unsigned)((from->rows + group - 1) / group)), kCountThreads, 0, false, true, stream, old, now, f, group))
            return rc;
    }
    if (int rc = launch(fork_assign_kernel<false>, dim3(blocks), kBookThreads, smem, true, true, stream, old, now, f, groups)) return rc;
    return with_pools(*pools, *pools, apply);
}

int nereus_cache_compact(const nereus_pages_t* pools, const nereus_page_table_t* from, const nereus_page_table_t* to, int64_t keep, int32_t* map,
                         int32_t* moves, int32_t* status, void* cuda_stream) {
    if (int rc = check_pages(pools)) return rc;
    if (int rc = check_books(from, false)) return rc;
    if (int rc = check_books(to, false)) return rc;
    if (from->columns != to->columns || from->rows != to->rows) return NEREUS_ERR_MISMATCH;
    if (!map || !status || (pools->pages > 1 && !moves)) return NEREUS_ERR_ARG;
    if (misaligned(map) || misaligned(status)) return NEREUS_ERR_ALIGN;
    if ((uintptr_t)moves & 7) return NEREUS_ERR_ALIGN;
    const Range written[] = {ints(map, pools->pages), ints(moves, pools->pages / 2 * 2), ints(status, 4)};
    if (int rc = check_apart(*pools, *from, *to, false, nullptr, 0, written, 3)) return rc;
    Device dev;
    if (int rc = device_of(&dev)) return rc;
    const Books    old = books_of(*from, pools->pages);
    const NewBooks now = new_books_of(*to);
    const Compact  c = {keep, map, moves, status};
    static std::atomic<bool> opted[kMaxDevices];
    if (!opted[dev.id].load()) {
        NEREUS_CUDA(cudaFuncSetAttribute(compact_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
        opted[dev.id].store(true);
    }
    if (int rc = launch(compact_kernel, dim3(cluster_of(pools->pages)), kBookThreads, 0, true, false, (cudaStream_t)cuda_stream, old, now, c)) return rc;
    return with_pools(*pools, *pools, [&](auto vector, auto& p) { return compact_apply<decltype(vector)>(p, old, now, c, dev, (cudaStream_t)cuda_stream); });
}

}  // extern "C"
