// pc_pages.hip -- pages of a KV cache on gfx950: forking, growing, freeing,
// compacting and storing, and the groups of a keyed batch.
//
// The pool's state is three integer arrays (holders of each page, page tables,
// lengths).  Every call has a kernel that checks its lists and a kernel that
// acts, and the second does nothing where the first set the status: a call
// happens whole or not at all.  Counts change by integer atomics, whose order
// does not matter; new pages go by rank among the free ones, so results do not
// depend on timing.  The kernels behind the check do not go by the status, which
// another call may set meanwhile, but by a word that one workgroup of their own
// call writes: in the workspace where there is one, else in the lengths (kGo).
#include "pc_pages.h"
#include "pc_wave.h"

namespace pcr {

namespace {

constexpr int kThreads = 1024;    // of the kernels that one workgroup runs alone

__device__ __forceinline__ int blocks_of(int tokens) { return (int)(((int64_t)tokens + kBlk - 1) / kBlk); }

__device__ __forceinline__ bool page_ok(const pc_pages &p, int page) { return (uint32_t)page < (uint32_t)p.n_pages; }

__device__ __forceinline__ bool len_ok(const pc_pages &p, int len) {
    return len >= 0 && (int64_t)len <= (int64_t)p.table_width * kBlk;
}

// Whether the status was set when the workgroup began: one read for all its
// threads, for kernels whose workgroups may set it meanwhile.
__device__ bool stopped(const int32_t *status) {
    __shared__ int32_t s;
    if (threadIdx.x == 0) s = __hip_atomic_load(status, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    return s != PC_OK;
}

// Every sequence of the list in the pool, and none twice (seen: a bit for
// each sequence of the pool).  One workgroup, all of its threads.
__device__ bool bad_list(const pc_pages &p, const int32_t *seq, int32_t n, uint32_t *seen) {
    const int words = (p.n_seqs + 31) / 32;
    for (int i = threadIdx.x; i < words; i += blockDim.x) seen[i] = 0;
    __syncthreads();
    bool bad = false;
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        const uint32_t s = (uint32_t)seq[i];
        const uint32_t bit = 1u << (s & 31);
        bad |= s >= (uint32_t)p.n_seqs || (atomicOr(&seen[s >> 5], bit) & bit);
    }
    __syncthreads();
    return bad;
}

// ------------------------------------------------------------------ copies

// 16 bytes a thread at a time.  Bound by memory: pages of 12 layers are copied at 5.5 TB/s (512 branches
// of 64 sequences), moved at 5.0 TB/s (2,000 pages of 786 KB), read and write together.
__device__ __forceinline__ void copy_page(const pc_pages &p, int which, int src, int dst) {
    const int64_t layer = (int64_t)(which >> 1) * p.layer_stride;
    uint16_t *base = static_cast<uint16_t *>((which & 1) ? p.d_v : p.d_k) + layer;
    const uint4 *s = reinterpret_cast<const uint4 *>(base + src * p.page_stride);
    uint4 *d = reinterpret_cast<uint4 *>(base + dst * p.page_stride);
    const int n = p.n_kv_heads * p.head_dim * kBlk / 8;
    for (int i = threadIdx.x; i < n; i += blockDim.x) d[i] = s[i];
}

// ------------------------------------------------------------------ fork, free

// Whether the lists are as they should be (child == nullptr: that of
// pc_pages_free).  One workgroup, all of its threads; a thread's own answer.
__device__ bool bad_lists(const pc_pages &p, const int32_t *seq, const int32_t *child, int32_t n, uint32_t *seen) {
    bool bad = bad_list(p, child ? child : seq, n, seen);
    if (child)
        for (int i = threadIdx.x; i < n; i += blockDim.x) {
            const uint32_t s = (uint32_t)seq[i], c = (uint32_t)child[i];
            bad |= s >= (uint32_t)p.n_seqs || (seen[s >> 5] >> (s & 31) & 1);
            bad |= c >= (uint32_t)p.n_seqs || p.d_len[c] != 0;
        }
    return bad;
}

// Whether sequence s's length and page numbers are in range, by `step` threads
// that begin at `at`; false where s is not in the pool (bad_lists says so).
__device__ bool bad_pages(const pc_pages &p, uint32_t s, int at, int step) {
    if (s >= (uint32_t)p.n_seqs) return false;
    const int len = p.d_len[s];
    if (!len_ok(p, len)) return true;
    const int32_t *row = p.d_table + (int64_t)s * p.table_width;
    const int nb = blocks_of(len);
    bool bad = false;
    for (int i = at; i < nb; i += step) bad |= !page_ok(p, row[i]);
    return bad;
}

// Lists and page numbers have been checked, unless the caller zeroed the status
// between two kernels of the call: none of them leads outside all the same.
__device__ void fork_one(const pc_pages &p, uint32_t from, int64_t to, int len, int at, int step) {
    const int nb = from < (uint32_t)p.n_seqs ? blocks_of(len) : 0;
    const int32_t *src = p.d_table + (int64_t)from * p.table_width;
    int32_t *dst = p.d_table + to * p.table_width;
    for (int i = at; i < nb; i += step) {
        const int page = src[i];
        dst[i] = page;
        if (page_ok(p, page)) atomicAdd(&p.d_refs[page], 1);
    }
    if (at == 0) p.d_len[to] = len;
}

__device__ void free_one(const pc_pages &p, int64_t s, int len, int at, int step) {
    const int32_t *row = p.d_table + s * p.table_width;
    const int nb = blocks_of(len);
    for (int i = at; i < nb; i += step) {
        const int page = row[i];
        if (page_ok(p, page)) atomicSub(&p.d_refs[page], 1);
    }
}

// Beside the length of a sequence that is about to be filled or emptied, between
// two kernels of one call.  No length that is in range has it; one out of range
// that looks like this becomes another one out of range.
constexpr int32_t kGo = 1 << 30;
constexpr int32_t kNoLength = 0x7fffffff;

__device__ __forceinline__ bool goes(const pc_pages &p, int32_t len) { return len >= kGo && len_ok(p, len - kGo); }

// Workgroup 0 looks at the lists, the others each at one sequence's pages.
__global__ __launch_bounds__(256) void check_lists(pc_pages p, const int32_t *seq, const int32_t *child, int32_t n,
                                                   int32_t *status) {
    if (stopped(status)) return;
    extern __shared__ uint32_t seen[];
    const bool bad = blockIdx.x == 0 ? bad_lists(p, seq, child, n, seen)
                                     : bad_pages(p, (uint32_t)seq[blockIdx.x - 1], threadIdx.x, blockDim.x);
    if (bad) atomicExch(status, PC_EINVAL);
}

// One workgroup reads the status once and says to all sequences whether the
// call happens.  A launch between the other two, 1.6 us: without it every
// workgroup, and every wave, read the status for itself, and what another call
// set at that moment stopped some of them.
__global__ __launch_bounds__(kThreads) void decide(pc_pages p, const int32_t *seq, const int32_t *child, int32_t n,
                                                   const int32_t *status) {
    __shared__ int32_t now;
    if (threadIdx.x == 0) now = __hip_atomic_load(status, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    for (int i0 = 0; i0 < n; i0 += kThreads) {
        const int i = i0 + threadIdx.x;
        const uint32_t from = i < n ? (uint32_t)seq[i] : ~0u, to = i < n && child ? (uint32_t)child[i] : from;
        const bool in = from < (uint32_t)p.n_seqs, ends = to < (uint32_t)p.n_seqs;      // if not, the call is refused
        const int32_t len = in ? p.d_len[from] : 0, old = ends ? p.d_len[to] : 0;
        if (i0 == 0) __syncthreads();       // behind the loads: now
        if (in && ends && now == PC_OK) p.d_len[to] = len | kGo;
        else if (ends && goes(p, old)) p.d_len[to] = kNoLength;
    }
}

__global__ __launch_bounds__(256) void fork_pages(pc_pages p, const int32_t *parent, const int32_t *child) {
    const uint32_t c = (uint32_t)child[blockIdx.x];
    if (c >= (uint32_t)p.n_seqs) return;
    const int32_t len = p.d_len[c];
    if (!goes(p, len)) return;
    __syncthreads();        // all have read it
    fork_one(p, parent[blockIdx.x], c, len - kGo, threadIdx.x, blockDim.x);
}

__global__ __launch_bounds__(256) void free_pages(pc_pages p, const int32_t *seq) {
    const uint32_t s = (uint32_t)seq[blockIdx.x];
    if (s >= (uint32_t)p.n_seqs) return;
    const int32_t len = p.d_len[s];
    if (!goes(p, len)) return;
    __syncthreads();        // all have read it
    free_one(p, s, len - kGo, threadIdx.x, blockDim.x);
    if (threadIdx.x == 0) p.d_len[s] = 0;
}

// Both steps by one workgroup, a wave to a sequence (see few).
__global__ __launch_bounds__(kThreads) void fork_or_free_few(pc_pages p, const int32_t *seq, const int32_t *child,
                                                             int32_t n, int32_t *status) {
    extern __shared__ uint32_t seen[];
    __shared__ int any_bad;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (stopped(status)) return;
    if (threadIdx.x == 0) any_bad = 0;
    bool bad = bad_lists(p, seq, child, n, seen);
    for (int i = wave; i < n; i += kThreads / 64) bad |= bad_pages(p, (uint32_t)seq[i], lane, 64);
    if (bad) any_bad = 1;
    __syncthreads();
    if (any_bad) {
        if (threadIdx.x == 0) *status = PC_EINVAL;
        return;
    }
    for (int i = wave; i < n; i += kThreads / 64) {
        if (child) {
            fork_one(p, seq[i], child[i], p.d_len[seq[i]], lane, 64);
        } else {
            const int len = p.d_len[seq[i]];
            free_one(p, seq[i], len, lane, 64);
            if (lane == 0) p.d_len[seq[i]] = 0;
        }
    }
}

// ------------------------------------------------------------------ free pages

// Bitmap and count of a chunk's free pages.
__global__ __launch_bounds__(256) void scan_refs(pc_pages p, PagesWs ws) {
    __shared__ int32_t sums[4];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int base = blockIdx.x * kChunkPages + w * (kChunkPages / 4);
    int count = 0;
#pragma unroll
    for (int i = 0; i < kChunkPages / 256; ++i) {
        const int page = base + i * 64 + lane;
        const uint64_t m = __ballot(page < p.n_pages && p.d_refs[page] == 0);
        if (lane == 0) ws.free_bits[base / 64 + i] = m;
        count += __popcll(m);
    }
    if (lane == 0) sums[w] = count;
    __syncthreads();
    if (threadIdx.x == 0) ws.chunk_free[blockIdx.x] = sums[0] + sums[1] + sums[2] + sums[3];
}

// A pool of so many pages or fewer is scanned by the one workgroup that plans;
// larger ones by kernels of their own before and after it.  A call that finds
// nothing to copy, one way / the other: 512 pages 6.7 / 10.5 us (extend) and 5.5 /
// 10.3 us (compact), 16,384 pages 9.6 / 12.1 and 12.4 / 15.9, 65,536 pages 18.3 /
// 11.8 and 35.6 / 16.1.
constexpr int kSmallPool = 16384;
static_assert(kSmallPool / 64 <= kThreads, "a thread for each word");

// Free pages as bits, with those before each word.
struct FreeBits {
    uint64_t bits[kSmallPool / 64];
    int32_t before[kSmallPool / 64];
    __device__ bool is_free(int page) const { return bits[page >> 6] >> (page & 63) & 1; }
    // free pages before this one
    __device__ int rank(int page) const {
        return before[page >> 6] + __popcll(bits[page >> 6] & ((1ull << (page & 63)) - 1));
    }
};

// Scans a small pool by one workgroup; all its free pages.
__device__ int scan_small(const pc_pages &p, FreeBits &f, int *lds) {
    const int lane = threadIdx.x & 63, words = (p.n_pages + 63) / 64;
#pragma unroll 4
    for (int w = threadIdx.x >> 6; w < words; w += kThreads / 64) {
        const int page = w * 64 + lane;
        const uint64_t m = __ballot(page < p.n_pages && p.d_refs[page] == 0);
        if (lane == 0) f.bits[w] = m;
    }
    __syncthreads();
    int all;
    const int t = threadIdx.x, x = block_sum<kThreads>(t < words ? (int)__popcll(f.bits[t]) : 0, &all, lds);
    if (t < words) f.before[t] = x;
    __syncthreads();
    return all;
}

// One chunk of a scanned pool, by 256 threads.
__device__ void load_chunk(const PagesWs &ws, FreeBits &f, int *lds) {
    const int t = threadIdx.x;
    const uint64_t m = t < 64 ? ws.free_bits[(int64_t)blockIdx.x * 64 + t] : 0;
    int all;
    const int x = ws.chunk_free[blockIdx.x] + block_sum<256>((int)__popcll(m), &all, lds);
    if (t < 64) {
        f.bits[t] = m;
        f.before[t] = x;
    }
    __syncthreads();
}

// Free pages of all chunks; chunk_free becomes those before the chunk.  One
// workgroup, all of its threads.
__device__ int sum_chunks(const PagesWs &ws, int *lds) {
    int before = 0;
    for (int c0 = 0; c0 < ws.n_chunks; c0 += kThreads) {
        const int c = c0 + threadIdx.x;
        const int v = c < ws.n_chunks ? ws.chunk_free[c] : 0;
        int all;
        const int x = block_sum<kThreads>(v, &all, lds);
        if (c < ws.n_chunks) ws.chunk_free[c] = before + x;
        before += all;
    }
    return before;
}

// ------------------------------------------------------------------ extend

// One workgroup: checks the list, says which last pages are copied, gives
// every sequence its ranks among the free pages, and takes the copied pages'
// holders off them.  A shared last page's count tells whether all its holders
// grow: each takes itself off, and where nothing is left the lowest place in
// the list, found by an atomic minimum in the same word, keeps the page.  (A
// barrier waits for a wave's atomics, and the loads that follow go past L1, so
// no fence is needed within the workgroup.)
template <bool kSmall>
__global__ __launch_bounds__(kThreads) void extend_plan(pc_pages p, const int32_t *seq, const int32_t *add, int32_t n,
                                                        PagesWs ws, int32_t *status) {
    if (threadIdx.x == 0) ws.head[3] = 0;
    if (stopped(status)) return;
    constexpr int kPer = PC_MAX_BATCH / kThreads;
    extern __shared__ uint32_t seen[];
    __shared__ FreeBits free_bits;
    __shared__ int lds[16];
    __shared__ int64_t lds64[16];
    __shared__ int any_bad, any_shared;
    int32_t *first = ws.entry, *have = first + n, *fresh = have + n, *copied = fresh + n;
    const int words = (p.n_seqs + 31) / 32;
    for (int i = threadIdx.x; i < words; i += kThreads) seen[i] = 0;
    if (threadIdx.x == 0) any_bad = any_shared = 0;
    __syncthreads();
    auto count = [&](int page) {
        return __hip_atomic_load(&p.d_refs[page], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    };
    int need[kPer], last[kPer];     // new pages; a shared last page, or -1
    bool keeps[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        const int i = e * kThreads + threadIdx.x;
        need[e] = 0;
        last[e] = -1;
        keeps[e] = false;
        if (i >= n) continue;
        const uint32_t s = (uint32_t)seq[i];
        const int a = add[i];
        bool bad = s >= (uint32_t)p.n_seqs || a < 0;
        if (!bad) {
            const uint32_t bit = 1u << (s & 31);
            const int len = p.d_len[s];
            bad = (atomicOr(&seen[s >> 5], bit) & bit) || !len_ok(p, len) ||
                  (int64_t)len + a > (int64_t)p.table_width * kBlk;
            if (!bad) {
                const int nb = blocks_of(len);
                need[e] = blocks_of(len + a) - nb;
                have[i] = nb;
                if (a > 0 && len % kBlk) {
                    const int page = p.d_table[(int64_t)s * p.table_width + nb - 1];
                    if (!page_ok(p, page)) {
                        bad = true;
                    } else if (count(page) > 1) {
                        last[e] = page;
                        any_shared = 1;
                    }
                }
            }
        }
        if (bad) any_bad = 1;
    }
    __syncthreads();
    if (any_bad) {
        if (threadIdx.x == 0) *status = PC_EINVAL;
        return;
    }
    const int n_free = kSmall ? scan_small(p, free_bits, lds) : sum_chunks(ws, lds);
    if (any_shared) {
#pragma unroll
        for (int e = 0; e < kPer; ++e)
            if (last[e] >= 0) atomicSub(&p.d_refs[last[e]], 1);
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kPer; ++e)
            if (last[e] >= 0 && count(last[e]) <= 0) atomicMin(&p.d_refs[last[e]], e * kThreads + (int)threadIdx.x - n);
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kPer; ++e)
            if (last[e] >= 0) {
                keeps[e] = count(last[e]) == e * kThreads + (int)threadIdx.x - n;
                if (!keeps[e]) ++need[e];
            }
    }
    int64_t total = 0;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        if (e * kThreads >= n) break;
        const int i = e * kThreads + threadIdx.x;
        int64_t all;
        const int64_t x = block_sum<kThreads>((int64_t)need[e], &all, lds64);
        if (i < n) {
            first[i] = (int32_t)(total + x);    // of use only where the pool has them all
            fresh[i] = need[e];
            copied[i] = keeps[e] ? -1 : last[e];
        }
        total += all;
    }
    const bool short_of = total > n_free;
    if (any_shared) {
        // kept pages have one holder again; where the pool is short, all is as before
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kPer; ++e)
            if (keeps[e])
                __hip_atomic_store(&p.d_refs[last[e]], short_of ? 0 : 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        if (short_of)
#pragma unroll
            for (int e = 0; e < kPer; ++e)
                if (last[e] >= 0) atomicAdd(&p.d_refs[last[e]], 1);
    }
    if (short_of) {
        if (threadIdx.x == 0) *status = PC_ENOPAGES;
        return;
    }
    if (threadIdx.x == 0) {
        ws.head[0] = (int32_t)total;
        ws.head[3] = 1;
    }
    if (kSmall && total) {
        // the lowest ones: no further than the word with the last of them
        for (int page = threadIdx.x; page < p.n_pages && free_bits.before[page >> 6] < total; page += kThreads)
            if (free_bits.is_free(page)) {
                const int rank = free_bits.rank(page);
                if (rank < total) {
                    ws.list[rank] = page;
                    p.d_refs[page] = 1;
                }
            }
    }
}

// The free pages of rank < head[0], listed by rank; they have a holder now.
__global__ __launch_bounds__(256) void list_free(pc_pages p, PagesWs ws) {
    if (ws.head[3] == 0) return;
    __shared__ FreeBits f;
    __shared__ int lds[4];
    const int total = ws.head[0], base = blockIdx.x * kChunkPages;
    if (ws.chunk_free[blockIdx.x] >= total) return;
    load_chunk(ws, f, lds);
    for (int at = threadIdx.x; at < kChunkPages; at += 256)
        if (f.is_free(at)) {        // no page behind the pool's last is
            const int rank = f.rank(at);
            if (rank < total) {
                ws.list[rank] = base + at;
                p.d_refs[base + at] = 1;
            }
        }
}

__global__ __launch_bounds__(256) void extend_pages(pc_pages p, const int32_t *seq, const int32_t *add, int32_t n,
                                                    PagesWs ws) {
    if (ws.head[3] == 0) return;
    const int i = blockIdx.x;
    const int first = ws.entry[i], have = ws.entry[n + i], fresh = ws.entry[2 * n + i], src = ws.entry[3 * n + i];
    if (blockIdx.y == 0) {
        const int64_t s = seq[i];
        int32_t *row = p.d_table + s * p.table_width + have - (src >= 0);
        for (int j = threadIdx.x; j < fresh; j += blockDim.x) row[j] = ws.list[first + j];
        if (threadIdx.x == 0) p.d_len[s] += add[i];
    }
    if (src >= 0) copy_page(p, blockIdx.y, src, ws.list[first]);
}

// ------------------------------------------------------------------ compact

// A page's part in the moves: the free places before n_live and the pages
// behind it are listed by rank.  free_before: free pages before this one.
__device__ __forceinline__ void list_move(const PagesWs &ws, int page, bool is_free, int free_before, int live, int holes) {
    if (is_free) {
        if (page < live) ws.list[free_before] = page;
    } else if (page >= live) {
        const int i = page - free_before - (live - holes);      // pages in use before it, less those that stay
        ws.moved[i] = page;
        ws.rank[page] = i;
    }
}

// One workgroup: pages in use, and how many of them lie behind that number.
template <bool kSmall>
__global__ __launch_bounds__(kThreads) void compact_plan(pc_pages p, PagesWs ws, int32_t *n_live, const int32_t *status) {
    if (threadIdx.x == 0) ws.head[3] = 0;
    if (stopped(status)) return;
    __shared__ FreeBits free_bits;
    __shared__ int lds[16];
    const int live = p.n_pages - (kSmall ? scan_small(p, free_bits, lds) : sum_chunks(ws, lds));
    __syncthreads();
    int holes = 0;
    if (live < p.n_pages && kSmall) {
        holes = free_bits.rank(live);
    } else if (live < p.n_pages) {
        // free pages before page `live`
        const int c = live / kChunkPages, in = live % kChunkPages, t = threadIdx.x;
        int x = 0;
        if (t < 64 && t * 64 < in) {
            const uint64_t m = ws.free_bits[(int64_t)c * 64 + t];
            const int bits = in - t * 64;
            x = __popcll(bits >= 64 ? m : m & ((1ull << bits) - 1));
        }
        int all;
        block_sum<kThreads>(x, &all, lds);
        holes = ws.chunk_free[c] + all;
    }
    if (kSmall) {
        for (int page = threadIdx.x; page < p.n_pages; page += kThreads)
            list_move(ws, page, free_bits.is_free(page), free_bits.rank(page), live, holes);
        for (int w = threadIdx.x; w < (p.n_pages + 63) / 64; w += kThreads) ws.free_bits[w] = free_bits.bits[w];
    }
    if (threadIdx.x == 0) {
        ws.head[0] = live;
        ws.head[1] = holes;
        ws.head[3] = 1;
        *n_live = live;
    }
}

__global__ __launch_bounds__(256) void list_moves(pc_pages p, PagesWs ws) {
    if (ws.head[3] == 0) return;
    __shared__ FreeBits f;
    __shared__ int lds[4];
    const int live = ws.head[0], holes = ws.head[1], base = blockIdx.x * kChunkPages;
    load_chunk(ws, f, lds);
    for (int at = threadIdx.x; at < kChunkPages && base + at < p.n_pages; at += 256)
        list_move(ws, base + at, f.is_free(at), f.rank(at), live, holes);
}

__global__ __launch_bounds__(256) void compact_pages(pc_pages p, int32_t *refs_to, int32_t *table_to, PagesWs ws,
                                                     int32_t *status) {
    if (ws.head[3] == 0) return;
    const int live = ws.head[0], moves = ws.head[1];
    const int64_t copies = (int64_t)moves * 2 * p.n_layers;
    for (int64_t u = blockIdx.x; u < copies; u += gridDim.x) {
        const int which = (int)(u / moves), i = (int)(u - (int64_t)which * moves);
        copy_page(p, which, ws.moved[i], ws.list[i]);
    }
    const int64_t step = (int64_t)gridDim.x * blockDim.x, at = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    auto is_free = [&](int page) { return ws.free_bits[page >> 6] >> (page & 63) & 1; };
    for (int64_t u = at; u < p.n_pages; u += step) {
        const int page = (int)u;
        if (page < live) {
            if (!is_free(page)) refs_to[page] = p.d_refs[page];
        } else if (is_free(page)) {
            refs_to[page] = 0;
        } else {    // both counts of a move by one thread: the two arrays may be one
            refs_to[ws.list[ws.rank[page]]] = p.d_refs[page];
            refs_to[page] = 0;
        }
    }
    const int64_t entries = (int64_t)p.n_seqs * p.table_width;
    bool bad = false;
    for (int64_t u = at; u < entries; u += step) {
        const int64_t s = u / p.table_width;
        int page = p.d_table[u];
        const int len = p.d_len[s];
        if (!len_ok(p, len)) {
            bad = true;
        } else if (u - s * p.table_width < blocks_of(len)) {
            if (!page_ok(p, page) || is_free(page)) bad = true;
            else if (page >= live) page = ws.list[ws.rank[page]];
        }
        table_to[u] = page;
    }
    if (bad) atomicExch(status, PC_EINVAL);
}

// ------------------------------------------------------------------ write

__global__ __launch_bounds__(256) void write_rows(pc_pages p, int32_t layer, const int32_t *seq, const int32_t *new_off,
                                                  int32_t n, int64_t n_tokens, pc_rows kn, pc_rows vn, int32_t *status) {
    if (stopped(status)) return;
    extern __shared__ uint32_t seen[];
    bool bad = false;
    const int i = blockIdx.x;
    if (i == n) {    // the last column looks at the list
        if (blockIdx.y == 0 && bad_list(p, seq, n, seen)) atomicExch(status, PC_EINVAL);
        return;
    }
    const uint32_t s = (uint32_t)seq[i];
    const int64_t r0 = new_off[i], r1 = new_off[i + 1];
    const int len = s < (uint32_t)p.n_seqs ? p.d_len[s] : -1;
    if (r0 < 0 || r1 < r0 || r1 > n_tokens || !len_ok(p, len) || r1 - r0 > len) {
        bad = true;
    } else {
        const int32_t *row = p.d_table + (int64_t)s * p.table_width;
        const int per_row = p.head_dim / 8, units = p.n_kv_heads * per_row;
        const int32_t head_stride = p.layout == PC_HEADS_FIRST ? kBlk * p.head_dim : p.head_dim;
        const int32_t token_stride = p.layout == PC_HEADS_FIRST ? p.head_dim : p.n_kv_heads * p.head_dim;
        uint16_t *kp = static_cast<uint16_t *>(p.d_k) + (int64_t)layer * p.layer_stride;
        uint16_t *vp = static_cast<uint16_t *>(p.d_v) + (int64_t)layer * p.layer_stride;
        // as many tokens at a time as a workgroup's threads have pieces for
        const int tokens = units < 256 ? 256 / units : 1, n_new = (int)(r1 - r0);
        const int my_token = (int)threadIdx.x / units, w0 = (int)threadIdx.x - my_token * units;
        for (int j = blockIdx.y * tokens + my_token; my_token < tokens && j < n_new; j += gridDim.y * tokens)
            for (int w = w0; w < units; w += 256) {
                const int h = w / per_row, c = w - h * per_row;
                const uint4 k = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(kn.d_data) +
                                                                 (r0 + j) * kn.token_stride + h * kn.head_stride + c * 8);
                const uint4 v = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(vn.d_data) +
                                                                 (r0 + j) * vn.token_stride + h * vn.head_stride + c * 8);
                const int pos = len - n_new + j, page = row[pos / kBlk];
                if (!page_ok(p, page) || p.d_refs[page] != 1) {
                    bad = true;
                    continue;
                }
                const int64_t to = page * p.page_stride + (pos % kBlk) * token_stride + h * head_stride + c * 8;
                *reinterpret_cast<uint4 *>(kp + to) = k;
                *reinterpret_cast<uint4 *>(vp + to) = v;
            }
    }
    if (bad) atomicExch(status, PC_EINVAL);
}

// ------------------------------------------------------------------ groups

// One workgroup of NT threads, for up to NT * kPer requests: the first request
// with the same key of block min_blocks - 1 by a hash table in LDS, then a sort
// by (that request, own number): a bitonic network whose exchanges within a
// wave go by registers, so that 10 of the 55 steps for 1,024 requests need a
// barrier (21 us before, with one at every step).  Leaves each request's group
// beside its number in d_order for the next kernel, and the first request's
// blocks in d_shared.
template <int NT, int kPer>
__global__ __launch_bounds__(NT) void group_requests(const uint64_t *keys, int64_t n_keys, const int64_t *key_off,
                                                     int32_t R, int32_t Rp, int32_t min_blocks, int32_t *order,
                                                     int32_t *group_off, int32_t *shared, int32_t *n_groups,
                                                     int32_t *status) {
    extern __shared__ __align__(16) uint64_t mark[];          // [Rp]
    int32_t *lead = reinterpret_cast<int32_t *>(mark + Rp);   // [Rp] then the sorted words
    int32_t *tab = lead + Rp;                                 // [2 Rp]
    __shared__ int lds[NT / 64];
    __shared__ int any_bad;
    const int tid = threadIdx.x;
    if (tid == 0) any_bad = 0;
    for (int i = tid; i < 2 * Rp; i += NT) tab[i] = -1;
    __syncthreads();
    int blocks[kPer], word[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        const int i = e * NT + tid;
        blocks[e] = 0;
        if (i < Rp) lead[i] = i;
        if (i >= R) continue;
        const int64_t a = key_off[i], b = key_off[i + 1];
        if (a < 0 || b < a || b > n_keys || b - a > 1 << 26) any_bad = 1;
        else blocks[e] = (int)(b - a);
        if (blocks[e] >= min_blocks) mark[i] = keys[a + min_blocks - 1];
    }
    __syncthreads();
    if (tid == 0) {
        *status = any_bad ? PC_EINVAL : PC_OK;
        if (any_bad) *n_groups = -1;
    }
    if (any_bad) return;
    const uint32_t slots = 2 * Rp;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        const int i = e * NT + tid;
        word[e] = i;        // a request that has this one's key
        if (i >= R || blocks[e] < min_blocks) continue;
        uint32_t at = (uint32_t)((mark[i] * 0x9E3779B97F4A7C15ull) >> 40) & (slots - 1);
        for (;;) {          // at most half of the slots are ever taken
            const int cur = atomicCAS(&tab[at], -1, i);
            if (cur < 0) break;
            if (mark[cur] == mark[i]) {
                word[e] = cur;
                atomicMin(&lead[cur], i);
                break;
            }
            at = (at + 1) & (slots - 1);
        }
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        const int i = e * NT + tid;
        word[e] = i < R ? lead[word[e]] * PC_MAX_BATCH + i : 0x7fffffff;
    }
    __syncthreads();
    int32_t *to = lead, *other = tab;       // exchanged in turn: one barrier a step
    for (int k = 2; k <= Rp; k <<= 1)
        for (int j = k >> 1; j > 0; j >>= 1) {
            int theirs[kPer];
            if (j >= NT) {
#pragma unroll
                for (int e = 0; e < kPer; ++e) {
                    theirs[e] = 0;
#pragma unroll
                    for (int x = 0; x < kPer; ++x)
                        if (x == (e ^ (j / NT))) theirs[e] = word[x];
                }
            } else if (j >= 64) {
#pragma unroll
                for (int e = 0; e < kPer; ++e)
                    if (e * NT + tid < Rp) to[e * NT + tid] = word[e];
                __syncthreads();
#pragma unroll
                for (int e = 0; e < kPer; ++e) theirs[e] = e * NT + tid < Rp ? to[(e * NT + tid) ^ j] : 0;
                int32_t *t = to;
                to = other;
                other = t;
            } else {
#pragma unroll
                for (int e = 0; e < kPer; ++e) theirs[e] = __shfl_xor(word[e], j);
            }
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                const int i = e * NT + tid;
                const bool least = ((i & j) == 0) == ((i & k) == 0);
                word[e] = least ? min(word[e], theirs[e]) : max(word[e], theirs[e]);
            }
        }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kPer; ++e)
        if (e * NT + tid < Rp) lead[e * NT + tid] = word[e];
    __syncthreads();
    int groups = 0;
    for (int p0 = 0; p0 < R; p0 += NT) {
        const int q = p0 + tid;
        const int x = q < R ? lead[q] : 0;
        const int l = x / PC_MAX_BATCH, i = x % PC_MAX_BATCH;
        const bool begins = q < R && (q == 0 || lead[q - 1] / PC_MAX_BATCH != l);
        int all;
        const int g = groups + block_sum<NT>((int)begins, &all, lds) + begins - 1;
        if (q < R) order[q] = g * PC_MAX_BATCH + i;
        if (begins) {
            const bool alone = q + 1 >= R || lead[q + 1] / PC_MAX_BATCH != l;
            group_off[g] = q;
            shared[g] = alone ? 0 : (int32_t)(key_off[i + 1] - key_off[i]);
        }
        groups += all;
    }
    for (int g = groups + tid; g <= R; g += NT) {
        group_off[g] = R;
        if (g < R) shared[g] = 0;
    }
    if (tid == 0) *n_groups = groups;
}

// A workgroup for each request: how many leading keys it has in common with
// its group's first one.  It goes by the number of groups, which this call alone
// writes, and not by the status.
__global__ __launch_bounds__(256) void group_shared(const uint64_t *keys, const int64_t *key_off, int32_t *order,
                                                    const int32_t *group_off, int32_t *shared,
                                                    const int32_t *n_groups) {
    if (*n_groups < 0) return;
    __shared__ int first_off;
    const int q = blockIdx.x;
    const int x = order[q], g = x / PC_MAX_BATCH, i = x % PC_MAX_BATCH;
    const int q0 = group_off[g];
    if (q > q0) {
        // the word of the group's first request may be the number alone already
        const int l = __hip_atomic_load(&order[q0], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) % PC_MAX_BATCH;
        const int64_t a = key_off[i], b = key_off[l];
        const int64_t na = key_off[i + 1] - a, nb = key_off[l + 1] - b;
        const int n = (int)(na < nb ? na : nb);
        if (threadIdx.x == 0) first_off = n;
        __syncthreads();
        for (int k0 = 0; k0 < n; k0 += 1024) {
            int off = 0x7fffffff;
#pragma unroll
            for (int e = 3; e >= 0; --e) {
                const int k = k0 + e * 256 + threadIdx.x;
                if (k < n && keys[a + k] != keys[b + k]) off = k;
            }
            if (off < n) atomicMin(&first_off, off);
            __syncthreads();
            const int found = first_off;
            __syncthreads();
            if (found < n) break;
        }
        if (threadIdx.x == 0) atomicMin(&shared[g], first_off);
    }
    __syncthreads();        // all waves have read their word: x
    if (threadIdx.x == 0) __hip_atomic_store(&order[q], i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

int64_t up(int64_t v) { return (v + 255) / 256 * 256; }

}  // namespace

int64_t pages_ws(const pc_pages &p, int64_t n, char *base, PagesWs *ws) {
    const int32_t chunks = (p.n_pages + kChunkPages - 1) / kChunkPages;
    int64_t o = 0;
    auto take = [&](int64_t bytes) { const int64_t at = o; o += up(bytes); return at; };
    const int64_t bits = take((int64_t)chunks * 512), cf = take(4LL * chunks), list = take(4LL * p.n_pages),
                  moved = take(4LL * p.n_pages), rank = take(4LL * p.n_pages), entry = take(16 * (n < 1 ? 1 : n)),
                  head = take(16);
    if (ws)
        *ws = PagesWs{reinterpret_cast<uint64_t *>(base + bits), reinterpret_cast<int32_t *>(base + cf),
                      reinterpret_cast<int32_t *>(base + list), reinterpret_cast<int32_t *>(base + moved),
                      reinterpret_cast<int32_t *>(base + rank), reinterpret_cast<int32_t *>(base + entry),
                      reinterpret_cast<int32_t *>(base + head), chunks};
    return o;
}

static size_t seen_bytes(const pc_pages &p) { return (size_t)((p.n_seqs + 31) / 32) * 4; }

// Whether one workgroup forks or frees by itself, a wave to a sequence.  A fork and a free of n sequences of so many
// blocks by it / by three kernels each: 1 of 14 6.0 / 10.3 us, 16 of 64 6.9 / 11.5, 16 of 200 9.5 / 12.1, 16 of 600
// 15.3 / 13.5, 1 of 4,000 52 / 24; with two to a wave 32 of 32 9.0 / 11.6, 32 of 128 11.7 / 11.6, with four 64 of 14
// 15.9 / 11.8.  The host knows how wide the table is, not how much of it is in use.
static bool few(const pc_pages &p, int32_t n) { return n <= 16 ? p.table_width <= 640 : n <= 32 && p.table_width <= 128; }

hipError_t launch_fork(const pc_pages &p, const int32_t *parent, const int32_t *child, int32_t n, int32_t *status,
                       hipStream_t st) {
    if (few(p, n)) {
        fork_or_free_few<<<1, kThreads, seen_bytes(p), st>>>(p, parent, child, n, status);
    } else {
        check_lists<<<n + 1, 256, seen_bytes(p), st>>>(p, parent, child, n, status);
        decide<<<1, kThreads, 0, st>>>(p, parent, child, n, status);
        fork_pages<<<n, 256, 0, st>>>(p, parent, child);
    }
    return hipGetLastError();
}

hipError_t launch_free(const pc_pages &p, const int32_t *seq, int32_t n, int32_t *status, hipStream_t st) {
    if (few(p, n)) {
        fork_or_free_few<<<1, kThreads, seen_bytes(p), st>>>(p, seq, nullptr, n, status);
    } else {
        check_lists<<<n + 1, 256, seen_bytes(p), st>>>(p, seq, nullptr, n, status);
        decide<<<1, kThreads, 0, st>>>(p, seq, nullptr, n, status);
        free_pages<<<n, 256, 0, st>>>(p, seq);
    }
    return hipGetLastError();
}

hipError_t launch_extend(const pc_pages &p, const int32_t *seq, const int32_t *add, int32_t n, const PagesWs &ws,
                         int32_t *status, hipStream_t st) {
    if (p.n_pages <= kSmallPool) {
        extend_plan<true><<<1, kThreads, seen_bytes(p), st>>>(p, seq, add, n, ws, status);
    } else {
        scan_refs<<<ws.n_chunks, 256, 0, st>>>(p, ws);
        extend_plan<false><<<1, kThreads, seen_bytes(p), st>>>(p, seq, add, n, ws, status);
        list_free<<<ws.n_chunks, 256, 0, st>>>(p, ws);
    }
    extend_pages<<<dim3(n, 2 * p.n_layers), 256, 0, st>>>(p, seq, add, n, ws);
    return hipGetLastError();
}

hipError_t launch_compact(const pc_pages &p, int32_t *refs_to, int32_t *table_to, int32_t *n_live, const PagesWs &ws,
                          int32_t *status, hipStream_t st) {
    if (p.n_pages <= kSmallPool) {
        compact_plan<true><<<1, kThreads, 0, st>>>(p, ws, n_live, status);
    } else {
        scan_refs<<<ws.n_chunks, 256, 0, st>>>(p, ws);
        compact_plan<false><<<1, kThreads, 0, st>>>(p, ws, n_live, status);
        list_moves<<<ws.n_chunks, 256, 0, st>>>(p, ws);
    }
    compact_pages<<<2048, 256, 0, st>>>(p, refs_to, table_to, ws, status);
    return hipGetLastError();
}

hipError_t launch_write(const pc_pages &p, int32_t layer, const int32_t *seq, const int32_t *new_off, int32_t n,
                        int64_t n_tokens, const pc_rows &k_new, const pc_rows &v_new, int32_t *status, hipStream_t st) {
    // workgroups enough for the case that one sequence has all the tokens, but not many more than the chip
    // holds at a time (22,000 tokens of 12 sequences: 2,048 41.3 us, 8,192 39.6 us, 32,768 50.2 us; bound by
    // memory, 4.4 TB/s)
    int64_t y = (n_tokens * p.n_kv_heads * (p.head_dim / 8) + 255) / 256;
    const int64_t most = 8192 / n > 1 ? 8192 / n : 1;
    y = y < 1 ? 1 : y > most ? most : y;
    write_rows<<<dim3(n + 1, (uint32_t)y), 256, seen_bytes(p), st>>>(p, layer, seq, new_off, n, n_tokens, k_new, v_new, status);
    return hipGetLastError();
}

hipError_t launch_groups(const uint64_t *keys, int64_t n_keys, const int64_t *key_off, int32_t n_req,
                         int32_t min_blocks, int32_t *order, int32_t *group_off, int32_t *shared, int32_t *n_groups,
                         int32_t *status, hipStream_t st) {
    int32_t rp = 2;
    while (rp < n_req) rp <<= 1;
    const size_t bytes = (size_t)rp * (8 + 4 + 8);
    auto launch = [&](auto *kernel, int threads) {
        if (bytes > 64 * 1024 - 256) {
            const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel),
                                                     hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
            if (e != hipSuccess) return e;
        }
        kernel<<<1, threads, bytes, st>>>(keys, n_keys, key_off, n_req, rp, min_blocks, order, group_off, shared,
                                          n_groups, status);
        return hipGetLastError();
    };
    // No more registers to sort than requests need: with four a thread, 1,024 of them took 22 us in place
    // of 13.  256 threads for few, whose barriers and sums cost less: 8 requests 6.4 us in place of 6.7, 256
    // 10.7 in place of 11.6 (both kernels).
    const hipError_t e = rp <= 256    ? launch(&group_requests<256, 1>, 256)
                         : rp <= 1024 ? launch(&group_requests<1024, 1>, 1024)
                         : rp <= 2048 ? launch(&group_requests<1024, 2>, 1024)
                                      : launch(&group_requests<1024, 4>, 1024);
    if (e != hipSuccess) return e;
    group_shared<<<n_req, 256, 0, st>>>(keys, key_off, order, group_off, shared, n_groups);
    return hipGetLastError();
}

}  // namespace pcr
