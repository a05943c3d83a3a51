// pc_attn.hip -- attention over paged K and V on gfx950, a batch's shared
// prefixes read once for all their requests.
//
// A batch is cut into segments: a group's queries against its shared tokens,
// and each request's queries against its own.  A segment is a small dense
// problem: rows (a query and one of the query heads of a KV head) against
// tokens.  Rows are cut into tiles, long token ranges into chunks (the plan),
// and every (tile, KV head, chunk) is one item.  Per item
//   m = max s,  l = sum 2^(s - m),  o = sum 2^(s - m) v / l,  s = q.k scale log2(e)
// in one pass over the tokens with a running m and l.  Items of one row are
// joined by w_i = 2^(lse_i - max lse), lse_i = m_i + log2(l_i).
//
// Both kernels form S^T = K Q^T and O^T = V^T P^T, so that a lane holds scores
// of one query in registers: the running statistics need one exchange between
// lane halves (or quarters), the scaling of O^T none, and P^T is the B operand
// of the second product as it lies, once the order of the tokens inside a
// matrix instruction's k is taken to be the order in which the first product
// leaves them.  V^T comes from row-major V by the transposing LDS read.
#include <type_traits>

#include "pc_pages.h"
#include "pc_wave.h"

namespace pcr {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// kLift: the weights are multiplied by 2^kLift on their way to the second product (and their sum with them), so that
// small ones keep their bits in a type of few exponents.
struct Bf16 {
    static constexpr float kLift = 0.f;
    typedef __bf16 x8 __attribute__((ext_vector_type(8)));
    static __device__ f32x16 mma32(s16x8 a, s16x8 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
    }
    static __device__ f32x4 mma16(s16x8 a, s16x8 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
    }
    // to nearest, ties to even
    static __device__ uint32_t pack(float a, float b) {
        return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
    }
    // what pack() left of the two
    static __device__ uint32_t pack_rest(float a, float b, uint32_t packed) {
        return pack(a - __builtin_bit_cast(float, packed << 16), b - __builtin_bit_cast(float, packed & 0xffff0000u));
    }
};
struct Fp16 {
    // 2^8 times this stays below the largest value, and 2^-32 of the greatest weight is what gets lost, in place of
    // 2^-25: behind a token that takes nearly all, 20,000 others may share 1/2,000
    static constexpr float kLift = 7.f;
    typedef _Float16 x8 __attribute__((ext_vector_type(8)));
    static __device__ f32x16 mma32(s16x8 a, s16x8 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
    }
    static __device__ f32x4 mma16(s16x8 a, s16x8 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
    }
    static __device__ uint32_t pack(float a, float b) {
        return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), f16x2));
    }
    static __device__ uint32_t pack_rest(float a, float b, uint32_t packed) {
        const f16x2 p = __builtin_bit_cast(f16x2, packed);
        return pack(a - (float)p[0], b - (float)p[1]);
    }
};

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kNegInf = -__builtin_inff();

using as3 = __attribute__((address_space(3))) void;

// 16 bytes a lane from memory to LDS, at l + 16 lane, waited for by hand: the
// compiler, told that LDS is written, would wait for all loads in flight
// before the next read of any LDS.  There is no output register to be
// overwritten.
__device__ __forceinline__ void load_lds16(const void *g, const void *l) {
    const uint32_t to = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(const as3 *)l);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(g) : "memory", "m0");
}
__device__ __forceinline__ void load_lds16(const void *base, uint32_t offset, const void *l) {
    const uint32_t to = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(const as3 *)l);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(base)
                 : "memory", "m0");
}
__device__ __forceinline__ s16x4 read_tr(const uint16_t *l) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)l);
}
__device__ __forceinline__ s16x8 join(s16x4 a, s16x4 b) {
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_of(float x) { return __builtin_amdgcn_logf(x); }

// The running maximum follows the scores only where they pass it by this much
// (in powers of two): weights up to 2^8 lose nothing in any of the types (see
// kLift), and most tiles are spared the scaling of O.
constexpr float kSlack = 8.f;

// Every load of the wave has landed in LDS.
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// ------------------------------------------------------------------ plan

constexpr int kPlanGroups = 16;

// A group's shared tokens are read for all its members at once where the row
// tiles that this saves, times the tokens, outweigh what it costs: the joint
// tiles' partial results, and the members' own ones, which without it go straight
// to the output, written and joined.  32 heads on 8 of K and V, together / each by
// itself: eight requests behind 3,300 shared tokens with 900 new tokens each 433 /
// 409 us, 100: 63 / 67, behind 2,100 with 17: 21 / 24; decoding, 64 requests behind 930
// tokens 21 / 30, 512 behind 48 tokens 64 / 58, behind 128 68 / 71, in groups of eight
// behind up to 240 77 / 81, behind up to 480 88 / 116 (99 by this rule), pairs behind
// up to 1,900 88 / 108 (99 by this rule).
constexpr int64_t kShareCost = 16 * kTileKv, kSplitCost = 4 * kTileKv;

// A segment as the plan holds it: segment i < n_req is the own tokens of the
// request at place i of the order, segment n_req + g group g's shared tokens.
struct Segment {
    int32_t t0, n_tok, kv0, kv1, seq, per, chunks, tiles, part;
    int32_t first;      // its first item on the wide list, or -1 - that on the narrow one
};

constexpr int kSmallGroup = 16;      // requests of a group that one thread goes through

// LDS of the plan, bytes: the arrays that attn_plan declares, and those sized by the batch.
template <int NT>
constexpr size_t kPlanLds = NT * (sizeof(Segment) + 4) + NT / 64 * (3 * 4 + 2 * 8) + PC_MAX_BATCH / kSmallGroup * 4 +
                            PC_MAX_BATCH / 8 + 64;
constexpr size_t plan_lds_bytes(size_t n_req) { return 4 * (7 * n_req + 3); }
constexpr size_t kLdsUnasked = 64 * 1024, kLdsMost = 160 * 1024;     // without an attribute, and with it
static_assert(kPlanLds<256> + plan_lds_bytes(256) <= kLdsUnasked, "a few requests");
static_assert(kPlanLds<1024> + plan_lds_bytes(PC_MAX_BATCH) <= kLdsMost, "the largest batch (161,804 bytes)");

// The last i of n with at[i] <= x, where at[0] <= x.
__device__ __forceinline__ int last_at(const int32_t *at, int n, int x) {
    int lo = 0;
    for (int step = 1 << (31 - __clz(n)); step; step >>= 1)
        if (lo + step < n && at[lo + step] <= x) lo += step;
    return lo;
}

// x / d by a 32-bit float where that is exact but for one (x below 2^22).
__device__ __forceinline__ uint32_t divide(uint32_t x, uint32_t d) {
    if (x >= 1u << 22) return x / d;
    uint32_t q = (uint32_t)((float)x * __builtin_amdgcn_rcpf((float)d));
    const int32_t r = (int32_t)(x - q * d);
    return r < 0 ? q - 1 : r >= (int32_t)d ? q + 1 : q;
}

// Makes the list of items.  It is bound by latency: a request's length is two
// dependent reads away, and what comes after is kept in LDS, where each query
// and each item finds its request or segment by a binary search.  Every
// workgroup works all segments out by itself and writes its share of the
// queries and items; the first one writes the rest.  128 requests with 3,000
// items took 20 us by one workgroup, most of it to write items; by 16 they take
// 11, one of them to see whether a tile's weights go in two pieces.
template <int NT>
__global__ __launch_bounds__(NT) void attn_plan(AttnPlanArgs a) {
    const pc_pages &p = a.p;
    const AttnWs &ws = a.ws;
    const int R = a.n_req, G = a.n_heads / p.n_kv_heads, Hk = p.n_kv_heads;
    extern __shared__ int32_t plan_lds[];
    int32_t *t0 = plan_lds;             // [R + 1] first query, in the order
    int32_t *goff = t0 + R + 1;         // [R + 1] group_off
    int32_t *q_off = goff + R + 1;      // [R + 1] of the requests, as their lengths and sequences:
    int32_t *len = q_off + R + 1;       // [R]
    int32_t *seq = len + R;             // [R]
    int32_t *place = seq + R;           // [R] the request at a place | its group (or kNoGroup) << 16
    int32_t *share = place + R;         // [R] blocks of the group, then tokens
    constexpr int kNoGroup = 0x7fff;
    static_assert(PC_MAX_BATCH < kNoGroup, "request and group in one word");
    __shared__ Segment seg[NT];
    __shared__ int32_t first_item[NT];
    __shared__ int32_t lds[3 * (NT / 64)];
    __shared__ int64_t lds64[2 * (NT / 64)];
    __shared__ int large[PC_MAX_BATCH / kSmallGroup];
    __shared__ int any_bad, stop, n_large;
    __shared__ uint32_t seen[PC_MAX_BATCH / 32];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const bool grouped = a.order != nullptr, first = blockIdx.x == 0;
    const int wg_tid = blockIdx.x * NT + tid, wg_step = gridDim.x * NT;     // of what the workgroups share
    if (tid < PC_MAX_BATCH / 32) seen[tid] = 0;
    if (tid == 0) any_bad = n_large = 0;
    if (first && tid < 64) reinterpret_cast<int32_t *>(ws.head)[tid] = 0;
    __syncthreads();
    // all that the caller gives, at once
    const int status = __hip_atomic_load(a.status, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const int n_groups = grouped ? *a.n_groups : 0;
    bool bad = n_groups < 0 || n_groups > R;
    for (int i = tid; i <= R; i += NT) {
        q_off[i] = a.q_off[i];
        goff[i] = grouped ? a.group_off[i] : 0;
        if (i == R) break;
        const uint32_t s = a.seq[i], r = grouped ? (uint32_t)a.order[i] : (uint32_t)i;
        share[i] = grouped ? a.shared[i] : 0;
        seq[i] = s;
        const int l = s < (uint32_t)p.n_seqs ? p.d_len[s] : -1;
        len[i] = l;
        bad |= l < 0 || (int64_t)l > (int64_t)p.table_width * kBlk;
        bad |= r >= (uint32_t)R || (atomicOr(&seen[r >> 5], 1u << (r & 31)) >> (r & 31) & 1);
        place[i] = (r < (uint32_t)R ? r : 0) | kNoGroup << 16;
    }
    // Only the first workgroup, which says in the end that there is a plan, goes by the status: another call may set
    // it meanwhile, and either all of the plan is there or nobody follows it.
    if (tid == 0) stop = first && status != PC_OK;
    __syncthreads();
    if (stop) return;
    // every request once, and their queries one behind the other: every query in one of them
    for (int i = tid; i < R; i += NT) bad |= q_off[i + 1] < q_off[i];
    bad |= q_off[0] != 0 || q_off[R] != a.n_tokens;
    for (int g = tid; g < n_groups && g < R; g += NT)
        bad |= goff[g] < 0 || goff[g + 1] < goff[g] || goff[g + 1] > R || (g == 0 && goff[0] != 0) ||
               (g == n_groups - 1 && goff[g + 1] != R);
    if (bad) any_bad = 1;
    __syncthreads();
    if (any_bad) {
        if (tid == 0) *a.status = PC_EINVAL;
        return;
    }
    auto request = [&](int j) { return place[j] & 0xffff; };
    auto group = [&](int j) { return place[j] >> 16; };
    int before = 0;
    for (int j0 = 0; j0 < R; j0 += NT) {
        const int j = j0 + tid;
        int n[1] = {0}, all[1];
        if (j < R) n[0] = q_off[request(j) + 1] - q_off[request(j)];
        block_scan<NT>(n, all, lds);
        if (j < R) t0[j] = before + n[0];
        before += all[0];
    }
    if (tid == 0) t0[R] = before;
    __syncthreads();
    // the tokens that all members of a group share: by a thread for small groups, a wave for others
    auto tiles_of = [&](int j) { return ((int64_t)(t0[j + 1] - t0[j]) * G + kWideRows - 1) / kWideRows; };
    auto shared_tokens = [&](int g, int least, int64_t separate) {
        const int64_t blocks = share[g], most = least / kBlk * kBlk;
        const int64_t tokens = blocks <= 0 ? 0 : min(most, blocks * kBlk);
        const int64_t joint = ((int64_t)(t0[goff[g + 1]] - t0[goff[g]]) * G + kWideRows - 1) / kWideRows;
        return (separate - joint) * tokens > kShareCost * joint + kSplitCost * separate ? (int)tokens : 0;
    };
    for (int g = tid; g < n_groups; g += NT) {
        const int j0 = goff[g], j1 = goff[g + 1];
        if (j1 - j0 > kSmallGroup) {
            large[atomicAdd(&n_large, 1)] = g;
            continue;
        }
        int least = 0x7fffffff;
        int64_t separate = 0;
        for (int j = j0; j < j1; ++j) {
            least = min(least, len[request(j)]);
            separate += tiles_of(j);
        }
        const int tokens = j1 - j0 < 2 ? 0 : shared_tokens(g, least, separate);
        if (tokens)
            for (int j = j0; j < j1; ++j) place[j] = request(j) | g << 16;
        share[g] = tokens;
    }
    __syncthreads();
    for (int i = wave; i < n_large; i += NT / 64) {
        const int g = large[i], j0 = goff[g], j1 = goff[g + 1];
        int least = 0x7fffffff;
        int64_t separate = 0;
        for (int j = j0 + lane; j < j1; j += 64) {
            least = min(least, len[request(j)]);
            separate += tiles_of(j);
        }
        separate = wave_last(wave_scan(separate));
#pragma unroll
        for (int d = 32; d; d >>= 1) least = min(least, __shfl_xor(least, d));
        const int tokens = shared_tokens(g, least, separate);
        if (tokens)
            for (int j = j0 + lane; j < j1; j += 64) place[j] = request(j) | g << 16;
        if (lane == 0) share[g] = tokens;
    }
    __syncthreads();
    // blocks of work on each list, and from them how long an item may be
    const int n_seg = R + n_groups;
    auto segment = [&](int i) {     // groups before the requests' own tokens: theirs are the longest items
        Segment x{};
        if (i < n_groups) {
            const int j0 = goff[i], j1 = goff[i + 1];
            if (share[i]) x = Segment{t0[j0], t0[j1] - t0[j0], 0, share[i], seq[request(j0)], 0, 0, 0, 0, 0};
        } else if (i < n_seg) {
            const int j = i - n_groups;
            const int r = request(j), g = group(j);
            x = Segment{t0[j], t0[j + 1] - t0[j], g == kNoGroup ? 0 : share[g], len[r], seq[r], 0, 0, 0, 0, 0};
        }
        return x;
    };
    int64_t work[2] = {0, 0}, all_work[2];      // wide, narrow
    for (int i = tid; i < n_seg; i += NT) {
        const Segment x = segment(i);
        const int64_t rows = (int64_t)x.n_tok * G, blocks = (x.kv1 - x.kv0 + kTileKv - 1) / kTileKv;
        if (rows > kNarrowRows) work[0] += (rows + kWideRows - 1) / kWideRows * blocks;
        else if (rows) work[1] += blocks;
    }
    block_scan<NT>(work, all_work, lds64);
    const int64_t by_wide = (all_work[0] * Hk + kWideItems - 1) / kWideItems,
                  by_narrow = (all_work[1] * Hk + kNarrowItems - 1) / kNarrowItems;
    // no more than the longest sequence has, for the 64-bit sums of many of these
    constexpr int64_t kMostBlocks = (1LL << 24) * kBlk / kTileKv;
    const int len_wide = (int)min(max(by_wide, (int64_t)kWideMinBlocks), kMostBlocks);
    const int len_narrow = (int)min(max(by_narrow, (int64_t)kNarrowMinBlocks), kMostBlocks);
    int n_wide = 0, n_narrow = 0, rows_at = 0;
    for (int i0 = 0; i0 < n_seg; i0 += NT) {
        const int i = i0 + tid;
        Segment x = segment(i);
        int chunks = 0;
        bool direct = false;
        const int64_t rows = (int64_t)x.n_tok * G;
        const int blocks = (x.kv1 - x.kv0 + kTileKv - 1) / kTileKv;
        const bool is_wide = rows > kNarrowRows;
        if (rows && blocks) {
            x.tiles = (int)((rows + kWideRows - 1) / kWideRows);
            const int most = is_wide ? len_wide : len_narrow;
            chunks = (blocks + most - 1) / most;
            const int per = (blocks + chunks - 1) / chunks;
            chunks = (blocks + per - 1) / per;
            x.per = per * kTileKv;
            x.chunks = chunks;
            direct = i >= n_groups && chunks == 1 && group(i - n_groups) == kNoGroup;
        }
        const int items = chunks * x.tiles * Hk;
        // items of this pass, the wide ones among them, partial rows
        int at[3] = {items, is_wide ? items : 0, direct ? 0 : chunks * x.n_tok * a.n_heads}, all[3];
        block_scan<NT>(at, all, lds);
        x.first = is_wide ? n_wide + at[1] : -1 - (n_narrow + at[0] - at[1]);
        x.part = direct ? -1 : rows_at + at[2];
        seg[tid] = x;
        first_item[tid] = at[0];
        // by every workgroup, for itself
        if (i < n_seg) ws.parts[i < n_groups ? R + i : i - n_groups] = AttnParts{x.part, direct ? -1 : chunks};
        __syncthreads();
        const int n_items = all[0], n_here = min(n_seg - i0, NT);
        // segments of long items first, so that short ones end the list (32 prompts of 300 tokens behind 3,000:
        // 245 us in place of 277); where each workgroup has at most one, and there are no others, the second
        // half of the workgroups, on the same CUs as the first, the other way round (one prompt of 2,000: 60 in
        // place of 63, eight of 900 behind 4,096 145 in place of 150)
        const bool pairs = n_seg <= NT && all[1] == all[0] && all[1] > kWideSlots / 2 && all[1] <= kWideSlots;
        if (pairs || all[1] > kWideSlots) {
            int before = n_wide;
            for (int k = 0; k < n_here; ++k) {
                const Segment &y = seg[k];
                if (y.first >= 0 && (y.per > x.per || (y.per == x.per && k < tid))) before += y.chunks * y.tiles * Hk;
            }
            __syncthreads();
            if (x.first >= 0) seg[tid].first = before;
            __syncthreads();
        }
        for (int u = wg_tid; u < n_items; u += wg_step) {
            const int k = last_at(first_item, n_here, u);
            const Segment y = seg[k];
            // the last tiles, which see most, first; then chunks, then heads
            const uint32_t off = u - first_item[k], rest = divide(off, Hk), head = off - rest * Hk;
            const uint32_t back = divide(rest, y.chunks), c = rest - back * y.chunks, tile = y.tiles - 1 - back;
            const int b = y.kv0 + (int)c * y.per;
            int to = (y.first >= 0 ? y.first : -1 - y.first) + (int)off;
            if (pairs) {
                const int half = kWideSlots / 2 / kXcds, turn = to / kXcds, turns = all[1] / kXcds;
                if (turn >= half && turn < turns) to += (half + turns - 1 - 2 * turn) * kXcds;
            }
            // a wide tile with a row of a request that would be narrow by itself; only shared tokens have such tiles,
            // and one without has fewer than ten requests
            int exact = 0;
            if (y.first >= 0 && i0 + k < n_groups) {
                const int t_first = y.t0 + (int)divide(tile * kWideRows, G),
                          t_last = y.t0 + min(y.n_tok - 1, (int)divide(tile * kWideRows + kWideRows - 1, G));
                for (int j = last_at(t0, R, t_first); !exact && j < R && t0[j] <= t_last; ++j)
                    exact = t0[j + 1] > t0[j] && (t0[j + 1] - t0[j]) <= kNarrowRows / G;
            }
            (y.first >= 0 ? ws.wide : ws.narrow)[to] =
                AttnItem{y.t0, y.n_tok, b, min(b + y.per, y.kv1), y.seq, (int32_t)(head | tile << 8),
                         y.part < 0 ? -1 : y.part + (int)c * y.n_tok * a.n_heads, exact};
        }
        n_wide += all[1];
        n_narrow += all[0] - all[1];
        rows_at += all[2];
        __syncthreads();
    }
    // the queries in the order, and where their partial results are
    for (int t = wg_tid; t < (int)a.n_tokens; t += wg_step) {
        const int j = last_at(t0, R, t), r = request(j), g = group(j), n = t0[j + 1] - t0[j];
        const AttnParts own = ws.parts[j], grp = g == kNoGroup ? AttnParts{0, 0} : ws.parts[R + g];
        const int g0 = g == kNoGroup ? t : t0[goff[g]], gn = g == kNoGroup ? 0 : t0[goff[g + 1]] - g0;
        const int q_row = q_off[r] + t - t0[j];
        ws.tok[t] = q_row;
        ws.lim[t] = a.causal ? len[r] - n + t - t0[j] + 1 : len[r];
        ws.row[t] = AttnRow{q_row, own.chunks, own.base + (t - t0[j]) * a.n_heads, n * a.n_heads,
                            grp.chunks, grp.base + (t - g0) * a.n_heads, gn * a.n_heads, 0};
    }
    if (!first) return;
    if (tid < kXcds) ws.next[tid * kNextStep] = 0;
    if (tid == 0)
        *ws.head = AttnHead{kPlanned, n_wide, n_narrow, R, (int32_t)a.n_tokens, a.n_heads, Hk, p.head_dim, p.n_seqs, p.table_width};
}

// A plan of this batch and pool is in the workspace: its lists, which say
// where to read and write, are not looked at otherwise.
__device__ __forceinline__ bool planned(const AttnArgs &a) {
    const AttnHead h = *a.ws.head;
    return h.magic == kPlanned && h.n_req == a.n_req && h.n_tokens == a.n_tokens && h.n_heads == a.n_heads &&
           h.n_kv_heads * a.group == a.n_heads && h.head_dim == a.head_dim && h.n_seqs == a.n_seqs &&
           h.table_width == a.table_width;
}

// ------------------------------------------------------------------ wide items

// Where 16-byte piece c of token t's row lies in LDS: at c ^ swap.  A row is 256
// or 128 bytes of the banks' 256.  K is read by 16 lanes at a time, the same
// piece of 16 tokens; V by 32 lanes of 8 bytes, which take 32 bytes each of four
// tokens and two neighbouring columns (wide) or of eight tokens (narrow): these
// permutations send each of them to other banks.
template <int D>
__device__ __forceinline__ int swap_k(int t) { return D == 128 ? t & 15 : t >> 1 & 7; }
template <int D>
__device__ __forceinline__ int swap_v(int t) { return D == 128 ? 4 * (t & 3) : 2 * (t & 2); }
template <int D>
__device__ __forceinline__ int swap_v_narrow(int t) { return D == 128 ? 2 * (t & 7) : t & 6; }

// A workgroup of four waves takes 128 rows, a wave 32 of them (the columns of
// 32 x 32 x 16 products), and 64 tokens of K and V at a time from LDS, where a
// second pair of buffers fills meanwhile.  16-byte pieces of a token's row are
// permuted in LDS (see swap_k and swap_v).  Prompts of 900 tokens behind 4,096
// cached ones run at 790 TFLOP/s, without the plan and the join (a library's
// product of 8192^3, which the chip's power bounds too: 1,206 to 1,380).  The
// matrix units are busy 38 % of the time and the vector units about as long; the products left out, the same prompts take 87
// us in place of 140, and no single part of the weights' work more than 12 us
// (the exponentials).  What did not help: eight waves in two teams that barriers
// kept half a tile apart (12 % longer), a wave that weighed one half of a tile
// between the products of the others (1 % longer), tiles of 32 tokens (6 %),
// wave priorities (the same).  Products of four independent sums in turn, their
// reads issued four products ahead, save 2 %.
//
// kWeights: in how many pieces the weights go into the second product.  One, rounded to the type of K and V, for
// prompts, two, exact to twice its bits, where a row is of a request with few (a token that decodes has the same
// precision whoever shares its prefix).  Two everywhere would take eight prompts of 900 behind 4,096 from 137 to 177 us
// and one of 8,192 from 281 to 362, for errors of 1.7e-3 in place of 2.3e-3 (bf16, whose results round by 1.7e-3);
// where the rows decode, reading the tokens hides them: 128 requests behind 8,192 tokens take 64.3 us in place of 62.2.
template <typename T, int D, int kWeights>
__device__ __forceinline__ void wide_item(const AttnArgs &a, const AttnItem it, uint16_t *lds, int *lds_lim, int *queue,
                                          int &next) {
    constexpr int kPieces = D / 8, kSteps = D / 16, kDb = D / 32, kBuf = kTileKv * D;   // K, K, V, V
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, half = lane >> 5;
    const uint16_t *zeros = reinterpret_cast<const uint16_t *>(reinterpret_cast<const char *>(a.ws.head) + kZeroOffset);
    const uint16_t *kp = static_cast<const uint16_t *>(a.k), *vp = static_cast<const uint16_t *>(a.v);
    const int head = it.head_tile & 255, tile = it.head_tile >> 8;
    const int row = tile * kWideRows + wave * 32 + col;
    const int tok = row / a.group, hq = head * a.group + row - tok * a.group;
    const bool active = tok < it.n_tok;
    const int lim = active ? min(a.ws.lim[it.t0 + tok], it.kv1) : 0;
    const int64_t q_row = active ? a.ws.tok[it.t0 + tok] : 0;
    s16x8 qf[kSteps];
    {
        const uint16_t *q = static_cast<const uint16_t *>(a.q) + q_row * a.q_token + hq * a.q_head + half * 8;
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
            qf[s] = active ? *reinterpret_cast<const s16x8 *>(q + 16 * s) : s16x8{0, 0, 0, 0, 0, 0, 0, 0};
    }
    int most = lim, least = lim;
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        most = max(most, __shfl_xor(most, d));
        least = min(least, __shfl_xor(least, d));
    }
    least = __builtin_amdgcn_readfirstlane(least);
    __syncthreads();        // the last item's readers of LDS
    if (lane == 0) lds_lim[wave] = most;
    __syncthreads();
    const int end = __builtin_amdgcn_readfirstlane(max(max(lds_lim[0], lds_lim[1]), max(lds_lim[2], lds_lim[3])));
    const int tiles = end > it.kv0 ? (end - it.kv0 + kTileKv - 1) / kTileKv : 0;
    const int32_t *table = a.table + (int64_t)it.seq * a.table_width;

    // a wave loads one page of each tile: 16 tokens.  The page's number is
    // read a tile ahead, so that it is there when its loads are issued.
    // (none: a zero that the compiler takes for a lane's own, or it would wait for the number
    // at once to have it in a scalar register)
    int none;
    asm volatile("v_mov_b32 %0, 0" : "=v"(none));
    auto page_of = [&](int n) { return table[min(it.kv0 + n * kTileKv + wave * kBlk, end - 1) / kBlk + none]; };
    uint32_t k_at[kPieces / 4], v_at[kPieces / 4];      // bytes of this lane's pieces in a page
#pragma unroll
    for (int i = 0; i < kPieces / 4; ++i) {
        const int u = i * 64 + lane, t = u / kPieces, c = u % kPieces;
        k_at[i] = 2 * (t * a.token_stride + (c ^ swap_k<D>(t)) * 8);
        v_at[i] = 2 * (t * a.token_stride + (c ^ swap_v<D>(t)) * 8);
    }
    auto fetch = [&](int n, int buf, int number) {
        const uint32_t page = min((uint32_t)__builtin_amdgcn_readfirstlane(number), (uint32_t)(a.n_pages - 1));
        const int t_first = it.kv0 + n * kTileKv + wave * kBlk;
        const int64_t from = (int64_t)page * a.page_stride + (int64_t)head * a.head_stride;
        const uint16_t *lk = lds + buf * kBuf + wave * kBlk * D, *lv = lk + 2 * kBuf;
#pragma unroll
        for (int i = 0; i < kPieces / 4; ++i) load_lds16(kp + from, k_at[i], lk + i * 512);
        if (t_first + kBlk <= end) {
#pragma unroll
            for (int i = 0; i < kPieces / 4; ++i) load_lds16(vp + from, v_at[i], lv + i * 512);
        } else {    // behind the end there may be anything, and zero times anything is to be zero
#pragma unroll
            for (int i = 0; i < kPieces / 4; ++i) {
                const char *v = reinterpret_cast<const char *>(vp + from) + v_at[i];
                load_lds16(t_first + (i * 64 + lane) / kPieces < end ? v : reinterpret_cast<const char *>(zeros),
                                 lv + i * 512);
            }
        }
    };
    f32x16 o[kDb];
#pragma unroll
    for (int i = 0; i < kDb; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[i][r] = 0;
    float m = kNegInf, l = 0;
    int page = 0;
    if (tiles) {
        fetch(0, 0, page_of(0));
        page = page_of(1);
    }
    for (int n = 0; n < tiles; ++n) {
        wait_loads();
        __syncthreads();
        if (n + 1 < tiles) {
            fetch(n + 1, (n + 1) & 1, page);
            page = page_of(n + 2);
        }
        const uint16_t *lk = lds + (n & 1) * kBuf, *lv = lk + 2 * kBuf;
        f32x16 s[2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[h][r] = 0;
#pragma unroll
        for (int st = 0; st < kSteps; ++st)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int at = (h * 32 + col) * D + (((2 * st + half) ^ swap_k<D>(col)) * 8);
                s[h] = T::mma32(*reinterpret_cast<const s16x8 *>(lk + at), qf[st], s[h]);
            }
        const int base = it.kv0 + n * kTileKv;
        if (base + kTileKv > least) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (base + h * 32 + (r >> 2) * 8 + half * 4 + (r & 3) >= lim) s[h][r] = kNegInf;
        }
        float top = kNegInf;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[h][r]);
        top = fmaxf(top, __shfl_xor(top, 32)) * a.scale_log2;
        if (__any(top > m + kSlack)) {
            const float now = fmaxf(m, top), f = now == kNegInf ? 1.f : exp2_of(m - now);
            l *= f;
#pragma unroll
            for (int i = 0; i < kDb; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[i][r] *= f;
            m = now;
        }
        const float use = m == kNegInf ? 0.f : m - T::kLift;
        s16x8 pf[4], rest[4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[h][r] = exp2_of(fmaf(s[h][r], a.scale_log2, -use));
                l += s[h][r];
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                union { uint32_t u[4]; s16x8 v; } w;
#pragma unroll
                for (int y = 0; y < 4; ++y) w.u[y] = T::pack(s[h][8 * x + 2 * y], s[h][8 * x + 2 * y + 1]);
                pf[2 * h + x] = w.v;
                if (kWeights == 1) continue;
#pragma unroll
                for (int y = 0; y < 4; ++y)
                    w.u[y] = T::pack_rest(s[h][8 * x + 2 * y], s[h][8 * x + 2 * y + 1], w.u[y]);
                rest[2 * h + x] = w.v;
            }
        }
        const int quad = (lane >> 2) & 3, g16 = (lane >> 4) & 1;
        const int vt = 4 * half + quad;     // token of this lane's address, within eight
#pragma unroll
        for (int st = 0; st < 4; ++st)
#pragma unroll
            for (int i = 0; i < kDb; ++i) {
                const int piece = (4 * i + 2 * g16 + ((lane & 3) >> 1)) ^ swap_v<D>(vt);
                const uint16_t *v = lv + vt * D + piece * 8 + (lane & 1) * 4;
                const s16x8 v8 = join(read_tr(v + st * 16 * D), read_tr(v + (st * 16 + 8) * D));
                o[i] = T::mma32(v8, pf[st], o[i]);
                if (kWeights == 2) o[i] = T::mma32(v8, rest[st], o[i]);
            }
        // four products' reads ahead of the first one
        __builtin_amdgcn_sched_group_barrier(0x100, 8, 1);
#pragma unroll
        for (int i = 0; i < 4 * kDb - 4; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, kWeights, 1);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 1);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 4 * kWeights, 1);
    }
    // no sooner: who takes an item long before it can begin keeps it from others.  Looked at behind the stores.
    if (queue && threadIdx.x == 0) next = atomicAdd(queue, 1);
    l += __shfl_xor(l, 32);
    if (active) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const float lse = l == 0.f ? kNegInf : m - T::kLift + log2_of(l);
        if (it.part < 0) {
            uint16_t *to = static_cast<uint16_t *>(a.out) + q_row * a.out_token + hq * a.out_head + 4 * half;
#pragma unroll
            for (int i = 0; i < kDb; ++i)
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    *reinterpret_cast<uint2 *>(to + 32 * i + 8 * b) =
                        make_uint2(T::pack(o[i][4 * b] * inv, o[i][4 * b + 1] * inv),
                                   T::pack(o[i][4 * b + 2] * inv, o[i][4 * b + 3] * inv));
            if (a.lse_out && half == 0) a.lse_out[q_row * a.n_heads + hq] = lse * kLn2;
        } else {
            const int64_t at = it.part + (int64_t)tok * a.n_heads + hq;
            float *to = a.ws.o + at * D + 4 * half;
#pragma unroll
            for (int i = 0; i < kDb; ++i)
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    *reinterpret_cast<float4 *>(to + 32 * i + 8 * b) =
                        make_float4(o[i][4 * b] * inv, o[i][4 * b + 1] * inv, o[i][4 * b + 2] * inv, o[i][4 * b + 3] * inv);
            if (half == 0) a.ws.lse[at] = lse;
        }
    }
}

// ------------------------------------------------------------------ narrow items

// Up to 16 rows: a wave by itself, with 16 x 16 x 32 products and 32 tokens
// (two pages) at a time, bound by memory.  K and V of the next tokens are
// loaded to registers while the present ones are weighed and multiplied; V
// goes on through a piece of LDS of the wave's own, for the transposing read.
// Four decoding requests of 60,000 tokens: 4.7 TB/s with the join (a copy:
// 5.2).  64 tokens at a time by loads straight to LDS: 3 % longer.
template <typename T, int D>
__device__ __forceinline__ void narrow_item(const AttnArgs &a, const AttnItem it, uint16_t *lv) {
    constexpr int kPieces = D / 8, kSteps = D / 32, kDb = D / 16, kStep = 32, kPages = kStep / kBlk;
    const int lane = threadIdx.x & 63;
    const int col = lane & 15, quarter = lane >> 4;
    const int head = it.head_tile & 255, end = it.kv1;
    const uint16_t *kp = static_cast<const uint16_t *>(a.k) + (int64_t)head * a.head_stride;
    const uint16_t *vp = static_cast<const uint16_t *>(a.v) + (int64_t)head * a.head_stride;
    const int32_t *table = a.table + (int64_t)it.seq * a.table_width;
    int none;       // see wide_item
    asm volatile("v_mov_b32 %0, 0" : "=v"(none));
    int number[kPages];
    auto look_up = [&](int base) {
#pragma unroll
        for (int h = 0; h < kPages; ++h) number[h] = table[min(base + h * kBlk, end - 1) / kBlk + none];
    };
    const int k_at = col * a.token_stride + quarter * 8, v_at = lane / kPieces * a.token_stride + lane % kPieces * 8,
              v_step = 64 / kPieces * a.token_stride;
    s16x8 kf[kPages][kSteps], vf[kPages][kSteps];
    auto load = [&](int base) {
#pragma unroll
        for (int h = 0; h < kPages; ++h) {
            const uint32_t page = min((uint32_t)__builtin_amdgcn_readfirstlane(number[h]), (uint32_t)(a.n_pages - 1));
            const uint16_t *k = kp + (int64_t)page * a.page_stride, *v = vp + (int64_t)page * a.page_stride;
#pragma unroll
            for (int st = 0; st < kSteps; ++st) kf[h][st] = *reinterpret_cast<const s16x8 *>(k + k_at + 32 * st);
#pragma unroll
            for (int st = 0; st < kSteps; ++st) vf[h][st] = *reinterpret_cast<const s16x8 *>(v + v_at + st * v_step);
        }
        if (base + kStep < end) look_up(base + kStep);
    };
    look_up(it.kv0);
    load(it.kv0);
    const int tok = col / a.group, hq = head * a.group + col - tok * a.group;
    const bool active = tok < it.n_tok;
    // a row behind the last reads the last query, and sees nothing
    const int at_tok = it.t0 + min(tok, it.n_tok - 1);
    const int lim = active ? min(a.ws.lim[at_tok], it.kv1) : 0;
    const int64_t q_row = a.ws.tok[at_tok];
    s16x8 qf[kSteps];
    {
        const uint16_t *q = static_cast<const uint16_t *>(a.q) + q_row * a.q_token + hq * a.q_head + quarter * 8;
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
            qf[s] = *reinterpret_cast<const s16x8 *>(q + 32 * s);
    }
    f32x4 o[kDb];
#pragma unroll
    for (int i = 0; i < kDb; ++i) o[i] = f32x4{0, 0, 0, 0};
    float m = kNegInf, l = 0;
    for (int base = it.kv0; base < end; base += kStep) {
        // V to LDS, a token's pieces permuted as in wide_item.  A wave's LDS operations stay in order, so
        // the last tokens' reads are done.  Behind the end there may be anything, and zero times anything
        // is to be zero.
        const bool whole = base + kStep <= end;
#pragma unroll
        for (int h = 0; h < kPages; ++h)
#pragma unroll
            for (int st = 0; st < kSteps; ++st) {
                const int u = st * 64 + lane, t = u / kPieces, c = u % kPieces;
                s16x8 v = vf[h][st];
                if (!whole && base + h * kBlk + t >= end) v = s16x8{0, 0, 0, 0, 0, 0, 0, 0};
                *reinterpret_cast<s16x8 *>(lv + (h * kBlk + t) * D + (c ^ swap_v_narrow<D>(t)) * 8) = v;
            }
        f32x4 s[kPages];
#pragma unroll
        for (int h = 0; h < kPages; ++h) {
            s[h] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int st = 0; st < kSteps; ++st) s[h] = T::mma16(kf[h][st], qf[st], s[h]);
        }
        if (base + kStep < end) load(base + kStep);
        float top = kNegInf;
#pragma unroll
        for (int h = 0; h < kPages; ++h)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (base + h * kBlk + quarter * 4 + r >= lim) s[h][r] = kNegInf;
                top = fmaxf(top, s[h][r]);
            }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32)) * a.scale_log2;
        if (__any(top > m + kSlack)) {
            const float now = fmaxf(m, top), f = now == kNegInf ? 1.f : exp2_of(m - now);
            l *= f;
#pragma unroll
            for (int i = 0; i < kDb; ++i) o[i] *= f;
            m = now;
        }
        const float use = m == kNegInf ? 0.f : m - T::kLift;
        union { uint32_t u[2 * kPages]; s16x8 v[kPages / 2]; } w, rest;
#pragma unroll
        for (int h = 0; h < kPages; ++h) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s[h][r] = exp2_of(fmaf(s[h][r], a.scale_log2, -use));
                l += s[h][r];
            }
            w.u[2 * h] = T::pack(s[h][0], s[h][1]);
            w.u[2 * h + 1] = T::pack(s[h][2], s[h][3]);
            // here the matrix units wait for memory: the weights go in two pieces, so that they are exact to
            // twice the type's bits
            rest.u[2 * h] = T::pack_rest(s[h][0], s[h][1], w.u[2 * h]);
            rest.u[2 * h + 1] = T::pack_rest(s[h][2], s[h][3], w.u[2 * h + 1]);
        }
        const int vt = 4 * quarter + ((lane >> 2) & 3);     // token of this lane's address, within a page
#pragma unroll
        for (int i = 0; i < kDb; ++i) {
            const int piece = (2 * i + ((lane & 3) >> 1)) ^ swap_v_narrow<D>(vt);
            const uint16_t *v = lv + vt * D + piece * 8 + (lane & 1) * 4;
#pragma unroll
            for (int h = 0; h < kPages; h += 2) {
                const s16x8 vt8 = join(read_tr(v + h * kBlk * D), read_tr(v + (h + 1) * kBlk * D));
                o[i] = T::mma16(vt8, w.v[h / 2], o[i]);
                o[i] = T::mma16(vt8, rest.v[h / 2], o[i]);
            }
        }
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (active) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const float lse = l == 0.f ? kNegInf : m - T::kLift + log2_of(l);
        if (it.part < 0) {
            uint16_t *to = static_cast<uint16_t *>(a.out) + q_row * a.out_token + hq * a.out_head + 4 * quarter;
#pragma unroll
            for (int i = 0; i < kDb; ++i)
                *reinterpret_cast<uint2 *>(to + 16 * i) = make_uint2(T::pack(o[i][0] * inv, o[i][1] * inv),
                                                                     T::pack(o[i][2] * inv, o[i][3] * inv));
            if (a.lse_out && quarter == 0) a.lse_out[q_row * a.n_heads + hq] = lse * kLn2;
        } else {
            const int64_t at = it.part + (int64_t)tok * a.n_heads + hq;
            float *to = a.ws.o + at * D + 4 * quarter;
#pragma unroll
            for (int i = 0; i < kDb; ++i)
                *reinterpret_cast<float4 *>(to + 16 * i) =
                    make_float4(o[i][0] * inv, o[i][1] * inv, o[i][2] * inv, o[i][3] * inv);
            if (quarter == 0) a.ws.lse[at] = lse;
        }
    }
}

// ------------------------------------------------------------------ items

// Wide items are bound by the matrix units and LDS, narrow ones by memory: of
// the two workgroups on a CU one begins with the wide list and one with the
// narrow one, so that both kinds run side by side.
//
// Wide items differ in length, as queries see only what precedes them, so a
// workgroup takes its next one when it is done with the last: from a counter for
// each XCD, which has an L2 of its own and takes every eighth item (workgroups go
// round the XCDs).  Heads are the fastest index of the list, so that an XCD's
// workgroups read the same heads' K and V, and it runs from long items to short
// ones.  One prompt of 8,192 tokens takes 528 us in place of 800 with turns fixed
// beforehand, one of 20,000 for 6 heads on one of K and V 570 us in place of 757,
// 32 of 300 behind 3,000 cached ones 240 in place of 275.  Where there are no more
// items than workgroups (with narrow ones beside them: than half of these), nothing is
// taken.  The join leaves the counters at 0.
template <typename T, int D>
__global__ __launch_bounds__(256, 2) void attn_items(AttnArgs a) {
    __shared__ __align__(1024) uint16_t lds[4 * kTileKv * D];
    __shared__ int lds_lim[4], lds_next;
    if (!planned(a)) return;
    const int n_wide = a.ws.head->n_wide, n_narrow = a.ws.head->n_narrow;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool wide_first = blockIdx.x < gridDim.x / 2;
    for (int phase = 0; phase < 2; ++phase) {
        if ((phase == 0) == wide_first) {
            const int xcd = blockIdx.x % kXcds, given = (n_narrow ? gridDim.x / 2 : gridDim.x) / kXcds;
            int *queue = given * kXcds < n_wide ? a.ws.next + xcd * kNextStep : nullptr;
            int turn = blockIdx.x / kXcds, next = 0;
            bool have = turn < given && turn * kXcds + xcd < n_wide;
            while (have || queue) {
                if (have) {
                    const AttnItem it = a.ws.wide[turn * kXcds + xcd];
                    if (it.exact) wide_item<T, D, 2>(a, it, lds, lds_lim, queue, next);
                    else wide_item<T, D, 1>(a, it, lds, lds_lim, queue, next);
                } else if (threadIdx.x == 0) next = atomicAdd(queue, 1);
                if (!queue) break;
                __syncthreads();
                if (threadIdx.x == 0) lds_next = given + next;
                __syncthreads();
                turn = __builtin_amdgcn_readfirstlane(lds_next);
                if (turn * kXcds + xcd >= n_wide) break;
                have = true;
            }
        } else {
            // a wave an item, those of the workgroups that begin here first
            const int half = gridDim.x / 2, first = wide_first ? 4 * half + (int)blockIdx.x : (int)blockIdx.x - half;
            for (int which = first + wave * half; which < n_narrow; which += gridDim.x * 4)
                narrow_item<T, D>(a, a.ws.narrow[which], lds + wave * kTileKv * D);
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------ join

// A wave for kHeads heads of a query.  A lane weighs one part of one head, 64 /
// kHeads parts at a time; the parts' values follow with 16 loads in flight, the
// last few parts' with fewer (up to 7 % of short attentions' time: most rows
// have two or three parts).
template <typename T, int D, int kHeads>
__global__ __launch_bounds__(256) void attn_join(AttnArgs a) {
    constexpr int kParts = 64 / kHeads, kFly = 16 / kHeads, kPer = D / 64, kTail = kFly < 8 ? 2 : 4;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int per_query = (a.n_heads + kHeads - 1) / kHeads;
    const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (block == 0 && threadIdx.x < kXcds && planned(a)) a.ws.next[threadIdx.x * kNextStep] = 0;
    const int64_t at = block * 4 + wave;
    const int64_t t = at / per_query;
    const int h0 = (int)(at - t * per_query) * kHeads;
    if (t >= a.n_tokens) return;
    const AttnRow x = a.ws.row[t];
    if (!planned(a)) return;
    if (x.own_chunks < 0) return;       // written already
    const int64_t q_row = x.q_row;
    const int n = x.own_chunks + x.grp_chunks, heads = min(a.n_heads - h0, kHeads);
    auto row = [&](int c) -> int64_t {      // of head h0
        return h0 + (c < x.grp_chunks ? x.grp_row + (int64_t)c * x.grp_step
                                      : x.own_row + (int64_t)(c - x.grp_chunks) * x.own_step);
    };
    const int my_head = lane / kParts, my_part = lane % kParts;
    float top = kNegInf, sum = 0, o[kHeads][kPer];
#pragma unroll
    for (int h = 0; h < kHeads; ++h)
#pragma unroll
        for (int e = 0; e < kPer; ++e) o[h][e] = 0;
    for (int c0 = 0; c0 < n; c0 += kParts) {
        const int c = c0 + my_part;
        const float lse = c < n && my_head < heads ? a.ws.lse[row(c) + my_head] : kNegInf;
        float now = fmaxf(top, lse);
#pragma unroll
        for (int d = kParts / 2; d; d >>= 1) now = fmaxf(now, __shfl_xor(now, d));
        const float use = now == kNegInf ? 0.f : now;
        const float f = exp2_of(top - use), w = exp2_of(lse - use);
        float all = w;
#pragma unroll
        for (int d = kParts / 2; d; d >>= 1) all += __shfl_xor(all, d);
        sum = sum * f + all;
        top = now;
#pragma unroll
        for (int h = 0; h < kHeads; ++h) {
            const float fh = __shfl(f, h * kParts);
#pragma unroll
            for (int e = 0; e < kPer; ++e) o[h][e] *= fh;
        }
        const int m = min(n - c0, kParts);
        auto add = [&](auto count, int k0) {
            constexpr int kCount = decltype(count)::value;
            float x[kCount][kHeads][kPer];
#pragma unroll
            for (int k = 0; k < kCount; ++k) {
                const float *from = a.ws.o + row(c0 + min(k0 + k, m - 1)) * D + kPer * lane;
#pragma unroll
                for (int h = 0; h < kHeads; ++h)
#pragma unroll
                    for (int e = 0; e < kPer; ++e) x[k][h][e] = from[min(h, heads - 1) * D + e];
            }
#pragma unroll
            for (int k = 0; k < kCount; ++k)
#pragma unroll
                for (int h = 0; h < kHeads; ++h) {
                    // a part without tokens has no values, and the weight 0
                    const float wk = k0 + k < m ? __shfl(w, h * kParts + k0 + k) : 0.f;
#pragma unroll
                    for (int e = 0; e < kPer; ++e) o[h][e] += wk == 0.f ? 0.f : wk * x[k][h][e];
                }
        };
        int k0 = 0;
        for (; k0 + kFly <= m; k0 += kFly) add(std::integral_constant<int, kFly>(), k0);
        for (; k0 < m; k0 += kTail) add(std::integral_constant<int, kTail>(), k0);
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const float joined = sum == 0.f ? kNegInf : (top + log2_of(sum)) * kLn2;
#pragma unroll
    for (int h = 0; h < kHeads; ++h) {
        const float ih = __shfl(inv, h * kParts);
        if (h >= heads) continue;
        uint16_t *to = static_cast<uint16_t *>(a.out) + q_row * a.out_token + (h0 + h) * a.out_head;
        if (kPer == 2) *reinterpret_cast<uint32_t *>(to + 2 * lane) = T::pack(o[h][0] * ih, o[h][kPer - 1] * ih);
        else to[lane] = (uint16_t)T::pack(o[h][0] * ih, 0.f);
    }
    if (a.lse_out && my_part == 0 && my_head < heads) a.lse_out[q_row * a.n_heads + h0 + my_head] = joined;
}

template <typename T, int D>
hipError_t launch(const AttnArgs &a, hipStream_t st) {
    attn_items<T, D><<<kWideSlots, 256, 0, st>>>(a);     // two workgroups to a CU
    // A wave to a row for up to four a SIMD: those of few queries have many parts, and a wave by itself reads 16
    // at a time.  More rows have mostly two or three parts, and with four rows to a wave more loads in flight.
    // The whole attention by one / by four: 128 rows of four requests of 60,000 tokens 80 / 89 us, 2,700 rows 29 /
    // 31, 4,096 62.6 / 62.5, 9,400 34 / 32, 32,000 169 / 169.
    const int64_t rows = a.n_tokens * a.n_heads, waves = a.n_tokens * ((a.n_heads + 3) / 4);
    if (rows <= 4096) {
        attn_join<T, D, 1><<<(uint32_t)((rows + 3) / 4), 256, 0, st>>>(a);
    } else {    // a grid's row has less than 2^32 threads
        const int64_t blocks = (waves + 3) / 4, x = blocks < 1 << 20 ? blocks : 1 << 20;
        attn_join<T, D, 4><<<dim3((uint32_t)x, (uint32_t)((blocks + x - 1) / x)), 256, 0, st>>>(a);
    }
    return hipGetLastError();
}

int64_t up(int64_t v) { return (v + 255) / 256 * 256; }

}  // namespace

int64_t attn_ws(int32_t n_req, int64_t n_tokens, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, char *base,
                AttnWs *ws) {
    // Partial rows: one for every (query, head) of each of its two segments, and
    // for each item beyond a segment's first of a (tile, KV head) a tile's rows;
    // of those there are at most as many as the plan aims at.
    const int64_t rows = 2 * n_tokens * n_heads + (int64_t)kWideRows * kWideItems + (int64_t)kNarrowRows * kNarrowItems;
    const int64_t q_rows = n_tokens * (n_heads / n_kv_heads);
    const int64_t wide = n_kv_heads * (2 * (q_rows / kWideRows + 1) + 2LL * n_req) + kWideItems;
    const int64_t narrow = n_kv_heads * 2LL * n_req + kNarrowItems;
    if (rows > 0x7fffffff || wide > 0x7fffffff) return -1;
    int64_t o = 0;
    auto take = [&](int64_t bytes) { const int64_t at = o; o += up(bytes); return at; };
    static_assert(PC_ATTN_HEAD_BYTES == 256 && sizeof(AttnHead) <= kZeroOffset, "the head, and the zeros behind it");
    const int64_t head = take(PC_ATTN_HEAD_BYTES), next = take(4 * kXcds * kNextStep), tok = take(4 * n_tokens), lim = take(4 * n_tokens), row = take(n_tokens * (int64_t)sizeof(AttnRow)),
                  parts = take(2LL * n_req * (int64_t)sizeof(AttnParts)),
                  w = take(wide * (int64_t)sizeof(AttnItem)), nr = take(narrow * (int64_t)sizeof(AttnItem)),
                  po = take(rows * head_dim * 4), pl = take(rows * 4);
    if (ws) {
        ws->head = reinterpret_cast<AttnHead *>(base + head);
        ws->next = reinterpret_cast<int32_t *>(base + next);
        ws->tok = reinterpret_cast<int32_t *>(base + tok);
        ws->lim = reinterpret_cast<int32_t *>(base + lim);
        ws->row = reinterpret_cast<AttnRow *>(base + row);
        ws->parts = reinterpret_cast<AttnParts *>(base + parts);
        ws->wide = reinterpret_cast<AttnItem *>(base + w);
        ws->narrow = reinterpret_cast<AttnItem *>(base + nr);
        ws->o = reinterpret_cast<float *>(base + po);
        ws->lse = reinterpret_cast<float *>(base + pl);
    }
    return o;
}

hipError_t launch_attn_plan(const AttnPlanArgs &a, hipStream_t st) {
    const size_t bytes = plan_lds_bytes(a.n_req);
    // A barrier and a sum over 16 wavefronts cost more than what few requests have to do: with 256 / 1,024
    // threads, one request 6.1 / 7.9 us, 64 8.2 / 10.0 us, 256 10.8 / 11.1 us, 512 14.5 / 12.2 us.
    if (a.n_req <= 256) {
        attn_plan<256><<<kPlanGroups, 256, bytes, st>>>(a);
        return hipGetLastError();
    }
    if (kPlanLds<1024> + bytes > kLdsUnasked) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&attn_plan<1024>),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
        if (e != hipSuccess) return e;
    }
    attn_plan<1024><<<kPlanGroups, 1024, bytes, st>>>(a);
    return hipGetLastError();
}

hipError_t launch_attn(const AttnArgs &a, int32_t dtype, hipStream_t st) {
    if (dtype == PC_BF16) return a.head_dim == 128 ? launch<Bf16, 128>(a, st) : launch<Bf16, 64>(a, st);
    return a.head_dim == 128 ? launch<Fp16, 128>(a, st) : launch<Fp16, 64>(a, st);
}

}  // namespace pcr
