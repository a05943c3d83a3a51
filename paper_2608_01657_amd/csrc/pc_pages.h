// pc_pages.h -- shapes shared between the host checks (pc_pages_abi.cpp) and
// the kernels of the page operators (pc_pages.hip) and of the attention over
// shared prefixes (pc_attn.hip).  Not part of the public ABI.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pc.h"

namespace pcr {

constexpr int kBlk = PC_BLOCK_TOKENS;     // tokens of a page

// ---- page operators ------------------------------------------------------

// A bitmap of the pages that nobody holds, in chunks of one workgroup's work.
constexpr int kChunkPages = 4096;

// The workspace of pc_pages_extend and pc_pages_compact.
struct PagesWs {
    uint64_t *free_bits;    // [n_chunks][64]
    int32_t *chunk_free;    // [n_chunks] free pages of the chunk, then those before it
    int32_t *list;          // [n_pages] the free page of a rank
    int32_t *moved;         // [n_pages] compact: the page that moves to it
    int32_t *rank;          // [n_pages] compact: rank of a page that moves
    int32_t *entry;         // [4][n] extend: first new rank, pages held before, new pages, copied page or -1
    int32_t *head;          // [4] extend: new pages; compact: pages in use, pages that move; [3]: whether to act
    int32_t n_chunks;
};
int64_t pages_ws(const pc_pages &p, int64_t n_list, char *base, PagesWs *ws);

hipError_t launch_fork(const pc_pages &p, const int32_t *parent, const int32_t *child, int32_t n, int32_t *status,
                       hipStream_t st);
hipError_t launch_free(const pc_pages &p, const int32_t *seq, int32_t n, int32_t *status, hipStream_t st);
hipError_t launch_extend(const pc_pages &p, const int32_t *seq, const int32_t *add, int32_t n, const PagesWs &ws,
                         int32_t *status, hipStream_t st);
hipError_t launch_compact(const pc_pages &p, int32_t *refs_to, int32_t *table_to, int32_t *n_live, const PagesWs &ws,
                          int32_t *status, hipStream_t st);
hipError_t launch_write(const pc_pages &p, int32_t layer, const int32_t *seq, const int32_t *new_off, int32_t n,
                        int64_t n_tokens, const pc_rows &k_new, const pc_rows &v_new, int32_t *status, hipStream_t st);
hipError_t launch_groups(const uint64_t *keys, int64_t n_keys, const int64_t *key_off, int32_t n_req,
                         int32_t min_blocks, int32_t *order, int32_t *group_off, int32_t *shared, int32_t *n_groups,
                         int32_t *status, hipStream_t st);

// ---- attention -----------------------------------------------------------

constexpr int kTileKv = 64;          // tokens of K and V that a wide tile takes at a time
constexpr int kWideRows = 128;       // query rows of a wide tile
constexpr int kNarrowRows = 16;      // query rows of a narrow tile
// Items that the plan aims at where it splits a long axis, and the fewest
// 64-token blocks of an item that it splits down to.  More items fill the chip
// more evenly, fewer have less to write and to join: 128 requests behind 8,192
// shared tokens take 84 us with 512 and 2,048 (a workgroup and a wave for every
// place on the chip), 75 us with these; four of 60,000 tokens 112 and 104 us.
constexpr int kWideItems = 256, kNarrowItems = 1024;
constexpr int kWideMinBlocks = 4, kNarrowMinBlocks = 2;

// One piece of work: a tile of query rows of one KV head against a range of
// tokens of one sequence's pages.
struct AttnItem {
    int32_t t0, n_tok;      // the segment's queries, in group order
    int32_t kv0, kv1;       // tokens
    int32_t seq;            // whose table row holds the pages
    int32_t head_tile;      // KV head | tile << 8
    int32_t part;           // partial row of (first query, head 0); -1: straight to the output
    int32_t exact;          // whether its weights go in two pieces (wide ones; narrow ones always do)
};
// Where a segment's partial results are: their first row, and how many parts
// each query has (-1: they go straight to the output).
struct AttnParts {
    int32_t base, chunks;
};
// The same for a query: its own tokens' parts and its group's, of head 0, and
// the rows from a part to the next.
struct AttnRow {
    int32_t q_row, own_chunks, own_row, own_step, grp_chunks, grp_row, grp_step, pad;
};
// What the plan was made for, and the sizes of its lists.
struct AttnHead {
    int32_t magic, n_wide, n_narrow, n_req, n_tokens, n_heads, n_kv_heads, head_dim, n_seqs, table_width;
};
constexpr int32_t kPlanned = 0x70634174;
struct AttnWs {
    AttnHead *head;         // 256 bytes, with kZeroOffset bytes of zeros from there on
    int32_t *next;          // [kXcds][kNextStep]: the first of each, items of the wide list that this XCD has taken
    int32_t *tok;           // [n_tokens] query row of the query at this place of the order
    int32_t *lim;           // [n_tokens] it sees the tokens before this one
    AttnRow *row;           // [n_tokens]
    AttnParts *parts;       // [2][n_req]: of the requests at their places, of groups
    AttnItem *wide, *narrow;
    float *o;               // [rows][head_dim] partial results, normalised
    float *lse;             // [rows] log2 of their sums of exponentials
};
constexpr int kZeroOffset = 128;
constexpr int kWideSlots = 512;      // workgroups of the items' kernel, two to a CU
constexpr int kXcds = 8, kNextStep = 32;     // a cache line to a counter
// Bytes of the workspace (< 0: more than 2^31 - 1 partial rows).
int64_t attn_ws(int32_t n_req, int64_t n_tokens, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, char *base,
                AttnWs *ws);

struct AttnPlanArgs {
    pc_pages p;
    const int32_t *seq, *q_off, *order, *group_off, *shared, *n_groups;
    int32_t n_req, n_heads, causal;
    int64_t n_tokens;
    AttnWs ws;
    int32_t *status;
};
hipError_t launch_attn_plan(const AttnPlanArgs &a, hipStream_t st);

struct AttnArgs {
    const void *k, *v, *q;
    void *out;
    float *lse_out;
    const int32_t *table;
    int64_t page_stride, q_token, q_head, out_token, out_head;   // elements
    int32_t head_stride, token_stride;                           // of a page, elements
    int32_t table_width, n_pages, n_heads, group;                // group: query heads of a KV head
    int32_t n_req, n_seqs, head_dim;
    float scale_log2;
    int64_t n_tokens;
    AttnWs ws;
};
hipError_t launch_attn(const AttnArgs &a, int32_t dtype, hipStream_t st);

}  // namespace pcr
