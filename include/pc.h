/*
 * pc.h -- C ABI of the MI355X prefix-cache replay library (libpcreplay.so).
 *
 * The library runs the data-parallel hot path of PrefixShield (arXiv
 * 2608.01657): cutting token sequences into full 16-token KV blocks with
 * chained 64-bit block keys, and replaying many independent multi-tenant
 * prefix-cache instances (LRU, S3-FIFO, PrefixShield) over those keys, one
 * wavefront per instance on runs of blocks, or one workgroup of four where
 * an instance does not fit that form, with admission debt metered per
 * accounting group.  Beside them it has the pages of a real KV cache (forking,
 * growing, freeing, compacting, storing), the groups of a batch that its
 * block keys show to share a prefix, and attention that reads such a prefix
 * once for its group.
 *
 * Conventions (every entry point):
 *   - Pointers named d_* are DEVICE pointers owned by the caller; they must
 *     stay valid until the work queued on `stream` has completed.  The
 *     library never allocates device memory.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).
 *     All calls except pc_get_stats and pc_last_error are asynchronous.
 *   - Return value: PC_OK (0) or a negative PC_E* code; pc_last_error()
 *     then describes the failure.  Host-side validation happens before any
 *     device work is queued; a rejected call queues nothing.
 *   - Replay and keys are integer: keys are uint64, balances and debts are int64
 *     in Q16 fixed point (2^16 = one block).
 */
#ifndef PC_H
#define PC_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define PC_OK 0
#define PC_EINVAL (-1)        /* bad argument (null pointer, size, range, ...)        */
#define PC_ENOMEM (-2)        /* caller-provided workspace too small                  */
#define PC_EDEVICE (-3)       /* HIP runtime or launch error                          */
#define PC_EUNSUPPORTED (-4)  /* a parameter the GPU path does not implement          */
#define PC_EINTERNAL (-5)     /* internal table overflow (never expected)             */
#define PC_ENOPAGES (-6)      /* a pool has too few pages that nobody holds           */

#define PC_BLOCK_TOKENS 16    /* the only block size the GPU path implements          */
#define PC_MAX_GROUPS 64
#define PC_MAX_CONTRACTS 4
#define PC_MAX_CAPACITY 32767

/* Thread-local description of the last failure on this host thread. */
const char *pc_last_error(void);

/* ------------------------------------------------------------------------
 * Block cutting.  Each request is cut into floor(len / 16) full blocks; a
 * partial tail gets no key (Sec. III-B: only full KV blocks are metered).
 *
 * pc_block_offsets: d_key_off[r] = sum_{i<r} floor(d_req_len[i] / 16) for
 * r = 0..n_req (n_req+1 int64 values, CSR offsets of each request's keys).
 * d_req_len values must be >= 0 (negative lengths count as 0 blocks).
 * ------------------------------------------------------------------------ */
int32_t pc_block_offsets(const int32_t *d_req_len, int64_t n_req, int32_t block_size,
                         int64_t *d_key_off, void *stream);

/* ------------------------------------------------------------------------
 * Chained block keys (PCH64; the paper keeps the serving engine's native
 * content hash, Sec. III-A and IV, so this key is the library's own).
 * For a request in namespace ns (its accounting group, Sec. II-C) with
 * tokens t (int32, reinterpreted as uint32):
 *   d_k   = sum_{i<8} ((t[16k+2i] + K[2i]) mod 2^32) * ((t[16k+2i+1] + K[2i+1]) mod 2^32)  mod 2^64
 *   H_-1  = fmix64(ns + 1),  H_k = A*H_{k-1} + fmix64(d_k) mod 2^64,  key_k = fmix64(H_k)
 * where fmix64 is the MurmurHash3 finalizer, A = 0x9E3779B97F4A7C15 and
 * K[i] = floor(frac(sqrt(p_i)) * 2^31) + 1 for the first 16 primes.
 *
 *   d_tokens   [n_tokens] int32, 4-byte aligned (else PC_EINVAL); a
 *              request may start at any token, and requests may alias.
 *   d_req_tok_off, d_req_len, d_req_ns  [n_req]: start, length, namespace;
 *              a request holds fewer than 2^30 tokens (4 GiB).
 *   d_key_off  [n_req+1] output of pc_block_offsets (or any offsets with
 *              room for floor(len/16) keys per request).
 *   d_keys     [n_keys] output.
 *   d_status   one int32 in device memory, set to PC_EINVAL by the kernel if
 *              any request's token or key range falls outside the buffers,
 *              or its length is negative or 2^30 or more (that request is
 *              skipped); the caller zeroes it beforehand.
 * ------------------------------------------------------------------------ */
int32_t pc_hash_blocks(const int32_t *d_tokens, int64_t n_tokens,
                       const int64_t *d_req_tok_off, const int32_t *d_req_len,
                       const int32_t *d_req_ns, const int64_t *d_key_off, int64_t n_req,
                       int32_t block_size, uint64_t *d_keys, int64_t n_keys,
                       int32_t *d_status, void *stream);

/* ------------------------------------------------------------------------
 * Replay.
 * ------------------------------------------------------------------------ */
/* Policies (Sec. V-A): LRU is the engine's free-queue order; S3-FIFO and
 * StaticQuota are the paper's baselines; PrefixShield is its method (Sec.
 * III).  StaticQuota gives every accounting group a fixed partition of
 * floor(capacity / n_groups) blocks with LRU inside it and no borrowing: a
 * request probes at most its partition (the rest counts as truncated) and
 * reclaims only its own group's blocks. */
enum { PC_LRU = 0, PC_S3FIFO = 1, PC_PREFIXSHIELD = 2, PC_STATICQUOTA = 3 };
enum { PC_FLAG_NO_SEGMENTATION = 1,   /* Sec. V-D ablation: one retention segment    */
       PC_FLAG_NO_DEBT_GATE = 2 };    /* Sec. V-D ablation: promote regardless of debt */

/* One request trace, all arrays in device memory.  Request r probes the
 * keys d_keys[d_key_off[r] .. d_key_off[r+1]).  Group = accounting group
 * (also the lookup namespace), contract = service contract, prefix =
 * logical prefix id, dense per (group, prefix) (Sec. III-A).  Ticks are the
 * monotonic accounting clock (Eq. 1); NULL means tick = request index. */
typedef struct {
    const uint64_t *d_keys;
    const int64_t *d_key_off;      /* [n_req+1], non-decreasing, within [0, n_keys] */
    const uint8_t *d_group;        /* [n_req] < n_groups                            */
    const uint8_t *d_contract;     /* [n_req] < the instance's n_contracts          */
    const uint32_t *d_prefix;      /* [n_req] < n_prefix                            */
    const int64_t *d_tick;         /* [n_req] >= 0, non-decreasing, or NULL         */
    int64_t n_req;
    int64_t n_keys;
    int64_t n_prefix;
    int32_t n_groups;              /* 1..64                                         */
    int32_t max_req_blocks;        /* >= every d_key_off[r+1]-d_key_off[r]          */
} pc_trace_desc;

/* A service contract (Eqs. 1-2).  The contracts of one instance are weighted
 * by w_c = rho_c / rho_min (Eq. 5), and 1/w_c is kept in Q16, so their refill
 * rates may differ by a factor 2^16 at most (else PC_EINVAL): Eq. 8's
 * per-victim decrement 1/W_g is then at least one Q16 unit. */
typedef struct {
    int64_t rho_q16;               /* refill rate per tick, > 0 (Prop. 1), <= 2^40  */
    int64_t beta_q16;              /* burst capacity, 0..2^50                        */
} pc_contract;

typedef struct {
    int32_t trace;                 /* index into the traces array                  */
    int32_t policy;                /* PC_LRU / PC_S3FIFO / PC_PREFIXSHIELD /
                                      PC_STATICQUOTA                                */
    int32_t capacity;              /* usable blocks, 1..PC_MAX_CAPACITY             */
    int32_t flags;                 /* PC_FLAG_*                                     */
    int32_t n_contracts;           /* 1..4                                          */
    int32_t s3_small_permille;     /* S3-FIFO small-queue share, 0..1000 (100)      */
    int32_t s3_move_threshold;     /* S3-FIFO small->main access count, >= 0 (1)    */
    int32_t reserved;              /* must be 0                                     */
    int64_t eps_q16;               /* debt tolerance epsilon, 0..2^50 (Sec. III-B)  */
    pc_contract contract[PC_MAX_CONTRACTS];
} pc_instance_desc;

/* Per instance, per accounting group; exact integers. */
typedef struct {
    uint64_t requests, probes, hits, misses, charged, evicted_owned, evictions_caused,
        promotions, gated, orphans, dups, truncated;
    int64_t debt_end_q16;          /* raw debt D_g (Eq. 3) at the last request's tick */
    int64_t debt_max_q16;          /* max over requests of D_g after the request      */
    int64_t debt_sum_q16;          /* sum over requests of D_g after the request      */
    int64_t resident_end, resident_max;
} pc_group_stats;

typedef struct {
    uint64_t evictions, s3_moves, s3_reinserts, s3_ghost_hits, s3_ghost_inserts;
    int64_t resident_end, resident_max;
    int32_t status;                /* PC_OK, or PC_EINVAL if a request was malformed
                                      (the instance stopped there; counters zeroed) */
    int32_t reserved;
} pc_instance_stats;

/* Device stats record of one instance: 64 pc_group_stats then one
 * pc_instance_stats.  d_stats for n_inst instances needs
 * n_inst * PC_STATS_RECORD_BYTES bytes. */
#define PC_STATS_RECORD_BYTES (64 * 136 + 64)

/* Workspace bytes for this batch (< 0: invalid input, see pc_last_error).
 * They include the trace analysis of the replay on runs: some 12 bytes per
 * key of every distinct key buffer, or, where its traces can read only part of
 * it, per key that they can (n_req * max_req_blocks); and 32 per request; where
 * that is at most 16 GiB.  pc_replay_batch also takes a workspace that only
 * lacks this part and then replays with the general kernels alone. */
int64_t pc_replay_workspace_bytes(const pc_trace_desc *traces, int32_t n_traces,
                                  const pc_instance_desc *inst, int32_t n_inst);

/* The same without the trace analysis: the least that pc_replay_batch takes,
 * for where device memory is short.  From here up to
 * pc_replay_workspace_bytes the general kernels alone replay the batch, with
 * the same results in a multiple of the time. */
int64_t pc_replay_workspace_min_bytes(const pc_trace_desc *traces, int32_t n_traces,
                                      const pc_instance_desc *inst, int32_t n_inst);

/* Where pc_replay_batch, given a workspace of workspace_bytes, leaves how it
 * replayed the instances: the byte offset of int32[n_inst] in the workspace
 * (the results do not depend on it), or 0: with the general kernels all. */
#define PC_ROUTE_GENERAL 0
#define PC_ROUTE_RUNS 1             /* one wavefront, on runs of blocks             */
#define PC_ROUTE_RUNS_WIDE 2        /* the same, with the widest windows            */
int64_t pc_replay_route_offset(const pc_trace_desc *traces, int32_t n_traces,
                               const pc_instance_desc *inst, int32_t n_inst,
                               int64_t workspace_bytes);

/* Per-instance replay state (the cache metadata: block keys and metadata,
 * stamps, the free-queue log, the block and ghost tables, per-request
 * scratch) that pc_replay_batch's general kernels would use for this batch:
 * bytes_out[i] bytes, laid out as layout_out[i] says:
 *   PC_LAYOUT_LDS     all of it in LDS
 *   PC_LAYOUT_HYBRID  block keys and prefix ids in the workspace, the rest
 *                     in LDS (chosen when it lets more instances share a CU)
 *   PC_LAYOUT_WS      all of it in the workspace (when it does not fit LDS)
 * Host only; validates like pc_replay_workspace_bytes.  The per-prefix
 * bitmaps and the S3-FIFO ghost ring live in the workspace and are not
 * counted. */
#define PC_LAYOUT_LDS 0
#define PC_LAYOUT_HYBRID 1
#define PC_LAYOUT_WS 2
int32_t pc_replay_state_bytes(const pc_trace_desc *traces, int32_t n_traces,
                              const pc_instance_desc *inst, int32_t n_inst,
                              int64_t *bytes_out, int32_t *layout_out);

/* Replay every instance over its trace, one wavefront or workgroup per
 * instance; queued on `stream` (instances of different LDS footprints run as
 * separate launches on library streams that fork from and join back into it).
 * Per request it runs the hooks of Alg. 1 (OnRequest, OnTouch with the debt
 * gate of Eq. 4, OnCacheFullBlocks metering Eqs. 1-3) and, when the cache is
 * full, the reclamation of Alg. 2 (PrefixShield: Eqs. 5-9; LRU, S3-FIFO and
 * StaticQuota: the baselines of Sec. V-A) under the same debt accounting.
 *   d_workspace   device memory of pc_replay_workspace_bytes() bytes or more
 *                 (see there), 256-byte aligned; its contents need not be
 *                 zeroed.
 *   d_stats       n_inst * PC_STATS_RECORD_BYTES bytes, written at the end.
 *   d_per_request optional (NULL): per-request int32 quadruples (hits, new
 *                 blocks, evictions, orphans); instance i's block starts at
 *                 4 * sum_{j<i} traces[inst[j].trace].n_req.
 * Instances are independent; their order does not affect any result. */
int32_t pc_replay_batch(const pc_trace_desc *traces, int32_t n_traces,
                        const pc_instance_desc *inst, int32_t n_inst,
                        void *d_workspace, int64_t workspace_bytes, void *d_stats,
                        int32_t *d_per_request, void *stream);

/* For callers that cannot allocate device memory (code under HIP graph
 * capture, serving loops and harnesses that forbid allocation): the same
 * replay as pc_replay_batch, with the workspace taken from a static device
 * array of PC_STATIC_WORKSPACE_BYTES that the library holds on every GPU it
 * runs on, until the process ends.  The call allocates no device memory and
 * no pinned host memory; the caller still passes d_stats and d_per_request
 * (as for pc_replay_batch).
 *   - A batch whose workspace exceeds PC_STATIC_WORKSPACE_BYTES even without
 *     the trace analysis (see pc_replay_workspace_bytes) is rejected with
 *     PC_ENOMEM, queuing nothing.
 *   - Every call on one GPU uses that GPU's one array.  The kernels clear
 *     what they need, so a call never depends on an earlier call's
 *     contents, but calls whose work overlaps on one GPU (other streams, or
 *     another host thread) race on the array and give undefined results:
 *     order them on one stream.
 *   - The descriptor upload copies from pageable host memory, which the
 *     runtime has read when the call returns. */
#define PC_STATIC_WORKSPACE_BYTES (64LL << 20)
int32_t pc_replay_batch_static(const pc_trace_desc *traces, int32_t n_traces,
                               const pc_instance_desc *inst, int32_t n_inst, void *d_stats,
                               int32_t *d_per_request, void *stream);

/* Synchronize `stream`, copy the stats of one instance (or of all n_inst
 * when instance == -1) to the host and decode them: per-group hits, misses
 * and evictions, charged blocks (Eq. 2), the raw debt D_g of Eq. 3 (final,
 * maximum and sum over requests, whose mean is the "mean debt" of Sec. V-D)
 * and occupancy (Table III).
 *   groups_out  [max_groups] (or [n_inst][max_groups] for instance == -1)
 *   inst_out    [1] (or [n_inst]) */
int32_t pc_get_stats(const void *d_stats, int32_t n_inst, int32_t instance,
                     pc_group_stats *groups_out, int32_t max_groups,
                     pc_instance_stats *inst_out, void *stream);

/* ------------------------------------------------------------------------
 * Pages of a KV cache, and attention over them.
 *
 * A pool holds the K and V of sequences in pages of PC_BLOCK_TOKENS tokens,
 * the blocks that pc_hash_blocks keys.  Token t of a sequence is in the page
 * table[seq][t / 16], at place t % 16.  Sequences may hold a page together
 * (a shared prefix, a fork): refs[page] counts its holders, and a page that
 * nobody holds has 0.  All of it is the caller's device memory; the calls
 * below change it on the stream that they are given, and calls on one pool
 * that change it must be ordered.
 *
 * Device-side status (d_status, one int32 in device memory that the caller
 * zeroes, while no call with it is under way; pc_prefix_groups alone writes one
 * of its own): a call that finds its lists or the pool's state out of range
 * sets it to PC_EINVAL, or PC_ENOPAGES, and does nothing else unless said
 * otherwise.  A call that finds it set does nothing, so that calls may be
 * queued one after another (or captured) and looked at once, at the end.
 * Calls that may overlap (on other streams) have a status of their own each, or
 * may be stopped by each other's errors, pc_pages_write in the middle and the others
 * as a whole.  A call that is refused or stopped may turn a length that is out of
 * range into another one that is.  No call reads or writes outside the
 * buffers described here, whatever the lists and tables hold.
 *
 * Every call can be captured into a HIP graph.  A workspace holds nothing
 * between calls (but for pc_attn, see there): calls that do not overlap may
 * share one, on one stream or in several graphs.
 * ------------------------------------------------------------------------ */
enum { PC_BF16 = 0, PC_FP16 = 1 };
enum { PC_HEADS_FIRST = 0,            /* a page is [n_kv_heads][16][head_dim]          */
       PC_TOKENS_FIRST = 1 };         /* a page is [16][n_kv_heads][head_dim]          */

#define PC_MAX_SEQS 262144            /* sequences of a pool                           */
#define PC_MAX_POOL_PAGES (1 << 27)
#define PC_MAX_BATCH 4096             /* requests of one batch, sequences that grow at once */
#define PC_ATTN_HEAD_BYTES 256        /* of an attention's workspace, zeroed by the caller once */

typedef struct {
    void *d_k, *d_v;                  /* page 0 of layer 0, 16-byte aligned            */
    int32_t *d_refs;                  /* [n_pages] holders                             */
    int32_t *d_table;                 /* [n_seqs][table_width]; entries at and behind a
                                         sequence's last page may hold anything        */
    int32_t *d_len;                   /* [n_seqs] tokens, 0..16 * table_width          */
    int64_t page_stride;              /* elements from a page to the next, >= one
                                         page's 16 * n_kv_heads * head_dim, a multiple
                                         of 8 (any value where n_pages is 1); the same
                                         for K and V                                   */
    int64_t layer_stride;             /* elements from a layer to the next, a multiple
                                         of 8 (any value where n_layers is 1)          */
    int32_t n_layers;                 /* >= 1; the layers share table, len and refs    */
    int32_t n_pages;                  /* 1..PC_MAX_POOL_PAGES                          */
    int32_t n_seqs;                   /* 1..PC_MAX_SEQS                                */
    int32_t table_width;              /* 1..2^24                                       */
    int32_t n_kv_heads;               /* 1..256                                        */
    int32_t head_dim;                 /* 64 or 128                                     */
    int32_t dtype;                    /* PC_BF16 / PC_FP16                             */
    int32_t layout;                   /* PC_HEADS_FIRST / PC_TOKENS_FIRST              */
} pc_pages;

/* Rows of K, V, queries or results: one of head_dim elements (contiguous, 16-byte
 * aligned) for each token and head. */
typedef struct {
    void *d_data;
    int64_t token_stride, head_stride;   /* elements, multiples of 8 (any value where there is one) */
} pc_rows;

/* Workspace bytes of pc_pages_extend for up to n sequences a call, and of
 * pc_pages_compact (any n >= 0).  < 0: invalid, see pc_last_error. */
int64_t pc_pages_workspace_bytes(const pc_pages *pages, int64_t n);

/* Child i takes over parent i's pages and length; each page has a holder
 * more.  A parent may have several children.  Children are distinct, empty
 * (length 0), and no parents. */
int32_t pc_pages_fork(const pc_pages *pages, const int32_t *d_parent, const int32_t *d_child, int32_t n,
                      int32_t *d_status, void *stream);

/* Sequence d_seq[i] grows by d_add[i] >= 0 tokens; the sequences are distinct,
 * PC_MAX_BATCH of them at most (else PC_EUNSUPPORTED).
 * New pages are the lowest that nobody holds, handed out in the order of the
 * list.  A last page that is filled in part and held by others too is copied
 * for a sequence that grows, K and V of every layer, the copy taking the first
 * of its new pages; but where all its holders are in the list and grow, the
 * first of them keeps it.  The pages that hold the new tokens are then the
 * sequence's alone.  Their K and V are as they were: pc_pages_write fills them.
 * A pool with too few pages sets the status to PC_ENOPAGES and is left as it was.
 *   d_workspace   pc_pages_workspace_bytes(pages, n) bytes, 256-byte aligned */
int32_t pc_pages_extend(const pc_pages *pages, const int32_t *d_seq, const int32_t *d_add, int32_t n,
                        void *d_workspace, int64_t workspace_bytes, int32_t *d_status, void *stream);

/* The distinct sequences d_seq[i] give their pages up (a holder less each) and
 * are empty.  Their table entries and the pages' K and V stay as they are
 * until the pages are handed out again. */
int32_t pc_pages_free(const pc_pages *pages, const int32_t *d_seq, int32_t n, int32_t *d_status, void *stream);

/* Pages in use move to the lowest page numbers: with n_live pages in use, the
 * i-th one at or behind n_live moves to the i-th unused place before it, K and
 * V of every layer.  New counts and tables go to d_refs_to [n_pages] and
 * d_table_to [n_seqs][table_width] (which may be the pool's own), n_live to
 * d_n_live.  Where they are not the pool's own, readers of the old table find
 * what they did: pages that moved keep their contents at the old place.
 * A page number out of the pool, or of a page that nobody holds, is passed on
 * as it is and sets the status to PC_EINVAL. */
int32_t pc_pages_compact(const pc_pages *pages, int32_t *d_refs_to, int32_t *d_table_to, int32_t *d_n_live,
                         void *d_workspace, int64_t workspace_bytes, int32_t *d_status, void *stream);

/* Stores K and V of the last tokens of n distinct sequences, in one layer: rows
 * d_new_off[i] .. d_new_off[i+1]-1 of k_new and v_new (n_tokens rows) are the
 * last tokens of sequence d_seq[i], which pc_pages_extend has made room for.
 * Where the status is set, rows may or may not have been stored: a token's page
 * out of the pool, or held by more than one sequence, is not written. */
int32_t pc_pages_write(const pc_pages *pages, int32_t layer, const int32_t *d_seq, const int32_t *d_new_off,
                       int32_t n, int64_t n_tokens, const pc_rows *k_new, const pc_rows *v_new,
                       int32_t *d_status, void *stream);

/* Groups of a batch by the block keys of its requests (d_keys, d_key_off: as
 * of pc_block_offsets and pc_hash_blocks).  Two requests with at least
 * min_blocks >= 1 full blocks are in one group if their keys of block
 * min_blocks - 1 are equal (keys are chained, so their blocks before it are
 * then equal too); a request with fewer blocks is in a group of its own.
 * Groups are in the order of their first requests, requests in a group in
 * their own order:
 *   d_order      [n_req] the requests, group by group
 *   d_group_off  [n_req+1] group g: d_order[d_group_off[g]] .. ; n_req from
 *                d_group_off[n_groups] on
 *   d_shared     [n_req] leading blocks with the same keys in all requests of
 *                group g; 0 for a group of one and behind the last group
 *   d_n_groups   [1]; -1 where the offsets are refused, which pc_attn_plan
 *                refuses in its turn
 * n_req is at most PC_MAX_BATCH (else PC_EUNSUPPORTED), a request has 2^26
 * blocks at most.  d_status, written by every call and not read: PC_OK, or
 * PC_EINVAL where the offsets fall or leave [0, n_keys] (only d_n_groups is
 * written beside it then). */
int32_t pc_prefix_groups(const uint64_t *d_keys, int64_t n_keys, const int64_t *d_key_off, int32_t n_req,
                         int32_t min_blocks, int32_t *d_order, int32_t *d_group_off, int32_t *d_shared,
                         int32_t *d_n_groups, int32_t *d_status, void *stream);

/* Attention of a batch over its pages, in two calls: a plan, once for a batch
 * of the lengths it then has, and the attention of one layer by that plan, as
 * often as there are layers.
 *   request r     the sequence d_seq[r] (one may come twice) and the queries
 *                 d_q_off[r] .. d_q_off[r+1]-1 of n_tokens (from 0 to n_tokens, each
 *                 in one request); its length L counts the tokens of these
 *                 queries, whose K and V are in the pages.
 *   causal        query i of n sees the tokens before L - n + i + 1; otherwise,
 *                 all L.  A query that sees none (also: of an empty sequence)
 *                 gives zeros, and -inf in lse.
 *   d_order ..    the groups, as pc_prefix_groups gives them; or all four NULL:
 *                 no request shares anything.  The pages of a group's shared
 *                 blocks have to hold the same tokens in all its requests: those
 *                 of the first one are read for all.  Shared blocks behind the
 *                 shortest request's last full one are taken as not shared.
 * A group's shared tokens are read once for the queries of all its requests
 * (where requests have many queries, or share little, also for each by itself,
 * if that is sooner done), each request's own tokens by itself, and long ranges in
 * several parts; the results are joined by their sums of exponentials.  Scores, sums and joined
 * values are in 32 bits; the weights are rounded to the pool's type before
 * the product with V, those of a request with up to 16 rows a KV head (a few
 * decoding queries) to twice its bits, over shared tokens as over its own.  Results
 * do not depend on timing.
 * K of a token that a query does not see, and K and V behind the length, may
 * hold anything.  V of the tokens within the length is finite: a weight of
 * zero times infinity or NaN is NaN.
 *   d_workspace   pc_attn_workspace_bytes() bytes, 256-byte aligned; it holds the
 *                 plan from pc_attn_plan until the last pc_attn of that plan
 *                 is done, and their partial results: they must not overlap.
 *                 Its first PC_ATTN_HEAD_BYTES are zeroed by the caller when the
 *                 memory becomes a workspace: a plan that it held before would
 *                 be taken for this one's. */
int64_t pc_attn_workspace_bytes(const pc_pages *pages, int32_t n_req, int64_t n_tokens, int32_t n_heads);

int32_t pc_attn_plan(const pc_pages *pages, const int32_t *d_seq, const int32_t *d_q_off, int32_t n_req,
                     int64_t n_tokens, int32_t n_heads, int32_t causal, const int32_t *d_order,
                     const int32_t *d_group_off, const int32_t *d_shared, const int32_t *d_n_groups,
                     void *d_workspace, int64_t workspace_bytes, int32_t *d_status, void *stream);

/* out[t][h] = softmax(scale * q[t][h] . K) V over the tokens that query t sees;
 * n_heads is a multiple of the KV heads, head h reads KV head
 * h / (n_heads / n_kv_heads).  n_req, n_tokens and n_heads are the plan's, and so
 * are the pool's table and lengths; K and V are of `layer`.  scale > 0, and
 * scale log2(e) a finite float.
 *   d_lse         optional (NULL): [n_tokens][n_heads] float, the natural
 *                 logarithm of each row's sum of exponentials
 * Without a plan of these n_req, n_tokens and n_heads for this pool's shape in
 * the workspace (also: where the plan set the status), nothing is written.  A
 * page number out of the pool reads another page, never memory outside. */
int32_t pc_attn(const pc_pages *pages, int32_t layer, const pc_rows *q, int32_t n_req, int64_t n_tokens,
                int32_t n_heads, float scale, const pc_rows *out, float *d_lse, void *d_workspace,
                int64_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* PC_H */
