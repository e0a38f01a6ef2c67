/*
 * foe.h - C ABI of the MI355X (gfx950) per-cluster MoE block of
 *         Federation of Experts (FoE).
 *
 * One FoE layer splits its MoE block into H expert groups ("clusters"), each
 * owning a contiguous block of experts (Section 3, notation table).  All groups
 * route the same cross-group averaged residual r_full with one router and each
 * keeps its own top-k/H experts (Section 3.1, routing equation); every group
 * then forms its partial x'[h] = r_full + sum_e w_h[i,e] FFN_e(r_full)
 * (Table 3, "MoE update" row) and the partials are averaged (Table 3,
 * "Cross-group avg." row; Section 3.1, "Layer boundaries").  Groups that share
 * a GPU combine their partials locally (Section 3.2).  This library runs that
 * block for C clusters co-resident on one GPU.
 *
 * Per cluster: T tokens, hidden size d, E experts, top-k k (the paper's k/H),
 * expert FFN size F, R = T*k (token, slot) pairs.
 *
 * Conventions shared by every entry point
 *  - Pointers are DEVICE pointers owned by the caller unless marked (host).
 *    Tensors are dense row-major; weights are [out, in] (K-contiguous).
 *  - dt selects the storage type of activations, weights and FFN outputs:
 *    FOE_F32 (fp32) or FOE_BF16 (bf16).  Router bias, routing weights and all
 *    accumulation are fp32 in both cases.  Indices are int32.
 *  - Every tensor pointer must be 16-byte aligned; d and F must be multiples
 *    of 8 (rows are moved as 128-bit vectors).
 *  - Limits: 0 <= T, 1 <= k <= E <= 256, 1 <= C <= 64, d, F >= 8.  T = 0 is an
 *    empty batch: outputs are empty and, for foe_permute, counts/offsets are
 *    written as zeros.
 *  - `stream` is a hipStream_t (NULL = the null stream).  Calls only enqueue
 *    work on it and return; the caller synchronises.  No call allocates device
 *    memory: scratch comes from the caller's workspace `ws` of `ws_bytes`
 *    bytes (16-byte aligned), sized with foe_workspace_bytes().
 *  - Return value: FOE_OK (0) or a negative foe_status.  All argument checks
 *    run on the host before anything is enqueued, so an error leaves device
 *    memory untouched.  foe_last_error() gives a message for the calling
 *    thread's last failure.
 *  - Outputs are bit-deterministic: the same inputs give the same bits on
 *    every call (no floating point atomics; fixed summation orders).
 *  - Device-side index data supplied by the caller (topk_idx, offsets,
 *    row_of) is not trusted for memory safety: out-of-range entries are
 *    skipped rather than dereferenced (documented per entry point).
 */
#ifndef FOE_H
#define FOE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    FOE_OK = 0,
    FOE_ERR_INVALID = -1,     /* bad shape, null/misaligned pointer, bad dtype */
    FOE_ERR_UNSUPPORTED = -2, /* valid request the library does not implement */
    FOE_ERR_WORKSPACE = -3,   /* ws_bytes below foe_workspace_bytes()        */
    FOE_ERR_HIP = -4          /* the HIP runtime reported an error            */
} foe_status;

typedef enum { FOE_F32 = 0, FOE_BF16 = 1 } foe_dtype;

/*
 * Routing weights of the selected experts (Section 3.1 routing equation; the
 * paper leaves renormalisation open):
 *   FOE_GATE_RENORM  softmax over the k selected scores of the group: the
 *                    global softmax renormalised over the selection (each
 *                    token's k weights of a group sum to 1)
 *   FOE_GATE_GLOBAL  the global softmax over the single score vector of all
 *                    C*E experts (all groups), taken at the selected experts
 *                    and not renormalised (OLMoE-style gating; each group's
 *                    weights sum to its share of the probability mass)
 */
typedef enum { FOE_GATE_RENORM = 0, FOE_GATE_GLOBAL = 1 } foe_gating;

/*
 * foe_route - router scores, per-group top-k and routing weights.
 * Section 3.1, routing equation: g[i] = Router(r_full[i]) and
 * I_h[i], w_h[i] = TopK over the group's experts of g[i].
 *
 *   x         [T,d] dt        the block input r_full (one row per token)
 *   w_router  [E,d] dt        this cluster's router rows (linear router)
 *   bias      [E]   fp32      added to the scores, or NULL
 *   topk_idx  [T,k] int32 out expert ids, descending score; equal scores ->
 *                             lower id first.  Scores are fp32 (fp32
 *                             accumulation of the dt products, plus bias).
 *   topk_w    [T,k] fp32  out softmax over the k selected scores (each row
 *                             sums to 1; equals the global softmax
 *                             renormalised over the selection)
 * Needs no workspace.
 */
int foe_route(foe_dtype dt, int T, int d, int E, int k,
              const void* x, const void* w_router, const float* bias,
              int32_t* topk_idx, float* topk_w, void* stream);

/*
 * foe_route_ex - foe_route for G groups sharing x, with a gating choice.
 * The G router matrices w_router [G,E,d] (and bias [G,E] or NULL) form one
 * score vector of G*E experts per token; group h takes its top-k over its own
 * block of E scores and writes topk_idx/topk_w [G,T,k] rows h*T.. (ids local
 * to the group, 0..E-1).  gating: FOE_GATE_RENORM (foe_route's weights) or
 * FOE_GATE_GLOBAL (softmax over all G*E scores, not renormalised).
 * FOE_ERR_UNSUPPORTED when G*E > 256 with G > 1.  Needs no workspace.
 */
int foe_route_ex(foe_dtype dt, int G, int T, int d, int E, int k, foe_gating gating,
                 const void* x, const void* w_router, const float* bias,
                 int32_t* topk_idx, float* topk_w, void* stream);

/*
 * foe_permute - expert histogram, prefix sum and stable token permutation:
 * the on-device form of the intra-group dispatch (Section 3.2; on one GPU the
 * local activation rate is 1 and dispatch never leaves the device).
 *
 *   topk_idx        [T,k]   int32  from foe_route (or any k ids per token)
 *   x               [T,d]   dt     rows to dispatch
 *   expert_counts   [E]     int32 out pairs per expert (may be NULL)
 *   expert_offsets  [E+1]   int32 out exclusive prefix sum; offsets[E] = number
 *                                  of valid pairs (T*k when all ids are valid)
 *   sorted_src      [T*k]   int32 out flat pair f = i*k + j held by permuted
 *                                  row p; order = (expert asc, token asc)
 *   row_of          [T*k]   int32 out inverse: row_of[f] = p (-1 for a pair
 *                                  whose id is outside [0,E); such pairs are
 *                                  dropped and trailing sorted_src/x_perm
 *                                  rows are left unwritten)
 *   x_perm          [T*k,d] dt    out x_perm[p] = x[sorted_src[p] / k]
 *   ws, ws_bytes    workspace of foe_workspace_bytes("permute", ...)
 */
int foe_permute(foe_dtype dt, int T, int d, int E, int k,
                const int32_t* topk_idx, const void* x,
                int32_t* expert_counts, int32_t* expert_offsets,
                int32_t* sorted_src, int32_t* row_of, void* x_perm,
                void* ws, size_t ws_bytes, void* stream);

/*
 * foe_expert_ffn - grouped SwiGLU expert FFN over the permuted rows
 * (Table 3 "MoE update": FFN_e applied to the rows routed to expert e).
 * Rows offsets[e] .. offsets[e+1]-1 of x_perm go through expert e:
 *   y = W_d[e] (silu(W_g[e] x) * (W_u[e] x)),  silu(z) = z / (1 + exp(-z)).
 * bf16: products in bf16 MFMA with fp32 accumulation; the hidden activation
 * is rounded to bf16 (nearest even) before the down projection.
 *
 *   rows            number of permuted rows (T*k)
 *   x_perm          [rows,d]  dt
 *   expert_offsets  [E+1]     int32 (device) segment bounds; bounds are
 *                             clamped to [0, rows] and a decreasing bound
 *                             gives an empty segment
 *   w_gate, w_up    [E,F,d]   dt
 *   w_down          [E,d,F]   dt
 *   y_perm          [rows,d]  dt out (rows outside every segment are not written)
 *   ws, ws_bytes    workspace of foe_workspace_bytes("expert_ffn", ...)
 * bf16 limits: rows*d and rows*F below 2^30 elements (else FOE_ERR_UNSUPPORTED).
 */
int foe_expert_ffn(foe_dtype dt, int E, int d, int F, int rows,
                   const void* x_perm, const int32_t* expert_offsets,
                   const void* w_gate, const void* w_up, const void* w_down,
                   void* y_perm, void* ws, size_t ws_bytes, void* stream);

/*
 * foe_combine - weighted un-permute (Table 3 "MoE update": the weighted sum
 * over the selected experts, plus r_full):
 *   out[i] = residual[i] + sum_{j<k} topk_w[i,j] * y_perm[row_of[i*k+j]]
 * summed in fp32 in slot order j = 0..k-1, rounded once to dt.
 *
 *   y_perm    [T*k,d] dt
 *   row_of    [T*k]   int32   entries outside [0, T*k) contribute nothing
 *   topk_w    [T,k]   fp32
 *   residual  [T,d]   dt      or NULL (then out = the weighted sum only)
 *   out       [T,d]   dt out
 */
int foe_combine(foe_dtype dt, int T, int d, int k,
                const void* y_perm, const int32_t* row_of, const float* topk_w,
                const void* residual, void* out, void* stream);

/*
 * foe_reduce - local reduction of C cluster partials (Table 3 "Cross-group
 * avg."; Section 3.1 final cross-group average; Section 3.2: groups sharing a
 * GPU combine partials locally):
 *   out = scale * sum_{h=0}^{C-1} (residual + partials[h])
 * accumulated in fp32 in the fixed order h = 0..C-1 (residual omitted when
 * NULL).  scale = 1/C is the paper's average.
 *
 *   partials  [C,T,d] dt;  residual [T,d] dt or NULL;  out [T,d] dt
 */
int foe_reduce(foe_dtype dt, int C, int T, int d,
               const void* partials, const void* residual, float scale,
               void* out, void* stream);

/*
 * foe_cluster_block - the whole block for C clusters sharing the input x
 * (all groups route and update the same r_full: Table 3 "Routing" and "MoE
 * update" rows), followed by the local reduction:
 *   out = reduce_scale * sum_h (x + delta_h),
 *   delta_h[i] = sum_{e in I_h[i]} w_h[i,e] FFN_{h,e}(x[i]).
 * One routing pass scores all clusters (one read of x when C*E <= 256) and
 * each cluster takes its top-k over its own experts; the dispatch of all
 * clusters is numbered in one pass (at decode sizes each FFN workgroup lists
 * its expert's pairs itself); one grouped FFN covers all C*E experts and
 * reads the rows of x through the permutation (no permuted copy of x is
 * written); the weighted sums of every cluster and the reduction are formed
 * in one pass (at decode sizes inside the down-projection kernel) and no
 * per-cluster partial is written.  Evaluated as reduce_scale * (C * x + S)
 * with S the fp32 sum of the weighted expert rows in the order
 * (h = 0..C-1, j = 0..k-1).  Weights are FOE_GATE_RENORM.
 *
 *   x         [T,d]       dt
 *   w_router  [C,E,d]     dt;   bias [C,E] fp32 or NULL
 *   w_gate    [C,E,F,d]   dt;   w_up [C,E,F,d] dt;   w_down [C,E,d,F] dt
 *   reduce_scale          1/C = the paper's average, 1 = a plain sum
 *   out       [T,d]       dt out
 *   ws, ws_bytes          workspace of foe_workspace_bytes("cluster_block", ...)
 * bf16 limits: T*d, C*T*k*d and C*T*k*F below 2^30 elements (else
 * FOE_ERR_UNSUPPORTED); C*T*k below 2^31.
 */
int foe_cluster_block(foe_dtype dt, int C, int T, int d, int E, int k, int F,
                      const void* x, const void* w_router, const float* bias,
                      const void* w_gate, const void* w_up, const void* w_down,
                      float reduce_scale, void* out,
                      void* ws, size_t ws_bytes, void* stream);

/*
 * foe_cluster_block_ex - foe_cluster_block with a gating choice (see
 * foe_gating).  FOE_GATE_GLOBAL normalises over all C*E scores of a token and
 * is supported for C == 1 or C*E <= 256 (else FOE_ERR_UNSUPPORTED).  Same
 * workspace as foe_cluster_block.
 */
int foe_cluster_block_ex(foe_dtype dt, int C, int T, int d, int E, int k, int F,
                         foe_gating gating, const void* x, const void* w_router,
                         const float* bias, const void* w_gate, const void* w_up,
                         const void* w_down, float reduce_scale, void* out,
                         void* ws, size_t ws_bytes, void* stream);

/*
 * foe_cluster_block_noalloc - foe_cluster_block (FOE_GATE_RENORM) for callers
 * that cannot allocate device memory or pass a workspace: code under HIP-graph
 * capture, tight serving loops, harnesses that forbid allocation.  Same
 * arguments as foe_cluster_block without ws / ws_bytes, same kernels, same
 * results bit for bit.
 *
 * Its scratch is a static device array of the library, one copy per GPU,
 * reserved when the library's code is first loaded on that GPU and held until
 * the process ends.  Its size is 128 MiB (134217728 bytes): enough for the
 * decode- and prefill-shaped blocks, e.g. C=1, T=8192, d=2048, E=16, k=2,
 * F=1024.  Sizes whose workspace
 * (foe_workspace_bytes("cluster_block", ...)) exceeds it are rejected with
 * FOE_ERR_UNSUPPORTED before anything is enqueued.  The call allocates no
 * device or host memory.
 *
 * Every call on one GPU uses that GPU's one array, which keeps the last call's
 * contents (the block clears what it needs itself): calls that overlap on one
 * GPU (two host threads, or two streams without an ordering between them)
 * race and give undefined results.  Calls ordered on one stream are safe.
 */
int foe_cluster_block_noalloc(foe_dtype dt, int C, int T, int d, int E, int k, int F,
                              const void* x, const void* w_router, const float* bias,
                              const void* w_gate, const void* w_up, const void* w_down,
                              float reduce_scale, void* out, void* stream);

/*
 * foe_group_attention - the per-group attention that feeds the block (Table 3,
 * FoE column, rows "Attn. residual" and "Cross-group avg."):
 *   r[h,i]    = x[h,i] + Attn_h(x[h,:])[i]     (every group its own representation)
 *   r_full[i] = (1/H) sum_h r[h,i]
 * computed as (1/H) (sum_h o[h,i] w_o[h]^T + sum_h x[h,i]) in fp32: the output
 * projections of all groups form one product over the concatenated head
 * outputs, and the residual sum (h = 0..H-1 in order) is added after it.
 * Attn_h: causal self-attention over the S tokens (positions 0..S-1) with one
 * key/value head and nq query heads sharing it (grouped-query attention),
 * scores q.k/sqrt(hd), rotary embedding on q and k pairing dimension i with
 * i+hd/2 at angle (s/scale)*theta^(-2i/hd), bias-free projections.
 *
 *   x        [H,S,d]          bf16
 *   w_qkv    [H,(nq+2)*hd,d]  bf16  rows: nq query heads, the key head, the value head
 *   w_o      [d,H*nq*hd]      bf16  the groups' output projections side by side:
 *                                   columns h*nq*hd .. (h+1)*nq*hd-1 belong to group h
 *   theta    rotary base (> 0);  scale: rotary scaling factor (> 0), positions / scale
 *   r_full   [S,d]            bf16 out
 *   ws, ws_bytes              workspace of foe_group_attention_workspace_bytes()
 * All pointers are device memory owned by the caller, 16-byte aligned (the
 * workspace too); the call enqueues work on `stream` and returns.  One of its
 * kernels (the residual sum, unless x is small) runs on a library-owned stream of
 * the current device, forked from `stream` and joined back to it by events, so all of the
 * call's work still follows earlier work on `stream` and precedes later work
 * (also under HIP-graph capture, where the fork and join become edges).  bf16 only
 * and hd = 96 or 128 (else FOE_ERR_UNSUPPORTED); H*S*d and H*S*(nq+2)*hd must stay
 * below 2^30 elements.  S = 0 is a no-op.  Scores have to stay below 2^29 in magnitude (a
 * row of larger ones may give NaN; foe_cache_attention takes any).
 */
int foe_group_attention(foe_dtype dt, int H, int S, int d, int nq, int hd, float theta,
                        float scale, const void* x, const void* w_qkv, const void* w_o,
                        void* r_full, void* ws, size_t ws_bytes, void* stream);

/* Workspace bytes of foe_group_attention (SIZE_MAX for invalid sizes). */
size_t foe_group_attention_workspace_bytes(int H, int S, int d, int nq, int hd);

/*
 * The 8-bit key/value cache: what a layer's attention keeps between calls, for
 * prompts in chunks and for decode steps (Section 3.1: each of the H groups has
 * one key/value head, shared by its nq query heads).
 *
 * A cache is a pool of n_pages pages of FOE_CACHE_PAGE tokens, for all groups:
 *   k_cache   [n_pages, H, 64, hd]     e4m3 codes (OCP fp8), a row per token; the keys
 *                                      are held after their rotation
 *   v_cache   [n_pages, H, 4, hd, 16]  e4m3 codes: per 16 tokens, each dim's 16 tokens
 *                                      side by side
 *   kv_scale  [n_pages, H, 2]          fp32, the page's key and value scale of a group:
 *                                      powers of two, at least 2^-100; value = code * scale
 *   mass      [n_pages, H, 64]         fp32, the attention weight that each token has
 *                                      received (for foe_cache_evict; optional elsewhere)
 * The scale of a group's 64 tokens is the smallest power of two s >= 2^-100 with
 * |x| <= 448 s for all of them.  A power of two costs a floating format no
 * precision, keeps the products' operands exact in bf16, and a scale that has to
 * grow rescales earlier codes without a second rounding (but among the 2^-9 s
 * steps of the smallest magnitudes).
 * The caller owns the pool and hands out pages:
 *   block_table [B, max_blocks] int32  pages of each sequence, in token order; token t of
 *                                      sequence b is in slot t % 64 of page
 *                                      block_table[b, t / 64]
 * A call's sequences b = 0 .. B-1 must not share a page that the call writes.
 * Entries outside [0, n_pages) are absent pages: nothing is stored there and
 * their tokens are not seen.  Lengths are cut to [0, 64 * max_blocks], row
 * ranges to [0, N].
 *
 * bf16 activations and hd = 96 or 128 only (else FOE_ERR_UNSUPPORTED).  Limits:
 * 1 <= H <= 64, 1 <= nq <= 64, B <= 65535, N*nq <= 2^22, n_pages >= 1,
 * 1 <= max_blocks <= 2^18, B*max_blocks <= 2^31.
 */
#define FOE_CACHE_PAGE 64

/*
 * foe_cache_append - rotates new tokens and stores their keys and values.
 * The batch packs the new rows of all sequences: sequence b has rows
 * row_start[b] .. row_start[b+1]-1 of N (possibly none), which become its tokens
 * ctx_len[b], ctx_len[b] + 1, ...
 *
 *   qkv       [H, N, nq+2, hd] dt   per group and row: nq query heads, the key, the value
 *   row_start [B+1]      int32      non-decreasing
 *   ctx_len   [B]        int32      tokens that each sequence holds before the call
 *   pos       [B]        int32      rotary position of a sequence's first new row, or NULL:
 *                                   ctx_len[b] (after an eviction positions run ahead)
 *   theta, scale                    rotary base and scaling as in foe_group_attention:
 *                                   dims i and i + hd/2 turn by (p/scale)*theta^(-2i/hd)
 *   q_out     [H, N, nq, hd] dt out the rotated queries (not qkv itself)
 *   k_cache, v_cache, kv_scale      updated: keys and values are quantised from fp32, a
 *                                   page that held tokens keeps a scale of at least its old
 *                                   one (when it grows, the codes of all its other slots
 *                                   are rescaled); else slots without a new token are left
 *                                   as they were
 * A token whose rotated key or value holds an element that is not finite, or of
 * 1.9375 * 2^127 or more in magnitude (its code would stand for 2^128), is stored
 * as a key of NaN codes and a zero value, and has no part in the scales: every
 * query that sees it gives NaN, and no other does.  Rows past the table's end give q_out
 * alone.  Needs no workspace.
 */
int foe_cache_append(foe_dtype dt, int H, int B, int N, int nq, int hd, int n_pages,
                     int max_blocks, float theta, float scale, const void* qkv,
                     const int32_t* row_start, const int32_t* ctx_len, const int32_t* pos,
                     const int32_t* block_table, void* q_out, void* k_cache, void* v_cache,
                     float* kv_scale, void* stream);

/*
 * foe_cache_append_tree - foe_cache_append for the rows of a tree of drafted tokens
 * (or any rows whose order in the batch is not their order in the text): row r of
 * sequence b stands depth[r] places behind its context, so it turns by pos[b] + depth[r].
 * The rows still become tokens ctx_len[b], ctx_len[b] + 1, ... of the cache, in their
 * order; foe_cache_attention_ex takes the same depths and each row's ancestors, and
 * foe_cache_accept keeps the rows of one path.
 *
 *   depth     [N]  int32   cut to [0, 2^20]
 */
int foe_cache_append_tree(foe_dtype dt, int H, int B, int N, int nq, int hd, int n_pages,
                          int max_blocks, float theta, float scale, const void* qkv,
                          const int32_t* row_start, const int32_t* ctx_len, const int32_t* pos,
                          const int32_t* depth, const int32_t* block_table, void* q_out,
                          void* k_cache, void* v_cache, float* kv_scale, void* stream);

/*
 * foe_cache_attention - causal attention of the new rows over the cache, after
 * foe_cache_append has stored them (same row_start and ctx_len):
 *   o[r,h,j] = sum_t p_t v_t,  p = softmax over t <= ctx_len[b] + i of q.k_t/sqrt(hd)
 * for row r = row_start[b] + i, group h and query head j.  A row that sees no
 * token (all its pages absent) gives zeros.
 *
 *   max_rows               upper bound (>= 1) of the rows of one sequence; it picks the
 *                          kernels (a decode step passes 1).  A sequence's rows past it are
 *                          left out
 *   q         [H, N, nq, hd] dt   rotated queries
 *   mass_in   [n_pages, H, 64] fp32, mass_out [n_pages, H, 64] fp32 out, or both NULL:
 *                          mass_out[t] = (t < ctx_len[b] ? mass_in[t] : 0) + the sum of p_t
 *                          over the call's rows and heads, for the tokens t of the
 *                          sequences that have rows (0 <= t < ctx_len[b] + rows); other
 *                          entries are not written.  mass_out may be mass_in itself
 *   out       [N, H, nq, hd] dt out   the layout of w_o's columns in foe_group_attention
 *   ws, ws_bytes           workspace of foe_cache_attention_workspace_bytes(), which no smaller
 *                          size takes more of: one for the largest H, B, N, nq, max_blocks and
 *                          max_rows of a caller's calls, with mass if any has it, serves them
 *                          all, one after another.  With mass it grows with the table's width
 *                          (scores of sequences of few columns are kept where all entries'
 *                          take at most 1 GiB, else formed again): tables need be no wider
 *                          than the longest sequence
 * bf16: products in bf16 MFMA with fp32 accumulation; softmax statistics, mass and
 * sums in fp32, the probabilities are rounded to bf16 for the product with v.
 * Scores may lie anywhere in fp32's range.  A row with a score of NaN or +inf, or
 * whose scores are all -inf (past fp32), gives NaN, and so do the masses of the
 * tokens that it sees.  The sums with v are normalised at the end: values up to
 * 2^94 in magnitude cannot take them past fp32.
 */
int foe_cache_attention(foe_dtype dt, int H, int B, int N, int nq, int hd, int n_pages,
                        int max_blocks, int max_rows, const void* q, const int32_t* row_start,
                        const int32_t* ctx_len, const int32_t* block_table, const void* k_cache,
                        const void* v_cache, const float* kv_scale, const float* mass_in,
                        float* mass_out, void* out, void* ws, size_t ws_bytes, void* stream);

/* Workspace bytes of foe_cache_attention (with_mass: mass_out is given; SIZE_MAX
 * for invalid sizes). */
size_t foe_cache_attention_workspace_bytes(int H, int B, int N, int nq, int hd, int max_blocks,
                                           int max_rows, int with_mass);

/*
 * foe_cache_attention_ex - foe_cache_attention with other masks and scores (each of the
 * arguments below may be left out: cap 0, pointers NULL).  With s = q.k_t/sqrt(hd),
 *   o[r,h,j] = sum_t p_t v_t,  p = softmax over the tokens that row r sees of
 *              cap * tanh(s / cap) - slope[h,j] * |place(r) - place(t)|
 *
 *   cap                    0 (the scores as they are) or in [2^-64, 2^64]
 *   slope     [H, nq]      fp32   slope of the distance bias of each head
 *   prefix    [B]  int32   the first prefix[b] tokens are seen by every row of sequence b (those
 *                          of its context and its rows up to max_rows), whatever their order
 *   tree      [N, tree_words] int32   bit i % 32 of word i / 32 of a row: it sees row i of its
 *                          sequence.  All rows see the context besides; a row sees itself
 *                          if its own bit says so.  NULL: itself and the rows before it
 *   tree_words             at least max_rows / 32, rounded up
 *   depth     [N]  int32   row r stands at place ctx_len[b] + depth[r], cut as in
 *                          foe_cache_append_tree.  NULL: row i of its sequence at ctx_len[b] + i.
 *                          Tokens of the context stand where they are in the cache: after
 *                          an eviction distances count the tokens that were kept, not those
 *                          of the text (each group keeps others).  Only the bias asks for
 *                          places
 *   ws, ws_bytes           workspace of foe_cache_attention_ex_workspace_bytes()
 * A row that sees no token gives zeros.  A mass counts the tokens that the rows see, and every
 * row, also those that foe_cache_accept then drops (see there for masses of the text alone).
 * Scores that pass fp32 are capped like any other; a NaN score gives a NaN row.  Capped and
 * biased scores have to stay within 2^100.
 */
int foe_cache_attention_ex(foe_dtype dt, int H, int B, int N, int nq, int hd, int n_pages,
                           int max_blocks, int max_rows, float cap, const float* slope,
                           const int32_t* prefix, const int32_t* tree, int tree_words,
                           const int32_t* depth, const void* q, const int32_t* row_start,
                           const int32_t* ctx_len, const int32_t* block_table, const void* k_cache,
                           const void* v_cache, const float* kv_scale, const float* mass_in,
                           float* mass_out, void* out, void* ws, size_t ws_bytes, void* stream);

/* Workspace bytes of foe_cache_attention_ex, whatever its scores and masks (SIZE_MAX
 * for invalid sizes); as with foe_cache_attention_workspace_bytes, smaller sizes take no more. */
size_t foe_cache_attention_ex_workspace_bytes(int H, int B, int N, int nq, int hd, int max_blocks,
                                              int max_rows, int with_mass);

/*
 * foe_cache_accept - keeps the accepted rows of a tree: of the new rows that
 * foe_cache_append_tree stored behind the context, those that path[b] names become tokens
 * ctx_len[b], ctx_len[b] + 1, ... of sequence b, in place, and the others are dropped.
 *
 *   row_start [B+1], ctx_len [B]  int32   as in foe_cache_append_tree
 *   path      [B, max_path] int32   rows of the sequence, ascending (every row of a tree stands
 *                          behind its ancestors); the path ends at the first entry that does
 *                          not ascend or is no row of the sequence (-1)
 *   k_cache, v_cache, kv_scale   updated: in the pages from the context's end to the last
 *                          kept token's, the scales follow from the values that the page then
 *                          holds (the rule of foe_cache_evict: dropped rows no longer count), and
 *                          codes are rescaled to them.  Slots past the last kept token are left as
 *                          they were.  Nothing changes where no row is kept
 *   mass      [n_pages, H, 64] fp32   moves with its token, or NULL
 *   new_len   [B]   int32 out   ctx_len[b] and the length of the path (a buffer of its own)
 * A row whose page is absent is kept as a zero key and value without mass; rows that fall
 * into an absent page are lost.  1 <= max_path <= 2^22.  Needs no workspace.
 * A mass that was written with the whole tree holds the dropped rows' weights too, and
 * foe_cache_evict would rank the context by drafts that are no part of the text.  Where that
 * counts, verify the tree without a mass, accept the path, and add the kept rows' weights by
 * a causal call with the mass: foe_cache_attention (or _ex with the same cap and slope) of
 * their queries alone, with this call's ctx_len and the row_start of the paths.
 */
int foe_cache_accept(int H, int B, int hd, int n_pages, int max_blocks, int max_path,
                     const int32_t* row_start, const int32_t* ctx_len, const int32_t* path,
                     const int32_t* block_table, void* k_cache, void* v_cache, float* kv_scale,
                     float* mass, int32_t* new_len, void* stream);

/*
 * foe_cache_evict - keeps the tokens that received the most attention.  Of a
 * sequence longer than `keep`, each group keeps the last `recent` tokens and,
 * of those before, the keep - recent of largest mass (equal masses: the
 * earlier token; NaN ranks above infinity).  Groups choose for themselves.
 * The kept tokens, in their order, become tokens 0, 1, ... of the pages of
 * dst_table; shorter sequences are moved whole.  Each page's scales follow
 * from the values that it then holds, and mass moves with its token.  Tokens of
 * absent pages rank last; one that is kept all the same is stored as a zero key
 * and value without mass, which later queries see.
 *
 *   keep, recent           0 <= recent <= keep, 1 <= keep <= 2^30
 *   length    [B]          int32  tokens of each sequence
 *   k_cache, v_cache, kv_scale, mass   the pool: read at block_table's pages, written at
 *                          dst_table's, which must be other pages
 *   dst_table [B, dst_blocks] int32    64 * dst_blocks >= keep; slots past the kept tokens
 *                          are left as they were
 *   kept      [B, H, keep] int32 out   the kept tokens' former numbers, ascending; -1 past
 *                          a shorter sequence's end
 *   new_len   [B]          int32 out   min(length, keep)
 *   ws, ws_bytes           workspace of foe_cache_evict_workspace_bytes() (none for tables of
 *                          up to 512 pages)
 */
int foe_cache_evict(int H, int B, int hd, int n_pages, int max_blocks, int keep, int recent,
                    const int32_t* length, const int32_t* block_table, const int32_t* dst_table,
                    int dst_blocks, void* k_cache, void* v_cache, float* kv_scale, float* mass,
                    int32_t* kept, int32_t* new_len, void* ws, size_t ws_bytes, void* stream);

/* Workspace bytes of foe_cache_evict (SIZE_MAX for invalid sizes). */
size_t foe_cache_evict_workspace_bytes(int H, int B, int max_blocks);

/*
 * foe_workspace_bytes - workspace size in bytes for `op` (host string:
 * "route", "permute", "expert_ffn", "combine", "reduce", "cluster_block").
 * Arguments an op does not use are ignored (pass 0); for "expert_ffn" T is the
 * number of rows and k must be 1.  Returns 0 when the op needs no workspace and
 * SIZE_MAX for an unknown op or invalid sizes (foe_last_error() says which).
 */
size_t foe_workspace_bytes(const char* op, foe_dtype dt, int C, int T, int d,
                           int E, int k, int F);

/* Message for the calling thread's last failed call ("" if none). */
const char* foe_last_error(void);

/*
 * Kernel timing (for measurement).  While enabled, every kernel the library
 * enqueues carries two HIP events that its dispatch stamps at its start and
 * end (on the same stream); the records accumulate until foe_profile_reset().
 * Reading waits on the events.
 *   foe_profile_enable(1/0)          start / stop recording (returns FOE_OK)
 *   foe_profile_reset()              drop all records
 *   foe_profile_kernel(name, &n, &ms)  launches and summed milliseconds of the
 *                                    kernel `name` (host string); FOE_ERR_INVALID
 *                                    if no launch of that name was recorded
 *   foe_profile_names(buf, len)      comma-separated names recorded so far
 *                                    (host buffer); returns the length needed
 */
int foe_profile_enable(int on);
int foe_profile_reset(void);
int foe_profile_kernel(const char* name, int* launches, double* total_ms);
int foe_profile_names(char* buf, size_t len);

#ifdef __cplusplus
}
#endif

#endif /* FOE_H */
