/*
 * libcure -- MI355X (gfx950) verify-and-repair hot path of CURE
 * (local uncertainty repair for block-parallel speculative decoding).
 *
 * Stream-ordered entry points cover one decoding iteration's data-parallel
 * work on the device:
 *
 *   cure_margins    top-1/top-2 margin and log-sum-exp per logits row, plus the
 *                   Uncertainty Focal Point (UFP) selection      (Sec. 3.3, Eq. 2)
 *   cure_tree_attn  tree-masked verification attention over the KV cache and
 *                   each node's own tree ancestors           (Sec. 3.2, 3.4, 3.5)
 *   cure_accept     accepted prefix per path and the best path     (Eq. 1, Eq. 4)
 *   cure_margins_accept  cure_margins over a tree's node logits followed by
 *                   cure_accept on their argmaxes, in the margin pass's launches
 *   cure_repair_tree  the budget-aware repair tree: ranked alternatives at the
 *                   UFPs, the Eq. 3 branch budget and the parent/token arrays
 *                                                       (Sec. 3.3, 3.4, Alg. 1)
 *   cure_commit     the winning path committed: its cache rows moved after the
 *                   context in every layer, the emitted tokens, the new context
 *                   length and the draft-cache replay start   (Sec. 3.5, Alg. 1)
 *   cure_rope_append  new rows' queries and keys normalised per head and rotated
 *                   by their positions, keys and values written to the cache
 *   cure_prompt_attn  causal attention of whole prompts, chunks of them or single
 *                   tokens, packed without padding: what fills the context
 *   cure_prefix_attn  cure_tree_attn for sequences that share a prefix, whose
 *                   keys and values are read once for all of them
 *   cure_margins_noalloc  cure_margins for callers that cannot allocate: its
 *                   scratch is a fixed array inside the library
 *   cure_read_ceiling  not a step of the method: a plain streaming read, the
 *                   practical HBM read rate the other calls are compared with
 *
 * Conventions shared by every entry point
 *  - All array arguments are DEVICE pointers (memory the caller allocated with
 *    hipMalloc or equivalent), except those whose name starts with host_.
 *    The library allocates no device memory and keeps no state beyond a cached
 *    device-property query (and the static scratch array of
 *    cure_margins_noalloc, part of its code object); the caller owns every
 *    buffer.
 *  - stream is a hipStream_t passed as void* (NULL = the legacy default stream).
 *    Calls only enqueue work: they return before the work runs, and the outputs
 *    are valid once the stream reaches that point.
 *  - The return value reports errors the host can see: invalid arguments,
 *    unsupported shapes, a too-small workspace and HIP launch failures. Errors
 *    in device data (a malformed tree) are reported through device status words.
 *    No C++ exception crosses this interface.
 *  - Workspaces: a call that takes a workspace needs at least the size its
 *    *_workspace_size function returns for the same arguments (0 means none is
 *    needed and the pointer may be NULL). A workspace holds scratch data only
 *    while the call's kernels run: it needs no initialisation and may be reused
 *    by any later call on the same stream. Two calls whose work may overlap on
 *    the GPU must not share a workspace, and neither must two calls that threads
 *    make on one stream at the same time: a call enqueues several kernels, and
 *    the other's could come between them.
 *  - bf16 values are raw IEEE bfloat16 bit patterns (uint16 storage).
 */
#ifndef CURE_H
#define CURE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum cure_status {
  CURE_OK = 0,
  CURE_ERR_INVALID_ARG = 1,   /* null pointer, negative size, inconsistent shapes   */
  CURE_ERR_UNSUPPORTED = 2,   /* shape outside what the kernels implement            */
  CURE_ERR_BAD_TREE = 3,      /* device status word only: parent[n] not in [-1, n-1] */
  CURE_ERR_HIP = 4,           /* a HIP runtime call or kernel launch failed          */
  CURE_ERR_WORKSPACE = 5      /* workspace null or smaller than required             */
} cure_status;

typedef enum cure_dtype { CURE_F32 = 0, CURE_BF16 = 1 } cure_dtype;

/* Flags for cure_tree_attn. */
#define CURE_ATTN_FORCE_VALU 1u   /* use the vector-ALU kernel even where MFMA applies */

#define CURE_MAX_TREE_NODES 256   /* largest tree (nodes per sequence) supported       */

/* Human-readable name of a status code (static storage, never NULL). */
const char* cure_status_string(int status);

/* Library version as 10000*major + 100*minor + patch. */
int cure_version(void);

/* ------------------------------------------------------------------------- */
/* Margin pass and UFP gate -- Sec. 3.3 Eq. (2) and Algorithm 1.
 *
 * For every row r of logits (batch*rows rows of vocab entries; row r of
 * sequence b starts at element (b*rows + r)*ld):
 *   top1_idx/top1_val  the largest entry,
 *   top2_idx/top2_val  the next entry in the order (value descending, index
 *                      ascending) -- ties go to the lowest index, so a maximum
 *                      that occurs twice gives top2 = its second index,
 *   margin             top1_val - top2_val, computed in float32,
 *   lse                log(sum_v exp(x_v)), natural log, float32.
 * Entries are widened exactly to float32; values must be finite or -inf.
 *
 * UFP gate (skipped when ufp_pos and ufp_cnt are both NULL): over the first
 * chain_len rows of each sequence, the positions with margin < tau (strict),
 * ordered by (margin ascending, position ascending), at most
 * floor(repair_budget / branch_depth) of them, so that branches of branch_depth
 * nodes never exceed the repair budget. ufp_pos is [batch][chain_len] int32,
 * filled with the selected positions in that order and padded with -1;
 * ufp_cnt is [batch] int32.
 *
 * Layout: logits row-major, ld >= vocab elements between rows; every per-row
 * output has batch*rows entries. Requires vocab >= 2, 0 <= chain_len <= rows
 * (chain_len >= 1 when the gate runs), branch_depth >= 1, repair_budget >= 0.
 * workspace: cure_margins_workspace_size(batch, rows, vocab) bytes.
 */
size_t cure_margins_workspace_size(int32_t batch, int32_t rows, int32_t vocab);

cure_status cure_margins(const void* logits, int32_t dtype, int32_t batch, int32_t rows,
                         int32_t vocab, int64_t ld,
                         float* top1_val, int32_t* top1_idx, float* top2_val,
                         int32_t* top2_idx, float* lse, float* margin,
                         int32_t chain_len, float tau, int32_t repair_budget,
                         int32_t branch_depth, int32_t* ufp_pos, int32_t* ufp_cnt,
                         void* workspace, size_t workspace_bytes, void* stream);

/* Margin pass with the acceptance walk as its epilogue -- Sec. 3.3 Eq. (2),
 * Algorithm 1, Sec. 3.1 Eq. (1), Sec. 3.5 Eq. (4).
 *
 * For logits whose rows are the nodes of each sequence's candidate tree (row
 * n of sequence b = node n, so rows is the tree arrays' n_max): exactly
 * cure_margins(...) followed by cure_accept(parent, token, top1_idx, root_tgt,
 * n_nodes, chain_len, batch, rows, ...), with every output of both, bit for
 * bit. The walk runs in the workgroup that finishes each sequence's rows, so
 * the pair costs the margin pass's launches only (no separate acceptance
 * launch). chain_len serves the UFP gate (when ufp_pos/ufp_cnt are given) and
 * the walk's resync flag.
 *   parent, token  [batch][rows] int32;  root_tgt, n_nodes  [batch] int32
 *   acc_len, best, bonus, resync  [batch] int32;  path  [batch][rows] int32
 * Requires everything cure_margins requires, chain_len >= 0 and rows <= 256
 * (CURE_ERR_UNSUPPORTED otherwise). workspace: cure_margins_workspace_size(
 * batch, rows, vocab) bytes.
 */
cure_status cure_margins_accept(const void* logits, int32_t dtype, int32_t batch, int32_t rows,
                                int32_t vocab, int64_t ld,
                                float* top1_val, int32_t* top1_idx, float* top2_val,
                                int32_t* top2_idx, float* lse, float* margin,
                                int32_t chain_len, float tau, int32_t repair_budget,
                                int32_t branch_depth, int32_t* ufp_pos, int32_t* ufp_cnt,
                                const int32_t* parent, const int32_t* token,
                                const int32_t* root_tgt, const int32_t* n_nodes,
                                int32_t* acc_len, int32_t* path, int32_t* best,
                                int32_t* bonus, int32_t* resync,
                                void* workspace, size_t workspace_bytes, void* stream);

/* Allocation-free margin pass, for callers that cannot allocate device memory
 * (code under HIP stream capture, tight serving loops, harnesses that forbid
 * hipMalloc): the same pass, outputs and UFP gate as cure_margins, with no
 * workspace argument. Its scratch (the chunk results of rows split across
 * workgroups, 32 bytes per row and chunk) lives in a fixed device array of
 * cure_margins_noalloc_scratch_bytes() bytes (256 KiB) inside the library,
 * one per GPU the library runs on, held until the process ends. The call
 * itself allocates nothing; its first use on a device looks up that device's
 * copy of the array (hipGetSymbolAddress).
 * Returns CURE_ERR_UNSUPPORTED when the call would need more scratch than the
 * array holds (never on a 256-CU MI355X, whose plans need at most 32 KiB),
 * CURE_ERR_HIP when the array cannot be found on the current device, else as
 * cure_margins. Every call on one GPU shares that GPU's array and leaves its
 * contents behind: calls whose work may overlap on the GPU (different streams
 * without ordering between them) race and must not be issued, nor may two
 * threads be inside this call at the same time. */
size_t cure_margins_noalloc_scratch_bytes(void);

cure_status cure_margins_noalloc(const void* logits, int32_t dtype, int32_t batch,
                                 int32_t rows, int32_t vocab, int64_t ld,
                                 float* top1_val, int32_t* top1_idx, float* top2_val,
                                 int32_t* top2_idx, float* lse, float* margin,
                                 int32_t chain_len, float tau, int32_t repair_budget,
                                 int32_t branch_depth, int32_t* ufp_pos, int32_t* ufp_cnt,
                                 void* stream);

/* ------------------------------------------------------------------------- */
/* Tree-attention verification -- Sec. 3.2 (phase 3), Sec. 3.4, Sec. 3.5.
 *
 * One forward attention layer of the target over every node of each
 * sequence's candidate tree. Node n of sequence b, query head h (key/value head
 * h / (hq/hkv)) attends to
 *   - the ctx_len[b] cached context rows, and
 *   - the tree rows of the nodes on its own root path, itself included,
 * with scores scale * <q, k>, natural-base softmax:
 *   o[b][n][h]   = sum_j softmax_j * v_j            (normalised)
 *   lse[b][n][h] = log sum_j exp(scale * <q, k_j>)
 *
 * Layout:
 *   q       [batch][n_max][hq][d]          dtype
 *   k, v    token rows of [hkv][d]         dtype; sequence b owns rows
 *           kv_off[b] .. kv_off[b] + ctx_len[b] + n_nodes[b] - 1: its context,
 *           then its tree nodes in node order
 *   o       [batch][n_max][hq][d]          out_dtype (CURE_F32 or CURE_BF16)
 *   lse     [batch][n_max][hq]             float32 (may be NULL)
 *   parent  [batch][n_max]                 int32, parent[n] in [-1, n-1]: the
 *           tree in topological order, -1 = attached to the context
 *   kv_off  [batch] int64, ctx_len/n_nodes [batch] int32 (device)
 *   host_ctx_len/host_n_nodes: host copies of ctx_len/n_nodes, used only to
 *           plan the split of each context across workgroups.
 * Rows n >= n_nodes[b] of o and lse are not written.
 * tree_status [batch] int32 (may be NULL): CURE_OK (also for a sequence with
 * no nodes), or CURE_ERR_BAD_TREE when sequence b's parent array is malformed
 * (that sequence's o/lse are then unspecified).
 * Supports d in {64, 128}, hq % hkv == 0, 0 <= n_nodes[b] <= min(n_max, 256)
 * (a sequence with no nodes is skipped).
 * kv_split: 0 = automatic, else the number of context splits per sequence.
 * flags: CURE_ATTN_FORCE_VALU or 0.
 * workspace: cure_tree_attn_workspace_size(...) bytes for the same arguments.
 *   It holds each context split's fp32 partial rows and their log-sum-exps;
 *   the splits are combined by a log-sum-exp merge.
 * Alignment (else CURE_ERR_INVALID_ARG): workspace 16 bytes; on the bf16
 * matrix-core path (bf16 inputs, d 64 or 128, scale > 0, no FORCE_VALU) also
 * q, k, v 16 bytes and o 8 bytes (bf16 out) or 16 bytes (fp32 out).
 * fp32 inputs run on the fp32 matrix instructions when q, k, v and o have that
 * alignment, and on the vector-ALU kernel otherwise.
 * The bf16 matrix-core kernels address a sequence's rows with 32-bit offsets:
 * (ctx_len + n_nodes + 64) * hkv * d * 2 bytes must stay below 2^31. Calls whose
 * host copies reach that take the vector-ALU kernel; where the device's sizes
 * exceed the host's copies, they must not pass it.
 */
size_t cure_tree_attn_workspace_size(int32_t batch, int32_t hq, int32_t hkv, int32_t d,
                                     int32_t n_max, const int32_t* host_ctx_len,
                                     const int32_t* host_n_nodes, int32_t kv_split);

cure_status cure_tree_attn(const void* q, const void* k, const void* v, void* o, float* lse,
                           int32_t dtype, int32_t out_dtype, int32_t batch, int32_t hq,
                           int32_t hkv, int32_t d, float scale, const int64_t* kv_off,
                           const int32_t* ctx_len, const int32_t* n_nodes,
                           const int32_t* parent, int32_t n_max,
                           const int32_t* host_ctx_len, const int32_t* host_n_nodes,
                           int32_t kv_split, uint32_t flags, int32_t* tree_status,
                           void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------- */
/* Acceptance walk -- Sec. 3.1 Eq. (1), Sec. 3.5 Eq. (4), greedy decoding.
 *
 * Per sequence b with n_nodes[b] nodes (all arrays [batch][n_max] int32 unless
 * noted):
 *   node n is accepted when its token equals the target's argmax before it --
 *   root_tgt[b] for parent[n] == -1, else tgt[parent[n]] -- and its parent is
 *   accepted. The winner is the accepted node of greatest depth, lowest index
 *   on ties (so branch 0, numbered first, wins ties).
 *   acc_len [batch]  depth(winner)+1, or 0 when nothing is accepted
 *   best    [batch]  the winner, or -1
 *   path    [batch][n_max] root->winner node indices, padded with -1
 *   bonus   [batch]  tgt[winner], or root_tgt[b] when nothing is accepted
 *   resync  [batch]  1 when the winning path holds a node >= chain_len (a repair
 *                    node, so the draft cache must be resynchronised), else 0;
 *                    -1 together with acc_len = -1 when the parent array is
 *                    malformed.
 * tgt is typically cure_margins' top1_idx over the target's node logits.
 * Supports 0 <= n_nodes[b] <= min(n_max, 256); with no nodes, acc_len = 0
 * and bonus = root_tgt.
 */
cure_status cure_accept(const int32_t* parent, const int32_t* token, const int32_t* tgt,
                        const int32_t* root_tgt, const int32_t* n_nodes, int32_t chain_len,
                        int32_t batch, int32_t n_max, int32_t* acc_len, int32_t* path,
                        int32_t* best, int32_t* bonus, int32_t* resync, void* stream);

/* ------------------------------------------------------------------------- */
/* Repair-tree construction -- Sec. 3.3 Eq. (3), Sec. 3.4, Algorithm 1.
 *
 * Builds each sequence's candidate tree from its draft block (branch 0) and
 * the UFPs that cure_margins selected. For UFP slot s (in the given,
 * ascending-margin order) at block position u = ufp_pos[b][s]:
 *   ranked      the draft row's entries in the order (value descending, index
 *               ascending), read from logits row u of sequence b;
 *   alternatives the ranked tokens other than chain_tok[b][u], best first;
 *   b_s         Eq. (3) on margin m = margin[b*rows + u]:
 *                 t = b_min + clip(1 - m / margin_scale, 0, 1) * (b_max - b_min)
 *                 b_s = clip(round_half_even(t), b_min, b_max)
 *               in float32, every operation rounded once; a NaN margin counts
 *               as certain (b_s = b_min);
 *   granted     min(b_s, remaining / branch_depth): whole branches only,
 *               remaining starting at repair_budget, slots taken in order.
 * Branch r of slot s is a chain of branch_depth nodes: its root carries
 * alternative r and hangs off chain node u - 1 (-1, the context, when u = 0);
 * node j > 0 carries suffix[b][u][r][j-1] (the token the drafter proposed
 * after that substitution) or -1 when suffix is NULL, and hangs off node j - 1.
 *
 * Node numbering (the tree is in topological order): nodes 0 .. chain_len-1 are
 * the chain (parent[i] = i - 1, token = chain_tok); then the branches, slot by
 * slot and within a slot by alternative rank, each branch's nodes consecutive.
 *
 * Layout:
 *   logits     [batch][rows][ld] dtype (the draft block's rows; the first
 *              chain_len rows of each sequence are the chain positions)
 *   margin     [batch][rows] float32, as cure_margins wrote it
 *   ufp_pos    [batch][chain_len] int32, ufp_cnt [batch] int32, as cure_margins
 *              wrote them (the slots used are the first min(ufp_cnt,
 *              repair_budget / branch_depth), cut at the first position
 *              outside [0, chain_len))
 *   chain_tok  [batch][chain_len] int32, the draft block
 *   suffix     [batch][chain_len][b_max][branch_depth-1] int32, or NULL
 *   parent, token  [batch][n_max] int32 outputs; entries at or past
 *              n_nodes[b] are not written
 *   n_nodes    [batch] int32 output: chain_len + branch_depth * (branches)
 *   branch_cnt [batch][chain_len] int32 output (may be NULL): branches granted
 *              per slot, 0 for unused slots
 * Requires 1 <= chain_len <= min(rows, 1024), branch_depth >= 1,
 * repair_budget >= 0, 0 <= b_min <= b_max <= 7, b_max >= 1,
 * vocab >= b_max + 1, vocab <= 524288, ld >= vocab, margin_scale > 0 and
 * finite, n_max >= chain_len + repair_budget (so every tree fits).
 * workspace: cure_repair_tree_workspace_size(...) bytes for the same arguments.
 */
size_t cure_repair_tree_workspace_size(int32_t batch, int32_t chain_len, int32_t vocab,
                                       int32_t repair_budget, int32_t branch_depth);

cure_status cure_repair_tree(const void* logits, int32_t dtype, int32_t batch, int32_t rows,
                             int32_t vocab, int64_t ld, const float* margin,
                             const int32_t* ufp_pos, const int32_t* ufp_cnt,
                             const int32_t* chain_tok, int32_t chain_len,
                             int32_t repair_budget, int32_t branch_depth, float margin_scale,
                             int32_t b_min, int32_t b_max, const int32_t* suffix,
                             int32_t n_max, int32_t* parent, int32_t* token, int32_t* n_nodes,
                             int32_t* branch_cnt, void* workspace, size_t workspace_bytes,
                             void* stream);

/* ------------------------------------------------------------------------- */
/* Committing the winning path -- Sec. 3.5 (cache resynchronisation), Alg. 1.
 *
 * The accepted tokens become context for the next step. For each sequence b
 * with a = acc_len[b] accepted nodes and winning path path[b][0 .. a-1] (node
 * indices, root first, as cure_accept writes them):
 *   cache       in every layer, cache row kv_off[b] + ctx_len[b] + j takes
 *               the contents of row kv_off[b] + ctx_len[b] + path[b][j], for
 *               j < a (tree node n's rows sit at ctx_len + n, as for
 *               cure_tree_attn), in K and in V. The move is in place; rows from
 *               ctx_len + a on keep whatever they held.
 *   new_ctx_len [batch] ctx_len[b] + a
 *   emit        [batch][n_max + 1] the a accepted tokens token[b][path[b][j]],
 *               then bonus[b], padded with -1
 *   emit_cnt    [batch] a + 1
 *   replay_start [batch] depth of the path's first node numbered >= chain_len
 *               (a repair node), else a: the emitted tokens from there to a-1
 *               are the ones to replay into the draft model's cache
 *   commit_status [batch] CURE_OK, or CURE_ERR_BAD_TREE when the sequence is
 *               not committable: acc_len < 0 (cure_accept's mark of a malformed
 *               tree), acc_len > n_nodes, n_nodes outside [0, n_max], a
 *               negative ctx_len or kv_off, or a path entry outside
 *               [0, n_nodes) or not above its predecessor. Such a sequence's
 *               cache is left untouched, new_ctx_len = ctx_len, emit_cnt = 0,
 *               replay_start = 0 and its emit row is all -1.
 *
 * Layout:
 *   k, v       n_layers caches; layer l's starts at element l * layer_stride
 *              of k and of v and holds token rows of [hkv][d] dtype elements
 *              (layer_stride is ignored when n_layers <= 1)
 *   kv_off [batch] int64, ctx_len, n_nodes, acc_len, bonus [batch] int32,
 *   path, token [batch][n_max] int32 -- all device memory
 * Requires hkv * d * sizeof(dtype) to be a multiple of 16 bytes, n_max <= 256,
 * batch <= 65535. Outputs must not overlap the inputs (new_ctx_len may not be
 * ctx_len itself: other workgroups still read ctx_len while it is written).
 * Every cache row kv_off[b] .. kv_off[b] + ctx_len[b] + n_nodes[b] - 1 of
 * every layer must exist. No workspace.
 */
cure_status cure_commit(void* k, void* v, int32_t dtype, int32_t n_layers, int64_t layer_stride,
                        int32_t hkv, int32_t d, int32_t batch, const int64_t* kv_off,
                        const int32_t* ctx_len, const int32_t* n_nodes, const int32_t* path,
                        const int32_t* acc_len, const int32_t* token, const int32_t* bonus,
                        int32_t chain_len, int32_t n_max, int32_t* new_ctx_len, int32_t* emit,
                        int32_t* emit_cnt, int32_t* replay_start, int32_t* commit_status,
                        void* stream);

/* ------------------------------------------------------------------------- */
/* Rotary positions and the cache rows of new tokens -- what an attention layer
 * does before cure_tree_attn or cure_prompt_attn can read its keys and values.
 *
 * For the n_rows[b] new rows of each sequence b (a prompt's tokens, or the nodes
 * of a candidate tree), row n of it:
 *   queries, keys  every head x of d columns is normalised where a weight is given,
 *                    x^ = x * rsqrt(mean(x^2) + eps) * weight,
 *                  and its first rot columns rotated in pairs (a, b) by the angle
 *                  t = pos * inv_freq[i]:
 *                    y_a = mscale * (x^_a cos t - x^_b sin t)
 *                    y_b = mscale * (x^_a sin t + x^_b cos t)
 *                  where pair i is columns (i, i + rot/2), or (2i, 2i + 1) with
 *                  CURE_ROPE_INTERLEAVED; columns from rot on are not rotated.
 *   pos            pos_off[b] + ctx_len[b] + n, or with a tree
 *                  pos_off[b] + ctx_len[b] + depth(n) (a root has depth 0), the
 *                  position that the node has once cure_commit has moved its path
 *   q_out          [row][hq][d] takes the queries, at the row that they came from
 *   k_cache, v_cache  row kv_off[b] + ctx_len[b] + n takes the keys and the values
 * Arithmetic in float32 (the angle's reduction in float64), one rounding at the end.
 *
 * Layout:
 *   q, k, v    rows of [hq][d], [hkv][d], [hkv][d] dtype elements, q_ld, k_ld and
 *              v_ld elements apart (so they may lie in one fused projection's
 *              output). Sequence b's first row is row_off[b], or b * n_max where
 *              row_off is NULL (rows padded to n_max per sequence). hq = 0: no
 *              queries, q and q_out are ignored; hkv = 0: no keys and values.
 *   n_rows     [batch] int32, at most n_max
 *   parent     [batch][n_max] int32 as for cure_tree_attn, or NULL: a sequence
 *   row_off, kv_off  [batch] int64;  ctx_len, pos_off  [batch] int32 (pos_off may be
 *              NULL: 0)
 *   q_weight, k_weight  [d] dtype, each may be NULL: not normalised
 *   inv_freq   [rot/2] float32 (cure_rope_frequencies computes the usual ones)
 *   rows       rows that q, k, v and q_out hold;  cache_rows  rows of the caches
 *   row_status [batch] int32 output: CURE_OK, or CURE_ERR_BAD_TREE when the
 *              sequence's parent array is malformed, its sizes are negative,
 *              n_rows exceeds n_max, or its rows or (where hkv > 0) cache rows reach past
 *              rows or cache_rows. Nothing of such a sequence is written.
 * q_out may be q itself where q_ld = hq * d. Rows and cache rows of different
 * sequences must not overlap, and q, k and v must not overlap the cache rows written.
 * Rows that belong to no sequence are not written.
 * n_max sizes the launch: with row_off, give the longest n_rows rather than all rows.
 * Supports d a multiple of 16 up to 256, rot a multiple of 16 up to d, n_max <= 256
 * with a tree, n_max (with row_off: n_max or rows) < 2^26 - 3, batch <= 65535. All row
 * pointers, weights and row distances must be multiples of 16 bytes (else
 * CURE_ERR_INVALID_ARG). No workspace.
 */
#define CURE_ROPE_INTERLEAVED 1u

cure_status cure_rope_append(const void* q, int64_t q_ld, const void* k, int64_t k_ld,
                             const void* v, int64_t v_ld, int32_t dtype, int64_t rows,
                             int32_t batch, int32_t n_max, const int64_t* row_off,
                             const int32_t* n_rows, const int32_t* parent,
                             const int64_t* kv_off, const int32_t* ctx_len,
                             const int32_t* pos_off, int32_t hq, int32_t hkv, int32_t d,
                             const void* q_weight, const void* k_weight, float eps,
                             const float* inv_freq, int32_t rot, uint32_t flags, float mscale,
                             void* q_out, void* k_cache, void* v_cache, int64_t cache_rows,
                             int32_t* row_status, void* stream);

/* Frequencies of a rotation over rot columns, computed on the host in float64:
 * f_i = base^(-2i/rot), i < rot/2, changed for contexts longer than the trained one
 * (factor >= 1 times as long; orig_len tokens where it is used) by scaling:
 *   CURE_ROPE_PLAIN   not at all
 *   CURE_ROPE_LINEAR  f_i / factor
 *   CURE_ROPE_BASE    base * factor^(rot/(rot-2)) in place of base
 *   CURE_ROPE_BANDS   by the turns u = orig_len * f_i / 2 pi that a pair makes: kept
 *                     from u >= p1 on, f_i / factor up to u <= p0, blended linearly in
 *                     u between (0 < p0 < p1, usually 1 and 4)
 *   CURE_ROPE_RAMP    by the pair's index: kept before the pair that makes p0 turns,
 *                     f_i / factor from the one that makes p1 (p0 > p1 > 0, usually 32
 *                     and 1), a linear ramp between; mscale = 0.1 ln(factor) + 1
 * Writes host_inv_freq [rot/2] and host_mscale (1 except for CURE_ROPE_RAMP), both
 * host memory. rot even and >= 0, base > 1.
 */
enum { CURE_ROPE_PLAIN = 0, CURE_ROPE_LINEAR = 1, CURE_ROPE_BASE = 2, CURE_ROPE_BANDS = 3,
       CURE_ROPE_RAMP = 4 };

cure_status cure_rope_frequencies(int32_t rot, double base, int32_t scaling, double factor,
                                  double orig_len, double p0, double p1, float* host_inv_freq,
                                  float* host_mscale);

/* ------------------------------------------------------------------------- */
/* Attention over prompts: causal, grouped heads, packed sequences.
 *
 * New token i < n_rows[b] of sequence b attends, in every query head h (key/value
 * head h / (hq/hkv)), to the cache rows kv_off[b] .. kv_off[b] + ctx_len[b] + i: the
 * context before it and the new tokens up to itself, whose keys and values are in the
 * cache already (cure_rope_append). Whole prompts have ctx_len 0, chunks of long
 * ones and single tokens what came before.
 *   o[r][h]   = sum_j softmax_j * v_j,  r = row_off[b] + i
 *   lse[r][h] = log sum_j exp(scale * <q, k_j>)
 *
 * Layout:
 *   q, o       [rows][hq][d] dtype / out_dtype; sequence b's rows are row_off[b] ..
 *              row_off[b] + n_rows[b] - 1; other rows of o and lse are not written
 *   k, v       cache rows of [hkv][d] dtype
 *   lse        [rows][hq] float32 (may be NULL)
 *   row_off, kv_off  [batch] int64;  n_rows, ctx_len  [batch] int32 (device)
 *   host_n_rows, host_ctx_len  host copies that the launch is planned from. The
 *              device's n_rows may be smaller (a captured call replayed on shorter
 *              prompts), not larger: tokens past the host's longest n_rows may get no
 *              output. ctx_len may differ either way. A sequence whose ctx_len is negative
 *              or whose rows do not lie within `rows` on the device is taken as empty.
 * The values that a row sees must be finite; keys and values after it (later
 * tokens, and whatever the cache holds behind the sequence) may be anything.
 * Supports d in {64, 128}, hq % hkv == 0, scale > 0 with scale * log2(e) finite,
 * batch <= 65535, n_rows * hq up to 2^28. o may be q where their types are one.
 * kv_split: 0 = automatic, else the number of splits of the longest context (fewer where
 * that has not as many steps of keys).
 * workspace: cure_prompt_attn_workspace_size(...) bytes for the same arguments,
 * 16-byte aligned, as q, k, v and o are. Beyond 1 GB it has room for the splits of the
 * host's sizes only; a sequence that is longer on the device is then computed in one split.
 * bf16: probabilities are rounded to bf16 for their product and lse sums the rounded
 * ones (within 2^-8 of the exact sum). float32: float32 throughout.
 */
size_t cure_prompt_attn_workspace_size(int32_t batch, int64_t rows, int32_t hq, int32_t hkv,
                                       int32_t d, const int32_t* host_n_rows,
                                       const int32_t* host_ctx_len, int32_t kv_split);

cure_status cure_prompt_attn(const void* q, const void* k, const void* v, void* o, float* lse,
                             int32_t dtype, int32_t out_dtype, int32_t batch, int64_t rows,
                             int32_t hq, int32_t hkv, int32_t d, float scale,
                             const int64_t* row_off, const int32_t* n_rows,
                             const int64_t* kv_off, const int32_t* ctx_len,
                             const int32_t* host_n_rows, const int32_t* host_ctx_len,
                             int32_t kv_split, void* workspace, size_t workspace_bytes,
                             void* stream);

/* Tree attention over a shared prefix: cure_tree_attn for a batch whose sequences all
 * begin with the same prefix_len tokens, stored once in cache rows prefix_off ..
 * prefix_off + prefix_len - 1. Node n of sequence b attends to those, to its
 * sequence's own ctx_len[b] rows from kv_off[b] on and to the tree rows on its root
 * path behind them. The prefix is read once for all nodes of all sequences, the own
 * rows by workgroups of the same launch, and log-sum-exps join the two.
 * Arguments, layout and outputs as for cure_tree_attn (ctx_len counts a sequence's
 * own rows only; the position of a node is prefix_len + ctx_len + depth, which
 * cure_rope_append's pos_off = prefix_len gives). prefix_len = 0 is cure_tree_attn.
 * kv_split: splits of the prefix, 0 = automatic.
 * A malformed tree is reported in tree_status, and that sequence's o and lse are then
 * unspecified. Where prefix_len > 0 a ctx_len that is negative on the device is reported as
 * well, and that sequence's o and lse are not written. The values that a node sees must be
 * finite; what it does not see may be anything. The device's n_nodes and ctx_len may differ
 * from the host's copies (n_nodes up to n_max).
 * Supports a scale as cure_prompt_attn, and where prefix_len > 0 batch <= 1024,
 * batch * n_max * hq/hkv below 2^31 - 4096, batch * n_max * hq up to 2^27 and batch * hkv
 * up to 2^22, and what cure_tree_attn supports. Alignment as for
 * cure_prompt_attn. workspace: cure_prefix_attn_workspace_size(...) bytes for the same
 * arguments; as there beyond 1 GB, where a sequence with more nodes or own rows on the device
 * has its own rows in one split.
 */
size_t cure_prefix_attn_workspace_size(int32_t batch, int32_t hq, int32_t hkv, int32_t d,
                                       int32_t n_max, int32_t prefix_len,
                                       const int32_t* host_ctx_len,
                                       const int32_t* host_n_nodes, int32_t kv_split);

cure_status cure_prefix_attn(const void* q, const void* k, const void* v, void* o, float* lse,
                             int32_t dtype, int32_t out_dtype, int32_t batch, int32_t hq,
                             int32_t hkv, int32_t d, float scale, int64_t prefix_off,
                             int32_t prefix_len, const int64_t* kv_off, const int32_t* ctx_len,
                             const int32_t* n_nodes, const int32_t* parent, int32_t n_max,
                             const int32_t* host_ctx_len, const int32_t* host_n_nodes,
                             int32_t kv_split, int32_t* tree_status, void* workspace,
                             size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------- */
/* Read ceiling -- a measurement aid, not a step of the method.
 *
 * Streams `bytes` of device memory (a multiple of 16) the way the margin pass
 * streams its rows: one workgroup per 256 KB chunk, 16-byte non-temporal
 * loads. Writes the XOR of each chunk's 32-bit words to chunk_xor[i] (device,
 * cure_read_ceiling_chunks(bytes) entries), so the read is needed and can be
 * checked. Its time is the practical HBM read rate the hot path's bandwidth is
 * compared against.
 */
size_t cure_read_ceiling_chunks(size_t bytes);

cure_status cure_read_ceiling(const void* buf, size_t bytes, uint32_t* chunk_xor, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CURE_H */
