/*
 * fsd.h -- C ABI of the MI355X (gfx950) candidate-verification library for
 * Fuzzy Speculative Decoding (FSD).
 *
 * One call verifies, for a batch of sequences, every candidate position a
 * draft model proposed: it turns the target-model and draft-model logits of
 * each position into next-token distributions, measures the divergence
 * between them, accepts the position when the divergence is within the
 * threshold T, finds the accepted prefix (or accepted tree path) and draws the
 * one extra token from the target distribution.
 *
 * Conventions shared by all entry points
 *   - Every tensor pointer is a DEVICE pointer owned by the caller; the
 *     library never allocates, frees or keeps it.  Tensors are dense and
 *     row-major.  Logits are binary32 (FSD_F32) or bfloat16 (FSD_BF16).
 *     Rows that start on 16-byte boundaries (V * element size a multiple of
 *     16 and aligned base pointers) are read fastest; any other alignment of
 *     whole elements is read with 128-bit loads as well.
 *   - -inf logits are legal (masked vocabulary entries).  A NaN or +inf logit,
 *     or a row that is -inf everywhere, in a row the method reads is reported
 *     per sequence in row_status (FSD_ROW_NONFINITE): that sequence gets
 *     accept_len / path_len 0, all its output tokens -1 and NaN divergences
 *     for the affected positions.
 *   - Calls are asynchronous on `hip_stream` (a hipStream_t, NULL = the null
 *     stream), do no host synchronisation and no host<->device copy.
 *   - `workspace` is device memory of at least fsd_workspace_bytes(...) bytes,
 *     256-byte aligned, private to the call while it runs; its contents need
 *     no initialisation and mean nothing afterwards.
 *   - The return value is an fsd_status.  Argument errors are found before
 *     anything is launched and leave all outputs untouched.
 *   - The vocabulary-reduction kernel is persistent: the wavefronts that share a
 *     row pair wait for each other's partial results, so its grid is sized to
 *     what an otherwise idle device holds at once.  So do the workgroups that
 *     share a sequence in two kernels after it: the walk of strict SD over a
 *     tree, and the selection of a warped call under top_p without top_k
 *     where it splits a long row.  (The draw's workgroups wait for nobody but
 *     the last of a sequence, which looks for the shares of those dispatched
 *     before it, and so does not depend on what else is resident.)  If other work occupies the
 *     GPU while a call runs (another stream, another process), some of its
 *     workgroups may start late; every wait is bounded (by
 *     1<<22 polls; see fsd_debug_set_spin_limit), and a wait that expires ends the call with
 *     FSD_ROW_INTERNAL in row_status for every sequence (lengths 0, tokens -1;
 *     a plain FSD call on a few sequences, which is one kernel, for every
 *     sequence it concerns) instead of hanging.  Run verify calls on a GPU that is theirs while they
 *     run, and treat FSD_ROW_INTERNAL as "call again".
 *   - Random numbers: Philox4x32-10 keyed by `seed`; `offset` selects the
 *     decode step (counter words 2,3), the sequence index is counter word 1 and
 *     the vocabulary (or position) index picks counter word 0 and the lane.
 *     Equal (seed, offset, inputs) give equal outputs on every launch.
 */
#ifndef FSD_H_
#define FSD_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    FSD_OK = 0,
    FSD_ERR_NULL = -1,      /* a required pointer is NULL */
    FSD_ERR_SHAPE = -2,     /* B, K, N, V, max_depth out of range, or T is NaN */
    FSD_ERR_DTYPE = -3,     /* dtype is not an fsd_dtype */
    FSD_ERR_DIV = -4,       /* div is not an fsd_div */
    FSD_ERR_WORKSPACE = -5, /* workspace NULL, misaligned or too small */
    FSD_ERR_MODE = -6,      /* mode is not an fsd_mode */
    FSD_ERR_LAUNCH = -7,    /* the HIP runtime refused a launch */
    FSD_ERR_TOO_LARGE = -8, /* fsd_verify_chain_static: sizes beyond its fixed scratch buffer */
    FSD_ERR_LAYOUT = -9     /* a stride, an alignment or an overlap that the call does not take */
} fsd_status;

/* (FSD_F16: queries, keys and values of fsd_attend_* and fsd_cache_append only; logits are FSD_F32 or FSD_BF16.) */
typedef enum { FSD_F32 = 0, FSD_BF16 = 1, FSD_F16 = 2 } fsd_dtype;

/* Divergence between the target distribution p and the draft distribution q
 * (paper App. C): KL is KL(p || q) (C.1), JS the Jensen-Shannon divergence
 * with the even mixture (C.2), TV the total-variation distance (C.3).
 * Natural logarithm. */
typedef enum { FSD_DIV_KL = 0, FSD_DIV_JS = 1, FSD_DIV_TV = 2 } fsd_div;

/* How the extra token is drawn from the target row (paper Sec. 4, "whatever
 * sampling method the user sets", and Sec. 6.3): an exact categorical draw
 * from softmax(logits) by Gumbel-max, or the argmax (lowest index on ties). */
typedef enum { FSD_SAMPLE = 0, FSD_GREEDY = 1 } fsd_mode;

/* bits of row_status[b] */
enum {
    FSD_ROW_NONFINITE = 1,  /* NaN / +inf / all -inf row among the rows read */
    FSD_ROW_BAD_PARENT = 2, /* tree: parent[j] outside [-1, j) */
    FSD_ROW_TOO_DEEP = 4,   /* tree: a node deeper than max_depth */
    FSD_ROW_BAD_TOKEN = 8,  /* strict SD: candidate token id outside [0, V) */
    FSD_ROW_INTERNAL = 16,  /* a bounded device-side wait expired (never expected) */
    FSD_ROW_BAD_CACHE = 32, /* cache calls: a length, block number, path node or position outside its range */
    FSD_ROW_NO_BLOCKS = 64  /* fsd_cache_fork: the cache has too few free blocks */
};

/* Limits: 1 <= V <= fsd_max_vocab(dtype) (524288 for both dtypes); 1 <= K, N,
 * max_depth <= 2048; 1 <= B <= 65535; B*K (B*N) < 2^24. */
int64_t fsd_max_vocab(int dtype);

/* Bytes of workspace a call with these sizes needs (rows_per_seq = K or N).
 * Returns 0 for arguments no call would accept. */
size_t fsd_workspace_bytes(int B, int rows_per_seq, int V, int dtype);

const char* fsd_status_string(int status);

/*
 * FSD verification of linear candidate sequences (paper Sec. 4, eq. 4).
 *
 *   target_logits [B, K+1, V]  row i < K: target model's logits for position i;
 *                              row K: the position after the last candidate
 *   draft_logits  [B, K, V]    draft model's logits for position i
 *   cand_tokens   [B, K]       the K candidate token ids (copied to the output;
 *                              the FSD decision does not depend on them)
 *   div, T                     accept position i iff div(p_i, q_i) <= T
 *                              (T may be +-inf; NaN is rejected)
 *   accept_len    [B]   out    n_b = number of leading accepted positions
 *   out_tokens    [B, K+1] out cand[b, :n_b], then the token drawn from
 *                              softmax(target[b, n_b]), then -1 padding
 *   divergences   [B, K] out   optional (NULL to skip), the chosen divergence.
 *                              p and q are evaluated in binary32: the value is
 *                              within 1e-5 (binary32 logits) or 2e-3 (bfloat16)
 *                              relative of the exact one from 2e-2 (binary32)
 *                              or 1e-4 (bfloat16) upwards; below that (nearly
 *                              equal rows) its ABSOLUTE error stays under
 *                              2.5e-7, measured on rows that differ by noise of
 *                              0.001 to 0.3, and bit-identical rows give 0
 *   row_status    [B]   out    optional (NULL to skip), see FSD_ROW_*
 *
 * A call only enqueues kernels on hip_stream (what it needs clear in the
 * workspace is cleared by its kernels, never by a memset), so it may be
 * recorded into a HIP graph; seed and offset are then part of the recording.
 */
int fsd_verify_chain(const void* target_logits, const void* draft_logits, const int32_t* cand_tokens,
                     int B, int K, int V, int dtype, int div, float T, int mode, uint64_t seed,
                     uint64_t offset, int32_t* accept_len, int32_t* out_tokens, float* divergences,
                     int32_t* row_status, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * fsd_verify_chain for callers that cannot allocate device memory or pass a
 * workspace: code under HIP graph capture, tight serving loops, harnesses that
 * forbid hipMalloc.  Same inputs, outputs, kernels and results as
 * fsd_verify_chain; the workspace is a buffer of FSD_STATIC_SCRATCH_BYTES bytes
 * that is part of the loaded library (one copy per GPU, held until the process
 * ends).  The call allocates and frees nothing.
 *
 *   - Sizes whose fsd_workspace_bytes(B, K, V, dtype) exceeds
 *     FSD_STATIC_SCRATCH_BYTES are refused with FSD_ERR_TOO_LARGE before
 *     anything is launched (B=64, K=8, V=128256 bfloat16 needs 2.1 MiB).
 *   - Every call on a GPU uses that GPU's one buffer, which keeps the last
 *     call's contents; the call clears what it needs cleared itself.  Calls that
 *     overlap in time on one GPU (different streams, or threads) race on it:
 *     keep them on one stream or serialise them.
 */
#define FSD_STATIC_SCRATCH_BYTES (4u << 20)
int fsd_verify_chain_static(const void* target_logits, const void* draft_logits, const int32_t* cand_tokens,
                            int B, int K, int V, int dtype, int div, float T, int mode, uint64_t seed,
                            uint64_t offset, int32_t* accept_len, int32_t* out_tokens, float* divergences,
                            int32_t* row_status, void* hip_stream);

/*
 * FSD verification of a token tree (paper Sec. 6.4: FSD on top of a
 * tree-drafting method; the rule below is this library's statement of it).
 *
 *   target_logits [B, N+1, V]  row 0: target logits at the root context;
 *                              row j+1: at the context that ends with node j
 *   draft_logits  [B, N, V]    row j: the draft logits node j was proposed from
 *   node_tokens   [B, N]       token id of node j
 *   parent        [B, N]       parent node of j, -1 for children of the root;
 *                              parent[j] < j (checked on the device)
 *   max_depth                  longest path the outputs can hold
 *
 * Node j is accepted iff div(softmax(target[parent[j]+1]), softmax(draft[j])) <= T
 * and its parent is accepted.  The deepest accepted node wins (lowest index on
 * ties); the extra token is drawn from the target row of the winner's context
 * (row 0 when no node is accepted).
 *
 *   path_len   [B]              out  depth of the winner (0 = none)
 *   path_nodes [B, max_depth]   out  node indices root-to-winner, -1 padded
 *   out_tokens [B, max_depth+1] out  tokens of the path, the drawn token, -1 padding
 *   divergences [B, N] out optional; row_status [B] out optional
 */
int fsd_verify_tree(const void* target_logits, const void* draft_logits, const int32_t* node_tokens,
                    const int32_t* parent, int B, int N, int max_depth, int V, int dtype, int div,
                    float T, int mode, uint64_t seed, uint64_t offset, int32_t* path_len,
                    int32_t* path_nodes, int32_t* out_tokens, float* divergences, int32_t* row_status,
                    void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Strict speculative decoding on the same tensors (paper Sec. 3, eq. 1-3), the
 * baseline FSD generalises: position i is accepted iff min(1, p_i(x_i)/q_i(x_i)) > y_i
 * with y_i uniform in (0,1) from the Philox stream; at the first rejection the
 * token is drawn from the normalised positive part of p - q, and from the row
 * after the last candidate when everything is accepted.
 *
 *   log_ratio [B, K] out  optional, ln p_i(x_i) - ln q_i(x_i)
 */
int sd_verify_chain(const void* target_logits, const void* draft_logits, const int32_t* cand_tokens,
                    int B, int K, int V, int dtype, int mode, uint64_t seed, uint64_t offset,
                    int32_t* accept_len, int32_t* out_tokens, float* log_ratio, int32_t* row_status,
                    void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Strict speculative decoding over a token tree: the tree analogue of
 * sd_verify_chain, for the tree-structured proposals of the methods the paper's
 * Sec. 2 cites (item 1) and Sec. 6.4 builds on.  The paper gives no procedure
 * of its own; this is the multi-round rejection rule of that family on the
 * tensors of fsd_verify_tree.  At the current context, with target
 * distribution p, the children are tried in index order: child j is accepted
 * iff min(1, p(x_j)/q_j(x_j)) > y_j (Sec. 3, eq. 1-2; y_j the uniform number
 * of index j) and the walk moves to the context after node j; after a
 * rejection p becomes the normalised positive part of p - q_j (Sec. 3, eq. 3)
 * before the next child is tried.  When no child is accepted the token is
 * drawn from the p in force: the target row itself at a node without
 * children, otherwise the residual of the last rejection.  Every emitted
 * token then follows the target distribution of its context.  With one child
 * per node the outputs are sd_verify_chain's.
 *
 *   inputs and path_len / path_nodes / out_tokens / row_status as in fsd_verify_tree
 *   log_ratio [B, N] out  optional: ln p(x_j) - ln q_j(x_j) with the p in
 *                         force when node j was tried, NaN for nodes never tried
 */
int sd_verify_tree(const void* target_logits, const void* draft_logits, const int32_t* node_tokens,
                   const int32_t* parent, int B, int N, int max_depth, int V, int dtype, int mode,
                   uint64_t seed, uint64_t offset, int32_t* path_len, int32_t* path_nodes,
                   int32_t* out_tokens, float* log_ratio, int32_t* row_status, void* workspace,
                   size_t workspace_bytes, void* hip_stream);

/*
 * fsd_verify_chain with the usual sampling-method warpers applied where the
 * token is drawn (paper Sec. 4: "whatever sampling method the user sets"), in
 * this order, on the target row the token comes from:
 *   temperature  s_v = z_v * binary32(1 / temperature), 1e-3 <= temperature <= 1e3;
 *   top_k        keep the entries with s_v >= the top_k-th largest s (ties at it
 *                are all kept); 0 or >= V switches it off;
 *   top_p        with q = softmax of the kept s, keep s_v >= t, t the largest
 *                value with sum_{s_v >= t} q_v >= top_p (ties kept); 1 = off;
 * then the Gumbel-max draw of fsd_verify_chain over the kept entries, on
 * s_v + G_v with the same random stream.  FSD_GREEDY ignores the warpers (the
 * argmax is always kept).  Acceptance does not depend on them.  With
 * temperature 1, top_k 0 and top_p 1 the call is fsd_verify_chain.
 */
int fsd_verify_chain_warped(const void* target_logits, const void* draft_logits, const int32_t* cand_tokens,
                            int B, int K, int V, int dtype, int div, float T, int mode, uint64_t seed,
                            uint64_t offset, float temperature, int top_k, float top_p, int32_t* accept_len,
                            int32_t* out_tokens, float* divergences, int32_t* row_status, void* workspace,
                            size_t workspace_bytes, void* hip_stream);

/*
 * fsd_verify_tree with the same warpers, applied to the target row after the
 * last node of the accepted path.  Arguments as in fsd_verify_tree and
 * fsd_verify_chain_warped.
 */
int fsd_verify_tree_warped(const void* target_logits, const void* draft_logits, const int32_t* node_tokens,
                           const int32_t* parent, int B, int N, int max_depth, int V, int dtype, int div,
                           float T, int mode, uint64_t seed, uint64_t offset, float temperature, int top_k,
                           float top_p, int32_t* path_len, int32_t* path_nodes, int32_t* out_tokens,
                           float* divergences, int32_t* row_status, void* workspace, size_t workspace_bytes,
                           void* hip_stream);

/*
 * Reducible FSD (paper Sec. 4.3, "Reducing FSD to standard SD"): position i is
 * accepted iff div(p_i, q_i) <= T (the rule of fsd_verify_chain) OR the strict
 * SD test of sd_verify_chain accepts the candidate token, with the same uniform
 * numbers; at the first rejection the token is drawn from the normalised
 * positive part of p - q, otherwise from the row after the last candidate.
 * With T <= 0 and no bit-identical rows the outputs equal sd_verify_chain's.
 * Tensors and outputs as in fsd_verify_chain, plus
 *
 *   log_ratio [B, K] out  optional, ln p_i(x_i) - ln q_i(x_i)
 */
int rfsd_verify_chain(const void* target_logits, const void* draft_logits, const int32_t* cand_tokens,
                      int B, int K, int V, int dtype, int div, float T, int mode, uint64_t seed,
                      uint64_t offset, int32_t* accept_len, int32_t* out_tokens, float* divergences,
                      float* log_ratio, int32_t* row_status, void* workspace, size_t workspace_bytes,
                      void* hip_stream);

/*
 * Threshold tuning on a dev set (paper Sec. 6.2 "Selecting T", paragraph "Tuning T on small dev set";
 * App. A: the threshold that accepts about the same share of candidate tokens
 * as strict SD).  From the divergences of a batch of candidate sequences (the
 * `divergences` output of fsd_verify_chain, any T) it finds the smallest
 * threshold, among the values that occur, at which the chain rule accepts at
 * least `target_fraction` of all B*K candidate positions; +inf if no threshold
 * does (NaN divergences are never accepted).  Exact: the result is one of the
 * input values.
 *
 *   divergences  [B, K] device, binary32, >= 0 or NaN
 *   target_fraction      0 < f <= 1 (e.g. sum(accept_len of strict SD) / (B*K))
 *   T_out        [1] device out   the threshold
 *   fraction_out [1] device out   optional, the share accepted at T_out
 *   workspace    device, 256-byte aligned, fsd_calibrate_workspace_bytes(B, K)
 *
 * Asynchronous on hip_stream like the verify calls; limits as there.
 */
size_t fsd_calibrate_workspace_bytes(int B, int K);
int fsd_calibrate_threshold(const float* divergences, int B, int K, float target_fraction, float* T_out,
                            float* fraction_out, void* workspace, size_t workspace_bytes, void* hip_stream);

/* ---------------------------------------------------------------------------
 * Around a verify call: the operators that make its logits and that use its
 * outputs.  A serving step is, per layer of the target model, fsd_attend_* over
 * the candidates; then, on the logits, fsd_condition_*; then a verify call; then
 * fsd_cache_append with the verify call's accept_len (path_len, path_nodes).
 *
 * These calls keep the conventions above (device pointers, asynchronous on
 * hip_stream, argument errors before anything is launched, nothing allocated),
 * and may be recorded into HIP graphs.  Their workgroups never wait for one
 * another: they can share the GPU with any other work.
 * ------------------------------------------------------------------------- */

/*
 * Penalties for repeated tokens, biases and a grammar's mask on the logits of
 * a verify call.  Every row is conditioned on the tokens of its OWN context: the
 * history, and the candidates on the way to it.  With z the logit of entry v,
 *
 *   seen(v)    v occurs in the history or on the way
 *   count(v)   how often it occurs in the generated part of the history (from
 *              prompt_len on) and on the way
 *   z1 = z / r where seen(v) and z > 0, z * r where seen(v) and z <= 0, else z
 *   z2 = z1 - frequency * count(v) - (count(v) > 0 ? presence : 0)
 *   z3 = z2 + bias(v);  -inf where the mask does not allow v
 *
 * in binary32 in this order (z / r as z * (1 / r), which costs one rounding of 2^-24 more), rounded
 * once to the logits' type; an entry that none of this touches keeps its bits.  A masked entry is -inf whatever it held
 * (NaN as well); a mask that allows nothing leaves a row of -inf, which a verify
 * call reports (FSD_ROW_NONFINITE).
 *
 * All members may be NULL / 0: what is missing does not apply.
 */
typedef struct {
    const int32_t* history;      /* [B, history_stride] token ids, in order; ids outside [0, V) are passed over */
    const int32_t* history_len;  /* [B] how many count (taken as within [0, history_stride]); NULL: all */
    const int32_t* prompt_len;   /* [B] how many of them are the prompt; NULL: none */
    int history_stride;          /* 0 .. 2^29 */
    int bias_count;
    const int32_t* bias_tokens;  /* [B, bias_count]; ids outside [0, V) are passed over; of equal ids the last counts */
    const float* bias_values;    /* [B, bias_count] */
    const float* repetition;     /* [B] r, > 0; NULL: 1 */
    const float* presence;       /* [B] */
    const float* frequency;      /* [B] */
    const uint32_t* allowed;     /* [B, allowed_contexts, ceil(V / 32)] bit v % 32 of word v / 32: v is allowed */
    int allowed_contexts;        /* 1: one mask a sequence; contexts of the call: one mask for each; 0 with allowed NULL */
} fsd_conditions;

/*
 *   logits      [B, rows, V]  rows = K+1: the target rows of fsd_verify_chain; rows = K: its draft
 *                             rows.  Row i stands behind candidates 0 .. i-1 (both kinds).
 *   cand_tokens [B, K]        candidate token ids (0 <= K <= 2048; may be NULL when K is 0: a
 *                             step without candidates); ids outside [0, V) are passed over
 *   out         [B, rows, V]  out; may be logits itself (in place), else no overlap with it (FSD_ERR_LAYOUT); both on addresses of whole elements
 *                             (FSD_F32 or FSD_BF16), B * rows < 2^24
 * A mask per context has K+1 of them, also for draft rows: context i stands behind candidates 0 .. i-1.
 */
int fsd_condition_chain(const void* logits, const int32_t* cand_tokens, int B, int K, int rows, int V, int dtype,
                        const fsd_conditions* conditions, void* out, void* hip_stream);

/*
 * The same for a token tree.  rows = N+1: the target rows of fsd_verify_tree (row 0: the root's
 * context, row j+1: the context that ends with node j); rows = N: its draft rows (row j: the
 * context of node j's parent).  A mask per context has N+1 of them, numbered like the target rows.
 * A parent outside [-1, j) is taken as -1 (the verify call flags it).  1 <= N <= 2048.
 * (Any tree; what takes time is the part of a row's way that the row before does not share: trees of some hundred levels are better numbered
 * so that neighbours' ways are alike.)
 */
int fsd_condition_tree(const void* logits, const int32_t* node_tokens, const int32_t* parent, int B, int N, int rows,
                       int V, int dtype, const fsd_conditions* conditions, void* out, void* hip_stream);

/*
 * A paged cache of keys and values in 8 bits (OCP e4m3), in blocks of
 * FSD_CACHE_BLOCK tokens, with one scale for each block and head:
 *
 *   k_codes [layers, num_blocks, kv_heads, 64, head_dim]       a key of a token is head_dim bytes in a row
 *   v_codes [layers, num_blocks, kv_heads, 4, head_dim, 16]    token t of a block: group t / 16, place t % 16
 *   k_scale, v_scale [layers, num_blocks, kv_heads]            value = code * scale, scale > 0
 *   block_table [B, max_blocks]   token t of sequence b is token t % 64 of block block_table[b][t / 64]
 *   cache_len   [B]               tokens of sequence b in the cache
 *
 * (Values lie by groups of 16 tokens because the attention's matrix instruction takes them with
 * the token index running fastest: 16 bytes of one head dimension are then one load, and a token that is
 * appended still touches 2 KB at head_dim 128, not the whole block.)
 * head_dim is 64, 128 or 256, kv_heads at most 1024.  What lies behind a sequence's last token in its last block is never
 * used: it may hold anything.  Blocks may be shared by sequences as long as nothing is appended to
 * them.  Code and scale arrays start on 16-byte boundaries.
 */
#define FSD_CACHE_BLOCK 64
typedef struct {
    void* k_codes;
    void* v_codes;
    float* k_scale;
    float* v_scale;
    const int32_t* block_table;
    const int32_t* cache_len;
    int layers, num_blocks, kv_heads, head_dim, max_blocks;
} fsd_cache;

/*
 * Rotation by position (of queries and keys): of the first `dim` elements of a head, pairs are turned by the
 * angle of their position, the rest is left alone.  FSD_ROPE_HALVES pairs elements i and i + dim/2,
 * FSD_ROPE_PAIRS 2i and 2i+1, i < dim/2:  a' = a cos - b sin,  b' = b cos + a sin  (binary32).
 *
 *   table [rows, dim] binary32, 16-byte aligned: row p holds the dim/2 cosines, then the dim/2 sines of
 *         position p.  dim: a multiple of 16, at most head_dim.
 */
typedef enum { FSD_ROPE_HALVES = 0, FSD_ROPE_PAIRS = 1 } fsd_rope;
typedef struct {
    const float* table;
    int rows, dim, style;
} fsd_rotation;

/*
 * Appends keys and values to the cache: of every sequence row 0 (the token emitted last, whose key
 * and value the cache does not hold yet) and the accepted candidates behind it.
 *
 *   k, v  [layers, B, R, kv_heads, head_dim]  rows as in fsd_attend_*: row 0, then row j+1 for
 *         candidate (node) j; FSD_F32, FSD_BF16 or FSD_F16.  token_stride: elements from one token's
 *         keys to the next one's (>= kv_heads * head_dim, a multiple of 8); sequences are R, layers B * R tokens apart.
 *   accept_len [B]             as the verify calls give it (path_len): accept_len + 1 rows are
 *                              appended; -1: none.  For a prompt of n tokens: n - 1.
 *   path_nodes [B, max_depth]  as fsd_verify_tree gives them; NULL for a chain (rows 0 .. accept_len)
 *   rotation                   of the keys, at positions cache_len, cache_len + 1, ...; NULL: none
 *   cache_len_out [B]          out  optional: cache_len + accept_len + 1.  Not cache_len itself (other
 *                              workgroups of the call still read that): copy it over afterwards.
 *   row_status [B]             out  optional
 * cache_len_out and row_status share no byte with cache_len, block_table, accept_len, path_nodes or one another (FSD_ERR_LAYOUT).
 *
 * A block's scale is the smallest power of two s with |x| <= 448 s for every (finite) x appended to it, but
 * at least 2^-100 and at least the scale the block has if it holds tokens of the sequence already: those are rounded again
 * to the new scale if it is larger (exact but for codes that leave the normal range, as s is a power of two).
 * Codes are the nearest e4m3 value of x / s, ties to even; a value that is not finite is held as NaN.
 *
 * Nothing of a sequence is appended, its cache_len_out is its cache_len and FSD_ROW_BAD_CACHE is
 * set, if accept_len is outside [-1, R) (or over max_depth), a path node outside [0, R-1), cache_len or the new length
 * outside [0, 64 * max_blocks], a block to be written outside [0, num_blocks) or a position outside the rotation's table.
 * Two sequences that append to one block in one call race on it, and so do two places of one sequence's table that name one.
 * R <= 2^20, B <= 65535.  Calls of up to 16 rows a sequence (R, or max_depth + 1): layers <= 65535; of more: layers * B *
 * kv_heads * (blocks that R rows can touch) < 2^24.
 */
int fsd_cache_append(const void* k, const void* v, int64_t token_stride, int B, int R, int dtype,
                     const int32_t* accept_len, const int32_t* path_nodes, int max_depth,
                     const fsd_rotation* rotation, const fsd_cache* cache, int32_t* cache_len_out,
                     int32_t* row_status, void* hip_stream);

/*
 * Attention of a step's rows over the cache and over one another: what the target model does in the
 * pass that verifies the candidates (or, with R = 1, in a step without candidates, or with a larger R on a piece of a
 * prompt).  Row 0 is the token emitted last, row i+1 candidate i; none of them is in the cache yet.
 * Row r sees all cache_len tokens of its sequence and, of the rows, 0 .. r.
 *
 *   q        [B, R, heads, head_dim]      FSD_BF16 or FSD_F16; heads a multiple of kv_heads: query head i
 *                                         reads key head i / (heads / kv_heads)
 *   k, v     [B, R, kv_heads, head_dim]   same type
 *   q_stride, kv_stride                   elements from one token to the next (multiples of 8;
 *                                         sequences are R tokens apart); q, k, v are 16-byte aligned
 *   row_count [B]  optional: rows of the sequence (taken as within [0, R]); what lies behind them (their nodes' parents as well)
 *                  is neither read nor written
 *   scale          of the products before the softmax (any finite number)
 *   rotation       of q and k, at position cache_len + (number of rows before it that the row sees); NULL: none
 *   layer          which of the cache's layers
 *   out      [B, R, heads, head_dim] dense, out, 16-byte aligned
 *   row_status [B] out optional: FSD_ROW_BAD_CACHE where cache_len is outside [0, 64 * max_blocks], a
 *                  block outside [0, num_blocks), row_count outside [0, R] or a position outside the rotation's table (the call then
 *                  takes the nearest length and position, and leaves such blocks out).  It shares no byte with cache_len, block_table,
 *                  row_count or parent (FSD_ERR_LAYOUT)
 *   workspace      fsd_attend_workspace_bytes(...) bytes, 256-byte aligned
 *
 * Products of 16-bit operands are summed in binary32; the rotated queries and keys and the softmax's weights
 * enter them with the 11 significant bits of binary16 (scaled so that they stay in its range; FSD_F16's queries and keys, which may use
 * all 11, in two parts), the codes exactly; statistics are binary32, the result is rounded once.  Magnitudes of values up to
 * 2^120 and value scales from 2^-100 to 2^111 are in range.  A NaN among the keys or codes a row sees makes its outputs NaN, and so does
 * an infinite query or key of FSD_F16 (of FSD_BF16 its products' signs decide: a score of -inf is a weight of 0), or
 * a value among the rows that is not finite (all head_dim outputs of the heads that read it); what a row does not see
 * changes its result by a rounding at most, whatever it holds.
 * 1 <= R <= 2049, 1 <= heads / kv_heads <= 64, heads <= 1024, B <= 65535, B * R < 2^24.
 */
size_t fsd_attend_workspace_bytes(int B, int R, int heads, int kv_heads, int head_dim);
int fsd_attend_chain(const void* q, const void* k, const void* v, int64_t q_stride, int64_t kv_stride, int B, int R,
                     int heads, int dtype, const int32_t* row_count, float scale, const fsd_rotation* rotation,
                     const fsd_cache* cache, int layer, void* out, int32_t* row_status, void* workspace,
                     size_t workspace_bytes, void* hip_stream);

/*
 * The same over a token tree: R = N+1 rows, row j+1 for node j, parent [B, N] as in fsd_verify_tree.
 * Row j+1 sees the cache, row 0 and the rows of the nodes on the way to node j, itself included.  A parent outside
 * [-1, j) is taken as -1 and flagged (FSD_ROW_BAD_PARENT).
 */
int fsd_attend_tree(const void* q, const void* k, const void* v, int64_t q_stride, int64_t kv_stride,
                    const int32_t* parent, int B, int R, int heads, int dtype, const int32_t* row_count, float scale,
                    const fsd_rotation* rotation, const fsd_cache* cache, int layer, void* out, int32_t* row_status,
                    void* workspace, size_t workspace_bytes, void* hip_stream);

/* ---------------------------------------------------------------------------
 * Around drafting: the continuations that a drafter proposes, or a beam search
 * keeps, and what follows them.  A step is fsd_beam_select on the logits of a
 * sequence's contexts (a tree's level, or a search's beams), then, for states,
 * fsd_beam_reorder, and for the paged cache fsd_cache_fork with the selection's
 * parents (as rows of the table).  fsd_cache_fork is also what a serving loop
 * calls where sequences begin, end, are rolled back or need room.
 *
 * The conventions are those of the calls around a verify call; workgroups never
 * wait for one another.
 * ------------------------------------------------------------------------- */

/*
 * The n best continuations of each sequence's beams.  With z the logits of beam w,
 *
 *   s(w, v) = scores[w] + z_v - log sum_u exp(z_u)     for v in [0, V) with z_v > -inf
 *   s(w, -1) = scores[w]                               of a finished beam (done[w] != 0), its only continuation
 *   ranked by s * weights[w], largest first; of equal ranks the lowest w, then the largest z, then the lowest v
 *
 * Normalisers, scores and ranks are held in binary64 (relative error of a row's sum of exponentials under 2^-33; z_v's distance from the row's normaliser is formed
 * without a loss where both are large: a row of V times the type's lowest number has V continuations of -log V; a row's only
 * entry has the beam's score itself); scores_out is rounded once
 * (a score below binary32's range, to -inf).
 *
 *   logits  [B, beams, V]  FSD_F32 or FSD_BF16, row_stride elements from one beam's row to the next (>= V, at most 2^32)
 *   scores  [B, beams]     -inf: the beam does not count, and its row is not read; NULL: 0
 *   weights [B, beams]     > 0 and finite, e.g. a power of the length that a continuation has; NULL: 1
 *   done    [B, beams]     finished beams, whose rows are not read; NULL: none
 *   scores_out [B, n], parent [B, n], tokens [B, n]   out: s, w and v (-1 for a finished beam); -inf, -1 and -1 behind the last continuation
 *                          where there are fewer than n
 *   row_status [B]         out  optional: FSD_ROW_NONFINITE where a row that is read holds NaN or +inf, or a beam that counts has
 *                          such a score or a weight that is not positive and finite: the sequence has no continuations then.  (A row that is -inf
 *                          everywhere is none of that: a grammar that has ended a beam.)
 *   workspace              fsd_beam_workspace_bytes(...) bytes, 256-byte aligned; those of some sizes are enough for smaller ones as well, of either dtype
 * No output shares a byte with another one, scores, weights, done or the workspace, and neither an output nor the workspace lies between the first and the last byte of the
 * logits (FSD_ERR_LAYOUT).
 * Entries of -inf cost nothing.  Where fewer than n entries of a part of a row lie above many equal ones (a mask of a finite number), the part is gone over 18 more times (FSD_F32: 34):
 * mask by -inf where that can be chosen.
 * 1 <= beams <= 256, 1 <= n <= 128, 1 <= V <= fsd_max_vocab(dtype), 1 <= B <= 65535.
 */
size_t fsd_beam_workspace_bytes(int B, int beams, int V, int n, int dtype);
int fsd_beam_select(const void* logits, int64_t row_stride, const float* scores, const float* weights, const int32_t* done, int B,
                    int beams, int V, int dtype, int n, float* scores_out, int32_t* parent, int32_t* tokens, int32_t* row_status,
                    void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * States in the order of the continuations: out[l, b, i] = states[l, b, parent[b, i]], zeros where parent is -1.
 *
 *   states [layers, B, beams, row_bytes]   bytes of any type, on any address; out [layers, B, n, row_bytes], no overlap with states
 *   parent [B, n]                          as fsd_beam_select gives it
 *   row_status [B] out  optional: FSD_ROW_BAD_PARENT where a parent is outside [-1, beams) (its rows are zeros); no overlap with parent or out
 * 1 <= layers, beams, n, B <= 65535, layers * B * max(beams, n) < 2^31, row_bytes from 1 to 2^40.
 */
int fsd_beam_reorder(const void* states, const int32_t* parent, int layers, int B, int beams, int n, size_t row_bytes, void* out,
                     int32_t* row_status, void* hip_stream);

/*
 * New sequences that continue old ones: beams that are kept, once or more than once; a prompt that several answers go out from; or the
 * same sequences with candidates rolled back, room for the next step, some ended and others begun.  The n new sequences take the place of the B
 * old ones (those of `cache`): what no new one keeps is free again.  A sequence that goes on is its own parent.
 *
 *   refs [num_blocks]     for every block the number of places of block tables that name it, these and any others (a stored prompt's, another
 *                         batch's); 0: free
 *   parent [n]            the old sequence that new sequence i continues; -1: none, it begins empty
 *   lengths [n]           tokens of it that are kept, in [0, cache_len[parent]]; NULL: all.  (Without a parent: none.)
 *   room [n]              tokens that will be appended before the next call: the blocks they need are there; NULL: 0
 *   block_table_out [n, max_blocks], cache_len_out [n], refs_out [num_blocks]   out: the same of the new sequences.  refs_out may be refs, else no
 *                         output shares a byte with an input or another output (FSD_ERR_LAYOUT)
 *   free_blocks [1]       out  optional: blocks free afterwards; negative: how many were lacking
 *   row_status [n]        out  optional
 *
 * A table's entry that is negative names nothing.  With have = lengths[i] tokens, full = have / 64 and need = ceil((have + room[i]) / 64):
 *   - places < full share the parent's blocks;
 *   - a place from full to need - 1 keeps its parent's block if no other place will name that: none of other tables (refs less the old sequences' places
 *     is 0), none of the new sequences' first `full`, and of the other places that want to keep it this is the lowest (sequence, place);
 *   - all else gets free blocks, the lowest numbers first, in order of (sequence, place).  (A block that only ended sequences held is free.)
 *     Place `full`, if the sequence has tokens in it (have % 64), is copied there from its parent's, in all layers: the scales, and the groups of 16
 *     tokens that hold any;
 *   - places from need on are -1.
 * Appending to the new sequences then touches no block that another place names.
 *
 * FSD_ROW_BAD_PARENT: parent outside [-1, B).  FSD_ROW_BAD_CACHE: cache_len, lengths or room outside its range (have + room at most 64 * max_blocks), or a
 * place of the parent's that holds some of its first `have` tokens names no block.  Such a sequence comes out empty.  FSD_ROW_NO_BLOCKS, for all of them: there are too few
 * free blocks; nothing is copied, refs_out is refs and every sequence comes out empty, so that the caller, who still has the old tables, can make room and call again.
 * Blocks of reserved places may hold anything.  The copied codes' cache is that of `cache` (written in place).
 * Blocks are given out from refs, so calls that give out blocks of one pool go one after another, each with the refs_out of the one before.
 * n, B <= 65535, n * max_blocks < 2^31 - 1, num_blocks <= 2^24.
 */
size_t fsd_cache_fork_workspace_bytes(int num_blocks, int n);
int fsd_cache_fork(const fsd_cache* cache, int B, const int32_t* refs, const int32_t* parent, const int32_t* lengths, const int32_t* room, int n,
                   int32_t* block_table_out, int32_t* cache_len_out, int32_t* refs_out, int32_t* free_blocks, int32_t* row_status,
                   void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Pages from one cache to another, or within one: block src_blocks[k] of `src` becomes block dst_blocks[k] of `dst`, in all layers: the scales, and
 * the groups of 16 tokens that hold any of its first tokens[k] (0 .. 64; NULL: all).  The caches have the same layers, kv_heads and head_dim; they are one cache (all four arrays)
 * or share none (FSD_ERR_LAYOUT).  Their tables and lengths are not looked at.
 *
 *   page_status [n] out  optional: FSD_ROW_BAD_CACHE where a block or tokens is out of range, which copies nothing.  A block of -1 copies nothing either,
 *                   and is no error
 * The order of pages is not given: a block that is written twice, or written and read, holds parts of any of them.
 * n >= 1; n * layers * kv_heads < 2^40.
 */
int fsd_cache_copy(const fsd_cache* src, const fsd_cache* dst, const int32_t* src_blocks, const int32_t* dst_blocks, const int32_t* tokens, int n,
                   int32_t* page_status, void* hip_stream);

/*
 * A cache's pages moved together: with U blocks in use (refs > 0), those numbered U and up move to the free blocks below U, the lowest to the lowest, in all
 * layers and whole.  Afterwards blocks 0 .. U-1 are in use and the rest is free.
 *
 *   refs [num_blocks]             as in fsd_cache_fork
 *   block_table_out [B, max_blocks] out: the table with the new numbers; -1 where it names nothing or a free block.  May be the cache's own table
 *   refs_out [num_blocks]         out  may be refs
 *   remap [num_blocks]            out  optional: a block's new number, -1 of a free one (for tables of others)
 *   used_blocks [1]               out  optional: U
 *   row_status [B]                out  optional: FSD_ROW_BAD_CACHE where a table's row names a free block or one outside [0, num_blocks)
 * Otherwise no output shares a byte with an input or another output (FSD_ERR_LAYOUT).  num_blocks <= 2^24, B <= 65535.
 */
size_t fsd_cache_compact_workspace_bytes(int num_blocks);
int fsd_cache_compact(const fsd_cache* cache, int B, const int32_t* refs, int32_t* block_table_out, int32_t* refs_out, int32_t* remap,
                      int32_t* used_blocks, int32_t* row_status, void* workspace, size_t workspace_bytes, void* hip_stream);

/* ---------------------------------------------------------------------------
 * Everything below is for tests, tuning and benchmarks, not for serving code.
 * These calls set or read PROCESS-WIDE state inside the library (the only such
 * state it has; the verify calls themselves keep none between calls, apart from
 * per-device constants looked up once).  They are not thread-safe: use them from
 * one thread while no verify call is in flight on another.
 * ------------------------------------------------------------------------- */

/*
 * Timing of the vocabulary-reduction kernel, for benchmarks.  After
 * fsd_profile_enable(1) every verify call launches that kernel with a pair of
 * events that take the start and the end of its dispatch on the call's stream
 * (what a kernel trace shows; up to 4096 pairs are kept; later calls are
 * not recorded).  Small calls, which otherwise take another kernel (see
 * fsd_debug_set_small_calls), launch it as well while this is on.  fsd_profile_collect waits for the recorded events, returns
 * the number of pairs and their mean / minimum duration in milliseconds, and
 * forgets them.  Not thread-safe; meant for a single benchmarking thread.
 */
int fsd_profile_enable(int on);
int fsd_profile_collect(float* mean_ms, float* min_ms);

/* Test hook: number of polls a wavefront spends waiting for the words of those
 * it shares a row pair or a sequence with before it gives up and the call
 * flags FSD_ROW_INTERNAL (default 1<<22).  It governs the waits of workgroups that have to be resident together; the
 * look for the shares of a draw, which are there whatever else is resident, has a fixed bound of its own
 * (1<<22).  Returns the previous value. */
unsigned fsd_debug_set_spin_limit(unsigned polls);

/* Test hook: a smaller number of polls for one of these waits alone, that of the
 * workgroups which share a row in a warped call's selection under top_p
 * (default: no smaller one).  Returns the previous value. */
unsigned fsd_debug_set_selection_spin_limit(unsigned polls);

/* Test hooks of the bfloat16 Jensen-Shannon reduction.  It evaluates App. C.2 in
 * entropy form (one logarithm per entry), whose absolute error (about 1e-7
 * for small results) does not shrink with the result; results below a floor (default 1e-3 nats)
 * are evaluated again in the pointwise form, whose error does.
 * fsd_debug_set_js_floor sets that floor (0: never again; +inf: always) and
 * returns the previous one; fsd_debug_set_exact_js(1) makes every bfloat16 JS
 * call use the pointwise form only and returns the previous setting. */
float fsd_debug_set_js_floor(float floor_nats);
int fsd_debug_set_exact_js(int on);

/* Test hook: the verify calls launch no kernel of their own to clear the
 * workspace's exchange words: the reduction kernel's wavefronts clear them and
 * wait for their team to have done so (calls with more than 4 MB of such words
 * apart).  0 makes every call launch the clearing kernel again; returns the
 * previous setting. */
int fsd_debug_set_self_clear(int on);

/* Tuning hook: shape of the vocabulary-reduction kernel.  `wavefronts` per
 * workgroup must be 4 (or 0 = default); `slots_per_thread` is the number of
 * 16-byte slots of each row a lane holds: 2, 4 or 8 (bfloat16: 2, 4 or 5), 0 =
 * the library's own choice (bfloat16: 48 vocabulary entries per lane for JS and
 * TV, 32 for KL and strict SD or 64 in large calls; binary32: 40, or 32 in calls of few
 * steps and for strict SD, or 16 in small calls).  A shape
 * that would need more than 256 wavefronts per row pair is ignored.  Results
 * do not depend on the shape beyond the rounding order of the partial sums. */
int fsd_debug_set_shape(int wavefronts, int slots_per_thread);

/* Test hook: grid size (workgroups) of the last vocabulary-reduction launch and
 * the number of its workgroups the device can hold at once, which caps it. */
void fsd_debug_last_launch(int* grid, int* resident);

/* Test hooks of the route a call takes.  Small FSD calls (pairs times vocabulary
 * up to a few million, none of the hooks above changed from its default) have all their pairs reduced
 * in one step of the whole device, and where the draw is small too are one launch;
 * fsd_debug_set_small_calls(0) sends them the way of the larger ones (persistent
 * teams, then the sampler, both at their own shapes) and returns the previous setting.
 * fsd_debug_last_route: of the last verify call, 0 = persistent teams, 1 = the
 * one-step reduction with the sampler behind it, 2 = one launch.  (A call that is being captured may take 1
 * where it takes 2 otherwise; the results are the same.) */
int fsd_debug_set_small_calls(int on);
int fsd_debug_last_route(void);

/* Test hook: workgroups a sequence of the last warped call's selection of kept
 * logits (1: one works alone, or there was nothing to select). */
int fsd_debug_last_selection(void);

/* Test hook: byte offset, inside a workspace of fsd_workspace_bytes(B,
 * rows_per_seq, V, dtype), of the B binary32 values fsd_verify_chain_warped
 * leaves there: per sequence the smallest scaled logit its warpers kept on the
 * row the token was drawn from (-inf when nothing is cut).  0 for bad shapes. */
size_t fsd_debug_warp_threshold_offset(int B, int rows_per_seq, int V, int dtype);

#ifdef __cplusplus
}
#endif
#endif /* FSD_H_ */
