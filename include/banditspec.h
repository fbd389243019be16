/*
 * banditspec.h -- C ABI of the B200 (sm_100a) library for one batched round of
 * speculative decoding with a bandit-chosen speculation length.
 *
 * One round, per sequence b of a batch of B independent sequences:
 *
 *   bs_bandit_select    choose the arm (speculation length gamma_b) for this round
 *   bs_softmax_verify   softmax statistics of every target / draft row, accept test,
 *                       first-rejection scan  -> accept_len[b] = tau_b
 *   bs_residual_sample  resample one token from Norm([P - Q]_+) at the rejected position,
 *                       or the bonus token from P when all drafts passed -> out_tokens, out_len
 *   bs_bandit_update    feed the accepted length y_b = tau_b + 1 back to the arm statistics
 *
 * plus bs_lmhead_verify, which computes the logits themselves (bf16 hidden states times
 * the bf16 output embedding on the tensor cores) fused with the softmax statistics.
 *
 * Conventions that hold for every entry point
 *  - Every array pointer is a DEVICE pointer owned by the caller unless the comment says
 *    "host".  The library allocates no device memory.  Its only process-wide state is a set of
 *    per-device values looked up on first use and never changed afterwards (the opt-in shared
 *    memory limit, kernel attributes, resident-CTA counts, the device address of the built-in
 *    scratch array of bs_softmax_verify_noalloc) and that scratch array itself; the values are
 *    held in atomics and every thread that finds one missing looks up the same answer, so calls
 *    may come from several host threads.
 *  - `stream` is a cudaStream_t passed as void*.  Calls are asynchronous on that stream,
 *    never synchronise, and may be captured in a CUDA graph.
 *  - The return value covers host-side argument checks and launch errors only.  Problems
 *    found in device DATA (token id outside [0,V), gamma outside [0,Gmax], non-finite
 *    normaliser) are recorded per sequence in the workspace and read back with
 *    bs_get_device_status; the kernels never trap.
 *  - Row-major layouts with the vocabulary contiguous.  Row j (0-based) of either model is
 *    the distribution of drafted token j+1, i.e. conditioned on the prompt and the first j
 *    drafted tokens; target row gamma_b is the bonus position.  Padded entries (j >= gamma_b
 *    for tokens / uniforms / draft rows, j > gamma_b for target rows) are never read.
 *  - temperature > 0: sampling mode, probabilities are softmax(logits / temperature).
 *    temperature == 0: greedy mode (the limit of Section 2): a drafted token passes iff it
 *    equals the arg-max of its target row (lowest index among equal maxima); draft logits
 *    are not read and may be NULL.
 */
#ifndef BANDITSPEC_H_
#define BANDITSPEC_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    BS_OK = 0,
    BS_ERR_INVALID_ARG = 1,   /* NULL pointer, negative or unsupported size, bad enum */
    BS_ERR_CUDA = 2,          /* a CUDA runtime call or launch failed */
    BS_ERR_UNSUPPORTED = 3,   /* valid request outside the implemented limits */
    BS_ERR_WORKSPACE = 4,     /* workspace too small or misaligned */
    BS_ERR_TIMEOUT = 5,       /* bs_get_device_status, bs_cache_get_device_status, bs_prompt_get_device_status: a bounded wait
                                 inside a kernel gave up */
    BS_ERR_DEVICE_DATA = 6    /* bs_get_device_status: some sequence carries a data error */
} bs_status;

typedef enum { BS_F32 = 0, BS_BF16 = 1 } bs_dtype;
typedef enum { BS_UCB = 0, BS_EXP3 = 1, BS_UCB_REWARD = 2 } bs_alg;

/* Per-sequence device status bits (bs_get_device_status). */
#define BS_DEV_BAD_GAMMA   1   /* gamma[b] outside [0, Gmax]; the sequence was processed as gamma = 0 */
#define BS_DEV_BAD_TOKEN   2   /* a drafted token outside [0, V); that position counts as rejected */
#define BS_DEV_NONFINITE   4   /* a softmax normaliser or residual mass was NaN / Inf / 0 */
#define BS_DEV_RESIDUAL_FALLBACK 8 /* [P-Q]_+ had zero mass at the rejected position; sampled from P instead */
#define BS_DEV_DRAFT_MISSING 16    /* bs_softmax_verify_drafted: a draft row below gamma_b was not produced by
                                      bs_draft_sample on this workspace; every draft of the sequence was rejected */
#define BS_DEV_BAD_TREE      32    /* bs_tree_verify_greedy: a node's parent is not an earlier node; the node counts as
                                      hanging under the prompt and never passes.  bs_cache_attention: the same reading;
                                      bs_cache_keep_path: a path whose nodes do not ascend, nothing was moved */
#define BS_DEV_BAD_LENGTH    64    /* bs_cache_*: a length that is negative, longer than the sequence's blocks or than its
                                      row of the block table; the sequence got no new tokens / was left out.
                                      bs_prompt_attention, bs_history_update, bs_logits_adjust: see there */
#define BS_DEV_NO_BLOCKS     128   /* bs_cache_plan: not enough free blocks; the sequence got no new tokens */
#define BS_DEV_NO_ROOM       256   /* bs_cache_plan: its tokens do not fit slot_map; the sequence got no new tokens */
#define BS_DEV_BAD_BLOCK     512   /* bs_cache_attention / bs_cache_keep_path: a block id outside [0, n_blocks) */
#define BS_DEV_TIMEOUT       1024  /* bs_cache_attention: a bounded wait gave up; every output of the call is undefined and
                                      its workspace has to be cleared with bs_workspace_init.  Set in status[0]; without
                                      a status array bs_cache_get_device_status still tells.  bs_prompt_attention: the
                                      same, without a workspace; bs_prompt_get_device_status still tells */

#define BS_DEV_BAD_MASK      2048  /* bs_logits_adjust: a mask number outside [-1, n_masks); the row got no mask */

/* Limits of this implementation. */
#define BS_MAX_GAMMA   31      /* Gmax <= 31 (one warp scans the accept flags) */
#define BS_MAX_ARMS    32      /* K <= 32 (one lane per arm) */
#define BS_MAX_BATCH   4096    /* B <= 4096 */
#define BS_MAX_VOCAB   (1 << 20) /* V <= 1048576 */
#define BS_MAX_SEQ_BLOCKS (1 << 18) /* blocks of one sequence in the key / value cache */

const char* bs_status_string(bs_status s);

/* Text of the last CUDA runtime error that made a call on this thread return BS_ERR_CUDA
 * (diagnostics only; "no error" if there was none). */
const char* bs_last_cuda_error(void);

/* ---- workspace ------------------------------------------------------------------ */

/* Bytes of device scratch bs_softmax_verify / bs_residual_sample / bs_lmhead_verify need for
 * a batch of B sequences, speculation lengths up to Gmax and vocabulary V (any dtype).
 * Returns 0 for arguments outside the limits. */
size_t bs_workspace_bytes(int B, int Gmax, int V);

/* Clears the workspace (arrival counters must start at zero; the kernels leave them at zero
 * again after every call).  Call once after allocating, 256-byte aligned. */
bs_status bs_workspace_init(void* workspace, size_t workspace_bytes, void* stream);

/* Copies the per-sequence status words of the LAST verify/residual call to host memory.
 * Synchronises the stream.  host_status: host array [B].  Returns BS_ERR_DEVICE_DATA if any
 * word is non-zero, BS_ERR_TIMEOUT if a bounded wait inside a kernel of that call gave up (its
 * outputs are then undefined and its arrival counters may be left non-zero: clear the workspace
 * with bs_workspace_init before using it again), BS_OK otherwise. */
bs_status bs_get_device_status(const void* workspace, size_t workspace_bytes, int B, int Gmax, int V,
                               int32_t* host_status, void* stream);

/* ---- verification (Algorithm 6 of the paper, from its second line on) ---------------- */

/* Softmax statistics (Section 2: softmax of logits / temperature), accept test
 * r <= min{1, P(x)/Q(x)} and first-rejection scan (Algorithm 6, for-loop).
 *
 *  target_logits  [B, Gmax+1, V]  dtype
 *  draft_logits   [B, Gmax,   V]  dtype; may be NULL iff temperature == 0
 *  draft_tokens   [B, Gmax] int32, the drafted tokens x~_1..x~_gamma
 *  gamma          [B] int32, speculation length of each sequence this round, 0 <= gamma <= Gmax
 *  u_accept       [B, Gmax] fp32 uniforms in (0,1); may be NULL iff temperature == 0
 *  accept_len     [B] int32 out: tau_b = number of leading accepted drafts
 *  p_tok, q_tok   [B, Gmax] fp32 out or NULL: P_j(x~_{j+1}), Q_j(x~_{j+1}) for j < gamma_b
 *                 (entries j >= gamma_b are set to 0; both zero-filled in greedy mode).
 *                 Arithmetic is fp32 with the rounding of (row maximum * log2(e) / temperature)
 *                 undone to first order: measured error of a probability below 3e-7 for
 *                 temperatures from 0.05 to 8 at logits of +-10
 *  workspace      from bs_workspace_bytes / bs_workspace_init; keeps the row statistics that
 *                 bs_residual_sample reads, so the two calls share it and run on one stream.
 * Reads every valid logit exactly once.  Two calls that share a workspace must not overlap. */
bs_status bs_softmax_verify(const void* target_logits, const void* draft_logits, bs_dtype dtype,
                            const int32_t* draft_tokens, const int32_t* gamma, const float* u_accept,
                            float temperature, int B, int Gmax, int V,
                            int32_t* accept_len, float* p_tok, float* q_tok,
                            void* workspace, size_t workspace_bytes, void* stream);

/* Resampling step (Algorithm 6, else-branch and the line after the loop): for each sequence,
 * with tau = accept_len[b]: if tau < gamma_b sample from Norm([P_tau - Q_tau]_+), otherwise
 * sample the bonus token from P_gamma.  One uniform per sequence, inverse CDF in vocabulary
 * order: the smallest v whose cumulative mass strictly exceeds u * total.  Greedy mode emits
 * the arg-max of target row tau.
 *
 *  same logits / dtype / tokens / gamma / temperature / sizes / workspace as the preceding
 *  bs_softmax_verify call on this stream (its row statistics are read from the workspace)
 *  accept_len   [B] int32 in
 *  u_resample   [B] fp32 uniforms in (0,1); may be NULL iff temperature == 0
 *  out_tokens   [B, Gmax+1] int32 out: the tau accepted drafts, then the sampled token, then -1
 *  out_len      [B] int32 out: y_b = tau_b + 1, the accepted length that is the bandit reward
 *               (Section 3: the bonus token counts, 1 <= y <= L+1) */
bs_status bs_residual_sample(const void* target_logits, const void* draft_logits, bs_dtype dtype,
                             const int32_t* draft_tokens, const int32_t* gamma, const int32_t* accept_len,
                             const float* u_resample, float temperature, int B, int Gmax, int V,
                             int32_t* out_tokens, int32_t* out_len,
                             void* workspace, size_t workspace_bytes, void* stream);

/* bs_softmax_verify without a caller-supplied workspace.  (No counterpart in the paper: this
 * exists for integration, not for the method.)
 *
 * For callers that cannot allocate device memory where the call is made: a decoding loop that
 * runs out of a pool sized at start-up, a plugin that only ever receives its input and output
 * buffers, or a latency-critical path where cudaMalloc is off limits because it synchronises the
 * device.  The scratch is a fixed array of BS_NOALLOC_SCRATCH_BYTES built into the library; every
 * GPU that loads the library holds that much memory until the process exits.
 *
 *  - Same arguments, outputs and arithmetic as bs_softmax_verify, minus the workspace.  The
 *    call allocates and frees nothing.
 *  - Limit: bs_workspace_bytes(B, Gmax, V) must not exceed BS_NOALLOC_SCRATCH_BYTES, otherwise
 *    BS_ERR_WORKSPACE is returned and nothing is launched (e.g. B=64, Gmax=8, V=128256 needs
 *    about 0.3 MB; B=256, Gmax=8, V=152064 about 1.4 MB).
 *  - The first call on each device looks up the device address of the array (with that device
 *    current).  Make that first call outside any stream capture.
 *  - All calls on a GPU share the one array.  It keeps what the previous call left; the counters
 *    and status words the kernel reads before writing are cleared on the stream at the start of
 *    every call.  Calls that overlap on the same GPU (different streams, different threads) race
 *    on it and give wrong results: serialise them.
 *  - The row statistics stay inside the library, so bs_residual_sample cannot follow this call;
 *    it serves callers that need accept_len and the token probabilities only.
 *  - The per-sequence status words and the abort word live in the array too, and
 *    bs_get_device_status cannot be pointed at it: device-detected data problems are handled as
 *    in bs_softmax_verify (an out-of-range token counts as rejected, an out-of-range gamma as
 *    gamma = 0, nothing traps) but are not reported, and a pipeline wait that gave up leaves
 *    accept_len / p_tok / q_tok of the unfinished sequences unwritten without a way to learn of
 *    it.  Callers that need the report use bs_softmax_verify with a workspace. */
#define BS_NOALLOC_SCRATCH_BYTES (2 << 20)
bs_status bs_softmax_verify_noalloc(const void* target_logits, const void* draft_logits, bs_dtype dtype,
                                    const int32_t* draft_tokens, const int32_t* gamma, const float* u_accept,
                                    float temperature, int B, int Gmax, int V,
                                    int32_t* accept_len, float* p_tok, float* q_tok, void* stream);

/* ---- verification and resampling in one launch, with early exit ------------------------------- */

/* Algorithm 6 from its second line on in the algorithm's own order: position after position,
 * stopping at the first rejection (its "break"), then the resampling step -- bs_softmax_verify
 * followed by bs_residual_sample, but rows behind the first rejected draft are not needed: a
 * sequence that stops at position tau costs 2 (tau + 1) rows (2 gamma + 1 when everything
 * passes) plus a second pass over the rows of the stop position, instead of 2 gamma + 1 + 2.
 * (The kernel may stream a sequence up to three positions ahead of its last decision, so a few
 * rows behind the stop can be read all the same; they change no result.)
 *
 *  arguments as bs_softmax_verify and bs_residual_sample (temperature 0 = greedy mode: target rows
 *  only, the emitted token is the arg-max of the stop row, draft logits and uniforms may be NULL)
 *  p_tok, q_tok  [B, Gmax] fp32 out or NULL: filled for the positions that were examined
 *                (j <= tau_b, j < gamma_b); the entries behind the stop are set to 0 (all of them
 *                in greedy mode)
 *  accept_len, out_tokens, out_len: as the two separate calls
 * The CTAs that share a sequence wait for one another: they form a thread-block cluster, or --
 * rows of a single 32 KB segment, very large batches -- the kernel is launched cooperatively, and
 * the call fails with BS_ERR_CUDA where that is not possible.  A wait that does not end
 * within about a second makes bs_get_device_status return BS_ERR_TIMEOUT.
 * Requirement: rows on 16-byte boundaries (V * element size a multiple of 16, base pointers
 * 16-byte aligned), else BS_ERR_UNSUPPORTED. */
bs_status bs_verify_walk(const void* target_logits, const void* draft_logits, bs_dtype dtype,
                         const int32_t* draft_tokens, const int32_t* gamma, const float* u_accept,
                         const float* u_resample, float temperature, int B, int Gmax, int V,
                         int32_t* accept_len, float* p_tok, float* q_tok, int32_t* out_tokens, int32_t* out_len,
                         void* workspace, size_t workspace_bytes, void* stream);

/* ---- drafting on the device (Algorithm 6, first line: x~_{j+1} ~ Q(. | pt, x~_{1:j})) ------------ */

/* Draws the drafted token of ONE position for every sequence that drafts it (position < gamma_b):
 * a categorical sample from softmax(draft row `position` / temperature) by inverse CDF in
 * vocabulary order with the uniform u_draft[b, position] (the smallest v whose cumulative mass
 * strictly exceeds u * total); at temperature 0 the arg-max of the row (lowest index among
 * equal maxima).  A draft model produces its rows one position at a time, so this is called once
 * per position, after the row has been written.
 *
 *  draft_logits [B, Gmax, V] dtype: only row `position` of each drafting sequence is read
 *  position     0 <= position < Gmax
 *  gamma        [B] int32: this round's speculation lengths
 *  u_draft      [B, Gmax] fp32 uniforms in (0,1); may be NULL iff temperature == 0
 *  draft_tokens [B, Gmax] int32: entry [b, position] is written for drafting sequences, others kept
 *  workspace    the round's verification workspace (bs_workspace_bytes / bs_workspace_init)
 * Besides the token, the call leaves the row's softmax statistics in the workspace and marks the
 * position as drafted, which is what bs_softmax_verify_drafted relies on.
 * Requirement: rows on 16-byte boundaries (V * element size a multiple of 16, base pointer
 * 16-byte aligned), else BS_ERR_UNSUPPORTED. */
bs_status bs_draft_sample(const void* draft_logits, bs_dtype dtype, int position, const int32_t* gamma,
                          const float* u_draft, float temperature, int B, int Gmax, int V,
                          int32_t* draft_tokens, void* workspace, size_t workspace_bytes, void* stream);

/* bs_softmax_verify for a round whose draft rows 0..gamma_b-1 all went through bs_draft_sample on
 * the same workspace: same arguments, outputs and arithmetic, but the draft rows are not streamed
 * again -- their statistics are taken from the workspace and only the logit of each drafted token
 * is read, so the call reads gamma_b + 1 rows per sequence instead of 2 gamma_b + 1.  A sequence
 * with an undrafted position below gamma_b gets accept_len = 0 and the status bit
 * BS_DEV_DRAFT_MISSING.  The drafted marks are consumed: the next round drafts again.
 * bs_residual_sample follows as after bs_softmax_verify.  Same alignment requirement as
 * bs_draft_sample. */
bs_status bs_softmax_verify_drafted(const void* target_logits, const void* draft_logits, bs_dtype dtype,
                                    const int32_t* draft_tokens, const int32_t* gamma, const float* u_accept,
                                    float temperature, int B, int Gmax, int V,
                                    int32_t* accept_len, float* p_tok, float* q_tok,
                                    void* workspace, size_t workspace_bytes, void* stream);

/* bs_verify_walk for a round whose draft rows went through bs_draft_sample on the same workspace
 * (see bs_softmax_verify_drafted): only target rows are walked, position after position; of each
 * draft row the statistics left by drafting and the logit of the drafted token are used, and the
 * draft row of the stop position is read once for the residual.  Same arguments, outputs and
 * requirements as bs_verify_walk; an undrafted position stops the sequence there with
 * BS_DEV_DRAFT_MISSING; the drafted marks are consumed. */
bs_status bs_verify_walk_drafted(const void* target_logits, const void* draft_logits, bs_dtype dtype,
                                 const int32_t* draft_tokens, const int32_t* gamma, const float* u_accept,
                                 const float* u_resample, float temperature, int B, int Gmax, int V,
                                 int32_t* accept_len, float* p_tok, float* q_tok, int32_t* out_tokens,
                                 int32_t* out_len, void* workspace, size_t workspace_bytes, void* stream);

/* ---- greedy verification of a tree of drafted tokens (Section 3, example (2): the tree structure of
 *      the draft is the hyperparameter an arm stands for; Section 2: greedy decoding) -------------- */

/* The paper prints no verification rule for trees; at temperature -> 0 it is determined by Section 2
 * alone.  The target is a point mass on its arg-max, so the accept rule of Algorithm 6 accepts a drafted
 * token iff it IS the target's arg-max at its parent.  Node 0 is the prompt; node n = 1..n_b carries the
 * drafted token node_tokens[b, n-1] and hangs under node_parent[b, n-1], an earlier node (0..n-1).
 * Row n of target_logits[b] is the target's next-token distribution after the path to node n (what
 * a forward pass with tree attention returns), row 0 the one after the prompt.  A node passes iff its
 * parent passes (the prompt does) and its token is the arg-max of its parent's row (lowest index
 * among equal maxima).  The accepted path ends at the deepest passing node (the lowest-numbered one
 * among equally deep ones, which only matters if the draft repeated a token among siblings); the
 * arg-max of that node's own row is emitted after it.  Sampling mode is not offered for trees.
 *
 *  target_logits [B, Nmax+1, V] dtype; rows above n_b are never read
 *  node_parent   [B, Nmax] int32; node_tokens [B, Nmax] int32; n_nodes [B] int32, 0 <= n_b <= Nmax
 *  accept_len    [B] out: tau_b = depth of the node the accepted path ends at
 *  out_nodes     [B, Nmax] out or NULL: the nodes of the accepted path in order (the caller keeps
 *                their key/value entries), -1 behind it
 *  out_tokens    [B, Nmax+1] out: the accepted tokens, then the emitted arg-max, -1 behind it
 *  out_len       [B] out: y_b = tau_b + 1, the reward of the arm (Section 3)
 *  workspace     bs_workspace_bytes(B, Nmax, V) bytes; Nmax <= BS_MAX_GAMMA
 * Device-detected problems: n_b outside [0, Nmax] (BS_DEV_BAD_GAMMA, processed as the empty tree), a
 * token outside [0, V) (BS_DEV_BAD_TOKEN, the node never passes), a parent that is not an earlier
 * node (BS_DEV_BAD_TREE).  Two launches: the row-statistics kernel of bs_softmax_verify in greedy
 * mode (one arg-max per row, every valid logit read once) and a walk over the nodes. */
bs_status bs_tree_verify_greedy(const void* target_logits, bs_dtype dtype, const int32_t* node_parent,
                                const int32_t* node_tokens, const int32_t* n_nodes, int B, int Nmax, int V,
                                int32_t* accept_len, int32_t* out_nodes, int32_t* out_tokens, int32_t* out_len,
                                void* workspace, size_t workspace_bytes, void* stream);

/* Per-sequence trees from a table of K tree shapes (the arms): sequence b gets the parents and the node
 * count of shape arm[b], as bs_bandit_select chose it (arm[b] < 0, an inactive sequence: the empty tree).
 *  shape_parent [K, Nmax] int32, shape_nodes [K] int32, arm [B] int32 (all device)
 *  node_parent  [B, Nmax] out, n_nodes [B] out */
bs_status bs_tree_expand_shapes(const int32_t* shape_parent, const int32_t* shape_nodes, const int32_t* arm, int K,
                                int B, int Nmax, int32_t* node_parent, int32_t* n_nodes, void* stream);

/* ---- fused LM head (Algorithm 6, second line: the models are evaluated on all drafted positions
 *      in parallel; the last step of that evaluation is logits = H W) -------------------------- */

/* Bytes of device scratch bs_lmhead_verify needs.  The first bs_workspace_bytes(B, Gmax, V) bytes
 * are an ordinary verification workspace (clear it with bs_workspace_init before the first call),
 * so the same pointer and size are then handed to bs_residual_sample and bs_get_device_status.
 * Returns 0 for arguments outside the limits. */
size_t bs_lmhead_workspace_bytes(int B, int Gmax, int V);

/* Computes the target and draft logits from the final hidden states on the tensor cores
 * (bf16 x bf16 products, fp32 accumulation), the softmax statistics of every row while the
 * logits are still on chip, and then the accept test and first-rejection scan of
 * bs_softmax_verify.  The fp32 logits are written out so that
 *   bs_residual_sample(logits_t_out, logits_d_out, BS_F32, ..., workspace, ...)
 * can follow on the same stream.
 *
 *  H_t  [B * (Gmax+1), d_t] bf16, d_t contiguous: row b * (Gmax+1) + j is the target model's final
 *       hidden state at drafted position j of sequence b (j = Gmax is the bonus position)
 *  W_t  [d_t, V] bf16, V contiguous: the target model's output embedding
 *  H_d  [B * Gmax, d_d] bf16, W_d [d_d, V] bf16: the same for the draft model; all four may be
 *       NULL (and d_d 0) iff temperature == 0 or Gmax == 0
 *  logits_t_out [B, Gmax+1, V] fp32 out;  logits_d_out [B, Gmax, V] fp32 out (NULL iff no draft product)
 *  draft_tokens, gamma, u_accept, temperature, accept_len, p_tok, q_tok: as bs_softmax_verify
 *  workspace    at least bs_lmhead_workspace_bytes(B, Gmax, V) bytes, 256-byte aligned
 * Every row of H is multiplied, padded positions (j > gamma_b) included: they must be readable
 * and their logits are written, but they take no part in the verification.
 * Requirements: V, d_t and d_d multiples of 8; all matrix pointers 16-byte aligned; otherwise
 * BS_ERR_UNSUPPORTED / BS_ERR_INVALID_ARG.  A pipeline wait inside the kernel that does not
 * complete within about a second makes bs_get_device_status return BS_ERR_TIMEOUT. */
bs_status bs_lmhead_verify(const void* H_t, const void* W_t, int d_t, const void* H_d, const void* W_d, int d_d,
                           const int32_t* draft_tokens, const int32_t* gamma, const float* u_accept,
                           float temperature, int B, int Gmax, int V,
                           float* logits_t_out, float* logits_d_out,
                           int32_t* accept_len, float* p_tok, float* q_tok,
                           void* workspace, size_t workspace_bytes, void* stream);

/* ---- the key / value cache of a round ------------------------------------------------------
 *
 * The target model evaluates the pending token and all drafts of a sequence in one pass (Algorithm 6,
 * second line), which in a transformer is an attention of 1 + gamma_b new tokens (a chain) or 1 + n_b (a tree;
 * row 0 is the root, row n node n) over the tokens so far.  These four calls keep those tokens' keys and values:
 *
 *   bs_cache_plan       block tables, slots and positions of the round's new tokens
 *   bs_cache_append     their keys and values into the cache (each layer)
 *   bs_cache_attention  attention of the new tokens over the cache (each layer)
 *   bs_cache_keep_path  trees only, after the verification: the accepted path to the front (each layer)
 *
 * Rejected tokens need no call: the next bs_cache_plan is told how many of them stay (`kept`, the out_len of the
 * verification) and their slots are written again.
 *
 * The cache is held in 8 bits: codes [n_blocks, Hkv, block_tokens, d] e4m3 and scales [n_blocks, Hkv] fp32, for the
 * keys and for the values; value = code * scale.  A block holds block_tokens (16, 32, 64 or 128) consecutive
 * tokens of one sequence.  d is 64 or 128.  block_table [B, max_blocks] int32 lists the blocks of every sequence in
 * order; entries behind those it holds are never read.  New tokens are packed: those of sequence b are rows
 * cu_new[b] .. cu_new[b + 1] - 1 of the query, key and value arrays.  block table, lengths and slots are the same
 * for all layers.  Scales are positive and finite; a block that nothing was written to needs none.  bs_cache_attention may
 * be given tables whose sequences share blocks (a common prefix); a block that a call writes to belongs to one sequence, and in
 * the tables of a plan every block stands in one place, but for the leading ones that n_shared of bs_cache_plan_next counts.
 * `status` [B] int32 or NULL: bs_cache_plan writes its BS_DEV_* bits, the other calls add theirs. */

/* Block tables and slot maps from lengths that are on the device.  One launch, two where T is above 8192.
 *
 *  seq_len     [B] in / out: tokens of every sequence in the cache.  kept[b] tokens of the round before are added first
 *  kept        [B] or NULL (= 0)
 *  n_new       [B]; n_new[b] + extra new tokens come (gamma and extra = 1 for a round, prompt lengths and 0 for prompts)
 *  active      [B] uint8 or NULL (= all); an inactive sequence keeps nothing, gets nothing and returns what it does not need
 *  block_table [B, max_blocks] in / out, n_held [B] in / out: the blocks every sequence holds
 *  free_blocks [n_blocks] in / out, n_free [1] in / out: the stack of free blocks, its top at n_free - 1
 *  kv_len      [B] out: seq_len + new tokens, what bs_cache_attention reads
 *  cu_new      [B + 1] out: prefix sums of the new tokens
 *  slot_map    [T] out: block * block_tokens + offset of every new token, -1 behind the last one
 *  positions   [T] out or NULL: position of every new token in its sequence, -1 behind the last one
 *
 * Afterwards sequence b holds ceil((seq_len + new) / block_tokens) blocks: surplus blocks are returned (a sequence
 * with seq_len = 0 and no new tokens returns all), missing ones taken, in the order of the sequences.  If the stack runs
 * out (or slot_map is full) at some sequence, it and every later one that needs a block (a slot) gets no new tokens
 * and keeps what it held: BS_DEV_NO_BLOCKS (BS_DEV_NO_ROOM).  A sequence whose lengths make no sense
 * (BS_DEV_BAD_LENGTH) is left as it is, with kv_len 0.  Freed entries of block_table are set to -1.  A plan whose
 * tokens are all given back restores the stack. */
bs_status bs_cache_plan(int32_t* seq_len, const int32_t* kept, const int32_t* n_new, int extra, const uint8_t* active,
                        int B, int block_tokens, int32_t* block_table, int max_blocks, int32_t* n_held,
                        int32_t* free_blocks, int n_blocks, int32_t* n_free, int32_t* kv_len, int32_t* cu_new,
                        int32_t* slot_map, int32_t* positions, int T, int32_t* status, void* stream);

/* The same where the round before may have refused sequences, and where sequences share a prefix.  A refused sequence has
 * no rows in the packed arrays, but the verification of the whole batch still returns an out_len for it; those tokens
 * were never in the cache.
 *
 *  last_cu [B + 1] or NULL: cu_new of the plan whose new tokens `kept` counts (the array cu_new itself may be passed: it is read
 *          before it is written).  A sequence that got no new tokens then keeps none, whatever kept says; one that is
 *          said to keep more than it got is BS_DEV_BAD_LENGTH.  NULL, and bs_cache_plan: kept is taken as it is, and
 *          has to be 0 where the plan before set a bit of status.
 *  n_shared [B] or NULL (= 0): the first n_shared[b] blocks of the row, full ones, are shared with other sequences and only
 *          read.  They count in n_held and are never returned, also when the sequence ends; a sequence whose new tokens would
 *          lie in them (seq_len < n_shared * block_tokens), or that holds fewer, is BS_DEV_BAD_LENGTH.  The caller knows who still
 *          reads them: the row of a sequence that ended is let go of with n_held[b] = n_shared[b] = 0, the last reader's with
 *          n_shared[b] = 0 alone, and then they go back to the stack with the rest. */
bs_status bs_cache_plan_next(int32_t* seq_len, const int32_t* kept, const int32_t* last_cu, const int32_t* n_shared,
                             const int32_t* n_new, int extra, const uint8_t* active, int B, int block_tokens,
                             int32_t* block_table, int max_blocks, int32_t* n_held, int32_t* free_blocks, int n_blocks,
                             int32_t* n_free, int32_t* kv_len, int32_t* cu_new, int32_t* slot_map, int32_t* positions, int T,
                             int32_t* status, void* stream);

/* Writes the new tokens' keys and values into their slots, quantised.
 *
 *  k, v      [T, Hkv, d] dtype, d contiguous; strides of a token and of a head in elements, multiples of 16 bytes,
 *            16-byte aligned (views of a fused projection are fine)
 *  slot_map  [T]: tokens with slot -1, or outside the cache, are skipped
 *
 * The scale of a (block, head) is the smallest power of two >= 2^-64 that brings the largest finite magnitude among
 * the new tokens to 448 or less, and no smaller than the block's present scale if the first new token is not the
 * first of its block; the codes of older tokens then follow (rounded once more only where they become subnormal).
 * Codes are rounded to nearest even, infinities become +-448 scales, NaN stays NaN.  The new tokens of a block must be
 * consecutive rows with consecutive slots, as bs_cache_plan gives them; two separate runs in one block, in
 * one call, are not supported. */
bs_status bs_cache_append(const void* k, const void* v, bs_dtype dtype, long long k_stride_t, long long k_stride_h,
                          long long v_stride_t, long long v_stride_h, const int32_t* slot_map, int T, int Hkv, int d,
                          void* k_cache, float* k_scale, void* v_cache, float* v_scale, int n_blocks, int block_tokens,
                          void* stream);

/* Bytes of scratch bs_cache_attention needs on the current device for these heads (any batch and length);
 * 0 for unsupported ones.  Clear it once with bs_workspace_init. */
size_t bs_cache_workspace_bytes(int Hq, int Hkv, int d);

/* Whether a bounded wait gave up in any bs_cache_attention on this workspace since it was cleared: BS_ERR_TIMEOUT, else
 * BS_OK.  Synchronises `stream`.  Clear the workspace with bs_workspace_init before it is used again. */
bs_status bs_cache_get_device_status(const void* workspace, size_t workspace_bytes, void* stream);

/* Attention of the new tokens over the cache: out_i = sum_j softmax_j(softmax_scale * q_i . k_j) v_j.
 *
 *  q, out       [T, Hq, d] bf16, d contiguous; strides of a token and of a head in elements, multiples of 8, 16-byte
 *               aligned.  Query head i reads key head i / (Hq / Hkv); Hq / Hkv <= 64
 *  cu_new, kv_len, block_table  from bs_cache_plan; kv_len includes the new tokens
 *  node_parent  NULL: a chain, new token i of sequence b sees positions <= kv_len[b] - n_new_b + i.
 *               [B, Nmax] (Nmax <= 31): trees as in bs_tree_verify_greedy, new token n sees the tokens before the tree,
 *               its ancestors and itself
 *  max_new      the largest number of new tokens of a sequence, as far as known on the host: chooses the tile, any
 *               value >= 1 gives the same result up to rounding
 *  workspace    bs_cache_workspace_bytes bytes, 256-byte aligned, cleared once; calls that may overlap need one each
 *
 * Keys and values enter the tensor cores as the e4m3 codes they are; a bf16 query is split into two e4m3 numbers, which
 * holds it exactly down to 2^-9 of its row's largest element; probabilities are split the same way, relative error at
 * most 2^-8 where they are within 2^-10 of the largest of their 128-token tile and absolute error 2^-18 of that
 * below.  Products accumulate in fp32, tiles are joined in fp32.
 * Range of the scales, which need not be powers of two: those of K at most 2^100, and softmax_scale x largest |q| of a row x scale of
 * K below 2^120; those of V from 2^-64 to 2^100, and the ones that a sequence reads within 2^96 of one another.  Outside it results
 * are undefined.  (bs_cache_append writes 2^-64 and more, and more than 2^100 only for values above 5e32.)
 * A token that sees nothing (kv_len < its position) gets zeros.  Rows of out behind cu_new[B] are left as they are, and so
 * are the rows of a sequence with BS_DEV_BAD_LENGTH (lengths outside the block table, cu_new not ascending or
 * above T; trees: more than Nmax + 1 new tokens).  BS_DEV_BAD_BLOCK: the rows of that sequence are undefined.
 * Results do not depend on the order in which CTAs run. */
bs_status bs_cache_attention(const void* q, long long q_stride_t, long long q_stride_h, const int32_t* cu_new,
                             const int32_t* kv_len, const int32_t* block_table, int max_blocks,
                             const int32_t* node_parent, int Nmax, const void* k_cache, const float* k_scale,
                             const void* v_cache, const float* v_scale, int n_blocks, int block_tokens, int B, int T, int Hq,
                             int Hkv, int d, int max_new, float softmax_scale, void* out, long long out_stride_t,
                             long long out_stride_h, int32_t* status, void* workspace, size_t workspace_bytes, void* stream);

/* After bs_tree_verify_greedy: moves the accepted path to the front of its tree, token seq_len + out_nodes[b, j] to
 * position seq_len + 1 + j for j < accept_len[b] (the root is in place), keys and values of one layer.
 *
 *  out_nodes [B, Nmax] and accept_len [B] from bs_tree_verify_greedy; seq_len [B] from bs_cache_plan of the round (tokens
 *  before the tree).
 * A destination block's scale becomes the largest of its own and those of the blocks its tokens come from.  A sequence
 * with BS_DEV_BAD_LENGTH, BS_DEV_BAD_TREE (nodes that do not ascend) or BS_DEV_BAD_BLOCK is left as it is, and so is one whose
 * status says that bs_cache_plan gave it no new tokens (pass the plan's status; with NULL its accept_len has to be 0). */
bs_status bs_cache_keep_path(const int32_t* out_nodes, const int32_t* accept_len, const int32_t* seq_len, int B, int Nmax,
                             const int32_t* block_table, int max_blocks, int Hkv, int d, void* k_cache, float* k_scale,
                             void* v_cache, float* v_scale, int n_blocks, int block_tokens, int32_t* status, void* stream);

/* ---- prompts and rotary positions ------------------------------------------------------------
 *
 * A prompt enters in the order bs_cache_plan, then in each layer bs_rotary, bs_prompt_attention, bs_cache_append; a round in the
 * order bs_cache_plan, then in each layer bs_rotary, bs_cache_append, bs_cache_attention.  (A prompt that comes in pieces
 * attends through bs_cache_attention, too.) */

/* Scaling of the frequencies base^(-2 i / rot) of pair i for contexts longer than `original`, the length that a model was
 * trained at. */
typedef enum {
    BS_ROTARY_PLAIN = 0,
    BS_ROTARY_LINEAR = 1,     /* all divided by factor */
    BS_ROTARY_BANDS = 2,      /* pairs that turn `high` times or more within the original length keep their frequency, those
                                 that turn `low` times or less are divided by factor, between the two it goes over linearly in the turns */
    BS_ROTARY_YARN = 3        /* pairs below the one that turns `high` times keep theirs, those above the one that turns `low`
                                 times are divided, between the two (rounded outwards) it goes over linearly in the pair's number; the
                                 amplitude is 0.1 ln(factor) + 1 */
} bs_rotary_scaling;

/* Frequencies for bs_rotary, computed on the HOST with 64 bits of mantissa: freq_host [rot / 2] turns a position x 2^64, off by
 * at most 2.3, and the amplitude.  rot
 * even, 2 to 256; base > 1; factor >= 1, 0 < low < high and original >= 1 where the scaling uses them. */
bs_status bs_rotary_frequencies(bs_rotary_scaling scaling, int rot, double base, double factor, double low, double high,
                                double original, uint64_t* freq_host, float* amplitude_host);

/* Rotates queries and keys to their positions: (a, b) -> amplitude (a cos w - b sin w, b cos w + a sin w) for every pair,
 * w = position x frequency.
 *
 *  q, q_out  [T, Hq, d], k, k_out [T, Hkv, d] dtype, d contiguous; strides of a token and a head in elements.  q_out may be q and
 *            k_out may be k (same strides); no other overlap of an output.  Hq or Hkv may be 0 (pointers NULL)
 *  positions [T] as bs_cache_plan gives them; rows with a negative one are left as they are (in q_out and k_out, too)
 *  freq      [rot / 2] DEVICE copy of what bs_rotary_frequencies made; rot <= d, elements from rot on are copied
 *  interleaved 0: pair i is elements i and i + rot / 2;  else: elements 2 i and 2 i + 1
 *  node_parent NULL: chains.  [B, Nmax]: trees as in bs_cache_attention, cu_new [B + 1] the plan's: row n of a sequence is rotated
 *            to position(row 0) + depth of node n, where bs_cache_keep_path will leave it if it is accepted.  A
 *            parent that is not an earlier node counts as the root; rows behind Nmax + 1 are left as they are
 * Angles are exact to 2^-31 turns at every position, then rounded to fp32 within the turn (2^-26 turns at most); sines, cosines and
 * products are fp32, results are rounded once.
 * Any strides work; those that are multiples of 16 bytes (and pointers) take the widest accesses. */
bs_status bs_rotary(const void* q, long long q_stride_t, long long q_stride_h, const void* k, long long k_stride_t,
                    long long k_stride_h, bs_dtype dtype, const int32_t* positions, const uint64_t* freq, float amplitude, int rot,
                    int interleaved, const int32_t* cu_new, const int32_t* node_parent, int B, int Nmax, int T, int Hq, int Hkv, int d,
                    void* q_out, long long qo_stride_t, long long qo_stride_h, void* k_out, long long ko_stride_t,
                    long long ko_stride_h, void* stream);

/* Causal attention of whole prompts to themselves: out_i = sum_{j <= i} softmax_j(softmax_scale * q_i . k_j) v_j within each
 * sequence.
 *
 *  q, out  [T, Hq, d], k, v [T, Hkv, d] bf16, d (64 or 128) contiguous; strides of a token and a head in elements, multiples of 8 and
 *          not negative, 16-byte aligned.  Query head i reads key head i / (Hq / Hkv); Hq / Hkv <= 64.  out overlaps no
 *          input (views of one buffer may lie between one another)
 *  cu_seqlens [B + 1]: sequence b is rows cu_seqlens[b] .. cu_seqlens[b + 1] - 1 (bs_cache_plan's cu_new, if all begin here).  Empty sequences
 *          are fine.  Rows of out behind cu_seqlens[B] are left as they are, what the other arrays hold there does not matter
 *  softmax_scale > 0 and, times log2(e), finite; T <= 2^30
 *  status  [B] or NULL: bits are added.  BS_DEV_BAD_LENGTH: a sequence outside [0, T], that ends before it begins, or that begins before
 *          the end of an earlier one: it is left out, no row is written for it; BS_DEV_TIMEOUT in status[0]: a bounded wait gave up, every output is undefined
 *          (without a status array bs_prompt_get_device_status tells)
 * Products accumulate in fp32, probabilities enter the second product as bf16.  Keys and values of later tokens may be NaN or
 * infinite without a trace; an element of v that is not finite makes that element of the rows that see it NaN or infinite.
 * Results do not depend on the order in which CTAs run. */
bs_status bs_prompt_attention(const void* q, long long q_stride_t, long long q_stride_h, const void* k, long long k_stride_t,
                              long long k_stride_h, const void* v, long long v_stride_t, long long v_stride_h,
                              const int32_t* cu_seqlens, int B, int T, int Hq, int Hkv, int d, float softmax_scale, void* out,
                              long long out_stride_t, long long out_stride_h, int32_t* status, void* stream);

/* Whether a bounded wait gave up in any bs_prompt_attention on the current device that had ended by now since the last such
 * answer: BS_ERR_TIMEOUT (once), else BS_OK.  Synchronises `stream`; calls on other streams are not waited for. */
bs_status bs_prompt_get_device_status(void* stream);

/* ---- what is done to logits before they are verified ---------------------------------------------
 *
 * History of a sequence's tokens: [B, V] int16, an entry is 2 x (times the token was emitted, up to 16383) + (1 if it is in the
 * prompt).  bs_history_update enters prompts when a sequence is admitted and the verification's out_tokens after every
 * round; bs_logits_adjust reads it before the next one. */

/* Enters tokens in the histories.
 *  history    [B, V] int16 in / out
 *  fresh      [B] uint8 or NULL (= 0): histories that begin anew, with no entry before this call's
 *  cu_prompt  [B + 1] or NULL: prompt tokens of sequence b are prompt_tokens[cu_prompt[b] .. cu_prompt[b + 1] - 1], of Tp
 *  out_tokens [B, W], out_len [B] or NULL: the first out_len[b] tokens were emitted (W <= BS_MAX_GAMMA + 1)
 *  status     [B] or NULL: bits are added.  BS_DEV_BAD_TOKEN: a token outside [0, V) was left out; BS_DEV_BAD_LENGTH: lengths outside
 *             the arrays, nothing of the sequence was entered
 * Two calls on the same history must not overlap. */
bs_status bs_history_update(int16_t* history, int B, int V, const uint8_t* fresh, const int32_t* cu_prompt,
                            const int32_t* prompt_tokens, int Tp, const int32_t* out_tokens, const int32_t* out_len, int W,
                            int32_t* status, void* stream);

/* Penalties, biases and grammar masks on the rows of a batch of logits, in this order:
 *   seen (in the prompt, emitted, or drafted on the way to this row):  x = x > 0 ? x / r : x r
 *   emitted or drafted c > 0 times:  x = x - f c - p
 *   listed:  x = x + its biases
 *   forbidden by the row's mask:  x = -inf
 *
 *  logits, out  [B, R, V] dtype, R <= BS_MAX_GAMMA + 1: target rows (R = Gmax + 1, extra = 1) or draft rows (R = Gmax, extra = 0).  out may
 *               be logits (only what changes is then written), or lies apart from them
 *  gamma        [B] or NULL (all R rows): rows row_begin <= j < min(row_end, gamma_b + extra) are adjusted, the others are neither
 *               read nor written
 *  draft_tokens [B, Nmax] or NULL, Nmax >= R - 1: row j stands behind tokens 0 .. j - 1 of a chain, or with node_parent [B, Nmax]
 *               (bs_tree_verify_greedy) behind node j and its ancestors.  They count as emitted; one outside [0, V) does not count
 *  history      [B, V] or NULL (= 0)
 *  repetition r > 0, presence p, frequency f  [B] fp32 or NULL (1, 0, 0); any of them needs a history or draft_tokens
 *  bias_begin   [B + 1] or NULL: entries bias_begin[b] .. bias_begin[b + 1] - 1 of bias_tokens and bias_values (n_bias of them) are those
 *               of sequence b; a token listed twice gets both, in the order of the list.  Meant for lists that are short
 *               against V: 32 entries cost about 10 instructions for every 256 tokens of the vocabulary
 *  masks        [n_masks, ceil(V / 32)]: bit v % 32 of word v / 32 is set where token v is allowed; mask_row [B, R] or NULL: the
 *               row's mask, -1 for none.  A row whose mask allows nothing becomes -inf throughout (BS_DEV_NONFINITE when it is verified)
 *  status       [B] or NULL: bits are added.  BS_DEV_BAD_GAMMA (outside [0, R - extra]; taken as 0), BS_DEV_BAD_MASK, BS_DEV_BAD_TOKEN (a drafted or
 *               a listed one), BS_DEV_BAD_TREE (a parent that is not an earlier node counts as the root), BS_DEV_BAD_LENGTH (biases
 *               outside their arrays, left out)
 * Arithmetic is fp32, rounded once.  A row's bits do not depend on the other rows of the call, on tokens drafted elsewhere than on its way,
 * or on what draft_tokens hold beyond gamma.  Any V works; a multiple of 8 with pointers on 16 bytes takes the widest accesses. */
bs_status bs_logits_adjust(const void* logits, void* out, bs_dtype dtype, const int32_t* gamma, int extra, int row_begin, int row_end,
                           const int32_t* draft_tokens, const int32_t* node_parent, int Nmax, const int16_t* history,
                           const float* repetition, const float* presence, const float* frequency, const int32_t* bias_begin,
                           const int32_t* bias_tokens, const float* bias_values, int n_bias, const uint32_t* masks, int n_masks,
                           const int32_t* mask_row, int B, int R, int V, int32_t* status, void* stream);

/* ---- arm selection (Algorithm 3, select and history lines) ---------------------------- */

/* Bytes of the opaque device state of B independent bandits with K arms. 0 if out of limits. */
size_t bs_bandit_state_bytes(bs_alg alg, int B, int K);

/* Resets the state: no pulls, no rounds.  arm_gamma: HOST array [K], speculation length of
 * each arm; L = max_i arm_gamma[i] is the maximum speculation length of the configuration.
 * delta: confidence parameter of UCBSpec (Algorithm 4 input; the regret proof uses 1/2);
 * ignored by EXP3Spec.  The state is plain device memory: copying its bytes checkpoints it. */
bs_status bs_bandit_init(void* state, size_t state_bytes, bs_alg alg, int B, int K,
                         const int32_t* arm_gamma_host, double delta, void* stream);

/* Chooses this round's arm for every active sequence.
 *  UCBSpec (Algorithm 4 / Algorithm 8): arm t in the first K rounds (t = completed rounds),
 *    then argmax_i  sumY_i/n_i + (L/2) sqrt((1+n_i)/n_i^2 (1 + 2 ln(K t^2 sqrt(1+n_i)/delta))),
 *    lowest index on ties.  u_arm is not read and may be NULL.
 *  EXP3Spec (Algorithm 5 / Algorithm 9): p_i proportional to exp(-eta_t S_i),
 *    eta_t = sqrt(ln K / (t K)) with t = completed rounds + 1; the arm is the smallest i whose
 *    cumulative probability strictly exceeds u_arm[b]; p of the chosen arm is kept for the update.
 *  u_arm   [B] fp32 uniforms in (0,1) (EXP3Spec)
 *  active  [B] uint8 or NULL (= all active); inactive sequences get arm = -1, gamma = 0
 *  arm     [B] int32 out;  gamma [B] int32 out = arm_gamma[arm]
 *  index_out [B, K] fp64 out or NULL: the UCB index values / EXP3 probabilities used (NaN
 *            during UCBSpec's round-robin prefix) -- for tests and logging. */
bs_status bs_bandit_select(void* state, size_t state_bytes, bs_alg alg, int B, int K,
                           const float* u_arm, const uint8_t* active,
                           int32_t* arm, int32_t* gamma, double* index_out, void* stream);

/* Records the outcome of the round for every active sequence.
 *  UCBSpec: n[arm] += 1, sumY[arm] += y, t += 1.
 *  EXP3Spec: S[arm] += (L + 1 - y) / (L * p_arm), t += 1  (loss estimate of Algorithm 9).
 *  arm [B] int32 in (as returned by select); reward_y [B] int32 in, 1 <= y <= L+1
 *  (out_len of bs_residual_sample); values outside that range are clamped. */
bs_status bs_bandit_update(void* state, size_t state_bytes, bs_alg alg, int B, int K,
                           const int32_t* arm, const int32_t* reward_y, const uint8_t* active,
                           void* stream);

/* bs_bandit_update of this round and bs_bandit_select of the next in one launch (Algorithm 3: the
 * history line of round t, then the select line of round t + 1), with the same results as the
 * two calls.
 *  reward_y [B] int32 (UCBSpec, EXP3Spec) or reward_r [B] fp64 (BS_UCB_REWARD): the other may be NULL
 *  u_arm_next [B] fp32: the uniforms of the next round's draw (EXP3Spec; else may be NULL)
 *  active: one mask for both steps (NULL = all active)
 *  arm [B] int32 in/out: the arms played this round on entry, the next round's arms on return
 *  gamma [B] int32 out: the next round's speculation lengths.  It must not be the array a kernel
 *  still in flight on another stream reads; on one stream the call is ordered like any other.
 *  index_out as in bs_bandit_select. */
bs_status bs_bandit_step(void* state, size_t state_bytes, bs_alg alg, int B, int K,
                         const int32_t* reward_y, const double* reward_r, const float* u_arm_next,
                         const uint8_t* active, int32_t* arm, int32_t* gamma, double* index_out,
                         void* stream);

/* Reads the sufficient statistics back to host arrays (any may be NULL).  Synchronises.
 *  UCBSpec: n_host [B,K] int64, sumY_host [B,K] int64, t_host [B] int64; S_host unused.
 *  EXP3Spec: S_host [B,K] fp64, n_host [B,K] int64 (pulls per arm, not used by the algorithm),
 *            t_host [B] int64; sumY_host unused. */
bs_status bs_bandit_read(const void* state, size_t state_bytes, bs_alg alg, int B, int K,
                         int64_t* n_host, int64_t* sumY_host, double* S_host, int64_t* t_host,
                         void* stream);

/* ---- throughput as the reward (Section 6.2) -------------------------------------------
 * Section 6.2 runs UCBSpec over the speculation lengths {0, ..., 4} (0 = canonical decoding,
 * Algorithm 1) with "the current throughput", generated tokens per second, as the reward, and
 * prints no formula.  Reading: alg = BS_UCB_REWARD is Algorithm 8 with the history holding
 * real rewards r in [0, W] and the radius factor L/2 (half the width of [1, L+1], where the
 * accepted length lives) replaced by W/2.  bs_bandit_state_bytes, bs_bandit_select and
 * bs_bandit_read take BS_UCB_REWARD; bs_bandit_init and bs_bandit_update do not (they return
 * BS_ERR_INVALID_ARG): use the two calls below.  bs_bandit_read: n_host [B,K] int64 pulls,
 * S_host [B,K] fp64 reward sums, t_host [B] int64; sumY_host unused. */

/* bs_bandit_init for BS_UCB_REWARD.  reward_width = W > 0, finite.  arm_gamma may be all
 * zero (L is not used by this algorithm). */
bs_status bs_bandit_init_reward(void* state, size_t state_bytes, int B, int K,
                                const int32_t* arm_gamma_host, double delta, double reward_width,
                                void* stream);

/* n[arm] += 1, sumR[arm] += r, t += 1 for every active sequence.
 *  arm [B] int32 device, as returned by select;  reward [B] fp64 device: values outside
 *  [0, W] are clamped into it, NaN counts as 0. */
bs_status bs_bandit_update_reward(void* state, size_t state_bytes, int B, int K,
                                  const int32_t* arm, const double* reward, const uint8_t* active,
                                  void* stream);

/* The round's throughput as a reward, on the device (fp64).
 *  out_len [B] int32 device: tokens sequence b emitted in the round (bs_residual_sample)
 *  seconds: HOST scalar > 0, finite: what the caller measured for the round
 *  whole_batch = 0: reward[b] = out_len[b] / seconds
 *  whole_batch = 1: reward[b] = (sum of out_len over the active sequences) / seconds for every
 *                   active b -- bandits that start together then stay together, so the batch
 *                   shares one speculation length, as one serving step does
 *  reward [B] fp64 device out; inactive sequences get 0. */
bs_status bs_throughput_reward(const int32_t* out_len, const uint8_t* active, int B, double seconds,
                               int whole_batch, double* reward, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* BANDITSPEC_H_ */
