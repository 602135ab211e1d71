/*
 * psd.h — C ABI of the PSD (Parallel Speculative Decoding for diffusion LLMs) per-step hot path
 * for NVIDIA B200 (sm_100a).
 *
 * One decoding step of PSD, seen from the LM head onwards, is four operations:
 *
 *   psd_confidence      x^_i = argmax_v p(v), c_i = max_v p(v) for every row of final hidden
 *                       states, p = softmax(hidden · W_lm^T)            (Sec. 3.1; Sec. 3.2 Stage 3)
 *   psd_verify_accept   hierarchical acceptance of a chain of drafts    (Sec. 3.2 Stage 3; Alg. 1 Stage 3)
 *   psd_select_unmask   transfer policy pi and the state update          (Sec. 3.2 Stage 1; Eq. (1))
 *   psd_build_drafts    speculative ordering sigma and draft assembly    (Sec. 3.2 Stage 2; Eq. (2))
 *
 * Conventions, common to every entry point unless it says otherwise:
 *   - Every array pointer is a DEVICE pointer owned by the caller.  The library allocates no
 *     device memory.  The computing entry points keep no state between calls; the only state the
 *     library holds is a handful of process-wide settings (psd_set_confidence_impl, psd_set_tuning)
 *     and a per-thread profiling hook (psd_set_kernel_events), all listed at the end of this file.
 *     The settings are plain atomics read at the start of a call: changing one while another thread
 *     is inside a call is not supported (PSD_TUNE_COMPACT_ROWS, for one, changes how much workspace
 *     psd_step needs and which entries of tokV / confV it writes), so set them before the threads
 *     that compute are started, or serialise.
 *   - Calls are asynchronous on `cuda_stream` (a cudaStream_t passed as void*; NULL = the
 *     default stream).  Outputs are valid once the stream has reached the end of the call.
 *   - The return value is PSD_OK or a negative psd_status code.  Argument errors are detected
 *     on the host before anything is launched; nothing is written in that case.
 *   - Layouts are row-major and dense.  A "block" is one sequence's active block of M slots.
 *     B = blocks, D = chain nodes per block in the verification batch (root included; the paper's
 *     draft depth d equals D-1), rows of the verification batch are ordered (b, d, i):
 *     row = (b*D + d)*M + i.
 *   - mask arrays hold 1 for a masked slot ([M] in the paper) and 0 for a committed one.
 *   - No exceptions, no output on stdout/stderr, plain C linkage.
 */
#ifndef PSD_H_
#define PSD_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum psd_status {
    PSD_OK = 0,
    PSD_ERR_NULL = -1,        /* a required pointer is NULL                                        */
    PSD_ERR_SHAPE = -2,       /* a size is out of range (see each call)                            */
    PSD_ERR_ALIGN = -3,       /* a pointer is not aligned as required                              */
    PSD_ERR_WORKSPACE = -4,   /* workspace smaller than psd_workspace_bytes()                      */
    PSD_ERR_POLICY = -5,      /* k_min < 1, 0 < k_max < k_min, depth out of range, stride < 0,
                                 unknown accept_mode, or tau is NaN                                 */
    PSD_ERR_CUDA = -6,        /* a CUDA runtime or driver call failed (launch, tensor-map encode)  */
    PSD_ERR_UNSUPPORTED = -7, /* a reserved argument was used                                      */
    PSD_ERR_TIMEOUT = -8,     /* device side only, via status_dev: a bounded wait inside a kernel
                                 ran out; the kernel returned early and its outputs are invalid    */
    PSD_ERR_INTERNAL = -9     /* device side only, via status_dev, and only from the library's debug
                                 build (compiled with PSD_DEBUG): a bounds or ring-order check inside
                                 a kernel failed; the offending access was skipped                  */
} psd_status;

/*
 * The device status word (`status_dev` of the entry points that take one): a device int32 that the
 * CALLER zeroes.  After the call it holds
 *     < 0   a psd_status code detected on the device (PSD_ERR_TIMEOUT; PSD_ERR_INTERNAL from the debug
 *           build); it is never replaced by a count;
 *     > 0   PSD_ERR_NONFINITE count: the number of scored rows whose logits held a NaN or an infinity,
 *           so that their confidence is NaN (such a row ranks below every number in the policy and
 *           never exceeds tau; nothing faults);
 *       0   neither.
 * Counts of successive calls add up when the word is not zeroed in between.
 */

/* Limits checked by the entry points. */
#define PSD_MAX_M 1024     /* slots per block                        */
#define PSD_MAX_DEPTH 64   /* chain nodes per block, root included   */

/* accept_mode: the form of the acceptance criterion A_pi(x~_{k,i}, x^_{p,i}, c_{p,i}) of
 * Algorithm 1 (the paper gives "sufficient confidence" as its example and leaves the form open). */
#define PSD_ACCEPT_AGREE_AND_CONF 0   /* x~ == x^_p  and  c_p > tau              (default) */
#define PSD_ACCEPT_AGREE_ONLY 1       /* x~ == x^_p                                         */
#define PSD_ACCEPT_AGREE_AND_POLICY 2 /* x~ == x^_p  and  i is in pi(parent's draft, c_p)  */

/*
 * Parameters of the transfer policy and of the draft chain, passed by value.
 *
 * The policy is confidence thresholding (App. B.2: unmask every masked position whose top-1
 * confidence exceeds tau, strictly), clamped to at least k_min positions (so that the decoding
 * loop of Algorithm 1 always progresses) and at most k_max.  k_min = k_max = 1 is greedy decoding,
 * k_min = k_max = k is fixed-k parallel decoding (Sec. 2.1).
 */
typedef struct psd_policy_t {
    float tau;           /* commit / acceptance threshold, compared with '>' in fp32              */
    int32_t k_min;       /* >= 1                                                                  */
    int32_t k_max;       /* >= k_min, or 0 for "no cap"                                           */
    int32_t depth;       /* D, 1 .. PSD_MAX_DEPTH; D = 1 means no speculation                     */
    int32_t stride;      /* slots each further depth speculates; 0 means k_min                    */
    int32_t accept_mode; /* PSD_ACCEPT_*                                                          */
    int32_t mask_id;     /* token id of [M]; written to no output, kept for callers' bookkeeping  */
} psd_policy_t;

/* Text for a psd_status code (static storage, never NULL). */
const char* psd_status_string(int code);

/*
 * Bytes of scratch that psd_confidence needs for n_rows x H x V.  Returns 0 for invalid sizes.
 * The scratch holds the per-row partial (max, sum-exp, argmax) triples of every vocabulary split.
 */
size_t psd_workspace_bytes(int32_t n_rows, int32_t H, int32_t V);

/*
 * Bytes of scratch for the paths that first copy the rows to score into a dense buffer: psd_confidence
 * with a row list, and psd_step / psd_decode_blocks with PSD_TUNE_COMPACT_ROWS on (n_rows = B*D*M).
 * Always >= psd_workspace_bytes.  Returns 0 for invalid sizes.
 */
size_t psd_compact_workspace_bytes(int32_t n_rows, int32_t H, int32_t V);

/*
 * psd_confidence — LM head + softmax max-probability + argmax, without ever storing logits.
 * (Sec. 3.1: x^_i and c_i; used for the single sequence of Stage 1 and for all drafts of the
 *  batched verification pass of Stage 3.)
 *
 * For each row r:  l_v = sum_j hidden[r,j] * w_lm[v,j]  (bf16 inputs, fp32 accumulation),
 *   out_token[r] = the lowest v attaining max_v l_v,
 *   out_conf[r]  = 1 / sum_v exp(l_v - max_v l_v)   ( = max_v softmax(l)_v ),
 *   out_lse[r]   = max_v l_v + ln sum_v exp(l_v - max_v l_v)      (optional).
 *
 *   hidden_bf16  [n_rows, H] bf16, 16-byte aligned, device
 *   w_lm_bf16    [V, H]      bf16, 16-byte aligned, device
 *   row_ids      NULL, or a device list [n_rows] int32 of the rows of hidden_bf16 to score (a gather list:
 *                output r belongs to hidden row row_ids[r]; hidden_bf16 may then have any number of rows;
 *                every id must be a valid row of it, the library does not check).
 *                The workspace must then hold psd_compact_workspace_bytes(n_rows, H, V)
 *   n_rows >= 1;  H >= 64 and a multiple of 64;  1 <= V < 2^31 - 256
 *   out_token    [n_rows] int32;  out_conf [n_rows] fp32;  out_lse [n_rows] fp32 or NULL
 *   workspace    >= psd_workspace_bytes(n_rows, H, V) bytes, 256-byte aligned, device; contents
 *                are overwritten; concurrent calls need distinct workspaces
 *   status_dev   NULL, or the device status word (see above): PSD_ERR_TIMEOUT if a bounded wait inside
 *                the kernel expired (outputs are then invalid), else the number of non-finite rows
 * Rows whose logits contain NaN produce out_conf = NaN and are counted in status_dev.
 */
int psd_confidence(const void* hidden_bf16, const void* w_lm_bf16, const int32_t* row_ids,
                   int32_t n_rows, int32_t H, int32_t V,
                   int32_t* out_token, float* out_conf, float* out_lse,
                   void* workspace, size_t workspace_bytes,
                   int32_t* status_dev, void* cuda_stream);

/*
 * psd_confidence_masked — psd_confidence on the rows whose row_mask is non-zero, without the host
 * knowing how many there are (Sec. 3.2 Stage 3 needs predictions only at "each masked position").
 * row_mask [n_rows] int32, device: typically the mask of the sequences themselves ([B, M] or
 * [B, D, M] flattened).  Outputs of flagged rows are written at the rows' own places; outputs of the
 * other rows are left untouched.  No host synchronisation: the rows are listed and copied into a dense
 * buffer on the device, and the fused kernel reads their number from device memory.
 * workspace >= psd_compact_workspace_bytes(n_rows, H, V).  Other arguments as for psd_confidence.
 */
int psd_confidence_masked(const void* hidden_bf16, const void* w_lm_bf16, const int32_t* row_mask,
                          int32_t n_rows, int32_t H, int32_t V,
                          int32_t* out_token, float* out_conf, float* out_lse,
                          void* workspace, size_t workspace_bytes, int32_t* status_dev, void* cuda_stream);

/*
 * ---- The vocabulary split over several GPUs ----------------------------------------------------------
 * softmax max / argmax over the whole vocabulary is an associative merge of per-range triples
 * (max logit, sum of exp(logit - max), lowest argmax), the same merge that combines the vocabulary
 * tiles inside psd_confidence.  A GPU that holds rows [v_offset, v_offset + V_shard) of W computes its
 * triple per row; the triples of all GPUs (12 bytes per row and GPU) are exchanged by the caller and
 * merged on every GPU.  (Sec. 3.1 defines x^ and c over the whole vocabulary; the split is this
 * library's, for LM heads sharded over GPUs.)
 *
 * psd_confidence_partial: out_max, out_sumexp [n_rows] fp32, out_arg [n_rows] int32 (GLOBAL vocabulary
 *   index); other arguments as for psd_confidence with V = V_shard.
 * psd_merge_partials: max, sumexp, arg are [n_shards, n_rows] (shard-major, e.g. the all-gathered
 *   outputs of psd_confidence_partial); out_token, out_conf, out_lse as for psd_confidence.  Equal
 *   maxima keep the lowest global index, so the result does not depend on the number of shards
 *   beyond the rounding order of the sums.  All its arrays are 4-byte aligned (PSD_ERR_ALIGN otherwise);
 *   it takes no status word (psd_confidence_partial has counted the non-finite rows of its shard).
 */
int psd_confidence_partial(const void* hidden_bf16, const void* w_shard_bf16, int32_t n_rows, int32_t H,
                           int32_t V_shard, int32_t v_offset, float* out_max, float* out_sumexp, int32_t* out_arg,
                           void* workspace, size_t workspace_bytes, int32_t* status_dev, void* cuda_stream);
int psd_merge_partials(const float* max, const float* sumexp, const int32_t* arg, int32_t n_shards, int32_t n_rows,
                       int32_t* out_token, float* out_conf, float* out_lse, void* cuda_stream);

/*
 * psd_select_unmask — the transfer policy T = pi(x, c) and the state update of Eq. (1).
 * (Sec. 3.2 Stage 1; App. B.2 for the threshold rule.)
 *
 * conf, tok are [B, n_nodes, M]; block b reads the rows of node node[b] (node 0 when node is
 * NULL).  A prediction tok < 0 is no token (psd_confidence_logits gives -1 where nothing may be chosen):
 * here and in the calls below its slot is not counted, committed or speculated, and agrees with nothing.
 * Over the other masked slots of block b, the candidates, ranked by (confidence descending, slot ascending;
 * NaN last):  n_thr = #{c_i > tau},  n = min(#candidates, k_max or inf, max(n_thr, k_min)),  T = the first
 * n.  Then tokens[b,i] = tok[i] and mask[b,i] = 0 for i in T; every other slot is left untouched.
 * n_sel[b] = 0 with slots still masked means that none of them has a token: the block is at a dead end, and
 * the same state will give the same answer again, so a loop has to change what is allowed there or stop.
 *
 *   tokens, mask [B, M] int32, in/out
 *   sel      [B, M] int32 out: 1 where i in T, else 0
 *   n_sel    [B]    int32 out: |T|
 *   sel_pos  [B, M] int32 out: the slots of T in rank order, then -1
 *   1 <= B; 1 <= M <= PSD_MAX_M; 1 <= n_nodes <= PSD_MAX_DEPTH; node values must lie in [0, n_nodes)
 */
int psd_select_unmask(const float* conf, const int32_t* tok, const int32_t* node, int32_t n_nodes,
                      int32_t* tokens, int32_t* mask, int32_t B, int32_t M, psd_policy_t p,
                      int32_t* sel, int32_t* n_sel, int32_t* sel_pos, void* cuda_stream);

/*
 * psd_build_drafts — speculative ordering and draft assembly for a chain of D = p.depth nodes.
 * (Sec. 3.2 Stage 2; Eq. (2); Algorithm 1 Stage 2.)
 *
 * conf, tok [B, n_nodes, M] are the cached predictions the step started from (node selection as in
 * psd_select_unmask); tokens, mask [B, M] are the state AFTER psd_select_unmask.  With m masked
 * slots left that have a token (tok >= 0), sigma orders them by (cached confidence descending, slot ascending; NaN last);
 * node d fills S_d = {sigma_1 .. sigma_{n_d}}, n_d = min(m, d * s), s = stride or k_min:
 *   draft_tokens[b,d,i] = tok[i] if i in S_d else tokens[b,i];   draft_mask[b,d,i] = mask[b,i] and i not in S_d.
 * Node 0 is the root (S_0 empty).  A block with m = 0 yields D copies of its state and n_fill = 0.
 *
 *   sigma   [B, M] int32 out, -1 after the first m entries
 *   n_fill  [B, D] int32 out
 *   draft_tokens, draft_mask [B, D, M] int32 out
 */
int psd_build_drafts(const float* conf, const int32_t* tok, const int32_t* node, int32_t n_nodes,
                     const int32_t* tokens, const int32_t* mask, int32_t B, int32_t M, psd_policy_t p,
                     int32_t* sigma, int32_t* n_fill, int32_t* draft_tokens, int32_t* draft_mask,
                     void* cuda_stream);

/*
 * psd_verify_accept — hierarchical acceptance over the chain, then the commit.
 * (Sec. 3.2 Stage 3; Algorithm 1 Stage 3.)
 *
 * tokV, confV [B, D, M] are psd_confidence's outputs on the D drafts built by psd_build_drafts
 * (sigma, n_fill, draft_tokens, draft_mask as written there, D = p.depth).  Node 0 is accepted;
 * node d >= 1 is accepted iff node d-1 is and every slot i = sigma_j, n_{d-1} < j <= n_d, passes
 * A_pi against node d-1's predictions (p.accept_mode).  k* is the accepted node that fills the
 * most slots, lowest index among equals.  Then tokens, mask <- draft k*, and every slot still
 * masked in draft k* whose confV[b,k*,i] > tau is committed to tokV[b,k*,i] as well (tokens below 0 agree
 * with nothing and are not committed).
 *
 *   tokens, mask     [B, M] int32 out (fully written)
 *   k_star           [B] int32 out
 *   n_spec_accepted  [B] int32 out: n_fill[b, k*]
 *   n_committed      [B] int32 out: n_spec_accepted plus the extra commits
 *   accepted         [B, D] int32 out or NULL: 1 for accepted nodes
 */
int psd_verify_accept(const int32_t* tokV, const float* confV,
                      const int32_t* sigma, const int32_t* n_fill,
                      const int32_t* draft_tokens, const int32_t* draft_mask,
                      int32_t B, int32_t M, psd_policy_t p,
                      int32_t* tokens, int32_t* mask,
                      int32_t* k_star, int32_t* n_spec_accepted, int32_t* n_committed,
                      int32_t* accepted, void* cuda_stream);

/*
 * psd_confidence_static — psd_confidence without a workspace argument and without any allocation.
 * (The paper has no counterpart: this entry point exists for deployment, not for the method.)
 *
 * For callers that cannot allocate device memory at the point of the call — a server whose own
 * pool already owns all free HBM, a plug-in invoked from another runtime's callback where
 * cudaMalloc and its implicit synchronisation are not allowed.  The scratch that psd_confidence
 * takes from its caller lives here in a fixed array inside the library image, of
 * PSD_STATIC_SCRATCH_BYTES; every GPU that loads the library holds that much until the process exits.
 *
 * Same arguments, outputs and numerics as psd_confidence (always the tcgen05 kernel), except:
 *   - no workspace; sizes with psd_workspace_bytes(n_rows, H, V) > PSD_STATIC_SCRATCH_BYTES are
 *     rejected with PSD_ERR_WORKSPACE (e.g. 128 rows x V = 126464 needs 1.5 MB and fits;
 *     8192 rows do not);
 *   - the first call on each device looks up the array's device address
 *     (cudaGetSymbolAddress, with that device current).  CUDA loads a library's device code lazily
 *     by default, so this look-up can be the moment the driver loads the module and reserves the
 *     array's memory: make one call per device at start-up, BEFORE the process hands the rest of
 *     the device memory to its pool and outside of any stream capture.  A first call made after
 *     the memory is gone fails with PSD_ERR_CUDA.  Later calls on that device touch no allocator;
 *   - it calls no cudaMalloc, cudaFree or other allocating routine;
 *   - all calls on a device share the one array, which keeps the previous call's contents.
 *     Nothing in it needs clearing (every entry read is written first by the same call), but two
 *     calls that overlap on the GPU (different streams, or different host threads) race on it:
 *     serialise them.
 */
#define PSD_STATIC_SCRATCH_BYTES (4u << 20)
int psd_confidence_static(const void* hidden_bf16, const void* w_lm_bf16,
                          int32_t n_rows, int32_t H, int32_t V,
                          int32_t* out_token, float* out_conf, float* out_lse,
                          int32_t* status_dev, void* cuda_stream);

/*
 * All pointers of one decoding step over a batch of B blocks.  Device pointers for psd_step,
 * HOST pointers (pinned memory recommended) for psd_step_host, except w_lm_bf16 which is a
 * device pointer in both.
 */
typedef struct psd_step_io_t {
    const void* hidden_bf16;  /* in  [B*D*M, H] final hidden states of the verification batch      */
    const void* w_lm_bf16;    /* in  [V, H] DEVICE                                                 */
    int32_t* sigma;           /* in/out [B, M]    drafts being verified -> drafts for the next step */
    int32_t* n_fill;          /* in/out [B, D]                                                     */
    int32_t* draft_tokens;    /* in/out [B, D, M]                                                  */
    int32_t* draft_mask;      /* in/out [B, D, M]                                                  */
    int32_t* tokV;            /* out [B, D, M] verifier predictions                                */
    float* confV;             /* out [B, D, M] verifier confidences                                */
    int32_t* tokens;          /* out [B, M] state after acceptance and the policy                  */
    int32_t* mask;            /* out [B, M]                                                        */
    int32_t* k_star;          /* out [B]                                                           */
    int32_t* n_spec_accepted; /* out [B]                                                           */
    int32_t* n_committed;     /* out [B] acceptance commits (the policy's are in n_sel)            */
    int32_t* sel;             /* out [B, M]                                                        */
    int32_t* n_sel;           /* out [B]                                                           */
    int32_t* sel_pos;         /* out [B, M]                                                        */
} psd_step_io_t;

/*
 * psd_step — one whole step on device buffers, on one stream, with no host synchronisation:
 *   psd_confidence on all B*D*M rows  ->  psd_verify_accept on the drafts in io
 *   ->  psd_select_unmask on node k*'s predictions  ->  psd_build_drafts for the next step
 * (the verification pass of Algorithm 1 doubles as the model call of the next iteration).
 * Argument rules are those of the four calls; D = p.depth.
 */
int psd_step(const psd_step_io_t* io, int32_t B, int32_t M, int32_t H, int32_t V, psd_policy_t p,
             void* workspace, size_t workspace_bytes, int32_t* status_dev, void* cuda_stream);

/*
 * Bytes of device staging that psd_step_host needs (inputs, outputs and the step's scratch, sized so
 * that PSD_TUNE_COMPACT_ROWS may be on).  Returns 0 for invalid sizes.
 */
size_t psd_step_host_bytes(int32_t B, int32_t M, int32_t H, int32_t V, int32_t D);

/*
 * Layout of ONE host block that holds every per-step array of psd_step_io_t except hidden_bf16 and
 * w_lm_bf16.  Returns the block's size in bytes (0 for invalid sizes) and, if offsets != NULL, the 15
 * byte offsets of sigma, n_fill, draft_tokens, draft_mask, tokV, confV, tokens, mask, k_star,
 * n_spec_accepted, n_committed, sel, n_sel, sel_pos and of a status word, in this order.  When the
 * io passed to psd_step_host points into such a block (pinned memory recommended), the draft state
 * is copied up in one transfer and all outputs come back in one; any other arrangement of host
 * arrays works too, with one transfer per array.
 */
size_t psd_step_host_block(int32_t B, int32_t M, int32_t D, size_t* offsets);

/*
 * psd_step_host — psd_step for callers whose per-step data lives in host memory.
 * Copies hidden and the draft state host->device into `staging`, runs psd_step, copies every
 * output of io back device->host, and waits for the stream.  io holds HOST pointers
 * (w_lm_bf16 excepted).  staging: device, 256-byte aligned, >= psd_step_host_bytes().
 * status_host: NULL, or receives the device status word (see "The device status word").
 * Synchronous: returns after the outputs are in host memory.
 * Batches of 2048 rows or more go up in two pieces (blocks are independent: the step on the first
 * blocks, then on the rest), the second piece's copy running under the first piece's kernels on an
 * internal stream; the first such call on a device creates that stream and three events, host-side
 * objects that live until the process exits.  Results are those of psd_step on the same pieces;
 * confidences can differ from one psd_step over the whole batch in the last bits (another tiling of
 * the rows), nothing else does.  With the one-block host layout the block's status word is
 * written by this call before the copy (the block goes up whole, which zeroes the device's word).
 */
int psd_step_host(const psd_step_io_t* io, int32_t B, int32_t M, int32_t H, int32_t V, psd_policy_t p,
                  void* staging, size_t staging_bytes, int32_t* status_host, void* cuda_stream);

/*
 * ---- General draft graph (multi-parent DAG) ------------------------------------------------------------
 * (Sec. 3.2 Stage 2: nodes k with subsets S_k of {sigma_1..sigma_m}, an edge (p, k) whenever S_p is a
 *  strict subset of S_k, a node may have several parents; Algorithm 1 Stage 3 for the acceptance.)
 *
 * The graph is fixed at inference time and expressed over RANKS of the speculative ordering: bit j of
 * ranks[k] set means that node k speculates sigma_{j+1} (the slot with the (j+1)-th highest cached
 * confidence among the residual masked slots).  Only the 64 best ranks can be speculated.  Node 0 is
 * the root (ranks[0] = 0).  When fewer than 64 residual slots exist, ranks beyond them drop out of
 * every node.  bit p of parents[k] set means that (p, k) is an edge; S_p must be a strict subset of
 * S_k.  The chain of psd_build_drafts is the special case ranks[d] = lowest d*stride bits,
 * parents[d] = {d-1}.
 */
#define PSD_MAX_DAG_NODES 64
typedef struct psd_dag_t {
    int32_t n_nodes;                      /* K, 1 .. PSD_MAX_DAG_NODES */
    int32_t reserved;
    uint64_t ranks[PSD_MAX_DAG_NODES];
    uint64_t parents[PSD_MAX_DAG_NODES];
} psd_dag_t;

/*
 * Fills *g (host memory) from n_nodes rank words and, optionally, parent words.  parents == NULL makes
 * every strict-subset pair an edge (the paper's edge set).  Returns PSD_ERR_SHAPE if node 0 is not the
 * root, n_nodes is out of range, or an edge is not between a strict subset and its superset.
 */
int psd_dag_init(psd_dag_t* g, int32_t n_nodes, const uint64_t* ranks, const uint64_t* parents);

/*
 * psd_build_drafts_dag — psd_build_drafts for a draft graph: sigma as there; node k fills
 * S_k = {sigma_{j+1} : bit j of g->ranks[k], j < m}; Eq. (2).  g is a HOST pointer.
 *   n_fill [B, K] out: |S_k|;  draft_tokens, draft_mask [B, K, M] out.  p is not used (kept for symmetry).
 */
int psd_build_drafts_dag(const float* conf, const int32_t* tok, const int32_t* node, int32_t n_nodes,
                         const int32_t* tokens, const int32_t* mask, int32_t B, int32_t M, psd_policy_t p,
                         const psd_dag_t* g, int32_t* sigma, int32_t* n_fill, int32_t* draft_tokens,
                         int32_t* draft_mask, void* cuda_stream);

/*
 * psd_verify_accept_dag — hierarchical acceptance over the graph, then the commit (Algorithm 1 Stage 3).
 * tokV, confV [B, K, M] are psd_confidence's outputs on the K drafts.  The root is accepted; in
 * topological order (fewer speculated ranks first, lower index among equals) node k is accepted iff
 * some accepted parent p passes A_pi(x~_{k,i}, x^_{p,i}, c_{p,i}) (p.accept_mode) on every slot of
 * S_k \ S_p; an empty difference passes.  k* = the accepted node with the largest |S_k|, lowest index
 * among equals.  Then as psd_verify_accept: tokens, mask <- draft k*, plus node k*'s own predictions
 * above tau.  accepted [B, K] out or NULL.  p.depth and p.stride are not used.
 */
int psd_verify_accept_dag(const int32_t* tokV, const float* confV, const int32_t* sigma,
                          const int32_t* draft_tokens, const int32_t* draft_mask, int32_t B, int32_t M,
                          psd_policy_t p, const psd_dag_t* g, int32_t* tokens, int32_t* mask, int32_t* k_star,
                          int32_t* n_spec_accepted, int32_t* n_committed, int32_t* accepted, void* cuda_stream);

/*
 * psd_step_dag — psd_step with the drafts of a graph: D = g->n_nodes in every shape of io; acceptance is
 * psd_verify_accept_dag, the next drafts psd_build_drafts_dag (p.depth and p.stride are not used).
 * Runs as separate launches (fused kernel, merge, acceptance, policy, drafts) on the stream.
 */
int psd_step_dag(const psd_step_io_t* io, int32_t B, int32_t M, int32_t H, int32_t V, psd_policy_t p,
                 const psd_dag_t* g, void* workspace, size_t workspace_bytes, int32_t* status_dev,
                 void* cuda_stream);

/*
 * ---- The whole decoding loop of Algorithm 1 over a batch of blocks ----------------------------------
 *
 * The transformer body is the caller's: a function that, given token states on the device, writes
 * their final hidden states.  n_seq sequences of M slots each: tokens, mask [n_seq, M] int32 (device),
 * hidden_bf16 [n_seq * M, H] bf16 (device, row (s, i) at s*M + i).  It must enqueue its work on
 * cuda_stream and return 0, or a negative value that psd_decode_blocks passes on.
 */
typedef int (*psd_body_fn)(void* user, const int32_t* tokens, const int32_t* mask, int32_t n_seq, int32_t M,
                           void* hidden_bf16, void* cuda_stream);

/* Order of operations inside one iteration of psd_decode_blocks. */
#define PSD_ORDER_TWO_PASSES 0 /* Algorithm 1 as printed: a pass on the state, policy, drafts, a batched
                                  pass on the D drafts, acceptance                                      */
#define PSD_ORDER_ONE_PASS 1   /* psd_step: the batched pass on the drafts also serves as the next
                                  iteration's pass on the state (acceptance, then policy on node k*)   */

typedef struct psd_decode_stats_t {
    int32_t iterations;     /* iterations of the while loop that ran                                  */
    int32_t forward_passes; /* calls of the body (batched over all blocks)                            */
    int32_t masked_left;    /* masked slots left over all blocks: 0 unless max_iterations ran out     */
} psd_decode_stats_t;

/* Bytes of device scratch psd_decode_blocks needs besides psd_confidence's workspace (0 = bad sizes). */
size_t psd_decode_scratch_bytes(int32_t B, int32_t M);

/*
 * psd_decode_blocks — Algorithm 1: repeat { forward pass, policy, drafts, batched verification pass,
 * hierarchical acceptance } until no block has a masked slot left, or max_iterations.
 * (Sec. 3.2; Algorithm 1, including its early break when Stage 1 resolves the block.)
 *
 * io holds DEVICE pointers.  io->tokens, io->mask [B, M] are the blocks' state, in and out: normally
 * every slot masked on entry (token = p.mask_id, mask = 1), but any state is accepted.  io->hidden_bf16
 * is scratch of [B*D*M, H] bf16 that the body fills (the library writes through the pointer although
 * the field is const).  Every other array of io is scratch/output with the shapes given at
 * psd_step_io_t; after the call they hold the last iteration's values.  D = p.depth; with D = 1
 * nothing is speculated and every iteration is one pass (plain parallel decoding).
 *
 *   g               NULL: the drafts are the chain of p.depth nodes; else a draft graph (HOST pointer),
 *                   and D = g->n_nodes in every shape above (p.depth, p.stride are then not used)
 *   order           PSD_ORDER_TWO_PASSES or PSD_ORDER_ONE_PASS
 *   scratch         device, 256-byte aligned, >= psd_decode_scratch_bytes(B, M)
 *   workspace       as for psd_confidence with n_rows = B*D*M
 *   passes          NULL or device [B] out: forward passes charged to each block (a block is charged
 *                   for a pass only while it still has masked slots) — M / passes[b] is the block's
 *                   tokens per forward pass
 *   done_iteration  NULL or device [B] out: index of the iteration that resolved the block, -1 if none
 *   trace           NULL or device [max_iterations, B, 4] out: per iteration and block
 *                   (n_sel, k_star, n_spec_accepted, n_committed); the last three are 0 in iterations
 *                   that stopped after Stage 1
 *   stats           host, out
 * The call is synchronous: after every state update the host waits for the stream and reads the number
 * of masked slots, which the counting kernel has written straight into a pinned host word, to decide
 * whether to go on.  It allocates no device memory; the first call of a host thread allocates that one
 * 64-byte pinned word, which lives until the process exits (if that fails, the count is copied instead).
 */
int psd_decode_blocks(psd_body_fn body, void* user, const psd_step_io_t* io, int32_t B, int32_t M, int32_t H,
                      int32_t V, psd_policy_t p, const psd_dag_t* g, int32_t order, int32_t max_iterations,
                      void* scratch, size_t scratch_bytes, void* workspace, size_t workspace_bytes,
                      int32_t* status_dev, int32_t* passes, int32_t* done_iteration, int32_t* trace,
                      psd_decode_stats_t* stats, void* cuda_stream);

/*
 * psd_table_body — a stand-in body for tests and benchmarks (the paper's body is a 7-8B transformer,
 * which is outside this library): a table look-up with no arithmetic.  user points to a
 * psd_table_body_t; hidden row (s, i) = table row ((b*M + i)*3 + c), where b = s / (n_seq / B) is the
 * sequence's block and c in {0, 1, 2} counts the committed neighbours of slot i (slots i-1 and i+1 of
 * the same sequence with mask 0).  tokens is not read.
 */
typedef struct psd_table_body_t {
    const void* table_bf16; /* [B, M, 3, H] bf16, device, 16-byte aligned */
    int32_t B;
    int32_t H;              /* multiple of 8 */
} psd_table_body_t;
int psd_table_body(void* user, const int32_t* tokens, const int32_t* mask, int32_t n_seq, int32_t M,
                   void* hidden_bf16, void* cuda_stream);

/*
 * ---- Around the step: attention of the drafts, upkeep of the prefix's cache, confidences from logits ----
 *
 * The verification pass runs the body on B*D drafts that differ only in their active block: the D drafts
 * of a sequence share its prefix (prompt and finished blocks), whose keys and values are cached once per
 * sequence.  (Sec. 3.2 Stage 3: the prefix's cache can be shared by the drafts.)  A NODE is one draft of
 * one sequence, n = b*D + d; a token of the batch is t = n*M + i.  Query heads h share key head
 * h / (Hq / Hkv).  With M = 1 the same calls serve token-by-token decoding of B*D continuations.
 */
#define PSD_BF16 0
#define PSD_FP16 1
#define PSD_FP32 2 /* psd_confidence_logits only */

/* Element strides of a cache [outer, token, head, Dh]; the innermost stride is 1. */
typedef struct psd_kv_strides_t {
    int64_t outer; /* sequence (prefix cache) or node (a draft's own keys); 0 shares one among all */
    int64_t token; /* > 0 */
    int64_t head;  /* 0 shares one among all heads */
} psd_kv_strides_t;

/* Shapes of psd_draft_attention and psd_prefix_weights (which reads the fields marked *). */
typedef struct psd_attention_t {
    int32_t B, D, M;     /* * sequences, drafts per sequence, query tokens per draft; all >= 1               */
    int32_t Hq, Hkv, Dh; /* * heads, key heads (Hq a multiple of Hkv, Hq/Hkv <= 128), 8 <= Dh <= 128, Dh % 8 == 0 */
    int32_t P;           /* * token capacity of the prefix cache, >= 0                                        */
    int32_t S;           /* capacity of a draft's own keys, >= 0                                              */
    int32_t dtype;       /* * PSD_BF16 or PSD_FP16: q, caches and out                                         */
    int32_t causal;      /* own keys: 0 every row sees all own_len keys of its node; 1 query i sees own key s
                            iff s <= own_len - M + i (its node's last M own keys are the queries' own)      */
    float scale;         /* * > 0, finite                                                                     */
    int32_t reserved;    /* 0 */
    int64_t q_token, q_head;     /* * element strides of q [B*D*M, Hq, Dh]                                    */
    int64_t out_token, out_head; /* element strides of out                                                    */
    psd_kv_strides_t kp, vp;     /* * (kp) prefix caches [B, P, Hkv, Dh]                                      */
    psd_kv_strides_t ko, vo;     /* own keys and values [B*D, S, Hkv, Dh]                                     */
} psd_attention_t;

/*
 * Bytes of scratch psd_draft_attention needs (0 = bad sizes; the smallest value for good ones is 256).  With the other
 * sizes fixed the answer grows with B, D, P and S, and it serves every call with smaller ones: a workspace made for a
 * service's largest batch, drafts and cache stays large enough when sequences finish.
 */
size_t psd_attention_workspace_bytes(int32_t B, int32_t D, int32_t M, int32_t Hq, int32_t Hkv, int32_t Dh, int32_t P,
                                     int32_t S);

/*
 * Names of the kernels that psd_draft_attention launches at these sizes (static storage; NULL = bad sizes):
 * "draft_attention_kernel" (one kernel walks the prefix and the own keys), "prefix_attention_kernel" (the drafts' own
 * keys follow an unsplit prefix), or "prefix_attention_kernel+draft_attention_kernel" (partial results over the prefix,
 * then the own keys and the join).  splits, if not NULL, receives the partial results per row (0 in the first form).
 * For reports: it computes nothing.
 */
const char* psd_attention_kernel_names(int32_t B, int32_t D, int32_t M, int32_t Hq, int32_t Hkv, int32_t Dh, int32_t P,
                                       int32_t S, int32_t* splits);

/*
 * psd_draft_attention — attention of all drafts' tokens over the shared prefix, read once for all of a
 * sequence's drafts, and over each draft's own keys.
 * For token t = (b, d, i) and head h, over the keys K_j = prefix keys j < prefix_len[b] of sequence b and
 * own keys of node (b, d) that `causal` lets it see:
 *   s_j = scale * q[t,h] . K_j,   lse[t,h] = ln sum_j exp(s_j),   out[t,h] = sum_j exp(s_j - lse) V_j.
 * A row without keys gives out = 0 and lse = -inf.  Scores, softmax statistics and sums are fp32, the
 * weights are rounded to the inputs' type before they multiply V (fp16: kept large enough that none is off by more
 * than 2^-32 of the row's largest beside its rounding), out is rounded once at the end.
 *   prefix_len [B] int32, device, or NULL for P everywhere;  own_len [B*D] int32, device, or NULL for S;
 *   values outside [0, P] ([0, S]) are clamped.  What lies past a length is never used, whatever it holds, and
 *   a draft's outputs never depend on another draft's keys (with `causal`, values of own keys that a row of the
 *   same draft does not see must be finite: they are multiplied by 0).  P = 0 (S = 0): the pointers may be NULL.
 *   q, k_*, v_*, out 16-byte aligned, their strides multiples of 8 elements (PSD_ERR_ALIGN otherwise)
 *   lse [B*D*M, Hq] fp32 or NULL;  workspace 256-byte aligned, >= psd_attention_workspace_bytes
 *   status_dev NULL, or the status word (PSD_ERR_TIMEOUT: outputs invalid)
 */
int psd_draft_attention(const void* q, const void* k_prefix, const void* v_prefix, const int32_t* prefix_len,
                        const void* k_own, const void* v_own, const int32_t* own_len, const psd_attention_t* a,
                        void* out, float* lse, void* workspace, size_t workspace_bytes, int32_t* status_dev,
                        void* cuda_stream);

/* Bytes of scratch psd_prefix_weights needs (0 = bad sizes); grows with B, D, M and P and serves calls with smaller ones. */
size_t psd_weights_workspace_bytes(int32_t B, int32_t D, int32_t M, int32_t Hq, int32_t Hkv, int32_t Dh, int32_t P);

/*
 * psd_prefix_weights — the attention weight that every prefix key has drawn, summed over the rows that read it:
 *   acc_out[b,h,j] = beta * acc_in[b,h,j] + sum over t of sequence b and heads g of key head h of
 *                    exp(scale * q[t,g] . K_j - lse[t,g])          for j < prefix_len[b],  0 for j >= prefix_len[b].
 * lse [B*D*M, Hq] fp32 is psd_draft_attention's (a row with lse = -inf, which saw no keys, adds nothing).
 *   acc_in, acc_out [B, Hkv, P] fp32; acc_in NULL counts as 0 and may be acc_out itself.  P >= 1.
 * The sum's order is fixed: equal inputs give equal bits.  Other arguments as for psd_draft_attention.
 */
int psd_prefix_weights(const void* q, const void* k_prefix, const int32_t* prefix_len, const float* lse,
                       const psd_attention_t* a, float beta, const float* acc_in, float* acc_out, void* workspace,
                       size_t workspace_bytes, int32_t* status_dev, void* cuda_stream);

/* Shapes of psd_prefix_evict. */
typedef struct psd_evict_t {
    int32_t B, Hkv, Dh;       /* as above                                                                    */
    int32_t P;                /* capacity of the cache, 1 .. 2^30                                             */
    int32_t keep;             /* keys to keep per sequence and key head, 1 .. 2^30                             */
    int32_t n_sink, n_recent; /* always keep the first n_sink and the last n_recent; both >= 0, sum <= keep   */
    int32_t dtype;            /* PSD_BF16 or PSD_FP16 */
    psd_kv_strides_t k, v;    /* [B, P, Hkv, Dh] */
    psd_kv_strides_t k_out, v_out; /* [B, keep, Hkv, Dh], not overlapping k and v; no stride 0 */
} psd_evict_t;

/*
 * psd_prefix_evict — cuts the cache to `keep` keys per sequence and key head: the first n_sink, the last n_recent and,
 * of the others, those with the highest score (equal scores: lower position first; NaN below every number), packed
 * in order of position.
 *   scores [B, Hkv, P] fp32 (psd_prefix_weights' acc_out);  prefix_len as above
 *   index      [B, Hkv, keep] int32 out: kept positions ascending, then -1
 *   scores_out [B, Hkv, keep] fp32 out or NULL: their scores, then 0;  len_out [B] int32 out or NULL: min(prefix_len, keep)
 *   k_out, v_out: kept keys and values; slots past len_out are left untouched.
 */
int psd_prefix_evict(const float* scores, const void* k, const void* v, const int32_t* prefix_len, const psd_evict_t* e,
                     void* k_out, void* v_out, int32_t* index, float* scores_out, int32_t* len_out, void* cuda_stream);

/* Edits of psd_confidence_logits; pointers are device pointers, each may be NULL (that edit is then not made). */
typedef struct psd_logits_edit_t {
    const int32_t* history;      /* [B, history_cap] tokens of the text so far; ids outside [0, V) are ignored     */
    const int32_t* history_len;  /* [B], clamped to [0, history_cap]; NULL = history_cap                           */
    const int32_t* draft_tokens; /* [B*D, M] tokens of the drafts: where draft_mask is 0 they count as text of      */
    const int32_t* draft_mask;   /* [B*D, M] their own draft (both or neither)                                    */
    const float* bias;           /* [bias_rows, V] fp32                                                           */
    const uint32_t* allow;       /* [allow_rows, ceil(V/32)]: bit v%32 of word v/32 set = token v may be chosen     */
    int32_t history_cap;         /* 0 .. 2^30 */
    int32_t bias_rows;           /* divides B*D*M: row r uses bias row r / (B*D*M / bias_rows)                      */
    int32_t allow_rows;          /* likewise                                                                       */
    float repetition;            /* > 0, finite; 1 = none */
    float presence, frequency;   /* finite; 0 = none */
    int32_t reserved;            /* 0 */
} psd_logits_edit_t;

/* Bytes of scratch psd_confidence_logits needs (0 = bad sizes); grows with n_rows and V and serves calls with fewer. */
size_t psd_logits_workspace_bytes(int32_t n_rows, int32_t V);

/*
 * psd_confidence_logits — psd_confidence for bodies that hand out logits, with penalties for repeated tokens, biases
 * and grammar masks.  For row r = (b, d, i) and token v with c = how often v occurs in the text of (b, d), in fp32, each
 * operation rounded on its own:
 *   c > 0:  x = l > 0 ? l / repetition : l * repetition;  x = x - (frequency * c + presence);   else x = l
 *   x = x + bias;   tokens whose allow bit is 0 drop out, whatever their logit holds.
 * out_token, out_conf, out_lse are those of psd_confidence over x.  A row in which no token is left (or all that are left
 * have x = -inf) gives token -1, confidence 0 and lse -inf; it is not counted as non-finite, and psd_select_unmask,
 * psd_build_drafts and psd_verify_accept take its slot for one without a token: it stays masked.  A NaN or +inf among the tokens left gives confidence NaN and is counted in status_dev (the token is then
 * that of the largest value that is no NaN, -1 if there is none above -inf).
 *   logits [B*D*M, V] bf16, fp16 or fp32 (dtype), rows row_stride >= V elements apart, aligned to their element;
 *     B*D*M and V at most 2^30
 *   edit: HOST pointer, NULL = no edits;  workspace >= psd_logits_workspace_bytes(B*D*M, V), 256-byte aligned
 */
int psd_confidence_logits(const void* logits, int32_t dtype, int64_t row_stride, int32_t B, int32_t D, int32_t M, int32_t V,
                          const psd_logits_edit_t* edit, int32_t* out_token, float* out_conf, float* out_lse,
                          void* workspace, size_t workspace_bytes, int32_t* status_dev, void* cuda_stream);

/*
 * ---- A step in 8 bits: rotation, the prefix's cache and the LM head in codes -----------------------------
 *
 * CODES are int8 numbers from -127 to 127 that stand for code * scale.  One scale serves a row of a matrix, or the
 * tokens of a block of one key head in a cache.  Over a unit x of numbers, in fp32, each operation rounded on its own:
 *   scale = max(max |x| * fp32(1/127), 2^-126),   r = 1 / scale,   code = rint(x * r)      (ties to even).
 * A unit that holds a NaN or an infinity gets the scale NaN and codes 0.  Scales made elsewhere are finite and >= 0, or NaN.
 */

/* How psd_rope_frequencies scales a context of `original` tokens by `factor`. */
#define PSD_ROPE_PLAIN 0     /* f[j] = base^(-2j/rotary)                                                              */
#define PSD_ROPE_LINEAR 1    /* f[j] / factor                                                                         */
#define PSD_ROPE_STRETCHED 2 /* base * factor^(rotary / (rotary - 2)) in place of base (rotary > 2)                   */
#define PSD_ROPE_BY_PARTS 3  /* with n = original * f[j] / 2 pi turns over the original context and
                                w = clamp((n - low) / (high - low), 0, 1):  w * f[j] + (1 - w) * f[j] / factor
                                (the ramp is linear in the turns n, not in the index j, and comes with a gain above 1:
                                a model whose ramp or gain differ needs a table or a gain of its own)                 */

/*
 * psd_rope_frequencies — the table that psd_rotate_qk reads, computed on the host in 64 bits.
 *   rotary even, 2 .. 128;  base > 1;  factor >= 1;  BY_PARTS: original >= 1, 0 <= low < high (others do not read them)
 *   frequency [rotary/2] HOST out, radians per position;  gain HOST out or NULL: 1, BY_PARTS 0.1 ln(factor) + 1
 */
int psd_rope_frequencies(int32_t rotary, double base, int32_t kind, double factor, double original, double low, double high,
                         double* frequency, float* gain);

/* Shapes of psd_rotate_qk. */
typedef struct psd_rotate_t {
    int32_t n_tokens;     /* T >= 1                                                                          */
    int32_t Hq, Hkv, Dh;  /* heads, 0 .. 16384, not both 0 (0: q, or k and v, are not read); 8 <= Dh <= 128, Dh % 8 == 0 */
    int32_t dtype;        /* PSD_BF16 or PSD_FP16: q, k, v, weights and outputs                               */
    int32_t rotary;       /* the first `rotary` numbers of a head are rotated: even, 0 .. Dh                  */
    int32_t interleaved;  /* pairs: 0 (j, j + rotary/2), 1 (2j, 2j + 1)                                       */
    int32_t n_slots;      /* with slots: rows of k_out and v_out                                              */
    float eps;            /* > 0, finite */
    float gain;           /* > 0, finite: factor of sines and cosines */
    int64_t q_token, q_head, k_token, k_head, v_token, v_head;                         /* element strides, > 0 */
    int64_t q_out_token, q_out_head, k_out_token, k_out_head, v_out_token, v_out_head;
} psd_rotate_t;

/*
 * psd_rotate_qk — norms of queries and keys for each head, their position rotation, and the filing of keys and values in a
 * cache, in one pass.  For token t and a head x of q (of k):
 *   y = x * w / sqrt(mean(x^2) + eps) with w = q_norm (k_norm), or y = x where that is NULL;
 *   (z_a, z_b) = gain * (y_a cos u - y_b sin u, y_b cos u + y_a sin u),  u = position[t] * frequency[j],
 * for the pairs (a, b) of the first `rotary` numbers; the others are y.  fp32 (the angles 64 bits), rounded once.
 *   q [T, Hq, Dh] -> q_out;  k [T, Hkv, Dh] -> k_out[at];  v [T, Hkv, Dh] (NULL: none) -> v_out[at] unchanged
 *   at = t, or slot[t] ([T] int32, device): tokens whose slot lies outside [0, n_slots) are not filed.  No slot is named
 *   twice in a call.  Rows of k_out and v_out that no token names are left as they are.
 *   position [T] int32 (any value), frequency [rotary/2] fp64, device; rotary = 0: both may be NULL
 *   q_norm, k_norm [Dh] or NULL.  Outputs are the inputs themselves (same strides, no slots) or do not overlap them.
 *   pointers 16-byte aligned (position, slot 4, frequency 8), strides multiples of 8 elements (PSD_ERR_ALIGN)
 */
int psd_rotate_qk(const void* q, const void* k, const void* v, const int32_t* position, const double* frequency,
                  const void* q_norm, const void* k_norm, const int32_t* slot, const psd_rotate_t* r, void* q_out, void* k_out,
                  void* v_out, void* cuda_stream);

/*
 * psd_quantize_rows — codes [n_rows, H] and scale [n_rows] of the rows of x [n_rows, H] (bf16 or fp16), one scale a row:
 * an LM head for psd_confidence_q8, for instance.
 *   H >= 8, H % 8 == 0;  row_stride >= H elements, code_stride >= H, both multiples of 8;  x 16-byte, codes 8-byte aligned
 */
int psd_quantize_rows(const void* x, int32_t dtype, int64_t row_stride, int64_t n_rows, int32_t H, int8_t* codes,
                      int64_t code_stride, float* scale, void* cuda_stream);

/* Shapes of psd_prefix_quantize. */
typedef struct psd_quantize_t {
    int32_t B, Hkv, Dh;               /* 8 <= Dh <= 128, Dh % 8 == 0                                              */
    int32_t P;                        /* capacity of the caches, 1 .. 2^30                                        */
    int32_t block;                    /* tokens per scale: 16, 32, 64 or 128                                      */
    int32_t dtype;                    /* PSD_BF16 or PSD_FP16: k, v                                               */
    int32_t span;                     /* end - begin at most (the host's bound, for the launch); 0 = P             */
    int32_t reserved;                 /* 0 */
    psd_kv_strides_t k, v;            /* [B, P, Hkv, Dh], elements                                                */
    psd_kv_strides_t k_codes, v_codes; /* [B, P, Hkv, Dh], bytes; no stride 0 where the dimension is more than one */
} psd_quantize_t;

/*
 * psd_prefix_quantize — tokens begin[b] .. end[b] - 1 of a prefix's keys and values enter its 8-bit cache.
 * One scale serves block j (tokens j * block .. (j + 1) * block - 1) of a key head, over the tokens of the block below
 * end[b]; a range that begins inside a block codes that block again from its first token, which k and v must still hold.
 *   begin, end [B] int32, device, clamped to [0, P]; NULL: 0, P.  end is cut to begin + span.  begin >= end: nothing.
 *   k_scale, v_scale [B, Hkv, ceil(P / block)] fp32.  Blocks without tokens of the range, and codes from end[b] on,
 *   are left as they are; what k and v hold there is not read.
 *   k, v 16-byte aligned, strides multiples of 8; codes 8-byte aligned, strides multiples of 8
 */
int psd_prefix_quantize(const void* k, const void* v, const int32_t* begin, const int32_t* end, const psd_quantize_t* q,
                        int8_t* k_codes, int8_t* v_codes, float* k_scale, float* v_scale, void* cuda_stream);

/* Bytes of scratch psd_draft_attention_q8 needs (0 = bad sizes); grows with B, D, P and S and serves calls with smaller ones. */
size_t psd_attention_q8_workspace_bytes(int32_t B, int32_t D, int32_t M, int32_t Hq, int32_t Hkv, int32_t Dh, int32_t P, int32_t S);

/* Names of the kernels that psd_draft_attention_q8 launches at these sizes, as psd_attention_kernel_names tells them: "prefix_rows_q8_kernel"
 * (few rows per key head) or "prefix_tiles_q8_kernel", and "+draft_attention_kernel" where partial results are joined; "draft_attention_kernel"
 * alone: a short prefix, or none. */
const char* psd_attention_q8_kernel_names(int32_t B, int32_t D, int32_t M, int32_t Hq, int32_t Hkv, int32_t Dh, int32_t P,
                                          int32_t S, int32_t* splits);

/*
 * psd_draft_attention_q8 — psd_draft_attention with a prefix in codes: key j of the prefix is k_codes[b, j, h] *
 * k_scale[b, h, j / block], and so are the values; the drafts' own keys and values are 16-bit as there.
 *   block 16, 32, 64 or 128;  Dh % 16 == 0;  a->kp, a->vp are in bytes, multiples of 16;  codes 16-byte aligned
 *   k_scale, v_scale [B, Hkv, ceil(P / block)] fp32; neither codes nor scales past a length are used.  A scale NaN makes
 *   the outputs that draw on its block NaN.  Scores, statistics and sums are fp32, the codes enter exactly.  Weights over the
 *   prefix are rounded to fp16 after they are multiplied by their value's scale: none is off by more than 2^-32 of the row's
 *   largest such product beside that, however far the scales of a sequence and head lie apart (up to 2^110, and for weights
 *   above 2^-110 of the row's largest; smaller ones may add nothing to out).  Weights over own keys are rounded to the inputs'
 *   type, as there.
 *   Other arguments as for psd_draft_attention.
 */
int psd_draft_attention_q8(const void* q, const int8_t* k_codes, const int8_t* v_codes, const float* k_scale,
                           const float* v_scale, int32_t block, const int32_t* prefix_len, const void* k_own,
                           const void* v_own, const int32_t* own_len, const psd_attention_t* a, void* out, float* lse,
                           void* workspace, size_t workspace_bytes, int32_t* status_dev, void* cuda_stream);

/* Bytes of scratch psd_confidence_q8 needs (0 = bad sizes); grows with n_rows, H and V. */
size_t psd_confidence_q8_workspace_bytes(int32_t n_rows, int32_t H, int32_t V);

/*
 * psd_confidence_q8 — psd_confidence over an LM head in codes.  The hidden rows [n_rows, H] (bf16 or fp16) are coded as
 * psd_quantize_rows does; with n = sum_j x_code[r,j] * w_code[v,j] (exact),
 *   l[r,v] = fp32(fp32(fp32(n) * w_scale[v]) * x_scale[r]),
 * and token, confidence and lse are those of psd_confidence over l (the lowest v among equal l).
 *   H % 64 == 0, H <= 131072;  hidden, w_codes [V, H] 16-byte aligned;  w_scale [V] fp32
 *   workspace 256-byte aligned;  status_dev as for psd_confidence: counts the rows without a finite confidence
 */
int psd_confidence_q8(const void* hidden, int32_t dtype, const int8_t* w_codes, const float* w_scale, int32_t n_rows, int32_t H,
                      int32_t V, int32_t* out_token, float* out_conf, float* out_lse, void* workspace, size_t workspace_bytes,
                      int32_t* status_dev, void* cuda_stream);

/*
 * Which kernel psd_confidence uses.  Process-wide; returns the previous value, or PSD_ERR_SHAPE for
 * an unknown value.
 *   0  (default) the tcgen05/TMA kernels, chosen by size: pairs of CTAs on one tile of 256 rows
 *      (cta_group::2) for 129..256 rows, one CTA per tile of 128 rows otherwise
 *   1  a plain CUDA-core kernel kept for cross-checking
 *   2  always the single-CTA tcgen05 kernel;  3  always the CTA-pair tcgen05 kernel (same results up
 *      to summation order)
 */
int psd_set_confidence_impl(int impl);

/*
 * Performance knobs (process-wide; results never depend on them).  Returns PSD_OK,
 * PSD_ERR_UNSUPPORTED for an unknown knob or PSD_ERR_SHAPE for a bad value.
 *   PSD_TUNE_BAND_BYTES  bytes of the operand that one band of the fused kernel's tile order keeps
 *                        in L2 while the other operand streams past it (default 36 MiB)
 */
#define PSD_TUNE_BAND_BYTES 1
/*   PSD_TUNE_PDL         1 (default): consecutive kernels of a step are launched with programmatic stream
 *                        serialization, so a kernel's set-up overlaps the end of the one before it (the
 *                        fused kernel itself starts early only when the batch is a single row tile);
 *                        2: the fused kernel starts early at every size; 0: plain stream order */
#define PSD_TUNE_PDL 2
/*   PSD_TUNE_TILE_ORDER  0 (default): the library picks the tile order with the smaller estimated DRAM
 *                        traffic; 1: bands of vocabulary tiles (W resident, hidden re-read per band);
 *                        2: bands of row tiles (hidden resident, W re-read per band) */
#define PSD_TUNE_TILE_ORDER 3
/*   PSD_TUNE_COMPACT_ROWS  psd_step scores only the rows of slots that are still masked in their draft
 *                        (Sec. 3.2 Stage 3: "each masked position"): 0 (default) off; 1 on when the
 *                        batch has more than 128 rows; 2 always.  With it on, the workspace must hold
 *                        psd_compact_workspace_bytes, and entries of tokV / confV that belong to
 *                        committed slots are left as they were (no stage reads them) */
#define PSD_TUNE_COMPACT_ROWS 4
/*   PSD_TUNE_WAIT_LIMIT  every wait on a barrier inside the tensor-core kernels gives up after this many
 *                        THOUSANDS of SM clock cycles (default 4 000 000: about 2 s); the kernel then reports
 *                        PSD_ERR_TIMEOUT through status_dev, lets its own copies and tensor-core work finish
 *                        (those waits keep the default limit), frees what it holds and returns normally */
#define PSD_TUNE_WAIT_LIMIT 5
/*   PSD_TUNE_SELFTEST_STALL  1: self-test of that give-up path.  In every CTA (in the leading CTA of every
 *                        pair) the loader, after its first K-slice, waits on a barrier that nothing ever
 *                        arrives on, so the wait runs out after PSD_TUNE_WAIT_LIMIT and the call ends with
 *                        PSD_ERR_TIMEOUT in status_dev and invalid outputs; nothing faults and the next call
 *                        (with 0 here) works as usual.  0 (default): off */
#define PSD_TUNE_SELFTEST_STALL 6
/* 1 if PSD_TUNE_COMPACT_ROWS makes a batch of n_rows rows take the compacted path, else 0. */
int psd_compact_rows_enabled(int32_t n_rows);
int psd_set_tuning(int knob, int value);

/*
 * Profiling aid.  When both events (cudaEvent_t passed as void*) are non-NULL, the next
 * psd_confidence call made by this host thread (directly or through psd_step / psd_step_host)
 * records `start_event` immediately before and `stop_event` immediately after its main kernel
 * (the fused LM-head + confidence kernel, not the combine pass) on the call's stream; the hook then
 * clears itself.  Passing NULLs clears it.  Always returns PSD_OK.
 */
int psd_set_kernel_events(void* start_event, void* stop_event);

/*
 * Name of the kernel that psd_confidence (and psd_step) launches for a batch of n_rows rows under the
 * current psd_set_confidence_impl setting: "confidence_tc_kernel", "confidence_tc2_kernel" or
 * "confidence_simt_kernel" (static storage).  For reports: it computes nothing.
 */
const char* psd_confidence_kernel_name(int32_t n_rows);

/* Number of kernel launches the library has issued in this process (all entry points). */
int64_t psd_launch_count(void);

#ifdef __cplusplus
}
#endif
#endif /* PSD_H_ */
