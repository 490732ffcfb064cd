/*
 * dbt.h -- C ABI of the grouped decode step of the Decode-Branch Transformer on B200.
 *
 * What the library computes (paper Section 4).  Two residual trajectories share every
 * large matrix: the primary path S_1 is a standard causal Transformer and is the only
 * writer of the persistent KV cache; the decode branch S_2 starts from its own token
 * embedding (Eq. embeddings), forms only a query (Eq. asymattn: Q~_2 = Q_2 + a*Q_1, read
 * against the primary K_1,V_1), is coupled in the MLP by b and c (Eq. mlp) and writes no
 * persistent state.  Logits of both paths go through one output matrix and are mixed with
 * alpha = clip_[0.5,1](sum_v p_v^2) (Eq. alpha, Eq. mixloss).  Inference follows Section
 * 4.4: a primary-only prefill over the prompt, then grouped steps -- both paths' rows
 * stacked through the shared matrices and one read of the primary cache serving both
 * queries ("Decode" paragraph; Section 4.5, Eq. decode_traffic).
 *
 * Conventions.
 *  - Every pointer is marked HOST or DEVICE.  All device memory (weights, KV pool,
 *    workspace, token / logit buffers) belongs to the caller; the library borrows it,
 *    never frees it and never writes the weights.  It must outlive the handle.
 *  - Matrices are row-major [out_features, in_features] (the paper's H W with W stored
 *    transposed), in `weight_dtype`.  Norm gains and the coupling vectors a, b, c are fp32.
 *  - Stacked activations are path-major: rows 0..B-1 primary, then B rows per decode branch.
 *  - KV pool layout: [n_layers][2 (K,V)][num_pages][n_kv_heads][page_size][head_dim] in
 *    `weight_dtype`; K is stored after RoPE.  Logical position t of sequence b lives in
 *    physical page page_table[b][t / page_size], slot t % page_size.
 *  - Calls enqueue work on the CUDA stream given at creation and return without waiting
 *    (the *_host variants wait).  Errors the host can see (bad arguments, capacity) are
 *    returned at once and enqueue nothing.  Errors only the device can see (a token id out
 *    of range) are recorded in a status word read by dbt_sync_status; the offending value is
 *    clamped so that no access leaves its buffer.  Nothing traps or aborts.
 *  - Not thread-safe per handle.
 */
#ifndef DBT_H
#define DBT_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct dbt_model dbt_model; /* opaque; owned by the library */

typedef enum {
    DBT_OK = 0,
    DBT_ERR_INVALID_ARG = 1,
    DBT_ERR_UNSUPPORTED = 2, /* shape / option outside what the kernels cover        */
    DBT_ERR_CAPACITY = 3,    /* max_batch, max_seq or the page pool would be exceeded */
    DBT_ERR_STATE = 4,
    DBT_ERR_CUDA = 5,
    DBT_ERR_DEVICE = 6,      /* the device status word is non-zero (dbt_sync_status)  */
    DBT_ERR_TIMEOUT = 7      /* a bounded wait inside a kernel ran out (dbt_sync_status) */
} dbt_status;

enum { DBT_DTYPE_F32 = 0, DBT_DTYPE_BF16 = 1 };
enum { DBT_ROUTER_INDEPENDENT = 0, DBT_ROUTER_REPLAY = 1 };

typedef struct {
    uint32_t struct_size; /* sizeof(dbt_config), for versioning */
    int32_t d_model, n_layers, n_q_heads, n_kv_heads, head_dim, d_ff, vocab;
    int32_t weight_dtype; /* DBT_DTYPE_*; the KV cache uses the same storage type */
    float rope_base;      /* RoPE base; half-split pairs (i, i+head_dim/2), 0-based positions,
                             the same position for both paths */
    float rms_eps;
    int32_t final_norm;       /* 1: RMSNorm before the shared output matrix */
    int32_t n_experts;        /* 0 = dense MLP (Eq. mlp); >0 = MoE (Eq. moe_layer) */
    int32_t d_expert;         /* hidden width of one routed expert */
    int32_t n_shared_experts; /* applied to every token of both paths, un-gated */
    int32_t k_primary;        /* k_1 of Eq. moe_budget */
    int32_t k_branch;         /* k_2 of Eq. moe_budget */
    int32_t router_mode;      /* DBT_ROUTER_* (replay: Section 4.3) */
    int32_t moe_b_coupling;   /* 1: b couples the shared expert's hidden state; 0: b unused in MoE */
    int32_t compute_matched;  /* 1: compute-matched MoE allocation (Appendix B.3): the branch evaluates no
                                 attention and no shared expert; A_2 = g_A*A_1 (Eq. matched_attention),
                                 M_2 = R_2(N_2;k_2) + g_G*G(N_1) (Eq. matched_shared_expert); a, b, c are
                                 not applied.  MoE models only (DBT_ERR_UNSUPPORTED otherwise). */
    int32_t n_paths;          /* K of Appendix C.1 ("More decode branches"): residual paths in all, the primary plus
                                 K-1 decode branches.  Each branch has its own embedding table and same-position
                                 state, reads the primary cache, shares a, b, c (and g_A, g_G) with the other
                                 branches, routes for itself in MoE layers; the readout mixes p with the mean of
                                 the branch distributions.  2 (or 0) is the main text's model; at most 8, and
                                 n_paths * n_q_heads / n_kv_heads <= 16 (DBT_ERR_UNSUPPORTED otherwise). */
    int32_t max_batch, max_seq;
    int32_t page_size; /* tokens per KV page; 16 */
    int32_t num_pages; /* pages in the pool, per layer and per K/V */
} dbt_config;

/* DEVICE pointers.  Unused entries (MoE fields of a dense model and vice versa) may be NULL. */
typedef struct {
    const float *attn_norm_g;                  /* [d]                                         */
    const void *wq, *wk, *wv, *wo;             /* [q_dim,d] [kv_dim,d] [kv_dim,d] [d,q_dim]   */
    const float *coup_a;                       /* [q_dim]                                     */
    const float *mlp_norm_g;                   /* [d]                                         */
    const void *w_gate, *w_up, *w_down;        /* dense: [F,d] [F,d] [d,F]                    */
    const float *coup_b;                       /* dense [F]; MoE [n_shared*d_expert]          */
    const float *coup_c;                       /* [d]                                         */
    const void *router;                        /* [E,d]                                       */
    const void *exp_gate, *exp_up, *exp_down;  /* [E,Fe,d] [E,Fe,d] [E,d,Fe]                  */
    const void *sh_gate, *sh_up, *sh_down;     /* [Fs,d] [Fs,d] [d,Fs], Fs = n_shared*Fe      */
    const float *gate_a, *gate_g;              /* [d] [d]  g_A, g_G (compute_matched only)    */
} dbt_layer_weights;

typedef struct {
    const void *embed_primary, *embed_branch;  /* DEVICE E_1 [V,d]; E_2..E_K one after another
                                                  [n_paths-1][V,d]                            */
    const float *embed_norm_g, *final_norm_g;  /* DEVICE [d]                                  */
    const void *lm_head;                       /* DEVICE shared output matrix [V,d]           */
    const dbt_layer_weights *layers;           /* HOST array [n_layers] of DEVICE pointers    */
} dbt_weights;

/* Bytes the caller must provide for the KV pool and the workspace (both DEVICE, 256-byte
 * aligned).  cfg HOST. */
dbt_status dbt_query_sizes(const dbt_config *cfg, size_t *kv_bytes, size_t *workspace_bytes);

/* Build a handle (Section 4: the model of both paths).  cfg, w HOST; kv_pool_dev,
 * workspace_dev DEVICE; cuda_stream a cudaStream_t (NULL = default stream).  Validates the
 * configuration (DBT_ERR_UNSUPPORTED for head_dim not in {64,128}, page_size != 16,
 * n_q_heads not a multiple of n_kv_heads, more than 16 queries per KV head over both
 * paths, k > n_experts, ...), builds the RoPE table and the default page table
 * (sequence b owns pages b*ceil(max_seq/page_size) ...), and zeroes all sequence lengths.
 * On failure *out is NULL. */
dbt_status dbt_create(const dbt_config *cfg, const dbt_weights *w, void *kv_pool_dev,
                      void *workspace_dev, void *cuda_stream, dbt_model **out);
void dbt_destroy(dbt_model *m);

/* HOST table [B][pages_per_seq] of physical page ids (distinct, < num_pages) for sequences
 * 0..B-1; pages_per_seq <= ceil(max_seq/page_size) bounds each sequence's capacity. */
dbt_status dbt_set_page_table(dbt_model *m, const int32_t *table_host, int32_t B, int32_t pages_per_seq);

/* Sequence lengths := 0 (the cache contents are left as they are). */
dbt_status dbt_reset(dbt_model *m);
/* Declare that sequences 0..B-1 already hold lens_host[b] cached positions (the caller
 * wrote the pool itself, e.g. a synthetic fill for timing).  lens_host HOST. */
dbt_status dbt_set_seq_lens(dbt_model *m, const int32_t *lens_host, int32_t B);
/* Current length of sequence b as the host tracks it (-1 on a bad argument). */
int32_t dbt_seq_len(const dbt_model *m, int32_t b);

/* Section 4.4 item 1, prompt-wide prefill: the primary path alone processes n positions of
 * sequences 0..B-1 (tokens_dev DEVICE int32 [B][n]) starting at their current lengths,
 * writes their K/V and advances the lengths.  No branch computation.
 * last_primary_logits_dev: DEVICE fp32 [B][V] for the last position, or NULL. */
dbt_status dbt_prefill(dbt_model *m, const int32_t *tokens_dev, int32_t B, int32_t n,
                       float *last_primary_logits_dev);

/* Section 4.4 items 1 and 2 in one call: the primary path alone processes the whole prompt x_1..x_S
 * (tokens_dev DEVICE int32 [B][S], sequences 0..B-1 from their current lengths), and the continuation boundary
 * -- one branch evaluation at the final prompt token, coupled to the primary's Q_1, H_1, M_1 of that position
 * and read against the completed cache -- predicts x_{S+1} from the mixture.  Outputs as dbt_decode_step.
 * How it runs: positions 1..S-1 as the prompt-wide prefill, position S as one grouped step, whose rows go
 * through the GEMMs of the last prompt chunk where they fit its row tiles (dense bf16 models).  The boundary
 * evaluation has to stream every shared matrix once for the branch row anyway; letting the primary row of
 * position S ride in that same pass produces the "retained intermediates" where they are consumed, costs no
 * extra memory traffic and needs no per-layer retention buffers.  The values are those of the paper's form
 * (prefill all S positions, then a branch-only evaluation).  Lengths advance by S. */
dbt_status dbt_prefill_boundary(dbt_model *m, const int32_t *tokens_dev, int32_t B, int32_t S, int32_t *next_tokens_dev,
                                float *logits_primary_dev, float *logits_branch_dev, float *alpha_dev);

/* Section 4.4 items 2-3, one grouped step ("Decode" paragraph): for each sequence b the token
 * tokens_dev[b] at position t_b = its length; the primary appends K_1,V_1[t_b]; both paths'
 * queries read positions 0..t_b of the primary cache; the shared matrices are applied to
 * the stacked rows; next_tokens_dev[b] = argmax of alpha*p + (1-alpha)*q (lowest index on
 * ties; with more than one decode branch q is the mean of the branch distributions, Appendix C.1).
 * Lengths advance by one.  All pointers DEVICE; outputs may be NULL: next_tokens_dev int32 [B] (may alias
 * tokens_dev), logits_primary_dev fp32 [B][V], logits_branch_dev fp32 [n_paths-1][B][V], alpha_dev fp32 [B].
 * To start from a prompt x_1..x_S: prefill x_1..x_{S-1}, then pass x_S to the first step
 * (the boundary step of Section 4.4 item 2). */
dbt_status dbt_decode_step(dbt_model *m, const int32_t *tokens_dev, int32_t B, int32_t *next_tokens_dev,
                           float *logits_primary_dev, float *logits_branch_dev, float *alpha_dev);

/* The comparison path: the same step with the branch rows absent (a standard decode step,
 * Background "decode").  Writes the same K/V bits as dbt_decode_step for the same inputs;
 * next token = argmax of the primary logits. */
dbt_status dbt_decode_step_primary_only(dbt_model *m, const int32_t *tokens_dev, int32_t B,
                                        int32_t *next_tokens_dev, float *logits_primary_dev);

/* Tokens drawn from the last step's output distribution instead of its argmax: for the sequences 0..B-1 of the last
 * dbt_decode_step, dbt_decode_step_primary_only or dbt_prefill_boundary of this handle (their *_host forms too), by the rules
 * of dbt_op_sample below with z = log(alpha p + (1 - alpha) q), the mixture of Eq. mixloss and Appendix C.1 (primary-only
 * steps: the primary logits), so that the temperature acts on the mixture.  s HOST, its entries DEVICE [B], all but uniforms may
 * be NULL.  next_tokens_dev int32 [B], logprobs_dev fp32 [B] or NULL.  May be called again for other numbers.
 * DBT_ERR_STATE: no step yet, or a dbt_prefill or dbt_reset since.  DBT_ERR_INVALID_ARG: B is not the last step's. */
typedef struct {
    uint32_t struct_size; /* sizeof(dbt_sampling) */
    int32_t reserved;     /* 0 */
    const float *uniforms, *temperature;
    const int32_t *top_k;
    const float *top_p, *min_p;
} dbt_sampling;
dbt_status dbt_sample_last(dbt_model *m, const dbt_sampling *s, int32_t B, int32_t *next_tokens_dev, float *logprobs_dev);

/* End-to-end variants with HOST buffers: copy tokens_host [B] to the device, run the step,
 * copy next_tokens_host [B] (and alpha_host [B] when non-NULL) back, wait for the stream.
 * Buffers should be pinned for the copies to be asynchronous. */
dbt_status dbt_decode_step_host(dbt_model *m, const int32_t *tokens_host, int32_t B,
                                int32_t *next_tokens_host, float *alpha_host);
dbt_status dbt_decode_step_primary_only_host(dbt_model *m, const int32_t *tokens_host, int32_t B,
                                             int32_t *next_tokens_host);

/* MoE only: DEVICE int32 [n_layers][n_paths][max_batch][kmax] (kmax = max(k_primary,k_branch)),
 * the expert ids each row used in the last decode step (-1 padded); and the number of
 * distinct experts loaded per layer in the last step, HOST int32 [n_layers] (waits for the
 * stream).  Equation moe_layer leaves near-ties in the router to rounding, so tests read the
 * choice back instead of assuming it. */
dbt_status dbt_last_experts(dbt_model *m, const int32_t **experts_dev, int32_t *kmax);
dbt_status dbt_last_expert_union(dbt_model *m, int32_t *count_per_layer_host);

/* Wait for the stream and read the device status word.  *device_status: 0 = clean; 1 = a token
 * id was out of range, 2 = a page id was out of range (*detail = the offending value; the value was
 * clamped and the step ran on): returns DBT_ERR_DEVICE; 3 = a bounded wait inside a kernel (on a
 * shared-memory barrier that a TMA copy or a tensor-core commit completes) ran out after about two
 * seconds: *detail = the wait site (100 + warp: operand ring of the GEMM, 200 + warp: its accumulator,
 * 300..: the decode attention kernel's page ring, 400..: the prompt attention kernel's, 500..: the
 * persistent per-expert GEMM's rings and accumulators, 600..: the paired-SM GEMMs, 700..: the experts' paired-SM GEMMs,
 * 800..: the cluster kernel of small fp32 steps), the CTA skipped its stores, released its tensor memory and
 * returned, so the step's results are invalid but the context stays usable: returns DBT_ERR_TIMEOUT.
 * The first code recorded wins until dbt_reset clears the word.  HOST pointers, may be NULL. */
dbt_status dbt_sync_status(dbt_model *m, int32_t *device_status, int32_t *detail);

/* The persistent state of the method is the primary path's KV cache alone (Background, "KV cache";
 * Section 4.4 "Decode": the branch writes no persistent entries).  These two calls move it between the
 * paged pool and HOST buffers in logical order [n_layers][B][T][kv_dim] (elements of `weight_dtype`, K after
 * RoPE), for sequences seq_ids_host[0..B-1] (HOST; NULL = sequences 0..B-1) and positions 0..T-1, through the
 * page table; they wait for the stream.  Export needs T <= the current length of each sequence
 * (DBT_ERR_STATE otherwise).  Import overwrites those positions and sets the length of each listed
 * sequence to T (the other sequences keep theirs).  T beyond a sequence's capacity: DBT_ERR_CAPACITY.
 * Uses: handing a prefilled cache to another process or a checker, restoring a session, tests. */
dbt_status dbt_kv_export(dbt_model *m, const int32_t *seq_ids_host, int32_t B, int32_t T, void *k_host, void *v_host);
dbt_status dbt_kv_import(dbt_model *m, const int32_t *seq_ids_host, int32_t B, int32_t T, const void *k_host,
                         const void *v_host);

/* Operator-level entry: the grouped skinny GEMM alone (Section 4.4 "Decode": the stacked rows
 * of both paths go through one shared matrix, each weight tile fetched once).
 * Y[r][f] = sum_k W[f][k] X[r][k] with W_dev DEVICE bf16 [n_out][K], X_dev DEVICE bf16 [R][K]
 * (1 <= R <= 256, K a multiple of 8, both 16-byte aligned), Y_dev DEVICE fp32 [R][n_out].
 * scratch_dev: DEVICE fp32 workspace of scratch_floats elements for the split-K partials
 * (at least splits * roundup(R) * n_out with roundup to 16/32/64/128/256); status_dev DEVICE
 * int32[2] (zeroed by the caller; afterwards {3, wait site} when a bounded device wait ran out -- the
 * codes of dbt_sync_status -- else still zero).
 * force_split > 0 asks for that split-K factor (lowered to ceil(K/64) and to a factor whose ranges
 * are all non-empty), 0 lets the library choose; *split_used (HOST, nullable) receives the factor
 * used.  Runs on the tensor cores (TMA + tcgen05); enqueues on cuda_stream. */
dbt_status dbt_op_gemm_tc(const void *W_dev, const void *X_dev, int32_t n_out, int32_t K, int32_t R,
                          int32_t force_split, float *Y_dev, float *scratch_dev, size_t scratch_floats,
                          int32_t *status_dev, void *cuda_stream, int32_t *split_used);

/* The same GEMM for callers that cannot allocate device memory.  (The paper has no
 * counterpart: this entry exists for the integration, not for the method.)  Some hosts of this
 * library run where cudaMalloc is off limits -- inside a region that is being captured into a
 * CUDA graph, in a process whose memory pool is owned and fully handed out by another runtime,
 * or under a policy that forbids allocation after start-up -- and so cannot provide the split-K
 * workspace that dbt_op_gemm_tc asks for.  Here that workspace is a fixed array inside the
 * library's device image: 2^21 floats (8 MiB), resident on every GPU that has loaded the
 * library until the process exits.  The call allocates nothing and frees nothing.
 *   - Arguments as dbt_op_gemm_tc without the scratch pair; inputs, Y_dev and status_dev are
 *     still the caller's.  Results are identical to dbt_op_gemm_tc for the same split factor.
 *   - Limit: roundup(R) * n_out * splits <= 2^21 (roundup to 16/32/64/128/256).  The library
 *     lowers its own split choice to fit; a request that cannot fit even unsplit, or a
 *     force_split that does not fit, returns DBT_ERR_CAPACITY with a message and enqueues
 *     nothing.
 *   - The first call on each device looks up the array's device address (no allocation, but a
 *     runtime query): make that first call outside any stream capture, with the target device
 *     current.
 *   - All calls on a device share the one array and leave their partial sums in it.  Nothing in
 *     it needs to start at zero -- every element that is read has been written by the same
 *     call -- but two calls whose kernels overlap on the GPU (different streams, or a second
 *     process thread) race on it: serialise them. */
dbt_status dbt_op_gemm_tc_static(const void *W_dev, const void *X_dev, int32_t n_out, int32_t K, int32_t R,
                                 int32_t force_split, float *Y_dev, int32_t *status_dev, void *cuda_stream,
                                 int32_t *split_used);

/* ---- Operators for sampled and drafted tokens -------------------------------------------------------------------
 * The paper's decode step takes one token per sequence and picks the likeliest (reading of Section 4.4).  The entries
 * below serve programs that draw tokens, and programs that verify several drafted tokens per sequence in one pass over
 * the weights: rotary positions (plain, or with the keys and values written into the cache's pages), attention of a tree
 * of drafted tokens over the paged cache, sampling, and the acceptance of one branch of the tree.
 *
 * Common rules.
 *  - All pointers are DEVICE unless marked; the device that they are on must be the current one; work is enqueued on
 *    cuda_stream (a stream of that device) and nothing waits.  No call allocates memory, keeps state or uses memory that
 *    another call uses too, beyond the caller's own buffers: calls on different streams may overlap as long as their
 *    output, workspace and status buffers differ.  All calls may be captured into CUDA graphs.
 *  - dtype is DBT_DTYPE_*: the type of activations and of the cache.  head strides and the like count elements.
 *  - A cache layer is [2 (K,V)][num_pages][n_kv_heads][16][head_dim] -- one layer of the handle's pool --, 16-byte aligned,
 *    head_dim 64 or 128; page_table int32 [B][pages_per_seq] with position t of sequence b in page table[b][t / 16],
 *    slot t % 16.  Unlike a handle's own table it lives on the device.
 *  - seq_lens int32 [B]: cached positions of each sequence, before its drafted nodes.  The nodes 0..n-1 of sequence b have
 *    their keys and values at positions seq_lens[b] .. seq_lens[b] + n - 1.  node_counts int32 [B], or NULL: n_b nodes of
 *    sequence b count (0..max_nodes; other values are clamped); NULL: all max_nodes.  What belongs to nodes behind n_b is
 *    neither read nor written.  max_nodes is at most 64.
 *  - parents int32 [B][max_nodes]: the parent of each node, less than the node's own number, or -1 (a root).
 *  - status_dev int32 [2], zeroed by the caller: errors that only the device sees, {code, detail} as dbt_sync_status
 *    reports them (2 = a page id out of range, or a position behind the table's last page, detail -1; 3 = a bounded wait
 *    ran out, detail = its site, 900 and up; 4 = a parent that is not below its node, detail = the parent).  The first
 *    one stays.  Accesses stay inside the buffers: a bad page id is read as page 0 and not written, a bad parent counts as -1.
 *  - A message for a refused call is in dbt_last_error(NULL) of the calling thread. */

/* Frequencies (angle per position) of the rot_dim / 2 rotated pairs, HOST double [rot_dim / 2], and the factor on rotated
 * queries and keys, HOST (1 where the kind has none).  base_i = base^(-2 i / rot_dim). */
enum {
    DBT_ROPE_PLAIN = 0,  /* base_i */
    DBT_ROPE_LINEAR = 1, /* base_i / factor: positions squeezed into the trained range */
    DBT_ROPE_BASE = 2,   /* base * factor^(rot_dim / (rot_dim - 2)) for base: the slowest pair slows by factor, the fastest keeps */
    DBT_ROPE_RAMP = 3,   /* pairs of at most `low` turns over trained_len slow by factor, of at least `high` turns keep, a linear ramp
                            over the pairs between, which begins at pair 0 at the earliest and ends at pair rot_dim - 1 at the latest
                            (behind the last pair where that one makes more than `low` turns); the factor on queries and keys is 0.1 ln(factor) + 1 */
    DBT_ROPE_BANDS = 4   /* by the turns over trained_len: up to `low` slow by factor, from `high` on keep, between them a blend
                            linear in the turns */
};
typedef struct {
    uint32_t struct_size; /* sizeof(dbt_rope_spec) */
    int32_t kind;         /* DBT_ROPE_* */
    int32_t rot_dim;      /* rotated elements of a head: even, >= 2 */
    int32_t reserved;     /* 0 */
    double base;          /* > 1 */
    double factor;        /* >= 1 (all kinds but PLAIN) */
    double trained_len;   /* > 0 (RAMP, BANDS) */
    double low, high;     /* 0 < low < high (RAMP, BANDS) */
} dbt_rope_spec;
dbt_status dbt_rope_frequencies(const dbt_rope_spec *spec_host, double *freq_host, float *scale_host);

/* Rotary positions: y = scale * R(position) x on the first rot_dim elements of every head, the others copied.
 * x, y [rows][heads][head_dim], head_dim contiguous, with strides between rows and heads; y may be x with the same
 * strides, else the two do not overlap.  positions int32 [rows]; freq double [rot_dim / 2] (dbt_rope_frequencies, on the
 * device); angles are formed and reduced in 64 bits.  interleaved 0: pairs (i, i + rot_dim / 2); 1: pairs (2i, 2i + 1).
 * inverse 1: the transposed map, R(-position) with the same scale, which is the gradient with respect to x. */
dbt_status dbt_op_rope(const void *x, void *y, const int32_t *positions, const double *freq, int64_t rows, int32_t heads,
                       int32_t head_dim, int32_t rot_dim, int64_t x_row_stride, int64_t x_head_stride, int64_t y_row_stride,
                       int64_t y_head_stride, float scale, int32_t interleaved, int32_t inverse, int32_t dtype,
                       void *cuda_stream);

/* A step's queries and keys of drafted nodes rotated by positions int32 [B][max_nodes], the queries written to q_out
 * [B][max_nodes][n_q_heads][head_dim] (contiguous; not q), the keys and values to the cache positions of their nodes.
 * q, k, v [B][max_nodes][heads][head_dim], head_dim contiguous, strides for batch, node and head. */
typedef struct {
    uint32_t struct_size; /* sizeof(dbt_rope_append_args) */
    int32_t dtype, B, max_nodes, n_q_heads, n_kv_heads, head_dim, rot_dim, interleaved;
    int32_t num_pages, pages_per_seq;
    float scale;
    const void *q, *k, *v;
    int64_t q_stride[3], k_stride[3], v_stride[3]; /* batch, node, head */
    void *q_out, *cache_layer;
    const int32_t *positions, *page_table, *seq_lens, *node_counts;
    const double *freq;
    int32_t *status_dev;
} dbt_rope_append_args;
dbt_status dbt_op_rope_append(const dbt_rope_append_args *args_host, void *cuda_stream);

/* Attention of drafted nodes: node i of sequence b attends to the cached positions 0 .. seq_lens[b]-1 and, among the nodes,
 * to itself and its ancestors.  q [B][max_nodes][n_q_heads][head_dim] with strides (head_dim contiguous), out
 * [B][max_nodes][n_q_heads][head_dim] contiguous, query head h reads KV head h / (n_q_heads / n_kv_heads); scores are
 * multiplied by softmax_scale (0: 1 / sqrt(head_dim)).  Softmax in fp32.  workspace: dbt_op_attn_tree_workspace bytes,
 * 256-byte aligned, nothing in it needs to be initialised. */
typedef struct {
    uint32_t struct_size; /* sizeof(dbt_attn_tree_args) */
    int32_t dtype, B, max_nodes, n_q_heads, n_kv_heads, head_dim;
    int32_t num_pages, pages_per_seq;
    float softmax_scale;
    const void *q, *cache_layer;
    int64_t q_stride[3]; /* batch, node, head */
    void *out;
    const int32_t *page_table, *seq_lens, *node_counts, *parents;
    void *workspace;
    size_t workspace_bytes;
    int32_t *status_dev;
} dbt_attn_tree_args;
/* Bytes of workspace that this call needs (pointers are not looked at). */
dbt_status dbt_op_attn_tree_workspace(const dbt_attn_tree_args *args_host, size_t *bytes_host);
dbt_status dbt_op_attn_tree(const dbt_attn_tree_args *args_host, void *cuda_stream);

/* A token per row of logits [rows][vocab] (DBT_DTYPE_*, row_stride elements apart), from one number u in [0, 1) a row
 * (uniforms fp32 [rows]).  With w_i = exp((z_i - max z) / temperature):
 *   top_k  > 0: the k largest logits stay (ties: the lower token id);
 *   top_p  < 1: of those, in falling order, the shortest run that holds at least top_p of their mass;
 *   min_p  > 0: of those the ones with w_i >= min_p.
 * The likeliest token always stays.  The token is the first, in rising order of ids, at which the running sum of the
 * remaining w exceeds u times their total.  temperature <= 0: the largest logit.  NaN logits count as -inf; a row without
 * any logit above -inf gives token -1 and log-probability -inf; where the largest is +inf, the infinite ones share all mass.
 * u below 0 counts as 0; at 1, above it or not a number the last token that is kept comes.
 * temperature, top_p, min_p fp32 [rows], top_k int32 [rows]; each may be NULL (1, off, off, off).  tokens int32 [rows];
 * logprobs fp32 [rows] or NULL: log of the token's share of the remaining mass (0 where the temperature is <= 0).
 * Masses are formed and summed in 64 bits.  2 <= vocab <= 262144. */
dbt_status dbt_op_sample(const void *logits, int32_t dtype, int32_t rows, int32_t vocab, int64_t row_stride,
                         const float *uniforms, const float *temperature, const int32_t *top_k, const float *top_p,
                         const float *min_p, int32_t *tokens, float *logprobs, void *cuda_stream);

/* Acceptance: from node 0 on, the walk goes to the child (lowest number first) whose token is the one sampled at the
 * current node, as long as there is one.  tokens, parents, sampled int32 [B][max_nodes].  Outputs: path int32
 * [B][max_nodes], the accepted nodes in order (node 0 first), -1 behind them; counts int32 [B]; next_tokens int32 [B], the
 * token sampled at the last accepted node (-1 for a sequence without nodes); new_lens int32 [B], seq_lens + count (a buffer
 * of its own, not seq_lens).  The accepted nodes' keys and values are moved to positions seq_lens[b] .. + count - 1 in all n_layers
 * layers of pool [n_layers][2][num_pages][n_kv_heads][16][head_dim]; the positions behind keep what they hold. */
typedef struct {
    uint32_t struct_size; /* sizeof(dbt_tree_accept_args) */
    int32_t dtype, B, max_nodes, n_layers, n_kv_heads, head_dim;
    int32_t num_pages, pages_per_seq;
    const int32_t *tokens, *parents, *sampled, *page_table, *seq_lens, *node_counts;
    void *pool;
    int32_t *path, *counts, *next_tokens, *new_lens;
    int32_t *status_dev;
} dbt_tree_accept_args;
dbt_status dbt_op_tree_accept(const dbt_tree_accept_args *args_host, void *cuda_stream);

/* Per-kernel timing for the roofline report (paper Eq. roofline, Eq. decode_traffic: time
 * against the bytes that must move).  Between begin and end every kernel launch is bracketed
 * by CUDA events on the handle's stream; end waits for the stream and sums, per kernel family,
 * the launches, the device time and the algorithmic bytes (weights read once, visible K/V read
 * once; 0 for kernels that move neither).  entries_host HOST [max_entries]. */
typedef struct {
    char name[32];
    int64_t launches;
    double total_ms;
    double bytes;
} dbt_profile_entry;
dbt_status dbt_profile_begin(dbt_model *m);
dbt_status dbt_profile_end(dbt_model *m, dbt_profile_entry *entries_host, int32_t max_entries, int32_t *n_entries);

/* Kernels launched by this handle since creation (for benchmark bookkeeping). */
int64_t dbt_launch_count(const dbt_model *m);
/* Last host-side error message of this handle (or of the failed dbt_create when m is NULL). */
const char *dbt_last_error(const dbt_model *m);
/* Library version string. */
const char *dbt_version(void);

#ifdef __cplusplus
}
#endif
#endif /* DBT_H */
