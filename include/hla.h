/*
 * hla.h — C ABI of the MI355X (gfx950) Higher-order Linear Attention library.
 *
 * The library computes the strictly causal (masked) second-order HLA of
 * "Higher-order Linear Attention" (arXiv 2510.27258):
 *
 *     o_t = q_t^T (S_t C_t - G_t)                               (Thm. 1)
 *         = sum_{j<=t} sum_{i<=j} (q_t.k_i)(q_j.k_i) v_j        (Sec. 3.1)
 *
 * with S_t = sum k k^T, C_t = sum q v^T, m_t = sum q and the masking summaries
 * G_t = sum_i k_i k_i^T C_{i-1}, h_t = sum_i k_i k_i^T m_{i-1} (Sec. 3 and
 * 3.1), its ratio-normalised form num/(den + eps) with den_t = q_t^T(S_t m_t -
 * h_t) (Thm. 1), and the unmasked operator q_t^T S_t C_t (Eq. hla-unnorm,
 * Eq. hla-row).  Sequences are processed by the chunk-parallel associative
 * scan of Sec. 4 (Eq. semidirect, Thm. 2, Rem. scan-modes); the decode step
 * applies the online updates of Sec. 3.1.
 *
 * Conventions for every call
 *   - Pointers to tensors are DEVICE pointers.  The caller owns all memory,
 *     including workspaces sized by the *_workspace_bytes queries.  The library
 *     never allocates device memory, never synchronises, and enqueues work
 *     only on `stream` (a hipStream_t; NULL = the default stream).  Results
 *     are available once that stream reaches the enqueued work.
 *   - Tensors are row-major and contiguous:
 *       q, k [B, H, n, d]   v [B, H, n, dv]   out [B, H, n, dv]
 *     q/k/v are `dtype` (HLA_FP32 or HLA_BF16: raw bfloat16 bit patterns);
 *     outputs and states are always fp32.  Base pointers must be 16-byte
 *     aligned.  Inputs are read-only; inputs and outputs must not alias.
 *   - A head's second-order state is one fp32 record of
 *     F = d*d + 2*d*dv + 2*d floats (hla2_state_floats), in the order
 *       S [d][d] | C [d][dv] | m [d] | G [d][dv] | h [d]
 *     i.e. (S^K, C^QV, m^Q, G, h) of Sec. 3.1.  A state array [B, H, F]
 *     stores the records of all heads back to back.  The all-zero record is
 *     the identity segment (Thm. 2).
 *   - Supported sizes: d, dv in {16, 32, 64, 128}; chunk in {16, 32, 64,
 *     128}; any n >= 1 (a short last chunk is exact) with
 *     n * max(d, dv) * 4 < 2^31 (one head's fp32 rows stay within 32-bit
 *     byte offsets: n < 4 194 304 at d = dv = 128), else HLA_ERR_UNSUPPORTED;
 *     B*H <= 65535.
 *     masked, normalized in {0, 1}; eps finite and >= 0 (added to the
 *     denominator as is, den + eps).  Decay is 1 (hla2_forward_decay takes
 *     a decay) and the ridge 0.
 *   - Every call returns an hla_status.  On failure nothing is enqueued and
 *     hla_last_error() describes the reason (a thread-local string).
 *     Results are deterministic: the same inputs give bit-identical outputs.
 *   - Size queries returning size_t (*_workspace_bytes, hla2_state_bytes)
 *     return 0 exactly when the arguments would be rejected, and then set
 *     hla_last_error(); every accepted argument list gives a size > 0.
 *     hla2_workspace_query returns the status itself.
 *   - The environment variable HLA_FUSED_SEGMENTS=<p>, when set, overrides
 *     how many segments per head the segment-walk plans (fused forward and
 *     its decayed form, the fp32 / fp64 walk, AHLA, backward, third order)
 *     cut each head into (fewer where the workspace holds fewer), for
 *     testing and tuning; any p >= 1 gives the same result up to fp32
 *     rounding order.  Workspace queries read it too: set it before the
 *     query.  A call checks its workspace against its own plan.
 *   - At d = dv = 128 (chunk 64 or 128, bf16, masked) the fused forward, and
 *     prefill where it writes outputs, writes every output row once: a summary
 *     walk gives each segment's bracket, and one walk per segment starts from
 *     its true carry.  HLA_FUSED_LEGACY=1 selects instead the walk whose
 *     outputs a second kernel corrects by the carry (the form of the other
 *     widths), for testing; both give the same result up to fp32 rounding
 *     order.
 */
#ifndef HLA_H
#define HLA_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  HLA_OK = 0,
  HLA_ERR_INVALID = 1,      /* null pointer, bad size, flag or alignment */
  HLA_ERR_UNSUPPORTED = 2,  /* valid but not implemented (e.g. d = 96)  */
  HLA_ERR_WORKSPACE = 3,    /* workspace missing or too small           */
  HLA_ERR_HIP = 4           /* a HIP launch or runtime call failed      */
} hla_status;

typedef enum { HLA_FP32 = 0, HLA_BF16 = 1 } hla_dtype;

/* Activation of a gated projection. */
typedef enum { HLA_ACT_SILU = 0, HLA_ACT_GELU = 1 } hla_act;

/* Forward algorithms selectable through hla2_forward_ex. */
typedef enum {
  HLA_ALGO_AUTO = 0,     /* library choice (fused when supported)             */
  HLA_ALGO_CHUNKED = 1,  /* fp32 / fp64 arithmetic: a segment walk (d = dv),
                            else per-chunk summaries, (+)-scan, readout       */
  HLA_ALGO_FUSED = 2     /* segment walk with the carry state kept on chip    */
} hla_algo;

/* Reason for the last failed call on this thread ("" if none). */
const char *hla_last_error(void);

/* Floats in one second-order state record: d*d + 2*d*dv + 2*d. */
size_t hla2_state_floats(int d, int dv);

/* ---------------------------------------------------------------------------
 * hla2_forward — masked (or unmasked) second-order HLA over whole sequences.
 * Thm. 1 (output), Sec. 4 (chunk-parallel scan).  out[b,h,t,:] = o_t of head
 * (b,h); with normalized = 1, num_t / (den_t + eps).  `chunk` is the scan's
 * chunk size; results do not depend on it beyond rounding (Thm. 2).
 * workspace: at least hla2_workspace_bytes(...) bytes of device memory (its
 * contents on entry are ignored).  Returns HLA_ERR_WORKSPACE if smaller.
 * ------------------------------------------------------------------------- */
size_t hla2_workspace_bytes(int B, int H, int n, int d, int dv, int chunk, int dtype);
int hla2_forward(const void *q, const void *k, const void *v, float *out,
                 int B, int H, int n, int d, int dv, int chunk, int masked, int normalized,
                 float eps, int dtype, void *workspace, size_t workspace_bytes, void *stream);

/* As hla2_forward with an explicit algorithm (hla_algo) and an optional
 * denominator output.  den: NULL, or (normalized = 1 only) fp32 [B, H, n]
 * receiving den_t of Thm. 1 (q_t^T (S_t m_t - h_t) masked, q_t^T S_t m_t
 * unmasked), without eps; den != NULL with normalized = 0 is HLA_ERR_INVALID.
 * HLA_ALGO_FUSED returns HLA_ERR_UNSUPPORTED for shapes it does not cover.
 * Sizes for HLA_ALGO_AUTO are those of the masked operator; unmasked it takes
 * HLA_ALGO_CHUNKED, whose size the caller then asks for. */
size_t hla2_workspace_bytes_ex(int B, int H, int n, int d, int dv, int chunk, int dtype, int algo);
int hla2_forward_ex(const void *q, const void *k, const void *v, float *out, float *den,
                    int B, int H, int n, int d, int dv, int chunk, int masked, int normalized,
                    float eps, int dtype, void *workspace, size_t workspace_bytes, int algo,
                    void *stream);

/* Workspace size of hla2_forward_ex as a status: on HLA_OK *bytes holds the
 * size; otherwise *bytes is 0 and hla_last_error() says why.  bytes must not
 * be NULL (HLA_ERR_INVALID). */
int hla2_workspace_query(int B, int H, int n, int d, int dv, int chunk, int dtype, int algo, size_t *bytes);

/* The segment plan of the fused path for these arguments, as the forward
 * without initial or final state uses it: *segments gets the number of
 * segments each head is cut into (walked in parallel, composed by
 * Eq. semidirect), *tile the token tile the walk advances by, and, unless the
 * pointers are NULL, *first_tiles the tiles of segment 0 and
 * *tiles_per_segment those of every later segment (the last holds the rest).
 * Returns HLA_ERR_UNSUPPORTED when the fused path does not cover the shape
 * (bf16 inputs, masked).  Reads HLA_FUSED_SEGMENTS like the forward. */
int hla2_fused_plan(int B, int H, int n, int d, int dv, int chunk, int *segments, int *tile, int *first_tiles,
                    int *tiles_per_segment);

/* 1 if hla2_forward_ex would accept `algo` for these arguments, else 0.
 * HLA_ALGO_FUSED covers bf16 inputs, masked = 1, n * max(d, dv) * 4 < 2^31
 * and (tile, d, dv) in {(64,64,64), (32,32,32), (64,32,32), (32,64,64),
 * (64,64,32), (64,32,64), (64,128,128), (32,128,128)}, where the tile is the
 * chunk for chunk 32 and 64, and 64 for chunk 128 (the scan is exact for any
 * chunking, Thm. 2, so the tile changes only the rounding order). */
int hla2_algo_supported(int algo, int n, int d, int dv, int chunk, int dtype, int masked);

/* ---------------------------------------------------------------------------
 * hla2_forward_noalloc — hla2_forward for callers that cannot allocate device
 * memory: code under HIP graph capture, tight serving loops, harnesses that
 * forbid hipMalloc.  Same arguments, checks and results as hla2_forward
 * (algorithm HLA_ALGO_AUTO), without the workspace arguments: the workspace
 * is a fixed array of HLA_NOALLOC_SCRATCH_BYTES bytes in the library's own
 * device memory, one per GPU, held until the process ends.  Sizes whose
 * workspace (hla2_workspace_query of the algorithm HLA_ALGO_AUTO takes for
 * the call's masked flag) exceeds it return HLA_ERR_WORKSPACE before
 * anything is enqueued.  The call allocates nothing.  Every call on one GPU
 * shares that GPU's array (no call needs it cleared: the workspace's
 * contents on entry are ignored), so calls that overlap on one GPU (other
 * streams, other threads) race and must be ordered by the caller.
 * ------------------------------------------------------------------------- */
#define HLA_NOALLOC_SCRATCH_BYTES ((size_t)128 << 20)
int hla2_forward_noalloc(const void *q, const void *k, const void *v, float *out,
                         int B, int H, int n, int d, int dv, int chunk, int masked, int normalized,
                         float eps, int dtype, void *stream);

/* ---------------------------------------------------------------------------
 * hla2_chunk_summaries — the summary of every chunk of `chunk` tokens with a
 * zero carry-in: the (+)-product of its token segments (Sec. 4.2, Rem.
 * scan-modes: chunk summary).  states: [B, H, M, F], M = ceil(n / chunk);
 * chunk c covers tokens [c*chunk, min(n, (c+1)*chunk)).
 * ------------------------------------------------------------------------- */
int hla2_chunk_summaries(const void *q, const void *k, const void *v, float *states,
                         int B, int H, int n, int d, int dv, int chunk, int dtype, void *stream);

/* ---------------------------------------------------------------------------
 * hla2_scan — exclusive scan under the masked semidirect product, Eq.
 * (semidirect): prefix[b,h,c] = init (+) states[b,h,0] (+) ... (+)
 * states[b,h,c-1] (Rem. scan-modes).  states, prefix: [B, H, M, F];
 * init: [B, H, F] or NULL (identity); total: [B, H, F] receives the inclusive
 * product of all M segments, or NULL.  prefix and total must not alias
 * states or init.
 * ------------------------------------------------------------------------- */
int hla2_scan(const float *states, const float *init, float *prefix, float *total,
              int B, int H, int M, int d, int dv, void *stream);

/* ---------------------------------------------------------------------------
 * Decode state (Sec. 3.1 online updates; Thm. 2 identity).  A descriptor
 * fixes, for the life of the state, the operator every prefill and step on
 * it applies (masked, normalized, eps) and the dtype of the tokens they take,
 * so a prefill and the steps after it cannot disagree.  The state itself is
 * caller-owned device memory holding one record of FP floats per head: the
 * fields of the record above with S packed symmetric (Sec. 5: only its upper
 * triangle is stored), FP = d(d+1)/2 + 2*d*dv + 2*d:
 *   S [d(d+1)/2] | C [d][dv] | m [d] | G [d][dv] | h [d].
 * S is stored as d/2 folded row pairs of d+1 floats: pair p holds row p of S
 * from column p (d-p values), then row d-1-p from column d-1-p (p+1 values);
 * element (a, j), a <= j, is at p*(d+1) + c with p = a, c = j-a when a < d/2,
 * else p = d-1-a, c = j+1.  hla2_state_export writes the full records.
 * S, C, m, G, h point at head 0's fields and head i's field X is
 * X + i * head_floats.  `check` is written by hla2_state_init: a call
 * given a descriptor whose other fields changed since then returns
 * HLA_ERR_INVALID.  The descriptor is a host object; pass it by pointer.
 * ------------------------------------------------------------------------- */
typedef struct {
  int B, H, d, dv;            /* heads B*H; key and value widths            */
  int masked, normalized;     /* operator of every prefill and step          */
  int dtype;                  /* HLA_FP32 or HLA_BF16: the tokens' dtype     */
  float eps;                  /* denominator offset, used when normalized    */
  float *data;                /* [B, H, FP] fp32 device memory, caller-owned */
  size_t head_floats;         /* FP = d*(d+1)/2 + 2*d*dv + 2*d               */
  float *S, *C, *m, *G, *h;   /* head 0's fields inside data                 */
  unsigned long long check;   /* set by hla2_state_init                      */
} hla2_state;

/* Device bytes of a state of B*H heads: B*H*FP*4 (0 if invalid). */
size_t hla2_state_bytes(int B, int H, int d, int dv);

/* Fill *st for the device buffer buf (at least hla2_state_bytes(B, H, d, dv)
 * bytes, 16-byte aligned) and enqueue its zeroing on `stream`: the all-zero
 * record is the identity segment of Thm. 2, the state before any token.
 * Argument rules as hla2_forward (sizes, flags, eps, dtype). */
int hla2_state_init(hla2_state *st, void *buf, size_t buf_bytes, int B, int H, int d, int dv, int masked,
                    int normalized, float eps, int dtype, void *stream);

/* ---------------------------------------------------------------------------
 * hla2_prefill — continue every head's state over n new tokens:
 *   state <- state (+) summary(tokens)          (Thm. 2)
 * and, if out != NULL, write the outputs of those tokens ([B, H, n, dv]) as
 * the serial recurrence started from the given state would (Sec. 3.1,
 * Thm. 1), with the state's operator.  q, k: [B, H, n, d], v: [B, H, n, dv]
 * in the state's dtype.  workspace: at least hla2_prefill_workspace_bytes(st,
 * n, chunk) bytes.
 * ------------------------------------------------------------------------- */
size_t hla2_prefill_workspace_bytes(const hla2_state *st, int n, int chunk);
int hla2_prefill(hla2_state *st, const void *q, const void *k, const void *v, int n, int chunk, float *out,
                 void *workspace, size_t workspace_bytes, void *stream);

/* ---------------------------------------------------------------------------
 * hla2_step — one decode step per head: the online updates of Sec. 3.1 and
 * the readout of Thm. 1 (Sec. 5 order), with the state's operator.
 * q_t, k_t: [B, H, d]; v_t: [B, H, dv] in the state's dtype; out_t: [B, H, dv]
 * fp32.  The state is updated in place.
 * ------------------------------------------------------------------------- */
int hla2_step(hla2_state *st, const void *q_t, const void *k_t, const void *v_t, float *out_t, void *stream);

/* ---------------------------------------------------------------------------
 * hla2_state_export — the state as full records (the paper's 5-tuple with S
 * as a d x d matrix): full is [B, H, F] fp32 device memory, F =
 * hla2_state_floats(d, dv), caller-owned, 16-byte aligned, not aliasing the
 * state.  Enqueued on `stream`; the state is not changed.
 * ------------------------------------------------------------------------- */
int hla2_state_export(const hla2_state *st, float *full, void *stream);

/* ---------------------------------------------------------------------------
 * hla2_forward_decay — second-order HLA with exponential time decay gamma
 * (decay section; decay-aware monoid of Sec. 4).  Token moments age as
 *   S_t = gamma S_{t-1} + k_t k_t^T,  C_t = gamma C_{t-1} + q_t v_t^T,  m_t = gamma m_{t-1} + q_t,
 * so the pair (i, j) enters row t with weight gamma^{(t-i)+(t-j)}:
 *   masked    o_t = sum_{j<=t} sum_{i<=j} gamma^{(t-i)+(t-j)} (q_t.k_i)(q_j.k_i) v_j
 *   unmasked  o_t = sum_{j<=t} sum_{i<=t} gamma^{(t-i)+(t-j)} (q_t.k_i)(q_j.k_i) v_j
 * i.e. q_t^T (S_t C_t - G_t) with G_t = gamma^2 G_{t-1} + gamma k_t k_t^T C_{t-1}
 * (the paper prints the cross-summary and the segment concatenation in two
 * forms that disagree; this is the reading whose masked output drops exactly
 * the pairs j < i of the unmasked decayed output and whose concatenation,
 * with rho^2 on G and h, is associative).  normalized divides by the same
 * sum without v_j, plus eps.  gamma = 1 is hla2_forward's operator.
 * bf16 inputs, masked, d = dv in {64, 128}, chunk 64 or 128 run on the fused
 * segment walk with decay (bf16 MFMA, every decay factor applied in fp32 before
 * the hi/lo split); everything else on the chunked path in fp32 (decayed
 * chunk summaries, the decayed (+)-scan, decayed readout).  Arguments as
 * hla2_forward, plus
 * gamma, finite, 0 < gamma <= 1 (else HLA_ERR_INVALID); gamma^(2*tile), with
 * tile = min(chunk, 64) the token tile both paths walk, must stay a normal
 * fp32 number (gamma >= 0.51 at chunk 64 and 128; HLA_ERR_UNSUPPORTED
 * otherwise).  workspace: hla2_forward_decay_workspace_bytes(...) bytes (enough
 * for either path).
 * ------------------------------------------------------------------------- */
size_t hla2_forward_decay_workspace_bytes(int B, int H, int n, int d, int dv, int chunk, int dtype);
int hla2_forward_decay(const void *q, const void *k, const void *v, float *out,
                       int B, int H, int n, int d, int dv, int chunk, int masked, int normalized,
                       float eps, float gamma, int dtype, void *workspace, size_t workspace_bytes,
                       void *stream);

/* ---------------------------------------------------------------------------
 * hla3_forward — third-order HLA over whole sequences (Sec. 7).
 * masked = 1: out[b,h,t,:] = q_t^T F_t with F_t the corrected third-order
 * state (Eq. hla3-corrected-state, Thm. 3): the sum, over triples (i, u, j)
 * <= t whose largest index is attained at least twice, of
 * (q_t.k_i)(k_i.q_u)(q_u.k_j) v_j.  Computed in fp32 by the chunk-parallel
 * scan of Sec. 7.3 (operator (x)_3, Thm. 4).
 * masked = 0: out[b,h,t,:] = q_t^T S^K_t S^Q_t P_t (Sec. 7.1), the same sum
 * over all triples (i, u, j) <= t; the summaries only add, so each segment is
 * walked from the running sum of the moments before it.
 * With normalized = 1 the row is divided by (den_t + eps), den_t the same sum
 * without v_j (q_t^T eta_t masked, q_t^T S^K_t S^Q_t m^K_t unmasked).
 * q, k: [B, H, n, d]; v: [B, H, n, dv], fp32 or bf16 (dtype); out: [B, H, n, dv]
 * fp32; all device pointers, 16-byte aligned, caller-owned.
 * Supported: d and dv in {16, 32}, chunk in {16, 32, 64, 128}; chunks above
 * 32 are walked in 32-token tiles (exact for any chunking, Thm. 4).  Other
 * sizes return HLA_ERR_UNSUPPORTED.
 * workspace: at least hla3_workspace_bytes(...) bytes of device memory (its
 * contents on entry are ignored); HLA_ERR_WORKSPACE if smaller.
 * ------------------------------------------------------------------------- */
size_t hla3_workspace_bytes(int B, int H, int n, int d, int dv, int chunk, int dtype);
int hla3_forward(const void *q, const void *k, const void *v, float *out,
                 int B, int H, int n, int d, int dv, int chunk, int masked, int normalized,
                 float eps, int dtype, void *workspace, size_t workspace_bytes, void *stream);

/* ---------------------------------------------------------------------------
 * hla2_backward — gradients of the masked, unnormalised second-order HLA
 * (the reverse scan of Sec. 4.2, written out): for a loss L with upstream
 * gradient g = dL/dout,
 *   dq_j = Phi_j g_j + S_j u_j,   dv_j = U_j^T r_j,   dk_i = (Z_i + Z_i^T) k_i,
 * with S_j = sum_{i<=j} k_i k_i^T, r_j = S_j q_j, Phi_j = sum_{j'<=j} r_j' v_j'^T,
 * U_j = sum_{t>=j} q_t g_t^T, u_j = U_j v_j, Z_i = sum_{j>=i} u_j q_j^T.
 * Computed on bf16 MFMA (fp32 operands split hi/lo, fp32 accumulation) as
 * seven causal or anti-causal first-order chunk scans over 64-token tiles.
 * q, k, v [B, H, n, d] bf16 (dtype = HLA_BF16); g [B, H, n, dv] fp32;
 * dq, dk [B, H, n, d] and dv [B, H, n, dv] fp32, written (not accumulated).
 * Device pointers, 16-byte aligned, caller-owned; outputs must not alias
 * inputs or each other.  Supported: d = dv in {64, 128}, chunk any supported
 * value (the tiling does not change the result beyond rounding), any n >= 1;
 * everything else returns HLA_ERR_UNSUPPORTED.  workspace: at least
 * hla2_backward_workspace_bytes(...) bytes (contents on entry ignored).
 * ------------------------------------------------------------------------- */
size_t hla2_backward_workspace_bytes(int B, int H, int n, int d, int dv, int chunk, int dtype);
int hla2_backward(const void *q, const void *k, const void *v, const float *g, float *dq, float *dk,
                  float *dv, int B, int H, int n, int d, int dv_dim, int chunk, int dtype,
                  void *workspace, size_t workspace_bytes, void *stream);

/* As hla2_backward with the gradients in grad_dtype: HLA_FP32, or HLA_BF16 for
 * dq, dk, dv bf16 (the same fp32 sums, rounded to nearest even once). */
size_t hla2_backward_workspace_bytes_ex(int B, int H, int n, int d, int dv, int chunk, int dtype, int grad_dtype);
int hla2_backward_ex(const void *q, const void *k, const void *v, const float *g, void *dq, void *dk,
                     void *dv, int B, int H, int n, int d, int dv_dim, int chunk, int dtype, int grad_dtype,
                     void *workspace, size_t workspace_bytes, void *stream);

/* ---------------------------------------------------------------------------
 * ahla_forward — asymmetric second-order HLA (AHLA, Sec. 6): the left-cascaded
 * product ((A A) (.) L) V with A = L (.) Q K^T (diagonal kept),
 *   o_t = sum_{j<=t} sum_{i=j..t} (q_t.k_i)(q_i.k_j) v_j     (Eq. AHLA-explicit)
 *       = q_t^T E_t,  E_t = E_{t-1} + k_t (q_t^T P_t),  P_t = P_{t-1} + k_t v_t^T
 * (Thm. AHLA; E_t uses P_t including token t).  With normalized = 1 the row
 * is divided by (q_t^T n_t + eps), n_t = n_{t-1} + k_t (q_t^T m_t), m_t the
 * key sum: the same double sum without v_j.  Decay is 1.
 * Computed on bf16 MFMA with fp32 accumulation by a segment scan under
 * (+)_AHLA (Eq. AHLA-semidirect): q, k, v [B, H, n, d] bf16 (dtype =
 * HLA_BF16), out [B, H, n, d] fp32; device pointers, 16-byte aligned,
 * caller-owned.  Supported: d = dv in {64, 128}, chunk in {64, 128} (walked
 * in 64-token tiles; exact for any chunking), any n >= 1; everything else
 * (fp32 inputs included) returns HLA_ERR_UNSUPPORTED.  workspace: at least
 * ahla_workspace_bytes(...) bytes of device memory (contents on entry
 * ignored); HLA_ERR_WORKSPACE if smaller.
 * ------------------------------------------------------------------------- */
size_t ahla_workspace_bytes(int B, int H, int n, int d, int dv, int chunk, int dtype);
int ahla_forward(const void *q, const void *k, const void *v, float *out,
                 int B, int H, int n, int d, int dv, int chunk, int normalized, float eps,
                 int dtype, void *workspace, size_t workspace_bytes, void *stream);

/* ---------------------------------------------------------------------------
 * The operators around the attention.  Their conventions differ from the
 * above where said:
 *   - Activations come as a projection leaves them, token by token: x
 *     [B, n, ...] with the elements of a token contiguous and any strides
 *     >= 0 between batches (_bs) and tokens (_ts), in elements (a stride of 0
 *     repeats a row; the stride of a dimension of size one is not used).
 *     Outputs are contiguous and must not alias inputs.
 *   - Outputs and gradients have the type of what they belong to (`dtype`,
 *     `w_dtype`, `dt_dtype`: HLA_FP32 or HLA_BF16), states of the scan and its
 *     per-head parameters are fp32.  All arithmetic is fp32 or better, rounded
 *     once on the way out unless said otherwise; the SiLU of bf16 inputs takes
 *     the hardware's approximate exponential and reciprocal (2^-17 of a value).
 *   - A pointer said to be optional may be NULL.
 * ------------------------------------------------------------------------- */

/* hla_conv_forward — short causal convolution along the tokens:
 *   z[b,t,c] = bias[c] + sum_{j<K} weight[c,j] x[b,t-K+1+j,c],
 *   y = z sigmoid(z) with silu = 1, else z.
 * x [B, n, D]; weight [D, K], bias [D] (optional) of w_dtype; y [B, n, D].
 * state (optional) [B, K-1, D] of dtype: the K-1 inputs before the first,
 * oldest first; replaced by the last K-1 inputs of [state; x].  Without it
 * they are zeros.  One call with n = 1 is a decode step.
 * K in {2, 3, 4}, any D, n <= 2^22, B <= 65535.  Pointers need the alignment
 * of their type; four channels kept together (D and the strides multiples of
 * four, addresses of four values' alignment) are faster. */
int hla_conv_forward(const void *x, long long x_bs, long long x_ts, const void *weight, const void *bias,
                     void *state, void *y, int B, int n, int D, int K, int silu, int dtype, int w_dtype,
                     void *stream);

/* hla_conv_backward — gradients of hla_conv_forward without a state: dx
 * [B, n, D], dweight [D, K] and dbias [D] (optional) for dy [B, n, D].
 * D (K + 1) < 2^28 - 63.
 * workspace: at least hla_conv_backward_workspace_bytes(...) bytes. */
size_t hla_conv_backward_workspace_bytes(int B, int n, int D, int K);
int hla_conv_backward(const void *x, long long x_bs, long long x_ts, const void *weight, const void *bias,
                      const void *dy, long long dy_bs, long long dy_ts, void *dx, void *dweight, void *dbias,
                      int B, int n, int D, int K, int silu, int dtype, int w_dtype, void *workspace,
                      size_t workspace_bytes, void *stream);

/* hla_qk_norm_rope — norm and position rotation of queries and keys, head by
 * head, from q [B, n, H, d] and k [B, n, Hk, d] (the heads of a token
 * contiguous) to q_out [B, H, n, d] and k_out [B, Hk, n, d]:
 *   u = weight x / sqrt(mean(x^2) + eps),
 *   (u_i, u_j) -> (u_i c - u_j s, u_j c + u_i s), c = cos[p, m], s = sin[p, m],
 * for the m-th pair of the first rot dimensions: (i, j) = (m, m + rot/2), or
 * (2m, 2m + 1) with interleaved = 1; the other dimensions keep u.
 * q_weight, k_weight (optional) [d]; cos, sin fp32 [positions, rot/2] (unused
 * with rot = 0).  p: pos[b, t] (optional; int64 with pos64 = 1, else int32;
 * pos_bs elements between batches, 0 for one row for all), without it t.  A
 * position outside [0, positions) gives NaN in the rotated dimensions.
 * d: a multiple of 8 from 16 to 256; rot even.  q, k and the outputs are
 * 16-byte aligned with strides of whole 16-byte pieces. */
int hla_qk_norm_rope(const void *q, long long q_bs, long long q_ts, const void *k, long long k_bs,
                     long long k_ts, const void *q_weight, const void *k_weight, const float *cos,
                     const float *sin, const void *pos, long long pos_bs, void *q_out, void *k_out, int B,
                     int n, int H, int Hk, int d, int rot, int positions, int interleaved, float eps,
                     int dtype, int w_dtype, int pos64, void *stream);

/* hla_qk_norm_rope_backward — its gradients: dq [B, n, H, d], dk [B, n, Hk, d]
 * and dq_weight, dk_weight [d] (optional) for dq_out [B, H, n, d] and dk_out
 * [B, Hk, n, d], both contiguous.  workspace: at least
 * hla_qk_norm_rope_backward_workspace_bytes(d) bytes. */
size_t hla_qk_norm_rope_backward_workspace_bytes(int d);
int hla_qk_norm_rope_backward(const void *q, long long q_bs, long long q_ts, const void *k, long long k_bs,
                              long long k_ts, const void *q_weight, const void *k_weight, const float *cos,
                              const float *sin, const void *pos, long long pos_bs, const void *dq_out,
                              const void *dk_out, void *dq, void *dk, void *dq_weight, void *dk_weight,
                              int B, int n, int H, int Hk, int d, int rot, int positions, int interleaved,
                              float eps, int dtype, int w_dtype, int pos64, void *workspace,
                              size_t workspace_bytes, void *stream);

/* hla_ssm_forward — selective state space scan with a scalar decay a head:
 *   dt_t = softplus(dt[b,t,h] + dt_bias[h])  (without the softplus: softplus = 0),
 *   h_t = exp(dt_t A[h]) h_{t-1} + dt_t Bm_t x_t^T,   y_t = h_t^T Cm_t + D[h] x_t.
 * x [B, n, H, P] (the heads of a token contiguous), dt [B, n, H] of dt_dtype,
 * Bm, Cm [B, n, G, N]: head h reads group h / (H / G); A, D (optional),
 * dt_bias (optional) fp32 [H]; y [B, n, H, P].  state (optional) fp32
 * [B, H, N, P]: the state before the first token, replaced by the one after
 * the last; without it the scan starts from zero.
 * P and N: multiples of 16 from 16 to 128; G divides H; B*H <= 65535;
 * B*H*n < 2^31, n <= 2^31 - 64.  A <= 0 is meant (a growing state may
 * overflow).  x, Bm, Cm: 16-byte aligned, strides of whole 16-byte pieces, the
 * rows of a sequence not overlapping.  bf16 inputs: scores and the state that
 * the outputs read are rounded to bf16 (2^-8 of a term, as the outputs are),
 * the state itself is kept in fp32.  An infinite or NaN input leaves every
 * output and state element that depends on it infinite or NaN (which of the
 * two depends on where the sequence is cut), and no other.
 * workspace: at least hla_ssm_workspace_bytes(...) bytes. */
size_t hla_ssm_workspace_bytes(int B, int n, int H, int P, int G, int N, int dtype);
int hla_ssm_forward(const void *x, long long x_bs, long long x_ts, const void *dt, long long dt_bs,
                    long long dt_ts, const float *A, const void *Bm, long long b_bs, long long b_ts,
                    const void *Cm, long long c_bs, long long c_ts, const float *D, const float *dt_bias,
                    float *state, void *y, int B, int n, int H, int P, int G, int N, int softplus,
                    int dtype, int dt_dtype, void *workspace, size_t workspace_bytes, void *stream);

/* hla_ssm_step — one token of it for every head, the state updated in place:
 * x [B, H, P], dt [B, H], Bm, Cm [B, G, N], y [B, H, P]; strides between
 * batches only.  No workspace.  B*H < 2^24. */
int hla_ssm_step(float *state, const void *x, long long x_bs, const void *dt, long long dt_bs, const float *A,
                 const void *Bm, long long b_bs, const void *Cm, long long c_bs, const float *D,
                 const float *dt_bias, void *y, int B, int H, int P, int G, int N, int softplus, int dtype,
                 int dt_dtype, void *stream);

/* hla_ssm_backward — gradients of hla_ssm_forward without a state, for dy
 * [B, n, H, P] (strides as x's): dx [B, n, H, P], dBm, dCm [B, n, G, N] (summed
 * over the heads of a group), ddt [B, n, H] of dt_dtype, and fp32 [H] dA, dD
 * (optional), ddt_bias (optional).  bf16 inputs (dtype = HLA_BF16); fp32 ones
 * return HLA_ERR_UNSUPPORTED.  Rounded to bf16 on the way: the weighted scores
 * and the gradient of the state that dx reads (2^-8 of a term), the weighted
 * products of dy and x that dB and dC read (2^-16).  The gradients of dt and of
 * the per-head parameters are fp32 and fp64 sums.  Inputs and dy are meant to be
 * finite: NaN in one token may reach the gradients of the 64-token tile around
 * it.  B, n, G and the heads a group has must fit a launch (2^32 threads, 512
 * for every 64 tokens, group and subset of a group's heads).
 * workspace: at least hla_ssm_backward_workspace_bytes(...) bytes (two states
 * for every 64 tokens of a head). */
size_t hla_ssm_backward_workspace_bytes(int B, int n, int H, int P, int G, int N, int dtype);
int hla_ssm_backward(const void *x, long long x_bs, long long x_ts, const void *dt, long long dt_bs,
                     long long dt_ts, const float *A, const void *Bm, long long b_bs, long long b_ts,
                     const void *Cm, long long c_bs, long long c_ts, const float *D, const float *dt_bias,
                     const void *dy, long long dy_bs, long long dy_ts, void *dx, void *ddt, float *dA,
                     void *dBm, void *dCm, float *dD, float *ddt_bias, int B, int n, int H, int P, int G,
                     int N, int softplus, int dtype, int dt_dtype, void *workspace, size_t workspace_bytes,
                     void *stream);

/* ---------------------------------------------------------------------------
 * The operators of a block around its mixer.  Activations, outputs, gradients
 * and optional pointers as for the operators around the attention; pointers
 * need the alignment of their type unless said otherwise, and 16-byte rows are
 * faster.  B*n < 2^31.
 * ------------------------------------------------------------------------- */

/* hla_gated_norm — the norm of a mixer's output with its gate, over the d
 * elements of a group (a head, or with G = 1 the whole token):
 *   norm_first = 0:  v = y z sigmoid(z),  out = w v / sqrt(mean v^2 + eps)
 *   norm_first = 1:  out = w y / sqrt(mean y^2 + eps) z sigmoid(z)
 * y [B, n, G, d] of y_dtype and z (optional: no gate) of dtype, any strides
 * >= 0 between batches, tokens and groups (_bs, _ts, _gs); weight (optional:
 * ones) of w_dtype, [d] or with per_group = 1 [G, d]; out [B, n, G, d] of dtype.
 * y_dtype is dtype or HLA_FP32.  d <= 16384, G <= 65535, eps finite and >= 0. */
int hla_gated_norm(const void *y, long long y_bs, long long y_ts, long long y_gs, const void *z, long long z_bs,
                   long long z_ts, long long z_gs, const void *weight, void *out, int B, int n, int G, int d,
                   int per_group, int norm_first, float eps, int y_dtype, int dtype, int w_dtype, void *stream);

/* hla_gated_norm_backward — its gradients for dout [B, n, G, d]: dy of y_dtype
 * with strides of its own (rows that do not overlap), dz [B, n, G, d] (unused
 * without a z), dweight (optional) like weight, an fp32 sum over tokens (and
 * groups) in a fixed order.  workspace: at least
 * hla_gated_norm_backward_workspace_bytes(...) bytes. */
size_t hla_gated_norm_backward_workspace_bytes(int B, int n, int G, int d, int per_group);
int hla_gated_norm_backward(const void *y, long long y_bs, long long y_ts, long long y_gs, const void *z,
                            long long z_bs, long long z_ts, long long z_gs, const void *weight, const void *dout,
                            void *dy, long long dy_bs, long long dy_ts, long long dy_gs, void *dz, void *dweight,
                            int B, int n, int G, int d, int per_group, int norm_first, float eps, int y_dtype,
                            int dtype, int w_dtype, void *workspace, size_t workspace_bytes, void *stream);

/* hla_residual_norm — the residual addition with the norms on both sides:
 *   u = y, or with post_weight (optional) post_weight y / sqrt(mean y^2 + eps)
 *   r = x + alpha scale u,  out = weight r / sqrt(mean r^2 + eps)
 * x [B, n, D] (the residual stream) and r of x_dtype, y (a block's output) and
 * out of dtype; weight, post_weight, scale [D] of w_dtype, each optional
 * (weight and scale: ones).  out is made from r before its rounding.  x_dtype
 * is dtype or HLA_FP32.  D <= 16384, alpha finite, eps finite and >= 0. */
int hla_residual_norm(const void *x, long long x_bs, long long x_ts, const void *y, long long y_bs, long long y_ts,
                      const void *weight, const void *post_weight, const void *scale, void *out, void *r, int B,
                      int n, int D, float alpha, float eps, int x_dtype, int dtype, int w_dtype, void *stream);

/* hla_residual_norm_backward — its gradients for dout [B, n, D] of dtype and dr
 * [B, n, D] of x_dtype (each optional, not both: no gradient): dx of x_dtype, dy
 * of dtype, and (optional) dweight, dpost_weight, dscale [D] of w_dtype, fp32
 * sums over the tokens in a fixed order.  workspace: at least
 * hla_residual_norm_backward_workspace_bytes(...) bytes. */
size_t hla_residual_norm_backward_workspace_bytes(int B, int n, int D);
int hla_residual_norm_backward(const void *x, long long x_bs, long long x_ts, const void *y, long long y_bs,
                               long long y_ts, const void *weight, const void *post_weight, const void *scale,
                               const void *dout, const void *dr, void *dx, void *dy, void *dweight,
                               void *dpost_weight, void *dscale, int B, int n, int D, float alpha, float eps,
                               int x_dtype, int dtype, int w_dtype, void *workspace, size_t workspace_bytes,
                               void *stream);

/* hla_glr_forward — gated linear recurrence of every channel:
 *   r = sigmoid(f + f_bias), i = sigmoid(g + g_bias), a = exp(-c softplus(decay) r)
 *   h_t = a_t h_{t-1} + sqrt(1 - a_t^2) i_t x_t,  y_t = h_t
 * x, f, g [B, n, D] of dtype; decay, f_bias, g_bias (the biases optional) fp32
 * [D]; y [B, n, D] of dtype.  state (optional) fp32 [B, D]: the state before
 * the first token, replaced by that after the last; without it zeros.  kept
 * (optional): hla_glr_kept_bytes(...) bytes for what the gradients need of the
 * forward.  c finite and >= 0, D and the strides between tokens at most 2^21.
 * An infinite or NaN x or state, or a NaN f or g, leaves the outputs of its
 * channel from its token on infinite or NaN, and no other.  An infinite f or g
 * shuts or opens its gate: the outputs take the formula's limit.
 * workspace: at least hla_glr_workspace_bytes(...) bytes. */
size_t hla_glr_workspace_bytes(int B, int n, int D);
size_t hla_glr_kept_bytes(int B, int n, int D);
int hla_glr_forward(const void *x, long long x_bs, long long x_ts, const void *f, long long f_bs, long long f_ts,
                    const void *g, long long g_bs, long long g_ts, const float *decay, const float *f_bias,
                    const float *g_bias, float *state, void *y, float *kept, int B, int n, int D, float c, int dtype,
                    void *workspace, size_t workspace_bytes, void *stream);

/* hla_glr_step — one token of it for every sequence, the state updated in
 * place: x, f, g, y [B, D]; strides between batches only.  No workspace. */
int hla_glr_step(float *state, const void *x, long long x_bs, const void *f, long long f_bs, const void *g,
                 long long g_bs, const float *decay, const float *f_bias, const float *g_bias, void *y, int B, int D,
                 float c, int dtype, void *stream);

/* hla_glr_backward — gradients of hla_glr_forward without a state, for dy
 * [B, n, D] and what the forward kept: dx, df, dg [B, n, D] of dtype, fp32 [D]
 * ddecay, df_bias, dg_bias (the biases' optional).  workspace: at least
 * hla_glr_backward_workspace_bytes(...) bytes. */
size_t hla_glr_backward_workspace_bytes(int B, int n, int D);
int hla_glr_backward(const void *x, long long x_bs, long long x_ts, const void *f, long long f_bs, long long f_ts,
                     const void *g, long long g_bs, long long g_ts, const float *decay, const float *f_bias,
                     const float *g_bias, const float *kept, const void *dy, long long dy_bs, long long dy_ts,
                     void *dx, void *df, void *dg, float *ddecay, float *df_bias, float *dg_bias, int B, int n, int D,
                     float c, int dtype, void *workspace, size_t workspace_bytes, void *stream);

/* hla_glu_forward — gated feed-forward projections
 *   h = act(x w_gate^T) * (x w_up^T),  act SiLU or GELU (by the error function)
 * x [B, n, D], w_gate, w_up [F, D], h [B, n, F], all bf16 (dtype = HLA_BF16;
 * fp32 returns HLA_ERR_UNSUPPORTED), sums in fp32, rounded once; GELU far below
 * zero is within 2e-5 of itself before that, down to x w_gate^T = -13.  D and F
 * are multiples of 8, at most 2^20; addresses and strides whole 16-byte pieces. */
int hla_glu_forward(const void *x, long long x_bs, long long x_ts, const void *w_gate, const void *w_up, void *h,
                    int B, int n, int D, int F, int act, int dtype, void *stream);

/* hla_glu_backward — its gradients for dh [B, n, F] (strides as x's): dx
 * [B, n, D], dw_gate, dw_up [F, D].  The gradients of the two projections are
 * rounded to bf16 before they meet weights and inputs (up to 2^-8 of a term).
 * workspace: at least hla_glu_backward_workspace_bytes(...) bytes. */
size_t hla_glu_backward_workspace_bytes(int B, int n, int D, int F);
int hla_glu_backward(const void *x, long long x_bs, long long x_ts, const void *w_gate, const void *w_up,
                     const void *dh, long long dh_bs, long long dh_ts, void *dx, void *dw_gate, void *dw_up, int B,
                     int n, int D, int F, int act, int dtype, void *workspace, size_t workspace_bytes, void *stream);

/* ---------------------------------------------------------------------------
 * Benchmark timing.  hla_profile_begin(max_records) creates 2*max_records HIP
 * events (host objects, no device memory) and starts bracketing every kernel
 * the library launches with events recorded on that kernel's stream;
 * hla_profile_end() stops.  After synchronising the stream,
 * hla_profile_summary(buf, len) writes one line per kernel name,
 * "name launches total_ms", and forgets the records.  Records beyond
 * max_records are not timed.  Not thread-safe; for benchmarks only.
 * ------------------------------------------------------------------------- */
int hla_profile_begin(int max_records);
int hla_profile_end(void);
int hla_profile_summary(char *buf, size_t len);

#ifdef __cplusplus
}
#endif

#endif /* HLA_H */
