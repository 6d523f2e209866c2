/*
 * vitattn.h — C ABI of the exact non-causal attention library for MI355X (gfx950).
 *
 * What it computes. One GPU's share of the self-attention of a long-sequence
 * Vision Transformer after a DeepSpeed-Ulysses all-to-all (paper Sec. II-E):
 * the full sequence of N patch tokens for H heads of B samples. Attention is
 * dense and bidirectional: every token attends to every token (Sec. I and III),
 * with no mask, bias or dropout. Per (b, h), with s = scale:
 *
 *     S = s Q K^T,  LSE_i = log sum_j exp(S_ij),  P = exp(S - LSE 1^T),  O = P V
 *
 * and the backward pass, given dO = dL/dO:
 *
 *     D_i = sum_c dO_ic O_ic,  dS = P o (dO V^T - D 1^T),
 *     dQ = s dS K,  dK = s dS^T Q,  dV = P^T dO.
 *
 * The tiling (the N x N matrices S and P are never stored), the saved per-row
 * logsumexp and the recomputation of P in the backward pass follow
 * FlashAttention-2, which the paper uses (Sec. II-F, V-B, V-E).
 *
 * Conventions shared by every entry point:
 *  - All tensor pointers are DEVICE pointers owned by the caller. The library
 *    never allocates, frees or retains them, and holds no per-call state.
 *  - Tensors are contiguous row-major [B][H][N][d] (d innermost); lse and the
 *    backward workspace are [B][H][N]. Element offsets use 64-bit arithmetic.
 *    vitattn_fwd_strided / vitattn_bwd_strided take any batch, head and row
 *    strides instead (e.g. the sequence-major [B][N][H][d] layout), see
 *    vitattn_strides below.
 *  - q, k, v and dout hold bfloat16 values as raw 16-bit patterns. o, lse, dq,
 *    dk and dv are fp32. Every pointer must be 16-byte aligned.
 *  - Supported head dims: any multiple of 8 from 8 to 160 (the paper's models
 *    use 64, 72, 128 and 160, Table I and Sec. V-C). The kernels compute in
 *    tiles of width 64, 96, 128 or 160 with the columns past d zero, so d = 72
 *    costs what d = 96 costs. Any N >= 1 with (N + 256) * row_stride * 2 below
 *    2^31 for every bf16 operand (the kernels address one head's rows with
 *    32-bit offsets; N up to 8,388,351 for dense d = 128) and B*H*N below 2^31.
 *    Every kernel launch must also stay below 2^32 work-items: 2*B*H*(N + 383)
 *    for the forward; for the backward and its stages also
 *    4*B*H*(N + 191) + 2^19 and B*H*N times 8, 16 or 32 (head dims up to 64,
 *    128, 160); B*H*N*d/4 + 256 for the merge. These bind only at head dims
 *    of 16 or less (wider rows run out of memory first); a call past them
 *    returns VITATTN_E_INVAL.
 *  - Work is enqueued on `stream` (a hipStream_t; NULL = the null stream) and
 *    the call returns without waiting. Execution faults surface at the
 *    caller's next synchronisation on that stream.
 *  - Arguments are validated before anything is launched; on any error status
 *    no output is written and no kernel is enqueued. Validation itself makes
 *    no HIP call, so it works on a machine without a GPU.
 *  - Results are bitwise deterministic for identical inputs, and a head's
 *    results do not depend on the call it is part of: one call over H heads
 *    gives the bits of H single-head calls, whatever the grid or the CU
 *    count. The only atomics are in the dK/dV stage: when its last round of
 *    key-block workgroups would be at most half full, and there are 256 query
 *    tiles of 64 or more, those key blocks may be split over two workgroups
 *    (one per half of the query tiles) that add into dK and dV rows zeroed
 *    first by the same call; two fp32 adds onto zero give the same bits in
 *    either order. With that many query tiles every key block, split or not, sums
 *    them as the same two rounded partial sums (split near the middle query
 *    tile) and adds them, and with fewer as one sum, so splitting changes no
 *    bit. Which blocks split, and how many queries or keys a workgroup takes,
 *    depends on the sizes and the device's CU count, looked up once per
 *    device at the first call (no stream work, so a graph capture may hold
 *    it).
 *  - Calls are thread-safe; concurrent calls on different streams are fine.
 */
#ifndef VITATTN_H
#define VITATTN_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

enum vitattn_status {
  VITATTN_OK = 0,
  VITATTN_E_INVAL = 1,       /* null/misaligned pointer, B/H/N < 1, non-finite or non-positive scale, size overflow */
  VITATTN_E_UNSUPPORTED = 2, /* head dim d not supported (see above) */
  VITATTN_E_WORKSPACE = 3,   /* workspace missing or smaller than vitattn_bwd_workspace_bytes() */
  VITATTN_E_HIP = 4,         /* the HIP runtime reported an error when launching */
  VITATTN_E_INTERNAL = 5,    /* unexpected internal failure */
  VITATTN_E_TOO_LARGE = 6    /* vitattn_bwd_noalloc only: B*H*N above VITATTN_NOALLOC_MAX_ROWS */
};

/*
 * Forward pass (the tiled online softmax of FlashAttention-2, cited in paper
 * Sec. II-F).
 *   q, k, v : bf16 [B][H][N][d], read only.
 *   o       : fp32 [B][H][N][d], written: O = softmax(scale * Q K^T) V.
 *   lse     : fp32 [B][H][N], written: natural-log logsumexp of each row of
 *             the scaled logits, LSE_i = log sum_j exp(scale * q_i . k_j).
 *   scale   : softmax scale, finite and > 0 (typically 1/sqrt(d)).
 * Returns a vitattn_status.
 */
int vitattn_fwd(const void* q, const void* k, const void* v, float* o, float* lse, int B, int H, int N, int d,
                float scale, void* stream);

/*
 * Bytes of device workspace vitattn_bwd needs: two fp32 [B][H][N] regions,
 * each padded to a multiple of 64 rows (256 bytes): the row statistic D and
 * LSE * log2(e). Returns 0 for invalid sizes.
 */
size_t vitattn_bwd_workspace_bytes(int B, int H, int N, int d);

/*
 * Backward pass: a D = rowsum(dO o O) preprocess, then one kernel that
 * accumulates dK and dV per key block and one that accumulates dQ per query
 * block, both recomputing P from q, k and lse (FlashAttention-2's backward,
 * cited in paper Sec. II-F).
 *   q, k, v   : bf16 [B][H][N][d], the forward inputs.
 *   o, lse    : fp32, the forward outputs of vitattn_fwd for the same inputs.
 *   dout      : bf16 [B][H][N][d], the gradient of the loss with respect to o.
 *   dq, dk, dv: fp32 [B][H][N][d], written.
 *   workspace : device buffer of at least vitattn_bwd_workspace_bytes() bytes,
 *               overwritten; it must not alias any other argument.
 * Returns a vitattn_status.
 */
int vitattn_bwd(const void* q, const void* k, const void* v, const float* o, const void* dout, const float* lse,
                float* dq, float* dk, float* dv, int B, int H, int N, int d, float scale, void* workspace,
                size_t workspace_bytes, void* stream);

/*
 * The three stages of vitattn_bwd, callable one by one (same arguments,
 * layouts and validation as vitattn_bwd; used to time each kernel). They
 * must run in this order on one stream, all with the same workspace:
 *   vitattn_bwd_rowdot: workspace <- -D_i = -sum_c dout_ic o_ic (stored negated)
 *                       and LSE_i*log2(e);
 *   vitattn_bwd_dkdv  : dk, dv from q, k, v, dout, lse and D in the workspace;
 *   vitattn_bwd_dq    : dq from q, k, v, dout, lse and D in the workspace.
 * Each stage validates its own arguments like vitattn_bwd does.
 */
int vitattn_bwd_rowdot(const float* o, const void* dout, const float* lse, int B, int H, int N, int d,
                       void* workspace, size_t workspace_bytes, void* stream);
int vitattn_bwd_dkdv(const void* q, const void* k, const void* v, const void* dout, const float* lse, float* dk,
                     float* dv, int B, int H, int N, int d, float scale, const void* workspace,
                     size_t workspace_bytes, void* stream);
int vitattn_bwd_dq(const void* q, const void* k, const void* v, const void* dout, const float* lse, float* dq,
                   int B, int H, int N, int d, float scale, const void* workspace, size_t workspace_bytes,
                   void* stream);

/*
 * Attention over one segment of the keys, and the merge of such partial
 * results. Sequence parallelism over contiguous segments (Long Sequence
 * Segmentation, paper Sec. I and II "Sequence Parallel"; one segment per
 * worker) hands one GPU its queries and the keys of one segment at a time.
 * Softmax over a union of key sets factors over the sets:
 *
 *     LSE_i = log sum_s exp(LSE_s,i),   O_i = sum_s exp(LSE_s,i - LSE_i) O_s,i
 *
 * and the backward pass of one segment, given the merged O and LSE, yields
 * that segment's complete dK and dV rows and its share of dQ.
 */

/*
 * Forward pass of Nq queries over Nk keys (vitattn_fwd is the case
 * Nq = Nk = N; same algorithm, conventions and validation).
 *   q        : bf16 [B][H][Nq][d];  k, v: bf16 [B][H][Nk][d].
 *   o        : fp32 [B][H][Nq][d], written; lse: fp32 [B][H][Nq], written.
 *   Nq, Nk   : each >= 1 and within the limits N obeys for vitattn_fwd.
 */
int vitattn_fwd_kv(const void* q, const void* k, const void* v, float* o, float* lse, int B, int H, int Nq, int Nk,
                   int d, float scale, void* stream);

/* flags of vitattn_bwd_kv and vitattn_bwd_strided */
#define VITATTN_BWD_ACCUMULATE_DQ 1 /* dq += this segment's share instead of dq = it */
#define VITATTN_BWD_STORE_DS 2      /* dS mode: dQ from stored dS (see vitattn_bwd_workspace_bytes_kv) */

/*
 * Workspace bytes of vitattn_bwd_kv / vitattn_bwd_strided for these sizes
 * and flags; 0 for invalid arguments. Without VITATTN_BWD_STORE_DS it equals
 * vitattn_bwd_workspace_bytes(B, H, Nq, d).
 *
 * The dS mode trades memory for matrix-core work. The dK/dV kernel already
 * forms dS = P o (dP - D) (bf16, the value it multiplies into dK); with
 * VITATTN_BWD_STORE_DS it also writes every dS block to the workspace, and dQ
 * = scale dS K then streams them (2 d flops per score) instead of recomputing
 * S and dP in a third kernel (6 d flops per score). The extra workspace is
 * 2 bytes per (query, key) pair of every head, rounded up to 64 queries and
 * 128 keys: B*H*Nq*Nk*2 bytes, 142 GB at B=1, H=2, N=188,416. Results differ
 * from the default mode only in the rounding of dS (the default dQ kernel
 * rounds an fp32 P times (dP - D) to bf16, this one a bf16 P times it).
 * Requires Nq <= 16,777,152.
 */
size_t vitattn_bwd_workspace_bytes_kv(int B, int H, int Nq, int Nk, int d, int flags);

/*
 * Backward pass of Nq queries over Nk keys (vitattn_bwd is the case
 * Nq = Nk = N, flags = 0).
 *   q, dout  : bf16 [B][H][Nq][d];  k, v: bf16 [B][H][Nk][d].
 *   o, lse   : fp32 [B][H][Nq][d] and [B][H][Nq]: the output and LSE of the
 *              attention the gradient flows through. For one key segment of a
 *              larger key set pass the MERGED o and lse of all keys: then
 *              dk, dv (fp32 [B][H][Nk][d], written) are exact for this
 *              segment's keys and dq (fp32 [B][H][Nq][d]) is its share.
 *   flags    : 0, or VITATTN_BWD_ACCUMULATE_DQ to add the share to dq (sum
 *              the segments of one key set by calling once per segment on
 *              one stream with dq zeroed first; the order of the sum is the
 *              order of the calls), and/or VITATTN_BWD_STORE_DS (below).
 *              Other bits: VITATTN_E_INVAL.
 *   workspace: at least vitattn_bwd_workspace_bytes_kv(B, H, Nq, Nk, d, flags)
 *              bytes (vitattn_bwd_workspace_bytes(B, H, Nq, d) without
 *              VITATTN_BWD_STORE_DS), else VITATTN_E_WORKSPACE.
 */
int vitattn_bwd_kv(const void* q, const void* k, const void* v, const float* o, const void* dout, const float* lse,
                   float* dq, float* dk, float* dv, int B, int H, int Nq, int Nk, int d, float scale, int flags,
                   void* workspace, size_t workspace_bytes, void* stream);

/*
 * Operands in other layouts. The layout an all-to-all or a fused QKV
 * projection produces is rarely the dense [B][H][N][d]: the sequence-major
 * [B][N][H][d] (paper Sec. II "Sequence Parallel") has strides
 * {N*H*d, d, H*d}, rows padded to a larger pitch have row > d, and a slice
 * of a [B][N][3][H][d] QKV tensor has row = 3*H*d. The kernels read and write
 * such operands in place; no copy is made.
 *
 * Element strides of one operand viewed as [B][H][N][d]; the d elements of a
 * row are contiguous. Every stride must be >= 0 and a multiple of 8 elements
 * for bf16 operands (4 for fp32), so rows stay 16-byte aligned, and
 * row >= d. Inputs may repeat a head or batch (stride 0, e.g. keys shared by
 * several query heads); an output may not overlap itself (checked: sorted by
 * stride, every dimension must step past the span of the smaller ones). Each
 * bf16 operand needs (rows + 256) * row * 2 < 2^31. Violations:
 * VITATTN_E_INVAL. lse and the workspace stay dense [B][H][Nq].
 */
typedef struct vitattn_strides {
  long long batch, head, row;
} vitattn_strides;

/* vitattn_fwd_kv with a layout per operand (same computation and validation). */
int vitattn_fwd_strided(const void* q, vitattn_strides sq, const void* k, vitattn_strides sk, const void* v,
                        vitattn_strides sv, float* o, vitattn_strides so, float* lse, int B, int H, int Nq, int Nk,
                        int d, float scale, void* stream);

/* vitattn_bwd_kv with a layout per operand (same computation, flags and
 * validation); sdo is the layout of dout. */
int vitattn_bwd_strided(const void* q, vitattn_strides sq, const void* k, vitattn_strides sk, const void* v,
                        vitattn_strides sv, const float* o, vitattn_strides so, const void* dout,
                        vitattn_strides sdo, const float* lse, float* dq, vitattn_strides sdq, float* dk,
                        vitattn_strides sdk, float* dv, vitattn_strides sdv, int B, int H, int Nq, int Nk, int d,
                        float scale, int flags, void* workspace, size_t workspace_bytes, void* stream);

/*
 * The backward pass of a bf16 training step: vitattn_bwd_strided (flags = 0)
 * with the conversions around it done by its kernels. grad is the fp32
 * gradient with respect to o (layout sg, strides multiples of 4); it is
 * rounded to bf16 into dout (bf16 [B][H][Nq][d], dense, written), which takes
 * the place of vitattn_bwd's dout. dq is written as bf16 [B][H][Nq][d], dk and
 * dv as bf16 [B][H][Nk][d] where vitattn_bwd_train_bf16_kv(Nq) is 1 and as
 * fp32 otherwise, all dense. The values are those of the separate conversions
 * (round to nearest even), bit for bit. dout must not alias grad
 * (dout == grad is rejected; partial overlap is not detected). The other
 * arguments, the validation and the status are vitattn_bwd_strided's.
 */
int vitattn_bwd_train_bf16_kv(int Nq);
int vitattn_bwd_train(const void* q, vitattn_strides sq, const void* k, vitattn_strides sk, const void* v,
                      vitattn_strides sv, const float* o, vitattn_strides so, const float* grad, vitattn_strides sg,
                      const float* lse, void* dout, void* dq, void* dk, void* dv, int B, int H, int Nq, int Nk, int d,
                      float scale, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Which forms of the kernels a call of these sizes takes on the current
 * device (flags as in vitattn_bwd_kv): the results do not depend on them, so
 * this serves tests and the reading of profiles. Launches nothing and needs no
 * GPU; without one it gives the forms of a device that tells nothing about
 * itself.
 *   fwd_waves, dq_waves : waves per workgroup, 32 query rows each
 *   dkdv_keys           : keys per dK/dV workgroup
 *   dkdv_whole          : key blocks (of that many keys) with one workgroup
 *   dkdv_split          : key blocks split over two workgroups
 *   dkdv_rest64         : workgroups of 64 keys that take the remaining keys
 */
typedef struct vitattn_forms {
  int fwd_waves, dq_waves, dkdv_keys, dkdv_whole, dkdv_split, dkdv_rest64;
} vitattn_forms;
int vitattn_launch_forms(int B, int H, int Nq, int Nk, int d, int flags, vitattn_forms* forms);

/* The two kernels of the dS mode as separate calls (dense operands, Nq = Nk =
 * N; the row-statistics stage vitattn_bwd_rowdot runs first), for timing each:
 * vitattn_bwd_dkdv_ds writes dK, dV and the dS blocks into the workspace,
 * vitattn_bwd_dq_from_ds then writes dQ from them. The workspace must hold
 * vitattn_bwd_workspace_bytes_kv(B, H, N, N, d, VITATTN_BWD_STORE_DS) bytes. */
int vitattn_bwd_dkdv_ds(const void* q, const void* k, const void* v, const void* dout, const float* lse, float* dk,
                        float* dv, int B, int H, int N, int d, float scale, void* workspace, size_t workspace_bytes,
                        void* stream);
int vitattn_bwd_dq_from_ds(const void* k, float* dq, int B, int H, int N, int d, float scale, const void* workspace,
                           size_t workspace_bytes, void* stream);

/* largest number of partial results vitattn_merge accepts */
#define VITATTN_MERGE_MAX_PARTS 65536

/*
 * Merge n_parts partial attention results over disjoint key segments into
 * the attention over all of them (the formula above).
 *   o_parts  : fp32 [n_parts][B][H][N][d], read; lse_parts: fp32
 *              [n_parts][B][H][N], read (each partial as written by
 *              vitattn_fwd_kv for its segment).
 *   o, lse   : fp32 [B][H][N][d] and [B][H][N], written; they must not alias
 *              the partials.
 *   n_parts  : 1 .. VITATTN_MERGE_MAX_PARTS, else VITATTN_E_INVAL.
 *   d        : any head dim the attention takes (a multiple of 8 up to 160),
 *              else VITATTN_E_UNSUPPORTED.
 * A NaN partial LSE makes the merged row NaN. Bound by HBM bandwidth.
 */
int vitattn_merge(const float* o_parts, const float* lse_parts, int n_parts, float* o, float* lse, int B, int H,
                  int N, int d, void* stream);

/*
 * Layouts around DeepSpeed-Ulysses' all-to-all (paper Sec. II "Sequence
 * Parallel"; two all-to-alls per attention in each pass, Sec. V). Each of P
 * ranks holds Nl tokens of all H heads (rank r: tokens r*Nl .. r*Nl+Nl-1);
 * attention needs the whole sequence N = P*Nl of Hl = H/P heads. With
 * rows of row_bytes bytes (one token of one head, e.g. d bf16 values):
 *
 *   pack       x    [B][Nl][H]       -> send [P][B][Hl][Nl]   send[p][b][j][i] = x[b][i][p*Hl+j]
 *   (all-to-all: chunk p of rank r's send buffer becomes chunk r of rank p's receive buffer)
 *   unpack     recv [P][B][Hl][Nl]   -> y    [B][Hl][P*Nl]    y[b][j][r*Nl+i] = recv[r][b][j][i]
 *   pack_out   y    [B][Hl][P*Nl]    -> send [P][B][Hl][Nl]   (inverse of unpack)
 *   unpack_out recv [P][B][Hl][Nl]   -> x    [B][Nl][H]       (inverse of pack)
 *
 * y is the contiguous [B][Hl][N][row] input (or output) of the attention
 * entry points. The collective itself is not part of this library.
 *   B, Nl, H, P: >= 1 with H divisible by P, B <= 65535, Nl*row_bytes/16 < 2^31
 *                and ceil(Nl*row_bytes/4096)*H < 2^24 (256 work-items per
 *                block, below 2^32 per launch).
 *   row_bytes  : a multiple of 16, >= 16.
 *   src, dst   : device pointers, 16-byte aligned, not overlapping
 *                (src == dst is rejected; partial overlap is not detected).
 * Pure copies, bound by HBM bandwidth. Returns a vitattn_status.
 */
int vitattn_ulysses_pack(const void* x, void* send, int B, int Nl, int H, int P, int row_bytes, void* stream);
int vitattn_ulysses_unpack(const void* recv, void* y, int B, int Nl, int H, int P, int row_bytes, void* stream);
int vitattn_ulysses_pack_out(const void* y, void* send, int B, int Nl, int H, int P, int row_bytes, void* stream);
int vitattn_ulysses_unpack_out(const void* recv, void* x, int B, int Nl, int H, int P, int row_bytes, void* stream);

/*
 * Channel aggregation by attention with a learnable query: the Agg-Ch-ViT
 * layer (paper Sec. II "Patch Embedding and Sequence Length") folds the C
 * channel tokens of each patch into one token. For M patch positions (batch
 * x patches) and H heads, one query q_h per head, shared by every patch,
 * attends over that patch's projected channel keys and values:
 *
 *   s_c = scale q_h . k_mhc,  lse_mh = log sum_c exp(s_c),  o_mh = sum_c exp(s_c - lse_mh) v_mhc
 *
 * and the backward pass (dq sums over every patch, as q is shared):
 *
 *   ds_c = p_c (do_mh . v_mhc - do_mh . o_mh),  dk_mhc = scale ds_c q_h,
 *   dv_mhc = p_c do_mh,  dq_h = scale sum_m sum_c ds_c k_mhc.
 *
 * Layouts (row-major): q bf16 [H][d]; k, v bf16 [M][H][C][d]; o fp32
 * [M][H][d]; lse fp32 [M][H]; dout bf16 [M][H][d]; dq fp32 [H][d]; dk, dv
 * fp32 [M][H][C][d]. M, H, C >= 1 (any C; the paper's case is C = 92) with
 * (M + 3)*H and H*d below 2^26 (64 work-items each per launch, below 2^32);
 * d in {64, 128}; scale finite and > 0. Bound by HBM bandwidth. dq is
 * reduced in a fixed order (no atomics): results are bitwise reproducible.
 */
int vitattn_agg_fwd(const void* q, const void* k, const void* v, float* o, float* lse, int M, int H, int C, int d,
                    float scale, void* stream);

/* Workspace bytes of vitattn_agg_bwd: dq partials, one per head and group of four
 * patches (ceil(M/4) x H x d floats); 0 for invalid sizes. */
size_t vitattn_agg_bwd_workspace_bytes(int M, int H, int C, int d);

/* o and lse are vitattn_agg_fwd's outputs for the same q, k, v; workspace is
 * overwritten and must not alias any other argument. */
int vitattn_agg_bwd(const void* q, const void* k, const void* v, const float* o, const void* dout, const float* lse,
                    float* dq, float* dk, float* dv, int M, int H, int C, int d, float scale, void* workspace,
                    size_t workspace_bytes, void* stream);

/*
 * vitattn_bwd without a workspace argument, for callers that cannot allocate
 * device memory (code under HIP graph capture, serving loops that must not
 * call hipMalloc, harnesses that forbid it). Same arguments (minus the
 * workspace), layouts, validation, kernels and results as vitattn_bwd: the
 * outputs are bitwise equal to vitattn_bwd's for the same inputs. The
 * workspace lives in a static device array of the library (32 MiB, one copy
 * per device the library runs on, held until the process ends), so:
 *   - B*H*N may be at most VITATTN_NOALLOC_MAX_ROWS, else VITATTN_E_TOO_LARGE
 *     (and nothing is launched);
 *   - the call itself allocates nothing (no hipMalloc, hipFree or allocating
 *     library routine). Its first call on a device looks up that device's
 *     copy of the array (hipGetSymbolAddress) with that device current; the
 *     stream must belong to the calling thread's current device;
 *   - every call on a device shares that device's array: calls that overlap
 *     in time on one device (other streams, other threads) race and must be
 *     serialised by the caller. Nothing in the array needs clearing between
 *     calls: each call rewrites every entry it reads.
 */
#define VITATTN_NOALLOC_MAX_ROWS 4194304
int vitattn_bwd_noalloc(const void* q, const void* k, const void* v, const float* o, const void* dout,
                        const float* lse, float* dq, float* dk, float* dv, int B, int H, int N, int d, float scale,
                        void* stream);

/* ------------------------------------------------------------------------
 * Operators around the attention of a block, and differential attention.
 * ------------------------------------------------------------------------ */

enum vitattn_type { VITATTN_BF16 = 0, VITATTN_FP16 = 1, VITATTN_FP32 = 2 };

/*
 * Layer norm of B*H*N rows of D elements: with mu the row's mean,
 * r = 1/sqrt(mean((x - mu)^2) + eps) and h = (x - mu) r,
 *
 *     y = h w + b,
 *     dx = r (g - mean(g) - h mean(g h)) with g = dy w,
 *     dw = sum over the rows of dy h,  db = sum over the rows of dy.
 *
 * A block's norm has B = H = 1; three row dimensions let the heads of q and k
 * be normalised where a projection left them.
 *   x, y, dy, dx: rows at any element strides >= 0 (the D elements of a row
 *                 contiguous, no alignment beyond the element's); all of
 *                 `type`. y and dx must not overlap themselves. y may be x (the
 *                 same strides); dx may be dy (the same strides), except where
 *                 dw or db is wanted and D is above 16,384 (fp32: 8,192). An output
 *                 (or workspace) whose address range meets that of any other
 *                 operand is rejected.
 *   w, b, dw, db: [D], contiguous, of `weight_type` (x's type or fp32). w and b
 *                 may be null (ones, zeros); so may dw and db (not wanted).
 *   mean, rstd  : fp32, one per row in the order [B][H][N]; the forward takes
 *                 null for both (not wanted).
 *   eps         : finite, >= 0.
 *   D           : 1 .. 2^24, else VITATTN_E_UNSUPPORTED; B*H*N below 2^31 - 2^22.
 *   workspace   : vitattn_layer_norm_bwd_workspace_bytes() bytes, 16-byte
 *                 aligned, if dw or db is wanted (partial sums; overwritten).
 * Sums and statistics are fp32 (fp64 in the lanes of rows past registers); a mean
 * of four times the spread or more is corrected to the fp32 number next to the true
 * one, so equal values have h = 0. y and dx are rounded once, to their type. dw
 * and db are summed in a fixed order that depends on the sizes alone (no
 * atomics): results are bitwise reproducible. Bound by HBM bandwidth.
 */
int vitattn_layer_norm_fwd(const void* x, vitattn_strides sx, const void* w, const void* b, void* y,
                           vitattn_strides sy, float* mean, float* rstd, int B, int H, int N, int D, float eps,
                           int type, int weight_type, void* stream);
size_t vitattn_layer_norm_bwd_workspace_bytes(int B, int H, int N, int D, int type);
int vitattn_layer_norm_bwd(const void* x, vitattn_strides sx, const void* w, const float* mean, const float* rstd,
                           const void* dy, vitattn_strides sdy, void* dx, vitattn_strides sdx, void* dw, void* db,
                           int B, int H, int N, int D, int type, int weight_type, void* workspace,
                           size_t workspace_bytes, void* stream);

/*
 * Dropout by a counter-based generator: element c of row r (rows counted in the
 * order [B][H][N], whatever their strides) is kept if its sixteen-bit number is at
 * least T = round(65536 p), and then multiplied with 65536 / (65536 - T). The numbers
 * of columns 8 g .. 8 g + 7 are the halves, the lower first, of the four words that
 * Philox 4x32 with ten rounds gives for the counter (g, r, offset mod 2^32, offset /
 * 2^32) and the key (seed mod 2^32, seed / 2^32). The mask depends on nothing else, so
 * the backward forms it again.
 *   p    : 0 .. 1.
 *   state: null, or two 64-bit numbers on the device that are added to seed and offset
 *          (mod 2^64) when the kernels run: a captured graph draws other masks when
 *          they change between replays.
 */
typedef struct vitattn_dropout_spec {
  unsigned long long seed, offset;
  const long long* state;
  double p;
} vitattn_dropout_spec;

/*
 * y = residual + dropout(x), or dropout(x) without a residual, of B*H*N rows of D
 * elements; the gradient of x is the same call on the gradient of y, without a
 * residual. A dropped element adds nothing, whatever it holds.
 *   x        : of `type`; residual (or null) and y of residual_type: type or fp32; without a
 *              residual type, or of an fp32 x also a 16-bit type. Rows at any element strides >= 0, the D elements of a
 *              row contiguous, no alignment beyond the element's. y must not overlap
 *              itself, and may be x or the residual (the same type and strides).
 *   sizes    : B*H*N below 2^31 - 2^22, B*H*N*ceil(D/8) below 2^34 - 2^14.
 * Products and the sum are one fp32 operation, rounded once. Bound by HBM bandwidth.
 */
int vitattn_dropout(const void* x, vitattn_strides sx, const void* residual, vitattn_strides sr, void* y,
                    vitattn_strides sy, int B, int H, int N, int D, int type, int residual_type,
                    const vitattn_dropout_spec* dropout, void* stream);

#define VITATTN_RMS_MAX_BYTES 32768 /* of a row of x: D up to 16,384 (fp32: 8,192) */

/*
 * Root-mean-square norm of B*H*N rows of D elements with the residual's addition:
 *
 *     h = residual + dropout(x),  r = 1/sqrt(mean(h^2) + eps),  n = h r,  y = n w
 *
 * and the backward, given dy and the gradient dh that h has from what follows it:
 *
 *     dres = r (g - n mean(g n)) + dh with g = dy w,  dx = dropout(dres),
 *     dw = sum over the rows of dy n.
 *
 * h is rounded to its type and normalised as it is stored. Without a residual (null,
 * and h null) h is x, in the backward too.
 *   x, y, dy, dx     : of `type`; residual, h, dh and dres of residual_type: type or
 *                      fp32 (type without a residual). Rows as for vitattn_dropout. y may
 *                      be x, h the residual, dx dy and dres dh (the same strides); any other
 *                      output that shares memory with another operand is rejected.
 *   w, dw            : [D], contiguous, of weight_type (type or fp32); either may be null.
 *   rstd             : fp32, one per row in the order [B][H][N]: r. Null in the forward:
 *                      not wanted.
 *   dh, dx, dres     : may be null (no such gradient; not wanted).
 *   dropout          : null: none. The forward's, in the backward; needs a residual.
 *   eps              : finite, >= 0.
 *   D                : row bytes up to VITATTN_RMS_MAX_BYTES, else VITATTN_E_UNSUPPORTED;
 *                      B*H*N below 2^31 - 2^22.
 *   workspace        : vitattn_rms_norm_bwd_workspace_bytes() bytes, 16-byte aligned, if dw
 *                      is wanted (partial sums; overwritten).
 * Sums and r are fp32, outputs rounded once. dw is summed in a fixed order that depends on
 * the sizes alone (no atomics): results are bitwise reproducible. Bound by HBM bandwidth.
 */
int vitattn_rms_norm_fwd(const void* x, vitattn_strides sx, const void* residual, vitattn_strides sr, const void* w,
                         void* h, vitattn_strides sh, void* y, vitattn_strides sy, float* rstd, int B, int H, int N,
                         int D, float eps, int type, int residual_type, int weight_type,
                         const vitattn_dropout_spec* dropout, void* stream);
size_t vitattn_rms_norm_bwd_workspace_bytes(int B, int H, int N, int D, int type);
int vitattn_rms_norm_bwd(const void* h, vitattn_strides sh, const void* w, const float* rstd, const void* dy,
                         vitattn_strides sdy, const void* dh, vitattn_strides sdh, void* dx, vitattn_strides sdx,
                         void* dres, vitattn_strides sdres, void* dw, int B, int H, int N, int D, int type,
                         int residual_type, int weight_type, const vitattn_dropout_spec* dropout, void* workspace,
                         size_t workspace_bytes, void* stream);

/*
 * The same norm with an output in 8 bits for a product that takes them: y holds e4m3
 * bytes (OCP, no infinities, largest 448) at element strides of one byte, and
 *
 *     scale = max(max |y| / 448, 2^-126),  byte = y / scale rounded to the nearest even
 *
 * with the largest magnitude of the fp32 y over the row (group 0; scale [B*H*N]) or over
 * each `group` of columns (32, 64 or 128; scale [B*H*N][ceil(D / group)]), dense. The quotient
 * of the fp32 y and the scale is rounded once. NaN stays NaN and does not count for a scale. Other groups: VITATTN_E_UNSUPPORTED.
 */
int vitattn_rms_norm_fp8(const void* x, vitattn_strides sx, const void* residual, vitattn_strides sr, const void* w,
                         void* h, vitattn_strides sh, void* y, vitattn_strides sy, float* scale, int group, int B,
                         int H, int N, int D, float eps, int type, int residual_type, int weight_type, void* stream);

/* types of the positions of vitattn_rotary */
enum vitattn_pos_type { VITATTN_POS_I32 = 0, VITATTN_POS_I64 = 1, VITATTN_POS_F32 = 2 };
#define VITATTN_ROTARY_INTERLEAVED 1 /* pair p is columns 2p and 2p + 1; else p and R + p */
#define VITATTN_ROTARY_INVERSE 2     /* turn by the opposite angles: the gradient */
#define VITATTN_ROTARY_JOINT 4       /* one run of frequencies over the pairs of all axes */
#define VITATTN_ROTARY_MAX_AXES 8
#define VITATTN_ROTARY_MAX_PAIRS 128

/*
 * Rotary positions with several axes (time, height, width): pair p of a row,
 * belonging to axis a, turns by the angle t f_p with t the row's position on
 * that axis. Axis a has sections[a] pairs (0 is allowed), in order; R = the sum
 * of all, and the columns from 2 R on are left as they are. Pair i of the n of
 * an axis has the frequency base^(-i/n); with VITATTN_ROTARY_JOINT pair p of
 * all R has base^(-p/R).
 *   q, k     : [B][Hq][N][d] and [B][Hk][N][d] (Hk = 0: no k), of `type`, at
 *              any element strides >= 0, the d elements of a row contiguous, no
 *              alignment beyond the element's.
 *   q_out, k_out: written, of the same type; they must not overlap themselves,
 *              nor each other (interleaved heads of one tensor do not).
 *              Each may be its input (the same strides); if both are, q and k
 *              may be interleaved heads of one tensor. Any other output whose
 *              address range meets an input's or the positions' is rejected.
 *   positions: [B or 1][N][n_axes] of pos_type at element strides pos_batch (0:
 *              shared by the samples), pos_row and pos_axis.
 *   d        : 2 R <= d <= 65,536; R <= 128, n_axes <= 8 (VITATTN_E_UNSUPPORTED
 *              above). B and Hq + Hk up to 65,535.
 * Angles are formed in fp64 (positions of 1e6 and more keep an fp32 sine),
 * products in fp32, rounded once. Bound by HBM bandwidth.
 */
int vitattn_rotary(const void* q, vitattn_strides sq, void* q_out, vitattn_strides sq_out, int Hq, const void* k,
                   vitattn_strides sk, void* k_out, vitattn_strides sk_out, int Hk, const void* positions,
                   long long pos_batch, long long pos_row, long long pos_axis, int pos_type, const int* sections,
                   int n_axes, double base, int B, int N, int d, int type, int flags, void* stream);

#define VITATTN_DIFF_MAX_D 80  /* head dim of q and k */
#define VITATTN_DIFF_MAX_E 160 /* head dim of v and o */

/*
 * Differential attention: each head takes the difference of two softmax maps
 * over the same values. q and k hold two maps per head, heads 2h and 2h + 1:
 *
 *     S_m = scale Q_m K_m^T,  P_m = softmax(S_m),  O_m = P_m V,  O = O_1 - lam_h O_2
 *
 * and the backward pass, given dO:
 *
 *     dP = dO V^T,  D_m,i = sum_c dO_ic O_m,ic,
 *     dS_1 = P_1 o (dP - D_1),  dS_2 = -lam_h P_2 o (dP - D_2),
 *     dQ_m = scale dS_m K_m,  dK_m = scale dS_m^T Q_m,  dV = (P_1 - lam_h P_2)^T dO,
 *     dlam_h = -sum over b, i of D_2,i.
 *
 *   q        : bf16 [B][2H][Nq][d];  k: bf16 [B][2H][Nk][d];  v: bf16 [B][H][Nk][e].
 *   lam      : [H], fp32 or bf16 (lam_type), contiguous.
 *   key_lens : null, or int32 [B]: sample b attends to its first key_lens[b]
 *              keys (brought into 0 .. Nk); the rest are not read. A sample
 *              without keys has O = 0, LSE = -inf and no gradients; so has a
 *              query whose scores are all -inf.
 *   o        : bf16 [B][H][Nq][e], written.
 *   maps     : fp32 [B][2H][Nq][e], dense: each map's output O_m, which the
 *              backward reads; lse: fp32 [B][2H][Nq], dense. Either may be null
 *              in the forward (inference). The maps are kept in fp32 since
 *              dP - D_m cancels to a small part where values share a mean.
 *   dq, dk, dv: bf16, the shapes of q, k and v, written (rows of keys past
 *              key_lens are zeros); dlam: [H] of lam_type, or null.
 *   d, e     : multiples of 8 up to VITATTN_DIFF_MAX_D and VITATTN_DIFF_MAX_E
 *              (e = 2 d is the usual choice), else VITATTN_E_UNSUPPORTED. The
 *              kernels compute in tiles of width (d, e) = (32, 64), (64, 64),
 *              (64, 128) or (96, 160), columns past d and e zero.
 *   strides  : as for vitattn_fwd_strided (2H heads for q, k, dq and dk), with
 *              (rows + 512) * row * 2 < 2^31.
 *   overlaps : an output (or the workspace) that shares memory with any other
 *              operand is rejected; interleaved views of one tensor do not.
 *   sizes    : B*H*(max(Nq, Nk) + 512) below 2^30.
 *   workspace: at least the bytes the matching function gives (the forward's is
 *              0 unless up to 256 queries meet many keys; then both passes split
 *              the keys over workgroups whose results are joined), 16-byte aligned.
 * Scores, statistics, sums and the difference are fp32; P and dS are rounded
 * to bf16 as operands of the matrix cores, o and the gradients once at the end. Results are
 * bitwise deterministic, and a head's results do not depend on the call it is
 * part of. No atomics.
 */
size_t vitattn_diff_fwd_workspace_bytes(int B, int H, int Nq, int Nk, int d, int e);
int vitattn_diff_fwd(const void* q, vitattn_strides sq, const void* k, vitattn_strides sk, const void* v,
                     vitattn_strides sv, const void* lam, int lam_type, const int* key_lens, void* o,
                     vitattn_strides so, float* maps, float* lse, int B, int H, int Nq, int Nk, int d, int e, float scale,
                     void* workspace, size_t workspace_bytes, void* stream);
size_t vitattn_diff_bwd_workspace_bytes(int B, int H, int Nq, int Nk, int d, int e);
int vitattn_diff_bwd(const void* q, vitattn_strides sq, const void* k, vitattn_strides sk, const void* v,
                     vitattn_strides sv, const void* lam, int lam_type, const int* key_lens, const float* maps,
                     const float* lse, const void* dout, vitattn_strides sdo, void* dq, vitattn_strides sdq, void* dk,
                     vitattn_strides sdk, void* dv, vitattn_strides sdv, void* dlam, int B, int H, int Nq, int Nk, int d,
                     int e, float scale, void* workspace, size_t workspace_bytes, void* stream);

#define VITATTN_SELECT_MAX 256          /* blocks that a group may choose */
#define VITATTN_SPARSE_MAX_TOPK 1024    /* listed blocks of a group that the attention takes */
#define VITATTN_SPARSE_MAX_BLOCK 1024   /* keys of a block */
#define VITATTN_SPARSE_MAX_BLOCKS 16384 /* blocks of a sample's keys */

/*
 * Attention over blocks of keys that a cheap score chooses. The Nk keys of a sample are
 * cut into nb = ceil(Nk / block) blocks of `block` keys, the Nq queries into groups of
 * q_block neighbours (1: each query by itself), and each group of each head attends to
 * topk blocks. The queries' H heads share the Hk heads of keys and values, H / Hk
 * neighbouring heads each.
 *
 * The means of the blocks' keys, in 8 bits: with m the mean of a block's keys (of the
 * sample's first key_lens[b]),
 *
 *     means = round(m (127 (1 / max|m|))),  scales = max|m| (1 / 127); -1 of a block without keys.
 *
 *   k       : bf16 [B][Hk][Nk][d]; strides as for vitattn_fwd_strided.
 *   key_lens: null, or int32 [B], brought into 0 .. Nk.
 *   means   : int8 [B][Hk][nb][P], dense, 16-byte aligned, P = d rounded up to a multiple of
 *             64, columns from d on zero; scales: fp32 [B][Hk][nb].
 *   block   : a multiple of 64 up to VITATTN_SPARSE_MAX_BLOCK, nb up to
 *             VITATTN_SPARSE_MAX_BLOCKS, d as for vitattn_fwd; else VITATTN_E_UNSUPPORTED.
 * Sums are fp64 (exact for values within 2^37 of each other), and so is each step of the
 * scaling; a mean that is not finite counts as 0. Bound by HBM bandwidth.
 */
int vitattn_block_means(const void* k, vitattn_strides sk, const int* key_lens, void* means, float* scales, int B,
                        int Hk, int Nk, int d, int block, void* stream);

/*
 * The choice: with x the mean of a group's queries and X = round(x (127 (1 / max|x|))), block
 * j has the score (X . means_j) scales_j, a whole number times an fp32 number, rounded
 * once. Written are the topk blocks of highest score in ascending order (of equal ones the
 * lowest), then -1 where there are fewer blocks with keys.
 *   q     : bf16 [B][H][Nq][d].
 *   blocks: int32 [B][H][ceil(Nq / q_block)][topk], dense.
 *   topk  : 1 .. VITATTN_SELECT_MAX, else VITATTN_E_UNSUPPORTED.
 *   sizes : B and H up to 65,535.
 */
int vitattn_block_select(const void* q, vitattn_strides sq, const void* means, const float* scales, int* blocks, int B,
                         int H, int Hk, int Nq, int d, int nb, int q_block, int topk, void* stream);

/*
 * The attention: row i of head h attends to the keys of the blocks blocks[b][h][i /
 * q_block][0 .. topk - 1] among the sample's first key_lens[b]:
 *
 *     S_ij = scale q_i . k_j,  LSE_i = log sum_j exp(S_ij),  P = exp(S - LSE),  O = P V
 *
 * and the backward as for vitattn_bwd, dK and dV summed over the heads that share them.
 * Numbers outside 0 .. nb - 1 stand for no block, a block given twice counts once, and the
 * order does not matter. A row without keys has O = 0, LSE = -inf and no gradients; so has a
 * row whose scores are all -inf, of finite q, k and v (sums that overflow). Where infinite
 * elements make scores -inf, O and LSE are those of the other keys, but gradients of the rows
 * and keys that hold the elements, and of those that attend to each other with them, may be
 * NaN. Keys that a row does not attend to do not reach it, also where they are not finite.
 *   q, o, dout, dq : bf16 [B][H][Nq][d]; k, v, dk, dv: bf16 [B][Hk][Nk][d]; strides as for
 *                    vitattn_fwd_strided, (rows + 1280) * row * 2 below 2^31.
 *   blocks         : int32, dense, from vitattn_block_select or any other choice.
 *   o32, lse       : fp32, dense, [B][H][Nq][d] and [B][H][Nq]: the unrounded output and LSE,
 *                    which the backward reads; either may be null in the forward.
 *   topk           : 1 .. VITATTN_SPARSE_MAX_TOPK; d, block and nb as above, H / Hk up to
 *                    2047; else VITATTN_E_UNSUPPORTED.
 *   sizes          : Nq up to 2^26, B*H*(Nq + 128) and B*Hk*nb*block below 2^30, B*H*(Nq + 4096)
 *                    below 2^32.
 *   workspace      : at least the bytes the matching function gives (0 if invalid; the
 *                    forward's is 0 unless up to 256 queries split their blocks over
 *                    workgroups), 16-byte aligned.
 *   overlaps       : an output (or the workspace) that shares memory with another operand
 *                    is rejected.
 * Fastest where q_block is a multiple of 64 (better 128): else 64 neighbouring rows go over
 * the union of what they chose. Scores, statistics and sums are fp32; P and dS are rounded to
 * bf16 as operands of the matrix cores, outputs once. Results are bitwise deterministic, and a
 * head's results do not depend on the call it is part of. Atomics count integers only.
 */
size_t vitattn_block_fwd_workspace_bytes(int B, int H, int Hk, int Nq, int Nk, int d, int block, int q_block, int topk);
int vitattn_block_fwd(const void* q, vitattn_strides sq, const void* k, vitattn_strides sk, const void* v,
                      vitattn_strides sv, const int* blocks, const int* key_lens, void* o, vitattn_strides so,
                      float* o32, float* lse, int B, int H, int Hk, int Nq, int Nk, int d, int block, int q_block,
                      int topk, float scale, void* workspace, size_t workspace_bytes, void* stream);
size_t vitattn_block_bwd_workspace_bytes(int B, int H, int Hk, int Nq, int Nk, int d, int block, int q_block, int topk);
int vitattn_block_bwd(const void* q, vitattn_strides sq, const void* k, vitattn_strides sk, const void* v,
                      vitattn_strides sv, const int* blocks, const int* key_lens, const float* o32, const float* lse,
                      const void* dout, vitattn_strides sdo, void* dq, vitattn_strides sdq, void* dk,
                      vitattn_strides sdk, void* dv, vitattn_strides sdv, int B, int H, int Hk, int Nq, int Nk, int d,
                      int block, int q_block, int topk, float scale, void* workspace, size_t workspace_bytes,
                      void* stream);

/* Human-readable name of a status code (static storage, never NULL). */
const char* vitattn_status_str(int status);

/* Library version string (static storage). */
const char* vitattn_version(void);

#ifdef __cplusplus
}
#endif

#endif /* VITATTN_H */
