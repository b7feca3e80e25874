/*
 * fibq.h -- C ABI of libfibq.so, the MI355X (gfx950) implementation of the
 * FibQuant random-access KV-cache codec (arXiv 2605.11478, "FibQuant:
 * Universal Vector Quantization for Random-Access KV-Cache Compression").
 *
 * Notation (Sec. 3.1): head dimension d, block dimension k (k | d), codebook
 * size N = 2^w, index width w = log2 N bits, rate b = w / k bits per
 * coordinate, shared orthogonal rotation Pi (d x d), shared codebook
 * C = {c_1..c_N} in the unit ball of R^k.
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * - Every function returns an int status (FIBQ_OK or a negative FIBQ_E*).
 *   Arguments are validated synchronously before anything is enqueued; on an
 *   error nothing is launched and no output is touched.  No C++ exception
 *   crosses the ABI and nothing aborts.
 * - (d, k, b, N) must satisfy: N a power of two with 1 <= w <= 16,
 *   |b * k - w| < 1e-9, 1 <= k <= d, d % k == 0.  Violations give
 *   FIBQ_EINVAL; valid shapes that have no kernel instantiation (see
 *   fibq_supported) give FIBQ_EUNSUPPORTED.
 * - Device entry points take device pointers (memory the caller allocated on
 *   the current HIP device and owns), enqueue their kernels on `stream`
 *   (a hipStream_t passed as void*, NULL = the default stream) and return
 *   without synchronising.  A launch failure is reported as FIBQ_EHIP.
 *   They allocate no device memory.
 * - Layouts are row-major and dense unless a stride argument says otherwise.
 * - The payload of one vector is P = ceil((d / k) * w / 8) bytes: a
 *   little-endian bit stream in which the index of block m occupies bits
 *   [m w, (m + 1) w) (byte j holds bits 8j .. 8j + 7, bit 0 least
 *   significant), trailing bits zero.  Indices are 0-based.  Vector v of a
 *   cache owns bytes [v P, (v + 1) P) of the payload array and element v of
 *   the norm array (IEEE binary16 bits): fixed rate, affine addresses
 *   (Sec. 3.1, Fig. 1 caption).
 * - The library keeps no global mutable state; concurrent calls on different
 *   streams are safe.
 */
#ifndef FIBQ_H
#define FIBQ_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define FIBQ_OK 0
#define FIBQ_EINVAL (-1)        /* bad shape, rate, pointer or argument      */
#define FIBQ_EUNSUPPORTED (-2)  /* valid, but no kernel for this shape        */
#define FIBQ_EHIP (-3)          /* HIP launch / runtime error                 */
#define FIBQ_EIO (-4)           /* codebook file missing, short or corrupt    */
#define FIBQ_EWORKSPACE (-5)    /* workspace missing or too small             */

#define FIBQ_F32 0
#define FIBQ_F16 1
#define FIBQ_BF16 2

/* Human-readable text for a status code (static storage, never NULL). */
const char* fibq_strerror(int status);

/* Library version as major * 10000 + minor * 100 + patch. */
int fibq_version(void);

/* Payload bytes per vector, P = ceil((d/k) * log2(N) / 8) (Sec. 3.1: the
 * fixed-rate (d log2 N)/k-bit payload).  Returns P > 0, or FIBQ_EINVAL for an
 * invalid (d, k, N) (N must be a power of two, 2 <= N <= 65536, k | d). */
int fibq_payload_bytes(int d, int k, int N);

/* FIBQ_OK if (d, k, N) has device kernels for encode, decode and attention,
 * FIBQ_EUNSUPPORTED if the shape is valid but not instantiated, FIBQ_EINVAL
 * if it is invalid.  Instantiated: d in {64, 128} with k in {1, 2, 4, 8, 16},
 * and d = 64 with the large-block codes k in {32, 64}; 2 <= N <= 16384 and
 * N k <= 2^20 (codebooks up to 4 MB; those above 64 KB are read from global
 * memory instead of LDS). */
int fibq_supported(int d, int k, int N);

/* ------------------------------------------------------------------ host --
 * Offline construction of the two shared objects.  Host memory only, no GPU
 * needed.  Random draws come from Philox4x32-10 normals (the stream is
 * defined in the design notes); results are deterministic for a seed and do
 * not depend on n_threads. */

/* Haar-random orthogonal rotation Pi (Sec. 3 overview, Fig. 1 caption: one
 * matrix shared by all layers, heads, tokens, K and V): Q of the QR
 * factorisation of a d x d standard-normal matrix with diag(R) > 0, computed
 * in float64 and rounded once to float.  R_out: host, d*d floats, row-major,
 * y_i = sum_j Pi[i*d + j] x_j.  1 <= d <= 1024, else FIBQ_EINVAL. */
int fibq_build_rotation(int d, uint64_t seed, float* R_out);

/* Radial-angular codebook (Sec. 3.3; App. A codebook-construction table):
 * Beta-quantile radii (Eq. radii_main; closed form Eq. radii_k2 at k = 2)
 * times quasi-uniform directions (planar Fibonacci spiral at k = 2,
 * Fibonacci sphere at k = 3, Roberts-Kronecker at k >= 4, +/-1 at k = 1),
 * then `restarts` Lloyd-Max runs of `iters` rounds on M samples of the
 * spherical-Beta source f_{d,k} (Lemma 1), each run starting from the
 * initial codebook rotated by its own Haar k x k matrix; the run with the
 * lowest training MSE is kept; its codewords are finally rounded to
 * binary16-representable values (round to nearest, ties to even), which the
 * fused attention kernel reads exactly from an fp16 table (the effect on the
 * distortion is below 1e-4 dB).  M <= 0 selects max(100000, 30 N).
 * n_threads <= 0 uses all hardware threads.
 * C_out: host, N*k floats (codeword n at n*k).  train_mse_out (nullable):
 * per-block training MSE of the kept codebook.
 * k = d is the full-vector code (Sec. 5, "why a full-vector code can win"):
 * the source is then the whole normalised vector and the same steps apply.
 * Same as fibq_build_codebook_init with init = FIBQ_INIT_BETA. */
int fibq_build_codebook(int d, int k, double b, int N, uint64_t seed, int64_t M,
                        int restarts, int iters, int n_threads, float* C_out,
                        double* train_mse_out);

/* Starting codebooks for the same Lloyd-Max polish.
 * FIBQ_INIT_BETA: N Beta-quantile shells, one direction each (Eq. radii_main).
 * FIBQ_INIT_SHELL: the large-d shortcut of App. D (App. A table, last row):
 *   every codeword at the typical radius sqrt(k/d).
 * FIBQ_INIT_MULTISHELL: C(S, M_a) of App. E Eq. multishell, S shells at the
 *   Beta quantiles (s - 1/2)/S, shell s holding directions s*M_a+1 .. (s+1)*M_a
 *   of the sequence above (at k = 3 the latitude bands restart per shell, the
 *   azimuth continues); every factor pair S * M_a = N is tried on the training
 *   sample and the one with the lowest training MSE starts the polish (ties:
 *   the smaller S).  Codewords are shell-major. */
#define FIBQ_INIT_BETA 0
#define FIBQ_INIT_SHELL 1
#define FIBQ_INIT_MULTISHELL 2

/* fibq_build_codebook with a choice of starting codebook (`init`, one of the
 * FIBQ_INIT_* values, else FIBQ_EINVAL).  `shells` > 0 fixes S for
 * FIBQ_INIT_MULTISHELL (it must divide N; e.g. S = sqrt(N) for
 * fibq_encode_radius_first); 0 searches all factor pairs; any other use is
 * FIBQ_EINVAL.  `metric` (host, k*k doubles, row-major; NULL for the squared
 * Euclidean error) replaces ||x - c||^2 by (x - c)^T M (x - c) throughout
 * the Lloyd-Max polish: the task-weighted / Mahalanobis objective of Sec. 3
 * (the discussion after Eq. lattn); the cell mean stays the optimal centroid,
 * the payload and decoder are unchanged.  M must be symmetric (to 1e-12 of
 * its largest entry) and positive definite, else FIBQ_EINVAL.  shells_out
 * (nullable) receives the number of radial shells of the starting codebook
 * (N, 1 or S). */
int fibq_build_codebook_init(int d, int k, double b, int N, uint64_t seed, int64_t M,
                             int restarts, int iters, int n_threads, int init, int shells,
                             const double* metric, float* C_out, double* train_mse_out,
                             int* shells_out);

/* Write / read the codebook file (C, Pi and the two seeds; little-endian;
 * magic "FIBQCB01", u32 d, k, N, 0, u64 seeds, f32 C, f32 Pi, u64 FNV-1a-64
 * of all preceding bytes).  fibq_load_codebook with C == NULL or R == NULL
 * only reports the shape (query mode); `seeds` (nullable) receives 2 values.
 * Errors: FIBQ_EIO (cannot open, short, bad magic or checksum),
 * FIBQ_EINVAL (NULL path / shape pointers). */
int fibq_save_codebook(const char* path, int d, int k, int N, const float* C,
                       const float* R, uint64_t rotation_seed,
                       uint64_t codebook_seed);
int fibq_load_codebook(const char* path, int* d, int* k, int* N, float* C,
                       float* R, uint64_t* seeds);

/* ---------------------------------------------------------------- device -- */

/* Encoder (Sec. 3.1, Eq. encode): for each of n_vec vectors x_v (row v of
 * `x`, d elements of `dtype`, rows x_row_stride elements apart,
 * x_row_stride >= d):
 *   nu = ||x_v||_2, stored as binary16 (round-to-nearest-even) in norms[v];
 *   y = Pi (x_v / nu) (unrounded nu), cut into d/k blocks y^(m);
 *   i_m = argmin_j ||y^(m) - c_j||^2 (ties: lowest index), packed into
 *   payload[v*P .. v*P + P).
 * An all-zero vector stores norm 0 and indices 0.  Norms above the binary16
 * range store +inf.  R: device, d*d floats (row-major, as built above).
 * C: device, N*k floats.  payload: device, n_vec*P bytes.  norms: device,
 * n_vec uint16.  n_vec == 0 is a no-op. */
int fibq_encode(const void* x, int dtype, int64_t n_vec, int64_t x_row_stride,
                int d, int k, double b, int N, const float* R, const float* C,
                uint8_t* payload, uint16_t* norms, void* stream);

/* Radius-first encoder (App. F, Stage 1), an approximate search for
 * multi-shell codebooks built with FIBQ_INIT_MULTISHELL and S = L shells
 * (C shell-major: shell l holds codewords l*N/L .. (l+1)*N/L - 1).  Block m
 * of y takes the shell l* whose radius r_l = sqrt(BetaInv((l + 1/2)/L; k/2,
 * beta_dk)) (Eq. multishell, the same radii as the builder) is nearest to
 * ||y^(m)||_2 (lower shell on ties) and stores l* N/L + the index of the
 * nearest codeword of that shell alone (ties: lowest index): O(L + N/L)
 * work per block instead of O(N).  Header, payload layout and the decoder
 * are those of fibq_encode; L = 1 is exactly fibq_encode's search.
 * L: a power of two dividing N, 1 <= L <= 256, else FIBQ_EINVAL.  Other
 * arguments, ownership and errors as fibq_encode. */
int fibq_encode_radius_first(const void* x, int dtype, int64_t n_vec, int64_t x_row_stride,
                             int d, int k, double b, int N, int L, const float* R,
                             const float* C, uint8_t* payload, uint16_t* norms, void* stream);

/* Stage 2 tables for fibq_encode_list (App. F, hierarchical direction code),
 * host side: for each of the L shells of the shell-major codebook C (host,
 * N*k floats), spherical k-means of the shell's codeword directions into K
 * parents, started from codewords 0, s, 2s, .. (s = (N/L)/K), `rounds`
 * rounds of assignment by the largest inner product (first parent on ties)
 * and mean-direction update (a parent that empties keeps its direction),
 * then a final assignment.  mu_out: L*K*k doubles (parent p of shell l at
 * (l*K + p)*k); offsets_out: L*(K+1) ints, members_out: N ints: parent p of
 * shell l owns members_out[l*N/L + offsets_out[l*(K+1) + p] ..
 * l*N/L + offsets_out[l*(K+1) + p + 1]), the shell-local indices of its
 * codewords in increasing order.  Requires L | N, 1 <= K <= min(N/L, 64),
 * rounds >= 0, non-NULL pointers; else FIBQ_EINVAL. */
int fibq_build_parent_lists(const float* C, int N, int k, int L, int K, int rounds,
                            double* mu_out, int32_t* offsets_out, int32_t* members_out);

/* List-decoding encoder (App. F, Stages 1 + 2 composed), approximate: the
 * shell is chosen as in fibq_encode_radius_first; the shell's K parents are
 * ranked by <y^(m), mu_p> (float64, first parent on ties) and the codewords
 * of the best T parents are searched (float32 screen, float64 re-score of
 * near ties; lowest index on ties); the index is l* N/L + the shell-local
 * index.  T = K searches the whole shell (the radius-first result).  mu,
 * offsets, members: device copies of fibq_build_parent_lists' outputs for
 * the same C, L and K (L*K*k doubles, L*(K+1) and N ints).  Offsets and
 * members are clamped into their shell on the device, so other table
 * contents cannot read out of bounds (they only give a different search).  d = 64 with k in {4, 8, 16, 32} or d = 128 with k in
 * {4, 8, 16} (else FIBQ_EUNSUPPORTED); 1 <= T <= min(K, 8); L as in
 * fibq_encode_radius_first.  Other arguments, ownership and errors as
 * fibq_encode. */
int fibq_encode_list(const void* x, int dtype, int64_t n_vec, int64_t x_row_stride, int d, int k,
                     double b, int N, int L, int K, int T, const double* mu,
                     const int32_t* offsets, const int32_t* members, const float* R,
                     const float* C, uint8_t* payload, uint16_t* norms, void* stream);

/* Random-access decoder (Sec. 3.1 decoder; Sec. 6 "table lookup followed by
 * inverse rotation"): x_hat_i = nu * Pi^T (c_{i_1}, ..., c_{i_{d/k}}) with nu
 * the stored binary16 norm.  Output row i (d floats of x_hat, device) is
 * the vector t = token_ids[i] of the cache (payload row t, norms[t]), or
 * t = i when token_ids is NULL.  payload/norms hold n_cache vectors;
 * token_ids (device, nullable) holds n_vec int64 ids.  An id outside
 * [0, n_cache) yields a row of NaNs (the kernel checks every id).  With
 * token_ids == NULL, n_vec <= n_cache is required.  x_hat must be 16-byte
 * aligned (rows are stored as float4).  Violations give FIBQ_EINVAL. */
int fibq_decode(const uint8_t* payload, const uint16_t* norms,
                const int64_t* token_ids, int64_t n_vec, int64_t n_cache,
                int d, int k, double b, int N, const float* R, const float* C,
                float* x_hat, void* stream);

/* Workspace bytes fibq_attn_decode needs for this problem (0 for an invalid
 * one).  The workspace holds the rotated queries, the per-block query-codeword
 * tables and the split-K partial softmax states. */
size_t fibq_attn_workspace_bytes(int64_t n_groups, int G, int64_t T, int d,
                                 int k, int N);

/* Fused dequantisation + single-query decode attention (Eq. lattn with K, V
 * replaced by the decoded cache; Sec. 3.1 decoder; random access makes the
 * fusion possible, Sec. 1 and App. F):
 *   for group g (a (layer, batch, kv-head) triple, flattened by the caller)
 *   and its G query heads h (GQA: q-head h of the group shares its K, V):
 *   o_{g,h} = sum_t softmax_t(scale * <q_{g,h}, K_hat_{g,t}>) V_hat_{g,t},
 *   t = 0 .. T-1, no mask.  scale <= 0 selects 1/sqrt(d).
 * Computed in rotated space: the query is rotated once (q~ = Pi q, so
 * <q, K_hat_t> = nu_t <q~, c_(t)>), scores are sums of per-block
 * query-codeword dot products, values are accumulated as
 * sum_t p_t nu_t c_(t) and rotated back once (Pi^T) per head.
 * q: device [n_groups][G][d] of q_dtype.  k_payload/v_payload: device
 * [n_groups][T_stride][P] bytes; k_norms/v_norms: device
 * [n_groups][T_stride] binary16 bits (T <= T_stride: only the first T
 * tokens of each group are read).  out: device [n_groups][G][d] float.
 * workspace: device, at least fibq_attn_workspace_bytes(...) bytes, else
 * FIBQ_EWORKSPACE.  T == 0 writes zeros.  1 <= G <= 16. */
int fibq_attn_decode(const void* q, int q_dtype, const uint8_t* k_payload,
                     const uint16_t* k_norms, const uint8_t* v_payload,
                     const uint16_t* v_norms, int64_t n_groups, int G,
                     int64_t T, int64_t T_stride, int d, int k, double b,
                     int N, const float* R, const float* C, float scale,
                     float* out, void* workspace, size_t workspace_bytes,
                     void* stream);

/* For callers that cannot allocate device memory (code under HIP graph
 * capture, serving loops or harnesses that forbid hipMalloc): the same
 * computation as fibq_attn_decode, with the same arguments, layouts, results
 * and errors, but without a workspace argument.  The workspace comes from a
 * static device array of FIBQ_ATTN_SCRATCH_BYTES bytes that the library owns:
 * one per GPU it runs on, held until the process ends, located on the first
 * call on each device.  The call allocates nothing (no hipMalloc / hipFree).
 * A problem whose fibq_attn_workspace_bytes exceeds FIBQ_ATTN_SCRATCH_BYTES
 * returns FIBQ_EWORKSPACE before anything is enqueued.  All calls on one GPU
 * share that GPU's array: calls that overlap in time on one GPU (different
 * streams or host threads without ordering) race and give wrong results;
 * calls ordered on one stream are safe. */
#define FIBQ_ATTN_SCRATCH_BYTES ((size_t)64 << 20)
int fibq_attn_decode_noalloc(const void* q, int q_dtype, const uint8_t* k_payload,
                             const uint16_t* k_norms, const uint8_t* v_payload,
                             const uint16_t* v_norms, int64_t n_groups, int G, int64_t T,
                             int64_t T_stride, int d, int k, double b, int N, const float* R,
                             const float* C, float scale, float* out, void* stream);

/* --------------------------------------------------------------- serving --
 * Operators of a serving loop on the compressed cache, for groups of different
 * lengths: a group g (layer, sequence, kv-head) holds lens[g] cached tokens
 * (device, int32) in rows 0 .. lens[g] - 1 of its T_stride rows.  Lengths live
 * on the device, so a captured call follows them.  Common limits (else
 * FIBQ_EINVAL): 0 <= n_groups <= 65535, T_stride < 2^30, fewer than 2^31
 * output elements.  Layouts, dtypes and the scale are those of
 * fibq_attn_decode.  Rows behind a group's last token may hold anything. */

/* Ancestor masks of a tree of M drafted tokens, host memory.  parents[i] is
 * the drafted token that token i follows, or -1 for one that follows the last
 * cached token; -1 <= parents[i] < i (parents come first), 1 <= M <= 64, else
 * FIBQ_EINVAL.  masks_out[i] gets bit i and the bits of i's ancestors. */
int fibq_tree_masks(const int32_t* parents, int M, uint64_t* masks_out);

/* Workspace bytes of fibq_attn_tree (0 for an invalid problem). */
size_t fibq_attn_tree_workspace_bytes(int64_t n_groups, int M, int G, int d, int k, int N);

/* Attention of a tree of drafted tokens over the compressed cache (the
 * verification step of speculative decoding; Eq. lattn with a mask, over the
 * decoded cache).  The M drafted tokens' keys and values have been encoded
 * into rows lens[g] .. lens[g] + M - 1 of their group, so an accepted token
 * has seen exactly the rows that decoding it by itself would have read:
 *   o_{g,i,h} = sum_{t in A} softmax_{t in A}(scale <q_{g,i,h}, K_hat_{g,t}>) V_hat_{g,t},
 *   A = {t < lens[g]} and {lens[g] + j : bit j of the mask of (g, i)}.
 * q: device [n_groups][M][G][d] of q_dtype; out: device, the same shape, float.
 * masks: device uint64 (bits from M on are ignored); the mask of (g, i) is
 * masks[g * mask_stride + i], mask_stride 0 (one tree for all groups) or >= M.
 * A row that sees no token gives zeros.  The rows of a group whose length is
 * outside [0, T_stride - M] are NaN, and nothing of its cache is read.
 * 1 <= M <= 64, 1 <= G <= 16.  M = 1 with mask 1 is single-query attention
 * over lens[g] + 1 tokens.  workspace: device, at least
 * fibq_attn_tree_workspace_bytes(...) bytes, 256-byte aligned, else
 * FIBQ_EWORKSPACE; calls that overlap in time need one each. */
int fibq_attn_tree(const void* q, int q_dtype, const uint8_t* k_payload,
                   const uint16_t* k_norms, const uint8_t* v_payload, const uint16_t* v_norms,
                   const int32_t* lens, const uint64_t* masks, int64_t mask_stride,
                   int64_t n_groups, int M, int G, int64_t T_stride, int d, int k, double b, int N,
                   const float* R, const float* C, float scale, float* out, void* workspace,
                   size_t workspace_bytes, void* stream);

/* Acceptance of a drafted path, in place: row lens[g] + i of K and V (payload
 * and norm) becomes row lens[g] + path[g * path_len + i] for i < n_acc[g] (all
 * are read before any is written), and new_lens[g] = lens[g] + n_acc[g].
 * new_lens may be lens, and overlaps no input otherwise.  P: payload bytes of a row (fibq_payload_bytes),
 * 1 <= P <= 256; 1 <= M <= 64 drafted tokens, 1 <= path_len <= 64.  A group
 * with a length outside [0, T_stride - M], a count outside
 * [0, min(path_len, M)] or a path entry (of the first n_acc[g]) outside [0, M)
 * keeps its rows and gets new_lens[g] = -1, which every operator of this
 * section treats as a bad length. */
int fibq_accept_draft(uint8_t* k_payload, uint16_t* k_norms, uint8_t* v_payload,
                      uint16_t* v_norms, const int32_t* lens, int64_t n_groups, int64_t T_stride,
                      int P, int M, const int32_t* path, int path_len, const int32_t* n_acc,
                      int32_t* new_lens, void* stream);

/* Workspace bytes of fibq_attn_decode_accum (0 for an invalid problem). */
size_t fibq_attn_decode_accum_workspace_bytes(int64_t n_groups, int G, int d, int k, int N);

/* fibq_attn_decode over groups of different lengths that also accumulates
 * every token's attention weight:
 *   out as fibq_attn_decode with T = lens[g];
 *   acc[g * T_stride + t] += sum_h softmax_t(scale <q_{g,h}, K_hat_{g,t}>), t < lens[g].
 * acc: device float [n_groups][T_stride], in place; elements from lens[g] on
 * are left as they are.  Each token's sum is taken in a fixed order (no
 * atomics).  lens[g] = 0 gives zeros; a length outside [0, T_stride] gives NaN
 * rows and leaves the group's acc.  workspace as in fibq_attn_tree. */
int fibq_attn_decode_accum(const void* q, int q_dtype, const uint8_t* k_payload,
                           const uint16_t* k_norms, const uint8_t* v_payload,
                           const uint16_t* v_norms, const int32_t* lens, float* acc,
                           int64_t n_groups, int G, int64_t T_stride, int d, int k, double b,
                           int N, const float* R, const float* C, float scale, float* out,
                           void* workspace, size_t workspace_bytes, void* stream);

/* Workspace bytes of fibq_evict (0 if it needs none). */
size_t fibq_evict_workspace_bytes(int64_t n_groups, int64_t T_stride);

/* Eviction by accumulated attention weight, into another cache.  A group of
 * lens[g] <= keep tokens keeps them all; a longer one keeps its last `recent`
 * tokens and, of the others, the keep - recent with the largest acc (equal
 * ones: lowest index first; NaN ranks below everything).  Kept tokens stay in
 * order: row i of the new cache is row index[g * keep + i] of the old one.
 * Payloads [n_groups][T_stride][P], norms and acc [n_groups][T_stride] are
 * copied to the *_out arrays of T_out >= keep rows per group; new_lens[g] is
 * the number kept, index (device int32 [n_groups][keep]) is -1 behind it, and
 * rows of the new cache behind it are left as they are.  A length outside
 * [0, T_stride] gives new_lens[g] = -1, an index of -1 and no rows.  lens and
 * acc must stay as they are until the call has run: it reads them more than
 * once (else nothing is accessed out of range, but what is kept is open).
 * 1 <= keep < 2^30, 0 <= recent <= keep, 1 <= P <= 256.  No output may overlap
 * an input or another output (FIBQ_EINVAL for the same address).  workspace: device, at least
 * fibq_evict_workspace_bytes(...) bytes, 256-byte aligned, else
 * FIBQ_EWORKSPACE. */
int fibq_evict(const uint8_t* k_payload, const uint16_t* k_norms, const uint8_t* v_payload,
               const uint16_t* v_norms, const float* acc, const int32_t* lens, int64_t n_groups,
               int64_t T_stride, int P, int64_t keep, int64_t recent, int64_t T_out,
               uint8_t* k_payload_out, uint16_t* k_norms_out, uint8_t* v_payload_out,
               uint16_t* v_norms_out, float* acc_out, int32_t* new_lens, int32_t* index,
               void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------- paged 8-bit cache --
 * Keys and values in 8 bits with one scale per page and head, for layers that
 * are not coded, with the block tables, the rotary positions and the attention
 * of a serving loop.  A page holds `page` tokens of one sequence;
 * sequence g's token t is row t % page of page table[g][t / page].
 * k_pages, v_pages: device [n_pages][H][page][d] bytes, 16-byte aligned, of
 * codes FIBQ_INT8 (-127 .. 127) or FIBQ_E4M3 (1-4-3 floating point, largest 448,
 * no infinities); k_scales, v_scales: device float [n_pages][H]; an element is
 * code x scale.  H key/value heads, G query heads on each (query head h uses
 * head h / G).  Lengths and tables live on the device (int32), so a captured
 * call follows them.  Common limits (else FIBQ_EINVAL): 0 <= n_seqs <= 65535,
 * 0 <= n_rows and fewer than 2^31 elements in a matrix of rows, page in
 * {16, 32, 64, 128}, max_pages * page < 2^30, 1 <= H <= 1024,
 * 1 <= n_pages < 2^31; d in {64, 128, 256} (else FIBQ_EUNSUPPORTED).  Rows are
 * those of all sequences, one sequence behind the other: sequence g has rows
 * starts[g] .. starts[g + 1] - 1. */
#define FIBQ_INT8 0
#define FIBQ_E4M3 1

#define FIBQ_ROPE_HALF 0        /* pair i: elements i and i + rot / 2 */
#define FIBQ_ROPE_INTERLEAVED 1 /* pair i: elements 2 i and 2 i + 1   */

/* Rotary positions: in every head of row r of q and k, pair i (x0, x1) of the
 * first `rot` elements becomes
 *   scale (x0 cos a - x1 sin a), scale (x1 cos a + x0 sin a),
 *   a = positions[r] freqs[i]  (inverse != 0: -a),
 * and the elements from rot on are copied.  The inverse with the same scale is
 * the gradient.  Angles are reduced in double; products and sums are float, and
 * the result is rounded once to dtype.  q: device, element e of head h of row r
 * at r * q_row_stride + h * q_head_stride + e, q_heads heads; k likewise, or
 * k_heads = 0.  Outputs likewise; an output may be its input (the same address
 * and strides) and has no memory in common with any other tensor.  positions:
 * device int32 [n_rows], any value; freqs: device double [rot / 2], radians per
 * position.  d even, 2 <= d <= 512, rot even, 2 <= rot <= d; heads in all at
 * most 2048; at most 2^25 rows. */
int fibq_rope(const void* q, const void* k, int dtype, int64_t n_rows, int q_heads, int k_heads,
              int d, int64_t q_row_stride, int64_t q_head_stride, int64_t k_row_stride,
              int64_t k_head_stride, const int32_t* positions, const double* freqs, int rot,
              int layout, float scale, int inverse, void* q_out, void* k_out,
              int64_t q_out_row_stride, int64_t q_out_head_stride, int64_t k_out_row_stride,
              int64_t k_out_head_stride, void* stream);

/* Workspace bytes of fibq_page_resize. */
size_t fibq_page_resize_workspace_bytes(int64_t n_seqs);

/* Block tables and slot maps from request lengths.  Request g holds lens[g]
 * tokens and gets grow[g] new ones, or gives -grow[g] of its last ones back.
 * Its tokens' pages are table[g * max_pages ..].  free_pages (device int32, room
 * for free_cap) is a stack of page ids, *n_free of them free.  In this order:
 *   starts[g] = the positive grow of the requests before g, summed (clipped to
 *     n_rows); starts has n_seqs + 1 entries;
 *   pages that a request needs no more go onto the stack (requests and pages in
 *     order; those behind free_cap are lost);
 *   pages for new tokens are taken from its top, first come, first served: a
 *     request whose pages, with those of all before it, are more than the stack
 *     holds gets none and is refused (one that needs no page never is);
 *   new_lens[g] = lens[g] + grow[g], or -1 for a refused request, for one whose
 *     old or new length is outside [0, max_pages * page], and for one whose rows
 *     end behind n_rows; such a request's table stays as it is;
 *   row r of request g, its i-th, gets position positions[r] = lens[g] + i and
 *     slot slots[r] = table[g][position / page] * page + position % page; rows of
 *     a request with new_lens -1 and rows behind the last get -1 and -1, and a
 *     page id outside [0, n_pages) gives slot -1;
 *   *new_free = the pages that are left.
 * A slot is a row of a cache of n_pages * page rows; fibq_decode takes slots as
 * token_ids.  new_lens may be lens, and new_free n_free; outputs overlap nothing
 * otherwise.  A refused request still holds lens[g] tokens and their pages: only
 * lens says so, so where requests may be refused new_lens is another tensor, and
 * lens takes the entries that are not -1 (in place the length is lost, and the
 * request's pages with it).  lens, grow, table and free_pages are not written by others while
 * the call runs.  1 <= page <= 65536 here; free_cap < 2^30, n_rows < 2^31. */
int fibq_page_resize(int32_t* table, const int32_t* lens, const int32_t* grow, int64_t n_seqs,
                     int64_t max_pages, int page, int64_t n_pages, int32_t* free_pages,
                     int64_t free_cap, const int32_t* n_free, int64_t n_rows, int32_t* new_lens,
                     int32_t* starts, int64_t* slots, int32_t* positions, int32_t* new_free,
                     void* workspace, size_t workspace_bytes, void* stream);

/* Writes rows of keys and values into the pages at their slots (-1 or any other
 * slot outside the pool: the row is left out).  A page and head's scale is the
 * least power of two, from 2^-126 on, that takes the largest magnitude written
 * since the page was begun (its first row written) to the codes' range; where it
 * grows, the rows before are rounded again to the new scale:
 *   s = max(s_old, least), code = round(x / s), code' = round(code s_old / s),
 * ties to even; s = 0 for a page of zeros.  s_old need not be a power of two.
 * An infinity or NaN among a head's new elements of a page makes its scale NaN
 * (until the page is begun again) and its new codes 0: rows that read the page
 * give NaN.  The rows of one page follow each other in the call at increasing
 * slots, and no page is written from two places of a call (else its contents are
 * open; nothing is accessed out of range).  k, v: element e of head h of row r at
 * r * row_stride + h * head_stride + e.  No memory is shared with the pages. */
int fibq_cache8_write(const void* k, const void* v, int dtype, int64_t n_rows,
                      int64_t k_row_stride, int64_t k_head_stride, int64_t v_row_stride,
                      int64_t v_head_stride, const int64_t* slots, int H, int d, int page,
                      int64_t n_pages, int codes, void* k_pages, float* k_scales, void* v_pages,
                      float* v_scales, void* stream);

/* Workspace bytes of fibq_attn_cache8 (0 for an invalid problem, or if it needs none). */
size_t fibq_attn_cache8_workspace_bytes(int64_t n_seqs, int64_t n_rows, int H, int G,
                                        int64_t max_pages, int page, int d);

/* Attention over the paged cache: for row i of the M rows of sequence g and query
 * head h,
 *   o = sum_t softmax_t(scale <q, K_t>) V_t over t < lens[g] - M + i + 1 if causal
 *   (the rows are the sequence's last M tokens), else over t < lens[g] (cross
 *   attention to states of another length).
 * scale <= 0 selects 1/sqrt(d).  q: device [n_rows][H * G][d] of q_dtype; out:
 * device float of the same shape.  table: device int32 [n_seqs][max_pages]; starts: device
 * int32 [n_seqs + 1], or NULL for one row per sequence (n_rows = n_seqs).  A row
 * that sees no token gives zeros; rows of a sequence whose length is outside
 * [0, max_pages * page], or less than its rows if causal, are NaN and nothing of
 * its cache is read.  A page id outside [0, n_pages) makes the rows that see its
 * tokens NaN.  Rows that belong to no sequence are left as they are; a sequence
 * whose starts are not 0 <= starts[g] <= starts[g + 1] <= n_rows has none, and rows
 * that two sequences claim are open.  What
 * lies behind a sequence's last token is never used, whatever it holds.  A score's
 * factors (scale, K scale, the row's power of two) are limited to 2^94 in magnitude, so
 * that finite queries and elements give finite rows; a row of queries that holds a NaN
 * or an infinity is NaN, and so are rows that see a page whose scale (times `scale`, for
 * K) is no finite number.  Codes 0x7f and 0xff of E4M3 (NaN) among a sequence's tokens
 * make the rows of that sequence open.  lens, starts and table are not written while the
 * call runs (else nothing is accessed out of range, but rows are open).
 * 1 <= G <= 16.  workspace: device, at least
 * fibq_attn_cache8_workspace_bytes(...) bytes, 256-byte aligned, else
 * FIBQ_EWORKSPACE; calls that overlap in time need one each. */
int fibq_attn_cache8(const void* q, int q_dtype, const void* k_pages, const float* k_scales,
                     const void* v_pages, const float* v_scales, int codes, const int32_t* table,
                     const int32_t* lens, const int32_t* starts, int64_t n_seqs, int64_t n_rows,
                     int H, int G, int64_t max_pages, int page, int64_t n_pages, int d,
                     int causal, float scale, float* out, void* workspace,
                     size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* FIBQ_H */
