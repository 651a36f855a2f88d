/*
 * cryptogen_requests.h -- what a model has learned, brought to the encrypted tokens of many requests
 * (libcryptogen_requests.so, beside the evaluator of cryptogen.h).
 *
 * The evaluator takes plaintexts that somebody has encoded, one token of one request at a time, and one
 * token index for all caches.  Here slot values are encoded on the GPU, projection matrices and low-rank
 * adapters become the diagonals a projection reads, the tokens of many requests go through a layer's
 * matrices in one call, each with the adapter it asks for, a learned position bias is added to scores, and
 * every request's rows are appended at its own length.  Positions, lengths and choices of adapters are read
 * on the GPU when the call runs, so that a captured call serves the next token by a replay.
 *
 * Conventions are those of cryptogen.h (device buffers of the caller, 16-byte aligned; canonical residues;
 * errors; outputs must not overlap inputs unless stated), with these additions:
 *   integers    int64 plaintext values are any representatives modulo t; slot s of a plaintext is its value at
 *               zeta^e, e = 3^i for s = i < N/2 and -3^i for s = N/2 + i (mod 2N), zeta the smallest
 *               primitive 2N-th root of unity modulo t.
 *   int32       arrays of one entry per request or bucket need only 4-byte alignment.
 *   device      every call needs the handle's device to be the current one (CG_EINVAL otherwise; for create it
 *               is the context's, and destroy waits for the current one).
 *   threads     a handle holds constant tables only: calls may run at once, with workspaces of their own.
 *   capture     every call but create and destroy can be captured.
 */
#ifndef CRYPTOGEN_REQUESTS_H
#define CRYPTOGEN_REQUESTS_H

#include "cryptogen.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct cg_req cg_req;

/* Tables for a context and the parameters it was created with (both stay the caller's; the context must
 * outlive the handle; others than the context's, or another current device than its own, are CG_EINVAL).  t must
 * be a prime with t = 1 mod 2N: only such a modulus has N slots (CG_EINVAL otherwise).  Synchronises the device,
 * as does cg_req_destroy. */
int cg_req_create(cg_req **out, cg_ctx *ctx, const cg_params *prm);
int cg_req_destroy(cg_req *req);

/* Plaintexts from their slot values, int64[batch][N]: the polynomials with coefficients in [0,t)
 * (uint64[batch][N], what cg_add_plain and cg_plain_prepare take), or their prepared form (what
 * cg_plain_prepare makes of them).  1 <= batch <= 65536. */
int cg_slots_encode(cg_req *req, void *stream, const int64_t *slots_dev, uint64_t *pt_dev, uint32_t batch);
int cg_slots_prepare(cg_req *req, void *stream, const int64_t *slots_dev, void *plain_dev, uint32_t batch);

/* The diagonals that cg_cpvm, cg_cpvm_hoisted and cg_cpvm_requests read, of
 *   M_u = W_u + A_(u / a_group) B_u   modulo t,   u < units:
 * w_dev int64[units][d1][d2] or NULL (no W), a_dev int64[ceil(units / a_group)][d1][rank] and b_dev
 * int64[units][rank][d2] or both NULL with rank = 0 (no low-rank part); not all of them NULL.  Layout as
 * at cg_cpvm: tiles of D1 = the power of two >= max(d1, d2, N/d2), at most N/2; n_diag = d2 D1 / N,
 * at most 64.  d2 a power of two, 2 <= d2 <= N/4; rank <= 4096.  diags_dev: prepared plaintexts
 * [units][n_diag].  units n_diag <= 65536.
 * ws_dev: cg_cpvm_prepare_workspace_bytes(...) bytes (where that is 0 ws_dev may be NULL). */
uint32_t cg_cpvm_diagonals(const cg_req *req, uint32_t d1, uint32_t d2);    /* n_diag; 0: sizes out of range */
size_t cg_cpvm_prepare_workspace_bytes(const cg_req *req, uint32_t units, uint32_t d1, uint32_t d2, uint32_t rank);
int cg_cpvm_prepare(cg_req *req, void *stream, const int64_t *w_dev, const int64_t *a_dev, const int64_t *b_dev,
                    uint32_t units, uint32_t a_group, uint32_t d1, uint32_t d2, uint32_t rank, void *diags_dev,
                    void *ws_dev);

/* The tokens of several requests times the same matrices, each with an adapter's added:
 *   y[r][u] = x_r (W_u + D_(pick[r], u)),   r < requests, u < units
 * as cg_cpvm_hoisted computes it (copies x_(r,c) = rotate_hoisted(x_r, 3^c), c < n_diag; the sum over c
 * of x_(r,c) times the prepared diagonals, here diags[u][c] + adapters[pick[r]][u][c]; then the sum over
 * residue classes modulo d2, block_round_bits and keys as there).  x_dev: one ciphertext per request in
 * that call's layout; diags_dev: prepared plaintexts [units][n_diag]; adapters_dev: prepared plaintexts
 * [n_adapters][units][n_diag] (of A B alone, from cg_cpvm_prepare without W) or NULL with n_adapters = 0;
 * pick_dev: int32[requests], read when the call runs: any value outside [0, n_adapters) means no adapter
 * (may be NULL when n_adapters is 0).  out_dev: [requests][units] ciphertexts.  Without an adapter the
 * results are those of cg_cpvm_hoisted for each request.  requests units <= 65536, requests n_diag
 * <= 65536.  ws_dev: cg_cpvm_requests_workspace_bytes(...) bytes. */
size_t cg_cpvm_requests_workspace_bytes(const cg_req *req, uint32_t requests, uint32_t units, uint32_t n_diag);
int cg_cpvm_requests(cg_req *req, void *stream, const uint64_t *x_dev, const void *diags_dev,
                     const void *adapters_dev, uint32_t n_adapters, const int32_t *pick_dev, uint32_t requests,
                     uint32_t units, uint32_t n_diag, uint32_t d2, uint32_t block_round_bits,
                     const void *const *gk_copies_dev_host, const void *const *gk_block_dev_host,
                     uint64_t *out_dev, void *ws_dev);

/* A learned relative position bias by buckets.  bucket(dist) = the last n with edges[n] <= dist (edges_dev:
 * int32[n_buckets] ascending, the distance at which each bucket begins); table_dev: int64[n_buckets][heads].
 * A distance below 0 (a later token) or below edges[0] gets no bias.
 *
 * cg_score_bias adds it to the scores of one new token per request (cg_decode_scores of requests * heads
 * heads), scores_dev [requests][heads][n_cts]: with j = c N/d2 + b,
 *   out[r][h][c] = scores + floor(Q/t) encode(slot b d2: table[bucket(pos[r] - j)][h], all others 0),
 * pos_dev int32[requests] being the new tokens' indices, read when the call runs (below 0: nothing is added).
 *
 * cg_prompt_bias adds it to the m = N/d2 diagonals of cg_prefill_qk, diags_dev [prompts][heads][m]: slot
 * i d2 of unit sigma H + r gets the bias of dist = i - j, j the key token that this diagonal holds for query i
 * ((row(i) xor sigma) H + (i + r) mod H, H = m/2, row(i) = i / H).
 *
 * out_dev may be the input (component 0 is then rewritten, component 1 not touched) and must not overlap it
 * otherwise.  d2 a power of two, 2 <= d2 <= N/4; requests heads n_cts <= 65536 (prompts heads m likewise);
 * 1 <= n_buckets <= 4096. */
int cg_score_bias(cg_req *req, void *stream, const uint64_t *scores_dev, uint32_t requests, uint32_t heads,
                  uint32_t n_cts, uint32_t d2, const int32_t *pos_dev, const int64_t *table_dev,
                  const int32_t *edges_dev, uint32_t n_buckets, uint64_t *out_dev);
int cg_prompt_bias(cg_req *req, void *stream, const uint64_t *diags_dev, uint32_t prompts, uint32_t heads,
                   uint32_t d2, const int64_t *table_dev, const int32_t *edges_dev, uint32_t n_buckets,
                   uint64_t *out_dev);

/* cg_kv_append of many requests at their own lengths: for r < requests and each of its caches c < per,
 *   cache[r][c][len / B] <- cache[r][c][len / B] + rows[r][c] * masks[len mod B],   len = lens[r], B = N/d2,
 * a ciphertext that receives its first token (len mod B = 0) being opened as there.  cache_dev: [requests][per]
 * [cache_stride_cts] ciphertexts; rows_dev: request r's `per` new rows at ciphertext r * row_stride_cts
 * (>= per); masks_dev as for cg_kv_append; lens_dev int32[requests], read when the call runs: a request with
 * len < 0 or a full cache (len >= B cache_stride_cts) is left as it is.  requests per <= 65536.
 * d2 a power of two, 1 <= d2 <= N/2. */
int cg_kv_append_requests(cg_req *req, void *stream, uint64_t *cache_dev, uint32_t cache_stride_cts,
                          uint32_t requests, uint32_t per, const int32_t *lens_dev, const uint64_t *rows_dev,
                          uint32_t row_stride_cts, const void *masks_dev, uint32_t d2);

#ifdef __cplusplus
}
#endif
#endif /* CRYPTOGEN_REQUESTS_H */
