/*
 * dipaco_kernels.h - kernel-level entry points of libdipaco.so.
 *
 * Most expose single kernels of the path step (Algorithm 1 inner loop of arXiv 2403.10616: the pieces of
 * f(x, theta_i) and its gradient) so that each can be checked against its plain definition and timed against
 * its own roofline.  Attention with a window and over a paged cache, and a step of drafted decoding over that cache, stand beside them
 * for programs that score or continue text piece by piece; no step calls them.  They follow the conventions of dipaco.h: caller-owned device pointers, 16-byte aligned,
 * work enqueued on `stream`, non-zero status = nothing enqueued.  dtype is a dipaco_dtype: the element type of
 * every `void*` operand (fp32 or bf16); accumulation is always fp32.
 */
#ifndef DIPACO_KERNELS_H
#define DIPACO_KERNELS_H

#include "dipaco.h"

#ifdef __cplusplus
extern "C" {
#endif

/* C[M,N] = opA(A) . opB(B) on the matrix cores.
 *   trans_a = 0: A is [M,K] row-major; 1: A is [K,M] row-major.   trans_b = 0: B is [K,N]; 1: B is [N,K].
 *   Supported: (0,0) forward, (0,1) input gradient, (1,0) with out_f32 = 1 weight gradient.
 * Epilogue in this order, each optional: + bias[N];  act = 1: aux_out[M,N] = value, value = GELU(value);
 * act = 2: value *= GELU'(aux_in[M,N]);  act = 3: aux_out[M,N] = GELU'(value), value = GELU(value);
 * act = 4: value *= aux_in[M,N];  + resid[M,N].  out_f32 = 1: C is fp32, else dtype.
 * splits > 1 (needs out_f32, no epilogue): K is cut into ranges whose partial products are written to
 * partial ([splits, M, N] fp32) and summed in index order.  The contiguous extent of each operand must be a
 * multiple of 16 bytes and N a multiple of 8. */
dipaco_status dipaco_k_gemm(int32_t dtype, int32_t trans_a, int32_t trans_b, int32_t out_f32, int32_t M, int32_t N,
                            int32_t K, const void* A, const void* B, void* C, const void* bias, const void* resid,
                            void* aux_out, const void* aux_in, int32_t act, int32_t splits, float* partial,
                            void* stream);

/* dipaco_k_gemm without split-K that also returns colsum_out[n] (device fp32 [N]) = sum over m of the values written
 * to C[m, n] (after the epilogue, before rounding to C's type), added in a fixed order: the bias gradient of a linear
 * layer when C is its output gradient.  colsum_scratch: device fp32, at least ceil(M / 32) * N elements. */
dipaco_status dipaco_k_gemm_colsum(int32_t dtype, int32_t trans_a, int32_t trans_b, int32_t M, int32_t N, int32_t K,
                                   const void* A, const void* B, void* C, const void* bias, const void* resid,
                                   void* aux_out, const void* aux_in, int32_t act, float* colsum_out,
                                   float* colsum_scratch, void* stream);

/* Force the GEMM workgroup tile for every later call in this process: 0 = automatic (default), 1 / 2 / 3 / 4 / 14 = the
 * kernel for every type, layout and size with its 32x64 / 64x128 / 96x128 / 128x128 / 160x128 tile (fp32 and weight
 * gradients: the nearest built one), 5 = the bf16 kernel with 256x256 tiles, for every shape it takes (K a multiple of
 * 32, 16-byte rows; other shapes and fp32 keep the automatic choice), 6 / 7 = the same kernel with its 256x256 / 256x128 tile forced,
 * 8 / 9 = the same with 128x512 / 512x128 tiles for weight gradients (fp32 output) and 256x256 for the rest,
 * 10 = the same with tile columns every 224 wherever N is a multiple of 224 (bf16 output), 11 = its eight-wave 256x256
 * tile with K tiles of 64 in a ring of two (K a multiple of 64, no split-K), 12 / 13 = the 256x256 tile computed with
 * 16x16x32 matrix-core instructions, K tiles of 32 in a ring of four / of 64 in a ring of two.
 * For tests (every tile shape must give the same parity) and tuning: a process-wide switch, not a per-call setting. */
dipaco_status dipaco_k_set_gemm_tile(int32_t tile);

/* Host-only (no GPU needed): the uneven split-K plan that the weight gradient C[M, N] = X^T dY with K = tokens is
 * launched with when at most max_slices K slices are allowed (dipaco_k_gemm with trans_a = 1, out_f32 = 1, bf16).
 * out (host int32 [12]): tile height and width of the shape taken (0, 0 when there is no such plan and the launch
 * cuts K into equal slices); tile rows / columns of the class of tiles inside C; tiles per class; K slices per class.
 * Classes: inside C, over its last rows, over its last columns, over both.  One workgroup per (tile, slice): their
 * total never exceeds the 256 compute units. */
dipaco_status dipaco_k_gemm_split_plan(int32_t M, int32_t N, int32_t K, int32_t max_slices, int32_t* out);

/* Host-only: how a bf16 step takes the gradients of a linear layer of k_in x n_out weights over `tokens` tokens, dW = X^T dY (in at most
 * max_slices K slices) and dX = dY W^T.  out (host int32 [4]): rows of dX's tile where both are one launch, 0 where they are
 * two; 1 if dW's tiles come first in it; K of the longest chain of sums in dW in one launch (0: two launches), and in two: the first never exceeds
 * the second.  k_in, n_out: multiples of 8. */
dipaco_status dipaco_k_gemm_pair_plan(int32_t tokens, int32_t k_in, int32_t n_out, int32_t max_slices, int32_t* out);

/* How the bf16 attention kernels deal the blocks of the causal triangle to workgroups, for every later call in this
 * process (tuning and tests): 0 = a long and a short block per workgroup, 1 = one block per workgroup, launched
 * longest first.  Results are identical. */
dipaco_status dipaco_k_set_attention_blocks(int32_t single_block);

/* Causal softmax attention.  qkv: [B*S, 3*H*dh], row = q | k | v, head h at columns h*dh of each third;
 * o: [B*S, H*dh];  lse: fp32 [B, H, S] = log sum_j exp(q_i.k_j / sqrt(dh)), j <= i.  dh in {32, 64, 128}.
 * Here and in the gradient a value that is not finite reaches exactly the rows that see it; bf16 with dh = 64: any row of
 * its block of 64 positions as well. */
dipaco_status dipaco_k_attention_fwd(int32_t dtype, const void* qkv, void* o, float* lse, int32_t B, int32_t S,
                                     int32_t H, int32_t dh, void* stream);

/* Gradient of the above: d_o [B*S, H*dh] -> dqkv [B*S, 3*H*dh].  dsum: fp32 scratch of 2 * B * H * S128 floats,
 * S128 = S rounded up to a multiple of 128 (per-query statistics passed between the two backward kernels).
 * colsum_out: NULL, or fp32 [3*H*dh] = the column sums of dqkv (the bias gradient of the QKV projection), added in a
 * fixed order; then colsum_scratch: fp32, at least max(ceil(B*S / 256), B * ceil(S / 128)) * 3*H*dh elements. */
dipaco_status dipaco_k_attention_bwd(int32_t dtype, const void* qkv, const void* o, const void* d_o, const float* lse,
                                     void* dqkv, float* dsum, float* colsum_out, float* colsum_scratch, int32_t B,
                                     int32_t S, int32_t H, int32_t dh, void* stream);

/* Causal softmax attention with a sliding window and sinks.  Position i of a document sees position j where j <= i and
 * (j > i - window or j < sinks): the last `window` positions, itself included, and the first `sinks` of the document.
 * window >= 1 (one that covers the sequence is plain causal attention), sinks >= 0.
 *   qkv [B*S, (H + 2*H_kv)*dh], row = q | k | v; H is a multiple of H_kv, and query head h reads key and value head
 *   h / (H / H_kv).  dh in {32, 64, 128}.  o [B*S, H*dh];  lse fp32 [B, H, S] = log of the sum of exp(q_i.k_j / sqrt(dh))
 *   over the positions that i sees.
 *   lengths: NULL, or device int32 [B]: document b is the first lengths[b] of its S rows (taken as 0 below 0, as S above).
 *   Rows behind it are padding: they are not read, whatever they hold, and o, lse and dqkv are written 0 there.
 * A value that is not finite reaches exactly the rows that see it.  B * S < 2^31, H * S <= 2^25,
 * (H + 2*H_kv) * dh <= 2^20.  Results are bit-reproducible.
 * bf16, here, in the gradient and over a paged cache, as in dipaco_k_attention_*: probabilities (and dS) enter their products with 16 bits for dh 32
 * and 128, whose results are as exact as their rounding to bf16, and rounded to bf16 for dh 64; sums, lse and D are fp32. */
dipaco_status dipaco_k_attention_window_fwd(int32_t dtype, const void* qkv, const int32_t* lengths, void* o, float* lse,
                                            int32_t B, int32_t S, int32_t H, int32_t H_kv, int32_t dh, int32_t window,
                                            int32_t sinks, void* stream);

/* Gradient of the above: d_o [B*S, H*dh] -> dqkv [B*S, (H + 2*H_kv)*dh], from the o and lse that it left; the gradients of a
 * key or value head are the sums over the query heads that read it.  dsum: fp32 scratch of 2 * B * H * S128 floats,
 * S128 = S rounded up to a multiple of 128.  dqkv must not overlap the inputs; it may hold partial sums while the call runs. */
dipaco_status dipaco_k_attention_window_bwd(int32_t dtype, const void* qkv, const int32_t* lengths, const void* o,
                                            const void* d_o, const float* lse, void* dqkv, float* dsum, int32_t B, int32_t S,
                                            int32_t H, int32_t H_kv, int32_t dh, int32_t window, int32_t sinks, void* stream);

/* A paged cache of keys and values, for documents that are read or written in pieces.
 *   cache      dtype [n_pages, 2, H_kv, page_size, dh], keys then values; page_size in {16, 32, 64, 128, 256}.
 *   pages      device int32 [B, pages_per_doc]: position p of document b is slot p % page_size of page
 *              pages[b, p / page_size].  An entry outside [0, n_pages) is no page: nothing is written for its positions and
 *              nobody sees them (pages that a window has left behind can be handed back).  Documents may share pages that
 *              are only read; a page that a call writes to belongs to one document.
 *   qkv        the new tokens, [T, (H + 2*H_kv)*dh], row = q | k | v.
 *   row_start  device int32 [B + 1], not decreasing, 0 .. T: rows row_start[b] .. row_start[b+1] - 1 are the new tokens
 *              of document b, none or more.  Rows behind row_start[B] belong to nobody.
 *   cache_len  device int32 [B]: positions that document b had in front of them: its first new token is position
 *              cache_len[b], 0 .. 2^31 - 2^24 (values outside are taken as the nearest inside).  A position behind the table,
 *              pages_per_doc * page_size or more, has no page: it is not written, nobody sees it, and its row sees what of
 *              the table lies in its window or among the sinks.
 *              All of these are read on the device: a captured graph follows their values.
 * T <= 2^23, T * H <= 2^25, B <= 2^20, B * H <= 2^22, pages_per_doc * page_size <= 2^28.
 * dipaco_k_cache_append writes the new tokens' keys and values into the pages. */
dipaco_status dipaco_k_cache_append(int32_t dtype, const void* qkv, const int32_t* row_start, const int32_t* cache_len,
                                    const int32_t* pages, void* cache, int32_t T, int32_t B, int32_t H, int32_t H_kv,
                                    int32_t dh, int32_t n_pages, int32_t page_size, int32_t pages_per_doc, void* stream);

/* Attention of the new tokens over the cache that they have been appended to (same row_start and cache_len), with the window
 * and sinks of dipaco_k_attention_window_fwd over positions: chunk by chunk, or token by token, the rows of that call.
 *   o [T, H*dh];  lse fp32 [T, H] or NULL.  A row that sees nothing (its pages are gone): o = 0, lse = -inf; one whose visible
 *   scores are all -inf: o = NaN, lse = -inf, as in that call.  Rows of nobody are left as they were.  max_new: no document has more new tokens in this call (rows beyond it are left as they were).
 * workspace: device, >= dipaco_k_attention_paged_workspace_bytes(...) (0 = invalid shape), contents undefined before and
 * after; calls that may overlap in time, captured ones included, need one each.  A value that is not finite reaches exactly
 * the rows that see it.  Results are bit-reproducible; those of one row may differ in rounding with the other rows of the call. */
size_t dipaco_k_attention_paged_workspace_bytes(int32_t T, int32_t B, int32_t max_new, int32_t H, int32_t H_kv, int32_t dh,
                                                int32_t page_size, int32_t pages_per_doc);
dipaco_status dipaco_k_attention_paged(int32_t dtype, const void* qkv, const int32_t* row_start, const int32_t* cache_len,
                                       const int32_t* pages, const void* cache, void* o, float* lse, int32_t T, int32_t B,
                                       int32_t max_new, int32_t H, int32_t H_kv, int32_t dh, int32_t n_pages,
                                       int32_t page_size, int32_t pages_per_doc, int32_t window, int32_t sinks,
                                       void* workspace, size_t workspace_bytes, void* stream);

/* Drafted decoding over a paged cache: a cheaper path, or anything else, proposes several tokens for each document, and the path runs all of
 * them in one step.  A document's new rows are a tree: row 0 is the last token that is certain, every other row a drafted
 * token.  A step is dipaco_k_draft_tree; per block of the path dipaco_k_cache_append (row i goes to slot cache_len + i) and
 * dipaco_k_attention_tree; dipaco_k_draft_verify on the logits of all rows; dipaco_k_cache_keep; then cache_len grows by `kept`.
 *   parent     device int32 [T]: the row's parent, counted from its document's row 0; an earlier row of the document.  Any other
 *              value: the row is a root.
 *   row_start, cache_len, pages, cache, T, B: as above.  max_new: no document has more rows in this call (rows beyond it are left as
 *              they were), at most 1024.
 * dipaco_k_draft_tree:
 *   depth      device int32 [T]: a row's ancestors, their number.  Its token stands at position cache_len + depth.
 *   seen       device uint64 [T, ceil(max_new / 64)]: bit a % 64 of word a / 64 where the row sees row a of its document: itself and
 *              its ancestors.  Rows of nobody are left as they were. */
dipaco_status dipaco_k_draft_tree(const int32_t* parent, const int32_t* row_start, int32_t* depth, uint64_t* seen, int32_t T, int32_t B,
                                  int32_t max_new, void* stream);

/* Attention of the rows over the cache that they have been appended to.  Row i of document b stands at position cache_len[b] + depth and
 * sees cached position j < cache_len[b] where j > position - window or j < sinks, and row a of the document (slot cache_len[b] + a) where
 * its bit of `seen` is set; window >= max_new, so that no row's ancestor lies in front of its window.
 *   depth, seen  as dipaco_k_draft_tree writes them for the same max_new.  Others may be given: a depth is taken as the nearest in 0 .. i, bits
 *                of rows that the document does not have are ignored, and a row may see any others, or none.
 * bf16: probabilities enter their product with 16 bits for every dh.  Everything else, the workspace included, as in dipaco_k_attention_paged. */
size_t dipaco_k_attention_tree_workspace_bytes(int32_t T, int32_t B, int32_t max_new, int32_t H, int32_t H_kv, int32_t dh,
                                               int32_t page_size, int32_t pages_per_doc);
dipaco_status dipaco_k_attention_tree(int32_t dtype, const void* qkv, const int32_t* row_start, const int32_t* cache_len, const int32_t* depth,
                                      const uint64_t* seen, const int32_t* pages, const void* cache, void* o, float* lse, int32_t T,
                                      int32_t B, int32_t max_new, int32_t H, int32_t H_kv, int32_t dh, int32_t n_pages,
                                      int32_t page_size, int32_t pages_per_doc, int32_t window, int32_t sinks, void* workspace,
                                      size_t workspace_bytes, void* stream);

/* Which drafts stay, by given random numbers, so that every token has the distribution that the target alone would give it.
 *   target, draft  dtype [T, V] logits of the path and of what drafted.  Row i's are those of the token behind it: the children of row i
 *                  were drawn from softmax(draft_i / draft_temperature) (distinct = 0: each by itself; 1: one after the other, none
 *                  twice).  draft = NULL: the drafts were not drawn but picked, whatever the random numbers will be.
 *   tokens         device int32 [T];  u device fp32 [T], v device fp32 [B]: uniform in [0, 1), independent of the drafts.
 * From node = row 0: r = softmax(target_node / temperature), at temperature 0 all of it at the largest logit (the first such);
 * q = softmax(draft_node / draft_temperature).  The children of node, in order, of token x:
 *     q(x) = 0, or x not in [0, V): passed over;
 *     u q(x) < r(x): taken, and the walk goes on from there;
 *     else r <- max(r - q, 0) over its sum, and for distinct = 1 q(x) <- 0 and q <- q over its sum.
 *   draft = NULL: q is 1 at x and 0 elsewhere.  Where no child is taken the next token is the first y with r(0) + .. + r(y) > v; an r
 *   whose sum is 0 is softmax(target_node / temperature) again.  Decided with 64-bit numbers, whose exponentials
 *   are right to 2^-36 of themselves.
 *   path   device int32 [B, max_new]: row 0 and the rows taken, in order, then -1.   kept device int32 [B]: their number, 0 for a document
 *          without rows.   next device int32 [B]: the next token; -1 for a document without rows, and where the target's logits are no
 *          distribution (a NaN, a +inf, or nothing above -inf), where the walk ends.  Draft logits that are none: no child is taken.
 * temperature >= 0, draft_temperature > 0 (not read without draft), both finite.  1 <= V <= 2^18, max_new <= 1024, T <= 2^23, B <= 2^20.
 * workspace: device, >= dipaco_k_draft_verify_workspace_bytes(T, B, V) (0 = invalid shape), contents undefined before and after; calls
 * that may overlap in time, captured ones included, need one each.  Results are bit-reproducible. */
size_t dipaco_k_draft_verify_workspace_bytes(int32_t T, int32_t B, int32_t V);
dipaco_status dipaco_k_draft_verify(int32_t dtype, const void* target, const void* draft, const int32_t* tokens, const int32_t* parent,
                                    const int32_t* row_start, const float* u, const float* v, int32_t* path, int32_t* kept, int32_t* next,
                                    int32_t T, int32_t B, int32_t max_new, int32_t V, float temperature, float draft_temperature,
                                    int32_t distinct, void* workspace, size_t workspace_bytes, void* stream);

/* The rows that stay move to their places: in every cache slot cache_len[b] + i takes the keys and values of slot cache_len[b] + path[b, i],
 * i < kept[b].  caches: host array of n_layers device pointers, each another layer's cache (the same one twice is
 * refused), of the same pages.  path [B, max_new] and kept as dipaco_k_draft_verify writes them; kept is taken as the nearest in 0 .. max_new, and a path ends at the first entry that does not rise or is
 * not in 0 .. max_new - 1.  A row whose slot, the old one or the new, has no page stays where it is.  */
dipaco_status dipaco_k_cache_keep(int32_t dtype, const int32_t* path, const int32_t* kept, const int32_t* cache_len, const int32_t* pages,
                                  void* const* caches, int32_t n_layers, int32_t B, int32_t max_new, int32_t H_kv, int32_t dh,
                                  int32_t n_pages, int32_t page_size, int32_t pages_per_doc, void* stream);

/* Measurement aid, no part of the method: register-only loops that show how the matrix cores and the vector ALU of a
 * SIMD share instruction issue (the inner loops of the attention kernels are priced with it).  One workgroup of
 * 256 * waves_per_simd threads per compute unit (256 workgroups) runs `iters` iterations of
 *   mode 0: 16 v_mfma_f32_32x32x16_bf16 on four independent accumulators;   mode 1: 256 independent v_fma_f32;
 *   mode 2: the 16 MFMA, then the 256 FMA;   mode 3: sixteen times (1 MFMA, 16 FMA) in program order;
 *   mode 4: 256 times (v_exp_f32, multiply, add);
 *   modes 5..8 (always 512 threads per workgroup, two waves per SIMD; waves_per_simd is ignored): what the chip sustains
 *   of the two bf16 matrix-core shapes, a wave's 128 x 64 outputs computed 32 deep per iteration (524,288 flop per wave
 *   and iteration) from operands held in registers: 5 / 6 = v_mfma_f32_32x32x16_bf16 on all-zero / pseudo-random
 *   operands, 7 / 8 = v_mfma_f32_16x16x32_bf16 likewise (the GEMM kernel's choice of shape rests on 6 against 8).
 * The caller times the launch.  out: device fp32, 256 * 256 * waves_per_simd elements (at least 256 * 512 for modes
 * 5..8), overwritten (keeps the loops alive).  mode in 0..8, waves_per_simd in 1..4, iters >= 1, else DIPACO_EINVAL. */
dipaco_status dipaco_k_issue_probe(int32_t mode, int32_t waves_per_simd, int32_t iters, float* out, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* DIPACO_KERNELS_H */
