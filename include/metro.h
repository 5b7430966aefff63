/*
 * metro.h -- C ABI of the MI355X (gfx950) METRO hot path.
 *
 * METRO = Minimum Expert Token ROuting (arxiv 2512.09277): choose one replica for every
 * (token, expert) pair so that the maximum number of *activated* expert replicas on any
 * expert-parallel rank is minimised (problem min-exp-routing, Sec. 4.1), then run the
 * memory-bound decode MoE layer of one rank on the pairs routed to it.
 *
 * Conventions for every call
 *   - All data pointers are DEVICE pointers owned by the caller; nothing is allocated,
 *     freed or synchronised inside.  Work is enqueued on `stream` (a hipStream_t passed as
 *     void*; NULL = the default stream) and the call returns at once.
 *   - Return value: METRO_OK or a negative METRO_ERR_* for arguments the host can check.
 *     On error nothing is enqueued.  Conditions only the device can see (an id out of
 *     range, an expert with tokens but no replica) are reported through `err_flag`.
 *   - Notation: N experts, top-k, G logical EP ranks, spr replica slots per rank,
 *     S = G*spr slots, slot s lives on rank s / spr; T tokens in the (global) batch;
 *     pair index p = t*k + j; H hidden size, I intermediate size.
 *   - Limits: 1 <= N <= 512, 1 <= G <= 64, 1 <= spr <= 64, S <= 2048, 1 <= k <= N,
 *     T*k < 2^24.
 */
#ifndef METRO_H_
#define METRO_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define METRO_OK 0
#define METRO_ERR_INVALID_ARG (-1)   /* null pointer, non-positive size, k > N, misaligned pointer */
#define METRO_ERR_UNSUPPORTED (-2)   /* a size beyond the limits above, unknown dtype */
#define METRO_ERR_WORKSPACE (-3)     /* workspace smaller than the *_workspace_bytes() figure */
#define METRO_ERR_HIP (-4)           /* the HIP runtime refused a launch */
#define METRO_ERR_TOO_LARGE (-5)     /* the problem needs more than the library's built-in scratch buffer */

/* bits of err_flag[layer] */
#define METRO_FLAG_BAD_ID 1          /* a top-k id outside [-1, N) */
#define METRO_FLAG_NO_REPLICA 2      /* an expert that has tokens is on no rank */
#define METRO_FLAG_BAD_PLACEMENT 4   /* a slot_to_expert entry outside [-1, N) */

#define METRO_DTYPE_F32 0
#define METRO_DTYPE_BF16 1

/* Text for a METRO_ERR_* code (static storage). */
const char* metro_status_string(int status);

/*
 * metro_route -- the greedy solve of min-exp-routing (Alg. 1, Sec. 4.3) for L independent
 * layers in one launch.  Experts are served in ascending id; each expert with at least one
 * pair (T[i] > 0) takes, among the ranks hosting it, the one with the fewest activated
 * experts so far, ties to the lowest rank; all of its pairs go to that replica (x from y,
 * Sec. 4.3).  The result is a deterministic, lock-free execution of Alg. 1.
 *
 *   topk_ids       [L,T,k] int32  global top-k expert ids of the whole batch; -1 = padded pair
 *   slot_to_expert [L,S]   int32  placement (matrix A of Sec. 4.1): expert held by each slot,
 *                                 -1 = empty slot; a second copy of an expert on the same rank
 *                                 is ignored (A is binary)
 *   pair_slot      [L,T,k] int32  out: chosen slot of every pair (-1 for padded pairs)
 *   expert_slot    [L,N]   int32  out: activated slot of every expert, -1 if it has no pair
 *   rank_active    [L,G]   int32  out: activated experts per rank (lambda = their maximum)
 *   rank_bitmap    [L,G]   uint64 out: bit l set iff local slot l of the rank is activated
 *   err_flag       [L]     int32  out: 0, or METRO_FLAG_* bits; outputs of a flagged layer are
 *                                 unspecified apart from being in range
 *
 * Shared memory, here and in the other routing calls: pair_slot may be the id tensor itself; outputs of the token
 * lists (see moe_permute) may lie anywhere in the ids or the placement of a call that routes and lists in one;
 * n_pairs may be group_offsets + spr.  Apart from that an output must not overlap an input or another output.
 */
int metro_route(const int32_t* topk_ids, const int32_t* slot_to_expert, int L, int T, int k, int N, int G,
                int spr, int32_t* pair_slot, int32_t* expert_slot, int32_t* rank_active,
                uint64_t* rank_bitmap, int32_t* err_flag, void* stream);

/*
 * metro_route_token_balanced -- the baseline the paper compares with (EPLB-style routing,
 * Sec. 2.3 and Sec. 6.1 "Compared baselines"): every expert's pairs are spread evenly over
 * its replicas.  The q-th pair of an expert, in flattened (t, j) order, goes to replica
 * q mod r, replicas taken in ascending slot id.  Same arguments as metro_route, without
 * expert_slot (an expert may activate several replicas).
 */
int metro_route_token_balanced(const int32_t* topk_ids, const int32_t* slot_to_expert, int L, int T, int k,
                               int N, int G, int spr, int32_t* pair_slot, int32_t* rank_active,
                               uint64_t* rank_bitmap, int32_t* err_flag, void* stream);

/*
 * moe_permute -- per-replica token lists of one rank ("route tokens", Sec. 4.3): the pairs
 * whose slot lies on `rank`, ordered by local slot l = slot - rank*spr and, within a slot,
 * by pair index (a stable counting sort).
 *
 *   pair_slot     [T,k]   int32  one layer's routing result
 *   group_offsets [spr+1] int32  out: rows of local slot l are [group_offsets[l], group_offsets[l+1])
 *   perm_pair     [T*k]   int32  out: pair index of every row; entries past n_pairs are not written
 *   pair_row      [T,k]   int32  out: row of each pair in the list, -1 if routed to another rank
 *   n_pairs       [1]     int32  out: number of rows (= group_offsets[spr])
 */
int moe_permute(const int32_t* pair_slot, int T, int k, int rank, int spr, int32_t* group_offsets,
                int32_t* perm_pair, int32_t* pair_row, int32_t* n_pairs, void* stream);

/*
 * metro_route_permute / metro_route_token_balanced_permute -- one layer's routing solve followed, in the same
 * launch, by the token lists of one rank ("route tokens", Sec. 4.3): exactly metro_route (or
 * metro_route_token_balanced) with L = 1 and then moe_permute(pair_slot, rank), without the second launch: a
 * pair's row follows from its place among the pairs of its expert.  Arguments and results as in those calls;
 * 0 <= rank < G.  Where buffers share memory (see metro_route) it is the two calls, in two launches.
 */
int metro_route_permute(const int32_t* topk_ids, const int32_t* slot_to_expert, int T, int k, int N, int G, int spr,
                        int rank, int32_t* pair_slot, int32_t* expert_slot, int32_t* rank_active,
                        uint64_t* rank_bitmap, int32_t* err_flag, int32_t* group_offsets, int32_t* perm_pair,
                        int32_t* pair_row, int32_t* n_pairs, void* stream);
int metro_route_token_balanced_permute(const int32_t* topk_ids, const int32_t* slot_to_expert, int T, int k, int N,
                                       int G, int spr, int rank, int32_t* pair_slot, int32_t* rank_active,
                                       uint64_t* rank_bitmap, int32_t* err_flag, int32_t* group_offsets,
                                       int32_t* perm_pair, int32_t* pair_row, int32_t* n_pairs, void* stream);

/*
 * moe_gate_topk -- router gate and top-k over the full (gathered) token set: the step that builds
 * the global top-k knowledge the routing solve consumes (Sec. 4.3: tokens are all-gathered and every
 * rank runs top-k on all of them).  The paper leaves the gate itself to the model; this is the
 * common softmax router:
 *     logit[t][e]  = x[t] . w_gate[e]
 *     topk_ids[t]  = the k experts with the largest logits, descending; equal logits: lower id first
 *     topk_w[t][j] = exp(logit[t][ids[t][j]]) / sum over the k selected of exp(logit)
 *     expert_count[e] = number of (token, expert) pairs that selected e      (T[i] of Sec. 4.1)
 * Batches are padded to fixed sizes where the layer is replayed from a captured graph (Sec. 5): tokens
 * t >= *n_valid are padding and get topk_ids -1 (which both routing calls skip), topk_w 0, and count nothing.
 *
 *   x        [T,H]   dtype     activations (rows H elements apart)
 *   w_gate   [N,H]   dtype     router weights, rows ldw >= H elements apart
 *   n_valid  [1]     int32     number of real tokens, read on the device (clamped to [0, T]); NULL = T
 *   topk_ids [T,k]   int32     out; valid input for metro_route / metro_route_token_balanced
 *   topk_w   [T,k]   float32   out; valid input for moe_unpermute
 *   expert_count [N] int32     out, may be NULL (asking for it adds one small launch)
 *   ws                         workspace of moe_gate_topk_workspace_bytes(); 256-byte aligned.  The figure for T tokens is enough
 *                              for every smaller batch; a call is refused only for less than its own batch needs
 *   dtype  METRO_DTYPE_BF16: bf16 operands, fp32 accumulation on the matrix cores when H % 32 == 0,
 *          N % 64 == 0, ldw % 8 == 0 and x, w_gate are 16-byte aligned; other shapes and
 *          METRO_DTYPE_F32 (fp32 products and sums) take a general kernel.  Logits are summed in a fixed order, so the
 *          result is deterministic; a NaN logit counts as the lowest finite number (above -infinity).
 * Limits: N <= 512, k <= min(N, 64), T*k < 2^24.  T == 0 writes nothing but expert_count (all zero).
 */
size_t moe_gate_topk_workspace_bytes(int T, int H, int N, int dtype);
int moe_gate_topk(const void* x, const void* w_gate, int ldw, int T, int H, int N, int k, int dtype,
                  const int32_t* n_valid, int32_t* topk_ids, float* topk_w, int32_t* expert_count, void* ws,
                  size_t ws_bytes, void* stream);

/*
 * moe_grouped_ffn -- SwiGLU expert FFN over the token lists of one rank.  Only slots with at
 * least one row are touched, so HBM weight traffic scales with the number of activated
 * experts (Sec. 3.2).  For row r of local slot l, token t = perm_pair[r] / k:
 *     gate = x[t] . w13[l][0:I]^T      up = x[t] . w13[l][I:2I]^T
 *     y_perm[r] = (silu(gate) * up) . w2[l]^T
 *
 *   x      [T,H]       dtype   activations of the whole batch
 *   w13    [spr,2I,H]  dtype   per local slot: rows 0..I-1 gate, I..2I-1 up (H contiguous);
 *                              consecutive rows are ldw13 >= H elements apart, slots 2I*ldw13
 *   w2     [spr,H,I]   dtype   per local slot: down projection (I contiguous), rows ldw2 >= I
 *                              elements apart, slots H*ldw2
 *   ldw13, ldw2                row pitches in elements, multiples of 8.  The weights are the
 *                              library's to lay out: a pitch that is a multiple of 4096 bytes makes
 *                              the rows that are read together fall on the same few HBM channels (36 slots
 *                              of 8 rows at H = 4096, I = 2048, both matrices: 4.8 instead of 6.1 TB/s),
 *                              so pad such rows, e.g. by 128 elements.
 *   y_perm [T*k,H]     dtype   out: rows 0..n_pairs-1 are written
 *   ws                         workspace of moe_grouped_ffn_workspace_bytes(); 256-byte aligned
 *   dtype  METRO_DTYPE_BF16: bf16 storage, fp32 accumulation on the matrix cores, the
 *          intermediate silu(gate)*up rounded to bf16; needs H % 128 == 0 and I % 128 == 0,
 *          other shapes take a slower general kernel.  METRO_DTYPE_F32: fp32 throughout.
 *   x, w13, w2, y_perm must be 16-byte aligned.
 */
size_t moe_grouped_ffn_workspace_bytes(int T, int k, int spr, int H, int I, int dtype);
int moe_grouped_ffn(const void* x, const int32_t* perm_pair, const int32_t* group_offsets, int T, int k,
                    int spr, int H, int I, int dtype, const void* w13, int ldw13, const void* w2, int ldw2,
                    void* y_perm, void* ws, size_t ws_bytes, void* stream);

/*
 * The two stages of moe_grouped_ffn as separate calls, in the order gate_up -> down, on the same
 * workspace and stream (moe_grouped_ffn is exactly that sequence).  They exist so that a caller can
 * put events between the stages or overlap other work; arguments as above.  Both read
 * group_offsets: every workgroup derives its own piece of work from it, there is no planning pass.
 *   gate_up  act = silu(x . w13[gate]^T) * (x . w13[up]^T), kept in the workspace
 *   down     y_perm = act . w2^T
 */
int moe_grouped_ffn_gate_up(const void* x, const int32_t* perm_pair, const int32_t* group_offsets, int T, int k,
                            int spr, int H, int I, int dtype, const void* w13, int ldw13, void* ws,
                            size_t ws_bytes, void* stream);
int moe_grouped_ffn_down(const int32_t* group_offsets, int T, int k, int spr, int H, int I, int dtype,
                         const void* w2, int ldw2, void* y_perm, void* ws, size_t ws_bytes, void* stream);

/*
 * moe_grouped_ffn_static_ws -- moe_grouped_ffn for callers that cannot allocate or size a workspace (code under
 * HIP-graph capture, tight serving loops, harnesses that forbid hipMalloc): the intermediate activations
 * live in an array built into the library, METRO_STATIC_WS_BYTES per GPU, held from library load until the
 * process ends.  Same arguments and results as moe_grouped_ffn without ws / ws_bytes; same kernels.
 *   - A problem whose moe_grouped_ffn_workspace_bytes() exceeds moe_grouped_ffn_static_ws_bytes()
 *     (bf16: T*k*I*2 + 256 bytes; the DeepSeek-V3-shaped decode batch T*k = 8192, I = 2048 just fits)
 *     is refused with METRO_ERR_TOO_LARGE and nothing is enqueued.
 *   - The call allocates nothing.  Its first use on a device looks up the array's address.
 *   - All calls on one GPU share that GPU's array: calls that may overlap in time (different streams,
 *     different threads) race on it; serialise them or use moe_grouped_ffn with separate workspaces.
 *     Nothing in the array has to be cleared between calls.
 */
#define METRO_STATIC_WS_BYTES ((size_t)(32u << 20) + 256u)
size_t moe_grouped_ffn_static_ws_bytes(void);
int moe_grouped_ffn_static_ws(const void* x, const int32_t* perm_pair, const int32_t* group_offsets, int T, int k,
                              int spr, int H, int I, int dtype, const void* w13, int ldw13, const void* w2,
                              int ldw2, void* y_perm, void* stream);

/*
 * moe_unpermute -- the rank's share of the combine step (Sec. 2.2): for every token,
 *     out[t] = sum over j ascending of topk_w[t,j] * y_perm[pair_row[t,j]]   (pairs served here),
 * accumulated in fp32; tokens with no pair on this rank get zeros.
 *
 *   y_perm [T*k,H] dtype, pair_row [T,k] int32, topk_w [T,k] float32, out [T,H] dtype.
 *   An entry of pair_row outside [0, T*k) counts as "not on this rank".
 */
int moe_unpermute(const void* y_perm, const int32_t* pair_row, const float* topk_w, int T, int k, int H,
                  int dtype, void* out, void* stream);

/*
 * moe_permute_rows / moe_permute_rows_backward -- the tokens' rows sorted by expert, and the gradient of that:
 *     x_perm[pair_row[t,j]] = x[t]                          (pairs on this rank)
 *     dx[t] = sum over j ascending of dx_perm[pair_row[t,j]]    (pairs on this rank), accumulated in fp32; zeros where there is none
 * Rows of x_perm that no pair names (those past n_pairs) are left as they were.  pair_row as in moe_unpermute; no row is named twice.
 *
 *   x, dx [T,H] dtype, pair_row [T,k] int32, x_perm, dx_perm [T*k,H] dtype.
 */
int moe_permute_rows(const void* x, const int32_t* pair_row, int T, int k, int H, int dtype, void* x_perm, void* stream);
int moe_permute_rows_backward(const void* dx_perm, const int32_t* pair_row, int T, int k, int H, int dtype, void* dx, void* stream);

/*
 * moe_unpermute_backward -- the gradient of moe_unpermute.  For every pair of this rank, r = pair_row[t,j]:
 *     dy_perm[r] = topk_w[t,j] * dout[t]
 *     dtopk_w[t,j] = sum over H of dout[t] * y_perm[r], products and sums in fp32 in a fixed order; 0 for pairs of other ranks
 * Rows of dy_perm that no pair names are left as they were; no row is named twice.
 *
 *   dout [T,H] dtype, y_perm, dy_perm [T*k,H] dtype, pair_row [T,k] int32, topk_w, dtopk_w [T,k] float32.
 */
int moe_unpermute_backward(const void* dout, const void* y_perm, const int32_t* pair_row, const float* topk_w, int T, int k, int H,
                           int dtype, void* dy_perm, float* dtopk_w, void* stream);

/*
 * 8-bit experts.  Values are OCP e4m3 (1 byte; largest 448), with one fp32 scale for each block of 128: a value stands for
 * byte * scale.  Activations have a scale for each 128 consecutive values of a row, scale [rows, ceil(K/128)]; a weight matrix one for
 * each 128 rows x 128 columns, scale [ceil(rows/128), ceil(K/128)].  The last block of a row or matrix may be short.
 * e4m3 rows are `ld` bytes apart, ld >= K, a multiple of 16 and, where a product reads them, at most 2^28, and start 16-byte aligned; a product
 * reads the bytes from K up to the next multiple of 16 (their values do not matter), so they must be there, behind the last row too.
 *
 * moe_quantize_fp8 -- rows of activations (or of a gradient).  With m = max(largest magnitude of a block, 1e-30):
 *     scale = m / 448        q = the e4m3 value nearest to x * (448 / m), ties to even        (each operation rounded to fp32)
 * A block that holds a NaN gets scale NaN and NaNs; one that holds an infinity scale infinity, NaN in its place and zeros elsewhere.
 *
 *   x      [R,K]  dtype    rows ldx >= K elements apart
 *   n_rows [1]    int32    rows to convert, read on the device (clamped to [0, R]); NULL = R.  Rows past it are left as they were
 *   q      [R,K]  e4m3     out, rows ldq bytes apart (bytes past K are not written)
 *   scale  [R, ceil(K/128)] float32 out        Limit: K <= 2^30
 */
int moe_quantize_fp8(const void* x, int ldx, int R, int K, int dtype, const int32_t* n_rows, void* q, int ldq, float* scale,
                     void* stream);

/*
 * moe_quantize_weights_fp8 -- the same for `slots` matrices [rows, K], in blocks of 128 x 128.  For w13 as moe_grouped_ffn_fp8 reads it,
 * pass the gate and up halves as matrices of their own: slots = 2*spr, rows = I.
 *
 *   w [slots,rows,K] dtype, rows ldw elements and slots rows*ldw elements apart; q [slots,rows,K] e4m3 out, likewise with ldq bytes;
 *   scale [slots, ceil(rows/128), ceil(K/128)] float32 out.       Limits: rows, K <= 2^30, fewer than 2^24 blocks.
 */
int moe_quantize_weights_fp8(const void* w, int ldw, int slots, int rows, int K, int dtype, void* q, int ldq, float* scale, void* stream);

/*
 * moe_grouped_mm_fp8 -- rows sorted by group (expert) times the weights of their group.  For row r of group l, with blocks b of K:
 *     y[r][n] = sum over b of xs[r][b] * ws[l][n/128][b] * (sum over k in b of x[r][k] * w[l][n][k])
 * products and sums in fp32, in a fixed order, which differs between batches of few and of many rows.  Only groups with at least one row are
 * touched.  The gradient of x is the same call with transposed weights and scales on quantized rows of dy.
 *
 *   x      e4m3, xs float32     perm_pair NULL: [T*k,K], row r itself;  else [T,K], row r is that of token perm_pair[r] / k
 *   group_offsets [groups+1] int32   rows of group l are [group_offsets[l], group_offsets[l+1])
 *   w      [groups,N,K] e4m3    rows ldw bytes apart, groups N*ldw;   ws [groups, ceil(N/128), ceil(K/128)] float32
 *   y      [T*k,N] dtype   out; rows past the last group are left as they were.  16-byte aligned
 * Limits: groups <= 64, K, N <= 2^20, T*k < 2^24.
 */
int moe_grouped_mm_fp8(const void* x, int ldx, const float* xs, const int32_t* perm_pair, const int32_t* group_offsets, int T, int k,
                       int groups, int K, int N, const void* w, int ldw, const float* ws, int dtype, void* y, void* stream);

/*
 * moe_grouped_ffn_fp8 -- moe_grouped_ffn on 8-bit experts, products and sums in fp32 as in moe_grouped_mm_fp8.  For row r of local slot l, token
 * t = perm_pair[r] / k:
 *     gate, up = x[t] . w13[l]^T          (as in moe_grouped_mm_fp8 with perm_pair)
 *     act = silu(gate) * up in fp32, then to e4m3 with a scale for each 128 as by moe_quantize_fp8
 *     y_perm[r] = act . w2[l]^T
 *
 *   x      [T,H] e4m3, xs [T, ceil(H/128)] float32
 *   w13    [spr,2I,H] e4m3   gate rows, then up rows; s13 [spr, 2*ceil(I/128), ceil(H/128)]: the blocks of up start at its first row
 *   w2     [spr,H,I] e4m3    s2 [spr, ceil(H/128), ceil(I/128)]
 *   y_perm [T*k,H] dtype     out: rows 0..n_pairs-1 are written.  16-byte aligned
 *   ws     workspace of moe_grouped_ffn_fp8_workspace_bytes(); 256-byte aligned.  The figure for T tokens is enough for every smaller batch
 * Weight pitches: as for moe_grouped_ffn, pad rows whose length is a multiple of 4096 bytes.
 * Limits: spr <= 64, H, I <= 2^20, T*k < 2^24.
 */
size_t moe_grouped_ffn_fp8_workspace_bytes(int T, int k, int spr, int H, int I);
int moe_grouped_ffn_fp8(const void* x, int ldx, const float* xs, const int32_t* perm_pair, const int32_t* group_offsets, int T, int k,
                        int spr, int H, int I, const void* w13, int ldw13, const float* s13, const void* w2, int ldw2, const float* s2,
                        int dtype, void* y_perm, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* METRO_H_ */
