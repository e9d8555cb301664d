/*
 * bcast_serve.h -- C ABI of the operators that a group of serving replicas runs on bytes it got by
 * a broadcast.
 *
 * After bcast_exec() every rank buffer holds the same bytes.  Where these are a model's weights and
 * the cache of a prompt that all requests start with, the next thing a replica does is answer
 * requests, and the rule of the tuned ring -- do not move again what the receiver already holds --
 * carries over: what all requests share is read once for all of them, and only what is a request's
 * own is added per request.  The operators of a decode step, in the order of their use:
 *
 *   bcast_serve_linear   a projection that all tokens share, plus the low-rank adapter of each
 *                        token's request
 *   bcast_serve_linear4  the same without adapters, the weights in 4 bits: a message 3.8 times
 *                        shorter.  bcast_serve_pack4 makes such weights before the broadcast,
 *                        bcast_serve_unpack4 makes numbers of them again
 *   bcast_serve_append   new tokens' queries and keys normed and rotated, keys and values put into
 *                        the requests' caches
 *   bcast_serve_attn     attention of the newest tokens of every request over a prefix that all
 *                        requests share, followed by the request's own tokens
 *   bcast_serve_verify   acceptance of drafted tokens against the target's probabilities from given
 *                        random numbers, and the choice of the token that follows them
 *   bcast_serve_logprobs log probabilities of given tokens, the rows' entropy, and their most
 *                        probable tokens
 *
 * They go forward only: what they compute has no backward pass here.
 *
 * Conventions
 *   - As in bcast.h: every function returns BCAST_OK or a negative BCAST_ERR_* code, nothing throws
 *     across this boundary, and work is enqueued on the caller's stream of the current device and
 *     not waited for.
 *   - Pointers are DEVICE pointers unless stated otherwise; strides count elements, not bytes.  The
 *     innermost dimension of every array is contiguous.
 *   - What the host can check (ranges, alignment, NULL, host pointers, capacity of the workspace) is
 *     checked before anything is launched: BCAST_ERR_INVAL, or BCAST_ERR_CAPACITY for the workspace.
 *     What only the device knows (adapter numbers, lengths, page numbers, token numbers) cannot be
 *     refused; each operator says what it makes of values out of range.  None of them leads to an
 *     access outside the arrays described.
 *   - Inputs may not overlap outputs or the workspace, unless an operator says so.
 *   - Workspace (where a call has one): scratch of at least bcast_serve_*_workspace() bytes, 256-byte aligned.  Its first
 *     BCAST_SERVE_STATUS_BYTES hold the status word and must have been zeroed once, before the first
 *     call; nothing else in it has to be initialised, and nothing in it is kept from one call for the
 *     next.  Calls that share a workspace must be ordered on the GPU (one stream, or events); calls
 *     with different workspaces may overlap.
 *   - The kernels' waits on the copy engine and on the tensor cores are bounded.  One that runs out
 *     sets the status word and ends the kernel early, its output incomplete: see bcast_serve_status().
 *     With the environment variable BCAST_SERVE_GIVE_UP=1 (for tests; read at the first call) the kernels
 *     begin as if a wait had run out.
 *   - The calls may be captured into a CUDA graph.
 */
#ifndef BCAST_SERVE_B200_H
#define BCAST_SERVE_B200_H

#include "bcast.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { BCAST_SERVE_BF16 = 0, BCAST_SERVE_FP16 = 1, BCAST_SERVE_FP32 = 2 };

#define BCAST_SERVE_STATUS_BYTES 256

/*
 * bcast_serve_linear -- y[t] = W x[t] + bias + scale[a] * B[a] (A[a] x[t]),  a = adapter[t].
 * A token whose adapter is outside 0..num_adapters-1 (-1, say) gets W x[t] + bias alone.  Sums are
 * held in 32 bits; the low-rank product u = scale[a] * A[a] x[t] is passed on as the sum of two numbers of
 * the data type (bf16: a relative error of 2^-16 at most; fp16: 2^-22, or 2^-25 as such where that is more;
 * u has to be in the type's range), y is rounded once.
 *   - Adapters that no token of the call names are not read.  Those that are hold finite numbers: a token's own x
 *     may hold NaN or infinity without touching other tokens, an adapter's values may not (tokens of one tile pass
 *     through the same products, multiplied by zero for the adapters they do not have).
 *   dtype         BCAST_SERVE_BF16 or BCAST_SERVE_FP16: x, weight, bias, lora_a, lora_b and y
 *   tokens        0 <= T <= 2^21;  1 <= k, n <= 2^24, k a multiple of 8
 *   num_adapters  0 <= L <= 65536 (0: none; lora_*, adapter and scale are then not looked at)
 *   rank          R, a multiple of 8, 8..128 (an adapter of lower rank is padded with zeros)
 *   x [T][k], weight [n][k], y [T][n]: rows at x_stride, weight_stride, y_stride
 *   bias [n] or NULL
 *   lora_a [L][R][k], lora_b [L][n][R]: adapters at *_stride[0], rows at *_stride[1]
 *   adapter [T] int32, scale [L] float
 * x, weight, lora_a and lora_b start on a 16-byte boundary and their strides are multiples of 8;
 * a stride is at least the length of what it steps over (y_stride >= n, and so on).
 */
typedef struct bcast_serve_linear_args {
    int32_t dtype, num_adapters, rank;
    int64_t tokens, k, n;
    const void *x, *weight, *bias, *lora_a, *lora_b;
    const int32_t *adapter;
    const float *scale;
    void *y;
    int64_t x_stride, weight_stride, y_stride, lora_a_stride[2], lora_b_stride[2];
    void *workspace;
    uint64_t workspace_bytes;
} bcast_serve_linear_args;

int bcast_serve_linear(const bcast_serve_linear_args *args /* HOST */, void *cuda_stream);
/* Bytes of workspace the call needs (pointers in args are not looked at), or a negative code. */
int64_t bcast_serve_linear_workspace(const bcast_serve_linear_args *args);

/*
 * bcast_serve_attn -- for request b, new token i and query head h (which reads key/value head
 * h / (q_heads / kv_heads)):
 *     out[b][i][h] = sum_j softmax_j(scale * q[b][i][h] . k_j) v_j
 * over the prefix_len tokens of the shared prefix and the first own_len[b] - new_tokens + i + 1 of
 * the request's own: own_len[b] counts the own tokens in the cache, the new ones among them (they are
 * the last, and causal among themselves).  Softmax statistics and sums are held in 32 bits.
 *   - A row that sees no token at all (no prefix, and own_len[b] <= new_tokens - 1 - i) gives zeros,
 *     and -infinity in lse.
 *   - own_len[b] is taken as 0 where negative and as own_cap where larger.  Nothing is read behind it:
 *     cache rows that hold no token yet may hold anything, NaN included.
 *   - A page number outside 0..num_pages-1 stands for a page of tokens that are not there.
 *   - The values of the tokens that are there are finite: a new token that may not see a later one still has it
 *     multiplied by a weight of zero.  A key may hold NaN: the rows that see it become NaN, in out and in lse, and no
 *     others.
 * Arguments
 *   dtype        BCAST_SERVE_BF16 or BCAST_SERVE_FP16
 *   0 <= batch, new_tokens <= 65535;  1 <= kv_heads <= 1024, q_heads a multiple of kv_heads, at most 65535;
 *   0 <= prefix_len, own_cap < 2^31 - 65536;  dim a multiple of 8, 8..128;  new_tokens * q_heads <= 2^19, and at most 2^24 rows
 *   (batch * new_tokens * q_heads) in all
 *   q, out       [batch][new_tokens][q_heads][dim], strides of the first three
 *   prefix_k/_v  [prefix_len][kv_heads][dim], strides of the first two (not looked at if prefix_len = 0)
 *   own_k/_v     rows:  [batch][own_cap][kv_heads][dim]      (page_table NULL)
 *                pages: [num_pages][page_size][kv_heads][dim], strides of the first three
 *                (not looked at if own_cap = 0)
 *   own_len      [batch] int32
 *   page_table   NULL or [batch][ceil(own_cap / page_size)] int32, rows at page_table_stride
 *   lse          NULL or [batch][new_tokens][q_heads] float: log of the sum of exp(scale * q . k_j)
 * q, out and the caches start on 16-byte boundaries and their strides are multiples of 8.  A stride of out
 * and of the prefix is at least dim; those of q and of the own caches may also be 0 (rows that several
 * requests share).
 */
typedef struct bcast_serve_attn_args {
    int32_t dtype, batch, new_tokens, q_heads, kv_heads, dim, page_size;
    float scale;
    int64_t prefix_len, own_cap, num_pages;
    const void *q, *prefix_k, *prefix_v, *own_k, *own_v;
    const int32_t *own_len, *page_table;
    void *out;
    float *lse;
    int64_t q_stride[3], out_stride[3], prefix_k_stride[2], prefix_v_stride[2], own_k_stride[3], own_v_stride[3];
    int64_t page_table_stride;
    void *workspace;
    uint64_t workspace_bytes;
} bcast_serve_attn_args;

int bcast_serve_attn(const bcast_serve_attn_args *args /* HOST */, void *cuda_stream);
int64_t bcast_serve_attn_workspace(const bcast_serve_attn_args *args);

/*
 * bcast_serve_verify -- speculative sampling.  Request b has drafted x_i = draft_tokens[b][i],
 * i < drafts, each drawn from q_i = draft_probs[b][i]; p_i = softmax(logits[b][i] / temperature[b]),
 * i <= drafts, are the target's distributions at the same places and one further.
 *   - The drafts are accepted from the first on while uniforms[b][i] * q_i(x_i) < p_i(x_i); their
 *     number is accepted[b] = c.
 *   - The token after them is argmax_v w(v) / noise[b][v], with w = max(p_c - q_c, 0) if c < drafts
 *     and w = p_c if all were accepted.  With noise drawn from the unit exponential distribution this
 *     is a draw from w / sum(w), and the whole output is distributed as if drawn from p.  Where w is
 *     zero everywhere, p_c takes its place.
 *   - Where temperature[b] is not above 0 (NaN among them), x_i is accepted while it is the token of the
 *     largest logit, and the token after the accepted ones is that of the largest logit.  At an infinite
 *     temperature every token whose logit is above -infinity is as likely as any other.
 *   - tokens[b] = the accepted drafts, the token after them, then -1.
 * Ties go to the lowest token number.  A logit that is NaN counts as -infinity; where some are
 * +infinity, these share the probability evenly.  A row without any logit above -infinity has no
 * probabilities: its draft is not accepted, and the token is -1.  A drafted token outside
 * 0..vocab-1 is not accepted.  Entries of noise that are not positive never win.
 *   dtype        of logits: BCAST_SERVE_BF16, BCAST_SERVE_FP16 or BCAST_SERVE_FP32
 *   0 <= batch <= 65535;  0 <= drafts <= 63;  1 <= vocab < 2^31 - 65536
 *   logits       [batch][drafts + 1][vocab], strides of the first two
 *   draft_probs  [batch][drafts][vocab] float, strides of the first two
 *   noise        [batch][vocab] float, rows at noise_stride
 *   draft_tokens [batch][drafts] int32, uniforms [batch][drafts] float, temperature [batch] float
 *   accepted     [batch] int32, tokens [batch][drafts + 1] int32
 * draft_probs, draft_tokens and uniforms are not looked at if drafts = 0.
 */
typedef struct bcast_serve_verify_args {
    int32_t dtype, batch, drafts;
    int64_t vocab;
    const void *logits;
    const float *draft_probs, *uniforms, *noise, *temperature;
    const int32_t *draft_tokens;
    int32_t *accepted, *tokens;
    int64_t logits_stride[2], draft_probs_stride[2], noise_stride;
    void *workspace;
    uint64_t workspace_bytes;
} bcast_serve_verify_args;

int bcast_serve_verify(const bcast_serve_verify_args *args /* HOST */, void *cuda_stream);
int64_t bcast_serve_verify_workspace(const bcast_serve_verify_args *args);

/*
 * bcast_serve_append -- the newest tokens of every request on their way from a projection to
 * bcast_serve_attn.  For request b, new token i < new_tokens (own_len as in bcast_serve_attn: the own
 * tokens in the cache, the new ones among them):
 *     slot = own_len[b] - new_tokens + i
 *     out[b][i][h]        = R(norm(q[b][i][h]) * q_norm)         for every query head
 *     own_k at slot, head = R(norm(k[b][i][h]) * k_norm),   own_v at slot, head = v[b][i][h]
 * with norm(x) = x / sqrt(mean(x^2) + eps) where norm weights are given, and x itself where not.
 * R turns the pairs of the first `rot` numbers of a head, pair p = 0..rot/2-1 being (p, p + rot/2), or
 * (2p, 2p + 1) where `interleaved`: (x, y) -> (x cos t - y sin t, x sin t + y cos t),
 *     t = position * inv_freq[p],  position = first + slot, or positions[b][i][axis[p]] where given.
 * The angle is reduced in whole numbers, to 2^-63 of a turn, for every finite inv_freq and every position; one below 2^-6 keeps
 * all of its digits.  Arithmetic is in 32 bits, results are rounded once; what is neither normed nor rotated is copied bit
 * for bit.
 *   - A token is padding if i < new_tokens - new_len[b] (where new_len is given: a request with fewer new tokens
 *     has them at the end), or if its slot is negative.  Padding goes nowhere, and its rows of out are zero.
 *   - Keys and values whose slot is not below own_cap, or whose page is outside 0..num_pages-1, are not
 *     stored; their queries are still written.  Nothing else of the caches is touched.
 *   - Where two tokens of a call have the same place (a page that stands in the table twice), either may
 *     stay.
 *   - An axis outside 0..axes-1 is taken as 0.  inv_freq is finite.  A normed head's sum of squares is in the range of
 *     32-bit floats.
 *   dtype        BCAST_SERVE_BF16 or BCAST_SERVE_FP16: q, k, v, q_norm, k_norm, out and the caches
 *   0 <= batch, new_tokens <= 65535, at most 2^24 tokens and 2^31 - 1 heads of them in all;  0 <= q_heads <= 65535, 1 <= kv_heads
 *   <= 1024;  dim a multiple of 8, 8..128;  rot a multiple of 16, 0..dim (0: no rotation; inv_freq, axis and positions are then not
 *   looked at);  0 <= first < 2^31;  0 <= own_cap < 2^31 - 65536;  0 <= axes <= 16 (0: by slot)
 *   q, out       [batch][new_tokens][q_heads][dim] (not looked at if q_heads = 0); out may be q itself
 *   k, v         [batch][new_tokens][kv_heads][dim]; strides of the first three
 *   q_norm, k_norm  NULL or [dim] each;  eps >= 0
 *   inv_freq     [rot / 2] float
 *   positions    [batch][new_tokens][axes] int32 if axes > 0, strides of the first two;  axis [rot / 2] int32, or NULL
 *                for axis 0 throughout
 *   own_k/_v, page_table, page_size, num_pages   as in bcast_serve_attn
 *   own_len [batch] int32, new_len NULL or [batch] int32
 * q, k, v, out, the norms and the caches start on 16-byte boundaries and their strides are multiples of 8; strides of
 * out and the caches are at least dim, those of q, k and v may be 0.
 */
typedef struct bcast_serve_append_args {
    int32_t dtype, batch, new_tokens, q_heads, kv_heads, dim, page_size, rot, interleaved, axes;
    float eps;
    int64_t own_cap, num_pages, first;
    const void *q, *k, *v, *q_norm, *k_norm;
    const float *inv_freq;
    const int32_t *positions, *axis, *own_len, *new_len, *page_table;
    void *out, *own_k, *own_v;
    int64_t q_stride[3], k_stride[3], v_stride[3], out_stride[3], own_k_stride[3], own_v_stride[3], positions_stride[2];
    int64_t page_table_stride;
} bcast_serve_append_args;

int bcast_serve_append(const bcast_serve_append_args *args /* HOST */, void *cuda_stream);

/*
 * bcast_serve_logprobs -- for every row of logits l, with p = softmax(l):
 *     logprobs[r]     = log p(tokens[r])
 *     entropy[r]      = -sum p log p
 *     top_tokens[r]   = the `top` tokens with the largest logits, the lower number first among equals
 *     top_logprobs[r] = their log p
 * Statistics are held in 32 bits.  The logits are read once, a few of them twice; up to all of them twice in rows with
 * -infinity, NaN, the lowest number of bf16 or fp32, or logits beyond 2^20, and more often where hundreds of equal ones are
 * among the largest.  No log p is above 0, no entropy below.
 *   - A logit that is NaN counts as -infinity; where some are +infinity, these share the probability evenly.
 *     Tokens that so have no probability, and those outside 0..vocab-1, have -infinity as their log p.  They are no
 *     alternatives: where there are fewer than `top` others, the row goes on with token -1 and -infinity.  A row
 *     without any logit above -infinity has the entropy 0.
 *   dtype     of logits: BCAST_SERVE_BF16, BCAST_SERVE_FP16 or BCAST_SERVE_FP32
 *   0 <= rows < 2^24;  1 <= vocab < 2^31 - 65536;  0 <= top <= 32
 *   logits    [rows][vocab], rows at logits_stride (which may be 0)
 *   tokens    [rows] int32;  logprobs [rows] float
 *   entropy   NULL or [rows] float
 *   top_tokens [rows][top] int32, top_logprobs [rows][top] float (not looked at if top = 0)
 */
typedef struct bcast_serve_logprobs_args {
    int32_t dtype, top;
    int64_t rows, vocab;
    const void *logits;
    const int32_t *tokens;
    float *logprobs, *entropy, *top_logprobs;
    int32_t *top_tokens;
    int64_t logits_stride;
} bcast_serve_logprobs_args;

int bcast_serve_logprobs(const bcast_serve_logprobs_args *args /* HOST */, void *cuda_stream);

/*
 * Microscaled 4-bit numbers: 32 neighbours of a row share a power of two.
 *   codes   [rows][k / 2] bytes, rows at codes_stride (bytes): number 2j in the low half of byte j.  A code is a
 *           sign and one of 0, 1/2, 1, 3/2, 2, 3, 4, 6.
 *   scales  a byte e per block, which stands for 2^(e - 127); 255: the block's numbers are NaN.  They lie in tiles
 *           of 128 rows x 4 blocks, [ceil(rows / 128)][ceil(k / 128)][32][4][4] bytes: block c of row r at
 *           [r / 128][c / 4][r % 32][r % 128 / 32][c % 4].  Places that stand for no block are zero.
 *
 * bcast_serve_pack4 -- values to codes and scales.  e is the largest magnitude's exponent less 2 (so that it
 * becomes 4 to 8), at least 0; a number divided by 2^(e - 127) goes to the nearest code, to the even one of two as near,
 * and to 6 above that.  A block with NaN or an infinity in it becomes NaN.
 * bcast_serve_unpack4 -- codes and scales to values, rounded once to the data type.
 *   dtype   of values: BCAST_SERVE_BF16, BCAST_SERVE_FP16 or BCAST_SERVE_FP32
 *   0 <= rows < 2^31 - 65536;  k a multiple of 32, 32..2^24;  at most 2^36 numbers, both rounded up to 128
 *   values  [rows][k], rows at values_stride: at least k, a multiple of 8; starts on a 16-byte boundary
 *   codes_stride at least k / 2, a multiple of 16; codes and scales start on 16-byte boundaries
 */
typedef struct bcast_serve_pack4_args {
    int32_t dtype;
    int64_t rows, k;
    void *values;              /* pack4: read only */
    uint8_t *codes, *scales;   /* unpack4: read only */
    int64_t values_stride, codes_stride;
} bcast_serve_pack4_args;

int bcast_serve_pack4(const bcast_serve_pack4_args *args /* HOST */, void *cuda_stream);
int bcast_serve_unpack4(const bcast_serve_pack4_args *args /* HOST */, void *cuda_stream);

/*
 * bcast_serve_linear4 -- y[t] = W x4[t] + bias: W in microscaled 4-bit numbers as bcast_serve_pack4 makes
 * them, x4[t] what pack4 makes of x[t].  Sums are held in 32 bits, y is rounded once.  A block of x[t] with NaN or an
 * infinity in it makes y[t] NaN, a block of W that is NaN its feature.
 * 4 bits on both sides are coarse: for normally distributed x and W, y is off by 0.16 of its size (root mean square; with W
 * alone in 4 bits it would be 0.115, with both in bf16 0.003).
 *   dtype        BCAST_SERVE_BF16 or BCAST_SERVE_FP16: x, bias and y
 *   tokens       0 <= T <= 2^21;  k a multiple of 32, 32..2^24, T * k at most 2^36, k rounded up to 128;  1 <= n <= 2^24
 *   x [T][k], y [T][n]: rows at x_stride (a multiple of 8), y_stride;  bias [n] or NULL
 *   codes, codes_stride, scales: of W [n][k], as above
 */
typedef struct bcast_serve_linear4_args {
    int32_t dtype;
    int64_t tokens, k, n;
    const void *x, *bias;
    const uint8_t *codes, *scales;
    void *y;
    int64_t x_stride, codes_stride, y_stride;
    void *workspace;
    uint64_t workspace_bytes;
} bcast_serve_linear4_args;

int bcast_serve_linear4(const bcast_serve_linear4_args *args /* HOST */, void *cuda_stream);
int64_t bcast_serve_linear4_workspace(const bcast_serve_linear4_args *args);

/*
 * bcast_serve_status -- did a kernel that used this workspace give up on a bounded wait?  Reads the
 * status word on cuda_stream and waits for that stream; clears the word and returns BCAST_ERR_TIMEOUT if
 * it was set, else BCAST_OK.
 */
int bcast_serve_status(void *workspace, void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* BCAST_SERVE_B200_H */
