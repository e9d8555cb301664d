// bcast_serve_attn: attention of every request's newest tokens over a prefix that all requests share and
// the request's own tokens behind it.
//
// Softmax over a set of tokens that is cut into parts: with m_p >= the largest score of part p (in powers of two),
// l_p = sum 2^(s - m_p) and o_p = sum 2^(s - m_p) v, the whole is  M = max m_p,
//   out = sum_p 2^(m_p - M) o_p / sum_p 2^(m_p - M) l_p.
// Three kernels, the second starting once the first is on its way (programmatic launch):
//   prefix kernel   a block per (key/value head, tile of rows, part of the prefix).  The rows are those of ALL
//                   requests -- request, new token and query head of the group --, so a prefix token is read once
//                   for 128 or 256 rows (cut_of) and the two products run on tcgen05
//   own kernel      a block per (request, key/value head, part of its own tokens): few rows against tokens that
//                   nobody else reads, so bound by reading them; warps take 16 tokens at a time through mma.sync.  A
//                   short prefix goes with them, and the prefix kernel is left out.
//   join kernel     the formula above, a block per row
// What bounds them, and what they take on one B200 (bf16, 8 key/value heads of 128, 4 query heads to each; time on the
// device, in brackets that of a public call among others of its kind):
//   64 requests x 4 new tokens, prefix 65536, up to 1024 own: 257 us, 1.08 PFLOP/s (300, the power cap).  A pair of 128-row tiles against
//     128 tokens takes about 3050 cycles, where its products need 2048: a tile's softmax (about 2000 cycles, half
//     of them on the exponentials) is longer than the other tile's products, and nothing is left to run under it
//   32 requests x 1, prefix 8192, up to 700 own in pages: 36 us for 80 MB (37).  The prefix kernel takes 14 us of it (4 to
//     its first scores, 5 for its four tiles, 3.5 for its sums), the own kernel 15 (latency: a block has 8 rounds
//     of loads), the join 5
//   one request, 8 heads of 64, 509 + 60 tokens: 7 us, two launches (9.5)
#include "serve_device.cuh"
#include "serve_internal.h"
#include "serve_tma.h"

#include <climits>

namespace bcast_serve {
namespace {

struct AttnDev {
    const void *q, *ok, *ov, *pk, *pv;
    const int32_t *own_len, *page_table;
    void *out;
    float *lse;
    float2 *part_ml;      // [parts][rows]: (m, l), m = -infinity where a part holds nothing
    float *part_o;        // [parts][rows][dim]
    int *status;
    int give_up;          // 1: begin as if a wait had run out
    int64_t qs[3], os[3], oks[3], ovs[3], pks[2], pvs[2];
    int64_t own_cap, num_pages, pts, rows;       // rows: batch * fresh * q_heads
    int32_t batch, fresh, q_heads, kv_heads, group, dim, page, page_shift, prefix_len;
    int32_t prefix_splits, prefix_parts, row_tiles, own_chunk, folded, fold_chunk, parts;
    float scale_log2;     // scale * log2(e): the softmax is taken in powers of two
};

// fp16 holds weights from 2^-24 to 2^16: shifting them by 2^7 keeps the small ones exact for longer (the factor
// is in l as well and cancels).  bf16 has the exponents of 32-bit floats.
template <typename T> constexpr float kShift = std::is_same_v<T, __half> ? 7.0f : 0.0f;

// Powers of two that a row's maximum may lag behind: weights up to 2^kSlack (and 2^kShift).  32-bit sums and bf16
// weights have the exponents for much more, fp16 weights end at 2^16.
template <typename T> constexpr float kSlack = std::is_same_v<T, __half> ? 8.0f : 24.0f;

// Weights are rounded to the data type before their product with V, as the tensor cores take both operands in it.  That
// costs as much as rounding the result does: errors against 64 bits are 1.25 to 1.44 times those of 32-bit arithmetic
// rounded once.  Sums of weights are taken before the rounding.
template <typename T> __device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// ------------------------------------------------------------------------------------------- own tokens
constexpr int kOwnWarps = 2, kOwnKeys = 16, kOwnRows = 16, kOwnStages = 3;

template <int DB> constexpr size_t own_smem() { return (size_t)kOwnWarps * kOwnStages * 2 * kOwnKeys * DB * 128; }

__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool there)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void ldmatrix(uint32_t *r, uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldmatrix_t(uint32_t *r, uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
template <typename T>
__device__ __forceinline__ void mma_sync(float *c, const uint32_t *a, uint32_t b0, uint32_t b1)
{
    if constexpr (std::is_same_v<T, __nv_bfloat16>)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Where a request's own token `at` lies: page (or request) and place in it; page -1 if it is not there.  Looked up
// whether or not the token is in the cache yet (the table has a place for it), so as not to wait for the length.
struct Place {
    int32_t page, slot;
};
__device__ __forceinline__ Place place_of(const AttnDev &d, bool own, int b, int at)
{
    if (at >= (own ? d.own_cap : (int64_t)d.prefix_len)) return Place{-1, 0};
    if (!own || !d.page_table) return Place{b, at};
    const int n = d.page_shift >= 0 ? at >> d.page_shift : at / d.page;
    const int32_t p = d.page_table[(int64_t)b * d.pts + n];
    return Place{p >= 0 && p < d.num_pages ? p : -1, at - n * d.page};
}
// Where chunk `c` of row `r` of a tile lies, rows of 128 or 256 bytes: the eight rows that a matrix load reads at a
// time are in different banks.
template <int ROW>
__device__ __forceinline__ uint32_t own_at(int r, int c) { return r * ROW + ((c ^ (r & 7)) << 4); }

// A warp holds 16 rows and walks over its share of the block's tokens, 16 at a time: scores by mma.m16n8k16 (rows x
// tokens), weights, then rows x dim.  Its K and V tiles go through three stages of its own (cp.async, no barrier
// between warps); the warps' results are joined at the end.  Two warps to a block, so that blocks are many and end at
// different times: 64 requests with up to 1000 own tokens take 55 us, with four warps 68.
template <typename T, int DB>
__global__ void __launch_bounds__(kOwnWarps * 32, 4)
serve_attn_own_kernel(const __grid_constant__ AttnDev d)
{
    constexpr int D = DB * 64, row_bytes = DB * 128, tile = kOwnKeys * row_bytes;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ float warp_m[kOwnWarps][kOwnRows], warp_l[kOwnWarps][kOwnRows];
    const int b = blockIdx.z, kv = blockIdx.y % d.kv_heads, r0 = blockIdx.y / d.kv_heads * kOwnRows, split = blockIdx.x;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, rows = d.fresh * d.group;
    launch_next();
    // the first parts are the shared prefix's where that is too short for a kernel of its own (Cut::fold)
    const bool own = split >= d.folded;
    const int chunk = own ? d.own_chunk : d.fold_chunk, k0 = (own ? split - d.folded : split) * chunk;
    // length, pages and queries: three loads that do not wait for one another
    Place ahead[2];                           // of the two tokens of a block that this lane copies parts of
#pragma unroll
    for (int h = 0; h < 2; h++) ahead[h] = place_of(d, own, b, k0 + warp * kOwnKeys + h * 8 + lane / 4);
    // queries, as the first operand's fragments; rows and columns that do not exist are zero
    uint32_t q[DB * 4][4];
#pragma unroll
    for (int half = 0; half < 2; half++) {
        const int r = r0 + half * 8 + lane / 4;
        const T *row = (const T *)d.q + b * d.qs[0] + r / d.group * d.qs[1] + (kv * d.group + r % d.group) * d.qs[2];
#pragma unroll
        for (int i = 0; i < DB * 8; i++) {
            const int c = i * 8 + lane % 4 * 2;
            q[i / 2][half + i % 2 * 2] = r < rows && c < d.dim ? *(const uint32_t *)(row + c) : 0u;
        }
    }
    const int len = own ? (int)min(max((int64_t)d.own_len[b], (int64_t)0), d.own_cap) : d.prefix_len;
    const int k1 = min(len, k0 + chunk), part = d.prefix_parts + split;
    int limit[2], seen_by_all = INT_MAX;      // own tokens that a row sees; that all rows do
#pragma unroll
    for (int half = 0; half < 2; half++) {
        const int r = r0 + half * 8 + lane / 4;
        limit[half] = r >= rows ? 0 : own ? len - d.fresh + r / d.group + 1 : INT_MAX;
        seen_by_all = min(seen_by_all, r < rows ? limit[half] : INT_MAX);
    }
    seen_by_all = __reduce_min_sync(~0u, seen_by_all);

    const uint32_t base = smem_u32(smem) + warp * kOwnStages * 2 * tile;
    const int blocks = k1 > k0 ? (k1 - k0 + kOwnKeys - 1) / kOwnKeys : 0, mine = (blocks - warp + kOwnWarps - 1) / kOwnWarps;
    const T *const karray = (const T *)(own ? d.ok : d.pk), *const varray = (const T *)(own ? d.ov : d.pv);
    const T *kbase = karray + kv * (own ? d.oks[2] : d.pks[1]) + lane % 4 * 8, *vbase = varray + kv * (own ? d.ovs[2] : d.pvs[1]) + lane % 4 * 8;
    const int64_t kpage = own ? d.oks[0] : 0, vpage = own ? d.ovs[0] : 0, kslot = own ? d.oks[1] : d.pks[0], vslot = own ? d.ovs[1] : d.pvs[0];
    // Four lanes copy a token, 64 bytes at a time: whole sectors, and one address per lane and token.  Its page is
    // looked up one block ahead, so that this is not in the way of the copies.  Returns which tokens are there, token k at
    // bit 4 (k % 8) of word k / 8.
    auto load = [&](int i, int stage) {
        uint2 bits;
        const uint32_t ks = base + stage * 2 * tile;
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const int r = h * 8 + lane / 4, at = k0 + (i * kOwnWarps + warp) * kOwnKeys + r;
            const Place p = ahead[h];
            ahead[h] = place_of(d, own, b, at + kOwnWarps * kOwnKeys);
            const bool ok = at < k1 && p.page >= 0;
            (h ? bits.y : bits.x) = __ballot_sync(~0u, ok);
            const T *kr = ok ? kbase + p.page * kpage + p.slot * kslot : karray;
            const T *vr = ok ? vbase + p.page * vpage + p.slot * vslot : varray;
#pragma unroll
            for (int j = 0; j < DB * 2; j++) {
                const int c = j * 4 + lane % 4;
                const bool in = ok && c * 8 < d.dim;
                copy16(ks + own_at<row_bytes>(r, c), in ? kr + j * 32 : karray, in);
                copy16(ks + tile + own_at<row_bytes>(r, c), in ? vr + j * 32 : varray, in);
            }
        }
        return bits;
    };
    uint2 there[kOwnStages] = {};             // of the next blocks, in order
#pragma unroll
    for (int i = 0; i < kOwnStages - 1; i++) {
        if (i < mine) there[i] = load(i, i);
        asm volatile("cp.async.commit_group;" ::: "memory");
    }

    float o[DB * 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {};
#pragma unroll
    for (int n = 0; n < DB * 8; n++) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.0f;
    int stage = 0, free = kOwnStages - 1;
    for (int i = 0; i < mine; i++) {
        if (i + kOwnStages - 1 < mine) there[kOwnStages - 1] = load(i + kOwnStages - 1, free);
        asm volatile("cp.async.commit_group;" ::: "memory");
        asm volatile("cp.async.wait_group %0;" ::"n"(kOwnStages - 1) : "memory");
        __syncwarp();
        const uint32_t ks = base + stage * 2 * tile, vs = ks + tile;
        const uint2 here = there[0];
#pragma unroll
        for (int k = 0; k + 1 < kOwnStages; k++) there[k] = there[k + 1];
        free = stage;
        stage = stage + 1 == kOwnStages ? 0 : stage + 1;
        const int at = k0 + (i * kOwnWarps + warp) * kOwnKeys;
        float sc[2][4] = {};
#pragma unroll
        for (int k = 0; k < DB * 4; k++) {
            uint32_t f[4];
            const int r = lane / 16 * 8 + lane % 8, c = k * 2 + lane / 8 % 2;
            ldmatrix(f, ks + own_at<row_bytes>(r, c));
            mma_sync<T>(sc[0], q[k], f[0], f[1]);
            mma_sync<T>(sc[1], q[k], f[2], f[3]);
        }
        // scores that nobody may see go to -infinity; most blocks have none
        float top[2] = {-INFINITY, -INFINITY};
        if (here.x == ~0u && here.y == ~0u && at + kOwnKeys <= seen_by_all) {
#pragma unroll
            for (int x = 0; x < 8; x++) {
                float &v = sc[x / 4][x % 4];
                v *= d.scale_log2;
                top[x / 2 % 2] = fmaxf(top[x / 2 % 2], v);
            }
        } else {
#pragma unroll
            for (int x = 0; x < 8; x++) {
                const int key = lane % 4 * 2 + x % 2;  // of eight
                float &v = sc[x / 4][x % 4];
                v = ((x < 4 ? here.x : here.y) >> 4 * key & 1u) && at + x / 4 * 8 + key < limit[x / 2 % 2] ? v * d.scale_log2 : -INFINITY;
                top[x / 2 % 2] = fmaxf(top[x / 2 % 2], v);
            }
        }
        // The maximum may lag by kSlack, as in the prefix kernel: only where it has to move do the four lanes of a row
        // settle on it and scale down what is summed so far.
        if (__any_sync(~0u, top[0] > m[0] + (m[0] == -INFINITY ? 0.0f : kSlack<T>) || top[1] > m[1] + (m[1] == -INFINITY ? 0.0f : kSlack<T>))) {
#pragma unroll
            for (int half = 0; half < 2; half++) {
                float t = fmaxf(top[half], __shfl_xor_sync(~0u, top[half], 1));
                t = fmaxf(fmaxf(t, __shfl_xor_sync(~0u, t, 2)), m[half]);
                const float fix = exp2_approx(m[half] - (t == -INFINITY ? 0.0f : t));
                m[half] = t;
                l[half] *= fix;
#pragma unroll
                for (int n = 0; n < DB * 8; n++) {
                    o[n][half * 2] *= fix;
                    o[n][half * 2 + 1] *= fix;
                }
            }
        }
        uint32_t p[4];
#pragma unroll
        for (int half = 0; half < 2; half++) {
            // nothing seen so far: 0 in the place of -infinity, so that 2^-infinity is 0 and NaN stays NaN
            const float less = kShift<T> - (m[half] == -INFINITY ? 0.0f : m[half]);
            float w[4];
#pragma unroll
            for (int x = 0; x < 4; x++) w[x] = exp2_approx(sc[x / 2][half * 2 + x % 2] + less);
            l[half] += (w[0] + w[1]) + (w[2] + w[3]);
            p[half] = pack2<T>(w[0], w[1]);
            p[half + 2] = pack2<T>(w[2], w[3]);
        }
#pragma unroll
        for (int n = 0; n < DB * 4; n++) {
            uint32_t f[4];
            const int r = lane / 8 % 2 * 8 + lane % 8, c = n * 2 + lane / 16;
            ldmatrix_t(f, vs + own_at<row_bytes>(r, c));
            mma_sync<T>(o[n * 2], p, f[0], f[1]);
            mma_sync<T>(o[n * 2 + 1], p, f[2], f[3]);
        }
        __syncwarp();
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();                          // the stages' memory is free

    float *all = (float *)smem;               // [warp][row][D]
#pragma unroll
    for (int half = 0; half < 2; half++) {
        float sum = l[half];
        sum += __shfl_xor_sync(~0u, sum, 1);
        sum += __shfl_xor_sync(~0u, sum, 2);
        const int r = half * 8 + lane / 4;
        if (lane % 4 == 0) {
            warp_m[warp][r] = m[half];
            warp_l[warp][r] = sum;
        }
        if (blocks > 0) {
#pragma unroll
            for (int n = 0; n < DB * 8; n++)
                *(float2 *)(all + (warp * kOwnRows + r) * D + n * 8 + lane % 4 * 2) = make_float2(o[n][half * 2], o[n][half * 2 + 1]);
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kOwnRows * (D / 4); i += kOwnWarps * 32) {
        const int r = i / (D / 4), c = i % (D / 4) * 4;
        if (r0 + r >= rows || c >= d.dim) continue;
        const int64_t row = ((int64_t)b * d.fresh + (r0 + r) / d.group) * d.q_heads + kv * d.group + (r0 + r) % d.group;
        if (blocks == 0) {
            if (c == 0) d.part_ml[part * d.rows + row] = make_float2(-INFINITY, 0.0f);
            continue;
        }
        float top = warp_m[0][r];
        for (int w = 1; w < kOwnWarps; w++) top = fmaxf(top, warp_m[w][r]);
        const float from = top == -INFINITY ? 0.0f : top;
        float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        float total = 0.0f;
        for (int w = 0; w < kOwnWarps; w++) {
            const float x = exp2_approx(warp_m[w][r] - from);
            const float4 v = *(const float4 *)(all + (w * kOwnRows + r) * D + c);
            sum.x += x * v.x;
            sum.y += x * v.y;
            sum.z += x * v.z;
            sum.w += x * v.w;
            total += x * warp_l[w][r];
        }
        // a row without weights may still hold NaN: l tells
        if (c == 0) d.part_ml[part * d.rows + row] = make_float2(total == 0.0f ? -INFINITY : from - kShift<T>, total);
        *(float4 *)(d.part_o + (part * d.rows + row) * d.dim + c) = sum;
    }
    // the join kernel waits for this one; so this one does not end before the prefix kernel has
    if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0) wait_previous();
}

// ------------------------------------------------------------------------------------------- shared prefix
constexpr int kTileKeys = 128, kPrefixThreads = 320;
constexpr int kKvStages = 4;
constexpr int kPolyEvery = 4;                 // every fourth pair of exponentials goes to the multiply-add units

// (on the way out the same memory holds 256 rows of sums)
template <int DB, bool TWO> constexpr size_t prefix_smem() { return (size_t)(TWO ? 2 : 1) * DB * 16384 + (size_t)kKvStages * DB * 16384 + 1024; }

// The state of one row's softmax.
struct Row {
    float m = -INFINITY;  // what the weights are taken against (a power of two); may lag the maximum
    float l = 0.0f;
};

// 2^x for two numbers at once on the multiply-add units, which have time left where the unit for exponentials
// has none: x = r + f with r the nearest integer (added to 1.5 * 2^23 it stands in the sum's low bits), 2^f on
// [-1/2, 1/2] by a polynomial (least largest relative error, fitted: 7.5e-5 in degree 3, 2.6e-6 in degree 4, against
// 2^-9 and 2^-12 of rounding the weight to the type), times 2^r, whose bits are r's in the place of the exponent.  (r
// added to the exponent of 2^f would spare the product, but turns a NaN into a number.)  Below 2^-126 gives 2^-126.
template <typename T>
__device__ __forceinline__ void exp2_pair(uint64_t x, float &a, float &b)
{
    unpair(x, a, b);
    asm("max.NaN.f32 %0, %0, 0fC2FC0000;" : "+f"(a));         // -126; NaN stays NaN
    asm("max.NaN.f32 %0, %0, 0fC2FC0000;" : "+f"(b));
    x = pair(a, b);
    const float magic = 12582912.0f;
    const uint64_t t = add2(x, pair(magic, magic));
    const uint64_t f = fma2(add2(t, pair(-magic, -magic)), pair(-1.0f, -1.0f), x);
    uint64_t y;
    if constexpr (std::is_same_v<T, __half>) {
        y = pair(0.009570102207362652f, 0.009570102207362652f);
        y = fma2(y, f, pair(0.05591785907745361f, 0.05591785907745361f));
        y = fma2(y, f, pair(0.240247443318367f, 0.240247443318367f));
        y = fma2(y, f, pair(0.6931217908859253f, 0.6931217908859253f));
        y = fma2(y, f, pair(0.9999992847442627f, 0.9999992847442627f));
    } else {
        y = pair(0.0551716685295105f, 0.0551716685295105f);
        y = fma2(y, f, pair(0.2426111251115799f, 0.2426111251115799f));
        y = fma2(y, f, pair(0.6932609677314758f, 0.6932609677314758f));
        y = fma2(y, f, pair(0.9999280571937561f, 0.9999280571937561f));
    }
    float ta, tb;
    unpair(t, ta, tb);
    unpair(mul2(y, pair(__uint_as_float((__float_as_uint(ta) << 23) + 0x3f800000u), __uint_as_float((__float_as_uint(tb) << 23) + 0x3f800000u))), a, b);
}

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float min3(float a, float b, float c)
{
    float r;
    asm("min.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// The first of 16-bit weight `w` times `x`, and the second.
template <typename T>
__device__ __forceinline__ uint32_t scale2(uint32_t w, float x)
{
    const T *v = (const T *)&w;
    return pack2<T>(to_f32(v[0]) * x, to_f32(v[1]) * x);
}

// One tile of a row's scores (tensor memory at `s`, this thread's lane) to weights, 32 tokens at a time, written
// over scores that have been read already as 16-bit pairs.  The weights are taken against a maximum that may lag: it
// moves to the largest of 32 scores only where that is more than kSlack above it, and from there on.  What was taken
// against an earlier one (the sums, the accumulator at `o` among them, and this tile's first weights) is scaled to
// the last one in a place of its own before anyone may read it, which few tiles get to.  So the scores are read
// once, no weight waits for the maximum of the tile, and there is one branch in it: a warp has only one other on its
// scheduler to hide its latencies, so instructions of its own that do not wait for one another have to.  `most` is
// signalled when the weights of the first 96 tokens are there to stay: their product with V runs under the
// last exponentials.
template <typename T, bool MASK>
__device__ __forceinline__ void softmax_tile(Row &row, uint32_t s, uint32_t o, bool first, int valid, int columns, float c, uint32_t most)
{
    const bool up = c >= 0.0f;
    const uint64_t cc = pair(c, c);
    const float start = row.m;
    float m[4];                                       // what the group's weights are taken against
    uint64_t sum[4];
    uint32_t x[2][32];
    tmem_load32(s, x[0]);
#pragma unroll
    for (int g = 0; g < 4; g++) {
        tmem_wait_load32(x[g & 1]);
        const float *v = (const float *)x[g & 1];
        if (g < 3) tmem_load32(s + (g + 1) * 32, x[(g + 1) & 1]);
        // the largest of scale * score; NaN leaves it alone and becomes a NaN weight
        float t0 = up ? -INFINITY : INFINITY, t1 = t0;
        if (MASK) {
#pragma unroll
            for (int i = 0; i < 32; i++)
                if (g * 32 + i < valid) t0 = up ? fmaxf(t0, v[i]) : fminf(t0, v[i]);
        } else if (up) {
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
                t0 = max3(t0, v[i], v[i + 1]);
                t1 = max3(t1, v[i + 2], v[i + 3]);
            }
            t0 = fmaxf(t0, t1);
        } else {
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
                t0 = min3(t0, v[i], v[i + 1]);
                t1 = min3(t1, v[i + 2], v[i + 3]);
            }
            t0 = fminf(t0, t1);
        }
        const float top = MASK && g * 32 >= valid ? -INFINITY : t0 * c;
        row.m = top > row.m + (row.m == -INFINITY ? 0.0f : kSlack<T>) ? top : row.m;
        m[g] = row.m;
        if (g == 3) {
            if (__any_sync(~0u, m[3] != m[0] || (!first && m[0] != start))) {
                const float fix = exp2_approx(start - m[3]);
                if (m[3] != start) {
                    row.l *= fix;
                }
                for (int i = 0; i < (first ? 0 : columns); i += 16) {
                    uint32_t y[16];
                    tmem_load16(o + i, y);
                    tmem_wait_load16(y);
#pragma unroll
                    for (int k = 0; k < 16; k++) y[k] = m[3] == start ? y[k] : __float_as_uint(__uint_as_float(y[k]) * fix);
                    tmem_store16(o + i, y);
                }
                tmem_wait_store();
#pragma unroll
                for (int i = 0; i < 3; i++) {
                    const float part = m[i] == m[3] ? 1.0f : exp2_approx(m[i] - m[3]);
                    sum[i] = mul2(sum[i], pair(part, part));
                    uint32_t y[16];
                    tmem_load16(s + i * 16, y);
                    tmem_wait_load16(y);
#pragma unroll
                    for (int k = 0; k < 16; k++) y[k] = scale2<T>(y[k], part);
                    tmem_store16(s + i * 16, y);
                }
            }
            tmem_wait_store();
            tc_fence_before();
            mbar_arrive(most);
        }
        const float less = kShift<T> - (row.m == -INFINITY ? 0.0f : row.m);
        const uint64_t ll = pair(less, less);
        uint32_t w[16];
        sum[g] = 0;                                   // a pair of 0.0f
#pragma unroll
        for (int i = 0; i < 16; i++) {
            const uint64_t z = fma2(pair(v[2 * i], v[2 * i + 1]), cc, ll);
            float a, b;
            if (i % kPolyEvery == kPolyEvery - 1) {
                exp2_pair<T>(z, a, b);
            } else {
                unpair(z, a, b);
                a = exp2_approx(a);
                b = exp2_approx(b);
            }
            if (MASK) {
                if (g * 32 + 2 * i >= valid) a = 0.0f;
                if (g * 32 + 2 * i + 1 >= valid) b = 0.0f;
            }
            sum[g] = add2(sum[g], pair(a, b));
            w[i] = pack2<T>(a, b);
        }
        tmem_store16(s + g * 16, w);
    }
    float a, b;
    unpair(add2(add2(sum[0], sum[1]), add2(sum[2], sum[3])), a, b);
    row.l += a + b;
    tmem_wait_store();
}

// TWO: two tiles of 128 rows, each with its own softmax warps and accumulator, take the same tokens, so that
// one tile's matrix products run under the other's exponentials.  Otherwise the two halves share 128 rows and take every
// other tile of tokens, and their results are joined at the end.
template <typename T, int DB, bool TWO>
__global__ void __launch_bounds__(kPrefixThreads, 1)
serve_attn_prefix_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                         const __grid_constant__ AttnDev d)
{
    constexpr int block = kTileKeys * 128, stage = DB * block, stages = kKvStages;       // 64 columns of a tile; a tile
    extern __shared__ uint8_t raw_smem[];
    __shared__ __align__(8) uint64_t bars[2 * stages + 10];
    __shared__ float2 half_ml[2][128];
    __shared__ uint32_t tmem_at;
    __shared__ int gave_up;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const int rows = d.batch * d.fresh * d.group;                     // of one key/value head
    const int rt = blockIdx.x % d.row_tiles, kv = blockIdx.x / d.row_tiles % d.kv_heads, split = blockIdx.x / d.row_tiles / d.kv_heads;
    const int r0 = rt * (TWO ? 256 : 128);
    const int tiles = (d.prefix_len + kTileKeys - 1) / kTileKeys;
    const int j0 = (int)((int64_t)tiles * split / d.prefix_splits), nt = (int)((int64_t)tiles * (split + 1) / d.prefix_splits) - j0;
    launch_next();

    uint8_t *smem = (uint8_t *)(((uintptr_t)raw_smem + 1023) & ~(uintptr_t)1023);
    uint8_t *qs = smem;
    const uint32_t q_at = smem_u32(qs), kv_at = q_at + (TWO ? 2 : 1) * stage;
    const uint32_t full = smem_u32(bars), empty = full + 8 * stages, q_full = empty + 8 * stages, s_full = q_full + 8,
                   p_most = s_full + 16, p_full = p_most + 16, o_full = p_full + 16, drained = o_full + 16;
    if (tid == 0) {
        gave_up = d.give_up;
        for (int i = 0; i < stages; i++) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
        }
        mbar_init(q_full, 256);
        for (int i = 0; i < 2; i++) {
            mbar_init(s_full + 8 * i, 1);
            mbar_init(p_most + 8 * i, 128);
            mbar_init(p_full + 8 * i, 128);
            mbar_init(o_full + 8 * i, 1);
        }
        mbar_init(drained, 1);
        mbar_init_fence();
        tma_prefetch(&map_k);
        tma_prefetch(&map_v);
    }
    if (warp == 9) tmem_alloc(smem_u32(&tmem_at), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_at;                                    // scores 0, 128; accumulators 256, 384
    int issued = 0;                                                   // loads, of the thread that issues them

    if (warp == 8) {
        if (lane == 0) {
            // ---- loads, in the order the matrix products take them
            Ring<stages> ring;
            auto load = [&](const CUtensorMap *map, int j) {
                // (the warp that issues the products goes on after it gave up: a slot may be free then that is not filled)
                if (!mbar_wait(empty + 8 * ring.slot, ring.parity ^ 1u, &gave_up) || *(volatile int *)&gave_up) return false;
                mbar_expect(full + 8 * ring.slot, stage);
                for (int i = 0; i < DB; i++)
                    tma_load(kv_at + ring.slot * stage + i * block, map, i * 64, (j0 + j) * kTileKeys, kv, full + 8 * ring.slot);
                issued++;
                ring.step();
                return true;
            };
            // the queries are on their way before the rest of the first tiles, which they would have to queue behind
            bool ok = load(&map_k, 0) && mbar_wait(q_full, 0, &gave_up);
            for (int j = 0; j < nt && ok; j++) {
                if (TWO) {
                    ok = load(&map_v, j) && (j + 1 == nt || load(&map_k, j + 1));
                } else {
                    ok = (j + 1 == nt || load(&map_k, j + 1)) && load(&map_v, j);
                }
            }
        }
        __syncwarp();
    } else if (warp == 9) {
        // ---- matrix products.  An instruction every 64 cycles is what keeps the tensor cores busy, so issuing them has
        // to be cheap: the whole warp goes through the loop together, descriptors differ by constants, and a wait that
        // gives up does not leave the loop -- the ones after it give up at once, and what is still issued only touches this
        // block's own memory.  (With one thread in a loop of its own that made descriptors as it went, a product
        // of 128 x 128 x 128 took 900 to 1800 cycles to issue and not 512.)
        const uint32_t lead = elect_one();            // (chosen outside this branch, it made a long prefix take 5 % longer)
        const uint32_t s_desc = mma_desc<T>(128, kTileKeys), o_desc = mma_desc<T>(128, (d.dim + 15) / 16 * 16, true);
        const uint64_t q_desc = smem_desc(q_at), k_desc = smem_desc(kv_at), v_desc = smem_desc(kv_at, block);
        Ring<stages> ring;
        // Every lane polls for itself; none may fall so far behind the one that issues that a barrier has gone on to its
        // next phase but one.
        auto wait = [&](uint32_t bar, uint32_t parity) {
            mbar_wait(bar, parity, &gave_up);
            __syncwarp();
            tc_fence_after();
        };
        auto take = [&]() {                                           // the next tile of K or V, once it is there
            wait(full + 8 * ring.slot, ring.parity);
            const int slot = ring.slot;
            ring.step();
            return slot;
        };
        auto scores = [&](int w, int slot) {                          // S_w = Q_w K^T; columns past the head size are zero
            const uint64_t a = q_desc + (TWO ? w : 0) * (stage >> 4), b = k_desc + slot * (stage >> 4);
            // Four products to a turn, not unrolled further.  (An earlier form, one thread going through all eight of a
            // head size above 64 under a bound of its own for each, gave wrong rows in the second tile of rows; reading
            // did not show why, and it is not to be gone back to.)
#pragma unroll 1
            for (int k = 0; k < DB; k++)
#pragma unroll
                for (int i = 0; i < 4; i++)
                    mma_ss_warp(lead, tmem + w * 128, a + k * (block >> 4) + 2 * i, b + k * (block >> 4) + 2 * i, s_desc, k > 0 || i > 0);
            mma_commit_warp(lead, s_full + 8 * w);
        };
        auto values = [&](int w, int slot, int it) {                  // O_w += P_w V, as the weights come
            const uint64_t b = v_desc + slot * (stage >> 4);
            const uint32_t o = tmem + 256 + w * 128, a = tmem + w * 128;
            wait(p_most + 8 * w, it & 1);
            mma_ts_warp(lead, o, a, b, o_desc, it > 0);
#pragma unroll
            for (int i = 1; i < 6; i++) mma_ts_warp(lead, o, a + i * 8, b + i * (2048 >> 4), o_desc, true);
            wait(p_full + 8 * w, it & 1);
#pragma unroll
            for (int i = 6; i < 8; i++) mma_ts_warp(lead, o, a + i * 8, b + i * (2048 >> 4), o_desc, true);
        };
        wait(q_full, 0);
        int ks = take();
        scores(0, ks);
        if (TWO) {
            scores(1, ks);
            mma_commit_warp(lead, empty + 8 * ks);
            for (int j = 0; j < nt; j++) {
                const int vs = take();
                const bool more = j + 1 < nt;
                values(0, vs, j);
                if (more) {
                    ks = take();
                    scores(0, ks);
                } else {
                    mma_commit_warp(lead, o_full);
                }
                values(1, vs, j);
                mma_commit_warp(lead, empty + 8 * vs);
                if (more) {
                    scores(1, ks);
                    mma_commit_warp(lead, empty + 8 * ks);
                } else {
                    mma_commit_warp(lead, o_full + 8);
                }
            }
        } else {
            mma_commit_warp(lead, empty + 8 * ks);
            if (nt > 1) {
                ks = take();
                scores(1, ks);
                mma_commit_warp(lead, empty + 8 * ks);
            }
            for (int j = 0; j < nt; j++) {
                const int w = j & 1, vs = take();
                values(w, vs, j / 2);
                mma_commit_warp(lead, empty + 8 * vs);
                if (j + 2 < nt) {
                    ks = take();
                    scores(w, ks);
                    mma_commit_warp(lead, empty + 8 * ks);
                } else {
                    mma_commit_warp(lead, o_full + 8 * w);
                }
            }
        }
        __syncwarp();
    } else {
        // ---- queries into the swizzled layout; rows and columns that do not exist are zero
        const int w = warp / 4, live = min(rows - r0, TWO ? 256 : 128);
        constexpr int batch = DB * 4;                                 // chunks of 16 bytes that a thread has under way
        for (int i0 = tid; i0 < (TWO ? 256 : 128) * DB * 8; i0 += batch * 256) {
            uint4 v[batch];
#pragma unroll
            for (int u = 0; u < batch; u++) {
                const int i = i0 + u * 256, row = i / (DB * 8), c = i % (DB * 8);
                v[u] = make_uint4(0, 0, 0, 0);
                if (row < live && c * 8 < d.dim) {
                    const uint32_t g = r0 + row, bt = g / (uint32_t)d.group, b = bt / (uint32_t)d.fresh;
                    v[u] = __ldg((const uint4 *)((const T *)d.q + b * d.qs[0] + (bt - b * d.fresh) * d.qs[1] +
                                                 (kv * d.group + (g - bt * d.group)) * d.qs[2] + c * 8));
                }
            }
#pragma unroll
            for (int u = 0; u < batch; u++) {
                const int i = i0 + u * 256, row = i / (DB * 8), c = i % (DB * 8);
                *(uint4 *)(qs + row / 128 * stage + c / 8 * block + swizzled(row % 128, c % 8, 128)) = v[u];
            }
        }
        fence_async_proxy();
        mbar_arrive(q_full);

        // ---- softmax: one thread per row
        const int quarter = warp % 4, r = (TWO ? w * 128 : 0) + quarter * 32 + lane;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16, s_at = tmem + lanes + w * 128, o_at = tmem + lanes + 256 + w * 128;
        const bool busy = (TWO ? w * 128 : 0) + quarter * 32 < live;  // some row of this warp exists
        const int mine = TWO ? nt : (nt - w + 1) / 2, columns = (d.dim + 15) / 16 * 16;
        Row state;
        bool ok = true;
        for (int it = 0; it < mine; it++) {
            ok = mbar_wait(s_full + 8 * w, it & 1, &gave_up);
            if (!__all_sync(~0u, ok)) {
                ok = false;
                break;
            }
            tc_fence_after();
            const int valid = d.prefix_len - (j0 + (TWO ? it : 2 * it + w)) * kTileKeys;
            if (!busy) mbar_arrive(p_most + 8 * w);
            else if (valid >= kTileKeys) softmax_tile<T, false>(state, s_at, o_at, it == 0, kTileKeys, columns, d.scale_log2, p_most + 8 * w);
            else softmax_tile<T, true>(state, s_at, o_at, it == 0, valid, columns, d.scale_log2, p_most + 8 * w);
            tc_fence_before();
            mbar_arrive(p_full + 8 * w);
        }
        // ---- the way out: a row's sums as they are, with what they were taken against
        if (mine > 0 && ok) ok = mbar_wait(o_full + 8 * w, 0, &gave_up);
        // What is written now goes over the tiles that products read.  All of them are done where both halves' sums are.
        // One tile of rows: products are issued in the order of the tiles of tokens, so after half 1's last only half 0's
        // last can be under way, and the other way round.  Half 1 waits for that.  Half 0 need not: it is half 1's that is
        // last where the tiles are even in number, and loads, taken K 0, K 1, V 0, K 2, V 1, ..., V n - 1, bring V n - 1 as
        // number 2 n - 1 then, into the last of four stages, behind what half 0 writes.
        if (ok && (TWO || (w == 1 && mine > 0))) ok = mbar_wait(o_full + 8 * (w ^ 1), 0, &gave_up);
        ok = __all_sync(~0u, ok);
        tc_fence_after();
        // Through shared memory, where the tiles were, and out row by row.
        constexpr int pitch = DB * 64 + 4;
        static_assert(8 * 32 * pitch * 4 <= (TWO ? 2 : 1) * stage + stages * stage);
        static_assert(TWO || (stages == 4 && 128 * pitch * 4 <= stage + 3 * stage));     // half 0's, up to the last stage
        float *sums = (float *)smem + (w * 128 + quarter * 32) * pitch;       // this warp's rows
        if (busy && ok && mine > 0)
            for (int c = 0; c < columns; c += 16) {
                float v[16];
                tmem_load16(o_at + c, (uint32_t *)v);
                tmem_wait_load16((uint32_t *)v);
#pragma unroll
                for (int k = 0; k < 16; k += 4) *(float4 *)(sums + lane * pitch + c + k) = *(const float4 *)(v + k);
            }
        float2 mine_ml = make_float2(state.l == 0.0f ? -INFINITY : (state.m == -INFINITY ? 0.0f : state.m) - kShift<T>, state.l);
        if (!TWO) {
            half_ml[w][quarter * 32 + lane] = mine_ml;
            asm volatile("bar.sync 1, 256;" ::: "memory");
        } else {
            __syncwarp();
        }
        // TWO: a warp its own 32 rows.  Otherwise the two halves of the tokens become one part, 16 rows to a warp.
        constexpr int out_rows = TWO ? 32 : 16;
        const int first = TWO ? r - lane : warp * 16, row_here = first + lane % out_rows;
        const uint32_t g = r0 + row_here, bt = g / (uint32_t)d.group;         // request and new token: rows come in that order
        const int64_t row = split * d.rows + (int64_t)bt * d.q_heads + kv * d.group + (g - bt * d.group);
        float keep = 1.0f, other = 0.0f;
        if (!TWO) {
            const float2 x = half_ml[0][row_here], y = half_ml[1][row_here];
            mine_ml = x;
            if (y.x != -INFINITY) {
                const float top = fmaxf(x.x, y.x);
                keep = exp2_approx(x.x - top);
                other = exp2_approx(y.x - top);
                mine_ml = make_float2(top, keep * x.y + other * y.y);
            }
        }
        if (ok && row_here < live && lane < out_rows) d.part_ml[row] = mine_ml;
        const int count = ok ? min(out_rows, live - first) : 0;
        const unsigned long long to = (unsigned long long)(d.part_o + row * d.dim);
        const float *from0 = (const float *)smem + first * pitch + lane * 4, *from1 = from0 + 128 * pitch;
#pragma unroll 4
        for (int k = 0; k < count; k++) {
            float *dst = (float *)__shfl_sync(~0u, to, k);
            const float a = __shfl_sync(~0u, keep, k), b = __shfl_sync(~0u, other, k);
            if (lane * 4 >= d.dim) continue;
            float4 v = *(const float4 *)(from0 + k * pitch);
            if (!TWO && b != 0.0f) {                  // (where it is zero the other half may hold nothing)
                const float4 u = *(const float4 *)(from1 + k * pitch);
                v = make_float4(a * v.x + b * u.x, a * v.y + b * u.y, a * v.z + b * u.z, a * v.w + b * u.w);
            }
            *(float4 *)(dst + lane * 4) = v;
        }
        tc_fence_before();
    }
    __syncthreads();
    tc_fence_after();
    // (nobody sets gave_up from here on)
    if (warp == 9) {
        if (gave_up) {                                                // what was issued ends before tensor memory is given up
            mma_commit_warp(elect_one(), drained);
            mbar_drain(drained, 0);
            __syncwarp();
        }
        tmem_free(tmem, 512);
    }
    if (warp == 8 && lane == 0 && gave_up) {                          // and loads, before the block's memory is
        drain_loads<stages>(full, issued);
        atomicExch(d.status, 1);
    }
}

// ------------------------------------------------------------------------------------------- join
constexpr int kJoinThreads = 128, kJoinParts = 256;       // most parts of a row: 64 of the prefix, and what own_cap allows

// A block to a row: the parts' factors first, then dim / 4 threads to a part and as many parts at a time as there
// are threads for, four columns to a thread.  (With a warp to a row, parts one after the other, a decode step of 32
// requests took 25 us here.)
template <typename T>
__global__ void __launch_bounds__(kJoinThreads)
serve_attn_join_kernel(const __grid_constant__ AttnDev d)
{
    __shared__ float factor[kJoinParts], warp_top[kJoinThreads / 32], warp_sum[kJoinThreads / 32];
    __shared__ float4 sums[kJoinThreads];
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
    wait_previous();
    float2 ml[kJoinParts / kJoinThreads];
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < kJoinParts / kJoinThreads; k++) {
        const int p = tid + k * kJoinThreads;
        ml[k] = p < d.parts ? d.part_ml[p * d.rows + row] : make_float2(-INFINITY, 0.0f);
        top = fmaxf(top, ml[k].x);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
    if (lane == 0) warp_top[warp] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kJoinThreads / 32; w++) top = fmaxf(top, warp_top[w]);
    const float from = top == -INFINITY ? 0.0f : top;
    float total = 0.0f;
#pragma unroll
    for (int k = 0; k < kJoinParts / kJoinThreads; k++) {
        // a part that holds nothing has sums that were never written
        const float x = ml[k].x == -INFINITY ? -1.0f : exp2_approx(ml[k].x - from);
        if (tid + k * kJoinThreads < d.parts) factor[tid + k * kJoinThreads] = x;
        if (x >= 0.0f) total += x * ml[k].y;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(~0u, total, o);
    if (lane == 0) warp_sum[warp] = total;
    __syncthreads();
    total = 0.0f;
#pragma unroll
    for (int w = 0; w < kJoinThreads / 32; w++) total += warp_sum[w];

    const int width = d.dim / 4, at_once = kJoinThreads / width, mine = tid / width, c = tid % width * 4;
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (mine < at_once) {
#pragma unroll 4
        for (int p = mine; p < d.parts; p += at_once) {
            const float x = factor[p];
            const float4 v = x >= 0.0f ? *(const float4 *)(d.part_o + (p * d.rows + row) * d.dim + c) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            sum.x += x * v.x;
            sum.y += x * v.y;
            sum.z += x * v.z;
            sum.w += x * v.w;
        }
    }
    sums[tid] = sum;
    __syncthreads();
    if (tid < width) {
        for (int k = 1; k < at_once; k++) {
            const float4 v = sums[k * width + tid];
            sum.x += v.x;
            sum.y += v.y;
            sum.z += v.z;
            sum.w += v.w;
        }
        const float inv = total == 0.0f ? 0.0f : 1.0f / total;
        const int h = (int)(row % d.q_heads), i = (int)(row / d.q_heads % d.fresh), b = (int)(row / d.q_heads / d.fresh);
        *(uint2 *)((T *)d.out + b * d.os[0] + i * d.os[1] + h * d.os[2] + c) =
            make_uint2(pack2<T>(sum.x * inv, sum.y * inv), pack2<T>(sum.z * inv, sum.w * inv));
        if (d.lse && tid == 0) d.lse[row] = total == 0.0f ? -INFINITY : (from + log2f(total)) * kLn2;
    }
}

int check_shape(const bcast_serve_attn_args &a)
{
    if (a.dtype != BCAST_SERVE_BF16 && a.dtype != BCAST_SERVE_FP16) return BCAST_ERR_INVAL;
    if (a.batch < 0 || a.batch > 65535 || a.new_tokens < 0 || a.new_tokens > 65535 || a.kv_heads < 1 || a.kv_heads > 1024 ||
        a.q_heads < a.kv_heads || a.q_heads > 65535 || a.q_heads % a.kv_heads)
        return BCAST_ERR_INVAL;
    if (a.dim < 8 || a.dim > 128 || a.dim % 8) return BCAST_ERR_INVAL;
    if (a.prefix_len < 0 || a.prefix_len > kMaxDim - 65536 || a.own_cap < 0 || a.own_cap > kMaxDim - 65536) return BCAST_ERR_INVAL;
    if ((int64_t)a.new_tokens * a.q_heads > (1 << 19) || (int64_t)a.batch * a.new_tokens * a.q_heads > (1 << 24)) return BCAST_ERR_INVAL;
    return BCAST_OK;
}

// How a call is cut: rows of a key/value head into tiles, the prefix and the own tokens into parts.
struct Cut {
    bool two;                                 // 256 rows to a block of the prefix kernel
    int64_t rows, row_tiles, prefix_splits, prefix_parts, own_tiles, own_chunk, own_splits, parts;
    int64_t folded, fold_chunk;               // parts of the prefix that the own kernel takes, among own_splits
};

Cut cut_of(const bcast_serve_attn_args &a)
{
    Cut c = {};
    const int64_t group = a.q_heads / a.kv_heads, head_rows = (int64_t)a.batch * a.new_tokens * group;
    c.rows = head_rows * a.kv_heads;
    // 256 rows to a block read the prefix half as often; 128 rows leave fewer of the last tile's rows empty and end sooner,
    // their two halves taking every other tile of tokens.  Measured (us, 256 / 128): 1024 rows to a head, prefix 65536
    // 248 / 255, prefix 16384 114 / 112; 256 rows, 8192 53 / 49; 640 rows, 16384 87 / 77; 520 rows, 20011 42 / 38.  So
    // 256 only where the rows come in pairs of tiles and every SM has 64 tiles of tokens to go through.
    const int64_t row_tiles = ceil_div(head_rows, 128);
    c.two = row_tiles % 2 == 0 && row_tiles / 2 * a.kv_heads * ceil_div(a.prefix_len, 128) >= 64 * kSms;
    c.own_tiles = ceil_div(a.new_tokens * group, kOwnRows);
    const int64_t own_blocks = (int64_t)a.batch * a.kv_heads * c.own_tiles;
    // A prefix that is little to read, even once per request and 16 rows, goes with the own tokens: one launch less, and
    // no blocks of 128 rows for a few.  Measured (us, with the own kernel / with its own), by what the own kernel then
    // reads: 2000 tokens 6.9 / 9.5; 8000 7.4 / 10.0; 32000 10.3 / 12.4, 13.2 / 17.8 and 12.8 / 13.9; 65000 16.4 / 16.1
    // and 21.9 / 18.3; 128000 17.2 / 15.7.
    const bool fold = a.prefix_len > 0 && c.rows > 0 && own_blocks * a.prefix_len <= 1 << 15;
    if (fold) {
        int64_t s = ceil_div(2 * kSms, own_blocks);
        s = s < ceil_div(a.prefix_len, 128) ? s : ceil_div(a.prefix_len, 128);
        s = s < 64 ? s : 64;
        c.fold_chunk = round_up(ceil_div(a.prefix_len, s), 32);
        c.folded = ceil_div(a.prefix_len, c.fold_chunk);
    }
    if (a.prefix_len > 0 && c.rows > 0 && !fold) {
        c.row_tiles = ceil_div(head_rows, c.two ? 256 : 128);
        const int64_t items = c.row_tiles * a.kv_heads, tiles = ceil_div(a.prefix_len, 128);
        // the number of parts that ends first, one block to an SM: a block costs its tiles and about six more to
        // begin and to end; a tenth more where there are more blocks than SMs, since the own kernel only starts when
        // the last of them has (and then has the SMs that are left to itself)
        int64_t best = INT64_MAX;
        for (int64_t s = 1; s <= tiles && s <= 64; s++) {
            const int64_t rounds = ceil_div(items * s, kSms), cost = rounds * (ceil_div(tiles, s) + 6) * (rounds > 1 ? 11 : 10);
            if (cost < best) {
                best = cost;
                c.prefix_splits = s;
            }
        }
        c.prefix_parts = c.prefix_splits;
    }
    if (a.own_cap > 0 && c.rows > 0) {
        // parts of 256 tokens, 512 once that makes six blocks to an SM (a decode step of 32 requests with up to 700 own
        // tokens: 36 us, with 512 38, with 128 39; 64 requests with up to 1024: 259, 251, 268), 128 where there are
        // too few blocks otherwise
        const int64_t more = ceil_div(2 * kSms, own_blocks);
        int64_t s = ceil_div(a.own_cap, own_blocks * ceil_div(a.own_cap, 512) >= 6 * kSms ? 512 : 256);
        if (s < more) s = more < ceil_div(a.own_cap, 128) ? more : ceil_div(a.own_cap, 128);
        s = s < kJoinParts - 64 ? s : kJoinParts - 64;
        c.own_chunk = round_up(ceil_div(a.own_cap, s), 64);
        c.own_splits = ceil_div(a.own_cap, c.own_chunk);
    }
    c.own_splits += c.folded;
    c.parts = c.prefix_parts + c.own_splits;
    return c;
}

int64_t workspace_of(const bcast_serve_attn_args &a, const Cut &c)
{
    return BCAST_SERVE_STATUS_BYTES + round_up(c.parts * c.rows * 8, 256) + c.parts * c.rows * a.dim * 4;
}

template <typename T, int DB>
int run_own(const bcast_serve_attn_args &a, const AttnDev &d, const Cut &c, cudaStream_t st)
{
    int rc;
    if ((rc = allow_smem<serve_attn_own_kernel<T, DB>>(own_smem<DB>()))) return rc;
    return launch(serve_attn_own_kernel<T, DB>, dim3((unsigned)c.own_splits, (unsigned)(a.kv_heads * c.own_tiles), a.batch),
                  dim3(kOwnWarps * 32), own_smem<DB>(), st, c.prefix_splits > 0, 1, d);
}

template <typename T, int DB, bool TWO>
int run_prefix(const bcast_serve_attn_args &a, const AttnDev &d, const Cut &c, cudaStream_t st)
{
    const auto type = std::is_same_v<T, __nv_bfloat16> ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    CUtensorMap mk, mv;
    int rc;
    if ((rc = tensor_map(&mk, type, a.prefix_k, {a.dim, a.prefix_len, a.kv_heads}, {a.prefix_k_stride[0], a.prefix_k_stride[1]}, {64, kTileKeys, 1})))
        return rc;
    if ((rc = tensor_map(&mv, type, a.prefix_v, {a.dim, a.prefix_len, a.kv_heads}, {a.prefix_v_stride[0], a.prefix_v_stride[1]}, {64, kTileKeys, 1})))
        return rc;
    const size_t smem = prefix_smem<DB, TWO>();
    if ((rc = allow_smem<serve_attn_prefix_kernel<T, DB, TWO>>(smem))) return rc;
    return launch(serve_attn_prefix_kernel<T, DB, TWO>, dim3((unsigned)(c.row_tiles * a.kv_heads * c.prefix_splits)), dim3(kPrefixThreads), smem, st,
                  false, 1, mk, mv, d);
}

template <typename T, int DB>
int run(const bcast_serve_attn_args &a, const AttnDev &d, const Cut &c, cudaStream_t st)
{
    int rc = BCAST_OK;
    if (c.prefix_splits) rc = c.two ? run_prefix<T, DB, true>(a, d, c, st) : run_prefix<T, DB, false>(a, d, c, st);
    if (!rc && c.own_splits) rc = run_own<T, DB>(a, d, c, st);
    if (rc) return rc;
    return launch(serve_attn_join_kernel<T>, dim3((unsigned)c.rows), dim3(kJoinThreads), 0, st, c.parts > 0, 1, d);
}

}  // namespace
}  // namespace bcast_serve

using namespace bcast_serve;

extern "C" {

int64_t bcast_serve_attn_workspace(const bcast_serve_attn_args *a)
{
    if (!a || check_shape(*a)) return BCAST_ERR_INVAL;
    return workspace_of(*a, cut_of(*a));
}

int bcast_serve_attn(const bcast_serve_attn_args *args, void *cuda_stream)
{
    if (!args) return BCAST_ERR_INVAL;
    int rc = check_shape(*args);
    if (rc) return rc;
    bcast_serve_attn_args given = *args;
    const bcast_serve_attn_args *const a = &given;
    if (given.page_table && given.num_pages == 0) given.own_cap = 0;      // a cache without pages holds no token
    if (a->batch == 0 || a->new_tokens == 0) return BCAST_OK;
    if (!(a->scale == a->scale) || a->scale > 1e30f || a->scale < -1e30f) return BCAST_ERR_INVAL;
    const bool paged = a->own_cap && a->page_table;
    for (int i = 0; i < 3; i++) {
        if (!stride_ok(a->q_stride[i], 0, 8) || !stride_ok(a->out_stride[i], a->dim, 8)) return BCAST_ERR_INVAL;
        if (a->own_cap && (!stride_ok(a->own_k_stride[i], 0, 8) || !stride_ok(a->own_v_stride[i], 0, 8))) return BCAST_ERR_INVAL;
    }
    for (int i = 0; i < 2 && a->prefix_len; i++)
        if (!stride_ok(a->prefix_k_stride[i], a->dim, 8) || !stride_ok(a->prefix_v_stride[i], a->dim, 8)) return BCAST_ERR_INVAL;
    if (paged && (a->page_size < 1 || a->num_pages < 0 || a->num_pages > kMaxDim ||
                  !stride_ok(a->page_table_stride, ceil_div(a->own_cap, a->page_size), 1)))
        return BCAST_ERR_INVAL;
    int device = 0;
    SERVE_TRY(cudaGetDevice(&device));
    if ((rc = check_array(a->q, 16, device)) || (rc = check_array(a->out, 16, device)) || (rc = check_array(a->own_len, 4, device)))
        return rc;
    if (a->prefix_len && ((rc = check_array(a->prefix_k, 16, device)) || (rc = check_array(a->prefix_v, 16, device)))) return rc;
    if (a->own_cap && ((rc = check_array(a->own_k, 16, device)) || (rc = check_array(a->own_v, 16, device)))) return rc;
    if (paged && (rc = check_array(a->page_table, 4, device))) return rc;
    if (a->lse && (rc = check_array(a->lse, 4, device))) return rc;
    if ((rc = check_workspace(a->workspace, a->workspace_bytes, bcast_serve_attn_workspace(a), device))) return rc;

    const Cut c = cut_of(*a);
    AttnDev d = {};
    d.q = a->q;
    d.ok = a->own_k;
    d.ov = a->own_v;
    d.pk = a->prefix_k;
    d.pv = a->prefix_v;
    for (int i = 0; i < 2; i++) {
        d.pks[i] = a->prefix_k_stride[i];
        d.pvs[i] = a->prefix_v_stride[i];
    }
    d.own_len = a->own_len;
    d.page_table = paged ? a->page_table : nullptr;
    d.out = a->out;
    d.lse = a->lse;
    d.status = (int *)a->workspace;
    d.give_up = give_up_at_once();
    d.part_ml = (float2 *)((char *)a->workspace + BCAST_SERVE_STATUS_BYTES);
    d.part_o = (float *)((char *)d.part_ml + round_up(c.parts * c.rows * 8, 256));
    for (int i = 0; i < 3; i++) {
        d.qs[i] = a->q_stride[i];
        d.os[i] = a->out_stride[i];
        d.oks[i] = a->own_k_stride[i];
        d.ovs[i] = a->own_v_stride[i];
    }
    d.own_cap = a->own_cap;
    d.num_pages = a->num_pages;
    d.pts = a->page_table_stride;
    d.rows = c.rows;
    d.batch = a->batch;
    d.fresh = a->new_tokens;
    d.q_heads = a->q_heads;
    d.kv_heads = a->kv_heads;
    d.group = a->q_heads / a->kv_heads;
    d.dim = a->dim;
    d.page = paged ? a->page_size : 1;
    d.page_shift = -1;
    for (int i = 0; i < 31; i++)
        if (d.page == 1 << i) d.page_shift = i;
    d.prefix_len = (int32_t)a->prefix_len;
    d.prefix_splits = (int32_t)c.prefix_splits;
    d.prefix_parts = (int32_t)c.prefix_parts;
    d.row_tiles = (int32_t)c.row_tiles;
    d.folded = (int32_t)c.folded;
    d.fold_chunk = (int32_t)c.fold_chunk;
    d.own_chunk = (int32_t)c.own_chunk;
    d.parts = (int32_t)c.parts;
    d.scale_log2 = a->scale * kLog2e;
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    if (a->dtype == BCAST_SERVE_BF16) return a->dim > 64 ? run<__nv_bfloat16, 2>(*a, d, c, st) : run<__nv_bfloat16, 1>(*a, d, c, st);
    return a->dim > 64 ? run<__half, 2>(*a, d, c, st) : run<__half, 1>(*a, d, c, st);
}

}  // extern "C"
