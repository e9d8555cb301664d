// bcast_serve_attn: attention of every request's newest tokens over a prefix that all requests share and
// the request's own tokens behind it.
//
// One block per row (request, new token, query head), one pass over the row's tokens in tiles with the
// running maximum m and sum l of the softmax: a tile's scores s_j change m to m', and what was summed so far
// is scaled by exp(m - m').
#include "serve_device.cuh"
#include "serve_internal.h"

namespace bcast_serve {
namespace {

constexpr int kRowThreads = 128;

struct AttnDev {
    const void *q, *pk, *pv, *ok, *ov;
    const int32_t *own_len, *page_table;
    void *out;
    float *lse;
    int64_t qs[3], os[3], pks[2], pvs[2], oks[3], ovs[3];
    int64_t prefix_len, own_cap, num_pages, pts;
    int32_t batch, fresh, q_heads, group, dim, page;
    float scale_log2;     // scale * log2(e): the softmax is taken in powers of two
};

// Row `at` of a request's own keys (or values), nullptr if its page is not there.
template <typename T>
__device__ __forceinline__ const T *own_row(const AttnDev &d, const void *base, const int64_t *s, int b, int64_t at, int kv)
{
    if (!d.page_table) return (const T *)base + b * s[0] + at * s[1] + kv * s[2];
    const int32_t p = d.page_table[(int64_t)b * d.pts + at / d.page];
    if (p < 0 || p >= d.num_pages) return nullptr;
    return (const T *)base + p * s[0] + at % d.page * s[1] + kv * s[2];
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads)
serve_attn_row_kernel(const __grid_constant__ AttnDev d)
{
    const int h = blockIdx.x, i = blockIdx.y, b = blockIdx.z, kv = h / d.group, tid = threadIdx.x;
    __shared__ float q[128], p[kRowThreads], red[kRowThreads / 32];
    if (tid < d.dim) q[tid] = to_f32(((const T *)d.q)[b * d.qs[0] + i * d.qs[1] + h * d.qs[2] + tid]) * d.scale_log2;
    const int64_t len = min(max((int64_t)d.own_len[b], (int64_t)0), d.own_cap);
    const int64_t own = max(len - d.fresh + i + 1, (int64_t)0), total = d.prefix_len + own;
    float m = -INFINITY, l = 0.0f, o = 0.0f;
    __syncthreads();
    for (int64_t j0 = 0; j0 < total; j0 += kRowThreads) {
        const int64_t j = j0 + tid;
        const T *k = nullptr;
        if (j < d.prefix_len) k = (const T *)d.pk + j * d.pks[0] + kv * d.pks[1];
        else if (j < total) k = own_row<T>(d, d.ok, d.oks, b, j - d.prefix_len, kv);
        float s = -INFINITY;
        if (k) {
            s = 0.0f;
            for (int c = 0; c < d.dim; c++) s += q[c] * to_f32(k[c]);
        }
        float top = s;
#pragma unroll
        for (int x = 16; x; x >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, x));
        if (tid % 32 == 0) red[tid / 32] = top;
        __syncthreads();
        for (int w = 0; w < kRowThreads / 32; w++) top = fmaxf(top, red[w]);
        // nothing seen so far: 0 in the place of -infinity, so that exp(-infinity) is 0 and NaN stays NaN
        const float next = fmaxf(m, top), base = next == -INFINITY ? 0.0f : next, fix = exp2f(m - base);
        p[tid] = exp2f(s - base);
        __syncthreads();
        l *= fix;
        o *= fix;
        m = next;
        for (int x = 0; x < kRowThreads && j0 + x < total; x++) {
            l += p[x];
            if (tid < d.dim && p[x] != 0.0f) {
                const int64_t at = j0 + x;
                const T *v = at < d.prefix_len ? (const T *)d.pv + at * d.pvs[0] + kv * d.pvs[1]
                                               : own_row<T>(d, d.ov, d.ovs, b, at - d.prefix_len, kv);
                o += p[x] * to_f32(v[tid]);
            }
        }
        __syncthreads();
    }
    if (tid < d.dim) ((T *)d.out)[b * d.os[0] + i * d.os[1] + h * d.os[2] + tid] = from_f32<T>(l == 0.0f ? 0.0f : o / l);
    if (d.lse && tid == 0)
        d.lse[((int64_t)b * d.fresh + i) * d.q_heads + h] = l == 0.0f ? -INFINITY : (m + log2f(l)) * kLn2;
}

int check_shape(const bcast_serve_attn_args &a)
{
    if (a.dtype != BCAST_SERVE_BF16 && a.dtype != BCAST_SERVE_FP16) return BCAST_ERR_INVAL;
    if (a.batch < 0 || a.batch > 65535 || a.new_tokens < 0 || a.new_tokens > 65535 || a.kv_heads < 1 || a.kv_heads > 1024 ||
        a.q_heads < a.kv_heads || a.q_heads > 65535 || a.q_heads % a.kv_heads)
        return BCAST_ERR_INVAL;
    if (a.dim < 8 || a.dim > 128 || a.dim % 8) return BCAST_ERR_INVAL;
    if (a.prefix_len < 0 || a.prefix_len > kMaxDim - 65536 || a.own_cap < 0 || a.own_cap > kMaxDim - 65536) return BCAST_ERR_INVAL;
    if ((int64_t)a.batch * a.new_tokens * a.q_heads > kMaxDim) return BCAST_ERR_INVAL;
    return BCAST_OK;
}

}  // namespace
}  // namespace bcast_serve

using namespace bcast_serve;

extern "C" {

int64_t bcast_serve_attn_workspace(const bcast_serve_attn_args *a)
{
    if (!a || check_shape(*a)) return BCAST_ERR_INVAL;
    return BCAST_SERVE_STATUS_BYTES;
}

int bcast_serve_attn(const bcast_serve_attn_args *a, void *cuda_stream)
{
    if (!a) return BCAST_ERR_INVAL;
    int rc = check_shape(*a);
    if (rc) return rc;
    if (a->batch == 0 || a->new_tokens == 0) return BCAST_OK;
    if (!(a->scale == a->scale) || a->scale > 1e30f || a->scale < -1e30f) return BCAST_ERR_INVAL;
    const bool paged = a->own_cap && a->page_table;
    for (int i = 0; i < 3; i++) {
        const int64_t least = i == 2 ? a->dim : 0;
        if (!stride_ok(a->q_stride[i], 0, 8) || !stride_ok(a->out_stride[i], least, 8)) return BCAST_ERR_INVAL;
        if (a->own_cap && (!stride_ok(a->own_k_stride[i], 0, 8) || !stride_ok(a->own_v_stride[i], 0, 8))) return BCAST_ERR_INVAL;
    }
    for (int i = 0; i < 2 && a->prefix_len; i++)
        if (!stride_ok(a->prefix_k_stride[i], 0, 8) || !stride_ok(a->prefix_v_stride[i], 0, 8)) return BCAST_ERR_INVAL;
    if (paged && (a->page_size < 1 || a->num_pages < 0 || a->num_pages > kMaxDim ||
                  !stride_ok(a->page_table_stride, ceil_div(a->own_cap, a->page_size), 1)))
        return BCAST_ERR_INVAL;
    Device dev;
    if ((rc = current_device(&dev))) return rc;
    if ((rc = check_array(a->q, 16, dev.id)) || (rc = check_array(a->out, 16, dev.id)) || (rc = check_array(a->own_len, 4, dev.id)))
        return rc;
    if (a->prefix_len && ((rc = check_array(a->prefix_k, 16, dev.id)) || (rc = check_array(a->prefix_v, 16, dev.id)))) return rc;
    if (a->own_cap && ((rc = check_array(a->own_k, 16, dev.id)) || (rc = check_array(a->own_v, 16, dev.id)))) return rc;
    if (paged && (rc = check_array(a->page_table, 4, dev.id))) return rc;
    if (a->lse && (rc = check_array(a->lse, 4, dev.id))) return rc;
    if ((rc = check_workspace(a->workspace, a->workspace_bytes, bcast_serve_attn_workspace(a), dev.id))) return rc;

    AttnDev d;
    d.q = a->q;
    d.pk = a->prefix_k;
    d.pv = a->prefix_v;
    d.ok = a->own_k;
    d.ov = a->own_v;
    d.own_len = a->own_len;
    d.page_table = paged ? a->page_table : nullptr;
    d.out = a->out;
    d.lse = a->lse;
    for (int i = 0; i < 3; i++) {
        d.qs[i] = a->q_stride[i];
        d.os[i] = a->out_stride[i];
        d.oks[i] = a->own_k_stride[i];
        d.ovs[i] = a->own_v_stride[i];
    }
    for (int i = 0; i < 2; i++) {
        d.pks[i] = a->prefix_k_stride[i];
        d.pvs[i] = a->prefix_v_stride[i];
    }
    d.prefix_len = a->prefix_len;
    d.own_cap = a->own_cap;
    d.num_pages = a->num_pages;
    d.pts = a->page_table_stride;
    d.batch = a->batch;
    d.fresh = a->new_tokens;
    d.q_heads = a->q_heads;
    d.group = a->q_heads / a->kv_heads;
    d.dim = a->dim;
    d.page = paged ? a->page_size : 1;
    d.scale_log2 = a->scale * kLog2e;
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    const dim3 grid(a->q_heads, a->new_tokens, a->batch);
    if (a->dtype == BCAST_SERVE_BF16) return launch(serve_attn_row_kernel<__nv_bfloat16>, grid, dim3(kRowThreads), 0, st, false, 1, d);
    return launch(serve_attn_row_kernel<__half>, grid, dim3(kRowThreads), 0, st, false, 1, d);
}

}  // extern "C"
