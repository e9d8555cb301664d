// bcast_serve_append: queries and keys of new tokens normed for each head and rotated by their positions, keys
// and values put into the requests' caches -- one pass over what a projection left.
//
// A head of up to 128 numbers is `L` lanes' (a power of two, 16 numbers to a lane), which hold the two 16-byte chunks
// whose numbers are each other's partners in the rotation, so that the rotation needs no exchange; the norm is one sum
// over the L lanes.  A warp takes one token: the cosines and sines of its rot / 2 pairs are made once, two pairs to a
// lane, dealt out by shuffles, and then it goes through heads, 32 / L at a time.
// Angles: inv_freq / 2 pi as a 64-bit fraction of a turn; multiplied by the position modulo 2^64 this leaves the
// fraction of a turn with nothing lost to the size of the position.
// Bound by memory: what is read is written once.
#include "serve_device.cuh"
#include "serve_internal.h"

namespace bcast_serve {
namespace {

constexpr int kAppendThreads = 128, kAtOnce = 4;      // heads of a lane whose loads are under way together

struct AppendDev {
    const void *q, *k, *v, *q_norm, *k_norm;
    const float *inv_freq;
    const int32_t *positions, *axis, *own_len, *new_len, *page_table;
    void *out, *ok, *ov;
    int64_t qs[3], ks[3], vs[3], os[3], oks[3], ovs[3], ps[2];
    int64_t own_cap, num_pages, pts, first, items;
    int32_t fresh, q_heads, kv_heads, dim, page, rot, interleaved, axes, groups, rounds;
    float eps;
};

// One lane's two chunks of a head.
struct Unit {
    uint4 a, b;
};

template <typename T>
__device__ __forceinline__ void widen8(const uint4 &raw, float *x)
{
    const T *v = (const T *)&raw;
#pragma unroll
    for (int i = 0; i < 8; i++) x[i] = to_f32(v[i]);
}
template <typename T>
__device__ __forceinline__ uint4 narrow8(const float *x)
{
    uint4 raw;
    T *v = (T *)&raw;
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = from_f32<T>(x[i]);
    return raw;
}

// Cosine and sine of pair p's angle.
__device__ __forceinline__ float2 turn_of(const AppendDev &d, int p, int64_t row_position, const int32_t *positions)
{
    if (p >= d.rot / 2) return make_float2(1.0f, 0.0f);
    int64_t position = row_position;
    if (positions) {
        const int a = d.axis ? d.axis[p] : 0;
        position = positions[(uint32_t)a < (uint32_t)d.axes ? a : 0];
    }
    const double turns = (double)d.inv_freq[p] * 0.15915494309189533577;      // 1 / (2 pi)
    const uint64_t step = __double2ull_rz((turns - floor(turns)) * 18446744073709551616.0);
    const float half_turns = (float)(int32_t)((step * (uint64_t)position) >> 32) * 4.656612873077392578125e-10f;  // 2^-31
    float2 r;
    sincospif(half_turns, &r.y, &r.x);
    return r;
}

template <typename T, int L>
__global__ void __launch_bounds__(kAppendThreads)
serve_append_kernel(const __grid_constant__ AppendDev d)
{
    constexpr int kHeads = 32 / L;                    // heads of a warp at a time
    const int lane = threadIdx.x % 32, u = lane % L;
    const int64_t item = (int64_t)blockIdx.x * (kAppendThreads / 32) + threadIdx.x / 32;
    if (item >= d.items) return;
    const int token = (int)(item / d.groups), group = (int)(item - (int64_t)token * d.groups);
    const int b = token / d.fresh, i = token - b * d.fresh;
    const int32_t length = d.own_len[b], fresh = d.new_len ? d.new_len[b] : d.fresh;
    const int64_t slot = (int64_t)length - d.fresh + i;
    const bool there = slot >= 0 && i >= (int64_t)d.fresh - fresh;
    const int heads = d.q_heads + 2 * d.kv_heads, h0 = group * d.rounds * kHeads + lane / L;
    // where the token goes
    int64_t page = b, place = slot;
    bool stored = there && slot < d.own_cap;
    if (stored && d.page_table) {
        const int32_t n = (int32_t)slot / d.page;
        page = d.page_table[(int64_t)b * d.pts + n];
        place = slot - (int64_t)n * d.page;
        stored = page >= 0 && page < d.num_pages;
    }
    // this lane's chunks
    const int units = d.rot / 16, chunks = d.dim / 8;
    const bool turned = u < units;
    const int ca = turned && !d.interleaved ? u : 2 * u, cb = turned && !d.interleaved ? u + units : 2 * u + 1;
    const bool has_a = ca < chunks, has_b = cb < chunks;

    // cosines and sines of pairs 8 u to 8 u + 7
    float cosine[8], sine[8];
    if (d.rot) {
        const int32_t *positions = d.axes ? d.positions + b * d.ps[0] + i * d.ps[1] : nullptr;
        const float2 even = turn_of(d, 2 * lane, d.first + slot, positions), odd = turn_of(d, 2 * lane + 1, d.first + slot, positions);
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const int from = 4 * u + j / 2;
            cosine[j] = __shfl_sync(~0u, j % 2 ? odd.x : even.x, from);
            sine[j] = __shfl_sync(~0u, j % 2 ? odd.y : even.y, from);
        }
    }
    for (int r0 = 0; r0 < d.rounds; r0 += kAtOnce) {
        Unit x[kAtOnce];
#pragma unroll
        for (int r = 0; r < kAtOnce; r++) {
            const int h = h0 + (r0 + r) * kHeads;
            const T *src = h < d.q_heads ? (const T *)d.q + b * d.qs[0] + i * d.qs[1] + h * d.qs[2]
                         : h < d.q_heads + d.kv_heads ? (const T *)d.k + b * d.ks[0] + i * d.ks[1] + (h - d.q_heads) * d.ks[2]
                                                      : (const T *)d.v + b * d.vs[0] + i * d.vs[1] + (h - d.q_heads - d.kv_heads) * d.vs[2];
            const bool read = r0 + r < d.rounds && h < heads && (h < d.q_heads ? there : stored);
            x[r].a = read && has_a ? *(const uint4 *)(src + ca * 8) : make_uint4(0, 0, 0, 0);
            x[r].b = read && has_b ? *(const uint4 *)(src + cb * 8) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int r = 0; r < kAtOnce; r++) {
            if (r0 + r >= d.rounds) break;
            const int h = h0 + (r0 + r) * kHeads;
            const bool query = h < d.q_heads, key = !query && h < d.q_heads + d.kv_heads;
            const T *weights = query ? (const T *)d.q_norm : key ? (const T *)d.k_norm : nullptr;
            const bool turn = turned && (query || key);
            Unit y = x[r];
            float xa[8], xb[8];
            widen8<T>(y.a, xa);
            widen8<T>(y.b, xb);
            if (d.q_norm || d.k_norm) {               // by every lane: the sum is over lanes
                float sum = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; j++) sum += xa[j] * xa[j] + xb[j] * xb[j];
#pragma unroll
                for (int o = L / 2; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
                if (weights) {
                    const float inv = rsqrtf(sum / (float)d.dim + d.eps);
                    float wa[8] = {}, wb[8] = {};
                    if (has_a) widen8<T>(__ldg((const uint4 *)(weights + ca * 8)), wa);
                    if (has_b) widen8<T>(__ldg((const uint4 *)(weights + cb * 8)), wb);
#pragma unroll
                    for (int j = 0; j < 8; j++) {
                        xa[j] = xa[j] * inv * wa[j];
                        xb[j] = xb[j] * inv * wb[j];
                    }
                }
            }
            if (turn && !d.interleaved) {
#pragma unroll
                for (int j = 0; j < 8; j++) {
                    const float p = xa[j], q = xb[j];
                    xa[j] = p * cosine[j] - q * sine[j];
                    xb[j] = p * sine[j] + q * cosine[j];
                }
            } else if (turn) {
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const float p = xa[2 * j], q = xa[2 * j + 1], s = xb[2 * j], t = xb[2 * j + 1];
                    xa[2 * j] = p * cosine[j] - q * sine[j];
                    xa[2 * j + 1] = p * sine[j] + q * cosine[j];
                    xb[2 * j] = s * cosine[4 + j] - t * sine[4 + j];
                    xb[2 * j + 1] = s * sine[4 + j] + t * cosine[4 + j];
                }
            }
            if (turn || weights) {
                y.a = narrow8<T>(xa);
                y.b = narrow8<T>(xb);
            }
            T *dst;
            if (query) {
                dst = (T *)d.out + b * d.os[0] + i * d.os[1] + h * d.os[2];
                if (!there) y = Unit{make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
            } else {
                if (h >= heads || !stored) continue;
                dst = key ? (T *)d.ok + page * d.oks[0] + place * d.oks[1] + (h - d.q_heads) * d.oks[2]
                          : (T *)d.ov + page * d.ovs[0] + place * d.ovs[1] + (h - d.q_heads - d.kv_heads) * d.ovs[2];
            }
            if (has_a) *(uint4 *)(dst + ca * 8) = y.a;
            if (has_b) *(uint4 *)(dst + cb * 8) = y.b;
        }
    }
}

int check_shape(const bcast_serve_append_args &a)
{
    if (a.dtype != BCAST_SERVE_BF16 && a.dtype != BCAST_SERVE_FP16) return BCAST_ERR_INVAL;
    if (a.batch < 0 || a.batch > 65535 || a.new_tokens < 0 || a.new_tokens > 65535 || (int64_t)a.batch * a.new_tokens > (1 << 24) ||
        a.q_heads < 0 || a.q_heads > 65535 || a.kv_heads < 1 || a.kv_heads > 1024 ||
        (int64_t)a.batch * a.new_tokens * (a.q_heads + 2 * a.kv_heads) > kMaxDim)
        return BCAST_ERR_INVAL;
    if (a.dim < 8 || a.dim > 128 || a.dim % 8 || a.rot < 0 || a.rot > a.dim || a.rot % 16 || a.axes < 0 || a.axes > 16) return BCAST_ERR_INVAL;
    if (a.own_cap < 0 || a.own_cap > kMaxDim - 65536 || a.first < 0 || a.first > kMaxDim) return BCAST_ERR_INVAL;
    if (!(a.eps >= 0.0f) || a.eps > 1e30f) return BCAST_ERR_INVAL;
    return BCAST_OK;
}

template <typename T>
int run(const AppendDev &d, int lanes, unsigned blocks, cudaStream_t st)
{
    const dim3 threads(kAppendThreads);
    switch (lanes) {
    case 1: return launch(serve_append_kernel<T, 1>, dim3(blocks), threads, 0, st, false, 1, d);
    case 2: return launch(serve_append_kernel<T, 2>, dim3(blocks), threads, 0, st, false, 1, d);
    case 4: return launch(serve_append_kernel<T, 4>, dim3(blocks), threads, 0, st, false, 1, d);
    default: return launch(serve_append_kernel<T, 8>, dim3(blocks), threads, 0, st, false, 1, d);
    }
}

}  // namespace
}  // namespace bcast_serve

using namespace bcast_serve;

extern "C" int bcast_serve_append(const bcast_serve_append_args *args, void *cuda_stream)
{
    if (!args) return BCAST_ERR_INVAL;
    const bcast_serve_append_args &a = *args;
    int rc = check_shape(a);
    if (rc) return rc;
    if (a.batch == 0 || a.new_tokens == 0) return BCAST_OK;
    const int64_t own_cap = a.page_table && a.num_pages == 0 ? 0 : a.own_cap;         // a cache without pages holds no token
    const bool paged = own_cap && a.page_table;
    for (int i = 0; i < 3; i++) {
        if (a.q_heads && (!stride_ok(a.q_stride[i], 0, 8) || !stride_ok(a.out_stride[i], a.dim, 8))) return BCAST_ERR_INVAL;
        if (!stride_ok(a.k_stride[i], 0, 8) || !stride_ok(a.v_stride[i], 0, 8)) return BCAST_ERR_INVAL;
        if (own_cap && (!stride_ok(a.own_k_stride[i], a.dim, 8) || !stride_ok(a.own_v_stride[i], a.dim, 8))) return BCAST_ERR_INVAL;
    }
    if (paged && (a.page_size < 1 || a.num_pages < 0 || a.num_pages > kMaxDim || !stride_ok(a.page_table_stride, ceil_div(own_cap, a.page_size), 1)))
        return BCAST_ERR_INVAL;
    if (a.rot && a.axes && (!stride_ok(a.positions_stride[0], 0, 1) || !stride_ok(a.positions_stride[1], 0, 1))) return BCAST_ERR_INVAL;
    int device = 0;
    SERVE_TRY(cudaGetDevice(&device));
    if (a.q_heads && ((rc = check_array(a.q, 16, device)) || (rc = check_array(a.out, 16, device)))) return rc;
    if ((rc = check_array(a.k, 16, device)) || (rc = check_array(a.v, 16, device)) || (rc = check_array(a.own_len, 4, device))) return rc;
    if (own_cap && ((rc = check_array(a.own_k, 16, device)) || (rc = check_array(a.own_v, 16, device)))) return rc;
    if (a.q_norm && (rc = check_array(a.q_norm, 16, device))) return rc;
    if (a.k_norm && (rc = check_array(a.k_norm, 16, device))) return rc;
    if (a.new_len && (rc = check_array(a.new_len, 4, device))) return rc;
    if (paged && (rc = check_array(a.page_table, 4, device))) return rc;
    if (a.rot) {
        if ((rc = check_array(a.inv_freq, 4, device))) return rc;
        if (a.axes && (rc = check_array(a.positions, 4, device))) return rc;
        if (a.axes && a.axis && (rc = check_array(a.axis, 4, device))) return rc;
    }

    AppendDev d = {};
    d.q = a.q;
    d.k = a.k;
    d.v = a.v;
    d.q_norm = a.q_norm;
    d.k_norm = a.k_norm;
    d.inv_freq = a.inv_freq;
    d.positions = a.positions;
    d.axis = a.axis;
    d.own_len = a.own_len;
    d.new_len = a.new_len;
    d.page_table = paged ? a.page_table : nullptr;
    d.out = a.out;
    d.ok = a.own_k;
    d.ov = a.own_v;
    for (int i = 0; i < 3; i++) {
        d.qs[i] = a.q_stride[i];
        d.ks[i] = a.k_stride[i];
        d.vs[i] = a.v_stride[i];
        d.os[i] = a.out_stride[i];
        d.oks[i] = a.own_k_stride[i];
        d.ovs[i] = a.own_v_stride[i];
    }
    d.ps[0] = a.positions_stride[0];
    d.ps[1] = a.positions_stride[1];
    d.own_cap = own_cap;
    d.num_pages = a.num_pages;
    d.pts = a.page_table_stride;
    d.first = a.first;
    d.fresh = a.new_tokens;
    d.q_heads = a.q_heads;
    d.kv_heads = a.kv_heads;
    d.dim = a.dim;
    d.page = paged ? a.page_size : 1;
    d.rot = a.rot;
    d.interleaved = a.interleaved != 0;
    d.axes = a.axes;
    d.eps = a.eps;
    const int lanes = a.dim <= 16 ? 1 : a.dim <= 32 ? 2 : a.dim <= 64 ? 4 : 8;
    const int64_t tokens = (int64_t)a.batch * a.new_tokens, rounds = ceil_div(a.q_heads + 2 * a.kv_heads, 32 / lanes);
    // Few tokens: a warp to every 32 / L heads; many: several rounds to a warp, which makes the cosines once for them.
    const bool few = tokens * rounds <= 16 * kSms;
    d.rounds = few ? 1 : (int32_t)(rounds < 2 * kAtOnce ? rounds : 2 * kAtOnce);
    d.groups = (int32_t)ceil_div(rounds, d.rounds);
    d.items = tokens * d.groups;
    const unsigned blocks = (unsigned)ceil_div(d.items, kAppendThreads / 32);
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    return a.dtype == BCAST_SERVE_BF16 ? run<__nv_bfloat16>(d, lanes, blocks, st) : run<__half>(d, lanes, blocks, st);
}
