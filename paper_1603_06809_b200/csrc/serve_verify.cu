// bcast_serve_verify: speculative sampling over a batch of requests.
//
// Two kernels.  The first gives every row of logits (request b, place i) its softmax statistics -- largest
// logit m and where, s = sum exp((l - m) / T) -- one pass with a running maximum and sum, a row cut into
// parts so that few rows still fill the GPU.  Accepting a draft needs nothing but those and two numbers
// (p = exp((l_x - m) / T) / s against u q_x), so the second kernel joins the parts of a request's rows, finds
// the first draft that fails, and runs the race argmax w_v / e_v over that one row: a cluster of blocks per
// request, joined through distributed shared memory.  Bound by memory: drafts + 1 rows of logits are read
// once, one row of logits (from L2 where it is still there), one of q and one of noise a second time.
#include "serve_device.cuh"
#include "serve_internal.h"

#include <cooperative_groups.h>

namespace cg = cooperative_groups;

namespace bcast_serve {
namespace {

constexpr int kMaxDrafts = 63;
constexpr int kStatThreads = 256, kPickThreads = 512;

// Statistics of one part of a row; of a row once joined.  z = l * log2(e) / T.
struct RowStat {
    float top, sum;       // largest logit; sum of 2^((l - top) * c)
    int32_t best, pad;    // lowest token with that logit, -1 if no logit is above -infinity
};

struct VerifyDev {
    const void *logits;
    const float *draft_probs, *uniforms, *noise, *temperature;
    const int32_t *draft_tokens;
    int32_t *accepted, *tokens;
    int64_t ls0, ls1, qs0, qs1, ns;
    int32_t vocab, drafts, parts, part_len;
    RowStat *stats;       // [batch][drafts + 1][parts]
};

// What a logit counts for: NaN is -infinity.
__device__ __forceinline__ float clean(float l) { return l != l ? -INFINITY : l; }

// Weight of a logit against the row's largest one; equal infinities share the row.
__device__ __forceinline__ float weight(float l, float top, float c)
{
    if (top == INFINITY) return l == INFINITY ? 1.0f : 0.0f;
    return exp2f((l - top) * c);
}

__device__ __forceinline__ RowStat join(const RowStat &a, const RowStat &b, float c)
{
    if (b.best < 0) return a;
    if (a.best < 0) return b;
    RowStat r;
    r.top = fmaxf(a.top, b.top);
    r.sum = a.sum * weight(a.top, r.top, c) + b.sum * weight(b.top, r.top, c);
    r.best = a.top > b.top ? a.best : b.top > a.top ? b.best : min(a.best, b.best);
    r.pad = 0;
    return r;
}

__device__ __forceinline__ RowStat shuffle_xor(const RowStat &a, int d)
{
    RowStat r;
    r.top = __shfl_xor_sync(~0u, a.top, d);
    r.sum = __shfl_xor_sync(~0u, a.sum, d);
    r.best = __shfl_xor_sync(~0u, a.best, d);
    r.pad = 0;
    return r;
}

// 1 / temperature in units of log2, kept finite; a request without temperature only needs its largest logit.
__device__ __forceinline__ float exponent_scale(float temperature)
{
    return temperature > 0.0f ? fminf(kLog2e / temperature, 1e30f) : 0.0f;
}

template <typename T>
__global__ void __launch_bounds__(kStatThreads)
serve_verify_stats_kernel(const __grid_constant__ VerifyDev d)
{
    launch_next();
    const int b = blockIdx.z, i = blockIdx.y, part = blockIdx.x;
    const int lo = part * d.part_len, hi = min(d.vocab, lo + d.part_len);
    const T *row = (const T *)d.logits + (int64_t)b * d.ls0 + (int64_t)i * d.ls1;
    const float c = exponent_scale(d.temperature[b]);
    RowStat s{-INFINITY, 0.0f, -1, 0};
    for (int v = lo + threadIdx.x; v < hi; v += kStatThreads) {
        const float l = clean(to_f32(row[v]));
        if (l > s.top) {
            s.sum = s.best < 0 ? 0.0f : s.sum * weight(s.top, l, c);
            s.top = l;
            s.best = v;
        }
        if (s.best >= 0) s.sum += weight(l, s.top, c);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) s = join(s, shuffle_xor(s, o), c);
    __shared__ RowStat warp_stat[kStatThreads / 32];
    if (threadIdx.x % 32 == 0) warp_stat[threadIdx.x / 32] = s;
    __syncthreads();
    if (threadIdx.x < 32) {
        s = threadIdx.x < kStatThreads / 32 ? warp_stat[threadIdx.x] : RowStat{-INFINITY, 0.0f, -1, 0};
#pragma unroll
        for (int o = 16; o; o >>= 1) s = join(s, shuffle_xor(s, o), c);
        if (threadIdx.x == 0) d.stats[((int64_t)b * (d.drafts + 1) + i) * d.parts + part] = s;
    }
}

// Best runner of a race so far: the larger ratio, the lower token number among equals.
struct Runner {
    float ratio;
    int32_t token;
};
__device__ __forceinline__ Runner faster(const Runner &a, const Runner &b)
{
    if (a.ratio != b.ratio) return a.ratio > b.ratio ? a : b;
    return (uint32_t)a.token < (uint32_t)b.token ? a : b;      // -1 is the largest
}
__device__ __forceinline__ Runner shuffle_xor(const Runner &a, int d)
{
    return Runner{__shfl_xor_sync(~0u, a.ratio, d), __shfl_xor_sync(~0u, a.token, d)};
}

template <typename T>
__global__ void __launch_bounds__(kPickThreads)
serve_verify_pick_kernel(const __grid_constant__ VerifyDev d)
{
    cg::cluster_group cluster = cg::this_cluster();
    const int b = blockIdx.y, rank = (int)cluster.block_rank(), blocks = (int)cluster.num_blocks();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, warps = kPickThreads / 32;
    __shared__ RowStat row_stat[kMaxDrafts + 1];
    __shared__ uint32_t failed[2];            // bit i: draft i fails
    __shared__ Runner warp_run[2][kPickThreads / 32];
    __shared__ Runner block_run[2];

    if (threadIdx.x < 2) failed[threadIdx.x] = 0;
    const float t = d.temperature[b], c = exponent_scale(t);
    wait_previous();
    __syncthreads();
    for (int i = warp; i <= d.drafts; i += warps) {
        RowStat s{-INFINITY, 0.0f, -1, 0};
        for (int p = lane; p < d.parts; p += 32) s = join(s, d.stats[((int64_t)b * (d.drafts + 1) + i) * d.parts + p], c);
#pragma unroll
        for (int o = 16; o; o >>= 1) s = join(s, shuffle_xor(s, o), c);
        if (lane == 0) {
            row_stat[i] = s;
            if (i < d.drafts) {
                const int32_t x = d.draft_tokens[(int64_t)b * d.drafts + i];
                bool good = x >= 0 && x < d.vocab && s.best >= 0;
                if (good && t > 0.0f) {
                    const float l = clean(to_f32(((const T *)d.logits)[(int64_t)b * d.ls0 + (int64_t)i * d.ls1 + x]));
                    const float q = d.draft_probs[(int64_t)b * d.qs0 + (int64_t)i * d.qs1 + x];
                    good = d.uniforms[(int64_t)b * d.drafts + i] * q < weight(l, s.top, c) / s.sum;
                } else if (good) {
                    good = x == s.best;
                }
                if (!good) atomicOr(&failed[i / 32], 1u << (i % 32));
            }
        }
    }
    __syncthreads();
    const int accepted = failed[0] ? __ffs(failed[0]) - 1 : failed[1] ? 31 + __ffs(failed[1]) : d.drafts;
    const RowStat s = row_stat[accepted];
    int32_t chosen = s.best;                       // no temperature, or no probabilities: the largest logit, or -1
    if (t > 0.0f && s.best >= 0) {                 // the same for every block of the cluster
        const T *row = (const T *)d.logits + (int64_t)b * d.ls0 + (int64_t)accepted * d.ls1;
        const float *noise = d.noise + (int64_t)b * d.ns;
        const float *q = accepted < d.drafts ? d.draft_probs + (int64_t)b * d.qs0 + (int64_t)accepted * d.qs1 : nullptr;
        const float inv = 1.0f / s.sum;
        Runner rest{0.0f, -1}, all{0.0f, -1};      // the race by max(p - q, 0), and by p
        for (int v = rank * kPickThreads + threadIdx.x; v < d.vocab; v += blocks * kPickThreads) {
            const float e = noise[v];
            if (!(e > 0.0f)) continue;
            const float p = weight(clean(to_f32(row[v])), s.top, c) * inv;
            const float w = q ? p - q[v] : p;
            if (w / e > rest.ratio) rest = Runner{w / e, v};
            if (p / e > all.ratio) all = Runner{p / e, v};
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            rest = faster(rest, shuffle_xor(rest, o));
            all = faster(all, shuffle_xor(all, o));
        }
        if (lane == 0) {
            warp_run[0][warp] = rest;
            warp_run[1][warp] = all;
        }
        __syncthreads();
        if (threadIdx.x < 2) {
            Runner r = warp_run[threadIdx.x][0];
            for (int w = 1; w < warps; w++) r = faster(r, warp_run[threadIdx.x][w]);
            block_run[threadIdx.x] = r;
        }
        cluster.sync();
        if (rank == 0 && threadIdx.x < 32) {
            rest = all = Runner{0.0f, -1};
            if (lane < blocks) {
                const Runner *o = cluster.map_shared_rank(block_run, lane);
                rest = o[0];
                all = o[1];
            }
#pragma unroll
            for (int o = 16; o; o >>= 1) {
                rest = faster(rest, shuffle_xor(rest, o));
                all = faster(all, shuffle_xor(all, o));
            }
            chosen = rest.token >= 0 ? rest.token : all.token;
        }
        cluster.sync();                            // a block's shared memory stays until rank 0 has read it
    }
    if (rank == 0 && threadIdx.x < 32) {
        if (lane == 0) d.accepted[b] = accepted;
        for (int i = lane; i <= d.drafts; i += 32)
            d.tokens[(int64_t)b * (d.drafts + 1) + i] =
                i < accepted ? d.draft_tokens[(int64_t)b * d.drafts + i] : i == accepted ? chosen : -1;
    }
}

// Parts of a row: enough blocks to fill the GPU four times over, none shorter than 2048 logits.
int stat_parts(const bcast_serve_verify_args &a)
{
    const int64_t rows = (int64_t)a.batch * (a.drafts + 1);
    const int64_t want = ceil_div(4 * kSms, rows < 1 ? 1 : rows);
    const int64_t most = ceil_div(a.vocab, 2048);
    return (int)(want < most ? want : most);
}

int check_shape(const bcast_serve_verify_args &a)
{
    if (a.dtype != BCAST_SERVE_BF16 && a.dtype != BCAST_SERVE_FP16 && a.dtype != BCAST_SERVE_FP32) return BCAST_ERR_INVAL;
    if (a.batch < 0 || a.batch > 65535 || a.drafts < 0 || a.drafts > kMaxDrafts || a.vocab < 1 || a.vocab > kMaxDim - 65536)
        return BCAST_ERR_INVAL;
    return BCAST_OK;
}

template <typename T>
int run(const VerifyDev &d, int batch, cudaStream_t st)
{
    int rc = launch(serve_verify_stats_kernel<T>, dim3(d.parts, d.drafts + 1, batch), dim3(kStatThreads), 0, st, false, 1, d);
    if (rc) return rc;
    const unsigned blocks = 8;
    return launch(serve_verify_pick_kernel<T>, dim3(blocks, batch), dim3(kPickThreads), 0, st, true, blocks, d);
}

}  // namespace
}  // namespace bcast_serve

using namespace bcast_serve;

extern "C" {

int64_t bcast_serve_verify_workspace(const bcast_serve_verify_args *a)
{
    if (!a || check_shape(*a)) return BCAST_ERR_INVAL;
    return BCAST_SERVE_STATUS_BYTES + (int64_t)a->batch * (a->drafts + 1) * stat_parts(*a) * (int64_t)sizeof(RowStat);
}

int bcast_serve_verify(const bcast_serve_verify_args *a, void *cuda_stream)
{
    if (!a) return BCAST_ERR_INVAL;
    int rc = check_shape(*a);
    if (rc) return rc;
    if (a->batch == 0) return BCAST_OK;
    const int64_t V = a->vocab;
    if (!stride_ok(a->logits_stride[0], 0, 1) || !stride_ok(a->logits_stride[1], 0, 1) || !stride_ok(a->noise_stride, 0, 1) ||
        (a->drafts && (!stride_ok(a->draft_probs_stride[0], 0, 1) || !stride_ok(a->draft_probs_stride[1], 0, 1))))
        return BCAST_ERR_INVAL;
    Device dev;
    if ((rc = current_device(&dev))) return rc;
    const uintptr_t size = a->dtype == BCAST_SERVE_FP32 ? 4 : 2;
    if ((rc = check_array(a->logits, size, dev.id)) || (rc = check_array(a->noise, 4, dev.id)) ||
        (rc = check_array(a->temperature, 4, dev.id)) || (rc = check_array(a->accepted, 4, dev.id)) ||
        (rc = check_array(a->tokens, 4, dev.id)))
        return rc;
    if (a->drafts && ((rc = check_array(a->draft_probs, 4, dev.id)) || (rc = check_array(a->draft_tokens, 4, dev.id)) ||
                      (rc = check_array(a->uniforms, 4, dev.id))))
        return rc;
    if ((rc = check_workspace(a->workspace, a->workspace_bytes, bcast_serve_verify_workspace(a), dev.id))) return rc;

    VerifyDev d;
    d.logits = a->logits;
    d.draft_probs = a->draft_probs;
    d.uniforms = a->uniforms;
    d.noise = a->noise;
    d.temperature = a->temperature;
    d.draft_tokens = a->draft_tokens;
    d.accepted = a->accepted;
    d.tokens = a->tokens;
    d.ls0 = a->logits_stride[0];
    d.ls1 = a->logits_stride[1];
    d.qs0 = a->draft_probs_stride[0];
    d.qs1 = a->draft_probs_stride[1];
    d.ns = a->noise_stride;
    d.vocab = (int32_t)V;
    d.drafts = a->drafts;
    d.parts = stat_parts(*a);
    d.part_len = (int32_t)ceil_div(V, d.parts);
    d.stats = (RowStat *)((char *)a->workspace + BCAST_SERVE_STATUS_BYTES);
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    switch (a->dtype) {
    case BCAST_SERVE_BF16: return run<__nv_bfloat16>(d, a->batch, st);
    case BCAST_SERVE_FP16: return run<__half>(d, a->batch, st);
    default: return run<float>(d, a->batch, st);
    }
}

int bcast_serve_status(void *workspace, void *cuda_stream)
{
    Device dev;
    int rc = current_device(&dev);
    if (rc) return rc;
    if ((rc = check_array(workspace, 256, dev.id))) return rc;
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    int32_t word = 0;
    SERVE_TRY(cudaMemcpyAsync(&word, workspace, sizeof word, cudaMemcpyDeviceToHost, st));
    SERVE_TRY(cudaStreamSynchronize(st));
    if (!word) return BCAST_OK;
    SERVE_TRY(cudaMemsetAsync(workspace, 0, sizeof word, st));
    SERVE_TRY(cudaStreamSynchronize(st));
    return BCAST_ERR_TIMEOUT;
}

}  // extern "C"
