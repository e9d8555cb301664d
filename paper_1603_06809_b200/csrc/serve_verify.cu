// bcast_serve_verify: speculative sampling over a batch of requests.
//
// Two kernels.  The first gives every row of logits (request b, place i) its softmax statistics -- largest
// logit m and where, s = sum exp((l - m) / T) -- one pass with a running maximum and sum, a row cut into
// parts so that few rows still fill the GPU.  Accepting a draft needs nothing but those and two numbers
// (p = exp((l_x - m) / T) / s against u q_x), so the second kernel joins the parts of a request's rows, finds
// the first draft that fails, and runs the race argmax w_v / e_v over that one row: a cluster of blocks per
// request, joined through distributed shared memory.  Bound by memory and, close behind, by the unit for
// exponentials: drafts + 1 rows of logits are read once, one row of logits a second time (from L2 where it is still
// there), one of q and one of noise.  128 requests x 8 rows of 131072 bf16 logits take 89 us on the device (the
// bytes at the measured copy rate: 62), one request with 5 rows of 32000 9 us; public calls among others 94 and 10.5.  (One kernel for both, a cluster per request that
// takes its rows one after the other, was slower everywhere: 105 and 15 us.)
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
    int32_t best, pad;    // -1 if no logit is above -infinity; without temperature the lowest token with the largest
};

struct VerifyDev {
    const void *logits;
    const float *draft_probs, *uniforms, *noise, *temperature;
    const int32_t *draft_tokens;
    int32_t *accepted, *tokens;
    int64_t ls0, ls1, qs0, qs1, ns;
    int32_t vocab, drafts, parts;
    RowStat *stats;       // [batch][drafts + 1][parts]
};

// What a logit counts for: NaN is -infinity.
__device__ __forceinline__ float clean(float l) { return l != l ? -INFINITY : l; }

// Weight of a logit against the row's largest one; equal infinities share the row.
__device__ __forceinline__ float weight(float l, float top, float c)
{
    if (top == INFINITY) return l == INFINITY ? 1.0f : 0.0f;
    return exp2_approx((l - top) * c);
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

// Does a request draw at random?  (Not at zero, below it, or at NaN.)
__device__ __forceinline__ bool samples(float temperature) { return temperature > 0.0f; }
// 1 / temperature in units of log2, kept finite and, for a request that samples, above zero: at an infinite temperature
// the smallest number there is makes every exponent round to 0 but that of a logit of -infinity, which 0 would turn into
// NaN.  A request without temperature only needs its largest logit.
__device__ __forceinline__ float exponent_scale(float temperature)
{
    return samples(temperature) ? fmaxf(fminf(kLog2e / temperature, 1e30f), 1.4e-45f) : 0.0f;
}

// Sixteen bytes of logits as floats.
template <typename T> constexpr int kVector = 16 / (int)sizeof(T);
template <typename T>
__device__ __forceinline__ void widen(const uint4 &raw, float *l)
{
    const T *v = (const T *)&raw;
#pragma unroll
    for (int k = 0; k < kVector<T>; k++) l[k] = to_f32(v[k]);
}

// N logits, token numbers at + 0..N-1, into a thread's statistics.  Without a temperature that is the largest logit
// and where it is.  With one it is their largest (fmaxf passes over NaN) and the sum of the weights against it: what is
// summed so far is scaled at most once, and the exponentials are independent of one another.  A sum that comes out
// NaN had NaN or an infinity in it and is taken again, entry by entry.  (Looking for the place of the largest logit
// there too made the kernel issue-bound: 14 instructions to a logit, 128 x 8 rows of 131072 in 65 us.)
template <int N, bool SAMPLE>
__device__ __forceinline__ void take(RowStat &s, const float *l, int at, float c)
{
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < N; k++) top = fmaxf(top, l[k]);
    if (!SAMPLE) {
        if (top > s.top) {
            s.top = top;
#pragma unroll
            for (int k = N - 1; k >= 0; k--)
                if (l[k] == top) s.best = at + k;
        }
        return;
    }
    if (top > s.top) {
        s.sum = s.best < 0 ? 0.0f : s.sum * weight(s.top, top, c);
        s.top = top;
        s.best = 0;
    }
    if (s.best < 0) return;
    const uint64_t from = pair(-s.top, -s.top), cc = pair(c, c);
    uint64_t sums = 0;                        // a pair of 0.0f
#pragma unroll
    for (int k = 0; k < N; k += 2) {
        float a, b;
        unpair(mul2(add2(pair(l[k], l[k + 1]), from), cc), a, b);
        sums = add2(sums, pair(exp2_approx(a), exp2_approx(b)));
    }
    float a, b;
    unpair(sums, a, b);
    a += b;
    if (a != a) {
        a = 0.0f;
#pragma unroll
        for (int k = 0; k < N; k++) a += weight(clean(l[k]), s.top, c);
    }
    s.sum += a;
}

constexpr int kFetch = 4;                     // vectors that a thread has under way

template <typename T>
__device__ __forceinline__ void fetch(uint4 *to, const uint4 *vec, int v, int end)
{
#pragma unroll
    for (int u = 0; u < kFetch; u++) to[u] = v + u * kStatThreads < end ? __ldg(vec + v + u * kStatThreads) : make_uint4(0, 0, 0, 0);
}

// A thread's share of the vectors v..end-1 of a row, vector 0 being token `at`; `next` holds the first of them, and
// the next ones are fetched before the last ones are worked on.
template <typename T, bool SAMPLE>
__device__ __forceinline__ void take_vectors(RowStat &s, uint4 *next, const uint4 *vec, int v, int end, int at, float c)
{
    constexpr int E = kVector<T>;
    for (; v < end; v += kFetch * kStatThreads) {
        uint4 raw[kFetch];
#pragma unroll
        for (int u = 0; u < kFetch; u++) raw[u] = next[u];
        fetch<T>(next, vec, v + kFetch * kStatThreads, end);
#pragma unroll
        for (int u = 0; u < kFetch; u++) {
            if (v + u * kStatThreads >= end) break;
            float l[E];
            widen<T>(raw[u], l);
            take<E, SAMPLE>(s, l, at + (v + u * kStatThreads) * E, c);
        }
    }
}

// A block takes one part of a row, in 16-byte vectors from the row's first aligned logit on, four under way per
// thread; the first part also takes the logits before that, the last one those after the last vector.
template <typename T>
__global__ void __launch_bounds__(kStatThreads)
serve_verify_stats_kernel(const __grid_constant__ VerifyDev d)
{
    constexpr int E = kVector<T>;
    launch_next();
    const int b = blockIdx.z, i = blockIdx.y, part = blockIdx.x;
    const T *row = (const T *)d.logits + (int64_t)b * d.ls0 + (int64_t)i * d.ls1;
    const int head = min(d.vocab, (int)((16 - ((uintptr_t)row & 15)) % 16 / sizeof(T))), vectors = (d.vocab - head) / E;
    const int v0 = (int)((int64_t)vectors * part / d.parts), v1 = (int)((int64_t)vectors * (part + 1) / d.parts);
    const uint4 *vec = (const uint4 *)(row + head);
    RowStat s{-INFINITY, 0.0f, -1, 0};
    uint4 next[kFetch];
    fetch<T>(next, vec, v0 + threadIdx.x, v1);
    const float t = d.temperature[b], c = exponent_scale(t);
    if (samples(t)) take_vectors<T, true>(s, next, vec, v0 + threadIdx.x, v1, head, c);
    else take_vectors<T, false>(s, next, vec, v0 + threadIdx.x, v1, head, c);
    // a thread's tokens come in ascending order but for the head, which thread order would put last
    if (part == 0 && (int)threadIdx.x < head) {
        const float l = clean(to_f32(row[threadIdx.x]));
        s = join(s, RowStat{l, 1.0f, l > -INFINITY ? (int)threadIdx.x : -1, 0}, c);
    }
    const int tail = head + vectors * E + threadIdx.x;
    if (part == d.parts - 1 && tail < d.vocab) {
        const float l = clean(to_f32(row[tail]));
        s = join(s, RowStat{l, 1.0f, l > -INFINITY ? tail : -1, 0}, c);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) s = join(s, shuffle_xor(s, o), c);
    __shared__ RowStat warp_stat[kStatThreads / 32];
    if (threadIdx.x % 32 == 0) warp_stat[threadIdx.x / 32] = s;
    __syncthreads();
    if (threadIdx.x < 32) {
        s = threadIdx.x < kStatThreads / 32 ? warp_stat[threadIdx.x] : RowStat{-INFINITY, 0.0f, -1, 0};
#pragma unroll
        for (int o = kStatThreads / 64; o; o >>= 1) s = join(s, shuffle_xor(s, o), c);
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

// (1 / x within 2^-23, a few instructions less than the division: two runners whose ratios are nearer to each other than
// the probabilities' own rounding may come in in either order)
__device__ __forceinline__ float reciprocal(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// One thread's share of a race over a row, `N` neighbouring tokens at a time (their addresses are multiples of N then).
// `q` may be nullptr: the race by p.
template <typename T, int N>
__device__ __forceinline__ Runner run_race(const T *row, const float *q, const float *noise, int vocab, int first, int step, const RowStat &s,
                                           float c)
{
    constexpr int U = N == 1 ? 8 : 4;
    const float inv = 1.0f / s.sum;
    Runner best{0.0f, -1};
    for (int v0 = first * N; v0 < vocab; v0 += U * step * N) {
        alignas(16) T l[U][N];
        alignas(16) float e[U][N], qq[U][N];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int v = v0 + u * step * N;
            if (v < vocab) {
                if constexpr (N == 1) {
                    l[u][0] = row[v];
                    e[u][0] = noise[v];
                    qq[u][0] = q ? q[v] : 0.0f;
                } else {
                    if constexpr (sizeof(T) == 4) *(uint4 *)l[u] = *(const uint4 *)(row + v);
                    else *(uint2 *)l[u] = *(const uint2 *)(row + v);
                    *(float4 *)e[u] = *(const float4 *)(noise + v);
                    *(float4 *)qq[u] = q ? *(const float4 *)(q + v) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                }
            } else {
#pragma unroll
                for (int k = 0; k < N; k++) {
                    l[u][k] = from_f32<T>(0.0f);
                    e[u][k] = -1.0f;
                    qq[u][k] = 0.0f;
                }
            }
        }
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
            for (int k = 0; k < N; k++) {
                const float p = weight(clean(to_f32(l[u][k])), s.top, c) * inv;
                const float ratio = (p - qq[u][k]) * reciprocal(e[u][k]);
                if (e[u][k] > 0.0f && ratio > best.ratio) best = Runner{ratio, v0 + u * step * N + k};
            }
    }
    return best;
}

template <typename T, int N>
__global__ void __launch_bounds__(kPickThreads, 2)
serve_verify_pick_kernel(const __grid_constant__ VerifyDev d)
{
    cg::cluster_group cluster = cg::this_cluster();
    const int b = blockIdx.y, rank = (int)cluster.block_rank(), blocks = (int)cluster.num_blocks();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, warps = blockDim.x / 32;
    __shared__ RowStat row_stat[kMaxDrafts + 1];
    __shared__ uint32_t failed[2];            // bit i: draft i fails
    __shared__ Runner warp_run[kPickThreads / 32], block_run[2];

    if (threadIdx.x < 2) failed[threadIdx.x] = 0;
    const float t = d.temperature[b], c = exponent_scale(t);
    __syncthreads();
    for (int i = warp; i <= d.drafts; i += warps) {
        // what needs no statistics, while the kernel before this one still runs
        int32_t x = -1;
        float l = -INFINITY, uq = 0.0f;
        if (i < d.drafts) {
            x = d.draft_tokens[(int64_t)b * d.drafts + i];
            if (x >= d.vocab) x = -1;
            if (x >= 0) {
                l = clean(to_f32(((const T *)d.logits)[(int64_t)b * d.ls0 + (int64_t)i * d.ls1 + x]));
                uq = d.uniforms[(int64_t)b * d.drafts + i] * d.draft_probs[(int64_t)b * d.qs0 + (int64_t)i * d.qs1 + x];
            }
        }
        wait_previous();
        RowStat s{-INFINITY, 0.0f, -1, 0};
        for (int p = lane; p < d.parts; p += 32) s = join(s, d.stats[((int64_t)b * (d.drafts + 1) + i) * d.parts + p], c);
#pragma unroll
        for (int o = 16; o; o >>= 1) s = join(s, shuffle_xor(s, o), c);
        if (lane == 0) {
            row_stat[i] = s;
            const bool good = x >= 0 && s.best >= 0 && (samples(t) ? uq < weight(l, s.top, c) / s.sum : x == s.best);
            if (i < d.drafts && !good) atomicOr(&failed[i / 32], 1u << (i % 32));
        }
    }
    wait_previous();
    __syncthreads();
    const int accepted = failed[0] ? __ffs(failed[0]) - 1 : failed[1] ? 31 + __ffs(failed[1]) : d.drafts;
    const RowStat s = row_stat[accepted];
    int32_t chosen = s.best;                       // no temperature, or no probabilities: the largest logit, or -1
    if (samples(t) && s.best >= 0) {                 // the same for every block of the cluster
        const T *row = (const T *)d.logits + (int64_t)b * d.ls0 + (int64_t)accepted * d.ls1;
        const float *noise = d.noise + (int64_t)b * d.ns;
        const float *q = accepted < d.drafts ? d.draft_probs + (int64_t)b * d.qs0 + (int64_t)accepted * d.qs1 : nullptr;
        // by max(p - q, 0), or by p; where nothing is left of p - q, once more by p
        for (int round = 0; round < 2; round++) {
            Runner best = run_race<T, N>(row, round ? nullptr : q, noise, d.vocab, rank * blockDim.x + threadIdx.x, blocks * blockDim.x, s, c);
#pragma unroll
            for (int o = 16; o; o >>= 1) best = faster(best, shuffle_xor(best, o));
            if (lane == 0) warp_run[warp] = best;
            __syncthreads();
            if (warp == 0) {
                best = lane < warps ? warp_run[lane] : Runner{0.0f, -1};
#pragma unroll
                for (int o = 16; o; o >>= 1) best = faster(best, shuffle_xor(best, o));
                if (lane == 0) block_run[round] = best;
            }
            cluster.sync();
            best = lane < blocks ? *cluster.map_shared_rank(&block_run[round], lane) : Runner{0.0f, -1};
#pragma unroll
            for (int o = 16; o; o >>= 1) best = faster(best, shuffle_xor(best, o));
            chosen = best.token;
            if (chosen >= 0 || !q) break;          // every thread of the cluster has the same
        }
        cluster.sync();                            // a block's shared memory stays until the others have read it
    }
    if (rank == 0 && threadIdx.x < 32) {
        if (lane == 0) d.accepted[b] = accepted;
        for (int i = lane; i <= d.drafts; i += 32)
            d.tokens[(int64_t)b * (d.drafts + 1) + i] =
                i < accepted ? d.draft_tokens[(int64_t)b * d.drafts + i] : i == accepted ? chosen : -1;
    }
}

// Parts of a row: two blocks to an SM, none shorter than 2048 logits.  (24 x 6 rows of 50001: 15.7 us, with four blocks to an
// SM 17.3, with eight 18.9; 16 x 8 rows of 131072: 24.3, 25.0, 26.0.)
int stat_parts(const bcast_serve_verify_args &a)
{
    const int64_t rows = (int64_t)a.batch * (a.drafts + 1);
    const int64_t want = ceil_div(2 * kSms, rows < 1 ? 1 : rows);
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
    // four tokens to a load where every row starts on 16 bytes (8 for 16-bit logits)
    const uintptr_t bits = (uintptr_t)d.logits / (sizeof(T) / 2) | (uintptr_t)d.ls0 * 2 | (uintptr_t)d.ls1 * 2 | (uintptr_t)d.vocab * 2;
    const uintptr_t floats = (uintptr_t)d.noise | (uintptr_t)d.ns * 4 | (d.drafts ? (uintptr_t)d.draft_probs | (uintptr_t)d.qs0 * 4 | (uintptr_t)d.qs1 * 4 : 0);
    const bool whole = bits % 8 == 0 && floats % 16 == 0;
    // blocks of a request's cluster: up to eight while all are resident at once, and twice the threads where that
    // still leaves room
    unsigned blocks = 1;
    while (blocks < 8 && 2 * blocks * (unsigned)batch <= 4 * kSms) blocks *= 2;
    return launch(whole ? serve_verify_pick_kernel<T, 4> : serve_verify_pick_kernel<T, 1>, dim3(blocks, batch), dim3(blocks < 8 ? kPickThreads / 2 : kPickThreads), 0,
                  st, true, blocks, d);
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
    int device = 0;
    SERVE_TRY(cudaGetDevice(&device));
    const uintptr_t size = a->dtype == BCAST_SERVE_FP32 ? 4 : 2;
    if ((rc = check_array(a->logits, size, device)) || (rc = check_array(a->noise, 4, device)) ||
        (rc = check_array(a->temperature, 4, device)) || (rc = check_array(a->accepted, 4, device)) ||
        (rc = check_array(a->tokens, 4, device)))
        return rc;
    if (a->drafts && ((rc = check_array(a->draft_probs, 4, device)) || (rc = check_array(a->draft_tokens, 4, device)) ||
                      (rc = check_array(a->uniforms, 4, device))))
        return rc;
    if ((rc = check_workspace(a->workspace, a->workspace_bytes, bcast_serve_verify_workspace(a), device))) return rc;

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
    int device = 0, rc;
    SERVE_TRY(cudaGetDevice(&device));
    if ((rc = check_array(workspace, 256, device))) return rc;
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
