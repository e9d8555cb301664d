// bcast_serve_logprobs: log probabilities of given tokens, the rows' entropy and their most probable tokens.
//
// One pass over a row with a running maximum m: s = sum e^(l - m) and w = sum e^(l - m) (l - m), so that
//   log p(x) = l_x - m - log s,   entropy = log s - w / s.
// A thread's m may lag behind its largest logit (the exponentials' range allows it), so few steps scale the sums.
// The most probable tokens cost the pass nothing but what the softmax needs anyway, the largest logit of each thread:
// the K-th largest of the threads' maxima bounds the row's K-th largest logit from below, and only the threads whose
// maximum reaches it can hold one of the K.  A warp looks through such a thread's logits once more (from L2), what
// reaches the bound goes to a list in shared memory, and an entry's place is the number of entries before it in
// the order (logit, then lower token).  Lists that overflow -- many equal logits, as behind a mask of the type's lowest
// value -- take bounds that are exact, and equals in the order of their numbers.
// A row is a block's, or a cluster's where the rows are few: its first block joins the parts through distributed
// shared memory.
#include "serve_device.cuh"
#include "serve_internal.h"

#include <cooperative_groups.h>

namespace cg = cooperative_groups;

namespace bcast_serve {
namespace {

constexpr int kProbThreads = 256, kWarps = kProbThreads / 32, kMaxTop = 32, kListSize = 1024, kMaxParts = 8;
constexpr int kInFlight = 4;                  // vectors that a thread has under way
constexpr float kLag = 8.0f;                  // how far a thread's maximum may lag: weights up to e^8
constexpr float kFloor = -150.0f;             // in powers of two: what is smaller counts as nothing

struct ProbDev {
    const void *logits;
    const int32_t *tokens;
    float *logprobs, *entropy, *top_logprobs;
    int32_t *top_tokens;
    int64_t stride;
    int32_t vocab, top, parts;
};

// Statistics of a set of logits: sum of e^(l - at), and of e^(l - at) * (l - at) in powers of two.
struct Sums {
    float at, s, w;
};
// (a plain struct, which shared memory may hold)
__device__ __forceinline__ Sums no_sums() { return Sums{-INFINITY, 0.0f, 0.0f}; }

// The statistics against another maximum, not below the present one.
__device__ __forceinline__ void move_to(Sums &a, float at)
{
    if (a.at == -INFINITY) {
        a.at = at;
        return;
    }
    const float z = fmaxf((a.at - at) * kLog2e, kFloor), f = exp2_approx(z);
    a.w = (a.w + z * a.s) * f;
    a.s *= f;
    a.at = at;
}
__device__ __forceinline__ void join(Sums &a, Sums b)
{
    const float at = fmaxf(a.at, b.at);
    if (at == -INFINITY) return;
    move_to(a, at);
    move_to(b, at);
    a.s += b.s;
    a.w += b.w;
}

// Whole numbers in the order of the logits.  (-infinity and NaN, which counts as it, are the lowest.)
__device__ __forceinline__ uint32_t key_of(float l)
{
    const uint32_t b = __float_as_uint(l != l ? -INFINITY : l + 0.0f);        // -0 is 0
    return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float(key >> 31 ? key & 0x7fffffffu : ~key); }
constexpr uint32_t kLowest = 0x007fffffu;     // of -infinity

// Sixteen bytes of logits.
template <typename T> constexpr int kPer = 16 / (int)sizeof(T);
template <typename T>
__device__ __forceinline__ uint4 no_logits()
{
    const uint32_t v = std::is_same_v<T, float> ? 0xff800000u : std::is_same_v<T, __half> ? 0xfc00fc00u : 0xff80ff80u;
    return make_uint4(v, v, v, v);
}
template <typename T>
__device__ __forceinline__ void widen(const uint4 &raw, float *l)
{
    const T *v = (const T *)&raw;
#pragma unroll
    for (int k = 0; k < kPer<T>; k++) l[k] = to_f32(v[k]);
}

// What one block leaves of its part of a row.
struct Part {
    Sums sums;
    float top;                                // largest logit
    int32_t infinite, count;                  // logits of +infinity; entries of `best`
    uint64_t best[kMaxTop];
};

// A part of a row: tokens before its first vector, vectors, tokens behind its last.
template <typename T>
struct Span {
    const T *row;
    const uint4 *vec;
    int32_t head, v0, v1, tail, tail_count;   // `head` tokens before vector 0
    __device__ __forceinline__ Span(const ProbDev &d, int64_t r, int part)
    {
        row = (const T *)d.logits + r * d.stride;
        const int before = min(d.vocab, (int)((16 - ((uintptr_t)row & 15)) % 16 / sizeof(T))), vectors = (d.vocab - before) / kPer<T>;
        vec = (const uint4 *)(row + before);
        v0 = (int)((int64_t)vectors * part / d.parts);
        v1 = (int)((int64_t)vectors * (part + 1) / d.parts);
        head = before;
        tail = before + vectors * kPer<T>;
        tail_count = part == d.parts - 1 ? d.vocab - tail : 0;
    }
    // The token at place `i` of the part's first tokens and last ones, -1 if there is none.
    __device__ __forceinline__ int edge(int i, int part) const
    {
        const int heads = part == 0 ? head : 0;
        return i < heads ? i : i - heads < tail_count ? tail + i - heads : -1;
    }
};

struct Shared {
    Part part;
    Sums warp_sums[kWarps];
    float warp_top[kWarps], warp_low[kWarps];
    int warp_count[kWarps];
    int listed;
    uint64_t list[kListSize];
};

__device__ __forceinline__ uint64_t entry_of(uint32_t key, int token) { return (uint64_t)key << 32 | (uint32_t)~token; }
__device__ __forceinline__ int token_of(uint64_t entry) { return (int)~(uint32_t)entry; }

__device__ __forceinline__ void put(Shared &sh, float l, int token, uint32_t least)
{
    const uint32_t key = key_of(l);
    if (key < least) return;
    const int at = atomicAdd(&sh.listed, 1);
    if (at < kListSize) sh.list[at] = entry_of(key, token);
}

// Everything of this block's part whose key is at least `least` goes to the list (as far as that goes); `mine`: this
// thread's largest key, its edge token's among them.
template <typename T>
__device__ __forceinline__ void collect(Shared &sh, const Span<T> &span, int part, uint32_t mine, uint32_t least)
{
    __syncthreads();
    if (threadIdx.x == 0) sh.listed = 0;
    __syncthreads();
    const int lane = threadIdx.x % 32;
    for (uint32_t todo = __ballot_sync(~0u, mine >= least); todo; todo &= todo - 1) {
        const int who = threadIdx.x - lane + __ffs(todo) - 1;
        for (int v = span.v0 + who + lane * kProbThreads; v < span.v1; v += 32 * kProbThreads) {
            float l[kPer<T>];
            widen<T>(__ldg(span.vec + v), l);
#pragma unroll
            for (int k = 0; k < kPer<T>; k++) put(sh, l[k], span.head + v * kPer<T> + k, least);
        }
    }
    const int token = span.edge(threadIdx.x, part);
    if (token >= 0) put(sh, to_f32(span.row[token]), token, least);
    __syncthreads();
}

// How many logits of the part have a key of at least `least`.
template <typename T>
__device__ __forceinline__ int count_of(Shared &sh, const Span<T> &span, int part, uint32_t least)
{
    int n = 0;
    for (int v = span.v0 + threadIdx.x; v < span.v1; v += kProbThreads) {
        float l[kPer<T>];
        widen<T>(__ldg(span.vec + v), l);
#pragma unroll
        for (int k = 0; k < kPer<T>; k++) n += key_of(l[k]) >= least;
    }
    const int token = span.edge(threadIdx.x, part);
    if (token >= 0) n += key_of(to_f32(span.row[token])) >= least;
    n = __reduce_add_sync(~0u, n);
    __syncthreads();
    if (threadIdx.x % 32 == 0) sh.warp_count[threadIdx.x / 32] = n;
    __syncthreads();
    n = 0;
#pragma unroll
    for (int w = 0; w < kWarps; w++) n += sh.warp_count[w];
    return n;
}

// The first tokens of the part whose key is `key`, in the order of their numbers, behind what is listed, until the list
// has `want` entries.
template <typename T>
__device__ __forceinline__ void add_equals(Shared &sh, const Span<T> &span, int part, uint32_t key, int want)
{
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int begin = part == 0 ? 0 : span.head + span.v0 * kPer<T>, end = span.head + span.v1 * kPer<T> + span.tail_count;
    int have = sh.listed;
    for (int t0 = begin; t0 < end && have < want; t0 += kProbThreads) {
        const int token = t0 + threadIdx.x;
        const bool equal = token < end && key_of(to_f32(span.row[token])) == key;
        const uint32_t bits = __ballot_sync(~0u, equal);
        __syncthreads();
        if (lane == 0) sh.warp_count[warp] = __popc(bits);
        __syncthreads();
        int at = have;
#pragma unroll
        for (int w = 0; w < kWarps; w++) {
            if (w < warp) at += sh.warp_count[w];
            have += sh.warp_count[w];
        }
        at += __popc(bits & ((1u << lane) - 1u));
        if (equal && at < want) sh.list[at] = entry_of(key, token);
    }
    __syncthreads();
    if (threadIdx.x == 0) sh.listed = min(have, want);
    __syncthreads();
}

// The part's `want` largest logits above -infinity, or as many as there are, in order, to part.best.
template <typename T>
__device__ __forceinline__ void pick(Shared &sh, const Span<T> &span, int part, float mine, float low, int want)
{
    const uint32_t key = key_of(mine);
    // The bound: a key that `want` threads' maxima reach, and few more.  `over`: one that fewer reach.
    uint32_t least = kLowest + 1, over = key_of(sh.part.top) + 1;
    bool exact = false;                       // `least` is the want-th largest of the threads' maxima
    if (__syncthreads_count(key > kLowest) >= want) {
        uint32_t next = max(key_of(low), least);
        for (;;) {
            const int reach = __syncthreads_count(key >= next);
            if (reach >= want) least = next;
            else over = next;
            exact = over - least <= 1;
            if (exact || (reach >= want && reach <= want + want / 2)) break;
            next = least + (over - least) / 2;
        }
    }
    collect(sh, span, part, key, least);
    if (sh.listed > kListSize) {
        // the exact bound, and only what is above it: where many are equal to it, that is little
        while (!exact) {
            const uint32_t next = least + (over - least) / 2;
            if (__syncthreads_count(key >= next) >= want) least = next;
            else over = next;
            exact = over - least <= 1;
        }
        collect(sh, span, part, key, least + 1);
        if (sh.listed > kListSize) {
            // the want-th largest logit itself: fewer than `want` are above it
            over = key_of(sh.part.top) + 1;
            while (over - least > 1) {
                const uint32_t next = least + (over - least) / 2;
                if (count_of(sh, span, part, next) >= want) least = next;
                else over = next;
            }
            collect(sh, span, part, key, least + 1);
        }
        if (sh.listed < want) add_equals(sh, span, part, least, want);
    }
    const int listed = sh.listed;
    for (int i = threadIdx.x; i < listed; i += kProbThreads) {
        const uint64_t e = sh.list[i];
        int place = 0;
        for (int j = 0; j < listed; j++) place += sh.list[j] > e;
        if (place < want) sh.part.best[place] = e;
    }
    if (threadIdx.x == 0) sh.part.count = min(listed, want);
}

// One batch of logits into a thread's sums and largest logit.
template <typename T>
__device__ __forceinline__ void take(Sums &a, float &top, const uint4 *raw)
{
    float most = -INFINITY;
    if constexpr (std::is_same_v<T, float>) {
#pragma unroll
        for (int u = 0; u < kInFlight; u++) {
            float l[4];
            widen<T>(raw[u], l);
            most = fmaxf(most, fmaxf(fmaxf(l[0], l[1]), fmaxf(l[2], l[3])));
        }
    } else {
        using T2 = std::conditional_t<std::is_same_v<T, __half>, __half2, __nv_bfloat162>;
        T2 m[4];
#pragma unroll
        for (int k = 0; k < 4; k++) {
            m[k] = ((const T2 *)raw)[k];
#pragma unroll
            for (int u = 1; u < kInFlight; u++) m[k] = __hmax2(m[k], ((const T2 *)(raw + u))[k]);     // passes over NaN
        }
        const T2 r = __hmax2(__hmax2(m[0], m[1]), __hmax2(m[2], m[3]));
        most = fmaxf(fmaxf(most, to_f32(r.x)), to_f32(r.y));
    }
    top = fmaxf(top, most);
    if (most > a.at + kLag) move_to(a, most);
    if (a.at == -INFINITY) return;
    const uint64_t from = pair(-a.at, -a.at), unit = pair(kLog2e, kLog2e);
    uint64_t s = 0, w = 0;                    // pairs of 0.0f
#pragma unroll
    for (int u = 0; u < kInFlight; u++) {
        float l[kPer<T>];
        widen<T>(raw[u], l);
#pragma unroll
        for (int k = 0; k < kPer<T>; k += 2) {
            float x, y;
            unpair(mul2(add2(pair(l[k], l[k + 1]), from), unit), x, y);
            x = fmaxf(x, kFloor);             // (NaN too)
            y = fmaxf(y, kFloor);
            const uint64_t e = pair(exp2_approx(x), exp2_approx(y));
            s = add2(s, e);
            w = fma2(e, pair(x, y), w);
        }
    }
    float x, y;
    unpair(s, x, y);
    a.s += x + y;
    unpair(w, x, y);
    a.w += x + y;
}

template <typename T>
__device__ __forceinline__ void fetch(uint4 *to, const Span<T> &span, int v)
{
#pragma unroll
    for (int u = 0; u < kInFlight; u++) to[u] = v + u * kProbThreads < span.v1 ? __ldg(span.vec + v + u * kProbThreads) : no_logits<T>();
}

template <typename T>
__global__ void __launch_bounds__(kProbThreads, 4)
serve_logprobs_kernel(const __grid_constant__ ProbDev d)
{
    __shared__ Shared sh;
    const cg::cluster_group cluster = cg::this_cluster();
    const int part = d.parts > 1 ? (int)cluster.block_rank() : 0, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int64_t r = blockIdx.x / d.parts;
    const Span<T> span(d, r, part);
    Sums a = no_sums();
    float top = -INFINITY;
    {
        uint4 next[kInFlight];
        int v = span.v0 + threadIdx.x;
        fetch(next, span, v);
        for (; v < span.v1; v += kInFlight * kProbThreads) {
            uint4 raw[kInFlight];
#pragma unroll
            for (int u = 0; u < kInFlight; u++) raw[u] = next[u];
            fetch(next, span, v + kInFlight * kProbThreads);
            take<T>(a, top, raw);
        }
    }
    const int edge = span.edge(threadIdx.x, part);
    if (edge >= 0) {
        const float l = to_f32(span.row[edge]);
        if (l > -INFINITY) {
            join(a, Sums{l, 1.0f, 0.0f});
            top = fmaxf(top, l);
        }
    }
    const float mine = top;
    float low = mine == -INFINITY ? INFINITY : mine;  // the lowest of the threads' largest logits
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        join(a, Sums{__shfl_xor_sync(~0u, a.at, o), __shfl_xor_sync(~0u, a.s, o), __shfl_xor_sync(~0u, a.w, o)});
        top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
        low = fminf(low, __shfl_xor_sync(~0u, low, o));
    }
    if (lane == 0) {
        sh.warp_sums[warp] = a;
        sh.warp_top[warp] = top;
        sh.warp_low[warp] = low;
    }
    __syncthreads();
    a = sh.warp_sums[0];
    for (int w = 0; w < kWarps; w++) {
        if (w) join(a, sh.warp_sums[w]);
        top = fmaxf(top, sh.warp_top[w]);
        low = fminf(low, sh.warp_low[w]);
    }
    if (threadIdx.x == 0) {
        sh.part.sums = a;
        sh.part.top = top;
        sh.part.count = 0;
    }
    __syncthreads();
    const int infinite = top == INFINITY ? count_of(sh, span, part, key_of(INFINITY)) : 0;
    if (threadIdx.x == 0) sh.part.infinite = infinite;
    if (d.top && top > -INFINITY) pick(sh, span, part, mine, low, d.top);
    if (d.parts > 1) cluster.sync();
    else __syncthreads();
    if (part == 0) {
        // the row's statistics, by every thread alike
        Sums all = sh.part.sums;
        int infinities = sh.part.infinite;
        float most = sh.part.top;
        for (int p = 1; p < d.parts; p++) {
            const Part *o = cluster.map_shared_rank(&sh.part, p);
            join(all, o->sums);
            infinities += o->infinite;
            most = fmaxf(most, o->top);
        }
        const bool share = most == INFINITY;          // among the infinite ones
        const float log_sum = share ? logf((float)infinities) : logf(all.s);
        auto logprob = [&](float l) {
            if (!(l > -INFINITY)) return -INFINITY;
            if (share) return l == INFINITY ? -log_sum : -INFINITY;
            return l - all.at - log_sum;
        };
        if (threadIdx.x == 0) {
            const int32_t x = d.tokens[r];
            d.logprobs[r] = x >= 0 && x < d.vocab ? logprob(to_f32(span.row[x])) : -INFINITY;
            if (d.entropy) d.entropy[r] = most == -INFINITY ? 0.0f : share ? log_sum : fmaxf(log_sum - all.w / all.s * kLn2, 0.0f);
        }
        if (d.top) {
            const Part *mine_of = nullptr;            // the parts' lists, a thread to an entry
            int total = 0;
            uint64_t e = 0;
            for (int p = 0; p < d.parts; p++) {
                const Part *o = d.parts > 1 ? cluster.map_shared_rank(&sh.part, p) : &sh.part;
                const int at = (int)threadIdx.x - total, n = o->count;
                if (at >= 0 && at < n) {
                    mine_of = o;
                    e = o->best[at];
                }
                total += n;
            }
            if (d.parts > 1) {                        // at most 8 x 32 entries, one to a thread
                if (mine_of) sh.list[threadIdx.x] = e;
                __syncthreads();
            }
            int place = threadIdx.x;
            if (d.parts > 1 && mine_of) {
                place = 0;
                for (int j = 0; j < total; j++) place += sh.list[j] > e;
            }
            float l = mine_of ? logprob(logit_of((uint32_t)(e >> 32))) : -INFINITY;
            if (mine_of && place < d.top) {
                const bool likely = !share || l > -INFINITY;
                d.top_tokens[r * d.top + place] = likely ? token_of(e) : -1;
                d.top_logprobs[r * d.top + place] = l;
            }
            if ((int)threadIdx.x >= total && (int)threadIdx.x < d.top) {
                d.top_tokens[r * d.top + threadIdx.x] = -1;
                d.top_logprobs[r * d.top + threadIdx.x] = -INFINITY;
            }
        }
    }
    if (d.parts > 1) cluster.sync();                  // a block's memory stays until the first one has read it
}

int check_shape(const bcast_serve_logprobs_args &a)
{
    if (a.dtype != BCAST_SERVE_BF16 && a.dtype != BCAST_SERVE_FP16 && a.dtype != BCAST_SERVE_FP32) return BCAST_ERR_INVAL;
    if (a.rows < 0 || a.rows >= 1 << 24 || a.vocab < 1 || a.vocab > kMaxDim - 65536 || a.top < 0 || a.top > kMaxTop) return BCAST_ERR_INVAL;
    return BCAST_OK;
}

}  // namespace
}  // namespace bcast_serve

using namespace bcast_serve;

extern "C" int bcast_serve_logprobs(const bcast_serve_logprobs_args *args, void *cuda_stream)
{
    if (!args) return BCAST_ERR_INVAL;
    const bcast_serve_logprobs_args &a = *args;
    int rc = check_shape(a);
    if (rc) return rc;
    if (a.rows == 0) return BCAST_OK;
    if (!stride_ok(a.logits_stride, 0, 1)) return BCAST_ERR_INVAL;
    int device = 0;
    SERVE_TRY(cudaGetDevice(&device));
    if ((rc = check_array(a.logits, a.dtype == BCAST_SERVE_FP32 ? 4 : 2, device)) || (rc = check_array(a.tokens, 4, device)) ||
        (rc = check_array(a.logprobs, 4, device)))
        return rc;
    if (a.entropy && (rc = check_array(a.entropy, 4, device))) return rc;
    if (a.top && ((rc = check_array(a.top_tokens, 4, device)) || (rc = check_array(a.top_logprobs, 4, device)))) return rc;

    ProbDev d = {};
    d.logits = a.logits;
    d.tokens = a.tokens;
    d.logprobs = a.logprobs;
    d.entropy = a.entropy;
    d.top_logprobs = a.top_logprobs;
    d.top_tokens = a.top_tokens;
    d.stride = a.logits_stride;
    d.vocab = (int32_t)a.vocab;
    d.top = a.top;
    // few rows: several blocks to one, of at least two batches of vectors to a thread
    d.parts = 1;
    while (d.parts < kMaxParts && a.rows * d.parts * 2 <= 4 * kSms && a.vocab >= (int64_t)d.parts * 2 * 16384) d.parts *= 2;
    const dim3 grid((unsigned)(a.rows * d.parts)), threads(kProbThreads);
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    switch (a.dtype) {
    case BCAST_SERVE_BF16: return launch(serve_logprobs_kernel<__nv_bfloat16>, grid, threads, 0, st, false, (unsigned)d.parts, d);
    case BCAST_SERVE_FP16: return launch(serve_logprobs_kernel<__half>, grid, threads, 0, st, false, (unsigned)d.parts, d);
    default: return launch(serve_logprobs_kernel<float>, grid, threads, 0, st, false, (unsigned)d.parts, d);
    }
}
