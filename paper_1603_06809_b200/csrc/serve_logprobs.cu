// bcast_serve_logprobs: log probabilities of given tokens, the rows' entropy and their most probable tokens.
//
// One pass over a row with a running maximum m: s = sum e^(l - m) and w = sum e^(l - m) (l - m), so that
//   log p(x) = l_x - m - log s,   entropy = log s - w / s.
// A thread's m may lag behind its largest logit (the exponentials' range allows it), so few steps scale the sums.
// A thread whose share holds -infinity, NaN, the lowest number of bf16 or fp32, or a largest logit beyond 2^20 takes its sums
// once more, one logit after the other.
// The most probable tokens cost the pass nothing but what the softmax needs anyway, the largest logit of each thread:
// the K-th largest of the threads' maxima bounds the row's K-th largest logit from below, and only the threads whose
// maximum reaches it can hold one of the K.  The bound comes from the warps' largest, 32 in all, one to a lane,
// sorted by every warp for itself.  A warp looks through such a thread's logits once more (from L2), what
// reaches the bound goes to a list in shared memory, and an entry's place is the number of entries before it in
// the order (logit, then lower token).  Lists that overflow -- many equal logits, as behind a mask of the type's lowest
// value -- take bounds that are exact, and equals in the order of their numbers.
// A row is a block's (of one warp, where rows are short and many), or a cluster's where the rows are few: its first block
// joins the parts, which the others send it through distributed shared memory (fetched by it, one after the other, a
// cluster's join took 5 us).
// What bounds it, and what it takes on one B200 (in brackets the bytes at the measured copy rate): 4096 rows of 131072 bf16
// logits 175 us without alternatives, 200 with eight (164): loads and exponentials (64 % of their unit) while a block streams,
// nothing while it reduces and picks.  37 rows of 50001 with twenty 10 us, one row of 32000 5: latency, of which a launch,
// the loads, the reductions and the pick have about a third each.  Bringing the next row's beginning to L2 during the pick
// cost 2 to 50 %.  With nine logits of ten at -infinity 4096 rows of 131072 bf16 take 405 us without alternatives, 450 with
// eight (as long with one of a thousand), 64 rows of 32000 8.4 and 10.7 (6.2 and 9.3 without a mask).
#include "serve_device.cuh"
#include "serve_internal.h"

#include <cooperative_groups.h>

namespace cg = cooperative_groups;

namespace bcast_serve {
namespace {

constexpr int kMaxTop = 32, kMaxParts = 8;
template <int P> constexpr int kListSize = P == 32 ? 256 : 1024;          // (blocks of one warp are many to an SM)
constexpr int kInFlight = 4;                  // vectors that a thread has under way
constexpr float kLag = 8.0f;                  // how far a thread's maximum may lag: weights up to e^8
constexpr float kFloor = -150.0f;             // in powers of two: what is smaller counts as nothing
constexpr float kFar = 1048576.0f;            // a maximum beyond it is subtracted first, not in one step with log2(e)

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
// Whole numbers in the order of the logits.  (-infinity and NaN, which counts as it, are the lowest.)
__device__ __forceinline__ uint32_t key_of(float l)
{
    const uint32_t b = __float_as_uint(l != l ? -INFINITY : l + 0.0f);        // -0 is 0
    return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float(key >> 31 ? key & 0x7fffffffu : ~key); }
constexpr uint32_t kLowest = 0x007fffffu;     // of -infinity

// The statistics of all lanes, the same in each.
__device__ __forceinline__ Sums warp_join(Sums a)
{
    const float at = logit_of(__reduce_max_sync(~0u, key_of(a.at)));
    if (at == -INFINITY) return a;
    move_to(a, at);
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        a.s += __shfl_xor_sync(~0u, a.s, o);
        a.w += __shfl_xor_sync(~0u, a.w, o);
    }
    return a;
}

// Sixteen bytes of logits.
template <typename T> constexpr int kPer = 16 / (int)sizeof(T);
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

// `P`: threads of a block.
template <int P>
struct Shared {
    Part parts[kMaxParts];                    // of the first block of a cluster: what all of them found
    Sums warp_sums[P / 32];
    uint32_t tops[32];                        // each warp's largest keys, 1024 / P of them
    int warp_count[P / 32];
    int listed;
    uint64_t list[kListSize<P>];
};

__device__ __forceinline__ uint64_t entry_of(uint32_t key, int token) { return (uint64_t)key << 32 | (uint32_t)~token; }
__device__ __forceinline__ int token_of(uint64_t entry) { return (int)~(uint32_t)entry; }

template <int P>
__device__ __forceinline__ void put(Shared<P> &sh, float l, int token, uint32_t least)
{
    const uint32_t key = key_of(l);
    if (key < least) return;
    const int at = atomicAdd(&sh.listed, 1);
    if (at < kListSize<P>) sh.list[at] = entry_of(key, token);
}

// What reaches `least` of one vector, `at` the number of its first token, goes to the list.
template <typename T, int P>
__device__ __forceinline__ void put_vector(Shared<P> &sh, const uint4 &raw, int at, uint32_t least)
{
    float l[kPer<T>];
    widen<T>(raw, l);
    float most = l[0];
#pragma unroll
    for (int k = 1; k < kPer<T>; k++) most = fmaxf(most, l[k]);
    if (key_of(most) < least) return;
#pragma unroll
    for (int k = 0; k < kPer<T>; k++) put(sh, l[k], at + k, least);
}

// Everything of this block's part whose key is at least `least` goes to the list (as far as that goes); `mine`: this
// thread's largest key, its edge token's among them; `held`: its vectors, where no thread has more than kInFlight.
template <typename T, int P>
__device__ __forceinline__ void collect(Shared<P> &sh, const Span<T> &span, int part, uint32_t mine, uint32_t least, const uint4 *held, bool again)
{
    if (again) {
        __syncthreads();
        if (threadIdx.x == 0) sh.listed = 0;
        __syncthreads();
    }
    if (span.v1 - span.v0 <= kInFlight * P) {
        if (mine >= least) {
#pragma unroll
            for (int u = 0; u < kInFlight; u++) {
                const int v = span.v0 + threadIdx.x + u * P;
                if (v < span.v1) put_vector<T, P>(sh, held[u], span.head + v * kPer<T>, least);
            }
        }
    } else {
        const int lane = threadIdx.x % 32, each = (span.v1 - span.v0 + P - 1) / P;
        const uint32_t which = __ballot_sync(~0u, mine >= least);
        if (__popc(which) * ((each + 31) / 32) < each) {
            // a warp to a thread's logits
            for (uint32_t todo = which; todo; todo &= todo - 1) {
                const int who = threadIdx.x - lane + __ffs(todo) - 1;
#pragma unroll 2
                for (int v = span.v0 + who + lane * P; v < span.v1; v += 32 * P)
                    put_vector<T, P>(sh, __ldg(span.vec + v), span.head + v * kPer<T>, least);
            }
        } else {
            // many threads of a short row: each its own (4096 rows of 3292, twenty alternatives: 30 us, so 37)
            for (int v = span.v0 + threadIdx.x; v < span.v1; v += kInFlight * P) {
                uint4 raw[kInFlight];
#pragma unroll
                for (int u = 0; u < kInFlight; u++)
                    if (v + u * P < span.v1) raw[u] = __ldg(span.vec + v + u * P);
#pragma unroll
                for (int u = 0; u < kInFlight; u++)
                    if (v + u * P < span.v1) put_vector<T, P>(sh, raw[u], span.head + (v + u * P) * kPer<T>, least);
            }
        }
    }
    const int token = span.edge(threadIdx.x, part);
    if (token >= 0) put(sh, to_f32(span.row[token]), token, least);
    __syncthreads();
}

// How many logits of the part have a key of at least `least`.
template <typename T, int P>
__device__ __forceinline__ int count_of(Shared<P> &sh, const Span<T> &span, int part, uint32_t least)
{
    int n = 0;
    for (int v = span.v0 + threadIdx.x; v < span.v1; v += P) {
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
    for (int w = 0; w < P / 32; w++) n += sh.warp_count[w];
    return n;
}

// The first tokens of the part whose key is `key`, in the order of their numbers, behind what is listed, until the list
// has `want` entries.
template <typename T, int P>
__device__ __forceinline__ void add_equals(Shared<P> &sh, const Span<T> &span, int part, uint32_t key, int want)
{
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int begin = part == 0 ? 0 : span.head + span.v0 * kPer<T>, end = span.head + span.v1 * kPer<T> + span.tail_count;
    int have = sh.listed;
    for (int t0 = begin; t0 < end && have < want; t0 += P) {
        const int token = t0 + threadIdx.x;
        const bool equal = token < end && key_of(to_f32(span.row[token])) == key;
        const uint32_t bits = __ballot_sync(~0u, equal);
        __syncthreads();
        if (lane == 0) sh.warp_count[warp] = __popc(bits);
        __syncthreads();
        int at = have;
#pragma unroll
        for (int w = 0; w < P / 32; w++) {
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

// The next of the warp's largest keys, and no longer this lane's where it is the first that has it.
__device__ __forceinline__ uint32_t next_top(uint32_t &left)
{
    const uint32_t top = __reduce_max_sync(~0u, left);
    if ((int)(threadIdx.x % 32) == __ffs(__ballot_sync(~0u, left == top)) - 1) left = 0;
    return top;
}
// The `want`-th largest of the 32 lanes' keys.
__device__ __forceinline__ uint32_t nth_of_lanes(uint32_t key, int want)
{
    const int lane = threadIdx.x % 32;
#pragma unroll
    for (int size = 2; size <= 32; size *= 2) {
#pragma unroll
        for (int d = size / 2; d; d /= 2) {
            const uint32_t other = __shfl_xor_sync(~0u, key, d);
            const bool up = (lane & size) != 0 && size < 32, low = (lane & d) == 0;   // (descending as a whole)
            key = low != up ? max(key, other) : min(key, other);
        }
    }
    return __shfl_sync(~0u, key, want - 1);
}

// The part's `want` largest logits above -infinity, or as many as there are, to the list; `mine`: the key of this thread's
// largest logit.  Behind a barrier after `tops` and `listed` were written.
template <typename T, int P>
__device__ __forceinline__ void pick(Shared<P> &sh, const Span<T> &span, int part, uint32_t mine, int want, const uint4 *held)
{
    // a key that `want` threads' maxima reach, and few more; where fewer threads have a logit, the lowest there is
    uint32_t least = max(nth_of_lanes(sh.tops[threadIdx.x % 32], want), kLowest + 1);
    collect<T, P>(sh, span, part, mine, least, held, false);
    if (sh.listed <= kListSize<P>) return;
    // only what is above the bound: where many are equal to it, that is little
    collect<T, P>(sh, span, part, mine, least + 1, held, true);
    if (sh.listed > kListSize<P>) {
        // the want-th largest logit itself: fewer than `want` are above it
        uint32_t over = key_of(INFINITY) + 1;
        while (over - least > 1) {
            const uint32_t next = least + (over - least) / 2;
            if (count_of<T, P>(sh, span, part, next) >= want) least = next;
            else over = next;
        }
        collect<T, P>(sh, span, part, mine, least + 1, held, true);
    }
    if (sh.listed < want) add_equals<T, P>(sh, span, part, least, want);
}

// N vectors of logits into a thread's sums and largest logit; `again`: the sums are to be taken another way, because of NaN,
// of -infinity (nothing, times an infinite exponent) or of numbers far out.
template <typename T, int N>
__device__ __forceinline__ void take(Sums &a, float &top, bool &again, const uint4 *raw)
{
    float most = -INFINITY;
    if constexpr (std::is_same_v<T, float>) {
#pragma unroll
        for (int u = 0; u < N; u++) {
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
            for (int u = 1; u < N; u++) m[k] = __hmax2(m[k], ((const T2 *)(raw + u))[k]);     // passes over NaN
        }
        const T2 r = __hmax2(__hmax2(m[0], m[1]), __hmax2(m[2], m[3]));
        most = fmaxf(fmaxf(most, to_f32(r.x)), to_f32(r.y));
    }
    top = fmaxf(top, most);
    if (most > a.at + kLag) move_to(a, most);
    if (a.at == -INFINITY) return;
    // l log2(e) - base in one step; the base is rounded, which is made good below
    const float base = a.at * kLog2e, off = fmaf(a.at, kLog2e, -base);
    const uint64_t from = pair(-base, -base), unit = pair(kLog2e, kLog2e);
    uint64_t s = 0, w = 0;                    // pairs of 0.0f
#pragma unroll
    for (int u = 0; u < N; u++) {
        float l[kPer<T>];
        widen<T>(raw[u], l);
#pragma unroll
        for (int k = 0; k < kPer<T>; k += 2) {
            const uint64_t z = fma2(pair(l[k], l[k + 1]), unit, from);
            float x, y;
            unpair(z, x, y);
            const uint64_t e = pair(exp2_approx(x), exp2_approx(y));
            s = add2(s, e);
            w = fma2(e, z, w);
        }
    }
    float x, y;
    unpair(s, x, y);
    const float sum = x + y;
    unpair(w, x, y);
    const float more = x + y, by = exp2_approx(-off);
    a.s += sum * by;
    a.w += (more - off * sum) * by;
    again = again || more != more || fabsf(a.at) > kFar;
}

// A thread's sums once more, one logit after the other, against its largest one.
template <typename T, int P>
__device__ __noinline__ Sums sums_again(const uint4 *vec, int v, int end, float top)
{
    Sums a{top, 0.0f, 0.0f};
    if (top == -INFINITY) return a;
#pragma unroll 1
    for (; v < end; v += P) {
        float l[kPer<T>];
        widen<T>(__ldg(vec + v), l);
#pragma unroll
        for (int k = 0; k < kPer<T>; k++) {
            const float z = fmaxf((l[k] - top) * kLog2e, kFloor), e = l[k] > -INFINITY ? exp2_approx(z) : 0.0f;
            a.s += e;
            a.w += e * z;
        }
    }
    return a;
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

template <typename T, int P>
__global__ void __launch_bounds__(P, 1024 / P)
serve_logprobs_kernel(const __grid_constant__ ProbDev d)
{
    __shared__ Shared<P> sh;
    wait_previous();
    launch_next();
    const cg::cluster_group cluster = cg::this_cluster();
    const int part = d.parts > 1 ? (int)cluster.block_rank() : 0, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int64_t r = blockIdx.x / d.parts;
    const Span<T> span(d, r, part);
    if (d.parts > 1) cluster_arrive();
    // the given token and its logit, under way early
    const int32_t given = part == 0 && threadIdx.x == 0 ? d.tokens[r] : -1;
    Sums a = no_sums();
    float top = -INFINITY;
    bool again = false;
    uint4 next[kInFlight];
    {
        // whole batches, the next one on its way while one is worked on, then what is left, vector by vector
        constexpr int step = kInFlight * P;
        int v = span.v0 + threadIdx.x;
#pragma unroll
        for (int u = 0; u < kInFlight; u++)
            if (v + u * P < span.v1) next[u] = __ldg(span.vec + v + u * P);
        for (; v + step - P < span.v1 && span.v1 - span.v0 > step; v += step) {
            uint4 raw[kInFlight];
#pragma unroll
            for (int u = 0; u < kInFlight; u++) raw[u] = next[u];
#pragma unroll
            for (int u = 0; u < kInFlight; u++)
                if (v + step + u * P < span.v1) next[u] = __ldg(span.vec + v + step + u * P);
            take<T, kInFlight>(a, top, again, raw);
        }
#pragma unroll
        for (int u = 0; u < kInFlight; u++)
            if (v + u * P < span.v1) take<T, 1>(a, top, again, next + u);
    }
    if (again) a = sums_again<T, P>(span.vec, span.v0 + threadIdx.x, span.v1, top);
    const float logit = given >= 0 && given < d.vocab ? to_f32(span.row[given]) : -INFINITY;
    const int edge = span.edge(threadIdx.x, part);
    if (edge >= 0) {
        const float l = to_f32(span.row[edge]);
        if (l > -INFINITY) {
            if (l > a.at) move_to(a, l);
            const float z = fmaxf((l - a.at) * kLog2e, kFloor), e = exp2_approx(z);
            a.s += e;
            a.w += e * z;
            top = fmaxf(top, l);
        }
    }
    const uint32_t mine = key_of(top);
    a = warp_join(a);
    if (lane == 0) sh.warp_sums[warp] = a;
    if constexpr (P == 32) {
        sh.tops[lane] = mine;
    } else {
        uint32_t left = mine;
        for (int k = 0; k < 1024 / P; k++) {          // (one to a warp at least: the row's largest logit is among them)
            const uint32_t key = k == 0 || k < d.top ? next_top(left) : 0;
            if (lane == 0) sh.tops[warp * (1024 / P) + k] = key;
        }
    }
    if (threadIdx.x == 0) sh.listed = 0;
    __syncthreads();
    top = logit_of(__reduce_max_sync(~0u, sh.tops[lane]));
    const int infinite = top == INFINITY ? count_of<T, P>(sh, span, part, key_of(INFINITY)) : 0;
    if (d.top) pick<T, P>(sh, span, part, mine, d.top, next);
    const int listed = d.top ? sh.listed : 0, count = min(listed, d.top);
    // an entry's place in the order; where the row has several blocks, the first one is sent the entries and the sums
    Shared<P> *const first = d.parts > 1 ? cluster.map_shared_rank(&sh, 0) : &sh;
    if (d.parts > 1) cluster_wait();                  // it has begun
    uint64_t entry[kListSize<P> / P];
    int place[kListSize<P> / P];
#pragma unroll
    for (int k = 0; k < kListSize<P> / P; k++) {
        const int i = threadIdx.x + k * P;
        place[k] = kListSize<P>;
        if (i >= listed) continue;
        entry[k] = sh.list[i];
        place[k] = 0;
#pragma unroll 8
        for (int j = 0; j < listed; j++) place[k] += sh.list[j] > entry[k];
        if (d.parts > 1 && place[k] < count) first->parts[part].best[place[k]] = entry[k];
    }
    Sums all = warp_join(lane < P / 32 ? sh.warp_sums[lane] : no_sums());
    int infinities = infinite, total = count;
    if (d.parts > 1) {
        if (threadIdx.x == 0) {
            Part &mine_there = first->parts[part];
            mine_there.sums = all;
            mine_there.top = top;
            mine_there.infinite = infinite;
            mine_there.count = count;
        }
        cluster_arrive();
        cluster_wait();
        if (part) return;
        // the statistics, by every thread alike, and the entries, one to a thread
        total = 0;
        bool has = false;
        for (int p = 0; p < d.parts; p++) {
            const Part &o = sh.parts[p];
            if (p) {
                infinities += o.infinite;
                top = fmaxf(top, o.top);
            }
            const int at = (int)threadIdx.x - total, n = o.count;
            if (at >= 0 && at < n) {
                entry[0] = o.best[at];
                has = true;
            }
            total += n;
        }
        all = warp_join(lane < d.parts ? sh.parts[lane].sums : no_sums());
        if (has) sh.list[threadIdx.x] = entry[0];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kListSize<P> / P; k++) place[k] = kListSize<P>;
        if (has) {
            place[0] = 0;
#pragma unroll 8
            for (int j = 0; j < total; j++) place[0] += sh.list[j] > entry[0];
        }
    }
    {
        const bool share = top == INFINITY;           // among the infinite ones
        const float log_sum = logf(share ? (float)infinities : all.s);
        auto logprob = [&](float l) {
            if (!(l > -INFINITY)) return -INFINITY;
            if (share) return l == INFINITY ? -log_sum : -INFINITY;
            return fminf(l - all.at - log_sum, 0.0f);     // (a sum of one term and little more may be rounded below it)
        };
        if (threadIdx.x == 0) {
            d.logprobs[r] = logprob(logit);
            if (d.entropy) d.entropy[r] = top == -INFINITY ? 0.0f : share ? log_sum : fmaxf(log_sum - all.w / all.s * kLn2, 0.0f);
        }
#pragma unroll
        for (int k = 0; k < kListSize<P> / P; k++) {
            if (place[k] >= d.top) continue;
            const float l = logit_of((uint32_t)(entry[k] >> 32));
            const bool likely = !share || l == INFINITY;
            d.top_tokens[r * d.top + place[k]] = likely ? token_of(entry[k]) : -1;
            d.top_logprobs[r * d.top + place[k]] = logprob(l);
        }
        if ((int)threadIdx.x >= total && (int)threadIdx.x < d.top) {
            d.top_tokens[r * d.top + threadIdx.x] = -1;
            d.top_logprobs[r * d.top + threadIdx.x] = -INFINITY;
        }
    }
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
    // Few rows: several blocks to one, of at least 2048 logits each, in powers of two.  As long as all of them find a place at
    // once, clusters together: up to 7/4 of the SMs (37 rows of 50001 fp16, twenty alternatives: 8 blocks to a row 11.0 us, 4 9.9);
    // up to four to an SM where each has 64 KB (148 rows of 50257 fp32: 1 block 16.2, 2 12.8; but 74 of 32000 bf16: 4 blocks 11.0,
    // 1 6.8).  Two save little of a row that one block takes in four rounds of loads, and their join costs 2 us (128 rows of 32000
    // bf16: 2 blocks 8.8, 1 7.0).
    const int64_t row_bytes = a.vocab * (a.dtype == BCAST_SERVE_FP32 ? 4 : 2);
    d.parts = 1;
    while (d.parts < kMaxParts && a.vocab >= d.parts * 2 * 2048ll) {
        const int64_t blocks = a.rows * d.parts * 2;
        if (blocks > 4 * kSms || (blocks * 4 > 7 * kSms && row_bytes < d.parts * 2 * 65536ll)) break;
        d.parts *= 2;
    }
    if (d.parts == 2 && a.vocab > 16384 && row_bytes < 131072) d.parts = 1;
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    // Short rows: fewer threads to a block, since most of its time is its reductions; a warp to a row where there are more rows
    // than blocks of 128 run at a time.  Measured (us, bf16, five alternatives; a warp / 128 threads): 4096 rows of 2000 logits
    // 17 / 27, of 8100 27 / 37, 1500 of 3292 11 / 13; but 1500 rows of 16000 23 / 22, 4096 of 32000 86 / 65, 600 of 3292 9.2 / 8.7.
    // (128 threads / 256: 4096 rows of 16000 48 / 55, of 32000 65 / 69, but of 131072 237 / 200.)  The K-th largest of a
    // warp's 32 maxima lists some -32 ln(1 - K/32) logits, 44 where K is 24; of 32 the bound is the smallest of them all, and
    // the list overflows (4096 rows of 3292: 123 / 39).
    const int threads = d.parts > 1 || a.vocab > 16384 ? 256 : row_bytes > 16384 || a.rows <= 8 * kSms || a.top > 24 ? 128 : 32;
    const auto go = [&](auto kernel) { return launch(kernel, dim3((unsigned)(a.rows * d.parts)), dim3(threads), 0, st, true, (unsigned)d.parts, d); };
    const auto of = [&](auto type) {
        using T = decltype(type);
        return threads == 256 ? go(serve_logprobs_kernel<T, 256>) : threads == 128 ? go(serve_logprobs_kernel<T, 128>) : go(serve_logprobs_kernel<T, 32>);
    };
    switch (a.dtype) {
    case BCAST_SERVE_BF16: return of(__nv_bfloat16());
    case BCAST_SERVE_FP16: return of(__half());
    default: return of(float());
    }
}
