// bcast_serve_append: queries and keys of new tokens normed for each head and rotated by their positions, keys
// and values put into the requests' caches -- one pass over what a projection left.
//
// A head of up to 128 numbers is 1, 2, 4 or 8 lanes', 16 numbers to a lane, which hold the two 16-byte chunks whose
// numbers are each other's partners in the rotation, so that the rotation needs no exchange; the norm is one sum over
// those lanes.  A token is a warp's, which takes as many heads at a time as it has lanes for ("a round": queries first, then
// keys, then values), or a half's or a quarter's of one where it has few heads.  Its cosines and sines are made once and, with
// the norm's weights, turned into one set of factors for all heads of a kind.  Rounds come through shared memory, four ahead.
// Angles: inv_freq / 2 pi as a 96-bit fraction of a turn, times the position, whole turns cut off: to 2^-63 of a turn, for every
// finite inv_freq and every position; small angles in floats.
// What bounds it, and what it takes on one B200 (bf16, 32 query and 8 key/value heads of 128; in brackets the bytes at the
// measured copy rate): 16384 tokens 64 us without norms (62), 74.5 with: issuing instructions, 2.7 to a cycle and SM, half of the
// time on conversions.  (Norms and rotation together spill 14 to 15 of the 96 registers that 18 warps to an SM leave, around
// the rounds: 1 % of the instructions.)  1024 tokens 10 us (4), 128 5.0: a token's chain of length, angle, head after head.
// One token with 12 heads of 64 2.6, a launch.  Measured against it: cosines by each block of a token's warps (92 us for 16384 normed
// tokens), blocks that stay and take token after token (81 to 136), loads into registers instead of shared memory (80).
#include "serve_device.cuh"
#include "serve_internal.h"

namespace bcast_serve {
namespace {

constexpr int kAppendThreads = 64, kAppendBlocks = 9;  // of a block; blocks to an SM
constexpr int kFill = 16 * kSms;              // warps that are enough
constexpr int kFlight = 4;                    // rounds of loads that a warp has under way

struct AppendDev {
    const void *q, *k, *v, *q_norm, *k_norm;
    const float *inv_freq;
    const int32_t *positions, *axis, *own_len, *new_len, *page_table;
    void *out, *ok, *ov;
    int64_t qs[3], ks[3], vs[3], os[3], oks[3], ovs[3], ps[2];
    int64_t own_cap, num_pages, pts, first;
    int32_t fresh, q_heads, kv_heads, dim, page, page_shift, rot, axes, groups, rounds, lanes_shift, width_shift, items, tokens;
    float eps, per_dim;
};

enum { kStraight = 0, kHalves = 1, kNeighbours = 2 }; // what is turned: nothing, (p, p + rot / 2), (2 p, 2 p + 1)

// One lane's two chunks of a head.
struct Unit {
    uint4 a, b;
};

// Eight 16-bit numbers as four pairs of floats, and back.
template <typename T>
__device__ __forceinline__ void widen8(const uint4 &raw, uint64_t *x)
{
    const uint32_t v[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int i = 0; i < 4; i++) {
        if constexpr (std::is_same_v<T, __nv_bfloat16>) {
            x[i] = pair(__uint_as_float(v[i] << 16), __uint_as_float(v[i] & 0xffff0000u));
        } else {
            const float2 f = __half22float2(*(const __half2 *)&v[i]);
            x[i] = pair(f.x, f.y);
        }
    }
}
template <typename T>
__device__ __forceinline__ uint4 narrow8(const uint64_t *x)
{
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        float a, b;
        unpair(x[i], a, b);
        if constexpr (std::is_same_v<T, __nv_bfloat16>) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(v[i]) : "f"(b), "f"(a));
        else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(v[i]) : "f"(b), "f"(a));
    }
    return make_uint4(v[0], v[1], v[2], v[3]);
}

// Cosine and sine of `position` times `inv_freq` = m 2^e, m a whole number of 24 bits.  The angle is reduced in whole numbers, as
// Payne and Hanek do it: m times the 128 bits of 1 / 2 pi that matter behind 2^e is the fraction of a turn that one position
// makes, that times the position the fraction that all of them make, whole turns cut off, to 2^-63.  What is left of the nearest
// quarter of a turn goes to sincospi as a float, so that small sines and cosines keep their digits.  An angle below 2^-6 needs no
// reduction and is multiplied out in floats: a fixed number of places behind the point would leave it few.
__device__ __forceinline__ float2 turn_of(float inv_freq, int64_t position)
{
    uint32_t k0 = 0x28be60dbu, k1 = 0x9391054au, k2 = 0x7f09d5f4u, k3 = 0x7d4d3770u;       // 1 / 2 pi, 32 bits each
    const uint32_t bits = __float_as_uint(inv_freq), field = bits >> 23 & 255u;
    const uint32_t m = (bits & 0x7fffffu) | (field ? 0x800000u : 0u);
    const uint32_t by = (uint32_t)(position < 0 ? -position : position);                   // below 2^32: both parts of a sum are below 2^31
    int e = (int)(field ? field : 1u) - 150;
    if (e > 0) {
        // (from 2^24 on: the bits from e on)
        uint32_t k4 = 0x36d8a566u, k5 = 0x4f10e410u, k6 = 0x7f9458eau, k7 = 0xf7aef158u;
        for (; e >= 32; e -= 32) {
            k0 = k1, k1 = k2, k2 = k3, k3 = k4;
            k4 = k5, k5 = k6, k6 = k7, k7 = 0;
        }
        k0 = __funnelshift_l(k1, k0, e);
        k1 = __funnelshift_l(k2, k1, e);
        k2 = __funnelshift_l(k3, k2, e);
        k3 = __funnelshift_l(k4, k3, e);
        e = 0;
    }
    uint64_t t = (uint64_t)m * k3;
    t = (uint64_t)m * k2 + (t >> 32);
    uint32_t s0 = (uint32_t)t;                        // s0 to s3: from 2^-96 up; the places below make less than 2^-64 of a turn
    t = (uint64_t)m * k1 + (t >> 32);
    uint32_t s1 = (uint32_t)t;
    t = (uint64_t)m * k0 + (t >> 32);
    uint32_t s2 = (uint32_t)t, s3 = (uint32_t)(t >> 32);
    // (angles from 2^-6 on have e of -61 at least)
    const int right = -e;
    if (right >= 32) {
        s0 = s1, s1 = s2, s2 = s3, s3 = 0;
    }
    s0 = __funnelshift_r(s0, s1, right);
    s1 = __funnelshift_r(s1, s2, right);
    s2 = __funnelshift_r(s2, s3, right);
    // s0 to s2 are 2^-96, 2^-64 and 2^-32 of a turn
    t = (uint64_t)s0 * by;
    t = (uint64_t)s1 * by + (t >> 32);
    const uint64_t turns = (t & 0xffffffffu) | (uint64_t)((uint32_t)(t >> 32) + s2 * by) << 32;
    uint32_t quarters = (uint32_t)((turns + (1ull << 61)) >> 62);
    float half_turns = (float)(int64_t)(turns - ((uint64_t)quarters << 62)) * 1.0842021724855044e-19f;      // 2^-63
    const float angle = fabsf(inv_freq) * (float)by;
    if (angle < 0.015625f) {
        half_turns = angle * 0.318309886f;
        quarters = 0;
    }
    float2 r, q;
    sincospif(half_turns, &r.y, &r.x);
    q = quarters & 1u ? make_float2(-r.y, r.x) : r;
    r = quarters & 2u ? make_float2(-q.x, -q.y) : q;
    if ((bits >> 31 != 0) != (position < 0)) r.y = -r.y;
    return r;
}

// What a lane's 16 numbers are multiplied by, norm weights and rotation in one, two numbers to an entry.  Halves:
//   y_a = x_a aa + x_b ab,  y_b = x_a ba + x_b bb       (aa = w_a cos, ab = -w_b sin, ba = w_a sin, bb = w_b cos)
// neighbours, within each chunk:
//   y = x aa + swapped(x) ab, and the same with bb and ba for the second
struct Factors {
    uint64_t aa[4], ab[4], ba[4], bb[4];
};

template <int TURN, bool NORM>
__device__ __forceinline__ void turn_and_weigh(uint64_t *a, uint64_t *b, const Factors &f, bool turned_a, bool turned_b)
{
#pragma unroll
    for (int j = 0; j < 4; j++) {
        const uint64_t p = a[j], q = b[j];
        float x, y;
        if (TURN == kHalves && turned_a) {            // (one with the other)
            a[j] = fma2(p, f.aa[j], mul2(q, f.ab[j]));
            b[j] = fma2(p, f.ba[j], mul2(q, f.bb[j]));
            continue;
        }
        if (TURN == kNeighbours && turned_a) {
            unpair(p, x, y);
            a[j] = fma2(p, f.aa[j], mul2(pair(y, x), f.ab[j]));
        } else if (NORM) {
            a[j] = mul2(p, f.aa[j]);
        }
        if (TURN == kNeighbours && turned_b) {
            unpair(q, x, y);
            b[j] = fma2(q, f.bb[j], mul2(pair(y, x), f.ba[j]));
        } else if (NORM) {
            b[j] = mul2(q, f.bb[j]);
        }
    }
}

// Sixteen bytes on their way to shared memory; nothing where `in` does not hold.
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool in)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p cp.async.cg.shared.global [%0], [%1], 16;\n\t}" ::"r"(dst), "l"(src), "r"((uint32_t)in) : "memory");
}

template <typename T, bool NORM, int TURN>
__global__ void __launch_bounds__(kAppendThreads, kAppendBlocks)
serve_append_kernel(const __grid_constant__ AppendDev d)
{
    __shared__ __align__(16) uint4 ring[kFlight][2][kAppendThreads];          // each lane's chunks of the next rounds
    __shared__ __align__(16) float turns_of[kAppendThreads / 8][2][64];       // each token's cosines and sines
    wait_previous();
    launch_next();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    // a token has `width` lanes, a head `lanes` of them
    const int lanes = 1 << d.lanes_shift, width = 1 << d.width_shift;
    const int u = lane & (lanes - 1), sub = (lane & (width - 1)) >> d.lanes_shift, at_once = width >> d.lanes_shift;
    const int item = blockIdx.x * (kAppendThreads / 32) + warp;
    if (item >= d.items) return;
    const int share = d.groups == 1 ? item : item / d.groups, group = item - share * d.groups;
    const int token = (share << (5 - d.width_shift)) + (lane >> d.width_shift);
    const bool exists = token < d.tokens;
    const int b = exists ? token / d.fresh : 0, i = exists ? token - b * d.fresh : 0;
    const int32_t length = d.own_len[b], fresh = d.new_len ? d.new_len[b] : d.fresh;
    const int64_t slot = (int64_t)length - d.fresh + i;
    // this lane's chunks (neighbouring lanes have neighbouring chunks, so that whole sectors come and go: partners in the
    // halves' rotation, or as many chunks apart as there are lanes)
    const int units = d.rot / 16, chunks = d.dim / 8;
    const bool paired = TURN == kHalves && u < units;
    const int ca = TURN != kHalves || paired ? u : 2 * u, cb = TURN != kHalves ? u + lanes : paired ? u + units : 2 * u + 1;
    const bool has_a = exists && ca < chunks, has_b = exists && cb < chunks;
    const bool turned_a = TURN == kHalves ? paired : TURN == kNeighbours && ca * 8 < d.rot, turned_b = TURN == kHalves ? paired : TURN == kNeighbours && cb * 8 < d.rot;
    const int gap = (cb - ca) * 8;

    // which rounds: of queries 0..q_rounds - 1, of keys and of values from there on
    const int q_rounds = (d.q_heads + at_once - 1) / at_once, kv_rounds = (d.kv_heads + at_once - 1) / at_once;
    const int r0 = group * d.rounds, r1 = min(r0 + d.rounds, q_rounds + 2 * kv_rounds);
    const auto kind_of = [&](int r) { return r < q_rounds ? 0 : r < q_rounds + kv_rounds ? 1 : 2; };
    const auto base_of = [&](int kind) { return kind == 0 ? 0 : kind == 1 ? q_rounds : q_rounds + kv_rounds; };
    const auto store = [&](T *dst, const Unit &x, bool in) {
        if (in) *(uint4 *)dst = x.a;
        if (in && has_b) *(uint4 *)(dst + gap) = x.b;
    };
    const Unit nothing = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
    bool there = true;                                // (of a token that is not padding)
    if (d.new_len) {                                  // there may be much padding, which is not read
        there = slot >= 0 && i >= (int64_t)d.fresh - fresh;
        if (!__any_sync(~0u, exists && there)) {
            T *dst = (T *)d.out + b * d.os[0] + i * d.os[1] + ca * 8;
            for (int r = r0; r < min(r1, q_rounds); r++) {
                const int h = r * at_once + sub;
                store(dst + h * d.os[2], nothing, has_a && h < d.q_heads);
            }
            return;
        }
    }

    // The loads, kFlight rounds ahead.  (Without new_len they need not wait for the lengths.)  What is not there is zero.
    const T *src = nullptr;
    int64_t src_step = 0;
    int ahead = r0, src_end = r0, src_left = 0;
    const uint32_t mine = smem_u32(&ring[0][0][threadIdx.x]);
    constexpr uint32_t chunk_b = sizeof(ring[0][0]), round_bytes = sizeof(ring[0]);
#pragma unroll
    for (int k = 0; k < kFlight; k++) ring[k][0][threadIdx.x] = ring[k][1][threadIdx.x] = make_uint4(0, 0, 0, 0);
    const bool read = has_a && there;
    const auto load = [&](int place) {
        if (ahead < r1) {
            if (ahead == src_end) {                   // the next kind begins
                const int kind = kind_of(ahead), h = (ahead - base_of(kind)) * at_once + sub;
                src = kind == 0 ? (const T *)d.q + b * d.qs[0] + i * d.qs[1] + h * d.qs[2]
                    : kind == 1 ? (const T *)d.k + b * d.ks[0] + i * d.ks[1] + h * d.ks[2] : (const T *)d.v + b * d.vs[0] + i * d.vs[1] + h * d.vs[2];
                src += ca * 8;
                src_step = (kind == 0 ? d.qs[2] : kind == 1 ? d.ks[2] : d.vs[2]) * at_once;
                src_left = read ? (kind ? d.kv_heads : d.q_heads) - h : 0;
                src_end = kind == 2 ? r1 : base_of(kind + 1);
            }
            copy16(mine + place * round_bytes, src, src_left > 0);
            copy16(mine + place * round_bytes + chunk_b, src + gap, src_left > 0 && has_b);
            src += src_step;
            src_left -= at_once;
            ahead++;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int k = 0; k < kFlight; k++) load(k);

    there = there && slot >= 0;
    float (*const turns)[64] = turns_of[warp * 4 + (lane >> d.width_shift)];
    if constexpr (TURN != kStraight) {
        const int32_t *positions = d.axes ? d.positions + b * d.ps[0] + i * d.ps[1] : nullptr;
#pragma unroll 2
        for (int p = lane & (width - 1); p < d.rot / 2; p += width) {
            const float f = __ldg(d.inv_freq + p);
            const int axis = d.axis ? __ldg(d.axis + p) : 0;
            const float2 turn = turn_of(f, positions ? (int64_t)__ldg(positions + ((uint32_t)axis < (uint32_t)d.axes ? axis : 0)) : d.first + slot);
            turns[0][p] = turn.x;
            turns[1][p] = turn.y;
        }
        __syncwarp();
    }
    // where the token goes
    int64_t page = b, to = slot;
    bool stored = there && slot < d.own_cap;
    if (stored && d.page_table) {
        const int32_t n = d.page_shift >= 0 ? (int32_t)slot >> d.page_shift : (int32_t)slot / d.page;
        page = d.page_table[(int64_t)b * d.pts + n];
        to = slot - (int64_t)n * d.page;
        stored = page >= 0 && page < d.num_pages;
    }

    int r = r0, place = 0;
#pragma unroll 1
    for (int kind = 0; kind < 3; kind++) {
        const int base = base_of(kind), end = min(r1, kind == 2 ? r1 : base_of(kind + 1));
        if (r >= end) continue;
        const int h = (r - base) * at_once + sub;
        T *dst = kind == 0 ? (T *)d.out + b * d.os[0] + i * d.os[1] + h * d.os[2]
               : kind == 1 ? (T *)d.ok + page * d.oks[0] + to * d.oks[1] + h * d.oks[2] : (T *)d.ov + page * d.ovs[0] + to * d.ovs[1] + h * d.ovs[2];
        dst += ca * 8;
        const int64_t dst_step = (kind == 0 ? d.os[2] : kind == 1 ? d.oks[2] : d.ovs[2]) * at_once;
        int left = has_a && (kind == 0 || stored) ? (kind ? d.kv_heads : d.q_heads) - h : 0;
        const T *weights = NORM && kind < 2 ? (const T *)(kind ? d.k_norm : d.q_norm) : nullptr;
        const bool norm = NORM && weights, turn = TURN != kStraight && kind < 2;
        Factors f;
        if (norm || turn) {
            const uint64_t one = pair(1.0f, 1.0f);
            uint64_t wa[4] = {one, one, one, one}, wb[4] = {one, one, one, one};
            if (norm && has_a) widen8<T>(__ldg((const uint4 *)(weights + ca * 8)), wa);
            if (norm && has_b) widen8<T>(__ldg((const uint4 *)(weights + cb * 8)), wb);
#pragma unroll
            for (int j = 0; j < 4; j++) {
                f.aa[j] = wa[j];
                f.bb[j] = wb[j];
                if (TURN == kHalves && paired) {
                    const uint64_t c = *(const uint64_t *)(turns[0] + 8 * u + 2 * j), s = *(const uint64_t *)(turns[1] + 8 * u + 2 * j);
                    f.aa[j] = mul2(wa[j], c);
                    f.ab[j] = mul2(mul2(wb[j], s), pair(-1.0f, -1.0f));
                    f.ba[j] = mul2(wa[j], s);
                    f.bb[j] = mul2(wb[j], c);
                }
                float x, y;
                if (TURN == kNeighbours && turned_a) {
                    const float c = turns[0][4 * ca + j], s = turns[1][4 * ca + j];
                    unpair(wa[j], x, y);
                    f.aa[j] = pair(x * c, y * c);
                    f.ab[j] = pair(-y * s, x * s);
                }
                if (TURN == kNeighbours && turned_b) {
                    const float c = turns[0][4 * cb + j], s = turns[1][4 * cb + j];
                    unpair(wb[j], x, y);
                    f.bb[j] = pair(x * c, y * c);
                    f.ba[j] = pair(-y * s, x * s);
                }
            }
        }
#pragma unroll 1
        for (; r < end; r++) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kFlight - 1) : "memory");
            Unit y;
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(y.a.x), "=r"(y.a.y), "=r"(y.a.z), "=r"(y.a.w) : "r"(mine + place * round_bytes) : "memory");
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(y.b.x), "=r"(y.b.y), "=r"(y.b.z), "=r"(y.b.w) : "r"(mine + place * round_bytes + chunk_b) : "memory");
            if (norm || turn) {
                uint64_t xa[4], xb[4];
                widen8<T>(y.a, xa);
                widen8<T>(y.b, xb);
                uint64_t by = 0;
                if (norm) {
                    uint64_t squares = mul2(xa[0], xa[0]);
#pragma unroll
                    for (int j = 1; j < 4; j++) squares = fma2(xa[j], xa[j], squares);
#pragma unroll
                    for (int j = 0; j < 4; j++) squares = fma2(xb[j], xb[j], squares);
                    float sum, more;
                    unpair(squares, sum, more);
                    sum += more;
                    for (int o = lanes / 2; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
                    const float inv = rsqrtf(sum * d.per_dim + d.eps);
                    by = pair(inv, inv);
                }
                if (kind < 2) turn_and_weigh<TURN, NORM>(xa, xb, f, turned_a, turned_b);
                if (norm) {
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        xa[j] = mul2(xa[j], by);
                        xb[j] = mul2(xb[j], by);
                    }
                }
                if (norm || turned_a) y.a = narrow8<T>(xa);
                if (norm || turned_b) y.b = narrow8<T>(xb);
            }
            if (!there) y = nothing;
            load(place);                              // into the place that was just read
            store(dst, y, left > 0);
            place = place + 1 == kFlight ? 0 : place + 1;
            dst += dst_step;
            left -= at_once;
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
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
int run(const AppendDev &d, bool norm, int turn, unsigned blocks, cudaStream_t st)
{
    const auto go = [&](auto kernel) { return launch(kernel, dim3(blocks), dim3(kAppendThreads), 0, st, true, 1, d); };
    switch (turn) {
    case kStraight: return norm ? go(serve_append_kernel<T, true, kStraight>) : go(serve_append_kernel<T, false, kStraight>);
    case kHalves: return norm ? go(serve_append_kernel<T, true, kHalves>) : go(serve_append_kernel<T, false, kHalves>);
    default: return norm ? go(serve_append_kernel<T, true, kNeighbours>) : go(serve_append_kernel<T, false, kNeighbours>);
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
    d.page_shift = -1;
    for (int i = 0; i < 31; i++)
        if (d.page == 1 << i) d.page_shift = i;
    d.rot = a.rot;
    d.axes = a.axes;
    d.eps = a.eps;
    d.per_dim = 1.0f / (float)a.dim;
    d.lanes_shift = a.dim <= 16 ? 0 : a.dim <= 32 ? 1 : a.dim <= 64 ? 2 : 3;
    const int64_t tokens = (int64_t)a.batch * a.new_tokens;
    // How many lanes a token has.  A warp, as a rule; half or a quarter of one, a warp's tokens then sharing its instructions,
    // where its heads leave much of the warp idle and the tokens still fill the SMs.  Measured (us, 32 / 8 lanes): 40362 tokens of
    // 2 + 2 + 2 heads of 64 50 / 24, 14514 of 16 + 2 + 2 normed 37 / 26; 16384 of 32 + 8 + 8 of 128 64 / 70, of 64 37 / 39.
    // So from 1.5 times on, by the rounds and two more for what comes before them.
    d.tokens = (int32_t)tokens;
    const auto rounds_of = [&](int shift) {
        const int64_t heads = (1 << shift) >> d.lanes_shift;
        return ceil_div(a.q_heads, heads) + 2 * ceil_div(a.kv_heads, heads);
    };
    d.width_shift = 5;
    for (int shift = 4; shift >= 3; shift--)
        if (shift >= d.lanes_shift && tokens << shift >= 32 * kFill && 3 * (rounds_of(shift) + 2) << shift <= 2 * (rounds_of(5) + 2) << 5) d.width_shift = shift;
    const int64_t rounds = rounds_of(d.width_shift);
    // Few tokens: a warp to every round; otherwise to all of a token's.
    const bool few = tokens * rounds <= 16 * kSms;
    d.rounds = (int32_t)(few ? 1 : rounds);
    d.groups = (int32_t)ceil_div(rounds, d.rounds);
    d.items = (int32_t)(ceil_div(tokens << d.width_shift, 32) * d.groups);
    const int64_t blocks = ceil_div(d.items, kAppendThreads / 32);
    const bool norm = a.q_norm || a.k_norm;
    const int turn = a.rot == 0 ? kStraight : a.interleaved ? kNeighbours : kHalves;
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    return a.dtype == BCAST_SERVE_BF16 ? run<__nv_bfloat16>(d, norm, turn, (unsigned)blocks, st) : run<__half>(d, norm, turn, (unsigned)blocks, st);
}
