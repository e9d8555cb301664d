// Microscaled 4-bit numbers: bcast_serve_pack4, bcast_serve_unpack4, and bcast_serve_linear4, the projection whose
// weights are held so.
//
//   block of 32 along k:  e = max(exponent of its largest magnitude - 2, -127),  code = e2m1(x / 2^e),  x ~ code * 2^e
//   y[t][f] = sum over blocks  2^(eW + ex) * (sum of 32 products of codes)  + bias
// The tensor cores take both operands as they lie (kind::mxf4: 64 values of k to an instruction, a scale to every 32 of
// a row), so W is read once, in 17/32 of a byte a number, and nothing is unpacked on the way.
//   pack kernel     x to codes and scales, four lanes to a block: the call's own x first, in the workspace (up to 8 tokens
//                   the product's blocks do it themselves)
//   product kernel  tiles of 128 features x NT tokens as in bcast_serve_linear: features on the 128 lanes of tensor memory,
//                   tokens the instruction's N.  A stage is 256 values of k: codes by TMA, rows of 128 bytes, and scales,
//                   which are laid out so that a stage's are one run of memory, by bulk copies; tcgen05.cp brings
//                   them to tensor memory, where the instruction wants them
// What bounds them, and what they take on one B200 (bf16; device time, in brackets the bytes at the measured copy rate):
// 65536 x 4096 to codes and back 214 us (208): memory.  8192 tokens, 4096 -> 4096 68 us (22), of which x 15: the product's 52
// are 5.3 PFLOP/s; its pairs of blocks wait on the ring of six stages, about 2700 cycles from a stage's last product to
// its next one's arrival, where the products of six stages take 2690.  The stages are 640 MB in all, 12.3 TB/s out of L2, about
// what a broadcast moves through it (12.5): those cycles may be a queue, which no deeper ring would shorten.  64 tokens, 4096 ->
// 4096 7.5 us, one, 2048 -> 2048 3.8: launches and the latency of the loads.
#include "serve_device.cuh"
#include "serve_internal.h"
#include "serve_tma.h"

#include <cooperative_groups.h>

namespace cg = cooperative_groups;

namespace bcast_serve {
namespace {

constexpr int kBlock = 32;                // numbers that share a scale
constexpr int kAtom = 512;                // bytes of the scales of 128 rows x 4 blocks

// ------------------------------------------------------------------------------------------- to 4 bits and back
constexpr int kPackThreads = 256, kPackRows = 4;      // rows of a thread, whose loads are under way together

// Division by a number that the host knows, as a multiplication (Granlund and Montgomery's): the quotient of n < 2^31 is
// (n + the upper half of n * mul) >> shift.
struct Divisor {
    uint32_t of, mul, shift;
    __device__ __forceinline__ uint32_t quotient(uint32_t n) const { return (__umulhi(n, mul) + n) >> shift; }
};
Divisor divisor(uint32_t of)
{
    Divisor d{of, 0, 0};
    while ((1ull << d.shift) < of) d.shift++;
    d.mul = (uint32_t)((((1ull << d.shift) - of) << 32) / of + 1);
    return d;
}

// Rows of codes, and scales in tiles of `tile` rows of `atoms` x 128 places each, of which each four blocks along k lie
// together: tile r / tile, then block / 4, then the atom.  (Of weights: tile = 128, one atom.)
struct PackDev {
    void *values;
    uint8_t *codes, *scales;
    int64_t vs, cs;
    int32_t rows, padded;                 // padded: rows that have a place among the scales, up to which zeros are written
    int32_t k, tiles_k, atoms;            // tiles_k: of four blocks, to a row
    Divisor eights, tile;                 // eights: threads to a row, a multiple of 16
    uint32_t threads;
};

// Where a thread works: eight numbers from 8 * eight on, of rows row0 to row0 + 3.  The rows' scales are in one tile and
// in one of its groups of 32, so 16 bytes apart from `scale` on.
struct Eights {
    int32_t row0, eight;
    int64_t scale;
    bool there;
    __device__ __forceinline__ explicit Eights(const PackDev &d)
    {
        const uint32_t at = blockIdx.x * kPackThreads + threadIdx.x, group = d.eights.quotient(at);
        row0 = (int32_t)group * kPackRows;
        eight = (int32_t)(at - group * d.eights.of);
        there = at < d.threads && eight * 8 < d.k;
        const uint32_t tile = d.tile.quotient(row0), r = (uint32_t)row0 - tile * d.tile.of, block = (uint32_t)eight / 4;
        scale = (((int64_t)tile * d.tiles_k + block / 4) * d.atoms + r / 128) * kAtom + r % 32 * 16 + r % 128 / 32 * 4 + block % 4;
    }
};

// The scale's byte from the largest magnitude's bits: its exponent field less 2; 255 for what is not finite.
__device__ __forceinline__ uint32_t scale_of(uint32_t most) { return most >= 0x7f800000u ? 255u : (uint32_t)max((int)(most >> 23) - 2, 0); }
// What a block's numbers are multiplied by before they are rounded: 2^(127 - e).
__device__ __forceinline__ float inverse_of(uint32_t e) { return __uint_as_float(e == 255 ? 0u : (254u - e) << 23); }
// The number a scale's byte stands for: 2^(e - 127).
__device__ __forceinline__ float power_of(uint32_t e) { return __uint_as_float(e == 255 ? 0x7fc00000u : e ? e << 23 : 0x00400000u); }

// Eight numbers to codes, the first in the lowest bits: to nearest, to the even code of two as near, 6 at most.
__device__ __forceinline__ uint32_t codes_of(const float *x)
{
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r) : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]));
    return r;
}
__device__ __forceinline__ void numbers_of(uint32_t codes, uint64_t *x)
{
    uint32_t h[4];
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\tcvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(codes));
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const float2 v = __half22float2(*(const __half2 *)&h[i]);
        x[i] = pair(v.x, v.y);
    }
}

template <typename T> struct Eight {
    uint4 v[sizeof(T) / 2];
};
// Eight numbers as four pairs of floats, and back.
template <typename T>
__device__ __forceinline__ void widen8(const Eight<T> &raw, uint64_t *x)
{
    const uint32_t *v = (const uint32_t *)&raw;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        if constexpr (std::is_same_v<T, float>) {
            x[i] = pair(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1]));
        } else if constexpr (std::is_same_v<T, __nv_bfloat16>) {
            x[i] = pair(__uint_as_float(v[i] << 16), __uint_as_float(v[i] & 0xffff0000u));
        } else {
            const float2 f = __half22float2(*(const __half2 *)&v[i]);
            x[i] = pair(f.x, f.y);
        }
    }
}
template <typename T>
__device__ __forceinline__ void narrow8(Eight<T> &raw, const uint64_t *x)
{
    uint32_t *v = (uint32_t *)&raw;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        float a, b;
        unpair(x[i], a, b);
        if constexpr (std::is_same_v<T, float>) {
            v[2 * i] = __float_as_uint(a);
            v[2 * i + 1] = __float_as_uint(b);
        } else if constexpr (std::is_same_v<T, __nv_bfloat16>) {
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(v[i]) : "f"(b), "f"(a));
        } else {
            asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(v[i]) : "f"(b), "f"(a));
        }
    }
}
// The largest magnitude's bits as a float's, over the four lanes of a block; NaN is the largest.  16-bit numbers are
// compared two at a time.
template <typename T>
__device__ __forceinline__ uint32_t largest(const Eight<T> &raw)
{
    const uint32_t *v = (const uint32_t *)&raw;
    if constexpr (std::is_same_v<T, float>) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) m = max(m, v[i] & 0x7fffffffu);
        m = max(m, __shfl_xor_sync(~0u, m, 1));
        return max(m, __shfl_xor_sync(~0u, m, 2));
    } else {
        const auto larger = [](uint32_t a, uint32_t b) {              // NaN, whose bits are above infinity's, stays
            uint32_t r;
            if constexpr (std::is_same_v<T, __nv_bfloat16>) asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
            else asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
            return r;
        };
        uint32_t m = larger(larger(v[0] & 0x7fff7fffu, v[1] & 0x7fff7fffu), larger(v[2] & 0x7fff7fffu, v[3] & 0x7fff7fffu));
        m = larger(m, __shfl_xor_sync(~0u, m, 1));
        m = larger(m, __shfl_xor_sync(~0u, m, 2));
        m = max(m & 0xffffu, m >> 16);
        if constexpr (std::is_same_v<T, __nv_bfloat16>) return m << 16;
        else return __float_as_uint(__half2float(__ushort_as_half((unsigned short)m)));
    }
}

// Four neighbouring lanes hold a block of 32, sixteen the four blocks whose scales are neighbours.
template <typename T>
__global__ void __launch_bounds__(kPackThreads)
serve_pack4_kernel(const __grid_constant__ PackDev d)
{
    // (in this order: the kernel of a product reads W before it waits for this one, and W may be what came before this one)
    wait_previous();
    launch_next();
    const Eights e(d);
    Eight<T> raw[kPackRows];
    const T *src = (const T *)d.values + e.row0 * d.vs + e.eight * 8;
#pragma unroll
    for (int r = 0; r < kPackRows; r++) {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) / 2); i++)
            raw[r].v[i] = e.there && e.row0 + r < d.rows ? __ldg((const uint4 *)src + i) : make_uint4(0, 0, 0, 0);
        src += d.vs;
    }
    uint8_t *codes = d.codes + e.row0 * d.cs + e.eight * 4;
#pragma unroll
    for (int r = 0; r < kPackRows; r++) {
        const uint32_t s = scale_of(largest<T>(raw[r]));
        uint64_t x[4];
        widen8<T>(raw[r], x);
        const float by = inverse_of(s);
        const uint64_t two = pair(by, by);
        float y[8];
#pragma unroll
        for (int i = 0; i < 4; i++) unpair(mul2(x[i], two), y[2 * i], y[2 * i + 1]);
        if (e.there && e.row0 + r < d.rows) *(uint32_t *)codes = s == 255 ? 0u : codes_of(y);
        codes += d.cs;
        uint32_t four = s | __shfl_down_sync(~0u, s, 4) << 8;
        four |= __shfl_down_sync(~0u, four, 8) << 16;
        // (what is past k read as zeros, whose scale is 0)
        if (threadIdx.x % 16 == 0 && e.there && e.row0 + r < d.padded) *(uint32_t *)(d.scales + e.scale + r * 16) = four;
    }
}

template <typename T>
__global__ void __launch_bounds__(kPackThreads)
serve_unpack4_kernel(const __grid_constant__ PackDev d)
{
    wait_previous();
    launch_next();
    const Eights e(d);
    if (!e.there) return;
    uint32_t codes[kPackRows], s[kPackRows];
#pragma unroll
    for (int r = 0; r < kPackRows; r++) {
        const bool in = e.row0 + r < d.rows;
        codes[r] = in ? __ldg((const uint32_t *)(d.codes + (e.row0 + r) * d.cs + e.eight * 4)) : 0u;
        s[r] = in ? __ldg(d.scales + e.scale + r * 16) : 0u;
    }
    T *dst = (T *)d.values + e.row0 * d.vs + e.eight * 8;
#pragma unroll
    for (int r = 0; r < kPackRows; r++) {
        if (e.row0 + r >= d.rows) break;
        uint64_t x[4];
        numbers_of(codes[r], x);
        const float by = power_of(s[r]);
        const uint64_t two = pair(by, by);
#pragma unroll
        for (int i = 0; i < 4; i++) x[i] = mul2(x[i], two);
        Eight<T> raw;
        narrow8<T>(raw, x);
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) / 2); i++) ((uint4 *)(dst + r * d.vs))[i] = raw.v[i];
    }
}

// ------------------------------------------------------------------------------------------- product
constexpr int kFeatures = 128;            // features per tile: the lanes of tensor memory
constexpr int kDepth = 256;               // values of k per stage: 128 bytes of codes, one swizzled row
constexpr int kProductThreads = 192, kFusedThreads = 320;
constexpr int kFusedTokens = 8;           // up to which the product's blocks pack x themselves
constexpr int kMaxSplit = 8;              // blocks of a cluster that share one tile's k

template <int NT, bool FUSED> struct Tile {
    static constexpr int codes_w = kFeatures * 128, codes_x = NT * 128, scales_w = 2 * kAtom, scales_x = 2 * kAtom;
    static constexpr int stage = codes_w + codes_x + scales_w + scales_x;
    static constexpr int stages = FUSED ? 8 : NT == 128 ? 3 : 4;   // FUSED: one to each warp that packs x
    static constexpr int at_w = NT, at_x = at_w + 8, used = at_x + 8;      // tensor memory's columns of scales
    static constexpr int columns = used <= 64 ? 64 : used <= 128 ? 128 : 256;
    static constexpr size_t smem = (size_t)stage * stages + 1024;  // + alignment
    static_assert(NT <= 128 && stage % 1024 == 0 && used <= columns, "");
    static_assert(NT * kFeatures * 4 <= stage * stages, "partial sums take the stages' place");
};

struct ProductDev {
    const void *bias, *x;
    int64_t xs;
    const uint8_t *scales_w, *scales_x;
    void *y;
    int *status;
    int give_up;                          // 1: begin as if a wait had run out
    int64_t ys;
    int32_t tokens, k, n, f_tiles, t_tiles, tiles_k;
};

// Descriptor of 32 rows of 16 bytes, one after the other, as tcgen05.cp takes them.
__device__ __forceinline__ uint64_t scales_desc(uint32_t src) { return (uint64_t)((src >> 4) & 0x3fffu) | (uint64_t)(128 >> 4) << 32 | 1ull << 46; }

// The instructions that follow are issued by the thread with `lead` set of a warp in uniform control flow, so that their
// operands stay in uniform registers, where they are wanted.  (One thread in a loop of its own took about 110 cycles to issue
// each: 8192 tokens, 4096 -> 4096 took 105 us, however much or little was loaded.)

// A tile; sixteen bytes and more, both ends on 16-byte boundaries; the bytes that a barrier is to wait for.
__device__ __forceinline__ void load_tile(uint32_t lead, uint32_t dst, const CUtensorMap *m, int x, int y, uint32_t bar)
{
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %5, 0;\n\t"
                 "@q cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n\t}"
                 ::"r"(dst), "l"((uint64_t)m), "r"(x), "r"(y), "r"(bar), "r"(lead) : "memory");
}
__device__ __forceinline__ void load_bytes(uint32_t lead, uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %4, 0;\n\t"
                 "@q cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n\t}"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar), "r"(lead) : "memory");
}
__device__ __forceinline__ void expect(uint32_t lead, uint32_t bar, uint32_t bytes)
{
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %2, 0;\n\t@q mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}"
                 ::"r"(bar), "r"(bytes), "r"(lead) : "memory");
}
// 32 rows to 32 lanes of four columns, the same for each of the four warps' lanes.
__device__ __forceinline__ void scales_to_tmem(uint32_t lead, uint32_t dst, uint64_t src)
{
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %2, 0;\n\t@q tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;\n\t}"
                 ::"r"(dst), "l"(src), "r"(lead) : "memory");
}
// Instruction descriptor, kind::mxf4: e2m1 operands, scales that are powers of two; `which` of a column's two pairs of
// scales the instruction takes.
__device__ __forceinline__ constexpr uint32_t mx4_desc(int m, int n, int which)
{
    return 1u << 7 | 1u << 10 | (uint32_t)(n >> 3) << 17 | 1u << 23 | (uint32_t)(m >> 4) << 24 | (uint32_t)(2 * which) << 4 | (uint32_t)(2 * which) << 29;
}
__device__ __forceinline__ void mma_mx4(uint32_t lead, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t scales_a, uint32_t scales_b, bool add)
{
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %6, 0;\n\tsetp.ne.u32 q, %7, 0;\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::mxf4.block_scale.block32 [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(scales_a), "r"(scales_b), "r"((uint32_t)add), "r"(lead) : "memory");
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

// Does `v` hold for all 128 threads of barrier `id`?
__device__ __forceinline__ bool all_of(int id, bool v)
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, %2, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"((uint32_t)v), "r"(id) : "memory");
    return r;
}
// Are four neighbouring results of a row to be written at once?
__device__ __forceinline__ bool whole_rows(const ProductDev &d, int features) { return features % 4 == 0 && d.ys % 4 == 0 && ((uintptr_t)d.y & 7) == 0; }

// One row's 256 values of k from `k0` on to codes and scales in shared memory, a warp to the row, as TMA and the scales'
// layout would have brought them.
template <typename T>
__device__ __forceinline__ void pack_row(uint8_t *codes, uint8_t *scales, int row, const Eight<T> &raw)
{
    const int lane = threadIdx.x % 32;
    const uint32_t s = scale_of(largest<T>(raw));
    uint64_t x[4];
    widen8<T>(raw, x);
    const float by = inverse_of(s);
    const uint64_t two = pair(by, by);
    float y[8];
#pragma unroll
    for (int i = 0; i < 4; i++) unpair(mul2(x[i], two), y[2 * i], y[2 * i + 1]);
    *(uint32_t *)(codes + swizzled(row, lane / 4, 128) + lane % 4 * 4) = s == 255 ? 0u : codes_of(y);
    uint32_t four = s | __shfl_down_sync(~0u, s, 4) << 8;
    four |= __shfl_down_sync(~0u, four, 8) << 16;
    if (lane % 16 == 0) *(uint32_t *)(scales + lane / 16 * kAtom + row % 32 * 16 + row / 32 * 4) = four;
}

// Grid: one tile of features and tokens, features first, to a block, or to a cluster that shares its k.  A block has one warp
// that loads, one that issues the matrix instructions and four that bring the accumulator from tensor memory to y.
// FUSED: few tokens, whose x eight warps pack for their own block, a stage to a warp: each block does it again for itself, but
// a call is one launch.  Device time in us with a kernel for x / without, k = 4096, n = 4096: 1 token, 2048 -> 2048 5.2 / 3.7 (a
// public call among others 9.5 / 5.8); 4 6.3 / 5.7; 16 6.7 / 8.8; 1, n = 16384 10.4 / 8.8.
template <typename T, int NT, bool FUSED>
__global__ void __launch_bounds__(FUSED ? kFusedThreads : kProductThreads, FUSED ? 1 : 2)
serve_linear4_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ ProductDev d)
{
    using S = Tile<NT, FUSED>;
    constexpr int threads = FUSED ? kFusedThreads : kProductThreads;
    extern __shared__ uint8_t raw_smem[];
    __shared__ __align__(8) uint64_t bars[3 * S::stages + 2];
    __shared__ uint32_t tmem_at;
    __shared__ int gave_up;

    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const cg::cluster_group cluster = cg::this_cluster();
    const int split = (int)cluster.num_blocks(), part = (int)cluster.block_rank();

    uint8_t *smem = (uint8_t *)(((uintptr_t)raw_smem + 1023) & ~(uintptr_t)1023);
    const uint32_t stage0 = smem_u32(smem);
    const uint32_t full = smem_u32(bars), empty = full + 8 * S::stages, filled = empty + 8 * S::stages, acc_full = filled + 8 * S::stages,
                   drained = acc_full + 8;

    // which tile, and of k which stages
    const int k_blocks = (d.k + kDepth - 1) / kDepth;
    const int kb0 = (int)((int64_t)k_blocks * part / split), kb1 = (int)((int64_t)k_blocks * (part + 1) / split);
    const int tile = blockIdx.x / split, f_tile = tile % d.f_tiles, t_tile = tile / d.f_tiles, f0 = f_tile * kFeatures, t0 = t_tile * NT;

    if (warp == 1) {
        tmem_alloc(smem_u32(&tmem_at), S::columns);
    } else if (tid == 0) {
        gave_up = d.give_up;
        for (int i = 0; i < S::stages; i++) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
            if (FUSED) mbar_init(filled + 8 * i, 1);
        }
        mbar_init(acc_full, 1);
        mbar_init(drained, 1);
        mbar_init_fence();
        if (!FUSED) tma_prefetch(&map_x);
        tma_prefetch(&map_w);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_at;
    if (FUSED) {
        wait_previous();
        launch_next();
    }

    int issued = 0;                                   // loads, of the thread that issues them
    if (warp == 0) {
        // ---- loads.  W is there already: its first stages are on their way before x is packed.
        const uint32_t lead = elect_one();
        Ring<S::stages> ring;
        auto load = [&](int kb, int slot, bool w) {
            const uint32_t bar = full + 8 * slot, at = stage0 + slot * S::stage, scales = at + S::codes_w + S::codes_x;
            const int kt = 2 * kb, have = min(2, d.tiles_k - kt);                  // tiles of scales
            if (w) {
                expect(lead, bar, S::codes_w + have * kAtom + (FUSED ? 0 : S::codes_x + have * kAtom));
                load_tile(lead, at, &map_w, kb * 64, f0, bar);
                load_bytes(lead, scales, d.scales_w + ((int64_t)f_tile * d.tiles_k + kt) * kAtom, have * kAtom, bar);
                issued++;
            } else {
                load_tile(lead, at + S::codes_w, &map_x, kb * 64, t0, bar);
                load_bytes(lead, scales + S::scales_w, d.scales_x + ((int64_t)t_tile * d.tiles_k + kt) * kAtom, have * kAtom, bar);
            }
        };
        const int ahead = min(S::stages, kb1 - kb0);
        for (int i = 0; i < ahead; i++) load(kb0 + i, i, true);
        if (!FUSED) wait_previous();                  // the codes and scales of x
        for (int kb = kb0; kb < kb1; kb++) {
            if (kb - kb0 >= ahead) {
                // (the warp that issues the products goes on after it gave up: a slot may be free then whose load is under way)
                if (!__all_sync(~0u, mbar_wait(empty + 8 * ring.slot, ring.parity ^ 1u, &gave_up) && !*(volatile int *)&gave_up)) break;
                load(kb, ring.slot, true);
            }
            if (!FUSED) load(kb, ring.slot, false);
            ring.step();
        }
        __syncwarp();
    } else if (warp == 1) {
        // ---- matrix instructions.  A wait that gives up does not leave the loop: the ones after it give up at once, and what
        // is still issued only touches this block's own memory.
        const uint32_t lead = elect_one();
        const uint64_t a0 = smem_desc(stage0), b0 = smem_desc(stage0 + S::codes_w), s0 = scales_desc(stage0 + S::codes_w + S::codes_x);
        Ring<S::stages> ring;
        for (int kb = kb0; kb < kb1; kb++) {
            mbar_wait(full + 8 * ring.slot, ring.parity, &gave_up);
            if (FUSED) mbar_wait(filled + 8 * ring.slot, ring.parity, &gave_up);
            __syncwarp();
            tc_fence_after();
            const uint64_t step = (uint64_t)(ring.slot * (S::stage >> 4)), a = a0 + step, b = b0 + step, s = s0 + step;
            const int steps = min(kDepth / 64, (d.k - kb * kDepth + 63) / 64);
#pragma unroll
            for (int h = 0; h < 2; h++) {
                if (2 * h >= steps) break;
                scales_to_tmem(lead, tmem + S::at_w + 4 * h, s + h * (kAtom >> 4));
                scales_to_tmem(lead, tmem + S::at_x + 4 * h, s + ((S::scales_w + h * kAtom) >> 4));
            }
#pragma unroll
            for (int i = 0; i < kDepth / 64; i++) {
                if (i >= steps) break;
                mma_mx4(lead, tmem, a + 2 * i, b + 2 * i, mx4_desc(kFeatures, NT, i % 2), tmem + S::at_w + i / 2 * 4, tmem + S::at_x + i / 2 * 4, kb > kb0 || i > 0);
            }
            mma_commit_warp(lead, empty + 8 * ring.slot);
            ring.step();
        }
        mma_commit_warp(lead, acc_full);
        __syncwarp();
    } else {
        if (FUSED) {
            // ---- x: a warp to a stage, every eighth, which so is always in the same place; four rows to a batch, of which
            // the next is under way while one is packed
            constexpr int at_once = 4;
            const T *x = (const T *)d.x + (int64_t)t0 * d.xs + lane * 8;
            const int live = min(NT, d.tokens - t0), slot = warp - 2;
            uint8_t *codes = smem + slot * S::stage + S::codes_w, *scales = codes + S::codes_x + S::scales_w;
            auto fetch = [&](Eight<T> *raw, int kb, int r0) {
#pragma unroll
                for (int r = 0; r < at_once; r++)
                    if (kb < kb1 && r0 + r < live)
                        raw[r].v[0] = kb * kDepth + lane * 8 < d.k ? __ldg((const uint4 *)(x + (r0 + r) * d.xs + (int64_t)kb * kDepth)) : make_uint4(0, 0, 0, 0);
            };
            Eight<T> next[at_once];
            int kb = kb0 + slot, r0 = 0;
            uint32_t parity = 1;
            fetch(next, kb, 0);
            while (kb < kb1) {
                Eight<T> raw[at_once];
#pragma unroll
                for (int r = 0; r < at_once; r++) raw[r] = next[r];
                const bool last = r0 + at_once >= live;
                fetch(next, last ? kb + S::stages : kb, last ? 0 : r0 + at_once);
                if (r0 == 0 && !__all_sync(~0u, mbar_wait(empty + 8 * slot, parity, &gave_up) && !*(volatile int *)&gave_up)) break;
#pragma unroll
                for (int r = 0; r < at_once; r++)
                    if (r0 + r < live) pack_row<T>(codes, scales, r0 + r, raw[r]);
                r0 += at_once;
                if (!last) continue;
                fence_async_proxy();
                __syncwarp();
                if (lane == 0) mbar_arrive(filled + 8 * slot);
                r0 = 0;
                kb += S::stages;
                parity ^= 1u;
            }
            __syncwarp();
        }
        // ---- the accumulator's way out.  A warp may touch the 32 lanes of its number modulo 4.
        const int quarter = warp % 4, f = quarter * 32 + lane;
        const bool ok = warp < 6 && all_of(1, mbar_wait(acc_full, 0, &gave_up));
        tc_fence_after();
        if (ok && split == 1) {
            const float bias = d.bias && f0 + f < d.n ? to_f32(((const T *)d.bias)[f0 + f]) : 0.0f;
            const uint32_t src = tmem + ((uint32_t)(quarter * 32) << 16);
            T *y = (T *)d.y + (int64_t)t0 * d.ys + f0 + f;
            const int live = f0 + f < d.n ? min(NT, d.tokens - t0) : 0;
#pragma unroll 2
            for (int c = 0; c < NT; c += 16) {
                uint32_t v[16];
                tmem_load16(src + c, v);
                tmem_wait_load16(v);
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    if (c + i < live) *y = from_f32<T>(__uint_as_float(v[i]) + bias);
                    y += d.ys;
                }
            }
        }
        tc_fence_before();
    }

    if (split > 1) {
        // The blocks' sums are joined: each puts its own where its stages were, block r of the cluster adds up all of
        // them for its share of the tokens, always in the same order.
        const int share = NT / split;
        if (warp >= 2 && warp < 6) {
            const int quarter = warp % 4, f = quarter * 32 + lane;
#pragma unroll 2
            for (int c = 0; c < NT; c += 16) {
                uint32_t v[16];
                tmem_load16(tmem + ((uint32_t)(quarter * 32) << 16) + c, v);
                tmem_wait_load16(v);
#pragma unroll
                for (int i = 0; i < 16; i++) ((uint32_t *)smem)[(c + i) * kFeatures + f] = v[i];
            }
            tc_fence_before();
        }
        __syncwarp();
        cluster_arrive();
        cluster_wait();
        const int features = min(kFeatures, d.n - f0), c0 = part * share, c1 = min(c0 + share, d.tokens - t0);
        const bool whole = whole_rows(d, features);
#pragma unroll 2
        for (int i = c0 * (kFeatures / 4) + tid; i < c1 * (kFeatures / 4); i += threads) {
            const int f = i % (kFeatures / 4) * 4, c = i / (kFeatures / 4);
            if (f >= features) continue;
            float4 p[kMaxSplit];
#pragma unroll
            for (int b = 0; b < kMaxSplit; b++)
                p[b] = b < split ? cluster.map_shared_rank((const float4 *)smem, b)[i] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            float v[4] = {};
#pragma unroll
            for (int b = 0; b < kMaxSplit; b++) {
                v[0] += p[b].x;
                v[1] += p[b].y;
                v[2] += p[b].z;
                v[3] += p[b].w;
            }
            T *y = (T *)d.y + (int64_t)(t0 + c) * d.ys + f0 + f;
            __align__(8) T r[4];
#pragma unroll
            for (int k = 0; k < 4; k++)
                r[k] = from_f32<T>(v[k] + (d.bias && f + k < features ? to_f32(((const T *)d.bias)[f0 + f + k]) : 0.0f));
            if (whole) {
                *(uint2 *)y = *(const uint2 *)r;
            } else {
#pragma unroll
                for (int k = 0; k < 4; k++)
                    if (f + k < features) y[k] = r[k];
            }
        }
        cluster_arrive();                             // a block's memory stays until the others have read it
        cluster_wait();
    }
    __syncthreads();
    tc_fence_after();
    // (nobody sets gave_up from here on)
    if (warp == 1) {
        if (gave_up) {                                // what was issued ends before tensor memory is given up
            if (lane == 0) {
                mma_commit(drained);
                mbar_drain(drained, 0);
            }
            __syncwarp();
        }
        tmem_free(tmem, S::columns);
    }
    if (tid == 0 && gave_up) {                        // and loads, before the block's memory is
        drain_loads<S::stages>(full, issued);
        atomicExch(d.status, 1);
    }
}

// ------------------------------------------------------------------------------------------- product, two SMs to a tile
// Many tokens: the two blocks of a cluster take 256 features x 224 tokens together.  Each holds its own 128 features' rows
// of W and half of the tokens' rows, which the pair's instruction (cta_group::2, issued by the first block) reads from
// both, so that each block fetches 240 rows for what takes 352 alone.  Accumulators and scales (its own features', all
// tokens') are in each block's tensor memory.  A warp of each block brings W, another one x; all four arrive on one barrier
// of the first block (four barriers to a stage cost the warp that issues the products more time than the products take), and
// the matrix instructions' completion arrives on both blocks'.
constexpr int kPairTokens = 224, kPairThreads = 352;

struct PairTile {
    static constexpr int half = kPairTokens / 2;
    static constexpr int codes_w = kFeatures * 128, codes_x = half * 128, scales_w = 2 * kAtom, scales_x = 4 * kAtom;
    static constexpr int stage = codes_w + codes_x + scales_w + scales_x, stages = 6;
    static constexpr int at_scales = 2 * kPairTokens, scales = 24;     // columns: two accumulators, then two stages' scales
    static constexpr size_t smem = (size_t)stage * stages + 1024;
    static_assert(stage % 1024 == 0 && codes_x % 1024 == 0 && at_scales + 2 * scales <= 512, "");
};

// The first block's copy of a barrier.
__device__ __forceinline__ uint32_t of_first(uint32_t bar)
{
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(bar));
    return r;
}
__device__ __forceinline__ void arrive_at(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void expect_at(uint32_t lead, uint32_t bar, uint32_t bytes)
{
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %2, 0;\n\t@q mbarrier.arrive.expect_tx.shared::cluster.b64 _, [%0], %1;\n\t}"
                 ::"r"(bar), "r"(bytes), "r"(lead) : "memory");
}
// Into this block's memory, arriving on a barrier of the pair's first block.
__device__ __forceinline__ void pair_load(uint32_t lead, uint32_t dst, const CUtensorMap *m, int x, int y, uint32_t bar)
{
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %5, 0;\n\t"
                 "@q cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n\t}"
                 ::"r"(dst), "l"((uint64_t)m), "r"(x), "r"(y), "r"(bar), "r"(lead) : "memory");
}
__device__ __forceinline__ void pair_scales(uint32_t lead, uint32_t dst, uint64_t src)
{
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %2, 0;\n\t@q tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;\n\t}"
                 ::"r"(dst), "l"(src), "r"(lead) : "memory");
}
__device__ __forceinline__ void pair_mma(uint32_t lead, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t scales_a, uint32_t scales_b, bool add)
{
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %6, 0;\n\tsetp.ne.u32 q, %7, 0;\n\t"
                 "@q tcgen05.mma.cta_group::2.kind::mxf4.block_scale.block32 [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(scales_a), "r"(scales_b), "r"((uint32_t)add), "r"(lead) : "memory");
}
// Both blocks' barriers of that place are arrived on.
__device__ __forceinline__ void pair_commit(uint32_t lead, uint32_t bar)
{
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %2, 0;\n\t"
                 "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n\t}"
                 ::"r"(bar), "h"((uint16_t)3), "r"(lead) : "memory");
}

template <typename T>
__global__ void __launch_bounds__(kPairThreads, 1) __cluster_dims__(2, 1, 1)
serve_linear4_pair_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w,
                          const __grid_constant__ CUtensorMap map_sx, const __grid_constant__ CUtensorMap map_sw, const __grid_constant__ ProductDev d)
{
    using S = PairTile;
    extern __shared__ uint8_t raw_smem[];
    __shared__ __align__(8) uint64_t bars[2 * S::stages + 2 * 2 + 1];
    __shared__ uint32_t tmem_at;
    __shared__ int gave_up, issued[5];                // of the first block: stages that the four brought, and whether the other block gave up

    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const int rank = (int)cg::this_cluster().block_rank();

    uint8_t *smem = (uint8_t *)(((uintptr_t)raw_smem + 1023) & ~(uintptr_t)1023);
    const uint32_t stage0 = smem_u32(smem);
    const uint32_t full = smem_u32(bars), empty = full + 8 * S::stages, acc_full = empty + 8 * S::stages, acc_empty = acc_full + 16, drained = acc_empty + 16;
    const int k_blocks = (d.k + kDepth - 1) / kDepth;
    const int first_tile = blockIdx.x / 2, f_pairs = (d.f_tiles + 1) / 2, tiles = f_pairs * d.t_tiles, tile_step = gridDim.x / 2;

    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tmem_at)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else if (tid == 0) {
        gave_up = d.give_up;
        for (int i = 0; i < S::stages; i++) {
            mbar_init(full + 8 * i, 4);
            mbar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; i++) {
            mbar_init(acc_full + 8 * i, 1);
            mbar_init(acc_empty + 8 * i, 16);         // a lane of each warp that empties it, in both blocks
        }
        mbar_init(drained, 1);
        mbar_init_fence();
        tma_prefetch(&map_x);
        tma_prefetch(&map_w);
        tma_prefetch(&map_sx);
        tma_prefetch(&map_sw);
    }
    tc_fence_before();
    __syncthreads();
    cluster_arrive();                                 // the other block's barriers are there too
    cluster_wait();
    tc_fence_after();
    const uint32_t tmem = tmem_at;
    // A wait for all lanes alike.  One that runs out ends the other block's waits too.
    const auto wait = [&](uint32_t bar, uint32_t parity) {
        const bool ok = __all_sync(~0u, mbar_wait(bar, parity, &gave_up));
        if (!ok && lane == 0) *(volatile int *)cg::this_cluster().map_shared_rank(&gave_up, rank ^ 1) = 1;
        return ok;
    };

    if (warp == 0 || warp == 2) {
        // ---- loads: W, or x.  W is there already, x once it is packed.
        const uint32_t lead = elect_one();
        const int which = warp / 2;
        int count = 0;
        Ring<S::stages> ring;
        bool ok = true;
        if (which) wait_previous();
        for (int tile = first_tile; tile < tiles && ok; tile += tile_step) {
            const int f_tile = tile % f_pairs * 2 + rank, t_tile = tile / f_pairs;
            for (int kb = 0; kb < k_blocks; kb++) {
                ok = wait(empty + 8 * ring.slot, ring.parity ^ 1u);
                if (!ok) break;
                const uint32_t bar = of_first(full + 8 * ring.slot), at = stage0 + ring.slot * S::stage, scales = at + S::codes_w + S::codes_x;
                if (which == 0) {
                    expect_at(lead, bar, S::codes_w + S::scales_w);
                    pair_load(lead, at, &map_w, kb * 64, f_tile * kFeatures, bar);
                    pair_load(lead, scales, &map_sw, kb * 256, f_tile, bar);
                } else {
                    // (where the tiles of scales are odd in number, the last of them comes with one that nobody uses)
                    expect_at(lead, bar, S::codes_x + S::scales_x);
                    pair_load(lead, at + S::codes_w, &map_x, kb * 64, t_tile * kPairTokens + rank * S::half, bar);
                    pair_load(lead, scales + S::scales_w, &map_sx, 0, t_tile * d.tiles_k + 2 * kb, bar);
                }
                count++;
                ring.step();
            }
        }
        if (lane == 0) cg::this_cluster().map_shared_rank(issued, 0)[2 * rank + which] = count;
        __syncwarp();
    } else if (warp == 1) {
        if (rank == 0) {
            // ---- matrix instructions, for both blocks.  (Nothing is told to be empty after a wait gave up.)
            const uint32_t lead = elect_one();
            const uint64_t a0 = smem_desc(stage0), b0 = smem_desc(stage0 + S::codes_w), s0 = scales_desc(stage0 + S::codes_w + S::codes_x);
            Ring<S::stages> ring;
            Ring<2> acc;
            uint32_t odd = 0;                         // which of two places the stage's scales go to
            bool ok = true;
            for (int tile = first_tile; tile < tiles && ok; tile += tile_step) {
                if (!(ok = wait(acc_empty + 8 * acc.slot, acc.parity ^ 1u))) break;
                const uint32_t out = tmem + acc.slot * kPairTokens;
                for (int kb = 0; kb < k_blocks; kb++) {
                    if (!(ok = wait(full + 8 * ring.slot, ring.parity))) break;
                    tc_fence_after();
                    const uint64_t step = (uint64_t)(ring.slot * (S::stage >> 4)), a = a0 + step, b = b0 + step, s = s0 + step;
                    const uint32_t to_w = tmem + S::at_scales + odd * S::scales, to_x = to_w + 8;
                    const int steps = min(kDepth / 64, (d.k - kb * kDepth + 63) / 64);
#pragma unroll
                    for (int h = 0; h < 2; h++) {
                        pair_scales(lead, to_w + 4 * h, s + h * (kAtom >> 4));
                        pair_scales(lead, to_x + 8 * h, s + ((S::scales_w + 2 * h * kAtom) >> 4));
                        pair_scales(lead, to_x + 8 * h + 4, s + ((S::scales_w + (2 * h + 1) * kAtom) >> 4));
                    }
#pragma unroll
                    for (int i = 0; i < kDepth / 64; i++) {
                        if (i >= steps) break;
                        pair_mma(lead, out, a + 2 * i, b + 2 * i, mx4_desc(2 * kFeatures, kPairTokens, i % 2), to_w + i / 2 * 4, to_x + i / 2 * 8, kb > 0 || i > 0);
                    }
                    pair_commit(lead, empty + 8 * ring.slot);
                    ring.step();
                    odd ^= 1u;
                }
                if (!ok) break;
                pair_commit(lead, acc_full + 8 * acc.slot);
                acc.step();
            }
        }
        __syncwarp();
    } else {
        // ---- the accumulators' way out: lane f of this block is one of its own 128 features.  Four warps take the tile's
        // first tokens, four the others.  (Through shared memory, to write a row's 256 bytes at once, it took no less: 16 us
        // for 1024 tokens, 4096 -> 4096, against 17, and 30 for 2048 against 25.)
        const int quarter = warp % 4, f = quarter * 32 + lane, side = (warp - 3) / 4, id = 1 + side;
        Ring<2> acc;
        for (int tile = first_tile; tile < tiles; tile += tile_step) {
            // (the four warps go on together, or none does)
            if (!all_of(id, wait(acc_full + 8 * acc.slot, acc.parity))) break;
            tc_fence_after();
            const uint32_t src = tmem + ((uint32_t)(quarter * 32) << 16) + acc.slot * kPairTokens + side * S::half;
            const int f0 = (tile % f_pairs * 2 + rank) * kFeatures, t0 = tile / f_pairs * kPairTokens + side * S::half;
            const float bias = d.bias && f0 + f < d.n ? to_f32(((const T *)d.bias)[f0 + f]) : 0.0f;
            T *y = (T *)d.y + (int64_t)t0 * d.ys + f0 + f;
            const int live = f0 + f < d.n ? min(S::half, d.tokens - t0) : 0;
            uint32_t v[2][16];
            tmem_load16(src, v[0]);
#pragma unroll
            for (int c = 0; c < S::half / 16; c++) {
                tmem_wait_load16(v[c & 1]);
                if (c + 1 < S::half / 16) {
                    tmem_load16(src + (c + 1) * 16, v[(c + 1) & 1]);
                } else {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) arrive_at(of_first(acc_empty + 8 * acc.slot));
                }
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    if (c * 16 + i < live) *y = from_f32<T>(__uint_as_float(v[c & 1][i]) + bias);
                    y += d.ys;
                }
            }
            acc.step();
        }
        tc_fence_before();
    }
    __syncthreads();
    tc_fence_after();
    // (nobody sets gave_up from here on)
    if (tid == 0 && rank) cg::this_cluster().map_shared_rank(issued, 0)[4] = gave_up;
    cluster_arrive();
    cluster_wait();
    if (rank == 0 && (gave_up || issued[4])) {        // what was issued ends before tensor memory and the blocks' memory are given up
        if (tid == 32) {
            pair_commit(1, drained);
            mbar_drain(drained, 0);
        }
        if (tid == 0) {
            // (a stage that only some of the four came to is arrived on for the others)
            int most = 0;
            for (int k = 0; k < 4; k++) most = max(most, issued[k]);
            for (int k = 0; k < 4; k++)
                for (int i = issued[k]; i < most; i++) mbar_arrive(full + 8 * (i % S::stages));
            drain_loads<S::stages>(full, most);
            atomicExch(d.status, 1);
        }
    }
    __syncthreads();
    cluster_arrive();                                 // the first block has no more use for the other's memory
    cluster_wait();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

// ------------------------------------------------------------------------------------------- host
int check_pack(const bcast_serve_pack4_args *a)
{
    if (!a) return BCAST_ERR_INVAL;
    if (a->dtype != BCAST_SERVE_BF16 && a->dtype != BCAST_SERVE_FP16 && a->dtype != BCAST_SERVE_FP32) return BCAST_ERR_INVAL;
    if (a->rows < 0 || a->rows > kMaxDim - 65536 || a->k < kBlock || a->k > 1 << 24 || a->k % kBlock) return BCAST_ERR_INVAL;
    if (round_up(a->rows, 128) * round_up(a->k, 128) > 1ll << 36) return BCAST_ERR_INVAL;
    if (a->rows == 0) return BCAST_OK;
    if (!stride_ok(a->values_stride, a->k, 8) || !stride_ok(a->codes_stride, a->k / 2, 16)) return BCAST_ERR_INVAL;
    int device = 0, rc;
    SERVE_TRY(cudaGetDevice(&device));
    if ((rc = check_array(a->values, 16, device)) || (rc = check_array(a->codes, 16, device)) || (rc = check_array(a->scales, 16, device))) return rc;
    return BCAST_OK;
}

// Rows of `k` numbers, scales in tiles of `tile` rows.
PackDev pack_dev(void *values, int64_t vs, uint8_t *codes, int64_t cs, uint8_t *scales, int64_t rows, int64_t k, int tile)
{
    PackDev d = {};
    d.values = values;
    d.codes = codes;
    d.scales = scales;
    d.vs = vs;
    d.cs = cs;
    d.rows = d.padded = (int32_t)rows;
    d.k = (int32_t)k;
    d.tiles_k = (int32_t)ceil_div(k, 4 * kBlock);
    d.eights = divisor((uint32_t)round_up(k / 8, 16));
    d.tile = divisor((uint32_t)tile);
    d.atoms = (int32_t)ceil_div(tile, 128);
    return d;
}
PackDev pack_dev(const bcast_serve_pack4_args &a) { return pack_dev(a.values, a.values_stride, a.codes, a.codes_stride, a.scales, a.rows, a.k, 128); }

template <typename F>
int over_rows(F kernel, PackDev d, cudaStream_t st)
{
    const int64_t threads = ceil_div(d.padded, kPackRows) * d.eights.of;
    d.threads = (uint32_t)threads;        // at most 2^31: the shapes' checks see to it
    return launch(kernel, dim3((unsigned)ceil_div(threads, kPackThreads)), dim3(kPackThreads), 0, st, true, 1, d);
}

// How a call is cut: tokens of a tile and parts of k.
struct Cut {
    int tile, split;
};

// Parts of k: the most, in powers of two, that make no more than `room` blocks, each of at least two stages.
int parts_of(int64_t blocks, int64_t room, int64_t k_blocks, int most)
{
    int s = 1;
    while (s < most && blocks * s * 2 <= room && k_blocks >= 4 * s) s *= 2;
    return s;
}

// Measured on one B200 (us, k = 4096, n = 4096 where nothing else is said), a tile of 128 tokens to a block / 224 to a pair:
// 333 tokens, 2080 -> 5003 11.5 / 10.1; 512 13.0 / 11.6; 1024 16.1 / 16.9; 1500 26.4 / 18.5; 200, n = 16384 16.4 / 13.6; 448, n =
// 16384 28.4 / 19.3.  So pairs from half of them on.  Fewer tokens than 129: blocks of a cluster share a tile's k, at most
// one block to an SM (twice as many: 64 tokens 9.5 instead of 7.7).
Cut cut_of(const bcast_serve_linear4_args &a)
{
    Cut c = {};
    const int64_t k_blocks = ceil_div(a.k, kDepth), f_tiles = ceil_div(a.n, kFeatures);
    c.tile = a.tokens <= 32 ? 32 : a.tokens <= 64 ? 64 : a.tokens <= 128 || ceil_div(a.tokens, kPairTokens) * f_tiles < kSms / 2 ? 128 : kPairTokens;
    c.split = c.tile > 128 ? 1 : parts_of(ceil_div(a.tokens, c.tile) * f_tiles, kSms, k_blocks, kMaxSplit);
    return c;
}

int check_shape(const bcast_serve_linear4_args &a)
{
    if (a.dtype != BCAST_SERVE_BF16 && a.dtype != BCAST_SERVE_FP16) return BCAST_ERR_INVAL;
    if (a.tokens < 0 || a.tokens > (1 << 21) || a.k < kBlock || a.k > (1 << 24) || a.k % kBlock || a.n < 1 || a.n > (1 << 24)) return BCAST_ERR_INVAL;
    if (a.tokens * round_up(a.k, 128) > 1ll << 36) return BCAST_ERR_INVAL;
    return BCAST_OK;
}

// x in the workspace, where it is packed by a kernel of its own.
int64_t x_codes_bytes(const bcast_serve_linear4_args &a) { return a.tokens <= kFusedTokens ? 0 : round_up(a.tokens * (a.k / 2), 256); }
int64_t x_scales_bytes(const bcast_serve_linear4_args &a, const Cut &c)
{
    return a.tokens <= kFusedTokens ? 0 : ceil_div(a.tokens, c.tile) * ceil_div(a.k, 4 * kBlock) * ceil_div(c.tile, 128) * kAtom;
}

template <typename T, int NT, bool FUSED>
int run_product(const bcast_serve_linear4_args &a, ProductDev d, const PackDev &p, const Cut &c, cudaStream_t st)
{
    using S = Tile<NT, FUSED>;
    d.f_tiles = (int32_t)ceil_div(a.n, kFeatures);
    d.t_tiles = (int32_t)ceil_div(a.tokens, NT);
    const int64_t tiles = (int64_t)d.f_tiles * d.t_tiles;
    // rows of codes as rows of 16-bit numbers, four codes each
    CUtensorMap mx, mw;
    int rc;
    if ((rc = tensor_map(&mw, CU_TENSOR_MAP_DATA_TYPE_UINT16, a.codes, {a.k / 4, a.n}, {a.codes_stride / 2}, {64, kFeatures}))) return rc;
    mx = mw;
    if (!FUSED && (rc = tensor_map(&mx, CU_TENSOR_MAP_DATA_TYPE_UINT16, p.codes, {a.k / 4, a.tokens}, {p.cs / 2}, {64, NT}))) return rc;
    if ((rc = allow_smem<serve_linear4_kernel<T, NT, FUSED>>(S::smem))) return rc;
    const int64_t blocks = tiles * c.split;
    if (blocks > kMaxDim) return BCAST_ERR_INVAL;
    return launch(serve_linear4_kernel<T, NT, FUSED>, dim3((unsigned)blocks), dim3(FUSED ? kFusedThreads : kProductThreads), S::smem, st, true, c.split,
                  mx, mw, d);
}

template <typename T>
int run_pairs(const bcast_serve_linear4_args &a, ProductDev d, const PackDev &p, cudaStream_t st)
{
    using S = PairTile;
    d.f_tiles = (int32_t)ceil_div(a.n, kFeatures);
    d.t_tiles = (int32_t)ceil_div(a.tokens, kPairTokens);
    CUtensorMap mx, mw, msx, msw;
    int rc;
    if ((rc = tensor_map(&mx, CU_TENSOR_MAP_DATA_TYPE_UINT16, p.codes, {a.k / 4, a.tokens}, {p.cs / 2}, {64, S::half}))) return rc;
    if ((rc = tensor_map(&mw, CU_TENSOR_MAP_DATA_TYPE_UINT16, a.codes, {a.k / 4, a.n}, {a.codes_stride / 2}, {64, kFeatures}))) return rc;
    if ((rc = flat_map(&msx, p.scales, 256, (int64_t)d.t_tiles * p.tiles_k, 256, 256, 2))) return rc;
    if ((rc = flat_map(&msw, a.scales, p.tiles_k * 128, d.f_tiles, p.tiles_k * 128, 256, 1))) return rc;
    if ((rc = allow_smem<serve_linear4_pair_kernel<T>>(S::smem))) return rc;
    const int64_t pairs = (int64_t)ceil_div(d.f_tiles, 2) * d.t_tiles;
    if (pairs > kMaxDim) return BCAST_ERR_INVAL;
    return launch(serve_linear4_pair_kernel<T>, dim3((unsigned)(2 * (pairs < kSms / 2 ? pairs : kSms / 2))), dim3(kPairThreads), S::smem, st, true, 1, mx,
                  mw, msx, msw, d);
}

template <typename T>
int run(const bcast_serve_linear4_args &a, const ProductDev &d, const PackDev &p, const Cut &c, cudaStream_t st)
{
    if (a.tokens <= kFusedTokens) return run_product<T, 32, true>(a, d, p, c, st);
    const int rc = over_rows(serve_pack4_kernel<T>, p, st);
    if (rc) return rc;
    switch (c.tile) {
    case 32: return run_product<T, 32, false>(a, d, p, c, st);
    case 64: return run_product<T, 64, false>(a, d, p, c, st);
    case 128: return run_product<T, 128, false>(a, d, p, c, st);
    default: return run_pairs<T>(a, d, p, st);
    }
}

}  // namespace
}  // namespace bcast_serve

using namespace bcast_serve;

extern "C" {

int bcast_serve_pack4(const bcast_serve_pack4_args *a, void *cuda_stream)
{
    int rc = check_pack(a);
    if (rc || a->rows == 0) return rc;
    PackDev d = pack_dev(*a);
    d.padded = (int32_t)round_up(a->rows, 128);
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    switch (a->dtype) {
    case BCAST_SERVE_BF16: return over_rows(serve_pack4_kernel<__nv_bfloat16>, d, st);
    case BCAST_SERVE_FP16: return over_rows(serve_pack4_kernel<__half>, d, st);
    default: return over_rows(serve_pack4_kernel<float>, d, st);
    }
}

int bcast_serve_unpack4(const bcast_serve_pack4_args *a, void *cuda_stream)
{
    int rc = check_pack(a);
    if (rc || a->rows == 0) return rc;
    const PackDev d = pack_dev(*a);
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    switch (a->dtype) {
    case BCAST_SERVE_BF16: return over_rows(serve_unpack4_kernel<__nv_bfloat16>, d, st);
    case BCAST_SERVE_FP16: return over_rows(serve_unpack4_kernel<__half>, d, st);
    default: return over_rows(serve_unpack4_kernel<float>, d, st);
    }
}

int64_t bcast_serve_linear4_workspace(const bcast_serve_linear4_args *a)
{
    if (!a || check_shape(*a)) return BCAST_ERR_INVAL;
    return BCAST_SERVE_STATUS_BYTES + x_codes_bytes(*a) + x_scales_bytes(*a, cut_of(*a));
}

int bcast_serve_linear4(const bcast_serve_linear4_args *a, void *cuda_stream)
{
    if (!a) return BCAST_ERR_INVAL;
    int rc = check_shape(*a);
    if (rc) return rc;
    if (a->tokens == 0) return BCAST_OK;
    if (!stride_ok(a->x_stride, a->k, 8) || !stride_ok(a->codes_stride, a->k / 2, 16) || !stride_ok(a->y_stride, a->n, 1)) return BCAST_ERR_INVAL;
    int device = 0;
    SERVE_TRY(cudaGetDevice(&device));
    if ((rc = check_array(a->x, 16, device)) || (rc = check_array(a->codes, 16, device)) || (rc = check_array(a->scales, 16, device)) ||
        (rc = check_array(a->y, 2, device)))
        return rc;
    if (a->bias && (rc = check_array(a->bias, 2, device))) return rc;
    if ((rc = check_workspace(a->workspace, a->workspace_bytes, bcast_serve_linear4_workspace(a), device))) return rc;

    const Cut c = cut_of(*a);
    // (what has no token is read too, as scales of columns that nobody keeps)
    uint8_t *codes = (uint8_t *)a->workspace + BCAST_SERVE_STATUS_BYTES;
    const PackDev p = pack_dev(const_cast<void *>(a->x), a->x_stride, codes, a->k / 2, codes + x_codes_bytes(*a), a->tokens, a->k, c.tile);
    ProductDev d = {};
    d.bias = a->bias;
    d.x = a->x;
    d.xs = a->x_stride;
    d.scales_w = a->scales;
    d.scales_x = p.scales;
    d.y = a->y;
    d.status = (int *)a->workspace;
    d.give_up = give_up_at_once();
    d.ys = a->y_stride;
    d.tiles_k = p.tiles_k;
    d.tokens = (int32_t)a->tokens;
    d.k = (int32_t)a->k;
    d.n = (int32_t)a->n;
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    return a->dtype == BCAST_SERVE_BF16 ? run<__nv_bfloat16>(*a, d, p, c, st) : run<__half>(*a, d, p, c, st);
}

}  // extern "C"
