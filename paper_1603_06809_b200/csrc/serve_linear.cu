// bcast_serve_linear: a projection that all tokens share, plus the low-rank adapter of each token's request.
//
//   y[t] = W x[t] + bias + B[a] u[t],   u[t] = scale[a] A[a] x[t],   a = adapter[t]
//
// Both products are the same matrix product over tiles of 128 features x NT tokens: rows of W (or of A[a]) are
// the first operand of tcgen05.mma, rows of x the second, both as they lie in memory (k contiguous).  With the
// features on the 128 lanes a decode step's few tokens are the instruction's N, which may be as small as 16.
//   low kernel   one item per tile of tokens, group of adapters among them (as many as have room on the 128
//                lanes) and part of k: sums in 32 bits, one array per part
//   main kernel  the product goes on past k: for every adapter among a tile's tokens, B[a] stands in the
//                place of W and u, zero for the tokens of other adapters, in the place of x.  The adapter's
//                part so costs R more columns of k and no pass over y of its own.  u goes through the tensor
//                cores as the sum of two numbers of the data type, so that 16 or more bits of it count.
// A block has one warp that loads tiles by TMA, one that issues the matrix instructions and four that fill
// in u and bring accumulators from tensor memory to y.
// What bounds it, and what it takes on one B200 (bf16, 4096 -> 4096; time on the device, in brackets that of a public
// call among others of its kind): 8192 tokens of 16 requests, 8 adapters of rank 64, 254 us, 1.12 PFLOP/s (290, the
// power cap) -- the product alone runs at 1.40 (a library's at 1.47), the rest is the low kernel, which is not
// overlapped, and its 6 more stages of k to a tile; 64 tokens with 32 adapters of rank 16, 19 us for 43 MB (20.5) --
// reading W takes until 10 us, then come u (1), eight stages of adapters (3) and the sum over the cluster (3); one
// token, 2048 -> 2048, 10 us: two launches' latency (11.6).
#include "serve_device.cuh"
#include "serve_internal.h"
#include "serve_tma.h"

#include <cooperative_groups.h>

namespace cg = cooperative_groups;

namespace bcast_serve {
namespace {

constexpr int kFeatures = 128;            // features per tile: the lanes of tensor memory
constexpr int kDepth = 64;                // values of k per stage: 128 bytes, one swizzled row
constexpr int kLinearThreads = 192;
constexpr int kMaxSplit = 8;              // blocks of a cluster that share one tile's k
constexpr int kMaxLowSplit = 16;

// Stages in flight.  Two blocks fit on an SM up to 128 tokens, so that the low and the main kernel, or one
// tile's end and the next one's beginning, overlap; the 256-token tile takes the SM for itself.
template <int NT> struct Tile {
    static constexpr int stage = kFeatures * 128 + NT * 128;
    static constexpr int stages = NT == 256 ? 4 : NT == 128 ? 3 : NT == 64 ? 4 : 5;
    static constexpr int accs = NT == 256 ? 2 : 1;                 // accumulators: a second one where blocks are persistent
    static constexpr int columns = accs * NT < 32 ? 32 : accs * NT;
    static constexpr size_t smem = (size_t)stage * stages + 1024;  // + alignment
    static_assert(NT * kFeatures * 4 <= stage * stages, "partial sums take the stages' place");
};

struct LinearDev {
    const void *bias;
    const int32_t *adapter;
    const float *scale;
    void *y;
    float *low;                           // [low_splits][T][R]: parts of A x
    int *status;
    int give_up;                          // 1: begin as if a wait had run out
    int64_t ys;
    int32_t tokens, k, n, adapters, rank, f_tiles, t_tiles, low_splits;
};

__device__ __forceinline__ bool known(int32_t a, const LinearDev &d) { return (uint32_t)a < (uint32_t)d.adapters; }

// Does `v` hold for all threads of the four warps after the first two?
__device__ __forceinline__ bool all_of_four(bool v)
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"((uint32_t)v) : "memory");
    return r;
}

// The adapters of a tile's tokens, each once, in the order of their first token.  For the four warps after
// the first two; `list` and `count` are complete for them on return.
template <int NT>
__device__ __forceinline__ void tile_adapters(const int32_t *ad, uint32_t *firsts, int32_t *list, int *count, const LinearDev &d)
{
    const int tid = threadIdx.x - 64, lane = tid % 32;
    bool first[(NT + 127) / 128];
#pragma unroll
    for (int i = 0; i * 128 < NT; i++) {
        const int t = tid + i * 128;
        const int32_t a = t < NT ? ad[t] : -1;
        // the first of its 32 tokens, and in none of the 32s before
        const uint32_t same = __match_any_sync(~0u, a);       // by every lane, whatever its token
        first[i] = known(a, d) && (same & ((1u << lane) - 1u)) == 0;
        const int4 *four = (const int4 *)ad;
        const int before = t < NT ? t / 32 * 8 : 0;
#pragma unroll 8
        for (int o = 0; o < before; o++) {
            const int4 v = four[o];
            if (v.x == a || v.y == a || v.z == a || v.w == a) first[i] = false;
        }
        const uint32_t bits = __ballot_sync(~0u, first[i]);
        if (lane == 0) firsts[t / 32] = bits;
    }
    asm volatile("bar.sync 1, 128;" ::: "memory");
    int total = 0;
#pragma unroll
    for (int i = 0; i * 128 < NT; i++) {
        const int t = tid + i * 128;
        int at = 0;
        for (int g = 0; g < t / 32; g++) at += __popc(firsts[g]);
        if (first[i]) list[at + __popc(firsts[t / 32] & ((1u << lane) - 1u))] = ad[t];
    }
#pragma unroll
    for (int g = 0; g < (NT + 31) / 32; g++) total += __popc(firsts[g]);
    if (tid == 0) *count = total;
    asm volatile("bar.sync 1, 128;" ::: "memory");
}

// How the adapters' part of k is laid out in a stage: rows of B[a] and of u are 32, 64 or 128 bytes, the next
// width above R.  Up to 64 bytes both numbers of u have room beside each other; otherwise a block of 64 columns
// comes by twice, once for each.
struct Adapters {
    int row, column_blocks, halves;
    __device__ __forceinline__ explicit Adapters(int rank)
    {
        row = rank <= 16 ? 32 : rank <= 32 ? 64 : 128;
        column_blocks = (rank + 63) / 64;
        halves = row < 128 ? 1 : 2;       // stages for one block of columns
    }
};

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

// Grid: LOW: x = parts of k x groups of a tile's adapters, y = tiles of tokens.  Main: one tile per cluster where
// a tile's k is split over a cluster, otherwise persistent blocks that take tiles in turn, features first.
template <typename T, int NT, bool LOW>
__global__ void __launch_bounds__(kLinearThreads, NT == 256 ? 1 : 2)
serve_linear_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w,
                    const __grid_constant__ CUtensorMap map_b, const __grid_constant__ LinearDev d)
{
    using S = Tile<NT>;
    extern __shared__ uint8_t raw_smem[];
    __shared__ __align__(8) uint64_t bars[4 * S::stages + 2 * S::accs + 3];
    __shared__ __align__(16) int32_t ad[NT];
    __shared__ int32_t list[NT];
    __shared__ uint32_t firsts[(NT + 127) / 128 * 4], tmem_at;
    __shared__ int count, gave_up;

    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const cg::cluster_group cluster = cg::this_cluster();
    const int split = LOW ? d.low_splits : (int)cluster.num_blocks(), part = LOW ? blockIdx.x % split : (int)cluster.block_rank();
    launch_next();

    uint8_t *smem = (uint8_t *)(((uintptr_t)raw_smem + 1023) & ~(uintptr_t)1023);
    const uint32_t stage0 = smem_u32(smem);
    const uint32_t full = smem_u32(bars), empty = full + 8 * S::stages, ready = empty + 8 * S::stages,
                   filled = ready + 8 * S::stages, acc_full = filled + 8 * S::stages, acc_empty = acc_full + 8 * S::accs,
                   meta = acc_empty + 8 * S::accs, taken = meta + 8, drained = taken + 8;

    // which tiles, and of k which stages
    const int k_blocks = (d.k + kDepth - 1) / kDepth;
    const int kb0 = (int)((int64_t)k_blocks * part / split), kb1 = (int)((int64_t)k_blocks * (part + 1) / split);
    const int first_tile = LOW ? blockIdx.y : blockIdx.x / split, tiles = LOW ? first_tile + 1 : d.f_tiles * d.t_tiles,
              tile_step = LOW ? 1 : gridDim.x / split;
    const Adapters form(d.rank);
    const int per = LOW ? kFeatures / d.rank : 1;     // adapters of a group

    if (warp >= 2) {
        if (LOW) {
            for (int t = tid - 64; t < NT; t += 128) {
                const int at = first_tile * NT + t;
                ad[t] = at < d.tokens ? d.adapter[at] : -1;
            }
            asm volatile("bar.sync 1, 128;" ::: "memory");
            tile_adapters<NT>(ad, firsts, list, &count, d);
        }
    } else if (warp == 1) {
        tmem_alloc(smem_u32(&tmem_at), S::columns);
    } else if (tid == 0) {
        gave_up = d.give_up;
        for (int i = 0; i < S::stages; i++) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
            mbar_init(ready + 8 * i, 1);
            mbar_init(filled + 8 * i, 128);
        }
        for (int i = 0; i < S::accs; i++) {
            mbar_init(acc_full + 8 * i, 1);
            mbar_init(acc_empty + 8 * i, 128);
        }
        mbar_init(meta, 128);
        if (S::accs > 1) mbar_init(taken, 1);
        mbar_init(drained, 1);
        mbar_init_fence();
        tma_prefetch(&map_x);
        tma_prefetch(&map_w);
        if (!LOW && d.adapters) tma_prefetch(&map_b);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_at;
    const int slot = blockIdx.x / split, mine = LOW ? min(per, count - slot * per) : 0;
    if (LOW && mine <= 0) {                           // fewer adapters among these tokens than there might be
        if (warp == 1) tmem_free(tmem, S::columns);
        return;
    }

    int issued = 0;                                   // loads, of the thread that issues them
    if (warp == 0) {
        if (lane == 0) {
            // ---- loads
            Ring<S::stages> ring;
            uint32_t meta_parity = 0;
            bool ok = true;
            for (int tile = first_tile; tile < tiles && ok; tile += tile_step) {
                const int f0 = LOW ? 0 : tile % d.f_tiles * kFeatures, t0 = (LOW ? tile : tile / d.f_tiles) * NT;
                for (int kb = kb0; kb < kb1; kb++) {
                    if (!LOW && kb == kb0 + S::stages && tile == first_tile && d.adapters) {
                        // while the first stages are on their way: the adapters' tiles too, as far as L2
                        if (!(ok = mbar_wait(meta, 0, &gave_up))) break;
                        for (int j = part; j < count; j += split)
                            for (int cb = 0; cb < form.column_blocks; cb++) tma_prefetch_box(&map_b, cb * kDepth, f0, list[j]);
                    }
                    if (!(ok = mbar_wait(empty + 8 * ring.slot, ring.parity ^ 1u, &gave_up))) break;
                    const uint32_t bar = full + 8 * ring.slot, at = stage0 + ring.slot * S::stage;
                    mbar_expect(bar, (LOW ? mine * d.rank : kFeatures) * 128 + NT * 128);
                    if (LOW) {
                        for (int j = 0; j < mine; j++) tma_load(at + j * d.rank * 128, &map_w, kb * kDepth, 0, list[slot * per + j], bar);
                    } else {
                        tma_load(at, &map_w, kb * kDepth, f0, bar);
                    }
                    tma_load(at + kFeatures * 128, &map_x, kb * kDepth, t0, bar);
                    issued++;
                    ring.step();
                }
                if (LOW || !d.adapters || !ok) continue;
                if (!(ok = mbar_wait(meta, meta_parity, &gave_up))) break;
                meta_parity ^= 1u;
                const int adapters = count;
                const int stages = (adapters - part + split - 1) / split * form.halves;
                for (int cb = 0; cb < form.column_blocks && ok; cb++)
                    for (int i = 0; i < stages; i++) {
                        if (!(ok = mbar_wait(empty + 8 * ring.slot, ring.parity ^ 1u, &gave_up))) break;
                        mbar_arrive(ready + 8 * ring.slot);
                        mbar_expect(full + 8 * ring.slot, kFeatures * form.row);
                        tma_load(stage0 + ring.slot * S::stage, &map_b, cb * kDepth, f0, list[part + i / form.halves * split], full + 8 * ring.slot);
                        issued++;
                        ring.step();
                    }
                if (S::accs > 1 && ok) mbar_arrive(taken);    // count and list are the next tile's now
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {
            // ---- matrix instructions
            constexpr uint32_t idesc = mma_desc<T>(kFeatures, NT);
            Ring<S::stages> ring;
            Ring<S::accs> acc;
            uint32_t meta_parity = 0, uses = 0;       // bit s: parity of the next use of stage s for an adapter
            bool ok = true;
            for (int tile = first_tile; tile < tiles && ok; tile += tile_step) {
                if (!(ok = mbar_wait(acc_empty + 8 * acc.slot, acc.parity ^ 1u, &gave_up))) break;
                tc_fence_after();
                const uint32_t out = tmem + acc.slot * NT;
                bool add = false;
                for (int kb = kb0; kb < kb1; kb++) {
                    if (!(ok = mbar_wait(full + 8 * ring.slot, ring.parity, &gave_up))) break;
                    tc_fence_after();
                    const uint32_t at = stage0 + ring.slot * S::stage;
                    const uint64_t a = smem_desc(at), b = smem_desc(at + kFeatures * 128);
#pragma unroll
                    for (int i = 0; i < kDepth / 16; i++) {
                        mma_ss(out, a + 2 * i, b + 2 * i, idesc, add);
                        add = true;
                    }
                    mma_commit(empty + 8 * ring.slot);
                    ring.step();
                }
                if (!LOW && d.adapters && ok) {
                    if (!(ok = mbar_wait(meta, meta_parity, &gave_up))) break;
                    meta_parity ^= 1u;
                    const int adapters = count;
                    const int stages = (adapters - part + split - 1) / split * form.halves;
                    for (int cb = 0; cb < form.column_blocks && ok; cb++)
                        for (int i = 0; i < stages; i++) {
                            if (!(ok = mbar_wait(full + 8 * ring.slot, ring.parity, &gave_up) &&
                                       mbar_wait(filled + 8 * ring.slot, uses >> ring.slot & 1u, &gave_up)))
                                break;
                            uses ^= 1u << ring.slot;
                            tc_fence_after();
                            const uint32_t at = stage0 + ring.slot * S::stage;
                            const uint64_t a = smem_desc(at, 16, form.row), b = smem_desc(at + kFeatures * 128, 16, form.row);
                            const int steps = (min(kDepth, d.rank - cb * kDepth) + 15) / 16;
                            for (int k = 0; k < steps; k++) {
                                mma_ss(out, a + 2 * k, b + 2 * k, idesc, true);
                                if (form.halves == 1) mma_ss(out, a + 2 * k, b + (NT * form.row >> 4) + 2 * k, idesc, true);
                            }
                            mma_commit(empty + 8 * ring.slot);
                            ring.step();
                        }
                }
                if (!ok) break;
                mma_commit(acc_full + 8 * acc.slot);
                acc.step();
            }
        }
        __syncwarp();
    } else {
        // ---- u, and the accumulators' way out.  A warp may touch the 32 lanes of its number modulo 4.
        const int quarter = warp % 4, f = quarter * 32 + lane, id = tid - 64;
        Ring<S::stages> ring;
        Ring<S::accs> acc;
        uint32_t uses = 0, taken_parity = 0;
        bool waited = false, alive = true;
        for (int tile = first_tile; tile < tiles; tile += tile_step) {
            const int f0 = LOW ? 0 : tile % d.f_tiles * kFeatures, t0 = (LOW ? tile : tile / d.f_tiles) * NT;
            bool ok = true;
            for (int kb = kb0; kb < kb1; kb++) ring.step();
            if (!LOW && d.adapters) {
                if (S::accs > 1 && tile != first_tile) {
                    // A tile without adapters sends nothing that says the loading thread has seen so; and all four warps
                    // go on to the barriers below, or none.
                    alive = alive && mbar_wait(taken, taken_parity, &gave_up);
                    taken_parity ^= 1u;
                    if (!(alive = all_of_four(alive))) break;
                }
                for (int t = id; t < NT; t += 128) ad[t] = t0 + t < d.tokens ? d.adapter[t0 + t] : -1;
                asm volatile("bar.sync 1, 128;" ::: "memory");
                tile_adapters<NT>(ad, firsts, list, &count, d);
                mbar_arrive(meta);
                if (!waited) wait_previous();         // the low kernel's u
                waited = true;
                // u of the tokens that have adapter j, zero for the others.  A thread holds its 16-byte chunks of all
                // tokens' u, both numbers, in registers: they are the same for every adapter that comes by.
                constexpr int held = NT < 16 ? 1 : NT * 8 / 128;
                const int chunks = form.row / 16, shift = 31 - __clz(chunks), stages = (count - part + split - 1) / split * form.halves;
                for (int cb = 0; cb < form.column_blocks && stages > 0 && ok; cb++) {
                    uint4 hi[held], lo[held];
#pragma unroll
                    for (int i = 0; i < held; i++) {
                        const int at = id + i * 128, t = at >> shift, col = cb * kDepth + (at & (chunks - 1)) * 8;
                        float u[8] = {};
                        if (t < NT && col < d.rank && known(ad[t], d)) {
                            const float4 *src = (const float4 *)(d.low + (int64_t)(t0 + t) * d.rank + col);
#pragma unroll 8
                            for (int k = 0; k < d.low_splits; k++, src += (int64_t)d.tokens * d.rank / 4) {
                                const float4 p = __ldcg(src), q = __ldcg(src + 1);
                                u[0] += p.x;
                                u[1] += p.y;
                                u[2] += p.z;
                                u[3] += p.w;
                                u[4] += q.x;
                                u[5] += q.y;
                                u[6] += q.z;
                                u[7] += q.w;
                            }
                            const float scale = d.scale[ad[t]];
#pragma unroll
                            for (int k = 0; k < 8; k++) u[k] *= scale;
                        }
                        __align__(16) T h[8], l[8];
#pragma unroll
                        for (int k = 0; k < 8; k++) {
                            h[k] = from_f32<T>(u[k]);
                            l[k] = from_f32<T>(u[k] - to_f32(h[k]));
                        }
                        hi[i] = *(const uint4 *)h;
                        lo[i] = *(const uint4 *)l;
                    }
                    for (int j = 0; j < stages; j++) {
                        if (!(ok = mbar_wait(ready + 8 * ring.slot, uses >> ring.slot & 1u, &gave_up))) break;
                        uses ^= 1u << ring.slot;
                        uint8_t *dst = smem + ring.slot * S::stage + kFeatures * 128;
                        const int32_t a = list[part + j / form.halves * split];
                        const bool first = form.halves == 1 || j % 2 == 0;
#pragma unroll
                        for (int i = 0; i < held; i++) {
                            const int at = id + i * 128, t = at >> shift;
                            if (t >= NT) continue;
                            const bool has = ad[t] == a;
                            const uint32_t to = swizzled(t, at & (chunks - 1), form.row);
                            const uint4 zero = make_uint4(0, 0, 0, 0);
                            *(uint4 *)(dst + to) = has ? (first ? hi[i] : lo[i]) : zero;
                            if (form.halves == 1) *(uint4 *)(dst + NT * form.row + to) = has ? lo[i] : zero;
                        }
                        fence_async_proxy();
                        mbar_arrive(filled + 8 * ring.slot);
                        ring.step();
                    }
                }
            }
            ok = ok && mbar_wait(acc_full + 8 * acc.slot, acc.parity, &gave_up);
            if (!__all_sync(~0u, ok)) {
                alive = false;                        // told to the other warps where they wait for this one
                if (S::accs > 1 && d.adapters) continue;
                break;
            }
            tc_fence_after();
            const uint32_t src = tmem + ((uint32_t)(quarter * 32) << 16) + acc.slot * NT;
            if (!LOW && split > 1) break;             // goes on below, with the other blocks of the cluster
            if (LOW) {
                // lane f is column f % R of the group's adapter f / R: kept for the tokens that have it
                const int32_t a = f < mine * d.rank ? list[slot * per + f / d.rank] : -1;
                float *low = d.low + ((int64_t)part * d.tokens + t0) * d.rank + f % d.rank;
#pragma unroll 1
                for (int c = 0; c < NT; c += 16) {
                    uint32_t v[16];
                    tmem_load16(src + c, v);
                    tmem_wait_load16(v);
#pragma unroll
                    for (int i = 0; i < 16; i++)
                        if (a >= 0 && ad[c + i] == a) low[(int64_t)(c + i) * d.rank] = __uint_as_float(v[i]);
                }
            } else {
                const float bias = d.bias && f0 + f < d.n ? to_f32(((const T *)d.bias)[f0 + f]) : 0.0f;
                T *y = (T *)d.y + (int64_t)t0 * d.ys + f0 + f;
                const int live = f0 + f < d.n ? min(NT, d.tokens - t0) : 0;
#pragma unroll 1
                for (int c = 0; c < NT; c += 16) {
                    uint32_t v[16];
                    tmem_load16(src + c, v);
                    tmem_wait_load16(v);
#pragma unroll
                    for (int i = 0; i < 16; i++)
                        if (c + i < live) y[(int64_t)(c + i) * d.ys] = from_f32<T>(__uint_as_float(v[i]) + bias);
                }
            }
            tc_fence_before();
            mbar_arrive(acc_empty + 8 * acc.slot);
            acc.step();
        }
        if (!waited && !LOW && d.adapters) wait_previous();
    }

    if (!LOW && split > 1) {
        // The blocks' sums are joined: each puts its own where its stages were, block r of the cluster adds up all
        // of them for its share of the tokens, always in the same order.  (Sending them to where they are added
        // instead of fetching them from there was slower: 4-byte remote stores, 32 us against 25 us for 333
        // tokens, 2056 -> 5003, when the rule still gave these two blocks to a tile; it gives one now, 27 us.)
        const int f0 = first_tile % d.f_tiles * kFeatures, t0 = first_tile / d.f_tiles * NT, share = NT / split;
        if (warp >= 2) {
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
        const bool whole = features % 4 == 0 && d.ys % 4 == 0 && ((uintptr_t)d.y & 7) == 0;
#pragma unroll 2
        for (int i = c0 * (kFeatures / 4) + tid; i < c1 * (kFeatures / 4); i += kLinearThreads) {
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

int check_shape(const bcast_serve_linear_args &a)
{
    if (a.dtype != BCAST_SERVE_BF16 && a.dtype != BCAST_SERVE_FP16) return BCAST_ERR_INVAL;
    if (a.tokens < 0 || a.tokens > (1 << 21) || a.k < 8 || a.k > (1 << 24) || a.k % 8 || a.n < 1 || a.n > (1 << 24))
        return BCAST_ERR_INVAL;
    if (a.num_adapters < 0 || a.num_adapters > 65536 || (a.num_adapters && (a.rank < 8 || a.rank > 128 || a.rank % 8)))
        return BCAST_ERR_INVAL;
    return BCAST_OK;
}

// How a call is cut.  Measured on one B200 (us, inputs not in L2), k = 4096, n = 4096 where nothing else is said:
//   main kernel, tokens of a tile x parts of k:  64 tokens: 64 x 4 20.1, 64 x 2 23.6, 32 x 2 20.3, 128 x 4 24.3;
//     128 tokens: 64 x 2 25.4, 64 x 4 25.8, 128 x 4 30.2;  512: 128 x 2 35, 128 x 1 37, 64 x 1 36, 256 x 2 76;
//     1024: 128 47, 64 58, 256 81;  2048: 128 88, 256 105;  8192: 256 260, 128 289.  So no more blocks than SMs
//     (twice as many: 2 us ahead at 512 tokens, level at 128),
//     and the widest tile, which reads W least often, once there are three rounds of it.
//   low kernel, parts of k (more parts end sooner, but the main kernel adds them up):  64 tokens: 16 parts 21.1, 8 21.9,
//     4 24.6;  512: 4 parts 37, 8 44, 2 40, 1 49;  1024: 2 parts 41, 4 47, 1 49.  So at most one for every
//     second SM, counting two groups of adapters to a tile.
struct Cut {
    int low_tile, low_splits, tile, split;    // tokens of a tile and parts of k, of the low and of the main kernel
    int64_t groups;                           // of adapters, at most, to a tile of the low kernel
};

// Parts of k: the most, in powers of two, that make no more than `room` blocks, each of at least four stages.
int parts_of(int64_t blocks, int64_t room, int64_t k_blocks, int most)
{
    int s = 1;
    while (s < most && blocks * s * 2 <= room && k_blocks >= 8 * s) s *= 2;
    return s;
}

Cut cut_of(const bcast_serve_linear_args &a)
{
    Cut c = {};
    const int64_t k_blocks = ceil_div(a.k, kDepth), f_tiles = ceil_div(a.n, kFeatures);
    const int small = a.tokens <= 16 ? 16 : a.tokens <= 32 ? 32 : 64;
    if (a.num_adapters) {
        c.low_tile = small;
        c.groups = ceil_div(a.num_adapters < c.low_tile ? a.num_adapters : c.low_tile, kFeatures / a.rank);
        c.low_splits = parts_of(ceil_div(a.tokens, c.low_tile) * (c.groups < 2 ? 1 : 2), kSms / 2, k_blocks, kMaxLowSplit);
    }
    c.tile = a.tokens <= 128 ? small : ceil_div(a.tokens, 256) * f_tiles < 3 * kSms ? 128 : 256;
    c.split = parts_of(ceil_div(a.tokens, c.tile) * f_tiles, kSms, k_blocks, kMaxSplit);
    return c;
}

template <typename T> constexpr CUtensorMapDataType kMapType =
    std::is_same_v<T, __nv_bfloat16> ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;

template <typename T, int NT>
int run_low(const bcast_serve_linear_args &a, LinearDev d, const Cut &c, cudaStream_t st)
{
    using S = Tile<NT>;
    d.t_tiles = (int32_t)ceil_div(a.tokens, NT);
    CUtensorMap mx, ma;
    int rc;
    if ((rc = tensor_map(&mx, kMapType<T>, a.x, {a.k, a.tokens}, {a.x_stride}, {kDepth, NT}))) return rc;
    if ((rc = tensor_map(&ma, kMapType<T>, a.lora_a, {a.k, a.rank, a.num_adapters}, {a.lora_a_stride[1], a.lora_a_stride[0]},
                         {kDepth, a.rank, 1})))
        return rc;
    if ((rc = allow_smem<serve_linear_kernel<T, NT, true>>(S::smem))) return rc;
    return launch(serve_linear_kernel<T, NT, true>, dim3((unsigned)(c.groups * c.low_splits), d.t_tiles), dim3(kLinearThreads), S::smem,
                  st, false, 1, mx, ma, ma, d);
}

template <typename T, int NT>
int run_main(const bcast_serve_linear_args &a, LinearDev d, const Cut &c, cudaStream_t st)
{
    using S = Tile<NT>;
    d.f_tiles = (int32_t)ceil_div(a.n, kFeatures);
    d.t_tiles = (int32_t)ceil_div(a.tokens, NT);
    const int64_t tiles = (int64_t)d.f_tiles * d.t_tiles;
    CUtensorMap mx, mw, mb;
    int rc;
    if ((rc = tensor_map(&mx, kMapType<T>, a.x, {a.k, a.tokens}, {a.x_stride}, {kDepth, NT}))) return rc;
    if ((rc = tensor_map(&mw, kMapType<T>, a.weight, {a.k, a.n}, {a.weight_stride}, {kDepth, kFeatures}))) return rc;
    mb = mw;
    const int columns = a.rank <= 16 ? 16 : a.rank <= 32 ? 32 : 64;   // as in Adapters
    if (d.adapters && (rc = tensor_map(&mb, kMapType<T>, a.lora_b, {a.rank, a.n, a.num_adapters}, {a.lora_b_stride[1], a.lora_b_stride[0]},
                                       {columns, kFeatures, 1})))
        return rc;
    if ((rc = allow_smem<serve_linear_kernel<T, NT, false>>(S::smem))) return rc;
    const int64_t blocks = c.split == 1 && S::accs > 1 && tiles > kSms ? kSms : tiles * c.split;
    return launch(serve_linear_kernel<T, NT, false>, dim3((unsigned)blocks), dim3(kLinearThreads), S::smem, st, d.adapters > 0, c.split, mx,
                  mw, mb, d);
}

template <typename T>
int run_type(const bcast_serve_linear_args &a, const LinearDev &d, const Cut &c, cudaStream_t st)
{
    int rc = BCAST_OK;
    if (d.adapters) {
        switch (c.low_tile) {
        case 16: rc = run_low<T, 16>(a, d, c, st); break;
        case 32: rc = run_low<T, 32>(a, d, c, st); break;
        default: rc = run_low<T, 64>(a, d, c, st);
        }
        if (rc) return rc;
    }
    switch (c.tile) {
    case 16: return run_main<T, 16>(a, d, c, st);
    case 32: return run_main<T, 32>(a, d, c, st);
    case 64: return run_main<T, 64>(a, d, c, st);
    case 128: return run_main<T, 128>(a, d, c, st);
    default: return run_main<T, 256>(a, d, c, st);
    }
}

}  // namespace
}  // namespace bcast_serve

using namespace bcast_serve;

extern "C" {

int64_t bcast_serve_linear_workspace(const bcast_serve_linear_args *a)
{
    if (!a || check_shape(*a)) return BCAST_ERR_INVAL;
    return BCAST_SERVE_STATUS_BYTES + (a->num_adapters ? (int64_t)cut_of(*a).low_splits * a->tokens * a->rank * 4 : 0);
}

int bcast_serve_linear(const bcast_serve_linear_args *a, void *cuda_stream)
{
    if (!a) return BCAST_ERR_INVAL;
    int rc = check_shape(*a);
    if (rc) return rc;
    if (a->tokens == 0) return BCAST_OK;
    if (!stride_ok(a->x_stride, a->k, 8) || !stride_ok(a->weight_stride, a->k, 8) || !stride_ok(a->y_stride, a->n, 1))
        return BCAST_ERR_INVAL;
    if (a->num_adapters &&
        (!stride_ok(a->lora_a_stride[1], a->k, 8) || !stride_ok(a->lora_a_stride[0], a->lora_a_stride[1] * (a->rank - 1) + a->k, 8) ||
         !stride_ok(a->lora_b_stride[1], a->rank, 8) || !stride_ok(a->lora_b_stride[0], a->lora_b_stride[1] * (a->n - 1) + a->rank, 8)))
        return BCAST_ERR_INVAL;
    int device = 0;
    SERVE_TRY(cudaGetDevice(&device));
    if ((rc = check_array(a->x, 16, device)) || (rc = check_array(a->weight, 16, device)) || (rc = check_array(a->y, 2, device)))
        return rc;
    if (a->bias && (rc = check_array(a->bias, 2, device))) return rc;
    if (a->num_adapters && ((rc = check_array(a->lora_a, 16, device)) || (rc = check_array(a->lora_b, 16, device)) ||
                            (rc = check_array(a->adapter, 4, device)) || (rc = check_array(a->scale, 4, device))))
        return rc;
    if ((rc = check_workspace(a->workspace, a->workspace_bytes, bcast_serve_linear_workspace(a), device))) return rc;

    LinearDev d = {};
    d.bias = a->bias;
    d.adapter = a->adapter;
    d.scale = a->scale;
    d.y = a->y;
    d.low = (float *)((char *)a->workspace + BCAST_SERVE_STATUS_BYTES);
    d.status = (int *)a->workspace;
    d.give_up = give_up_at_once();
    d.ys = a->y_stride;
    d.tokens = (int32_t)a->tokens;
    d.k = (int32_t)a->k;
    d.n = (int32_t)a->n;
    d.adapters = a->num_adapters;
    d.rank = a->num_adapters ? a->rank : 0;
    const Cut c = cut_of(*a);
    d.low_splits = c.low_splits;
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    return a->dtype == BCAST_SERVE_BF16 ? run_type<__nv_bfloat16>(*a, d, c, st) : run_type<__half>(*a, d, c, st);
}

}  // extern "C"
