// bcast_serve_linear: a projection that all tokens share, plus the low-rank adapter of each token's request.
//
//   y[t] = W x[t] + bias + B[a] u[t],   u[t] = scale[a] A[a] x[t],   a = adapter[t]
//
// Both products are the same matrix product over tiles of 128 features x NT tokens: rows of W (or of A[a]) are
// the first operand of tcgen05.mma, rows of x the second, both as they lie in memory (k contiguous).  With the
// features on the 128 lanes a decode step's few tokens are the instruction's N, which may be as small as 16.
//   low kernel   one item per tile of tokens and adapter among them: u, kept as the sum of two numbers of
//                the data type, so that 16 or more bits of it pass through the tensor cores
//   main kernel  the product goes on past k: for every adapter among a tile's tokens, B[a] stands in the
//                place of W and u, zero for the tokens of other adapters, in the place of x.  The adapter's
//                part so costs R more columns of k and no pass over y of its own.
// A block has one warp that loads tiles by TMA, one that issues the matrix instructions and four that fill
// in u and bring accumulators from tensor memory to y.
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
    void *low[2];                         // [T][R]: u rounded to the type, and what that left
    int *status;
    int64_t ys;
    int32_t tokens, k, n, adapters, rank, f_tiles, t_tiles;
};

__device__ __forceinline__ bool known(int32_t a, const LinearDev &d) { return (uint32_t)a < (uint32_t)d.adapters; }

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
        first[i] = t < NT && known(ad[t < NT ? t : 0], d);
        if (first[i])
            for (int o = 0; o < t; o++)
                if (ad[o] == ad[t]) first[i] = false;
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

// Grid: LOW: x = blocks of a cluster x adapters of a tile, y = tiles of tokens.  Main: one tile per cluster where
// a tile's k is split over a cluster, otherwise persistent blocks that take tiles in turn, features first.
template <typename T, int NT, bool LOW>
__global__ void __launch_bounds__(kLinearThreads, NT == 256 ? 1 : 2)
serve_linear_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w,
                    const __grid_constant__ CUtensorMap map_b, const __grid_constant__ LinearDev d)
{
    using S = Tile<NT>;
    extern __shared__ uint8_t raw_smem[];
    __shared__ __align__(8) uint64_t bars[4 * S::stages + 2 * S::accs + 2];
    __shared__ __align__(16) int32_t ad[NT];
    __shared__ int32_t list[NT];
    __shared__ uint32_t firsts[(NT + 127) / 128 * 4], tmem_at;
    __shared__ int count, gave_up;

    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const cg::cluster_group cluster = cg::this_cluster();
    const int split = (int)cluster.num_blocks(), part = (int)cluster.block_rank();
    launch_next();

    uint8_t *smem = (uint8_t *)(((uintptr_t)raw_smem + 1023) & ~(uintptr_t)1023);
    const uint32_t stage0 = smem_u32(smem);
    const uint32_t full = smem_u32(bars), empty = full + 8 * S::stages, ready = empty + 8 * S::stages,
                   filled = ready + 8 * S::stages, acc_full = filled + 8 * S::stages, acc_empty = acc_full + 8 * S::accs,
                   meta = acc_empty + 8 * S::accs, drained = meta + 8;

    // which tiles, and of k which stages
    const int k_blocks = (d.k + kDepth - 1) / kDepth;
    const int kb0 = (int)((int64_t)k_blocks * part / split), kb1 = (int)((int64_t)k_blocks * (part + 1) / split);
    const int first_tile = LOW ? blockIdx.y : blockIdx.x / split, tiles = LOW ? first_tile + 1 : d.f_tiles * d.t_tiles,
              tile_step = LOW ? 1 : gridDim.x / split;
    const int r_blocks = (d.rank + kDepth - 1) / kDepth;

    if (warp >= 2) {
        if (LOW) {
            for (int t = tid - 64; t < NT; t += 128) {
                const int at = first_tile * NT + t;
                ad[t] = at < d.tokens ? d.adapter[at] : -1;
            }
            asm volatile("bar.sync 1, 128;" ::: "memory");
            tile_adapters<NT>(ad, firsts, list, &count, d);
        }
    } else if (tid == 0) {
        gave_up = 0;
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
        mbar_init(drained, 1);
        mbar_init_fence();
        tma_prefetch(&map_x);
        tma_prefetch(&map_w);
        if (!LOW && d.adapters) tma_prefetch(&map_b);
    }
    __syncthreads();
    const int slot = blockIdx.x / split;
    if (LOW && slot >= count) return;                 // the whole cluster: it sees the same tile
    const int32_t mine = LOW ? list[slot] : -1;
    if (warp == 1) tmem_alloc(smem_u32(&tmem_at), S::columns);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_at;

    if (warp == 0) {
        if (lane == 0) {
            // ---- loads
            Ring<S::stages> ring;
            uint32_t meta_parity = 0;
            int issued = 0;
            bool ok = true;
            for (int tile = first_tile; tile < tiles && ok; tile += tile_step) {
                const int f0 = LOW ? 0 : tile % d.f_tiles * kFeatures, t0 = (LOW ? tile : tile / d.f_tiles) * NT;
                for (int kb = kb0; kb < kb1; kb++) {
                    if (!(ok = mbar_wait(empty + 8 * ring.slot, ring.parity ^ 1u, &gave_up))) break;
                    const uint32_t bar = full + 8 * ring.slot, at = stage0 + ring.slot * S::stage;
                    mbar_expect(bar, (LOW ? (uint32_t)d.rank : (uint32_t)kFeatures) * 128 + NT * 128);
                    if (LOW) tma_load(at, &map_w, kb * kDepth, 0, mine, bar);
                    else tma_load(at, &map_w, kb * kDepth, f0, bar);
                    tma_load(at + kFeatures * 128, &map_x, kb * kDepth, t0, bar);
                    issued++;
                    ring.step();
                }
                if (LOW || !d.adapters || !ok) continue;
                if (!(ok = mbar_wait(meta, meta_parity, &gave_up))) break;
                meta_parity ^= 1u;
                const int adapters = count;
                for (int j = part; j < adapters && ok; j += split)
                    for (int rb = 0; rb < 2 * r_blocks; rb++) {
                        if (!(ok = mbar_wait(empty + 8 * ring.slot, ring.parity ^ 1u, &gave_up))) break;
                        mbar_arrive(ready + 8 * ring.slot);
                        mbar_expect(full + 8 * ring.slot, kFeatures * 128);
                        tma_load(stage0 + ring.slot * S::stage, &map_b, rb / 2 * kDepth, f0, list[j], full + 8 * ring.slot);
                        issued++;
                        ring.step();
                    }
            }
            if (gave_up) {                            // loads still under way end before the block does
                Ring<S::stages> r;
                for (int i = 0; i < issued; i++) {
                    if (i + S::stages >= issued) mbar_drain(full + 8 * r.slot, r.parity);
                    r.step();
                }
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
                    for (int j = part; j < adapters && ok; j += split)
                        for (int rb = 0; rb < 2 * r_blocks; rb++) {
                            if (!(ok = mbar_wait(full + 8 * ring.slot, ring.parity, &gave_up) &&
                                       mbar_wait(filled + 8 * ring.slot, uses >> ring.slot & 1u, &gave_up)))
                                break;
                            uses ^= 1u << ring.slot;
                            tc_fence_after();
                            const uint32_t at = stage0 + ring.slot * S::stage;
                            const uint64_t a = smem_desc(at), b = smem_desc(at + kFeatures * 128);
                            const int steps = (min(kDepth, d.rank - rb / 2 * kDepth) + 15) / 16;
                            for (int i = 0; i < steps; i++) mma_ss(out, a + 2 * i, b + 2 * i, idesc, true);
                            mma_commit(empty + 8 * ring.slot);
                            ring.step();
                        }
                }
                if (!ok) break;
                mma_commit(acc_full + 8 * acc.slot);
                acc.step();
            }
            if (gave_up) {
                mma_commit(drained);                  // what was issued ends before its operands' memory is given up
                mbar_drain(drained, 0);
            }
        }
        __syncwarp();
    } else {
        // ---- u, and the accumulators' way out.  A warp may touch the 32 lanes of its number modulo 4.
        const int quarter = warp % 4, f = quarter * 32 + lane, id = tid - 64;
        Ring<S::stages> ring;
        Ring<S::accs> acc;
        uint32_t uses = 0;
        bool waited = false;
        for (int tile = first_tile; tile < tiles; tile += tile_step) {
            const int f0 = LOW ? 0 : tile % d.f_tiles * kFeatures, t0 = (LOW ? tile : tile / d.f_tiles) * NT;
            bool ok = true;
            for (int kb = kb0; kb < kb1; kb++) ring.step();
            if (!LOW && d.adapters) {
                for (int t = id; t < NT; t += 128) ad[t] = t0 + t < d.tokens ? d.adapter[t0 + t] : -1;
                asm volatile("bar.sync 1, 128;" ::: "memory");
                tile_adapters<NT>(ad, firsts, list, &count, d);
                mbar_arrive(meta);
                if (!waited) wait_previous();         // the low kernel's u
                waited = true;
                const int adapters = count;
                for (int j = part; j < adapters && ok; j += split)
                    for (int rb = 0; rb < 2 * r_blocks; rb++) {
                        if (!(ok = mbar_wait(ready + 8 * ring.slot, uses >> ring.slot & 1u, &gave_up))) break;
                        uses ^= 1u << ring.slot;
                        uint8_t *dst = smem + ring.slot * S::stage + kFeatures * 128;
                        const T *low = (const T *)d.low[rb & 1] + rb / 2 * kDepth;
                        const int chunks = min(kDepth, d.rank - rb / 2 * kDepth) / 8;
                        for (int i = id; i < NT * 8; i += 128) {
                            const int t = i / 8, c = i % 8;
                            uint4 v = make_uint4(0, 0, 0, 0);
                            if (c < chunks && ad[t] == list[j]) v = __ldcg((const uint4 *)(low + (int64_t)(t0 + t) * d.rank) + c);
                            *(uint4 *)(dst + t * 128 + ((c ^ (t & 7)) << 4)) = v;
                        }
                        fence_async_proxy();
                        mbar_arrive(filled + 8 * ring.slot);
                        ring.step();
                    }
            }
            ok = ok && mbar_wait(acc_full + 8 * acc.slot, acc.parity, &gave_up);
            if (!__all_sync(~0u, ok)) break;
            tc_fence_after();
            const uint32_t src = tmem + ((uint32_t)(quarter * 32) << 16) + acc.slot * NT;
            const bool write = !LOW && split == 1;
            const float bias = write && d.bias && f0 + f < d.n ? to_f32(((const T *)d.bias)[f0 + f]) : 0.0f;
            T *y = (T *)d.y + (int64_t)t0 * d.ys + f0 + f;
            const int live = f0 + f < d.n ? min(NT, d.tokens - t0) : 0;
#pragma unroll 1
            for (int c = 0; c < NT; c += 16) {
                uint32_t v[16];
                tmem_load16(src + c, v);
                tmem_wait_load16(v);
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    if (write) {
                        if (c + i < live) y[(int64_t)(c + i) * d.ys] = from_f32<T>(__uint_as_float(v[i]) + bias);
                    } else {
                        ((float *)smem)[(c + i) * kFeatures + f] = __uint_as_float(v[i]);
                    }
                }
            }
            tc_fence_before();
            mbar_arrive(acc_empty + 8 * acc.slot);
            acc.step();
        }
        if (!waited && !LOW && d.adapters) wait_previous();
    }
    __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_free(tmem, S::columns);
    if (tid == 0 && gave_up) atomicExch(d.status, 1);

    if (LOW || split > 1) {
        // the blocks' partial sums joined, each block for its share of the tokens, always in the same order
        cluster.sync();
        const int f0 = LOW ? 0 : first_tile % d.f_tiles * kFeatures, t0 = (LOW ? first_tile : first_tile / d.f_tiles) * NT;
        const int c0 = NT * part / split, c1 = min(NT * (part + 1) / split, d.tokens - t0);
        const int features = LOW ? d.rank : min(kFeatures, d.n - f0);
        const float scale = LOW ? d.scale[mine] : 1.0f;
        for (int i = c0 * kFeatures + tid; i < c1 * kFeatures; i += kLinearThreads) {
            const int f = i % kFeatures, c = i / kFeatures;
            if (f >= features || (LOW && ad[c] != mine)) continue;
            float v = 0.0f;
            for (int s = 0; s < split; s++) v += cluster.map_shared_rank((float *)smem, s)[i];
            if (LOW) {
                v *= scale;
                const T hi = from_f32<T>(v);
                const int64_t at = (int64_t)(t0 + c) * d.rank + f;
                ((T *)d.low[0])[at] = hi;
                ((T *)d.low[1])[at] = from_f32<T>(v - to_f32(hi));
            } else {
                if (d.bias) v += to_f32(((const T *)d.bias)[f0 + f]);
                ((T *)d.y)[(int64_t)(t0 + c) * d.ys + f0 + f] = from_f32<T>(v);
            }
        }
        cluster.sync();
    }
}

int check_shape(const bcast_serve_linear_args &a)
{
    if (a.dtype != BCAST_SERVE_BF16 && a.dtype != BCAST_SERVE_FP16) return BCAST_ERR_INVAL;
    if (a.tokens < 0 || a.tokens > (1 << 22) || a.k < 8 || a.k > (1 << 24) || a.k % 8 || a.n < 1 || a.n > (1 << 24))
        return BCAST_ERR_INVAL;
    if (a.num_adapters < 0 || a.num_adapters > 65536 || (a.num_adapters && (a.rank < 8 || a.rank > 128 || a.rank % 8)))
        return BCAST_ERR_INVAL;
    return BCAST_OK;
}

// Bytes of one of the two arrays of u.
int64_t low_bytes(const bcast_serve_linear_args &a)
{
    return a.num_adapters ? round_up(a.tokens * a.rank * 2, 256) : 0;
}

int token_tile(int64_t tokens) { return tokens <= 16 ? 16 : tokens <= 32 ? 32 : tokens <= 64 ? 64 : tokens <= 128 ? 128 : 256; }

// Blocks that share a tile's k: as many as it takes to give every SM one, each with at least four stages.
int split_of(int64_t tiles, int64_t k_blocks)
{
    int s = 1;
    while (s < kMaxSplit && tiles * s * 2 <= kSms * 2 && k_blocks >= 8 * s) s *= 2;
    return s;
}

template <typename T, int NT>
int run(const bcast_serve_linear_args &a, LinearDev d, cudaStream_t st)
{
    using S = Tile<NT>;
    const auto type = std::is_same_v<T, __nv_bfloat16> ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    d.f_tiles = (int32_t)ceil_div(a.n, kFeatures);
    d.t_tiles = (int32_t)ceil_div(a.tokens, NT);
    const int64_t k_blocks = ceil_div(a.k, kDepth), tiles = (int64_t)d.f_tiles * d.t_tiles;
    CUtensorMap mx, mw, ma, mb;
    int rc;
    if ((rc = tensor_map(&mx, type, a.x, {a.k, a.tokens}, {a.x_stride}, {kDepth, NT}))) return rc;
    if ((rc = tensor_map(&mw, type, a.weight, {a.k, a.n}, {a.weight_stride}, {kDepth, kFeatures}))) return rc;
    ma = mb = mw;
    const auto low = serve_linear_kernel<T, NT, true>, main = serve_linear_kernel<T, NT, false>;
    if (d.adapters) {
        if ((rc = tensor_map(&ma, type, a.lora_a, {a.k, a.rank, a.num_adapters}, {a.lora_a_stride[1], a.lora_a_stride[0]}, {kDepth, a.rank, 1})))
            return rc;
        if ((rc = tensor_map(&mb, type, a.lora_b, {a.rank, a.n, a.num_adapters}, {a.lora_b_stride[1], a.lora_b_stride[0]},
                             {kDepth, kFeatures, 1})))
            return rc;
        const int64_t slots = a.num_adapters < NT ? a.num_adapters : NT;
        const int split = split_of(slots * d.t_tiles, k_blocks);
        if ((rc = allow_smem<serve_linear_kernel<T, NT, true>>(S::smem))) return rc;
        if ((rc = launch(low, dim3((unsigned)(slots * split), d.t_tiles), dim3(kLinearThreads), S::smem, st, false, split, mx, ma, ma, d)))
            return rc;
    }
    if ((rc = allow_smem<serve_linear_kernel<T, NT, false>>(S::smem))) return rc;
    const int split = S::accs > 1 ? 1 : split_of(tiles, k_blocks);
    const int64_t blocks = S::accs > 1 ? (tiles < kSms ? tiles : kSms) : tiles * split;
    return launch(main, dim3((unsigned)blocks), dim3(kLinearThreads), S::smem, st, d.adapters > 0, split, mx, mw, mb, d);
}

template <typename T>
int run_type(const bcast_serve_linear_args &a, const LinearDev &d, cudaStream_t st)
{
    switch (token_tile(a.tokens)) {
    case 16: return run<T, 16>(a, d, st);
    case 32: return run<T, 32>(a, d, st);
    case 64: return run<T, 64>(a, d, st);
    case 128: return run<T, 128>(a, d, st);
    default: return run<T, 256>(a, d, st);
    }
}

}  // namespace
}  // namespace bcast_serve

using namespace bcast_serve;

extern "C" {

int64_t bcast_serve_linear_workspace(const bcast_serve_linear_args *a)
{
    if (!a || check_shape(*a)) return BCAST_ERR_INVAL;
    return BCAST_SERVE_STATUS_BYTES + 2 * low_bytes(*a);
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
    Device dev;
    if ((rc = current_device(&dev))) return rc;
    if ((rc = check_array(a->x, 16, dev.id)) || (rc = check_array(a->weight, 16, dev.id)) || (rc = check_array(a->y, 2, dev.id)))
        return rc;
    if (a->bias && (rc = check_array(a->bias, 2, dev.id))) return rc;
    if (a->num_adapters && ((rc = check_array(a->lora_a, 16, dev.id)) || (rc = check_array(a->lora_b, 16, dev.id)) ||
                            (rc = check_array(a->adapter, 4, dev.id)) || (rc = check_array(a->scale, 4, dev.id))))
        return rc;
    if ((rc = check_workspace(a->workspace, a->workspace_bytes, bcast_serve_linear_workspace(a), dev.id))) return rc;

    LinearDev d = {};
    d.bias = a->bias;
    d.adapter = a->adapter;
    d.scale = a->scale;
    d.y = a->y;
    d.low[0] = (char *)a->workspace + BCAST_SERVE_STATUS_BYTES;
    d.low[1] = (char *)d.low[0] + low_bytes(*a);
    d.status = (int *)a->workspace;
    d.ys = a->y_stride;
    d.tokens = (int32_t)a->tokens;
    d.k = (int32_t)a->k;
    d.n = (int32_t)a->n;
    d.adapters = a->num_adapters;
    d.rank = a->num_adapters ? a->rank : 0;
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    return a->dtype == BCAST_SERVE_BF16 ? run_type<__nv_bfloat16>(*a, d, st) : run_type<__half>(*a, d, st);
}

}  // extern "C"
