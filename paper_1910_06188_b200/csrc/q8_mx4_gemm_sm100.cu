// Product of an MXFP4 activation with MXFP4 weights on Blackwell tensor cores (sm_100a), plain or grouped by expert:
//
//   Y[t, n] = act(sum_k x[t, k] w[e][n, k] + b[e][n])     for the slots t of expert e
//
// The weights are the A operand (accumulator rows = TMEM lanes = output features), the tokens the B operand (accumulator columns).
// So a tile is as narrow as its tokens are few, an expert with three rows costs 16 columns, a lane of the epilogue has one bias
// value for the whole tile, and what a warp stores of one column is 32 neighbouring features of a token.
//
//   warp 0      producer of the weights: a tile of 128 rows x 256 codes with its scales is one contiguous copy
//   warp 2      producer of the tokens: rows of such tiles, and their scales
//   warp 1      MMA issuer: copies the scales to TMEM (tcgen05.cp), issues tcgen05.mma kind::mxf4 (64 codes a time, one scale per
//               32), fp32 accumulators in TMEM, double buffered
//   warps 3..   epilogue: tcgen05.ld, bias, GELU, conversion, store
//
// Few tokens (X not void): no quantise pass; the epilogue warps first quantise the tokens of the tile into the operand stages themselves,
// while the weights, which are what such a product waits for, are on their way.
//
// A plain product with few tiles and a long K: the K axis of a tile is split over a cluster of CTAs, whose sums are joined through distributed
// shared memory, each CTA finishing a share of the tokens (join()).
//
// CTAS = 2 (cta_group::2): a pair of SMs shares a tile of 256 features; each loads its own 128 rows of weights, half of the tokens and the
// scales of all of them.  A plain product is the grouped one with a single expert.  Every wait on an mbarrier is bounded: after
// ~2 s the CTA raises Q8_ERR_TIMEOUT in the status word, all roles leave their loops, copies and products in flight are waited for
// (bounded), TMEM is freed.  No copy is multicast.  Without a limit are the waits for the kernel before, for the CTAs of a cluster, for the CTA's own warps
// and for TMEM; what ends them is resident (a cluster starts as a whole) or complete before this kernel's last CTA, and no other CTA of the library that holds TMEM
// fits beside this one's shared memory.
//
// Bounds: many tokens the tensor pipe (8192 x 8192 -> 8192 bf16 180 us = 6.1 PFLOP/s at 1.55 GHz, the pipe 86 % active; 4096 x 8192 -> 8192 91 to 97 us),
// with short K or fp32 outputs the epilogue's stores (24576 x 1024 -> 4096 fp32 with GELU 83 to 87 us for 403 MB of output); few tokens the
// weights (24 x 4096 -> 65536 28 us, DRAM 63 %), and the smallest the chain load, round, multiply, store (1 x 1024 -> 4096 4.7 us).

#include <cuda.h>

#include "q8_gemm_common.cuh"
#include "q8_mx4.cuh"

namespace q8 {

namespace {

using namespace ptx;
using namespace mx4;
using gemm_detail::encode_tiled_fn;
using gemm_detail::gelu_fast_x2;

constexpr int kAccStages = 2;
constexpr int kScaleBytes = 2 * kAtomBytes;  // of a tile
constexpr int kScaleCols = 4 * 2 + 8 * 2;    // TMEM columns of a stage's scales: 128 weight rows, 256 token rows, two atoms each
constexpr int kFusedStages = 9;
constexpr int kFusedTokens = 32;                // of a tile

// A tile: expert and its first row block of tokens, the tile's first token (in the expert and as a row of Y), how many it has, its first feature.
struct __align__(16) Tile {
    int32_t expert, block, first, row, count, feature, pad[2];
};
constexpr int kListed = 64;  // tiles of a CTA that are worked out at the start
template <int CTAS, int BN, int EW, bool FUSED>
struct Cfg {
    static constexpr int kThreads = 96 + 32 * EW;
    static constexpr int kBBytes = BN / CTAS * 128;
    static constexpr int kSbBytes = (BN > kTileRows ? 2 : 1) * kScaleBytes;  // of each row block that a tile's tokens may lie in
    static constexpr int kStageBytes = kTileBytes + kBBytes + kSbBytes;
    static constexpr int kTableBytes = 3 * (kMaxExperts + 1) * 4 + 4 + kListed * (int)sizeof(Tile);
    static constexpr int kBudget = 227 * 1024 - 1024 - kTableBytes - 512;
    static constexpr int kStages = FUSED ? kFusedStages : kBudget / kStageBytes > 8 ? 8 : kBudget / kStageBytes;
    // Two accumulators of 256 columns leave no room for the scales: they share 48 columns, which the epilogue empties first.
    static constexpr int kAccStride = BN == 256 ? 512 - 2 * kScaleCols - 256 : BN;
    static constexpr int kScaleCol0 = kAccStride + BN;
    static constexpr int kTmemCols = kScaleCol0 + 2 * kScaleCols <= 128 ? 128 : kScaleCol0 + 2 * kScaleCols <= 256 ? 256 : 512;
    static constexpr int kBarrierBytes = (2 * kStages + 2 * kAccStages + 1) * 8 + 32;
    static constexpr int kSmemBytes = 1024 + kStages * kStageBytes + kTableBytes + kBarrierBytes;
    static_assert(kScaleCol0 + 2 * kScaleCols <= 512, "TMEM columns");
    static_assert(kSmemBytes <= 232448 && kStages >= 3, "shared memory budget");
    static_assert(kBBytes % 1024 == 0 && (FUSED ? CTAS == 1 && BN == kFusedTokens : CTAS == 1 ? BN == 64 || BN == 128 : BN == 256) && (EW == 8 || EW == 16), "tile");
    // Instruction descriptor of kind::mxf4: E2M1 operands, both K-major, UE8M0 scales, M = 128 or 256 for the pair; N / 8 in bits
    // 17..22, which half of a scale word serves in bits 4..5 (B) and 29..30 (A).
    static constexpr uint32_t kInstrDesc = (1u << 7) | (1u << 10) | (1u << 23) | ((uint32_t)CTAS << 27);
};

// The instructions below are issued by one elected lane.  Descriptors of shared memory are given by their lower words, in which the
// address (in units of 16 bytes) is the only part that changes; what is constant is put together in line.
constexpr uint32_t kOperandHigh = (1024 >> 4) | (1u << 14) | (2u << 29);  // K-major, 128-byte swizzle, 8-row groups 1024 bytes apart
constexpr uint32_t kScalesHigh = (128 >> 4) | (1u << 14);                 // no swizzle, groups of 8 rows of 16 bytes 128 bytes apart
__device__ __forceinline__ uint32_t operand_low(uint32_t saddr) { return ((saddr & 0x3FFFFu) >> 4) | (1u << 16); }
__device__ __forceinline__ uint32_t scales_low(uint32_t saddr) { return (saddr & 0x3FFFFu) >> 4; }

template <int CTAS>
__device__ __forceinline__ void mma_mxf4(uint32_t tmem_d, uint32_t a_low, uint32_t b_low, uint32_t idesc, uint32_t tmem_sa, uint32_t tmem_sb,
                                         uint32_t accumulate)
{
    if constexpr (CTAS == 2)
        asm volatile(
            "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
            "setp.ne.b32 p, %6, 0;\n\t"
            "mov.b64 da, {%1, %7};\n\tmov.b64 db, {%2, %7};\n\t"
            "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], da, db, %3, [%4], [%5], p;\n\t}"
            ::"r"(tmem_d), "r"(a_low), "r"(b_low), "r"(idesc), "r"(tmem_sa), "r"(tmem_sb), "r"(accumulate), "n"(kOperandHigh)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
            "setp.ne.b32 p, %6, 0;\n\t"
            "mov.b64 da, {%1, %7};\n\tmov.b64 db, {%2, %7};\n\t"
            "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], da, db, %3, [%4], [%5], p;\n\t}"
            ::"r"(tmem_d), "r"(a_low), "r"(b_low), "r"(idesc), "r"(tmem_sa), "r"(tmem_sb), "r"(accumulate), "n"(kOperandHigh)
            : "memory");
}
// 512 bytes of shared memory (32 lanes x 16 bytes) to four columns of each of the four lane quarters; with CTAS = 2 in both CTAs, each from
// its own shared memory
template <int CTAS>
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint32_t low)
{
    if constexpr (CTAS == 2)
        asm volatile("{\n\t.reg .b64 d;\n\tmov.b64 d, {%1, %2};\n\ttcgen05.cp.cta_group::2.32x128b.warpx4 [%0], d;\n\t}" ::"r"(tmem), "r"(low), "n"(kScalesHigh) : "memory");
    else
        asm volatile("{\n\t.reg .b64 d;\n\tmov.b64 d, {%1, %2};\n\ttcgen05.cp.cta_group::1.32x128b.warpx4 [%0], d;\n\t}" ::"r"(tmem), "r"(low), "n"(kScalesHigh) : "memory");
}
// Untiled copy global -> shared; both 16-byte aligned, bytes a multiple of 16.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}
struct Plan {
    int32_t tiles;     // of a plain product
    int32_t tile_n;    // tokens of a full tile
    int32_t tiles_m;   // tiles of features
    uint32_t inv_m;    // floor(2^32 / tiles_m), at most 2^32 - 1: its high products are the quotients or one below
    int32_t num_kb;    // stages of a tile
    int32_t k_blocks;  // blocks of 32 along K
    int32_t w_blocks;  // row blocks of one expert's weights
    int32_t split;     // CTAs that share the K axis of a tile
    int32_t x_vec;     // bytes that loads of the tokens' values may take at once
};

// The tensor maps of a pair: weights, boxes of 128, 64 and 32 rows of tokens, scales.  One CTA copies without any.
template <int CTAS>
struct Maps {
    CUtensorMap w, x, x64, x32, s;
};
template <>
struct Maps<1> {};

// Tile t, those of an expert ordered features first; false behind the last one.  (A plain product needs no table.)
template <int TILE_M>
__device__ __forceinline__ bool find_tile(int32_t t, const ExpertTable &table, const Mx4GemmArgs &a, const Plan &p, Tile &out)
{
    uint32_t local = (uint32_t)t;
    int32_t end = (int32_t)a.M;
    out.expert = out.block = out.row = 0;
    if (a.offsets == nullptr) {
        if (t >= p.tiles) return false;
    } else {
        if (t >= table.tile[a.E]) return false;
        int e = 0, hi = a.E - 1;  // the last expert whose tiles begin at or before t: those without tokens have none
        while (e < hi) {
            const int mid = (e + hi + 1) >> 1;
            if (table.tile[mid] <= t) e = mid;
            else hi = mid - 1;
        }
        local -= (uint32_t)table.tile[e];
        out.expert = e;
        out.block = table.block[e];
        out.row = table.start[e];
        end = table.start[e + 1];
    }
    uint32_t n = __umulhi(local, p.inv_m);
    if (local - n * (uint32_t)p.tiles_m >= (uint32_t)p.tiles_m) ++n;
    out.first = (int32_t)n * p.tile_n;
    out.row += out.first;
    out.count = min(p.tile_n, end - out.row);
    out.feature = (int32_t)(local - n * p.tiles_m) * TILE_M;
    return true;
}

__device__ __forceinline__ void mbar_arrive_many(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
// Bounded wait whose first try is in line.
__device__ __noinline__ bool wait_on(uint32_t bar, uint32_t parity, volatile int *abort_flag, int32_t *status)
{
    return mbar_wait(bar, parity, abort_flag, status);
}
__device__ __forceinline__ bool wait_for(uint32_t bar, uint32_t parity, volatile int *abort_flag, int32_t *status)
{
    return mbar_try_wait(bar, parity) || wait_on(bar, parity, abort_flag, status);
}

// The tokens of a tile into the stages of the operand ring.  A warp takes every EW-th stage and all its rows, four at a time, the values of
// the next four on their way while it rounds these; with fewer stages than warps some share the rows of one.  (All warps on one stage
// after the other: 24 x 4096 -> 16384 18.9 us.  The fence at the end of a stage waits for loads in flight, so none are over it.)
template <int EW, int STAGES, int B_BYTES, int SB_BYTES, typename X>
__device__ __forceinline__ bool quantize_tokens(const Mx4GemmArgs &a, const Plan &plan, const Tile &tile, int32_t kb_lo, int32_t kb_hi, int ew, int32_t stage0, uint8_t *smem_b, uint8_t *smem_sb,
                                                uint64_t *full_bar, uint64_t *empty_bar, volatile int *abort_flag)
{
    const int lane = threadIdx.x & 31;
    const int stages = kb_hi - kb_lo, share = stages >= EW ? 1 : stages * 2 >= EW ? 2 : stages * 4 >= EW ? 4 : EW;  // warps of a stage
    const int every = EW / share, r0 = ew % share, step = 4 * share;
    const X *values = reinterpret_cast<const X *>(a.values) + (int64_t)tile.row * a.ldx;
    bool odd = false;
    for (int kb = kb_lo + ew / share; kb < kb_hi; kb += every) {
        const uint32_t n = (uint32_t)(stage0 + kb - kb_lo), s = n % STAGES, parity = (n / STAGES) & 1u;
        Columns<X, true> v[4], next[4];
        auto load = [&](int row, Columns<X, true> (&to)[4]) {
#pragma unroll
            for (int j = 0; j < 4; ++j, row += share) to[j].load(values + (int64_t)row * a.ldx, kb * kTileK + lane * 8, (int32_t)a.K, row < tile.count, plan.x_vec);
        };
        if (r0 < tile.count) load(r0, v);
        if (!__all_sync(0xffffffffu, wait_for(smem_u32(empty_bar + s), parity ^ 1u, abort_flag, a.status))) return false;
        for (int row = r0; row < tile.count; row += step) {
            if (row + step < tile.count) load(row + step, next);
            // (rows behind the last are rounded and dropped, so that the four can be worked on together)
            uint32_t words[4][kWords<X>], codes[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < kWords<X>; ++i) words[j][i] = v[j].w[i];
            const uint32_t scales = scale_words(quantize_rows<X, 4>(words, codes, odd), lane);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (row + share * j < tile.count) *reinterpret_cast<uint32_t *>(smem_b + s * B_BYTES + code_place(row + share * j, lane)) = codes[j];
            const int mine = row + share * ((lane >> 2) & 3);
            if ((lane & 3) == 0 && mine < tile.count)
                *reinterpret_cast<uint32_t *>(smem_sb + s * SB_BYTES + scale_place(mine, (lane >> 4) * 4) - kCodeBytes) = scales;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = next[j];
        }
        fence_proxy_async_smem();  // what the tensor cores read they read through the asynchronous proxy
        __syncwarp();
        if (lane == 0) mbar_arrive_many(smem_u32(full_bar + s), (uint32_t)every);
    }
    if (odd && lane == 0 && a.status != nullptr) atomicOr(a.status, 1 << Q8_ERR_SCALE);
    return true;
}

__device__ __forceinline__ void store_remote(uint32_t cluster_addr, float v)
{
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(cluster_addr), "f"(v) : "memory");
}
// The sums of a tile whose K axis a cluster shares: CTA r of S finishes the tokens from r ceil(count / S) on.  Every CTA stores what it has of each
// token in shared memory of the CTA that finishes it (the operand ring, which no CTA uses any more after the first barrier), and that one adds
// the parts in their order.  All threads of the cluster.
template <int EW, typename T>
__device__ __forceinline__ void join(const Mx4GemmArgs &a, const Plan &plan, const Tile &tile, int32_t part, uint32_t tmem_base, float *parts)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quarter = warp & 3, group = (warp - 3) >> 2, place = quarter * 32 + lane;
    __syncwarp();
    cluster_sync_all();
    const int share = (tile.count + plan.split - 1) / plan.split;
    if (warp >= 3) {
        tc_fence_after();
        for (int col = group * 32; col < tile.count; col += 8 * EW) {
            uint32_t v[32];
            tmem_ld_32x32(tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)col, v);
            tmem_ld_wait();
            int owner = col / share, in = col - owner * share;
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                if (col + j < tile.count) store_remote(map_to_cta(smem_u32(parts + (part * share + in) * kTileRows + place), (uint32_t)owner), __uint_as_float(v[j]));
                if (++in == share) {
                    in = 0;
                    ++owner;
                }
            }
        }
        tc_fence_before();
    }
    __syncwarp();
    cluster_sync_all();
    const int feature = tile.feature + place;
    if (warp >= 3 && feature < a.N) {
        const float bias = a.bias != nullptr ? __ldcg(a.bias + feature) : 0.0f;
        const int first = part * share, mine = min(share, tile.count - first);
        for (int i = group; i < mine; i += EW / 4) {
            float y = parts[i * kTileRows + place];
            for (int q = 1; q < plan.split; ++q) y += parts[(q * share + i) * kTileRows + place];
            y += bias;
            float other;
            if (a.act == Q8_ACT_GELU) gelu_fast_x2(pack_f32x2(y, y), y, other);
            reinterpret_cast<T *>(a.Y)[(int64_t)(tile.row + first + i) * a.ldy + feature] = from_float<T>(y);
        }
    }
}

template <int CTAS, int BN, int EW, typename T, typename X>
__global__ void __launch_bounds__(96 + 32 * EW, 1)
mx4_gemm_kernel(const __grid_constant__ Maps<CTAS> maps, Mx4GemmArgs a, Plan plan)
{
    constexpr bool FUSED = !std::is_void<X>::value;
    using C = Cfg<CTAS, BN, EW, FUSED>;
    constexpr int TILE_M = kTileRows * CTAS;
    constexpr int kStep = CTAS == 2 ? 64 : 16;  // widths of tiles are multiples of this
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *smem_a = smem;  // codes and scales of the weights
    uint8_t *smem_b = smem_a + C::kStages * kTileBytes;
    uint8_t *smem_sb = smem_b + C::kStages * C::kBBytes;
    uint64_t *full_bar = reinterpret_cast<uint64_t *>(smem_sb + C::kStages * C::kSbBytes);
    uint64_t *empty_bar = full_bar + C::kStages;
    uint64_t *tmem_full_bar = empty_bar + C::kStages;
    uint64_t *tmem_empty_bar = tmem_full_bar + kAccStages;
    uint64_t *drain_bar = tmem_empty_bar + kAccStages;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(drain_bar + 1);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    ExpertTable table;
    table.start = reinterpret_cast<int32_t *>(tmem_slot + 4);
    table.block = table.start + kMaxExperts + 1;
    table.tile = table.block + kMaxExperts + 1;
    Tile *list = reinterpret_cast<Tile *>((reinterpret_cast<uintptr_t>(table.tile + kMaxExperts + 1) + 15) & ~uintptr_t(15));

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CTAS == 2 ? cluster_ctarank() : 0u;
    const bool leader = rank == 0;
    if (warp == 0) {  // a lane a barrier
        constexpr int kBarriers = 2 * C::kStages + 2 * kAccStages + 1;
        static_assert(kBarriers <= 32, "barriers");
        // full: both producers (the leader's), with the byte counts, or the weights' and the warps that quantise; tmem_empty: the epilogue's warps
        if (lane < kBarriers)
            mbar_init(smem_u32(full_bar + lane), lane < C::kStages ? (FUSED ? 1 + EW : 2)
                                                 : lane >= 2 * C::kStages + kAccStages && lane < 2 * C::kStages + 2 * kAccStages ? EW * CTAS : 1);
        if (lane == 0) *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // A pair allocates together, so both of its CTAs have started first; after this the peer's barriers exist as well.
    if (CTAS == 2) {
        __syncwarp();
        cluster_sync_all();
    }
    if (warp == 1) {
        if (CTAS == 2) tmem_alloc_pair(smem_u32(tmem_slot), C::kTmemCols);
        else tmem_alloc(smem_u32(tmem_slot), C::kTmemCols);
    }
    const int32_t split = CTAS == 1 ? plan.split : 1, unit = CTAS * split;  // CTAs of a tile
    const int32_t first_tile = blockIdx.x / unit, tile_step = gridDim.x / unit;
    const int32_t part = split > 1 ? blockIdx.x % split : 0;  // stages of the tile that are this CTA's
    const int32_t kb_lo = split > 1 ? part * plan.num_kb / split : 0, kb_hi = split > 1 ? (part + 1) * plan.num_kb / split : plan.num_kb;
    if (warp == 2) {
        if (a.offsets != nullptr) {
            const bool bad = build_expert_table(table, a.offsets, a.E, (int32_t)a.M, plan.tile_n, plan.tiles_m);
            if (bad && lane == 0 && blockIdx.x == 0 && a.status != nullptr) atomicOr(a.status, 1 << Q8_ERR_INDEX);
        }
        // A lane a tile: looked up by every role for every tile, between two of them, they took 400 cycles each time.
        const int32_t all = a.offsets != nullptr ? table.tile[a.E] : plan.tiles;
#pragma unroll 1
        for (int i = lane; i < kListed; i += 32) {
            Tile found;
            if (!find_tile<TILE_M>(first_tile + i * tile_step, table, a, plan, found)) found.count = 0;
            list[i] = found;
            if (first_tile + (i - lane + 31) * tile_step >= all) break;  // (the last of these 32 ended the list)
        }
    }
    // The i-th tile of this CTA; false behind the last one.
    auto get_tile = [&](int32_t i, Tile &tile) {
        if (i >= kListed) return find_tile<TILE_M>(first_tile + i * tile_step, table, a, plan, tile);
        tile = list[i];
        return tile.count > 0;
    };
    // A plain product's weight producer, which made the barriers and needs neither the list nor TMEM, goes ahead without the others.
    tc_fence_before();
    __syncwarp();
    const bool goes_ahead = CTAS == 1 && a.offsets == nullptr && warp == 0;
    if (goes_ahead) asm volatile("barrier.cta.arrive 1, %0;" ::"n"(C::kThreads) : "memory");
    else asm volatile("barrier.cta.sync 1, %0;" ::"n"(C::kThreads) : "memory");
    tc_fence_after();
    const uint32_t tmem_base = *reinterpret_cast<volatile uint32_t *>(tmem_slot);  // (not yet there for that producer, which does not use it)
    // The next kernel is parked beside single CTAs with one tile each, or with up to three where they quantise their tokens themselves, and only once
    // this CTA has its tensor memory, whose allocation waits without a limit.  Longer products and pairs have nothing parked beside them: they
    // let the next one start when they end.  (Let in early / when it ends, us, replayed: 1 x 1024 -> 4096 4.1 / 5.0, 1 x 8192 -> 512 5.8 / 7.4, 1 x 1024 -> 32768 7.2 /
    // 8.0, 1000 slots of 7 experts 8.1 / 9.7, but with two or three tiles behind a quantise pass 24 x 4096 -> 32768 18.3 / 16.4, 640 x 512 -> 4096 9.6 / 7.9, 32 slots
    // on 64 experts 12.4 / 11.0.)
    constexpr int kRoundsBeside = FUSED ? 3 : 1;
    if (!goes_ahead) grid_dependency_release_next(CTAS == 1 && (a.offsets != nullptr ? table.tile[a.E] : plan.tiles) <= kRoundsBeside * tile_step);

    Tile tile;
    auto width_of = [&](const Tile &t) { return (t.count + kStep - 1) / kStep * kStep; };
    if (warp == 0 || (warp == 2 && !FUSED)) {
        // ---------------- producers ----------------
        // A pair's loads all report to the leader's barrier, which its MMA warp waits on.  The tensor maps of the pair see tiles as rows of 128
        // bytes: 136 of them to a tile, the last 8 its scales.
        const bool weights = warp == 0;
        // The quantise pass in front of a grouped product has waited for all kernels before it when this one starts, and writes neither weights
        // nor offsets, so these may be read before it ends: as much as the ring holds (32 slots on 64 experts 12.7 -> 11.7 us).  (Asking for
        // the rest into L2 as well holds up the loads behind it: 24 x 4096 -> 16384 9.9 -> 10.6 us, 32 slots on 64 experts 9.5 -> 12.)
        const bool early = CTAS == 1 && a.offsets != nullptr;
        // One lane does all of it: a warp that waits together and then lets one lane issue takes 500 cycles a stage, more than the products.
        if (elect_one()) {
            int s = 0;
            uint32_t phase = 0;
            int64_t issued = 0;
            bool ok = true, waited = false;
            // (a plain product's weight producer does not wait for the list)
            const bool ahead = CTAS == 1 && a.offsets == nullptr && weights;
            for (int32_t i = 0; ok && (ahead ? find_tile<TILE_M>(first_tile + i * tile_step, table, a, plan, tile) : get_tile(i, tile)); ++i) {
                const int width = width_of(tile), mine = width / CTAS;
                const int64_t w_tile = ((int64_t)tile.expert * plan.w_blocks + tile.feature / kTileRows + rank) * plan.num_kb;
                const int first = tile.first + (int)rank * mine, sub = first % kTileRows;
                const int64_t x_tile = ((int64_t)tile.block + first / kTileRows) * plan.num_kb;
                const int64_t s_tile = ((int64_t)tile.block + tile.first / kTileRows) * plan.num_kb;
                const bool two_scales = tile.first % kTileRows + width > kTileRows;  // the tile's tokens lie in two row blocks
                const int in_first = min(mine, kTileRows - sub);                     // of this CTA's tokens, those in the first row block
                const uint32_t bytes = CTAS == 1 ? (weights ? kTileBytes : (uint32_t)mine * 128 + kScaleBytes)
                                                 : 2 * (weights ? kTileBytes + kScaleBytes : (uint32_t)mine * 128 + kScaleBytes * (two_scales ? 1 : 0));
                if (!waited && !(weights && early)) grid_dependency_wait();
                waited = true;
                const uint8_t *w = a.W + (w_tile + kb_lo) * kTileBytes, *x = a.X + (x_tile + kb_lo) * kTileBytes;
                bool ready = mbar_try_wait(smem_u32(empty_bar + s), phase ^ 1u);
                for (int kb = kb_lo; kb < kb_hi; ++kb) {
                    ok = ready || wait_on(smem_u32(empty_bar + s), phase ^ 1u, abort_flag, a.status);
                    if (!ok) break;
                    const int s_next = s + 1 == C::kStages ? 0 : s + 1;
                    if (kb + 1 < kb_hi) ready = mbar_try_wait(smem_u32(empty_bar + s_next), phase ^ (s_next == 0 ? 0u : 1u));  // (its answer is there by the time it is needed)
                    const uint32_t fb = smem_u32(full_bar + s);
                    const uint32_t dst_b = smem_u32(smem_b + s * C::kBBytes), dst_s = smem_u32(smem_sb + s * C::kSbBytes);
                    if constexpr (CTAS == 1) {
                        mbar_expect_tx(fb, bytes);
                        if (weights) {
                            bulk_load(smem_u32(smem_a + s * kTileBytes), w, kTileBytes, fb);
                            w += kTileBytes;
                        } else {
                            bulk_load(dst_b, x + sub * 128, (uint32_t)mine * 128, fb);
                            bulk_load(dst_s, x + kCodeBytes, kScaleBytes, fb);
                            x += kTileBytes;
                        }
                    } else {
                        if (leader) mbar_expect_tx(fb, bytes);
                        const uint32_t fb_leader = map_to_cta(fb, 0);
                        constexpr int kRowsPerTile = kTileBytes / 128;
                        if (weights) {
                            tma_load_2d_pair(smem_u32(smem_a + s * kTileBytes), &maps.w, 0, (int32_t)(w_tile + kb) * kRowsPerTile, fb_leader);
                            tma_load_2d_pair(dst_s, &maps.s, 0, (int32_t)(s_tile + kb) * kRowsPerTile + kTileRows, fb_leader);
                        } else {
                            // 32, 64, 96 or 128 rows, in a box or two that end with the row block or with the tile's half
                            if (mine == kTileRows) {
                                tma_load_2d_pair(dst_b, &maps.x, 0, (int32_t)(x_tile + kb) * kRowsPerTile, fb_leader);
                            } else {
                                int box;
                                for (int r = 0; r < mine; r += box) {
                                    const bool second = r >= in_first;
                                    const int32_t at = (int32_t)(x_tile + kb + (second ? plan.num_kb : 0)) * kRowsPerTile + (second ? r - in_first : sub + r);
                                    box = (second ? mine : in_first) - r >= 64 ? 64 : 32;
                                    tma_load_2d_pair(dst_b + r * 128, box == 64 ? &maps.x64 : &maps.x32, 0, at, fb_leader);
                                }
                            }
                            if (two_scales)
                                tma_load_2d_pair(dst_s + kScaleBytes, &maps.s, 0, (int32_t)(s_tile + kb + plan.num_kb) * kRowsPerTile + kTileRows, fb_leader);
                        }
                    }
                    ++issued;
                    s = s_next;
                    if (s == 0) phase ^= 1u;
                }
            }
            // Every stage has been given back before the CTA ends: the issuer's last commits arrive at these barriers, a pair's at the peer's
            // too, and nothing else waits for them.
            for (int i = 0; ok && i < C::kStages; ++i) {
                ok = wait_for(smem_u32(empty_bar + s), phase ^ 1u, abort_flag, a.status);
                if (++s == C::kStages) { s = 0; phase ^= 1u; }
            }
            if (!ok) {
                // Aborting: this warp's copies land before the CTA gives up its shared memory (bounded: the other producer may have stopped
                // a stage earlier, and its barrier then never completes).
                const uint64_t t0 = global_timer_ns();
                if (leader) {
                    for (int64_t i = 1; i <= (issued < C::kStages ? issued : C::kStages); ++i) {
                        const int64_t k = issued - i;
                        while (!mbar_try_wait(smem_u32(full_bar + k % C::kStages), (uint32_t)(k / C::kStages) & 1u) && global_timer_ns() - t0 < 50000000ull) {}
                    }
                } else {
                    while (global_timer_ns() - t0 < 1000000ull) {}  // the peer cannot poll the leader's barrier
                }
            }
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer (the leader's drives the pair) ----------------
        if (leader && elect_one()) {
            auto commit = [&](uint64_t *bar) {
                if (CTAS == 2) umma_commit_pair(smem_u32(bar));
                else umma_commit(smem_u32(bar));
            };
            int s = 0, as = 0;
            uint32_t phase = 0, aphase = 0;
            const uint32_t a0 = operand_low(smem_u32(smem_a)), b0 = operand_low(smem_u32(smem_b));
            const uint32_t sa0 = scales_low(smem_u32(smem_a + kCodeBytes)), sb0 = scales_low(smem_u32(smem_sb));
            uint32_t scale_col = tmem_base + C::kScaleCol0;
            const uint32_t scale_sum = 2 * scale_col + kScaleCols;
            const int last_blocks = plan.k_blocks - (plan.num_kb - 1) * (kTileK / kBlock);  // of the last stage
            bool ok = true;
            for (int32_t i = 0; ok && get_tile(i, tile); ++i) {
                // the tile before last has left this accumulator, or the last one the columns that it shares with it
                constexpr bool kShared = C::kAccStride < BN;
                ok = wait_for(smem_u32(tmem_empty_bar + (kShared ? as ^ 1 : as)), kShared && as == 1 ? aphase : aphase ^ 1u, abort_flag, a.status);
                if (!ok) break;
                tc_fence_after();
                const int width = width_of(tile);
                const uint32_t tmem_d = tmem_base + (uint32_t)(as * C::kAccStride);
                const uint32_t idesc = C::kInstrDesc | ((uint32_t)(width >> 3) << 17);
                // Where the tile's first token is in its row block: a multiple of 64, so that the scales start at an even column, as they have to.
                // (Tokens that were quantised here are at the start of the stage, wherever the tile begins.)
                const int sub = FUSED ? 0 : tile.first % kTileRows;
                const uint32_t sub_col = (uint32_t)sub >> 5;
                const bool two_blocks = sub + width > kTileRows;
                bool ready = mbar_try_wait(smem_u32(full_bar + s), phase);
                for (int kb = kb_lo; kb < kb_hi; ++kb) {
                    ok = ready || wait_on(smem_u32(full_bar + s), phase, abort_flag, a.status);
                    if (!ok) break;
                    const int s_next = s + 1 == C::kStages ? 0 : s + 1;
                    if (kb + 1 < kb_hi) ready = mbar_try_wait(smem_u32(full_bar + s_next), phase ^ (s_next == 0 ? 1u : 0u));  // (behind the last tile nothing would end this wait)
                    tc_fence_after();
                    const uint32_t da = a0 + (uint32_t)s * (kTileBytes >> 4), db = b0 + (uint32_t)s * (C::kBBytes >> 4);
                    const uint32_t dsa = sa0 + (uint32_t)s * (kTileBytes >> 4), dsb = sb0 + (uint32_t)s * (C::kSbBytes >> 4);
                    // scales of this stage: per atom 4 columns for the weights, 8 for the tokens; the two buffers take turns
                    const uint32_t sa_col = scale_col, sb_col = sa_col + 8;
                    scale_col = scale_sum - scale_col;
                    // Blocks 0 and 1 or 2 and 3 of an atom serve a product: half 0 or 2 of its words.
                    auto product = [&](int k, uint32_t accumulate) {
                        const uint32_t half = (uint32_t)(k & 1) * 2;
                        mma_mxf4<CTAS>(tmem_d, da + (uint32_t)(2 * k), db + (uint32_t)(2 * k), idesc | (half << 4) | (half << 29), sa_col + 4 * (k >> 1),
                                       sb_col + 8 * (k >> 1) + sub_col, accumulate);
                    };
                    auto scales = [&](int atom) {
                        copy_scales<CTAS>(sa_col + 4 * atom, dsa + (uint32_t)(atom * (kAtomBytes >> 4)));
                        copy_scales<CTAS>(sb_col + 8 * atom, dsb + (uint32_t)(atom * (kAtomBytes >> 4)));
                        if (BN > 128 && two_blocks) copy_scales<CTAS>(sb_col + 8 * atom + 4, dsb + (uint32_t)((2 + atom) * (kAtomBytes >> 4)));
                    };
                    if (kb + 1 < plan.num_kb || last_blocks == kTileK / kBlock) {  // (a whole tile: without a test at every instruction)
                        scales(0);
                        scales(1);
                        product(0, kb != kb_lo);
                        product(1, 1);
                        product(2, 1);
                        product(3, 1);
                    } else {
                        scales(0);
                        if (last_blocks > 4) scales(1);
                        product(0, kb != kb_lo);
#pragma unroll 1
                        for (int k = 1; 2 * k < last_blocks; ++k) product(k, 1);
                    }
                    commit(empty_bar + s);
                    if (kb + 1 == kb_hi) commit(tmem_full_bar + as);
                    s = s_next;
                    if (s == 0) phase ^= 1u;
                }
                if (!ok) break;
                if (++as == kAccStages) { as = 0; aphase ^= 1u; }
            }
            if (!ok) {
                // Aborting: wait (bounded) for the tensor core to finish what was issued.
                commit(drain_bar);
                const uint64_t t0 = global_timer_ns();
                while (!mbar_try_wait(smem_u32(drain_bar), 0) && global_timer_ns() - t0 < 50000000ull) {}
            }
        }
    } else if (warp >= 3) {
        // ---------------- epilogue ----------------
        const int ew = warp - 3;
        const int quarter = warp & 3;  // TMEM lanes 32 * quarter .. + 31
        constexpr int kGroups = EW / 4;  // warps that share a quarter take every kGroups-th run of 32 columns
        const int group = ew >> 2;
        int as = 0;
        uint32_t aphase = 0;
        bool waited = false;
        int32_t stage0 = 0;  // stages of the tiles before
        for (int32_t n = 0; get_tile(n, tile); ++n) {
            if constexpr (FUSED) {
                if (!waited) grid_dependency_wait();
                waited = true;
                const bool done = quantize_tokens<EW, C::kStages, C::kBBytes, C::kSbBytes, X>(a, plan, tile, kb_lo, kb_hi, ew, stage0, smem_b, smem_sb, full_bar, empty_bar, abort_flag);
                if (!done) break;
                stage0 += kb_hi - kb_lo;
            }
            const int feature0 = tile.feature + (int)rank * kTileRows + quarter * 32, feature = feature0 + lane;
            const bool mine = feature < a.N;
            if (!waited) grid_dependency_wait();  // (an earlier kernel may have written the bias, which is not read-only data therefore, or still read Y)
            waited = true;
            const float bias = mine && a.bias != nullptr ? __ldcg(a.bias + (int64_t)tile.expert * a.N + feature) : 0.0f;
            const bool ok = __all_sync(0xffffffffu, wait_for(smem_u32(tmem_full_bar + as), aphase, abort_flag, a.status));
            if (!ok) break;
            tc_fence_after();
            if (CTAS == 1 && split > 1) break;  // (its only tile: on to the join)
            const uint32_t acc = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(as * C::kAccStride);
            auto release = [&]() {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (CTAS == 2) mbar_arrive_cluster_relaxed(map_to_cta(smem_u32(tmem_empty_bar + as), 0));
                    else mbar_arrive(smem_u32(tmem_empty_bar + as));
                }
            };
            // With shared columns the first accumulator is emptied from its end, the second from its beginning, and both are handed on once no
            // warp has shared columns left to read; a warp gets to the next tile only after all of this one, so the rest is empty in time.
            constexpr int kRounds = (BN / 32 + kGroups - 1) / kGroups;
            bool released = false;
#pragma unroll 1
            for (int i = 0; i < kRounds; ++i) {
                const int block = C::kAccStride < BN && as == 0 ? BN / 32 - 1 - (i * kGroups + group) : i * kGroups + group, col = block * 32;
                if (col >= tile.count || col >= BN) continue;
                uint32_t v[32];
                tmem_ld_32x32(acc + (uint32_t)col, v);
                tmem_ld_wait();
                if (C::kAccStride < BN ? !released : col + 32 * kGroups >= tile.count) {
                    release();
                    released = true;
                }
                if (feature0 >= a.N) continue;
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) + bias);
                if (a.act == Q8_ACT_GELU) {
#pragma unroll
                    for (int j = 0; j < 32; j += 2) {
                        float y0, y1;
                        gelu_fast_x2(pack_f32x2(__uint_as_float(v[j]), __uint_as_float(v[j + 1])), y0, y1);
                        v[j] = __float_as_uint(y0);
                        v[j + 1] = __float_as_uint(y1);
                    }
                }
                if (mine) {
                    T *y = reinterpret_cast<T *>(a.Y) + (int64_t)(tile.row + col) * a.ldy + feature;
                    if (col + 32 <= tile.count) {
#pragma unroll
                        for (int j = 0; j < 32; ++j, y += a.ldy) *y = from_float<T>(__uint_as_float(v[j]));
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j, y += a.ldy)
                            if (col + j < tile.count) *y = from_float<T>(__uint_as_float(v[j]));
                    }
                }
            }
            if (!released) release();
            if (++as == kAccStages) { as = 0; aphase ^= 1u; }
        }
    }

    if constexpr (CTAS == 1) {
        if (split > 1) join<EW, T>(a, plan, list[0], part, tmem_base, reinterpret_cast<float *>(smem));
    }

    // ---------------- teardown (reached by every thread, also when aborting) ----------------
    __syncwarp();            // (the idle lanes of a producer wait here: in the next line they would hold up the one that works)
    grid_dependency_wait();  // also where a CTA had no tile: this kernel ends after the one before it
    tc_fence_before();
    __syncthreads();
    if (CTAS == 2) {
        __syncwarp();
        cluster_sync_all();  // the peer has finished with this CTA's barriers and with the shared accumulators
    }
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        if (CTAS == 2) tmem_dealloc_pair(tmem_base, C::kTmemCols);
        else tmem_dealloc(tmem_base, C::kTmemCols);
    }
}

// ------------------------------------------------------------------ host side
// Tiles as rows of 128 bytes, boxes of box_rows of them; what lies behind the last reads as zero.
bool tiles_map(CUtensorMap *map, const uint8_t *base, int64_t tiles, int box_rows)
{
    const auto fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {128, (cuuint64_t)(tiles * (kTileBytes / 128))}, strides[1] = {128};
    const cuuint32_t box[2] = {128, (cuuint32_t)box_rows}, estr[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
template <int CTAS, int BN, int EW, typename T, typename X>
cudaError_t launch_typed(const Mx4GemmArgs &a, Plan plan, int64_t tiles, cudaStream_t s)
{
    plan.tiles = (int32_t)tiles;
    plan.inv_m = plan.tiles_m > 1 ? (uint32_t)((uint64_t(1) << 32) / plan.tiles_m) : 0xffffffffu;
    using C = Cfg<CTAS, BN, EW, !std::is_void<X>::value>;
    auto kernel = mx4_gemm_kernel<CTAS, BN, EW, T, X>;
    static bool attr_set[64] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!attr_set[dev]) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmemBytes);
        if (e != cudaSuccess) return e;
        attr_set[dev] = true;
    }
    Maps<CTAS> maps;
    if constexpr (CTAS == 2) {
        const int64_t w_tiles = (int64_t)a.E * plan.w_blocks * plan.num_kb;
        const int64_t x_tiles = (a.offsets != nullptr ? most_row_blocks(a.M, a.E) : ceil_div(a.M, kTileRows)) * plan.num_kb;
        if (!tiles_map(&maps.w, a.W, w_tiles, kTileBytes / 128) || !tiles_map(&maps.x, a.X, x_tiles, kTileRows) || !tiles_map(&maps.x64, a.X, x_tiles, 64) ||
            !tiles_map(&maps.x32, a.X, x_tiles, 32) || !tiles_map(&maps.s, a.X, x_tiles, kScaleBytes / 128))
            return cudaErrorInvalidValue;
    }
    const int64_t units = sm_count() / (CTAS * plan.split);
    const int grid = (int)(tiles < units ? tiles : units) * CTAS * plan.split;
    LaunchInfo &li = last_launch_info();
    li.gemm_kernel = 1;
    li.block_n = plan.tile_n;
    li.ctas = CTAS * plan.split;
    li.epilogue_warps = EW;
    li.grid = grid;
    li.launches += 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(C::kThreads);
    cfg.dynamicSmemBytes = C::kSmemBytes;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CTAS * plan.split;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = CTAS * plan.split > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, maps, a, plan);
}

template <int CTAS, int BN, int EW, typename X = void>
cudaError_t launch_shape(const Mx4GemmArgs &a, const Plan &plan, int64_t tiles, cudaStream_t s)
{
    switch (a.y_dtype) {
        case Q8_F32: return launch_typed<CTAS, BN, EW, float, X>(a, plan, tiles, s);
        case Q8_F16: return launch_typed<CTAS, BN, EW, __half, X>(a, plan, tiles, s);
        default: return launch_typed<CTAS, BN, EW, __nv_bfloat16, X>(a, plan, tiles, s);
    }
}

}  // namespace

// CTAs that share the K axis of each of so many tiles of `tokens` tokens: a stage takes 0.21 us, the join 2.2 and 0.03 more for each token; clusters of 8
// find room on the device together up to 12 (16 of them take two rounds: 1 x 8192 -> 2048 9.6 -> 11.8 us).  Shared / not, us: 1 x 8192 -> 512 5.7 / 9.4, 64
// rows 8.5 / 10.2, 1 x 20000 -> 300 6.8 / 19.3, 1 x 4096 -> 1024 5.8 / 6.1, but 64 rows 8.4 / 7.1 and 1 x 2048 -> 256 5.5 / 4.3.
int split_of(int64_t tiles, int num_kb, int64_t tokens)
{
    int best = 1;
    double most = 0.2;
    for (int split : {2, 4, 8}) {
        if (num_kb < 2 * split || tiles * split > (split == 8 ? 96 : 112) || tiles * split > sm_count()) break;
        const double gain = 0.21 * num_kb * (split - 1) / split - 2.2 - 0.03 * (double)tokens;
        if (gain > most) {
            best = split;
            most = gain;
        }
    }
    return best;
}

// Microseconds of `rounds` tiles one after the other: set-up, and for each tile its stages and what is not hidden under the next one's.
// Fitted to 300 products (100 to 8192 tokens, K = 256 to 4096, 256 to 4096 features, bf16 without and fp32 with GELU) timed with
// each width, 5 % off for single CTAs, 11 % for pairs.  Taking the fastest by it costs 0.6 % on average; 192 wide tiles of one CTA, or pairs as soon as
// each has work, 5.8 % and up to 45 % (4096 x 4096 -> 1024: 64 / 128 / 192 wide 16.0 / 11.2 / 14.9 us, pairs 10.3).
double tile_cost(int n, int64_t rounds, int num_kb, bool gelu)
{
    const double start = n == 64 ? 2.2 : n == 128 ? 2.3 : 2.5;
    const double stage = n == 64 ? 0.183 : n == 128 ? 0.210 : 0.290;
    const double tile = gelu ? (n == 64 ? 0.89 : n == 128 ? 1.53 : 2.99) : (n == 64 ? 0.54 : n == 128 ? 0.87 : 1.80);
    return start + (double)rounds * (stage * num_kb + tile);
}

// One launch instead of two, against tokens that every CTA reads and rounds itself, behind the weights that fill the way into its SM: about
// 1 us for every four tokens and 8 stages.  (Fused / not, us, replayed and then called from Python: 1 x 1024 -> 4096 4.0 / 5.0 and 4.3 / 6.9, 16 x 1024 ->
// 4096 5.5 / 4.8 and 5.7 / 6.9, 32 x 1024 -> 4096 7.4 / 4.9 and 7.6 / 7.1, 4 x 4096 -> 16384 8.4 / 9.8 and 8.5 / 9.9, 8 x 4096 -> 16384 10.2 / 9.7 and
// 10.5 / 9.8, 4 x 8192 -> 8192 10.6 / 11.8 and 10.9 / 12.0.)
bool mx4_fused_preferred(int64_t M, int64_t K) { return M <= 4 || (M <= kFusedTokens && M * K <= 16384); }

cudaError_t launch_mx4_gemm(const Mx4GemmArgs &a, cudaStream_t s)
{
    Plan p = {};
    p.num_kb = (int32_t)tiles_along(a.K);
    p.k_blocks = (int32_t)ceil_div(a.K, kBlock);
    p.w_blocks = (int32_t)ceil_div(a.N, kTileRows);
    p.tiles_m = p.w_blocks;
    const int64_t hit = a.E < a.M ? a.E : a.M;  // experts with tokens, at most
    const int64_t extra = a.E > 1 ? hit : 0;    // tiles of tokens that are not full, at most
    const int64_t pairs = ceil_div(a.N, 2 * kTileRows);
    p.split = 1;
    if (a.values != nullptr) {
        p.tile_n = kFusedTokens;
        p.x_vec = value_alignment(a.values, a.ldx, a.x_dtype == Q8_F32 ? 4 : 2);
        const int64_t tiles = ceil_div(a.M, p.tile_n) * p.tiles_m;
        p.split = split_of(tiles, p.num_kb, a.M);
        switch (a.x_dtype) {
            case Q8_F32: return launch_shape<1, kFusedTokens, 8, float>(a, p, tiles, s);
            case Q8_F16: return launch_shape<1, kFusedTokens, 8, __half>(a, p, tiles, s);
            default: return launch_shape<1, kFusedTokens, 8, __nv_bfloat16>(a, p, tiles, s);
        }
    }
    // The width of a tile whose rounds over the device take the shortest time.
    const int sms = sm_count();
    int best = 0;
    double best_cost = 0.0;
    for (int n : {64, 128, 256}) {
        const int64_t tokens = ceil_div(a.M, n) + extra / 2, tiles = (tokens > hit ? tokens : hit) * (n == 256 ? pairs : p.w_blocks);
        const double cost = tile_cost(n, ceil_div(tiles, n == 256 ? sms / 2 : sms), p.num_kb, a.act == Q8_ACT_GELU);
        if (best == 0 || cost < best_cost) {
            best = n;
            best_cost = cost;
        }
    }
    p.tile_n = best;
    if (best == 256) p.tiles_m = (int32_t)pairs;
    const int64_t tiles = (ceil_div(a.M, best) + extra) * p.tiles_m;  // at most
    if (best == 64 && a.offsets == nullptr) p.split = split_of(tiles, p.num_kb, a.M < 64 ? a.M : 64);
    if (best == 64) return launch_shape<1, 64, 8>(a, p, tiles, s);
    if (best == 128) return launch_shape<1, 128, 8>(a, p, tiles, s);
    // GELU keeps 16 warps busy; without it 8 with more registers are faster (24576 x 1024 -> 4096 bf16, 8 / 16 warps: 60 / 62 us, with GELU 95 / 82;
    // 8192 x 2048 -> 8192 60 / 67 and 80 / 77).
    return a.act == Q8_ACT_GELU ? launch_shape<2, 256, 16>(a, p, tiles, s) : launch_shape<2, 256, 8>(a, p, tiles, s);
}

}  // namespace q8
