// Product of an MXFP4 activation with MXFP4 weights on Blackwell tensor cores (sm_100a), plain or grouped by expert:
//
//   Y[t, n] = act(sum_k x[t, k] w[e][n, k] + b[e][n])     for the slots t of expert e
//
// The weights are the A operand (accumulator rows = TMEM lanes = output features), the tokens the B operand (accumulator columns).
// So a tile is as narrow as its tokens are few, an expert with three rows costs 16 columns, a lane of the epilogue has one bias
// value for the whole tile, and a warp's store of one column is 32 neighbouring features of a token: whole sectors of Y without any
// staging.
//
//   warp 0      TMA producer of the weights: 128-byte-swizzled boxes of 128 rows x 256 codes, and their scales
//   warp 2      the same for the tokens
//   warp 1      MMA issuer: copies the scales to TMEM (tcgen05.cp), issues tcgen05.mma kind::mxf4 (64 codes a time, one scale per
//               32), fp32 accumulators in TMEM, double buffered
//   warps 3..   epilogue: tcgen05.ld, bias, GELU, conversion, store
//
// A plain product is the grouped one with a single expert.  Every wait on an mbarrier is bounded: after ~2 s the CTA raises
// Q8_ERR_TIMEOUT in the status word, all roles leave their loops, copies and products in flight are waited for (bounded), TMEM is freed.

#include <cuda.h>

#include "q8_gemm_common.cuh"
#include "q8_mx4.cuh"

namespace q8 {

namespace {

using namespace ptx;
using namespace mx4;
using gemm_detail::encode_tiled_fn;
using gemm_detail::gelu_fast_x2;

constexpr int kTileM = 128;           // weight rows of a tile
constexpr int kStageK = 256;          // codes of a stage row: one 128-byte swizzle span
constexpr int kStageRowBytes = 128;
constexpr int kMmaK = 64;
constexpr int kAccStages = 2;
constexpr int kBoxRows = 32;          // tokens of the small box, for tiles that are not full
constexpr int kScaleCols = 4 * 2 + 8 * 2;  // TMEM columns of a stage's scales: 128 weight rows, 256 token rows, two atoms each

template <int BN, int EW>
struct Cfg {
    static constexpr int kThreads = 96 + 32 * EW;
    static constexpr int kABytes = kTileM * kStageRowBytes;
    static constexpr int kBBytes = BN * kStageRowBytes;
    static constexpr int kSaBytes = 2 * kAtomBytes;
    static constexpr int kSbBytes = 4 * kAtomBytes;  // two row blocks: a tile of 192 may start in the middle of one
    static constexpr int kStageBytes = kABytes + kBBytes + kSaBytes + kSbBytes;
    static constexpr int kTableBytes = 2 * (kMaxExperts + 1) * 4 + 8;
    static constexpr int kBudget = 227 * 1024 - 1024 - kTableBytes - 512;
    static constexpr int kStages = kBudget / kStageBytes > 8 ? 8 : kBudget / kStageBytes;
    static constexpr int kScaleCol0 = kAccStages * BN;
    static constexpr int kTmemCols = kScaleCol0 + 2 * kScaleCols <= 128 ? 128 : kScaleCol0 + 2 * kScaleCols <= 256 ? 256 : 512;
    static constexpr int kBarrierBytes = (2 * kStages + 2 * kAccStages + 1) * 8 + 16;
    static constexpr int kSmemBytes = 1024 + kStages * kStageBytes + kTableBytes + kBarrierBytes;
    static_assert(kScaleCol0 + 2 * kScaleCols <= 512, "TMEM columns");
    static_assert(kSmemBytes <= 232448 && kStages >= 3, "shared memory budget");
    static_assert(BN % kBoxRows == 0 && BN <= 192, "tile width");
};

// Instruction descriptor of kind::mxf4: E2M1 operands, both K-major, UE8M0 scales, M = 128; N / 8 in bits 17..22, which half of a
// scale word serves in bits 4..5 (B) and 29..30 (A).
constexpr uint32_t kInstrDesc = (1u << 7) | (1u << 10) | (1u << 23) | ((uint32_t)(kTileM >> 7) << 27);

__device__ __forceinline__ void mma_mxf4_elected(uint32_t elected, uint32_t tmem_d, uint64_t desc_a, uint64_t desc_b, uint32_t idesc,
                                                 uint32_t tmem_sa, uint32_t tmem_sb, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "setp.ne.b32 e, %7, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(tmem_d), "l"(desc_a), "l"(desc_b), "r"(idesc), "r"(tmem_sa), "r"(tmem_sb), "r"(accumulate), "r"(elected)
        : "memory");
}
// 512 bytes of shared memory (32 lanes x 16 bytes) to four columns of each of the four lane quarters
__device__ __forceinline__ void copy_scales_elected(uint32_t elected, uint32_t tmem, uint64_t desc)
{
    asm volatile(
        "{\n\t.reg .pred e;\n\t"
        "setp.ne.b32 e, %2, 0;\n\t"
        "@e tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;\n\t}"
        ::"r"(tmem), "l"(desc), "r"(elected)
        : "memory");
}
// Untiled copy global -> shared; both 16-byte aligned, bytes a multiple of 16.
__device__ __forceinline__ void bulk_load_elected(uint32_t elected, uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile(
        "{\n\t.reg .pred e;\n\t"
        "setp.ne.b32 e, %4, 0;\n\t"
        "@e cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n\t}"
        ::"r"(dst), "l"(src), "r"(bytes), "r"(bar), "r"(elected)
        : "memory");
}
// An atom of scales in shared memory: no swizzle, 8 rows of 16 bytes contiguous, 128 bytes from one group of 8 to the next.
__device__ __forceinline__ uint64_t scale_desc(uint32_t saddr)
{
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)(128 >> 4) << 32) | (1ull << 46);
}

struct Plan {
    int32_t tile_n;    // tokens of a full tile
    int32_t tiles_m;   // tiles of weight rows
    int32_t num_kb;    // stages of a tile
    int32_t k_blocks;  // blocks of 32 along K
    int32_t atoms;     // atoms of scales along K
    int32_t w_row_blocks;  // row blocks of scales of one expert's weights
};

// A tile: expert, its first token (in the expert and as a row of X and Y), how many tokens it has, its first feature.
struct Tile {
    int32_t expert, first, row, count, feature;
    __device__ __forceinline__ int width() const { return (count + 15) & ~15; }
};
// Walks the tiles that a CTA takes, in rising order; tiles of an expert are ordered features first.
struct TileWalk {
    int32_t expert = 0, base = 0, next_base = 0;
    __device__ __forceinline__ bool find(int32_t t, const ExpertTable &table, int E, const Plan &p, Tile &out)
    {
        while (true) {
            if (expert >= E) return false;
            const int32_t count = table.start[expert + 1] - table.start[expert];
            const int32_t tiles = (count + p.tile_n - 1) / p.tile_n * p.tiles_m;
            if (t < base + tiles) {
                const int32_t local = t - base, n = local / p.tiles_m;
                out.expert = expert;
                out.first = n * p.tile_n;
                out.row = table.start[expert] + out.first;
                out.count = min(p.tile_n, count - out.first);
                out.feature = (local - n * p.tiles_m) * kTileM;
                return true;
            }
            base += tiles;
            ++expert;
        }
    }
};

template <int BN, int EW, typename T>
__global__ void __launch_bounds__(96 + 32 * EW, 1)
mx4_gemm_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
                const __grid_constant__ CUtensorMap map_x32, Mx4GemmArgs a, Plan plan)
{
    using C = Cfg<BN, EW>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *smem_a = smem;
    uint8_t *smem_b = smem_a + C::kStages * C::kABytes;
    uint8_t *smem_sa = smem_b + C::kStages * C::kBBytes;
    uint8_t *smem_sb = smem_sa + C::kStages * C::kSaBytes;
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

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < C::kStages; ++s) {
            mbar_init(smem_u32(full_bar + s), 2);  // both producers, with their byte counts
            mbar_init(smem_u32(empty_bar + s), 1);
        }
        for (int s = 0; s < kAccStages; ++s) {
            mbar_init(smem_u32(tmem_full_bar + s), 1);
            mbar_init(smem_u32(tmem_empty_bar + s), EW);
        }
        mbar_init(smem_u32(drain_bar), 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc(smem_u32(tmem_slot), C::kTmemCols);
    // Offsets and weights are there already when the kernel before this one is the quantise pass of the same call; else that
    // kernel may have written them.
    if (!a.weights_early) grid_dependency_wait();
    if (warp == 2) {
        const bool bad = build_expert_table(table, a.offsets, a.E, (int32_t)a.M);
        if (bad && lane == 0 && blockIdx.x == 0 && a.status != nullptr) atomicOr(a.status, 1 << Q8_ERR_INDEX);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    grid_dependency_release_next(true);

    const int32_t first_tile = blockIdx.x, tile_step = gridDim.x;
    TileWalk walk;
    Tile tile;
    if (warp == 0 || warp == 2) {
        // ---------------- producers ----------------
        const bool weights = warp == 0;
        if (!weights) grid_dependency_wait();
        const uint32_t elected = elect_one();
        int s = 0;
        uint32_t phase = 0;
        int64_t issued = 0;
        bool ok = true;
        for (int32_t t = first_tile; ok && walk.find(t, table, a.E, plan, tile); t += tile_step) {
            const int64_t atom_row = (int64_t)plan.atoms * kAtomBytes;
            const int w_row = (int)((int64_t)tile.expert * a.N + tile.feature);
            const uint8_t *sa = a.Ws + ((int64_t)tile.expert * plan.w_row_blocks + tile.feature / kAtomRows) * atom_row;
            const uint8_t *sb = a.Xs + ((int64_t)table.block[tile.expert] + tile.first / kAtomRows) * atom_row;
            const bool two_blocks = tile.first % kAtomRows + tile.width() > kAtomRows;
            const bool whole = tile.width() > BN - kBoxRows;
            const int boxes = (tile.width() + kBoxRows - 1) / kBoxRows;
            for (int kb = 0; kb < plan.num_kb; ++kb) {
                ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(empty_bar + s), phase ^ 1u, abort_flag, a.status));
                if (!ok) break;
                const uint32_t fb = smem_u32(full_bar + s);
                const uint32_t scale_bytes = (uint32_t)min(2, plan.atoms - 2 * kb) * kAtomBytes;
                if (weights) {
                    mbar_expect_tx_elected(elected, fb, C::kABytes + scale_bytes);
                    tma_load_2d_elected(elected, smem_u32(smem_a + s * C::kABytes), &map_w, kb * kStageRowBytes, w_row, fb);
                    bulk_load_elected(elected, smem_u32(smem_sa + s * C::kSaBytes), sa + kb * 2 * kAtomBytes, scale_bytes, fb);
                } else {
                    const uint32_t dst = smem_u32(smem_b + s * C::kBBytes), dst_s = smem_u32(smem_sb + s * C::kSbBytes);
                    mbar_expect_tx_elected(elected, fb, (uint32_t)(whole ? C::kBBytes : boxes * kBoxRows * kStageRowBytes) +
                                                            scale_bytes * (two_blocks ? 2 : 1));
                    if (whole) {
                        tma_load_2d_elected(elected, dst, &map_x, kb * kStageRowBytes, tile.row, fb);
                    } else {
                        for (int i = 0; i < boxes; ++i)
                            tma_load_2d_elected(elected, dst + i * kBoxRows * kStageRowBytes, &map_x32, kb * kStageRowBytes, tile.row + i * kBoxRows, fb);
                    }
                    bulk_load_elected(elected, dst_s, sb + kb * 2 * kAtomBytes, scale_bytes, fb);
                    if (two_blocks) bulk_load_elected(elected, dst_s + 2 * kAtomBytes, sb + atom_row + kb * 2 * kAtomBytes, scale_bytes, fb);
                }
                ++issued;
                if (++s == C::kStages) { s = 0; phase ^= 1u; }
            }
        }
        if (!ok) {
            // Aborting: this warp's copies land before the CTA gives up its shared memory (bounded: the other producer may have stopped
            // a stage earlier, and its barrier then never completes).
            const uint64_t t0 = global_timer_ns();
            for (int64_t i = 1; i <= (issued < C::kStages ? issued : C::kStages); ++i) {
                const int64_t k = issued - i;
                while (!mbar_try_wait(smem_u32(full_bar + k % C::kStages), (uint32_t)(k / C::kStages) & 1u) && global_timer_ns() - t0 < 50000000ull) {}
            }
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer ----------------
        const uint32_t elected = elect_one();
        auto uniform = [&](bool mine) { return (bool)__all_sync(0xffffffffu, mine); };
        int s = 0, as = 0;
        uint32_t phase = 0, aphase = 0;
        uint32_t scale_buffer = 0;
        bool ok = true;
        for (int32_t t = first_tile; ok && walk.find(t, table, a.E, plan, tile); t += tile_step) {
            ok = uniform(mbar_wait(smem_u32(tmem_empty_bar + as), aphase ^ 1u, abort_flag, a.status));
            if (!ok) break;
            tc_fence_after();
            const uint32_t tmem_d = tmem_base + (uint32_t)(as * BN);
            const uint32_t idesc = kInstrDesc | ((uint32_t)(tile.width() >> 3) << 17);
            const int sub = tile.first % kAtomRows;  // a multiple of 32
            const bool two_blocks = sub + tile.width() > kAtomRows;
            for (int kb = 0; kb < plan.num_kb; ++kb) {
                ok = uniform(mbar_wait(smem_u32(full_bar + s), phase, abort_flag, a.status));
                if (!ok) break;
                tc_fence_after();
                const uint64_t da = smem_desc_sw128(smem_u32(smem_a + s * C::kABytes));
                const uint64_t db = smem_desc_sw128(smem_u32(smem_b + s * C::kBBytes));
                const uint64_t dsa = scale_desc(smem_u32(smem_sa + s * C::kSaBytes)), dsb = scale_desc(smem_u32(smem_sb + s * C::kSbBytes));
                // scales of this stage: per atom 4 columns for the weights, 8 for the tokens; the two buffers take turns
                const uint32_t sa_col = tmem_base + (uint32_t)(C::kScaleCol0) + scale_buffer, sb_col = sa_col + 8;
                scale_buffer = scale_buffer == 0 ? kScaleCols : 0;
                const int blocks = min(kStageK / kBlock, plan.k_blocks - kb * (kStageK / kBlock));
#pragma unroll
                for (int atom = 0; atom < 2; ++atom) {
                    if (4 * atom >= blocks) break;
                    copy_scales_elected(elected, sa_col + 4 * atom, dsa + (uint64_t)(atom * (kAtomBytes >> 4)));
                    copy_scales_elected(elected, sb_col + 8 * atom, dsb + (uint64_t)(atom * (kAtomBytes >> 4)));
                    if (two_blocks) copy_scales_elected(elected, sb_col + 8 * atom + 4, dsb + (uint64_t)((2 + atom) * (kAtomBytes >> 4)));
                }
#pragma unroll
                for (int k = 0; k < kStageK / kMmaK; ++k) {
                    if (2 * k >= blocks) break;
                    const uint32_t half = (uint32_t)(k & 1) * 2;  // blocks 0 and 1 or 2 and 3 of the atom
                    mma_mxf4_elected(elected, tmem_d, da + (uint64_t)(2 * k), db + (uint64_t)(2 * k), idesc | (half << 4) | (half << 29),
                                     sa_col + 4 * (k >> 1), sb_col + 8 * (k >> 1) + (uint32_t)(sub >> 5), (uint32_t)((kb | k) != 0));
                }
                umma_commit_elected(elected, smem_u32(empty_bar + s));
                if (++s == C::kStages) { s = 0; phase ^= 1u; }
            }
            if (!ok) break;
            umma_commit_elected(elected, smem_u32(tmem_full_bar + as));
            if (++as == kAccStages) { as = 0; aphase ^= 1u; }
        }
        if (!ok) {
            // Aborting: wait (bounded) for the tensor core to finish what was issued.
            umma_commit_elected(elected, smem_u32(drain_bar));
            const uint64_t t0 = global_timer_ns();
            while (!mbar_try_wait(smem_u32(drain_bar), 0) && global_timer_ns() - t0 < 50000000ull) {}
        }
    } else {
        // ---------------- epilogue ----------------
        const int ew = warp - 3;
        const int quarter = warp & 3;  // TMEM lanes 32 * quarter .. + 31
        constexpr int kGroups = EW / 4;  // warps that share a quarter take every kGroups-th run of 32 columns
        const int group = ew >> 2;
        int as = 0;
        uint32_t aphase = 0;
        grid_dependency_wait();  // before anything is written: an earlier kernel may still read Y
        for (int32_t t = first_tile; walk.find(t, table, a.E, plan, tile); t += tile_step) {
            const int feature = tile.feature + quarter * 32 + lane;
            const bool mine = feature < a.N;
            const float bias = mine && a.bias != nullptr ? __ldg(a.bias + (int64_t)tile.expert * a.N + feature) : 0.0f;
            const bool ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(tmem_full_bar + as), aphase, abort_flag, a.status));
            if (!ok) break;
            tc_fence_after();
            T *y = reinterpret_cast<T *>(a.Y) + (int64_t)tile.row * a.ldy + feature;
            const uint32_t acc = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(as * BN);
            for (int col = group * 32; col < tile.count; col += 32 * kGroups) {
                uint32_t v[32];
                tmem_ld_32x32(acc + (uint32_t)col, v);
                tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < 32; j += 2) {
                    float y0 = __uint_as_float(v[j]) + bias, y1 = __uint_as_float(v[j + 1]) + bias;
                    if (a.act == Q8_ACT_GELU) gelu_fast_x2(pack_f32x2(y0, y1), y0, y1);
                    if (mine && col + j < tile.count) y[(int64_t)(col + j) * a.ldy] = from_float<T>(y0);
                    if (mine && col + j + 1 < tile.count) y[(int64_t)(col + j + 1) * a.ldy] = from_float<T>(y1);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(tmem_empty_bar + as));
            if (++as == kAccStages) { as = 0; aphase ^= 1u; }
        }
    }

    // ---------------- teardown (reached by every thread, also when aborting) ----------------
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc(tmem_base, C::kTmemCols);
    }
}

// ------------------------------------------------------------------ host side
// Codes [rows, pitch bytes] in boxes of 128 bytes x box_rows, 128-byte swizzle; what lies outside reads as zero.
bool codes_map(CUtensorMap *map, const uint8_t *base, int64_t rows, int64_t pitch, int box_rows)
{
    const auto fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)pitch, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)pitch};
    const cuuint32_t box[2] = {kStageRowBytes, (cuuint32_t)box_rows}, estr[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int BN, int EW, typename T>
cudaError_t launch_typed(const Mx4GemmArgs &a, const Plan &plan, int64_t tiles, cudaStream_t s)
{
    using C = Cfg<BN, EW>;
    auto kernel = mx4_gemm_kernel<BN, EW, T>;
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
    const int64_t pitch = code_pitch(a.K);
    CUtensorMap mw, mx, mx32;
    if (!codes_map(&mw, a.Wq, (int64_t)a.E * a.N, pitch, kTileM) || !codes_map(&mx, a.Xq, a.M, pitch, BN) || !codes_map(&mx32, a.Xq, a.M, pitch, kBoxRows))
        return cudaErrorInvalidValue;
    const int sms = sm_count();
    const int grid = (int)(tiles < sms ? tiles : sms);
    LaunchInfo &li = last_launch_info();
    li.gemm_kernel = 1;
    li.block_n = plan.tile_n;
    li.ctas = 1;
    li.grid = grid;
    li.launches += 1;
    return launch_overlapping_tail(kernel, dim3(grid), dim3(C::kThreads), C::kSmemBytes, s, mw, mx, mx32, a, plan);
}

template <int BN, int EW>
cudaError_t launch_shape(const Mx4GemmArgs &a, const Plan &plan, int64_t tiles, cudaStream_t s)
{
    switch (a.y_dtype) {
        case Q8_F32: return launch_typed<BN, EW, float>(a, plan, tiles, s);
        case Q8_F16: return launch_typed<BN, EW, __half>(a, plan, tiles, s);
        default: return launch_typed<BN, EW, __nv_bfloat16>(a, plan, tiles, s);
    }
}

}  // namespace

cudaError_t launch_mx4_gemm(const Mx4GemmArgs &a, cudaStream_t s)
{
    Plan p;
    p.tiles_m = (int32_t)ceil_div(a.N, kTileM);
    p.num_kb = (int32_t)ceil_div(a.K, kStageK);
    p.k_blocks = (int32_t)ceil_div(a.K, kBlock);
    p.atoms = (int32_t)scale_atoms(a.K);
    p.w_row_blocks = (int32_t)ceil_div(a.N, kAtomRows);
    const int64_t hit = a.E < a.M ? a.E : a.M;        // experts with tokens, at most
    const int64_t mean = ceil_div(a.M, a.E);
    const int sms = sm_count();
    // widest tile that still gives every SM one
    p.tile_n = 192;
    for (int n : {128, 64})
        if (mean <= n || (a.E == 1 && ceil_div(a.M, p.tile_n) * p.tiles_m < sms)) p.tile_n = n;
    const int64_t tiles = (ceil_div(a.M, p.tile_n) + (a.E > 1 ? hit : 0)) * p.tiles_m;  // at most
    if (tiles > 0x7fffffff) return cudaErrorInvalidValue;
    return p.tile_n == 64 ? launch_shape<64, 8>(a, p, tiles, s) : p.tile_n == 128 ? launch_shape<128, 8>(a, p, tiles, s) : launch_shape<192, 8>(a, p, tiles, s);
}

}  // namespace q8
