// Quantisation to microscaled 4-bit floating point, back, and both at once (training), streaming passes bound by HBM.
//
// A lane takes 8 neighbouring values of a row, so four lanes share a block: the exponent of its maximum is the largest of the lanes', two
// shuffles, the scale that exponent less 2, the codes four conversions of two values each.  A warp takes 256 columns of
// up to four rows, whose loads are all issued before the first is used.  For a plain matrix these are the rows r, r + 32,
// r + 64 and r + 96 that lie side by side in an atom of scales, whose scales leave as 16 bytes of four lanes.
//
// Measured: fp32 is bound by memory (49152 x 1024 into tiles 34.6 us, DRAM 77 %; 4096 x 1024 with the gradient's copy 12.5 us = 82 % of the copy rate), 16-bit
// values by instructions (8192 x 8192 bf16 30.9 us, ALU pipe 69 %, DRAM 56 %; in training 12288 x 4096 37 us = 5.4 TB/s).  Into tiles and
// back, 24576 x 1024 fp32: 39 us for two passes, 89 % of the copy rate.

#include "q8_mx4.cuh"

namespace q8 {

namespace {

using namespace mx4;

constexpr int kThreads = 128;
constexpr int kWarps = kThreads / 32;
constexpr int kChunk = kTileK;  // columns of a warp

enum Kind { kMatrix, kFake, kSlots1, kSlots4 };
template <int KIND>
constexpr int kRows = KIND == kSlots1 ? 1 : 4;

// The other way: columns k0 .. k0 + 7 of a row from every lane.  Unaligned, a lane stores the aligned 16 or 32 bytes that end with its first
// values and begin with the last ones of the lane before; the first and last lanes and those at the row's end store value by value.
template <typename T, bool ALIGNED>
__device__ __forceinline__ void store_columns(T *row, int32_t k0, int32_t K, int vec, const float (&v)[8])
{
    constexpr int N = kWords<T>;
    uint32_t w[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if constexpr (sizeof(T) == 4) {
            w[i] = __float_as_uint(v[i]);
        } else {
            const T h[2] = {from_float<T>(v[2 * i]), from_float<T>(v[2 * i + 1])};
            memcpy(&w[i], h, 4);
        }
    }
    if constexpr (ALIGNED) {
        T *p = row + k0;
        if (k0 + 8 > K || vec == 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (k0 + i < K) p[i] = from_float<T>(v[i]);
        } else if (sizeof(T) == 4 && vec >= 32) {
            asm volatile("st.global.cs.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                         ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[N - 4]), "r"(w[N - 3]), "r"(w[N - 2]), "r"(w[N - 1])
                         : "memory");
        } else {
#pragma unroll
            for (int i = 0; i < N / 4; ++i) __stcs(reinterpret_cast<uint4 *>(p) + i, make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]));
        }
    } else {
        const int lane = threadIdx.x & 31;
        const uint32_t off = (uint32_t)reinterpret_cast<uintptr_t>(row) & 15u, shift = 16u - off;  // bytes
        uint32_t z[N + 5];
#pragma unroll
        for (int i = 0; i < 4; ++i) z[i] = __shfl_up_sync(0xffffffffu, w[N - 4 + i], 1);
#pragma unroll
        for (int i = 0; i < N; ++i) z[4 + i] = w[i];
        z[N + 4] = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = shift & 16 ? z[i + 4] : z[i];
#pragma unroll
        for (int i = N; i < N + 4; ++i) z[i] = shift & 16 ? 0u : z[i];
#pragma unroll
        for (int i = 0; i < N + 2; ++i) z[i] = shift & 8 ? z[i + 2] : z[i];
#pragma unroll
        for (int i = 0; i < N + 1; ++i) z[i] = shift & 4 ? z[i + 1] : z[i];
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < N; ++i) z[i] = __funnelshift_r(z[i], z[i + 1], (shift & 2) * 8);
        }
        const int32_t before = (int32_t)(off / sizeof(T)), first = k0 - before;
        if ((lane > 0 || off == 0) && first + 8 <= K) {
#pragma unroll
            for (int i = 0; i < N / 4; ++i) __stcs(reinterpret_cast<uint4 *>(row + first) + i, make_uint4(z[4 * i], z[4 * i + 1], z[4 * i + 2], z[4 * i + 3]));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                T one;
                const uint32_t bits = sizeof(T) == 4 ? z[i % N] : z[i / 2] >> (16 * (i & 1));
                memcpy(&one, &bits, sizeof(T));
                if (first + i < K && (lane > 0 || first + i >= k0)) row[first + i] = one;
            }
        }
        if (lane == 31) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i >= 8 - before && k0 + i < K) row[k0 + i] = from_float<T>(v[i]);
        }
    }
}

template <typename T, bool ALIGNED, int R>
__device__ __forceinline__ void settle_rows(Columns<T, ALIGNED> (&v)[R], uint32_t (&words)[R][kWords<T>])
{
#pragma unroll
    for (int j = 0; j < R; ++j) {
        v[j].settle();
#pragma unroll
        for (int i = 0; i < kWords<T>; ++i) words[j][i] = v[j].w[i];
    }
}

// (Rows and tasks are counted in 32 bits: with 64-bit divisions the indices took as many instructions as the arithmetic.)
template <typename T, int KIND, bool ALIGNED>
__global__ void __launch_bounds__(kThreads) mx4_quantize_kernel(Mx4QuantizeArgs a, uint32_t tasks, uint32_t chunks, uint32_t splits, uint32_t row_lanes, int vec, int vec_out)
{
    constexpr int R = kRows<KIND>;
    constexpr bool kSlots = KIND == kSlots1 || KIND == kSlots4;
    constexpr int kRowStep = KIND == kMatrix ? 32 : 1;
    __shared__ int32_t table_words[kSlots ? 2 * (kMaxExperts + 1) : 1];
    // The product behind slots reads offsets and weights at once, so it starts when everything before this kernel has ended; the one behind a
    // matrix reads nothing before this kernel's end and may be set up as early as can be (16 x 4096 -> 1024 9.1 -> 8.7 us, 64 rows 8.2 -> 7.8).
    if (!kSlots) grid_dependency_release_next(true);
    grid_dependency_wait();
    if (kSlots) grid_dependency_release_next(true);
    const int lane = threadIdx.x & 31;
    const uint32_t task = blockIdx.x * kWarps + (threadIdx.x >> 5);
    ExpertTable table{table_words, table_words + kMaxExperts + 1, nullptr};
    bool bad_index = false;
    if (kSlots) {
        if (threadIdx.x < 32) bad_index = build_expert_table(table, a.offsets, a.E, (int32_t)a.rows, 1, 1);
        __syncthreads();
    }
    if (task >= tasks) return;
    const uint32_t line = task / splits, part = task - line * splits;  // a part of the tiles of a row: one, or every splits-th
    const int32_t rows = (int32_t)a.rows;
    bool odd = false;
    if constexpr (kSlots) {
        // R slots in a row; what a slot's index and expert say is worked out once for all of its tiles.
        const int32_t first = (int32_t)line * R;
        int expert = 0, hi = a.E;  // the expert that owns the first slot: the last one that starts at or before it
        while (expert < hi) {
            const int mid = (expert + hi) >> 1;
            if (table.start[mid + 1] <= first) expert = mid + 1;
            else hi = mid;
        }
        const T *x[R];
        uint8_t *to[R];
        bool there[R];
        uint32_t r[R];
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int32_t slot = first + j;
            int64_t from = slot;
            if (a.index != nullptr && slot < rows) from = __ldcg(a.index + slot);
            while (expert < a.E && table.start[expert + 1] <= slot) ++expert;
            const bool owned = slot < rows && expert < a.E && slot >= table.start[expert];
            there[j] = owned && from >= 0 && from < a.x_rows;  // else it counts as a row of zeros
            bad_index |= owned && !there[j];
            x[j] = reinterpret_cast<const T *>(a.X) + (there[j] ? from : 0) * a.ld;
            const uint32_t in_expert = owned ? (uint32_t)(slot - table.start[expert]) : 0u;
            r[j] = in_expert % kTileRows;
            to[j] = owned ? a.out + (int64_t)(table.block[expert] + in_expert / kTileRows) * chunks * kTileBytes : nullptr;
        }
        Columns<T, ALIGNED> v[R], next[R];
        auto load = [&](uint32_t chunk, Columns<T, ALIGNED> (&w)[R]) {
#pragma unroll
            for (int j = 0; j < R; ++j) w[j].load(x[j], (int32_t)chunk * kChunk + lane * 8, (int32_t)a.K, there[j], vec);
        };
        // where this lane's scales go: those of one row for each (lane / 4) % 4, or of the only one
        const int mine = R == 1 ? 0 : (lane >> 2) & 3;
        uint8_t *scales_to = to[0];
        int scales_row = (int)r[0];
#pragma unroll
        for (int j = 1; j < R; ++j) {
            scales_to = mine == j ? to[j] : scales_to;
            scales_row = mine == j ? (int)r[j] : scales_row;
        }
        if ((lane & (R == 1 ? 15 : 3)) != 0) scales_to = nullptr;
        load(part, v);
        for (uint32_t chunk = part; chunk < chunks; chunk += splits) {
            if (chunk + splits < chunks) load(chunk + splits, next);
            uint32_t words[R][kWords<T>], codes[R];
            settle_rows(v, words);
            const uint32_t e = quantize_rows<T, R>(words, codes, odd);
            uint32_t scales;
            if constexpr (R == 1) {
                scales = e << (8 * ((lane >> 2) & 3));
                scales |= __shfl_xor_sync(0xffffffffu, scales, 4);
                scales |= __shfl_xor_sync(0xffffffffu, scales, 8);
            } else {
                scales = scale_words(e, lane);
            }
            const int64_t at = (int64_t)chunk * kTileBytes;
#pragma unroll
            for (int j = 0; j < R; ++j)
                if (to[j] != nullptr) *reinterpret_cast<uint32_t *>(to[j] + at + code_place((int)r[j], lane)) = codes[j];
            if (scales_to != nullptr) *reinterpret_cast<uint32_t *>(scales_to + at + scale_place(scales_row, (lane >> 4) * 4)) = scales;
#pragma unroll
            for (int j = 0; j < R; ++j) v[j] = next[j];
        }
    } else {
        int32_t first, end = rows;
        uint8_t *tile = nullptr;
        uint32_t r0 = 0;
        if (KIND == kMatrix) {  // the row r0 of a block of 128, r0 < row_lanes, and those 32, 64 and 96 further
            const uint32_t block = line / row_lanes;
            r0 = line - block * row_lanes;
            uint32_t in_group = block;
            first = 0;
            if (a.groups > 1) {
                const uint32_t blocks = (uint32_t)(rows + kTileRows - 1) / kTileRows, group = block / blocks;
                in_group = block - group * blocks;
                first = (int32_t)group * rows;
                end = first + rows;
            }
            first += (int32_t)(in_group * kTileRows + r0);
            tile = a.out + ((int64_t)block * chunks + part) * kTileBytes;
        } else {
            first = (int32_t)line * R;
        }
        const int32_t k0 = (int32_t)part * kChunk + lane * 8;
        Columns<T, ALIGNED> v[R];
        const T *x = reinterpret_cast<const T *>(a.X) + first * a.ld;
#pragma unroll
        for (int j = 0; j < R; ++j, x += kRowStep * a.ld) v[j].load(x, k0, (int32_t)a.K, first + j * kRowStep < end, vec);
        uint32_t words[R][kWords<T>], codes[R];
        settle_rows(v, words);
        const uint32_t e = quantize_rows<T, R>(words, codes, odd);
        if constexpr (KIND == kFake) {
#pragma unroll
            for (int j = 0; j < R; ++j) {
                float back[8];
                unpack_e2m1(codes[j], back);
                const float s = scale_value(e >> (8 * j) & 0xffu);
#pragma unroll
                for (int i = 0; i < 8; ++i) back[i] = __fmul_rn(back[i], s);
                const int32_t row = first + j;
                if (row < end) store_columns<T, ALIGNED>(reinterpret_cast<T *>(a.Xhat) + row * a.ldo, k0, (int32_t)a.K, vec_out, back);
            }
        } else {
            const uint32_t scales = scale_words(e, lane);
#pragma unroll
            for (int j = 0; j < R; ++j)
                if (first + 32 * j < end) *reinterpret_cast<uint32_t *>(tile + code_place((int)r0, lane) + 32 * 128 * j) = codes[j];
            if ((lane & 3) == 0) *reinterpret_cast<uint32_t *>(tile + scale_place((int)r0, (lane >> 4) * 4) + (lane & 12)) = scales;
        }
    }
    if (a.status != nullptr && lane == 0) {  // (the whole warp has the same)
        const uint32_t flags = (odd ? 1u << Q8_ERR_SCALE : 0u) | (bad_index ? 1u << Q8_ERR_INDEX : 0u);
        if (flags != 0) atomicOr(a.status, (int32_t)flags);
    }
}

template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(kThreads)
mx4_dequantize_kernel(const uint8_t *tiles, uint32_t groups, uint32_t rows, int32_t K, T *Y, int64_t ldy, uint32_t tasks, uint32_t chunks, int vec)
{
    grid_dependency_wait();
    const int lane = threadIdx.x & 31;
    const uint32_t task = blockIdx.x * kWarps + (threadIdx.x >> 5);
    if (task >= tasks) return;
    const uint32_t line = task / chunks, chunk = task - line * chunks, first = line * 4, all = groups * rows;
    const int32_t k0 = (int32_t)chunk * kChunk + lane * 8;
    const uint32_t blocks = (rows + kTileRows - 1) / kTileRows;
    uint32_t c[4], E[4];
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) {
        const uint32_t row = min(first + j, all - 1), group = groups > 1 ? row / rows : 0, r = row - group * rows;
        const uint8_t *tile = tiles + ((int64_t)(group * blocks + r / kTileRows) * chunks + chunk) * kTileBytes;
        // (not as read-only data: a kernel that writes them may end after this one has started)
        c[j] = __ldcg(reinterpret_cast<const uint32_t *>(tile + code_place((int)(r % kTileRows), lane)));
        E[j] = __ldcg(tile + scale_place((int)(r % kTileRows), lane >> 2));
    }
    T *y = Y + first * ldy;
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j, y += ldy) {
        if (first + j >= all) break;
        float v[8];
        unpack_e2m1(c[j], v);
        const float s = E[j] == 255 ? __uint_as_float(0x7fc00000u) : scale_value(E[j]);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __fmul_rn(v[i], s);
        store_columns<T, ALIGNED>(y, k0, K, vec, v);
    }
}

cudaError_t grid_of(int64_t tasks, dim3 *grid)
{
    if (tasks > 0x7fffffff) return cudaErrorInvalidConfiguration;  // more than 2^41 values
    *grid = dim3((unsigned)ceil_div(tasks, kWarps));
    return cudaSuccess;
}

bool worth_shifting(int64_t rows, int64_t K) { return K >= 256 && rows * K >= (1 << 20); }

template <typename T, int KIND>
cudaError_t launch_kind(const Mx4QuantizeArgs &a, cudaStream_t s)
{
    const int64_t chunks = ceil_div(a.K, kChunk), row_lanes = a.rows < 32 ? a.rows : 32;
    const int64_t lines = KIND == kMatrix ? a.groups * ceil_div(a.rows, kTileRows) * row_lanes : ceil_div(a.rows, kRows<KIND>);
    int64_t splits = chunks;
    if (KIND == kSlots4) {  // as many warps as the device holds, a warp as many tiles of its rows as that leaves
        const int64_t room = 24 * sm_count() / lines;
        splits = room < 1 ? 1 : room < chunks ? room : chunks;
    }
    dim3 grid;
    cudaError_t e = grid_of(lines * splits, &grid);
    if (e != cudaSuccess) return e;
    const int vec = value_alignment(a.X, a.ld, sizeof(T)), vec_out = value_alignment(a.Xhat, a.ldo, sizeof(T));
    auto kernel = KIND == kSlots1 || KIND == kSlots4 || (vec > 0 && vec_out > 0) || !worth_shifting(a.groups * a.rows, a.K) ? mx4_quantize_kernel<T, KIND, true>
                                                                                                                     : mx4_quantize_kernel<T, KIND, false>;
    return launch_overlapping_tail(kernel, grid, dim3(kThreads), 0, s, a, lines * splits, chunks, splits, row_lanes, vec, vec_out);
}

template <typename T>
cudaError_t launch_type(const Mx4QuantizeArgs &a, cudaStream_t s)
{
    if (a.Xhat != nullptr) return launch_kind<T, kFake>(a, s);
    if (a.offsets == nullptr) return launch_kind<T, kMatrix>(a, s);
    // one row to a warp while that leaves room for every warp at once
    return a.rows * ceil_div(a.K, kChunk) <= 16 * sm_count() ? launch_kind<T, kSlots1>(a, s) : launch_kind<T, kSlots4>(a, s);
}

template <typename T>
cudaError_t launch_back(T *Y, int64_t ldy, dim3 grid, cudaStream_t s, const uint8_t *tiles, int64_t groups, int64_t rows, int64_t K, int64_t tasks, int64_t chunks)
{
    const int vec = value_alignment(Y, ldy, sizeof(T));
    auto kernel = vec > 0 || !worth_shifting(groups * rows, K) ? mx4_dequantize_kernel<T, true> : mx4_dequantize_kernel<T, false>;
    return launch_overlapping_tail(kernel, grid, dim3(kThreads), 0, s, tiles, groups, rows, K, Y, ldy, tasks, chunks, vec);
}

}  // namespace

cudaError_t launch_mx4_quantize(const Mx4QuantizeArgs &a, int dtype, cudaStream_t s)
{
    last_launch_info().launches += 1;
    switch (dtype) {
        case Q8_F32: return launch_type<float>(a, s);
        case Q8_F16: return launch_type<__half>(a, s);
        default: return launch_type<__nv_bfloat16>(a, s);
    }
}

cudaError_t launch_mx4_dequantize(const uint8_t *tiles, int64_t groups, int64_t rows, int64_t K, void *Y, int dtype, int64_t ldy, cudaStream_t s)
{
    last_launch_info().launches += 1;
    const int64_t chunks = ceil_div(K, kChunk), tasks = ceil_div(groups * rows, 4) * chunks;
    dim3 grid;
    cudaError_t e = grid_of(tasks, &grid);
    if (e != cudaSuccess) return e;
    switch (dtype) {
        case Q8_F32: return launch_back(static_cast<float *>(Y), ldy, grid, s, tiles, groups, rows, K, tasks, chunks);
        case Q8_F16: return launch_back(static_cast<__half *>(Y), ldy, grid, s, tiles, groups, rows, K, tasks, chunks);
        default: return launch_back(static_cast<__nv_bfloat16 *>(Y), ldy, grid, s, tiles, groups, rows, K, tasks, chunks);
    }
}

}  // namespace q8
