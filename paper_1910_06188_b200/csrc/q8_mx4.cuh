// Microscaled 4-bit floating point (MXFP4): the format, its layout in memory and the work lists of the expert-grouped product.
//
// A block of 32 neighbouring values x of a row shares the scale s = 2^(E - 127), E = max(exponent field of max|x| - 2, 0), so
// that the largest value lies in [4, 8) s; each value is held as the E2M1 number nearest to x / s (0, 0.5, 1, 1.5, 2, 3, 4, 6
// and their negatives; ties to the even mantissa, 6 from there on).  x / s is a product with a power of two and exact wherever
// the rounding depends on it, so the codes are the same whichever way they are computed.
//
// Layout of [rows, K]:
//   codes   row-major, two to a byte (the lower index in the lower half), rows of 16 ceil(K / 32) bytes: whole blocks, 16-byte
//           pitch; codes behind column K are 0
//   scales  the order in which the tensor cores take them: atoms of 128 rows x 128 columns (4 blocks), 512 bytes each, atoms of
//           a row of atoms one after the other; in an atom row r, block b is byte 16 (r % 32) + 4 (r / 32) + b.  Bytes of blocks
//           behind the last one are 0; those of rows behind the last one are of no account.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "q8_internal.cuh"

namespace q8 {
namespace mx4 {

constexpr int kBlock = 32;         // values that share a scale
constexpr int kAtomRows = 128;     // rows, and
constexpr int kAtomK = 128;        // columns of an atom of scales
constexpr int kAtomBytes = 512;
constexpr int kMaxExperts = 1024;

__host__ __device__ inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
__host__ __device__ inline int64_t code_pitch(int64_t K) { return 16 * ceil_div(K, kBlock); }
__host__ __device__ inline int64_t scale_atoms(int64_t K) { return ceil_div(K, kAtomK); }
// Row blocks of scales that T slots of E experts can need: every expert starts a block of its own.
inline int64_t most_row_blocks(int64_t T, int64_t E) { return T / kAtomRows + (E < T ? E : T); }

// ---- experts
// The slots [start[e], start[e + 1]) of each expert and the first of its row blocks of scales, in shared memory.
struct ExpertTable {
    int32_t *start;  // E + 1
    int32_t *block;  // E + 1
};
// Written by one warp.  Offsets outside [0, T] or below an earlier one (a caller's mistake) are moved to the nearest allowed value, so that
// every slot belongs to one expert at most and no access leaves the tensors; returns whether there were any.  A lane takes
// neighbouring experts, so the 32 runs need one scan.  offsets == nullptr: one expert with all T slots.
__device__ __forceinline__ bool build_expert_table(const ExpertTable &t, const int32_t *offsets, int E, int32_t T)
{
    const int lane = threadIdx.x & 31;
    if (offsets == nullptr) {
        if (lane == 0) {
            t.start[0] = 0;
            t.start[1] = T;
            t.block[0] = 0;
            t.block[1] = (T + kAtomRows - 1) / kAtomRows;
        }
        __syncwarp();
        return false;
    }
    const int run = (E + 32) / 32;  // ceil((E + 1) / 32)
    const int lo = min(lane * run, E + 1), hi = min(lo + run, E + 1);
    int32_t top = 0;
    bool bad = false;
    for (int i = lo; i < hi; ++i) {
        const int32_t v = __ldg(offsets + i);
        bad |= v < 0 || v > T || v < top;
        top = max(top, min(max(v, 0), T));
        t.start[i] = top;
    }
    int32_t before = top;  // maximum over this and all lower lanes
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int32_t o = __shfl_up_sync(0xffffffffu, before, d);
        if (lane >= d) before = max(before, o);
    }
    before = __shfl_up_sync(0xffffffffu, before, 1);
    if (lane == 0) before = 0;
    for (int i = lo; i < hi; ++i) {
        bad |= t.start[i] < before;
        t.start[i] = max(t.start[i], before);
    }
    __syncwarp();
    int32_t sum = 0;
    for (int i = lo; i < min(hi, E); ++i) sum += (t.start[i + 1] - t.start[i] + kAtomRows - 1) / kAtomRows;
    int32_t at = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int32_t o = __shfl_up_sync(0xffffffffu, at, d);
        if (lane >= d) at += o;
    }
    at -= sum;
    for (int i = lo; i < hi; ++i) {
        t.block[i] = at;
        if (i < E) at += (t.start[i + 1] - t.start[i] + kAtomRows - 1) / kAtomRows;
    }
    bad = __any_sync(0xffffffffu, bad);
    __syncwarp();
    return bad;
}

// ---- values
template <typename T>
__device__ __forceinline__ float to_float(T v)
{
    if constexpr (sizeof(T) == 4) return v;
    else if constexpr (std::is_same<T, __half>::value) return __half2float(v);
    else return __bfloat162float(v);
}
template <typename T>
__device__ __forceinline__ T from_float(float v)
{
    if constexpr (sizeof(T) == 4) return v;
    else if constexpr (std::is_same<T, __half>::value) return __float2half_rn(v);
    else return __float2bfloat16_rn(v);
}

// Eight E2M1 codes, the first in the lowest four bits (nearest even, saturating; the conversion instruction of sm_100a).
__device__ __forceinline__ uint32_t pack_e2m1(const float (&v)[8])
{
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r)
        : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}
// The values of eight codes: a code's exponent and mantissa bits at their places in an fp32 number are that value times 2^-126
// (0.5 a subnormal).  (The conversion instruction back from E2M1 gave zeros where it followed pack_e2m1() in one kernel.)
__device__ __forceinline__ void unpack_e2m1(uint32_t codes, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t c = codes >> (4 * i);
        v[i] = __fmul_rn(__uint_as_float((c & 7) << 22 | (c & 8) << 28), __uint_as_float(253u << 23));
    }
}
// 2^(E - 127) and its inverse, E <= 252 (an exponent of 0 is the subnormal 2^-127).
__device__ __forceinline__ float scale_value(uint32_t E) { return __uint_as_float(E == 0 ? 0x00400000u : E << 23); }
__device__ __forceinline__ float inverse_scale(uint32_t E) { return __uint_as_float((254u - E) << 23); }

}  // namespace mx4

// ---- launchers (q8_mx4.cu, q8_mx4_gemm_sm100.cu); arguments are checked by the entry points
struct Mx4QuantizeArgs {
    const void *X;        // [groups, rows, K], rows ld values apart, groups rows * ld
    int64_t ld;
    int64_t groups, rows, K;
    uint8_t *codes, *scales;
    void *Xhat = nullptr;  // instead of codes and scales: the values, in X's type, rows ldo values apart
    int64_t ldo = 0;
    int32_t *status;
    // slots of experts: rows is the number of slots, groups 1
    const int32_t *offsets = nullptr;  // [E + 1]
    int E = 0;
    const int32_t *index = nullptr;  // row of X of each slot; none: the slot's own
    int64_t x_rows = 0;              // rows that X has
};
cudaError_t launch_mx4_quantize(const Mx4QuantizeArgs &a, int dtype, cudaStream_t s);
cudaError_t launch_mx4_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t groups, int64_t rows, int64_t K, void *Y,
                                  int dtype, int64_t ldy, cudaStream_t s);

struct Mx4GemmArgs {
    const uint8_t *Xq, *Xs;  // activation codes [M, K] and scales
    const uint8_t *Wq, *Ws;  // weights [E, N, K], scales of each expert in row blocks of its own
    const float *bias;       // [E, N] or nullptr
    void *Y;                 // [M, N], rows ldy values apart
    int64_t ldy;
    int y_dtype;
    int64_t M, N, K;
    int act;
    const int32_t *offsets = nullptr;  // [E + 1], or nullptr with E == 1
    int E = 1;
    int32_t *status;
    bool weights_early = false;  // the kernel before this one in the stream waited for all before it and writes neither weights nor offsets
};
cudaError_t launch_mx4_gemm(const Mx4GemmArgs &a, cudaStream_t s);

}  // namespace q8
