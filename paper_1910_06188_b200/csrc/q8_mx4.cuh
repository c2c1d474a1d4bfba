// Microscaled 4-bit floating point (MXFP4): the format, its layout in memory and the work lists of the expert-grouped product.
//
// A block of 32 neighbouring values x of a row shares the scale s = 2^(E - 127), E = max(exponent field of max|x| - 2, 0), so
// that the largest value lies in [4, 8) s; each value is held as the E2M1 number nearest to x / s (0, 0.5, 1, 1.5, 2, 3, 4, 6
// and their negatives; ties to the even mantissa, 6 from there on).  x / s is a product with a power of two and exact wherever
// the rounding depends on it, so the codes are the same whichever way they are computed.
//
// Layout of [rows, K]: tiles of 128 rows x 256 columns, the tiles of a row of tiles one after the other, each as the tensor
// cores take it from shared memory, so that a tile is one contiguous copy:
//   16384 bytes of codes   row r at 128 r, in eight pieces of 16 bytes (32 codes, one block); piece p stands at place p ^ (r % 8); two
//                          codes to a byte, the lower column in the lower half; codes behind column K are 0
//   1024 bytes of scales   two atoms of 128 rows x 4 blocks: row r, block b of the atom is byte 16 (r % 32) + 4 (r / 32) + b;
//                          scales of blocks behind the last one are 0
// What rows behind the last one hold is of no account.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "q8_internal.cuh"
#include "q8_sm100_ptx.cuh"

namespace q8 {
namespace mx4 {

constexpr int kBlock = 32;       // values that share a scale
constexpr int kTileRows = 128;   // rows, and
constexpr int kTileK = 256;      // columns of a tile
constexpr int kAtomBytes = 512;  // scales of 128 rows x 128 columns
constexpr int kCodeBytes = kTileRows * kTileK / 2;
constexpr int kTileBytes = kCodeBytes + 2 * kAtomBytes;
constexpr int kMaxExperts = 1024;

__host__ __device__ inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
__host__ __device__ inline int64_t tiles_along(int64_t K) { return ceil_div(K, kTileK); }
// Places in a tile: the 4 bytes with the codes of columns 8 i .. 8 i + 7, the scale of block b (0 .. 7), row r
__host__ __device__ inline int code_place(int r, int i) { return r * 128 + ((((i >> 2) ^ r) & 7) << 4) + ((i & 3) << 2); }
__host__ __device__ inline int scale_place(int r, int b) { return kCodeBytes + (b >> 2) * kAtomBytes + (r & 31) * 16 + (r >> 5) * 4 + (b & 3); }
// Row blocks that T slots of E experts can need: every expert starts a block of its own.
inline int64_t most_row_blocks(int64_t T, int64_t E) { return T / kTileRows + (E < T ? E : T); }

// ---- experts
// The slots [start[e], start[e + 1]) of each expert, the first of its row blocks and of its tiles, in shared memory.
struct ExpertTable {
    int32_t *start;  // E + 1
    int32_t *block;  // E + 1
    int32_t *tile;   // E + 1, or nullptr
};
__device__ __forceinline__ int32_t scan_sum(int32_t v, int lane)
{
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int32_t o = __shfl_up_sync(0xffffffffu, v, d);
        if (lane >= d) v += o;
    }
    return v;
}
// Written by one warp, a lane a run of neighbouring experts.  Offsets outside [0, T] or below an earlier one (a caller's mistake)
// are moved to the nearest allowed value, so that every slot belongs to one expert at most and no access leaves the tensors; returns
// whether there were any.  An expert has ceil(slots / tile_n) tiles_m tiles.
__device__ __forceinline__ bool build_expert_table(const ExpertTable &t, const int32_t *offsets, int E, int32_t T, int32_t tile_n, int32_t tiles_m)
{
    const int lane = threadIdx.x & 31;
    const int run = (E + 32) / 32, lo = min(lane * run, E + 1), hi = min(lo + run, E + 1);  // of E + 1 offsets
    for (int i = lane; i <= E; i += 32) t.start[i] = __ldcg(offsets + i);  // (from L2: the product reads them before its dependency wait)
    __syncwarp();
    bool bad = false;
    int32_t top = 0;
    for (int i = lo; i < hi; ++i) {
        const int32_t v = t.start[i];
        bad |= v < top || v > T;
        top = max(top, min(v, T));
        t.start[i] = top;
    }
    int32_t before = top;  // what the lanes before have at most
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int32_t o = __shfl_up_sync(0xffffffffu, before, d);
        if (lane >= d) before = max(before, o);
    }
    before = __shfl_up_sync(0xffffffffu, before, 1);
    if (lane == 0) before = 0;
    for (int i = lo; i < hi && t.start[i] < before; ++i) {
        bad = true;
        t.start[i] = before;
    }
    __syncwarp();
    int32_t blocks = 0, tiles = 0;
    for (int i = lo; i < min(hi, E); ++i) {
        const int32_t count = t.start[i + 1] - t.start[i];
        blocks += (count + kTileRows - 1) / kTileRows;
        if (t.tile != nullptr) tiles += (int32_t)((uint32_t)(count + tile_n - 1) / (uint32_t)tile_n) * tiles_m;
    }
    int32_t block = scan_sum(blocks, lane) - blocks, tile = t.tile != nullptr ? scan_sum(tiles, lane) - tiles : 0;
    for (int i = lo; i < hi; ++i) {
        t.block[i] = block;
        if (t.tile != nullptr) t.tile[i] = tile;
        const int32_t count = i < E ? t.start[i + 1] - t.start[i] : 0;
        block += (count + kTileRows - 1) / kTileRows;
        if (t.tile != nullptr) tile += (int32_t)((uint32_t)(count + tile_n - 1) / (uint32_t)tile_n) * tiles_m;
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
// 2^(E - 127) (an exponent of 0 is the subnormal 2^-127).
__device__ __forceinline__ float scale_value(uint32_t E) { return __uint_as_float(E == 0 ? 0x00400000u : E << 23); }

// Eight values as they lie in memory: four words of two, or eight words of one.
template <typename T>
constexpr int kWords = sizeof(T) == 4 ? 8 : 4;

// `count` values from p on, those outside [from, to) left out as 0, into words.
template <typename T, int WORDS>
__device__ __forceinline__ void load_single(const T *p, int from, int to, uint32_t *w)
{
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
        if constexpr (sizeof(T) == 4) {
            w[i] = i >= from && i < to ? reinterpret_cast<const uint32_t *>(p)[i] : 0u;
        } else {
            const uint16_t *h = reinterpret_cast<const uint16_t *>(p);
            const uint32_t lo = 2 * i >= from && 2 * i < to ? h[2 * i] : 0u, hi = 2 * i + 1 >= from && 2 * i + 1 < to ? h[2 * i + 1] : 0u;
            w[i] = lo | hi << 16;
        }
    }
}
__device__ __forceinline__ void load16(const void *p, uint32_t *w)
{
    const uint4 a = __ldcs(reinterpret_cast<const uint4 *>(p));
    w[0] = a.x;
    w[1] = a.y;
    w[2] = a.z;
    w[3] = a.w;
}

// What a lane of a warp that takes 256 columns of a row reads of its columns k0 .. k0 + 7 (k0 = 8 lane + a multiple of 256), columns at
// and behind K being 0.  ALIGNED: rows begin at multiples of 16 (vec) or 32 bytes.  Else a lane reads the aligned 16 or 32 bytes that its
// first value lies in, the last lane the 16 behind them too, and settle() moves the bytes to their places; what of that is not of the
// row is not read.  (Value by value, rows of 3532 bf16 took 6 times as long as rows of 3536.)  Few values, the slots of experts and tokens that the
// product quantises itself take ALIGNED at any address, value by value where vec is 0: the grouped layer on 16384 slots of 2048 bf16 97.8 us with
// rows 2048 apart, 116 to 120 with rows 2049 apart.
template <typename T, bool ALIGNED>
struct Columns {
    uint32_t w[kWords<T>], behind[ALIGNED ? 1 : 4];
    uint32_t shift;  // bytes

    __device__ __forceinline__ void load(const T *row, int32_t k0, int32_t K, bool there, int vec)
    {
        constexpr int kBytes = 8 * (int)sizeof(T);
        if (!there) K = 0;
        if constexpr (ALIGNED) {
            const T *p = row + k0;
            if (k0 + 8 > K || vec == 0) {
                load_single<T, kWords<T>>(p, 0, K - k0, w);
            } else if (sizeof(T) == 4 && vec >= 32) {
                asm volatile("ld.global.cs.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                             : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[kWords<T> - 4]), "=r"(w[kWords<T> - 3]), "=r"(w[kWords<T> - 2]), "=r"(w[kWords<T> - 1])
                             : "l"(p));
            } else {
#pragma unroll
                for (int i = 0; i < kWords<T> / 4; ++i) load16(reinterpret_cast<const uint4 *>(p) + i, w + 4 * i);
            }
        } else {
            shift = (uint32_t)reinterpret_cast<uintptr_t>(row) & 15u;
            const int32_t first = k0 - (int32_t)(shift / sizeof(T));  // the value that the aligned bytes begin with
            const T *p = row + first;
            if (first >= 0 && first + 8 <= K) {
#pragma unroll
                for (int i = 0; i < kBytes / 16; ++i) load16(reinterpret_cast<const uint4 *>(p) + i, w + 4 * i);
            } else {
                load_single<T, kWords<T>>(p, -first, K - first, w);
            }
            if ((threadIdx.x & 31) == 31) {
                constexpr int kNext = 16 / (int)sizeof(T);
                if (first + 8 + kNext <= K) load16(p + 8, behind);
                else load_single<T, 4>(p + 8, 0, K - first - 8, behind);
            }
        }
    }
    // The eight values (the whole warp together).
    __device__ __forceinline__ void settle()
    {
        if constexpr (!ALIGNED) {
            constexpr int N = kWords<T>;
            uint32_t z[N + 4];
#pragma unroll
            for (int i = 0; i < N; ++i) z[i] = w[i];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                z[N + i] = __shfl_down_sync(0xffffffffu, w[i], 1);
                if ((threadIdx.x & 31) == 31) z[N + i] = behind[i];
            }
#pragma unroll
            for (int i = 0; i < N + 2; ++i) z[i] = shift & 8 ? z[i + 2] : z[i];
#pragma unroll
            for (int i = 0; i < N + 1; ++i) z[i] = shift & 4 ? z[i + 1] : z[i];
#pragma unroll
            for (int i = 0; i < N; ++i) w[i] = sizeof(T) == 4 ? z[i] : __funnelshift_r(z[i], z[i + 1], (shift & 2) * 8);
        }
    }
};
template <typename T>
__device__ __forceinline__ void unpack8(const uint32_t (&w)[kWords<T>], float (&v)[8])
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
    } else if constexpr (std::is_same<T, __half>::value) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
            v[2 * i] = f.x;
            v[2 * i + 1] = f.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
}
// The exponent field (of fp32) of max|v|; 255 where one of the values is NaN or infinite.
template <typename T>
__device__ __forceinline__ uint32_t top_field(const uint32_t (&w)[kWords<T>])
{
    if constexpr (sizeof(T) == 4) {
        float m = __uint_as_float(w[0]);
#pragma unroll
        for (int i = 1; i < 8; ++i) asm("max.NaN.xorsign.abs.f32 %0, %0, %1;" : "+f"(m) : "f"(__uint_as_float(w[i])));
        return __float_as_uint(m) << 1 >> 24;
    } else {  // magnitudes order like their bits, two to a word
        uint32_t m = w[0] & 0x7fff7fffu;
#pragma unroll
        for (int i = 1; i < 4; ++i) m = __vmaxu2(m, w[i] & 0x7fff7fffu);
        m = __vmaxu2(m, m >> 16);
        if constexpr (std::is_same<T, __half>::value) return __float_as_uint(__half2float(__ushort_as_half((unsigned short)m))) >> 23;
        else return (m >> 7) & 0xffu;
    }
}
// The same without what is not a number; NaN becomes 0.
template <typename T>
__device__ __forceinline__ uint32_t top_finite_field(uint32_t (&w)[kWords<T>])
{
    float v[8];
    unpack8<T>(w, v);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t bits = __float_as_uint(v[i]) & 0x7fffffffu;
        if (bits > 0x7f800000u) w[sizeof(T) == 4 ? i : i / 2] &= sizeof(T) == 4 ? 0u : i & 1 ? 0xffffu : 0xffff0000u;
        if (bits < 0x7f800000u) top = max(top, bits);
    }
    return top >> 23;
}

// E of the block that this lane and its three neighbours hold of R rows (1 or 4), a byte a row, and the lane's codes of each row.  NaN becomes
// 0; neither NaN nor an infinity is in a maximum (`odd` says that there was one).  The rows share their shuffles, two exponents to a word:
// that, one test for all four of what is not a number, and the four by four bytes of scale_words() take 50 instructions a row less than rows by themselves.
template <typename T, int R>
__device__ __forceinline__ uint32_t quantize_rows(uint32_t (&w)[R][kWords<T>], uint32_t (&codes)[R], bool &odd)
{
    static_assert(R == 1 || R == 4, "rows");
    constexpr int N = R == 1 ? 1 : 2;
    uint32_t f[R], pair[N];
#pragma unroll
    for (int j = 0; j < R; ++j) f[j] = top_field<T>(w[j]);
    uint32_t all = f[0];
#pragma unroll
    for (int j = 1; j < R; ++j) all = max(all, f[j]);
    if (__any_sync(0xffffffffu, all == 255)) {
        odd = true;
#pragma unroll
        for (int j = 0; j < R; ++j) f[j] = top_finite_field<T>(w[j]);
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
        pair[n] = R == 1 ? f[0] : __byte_perm(f[2 * n % R], f[(2 * n + 1) % R], 0x5410);
        pair[n] = __vmaxu2(pair[n], __shfl_xor_sync(0xffffffffu, pair[n], 1));
        pair[n] = __vmaxu2(pair[n], __shfl_xor_sync(0xffffffffu, pair[n], 2));
        pair[n] = __vmaxu2(pair[n], 0x00020002u) - 0x00020002u;  // the fields less 2, at least 0: E
    }
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const uint32_t rest = 0x00fe00feu - pair[j / 2];  // 254 - E
        const float inv = __uint_as_float(j & 1 ? (rest & 0x00ff0000u) << 7 : rest << 23);
        const uint64_t inv2 = ptx::pack_f32x2(inv, inv);
        float v[8];
        unpack8<T>(w[j], v);
#pragma unroll
        for (int i = 0; i < 8; i += 2) ptx::unpack_f32x2(ptx::mul_f32x2(ptx::pack_f32x2(v[i], v[i + 1]), inv2), v[i], v[i + 1]);
        codes[j] = pack_e2m1(v);
    }
    return R == 1 ? pair[0] & 0xffu : __byte_perm(pair[0], pair[N - 1], 0x6420);
}
// The scale word of row i of the four for the lanes with (lane / 4) % 4 = i: the bytes of the four blocks that every 16 lanes hold, from the
// bytes of four rows that each lane has (a four by four transposition in two exchanges).
__device__ __forceinline__ uint32_t scale_words(uint32_t e, int lane)
{
    uint32_t q = __shfl_xor_sync(0xffffffffu, e, 4);
    e = __byte_perm(e, q, lane & 4 ? 0x3715 : 0x6240);
    q = __shfl_xor_sync(0xffffffffu, e, 8);
    return __byte_perm(e, q, lane & 8 ? 0x3276 : 0x5410);
}

// The largest access of up to 32 bytes that the rows are aligned for.  (fp32 in two halves of 16 bytes writes half sectors: dequantising
// 24576 x 1024 30 us, in one piece 17.)
inline int value_alignment(const void *p, int64_t ld, int size)
{
    const uint64_t all = reinterpret_cast<uintptr_t>(p) | (uint64_t)(ld * size);
    return all % 32 == 0 ? 32 : all % 16 == 0 ? 16 : 0;
}

}  // namespace mx4

// ---- launchers (q8_mx4.cu, q8_mx4_gemm_sm100.cu); arguments are checked by the entry points
struct Mx4QuantizeArgs {
    const void *X;  // [groups, rows, K], rows ld values apart, groups rows * ld
    int64_t ld;
    int64_t groups, rows, K;
    uint8_t *out;          // tiles
    void *Xhat = nullptr;  // instead: the values, in X's type, rows ldo values apart
    int64_t ldo = 0;
    int32_t *status;
    // slots of experts: rows is the number of slots, groups 1
    const int32_t *offsets = nullptr;  // [E + 1]
    int E = 0;
    const int32_t *index = nullptr;  // row of X of each slot; none: the slot's own
    int64_t x_rows = 0;              // rows that X has
};
cudaError_t launch_mx4_quantize(const Mx4QuantizeArgs &a, int dtype, cudaStream_t s);
cudaError_t launch_mx4_dequantize(const uint8_t *tiles, int64_t groups, int64_t rows, int64_t K, void *Y, int dtype, int64_t ldy, cudaStream_t s);

struct Mx4GemmArgs {
    const uint8_t *X;   // activation tiles, each expert's slots in row blocks of their own
    const uint8_t *W;   // weight tiles, each expert's in row blocks of their own
    const float *bias;  // [E, N] or nullptr
    void *Y;            // [M, N], rows ldy values apart
    int64_t ldy;
    int y_dtype;
    int64_t M, N, K;
    int act;
    const int32_t *offsets = nullptr;  // [E + 1], or nullptr with E == 1; with them the kernel before in the stream is the quantise pass of the slots
    int E = 1;
    int32_t *status;
    // Few tokens: taken and quantised by the product itself, X not used.
    const void *values = nullptr;
    int x_dtype = 0;
    int64_t ldx = 0;
};
cudaError_t launch_mx4_gemm(const Mx4GemmArgs &a, cudaStream_t s);
bool mx4_fused_preferred(int64_t M, int64_t K);  // whether to leave the quantisation of a plain activation to the product

}  // namespace q8
