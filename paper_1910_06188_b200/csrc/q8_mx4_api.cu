// extern "C" entry points of the MXFP4 operators: argument checks and launches.

#include "q8_mx4.cuh"

using namespace q8;
using namespace q8::mx4;

namespace {

constexpr int64_t kMaxRows = (int64_t(1) << 31) - 512;  // rows and tile ends are 32-bit coordinates on the device
constexpr int64_t kMaxK = int64_t(1) << 24;
constexpr int64_t kMaxSpan = int64_t(1) << 56;  // rows * pitch, in values: offsets in bytes fit 64 bits with room

bool span_too_long(int64_t rows, int64_t ld) { return ld > kMaxSpan / (rows > 0 ? rows : 1); }

bool aligned_to(const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
bool known_dtype(int d) { return d == Q8_F32 || d == Q8_F16 || d == Q8_BF16; }
size_t dtype_bytes(int d) { return d == Q8_F32 ? 4 : 2; }
// Where conditions go that the caller gave no word for.
static __device__ int32_t g_status[1];
int32_t *own_status_word()
{
    static int32_t *cached[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return nullptr;
    if (cached[dev] == nullptr) {
        void *p = nullptr;
        if (cudaGetSymbolAddress(&p, g_status) != cudaSuccess) return nullptr;
        cached[dev] = static_cast<int32_t *>(p);
    }
    return cached[dev];
}
int32_t *word_or_own(int32_t *dev_status) { return dev_status != nullptr ? dev_status : own_status_word(); }
q8_status cuda_status(cudaError_t e) { return e == cudaSuccess ? Q8_OK : Q8_ERR_CUDA; }

// [groups, rows, K] with rows ld values apart
q8_status check_matrix(int64_t groups, int64_t rows, int64_t K, int64_t ld)
{
    if (groups < 0 || rows < 0 || K <= 0 || K > kMaxK || ld < K) return Q8_ERR_SHAPE;
    if (groups > kMaxRows || rows > kMaxRows || (rows > 0 && groups > kMaxRows / rows)) return Q8_ERR_SHAPE;
    return span_too_long(groups * rows, ld) ? Q8_ERR_SHAPE : Q8_OK;
}

q8_status check_layer(int64_t M, int64_t N, int64_t K, int64_t E, int64_t ldy)
{
    if (M < 0 || N < 0 || K <= 0 || E < 0) return Q8_ERR_SHAPE;
    if (M > kMaxRows || N > kMaxRows || K > kMaxK || E > kMaxExperts || ldy < N || span_too_long(M, ldy)) return Q8_ERR_SHAPE;
    if (E > 0 && N > kMaxRows / E) return Q8_ERR_SHAPE;
    // tiles are counted in 32 bits
    if (((M + 63) / 64 + E) * ((N + 127) / 128) > 0x7fff0000) return Q8_ERR_SHAPE;
    return Q8_OK;
}

// Whether rows of `a` and of `b` bytes, pa and pb bytes apart, have any byte in common.  (Rows side by side in one wider matrix do not.)
bool rows_overlap(const void *x, int64_t rows_x, int64_t a, int64_t pa, const void *y, int64_t rows_y, int64_t b, int64_t pb)
{
    const uintptr_t x0 = reinterpret_cast<uintptr_t>(x), y0 = reinterpret_cast<uintptr_t>(y);
    if (rows_x == 0 || rows_y == 0 || x0 + (uintptr_t)((rows_x - 1) * pa + a) <= y0 || y0 + (uintptr_t)((rows_y - 1) * pb + b) <= x0) return false;
    if (pa != pb) return true;
    const int64_t d = (int64_t)(y0 >= x0 ? (y0 - x0) % (uintptr_t)pa : (pa - (int64_t)((x0 - y0) % (uintptr_t)pa)) % pa);
    return d < a || d + b > pa;
}

// The same for rows and one piece of memory, such as tiles, a workspace or a bias.  (A piece between two rows touches neither.)
bool rows_touch(const void *x, int64_t rows, int64_t a, int64_t pa, const void *piece, size_t bytes)
{
    const int64_t b = (int64_t)bytes;
    return piece != nullptr && bytes > 0 && rows_overlap(x, rows, a, pa, piece, 1, b, b < pa ? pa : b);
}

bool pieces_touch(const void *x, size_t a, const void *y, size_t b)
{
    const uintptr_t x0 = reinterpret_cast<uintptr_t>(x), y0 = reinterpret_cast<uintptr_t>(y);
    return x != nullptr && y != nullptr && a > 0 && b > 0 && x0 < y0 + b && y0 < x0 + a;
}

// Whether a layer would write what it also reads: Y over weights, bias, offsets or rows, the workspace over any of them or over Y.
bool layer_overlaps(const Mx4GemmArgs &g, const int32_t *index, const void *workspace, size_t scratch)
{
    const int64_t size = (int64_t)dtype_bytes(g.y_dtype);
    const struct { const void *p; size_t bytes; } read[] = {{g.W, q8_mx4_bytes(g.E, g.N, g.K)},
                                                            {g.bias, (size_t)g.E * (size_t)g.N * sizeof(float)},
                                                            {g.offsets, ((size_t)g.E + 1) * sizeof(int32_t)},
                                                            {index, (size_t)g.M * sizeof(int32_t)}};
    for (const auto &r : read)
        if (rows_touch(g.Y, g.M, g.N * size, g.ldy * size, r.p, r.bytes) || pieces_touch(workspace, scratch, r.p, r.bytes)) return true;
    return rows_touch(g.Y, g.M, g.N * size, g.ldy * size, workspace, scratch);
}

// The activation into the workspace and the product from there, or both in one kernel where the tokens are few.
q8_status quantize_and_multiply(Mx4GemmArgs g, const void *X, int x_dtype, int64_t ldx, int64_t x_rows, const int32_t *index, void *workspace,
                                cudaStream_t s)
{
    if (g.offsets == nullptr && mx4_fused_preferred(g.M, g.K)) {
        g.values = X;
        g.x_dtype = x_dtype;
        g.ldx = ldx;
        return cuda_status(launch_mx4_gemm(g, s));
    }
    Mx4QuantizeArgs a = {};
    a.X = X;
    a.ld = ldx;
    a.groups = 1;
    a.rows = g.M;
    a.K = g.K;
    a.out = static_cast<uint8_t *>(workspace);
    a.status = g.status;
    a.offsets = g.offsets;
    a.E = g.E;
    a.index = index;
    a.x_rows = x_rows;
    const cudaError_t e = launch_mx4_quantize(a, x_dtype, s);
    if (e != cudaSuccess) return Q8_ERR_CUDA;
    g.X = a.out;
    return cuda_status(launch_mx4_gemm(g, s));
}

}  // namespace

extern "C" {

size_t q8_mx4_bytes(int64_t groups, int64_t rows, int64_t K)
{
    if (check_matrix(groups, rows, K, K) != Q8_OK) return 0;
    return (size_t)groups * (size_t)ceil_div(rows, kTileRows) * (size_t)tiles_along(K) * kTileBytes;
}

q8_status q8_mx4_status_word(void **dev_status)
{
    if (dev_status == nullptr) return Q8_ERR_NULL;
    *dev_status = own_status_word();
    return *dev_status != nullptr ? Q8_OK : Q8_ERR_CUDA;
}

q8_status q8_mx4_quantize(const void *X, int dtype, int64_t groups, int64_t rows, int64_t K, int64_t ldx, uint8_t *T, int32_t *dev_status,
                          void *stream)
{
    last_launch_info() = LaunchInfo();
    if (!known_dtype(dtype)) return Q8_ERR_ARG;
    const q8_status st = check_matrix(groups, rows, K, ldx);
    if (st != Q8_OK) return st;
    if (groups == 0 || rows == 0) return Q8_OK;
    if (!X || !T) return Q8_ERR_NULL;
    if (!aligned_to(X, dtype_bytes(dtype)) || !aligned_to(T, 16) || !aligned_to(dev_status, 4)) return Q8_ERR_ALIGN;
    const int64_t size = (int64_t)dtype_bytes(dtype);
    if (rows_touch(X, groups * rows, K * size, ldx * size, T, q8_mx4_bytes(groups, rows, K))) return Q8_ERR_ARG;
    Mx4QuantizeArgs a = {};
    a.X = X;
    a.ld = ldx;
    a.groups = groups;
    a.rows = rows;
    a.K = K;
    a.out = T;
    a.status = word_or_own(dev_status);
    return cuda_status(launch_mx4_quantize(a, dtype, static_cast<cudaStream_t>(stream)));
}

q8_status q8_mx4_dequantize(const uint8_t *T, int64_t groups, int64_t rows, int64_t K, void *Y, int dtype, int64_t ldy,
                            void *stream)
{
    last_launch_info() = LaunchInfo();
    if (!known_dtype(dtype)) return Q8_ERR_ARG;
    const q8_status st = check_matrix(groups, rows, K, ldy);
    if (st != Q8_OK) return st;
    if (groups == 0 || rows == 0) return Q8_OK;
    if (!Y || !T) return Q8_ERR_NULL;
    if (!aligned_to(Y, dtype_bytes(dtype)) || !aligned_to(T, 16)) return Q8_ERR_ALIGN;
    const int64_t size = (int64_t)dtype_bytes(dtype);
    if (rows_touch(Y, groups * rows, K * size, ldy * size, T, q8_mx4_bytes(groups, rows, K))) return Q8_ERR_ARG;
    return cuda_status(launch_mx4_dequantize(T, groups, rows, K, Y, dtype, ldy, static_cast<cudaStream_t>(stream)));
}

q8_status q8_mx4_fake_quantize(const void *X, int dtype, int64_t rows, int64_t K, int64_t ldx, void *Xhat, int64_t ldo, int32_t *dev_status, void *stream)
{
    last_launch_info() = LaunchInfo();
    if (!known_dtype(dtype)) return Q8_ERR_ARG;
    q8_status st = check_matrix(1, rows, K, ldx);
    if (st == Q8_OK) st = check_matrix(1, rows, K, ldo);
    if (st != Q8_OK) return st;
    if (rows == 0) return Q8_OK;
    if (!X || !Xhat) return Q8_ERR_NULL;
    if (!aligned_to(X, dtype_bytes(dtype)) || !aligned_to(Xhat, dtype_bytes(dtype)) || !aligned_to(dev_status, 4)) return Q8_ERR_ALIGN;
    const int64_t size = (int64_t)dtype_bytes(dtype);
    if ((X != Xhat || ldx != ldo) && rows_overlap(X, rows, K * size, ldx * size, Xhat, rows, K * size, ldo * size)) return Q8_ERR_ARG;
    Mx4QuantizeArgs a = {};
    a.X = X;
    a.ld = ldx;
    a.groups = 1;
    a.rows = rows;
    a.K = K;
    a.Xhat = Xhat;
    a.ldo = ldo;
    a.status = word_or_own(dev_status);
    return cuda_status(launch_mx4_quantize(a, dtype, static_cast<cudaStream_t>(stream)));
}

q8_status q8_mx4_ste_backward(const void *grad_out, int dtype, int64_t numel, void *grad_in, void *stream)
{
    last_launch_info() = LaunchInfo();
    if (!known_dtype(dtype)) return Q8_ERR_ARG;
    if (numel < 0 || numel > kMaxSpan) return Q8_ERR_SHAPE;
    if (numel == 0 || grad_in == grad_out) return Q8_OK;
    if (!grad_out || !grad_in) return Q8_ERR_NULL;
    const size_t size = dtype_bytes(dtype);
    if (!aligned_to(grad_out, size) || !aligned_to(grad_in, size)) return Q8_ERR_ALIGN;
    if (pieces_touch(grad_out, (size_t)numel * size, grad_in, (size_t)numel * size)) return Q8_ERR_ARG;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    return cuda_status(size == 4 ? launch_copy(static_cast<const float *>(grad_out), numel, static_cast<float *>(grad_in), s)
                                 : launch_copy_16(static_cast<const uint16_t *>(grad_out), numel, static_cast<uint16_t *>(grad_in), s));
}

size_t q8_mx4_linear_workspace_bytes(int64_t M, int64_t K) { return M >= 0 && K > 0 && mx4_fused_preferred(M, K) ? 0 : q8_mx4_bytes(1, M, K); }

size_t q8_mx4_linear_grouped_workspace_bytes(int64_t T, int64_t experts, int64_t K)
{
    if (T < 0 || T > kMaxRows || experts < 0 || experts > kMaxExperts || K <= 0 || K > kMaxK) return 0;
    return (size_t)most_row_blocks(T, experts) * (size_t)tiles_along(K) * kTileBytes;
}

q8_status q8_mx4_linear_q(const uint8_t *Xq, const uint8_t *Wq, const float *bias, int act, void *Y, int y_dtype,
                          int64_t ldy, int64_t M, int64_t N, int64_t K, int32_t *dev_status, void *stream)
{
    last_launch_info() = LaunchInfo();
    if (!known_dtype(y_dtype) || (act != Q8_ACT_NONE && act != Q8_ACT_GELU)) return Q8_ERR_ARG;
    const q8_status st = check_layer(M, N, K, 1, ldy);
    if (st != Q8_OK) return st;
    if (M == 0 || N == 0) return Q8_OK;
    if (!Xq || !Wq || !Y) return Q8_ERR_NULL;
    if (!aligned_to(Xq, 16) || !aligned_to(Wq, 16) || !aligned_to(bias, 4) ||
        !aligned_to(Y, dtype_bytes(y_dtype)) || !aligned_to(dev_status, 4))
        return Q8_ERR_ALIGN;
    Mx4GemmArgs g = {};
    g.X = Xq;
    g.W = Wq;
    g.bias = bias;
    g.Y = Y;
    g.ldy = ldy;
    g.y_dtype = y_dtype;
    g.M = M;
    g.N = N;
    g.K = K;
    g.act = act;
    g.E = 1;
    const int64_t ys = (int64_t)dtype_bytes(y_dtype);
    if (layer_overlaps(g, nullptr, nullptr, 0) || rows_touch(Y, M, N * ys, ldy * ys, Xq, q8_mx4_bytes(1, M, K))) return Q8_ERR_ARG;
    g.status = word_or_own(dev_status);
    return cuda_status(launch_mx4_gemm(g, static_cast<cudaStream_t>(stream)));
}

q8_status q8_mx4_linear(const void *X, int x_dtype, int64_t ldx, const uint8_t *Wq, const float *bias, int act, void *Y, int y_dtype,
                        int64_t ldy, int64_t M, int64_t N, int64_t K, void *workspace, size_t workspace_bytes, int32_t *dev_status, void *stream)
{
    last_launch_info() = LaunchInfo();
    if (!known_dtype(x_dtype) || !known_dtype(y_dtype) || (act != Q8_ACT_NONE && act != Q8_ACT_GELU)) return Q8_ERR_ARG;
    q8_status st = check_layer(M, N, K, 1, ldy);
    if (st == Q8_OK) st = check_matrix(1, M, K, ldx);
    if (st != Q8_OK) return st;
    if (M == 0 || N == 0) return Q8_OK;
    if (!X || !Wq || !Y || (!workspace && q8_mx4_linear_workspace_bytes(M, K) > 0)) return Q8_ERR_NULL;
    if (!aligned_to(X, dtype_bytes(x_dtype)) || !aligned_to(Wq, 16) || !aligned_to(bias, 4) ||
        !aligned_to(Y, dtype_bytes(y_dtype)) || !aligned_to(dev_status, 4) || !aligned_to(workspace, 256))
        return Q8_ERR_ALIGN;
    if (workspace_bytes < q8_mx4_linear_workspace_bytes(M, K)) return Q8_ERR_WORKSPACE;
    const int64_t xs = (int64_t)dtype_bytes(x_dtype), ys = (int64_t)dtype_bytes(y_dtype);
    const size_t scratch = q8_mx4_linear_workspace_bytes(M, K);
    Mx4GemmArgs g = {};
    g.W = Wq;
    g.bias = bias;
    g.Y = Y;
    g.ldy = ldy;
    g.y_dtype = y_dtype;
    g.M = M;
    g.N = N;
    g.K = K;
    g.act = act;
    g.E = 1;
    if (layer_overlaps(g, nullptr, workspace, scratch) || rows_overlap(X, M, K * xs, ldx * xs, Y, M, N * ys, ldy * ys) ||
        rows_touch(X, M, K * xs, ldx * xs, workspace, scratch))
        return Q8_ERR_ARG;
    g.status = word_or_own(dev_status);
    return quantize_and_multiply(g, X, x_dtype, ldx, M, nullptr, workspace, static_cast<cudaStream_t>(stream));
}

q8_status q8_mx4_linear_grouped(const void *X, int x_dtype, int64_t ldx, int64_t x_rows, const int32_t *rows, const int32_t *offsets, int64_t experts,
                                const uint8_t *Wq, const float *bias, int act, void *Y, int y_dtype, int64_t ldy, int64_t T, int64_t N,
                                int64_t K, void *workspace, size_t workspace_bytes, int32_t *dev_status, void *stream)
{
    last_launch_info() = LaunchInfo();
    if (!known_dtype(x_dtype) || !known_dtype(y_dtype) || (act != Q8_ACT_NONE && act != Q8_ACT_GELU)) return Q8_ERR_ARG;
    q8_status st = check_layer(T, N, K, experts, ldy);
    if (st == Q8_OK) st = check_matrix(1, x_rows, K, ldx);
    if (st != Q8_OK) return st;
    if (!rows && x_rows < T) return Q8_ERR_SHAPE;
    if (T == 0 || N == 0 || experts == 0) return Q8_OK;
    if ((!X && x_rows > 0) || !offsets || !Wq || !Y || !workspace) return Q8_ERR_NULL;
    if (!aligned_to(X, dtype_bytes(x_dtype)) || !aligned_to(rows, 4) || !aligned_to(offsets, 4) || !aligned_to(Wq, 16) ||
        !aligned_to(bias, 4) || !aligned_to(Y, dtype_bytes(y_dtype)) || !aligned_to(dev_status, 4) || !aligned_to(workspace, 256))
        return Q8_ERR_ALIGN;
    if (workspace_bytes < q8_mx4_linear_grouped_workspace_bytes(T, experts, K)) return Q8_ERR_WORKSPACE;
    const int64_t xs = (int64_t)dtype_bytes(x_dtype), ys = (int64_t)dtype_bytes(y_dtype);
    const size_t scratch = q8_mx4_linear_grouped_workspace_bytes(T, experts, K);
    Mx4GemmArgs g = {};
    g.W = Wq;
    g.bias = bias;
    g.Y = Y;
    g.ldy = ldy;
    g.y_dtype = y_dtype;
    g.M = T;
    g.N = N;
    g.K = K;
    g.act = act;
    g.offsets = offsets;
    g.E = (int)experts;
    if (layer_overlaps(g, rows, workspace, scratch) || rows_overlap(X, x_rows, K * xs, ldx * xs, Y, T, N * ys, ldy * ys) ||
        rows_touch(X, x_rows, K * xs, ldx * xs, workspace, scratch))
        return Q8_ERR_ARG;
    g.status = word_or_own(dev_status);
    return quantize_and_multiply(g, X, x_dtype, ldx, x_rows, rows, workspace, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
