// Newton-Schulz orthogonalisation of a stack of matrices: X0 = U / (|U|_F + eps), then per
// step, with A the Gram matrix of X on its smaller side,
//   X <- a X + (b A + c A^2) X    (rows <= cols, A = X X^T),
//   X <- a X + X (b A + c A^2)    (else, A = X^T X),
// all in fp32 (mec_linear_f32.hip): an error of one product grows by the factor a = 3.4 per
// step in the directions of small singular values, 140 times over the steps after the
// first, which fp32 has room for and bf16 (2^-9 a rounding) has not.
#include "mec_product.h"

namespace mec {
namespace {

constexpr int kShares = 64;  // of a matrix, for its norm

struct OrthParams {
    const void* U;
    float* X;
    double* part;     // batch x kShares sums of squares
    int64_t n;        // elements of a matrix
    int64_t per;      // and of a share
    float eps;
};

// The squares in fp64: those of gradients far from 1 leave fp32's range.
template <class E>
__global__ __launch_bounds__(256) void norm_squares_kernel(OrthParams p) {
    __shared__ double sums[4];
    const E* const u = static_cast<const E*>(p.U) + (int64_t)blockIdx.y * p.n;
    const int64_t end = (blockIdx.x + 1) * p.per < p.n ? (blockIdx.x + 1) * p.per : p.n;
    double s = 0.0;
    for (int64_t i = blockIdx.x * p.per + threadIdx.x; i < end; i += 256) {
        const double x = (double)to_float(u[i]);
        s += x * x;
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d, 64);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) p.part[blockIdx.y * kShares + blockIdx.x] = sums[0] + sums[1] + sums[2] + sums[3];
}

template <class E>
__global__ __launch_bounds__(256) void scale_kernel(OrthParams p) {
    double s = 0.0;
    for (int i = 0; i < kShares; ++i) s += p.part[blockIdx.y * kShares + i];
    const double by = 1.0 / (sqrt(s) + (double)p.eps);
    const E* const u = static_cast<const E*>(p.U) + (int64_t)blockIdx.y * p.n;
    float* const x = p.X + (int64_t)blockIdx.y * p.n;
    const int64_t end = (blockIdx.x + 1) * p.per < p.n ? (blockIdx.x + 1) * p.per : p.n;
    for (int64_t i = blockIdx.x * p.per + threadIdx.x; i < end; i += 256) x[i] = (float)((double)to_float(u[i]) * by);
}

__global__ __launch_bounds__(256) void to_bf16_kernel(const float* x, uint16_t* o, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) o[i] = from_float<uint16_t>(x[i]);
}

int64_t round16(int64_t bytes) { return (bytes + 15) / 16 * 16; }

}  // namespace

// Two copies of X, A and the polynomial's matrix, and the partial norms; the output is the
// second copy of X where it is fp32.
int64_t orth_workspace_bytes(int32_t batch, int64_t rows, int64_t cols, int) {
    const int64_t m = rows < cols ? rows : cols;
    return 16 + 2 * round16(batch * rows * cols * 4) + 2 * round16(batch * m * m * 4) + (int64_t)batch * kShares * 8;
}

hipError_t launch_orth(const void* U, void* O, void* workspace, int32_t batch, int64_t rows, int64_t cols, int32_t steps,
                       float a, float b, float c, float eps, int dtype, hipStream_t stream) {
    const int64_t n = rows * cols, m = rows < cols ? rows : cols;
    char* at = reinterpret_cast<char*>(((uintptr_t)workspace + 15) / 16 * 16);
    float* X[2];
    X[0] = reinterpret_cast<float*>(at);
    at += round16(batch * n * 4);
    X[1] = reinterpret_cast<float*>(at);
    at += round16(batch * n * 4);
    float* const A = reinterpret_cast<float*>(at);
    at += round16(batch * m * m * 4);
    float* const P = reinterpret_cast<float*>(at);
    at += round16(batch * m * m * 4);

    OrthParams q{};
    q.U = U;
    q.X = X[0];
    q.part = reinterpret_cast<double*>(at);
    q.n = n;
    q.per = (n + kShares - 1) / kShares;
    q.eps = eps;
    const dim3 grid(kShares, (uint32_t)batch);
    if (dtype) {
        hipLaunchKernelGGL(norm_squares_kernel<uint16_t>, grid, dim3(256), 0, stream, q);
        hipLaunchKernelGGL(scale_kernel<uint16_t>, grid, dim3(256), 0, stream, q);
    } else {
        hipLaunchKernelGGL(norm_squares_kernel<float>, grid, dim3(256), 0, stream, q);
        hipLaunchKernelGGL(scale_kernel<float>, grid, dim3(256), 0, stream, q);
    }
    hipError_t e = hipGetLastError();
    for (int32_t s = 0; s < steps && e == hipSuccess; ++s) {
        float* const from = X[s & 1];
        float* const to = s + 1 == steps && !dtype ? static_cast<float*>(O) : X[(s + 1) & 1];
        Product p{};
        p.batch = batch;
        p.splits = 1;
        p.alpha = 1.0f;
        // A
        p.A = p.B = from;
        p.Y = A;
        p.lda = p.ldb = cols;
        p.M = p.N = (int32_t)m;
        p.ldy = m;
        p.K = (int32_t)(n / m);
        p.a_batch = p.b_batch = n;
        p.y_batch = p.r_batch = m * m;
        e = launch_product(rows <= cols ? Layout::kXKt : Layout::kXtK, p, 0, stream);
        if (e != hipSuccess) break;
        // P = c A^2 + b A (A is symmetric: A A^T)
        p.A = p.B = A;
        p.Y = P;
        p.R = A;
        p.ldr = p.lda = p.ldb = m;
        p.K = (int32_t)m;
        p.a_batch = p.b_batch = m * m;
        p.alpha = c;
        p.beta = b;
        e = launch_product(Layout::kXKt, p, 0, stream);
        if (e != hipSuccess) break;
        // X
        p.alpha = 1.0f;
        p.beta = a;
        p.R = from;
        p.Y = to;
        p.M = (int32_t)rows;
        p.N = (int32_t)cols;
        p.ldr = p.ldy = cols;
        p.y_batch = p.r_batch = n;
        if (rows <= cols) {
            p.A = P;
            p.lda = m;
            p.a_batch = m * m;
            p.B = from;
            p.ldb = cols;
            p.b_batch = n;
            e = launch_product(Layout::kXK, p, 0, stream);
        } else {
            p.A = from;
            p.lda = cols;
            p.a_batch = n;
            p.B = P;
            p.ldb = m;
            p.b_batch = m * m;
            e = launch_product(Layout::kXKt, p, 0, stream);
        }
    }
    if (e == hipSuccess && dtype) {
        const int64_t total = batch * n, blocks = (total + 255) / 256;
        hipLaunchKernelGGL(to_bf16_kernel, dim3((uint32_t)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, stream, X[steps & 1],
                           static_cast<uint16_t*>(O), total);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace mec
