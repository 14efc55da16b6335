// Newton-Schulz orthogonalisation of a stack of matrices: X0 = U / (|U|_F + eps), then per
// step, with A the Gram matrix of X on its smaller side (m of m x n, r = n / m),
//   X <- (a I + b A + c A^2) X    (rows <= cols, A = X X^T; else A = X^T X, from the right),
// all in fp32 (mec_linear_f32.hip): an error of one product grows by the factor a = 3.4 per
// step in the directions of small singular values, 140 times over the steps after the
// first, which fp32 has room for and bf16 (2^-8 a rounding) has not.
//
// Two steps at once: with P = a I + b A + c A^2 the Gram matrix after the step is P A P, so a
// pair of steps needs one Gram matrix of X and one product with X, for P' P, and the rest on
// m x m matrices (which commute, being polynomials of A): P A, (P A) P and P' P. In products
// of m x m x m that is 2r + 5 against 4r + 2. The error of A is relative to its largest value,
// and a step multiplies it in the small singular directions, so a pair costs least where
// all singular values are alike or what it spoils is not multiplied again: the first two
// steps (all below the polynomial's range yet) and the last two. The steps between them are
// taken one by one. What a pair loses depends on the steps around it and on the coefficients:
// error against 64 bits over that of single steps, worst of Gaussian, low-rank, two-valued and
// log-spaced spectra of 256 x 2304, 53 x 2016, 32 x 2160, 200 x 400 and 128 x 1152,
//   3.4445, -4.7750, 2.0315   5 to 10 steps 1.7 (1.0 to 1.1 at the median), but 2 steps 3.8, 4 (as
//                             2 + 2) 3.2, and 5 as 1 + 2 + 2 6, as 3 + 2 12, at once 70
//   1.5, -0.5, 0              2 steps 6.4, 5 steps 6.1
//   1.875, -1.25, 0.375       2 steps 3.4
//   2, -1.5, 0.5              4 steps 3.6, 5 steps 2.5
//   4, -6, 2.5                3 steps 3.1, 5 steps 19
// so that only 5 steps and more with the first of these are taken so; all others singly.
#include "mec_product.h"

namespace mec {
namespace {

constexpr int kShares = 128;  // of a matrix, for its norm

struct OrthParams {
    const void* U;
    float* X;
    double* part;     // batch x kShares sums of squares
    int64_t n;        // elements of a matrix
    int64_t per;      // and of a share
    float eps;
};

// The squares in fp64: those of gradients far from 1 leave fp32's range.
template <class E, int THREADS>
__device__ inline double sum_squares(const E* u, int64_t from, int64_t end) {
    __shared__ double sums[THREADS / 64];
    double s = 0.0;
#pragma unroll 2
    for (int64_t i = from + threadIdx.x * 8; i < end; i += THREADS * 8) {
        Pack8<E> w;
        const int have = end - i < 8 ? (int)(end - i) : 8;
        w.load(u + i, have);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < have) s += (double)w.get(e) * (double)w.get(e);
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d, 64);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
    __syncthreads();
    s = sums[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) s += sums[w];
    return s;
}

// x = by u
template <class E, int THREADS>
__device__ inline void scaled(const E* u, float* x, int64_t from, int64_t end, double by) {
#pragma unroll 2
    for (int64_t i = from + threadIdx.x * 8; i < end; i += THREADS * 8) {
        Pack8<E> w;
        const int have = end - i < 8 ? (int)(end - i) : 8;
        w.load(u + i, have);
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (float)((double)w.get(e) * by);
        Pack8<float> o;
        o.round(v);
        o.store(x + i, have);
    }
}

template <class E>
__global__ __launch_bounds__(256) void norm_squares_kernel(OrthParams p) {
    const E* const u = static_cast<const E*>(p.U) + (int64_t)blockIdx.y * p.n;
    const int64_t end = (blockIdx.x + 1) * p.per < p.n ? (blockIdx.x + 1) * p.per : p.n;
    const double s = sum_squares<E, 256>(u, blockIdx.x * p.per, end);
    if (threadIdx.x == 0) p.part[blockIdx.y * kShares + blockIdx.x] = s;
}

template <class E>
__global__ __launch_bounds__(256) void scale_kernel(OrthParams p) {
    double s = 0.0;
#pragma unroll 16
    for (int i = 0; i < kShares; ++i) s += p.part[blockIdx.y * kShares + i];
    const int64_t end = (blockIdx.x + 1) * p.per < p.n ? (blockIdx.x + 1) * p.per : p.n;
    scaled<E, 256>(static_cast<const E*>(p.U) + blockIdx.y * p.n, p.X + blockIdx.y * p.n, blockIdx.x * p.per, end,
                   1.0 / (sqrt(s) + (double)p.eps));
}

// small matrices: one workgroup each, in one launch
constexpr int64_t kOneLaunch = 65536;
template <class E>
__global__ __launch_bounds__(1024) void norm_scale_kernel(OrthParams p) {
    const E* const u = static_cast<const E*>(p.U) + (int64_t)blockIdx.x * p.n;
    float* const x = p.X + (int64_t)blockIdx.x * p.n;
    scaled<E, 1024>(u, x, 0, p.n, 1.0 / (sqrt(sum_squares<E, 1024>(u, 0, p.n)) + (double)p.eps));
}

template <class E>
hipError_t normalise(const OrthParams& q, int32_t batch, hipStream_t stream) {
    if (q.n <= kOneLaunch) {
        hipLaunchKernelGGL(norm_scale_kernel<E>, dim3((uint32_t)batch), dim3(1024), 0, stream, q);
    } else {
        hipLaunchKernelGGL(norm_squares_kernel<E>, dim3(kShares, (uint32_t)batch), dim3(256), 0, stream, q);
        hipLaunchKernelGGL(scale_kernel<E>, dim3(kShares, (uint32_t)batch), dim3(256), 0, stream, q);
    }
    return hipGetLastError();
}

int64_t round16(int64_t bytes) { return (bytes + 15) / 16 * 16; }

// m x m matrices for each of the stack: A, A after a step, P A (then P' P), P, P'; before those
// all but A hold the shares of A's sum: 6, or up to 32 of small ones (32 MB).
constexpr int kSquares = 5;
int32_t gram_shares(int64_t m, int32_t batch) {
    const int64_t fit = (int64_t(32) << 20) / (m * m * 4 * batch);
    return (int32_t)(fit < 6 ? 6 : fit < 32 ? fit : 32);
}

// A pair of steps at once loses less than twice a single step's precision (above) ...
bool pairs_precise(int32_t steps, float a, float b, float c) {
    return steps >= 5 && a == 3.4445f && b == -4.7750f && c == 2.0315f;
}
// ... and is faster: the modelled times of the products that differ.
bool pairs_faster(int64_t m, int64_t n, int32_t batch) {
    auto us = [&](int64_t M, int64_t N, int64_t K) { return plan_product(Layout::kXKt, 0, M, N, K, batch, 1, M == N).us; };
    return us(m, m, n) + us(n, m, m) > 3 * us(m, m, m);
}

// The polynomial and the product with X in one launch: where the polynomial's rows, made again
// for every 32 x 32 outputs, cost less than a launch: one round of workgroups (363 x 96 88 us
// without, so 70; 8 of 64 x 1000, two rounds, 100 and 112), and pairs of steps do not save
// more on A (5000 x 32 119 and 129).
bool step_preferred(int64_t m, int64_t rows, int64_t cols, int32_t batch) {
    return m <= kOrthStepMax && rows <= 2048 && cols <= 2048 && ((rows + 31) / 32) * ((cols + 31) / 32) * batch <= 256;
}

// The products of a step of m = min(rows, cols): the Gram matrix, in shares if that helps, and
// products of two m x m matrices.
ProductPlan gram_plan(int32_t batch, int64_t rows, int64_t cols) {
    const bool wide = rows <= cols;
    const int64_t m = wide ? rows : cols, n = wide ? cols : rows;
    return plan_product(wide ? Layout::kXKt : Layout::kXtK, 0, m, m, n, batch, gram_shares(m, batch), true);
}
ProductPlan square_plan(int32_t batch, int64_t m) { return plan_product(Layout::kXKt, 0, m, m, m, batch, 1, true); }

// How the steps are taken: by products, in a launch each, or in pairs at both ends.
enum class Steps { kSingle, kOneLaunch, kPairs };
Steps plan_steps(int32_t batch, int64_t rows, int64_t cols, int32_t steps, float a, float b, float c) {
    const int64_t m = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
    if (step_preferred(m, rows, cols, batch)) return Steps::kOneLaunch;
    return pairs_precise(steps, a, b, c) && pairs_faster(m, n, batch) ? Steps::kPairs : Steps::kSingle;
}

}  // namespace

bool orth_pairs(int32_t batch, int64_t rows, int64_t cols, int32_t steps, float a, float b, float c) {
    return plan_steps(batch, rows, cols, steps, a, b, c) == Steps::kPairs;
}

ProductPlan orth_plan(int32_t batch, int64_t rows, int64_t cols, bool gram) {
    return gram ? gram_plan(batch, rows, cols) : square_plan(batch, rows < cols ? rows : cols);
}

// Two copies of X, the m x m matrices and the partial norms; the output is the second copy's
// last use.
int64_t orth_workspace_bytes(int32_t batch, int64_t rows, int64_t cols, int) {
    const int64_t m = rows < cols ? rows : cols;
    return 16 + 2 * round16(batch * rows * cols * 4) +
           (1 + gram_shares(m, batch)) * round16(batch * m * m * 4) + (int64_t)batch * kShares * 8;
}

hipError_t launch_orth(const void* U, void* O, void* workspace, int32_t batch, int64_t rows, int64_t cols, int32_t steps,
                       float a, float b, float c, float eps, int dtype, hipStream_t stream) {
    const bool wide = rows <= cols;
    const int64_t m = wide ? rows : cols, n = wide ? cols : rows, mm = m * m;
    char* at = reinterpret_cast<char*>(((uintptr_t)workspace + 15) / 16 * 16);
    auto take = [&](int64_t bytes) {
        void* const p = at;
        at += round16(bytes);
        return static_cast<float*>(p);
    };
    float* const X[2] = {take(batch * m * n * 4), take(batch * m * n * 4)};
    float* S[kSquares];
    const int32_t shares = gram_shares(m, batch);
    for (float*& s : S) s = take(batch * mm * 4);
    take((1 + shares - kSquares) * round16(batch * mm * 4));  // S[1] on holds the shares

    OrthParams q{};
    q.U = U;
    q.X = X[0];
    q.part = reinterpret_cast<double*>(at);
    q.n = m * n;
    q.per = ((q.n + kShares - 1) / kShares + 7) / 8 * 8;
    q.eps = eps;
    hipError_t e = dtype ? normalise<uint16_t>(q, batch, stream) : normalise<float>(q, batch, stream);

    const ProductPlan grams = gram_plan(batch, rows, cols), squares = square_plan(batch, m);
    Product base{};
    base.batch = batch;
    base.splits = 1;
    base.alpha = 1.0f;
    // alpha S1 S2 of symmetric (or commuting) m x m matrices, to Y, which is not R
    auto square = [&](const float* s1, const float* s2, float* y, float alpha, const float* r, float beta, float diag) {
        if (e != hipSuccess) return;
        Product p = base;
        p.A = s1;
        p.B = s2;
        p.Y = y;
        p.R = r;
        p.lda = p.ldb = p.ldy = p.ldr = m;
        p.M = p.N = p.K = (int32_t)m;
        p.a_batch = p.b_batch = p.y_batch = p.r_batch = mm;
        p.alpha = alpha;
        p.beta = beta;
        p.diag = diag;
        p.symmetric = 1;
        e = launch_product(squares, Layout::kXKt, p, 0, stream);
    };
    int copy = 0;
    const Steps how = plan_steps(batch, rows, cols, steps, a, b, c);
    const bool one = how == Steps::kOneLaunch, pairs = how == Steps::kPairs;
    for (int32_t left = steps; left > 0 && e == hipSuccess;) {
        const bool two = pairs && left >= 2 && (left == steps || left == 2);
        left -= two ? 2 : 1;
        float *const A = S[0], *const A2 = S[1], *const T = S[2], *const P = S[3], *const P2 = S[4];
        const float* const from = X[copy];
        Product p = base;  // A
        p.A = p.B = from;
        p.Y = A;
        p.lda = p.ldb = cols;
        p.M = p.N = (int32_t)m;
        p.ldy = m;
        p.K = (int32_t)n;
        p.a_batch = p.b_batch = m * n;
        p.y_batch = mm;
        p.symmetric = 1;
        p.part = S[1];  // the other squares are free now
        e = launch_product(grams, wide ? Layout::kXKt : Layout::kXtK, p, 0, stream);
        if (e == hipSuccess && grams.splits > 1) e = launch_sum_parts(S[1], grams.splits, batch * mm, A, 0, stream);
        copy ^= 1;
        void* const to = left ? static_cast<void*>(X[copy]) : O;
        if (one) {
            if (e == hipSuccess)
                e = launch_orth_step({A, from, to, (int32_t)m, (int32_t)rows, (int32_t)cols, !left && dtype, a, b, c}, batch, stream);
            continue;
        }
        square(A, A, P, c, A, b, two ? a : 0.0f);  // a single step adds a X itself
        if (two) {
            square(P, A, T, 1.0f, nullptr, 0.0f, 0.0f);
            square(T, P, A2, 1.0f, nullptr, 0.0f, 0.0f);
            square(A2, A2, P2, c, A2, b, a);
            square(P2, P, T, 1.0f, nullptr, 0.0f, 0.0f);
        }
        const float* const Q = two ? T : P;
        if (e != hipSuccess) break;
        p = base;  // X
        if (!two) {
            p.R = from;
            p.beta = a;
        }
        p.Y = to;
        p.y_bf16 = !left && dtype;
        p.M = (int32_t)rows;
        p.N = (int32_t)cols;
        p.K = (int32_t)m;
        p.ldr = p.ldy = cols;
        p.y_batch = p.r_batch = m * n;
        p.A = wide ? Q : from;
        p.lda = wide ? m : cols;
        p.a_batch = wide ? mm : m * n;
        p.B = wide ? from : Q;
        p.ldb = wide ? cols : m;
        p.b_batch = wide ? m * n : mm;
        e = launch_product(wide ? Layout::kXK : Layout::kXKt, p, 0, stream);
    }
    return e;
}

}  // namespace mec
