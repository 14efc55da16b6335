// Host side of the C ABI declared in include/mec.h: argument validation,
// output-size arithmetic (Eq. (1), floor reading), workspace sizes, and the
// choice of kernels. Every check happens before anything is enqueued.
#include "mec.h"

#include <stdint.h>
#include <stdio.h>

#include <algorithm>
#include <initializer_list>

#include "mec_internal.h"
#include "mec_product.h"

namespace {

// Largest tensor this build accepts, in elements. Far above the 288 GB of one
// MI355X; it keeps every int64 product in this file from overflowing.
constexpr int64_t kMaxElems = int64_t(1) << 40;

bool valid_dtype(int dtype) { return dtype == MEC_F32 || dtype == MEC_BF16; }
int64_t elem_bytes(int dtype) { return dtype == MEC_F32 ? 4 : 2; }

// Product of non-negative factors, or -1 once it exceeds kMaxElems.
int64_t checked_product(std::initializer_list<int64_t> factors) {
    int64_t r = 1;
    for (int64_t f : factors) {
        if (f < 0) return -1;
        if (f != 0 && r > kMaxElems / f) return -1;
        r *= f;
    }
    return r;
}

// Fills s from the arguments; returns MEC_OK or MEC_ERR_INVALID_ARG.
int make_shape(mec::Shape& s, int i_n, int i_h, int i_w, int i_c, int k_h, int k_w, int k_c,
               int s_h, int s_w) {
    if (i_n < 1 || i_h < 1 || i_w < 1 || i_c < 1 || k_h < 1 || k_w < 1 || k_c < 1 || s_h < 1 ||
        s_w < 1)
        return MEC_ERR_INVALID_ARG;
    if (k_h > i_h || k_w > i_w) return MEC_ERR_INVALID_ARG;
    s.i_n = i_n; s.i_h = i_h; s.i_w = i_w; s.i_c = i_c;
    s.k_h = k_h; s.k_w = k_w; s.k_c = k_c; s.s_h = s_h; s.s_w = s_w;
    s.o_h = (s.i_h - s.k_h) / s.s_h + 1;  // Eq. (1), floor
    s.o_w = (s.i_w - s.k_w) / s.s_w + 1;
    s.R = s.k_w * s.i_c;
    s.pairs = s.i_n * s.o_w;
    if (checked_product({s.i_n, s.i_h, s.i_w, s.i_c}) < 0 ||
        checked_product({s.k_h, s.k_w, s.i_c, s.k_c}) < 0 ||
        checked_product({s.i_n, s.o_h, s.o_w, s.k_c}) < 0 ||
        checked_product({s.i_n, s.o_w, s.i_h, s.k_w, s.i_c}) < 0 ||
        checked_product({s.i_n, s.o_h, s.o_w, s.k_h, s.k_w, s.i_c}) < 0)
        return MEC_ERR_INVALID_ARG;
    // the kernels index one L row (R elements) and one block's rows in 32 bits
    if (s.R > (int64_t(1) << 26)) return MEC_ERR_INVALID_ARG;
    return MEC_OK;
}

int64_t lowered_elems(const mec::Shape& s) { return s.i_n * s.o_w * s.i_h * s.k_w * s.i_c; }
int64_t im2col_elems(const mec::Shape& s) { return s.i_n * s.o_h * s.o_w * s.k_h * s.k_w * s.i_c; }

// The product phase of im2col + GEMM as MEC's product phase of a 1x1,
// stride-1 convolution: the image has pixels (n, y, x), each with the
// k_h*k_w*i_c values of its patch as channels; its MEC lowered tensor is the
// (n, x, y)-ordered im2col matrix.
mec::Shape im2col_product_shape(const mec::Shape& s) {
    mec::Shape v = s;
    v.i_h = s.o_h;
    v.i_w = s.o_w;
    v.i_c = s.k_h * s.k_w * s.i_c;
    v.k_h = v.k_w = v.s_h = v.s_w = 1;
    v.o_h = s.o_h;
    v.o_w = s.o_w;
    v.R = v.i_c;
    v.pairs = s.i_n * s.o_w;
    return v;
}

bool aligned(const void* p, int64_t bytes) { return ((uintptr_t)p % (uintptr_t)bytes) == 0; }

thread_local char g_last_error[256];

// Launch status -> MEC status; a failure records which launch and why.
int hip_status(hipError_t e, const char* what) {
    if (e == hipSuccess) return MEC_OK;
    snprintf(g_last_error, sizeof g_last_error, "%s: %s (%s)", what, hipGetErrorName(e),
             hipGetErrorString(e));
    return MEC_ERR_HIP;
}

// A HIP error left pending by earlier, unrelated work would be reported by the
// hipGetLastError that follows our launch; take it off first.
void clear_stale_error() {
    g_last_error[0] = 0;
    (void)hipGetLastError();
}

}  // namespace

extern "C" {

int mec_output_dims(int i_h, int i_w, int k_h, int k_w, int s_h, int s_w, int* o_h, int* o_w) {
    if (i_h < 1 || i_w < 1 || k_h < 1 || k_w < 1 || s_h < 1 || s_w < 1 || k_h > i_h || k_w > i_w)
        return MEC_ERR_INVALID_ARG;
    if (o_h) *o_h = (i_h - k_h) / s_h + 1;
    if (o_w) *o_w = (i_w - k_w) / s_w + 1;
    return MEC_OK;
}

int64_t mec_workspace_bytes(int i_n, int i_h, int i_w, int i_c, int k_h, int k_w, int k_c,
                            int s_h, int s_w, int dtype, int algo) {
    mec::Shape s;
    int rc = make_shape(s, i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w);
    if (rc != MEC_OK) return rc;
    if (!valid_dtype(dtype)) return MEC_ERR_INVALID_ARG;
    if (algo == MEC_ALGO_FUSED) return 0;
    if (algo == MEC_ALGO_IM2COL) return im2col_elems(s) * elem_bytes(dtype);
    if (algo != MEC_ALGO_LOWERED) return MEC_ERR_INVALID_ARG;
    return lowered_elems(s) * elem_bytes(dtype);
}

int64_t mec_im2col_bytes(int i_n, int i_h, int i_w, int i_c, int k_h, int k_w, int k_c, int s_h,
                         int s_w, int dtype) {
    mec::Shape s;
    int rc = make_shape(s, i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w);
    if (rc != MEC_OK) return rc;
    if (!valid_dtype(dtype)) return MEC_ERR_INVALID_ARG;
    return im2col_elems(s) * elem_bytes(dtype);
}

int mec_lower(const void* I, void* L, int i_n, int i_h, int i_w, int i_c, int k_h, int k_w,
              int k_c, int s_h, int s_w, int dtype, void* stream) {
    mec::Shape s;
    int rc = make_shape(s, i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w);
    if (rc != MEC_OK) return rc;
    if (!valid_dtype(dtype) || !I || !L) return MEC_ERR_INVALID_ARG;
    const int64_t es = elem_bytes(dtype);
    if (!aligned(I, es) || !aligned(L, es)) return MEC_ERR_ALIGNMENT;
    clear_stale_error();
    return hip_status(mec::launch_lower(s, I, L, (int)es, (hipStream_t)stream), "lowering");
}

int mec_im2col(const void* I, void* M, int i_n, int i_h, int i_w, int i_c, int k_h, int k_w,
               int k_c, int s_h, int s_w, int dtype, void* stream) {
    mec::Shape s;
    int rc = make_shape(s, i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w);
    if (rc != MEC_OK) return rc;
    if (!valid_dtype(dtype) || !I || !M) return MEC_ERR_INVALID_ARG;
    const int64_t es = elem_bytes(dtype);
    if (!aligned(I, es) || !aligned(M, es)) return MEC_ERR_ALIGNMENT;
    clear_stale_error();
    return hip_status(mec::launch_im2col(s, I, M, (int)es, (hipStream_t)stream), "im2col");
}

int mec_gemm(const void* L, const void* K, float* O, int i_n, int i_h, int i_w, int i_c, int k_h,
             int k_w, int k_c, int s_h, int s_w, int dtype, void* stream) {
    mec::Shape s;
    int rc = make_shape(s, i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w);
    if (rc != MEC_OK) return rc;
    if (!valid_dtype(dtype) || !L || !K || !O) return MEC_ERR_INVALID_ARG;
    const int64_t es = elem_bytes(dtype);
    if (!aligned(L, es) || !aligned(K, es) || !aligned(O, 4)) return MEC_ERR_ALIGNMENT;
    if (!mec::gemm_supported(s, dtype, false)) return MEC_ERR_UNSUPPORTED;
    clear_stale_error();
    return hip_status(mec::launch_gemm(s, L, K, O, dtype, false, (hipStream_t)stream),
                      "slab products");
}

int mec_conv2d(const void* I, const void* K, float* O, void* workspace, size_t workspace_bytes,
               int i_n, int i_h, int i_w, int i_c, int k_h, int k_w, int k_c, int s_h, int s_w,
               int dtype, int algo, void* stream) {
    mec::Shape s;
    int rc = make_shape(s, i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w);
    if (rc != MEC_OK) return rc;
    if (!valid_dtype(dtype) ||
        (algo != MEC_ALGO_LOWERED && algo != MEC_ALGO_FUSED && algo != MEC_ALGO_IM2COL) || !I ||
        !K || !O)
        return MEC_ERR_INVALID_ARG;
    const int64_t es = elem_bytes(dtype);
    if (!aligned(I, es) || !aligned(K, es) || !aligned(O, 4)) return MEC_ERR_ALIGNMENT;
    if (algo != MEC_ALGO_FUSED) {
        const int64_t need = (algo == MEC_ALGO_IM2COL ? im2col_elems(s) : lowered_elems(s)) * es;
        if (!workspace || (uint64_t)workspace_bytes < (uint64_t)need) return MEC_ERR_WORKSPACE;
        if (!aligned(workspace, es)) return MEC_ERR_ALIGNMENT;
    }
    const mec::Shape g = algo == MEC_ALGO_IM2COL ? im2col_product_shape(s) : s;
    if (g.R > (int64_t(1) << 26) || !mec::gemm_supported(g, dtype, algo == MEC_ALGO_FUSED))
        return MEC_ERR_UNSUPPORTED;
    const hipStream_t st = (hipStream_t)stream;
    clear_stale_error();
    if (algo == MEC_ALGO_FUSED)
        return hip_status(mec::launch_gemm(s, I, K, O, dtype, true, st), "fused slab products");
    if (algo == MEC_ALGO_IM2COL) {
        rc = hip_status(mec::launch_im2col(s, I, workspace, (int)es, st), "im2col");
        if (rc != MEC_OK) return rc;
        return hip_status(mec::launch_gemm(g, workspace, K, O, dtype, false, st), "im2col product");
    }
    rc = hip_status(mec::launch_lower(s, I, workspace, (int)es, st), "lowering");
    if (rc != MEC_OK) return rc;
    if (mec::gemm_from_input(s, I, K, dtype))
        return hip_status(mec::launch_gemm(s, I, K, O, dtype, true, st), "slab products from the input");
    return hip_status(mec::launch_gemm(s, workspace, K, O, dtype, false, st), "slab products");
}

// ---------------------------------------------------------------- training passes

namespace {

// Common checks of the training entry points: shape, dtype (fp32 only),
// and the 32-bit index ranges of the kernels.
int grad_shape(mec::Shape& s, int i_n, int i_h, int i_w, int i_c, int k_h, int k_w, int k_c,
               int s_h, int s_w, int dtype) {
    int rc = make_shape(s, i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w);
    if (rc != MEC_OK) return rc;
    if (!valid_dtype(dtype)) return MEC_ERR_INVALID_ARG;
    if (dtype != MEC_F32) return MEC_ERR_UNSUPPORTED;
    if (s.i_n * s.i_h * s.i_w * s.i_c >= (int64_t(1) << 31)) return MEC_ERR_UNSUPPORTED;
    return MEC_OK;
}

}  // namespace

int64_t mec_grad_workspace_bytes(int i_n, int i_h, int i_w, int i_c, int k_h, int k_w, int k_c,
                                 int s_h, int s_w, int dtype, int pass) {
    mec::Shape s;
    int rc = grad_shape(s, i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w, dtype);
    if (rc != MEC_OK) return rc;
    switch (pass) {
        case MEC_GRAD_INPUT: return mec::dgrad_workspace_bytes(s);
        case MEC_GRAD_KERNEL:  // the products read L's rows from I: partial sums only
        case MEC_GRAD_KERNEL_FROM_L: return mec::wgrad_partial_bytes(s);
        default: return MEC_ERR_INVALID_ARG;
    }
}

int mec_fold(const float* dL, float* dI, int i_n, int i_h, int i_w, int i_c, int k_h, int k_w,
             int k_c, int s_h, int s_w, void* stream) {
    mec::Shape s;
    int rc = grad_shape(s, i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w, MEC_F32);
    if (rc != MEC_OK) return rc;
    if (!dL || !dI) return MEC_ERR_INVALID_ARG;
    if (!aligned(dL, 4) || !aligned(dI, 4)) return MEC_ERR_ALIGNMENT;
    clear_stale_error();
    return hip_status(mec::launch_fold(s, dL, dI, (hipStream_t)stream), "fold");
}

int mec_dgrad_gemm(const float* G, const float* K, float* dL, int i_n, int i_h, int i_w, int i_c,
                   int k_h, int k_w, int k_c, int s_h, int s_w, int dtype, void* stream) {
    mec::Shape s;
    int rc = grad_shape(s, i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w, dtype);
    if (rc != MEC_OK) return rc;
    if (!G || !K || !dL) return MEC_ERR_INVALID_ARG;
    if (!aligned(G, 4) || !aligned(K, 4) || !aligned(dL, 4)) return MEC_ERR_ALIGNMENT;
    if (!mec::dgrad_supported(s)) return MEC_ERR_UNSUPPORTED;
    clear_stale_error();
    return hip_status(mec::launch_dgrad_dl(s, G, K, dL, (hipStream_t)stream), "dgrad products");
}

int mec_conv2d_dgrad(const float* G, const void* K, float* dI, void* workspace,
                     size_t workspace_bytes, int i_n, int i_h, int i_w, int i_c, int k_h, int k_w,
                     int k_c, int s_h, int s_w, int dtype, void* stream) {
    mec::Shape s;
    int rc = grad_shape(s, i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w, dtype);
    if (rc != MEC_OK) return rc;
    if (!G || !K || !dI) return MEC_ERR_INVALID_ARG;
    if (!aligned(G, 4) || !aligned(K, 4) || !aligned(dI, 4)) return MEC_ERR_ALIGNMENT;
    if (!workspace || (uint64_t)workspace_bytes < (uint64_t)mec::dgrad_workspace_bytes(s))
        return MEC_ERR_WORKSPACE;
    if (!aligned(workspace, 4)) return MEC_ERR_ALIGNMENT;
    const hipStream_t st = (hipStream_t)stream;
    clear_stale_error();
    if (mec::dgrad_phases_ok(s))
        return hip_status(mec::launch_dgrad_phases(s, G, static_cast<const float*>(K), dI,
                                                   workspace, st),
                          "dgrad as sub-pixel phases of the padded gradient");
    if (!mec::dgrad_supported(s)) return MEC_ERR_UNSUPPORTED;
    float* dL = static_cast<float*>(workspace);
    rc = hip_status(mec::launch_dgrad_dl(s, G, static_cast<const float*>(K), dL, st),
                    "dgrad products");
    if (rc != MEC_OK) return rc;
    return hip_status(mec::launch_fold(s, dL, dI, st), "fold");
}

int mec_wgrad_gemm(const void* L, const float* G, float* dK, void* workspace,
                   size_t workspace_bytes, int i_n, int i_h, int i_w, int i_c, int k_h, int k_w,
                   int k_c, int s_h, int s_w, int dtype, void* stream) {
    mec::Shape s;
    int rc = grad_shape(s, i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w, dtype);
    if (rc != MEC_OK) return rc;
    if (!L || !G || !dK) return MEC_ERR_INVALID_ARG;
    if (!aligned(L, 4) || !aligned(G, 4) || !aligned(dK, 4)) return MEC_ERR_ALIGNMENT;
    if (!mec::wgrad_supported(s)) return MEC_ERR_UNSUPPORTED;
    if (!workspace || (uint64_t)workspace_bytes < (uint64_t)mec::wgrad_partial_bytes(s))
        return MEC_ERR_WORKSPACE;
    if (!aligned(workspace, 4)) return MEC_ERR_ALIGNMENT;
    clear_stale_error();
    return hip_status(mec::launch_wgrad(s, static_cast<const float*>(L), G,
                                        static_cast<float*>(workspace), dK, (hipStream_t)stream),
                      "wgrad products");
}

int mec_conv2d_wgrad(const void* I, const float* G, float* dK, void* workspace,
                     size_t workspace_bytes, int i_n, int i_h, int i_w, int i_c, int k_h, int k_w,
                     int k_c, int s_h, int s_w, int dtype, void* stream) {
    mec::Shape s;
    int rc = grad_shape(s, i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w, dtype);
    if (rc != MEC_OK) return rc;
    if (!I || !G || !dK) return MEC_ERR_INVALID_ARG;
    if (!aligned(I, 4) || !aligned(G, 4) || !aligned(dK, 4)) return MEC_ERR_ALIGNMENT;
    if (!mec::wgrad_supported(s)) return MEC_ERR_UNSUPPORTED;
    if (!workspace || (uint64_t)workspace_bytes < (uint64_t)mec::wgrad_partial_bytes(s))
        return MEC_ERR_WORKSPACE;
    if (!aligned(workspace, 4)) return MEC_ERR_ALIGNMENT;
    const hipStream_t st = (hipStream_t)stream;
    float* part = static_cast<float*>(workspace);
    clear_stale_error();
    // the products read L's rows straight from I: no lowering pass
    return hip_status(mec::launch_wgrad(s, static_cast<const float*>(I), G, part, dK, st, true),
                      "wgrad products from I");
}

// ---------------------------------------------------------------- layer operators

namespace {

// Widths and pitches that the kernels' 32-bit offsets within a tile hold, and rows that
// their grids do.
constexpr int64_t kMaxWidth = int64_t(1) << 20, kMaxRows = int64_t(1) << 30;

// rows of `width` elements, `pitch` apart
int check_rows(int64_t rows, int64_t width, int64_t pitch) {
    if (rows < 1 || width < 1 || pitch < width) return MEC_ERR_INVALID_ARG;
    if (rows > kMaxRows || pitch > kMaxWidth) return MEC_ERR_UNSUPPORTED;
    return checked_product({rows, pitch}) < 0 ? MEC_ERR_INVALID_ARG : MEC_OK;
}

int first_error(std::initializer_list<int> codes) {
    for (int c : codes)
        if (c != MEC_OK) return c;
    return MEC_OK;
}

// A product by its plan, the shares of its reduction (in p.part) added up; without an
// epilogue of its own Y is dense.
hipError_t launch_shared(const mec::ProductPlan& plan, mec::Layout layout, mec::Product p, int dtype, hipStream_t stream) {
    const hipError_t e = mec::launch_product(plan, layout, p, dtype, stream);
    if (e != hipSuccess || plan.splits == 1) return e;
    if (layout != mec::Layout::kXK) return mec::launch_sum_parts(p.part, plan.splits, (int64_t)p.M * p.N, p.Y, dtype, stream);
    p.splits = plan.splits;
    return mec::launch_finish_parts(p, dtype, stream);
}

bool valid_act(int act) { return act >= MEC_ACT_NONE && act <= MEC_ACT_GELU; }

constexpr int32_t kMaxShares = 64;  // of a product's reduction

// the sums of a product's shares
int64_t parts_bytes(const mec::ProductPlan& plan, int64_t M, int64_t N) { return plan.splits > 1 ? plan.splits * M * N * 4 : 0; }

mec::ProductPlan linear_plan(int64_t rows, int64_t i_c, int64_t k_c, int dtype) {
    return mec::plan_product(mec::Layout::kXK, dtype, rows, k_c, i_c, 1, kMaxShares);
}

// What a backward pass does by its sizes and activation, and the workspace for it: partial sums
// and, 16-byte aligned behind them, dZ's second part where there is one. (ReLU's dZ is G or 0, so
// that rounding it leaves nothing over.)
struct GradPlan {
    mec::ProductPlan x, k, pair;
    int64_t sums, bytes;
    bool two;
};
GradPlan grad_plan(int64_t rows, int64_t i_c, int64_t k_c, int dtype, int act) {
    GradPlan g;
    g.two = dtype == MEC_BF16 && act > MEC_ACT_RELU;
    mec::Operands with;
    with.two = g.two;
    g.x = mec::plan_product(mec::Layout::kXKt, dtype, rows, i_c, k_c, 1, kMaxShares, false, with);
    g.k = mec::plan_product(mec::Layout::kXtK, dtype, i_c, k_c, rows, 1, kMaxShares, false, with);
    g.pair = mec::plan_pair(g.x, g.k, dtype, rows, i_c, k_c, kMaxShares, g.two);
    const int64_t shares = mec::act_grad_shares(rows, k_c);  // one share goes straight to dbias
    g.sums = std::max({parts_bytes(g.x, rows, i_c), parts_bytes(g.k, i_c, k_c), parts_bytes(g.pair, i_c, k_c),
                       shares > 1 ? shares * k_c * 4 : int64_t(0)});
    g.bytes = g.sums + (g.two ? 16 + 2 * rows * k_c : 0);
    return g;
}

// How dX and dK are computed where both are wanted.
enum class GradRoute { kApart = 0, kSmallPair = 1, kTilePair = 2 };
GradRoute grad_route(const GradPlan& plan, const mec::ProductPlan& px, const mec::ProductPlan& pk, bool clean) {
    if (px.kernel == 0 && pk.kernel == 0) return GradRoute::kSmallPair;
    return plan.pair.kernel && clean ? GradRoute::kTilePair : GradRoute::kApart;
}

}  // namespace

int mec_linear(const void* X, const void* K, const float* bias, const void* R, void* Y, void* Z, int64_t rows, int i_c,
               int k_c, int64_t x_pitch, int64_t r_pitch, int64_t y_pitch, int dtype, int act, int residual_first,
               void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = first_error({check_rows(rows, i_c, x_pitch), check_rows(rows, k_c, y_pitch),
                                R ? check_rows(rows, k_c, r_pitch) : MEC_OK});
    if (rc != MEC_OK) return rc;
    if (!valid_dtype(dtype) || !valid_act(act) || !X || !K || !Y) return MEC_ERR_INVALID_ARG;
    const int64_t es = elem_bytes(dtype);
    if (!aligned(X, es) || !aligned(K, es) || !aligned(bias, 4) || !aligned(R, es) || !aligned(Y, es) || !aligned(Z, es))
        return MEC_ERR_ALIGNMENT;
    const mec::ProductPlan plan = linear_plan(rows, i_c, k_c, dtype);
    const int64_t need = parts_bytes(plan, rows, k_c);
    if (need && (!workspace || (uint64_t)workspace_bytes < (uint64_t)need)) return MEC_ERR_WORKSPACE;
    if (!aligned(workspace, 4)) return MEC_ERR_ALIGNMENT;
    mec::Product p{};
    p.A = X;
    p.B = K;
    p.Y = Y;
    p.Z = Z;
    p.R = R;
    p.bias = bias;
    p.lda = x_pitch;
    p.ldb = p.ldz = k_c;
    p.ldr = r_pitch;
    p.ldy = y_pitch;
    p.M = (int32_t)rows;
    p.N = k_c;
    p.K = i_c;
    p.act = act;
    p.res_first = residual_first != 0;
    p.alpha = p.beta = 1.0f;
    p.batch = 1;
    p.part = static_cast<float*>(workspace);
    const mec::ProductPlan refined = mec::refine_plan(plan, mec::Layout::kXK, dtype, p);
    if (refined.kernel < 0) return MEC_ERR_UNSUPPORTED;
    clear_stale_error();
    return hip_status(launch_shared(refined, mec::Layout::kXK, p, dtype, (hipStream_t)stream), "linear");
}

int64_t mec_linear_workspace_bytes(int64_t rows, int i_c, int k_c, int dtype) {
    const int rc = first_error({check_rows(rows, i_c, i_c), check_rows(rows, k_c, k_c)});
    if (rc != MEC_OK) return rc;
    if (!valid_dtype(dtype)) return MEC_ERR_INVALID_ARG;
    const mec::ProductPlan plan = linear_plan(rows, i_c, k_c, dtype);
    return plan.kernel < 0 ? MEC_ERR_UNSUPPORTED : parts_bytes(plan, rows, k_c);
}

int64_t mec_linear_grad_workspace_bytes(int64_t rows, int i_c, int k_c, int dtype) {
    const int rc = first_error({check_rows(rows, i_c, i_c), check_rows(rows, k_c, k_c)});
    if (rc != MEC_OK) return rc;
    if (!valid_dtype(dtype)) return MEC_ERR_INVALID_ARG;
    return std::max(grad_plan(rows, i_c, k_c, dtype, MEC_ACT_NONE).bytes, grad_plan(rows, i_c, k_c, dtype, MEC_ACT_GELU).bytes);
}

int64_t mec_linear_grad_act_workspace_bytes(int64_t rows, int i_c, int k_c, int dtype, int act) {
    const int rc = first_error({check_rows(rows, i_c, i_c), check_rows(rows, k_c, k_c)});
    if (rc != MEC_OK) return rc;
    if (!valid_dtype(dtype) || !valid_act(act)) return MEC_ERR_INVALID_ARG;
    return grad_plan(rows, i_c, k_c, dtype, act).bytes;
}

int mec_linear_grad(const void* G, const void* X, const void* K, const void* Z, void* dZ, void* dX, void* dK, float* dbias,
                    void* workspace, size_t workspace_bytes, int64_t rows, int i_c, int k_c, int64_t g_pitch,
                    int64_t x_pitch, int dtype, int act, void* stream) {
    int rc = first_error({check_rows(rows, k_c, g_pitch), X ? check_rows(rows, i_c, x_pitch) : check_rows(rows, i_c, i_c)});
    if (rc != MEC_OK) return rc;
    if (!valid_dtype(dtype) || !valid_act(act) || !G || (dX && !K) || (dK && !X) || (act != MEC_ACT_NONE && (!Z || !dZ)))
        return MEC_ERR_INVALID_ARG;
    const int64_t es = elem_bytes(dtype);
    if (!aligned(G, es) || !aligned(X, es) || !aligned(K, es) || !aligned(Z, es) || !aligned(dZ, es) || !aligned(dX, es) ||
        !aligned(dK, es) || !aligned(dbias, 4))
        return MEC_ERR_ALIGNMENT;
    const GradPlan plan = grad_plan(rows, i_c, k_c, dtype, act);
    if ((dX || dK || dbias) && plan.bytes && (!workspace || (uint64_t)workspace_bytes < (uint64_t)plan.bytes))
        return MEC_ERR_WORKSPACE;
    if (!aligned(workspace, 4)) return MEC_ERR_ALIGNMENT;
    if ((dX && plan.x.kernel < 0) || (dK && plan.k.kernel < 0)) return MEC_ERR_UNSUPPORTED;  // (the same with other operands)
    const hipStream_t st = (hipStream_t)stream;
    float* const part = static_cast<float*>(workspace);
    char* const low = plan.two && (dX || dK) ? reinterpret_cast<char*>(((uintptr_t)workspace + plan.sums + 15) / 16 * 16) : nullptr;
    clear_stale_error();
    if (act != MEC_ACT_NONE || dbias) {
        rc = hip_status(mec::launch_act_grad(G, g_pitch, Z, act == MEC_ACT_NONE ? nullptr : dZ, low, dbias, part, rows, k_c,
                                             act, dtype, st), "gradients of the activation and the bias");
        if (rc != MEC_OK) return rc;
    }
    const void* const dz = act == MEC_ACT_NONE ? G : dZ;
    const int64_t z_pitch = act == MEC_ACT_NONE ? g_pitch : k_c;
    mec::Product x{}, k{};
    x.alpha = k.alpha = 1.0f;
    x.batch = x.splits = k.batch = k.splits = 1;
    x.A = dz;
    x.lda = z_pitch;
    x.B = K;
    x.ldb = k_c;
    x.Y = dX;
    x.ldy = i_c;
    x.M = (int32_t)rows;
    x.N = i_c;
    x.K = k_c;
    k.A = X;
    k.lda = x_pitch;
    k.B = dz;
    k.ldb = z_pitch;
    k.Y = dK;
    k.ldy = k_c;
    k.M = i_c;
    k.N = k_c;
    k.K = (int32_t)rows;
    k.part = part;
    x.part = part;
    x.second = k.second = low ? (int64_t)((uintptr_t)low - (uintptr_t)dZ) : 0;
    const mec::ProductPlan px = mec::refine_plan(plan.x, mec::Layout::kXKt, dtype, x);
    const mec::ProductPlan pk = mec::refine_plan(plan.k, mec::Layout::kXtK, dtype, k);
    const GradRoute route = dX && dK ? grad_route(plan, px, pk, !dtype || (mec::clean_rows(mec::Layout::kXKt, x) &&
                                                                          mec::clean_rows(mec::Layout::kXtK, k)))
                                     : GradRoute::kApart;
    if (route == GradRoute::kSmallPair)
        return hip_status(mec::launch_product_small_pair(x, k, dtype, st), "gradients of the input and the kernel");
    if (route == GradRoute::kTilePair) {
        k.splits = plan.pair.splits;
        rc = hip_status(dtype ? mec::launch_product_bf16_pair(x, k, st) : mec::launch_product_f32_pair(x, k, st),
                        "gradients of the input and the kernel");
        if (rc == MEC_OK && k.splits > 1)
            rc = hip_status(mec::launch_sum_parts(part, k.splits, (int64_t)i_c * k_c, dK, dtype, st), "sum of the kernel's gradient");
        return rc;
    }
    if (dX) {
        rc = hip_status(launch_shared(px, mec::Layout::kXKt, x, dtype, st), "gradient of the input");
        if (rc != MEC_OK) return rc;
    }
    return dK ? hip_status(launch_shared(pk, mec::Layout::kXtK, k, dtype, st), "gradient of the kernel") : MEC_OK;
}

int mec_layer_norm(const void* X, const float* gamma, const float* beta, void* Y, float* mean, float* rstd, int64_t rows,
                   int channels, int64_t x_pitch, int64_t y_pitch, float eps, int dtype, void* stream) {
    const int rc = first_error({check_rows(rows, channels, x_pitch), check_rows(rows, channels, y_pitch)});
    if (rc != MEC_OK) return rc;
    if (!valid_dtype(dtype) || !X || !Y || !(eps >= 0.0f)) return MEC_ERR_INVALID_ARG;
    const int64_t es = elem_bytes(dtype);
    if (!aligned(X, es) || !aligned(Y, es) || !aligned(gamma, 4) || !aligned(beta, 4) || !aligned(mean, 4) || !aligned(rstd, 4))
        return MEC_ERR_ALIGNMENT;
    clear_stale_error();
    return hip_status(mec::launch_norm(X, x_pitch, gamma, beta, Y, y_pitch, mean, rstd, rows, channels, eps, dtype,
                                       (hipStream_t)stream), "layer norm");
}

int64_t mec_layer_norm_grad_workspace_bytes(int64_t rows, int channels, int dtype) {
    const int rc = check_rows(rows, channels, channels);
    if (rc != MEC_OK) return rc;
    if (!valid_dtype(dtype)) return MEC_ERR_INVALID_ARG;
    return mec::norm_grad_blocks(rows) * 2 * channels * 4;
}

int mec_layer_norm_grad(const void* G, const void* X, const float* gamma, const float* mean, const float* rstd, void* dX,
                        float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes, int64_t rows, int channels,
                        int64_t g_pitch, int64_t x_pitch, int dtype, void* stream) {
    const int rc = first_error({check_rows(rows, channels, g_pitch), check_rows(rows, channels, x_pitch)});
    if (rc != MEC_OK) return rc;
    if (!valid_dtype(dtype) || !G || !X || !mean || !rstd) return MEC_ERR_INVALID_ARG;
    const int64_t es = elem_bytes(dtype);
    if (!aligned(G, es) || !aligned(X, es) || !aligned(dX, es) || !aligned(gamma, 4) || !aligned(mean, 4) ||
        !aligned(rstd, 4) || !aligned(dgamma, 4) || !aligned(dbeta, 4))
        return MEC_ERR_ALIGNMENT;
    if ((dgamma || dbeta) &&
        (!workspace || (uint64_t)workspace_bytes < (uint64_t)mec_layer_norm_grad_workspace_bytes(rows, channels, dtype)))
        return MEC_ERR_WORKSPACE;
    if (!aligned(workspace, 4)) return MEC_ERR_ALIGNMENT;
    if (!dX && !dgamma && !dbeta) return MEC_OK;
    clear_stale_error();
    return hip_status(mec::launch_norm_grad(G, g_pitch, X, x_pitch, gamma, mean, rstd, dX, dgamma, dbeta,
                                            static_cast<float*>(workspace), rows, channels, dtype, (hipStream_t)stream),
                      "layer norm gradients");
}

namespace {

int check_stack(int batch, int rows, int cols, int dtype) {
    if (batch < 1 || rows < 1 || cols < 1 || !valid_dtype(dtype)) return MEC_ERR_INVALID_ARG;
    if (batch > 65535 || rows > kMaxWidth || cols > kMaxWidth) return MEC_ERR_UNSUPPORTED;
    return checked_product({batch, rows, cols}) < 0 ? MEC_ERR_INVALID_ARG : MEC_OK;
}

}  // namespace

int64_t mec_orthogonalize_workspace_bytes(int batch, int rows, int cols, int dtype) {
    const int rc = check_stack(batch, rows, cols, dtype);
    return rc != MEC_OK ? rc : mec::orth_workspace_bytes(batch, rows, cols, dtype);
}

int mec_orthogonalize(const void* U, void* O, void* workspace, size_t workspace_bytes, int batch, int rows, int cols,
                      int steps, float a, float b, float c, float eps, int dtype, void* stream) {
    const int rc = check_stack(batch, rows, cols, dtype);
    if (rc != MEC_OK) return rc;
    if (!U || !O || steps < 1 || steps > 100 || !(eps >= 0.0f)) return MEC_ERR_INVALID_ARG;
    const int64_t es = elem_bytes(dtype);
    if (!aligned(U, es) || !aligned(O, es)) return MEC_ERR_ALIGNMENT;
    if (!workspace || (uint64_t)workspace_bytes < (uint64_t)mec::orth_workspace_bytes(batch, rows, cols, dtype))
        return MEC_ERR_WORKSPACE;
    clear_stale_error();
    return hip_status(mec::launch_orth(U, O, workspace, batch, rows, cols, steps, a, b, c, eps, dtype, (hipStream_t)stream),
                      "orthogonalisation");
}

// ---------------------------------------------------------------- for the tests
// What mec_internal.h declares for them: the kernel that a call takes, and a call of one
// kernel on any shape that it holds.

int mec_internal_gemm_route(const void* I, const void* K, int i_n, int i_h, int i_w, int i_c, int k_h, int k_w, int k_c,
                            int s_h, int s_w, int dtype, int algo, int* from_input) {
    mec::Shape s;
    const int rc = make_shape(s, i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w);
    if (rc != MEC_OK) return rc;
    if (!valid_dtype(dtype) || (algo != MEC_ALGO_LOWERED && algo != MEC_ALGO_FUSED && algo != -1))
        return MEC_ERR_INVALID_ARG;
    const bool fused = algo == MEC_ALGO_FUSED || (algo == MEC_ALGO_LOWERED && mec::gemm_from_input(s, I, K, dtype));
    if (from_input) *from_input = fused;
    return (int)mec::gemm_route(s, I, K, dtype, fused, nullptr);
}

int mec_internal_gemm(int kernel, const void* A, const void* K, float* O, int i_n, int i_h, int i_w, int i_c, int k_h,
                      int k_w, int k_c, int s_h, int s_w, int dtype, int fused, void* stream) {
    mec::Shape s;
    const int rc = make_shape(s, i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w);
    if (rc != MEC_OK) return rc;
    if (!valid_dtype(dtype) || !A || !K || !O) return MEC_ERR_INVALID_ARG;
    const int64_t es = elem_bytes(dtype);
    if (!aligned(A, es) || !aligned(K, es) || !aligned(O, 4)) return MEC_ERR_ALIGNMENT;
    bool holds = false;
    switch ((mec::GemmKernel)kernel) {
        case mec::GemmKernel::kSmall: holds = mec::gemm_small_holds(s, dtype, fused); break;
        case mec::GemmKernel::kFirst: holds = dtype == MEC_BF16 && fused && mec::gemm_first_holds(s, A); break;
        case mec::GemmKernel::kPatch: holds = dtype == MEC_BF16 && fused && mec::gemm_patch_holds(s, A, K); break;
        case mec::GemmKernel::kTile: holds = dtype == MEC_F32 && mec::gemm_tile_holds(s, fused, nullptr); break;
        case mec::GemmKernel::kFixed: holds = mec::gemm_supported(s, dtype, fused); break;
        default: return MEC_ERR_INVALID_ARG;
    }
    if (!holds) return MEC_ERR_UNSUPPORTED;
    clear_stale_error();
    return hip_status(mec::launch_gemm_by((mec::GemmKernel)kernel, s, A, K, O, dtype, fused, (hipStream_t)stream),
                      "one kernel's slab products");
}

int mec_internal_wgrad(int kernel, const void* A, const float* G, float* dK, void* workspace, size_t workspace_bytes,
                       int i_n, int i_h, int i_w, int i_c, int k_h, int k_w, int k_c, int s_h, int s_w, int fused,
                       void* stream) {
    mec::Shape s;
    const int rc = grad_shape(s, i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w, MEC_F32);
    if (rc != MEC_OK) return rc;
    if (!A || !G || !dK) return MEC_ERR_INVALID_ARG;
    if (!aligned(A, 4) || !aligned(G, 4) || !aligned(dK, 4) || !aligned(workspace, 4)) return MEC_ERR_ALIGNMENT;
    if (!mec::wgrad_supported(s)) return MEC_ERR_UNSUPPORTED;
    if (!workspace || (uint64_t)workspace_bytes < (uint64_t)mec::wgrad_partial_bytes(s)) return MEC_ERR_WORKSPACE;
    switch ((mec::WgradKernel)kernel) {
        case mec::WgradKernel::kTile: if (!mec::wgrad_tile_holds(s)) return MEC_ERR_UNSUPPORTED; break;
        case mec::WgradKernel::kSlab: if (!mec::wgrad_slab_ok(s)) return MEC_ERR_UNSUPPORTED; break;
        case mec::WgradKernel::kGeneral: if (mec::wgrad_slab_ok(s)) return MEC_ERR_UNSUPPORTED; break;
        default: return MEC_ERR_INVALID_ARG;
    }
    clear_stale_error();
    return hip_status(mec::launch_wgrad_by((mec::WgradKernel)kernel, s, static_cast<const float*>(A), G,
                                           static_cast<float*>(workspace), dK, (hipStream_t)stream, fused),
                      "one kernel's wgrad products");
}

int mec_internal_product_with(int kernel, int layout, int dtype, int M, int N, int K, const mec_internal_operands* o, void* stream) {
    if (layout < 0 || layout > 2 || !valid_dtype(dtype) || !o || !o->A || !o->B || !o->Y || M < 1 || N < 1 || K < 1 ||
        o->splits < 1 || (o->splits > 1 && !o->part) || o->batch < 1 || !valid_act(o->act))
        return MEC_ERR_INVALID_ARG;
    mec::Product p{};
    p.A = o->A;
    p.B = o->B;
    p.Y = o->Y;
    p.Z = o->Z;
    p.R = o->R;
    p.bias = o->bias;
    p.part = o->part;
    p.lda = o->lda;
    p.ldb = o->ldb;
    p.ldy = o->ldy;
    p.ldz = o->ldz;
    p.ldr = o->ldr;
    p.M = M;
    p.N = N;
    p.K = K;
    p.act = o->act;
    p.res_first = o->res_first;
    p.alpha = o->alpha;
    p.beta = o->beta;
    p.diag = o->diag;
    p.batch = o->batch;
    p.a_batch = o->a_batch;
    p.b_batch = o->b_batch;
    p.y_batch = p.r_batch = (int64_t)M * o->ldy;
    p.symmetric = o->symmetric;
    p.second = o->second;
    clear_stale_error();
    const hipStream_t st = (hipStream_t)stream;
    const hipError_t e = mec::launch_product({kernel, o->splits, 0.0}, (mec::Layout)layout, p, dtype, st);
    if (e == hipErrorNotSupported) return MEC_ERR_UNSUPPORTED;
    const int rc = hip_status(e, "one kernel's product");
    if (rc != MEC_OK || o->splits == 1) return rc;
    return hip_status(mec::launch_sum_parts(o->part, o->splits, (int64_t)o->batch * M * N, o->Y, dtype, st), "sum");
}

int mec_internal_orth_pairs(int batch, int rows, int cols, int steps, float a, float b, float c) {
    return mec::orth_pairs(batch, rows, cols, steps, a, b, c);
}

int mec_internal_orth_plan(int batch, int rows, int cols, int gram) {
    const mec::ProductPlan p = mec::orth_plan(batch, rows, cols, gram != 0);
    return p.kernel < 0 ? MEC_ERR_UNSUPPORTED : p.kernel + 16 * p.splits;
}

int mec_internal_linear_grad_route(int rows, int i_c, int k_c, int dtype, int act) {
    if (rows < 1 || i_c < 1 || k_c < 1 || !valid_dtype(dtype) || !valid_act(act)) return MEC_ERR_INVALID_ARG;
    const GradPlan g = grad_plan(rows, i_c, k_c, dtype, act);
    const bool clean = !dtype || (i_c % 8 == 0 && k_c % 8 == 0);
    mec::Operands with;
    with.clean = clean;
    with.two = g.two;
    auto refined = [&](const mec::ProductPlan& p, mec::Layout layout, int M, int N, int K) {
        return clean ? p : mec::plan_product(layout, dtype, M, N, K, 1, p.splits, false, with);
    };
    const mec::ProductPlan px = refined(g.x, mec::Layout::kXKt, rows, i_c, k_c), pk = refined(g.k, mec::Layout::kXtK, i_c, k_c, rows);
    const GradRoute route = grad_route(g, px, pk, clean);
    return (int)route + 16 * (route == GradRoute::kTilePair ? g.pair.splits : pk.splits);
}

int mec_internal_dword_granule(int odd, int k) {
    const mec::DwordGranule g = mec::dword_granule(odd != 0, k);
    return (k + g.wide) | (k + g.single) << 16;
}

int mec_internal_product_plan(int layout, int dtype, int M, int N, int K, int batch, int may_split) {
    const mec::ProductPlan p = mec::plan_product((mec::Layout)layout, dtype, M, N, K, batch, may_split ? kMaxShares : 1);
    return p.kernel < 0 ? MEC_ERR_UNSUPPORTED : p.kernel + 16 * p.splits;
}

int mec_internal_product(int kernel, int layout, const void* A, const void* B, void* Y, float* part, int splits, int M, int N,
                         int K, int64_t lda, int64_t ldb, int64_t ldy, int dtype, void* stream) {
    if (layout < 0 || layout > 2 || !valid_dtype(dtype) || !A || !B || !Y || M < 1 || N < 1 || K < 1 || splits < 1 ||
        (splits > 1 && !part))
        return MEC_ERR_INVALID_ARG;
    mec::Product p{};
    p.A = A;
    p.B = B;
    p.Y = Y;
    p.part = part;
    p.lda = lda;
    p.ldb = ldb;
    p.ldy = ldy;
    p.M = M;
    p.N = N;
    p.K = K;
    p.alpha = 1.0f;
    p.batch = 1;
    clear_stale_error();
    const hipError_t e = mec::launch_product({kernel, splits, 0.0}, (mec::Layout)layout, p, dtype, (hipStream_t)stream);
    if (e == hipErrorNotSupported) return MEC_ERR_UNSUPPORTED;
    int rc = hip_status(e, "one kernel's product");
    if (rc == MEC_OK && splits > 1)
        rc = hip_status(mec::launch_sum_parts(part, splits, (int64_t)M * N, Y, dtype, (hipStream_t)stream), "sum");
    return rc;
}

int mec_internal_wgrad_route(int i_n, int i_h, int i_w, int i_c, int k_h, int k_w, int k_c, int s_h, int s_w) {
    mec::Shape s;
    const int rc = grad_shape(s, i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w, MEC_F32);
    if (rc != MEC_OK) return rc;
    return (int)mec::wgrad_route(s);
}

int mec_internal_dgrad_gemm(int tile, const float* G, const float* K, float* dL, int i_n, int i_h, int i_w, int i_c,
                            int k_h, int k_w, int k_c, int s_h, int s_w, void* stream) {
    mec::Shape s;
    const int rc = grad_shape(s, i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w, MEC_F32);
    if (rc != MEC_OK) return rc;
    if (!G || !K || !dL) return MEC_ERR_INVALID_ARG;
    if (!aligned(G, 4) || !aligned(K, 4) || !aligned(dL, 4)) return MEC_ERR_ALIGNMENT;
    if (tile ? !mec::dgrad_tile_holds(s) : !mec::dgrad_supported(s)) return MEC_ERR_UNSUPPORTED;
    clear_stale_error();
    return hip_status(tile ? mec::launch_dgrad_tile(s, G, K, dL, (hipStream_t)stream)
                           : mec::launch_dgrad_fp32(s, G, K, dL, (hipStream_t)stream),
                      "one kernel's dgrad products");
}

int64_t mec_noalloc_scratch_bytes(void) { return mec::kNoAllocScratchBytes; }

int mec_conv2d_wgrad_noalloc(const void* I, const float* G, float* dK, int i_n, int i_h, int i_w,
                             int i_c, int k_h, int k_w, int k_c, int s_h, int s_w, int dtype,
                             void* stream) {
    mec::Shape s;
    int rc = grad_shape(s, i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w, dtype);
    if (rc != MEC_OK) return rc;
    if (!I || !G || !dK) return MEC_ERR_INVALID_ARG;
    if (!aligned(I, 4) || !aligned(G, 4) || !aligned(dK, 4)) return MEC_ERR_ALIGNMENT;
    if (!mec::wgrad_supported(s)) return MEC_ERR_UNSUPPORTED;
    // the same partial sums as mec_conv2d_wgrad, in the static array
    if (mec::wgrad_partial_bytes(s) > mec::kNoAllocScratchBytes) return MEC_ERR_SCRATCH;
    const hipStream_t st = (hipStream_t)stream;
    clear_stale_error();
    void* part = nullptr;
    rc = hip_status(mec::noalloc_scratch(st, &part), "address of the static scratch");
    if (rc != MEC_OK) return rc;
    return hip_status(mec::launch_wgrad(s, static_cast<const float*>(I), G, static_cast<float*>(part), dK,
                                        st, true),
                      "wgrad products from I, partial sums in the static scratch");
}

const char* mec_strerror(int status) {
    switch (status) {
        case MEC_OK: return "success";
        case MEC_ERR_INVALID_ARG: return "invalid argument (dimension, stride, enum or pointer)";
        case MEC_ERR_WORKSPACE: return "workspace missing or smaller than mec_workspace_bytes";
        case MEC_ERR_ALIGNMENT: return "pointer not aligned to its element size";
        case MEC_ERR_HIP: return "HIP runtime error at kernel launch";
        case MEC_ERR_UNSUPPORTED: return "shape beyond this build's kernel limits";
        case MEC_ERR_SCRATCH: return "the call needs more than the library's static scratch holds";
        default: return "unknown status";
    }
}

const char* mec_last_error(void) { return g_last_error; }

}  // extern "C"
