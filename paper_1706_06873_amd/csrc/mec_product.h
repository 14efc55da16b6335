// Matrix products of the layer operators (mec_linear.hip in bf16, mec_linear_f32.hip in
// fp32): what they compute, and the epilogue that both share.
//
//   acc = A B, then per output (m, n), all in fp32:
//   z = alpha*acc + bias[n] (+ beta*R[m, n] with res_first) (+ diag where m = n),  Z = z,
//   Y = act(z) (+ beta*R[m, n] without it)
//
// A is M x K, stored [m][k] or [k][m]; B is K x N, stored [n][k] or [k][n]: the layouts of
// Y = X K ([m][k], [k][n]), dX = dZ K^T ([m][k], [n][k]) and dK = X^T dZ ([k][m], [k][n]).
#pragma once

#include <stdint.h>

#include "mec_internal.h"

namespace mec {

enum class Layout { kXK = 0, kXKt = 1, kXtK = 2 };  // the three above

enum Act { kActNone = 0, kActRelu = 1, kActSilu = 2, kActGelu = 3 };

struct Product {
    const void* A;
    const void* B;
    void* Y;
    void* Z;         // or nullptr
    const void* R;   // or nullptr
    const float* bias;  // or nullptr
    float* part;     // with splits > 1: splits x batch x M x N partial sums in place of Y
    int64_t lda, ldb, ldy, ldz, ldr;  // elements per row as stored
    int32_t M, N, K;
    int32_t act, res_first;
    float alpha, beta;
    int32_t splits;  // of the reduction
    int32_t batch;   // equal products, the strides below apart (elements)
    int64_t a_batch, b_batch, y_batch, r_batch;
    float diag;      // added to z where m = n
    int32_t symmetric;  // A B and R are symmetric (fp32, no act): the 64 x 64 tiles leave out those above the diagonal
    int32_t y_bf16;  // fp32 products: Y is bf16
    // bf16, dX and dK: dZ is the sum of two matrices alike, the second (what rounding it to bf16
    // left over) this many bytes from the first; 0: one matrix
    int64_t second;

    // filled by the launch
    int32_t m_tiles, n_tiles, chunks;  // chunks of the reduction per split
    int32_t clean;                     // 16-byte rows of A and B
};

// What a launch holds in one dimension of its grid.
constexpr int64_t kMaxThreads = (int64_t(1) << 32) - 1;

// Which kernel computes a product, and the shares of its reduction.
struct ProductPlan {
    int kernel;  // 0 the small one, from 1 the tiles; -1: more outputs than a launch of any holds
    int32_t splits;
    double us;   // by the model
};
// What the sizes do not say: 16-byte rows (clean), a residual, a saved argument of the
// activation, dZ in two parts.
struct Operands {
    bool clean = true, R = false, Z = false, two = false;
};
// max_splits: as many shares as the caller has room for partial sums (batch x M x N each)
ProductPlan plan_product(Layout layout, int dtype, int64_t M, int64_t N, int64_t K, int32_t batch, int32_t max_splits,
                         bool symmetric = false, const Operands& with = {});
// the plan by the sizes alone, for the operands as they are: in no more shares
ProductPlan refine_plan(const ProductPlan& plan, Layout layout, int dtype, const Product& p);
// dX (rows x i_c) and dK (i_c x k_c) by tiles in one launch: kernel 3 and dK's shares, or
// kernel 0 where two launches by those plans are as fast, or one does not hold both
ProductPlan plan_pair(const ProductPlan& x, const ProductPlan& k, int dtype, int64_t rows, int64_t i_c, int64_t k_c,
                      int32_t max_splits, bool two);
// A's and B's rows are whole 16-byte granules (bf16)
bool clean_rows(Layout layout, const Product& p);

// Granule k .. k + 7 of a row of more than 8 bf16 elements by whole dwords, without a byte from
// outside the row: 16 bytes from element k + wide on, and element k + single by itself. `odd`: the
// granule begins inside a dword.
struct DwordGranule {
    int32_t wide, single;
};
constexpr DwordGranule dword_granule(bool odd, int32_t k) {
    return !odd ? DwordGranule{0, 7} : k == 0 ? DwordGranule{1, 0} : DwordGranule{-1, 7};
}

// Enqueue the product (dtype of A, B, Z, R, Y), with p.splits shares that leave their partial
// sums where it is above 1. hipErrorNotSupported where there is no such kernel.
hipError_t launch_product(const ProductPlan& plan, Layout layout, Product p, int dtype, hipStream_t stream);
hipError_t launch_product_bf16(Layout layout, Product p, int tile, hipStream_t stream);  // mec_linear.hip
hipError_t launch_product_f32(Layout layout, Product p, int tile, hipStream_t stream);   // mec_linear_f32.hip
constexpr int64_t kMaxSmallBlocks = 0x1fffff;  // of 1024 threads, in a launch
hipError_t launch_product_small(Layout layout, Product p, int dtype, hipStream_t stream);  // mec_linear_small.hip
// A step of the orthogonalisation from A = X X^T or X^T X (m x m) in one launch.
constexpr int kOrthStepMax = 128;  // m
struct OrthStep {
    const float* A;
    const float* X;
    void* Y;  // not X; bf16 where bf16
    int32_t m, rows, cols, bf16;
    float a, b, c;
};
hipError_t launch_orth_step(const OrthStep& p, int32_t batch, hipStream_t stream);
// the two products of a backward pass, x of layout kXKt (in one share) and k of kXtK, in one launch:
// by 64 x 64 tiles, 64 x 128 tiles (clean rows), or both small
hipError_t launch_product_f32_pair(Product x, Product k, hipStream_t stream);
hipError_t launch_product_bf16_pair(Product x, Product k, hipStream_t stream);
hipError_t launch_product_small_pair(Product x, Product k, int dtype, hipStream_t stream);
// by the plan, in one share
hipError_t launch_product(Layout layout, const Product& p, int dtype, hipStream_t stream);

// Y, Z of a product (one, not a batch) from the sums of its shares in p.part
hipError_t launch_finish_parts(const Product& p, int dtype, hipStream_t stream);
// out[j] = sum over i < count of part[i*n + j], in a fixed order; out fp32 or bf16
hipError_t launch_sum_parts(const float* part, int64_t count, int64_t n, void* out, int dtype, hipStream_t stream);
// the same for 2 n columns, the first n to out and the others to out2 (either may be nullptr)
hipError_t launch_sum_pairs(const float* part, int64_t count, int64_t n, float* out, float* out2, hipStream_t stream);

// dZ = G act'(Z) (dZ nullptr: act is none and dZ is G) and, unless nullptr, low, what rounding
// dZ to bf16 left over, rounded to bf16 (both dense), and dbias, by way of the partial column
// sums of act_grad_shares shares of the rows in part
int32_t act_grad_shares(int64_t rows, int64_t N);
hipError_t launch_act_grad(const void* G, int64_t ldg, const void* Z, void* dZ, void* low, float* dbias, float* part,
                           int64_t rows, int32_t N, int act, int dtype, hipStream_t stream);

// mec_norm.hip
hipError_t launch_norm(const void* X, int64_t ldx, const float* gamma, const float* beta, void* Y, int64_t ldy, float* mean,
                       float* rstd, int64_t rows, int32_t C, float eps, int dtype, hipStream_t stream);
int64_t norm_grad_blocks(int64_t rows);  // each leaves 2 C partial sums
hipError_t launch_norm_grad(const void* G, int64_t ldg, const void* X, int64_t ldx, const float* gamma, const float* mean,
                            const float* rstd, void* dX, float* dgamma, float* dbeta, float* part, int64_t rows, int32_t C,
                            int dtype, hipStream_t stream);

// mec_orth.hip
ProductPlan orth_plan(int32_t batch, int64_t rows, int64_t cols, bool gram);  // of its Gram matrices, or its squares
bool orth_pairs(int32_t batch, int64_t rows, int64_t cols, int32_t steps, float a, float b, float c);  // steps in pairs
int64_t orth_workspace_bytes(int32_t batch, int64_t rows, int64_t cols, int dtype);
hipError_t launch_orth(const void* U, void* O, void* workspace, int32_t batch, int64_t rows, int64_t cols, int32_t steps,
                       float a, float b, float c, float eps, int dtype, hipStream_t stream);

}  // namespace mec

#if defined(__HIP__)
#include "mec_mfma.h"

namespace mec {

typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));
typedef float f32x4v __attribute__((ext_vector_type(4)));

// e^x and 1/x: within an ulp or two of the type for fp32 outputs; for bf16 outputs (FAST) the
// hardware's exp2 and reciprocal, whose 2^-22 or so (e^x: 2^-24 |x|) the rounding covers
template <bool FAST>
__device__ inline float exp_of(float x) { return FAST ? __expf(x) : expf(x); }
template <bool FAST>
__device__ inline float reciprocal(float x) { return FAST ? __builtin_amdgcn_rcpf(x) : 1.0f / x; }

constexpr float kGeluC = 0.7978845608028654f, kGeluA = 0.044715f;  // sqrt(2/pi)

// act(z), with s(x) = 1 / (1 + e^-x). GELU is the tanh form, z/2 (1 + tanh(c (z + a z^3)))
// = z s(2 c (z + a z^3)), which keeps its relative accuracy where tanh nears -1. NaN stays
// NaN in all of them.
template <bool FAST>
__device__ inline float act_value(int act, float z) {
    if (act == kActRelu) return z < 0.0f ? 0.0f : z;
    if (act == kActNone) return z;
    const float t = act == kActSilu ? z : 2.0f * kGeluC * (z + kGeluA * z * z * z);
    return z * reciprocal<FAST>(1.0f + exp_of<FAST>(-t));
}
// act'(z) for the two smooth ones. s (1 - s) is taken as e^-|t| s(|t|)^2, without the
// cancellation of 1 - s; past |z| = 12 GELU's slope is 0 or 1 to fp32 (s (1 - s) < e^-100)
// where z^3 may overflow.
template <bool FAST>
__device__ inline float act_slope(int act, float z) {
    if (act == kActGelu && fabsf(z) > 12.0f) return z > 0.0f ? 1.0f : 0.0f;
    const float t = act == kActSilu ? z : 2.0f * kGeluC * (z + kGeluA * z * z * z);
    const float e = exp_of<FAST>(-fabsf(t)), r = reciprocal<FAST>(1.0f + e);
    const float s = t < 0.0f ? e * r : r, q = e * r * r;
    if (act == kActSilu) return q == 0.0f ? s : s + z * q;
    return s + z * q * (2.0f * kGeluC) * (1.0f + 3.0f * kGeluA * z * z);
}

__device__ inline float to_float(uint16_t x) { return __builtin_bit_cast(float, (uint32_t)x << 16); }
__device__ inline float to_float(float x) { return x; }
template <class E>
__device__ inline E from_float(float x);
template <>
__device__ inline float from_float<float>(float x) { return x; }
template <>
__device__ inline uint16_t from_float<uint16_t>(float x) {  // to nearest even
    return __builtin_bit_cast(uint16_t, (__bf16)x);
}

// 8 consecutive elements of a 16-byte aligned row
__device__ inline void load8v(const uint16_t* src, float* v) {
    const u32x4v w = *reinterpret_cast<const u32x4v*>(src);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[2 * e] = __builtin_bit_cast(float, w[e] << 16);
        v[2 * e + 1] = __builtin_bit_cast(float, w[e] & 0xffff0000u);
    }
}
__device__ inline void load8v(const float* src, float* v) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const f32x4v w = *reinterpret_cast<const f32x4v*>(src + 4 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * h + e] = w[e];
    }
}
__device__ inline void store8v(uint16_t* dst, const float* v) {
    u32x4v w;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        w[e] = (uint32_t)from_float<uint16_t>(v[2 * e]) | (uint32_t)from_float<uint16_t>(v[2 * e + 1]) << 16;
    *reinterpret_cast<u32x4v*>(dst) = w;
}
__device__ inline void store8v(float* dst, const float* v) {
#pragma unroll
    for (int h = 0; h < 2; ++h) *reinterpret_cast<f32x4v*>(dst + 4 * h) = f32x4v{v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
}

// 16 bytes at any 2-byte boundary
__device__ inline u32x4v load_any(const uint16_t* src) {
    struct __attribute__((packed, aligned(2))) Any {
        u32x4v v;
    };
    return reinterpret_cast<const Any*>(src)->v;
}
// its first `have` elements, then zeros: 8, 4 and 2 bytes, as `have` is made of
__device__ inline u32x4v load_some(const uint16_t* src, int64_t have) {
    if (have >= 8) return load_any(src);
    typedef uint32_t u32x2v __attribute__((ext_vector_type(2)));
    struct __attribute__((packed, aligned(2))) Any2 {
        u32x2v v;
    };
    struct __attribute__((packed, aligned(2))) Any1 {
        uint32_t v;
    };
    u32x4v w = {0, 0, 0, 0};
    if (have <= 0) return w;
    const int n = (int)have, two = n & 4, one = n & 6;
    uint32_t pair = 0, last = 0;
    if (n & 4) {
        const u32x2v x = reinterpret_cast<const Any2*>(src)->v;
        w[0] = x[0];
        w[1] = x[1];
    }
    if (n & 2) pair = reinterpret_cast<const Any1*>(src + two)->v;
    if (n & 1) last = src[one];
    // pair goes to dword two / 2 (0 or 2), last to dword one / 2
    if (n & 2) {
        if (two) w[2] = pair;
        else w[0] = pair;
    }
    if (n & 1) {
        if (one == 0) w[0] = last;
        else if (one == 2) w[1] = last;
        else if (one == 4) w[2] = last;
        else w[3] = last;
    }
    return w;
}
// the first `have` of 8 elements to memory, likewise
__device__ inline void store_some(uint16_t* dst, u32x4v w, int have) {
    typedef uint32_t u32x2v __attribute__((ext_vector_type(2)));
    struct __attribute__((packed, aligned(2))) Any4 {
        u32x4v v;
    };
    struct __attribute__((packed, aligned(2))) Any2 {
        u32x2v v;
    };
    struct __attribute__((packed, aligned(2))) Any1 {
        uint32_t v;
    };
    if (have >= 8) {
        reinterpret_cast<Any4*>(dst)->v = w;
    } else if (have > 0) {
        const int two = have & 4, one = have & 6;
        if (have & 4) reinterpret_cast<Any2*>(dst)->v = u32x2v{w[0], w[1]};
        if (have & 2) reinterpret_cast<Any1*>(dst + two)->v = two ? w[2] : w[0];
        if (have & 1) dst[one] = (uint16_t)(one == 0 ? w[0] : one == 2 ? w[1] : one == 4 ? w[2] : w[3]);
    }
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;

// Transposing read of 4 k for each of 16 columns: lane p of 16 gives the address of columns
// 4*(p % 4) .. + 3 of row k + p / 4, and gets rows k .. k + 3 of column p.
__device__ inline s16x4 read_tr(const char* at) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(lds_char*)at);
}
__device__ inline bf16x8 join_tr(s16x4 a, s16x4 b) {
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// one output (m, n) from its sum v
template <class E>
__device__ inline void finish(const Product& p, int64_t m, int32_t n, int32_t bat, float v) {
    constexpr bool FAST = sizeof(E) == 2;
    const float r = p.R ? p.beta * to_float(static_cast<const E*>(p.R)[bat * p.r_batch + m * p.ldr + n]) : 0.0f;
    v *= p.alpha;
    if (p.bias) v += p.bias[n];
    if (p.R && p.res_first) v += r;
    if (m == n) v += p.diag;
    if (p.Z) static_cast<E*>(p.Z)[m * p.ldz + n] = from_float<E>(v);
    if (p.act == kActRelu) v = act_value<FAST>(kActRelu, v);
    else if (p.act == kActSilu) v = act_value<FAST>(kActSilu, v);
    else if (p.act == kActGelu) v = act_value<FAST>(kActGelu, v);
    if (p.R && !p.res_first) v += r;
    const int64_t at = bat * p.y_batch + m * p.ldy + n;
    if (sizeof(E) == 4 && p.y_bf16) static_cast<uint16_t*>(p.Y)[at] = from_float<uint16_t>(v);
    else static_cast<E*>(p.Y)[at] = from_float<E>(v);
}

// the operands of product `bat` of a batch
template <class E>
__device__ inline const E* a_of(const Product& p, int32_t bat) {
    return static_cast<const E*>(p.A) + bat * p.a_batch;
}
template <class E>
__device__ inline const E* b_of(const Product& p, int32_t bat) {
    return static_cast<const E*>(p.B) + bat * p.b_batch;
}

// 8 elements as they lie in memory, at any boundary of the element's size
template <class E>
struct Pack8 {
    static constexpr int W = sizeof(E) / 2;
    struct __attribute__((packed, aligned(sizeof(E)))) Any {
        u32x4v v;
    };
    u32x4v w[W];
    // the first `have` of them
    __device__ inline void load(const E* src, int have) {
        if constexpr (sizeof(E) == 2) {
            w[0] = load_some(src, have);
        } else if (have >= 8) {
#pragma unroll
            for (int i = 0; i < W; ++i) w[i] = reinterpret_cast<const Any*>(src)[i].v;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < have) w[e / 4][e % 4] = __builtin_bit_cast(uint32_t, src[e]);
        }
    }
    __device__ inline void store(E* dst, int have) const {
        if constexpr (sizeof(E) == 2) {
            store_some(dst, w[0], have);
        } else if (have >= 8) {
#pragma unroll
            for (int i = 0; i < W; ++i) reinterpret_cast<Any*>(dst)[i].v = w[i];
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < have) dst[e] = __builtin_bit_cast(float, (uint32_t)w[e / 4][e % 4]);
        }
    }
    __device__ inline float get(int e) const {
        if constexpr (sizeof(E) == 4) {
            return __builtin_bit_cast(float, (uint32_t)w[e / 4][e % 4]);
        } else {
            const uint32_t x = w[0][e / 2];
            return __builtin_bit_cast(float, e % 2 ? x & 0xffff0000u : x << 16);
        }
    }
    __device__ inline void round(const float* v) {
        if constexpr (sizeof(E) == 4) {
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e / 4][e % 4] = __builtin_bit_cast(uint32_t, v[e]);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                w[0][e] = (uint32_t)from_float<uint16_t>(v[2 * e]) | (uint32_t)from_float<uint16_t>(v[2 * e + 1]) << 16;
        }
    }
};

// A wave's BM x BN blocks of 32 x 32 sums, as the products leave them with B's columns as
// the instruction's rows (lane l holds m = l % 32 and, in register v, n = acc_row(v, l)),
// through `mine`, 32 rows of 32*BN + 4 floats of LDS that only this wave uses: rows are
// read back whole, so that Y, Z and R move in runs of 64*BN (bf16) or 128*BN bytes. The
// loads and LDS reads of 32 rows are all in flight at once (8192 x 8192 x 64 in bf16 37 us;
// 60 with 8 rows after another).
template <class E, int BM, int BN>
__device__ inline void epilogue(const Product& p, const floatx16 (&acc)[BM][BN], float* mine, int32_t m0, int32_t n0,
                                int32_t bat, int32_t split, int lane) {
    constexpr int PITCH = 32 * BN + 4, LPR = 4 * BN, RPP = 64 / LPR, PASSES = 32 / RPP;
    constexpr bool FAST = sizeof(E) == 2;
    const int row0 = lane / LPR, col = (lane % LPR) * 8;
    const int32_t have = p.N - n0 - col;  // columns from this lane's first on
    const int32_t rows = p.M - m0 - row0;
    const bool part = p.splits > 1, diagonal = p.diag != 0.0f;
    const bool half = sizeof(E) == 4 && p.y_bf16;
    const int64_t m = m0 + row0, n = n0 + col;
    const int64_t yat = bat * p.y_batch + m * p.ldy + n;
    E* const y = static_cast<E*>(p.Y) + yat;
    uint16_t* const y16 = static_cast<uint16_t*>(p.Y) + yat;
    E* const z = static_cast<E*>(p.Z) + m * p.ldz + n;
    const E* const r = static_cast<const E*>(p.R) + bat * p.r_batch + m * p.ldr + n;
    float* const q = p.part + (((int64_t)split * p.batch + bat) * p.M + m) * p.N + n;
    float bias[8] = {};
    if (p.bias && !part)
#pragma unroll
        for (int e = 0; e < 8; ++e) bias[e] = e < have ? p.bias[n + e] : 0.0f;
#pragma unroll
    for (int i = 0; i < BM; ++i) {
        Pack8<E> rr[PASSES];
        if (p.R && !part)
#pragma unroll
            for (int s = 0; s < PASSES; ++s)
                if (i * 32 + s * RPP < rows) rr[s].load(r + (i * 32 + s * RPP) * p.ldr, have);
        asm volatile("" ::: "memory");  // the wave's LDS accesses stay in this order
#pragma unroll
        for (int j = 0; j < BN; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                *reinterpret_cast<f32x4v*>(mine + (lane & 31) * PITCH + j * 32 + k * 8 + (lane >> 5) * 4) =
                    f32x4v{acc[i][j][4 * k], acc[i][j][4 * k + 1], acc[i][j][4 * k + 2], acc[i][j][4 * k + 3]};
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_wave_barrier();
        float v[PASSES][8];
#pragma unroll
        for (int s = 0; s < PASSES; ++s) load8v(mine + (s * RPP + row0) * PITCH + col, v[s]);
        if (part) {
#pragma unroll
            for (int s = 0; s < PASSES; ++s) {
                Pack8<float> o;
                o.round(v[s]);
                if (i * 32 + s * RPP < rows) o.store(q + (int64_t)(i * 32 + s * RPP) * p.N, have);
            }
        } else {
#pragma unroll
            for (int s = 0; s < PASSES; ++s)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[s][e] = v[s][e] * p.alpha + bias[e];
            if (p.R && p.res_first)
#pragma unroll
                for (int s = 0; s < PASSES; ++s)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[s][e] += p.beta * rr[s].get(e);
            if (diagonal)
#pragma unroll
                for (int s = 0; s < PASSES; ++s)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (m0 + i * 32 + s * RPP + row0 == n0 + col + e) v[s][e] += p.diag;
            if (p.Z)
#pragma unroll
                for (int s = 0; s < PASSES; ++s) {
                    Pack8<E> o;
                    o.round(v[s]);
                    if (i * 32 + s * RPP < rows) o.store(z + (i * 32 + s * RPP) * p.ldz, have);
                }
            if (p.act == kActRelu) {
#pragma unroll
                for (int s = 0; s < PASSES; ++s)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[s][e] = act_value<FAST>(kActRelu, v[s][e]);
            } else if (p.act == kActSilu) {
#pragma unroll
                for (int s = 0; s < PASSES; ++s)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[s][e] = act_value<FAST>(kActSilu, v[s][e]);
            } else if (p.act == kActGelu) {
#pragma unroll
                for (int s = 0; s < PASSES; ++s)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[s][e] = act_value<FAST>(kActGelu, v[s][e]);
            }
            if (p.R && !p.res_first)
#pragma unroll
                for (int s = 0; s < PASSES; ++s)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[s][e] += p.beta * rr[s].get(e);
#pragma unroll
            for (int s = 0; s < PASSES; ++s)
                if (i * 32 + s * RPP < rows) {
                    if (half) {
                        Pack8<uint16_t> o;
                        o.round(v[s]);
                        o.store(y16 + (i * 32 + s * RPP) * p.ldy, have);
                    } else {
                        Pack8<E> o;
                        o.round(v[s]);
                        o.store(y + (i * 32 + s * RPP) * p.ldy, have);
                    }
                }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_wave_barrier();
    }
}

// The mirror image of a wave's block of a symmetric Y (a tile below the diagonal): register v
// of the 32 lanes with one n holds 32 consecutive m, a run of a row of the image.
__device__ inline void mirror(const Product& p, const floatx16& acc, int32_t m0, int32_t n0, int32_t bat, int32_t split, int lane) {
    const int32_t m = m0 + (lane & 31);
    if (m >= p.M) return;
    const bool part = p.splits > 1;
    float r[16] = {};
    if (p.R && !part)
#pragma unroll
        for (int v = 0; v < 16; ++v) {  // all in flight at once, before any store that might change them
            const int64_t n = n0 + acc_row(v, lane);
            r[v] = static_cast<const float*>(p.R)[bat * p.r_batch + (n < p.N ? n : p.N - 1) * p.ldr + m];
        }
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        const int64_t n = n0 + acc_row(v, lane);
        if (n >= p.N) continue;
        if (part) p.part[(((int64_t)split * p.batch + bat) * p.M + n) * p.N + m] = acc[v];
        else static_cast<float*>(p.Y)[bat * p.y_batch + n * p.ldy + m] = acc[v] * p.alpha + p.beta * r[v];
    }
}
// Tile t of those of a symmetric Y on and below the diagonal, row by row
__device__ inline void tile_of_half(uint32_t t, uint32_t& mt, uint32_t& nt) {
    mt = (uint32_t)((sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
    while (mt * (mt + 1) / 2 > t) --mt;  // (the root is rounded)
    while ((mt + 1) * (mt + 2) / 2 <= t) ++mt;
    nt = t - mt * (mt + 1) / 2;
}

// Of dZ's two parts the second is finite, but times an infinity it makes a NaN where it is 0 or of
// the other sign. Where the operand that dZ is multiplied with holds an infinity, sums that are not
// finite are therefore taken again from the first part alone, which spreads infinities and NaNs as
// dZ does. (50176 x 512 -> 2048 with GELU, event to event: 728 us, with one NaN in G 992, NaNs alone
// 1765, an infinity in X and K 1873; every sum that was not finite taken again 2854 and 12213.)
__device__ inline bool not_finite(const floatx16& acc) {
    bool any = false;
#pragma unroll
    for (int v = 0; v < 16; ++v) any |= !__builtin_isfinite(acc[v]);
    return __any(any);
}
// whether a wave's 32 rows (or columns) of a matrix hold an infinity: this lane's, with its elements x_k apart
__device__ inline bool holds_infinity(const uint16_t* x, int64_t x_k, int32_t K, int lane) {
    bool any = false;
    for (int32_t s = 0; s < K; s += 32) {  // (past the end: its last element)
        uint32_t v[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int32_t k = s + 16 * (lane >> 5) + e;
            v[e] = x[(k < K ? k : K - 1) * x_k];
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) any |= (v[e] & 0x7fffu) == 0x7f80u;
    }
    return __any(any);
}
// the sums that are not finite, from memory: this lane's row of A and column of B
__device__ inline void take_again(floatx16& acc, const uint16_t* a, int64_t a_k, const uint16_t* b, int64_t b_k, int32_t K, int lane) {
    floatx16 sum = {};
#pragma clang loop unroll(disable)
    for (int32_t s = 0; s < K; s += 16) {
        uint32_t v[8], w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int32_t k = s + 8 * (lane >> 5) + e, at = k < K ? k : K - 1;
            v[e] = a[at * a_k];
            w[e] = b[at * b_k];
        }
        u32x4v x = {0, 0, 0, 0}, y = {0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (s + 8 * (lane >> 5) + e < K) {
                x[e / 2] |= v[e] << (e % 2 * 16);
                y[e / 2] |= w[e] << (e % 2 * 16);
            }
        sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, y), __builtin_bit_cast(bf16x8, x), sum, 0, 0, 0);
    }
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[v] = __builtin_isfinite(acc[v]) ? acc[v] : sum[v];
}

// Tile t of a grid of m_tiles x n_tiles: runs of `group` rows of tiles, column by column,
// so that the workgroups in flight share rows of A and columns of B in their XCD's L2.
__device__ inline void tile_of(uint32_t t, uint32_t m_tiles, uint32_t n_tiles, uint32_t group, uint32_t& mt, uint32_t& nt) {
    const uint32_t per = group * n_tiles, g = t / per, first = g * group;
    const uint32_t rows = m_tiles - first < group ? m_tiles - first : group;
    const uint32_t r = t - g * per;
    nt = r / rows;
    mt = first + r - nt * rows;
}

}  // namespace mec
#endif
