// Layer norm of rows of channels, forward and backward; fp32 or bf16, everything between in
// fp32.
//
//   y = (x - mu) rstd gamma + beta,  mu = mean(x),  rstd = 1 / sqrt(mean((x - mu)^2) + eps)
//   with xh = (x - mu) rstd and w = g gamma:
//   dx = rstd (w - mean(w) - xh mean(w xh)),  dgamma = sum_rows g xh,  dbeta = sum_rows g
//
// Bound by memory: each row is read once, into registers, by TPR threads that hold ITEMS
// vectors of it each; mean, then the squares about that mean (no difference of large sums),
// then the output. Rows longer than the registers hold are read again from the caches for
// each of these. The backward pass keeps a thread's own columns' sums in registers over all
// rows its workgroup takes, writes one row of partial sums per workgroup and adds those in
// a fixed order in a second launch; rows past 8192 channels in fp32 and 16384 in bf16, more than
// registers hold beside those sums, are read once for dgamma and dbeta and twice for dX, element by
// element: 4096 x 8192 in fp32 89 us (4.5 TB/s), x 8196 175 (2.3); 2048 x 16384 in bf16 54 (3.8), x
// 16392 110 (1.8). The forward pass, re-read from the caches past 16384 and 32768: 4096 x 8192 in
// fp32 51 (5.3), 1024 x 32768 82 (3.3).
#include "mec_product.h"

namespace mec {
namespace {

struct NormParams {
    const void* X;
    const void* G;        // backward
    const float* gamma;   // or nullptr: ones
    const float* beta;    // or nullptr: zeros
    void* Y;              // Y, or dX (or nullptr)
    float* mean;          // forward: written unless nullptr; backward: read
    float* rstd;
    float* part;          // backward: workgroups x 2 x C, or nullptr
    int64_t rows, ldx, ldg, ldy;
    int32_t C;
    float eps;
};

// V consecutive elements (16 bytes' worth) at any boundary of the element's size, of which
// `have` are the row's; the others come as zeros and are not written. (The same instructions
// as for 16-byte rows; single elements took 725 us where these take 221, 108934 rows of 1619
// in bf16.)
struct __attribute__((packed, aligned(4))) AnyF {
    f32x4v v;
};
template <int V, class E>
__device__ inline void load_v(const E* src, int have, float* v) {
    if constexpr (sizeof(E) == 2) {
        static_assert(V == 8, "16 bytes");
        const u32x4v w = load_some(src, have);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[2 * e] = __builtin_bit_cast(float, w[e] << 16);
            v[2 * e + 1] = __builtin_bit_cast(float, w[e] & 0xffff0000u);
        }
    } else if (have >= V) {
#pragma unroll
        for (int h = 0; h < V; h += 4) {
            const f32x4v w = reinterpret_cast<const AnyF*>(src + h)->v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[h + e] = w[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = e < have ? src[e] : 0.0f;
    }
}
template <int V, class E>
__device__ inline void store_v(E* dst, int have, const float* v) {
    if constexpr (sizeof(E) == 2) {
        Pack8<E> w;
        w.round(v);
        w.store(dst, have);
    } else if (have >= V) {
#pragma unroll
        for (int h = 0; h < V; h += 4) reinterpret_cast<AnyF*>(dst + h)->v = f32x4v{v[h], v[h + 1], v[h + 2], v[h + 3]};
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (e < have) dst[e] = v[e];
    }
}

// Sum of N values over the TPR threads of a row, in every one of them. `lds` holds two
// sets of waves x N floats that calls use in turn (`turn`), so that one barrier per call
// is enough: a set is written again only after the barrier of the call between.
template <int TPR, int THREADS, int N>
__device__ inline void row_sum(float (&v)[N], float* lds, int& turn) {
    constexpr int W = TPR < 64 ? TPR : 64;
#pragma unroll
    for (int s = W / 2; s > 0; s >>= 1)
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] += __shfl_xor(v[e], s, 64);
    if constexpr (TPR > 64) {
        constexpr int WAVES = TPR / 64;
        float* const set = lds + turn * (THREADS / 64) * N;
        turn ^= 1;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int e = 0; e < N; ++e) set[(threadIdx.x >> 6) * N + e] = v[e];
        __syncthreads();
        const float* const row = set + threadIdx.x / TPR * WAVES * N;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            float s = row[e];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) s += row[w * N + e];
            v[e] = s;
        }
    }
}

// TPR threads per row, ITEMS vectors of V elements each; ITEMS = 0: any length, re-read.
template <class E, int V, int TPR, int THREADS, int ITEMS>
__global__ __launch_bounds__(THREADS) void norm_kernel(NormParams p) {
    constexpr int RPB = THREADS / TPR;
    __shared__ float lds[TPR > 64 ? 2 * THREADS / 64 : 1];
    const int t = threadIdx.x % TPR;
    const float inv = 1.0f / (float)p.C;
    int turn = 0;
    auto squares = [&](float* v, int have, float mean, float& sq) {  // v about the mean, and their squares
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = e < have ? v[e] - mean : 0.0f;
#pragma unroll
        for (int e = 0; e < V; ++e) sq += v[e] * v[e];
    };
    auto finish = [&](float* v, E* y, int c, float rstd) {
        const int have = p.C - c;
        float g[V], b[V];
        if (p.gamma) load_v<V>(p.gamma + c, have, g);
        if (p.beta) load_v<V>(p.beta + c, have, b);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float o = v[e] * rstd;
            if (p.gamma) o *= g[e];
            if (p.beta) o += b[e];
            v[e] = o;
        }
        store_v<V>(y + c, have, v);
    };
    // every thread of a workgroup makes the same number of turns (the sums have barriers)
    for (int64_t first = (int64_t)blockIdx.x * RPB; first < p.rows; first += (int64_t)gridDim.x * RPB) {
        const int64_t row = first + threadIdx.x / TPR;
        const bool here = row < p.rows;
        const E* const x = static_cast<const E*>(p.X) + (here ? row : p.rows - 1) * p.ldx;
        E* const y = static_cast<E*>(p.Y) + row * p.ldy;
        float sum[1] = {0.0f}, sq[1] = {0.0f}, mean, rstd;
        if constexpr (ITEMS > 0) {
            float v[ITEMS][V];
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                const int c = (i * TPR + t) * V;
                load_v<V>(x + c, p.C - c, v[i]);
            }
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                for (int e = 0; e < V; ++e) sum[0] += v[i][e];
            row_sum<TPR, THREADS, 1>(sum, lds, turn);
            mean = sum[0] * inv;
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) squares(v[i], p.C - (i * TPR + t) * V, mean, sq[0]);
            row_sum<TPR, THREADS, 1>(sq, lds, turn);
            rstd = 1.0f / sqrtf(sq[0] * inv + p.eps);
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                const int c = (i * TPR + t) * V;
                if (here && c < p.C) finish(v[i], y, c, rstd);
            }
        } else {
            float v[V];
            for (int c = t * V; c < p.C; c += TPR * V) {
                load_v<V>(x + c, p.C - c, v);
#pragma unroll
                for (int e = 0; e < V; ++e) sum[0] += v[e];
            }
            row_sum<TPR, THREADS, 1>(sum, lds, turn);
            mean = sum[0] * inv;
            for (int c = t * V; c < p.C; c += TPR * V) {
                load_v<V>(x + c, p.C - c, v);
                squares(v, p.C - c, mean, sq[0]);
            }
            row_sum<TPR, THREADS, 1>(sq, lds, turn);
            rstd = 1.0f / sqrtf(sq[0] * inv + p.eps);
            for (int c = t * V; c < p.C; c += TPR * V) {
                load_v<V>(x + c, p.C - c, v);
#pragma unroll
                for (int e = 0; e < V; ++e) v[e] -= mean;
                finish(v, y, c, rstd);
            }
        }
        if (here && t == 0) {
            if (p.mean) p.mean[row] = mean;
            if (p.rstd) p.rstd[row] = rstd;
        }
    }
}

// The sums of a workgroup's row groups, joined in LDS a quantity at a time, to its row of
// partial sums.
template <int V, int TPR, int THREADS>
__device__ inline void join_columns(const float* v, float* lds, float* to, int c, int32_t C) {
    constexpr int RPB = THREADS / TPR;
    if constexpr (RPB > 1) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < V; ++e) lds[threadIdx.x * V + e] = v[e];
        __syncthreads();
        if (threadIdx.x < TPR && c < C) {
            float s[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                s[e] = v[e];
#pragma unroll
                for (int r = 1; r < RPB; ++r) s[e] += lds[(r * TPR + threadIdx.x) * V + e];
            }
            store_v<V>(to + c, C - c, s);
        }
    } else {
        if (c < C) store_v<V>(to + c, C - c, v);
    }
}

template <class E, int V, int TPR, int THREADS, int ITEMS>
__global__ __launch_bounds__(THREADS) void norm_grad_kernel(NormParams p) {
    constexpr int RPB = THREADS / TPR;
    constexpr int JOIN = RPB > 1 ? THREADS * V : 1, RED = TPR > 64 ? 4 * THREADS / 64 : 1;
    __shared__ float lds[JOIN > RED ? JOIN : RED];
    const int t = threadIdx.x % TPR;
    const float inv = 1.0f / (float)p.C;
    int turn = 0;
    float dg[ITEMS][V] = {}, db[ITEMS][V] = {};
    float gm[ITEMS][V];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int c = (i * TPR + t) * V;
        if (p.gamma) load_v<V>(p.gamma + c, p.C - c, gm[i]);
        else
#pragma unroll
            for (int e = 0; e < V; ++e) gm[i][e] = 1.0f;
    }
    for (int64_t first = (int64_t)blockIdx.x * RPB; first < p.rows; first += (int64_t)gridDim.x * RPB) {
        const int64_t at = first + threadIdx.x / TPR;
        const bool here = at < p.rows;
        const int64_t row = here ? at : p.rows - 1;
        const E* const x = static_cast<const E*>(p.X) + row * p.ldx;
        const E* const g = static_cast<const E*>(p.G) + row * p.ldg;
        const float mean = p.mean[row], rstd = p.rstd[row];
        float xh[ITEMS][V], w[ITEMS][V], sum[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int c = (i * TPR + t) * V;
            if (here && c < p.C) {
                load_v<V>(x + c, p.C - c, xh[i]);
                load_v<V>(g + c, p.C - c, w[i]);
#pragma unroll
                for (int e = 0; e < V; ++e) {  // (past the row's end g is 0)
                    xh[i][e] = (xh[i][e] - mean) * rstd;
                    dg[i][e] += w[i][e] * xh[i][e];
                    db[i][e] += w[i][e];
                    w[i][e] *= gm[i][e];
                    sum[0] += w[i][e];
                    sum[1] += w[i][e] * xh[i][e];
                }
            }
        }
        if (p.Y) {
            row_sum<TPR, THREADS, 2>(sum, lds, turn);
            const float mw = sum[0] * inv, mx = sum[1] * inv;
            E* const y = static_cast<E*>(p.Y) + row * p.C;
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                const int c = (i * TPR + t) * V;
                if (here && c < p.C) {
#pragma unroll
                    for (int e = 0; e < V; ++e) w[i][e] = rstd * (w[i][e] - mw - xh[i][e] * mx);
                    store_v<V>(y + c, p.C - c, w[i]);
                }
            }
        }
    }
    if (!p.part) return;
    float* const to = p.part + (int64_t)blockIdx.x * 2 * p.C;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int c = (i * TPR + t) * V;
        join_columns<V, TPR, THREADS>(dg[i], lds, to, c, p.C);
        join_columns<V, TPR, THREADS>(db[i], lds, to + p.C, c, p.C);
    }
}

// Rows longer than the registers hold: the partial sums of 256 columns ...
template <class E>
__global__ __launch_bounds__(256) void norm_columns_kernel(NormParams p, int64_t rows_per_share) {
    const int c = (int)(blockIdx.x * 256 + threadIdx.x);
    if (c >= p.C) return;
    const int64_t r0 = (int64_t)blockIdx.y * rows_per_share;
    const int64_t r1 = r0 + rows_per_share < p.rows ? r0 + rows_per_share : p.rows;
    float dg = 0.0f, db = 0.0f;
    for (int64_t r = r0; r < r1; ++r) {
        const float g = to_float(static_cast<const E*>(p.G)[r * p.ldg + c]);
        dg += g * ((to_float(static_cast<const E*>(p.X)[r * p.ldx + c]) - p.mean[r]) * p.rstd[r]);
        db += g;
    }
    float* const to = p.part + (int64_t)blockIdx.y * 2 * p.C;
    to[c] = dg;
    to[p.C + c] = db;
}
// ... and dX, a row per workgroup, read twice
template <class E>
__global__ __launch_bounds__(1024) void norm_long_grad_kernel(NormParams p) {
    __shared__ float lds[4 * 1024 / 64];
    const float inv = 1.0f / (float)p.C;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const E* const x = static_cast<const E*>(p.X) + row * p.ldx;
        const E* const g = static_cast<const E*>(p.G) + row * p.ldg;
        E* const y = static_cast<E*>(p.Y) + row * p.C;
        const float mean = p.mean[row], rstd = p.rstd[row];
        float sum[2] = {0.0f, 0.0f};
        for (int c = (int)threadIdx.x; c < p.C; c += 1024) {
            const float xh = (to_float(x[c]) - mean) * rstd, w = to_float(g[c]) * (p.gamma ? p.gamma[c] : 1.0f);
            sum[0] += w;
            sum[1] += w * xh;
        }
        row_sum<1024, 1024, 2>(sum, lds, turn);
        const float mw = sum[0] * inv, mx = sum[1] * inv;
        for (int c = (int)threadIdx.x; c < p.C; c += 1024) {
            const float xh = (to_float(x[c]) - mean) * rstd, w = to_float(g[c]) * (p.gamma ? p.gamma[c] : 1.0f);
            y[c] = from_float<E>(rstd * (w - mw - xh * mx));
        }
    }
}

constexpr int64_t kMaxBlocks = int64_t(1) << 21;

template <class E, int V, int TPR, int THREADS, int ITEMS>
hipError_t forward(const NormParams& p, hipStream_t stream) {
    const int64_t blocks = (p.rows + THREADS / TPR - 1) / (THREADS / TPR);
    hipLaunchKernelGGL((norm_kernel<E, V, TPR, THREADS, ITEMS>), dim3((uint32_t)(blocks < kMaxBlocks ? blocks : kMaxBlocks)),
                       dim3(THREADS), 0, stream, p);
    return hipGetLastError();
}

// Threads per row: as few as hold it in at most 4 vectors each, whole waves from 64 on.
template <class E, int V>
hipError_t forward(const NormParams& p, hipStream_t stream) {
    const int64_t v = (p.C + V - 1) / V;
    if (v <= 8) return forward<E, V, 8, 256, 1>(p, stream);
    if (v <= 16) return forward<E, V, 16, 256, 1>(p, stream);
    if (v <= 32) return forward<E, V, 32, 256, 1>(p, stream);
    if (v <= 64) return forward<E, V, 64, 256, 1>(p, stream);
    if (v <= 128) return forward<E, V, 64, 256, 2>(p, stream);
    if (v <= 256) return forward<E, V, 128, 256, 2>(p, stream);
    if (v <= 512) return forward<E, V, 256, 256, 2>(p, stream);
    if (v <= 1024) return forward<E, V, 256, 256, 4>(p, stream);
    if (v <= 2048) return forward<E, V, 512, 512, 4>(p, stream);
    if (v <= 4096) return forward<E, V, 1024, 1024, 4>(p, stream);
    return forward<E, V, 1024, 1024, 0>(p, stream);
}

template <class E, int V, int TPR, int THREADS, int ITEMS>
hipError_t backward(const NormParams& p, uint32_t blocks, hipStream_t stream) {
    hipLaunchKernelGGL((norm_grad_kernel<E, V, TPR, THREADS, ITEMS>), dim3(blocks), dim3(THREADS), 0, stream, p);
    return hipGetLastError();
}

template <class E, int V>
hipError_t backward(const NormParams& p, uint32_t blocks, hipStream_t stream) {
    const int64_t v = (p.C + V - 1) / V;
    if (v <= 8) return backward<E, V, 8, 256, 1>(p, blocks, stream);
    if (v <= 16) return backward<E, V, 16, 256, 1>(p, blocks, stream);
    if (v <= 32) return backward<E, V, 32, 256, 1>(p, blocks, stream);
    if (v <= 64) return backward<E, V, 64, 256, 1>(p, blocks, stream);
    if (v <= 128) return backward<E, V, 64, 256, 2>(p, blocks, stream);
    if (v <= 256) return backward<E, V, 128, 256, 2>(p, blocks, stream);
    if (v <= 512) return backward<E, V, 256, 256, 2>(p, blocks, stream);
    if (v <= 1024) return backward<E, V, 512, 512, 2>(p, blocks, stream);
    if (v <= 2048) return backward<E, V, 1024, 1024, 2>(p, blocks, stream);
    if (p.part) {
        const int64_t per = (p.rows + blocks - 1) / blocks;
        hipLaunchKernelGGL(norm_columns_kernel<E>, dim3((uint32_t)((p.C + 255) / 256), blocks), dim3(256), 0, stream, p, per);
    }
    if (p.Y)
        hipLaunchKernelGGL(norm_long_grad_kernel<E>, dim3((uint32_t)(p.rows < kMaxBlocks ? p.rows : kMaxBlocks)), dim3(1024), 0,
                           stream, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm(const void* X, int64_t ldx, const float* gamma, const float* beta, void* Y, int64_t ldy, float* mean,
                       float* rstd, int64_t rows, int32_t C, float eps, int dtype, hipStream_t stream) {
    NormParams p{};
    p.X = X;
    p.gamma = gamma;
    p.beta = beta;
    p.Y = Y;
    p.mean = mean;
    p.rstd = rstd;
    p.rows = rows;
    p.ldx = ldx;
    p.ldy = ldy;
    p.C = C;
    p.eps = eps;
    return dtype ? forward<uint16_t, 8>(p, stream) : forward<float, 4>(p, stream);
}

// Workgroups of the backward pass, each of which leaves 2 C partial sums: one per row up to
// 256 (49 rows of 2048: one per 16 rows 18.5 us, so 7.5), then one per 16 rows, so that the
// partial sums stay a small part of the traffic, up to 1024.
int64_t norm_grad_blocks(int64_t rows) {
    const int64_t few = rows < 256 ? rows : 256, many = (rows + 15) / 16;
    return many < few ? few : many < 1024 ? many : 1024;
}

hipError_t launch_norm_grad(const void* G, int64_t ldg, const void* X, int64_t ldx, const float* gamma, const float* mean,
                            const float* rstd, void* dX, float* dgamma, float* dbeta, float* part, int64_t rows, int32_t C,
                            int dtype, hipStream_t stream) {
    NormParams p{};
    p.X = X;
    p.G = G;
    p.gamma = gamma;
    p.Y = dX;
    p.mean = const_cast<float*>(mean);
    p.rstd = const_cast<float*>(rstd);
    p.part = dgamma || dbeta ? part : nullptr;
    p.rows = rows;
    p.ldx = ldx;
    p.ldg = ldg;
    p.ldy = C;
    p.C = C;
    const uint32_t blocks = (uint32_t)norm_grad_blocks(rows);
    const hipError_t e = dtype ? backward<uint16_t, 8>(p, blocks, stream) : backward<float, 4>(p, blocks, stream);
    if (e != hipSuccess || !p.part) return e;
    return launch_sum_pairs(part, blocks, C, dgamma, dbeta, stream);
}

}  // namespace mec
