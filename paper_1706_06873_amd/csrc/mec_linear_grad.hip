// What the gradients of the layer operators need beside their products: dZ = G act'(Z) with
// the column sums of dZ, and the sums of partial sums. dZ in bf16 comes in two parts, the output
// and what its rounding left over: the products take both, since the rounding of dZ alone (2^-8
// at most) would weigh as much in dX and dK as the rounding of their own.
//
// act_grad_kernel is one pass over G and Z, bound by memory. A workgroup takes a strip of
// columns and a share of the rows; a thread keeps the sums of its own columns in registers
// over all of its rows, the workgroup joins them in LDS and writes one row of partial sums,
// and sum_parts adds those in a fixed order: no atomics, the same bits every time.
#include "mec_product.h"

namespace mec {
namespace {

struct ActGradParams {
    const void* G;
    const void* Z;
    void* dZ;     // or nullptr (then act is none)
    void* low;    // dZ's second part, or nullptr
    float* part;  // shares x N, or nullptr
    int64_t ldg, rows, rows_per_share;
    int32_t N, act;
};

// Strips of 8 TX columns, THREADS / TX rows at a time; rows at any boundary (Pack8).
template <class E, int TX, int THREADS>
__global__ __launch_bounds__(THREADS) void act_grad_kernel(ActGradParams p) {
    constexpr int TY = THREADS / TX, U = 2;  // rows of a thread in flight
    constexpr bool FAST = sizeof(E) == 2;
    __shared__ __align__(16) float sums[THREADS * 8];
    const int tx = threadIdx.x % TX, ty = threadIdx.x / TX;
    const int32_t n = (int32_t)(blockIdx.x * TX + tx) * 8, have = p.N - n;
    const int64_t r0 = (int64_t)blockIdx.y * p.rows_per_share;
    const int64_t r1 = r0 + p.rows_per_share < p.rows ? r0 + p.rows_per_share : p.rows;
    float sum[8] = {};
    if (have > 0) {
        for (int64_t r = r0 + ty; r < r1; r += U * TY) {
            Pack8<E> g[U], z[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t row = r + u * TY < r1 ? r + u * TY : r;
                g[u].load(static_cast<const E*>(p.G) + row * p.ldg + n, have);
                if (p.act != kActNone) z[u].load(static_cast<const E*>(p.Z) + row * p.N + n, have);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (r + u * TY >= r1) break;
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = g[u].get(e);
                if (p.act == kActRelu) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = z[u].get(e) > 0.0f ? x[e] : 0.0f;
                } else if (p.act == kActSilu) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] *= act_slope<FAST>(kActSilu, z[u].get(e));
                } else if (p.act == kActGelu) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] *= act_slope<FAST>(kActGelu, z[u].get(e));
                }
                if (p.dZ) {
                    Pack8<E> o;
                    o.round(x);
                    o.store(static_cast<E*>(p.dZ) + (r + u * TY) * p.N + n, have);
                    if (p.low) {
                        float y[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) y[e] = __builtin_isfinite(o.get(e)) ? x[e] - o.get(e) : 0.0f;
                        o.round(y);
                        o.store(static_cast<E*>(p.low) + (r + u * TY) * p.N + n, have);
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] += x[e];
            }
        }
    }
    if (!p.part) return;  // (the same for every thread)
    // joined in halves: row groups y and y + s
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[threadIdx.x * 8 + e] = sum[e];
#pragma unroll
    for (int s = TY / 2; s > 0; s >>= 1) {
        __syncthreads();
        if (ty < s)
#pragma unroll
            for (int e = 0; e < 8; ++e) sums[threadIdx.x * 8 + e] = sum[e] += sums[(threadIdx.x + s * TX) * 8 + e];
    }
    if (ty == 0 && have > 0) {
        Pack8<float> o;
        o.round(sum);
        o.store(p.part + (int64_t)blockIdx.y * p.N + n, have);
    }
}

// Partial sums part[i*n + j], i < count: output j < n0 goes to out[j], the others to
// out2[j - n0]; either may be nullptr.
template <class E>
struct SumParams {
    const float* part;
    E* out;
    E* out2;
    int64_t n, n0;
    int32_t count;
    __device__ inline void put(int64_t j, float s) const {
        if (j < n0) {
            if (out) out[j] = from_float<E>(s);
        } else if (out2) {
            out2[j - n0] = from_float<E>(s);
        }
    }
};

// One output per thread, count partial sums one after another.
template <class E>
__global__ __launch_bounds__(256) void sum_few_kernel(SumParams<E> p) {
    for (int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x; j < p.n; j += (int64_t)gridDim.x * 256) {
        float s = 0.0f;
#pragma unroll 4
        for (int32_t i = 0; i < p.count; ++i) s += p.part[i * p.n + j];
        p.put(j, s);
    }
}

// 64 outputs per workgroup: 16 waves take every 16th partial sum, then join.
template <class E>
__global__ __launch_bounds__(1024) void sum_many_kernel(SumParams<E> p) {
    __shared__ float sums[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t j = (int64_t)blockIdx.x * 64 + lane;
    float s = 0.0f;
    if (j < p.n)
#pragma unroll 8
        for (int32_t i = wave; i < p.count; i += 16) s += p.part[i * p.n + j];
    sums[wave][lane] = s;
    __syncthreads();
    if (wave || j >= p.n) return;
#pragma unroll
    for (int w = 1; w < 16; ++w) s += sums[w][lane];
    p.put(j, s);
}

template <class E>
hipError_t sum_parts(const float* part, int64_t count, int64_t n, int64_t n0, void* out, void* out2, hipStream_t stream) {
    SumParams<E> p{part, static_cast<E*>(out), static_cast<E*>(out2), n, n0, (int32_t)count};
    if (count <= 32 || n > (int64_t(1) << 20)) {
        const int64_t blocks = (n + 255) / 256;
        hipLaunchKernelGGL(sum_few_kernel<E>, dim3((uint32_t)(blocks < 8192 ? blocks : 8192)), dim3(256), 0, stream, p);
    } else {
        hipLaunchKernelGGL(sum_many_kernel<E>, dim3((uint32_t)((n + 63) / 64)), dim3(1024), 0, stream, p);
    }
    return hipGetLastError();
}

// What a product's epilogue does, for one whose reduction was shared: 8 columns of a row per
// thread, then bias, activation and residual. WAYS threads add every WAYS-th share each, and
// the first of them joins the sums in order.
template <class E, int WAYS>
__global__ __launch_bounds__(256) void finish_parts_kernel(Product p, uint32_t granules, uint32_t count) {
    constexpr bool FAST = sizeof(E) == 2;
    constexpr uint32_t PER = 256 / WAYS;
    __shared__ __align__(16) float sums[WAYS > 1 ? 256 * 8 : 1];
    const uint32_t at = threadIdx.x % PER, way = threadIdx.x / PER;
    const int64_t stride = (int64_t)p.M * p.N;
    for (uint32_t first = blockIdx.x * PER; first < count; first += gridDim.x * PER) {
        const uint32_t i = first + at < count ? first + at : count - 1;
        const int64_t m = i / granules;
        const int32_t n = (int32_t)(i - (uint32_t)m * granules) * 8, have = p.N - n;
        Pack8<E> r;
        if (p.R && way == 0) r.load(static_cast<const E*>(p.R) + m * p.ldr + n, have);
        const float* const part = p.part + m * p.N + n;
        float v[8] = {};
#pragma unroll 4
        for (int32_t s = (int32_t)way; s < p.splits; s += WAYS) {
            Pack8<float> w;
            w.load(part + s * stride, have);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += e < have ? w.get(e) : 0.0f;
        }
        if constexpr (WAYS > 1) {
            __syncthreads();
            store8v(sums + threadIdx.x * 8, v);
            __syncthreads();
            if (way == 0)
#pragma unroll
                for (int w = 1; w < WAYS; ++w)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] += sums[(w * PER + at) * 8 + e];
        }
        if (way || first + at >= count) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[e] *= p.alpha;
            if (p.bias && e < have) v[e] += p.bias[n + e];
            if (p.R && p.res_first) v[e] += p.beta * r.get(e);
        }
        Pack8<E> o;
        if (p.Z) {
            o.round(v);
            o.store(static_cast<E*>(p.Z) + m * p.ldz + n, have);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (p.act == kActRelu) v[e] = act_value<FAST>(kActRelu, v[e]);
            else if (p.act == kActSilu) v[e] = act_value<FAST>(kActSilu, v[e]);
            else if (p.act == kActGelu) v[e] = act_value<FAST>(kActGelu, v[e]);
            if (p.R && !p.res_first) v[e] += p.beta * r.get(e);
        }
        o.round(v);
        o.store(static_cast<E*>(p.Y) + m * p.ldy + n, have);
    }
}
template <class E, int WAYS>
hipError_t finish_parts(const Product& p, hipStream_t stream) {
    const int64_t granules = (p.N + 7) / 8, count = granules * p.M;
    if (count > 0x7fffffff || p.batch != 1) return hipErrorInvalidValue;
    const int64_t blocks = (count * WAYS + 255) / 256;
    hipLaunchKernelGGL((finish_parts_kernel<E, WAYS>), dim3((uint32_t)(blocks < 8192 ? blocks : 8192)), dim3(256), 0, stream, p,
                       (uint32_t)granules, (uint32_t)count);
    return hipGetLastError();
}

template <class E, int TX, int THREADS>
hipError_t act_grad(const ActGradParams& p, uint32_t shares, hipStream_t stream) {
    const uint32_t strips = (uint32_t)((p.N + 8 * TX - 1) / (8 * TX));
    hipLaunchKernelGGL((act_grad_kernel<E, TX, THREADS>), dim3(strips, shares), dim3(THREADS), 0, stream, p);
    return hipGetLastError();
}

// Few rows (one share): 64 at a time, so that the column sums need no second launch. Else
// strips of 1024 columns where those fill the GPU, or of 256 (800 rows of 2048 in bf16, 25
// shares: 21 us in wide strips, so 10) or 128.
template <class E>
hipError_t act_grad(const ActGradParams& p, uint32_t shares, hipStream_t stream) {
    if (shares == 1) return act_grad<E, 16, 1024>(p, shares, stream);
    if (p.N > 512 && (int64_t)shares * ((p.N + 1023) / 1024) >= 512) return act_grad<E, 128, 256>(p, shares, stream);
    return p.N > 128 ? act_grad<E, 32, 256>(p, shares, stream) : act_grad<E, 16, 256>(p, shares, stream);
}

}  // namespace

hipError_t launch_finish_parts(const Product& p, int dtype, hipStream_t stream) {
    if (p.splits > 6) return dtype ? finish_parts<uint16_t, 8>(p, stream) : finish_parts<float, 8>(p, stream);
    return dtype ? finish_parts<uint16_t, 1>(p, stream) : finish_parts<float, 1>(p, stream);
}
hipError_t launch_sum_parts(const float* part, int64_t count, int64_t n, void* out, int dtype, hipStream_t stream) {
    return dtype ? sum_parts<uint16_t>(part, count, n, n, out, nullptr, stream)
                 : sum_parts<float>(part, count, n, n, out, nullptr, stream);
}
hipError_t launch_sum_pairs(const float* part, int64_t count, int64_t n, float* out, float* out2, hipStream_t stream) {
    return sum_parts<float>(part, count, 2 * n, n, out, out2, stream);
}

// Shares of the rows: one up to 256 rows; else enough to fill the GPU, of about 32 rows at least
// (257 in 9 shares of 29), and partial sums that stay a small part of the traffic.
int32_t act_grad_shares(int64_t rows, int64_t N) {
    if (rows <= 256) return 1;
    const int64_t strips = (N + 511) / 512;
    int64_t shares = (rows + 31) / 32, most = 2048 / strips > 1 ? 2048 / strips : 1;
    return (int32_t)(shares < most ? shares : most);
}

hipError_t launch_act_grad(const void* G, int64_t ldg, const void* Z, void* dZ, void* low, float* dbias, float* part,
                           int64_t rows, int32_t N, int act, int dtype, hipStream_t stream) {
    const int32_t shares = act_grad_shares(rows, N);
    ActGradParams p{};
    p.G = G;
    p.Z = Z;
    p.dZ = dZ;
    p.low = low;
    p.part = !dbias ? nullptr : shares == 1 ? dbias : part;
    p.ldg = ldg;
    p.rows = rows;
    p.rows_per_share = (rows + shares - 1) / shares;
    p.N = N;
    p.act = act;
    const hipError_t e = dtype ? act_grad<uint16_t>(p, (uint32_t)shares, stream) : act_grad<float>(p, (uint32_t)shares, stream);
    if (e != hipSuccess || !dbias || shares == 1) return e;
    return launch_sum_parts(part, shares, N, dbias, 0, stream);
}

}  // namespace mec
