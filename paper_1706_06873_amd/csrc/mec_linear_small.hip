// Matrix products of the layer operators with few outputs, where the tile kernels would
// leave the GPU to a few workgroups that take one chunk after another: a workgroup computes
// 32 x 32 outputs, its 16 waves share the reduction (each takes one run of it, with loads of
// its own and no barriers) and their sums are joined in LDS in the order of the waves. Bound
// by the latency of a few rounds of loads.
//
// fp32: operands go from memory to registers, are split there and multiplied (mec_split.h).
// bf16: operands stored along the reduction likewise (a fragment is 16 bytes of a row); those
// stored across it pass through a patch of LDS of the wave's own, for the transposing reads.
#include "mec_product.h"
#include "mec_split.h"

namespace mec {
namespace {

constexpr int kWaves = 16, kPitch = 36;  // floats of a row of a wave's sums in LDS

struct Slice {
    int32_t k0, k1;  // this wave's run of the reduction
};

// a wave's sums to LDS
__device__ inline void put_sums(const floatx16& acc, float* sums, int wave, int lane) {
    float* const mine = sums + wave * 32 * kPitch + (lane & 31) * kPitch + (lane >> 5) * 4;
#pragma unroll
    for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4v*>(mine + q * 8) = f32x4v{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
}

// The sums of the waves, joined: thread t finishes output (t / 32, t % 32).
template <class E>
__device__ inline void join(const Product& p, const floatx16& acc, float* sums, int32_t m0, int32_t n0, int32_t bat, int waves,
                            int wave, int lane) {
    if (wave < waves) put_sums(acc, sums, wave, lane);
    __syncthreads();
    const int m = (int)threadIdx.x / 32, n = (int)threadIdx.x % 32;
    if (m0 + m >= p.M || n0 + n >= p.N) return;
    float v = 0.0f;
    for (int w = 0; w < waves; ++w) v += sums[w * 32 * kPitch + m * kPitch + n];
    finish<E>(p, m0 + m, n0 + n, bat, v);
}

struct Place {
    int32_t m0, n0, bat, waves;
    Slice k;
};
// tile `b` of all of p's
__device__ inline Place place(const Product& p, uint32_t b, int wave) {
    Place t;
    const uint32_t tiles = (uint32_t)p.m_tiles * (uint32_t)p.n_tiles;
    t.bat = (int32_t)(b / tiles);
    const uint32_t r = b - (uint32_t)t.bat * tiles, mt = r / (uint32_t)p.n_tiles;
    t.m0 = (int32_t)mt * 32;
    t.n0 = (int32_t)(r - mt * (uint32_t)p.n_tiles) * 32;
    const int32_t run = p.chunks * 16;  // of the reduction, a wave
    t.waves = (p.K + run - 1) / run;
    t.k.k0 = wave * run;
    t.k.k1 = t.k.k0 + run < p.K ? t.k.k0 + run : p.K;
    return t;
}

// ---------------------------------------------------------------- fp32
// 8 k of row (column) r: stored along (stride 1) or across (stride ld) the reduction
template <bool TR>
__device__ inline void fetch(const float* base, int64_t ld, int32_t k, int32_t k1, float* x) {
    if constexpr (TR) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int32_t at = k + e < k1 ? k + e : k1 - 1;
            const float v = base[at * ld];
            x[e] = k + e < k1 ? v : 0.0f;
        }
    } else if (k + 8 <= k1) {
        struct __attribute__((packed, aligned(4))) Any {
            f32x4v v;
        };
        const f32x4v a = reinterpret_cast<const Any*>(base + k)->v, b = reinterpret_cast<const Any*>(base + k + 4)->v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] = a[e];
            x[4 + e] = b[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = k + e < k1 ? base[k + e] : 0.0f;
    }
}

// A wave's 32 x 32 sums over k0 <= k < k1 (a multiple of 16 from each other, or k1 the last):
// fa and fb fetch this lane's 8 k from k on of its row and of its column. U: steps of 16 k in
// flight.
template <int U, class FA, class FB>
__device__ inline floatx16 run_f32(int32_t k0, int32_t k1, int lane, FA fa, FB fb) {
    const int32_t half = 8 * (lane >> 5);
    floatx16 acc = {}, low = {};
    uint32_t lost = 0;
    for (int32_t k = k0; k < k1; k += 16 * U) {
        float x[U][8], y[U][8];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            fa(k + 16 * u + half, x[u]);
            fb(k + 16 * u + half, y[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            u32x4 xs[3], ys[3];
            split8(x[u], xs[0], xs[1], xs[2], lost);
            split8(y[u], ys[0], ys[1], ys[2], lost);
            auto mm = [&](int i, int j, floatx16& to) {
                to = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, ys[j]), __builtin_bit_cast(bf16x8, xs[i]),
                                                             to, 0, 0, 0);
            };
            mm(0, 0, acc);
            mm(1, 0, low);
            mm(0, 1, low);
            mm(1, 1, low);
            mm(2, 0, low);
            mm(0, 2, low);
        }
    }
    uint32_t most = 0;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        acc[v] += low[v];
        const float x = acc[v];
        const uint32_t bits = __builtin_bit_cast(uint32_t, x) & 0x7fffffffu;
        most = bits > most ? bits : most;
    }
    if (__any((lost & 0xffffu) != 0) || __any(most >= 0x7f800000u)) {  // values the split does not hold
        floatx16 sum = {};
        plain_products(
            sum, (uint32_t)(k1 - k0 + 15) / 16u, [&](uint32_t s, float* x) { fb(k0 + (int32_t)s * 16 + half, x); },
            [&](uint32_t s, float* x) { fa(k0 + (int32_t)s * 16 + half, x); });
        acc = sum;
    }
    return acc;
}
template <Layout L>
__device__ inline void small_f32(const Product& p, uint32_t b0, float* sums) {
    constexpr bool AT = L == Layout::kXtK, BT = L != Layout::kXKt;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Place t = place(p, b0, wave);
    floatx16 acc = {};
    if (wave < t.waves) {
        // rows and columns past the last are copies of it
        const int32_t m = t.m0 + (lane & 31) < p.M ? t.m0 + (lane & 31) : p.M - 1;
        const int32_t n = t.n0 + (lane & 31) < p.N ? t.n0 + (lane & 31) : p.N - 1;
        const float* const a = a_of<float>(p, t.bat) + (AT ? (int64_t)m : m * p.lda);
        const float* const b = b_of<float>(p, t.bat) + (BT ? (int64_t)n : n * p.ldb);
        acc = run_f32<2>(
            t.k.k0, t.k.k1, lane, [&](int32_t k, float* x) { fetch<AT>(a, p.lda, k, t.k.k1, x); },
            [&](int32_t k, float* x) { fetch<BT>(b, p.ldb, k, t.k.k1, x); });
    }
    join<float>(p, acc, sums, t.m0, t.n0, t.bat, t.waves, wave, lane);
}

// A step of the orthogonalisation from A, X' = a X + P X (WIDE; else X P), P = b A + c A A, for m
// up to 128: each workgroup makes the 32 rows of P that its 32 x 32 outputs need (16 waves: up
// to 4 blocks of columns, the reduction in 4 runs) and keeps them in LDS for the product with
// X. More arithmetic than P in a launch of its own, but a launch less to wait for (363 x 96: 6.9
// us, P and X one after the other 11).
template <bool WIDE>
__global__ __launch_bounds__(64 * kWaves) void orth_step_kernel(OrthStep p) {
    constexpr int kRow = kOrthStepMax + 4;
    __shared__ __align__(16) float sums[kWaves * 32 * kPitch];
    __shared__ __align__(16) float P[32 * kRow];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = lane & 31;
    const int tr = (int)threadIdx.x / 32, tc = (int)threadIdx.x % 32;
    const uint32_t n_tiles = (uint32_t)(p.cols + 31) / 32, tiles = (uint32_t)((p.rows + 31) / 32) * n_tiles;
    const uint32_t b = xcd_remap(blockIdx.x, gridDim.x), bat = b / tiles, mt = (b - bat * tiles) / n_tiles;
    const int32_t r0 = (int32_t)mt * 32, c0 = (int32_t)(b - bat * tiles - mt * n_tiles) * 32, own = WIDE ? r0 : c0, m = p.m;
    const float* const A = p.A + (int64_t)bat * m * m;
    const int64_t x_at = (int64_t)bat * p.rows * p.cols;
    const float* const X = p.X + x_at;
    auto last = [](int32_t i, int32_t n) { return i < n ? i : n - 1; };

    // the wave's part of X, and what this thread adds
    float x[8] = {};
    const int32_t k2 = 16 * wave;
    if (k2 < m) {
        if constexpr (WIDE) fetch<true>(X + last(c0 + l, p.cols), p.cols, k2 + 8 * (lane >> 5), m, x);
        else fetch<false>(X + (int64_t)last(r0 + l, p.rows) * p.cols, 0, k2 + 8 * (lane >> 5), m, x);
    }
    const bool stored = r0 + tr < p.rows && c0 + tc < p.cols;
    const int64_t at = (int64_t)(r0 + tr) * p.cols + c0 + tc;
    const float own_x = stored ? X[at] : 0.0f;

    // P's rows
    const int t = wave & 3, run = ((m + 15) / 16 + 3) / 4 * 16;  // column block, k of a run
    const int32_t k0 = (wave >> 2) * run, k1 = k0 + run < m ? k0 + run : m;
    float own_a[kOrthStepMax / 32];
#pragma unroll
    for (int i = 0; i < kOrthStepMax / 32; ++i)
        own_a[i] = own + tr < m && i * 32 + tc < m ? A[(own + tr) * m + i * 32 + tc] : 0.0f;
    if (t * 32 < m && k0 < k1) {
        const float* const ra = A + last(own + l, m) * m;
        const float* const rb = A + last(t * 32 + l, m) * m;  // (A is symmetric)
        put_sums(run_f32<2>(
                     k0, k1, lane, [&](int32_t k, float* v) { fetch<false>(ra, 0, k, k1, v); },
                     [&](int32_t k, float* v) { fetch<false>(rb, 0, k, k1, v); }),
                 sums, wave, lane);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kOrthStepMax / 32; ++i) {
        if (i * 32 >= m) break;
        float v = 0.0f;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float s = sums[(i + 4 * q) * 32 * kPitch + tr * kPitch + tc];
            v += q * run < m ? s : 0.0f;
        }
        P[tr * kRow + i * 32 + tc] = own + tr < m && i * 32 + tc < m ? p.b * own_a[i] + p.c * v : 0.0f;
    }
    __syncthreads();

    if (k2 < m) {
        auto ours = [&](int32_t k, float* v) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = P[l * kRow + k + e];
        };
        auto theirs = [&](int32_t, float* v) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = x[e];
        };
        const floatx16 acc = WIDE ? run_f32<1>(k2, k2 + 16, lane, ours, theirs) : run_f32<1>(k2, k2 + 16, lane, theirs, ours);
        put_sums(acc, sums, wave, lane);
    }
    __syncthreads();
    if (!stored) return;
    float v = 0.0f;
    for (int w = 0; w * 16 < m; ++w) v += sums[w * 32 * kPitch + tr * kPitch + tc];
    v += p.a * own_x;
    if (p.bf16) static_cast<uint16_t*>(p.Y)[x_at + at] = from_float<uint16_t>(v);
    else static_cast<float*>(p.Y)[x_at + at] = v;
}

// ---------------------------------------------------------------- bf16
constexpr int kRun = 64;                  // k per turn: 4 fragments of each operand
constexpr int kPatch = kRun * 32 * 2;     // bytes of a wave's patch: 64 rows of 32 columns

// The 4 fragments of an operand for the 64 k from k on, in two parts: loads, and what makes
// fragments of them. CLEAN: 16-byte rows of whole granules; else granules are read whole at
// any boundary, but for those that the row or the reduction cuts off. Rows along the
// reduction at odd elements go dword by dword (whole loads of 64 rows that begin inside
// a dword: 64 x 256 <- 3239 41.7 us, so 24.2; at even elements 14.7 and 24).
// Elements k .. k + 7 of a row of more than 8, by whole dwords of the row's own.
__device__ inline u32x4v load_dwords(const uint16_t* row, int32_t k) {
    struct __attribute__((packed, aligned(4))) Any {
        u32x4v v;
    };
    const bool odd = ((uintptr_t)row & 2) != 0, start = odd && k == 0;  // (k is a multiple of 8)
    const DwordGranule g = dword_granule(odd, k);
    const u32x4v w = reinterpret_cast<const Any*>(row + (k + g.wide))->v;
    const uint32_t one = row[k + g.single], by = odd ? 16u : 0u;
    // what the granule is cut from: the single element before or after the others
    const uint32_t q[5] = {start ? one << 16 : w[0], start ? w[0] : w[1], start ? w[1] : w[2], start ? w[2] : w[3], start ? w[3] : one};
    return u32x4v{__builtin_amdgcn_alignbit(q[1], q[0], by), __builtin_amdgcn_alignbit(q[2], q[1], by),
                  __builtin_amdgcn_alignbit(q[3], q[2], by), __builtin_amdgcn_alignbit(q[4], q[3], by)};
}

template <bool TR, bool CLEAN>
struct Turn {
    u32x4v w[4];
    // base: the tile's first row (column); r: rows (columns) there are from it on
    __device__ inline void load(const uint16_t* base, int64_t ld, int32_t r, int32_t k, int32_t k1, int lane) {
        const bool whole = k1 % 8 == 0, odd = (((uint64_t)base >> 1 | (uint64_t)ld) & 1) != 0 && k1 > 8;  // uniform
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (TR) {  // row k + 16 i + lane / 4, granule lane % 4 of its 32 columns
                const int32_t at = k + 16 * i + (lane >> 2), c = (lane & 3) * 8;
                const uint16_t* const src = base + (at < k1 ? at : k1 - 1) * ld;
                if constexpr (CLEAN) {
                    w[i] = *reinterpret_cast<const u32x4v*>(src + (c < r ? c : r - 8));
                    if (at >= k1) w[i] = u32x4v{0, 0, 0, 0};
                } else if (r >= 32) {  // (uniform)
                    w[i] = load_any(src + c);
                    if (at >= k1) w[i] = u32x4v{0, 0, 0, 0};
                } else {
                    w[i] = load_some(src + c, at < k1 ? r - c : 0);
                }
            } else {
                const int32_t at = k + 16 * i + 8 * (lane >> 5);
                const uint16_t* const src = base + ((lane & 31) < r ? (lane & 31) : r - 1) * ld;
                if constexpr (CLEAN) w[i] = *reinterpret_cast<const u32x4v*>(src + (at < k1 ? at : k1 - 8));
                else if (whole && !odd) w[i] = load_any(src + (at < k1 ? at : k1 - 8));
                else if (whole) w[i] = load_dwords(src, at < k1 ? at : k1 - 8);
                else w[i] = load_some(src + at, k1 - at);
                if (at >= k1) w[i] = u32x4v{0, 0, 0, 0};
            }
        }
    }
    // rows of the patch are 64 bytes; their two 16-column blocks change places every second
    // pair of rows, so that the 4 rows that 16 lanes read lie on different banks
    __device__ inline void put(char* patch, int lane) const {
        if constexpr (TR)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = 16 * i + (lane >> 2), c = lane & 3;
                *reinterpret_cast<u32x4v*>(patch + row * 64 + ((c ^ (row & 2)) << 4)) = w[i];
            }
    }
    __device__ inline bf16x8 frag(const char* patch, int i, int lane) const {
        if constexpr (!TR) return __builtin_bit_cast(bf16x8, w[i]);
        const int q = lane & 15, block = (lane >> 4) & 1;
        s16x4 h[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int row = 16 * i + 8 * (lane >> 5) + 4 * s + (q >> 2);
            h[s] = read_tr(patch + row * 64 + (((block << 1) ^ (row & 2)) << 4) + (q & 3) * 8);
        }
        return join_tr(h[0], h[1]);
    }
};

template <Layout L>
constexpr int kPatches = (L == Layout::kXtK ? kPatch : 0) + (L != Layout::kXKt ? kPatch : 0);  // of a wave
constexpr int kSums = kWaves * 32 * kPitch * 4;
template <Layout L>
constexpr int kLds = kWaves * kPatches<L> > kSums ? kWaves * kPatches<L> : kSums;

template <Layout L, bool CLEAN>
__device__ inline void small_bf16(const Product& p, uint32_t b0, char* lds) {
    constexpr bool AT = L == Layout::kXtK, BT = L != Layout::kXKt;
    constexpr int PATCHES = kPatches<L>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Place t = place(p, b0, wave);
    floatx16 acc = {};
    if (wave < t.waves) {
        const uint16_t* const a = a_of<uint16_t>(p, t.bat) + (AT ? (int64_t)t.m0 : t.m0 * p.lda);
        const uint16_t* const b = b_of<uint16_t>(p, t.bat) + (BT ? (int64_t)t.n0 : t.n0 * p.ldb);
        char* const patch_b = lds + wave * PATCHES;
        char* const patch_a = patch_b + (BT ? kPatch : 0);
        Turn<AT, CLEAN> ta;
        Turn<BT, CLEAN> tb;
        // dZ (A of dX, B of dK) in two parts: turns of the one and of the other
        const int64_t second = L != Layout::kXK ? p.second / 2 : 0;
        auto load = [&](int32_t k, int64_t part) {
            ta.load(a + (AT ? 0 : part), p.lda, p.M - t.m0, k, t.k.k1, lane);
            tb.load(b + (AT ? part : 0), p.ldb, p.N - t.n0, k, t.k.k1, lane);
        };
        int64_t part = 0;
        load(t.k.k0, part);
        for (int32_t k = t.k.k0; k < t.k.k1;) {
            bf16x8 fa[4], fb[4];
            ta.put(patch_a, lane);
            tb.put(patch_b, lane);
            if constexpr (AT || BT) {  // the wave's LDS accesses stay in this order
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                __builtin_amdgcn_wave_barrier();
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                fa[i] = ta.frag(patch_a, i, lane);
                fb[i] = tb.frag(patch_b, i, lane);
            }
            if (L == Layout::kXK || part == second) k += kRun;
            if (L != Layout::kXK) part = second - part;
            if (k < t.k.k1) load(k, part);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[i], fa[i], acc, 0, 0, 0);
            if constexpr (AT || BT) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                __builtin_amdgcn_wave_barrier();
            }
        }
        if (second && not_finite(acc)) {
            const int32_t m = (lane & 31) < p.M - t.m0 ? (lane & 31) : p.M - t.m0 - 1;
            const int32_t n = (lane & 31) < p.N - t.n0 ? (lane & 31) : p.N - t.n0 - 1;
            const int64_t aks = AT ? p.lda : 1, bks = BT ? p.ldb : 1;
            const uint16_t* const row = a + m * (AT ? 1 : p.lda) + t.k.k0 * aks;
            const uint16_t* const column = b + n * (BT ? 1 : p.ldb) + t.k.k0 * bks;
            if (holds_infinity(AT ? row : column, AT ? aks : bks, t.k.k1 - t.k.k0, lane))
                take_again(acc, row, aks, column, bks, t.k.k1 - t.k.k0, lane);
        }
    }
    __syncthreads();
    join<uint16_t>(p, acc, reinterpret_cast<float*>(lds), t.m0, t.n0, t.bat, t.waves, wave, lane);
}

// One product, or (pair) the two of a backward pass, dX = dZ K^T and dK = X^T dZ, side by side
// in one launch: the launch is what a small pass waits for (3 us of host time each).
template <Layout L>
__global__ __launch_bounds__(64 * kWaves) void small_f32_kernel(Product p) {
    __shared__ __align__(16) float sums[kWaves * 32 * kPitch];
    small_f32<L>(p, xcd_remap(blockIdx.x, gridDim.x), sums);
}
__global__ __launch_bounds__(64 * kWaves) void small_f32_pair_kernel(Product x, Product k, uint32_t x_blocks) {
    __shared__ __align__(16) float sums[kWaves * 32 * kPitch];
    if (blockIdx.x < x_blocks) small_f32<Layout::kXKt>(x, xcd_remap(blockIdx.x, x_blocks), sums);
    else small_f32<Layout::kXtK>(k, blockIdx.x - x_blocks, sums);
}
template <Layout L, bool CLEAN>
__global__ __launch_bounds__(64 * kWaves) void small_bf16_kernel(Product p) {
    __shared__ __align__(16) char lds[kLds<L>];
    small_bf16<L, CLEAN>(p, xcd_remap(blockIdx.x, gridDim.x), lds);
}
template <bool CLEAN>
__global__ __launch_bounds__(64 * kWaves) void small_bf16_pair_kernel(Product x, Product k, uint32_t x_blocks) {
    __shared__ __align__(16) char lds[kLds<Layout::kXtK>];
    if (blockIdx.x < x_blocks) small_bf16<Layout::kXKt, CLEAN>(x, xcd_remap(blockIdx.x, x_blocks), lds);
    else small_bf16<Layout::kXtK, CLEAN>(k, blockIdx.x - x_blocks, lds);
}

template <Layout L>
hipError_t run(const Product& p, int dtype, uint32_t blocks, hipStream_t stream) {
    const dim3 grid(blocks), block(64 * kWaves);
    if (!dtype) hipLaunchKernelGGL(small_f32_kernel<L>, grid, block, 0, stream, p);
    else if (p.clean) hipLaunchKernelGGL((small_bf16_kernel<L, true>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((small_bf16_kernel<L, false>), grid, block, 0, stream, p);
    return hipGetLastError();
}

// Fills what the kernels need; the workgroups, or 0 past the grid.
uint32_t prepare(Product& p, Layout layout, int dtype) {
    p.m_tiles = (p.M + 31) / 32;
    p.n_tiles = (p.N + 31) / 32;
    const int64_t blocks = (int64_t)p.m_tiles * p.n_tiles * p.batch;
    // a wave's run: whole steps of 16 k
    const int64_t steps = ((int64_t)p.K + 15) / 16;
    p.chunks = (int32_t)((steps + kWaves - 1) / kWaves);
    if (dtype) p.clean = clean_rows(layout, p) && p.a_batch % 8 == 0 && p.b_batch % 8 == 0;
    return blocks > kMaxSmallBlocks || p.splits > 1 ? 0 : (uint32_t)blocks;
}

}  // namespace

hipError_t launch_orth_step(const OrthStep& p, int32_t batch, hipStream_t stream) {
    const int64_t blocks = (int64_t)((p.rows + 31) / 32) * ((p.cols + 31) / 32) * batch;
    if (p.m > kOrthStepMax || p.m != (p.rows < p.cols ? p.rows : p.cols) || blocks > kMaxSmallBlocks) return hipErrorInvalidValue;
    const dim3 grid((uint32_t)blocks), block(64 * kWaves);
    if (p.rows <= p.cols) hipLaunchKernelGGL(orth_step_kernel<true>, grid, block, 0, stream, p);
    else hipLaunchKernelGGL(orth_step_kernel<false>, grid, block, 0, stream, p);
    return hipGetLastError();
}

hipError_t launch_product_small(Layout layout, Product p, int dtype, hipStream_t stream) {
    const uint32_t blocks = prepare(p, layout, dtype);
    if (!blocks) return hipErrorInvalidValue;
    switch (layout) {
        case Layout::kXK: return run<Layout::kXK>(p, dtype, blocks, stream);
        case Layout::kXKt: return run<Layout::kXKt>(p, dtype, blocks, stream);
        default: return run<Layout::kXtK>(p, dtype, blocks, stream);
    }
}

hipError_t launch_product_small_pair(Product x, Product k, int dtype, hipStream_t stream) {
    const uint32_t bx = prepare(x, Layout::kXKt, dtype), bk = prepare(k, Layout::kXtK, dtype);
    if (!bx || !bk) return hipErrorInvalidValue;
    const dim3 grid(bx + bk), block(64 * kWaves);
    if (!dtype) hipLaunchKernelGGL(small_f32_pair_kernel, grid, block, 0, stream, x, k, bx);
    else if (x.clean && k.clean) hipLaunchKernelGGL(small_bf16_pair_kernel<true>, grid, block, 0, stream, x, k, bx);
    else hipLaunchKernelGGL(small_bf16_pair_kernel<false>, grid, block, 0, stream, x, k, bx);
    return hipGetLastError();
}

}  // namespace mec
