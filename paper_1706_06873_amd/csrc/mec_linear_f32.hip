// fp32 matrix products of the layer operators (mec_product.h) on the bf16 matrix cores: each
// operand value is split without loss into three bf16 values and a product is six bf16
// products (mec_gemm_tile.hip says how exact that is, and mec_split.h what happens to values
// that the split does not hold). A workgroup computes a tile of Y, 32*BM*WM x 32*BN*WN, from
// chunks of 32 of the reduction in two stages of LDS; chunks travel through registers, where
// they are split.
#include "mec_product.h"
#include "mec_split.h"

namespace mec {
namespace {

constexpr int kKT = 32, kG = kKT / 8;  // chunk of the reduction, groups of 8 in it

// KW groups of WM x WN waves share the reduction of a tile, each with stages of its own: what
// several tiles on a compute unit do for one another where there are that many (1024 x 1024 x
// 4096, a tile per compute unit, 88 us, so 69; two groups likewise, but for short reductions).
// TAIL: an operand stored along the reduction ends inside a group of 8.
template <int BM, int BN, int WM, int WN, int KW, Layout L, bool TAIL>
struct Cfg {
    static constexpr int kBM = BM, kBN = BN, kWM = WM, kWN = WN, kKW = KW;
    static constexpr bool kAT = L == Layout::kXtK, kBT = L != Layout::kXKt;  // stored across the reduction
    static constexpr bool kTail = TAIL;
    static constexpr int TM = 32 * BM * WM, TN = 32 * BN * WN, WAVES = WM * WN, THREADS = 64 * WAVES;  // of a group
    static constexpr int APL = TM * kKT * 2, BPL = TN * kKT * 2, STAGE = 3 * (APL + BPL);  // bytes (of a plane)
    static constexpr int EPI = WAVES * 32 * (32 * BN + 4) * 4;
    static constexpr int JOIN = (KW - 1) * WAVES * 4096;  // sums of a group's waves
    static_assert(KW == 1 || (BM * BN == 1 && EPI + JOIN <= 2 * KW * STAGE), "groups");
    static constexpr int LDS = 2 * KW * STAGE > EPI ? 2 * KW * STAGE : EPI;
    static constexpr int kPerSimd = WAVES * KW >= 8 ? WAVES * KW / 4 : (LDS <= 53 * 1024 ? 3 : LDS <= 80 * 1024 ? 2 : 1);
    static_assert(TM * kG % THREADS == 0 && TN * kG % THREADS == 0 && THREADS % TM == 0 && THREADS % TN == 0 && LDS <= 158 * 1024, "tile");
};

// One operand's T rows (stored along the reduction) or columns (TR: across it) of a tile.
template <int T, int THREADS, bool TR, bool TAIL>
struct Operand {
    static constexpr int ITEMS = T * kG / THREADS;
    const char* base;  // uniform: the tile's first row and the chunk's first k
    int64_t bytes;     // uniform: from base to the end of what may be read
    int64_t step;      // bytes from chunk to chunk
    int32_t left;      // elements of the reduction from base on
    uint32_t voff[TR ? 8 : ITEMS];
    uint32_t pitch;    // TR: bytes between the groups of two items
    uint32_t lds[ITEMS];
    int32_t k_at;      // first k of this thread's group in a chunk

    __device__ inline void init(const void* mem, int64_t ld, int32_t r0, int32_t count, int64_t k0, int64_t k1, int tid) {
        left = (int32_t)(k1 - k0);
        if constexpr (TR) {
            const int col = tid % T, g = __builtin_amdgcn_readfirstlane(tid / T);
            base = uniform(static_cast<const char*>(mem) + 4 * (k0 * ld + r0));
            bytes = 4 * ((int64_t)left * ld - r0);  // rows past k1 lie past it
            step = 4 * kKT * ld;
            pitch = (uint32_t)(THREADS / T) * 32u * (uint32_t)ld;
            const int c = r0 + col < count ? col : count - 1 - r0;
#pragma unroll
            for (int e = 0; e < 8; ++e) voff[e] = 4u * (uint32_t)((g * 8 + e) * ld + c);
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) lds[i] = swz((uint32_t)col, (uint32_t)(g + i * (THREADS / T)));
        } else {
            const int g = tid % kG, row = tid / kG;
            base = uniform(static_cast<const char*>(mem) + 4 * (r0 * ld + k0));
            bytes = 4 * ((int64_t)(count - 1 - r0) * ld + left);
            step = 4 * kKT;
            k_at = 8 * g;
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                int r = row + i * (THREADS / kG);
                lds[i] = swz((uint32_t)r, (uint32_t)g);
                if (r0 + r >= count) r = count - 1 - r0;  // rows past the last are not stored
                voff[i] = 4u * (uint32_t)(r * ld + 8 * g);
            }
        }
    }
    // this chunk to registers, and on to the next. k past the last come as zeros.
    __device__ inline void load(float (*x)[8]) {
        const __amdgpu_buffer_rsrc_t rs = buffer(base, bytes > 0x7fffffff ? 0x7fffffff : bytes > 0 ? (int)bytes : 0);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            if constexpr (TR) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    x[i][e] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rs, voff[e] + i * pitch, 0, 0));
            } else {
                load8(rs, k_at < left ? voff[i] : 0x80000000u, x[i]);
                if constexpr (TAIL) {
#pragma unroll
                    for (int e = 1; e < 8; ++e) x[i][e] = k_at + e < left ? x[i][e] : 0.0f;
                }
            }
        }
        base += step;
        bytes -= step;
        left -= kKT;
    }
    __device__ inline void put(const float (*x)[8], char* __restrict__ to, uint32_t& lost) const {
        constexpr int PL = T * kKT * 2;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            u32x4 h, m, l;
            split8(x[i], h, m, l, lost);
            *reinterpret_cast<u32x4*>(to + lds[i]) = h;
            *reinterpret_cast<u32x4*>(to + PL + lds[i]) = m;
            *reinterpret_cast<u32x4*>(to + 2 * PL + lds[i]) = l;
        }
    }
};

// A 32 x 32 block in plain fp32, for values that the split does not hold: this lane's row of
// A and column of B, with their elements a_k and b_k apart.
__device__ __attribute__((noinline)) floatx16 plain_block(const float* a, int64_t a_k, const float* b, int64_t b_k, int32_t K, int lane) {
    floatx16 sum = {};
    auto fetch = [&](const float* from, int64_t ks, uint32_t s, float* x) {
        const int32_t k = (int32_t)(s * 16u) + 8 * (lane >> 5);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = k + e < K ? from[(k + e) * ks] : 0.0f;
    };
    plain_products(
        sum, ((uint32_t)K + 15u) / 16u, [&](uint32_t s, float* x) { fetch(b, b_k, s, x); },
        [&](uint32_t s, float* x) { fetch(a, a_k, s, x); });
    return sum;
}

// Workgroup b's tile. all: C::LDS bytes of LDS; lost_s, there too: some thread's split left
// bits out.
template <class C>
__device__ inline void product_f32(const Product& p, uint32_t b, char* all, uint32_t& lost_s) {
    constexpr int BM = C::kBM, BN = C::kBN;
    using OpA = Operand<C::TM, C::THREADS, C::kAT, C::kTail>;
    using OpB = Operand<C::TN, C::THREADS, C::kBT, C::kTail>;
    const int group = C::kKW > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / C::THREADS) : 0;
    const int tid = (int)threadIdx.x - group * C::THREADS, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    char* const lds = all + group * 2 * C::STAGE;
    const int wm = wave % C::kWM, wn = wave / C::kWM;
    constexpr bool SQUARE = C::TM == C::TN && BM * BN == 1;  // holds symmetric products
    const bool symmetric = SQUARE && p.symmetric;
    const uint32_t tiles = symmetric ? (uint32_t)p.m_tiles * ((uint32_t)p.m_tiles + 1) / 2 : (uint32_t)p.m_tiles * (uint32_t)p.n_tiles;
    const uint32_t share = b / tiles;  // of the reduction, for each product of a batch
    const int32_t split = (int32_t)(share / (uint32_t)p.batch), bat = (int32_t)(share - (uint32_t)split * (uint32_t)p.batch);
    uint32_t mt, nt;
    if (symmetric) tile_of_half(b - share * tiles, mt, nt);
    else tile_of(b - share * tiles, (uint32_t)p.m_tiles, (uint32_t)p.n_tiles, 8u, mt, nt);
    const int32_t m0 = (int32_t)mt * C::TM, n0 = (int32_t)nt * C::TN;
    const int64_t s0 = (int64_t)split * p.chunks * kKT;  // the share, and this group's run of it (or none)
    const int64_t s1 = s0 + (int64_t)p.chunks * kKT < p.K ? s0 + (int64_t)p.chunks * kKT : p.K;
    const int chunks = (int)((s1 - s0 + C::kKW * kKT - 1) / (C::kKW * kKT));
    const int64_t k0 = s0 + (int64_t)group * chunks * kKT < s1 ? s0 + (int64_t)group * chunks * kKT : s1;
    const int64_t k1 = k0 + (int64_t)chunks * kKT < s1 ? k0 + (int64_t)chunks * kKT : s1;
    const float* const A = a_of<float>(p, bat);
    const float* const B = b_of<float>(p, bat);

    if (threadIdx.x == 0) lost_s = 0;  // (ordered by the first barriers)
    OpA oa;
    OpB ob;
    oa.init(A, p.lda, m0, p.M, k0, k1, tid);
    ob.init(B, p.ldb, n0, p.N, k0, k1, tid);
    struct Regs {
        float a[OpA::ITEMS][8], b[OpB::ITEMS][8];
    };
    uint32_t lost = 0;
    auto load = [&](Regs& r) {
        oa.load(r.a);
        ob.load(r.b);
    };
    auto stage = [&](const Regs& r, char* __restrict__ to) {
        oa.put(r.a, to, lost);
        ob.put(r.b, to + 3 * C::APL, lost);
    };
    floatx16 acc[BM][BN] = {}, low[BM][BN] = {};
    struct Frags {
        bf16x8 a[BM][3], b[BN][3];
    };
    auto read = [&](Frags& f, const char* __restrict__ from, int kk) {
        const uint32_t g = (uint32_t)(2 * kk + (lane >> 5));
#pragma unroll
        for (int q = 0; q < 3; ++q) {
#pragma unroll
            for (int i = 0; i < BM; ++i)
                f.a[i][q] = *reinterpret_cast<const bf16x8*>(from + q * C::APL + swz((uint32_t)((wm * BM + i) * 32 + (lane & 31)), g));
#pragma unroll
            for (int j = 0; j < BN; ++j)
                f.b[j][q] = *reinterpret_cast<const bf16x8*>(from + 3 * C::APL + q * C::BPL + swz((uint32_t)((wn * BN + j) * 32 + (lane & 31)), g));
        }
    };
    // B's columns are the instruction's rows (see the epilogue)
    auto products = [&](const Frags& f) {
#define MEC_MM(X, Y, ACC)                              \
    _Pragma("unroll") for (int i = 0; i < BM; ++i)     \
        _Pragma("unroll") for (int j = 0; j < BN; ++j) \
            ACC[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.b[j][Y], f.a[i][X], ACC[i][j], 0, 0, 0);
        MEC_MM(0, 0, acc)
        MEC_MM(1, 0, low)
        MEC_MM(0, 1, low)
        MEC_MM(1, 1, low)
        MEC_MM(2, 0, low)
        MEC_MM(0, 2, low)
#undef MEC_MM
    };
    // One chunk at a time in registers: it is requested under the second half of a chunk's
    // products and split into the other stage under the first half of the next one's. (Two and
    // four chunks in registers: 1024 x 1024 x 1024 in 64 x 64 tiles 25.5 us, 29.2, 39.7.)
    Frags f;
    Regs r;
    load(r);
    stage(r, lds);
    load(r);
    __syncthreads();
    auto step = [&](const char* __restrict__ cur, char* __restrict__ nxt) {
        read(f, cur, 0);
        stage(r, nxt);
        products(f);
        read(f, cur, 1);
        load(r);
        products(f);
        __syncthreads();
    };
    for (int c = 0; c < chunks; c += 2) {  // (chunks past the last are zeros, or another group's)
        step(lds, lds + C::STAGE);
        if (C::kKW > 1 && c + 1 == chunks) break;
        step(lds + C::STAGE, lds);
    }

    // Values the split does not hold. Rows and columns past the last are copies of the
    // last, so all accumulators count.
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < BM; ++i)
#pragma unroll
        for (int j = 0; j < BN; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const float x = acc[i][j][v] + low[i][j][v];
                acc[i][j][v] = x;
                const uint32_t bits = __builtin_bit_cast(uint32_t, x) & 0x7fffffffu;
                most = bits > most ? bits : most;
            }
    if (lost & 0xffffu) lost_s = 1;
    __syncthreads();
    float* const mine = reinterpret_cast<float*>(all) + wave * 32 * (32 * BN + 4);
    const int32_t mw = m0 + wm * BM * 32, nw = n0 + wn * BN * 32;
    if (lost_s || __any(most >= 0x7f800000u)) {
        const int64_t ars = C::kAT ? 1 : p.lda, aks = C::kAT ? p.lda : 1;
        const int64_t brs = C::kBT ? 1 : p.ldb, bks = C::kBT ? p.ldb : 1;
#pragma unroll
        for (int i = 0; i < BM; ++i)
#pragma unroll
            for (int j = 0; j < BN; ++j) {
                int32_t m = mw + i * 32 + (lane & 31), n = nw + j * 32 + (lane & 31);
                m = m < p.M ? m : p.M - 1;
                n = n < p.N ? n : p.N - 1;
                acc[i][j] = plain_block(A + m * ars + k0 * aks, aks, B + n * brs + k0 * bks, bks, (int32_t)(k1 - k0), lane);
            }
    }
    if constexpr (C::kKW > 1) {  // the groups' sums, joined in their order by the first
        float* const sums = reinterpret_cast<float*>(all + C::EPI) + wave * 1024 + lane * 4;
        if (group) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<f32x4v*>(sums + (group - 1) * C::WAVES * 1024 + q * 256) =
                    f32x4v{acc[0][0][4 * q], acc[0][0][4 * q + 1], acc[0][0][4 * q + 2], acc[0][0][4 * q + 3]};
        }
        __syncthreads();
        if (group) return;
#pragma unroll
        for (int g = 1; g < C::kKW; ++g)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x4v s = *reinterpret_cast<const f32x4v*>(sums + (g - 1) * C::WAVES * 1024 + q * 256);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[0][0][4 * q + e] += s[e];
            }
    }
    if constexpr (SQUARE) {
        if (symmetric && mt != nt) mirror(p, acc[0][0], mw, nw, bat, split, lane);
    }
    epilogue<float, BM, BN>(p, acc, mine, mw, nw, bat, split, lane);
}

template <class C>
__global__ __launch_bounds__(C::THREADS * C::kKW, C::kPerSimd) void product_f32_kernel(Product p) {
    __shared__ __align__(16) char all[C::LDS];
    __shared__ uint32_t lost_s;
    product_f32<C>(p, xcd_remap(blockIdx.x, gridDim.x), all, lost_s);
}

// The two products of a backward pass, dX = dZ K^T and dK = X^T dZ, side by side in one launch: the
// tiles of one fill the compute units that the other's last round leaves.
template <class X, class K>
__global__ __launch_bounds__(X::THREADS, X::kPerSimd) void product_f32_pair_kernel(Product x, Product k, uint32_t x_blocks) {
    static_assert(X::LDS == K::LDS && X::kKW == 1 && K::kKW == 1, "one shape of tiles");
    __shared__ __align__(16) char all[X::LDS];
    __shared__ uint32_t lost_s;
    if (blockIdx.x < x_blocks) product_f32<X>(x, xcd_remap(blockIdx.x, x_blocks), all, lost_s);
    else product_f32<K>(k, xcd_remap(blockIdx.x - x_blocks, gridDim.x - x_blocks), all, lost_s);
}

// Fills what the kernels need; the workgroups, or 0 past the grid or for shares that leave some empty.
template <class C>
uint32_t prepare(Product& p) {
    p.m_tiles = (p.M + C::TM - 1) / C::TM;
    p.n_tiles = (p.N + C::TN - 1) / C::TN;
    // shares are whole multiples of 64 elements, as plan_product counts them
    const int64_t chunks = 2 * (((int64_t)p.K + 63) / 64);
    p.chunks = 2 * (int32_t)((chunks / 2 + p.splits - 1) / p.splits);
    const int64_t tiles = p.symmetric ? (int64_t)p.m_tiles * (p.m_tiles + 1) / 2 : (int64_t)p.m_tiles * p.n_tiles;
    const int64_t blocks = tiles * p.splits * p.batch;
    return blocks > kMaxThreads / (C::THREADS * C::kKW) || (p.splits - 1) * (int64_t)p.chunks >= chunks ? 0 : (uint32_t)blocks;
}

template <int BM, int BN, int WM, int WN, int KW, Layout L>
hipError_t run(Product p, hipStream_t stream) {
    using C = Cfg<BM, BN, WM, WN, KW, L, false>;
    const uint32_t blocks = prepare<C>(p);
    if (!blocks) return hipErrorInvalidValue;
    if constexpr (L != Layout::kXtK) {
        if (p.K % 8) {
            using G = Cfg<BM, BN, WM, WN, KW, L, true>;
            hipLaunchKernelGGL(product_f32_kernel<G>, dim3(blocks), dim3(G::THREADS * KW), 0, stream, p);
            return hipGetLastError();
        }
    }
    hipLaunchKernelGGL(product_f32_kernel<C>, dim3(blocks), dim3(C::THREADS * KW), 0, stream, p);
    return hipGetLastError();
}

template <Layout L>
hipError_t pick(const Product& p, int tile, hipStream_t stream) {
    switch (tile) {
        case 1: return run<1, 2, 4, 1, 1, L>(p, stream);
        case 2: return run<2, 2, 4, 2, 1, L>(p, stream);
        case 3: return run<1, 1, 2, 2, 1, L>(p, stream);
        case 4: return run<1, 1, 2, 2, 3, L>(p, stream);
        default: return hipErrorNotSupported;
    }
}

}  // namespace

hipError_t launch_product_f32_pair(Product x, Product k, hipStream_t stream) {
    using X = Cfg<1, 1, 2, 2, 1, Layout::kXKt, false>;
    using XTail = Cfg<1, 1, 2, 2, 1, Layout::kXKt, true>;
    using K = Cfg<1, 1, 2, 2, 1, Layout::kXtK, false>;
    const uint32_t bx = prepare<X>(x), bk = prepare<K>(k);
    if (!bx || !bk || (int64_t)bx + bk > kMaxThreads / X::THREADS) return hipErrorInvalidValue;
    const dim3 grid(bx + bk), block(X::THREADS);
    if (x.K % 8) hipLaunchKernelGGL((product_f32_pair_kernel<XTail, K>), grid, block, 0, stream, x, k, bx);
    else hipLaunchKernelGGL((product_f32_pair_kernel<X, K>), grid, block, 0, stream, x, k, bx);
    return hipGetLastError();
}

hipError_t launch_product_f32(Layout layout, Product p, int tile, hipStream_t stream) {
    switch (layout) {
        case Layout::kXK: return pick<Layout::kXK>(p, tile, stream);
        case Layout::kXKt: return pick<Layout::kXKt>(p, tile, stream);
        default: return pick<Layout::kXtK>(p, tile, stream);
    }
}

}  // namespace mec
