// bf16 matrix products of the layer operators (mec_product.h), on v_mfma_f32_32x32x16_bf16.
//
// A workgroup computes a tile of Y, 32*BM*WM x 32*BN*WN, from chunks of KT (64 or 32) of the
// reduction in stages of LDS: while one chunk's products run, the next (of 4 stages: the next
// three) are on their way. Operands are staged as they are stored:
//   stored along the reduction ([m][k], [n][k])  rows of KT k; granule g (8 k) of row r at
//     g ^ (r & 7) (KT 32: g ^ (r / 2 & 3)); a fragment (8 k of one row per lane) is one
//     16-byte read
//   stored across it ([k][m], [k][n])  rows of one k; the 32-byte blocks (16 columns) of row
//     k at block ^ (k & 7); a fragment is two transposing reads (ds_read_b64_tr_b16: 16
//     lanes read 4 rows of 16 columns and each gets 4 k of one column)
// Both orders put the lanes that read together on different banks. Rows of whole 16-byte
// granules go straight to LDS (buffer_load .. lds; what lies past the end of the reduction
// is past the resource's end and arrives as zeros); others go through registers.
//
// dZ of the two gradients may come as two matrices whose sum it is (Product::second): chunks
// of the one and of the other take turns, against the same chunk of the other operand, so
// that dX and dK are as from dZ in 16 significant bits, at twice the products.
#include "mec_product.h"
#include "mec_split.h"

namespace mec {
namespace {

// BM x BN 32 x 32 blocks per wave, WM x WN waves, chunks of KT, S stages of LDS (DMA).
template <int BM, int BN, int WM, int WN, int KT, int S, Layout L, bool DMA>
struct Cfg {
    static constexpr int kKT = KT, kS = DMA ? S : 2;
    static constexpr int kBM = BM, kBN = BN, kWM = WM, kWN = WN;
    static constexpr bool kAT = L == Layout::kXtK;   // A stored [k][m]
    static constexpr bool kBT = L != Layout::kXKt;   // B stored [k][n]
    static constexpr bool kDMA = DMA;
    static constexpr bool kGrad = L != Layout::kXK;  // dZ, A of dX and B of dK, may come in two parts
    static constexpr int TM = 32 * BM * WM, TN = 32 * BN * WN, WAVES = WM * WN, THREADS = 64 * WAVES;
    static constexpr int AB = TM * kKT * 2, BB = TN * kKT * 2, STAGE = AB + BB;  // bytes
    static constexpr int kLoads = (TM + TN) * (KT / 8) / THREADS;                // granules per thread
    static constexpr int EPI = WAVES * 32 * (32 * BN + 4) * 4;
    static constexpr int LDS = kS * STAGE > EPI ? kS * STAGE : EPI;
    static_assert(TM * (KT / 8) % THREADS == 0 && TN * (KT / 8) % THREADS == 0 && LDS <= 160 * 1024, "tile");
    static_assert((kS - 2) * kLoads < 64, "loads in flight");
};

// A raw buffer of `bytes` from `base` (both uniform), as the load's four scalar registers.
__device__ inline u32x4v resource(const char* base, int64_t bytes) {
    const uint64_t a = (uint64_t)base;
    return u32x4v{(uint32_t)a, (uint32_t)(a >> 32) & 0xffffu, bytes > 0x7fffffff ? 0x7fffffffu : (uint32_t)bytes, 0x00027000u};
}

// 16 bytes per lane from the buffer at voff straight to LDS, at lds + 16 * lane; zeros from
// past its end. The compiler does not see the load: the caller waits on vmcnt before the
// data is read. M0 holds the LDS address; it cannot be declared clobbered and is put back.
__device__ inline void to_lds16(u32x4v rsrc, uint32_t voff, uint32_t lds) {
    uint32_t saved;
    asm volatile(
        "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds\n\ts_mov_b32 m0, %0"
        : "=&s"(saved)
        : "s"(lds), "v"(voff), "s"(rsrc)
        : "memory");
}

// w without its first s elements (0 to 8), zeros after the last
__device__ inline u32x4v shifted_down(u32x4v w, int s) {
    if (s & 1) w = u32x4v{w[0] >> 16 | w[1] << 16, w[1] >> 16 | w[2] << 16, w[2] >> 16 | w[3] << 16, w[3] >> 16};
    if (s & 2) w = u32x4v{w[1], w[2], w[3], 0};
    if (s & 4) w = u32x4v{w[2], w[3], 0, 0};
    if (s & 8) w = u32x4v{0, 0, 0, 0};
    return w;
}

// One operand's T rows (stored along the reduction) or columns (TR: across it) of a tile.
// Items of 16 bytes per thread.
template <int T, int THREADS, int KT, bool TR, bool DMA>
struct Operand {
    static constexpr int G = KT / 8;  // granules along a chunk
    static constexpr int ITEMS = T * G / THREADS;
    static constexpr int SW = T / 16 < 8 ? T / 16 - 1 : 7;
    const char* base;   // uniform: the tile's first row and the chunk's first k
    int64_t step;       // bytes from chunk to chunk
    int64_t left;       // uniform: DMA, TR: bytes of rows from base on; else elements of the reduction from base on
    int64_t ld;         // elements
    uint32_t voff[TR && DMA ? 1 : ITEMS];  // bytes from base
    int32_t have;       // TR: columns from this thread's on
    int32_t k_at;       // first k of this thread's granule(s)
    bool inner;         // uniform; not DMA, TR: every column of the tile is there
    bool room;          // uniform; not DMA, not TR: rows have 8 elements before the reduction's end

    static __device__ inline int swizzle(int row) { return KT == 64 ? row & 7 : (row >> 1) & 3; }

    // rows r0 .. of `count` rows (columns) of `ld` elements, reduction from k0 to k1
    __device__ inline void init(const void* mem, int64_t ld_, int32_t r0, int32_t count, int64_t k0, int64_t k1, int tid) {
        ld = ld_;
        if constexpr (TR) {
            const int pos = tid % (T / 8), k = tid / (T / 8);
            const int col = (((pos >> 1) ^ (k & SW)) * 2 + (pos & 1)) * 8;
            base = uniform(static_cast<const char*>(mem) + 2 * (k0 * ld + r0));
            step = 2 * KT * ld;
            have = count - r0 - col;
            k_at = k;
            if constexpr (DMA) {
                // columns past the last read the last 8 instead (count is a multiple of 8)
                voff[0] = 2u * (uint32_t)(k * ld + (have > 0 ? col : count - r0 - 8));
                left = 2 * ((k1 - k0) * ld - r0);
            } else {
#pragma unroll
                for (int i = 0; i < ITEMS; ++i) voff[i] = 2u * (uint32_t)((k + i * (THREADS * 8 / T)) * ld + (have > 0 ? col : 0));
                inner = r0 + T <= count;
                left = k1 - k0;
            }
        } else {
            const int row = tid / G, kg = (tid % G) ^ swizzle(row);
            base = uniform(static_cast<const char*>(mem) + 2 * (r0 * ld + k0));
            step = 2 * KT;
            left = k1 - k0;
            room = k1 >= 8;
            k_at = 8 * kg;
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                int r = row + i * (THREADS / G);
                if (r0 + r >= count) r = count - 1 - r0;  // rows past the last are not stored
                voff[i] = 2u * (uint32_t)(r * ld + 8 * kg);
            }
        }
    }
    // To the next chunk, or (on false) not along the reduction, and `jump` bytes to dZ's other part.
    __device__ inline void next(bool on, int64_t jump) {
        base += (on ? step : 0) + jump;
        left -= on ? (TR && DMA ? step : KT) : 0;
    }
    // DMA: this chunk to LDS at `to`
    __device__ inline void stage(uint32_t to, int wave) const {
        if constexpr (TR) {
            const u32x4v rs = resource(base, left > 0 ? left : 0);
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
                to_lds16(rs, voff[0] + (uint32_t)(i * (THREADS * 8 / T)) * 2u * (uint32_t)ld, to + (uint32_t)(i * THREADS + wave * 64) * 16u);
        } else {
            const u32x4v rs = resource(base, 0x7fffffff);
            const bool past = k_at >= left;
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
                to_lds16(rs, past ? 0x80000000u : voff[i], to + (uint32_t)(i * THREADS + wave * 64) * 16u);
        }
    }
    // else: this chunk to registers, and from there to LDS. All its loads are in flight
    // together: a granule that the row cuts off is read whole where what follows it in memory
    // is the matrix too (TR: columns past the last are not stored), or from 8 elements before
    // the row's end and shifted down (element by element, every load waited for in turn,
    // 99580 x 240 x 816 of dK took 253 us, so 196).
    __device__ inline void load(u32x4v* r) const {
        auto at = [&](int i) { return reinterpret_cast<const uint16_t*>(base + voff[i]); };
        if (left >= KT && (!TR || inner || left >= KT + 8)) {  // (uniform)
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) r[i] = load_any(at(i));
        } else if (TR || !room) {
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                if constexpr (TR) r[i] = load_some(at(i), k_at + i * (THREADS * 8 / T) < left ? have : 0);
                else r[i] = load_some(at(i), left - k_at);
            }
        } else {
            const int64_t over = k_at + 8 - left;
            const int shift = over < 0 ? 0 : over < 8 ? (int)over : 8;
            const int64_t back = over > 0 ? over : 0;
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) r[i] = load_any(at(i) - back);
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) r[i] = shifted_down(r[i], shift);
        }
    }
    static __device__ inline void put(const u32x4v* r, char* to, int tid) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) *reinterpret_cast<u32x4v*>(to + (i * THREADS + tid) * 16) = r[i];
    }
    // the fragment of 32-row block blk for the 16 k from 16*kk on
    static __device__ inline bf16x8 frag(const char* from, int blk, int kk, int lane) {
        if constexpr (TR) {
            const int p = lane & 15, c16 = blk * 2 + ((lane >> 4) & 1);
            s16x4 h[2];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int k = kk * 16 + 8 * (lane >> 5) + 4 * s + (p >> 2);
                h[s] = read_tr(from + k * (T * 2) + ((c16 ^ (k & SW)) << 5) + (p & 3) * 8);
            }
            return join_tr(h[0], h[1]);
        } else {
            const int r = blk * 32 + (lane & 31), g = 2 * kk + (lane >> 5);
            return *reinterpret_cast<const bf16x8*>(from + r * (KT * 2) + ((g ^ swizzle(r)) << 4));
        }
    }
};

// Workgroup b's tile, in C::LDS bytes of LDS.
template <class C>
__device__ inline void product_bf16(const Product& p, uint32_t b, char* lds) {
    constexpr int BM = C::kBM, BN = C::kBN, KT = C::kKT;
    using OpA = Operand<C::TM, C::THREADS, C::kKT, C::kAT, C::kDMA>;
    using OpB = Operand<C::TN, C::THREADS, C::kKT, C::kBT, C::kDMA>;
    const int tid = threadIdx.x, lane = tid & 63, wave = (int)uniform((uint32_t)tid >> 6);
    const int wm = wave % C::kWM, wn = wave / C::kWM;
    const uint32_t tiles = (uint32_t)p.m_tiles * (uint32_t)p.n_tiles;
    const uint32_t split = b / tiles;
    uint32_t mt, nt;
    tile_of(b - split * tiles, (uint32_t)p.m_tiles, (uint32_t)p.n_tiles, 8u, mt, nt);
    const int32_t m0 = (int32_t)mt * C::TM, n0 = (int32_t)nt * C::TN;
    const int64_t k0 = (int64_t)split * p.chunks * KT;
    const int64_t k1 = k0 + (int64_t)p.chunks * KT < p.K ? k0 + (int64_t)p.chunks * KT : p.K;
    const bool two = C::kGrad && p.second != 0;
    const int chunks = (int)((k1 - k0 + KT - 1) / KT) << (two ? 1 : 0);

    OpA a;
    OpB bb;
    a.init(p.A, p.lda, m0, p.M, k0, k1, tid);
    bb.init(p.B, p.ldb, n0, p.N, k0, k1, tid);
    const uint32_t at = (uint32_t)(uintptr_t)(lds_char*)lds;

    floatx16 acc[BM][BN] = {};
    struct Frags {
        bf16x8 a[BM], b[BN];
    };
    auto read = [&](Frags& f, const char* from, int kk) {
#pragma unroll
        for (int i = 0; i < BM; ++i) f.a[i] = OpA::frag(from, wm * BM + i, kk, lane);
#pragma unroll
        for (int j = 0; j < BN; ++j) f.b[j] = OpB::frag(from + C::AB, wn * BN + j, kk, lane);
    };
    auto multiply = [&](const Frags& f) {
#pragma unroll
        for (int i = 0; i < BM; ++i)
#pragma unroll
            for (int j = 0; j < BN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.b[j], f.a[i], acc[i][j], 0, 0, 0);
    };
    auto products = [&](const char* from) {
#pragma unroll
        for (int kk = 0; kk < KT / 16; ++kk) {
            Frags f;
            read(f, from, kk);
            multiply(f);
        }
    };
    bool on = !two;
    int64_t jump = two ? p.second : 0;
    auto next = [&] {
        a.next(on, C::kAT ? 0 : jump);
        bb.next(on, C::kAT ? jump : 0);
        on = on != two;
        jump = -jump;
    };
    auto stage = [&](uint32_t to) {
        a.stage(at + to, wave);
        bb.stage(at + to + C::AB, wave);
        next();
    };
    if constexpr (C::kDMA && C::kS > 2) {
        // S - 1 chunks on their way; those past the last are zeros, so that the loads in
        // flight stay the same number. Fragments are read one step of 16 k ahead of their
        // products, across the chunks' borders too.
        constexpr int S = C::kS, STEPS = KT / 16;
        uint32_t now = 0, then = (S - 1) * C::STAGE;
        auto after = [&](uint32_t x) { return x + C::STAGE == S * C::STAGE ? 0u : x + C::STAGE; };
#pragma unroll
        for (int s = 0; s < S - 1; ++s) stage(s * C::STAGE);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((S - 2) * C::kLoads) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        Frags f[2];
        read(f[0], lds, 0);
        static_assert(STEPS % 2 == 0, "the first fragments of a chunk go to f[0]");
        for (int c = 0; c < chunks; ++c) {
#pragma unroll
            for (int kk = 0; kk < STEPS; ++kk) {
                if (kk + 1 < STEPS) {
                    read(f[(kk + 1) % 2], lds + now, kk + 1);
                } else {
                    // the next chunk has arrived for every wave, and none reads the last one's
                    // stage any more: its fragments went into products before this chunk's
                    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((S - 3) * C::kLoads) : "memory");
                    __builtin_amdgcn_s_barrier();
                    asm volatile("" ::: "memory");
                    now = after(now);
                    read(f[(kk + 1) % 2], lds + now, 0);
                    stage(then);
                    then = after(then);
                }
                multiply(f[kk % 2]);
                if constexpr (BM * BN > 1) {
#pragma unroll
                    for (int g = 0; g < BM * BN; ++g) {
                        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // MFMA
                        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);  // LDS read
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    } else if constexpr (C::kDMA) {
        stage(0);
        for (int c = 0; c < chunks; ++c) {
            const uint32_t now = (c & 1) * C::STAGE, then = C::STAGE - now;
            // this chunk has arrived for every wave, and none reads the other stage any more
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (c + 1 < chunks) stage(then);
            products(lds + now);
        }
    } else {
        u32x4v ra[OpA::ITEMS], rb[OpB::ITEMS];
        a.load(ra);
        bb.load(rb);
        OpA::put(ra, lds, tid);
        OpB::put(rb, lds + C::AB, tid);
        for (int c = 0; c < chunks; ++c) {
            const uint32_t now = (c & 1) * C::STAGE, then = C::STAGE - now;
            __syncthreads();
            const bool more = c + 1 < chunks;
            if (more) {
                next();
                a.load(ra);
                bb.load(rb);
            }
            products(lds + now);
            if (more) {
                OpA::put(ra, lds + then, tid);
                OpB::put(rb, lds + then + C::AB, tid);
            }
        }
    }
    if constexpr (C::kGrad) {
        bool odd = false;
        if (two)
#pragma unroll
            for (int i = 0; i < BM; ++i)
#pragma unroll
                for (int j = 0; j < BN; ++j) odd |= not_finite(acc[i][j]);
        if (odd) {
            const int64_t ars = C::kAT ? 1 : p.lda, aks = C::kAT ? p.lda : 1, brs = C::kBT ? 1 : p.ldb, bks = C::kBT ? p.ldb : 1;
            const int32_t len = (int32_t)(k1 - k0);
            auto row = [&](int i) {
                const int32_t m = m0 + (wm * BM + i) * 32 + (lane & 31);
                return static_cast<const uint16_t*>(p.A) + k0 * aks + (m < p.M ? m : p.M - 1) * ars;
            };
            auto column = [&](int j) {
                const int32_t n = n0 + (wn * BN + j) * 32 + (lane & 31);
                return static_cast<const uint16_t*>(p.B) + k0 * bks + (n < p.N ? n : p.N - 1) * brs;
            };
#pragma unroll
            for (int o = 0; o < (C::kAT ? BM : BN); ++o)
                if (holds_infinity(C::kAT ? row(o) : column(o), C::kAT ? aks : bks, len, lane))
#pragma unroll
                    for (int q = 0; q < (C::kAT ? BN : BM); ++q)
                        take_again(acc[C::kAT ? o : q][C::kAT ? q : o], row(C::kAT ? o : q), aks, column(C::kAT ? q : o), bks, len, lane);
        }
    }
    __syncthreads();
    float* const mine = reinterpret_cast<float*>(lds) + wave * 32 * (32 * BN + 4);
    epilogue<uint16_t, BM, BN>(p, acc, mine, m0 + wm * BM * 32, n0 + wn * BN * 32, 0, (int32_t)split, lane);
}

template <class C>
__global__ __launch_bounds__(C::THREADS) void product_bf16_kernel(Product p) {
    __shared__ __align__(16) char lds[C::LDS];
    product_bf16<C>(p, xcd_remap(blockIdx.x, gridDim.x), lds);
}

// The two products of a backward pass in one launch, as in fp32.
template <class X, class K>
__global__ __launch_bounds__(X::THREADS) void product_bf16_pair_kernel(Product x, Product k, uint32_t x_blocks) {
    static_assert(X::LDS == K::LDS && X::THREADS == K::THREADS, "one shape of tiles");
    __shared__ __align__(16) char lds[X::LDS];
    if (blockIdx.x < x_blocks) product_bf16<X>(x, xcd_remap(blockIdx.x, x_blocks), lds);
    else product_bf16<K>(k, xcd_remap(blockIdx.x - x_blocks, gridDim.x - x_blocks), lds);
}

// Fills what the kernels need; the workgroups, or 0 past the grid or for shares that leave some empty.
template <class C>
uint32_t prepare(Product& p) {
    constexpr int KT = C::kKT;
    p.m_tiles = (p.M + C::TM - 1) / C::TM;
    p.n_tiles = (p.N + C::TN - 1) / C::TN;
    // shares are whole multiples of 64 elements
    const int64_t chunks = 64 / KT * (((int64_t)p.K + 63) / 64);
    p.chunks = 64 / KT * (int32_t)((chunks / (64 / KT) + p.splits - 1) / p.splits);
    const int64_t blocks = (int64_t)p.m_tiles * p.n_tiles * p.splits;
    return blocks > kMaxThreads / C::THREADS || (p.splits - 1) * (int64_t)p.chunks >= chunks ? 0 : (uint32_t)blocks;
}

template <int BM, int BN, int WM, int WN, int KT, int S, Layout L>
hipError_t run(Product p, hipStream_t stream) {
    using C = Cfg<BM, BN, WM, WN, KT, S, L, true>;
    const uint32_t blocks = prepare<C>(p);
    if (!blocks) return hipErrorInvalidValue;
    if (p.clean) {
        hipLaunchKernelGGL(product_bf16_kernel<C>, dim3(blocks), dim3(C::THREADS), 0, stream, p);
    } else {
        using G = Cfg<BM, BN, WM, WN, KT, 2, L, false>;
        hipLaunchKernelGGL(product_bf16_kernel<G>, dim3(blocks), dim3(G::THREADS), 0, stream, p);
    }
    return hipGetLastError();
}

template <Layout L>
hipError_t pick(const Product& p, int tile, hipStream_t stream) {
    switch (tile) {
        case 1: return run<2, 2, 2, 2, 64, 2, L>(p, stream);
        case 2: return run<4, 2, 2, 4, 32, 4, L>(p, stream);
        case 3: return run<1, 2, 2, 2, 64, 2, L>(p, stream);
        case 4: return run<1, 1, 2, 2, 64, 2, L>(p, stream);
        case 5: return run<1, 1, 2, 2, 64, 4, L>(p, stream);
        default: return hipErrorNotSupported;
    }
}

}  // namespace

hipError_t launch_product_bf16_pair(Product x, Product k, hipStream_t stream) {
    using X = Cfg<1, 2, 2, 2, 64, 2, Layout::kXKt, true>;
    using K = Cfg<1, 2, 2, 2, 64, 2, Layout::kXtK, true>;
    if (!clean_rows(Layout::kXKt, x) || !clean_rows(Layout::kXtK, k)) return hipErrorInvalidValue;
    const uint32_t bx = prepare<X>(x), bk = prepare<K>(k);
    if (!bx || !bk || (int64_t)bx + bk > kMaxThreads / X::THREADS) return hipErrorInvalidValue;
    hipLaunchKernelGGL((product_bf16_pair_kernel<X, K>), dim3(bx + bk), dim3(X::THREADS), 0, stream, x, k, bx);
    return hipGetLastError();
}

hipError_t launch_product_bf16(Layout layout, Product p, int tile, hipStream_t stream) {
    p.clean = clean_rows(layout, p);
    switch (layout) {
        case Layout::kXK: return pick<Layout::kXK>(p, tile, stream);
        case Layout::kXKt: return pick<Layout::kXKt>(p, tile, stream);
        default: return pick<Layout::kXtK>(p, tile, stream);
    }
}

}  // namespace mec
