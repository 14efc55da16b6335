// Which kernel computes a product of the layer operators. The times of each are modelled and
// the least taken: a tile kernel's busiest compute unit takes ceil(tiles / 256) tiles, as many
// at a time as fit, at the cost below per chunk of the reduction with 1, 2, .. resident and
// per tile for its start and end; the small kernel's one workgroup at a time, at a cost per
// round and per element of the reduction. All in us, measured on this GPU on long and short
// reductions over few and many tiles (M x N x K, us): bf16 16384 x 4096 x 4096 256x256 471,
// 128x128 526, 64x128 619, 64x64 746; 1024 x 1024 x 1024 34, 16.0, 11.5, 8.5 and small 19;
// 512 x 512 x 64 small 4.0, 128x128 7.4. fp32 16384 x 4096 x 1024 256x128 694, 128x64 862,
// 64x64 928; 1024 x 1024 x 1024 69, 37, 25 (in three groups 22) and small 36; 512 x 512 x 512
// small 6.7.
#include "mec_product.h"

namespace mec {
namespace {

struct TileCost {
    int tm, tn, threads, fit;
    double chunk[5], ends, residual, saved;  // residual, saved: what R and Z add to the ends
};
// by the kernels' numbers, from 1. Large tiles wait longer for a residual than small ones, of
// which others run meanwhile: 1577088 x 64 -> 256 in bf16 281, 239, 297, 367 us, with Z 440, 409,
// 458, 555, with R 415, 367, 329, 365, with both 531, 496, 455, 499; in fp32 744, 661, 804, with Z
// 1128, 1000, 1219, with R 833, 819, 970, with both 1031, 1087, 1178.
constexpr TileCost kBf16[] = {{128, 128, 256, 2, {0.57, 1.00}, 4.2, 2.5, 3.6},
                              {256, 256, 512, 1, {1.45}, 8.5, 5.3, 6.8},
                              {64, 128, 256, 3, {0.40, 0.70, 0.85}, 3.5, 0.4, 2.2},
                              {64, 64, 256, 5, {0.32, 0.50, 0.65, 0.80, 0.85}, 3.4, 0.0, 2.2},
                              {64, 64, 256, 2, {0.26, 0.38}, 3.8, 0.4, 1.0}};
// the same by way of registers (rows that are no whole 16-byte granules): 1886 x 3185 -> 2368
// 95, 157, 81, 110 where 3184 takes 50, 62, 50, 62; 11471 x 2505 -> 48 65, 124, 51, 43
constexpr TileCost kBf16Any[] = {{128, 128, 256, 2, {1.50, 1.80}, 4.2, 2.5, 3.6},
                                 {256, 256, 512, 1, {2.90}, 8.5, 5.3, 6.8},
                                 {64, 128, 256, 3, {1.19, 1.35, 1.55}, 3.5, 0.4, 2.2},
                                 {64, 64, 256, 5, {0.80, 1.10, 1.45, 1.80, 2.10}, 3.4, 0.0, 2.2}};
constexpr TileCost kF32[] = {{128, 64, 256, 2, {0.90, 1.55}, 4.8, 0.9, 3.2},
                             {256, 128, 512, 1, {2.3}, 10.0, 3.3, 6.5},
                             {64, 64, 256, 3, {0.64, 0.95, 1.15}, 5.0, 1.0, 2.5},
                             {64, 64, 768, 1, {0.48}, 7.0, 1.0, 2.5}};

constexpr int kPair = 3;          // the kernel whose tiles a pair of products takes
constexpr int kSymmetricF32 = 3;  // the fp32 kernels from this one on have square tiles

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

double tile_time(const TileCost& t, int64_t tiles, int64_t chunks, double ends) {
    const int64_t busiest = ceil_div(tiles, 256), rounds = busiest / t.fit, rest = busiest % t.fit;
    double us = (double)rounds * ((double)chunks * t.chunk[t.fit - 1] + ends);
    if (rest) us += (double)chunks * t.chunk[rest - 1] + ends;
    return us;
}

}  // namespace

ProductPlan plan_product(Layout layout, int dtype, int64_t M, int64_t N, int64_t K, int32_t batch, int32_t max_splits,
                         bool symmetric, const Operands& with) {
    const bool clean = with.clean;
    const TileCost* const tiles = !dtype ? kF32 : clean ? kBf16 : kBf16Any;
    const int count = dtype && clean ? 5 : 4;
    const int64_t parts = with.two ? 2 : 1;  // chunks of each take turns
    const int64_t chunks = parts * ceil_div(K, dtype ? 64 : 32), shares = ceil_div(K, 64);
    // A call of one product in shares takes its caller's thread a second launch and a workspace
    // (13 us, so 8; 1 x 2048 x 1000 in bf16 in one launch 7.5 us, in shares 14.0): below that
    // the GPU's time is not what counts. Where other launches stand around it anyway
    // (dK, a symmetric product) it is.
    const bool alone = layout != Layout::kXtK && !symmetric;
    ProductPlan best{-1, 1, 1e30};
    double least = 1e30;
    auto offer = [&](int32_t kernel, int64_t splits, double us) {
        const double host = !alone ? 0.0 : splits > 1 ? 13.0 : 8.0, t = us > host ? us : host;
        if (t < least || (t == least && us < best.us)) {
            least = t;
            best = {kernel, (int32_t)splits, us};
        }
    };
    const double per_k = !dtype ? 0.0066 : clean ? 0.0027 : layout == Layout::kXKt ? 0.0075 : 0.0040;
    const int64_t small = ceil_div(M, 32) * ceil_div(N, 32) * batch;
    if (small <= kMaxSmallBlocks) offer(0, 1, (double)ceil_div(small, 256) * (4.0 + per_k * (double)(parts * K)));
    for (int i = 0; i < count; ++i) {
        int64_t n = ceil_div(M, tiles[i].tm) * ceil_div(N, tiles[i].tn);
        if (symmetric && !dtype && i + 1 >= kSymmetricF32) n = (n + ceil_div(M, tiles[i].tm)) / 2;
        n *= batch;
        for (int64_t s = 1; s <= max_splits; s = s < 4 ? s + 1 : s + s / 4) {
            // shares of at least 4 chunks of 64, none empty, and partial sums of at most 256 MB
            if (s > 1 && (shares < 4 * s || s * batch * M * N > (int64_t(1) << 26))) break;
            const int64_t per = ceil_div(shares, s), real = ceil_div(shares, per);
            if (n * real > kMaxThreads / tiles[i].threads) break;
            const double ends = tiles[i].ends + (s > 1 ? 0.0 : (with.R ? tiles[i].residual : 0.0) + (with.Z ? tiles[i].saved : 0.0));
            double us = tile_time(tiles[i], n * real, s > 1 ? parts * per * (dtype ? 1 : 2) : chunks, ends);
            // the sum of the shares: a launch, its reads, and what else moves (the epilogue's
            // output; a mirror image's 4-byte stores)
            if (real > 1) us += (alone ? 4.0 : 3.0) + (double)((alone ? real + 1 : symmetric ? 2 * real : real) * batch * M * N) / 1.2e6;
            offer(i + 1, real, us);
        }
    }
    return best;
}

ProductPlan plan_pair(const ProductPlan& px, const ProductPlan& pk, int dtype, int64_t rows, int64_t i_c, int64_t k_c,
                      int32_t max_splits, bool two) {
    ProductPlan best{0, 1, 0.0};
    // What two launches take, by their models and a launch's own 3 us; the model of the pair is a
    // little too high (1000 x 1000 x 1000 49 where it took 44, two launches 50; 4608 x 256 x 1024
    // 57, 53 and 62; 20000 x 256 x 1024 166, 177 and 160; 11679 x 920 x 1619 508, 549 and 467;
    // bf16 2447 x 872 x 2144 40 and 60, 6272 x 1024 x 256 28 and 34, but 800 x 512 x 2048 27 and 24).
    best.us = 3.0 + 1.05 * (px.us + pk.us);
    const TileCost& t = (dtype ? kBf16 : kF32)[kPair - 1];
    const int64_t step = dtype ? 64 : 32;
    const int64_t nx = ceil_div(rows, t.tm) * ceil_div(i_c, t.tn), nk = ceil_div(i_c, t.tm) * ceil_div(k_c, t.tn);
    const int64_t shares = ceil_div(rows, 64);
    auto tile = [&](int64_t chunks) { return (double)(two ? 2 * chunks : chunks) * t.chunk[t.fit - 1] + t.ends; };
    for (int64_t s = 1; s <= max_splits; s = s < 4 ? s + 1 : s + s / 4) {
        if (s > 1 && (shares < 4 * s || s * i_c * k_c > (int64_t(1) << 26))) break;
        const int64_t per = ceil_div(shares, s), real = ceil_div(shares, per);
        if (nx + nk * real > kMaxThreads / t.threads) break;
        const double x = tile(ceil_div(k_c, step)), k = tile(real > 1 ? per * 64 / step : ceil_div(rows, step));
        // the compute units are full but for the last tile's time
        double us = ((double)nx * x + (double)(nk * real) * k) / (256.0 * t.fit);
        us += 0.5 * (x > k ? x : k);
        if (real > 1) us += 3.0 + (double)(real * i_c * k_c) / 1.2e6;
        if (us < best.us) best = {kPair, (int32_t)real, us};
    }
    return best;
}

bool clean_rows(Layout layout, const Product& p) {
    auto rows16 = [](const void* base, int64_t ld) { return ((uintptr_t)base & 15u) == 0 && ld % 8 == 0; };
    // the dimension that each operand's rows run along has to be whole granules
    const int64_t a_run = layout == Layout::kXtK ? p.M : p.K, b_run = layout == Layout::kXKt ? p.K : p.N;
    return rows16(p.A, p.lda) && rows16(p.B, p.ldb) && a_run % 8 == 0 && b_run % 8 == 0;
}

ProductPlan refine_plan(const ProductPlan& plan, Layout layout, int dtype, const Product& p) {
    const Operands with{!dtype || clean_rows(layout, p), p.R != nullptr, p.Z != nullptr, p.second != 0};
    return with.clean && !with.R && !with.Z ? plan : plan_product(layout, dtype, p.M, p.N, p.K, 1, plan.splits, false, with);
}

hipError_t launch_product(const ProductPlan& plan, Layout layout, Product p, int dtype, hipStream_t stream) {
    p.splits = plan.splits;
    p.symmetric = p.symmetric && !dtype && plan.kernel >= kSymmetricF32;
    if (plan.kernel < 0) return hipErrorNotSupported;
    if (plan.kernel == 0) return p.splits > 1 ? hipErrorNotSupported : launch_product_small(layout, p, dtype, stream);
    return dtype ? launch_product_bf16(layout, p, plan.kernel, stream) : launch_product_f32(layout, p, plan.kernel, stream);
}

hipError_t launch_product(Layout layout, const Product& p, int dtype, hipStream_t stream) {
    return launch_product(plan_product(layout, dtype, p.M, p.N, p.K, p.batch, 1, p.symmetric != 0), layout, p, dtype, stream);
}

}  // namespace mec
