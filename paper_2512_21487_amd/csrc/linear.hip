// Which kernel a matrix product with an epilogue runs on, and its launch.
#include <cmath>

#include "linear_kernels.h"

namespace moe_ep {

namespace {

// What a tile costs, us: `fixed` and, per K step, `alone` where most compute units have none, `full` where all have (power and
// L2 are shared).  Fitted to launches of 256 x 256 to 16384 x 5120 results, K from 256 to 8192.
struct Tiling { int rows, cols, slots, per_cu; double alone, full, fixed; };
constexpr Tiling kTilings[] = {
    {256, 256, 2, 1, 1.02, 1.40, 12.0}, {256, 192, 2, 1, 0.84, 1.13, 9.5}, {192, 256, 2, 1, 0.85, 1.13, 9.0},
    {128, 128, 4, 1, 0.33, 0.44, 5.0}, {64, 64, 4, 2, 0.15, 0.37, 1.2}};

// a launch lasts as many rounds as its busiest compute unit has tiles
double tiled_us(const Tiling& t, const LinearArgs& a, int n_cu)
{
    const double tiles = (double)((a.R + t.rows - 1) / t.rows) * ((a.N + t.cols - 1) / t.cols), slots = (double)n_cu * t.per_cu;
    const double rounds = std::ceil(tiles / slots), fill = tiles / (rounds * slots);
    return rounds * ((a.K + 63) / 64 * (t.alone + (t.full - t.alone) * fill) + t.fixed);
}

// the tiling of kTilings that costs least
int cheapest_tiling(const LinearArgs& a, int n_cu)
{
    int best = 0;
    double us = 0.0;
    for (int i = 0; i < (int)(sizeof kTilings / sizeof *kTilings); ++i) {
        const double t = tiled_us(kTilings[i], a, n_cu);
        if (kTilings[i].slots <= (a.K + 63) / 64 && (us == 0.0 || t < us)) { us = t; best = i; }
    }
    return best;
}

// The largest of the split tiles that still gives enough compute units work: half of them, three quarters where every tile also takes fp32
// weights apart.  64 x 32 / 64 x 16 / 32 x 16 / 16 x 16 tiles, us: 64 x 5120 x 1536 10 / 12 / 15 / 13; 33, 64 x 2048 x 1408 7.2 / 6.2 / 5.2 / 5.4,
// 7.3 / 6.4 / 5.2 / 5.5; 64 x 1536 x 5120 22 / 18 / 13 / 14; 24 x 1536 x 5120 18 / 15 / 12 / 9; 17, 32 x 5120 x 1536 8.9 / 11 / 10 / 8.9, 9.2 / 11 / 11 / 9.7;
// fp32 weights, 4096 x 128 x 4096 27 / 32 / 43 / 62, 1024 x 256 x 4096 23 / 16 / 23 / 33, 256 x 160 x 5120 25 / 17 / 12 / 10.  (Of 33 to 64 rows the
// rule takes 64 x 16 where 32 x 16 is up to a fifth faster: half of the compute units is too few there.)  64 x 32 with four wavefronts instead of
// eight, many tiles: 4096 x 256 x 2048 25 / 28, 8192 x 256 x 4096 87 / 94; 4096 x 128 x 4096, few, 31 / 27.
int split_kernel(const LinearArgs& a, int n_cu)
{
    const auto tiles = [&](int mb, int nb) { return (double)((a.R + mb * 16 - 1) / (mb * 16)) * ((a.N + nb * 16 - 1) / (nb * 16)); };
    const double enough = a.w32 ? 0.75 * n_cu : 0.5 * n_cu;
    if (a.R > 32 && tiles(4, 2) >= 2 * n_cu) return kLinearSplit64x32by4;
    if (a.R > 32 && tiles(4, 2) >= enough) return kLinearSplit64x32;
    if (a.R > 32 && tiles(4, 1) >= enough) return kLinearSplit64x16;
    if (a.R > 16 && tiles(2, 1) >= enough) return kLinearSplit32x16;
    return kLinearSplit16x16;
}

}  // namespace

int linear_kernel(const LinearArgs& a, int n_cu)
{
    const auto tiles = [&](int edge) { return (double)((a.R + edge - 1) / edge) * ((a.N + edge - 1) / edge); };
    // Few blocks of 16 x 16 for a matrix instruction, and little to multiply.  Rows / split, us: 1, 16, 33 x 160 x 5120, fp32 weights, 3.1 / 8.6,
    // 5.1 / 8.6, 6.5 / 8.7; 64, 256 x 128 x 4096 6.6 / 7.5, 17 / 9.1; bf16 weights, 1, 8 x 2048 x 1408 3.6 / 3.8, 7.6 / 3.9.
    const double products = (double)a.R * a.N * a.K;
    if ((products <= 40e6 && tiles(16) < n_cu / 2) || products <= 3e6) return a.R <= 8 ? kLinearRows1x1 : a.R <= 16 ? kLinearRows4x1 : kLinearRows4x2;
    // The tiled kernels move 16 bytes at a time, and are a K step ahead at least.  Of few tiles, each a compute unit's, a long K is better shared:
    // tiled / split, us: 64 x 1536 x 5120 17 / 9.7; 64 x 5120 x 2048 9.8 / 9.5, 256 x 2048 x 2048 9.6 / 12.
    const bool by_16 = !a.w32 && a.K > 64 && a.K % 8 == 0 && a.ldx % 8 == 0 && a.ldw % 8 == 0 && !((reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.w)) & 15);
    if (by_16 && a.R > 64 && tiles(64) >= n_cu / 4) return kLinearTiled + cheapest_tiling(a, n_cu);
    // Operands that are not on 16 bytes: 64 x 64 tiles / 128 x 64 tiles / split, us: 1531 x 1409 x 2049 39 / 43 / 49, 3112 x 839 x 182 8.9 / 11 / 12,
    // 8192 x 2048 x 2049 197 / 149 / 260, 16384 x 5120 x 1001 486 / 426 / 755; of few tiles 300 x 1409 x 2049 27 / 37 / 14.
    if (!a.w32 && !by_16 && a.K > 64) {
        if (2 * tiles(128) >= 4 * n_cu) return kLinearStaged128x64;
        if (tiles(64) >= 1.5 * n_cu) return kLinearStaged64x64;
    }
    return split_kernel(a, n_cu);
}

int linear_tile_rows(int kernel)
{
    if (kernel < kLinearTiled) return 0;
    if (kernel < kLinearStaged128x64) return kTilings[kernel - kLinearTiled].rows;
    switch (kernel) {
    case kLinearStaged128x64: return 128;
    case kLinearSplit32x16: return 32;
    case kLinearSplit16x16: return 16;
    default: return 64;
    }
}

int adapter_kernel(const LinearArgs& a, int n_cu)
{
    const int kernel = linear_kernel(a, n_cu);
    if (kernel < kLinearTiled) return kLinearSplit16x16;
    const double tiles = (double)((a.R + 191) / 192) * ((a.N + 255) / 256);
    return a.K < 256 && kernel < kLinearTiled + 3 && 2.5 * tiles < n_cu ? kLinearSplit64x32by4 : kernel;
}

hipError_t launch_linear(const LinearArgs& a, int n_cu, hipStream_t s)
{
    if (a.R <= 0) return hipSuccess;
    if (a.N < 1 || a.K < 1) return hipErrorInvalidValue;
    switch (const int kernel = linear_kernel(a, n_cu)) {
    case kLinearRows1x1: return launch_rows<1, 1>(a, s);
    case kLinearRows4x1: return launch_rows<4, 1>(a, s);
    case kLinearRows4x2: return launch_rows<4, 2>(a, s);
    default: return launch_chosen(kernel, a, NoAdapters{}, n_cu, s);
    }
}

}  // namespace moe_ep
