// Low-rank adapters of many requests beside a shared projection: act(x W^T + bias + scale_a (x A_a^T) B_a^T) + residual, a = index[row], of more than kGathered rows.
// Two launches.  The first makes scale_a x A_a^T of every row with an adapter, and for every row tile of the second the list of its rows' adapters.  The
// second is the product's own kernel (linear_kernels.h), whose reduction goes on behind K with these products and B_a: the
// wide result is neither written twice nor read again.
#include "linear_kernels.h"

namespace moe_ep {

namespace {

// the list of a tile of up to 256 rows, by one wavefront
__device__ __forceinline__ void make_list(const LinearArgs& a, const AdapterArgs& x, long long tile, int lane)
{
    int32_t* const list = x.lists + tile * adapter_list(x.tile);
    const int masks = (x.tile + 31) / 32;
    int mine[4], count = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const long long row = tile * x.tile + i * 64 + lane;
        mine[i] = i * 64 + lane < x.tile && row < a.R ? adapter_of(x, (int)row) : -1;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        Distinct d(mine[i]);
        int adapter;
        unsigned long long who[4] = {0, 0, 0, 0};
        while (d.next(adapter, who[i])) {
#pragma unroll
            for (int j = i + 1; j < 4; ++j) {
                who[j] = __ballot(mine[j] == adapter);
                if (mine[j] == adapter) mine[j] = -1;
            }
            // lane 0 writes the number, lane 1 + m the rows 32 m ..
            uint32_t v = (uint32_t)adapter;
#pragma unroll
            for (int m = 0; m < 8; ++m)
                if (lane == 1 + m) v = (uint32_t)(who[m >> 1] >> (m & 1) * 32);
            if (lane <= masks) list[1 + count * (1 + masks) + lane] = (int32_t)v;
            ++count;
        }
    }
    if (lane == 0) list[0] = count;
}

__device__ __forceinline__ void store_zeros(const AdapterArgs& x, long long row)
{
    *reinterpret_cast<u32x4_t*>(x.low + row * adapter_pitch(x.width) + x.width) = u32x4_t{0, 0, 0, 0};
}

// Rows on 16 bytes, zeros behind the last element: a wavefront has a row, 4 KB of it on their way.  `number`: of the launch's copying wavefronts
__device__ __forceinline__ void align_rows(const AlignArgs& c, int number, int wavefronts, int lane)
{
    constexpr int STEP = 64 * 8, AHEAD = 4;
    for (int at = number; at < c.x.rows + c.w.rows; at += wavefronts) {
        const bool of_x = at < c.x.rows;
        const AlignArgs::Rows& r = of_x ? c.x : c.w;
        const size_t row = of_x ? at : at - c.x.rows;
        const uint16_t* const from = r.from + row * r.ld;
        uint16_t* const to = r.to + row * c.pitch;
        int k = lane * 8;
        for (; k + (AHEAD - 1) * STEP + 8 <= c.K; k += AHEAD * STEP) {
            u32x4_t v[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) v[i] = *reinterpret_cast<const u32x4_any2*>(from + k + i * STEP);
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) *reinterpret_cast<u32x4_t*>(to + k + i * STEP) = v[i];
        }
        for (; k < c.pitch; k += STEP) *reinterpret_cast<u32x4_t*>(to + k) = load_part<8>(from + k, c.K - k, c.K);
    }
}

// Many rows: a workgroup has MB * 16 of them and NB * 16 ranks, and of the rows' adapters each `groups`th.
template <int MB, int NB, int WAVES, int DEPTH>
__global__ __launch_bounds__(WAVES * 64) void adapters_down_tiles_kernel(LinearArgs a, AdapterArgs x, AlignArgs c, int list_tiles, int groups)
{
    extern __shared__ uint4 lds4[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long long list_groups = (list_tiles + WAVES - 1) / WAVES, b = workgroup() - list_groups;
    if (b < 0) {
        const long long tile = workgroup() * WAVES + wave;
        if (tile < list_tiles) make_list(a, x, tile, lane);
        return;
    }
    const int blocks = (x.rank + NB * 16 - 1) / (NB * 16);
    const int r0 = (int)(b % blocks) * (NB * 16), group = (int)(b / blocks % groups);
    const long long m0 = b / blocks / groups * (MB * 16);
    if (m0 >= a.R) {
        // the copies are behind: these have a chain of K steps, those fill what they leave
        const long long number = b - (((long long)a.R + MB * 16 - 1) / (MB * 16)) * blocks * groups;
        if (number < c.workgroups) align_rows(c, (int)number * WAVES + wave, c.workgroups * WAVES, lane);
        return;
    }
    const bool mine = lane < MB * 16 && m0 + lane < a.R;
    if (r0 == 0 && group == 0 && wave == 0 && mine) store_zeros(x, m0 + lane);
    Distinct tile(mine ? adapter_of(x, (int)(m0 + lane)) : -1);
    int adapter;
    unsigned long long who;
    for (int at = 0; tile.next(adapter, who); ++at) {
        if (at % groups != group) continue;
        down<MB, NB, WAVES, DEPTH>(a, x, lds4, lane, wave, adapter, r0, m0 + __builtin_ctzll(who), [&](int i) { return who >> i & 1 ? m0 + i : -1ll; });
    }
}

template <int MB, int NB, int WAVES, int DEPTH>
hipError_t launch_tiles(const LinearArgs& a, const AdapterArgs& x, const AlignArgs& c, int groups, hipStream_t s)
{
    constexpr int bytes = WAVES * SplitCfg<MB, NB, false>::BYTES;
    static_assert(bytes <= 160 * 1024, "LDS of a compute unit");
    static std::atomic<uint64_t> told{0};
    const hipError_t e = allow_lds(&adapters_down_tiles_kernel<MB, NB, WAVES, DEPTH>, bytes, told);
    if (e != hipSuccess) return e;
    const long long list_tiles = ((long long)a.R + x.tile - 1) / x.tile;
    const long long tiles = ((long long)a.R + MB * 16 - 1) / (MB * 16), blocks = (x.rank + NB * 16 - 1) / (NB * 16);
    const long long grid = c.workgroups + (list_tiles + WAVES - 1) / WAVES + tiles * blocks * groups;
    hipLaunchKernelGGL((adapters_down_tiles_kernel<MB, NB, WAVES, DEPTH>), grid_of(grid), dim3(WAVES * 64), bytes, s, a, x, c, (int)list_tiles, groups);
    return hipGetLastError();
}

// Tiles of few rows spread a few hundred of them over the compute units, tall ones read A less often.  16 rows x 16 ranks (a), two workgroups with 16 x 32 (b), two with 32 x 64 (c), 32 x
// 64 (d), 64 x 64 (e): the whole call of R x 1024 x 4096, 16 prompts, us: rank 16, R 600 31 / 30 / 40 / 47 / 75, 4096 52 / 57 / 56 / 62 / 76, 16384 159 / 192 / 174 / 166 / 164; rank 64, 1024 35 /
// 34 / 44 / 50 / 70, 2048 54 / 53 / 50 / 57 / 76, 4096 77 / 78 / 63 / 68 / 81, 8192 142 / 155 / 116 / 116 / 123, 16384 245 / 280 / 196 / 182 / 175; rank 128, 4096 108 / 119 / 84 / 79 / 93, 16384 366 /
// 442 / 271 / 221 / 232; of 16384 x 5120 x 5120, rank 64, (d) 742, (e) 729.  Tiles of 64 x 64 filled by direct loads into a ring took as long as (e), and longer of fewer rows.
hipError_t launch_adapters_down(const LinearArgs& a, const AdapterArgs& x, const AlignArgs& c, int n_cu, hipStream_t s)
{
    if (x.rank <= 16) return launch_tiles<1, 1, 16, 2>(a, x, c, 1, s);
    if (a.R < 2048) return launch_tiles<1, 2, 8, 4>(a, x, c, 2, s);
    if (a.R < 8192) return launch_tiles<2, 4, 8, 2>(a, x, c, 2, s);
    if (a.R < 64 * n_cu) return launch_tiles<2, 4, 8, 1>(a, x, c, 1, s);
    return launch_tiles<4, 4, 8, 1>(a, x, c, 1, s);
}

}  // namespace

int adapter_plan(const LinearArgs& a, int n_cu, bool* copies)
{
    const bool of_x = rows_off_16(a.K, a.ldx), of_w = rows_off_16(a.K, a.ldw);
    LinearArgs copied = a;
    if (of_x || of_w) copied.K = adapter_pitch_of(a.K);
    if (of_x) { copied.x = nullptr; copied.ldx = copied.K; }   // on 16 bytes, wherever
    if (of_w) { copied.w = nullptr; copied.ldw = copied.K; }
    const int kernel = adapter_kernel(copied, n_cu);
    // Only where the product is then one of tiles filled by direct loads.  Else the operands are taken as they are, by what is chosen for such.  (Of a short K the shared reduction
    // in tiles of 64 x 32, which copies would have led to, takes them as well, but is no better where there are many tiles.  That choice / that reduction, us: 1531 x 1409 x 131 19 / 26, 4100 x 700 x 65 21 / 27,
    // 7933 x 299 x 131 23 / 31, 2000 x 2048 x 192, rows 195 apart, 22 / 26; of few 800 x 1100 x 129 19 / 14, 5692 x 128 x 131 22 / 17, 2000 x 299 x 130 18 / 14.)
    *copies = (of_x || of_w) && kernel >= kLinearTiled && kernel < kLinearStaged128x64;
    return *copies || !(of_x || of_w) ? kernel : adapter_kernel(a, n_cu);
}

hipError_t launch_linear_adapters(const LinearArgs& a, AdapterArgs x, uint16_t* aligned_x, uint16_t* aligned_w, int n_cu, hipStream_t s)
{
    if (a.R <= 0) return hipSuccess;
    if (a.N < 1 || a.K < 1 || a.w32 || x.n < 1 || x.rank < 8 || x.rank > kRankMost || x.rank % 8) return hipErrorInvalidValue;
    if ((aligned_x != nullptr) != rows_off_16(a.K, a.ldx) || (aligned_w != nullptr) != rows_off_16(a.K, a.ldw)) return hipErrorInvalidValue;
    LinearArgs product = a;
    AlignArgs c{};
    bool copies;
    const int kernel = adapter_plan(a, n_cu, &copies);
    if (copies) {
        c.K = a.K;
        c.pitch = adapter_pitch_of(a.K);
        product.K = c.pitch;
        if (aligned_x) {
            c.x = {a.x, aligned_x, a.ldx, a.R};
            product.x = aligned_x;
            product.ldx = c.pitch;
        }
        if (aligned_w) {
            c.w = {static_cast<const uint16_t*>(a.w), aligned_w, a.ldw, a.N};
            product.w = aligned_w;
            product.ldw = c.pitch;
        }
        c.workgroups = (int)fmin(((double)c.x.rows + c.w.rows + 7) / 8, 4.0 * n_cu);   // a row for a wavefront, eight wavefronts or sixteen
    }
    x.tile = linear_tile_rows(kernel);
    const hipError_t e = launch_adapters_down(a, x, c, n_cu, s);
    return e == hipSuccess ? launch_chosen(kernel, product, x, n_cu, s) : e;
}

}  // namespace moe_ep
