// Adapters of up to kGathered rows, a decode step of many requests: the product and x A_a^T in one launch, x A_a^T B_a^T and the epilogue in another.  The rows of such a
// batch have their adapters in no order, so that a tile of the product would meet most of them; groups of rows of one adapter meet one.
#include "linear_kernels.h"

namespace moe_ep {

namespace {

// A wavefront has a group of up to 16 rows and NB * 16 columns: x W^T of them, as the product left it, and the product of their x A^T (as kParts bf16 numbers) with B, straight
// from memory in the order that the matrix instruction wants: 64 bytes of a row, 16 rows at a time.
template <int NB>
__global__ __launch_bounds__(256) void adapters_up_kernel(LinearArgs a, AdapterArgs x, const float* wide, const int32_t* table, int slices)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = blockIdx.x / slices;
    const int n0 = ((int)(blockIdx.x % slices) * 4 + wave) * (NB * 16);
    const int32_t* const entry = table + group * kGroupEntry;
    const int adapter = entry[0], row = lane & 15, kh = lane >> 4, m = entry[1 + row];
    if (adapter < -1 || n0 >= a.N) return;
    const Epilogue<NB> e(a, n0, kh);
    typename Epilogue<NB>::Residual res;
    const bool there = m >= 0;
    if (a.residual && there) e.fetch(m, res);
    f32x4_t v[NB];
    const float* const from = wide + (size_t)(there ? m : 0) * a.N + n0 + kh * 4;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        v[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        if (e.group(b)) v[b] = *reinterpret_cast<const f32x4_any4*>(from + b * 16);
        else
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (n0 + kh * 4 + b * 16 + i < a.N) v[b][i] = from[b * 16 + i];
    }
    if (adapter >= 0) {
        const uint16_t* const low = x.low + (size_t)(there ? m : 0) * adapter_pitch(x.width);
        const uint16_t* const up = x.up + (size_t)adapter * a.N * x.rank;
#pragma unroll 4
        for (int k = kh * 8; k - kh * 8 < x.rank; k += 32) {
            const bool in = k < x.rank;
            u32x4_t u[NB], l[kParts];
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                u[b] = u32x4_t{0, 0, 0, 0};
                if (in) u[b] = *reinterpret_cast<const u32x4_t*>(up + (size_t)min(n0 + b * 16 + row, a.N - 1) * x.rank + k);
            }
#pragma unroll
            for (int p = 0; p < kParts; ++p) {
                l[p] = u32x4_t{0, 0, 0, 0};
                if (in && there) l[p] = *reinterpret_cast<const u32x4_t*>(low + p * x.rank + k);
            }
#pragma unroll
            for (int p = kParts - 1; p >= 0; --p)
#pragma unroll
                for (int b = 0; b < NB; ++b)
                    v[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, u[b]), __builtin_bit_cast(bf16x8_t, l[p]), v[b], 0, 0, 0);
        }
    }
    e.store(m, there, v, res);
}

template <int NB>
hipError_t launch_up(const LinearArgs& a, const AdapterArgs& x, const float* wide, const int32_t* table, int groups, hipStream_t s)
{
    const long long slices = ((long long)a.N + NB * 64 - 1) / (NB * 64), grid = groups * slices;
    if (grid > 0x7fffffffll / 256) return hipErrorInvalidValue;
    hipLaunchKernelGGL((adapters_up_kernel<NB>), dim3((unsigned)grid), dim3(256), 0, s, a, x, wide, table, (int)slices);
    return hipGetLastError();
}

// the product that leaves x W^T in fp32
LinearArgs product_of(const LinearArgs& a, float* wide)
{
    LinearArgs product = a;
    product.out = wide;
    product.ldo = a.N;
    product.out32 = true;
    product.bias = nullptr;
    product.residual = nullptr;
    product.act = kActNone;
    return product;
}

// groups, shares, workgroups
void share_groups(GroupArgs& g, int R, int n, int rank, int n_cu)
{
    g.groups = adapter_groups(R, n);
    const int blocks = (rank + 15) / 16;
    // two workgroups for a compute unit, beside the product's own (512 x 4096 x 4096, 400 adapters of rank 32, one / two / four 92 / 92 / 111 us, of rank 128 166 / 165 / 167)
    g.shares = g.groups * blocks <= 2 * n_cu ? blocks : 2 * n_cu / g.groups > 1 ? 2 * n_cu / g.groups : 1;
    g.workgroups = (g.groups * g.shares + 7) / 8 * 8;
}

}  // namespace

// Of up to 32 rows the weights bound it, and what is on its way from memory: 32 columns a workgroup and two K steps ahead, eight wavefronts, so that compute units have two workgroups
// or more, x A^T beside the product among them.  The product's own kernel / this, rank 16, us: 1, 12 x 5120 x 5120 17.5 / 15.0, 18.0 / 15.4, 2 x 4096 x 4096 15.8 / 13.3,
// 17 x 4096 x 4096 18.2 / 14.8, 32 x 5120 x 5120 22 / 17; of few columns both are as fast, 1 x 160 x 5120 12.5 / 12.4.  Nor do workgroups of sixteen wavefronts, one a
// compute unit, go with many that make x A^T: 111 x 448 x 2240, rank 128 of 58, 32 / 23, 64 x 1536 x 2048, rank 64 of 64, 17 / 15; with few, 48 x 512 x 5120, rank 16 of 48, 14 / 14.
int grouped_plan(const LinearArgs& a, int n, int rank, int n_cu)
{
    GroupArgs g{};
    share_groups(g, a.R, n, rank, n_cu);
    const int kernel = adapter_kernel(product_of(a, nullptr), n_cu);
    const bool sixteen = kernel == kLinearSplit16x16 || kernel == kLinearSplit32x16;
    return a.R <= 16 ? kGroupedRows16 : a.R <= 32 || (sixteen && 2 * g.workgroups > n_cu) ? kGroupedRows32 : kernel;
}

hipError_t launch_linear_grouped(const LinearArgs& a, const AdapterArgs& x, float* wide, int32_t* table, int n_cu, hipStream_t s)
{
    if (a.R <= 0) return hipSuccess;
    if (a.R > kGathered || a.N < 1 || a.K < 1 || a.w32 || x.n < 1 || x.rank < 8 || x.rank > kRankMost || x.rank % 8) return hipErrorInvalidValue;
    const LinearArgs product = product_of(a, wide);
    GroupArgs g{};
    g.adapters = x;
    g.table = table;
    share_groups(g, a.R, x.n, x.rank, n_cu);
    const int kernel = grouped_plan(a, x.n, x.rank, n_cu);
    const hipError_t e = kernel == kGroupedRows16 ? launch_split<1, 2, 8, 2>(product, g, s) : kernel == kGroupedRows32 ? launch_split<2, 2, 8, 2>(product, g, s)
                                                                                          : launch_chosen(kernel, product, g, n_cu, s);
    return e == hipSuccess ? launch_up<2>(a, x, wide, table, g.groups, s) : e;
}

}  // namespace moe_ep
