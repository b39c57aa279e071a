// gbmuf_product.hip -- matrix products on gfx950's matrix cores for the local half: out = a b' over 16-bit numbers.
#include "gbmuf_stage.h"

namespace gbmuf {
namespace {

// One tile of TM x TN by WM x WN waves.
template <int T, bool SPLIT, int TM, int TN, int WM, int WN, int ACROSS>
__global__ __launch_bounds__(64 * WM * WN) void product_kernel(ProductArgs a)
{
    __shared__ __align__(1024) uint16_t lds[2][(TM + TN) * kStep];
    static_assert(leave_bytes<TM, TN, WM, WN>() <= sizeof(lds), "the result leaves through the stages");
    const Share share = share_of<TM, TN>(a.t, static_cast<int>(blockIdx.x), (a.K + kStep - 1) / kStep);
    v16f acc[TM / WM / 32][TN / WN / 32];
    sum_tile<T, SPLIT, TM, TN, WM, WN, ACROSS>(acc, lds, a, share);
    __syncthreads();
    leave<TM, TN, WM, WN, SPLIT>(acc, &lds[0][0], a, share);
}

// Joins the parts of split tiles, in their order: 32 rows of a tile a workgroup, 8 columns a thread.
template <int TILE>
__global__ __launch_bounds__(256) void join_kernel(JoinArgs a)
{
    constexpr int kChunks = TILE / 32, kLanes = TILE / 8;
    const int rest = a.t.rest(), tile = static_cast<int>(blockIdx.x) / kChunks, chunk = static_cast<int>(blockIdx.x) % kChunks;
    const TileAt at = tile_at(a.t, a.t.whole + tile);
    const int column = static_cast<int>(threadIdx.x) % kLanes * 8, n = at.tn * TILE + column;
    if (n >= a.t.N) return;
    for (int r = chunk * 32 + static_cast<int>(threadIdx.x) / kLanes; r < chunk * 32 + 32; r += 256 / kLanes) {
        const int m = at.tm * TILE + r;
        if (m >= a.t.M) return;
        const float *from = a.t.partial + static_cast<int64_t>(tile) * (TILE * TILE) + r * TILE + column;
        const int64_t next = static_cast<int64_t>(rest) * (TILE * TILE);
        Eight s = read8<kF32>(from, 0);
#pragma unroll 4
        for (int p = 1; p < a.t.splits; ++p) {
            const Eight v = read8<kF32>(from, p * next);
            s.v[0] += v.v[0];
            s.v[1] += v.v[1];
        }
        finish8(a.e, at.g, m, n, a.t.N - n, s);
    }
}

}  // namespace

int launch_product(const ProductArgs &a, int32_t type, int tile, hipStream_t stream)
{
    if (a.t.count() <= 0) return GBMUF_OK;
    ProductArgs args = a;
    void *argv[] = {&args};
    using Fn = void (*)(ProductArgs);
    static constexpr Fn split[2] = {product_kernel<kF16, true, 128, 128, 2, 2, 0>, product_kernel<kF16, true, 256, 256, 2, 4, 0>};
    static constexpr Fn plain[2][3][2] = {
        {{product_kernel<kBf16, false, 128, 128, 2, 2, 0>, product_kernel<kBf16, false, 256, 256, 2, 4, 0>},
         {product_kernel<kBf16, false, 128, 128, 2, 2, 2>, product_kernel<kBf16, false, 256, 256, 2, 4, 2>},
         {product_kernel<kBf16, false, 128, 128, 2, 2, 3>, product_kernel<kBf16, false, 256, 256, 2, 4, 3>}},
        {{product_kernel<kF16, false, 128, 128, 2, 2, 0>, product_kernel<kF16, false, 256, 256, 2, 4, 0>},
         {product_kernel<kF16, false, 128, 128, 2, 2, 2>, product_kernel<kF16, false, 256, 256, 2, 4, 2>},
         {product_kernel<kF16, false, 128, 128, 2, 2, 3>, product_kernel<kF16, false, 256, 256, 2, 4, 3>}}};
    const Fn fn = type == kF32 ? split[tile == 256] : plain[type == kF16][a.across == 0 ? 0 : a.across - 1][tile == 256];
    const hipError_t err = hipLaunchKernel(reinterpret_cast<const void *>(fn), dim3(static_cast<unsigned>(a.t.blocks())),
                                           dim3(tile == 256 ? 512 : 256), argv, 0, stream);
    return err == hipSuccess ? GBMUF_OK : hip_failed("hipLaunchKernel(product)", err, GBMUF_EDEVICE);
}

int launch_join(const JoinArgs &a, hipStream_t stream)
{
    if (a.t.splits <= 1 || a.t.rest() <= 0) return GBMUF_OK;
    JoinArgs args = a;
    void *argv[] = {&args};
    const auto fn = a.tile == 64 ? join_kernel<64> : a.tile == 128 ? join_kernel<128> : join_kernel<256>;
    const hipError_t err = hipLaunchKernel(reinterpret_cast<const void *>(fn), dim3(static_cast<unsigned>(a.t.rest() * (a.tile / 32))), dim3(256), argv, 0,
                                           stream);
    return err == hipSuccess ? GBMUF_OK : hip_failed("hipLaunchKernel(join)", err, GBMUF_EDEVICE);
}

}  // namespace gbmuf
