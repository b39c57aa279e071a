// gbmuf_vocab.hip -- logits of many rows against a large vocabulary on gfx950's matrix cores, and what losses make of them: out = a b' is never
// written.
#include "gbmuf_loss.h"
#include "gbmuf_stage.h"

namespace gbmuf {
namespace {

// One tile of TM x TN logits by WM x WN waves.
template <int T, bool SPLIT, int TM, int TN, int WM, int WN, bool BACKWARD>
__global__ __launch_bounds__(64 * WM * WN) void vocab_kernel(ProductArgs a, LossArgs l)
{
    __shared__ __align__(1024) uint16_t lds[2][(TM + TN) * kStep];
    static_assert(loss_bytes<TM, TN, WM, WN>() <= sizeof(lds), "what follows takes the stages' place");
    const Share share = share_of<TM, TN>(a.t, static_cast<int>(blockIdx.x), (a.K + kStep - 1) / kStep);
    v16f acc[TM / WM / 32][TN / WN / 32];
    sum_tile<T, SPLIT, TM, TN, WM, WN, 0>(acc, lds, a, share);
    __syncthreads();
    leave_loss<TM, TN, WM, WN, SPLIT, BACKWARD>(acc, &lds[0][0], a.t, l, Scales{a.a_max, a.b_max, a.a_max_batch, a.b_max_batch}, share.at);
    if constexpr (!BACKWARD) {
        __syncthreads();
        store_parts<TM, TN, WM, WN, 64 * WM * WN>(&lds[0][0], a.t, l, share.at);
    }
}

}  // namespace

int launch_vocab(const ProductArgs &a, const LossArgs &l, int32_t type, int tile, bool backward, hipStream_t stream)
{
    if (a.t.count() <= 0) return GBMUF_OK;
    ProductArgs args = a;
    LossArgs loss = l;
    void *argv[] = {&args, &loss};
    using Fn = void (*)(ProductArgs, LossArgs);
    static constexpr Fn fns[3][2][2] = {
        {{vocab_kernel<kF16, true, 128, 128, 2, 2, false>, vocab_kernel<kF16, true, 256, 256, 2, 4, false>},
         {vocab_kernel<kF16, true, 128, 128, 2, 2, true>, vocab_kernel<kF16, true, 256, 256, 2, 4, true>}},
        {{vocab_kernel<kBf16, false, 128, 128, 2, 2, false>, vocab_kernel<kBf16, false, 256, 256, 2, 4, false>},
         {vocab_kernel<kBf16, false, 128, 128, 2, 2, true>, vocab_kernel<kBf16, false, 256, 256, 2, 4, true>}},
        {{vocab_kernel<kF16, false, 128, 128, 2, 2, false>, vocab_kernel<kF16, false, 256, 256, 2, 4, false>},
         {vocab_kernel<kF16, false, 128, 128, 2, 2, true>, vocab_kernel<kF16, false, 256, 256, 2, 4, true>}}};
    const hipError_t err = hipLaunchKernel(reinterpret_cast<const void *>(fns[type][backward ? 1 : 0][tile == 256 ? 1 : 0]),
                                           dim3(static_cast<unsigned>(a.t.blocks())), dim3(tile == 256 ? 512 : 256), argv, 0, stream);
    return err == hipSuccess ? GBMUF_OK : hip_failed("hipLaunchKernel(logits)", err, GBMUF_EDEVICE);
}

}  // namespace gbmuf
