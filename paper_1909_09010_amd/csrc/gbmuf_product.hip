// gbmuf_product.hip -- matrix products on gfx950's matrix cores for the local half: out = a b' over 16-bit numbers.
#include "gbmuf_stage.h"

namespace gbmuf {
namespace {

// One tile of TM x TN, WM x WN waves.  Two stages in LDS: while one is multiplied the next step arrives in the other.  A wave
// loads a turn's operands while it multiplies the turn before, and the waves meet before the last turn of a step, whose operands they then
// all hold: the next step's first turn is loaded, and the step after it sent for, under that last turn.
template <int T, bool SPLIT, int TM, int TN, int WM, int WN, int ACROSS>
__global__ __launch_bounds__(64 * WM * WN) void product_kernel(ProductArgs a)
{
    constexpr int THREADS = 64 * WM * WN, FM = TM / WM / 32, FN = TN / WN / 32, kTurns = SPLIT ? 2 : 4;
    __shared__ __align__(1024) uint16_t lds[2][(TM + TN) * kStep];
    static_assert(leave_bytes<TM, TN, WM, WN>() <= sizeof(lds), "the result leaves through the stages");

    const Share share = share_of<TM, TN>(a.t, static_cast<int>(blockIdx.x), (a.K + kStep - 1) / kStep);
    const int64_t g = share.at.g;
    const int m0 = share.at.tm * TM, n0 = share.at.tn * TN, first = share.first, last = share.last;
    const int full = min(last, a.K / kStep);               // steps [first, full) are whole
    std::conditional_t<(ACROSS & 1) != 0, StageAcross<TM, THREADS>, Stage<TM, THREADS>> sa;
    std::conditional_t<(ACROSS & 2) != 0, StageAcross<TN, THREADS>, Stage<TN, THREADS>> sb;
    sa.init(a.a + g * a.a_batch, a.lda, m0, a.t.M);
    sb.init(a.b + g * a.b_batch, a.ldb, n0, a.t.N);

    const int wave = threadIdx.x >> 6, wm = (wave % WM) * (TM / WM), wn = (wave / WM) * (TN / WN);
    v16f acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

    constexpr int kReads = (SPLIT ? 2 : 1) * ((ACROSS & 1 ? 0 : FM) + (ACROSS & 2 ? 0 : FN)), kMfmas = (SPLIT ? 3 : 1) * FM * FN;
    Turn<T, SPLIT, TM, TN, FM, FN, ACROSS> turn[2];
    if (first < full) {
        sa.load(lds[0], first * kStep);
        sb.load(lds[0] + TM * kStep, first * kStep);
        meet<true>();
        if (first + 1 < full) {
            sa.load(lds[1], (first + 1) * kStep);
            sb.load(lds[1] + TM * kStep, (first + 1) * kStep);
        }
        turn[0].template load<0>(lds[0], wm, wn);
        for (int s = first; s < full; ++s) {
            uint16_t *now = lds[(s - first) & 1], *next = lds[(s - first + 1) & 1];
            repeat<kTurns - 1>([&](auto t) {
                turn[(t + 1) & 1].template load<t + 1>(now, wm, wn);
                turn[t & 1].multiply(acc);
                interleave<kReads, kMfmas>();
                __builtin_amdgcn_sched_barrier(0);
            });
            meet<true>();
            if (s + 2 < full) {
                sa.load(now, (s + 2) * kStep);
                sb.load(now + TM * kStep, (s + 2) * kStep);
            }
            turn[0].template load<0>(next, wm, wn);         // of the last step: not used
            turn[(kTurns - 1) & 1].multiply(acc);
            interleave<kReads, kMfmas>();
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    if (full < last) {                                     // at most one step; nothing is in flight, the waves may be in the last turn
        __syncthreads();
        sa.load_rest(lds[0], full * kStep, a.K);
        sb.load_rest(lds[0] + TM * kStep, full * kStep, a.K);
        __syncthreads();
        repeat<kTurns>([&](auto t) {
            turn[0].template load<t>(lds[0], wm, wn);
            turn[0].multiply(acc);
        });
    }
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
