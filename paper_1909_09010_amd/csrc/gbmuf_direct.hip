// gbmuf_direct.hip -- products in f32 arithmetic straight from where the matrices lie, in tiles: no pass over the operands goes before
// them, so they are what small and ordinary sizes take.
#include "gbmuf_tile.h"

namespace gbmuf {
namespace {

constexpr int kDepth = 32;       // values of k per step (64 by tiles of 64 x 64 gain nothing, and cost the gradients half their waves)
constexpr int kThreads = 256;

template <int T>
__device__ __forceinline__ v4f read_left(const void *p, int64_t i, int left)
{
    if (left >= 4) return read4<T>(p, i);
    v4f v = {0.0f, 0.0f, 0.0f, 0.0f};
    if (left > 0) v[0] = load_one(p, i, T);
    if (left > 1) v[1] = load_one(p, i + 1, T);
    if (left > 2) v[2] = load_one(p, i + 2, T);
    return v;
}

// One step's share of an operand: R rows of the result by kDepth values of k.  ALONG_K: k lies side by side in memory, LDS holds [row][k] with the 16-byte
// chunk c of row r at place c ^ ((r / 2) & 7), 16 rows in all banks; else rows do, and LDS holds [k][row].  Whatever lies beyond the matrix is zero.
template <int T, bool ALONG_K, int R, bool SLOPE = false>
struct Stage {
    static constexpr int kChunks = R * kDepth / 4 / kThreads;
    static constexpr int kPitch = ALONG_K ? kDepth : R + 8;        // + 8: the two halves of a wave read k 4 apart, in other banks
    static constexpr int kFloats = ALONG_K ? R * kDepth : kDepth * kPitch;
    v4f v[kChunks], z[kChunks];

    static __device__ __forceinline__ int major(int i)
    {
        constexpr int per = (ALONG_K ? kDepth : R) / 4;
        return (i * kThreads + static_cast<int>(threadIdx.x)) / per;
    }
    static __device__ __forceinline__ int minor(int i)
    {
        constexpr int per = (ALONG_K ? kDepth : R) / 4;
        return (i * kThreads + static_cast<int>(threadIdx.x)) % per * 4;
    }

    __device__ __forceinline__ void load(const Source &s, int64_t g, int row0, int k0, int rows, int K)
    {
        const int64_t first = static_cast<int64_t>(ALONG_K ? row0 : k0), side = ALONG_K ? k0 : row0;
        if (row0 + R <= rows && k0 + kDepth <= K) {            // no guard between the loads: they are all in flight
#pragma unroll
            for (int i = 0; i < kChunks; ++i) v[i] = read4<T>(s.p, g * s.batch + (first + major(i)) * s.ld + side + minor(i));
            if (SLOPE && s.act)
#pragma unroll
                for (int i = 0; i < kChunks; ++i) z[i] = read4<T>(s.pre, g * s.p_batch + (first + major(i)) * s.ldp + side + minor(i));
            return;
        }
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            const int left = first + major(i) < (ALONG_K ? rows : K) ? static_cast<int>((ALONG_K ? K : rows) - side) - minor(i) : 0;
            v[i] = read_left<T>(s.p, g * s.batch + (first + major(i)) * s.ld + side + minor(i), left);
            if (SLOPE && s.act) z[i] = read_left<T>(s.pre, g * s.p_batch + (first + major(i)) * s.ldp + side + minor(i), left);
        }
    }

    template <int ACT>
    __device__ __forceinline__ void times_slope()
    {
#pragma unroll
        for (int i = 0; i < kChunks; ++i)
#pragma unroll
            for (int c = 0; c < 4; ++c) v[i][c] *= slope(z[i][c], ACT);
    }

    // applies the slope; what was beyond the matrix stays zero
    __device__ __forceinline__ void shape(const Source &s)
    {
        if (!SLOPE) return;
        switch (s.act) {
            case GBMUF_ACT_RELU: return times_slope<GBMUF_ACT_RELU>();
            case GBMUF_ACT_GELU: return times_slope<GBMUF_ACT_GELU>();
            case GBMUF_ACT_SILU: return times_slope<GBMUF_ACT_SILU>();
            case GBMUF_ACT_SIGMOID: return times_slope<GBMUF_ACT_SIGMOID>();
            case GBMUF_ACT_TANH: return times_slope<GBMUF_ACT_TANH>();
            default: return;
        }
    }

    __device__ __forceinline__ void put(float *lds) const
    {
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            float *to = ALONG_K ? lds + major(i) * kPitch + (((minor(i) >> 2) ^ ((major(i) >> 1) & 7)) << 2) : lds + major(i) * kPitch + minor(i);
            *reinterpret_cast<v4f *>(to) = v[i];
        }
    }

    // the values of row `row` at k = 4 (2 t + half) + 0 .. 3
    static __device__ __forceinline__ v4f get(const float *lds, int row, int chunk)
    {
        if constexpr (ALONG_K) return *reinterpret_cast<const v4f *>(lds + row * kPitch + ((chunk ^ ((row >> 1) & 7)) << 2));
        const float *p = lds + chunk * 4 * kPitch + row;
        return v4f{p[0], p[kPitch], p[2 * kPitch], p[3 * kPitch]};
    }
};

template <int T, bool A_ALONG_K, bool B_ALONG_K, int TILE>
constexpr size_t direct_lds()
{
    constexpr size_t stages = (Stage<T, A_ALONG_K, TILE>::kFloats + Stage<T, B_ALONG_K, TILE>::kFloats) * sizeof(float);
    constexpr size_t out = leave_bytes<TILE, TILE, 2, 2>();
    return stages > out ? stages : out;
}

// One tile of TILE x TILE by 2 x 2 waves.
template <int T, bool A_ALONG_K, bool B_ALONG_K, int TILE, bool SLOPE>
__device__ __forceinline__ void direct_tile(const DirectArgs &a, int id, float *lds)
{
    constexpr int F = TILE / 64;
    using A = Stage<T, A_ALONG_K, TILE, SLOPE>;
    using B = Stage<T, B_ALONG_K, TILE>;
    const Share share = share_of<TILE, TILE>(a.t, id, (a.K + kDepth - 1) / kDepth);
    const int64_t g = share.at.g;
    const int tn = share.at.tn, m0 = share.at.tm * TILE, n0 = tn * TILE, first = share.first, last = share.last;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = (wave & 1) * (TILE / 2), wn = (wave >> 1) * (TILE / 2);
    float *la = lds, *lb = lds + A::kFloats;
    v16f acc[F][F];
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
        for (int j = 0; j < F; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
    v4f sums = {0.0f, 0.0f, 0.0f, 0.0f};
    A x;
    B w;
    if (first < last) {
        x.load(a.a, g, m0, first * kDepth, a.t.M, a.K);
        w.load(a.b, g, n0, first * kDepth, a.t.N, a.K);
    }
    for (int s = first; s < last; ++s) {
        x.shape(a.a);
        x.put(la);
        w.put(lb);
        if (A_ALONG_K && a.copy && tn == 0)
#pragma unroll
            for (int i = 0; i < A::kChunks; ++i) {
                const int m = m0 + A::major(i), k = s * kDepth + A::minor(i);
                if (m >= a.t.M) continue;
                const int64_t at = g * a.copy_batch + m * a.copy_ld + k;
                if (k + 4 <= a.K) write4<T>(a.copy, at, x.v[i]);
                else
                    for (int c = 0; c < 3; ++c)
                        if (k + c < a.K) store_one(a.copy, at + c, T, x.v[i][c]);
            }
        if (!A_ALONG_K && a.sums)
#pragma unroll
            for (int i = 0; i < A::kChunks; ++i) sums += x.v[i];      // a thread's rows are the same in every chunk
        __syncthreads();
        if (s + 1 < last) {
            x.load(a.a, g, m0, (s + 1) * kDepth, a.t.M, a.K);
            w.load(a.b, g, n0, (s + 1) * kDepth, a.t.N, a.K);
        }
#pragma unroll
        for (int t = 0; t < kDepth / 8; ++t) {
            v4f p[F], q[F];
#pragma unroll
            for (int i = 0; i < F; ++i) p[i] = A::get(la, wm + i * 32 + (lane & 31), 2 * t + (lane >> 5));
#pragma unroll
            for (int j = 0; j < F; ++j) q[j] = B::get(lb, wn + j * 32 + (lane & 31), 2 * t + (lane >> 5));
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int i = 0; i < F; ++i)
#pragma unroll
                    for (int j = 0; j < F; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(q[j][c], p[i][c], acc[i][j], 0, 0, 0);
        }
        __syncthreads();
    }
    if (!A_ALONG_K && a.sums && tn == 0) {
        constexpr int per4 = TILE / 4, groups = kThreads / per4;     // threads t, t + per4 .. hold the same rows
        reinterpret_cast<v4f *>(lds)[threadIdx.x] = sums;
        __syncthreads();
        if (threadIdx.x < TILE) {
            float v = 0.0f;
#pragma unroll
            for (int i = 0; i < groups; ++i) v += lds[i * TILE + threadIdx.x];
            const int m = m0 + static_cast<int>(threadIdx.x);
            if (m < a.t.M) {
                const int64_t at = g * a.sums_batch + m;
                if (a.accumulate) v += load_one(a.sums, at, a.sums_type);
                store_one(a.sums, at, a.sums_type, v);
            }
        }
        __syncthreads();
    }
    leave<TILE, TILE, 2, 2, false>(acc, lds, a, share);
}

template <int T, int TILE>
__global__ __launch_bounds__(kThreads) void direct_forward_kernel(DirectArgs a)
{
    __shared__ __align__(16) float lds[direct_lds<T, true, true, TILE>() / 4];
    direct_tile<T, true, true, TILE, false>(a, static_cast<int>(blockIdx.x), lds);
}

// dx = dz w (dz lies along the sum, w across it) and dw = dz' x (both across), in one launch: the first workgroups are dx's.
template <int T, int TILE>
__global__ __launch_bounds__(kThreads) void direct_backward_kernel(DirectArgs dx, DirectArgs dw)
{
    __shared__ __align__(16) float lds[direct_lds<T, false, false, TILE>() / 4];
    static_assert(direct_lds<T, false, false, TILE>() >= direct_lds<T, true, false, TILE>(), "one piece of LDS for both");
    const int n = dx.t.blocks(), id = static_cast<int>(blockIdx.x);
    if (id < n) direct_tile<T, true, false, TILE, true>(dx, id, lds);
    else direct_tile<T, false, false, TILE, true>(dw, id - n, lds);
}

}  // namespace

int launch_direct_forward(const DirectArgs &a, int32_t type, int tile, hipStream_t stream)
{
    const int32_t blocks = a.t.blocks();
    if (blocks <= 0) return GBMUF_OK;
    using Fn = void (*)(DirectArgs);
    static constexpr Fn fns[3][2] = {{direct_forward_kernel<kF32, 64>, direct_forward_kernel<kF32, 128>},
                                     {direct_forward_kernel<kBf16, 64>, direct_forward_kernel<kBf16, 128>},
                                     {direct_forward_kernel<kF16, 64>, direct_forward_kernel<kF16, 128>}};
    DirectArgs args = a;
    void *argv[] = {&args};
    const hipError_t err = hipLaunchKernel(reinterpret_cast<const void *>(fns[type][tile == 128]), dim3(static_cast<unsigned>(blocks)), dim3(kThreads),
                                           argv, 0, stream);
    return err == hipSuccess ? GBMUF_OK : hip_failed("hipLaunchKernel(direct product)", err, GBMUF_EDEVICE);
}

int launch_direct_backward(const DirectArgs &dx, const DirectArgs &dw, int32_t type, int tile, hipStream_t stream)
{
    const int32_t blocks = dx.t.blocks() + dw.t.blocks();
    if (blocks <= 0) return GBMUF_OK;
    using Fn = void (*)(DirectArgs, DirectArgs);
    static constexpr Fn fns[3][2] = {{direct_backward_kernel<kF32, 64>, direct_backward_kernel<kF32, 128>},
                                     {direct_backward_kernel<kBf16, 64>, direct_backward_kernel<kBf16, 128>},
                                     {direct_backward_kernel<kF16, 64>, direct_backward_kernel<kF16, 128>}};
    DirectArgs x = dx, w = dw;
    void *argv[] = {&x, &w};
    const hipError_t err = hipLaunchKernel(reinterpret_cast<const void *>(fns[type][tile == 128]), dim3(static_cast<unsigned>(blocks)), dim3(kThreads),
                                           argv, 0, stream);
    return err == hipSuccess ? GBMUF_OK : hip_failed("hipLaunchKernel(direct gradients)", err, GBMUF_EDEVICE);
}

}  // namespace gbmuf
