// gbmuf_direct.hip -- products in f32 arithmetic straight from where the matrices lie, in tiles: no pass over the operands goes before
// them, so they are what small and ordinary sizes take.
#include "gbmuf_tile.h"

namespace gbmuf {
namespace {

constexpr int kDepth = 32;       // values of k per step (64 by tiles of 64 x 64 gain nothing, and cost the gradients half their waves)
constexpr int kThreads = 256;
constexpr int kTile = 64;        // (128 x 128: gradients of 8 x 128 x 650 x 650 f32 88 us where these take 44, and nowhere less than these)

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
// chunk c of row r at place c ^ ((r / 2) & 7), 16 rows in all banks; else rows do, and LDS holds [k][row].  What lies beyond the matrix along k is zero.
// Threads work in groups of 256, each on steps of its own.
__device__ __forceinline__ int thread_of() { return static_cast<int>(threadIdx.x) & (kThreads - 1); }

template <int T, bool ALONG_K, bool SLOPE = false>
struct Stage {
    static constexpr int kChunks = kTile * kDepth / 4 / kThreads;
    static constexpr int kPitch = ALONG_K ? kDepth : kTile + 8;        // + 8: the two halves of a wave read k 4 apart, in other banks
    static constexpr int kFloats = ALONG_K ? kTile * kDepth : kDepth * kPitch;
    v4f v[kChunks], z[kChunks];

    static __device__ __forceinline__ int major(int i)
    {
        constexpr int per = (ALONG_K ? kDepth : kTile) / 4;
        return (i * kThreads + thread_of()) / per;
    }
    static __device__ __forceinline__ int minor(int i)
    {
        constexpr int per = (ALONG_K ? kDepth : kTile) / 4;
        return (i * kThreads + thread_of()) % per * 4;
    }

    using Value = typename Num<T>::type;
    const Value *p[kChunks], *pre[kChunks];

    // Where the chunks of step 0 are read; those of rows beyond the matrix, whose results are not stored, at its end.
    __device__ __forceinline__ void init(const Source &s, int64_t g, int row0, int rows)
    {
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            const int64_t row = ALONG_K ? min(row0 + major(i), rows - 1) : major(i), side = ALONG_K ? minor(i) : min(row0 + minor(i), max(rows - 4, 0));
            p[i] = static_cast<const Value *>(s.p) + g * s.batch + row * s.ld + side;
            if (SLOPE && s.act) pre[i] = static_cast<const Value *>(s.pre) + g * s.p_batch + row * s.ldp + side;
        }
    }

    __device__ __forceinline__ void load(const Source &s, int64_t g, int row0, int k0, int rows, int K)
    {
        if (k0 + kDepth <= K && (ALONG_K || row0 + kTile <= rows || rows % 4 == 0)) {            // no guard between the loads: they are all in flight
            const int64_t k = k0;
#pragma unroll
            for (int i = 0; i < kChunks; ++i) v[i] = read4<T>(p[i], ALONG_K ? k : k * s.ld);
            if (SLOPE && s.act)
#pragma unroll
                for (int i = 0; i < kChunks; ++i) z[i] = read4<T>(pre[i], ALONG_K ? k : k * s.ldp);
            return;
        }
        const int64_t first = static_cast<int64_t>(ALONG_K ? row0 : k0), side = ALONG_K ? k0 : row0;
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

    // applies the slope
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

template <int T, bool A_ALONG_K, bool B_ALONG_K, int GROUPS>
constexpr size_t direct_lds()
{
    constexpr size_t stages = GROUPS * (Stage<T, A_ALONG_K>::kFloats + Stage<T, B_ALONG_K>::kFloats) * sizeof(float);
    constexpr size_t out = leave_bytes<kTile, kTile, 2, 2>(), parts = (GROUPS - 1) * kTile * kTile * sizeof(float), sums = GROUPS * kThreads * sizeof(v4f);
    constexpr size_t most = stages > out ? stages : out, more = parts > sums ? parts : sums;
    return most > more ? most : more;
}

// One tile of 64 x 64 by 2 x 2 waves, or by GROUPS times as many that take every GROUPS-th step each and are added up in the end: a step
// takes a microsecond or so however little it computes, and where there are few tiles nothing else hides that.
template <int T, bool A_ALONG_K, bool B_ALONG_K, bool SLOPE, int GROUPS>
__device__ __forceinline__ void direct_tile(const DirectArgs &a, int id, float *lds)
{
    using A = Stage<T, A_ALONG_K, SLOPE>;
    using B = Stage<T, B_ALONG_K>;
    const Share share = share_of<kTile, kTile>(a.t, id, (a.K + kDepth - 1) / kDepth);
    const int64_t g = share.at.g;
    const int tn = share.at.tn, m0 = share.at.tm * kTile, n0 = tn * kTile;
    const int group = GROUPS > 1 ? static_cast<int>(threadIdx.x) / kThreads : 0, first = share.first + group, last = share.last;
    const int turns = (share.last - share.first + GROUPS - 1) / GROUPS;            // of every group, though its last may be empty
    const int lane = threadIdx.x & 63, wave = thread_of() >> 6, wm = (wave & 1) * (kTile / 2), wn = (wave >> 1) * (kTile / 2);
    float *la = lds + group * (A::kFloats + B::kFloats), *lb = la + A::kFloats;
    v16f acc[1][1];
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[0][0][r] = 0.0f;
    v4f sums = {0.0f, 0.0f, 0.0f, 0.0f};
    A x;
    B w;
    x.init(a.a, g, m0, a.t.M);
    w.init(a.b, g, n0, a.t.N);
    if (first < last) {
        x.load(a.a, g, m0, first * kDepth, a.t.M, a.K);
        w.load(a.b, g, n0, first * kDepth, a.t.N, a.K);
    }
    for (int turn = 0; turn < turns; ++turn) {
        const int s = first + turn * GROUPS;
        if (s < last) {
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
        }
        __syncthreads();
        if (s + GROUPS < last) {
            x.load(a.a, g, m0, (s + GROUPS) * kDepth, a.t.M, a.K);
            w.load(a.b, g, n0, (s + GROUPS) * kDepth, a.t.N, a.K);
        }
        if (s < last)
#pragma unroll
            for (int t = 0; t < kDepth / 8; ++t) {
                const v4f p = A::get(la, wm + (lane & 31), 2 * t + (lane >> 5)), q = B::get(lb, wn + (lane & 31), 2 * t + (lane >> 5));
#pragma unroll
                for (int c = 0; c < 4; ++c) acc[0][0] = __builtin_amdgcn_mfma_f32_32x32x2f32(q[c], p[c], acc[0][0], 0, 0, 0);
            }
        __syncthreads();
    }
    if (!A_ALONG_K && a.sums && tn == 0) {
        constexpr int per4 = kTile / 4, same = GROUPS * kThreads / per4;      // threads t, t + per4 .. hold the same rows
        reinterpret_cast<v4f *>(lds)[threadIdx.x] = sums;
        __syncthreads();
        if (threadIdx.x < kTile) {
            float v = 0.0f;
#pragma unroll 8
            for (int i = 0; i < same; ++i) v += lds[i * kTile + threadIdx.x];
            const int m = m0 + static_cast<int>(threadIdx.x);
            if (m < a.t.M) {
                const int64_t at = g * a.sums_batch + m;
                if (a.accumulate) v += load_one(a.sums, at, a.sums_type);
                store_one(a.sums, at, a.sums_type, v);
            }
        }
        __syncthreads();
    }
    if constexpr (GROUPS > 1) {
        v4f *part = reinterpret_cast<v4f *>(lds);
        if (group > 0)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                part[((group - 1) * 4 + q) * kThreads + thread_of()] = v4f{acc[0][0][4 * q], acc[0][0][4 * q + 1], acc[0][0][4 * q + 2], acc[0][0][4 * q + 3]};
        __syncthreads();
        if (group == 0)
#pragma unroll
            for (int i = 0; i < (GROUPS - 1) * 4; ++i) {
                const v4f v = part[i * kThreads + thread_of()];
#pragma unroll
                for (int c = 0; c < 4; ++c) acc[0][0][i % 4 * 4 + c] += v[c];
            }
        __syncthreads();
        if (group > 0) return;
    }
    leave<kTile, kTile, 2, 2, false>(acc, lds, a, share);
}

template <int T, int GROUPS>
__global__ __launch_bounds__(GROUPS *kThreads) void direct_forward_kernel(DirectArgs a)
{
    __shared__ __align__(16) float lds[direct_lds<T, true, true, GROUPS>() / 4];
    direct_tile<T, true, true, false, GROUPS>(a, static_cast<int>(blockIdx.x), lds);
}

// dx = dz w (dz lies along the sum, w across it) and dw = dz' x (both across), in one launch: the first workgroups are dx's.
template <int T, int GROUPS>
__global__ __launch_bounds__(GROUPS *kThreads) void direct_backward_kernel(DirectArgs dx, DirectArgs dw)
{
    __shared__ __align__(16) float lds[direct_lds<T, false, false, GROUPS>() / 4];
    static_assert(direct_lds<T, false, false, GROUPS>() >= direct_lds<T, true, false, GROUPS>(), "one piece of LDS for both");
    const int n = dx.t.blocks(), id = static_cast<int>(blockIdx.x);
    if (id < n) direct_tile<T, true, false, true, GROUPS>(dx, id, lds);
    else direct_tile<T, false, false, true, GROUPS>(dw, id - n, lds);
}

// Up to one workgroup a CU: four groups of threads each.
bool grouped(int32_t blocks) { return blocks <= 256; }

}  // namespace

int launch_direct_forward(const DirectArgs &a, hipStream_t stream)
{
    const int32_t blocks = a.t.blocks();
    if (blocks <= 0) return GBMUF_OK;
    DirectArgs args = a;
    void *argv[] = {&args};
    const hipError_t err = hipLaunchKernel(reinterpret_cast<const void *>(grouped(blocks) ? direct_forward_kernel<kF32, 4> : direct_forward_kernel<kF32, 1>),
                                           dim3(static_cast<unsigned>(blocks)), dim3(grouped(blocks) ? 4 * kThreads : kThreads), argv, 0, stream);
    return err == hipSuccess ? GBMUF_OK : hip_failed("hipLaunchKernel(direct product)", err, GBMUF_EDEVICE);
}

int launch_direct_backward(const DirectArgs &dx, const DirectArgs &dw, int32_t type, hipStream_t stream)
{
    const int32_t blocks = dx.t.blocks() + dw.t.blocks();
    if (blocks <= 0) return GBMUF_OK;
    using Fn = void (*)(DirectArgs, DirectArgs);
    static constexpr Fn fns[3][2] = {{direct_backward_kernel<kF32, 1>, direct_backward_kernel<kF32, 4>},
                                     {direct_backward_kernel<kBf16, 1>, direct_backward_kernel<kBf16, 4>},
                                     {direct_backward_kernel<kF16, 1>, direct_backward_kernel<kF16, 4>}};
    DirectArgs x = dx, w = dw;
    void *argv[] = {&x, &w};
    const hipError_t err = hipLaunchKernel(reinterpret_cast<const void *>(fns[type][grouped(blocks) ? 1 : 0]), dim3(static_cast<unsigned>(blocks)),
                                           dim3(grouped(blocks) ? 4 * kThreads : kThreads), argv, 0, stream);
    return err == hipSuccess ? GBMUF_OK : hip_failed("hipLaunchKernel(direct gradients)", err, GBMUF_EDEVICE);
}

}  // namespace gbmuf
