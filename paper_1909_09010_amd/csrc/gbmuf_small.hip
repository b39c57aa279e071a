// gbmuf_small.hip -- gradients of losses of up to 64 rows and 64 features: the logits, their gradient and both products of a piece of the vocabulary in one workgroup.
#include "gbmuf_loss.h"

namespace gbmuf {
namespace {

constexpr int kWords = kSmallWords, kSlab = kSmallColumns, kThreads = 256, kPitch = kWords + 1;     // + 1: rows of dz are read down their columns too

// 64 rows of kSlab values as f32, the 16-byte chunk c of row r at place c ^ (r % 16): 16 rows lie in all banks at any chunk.
__device__ __forceinline__ int slab_at(int r, int k) { return r * kSlab + (((k >> 2) ^ (r & 15)) << 2) + (k & 3); }

// A thread's share of a slab of R rows on its way to LDS: 4 values of every 16th row.
template <int T, int R>
struct Slab {
    v4f v[R / 16];

    // rows behind the last are read as the last one, and what lies behind the columns as zeros
    __device__ __forceinline__ void load(const void *p, int64_t ld, int rows, int K)
    {
        const int k = static_cast<int>(threadIdx.x & 15) * 4;
#pragma unroll
        for (int i = 0; i < R / 16; ++i) {
            const int64_t at = min(i * 16 + static_cast<int>(threadIdx.x >> 4), rows - 1) * ld + k;
            v[i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
            if (k + 4 <= K) v[i] = read4<T>(p, at);
            else
#pragma unroll
                for (int c = 0; c < 3; ++c)
                    if (k + c < K) v[i][c] = load_one(p, at + c, T);
        }
    }

    // keep: which rows count; zeros in place of the others
    __device__ __forceinline__ void put(float *lds, const int32_t *keep) const
    {
#pragma unroll
        for (int i = 0; i < R / 16; ++i) {
            const int r = i * 16 + static_cast<int>(threadIdx.x >> 4);
            const bool is = !keep || keep[r] != kDead;
            *reinterpret_cast<v4f *>(lds + slab_at(r, static_cast<int>(threadIdx.x & 15) * 4)) =
                v4f{is ? v[i][0] : 0.0f, is ? v[i][1] : 0.0f, is ? v[i][2] : 0.0f, is ? v[i][3] : 0.0f};
        }
    }
};

__device__ __forceinline__ v16f zeros()
{
    v16f z;
#pragma unroll
    for (int r = 0; r < 16; ++r) z[r] = 0.0f;
    return z;
}

// A workgroup takes 64 words for all rows: z = x w' first, then dz in LDS, and from it dw = dz' x, which is whole, and its part of dx = dz w, which
// another launch adds up.  Bound by its chain of loads, barriers and 96 matrix instructions a wave (up to 32 rows 32 fewer, on two waves), which 3 workgroups
// of 49 KB on a CU, of up to 32 rows 4 of 33 KB, do beside each other.  us, with that launch / by the launches of larger sizes (dz, both products, joining),
// workers x rows x vocabulary x features: f16 4 x 40 x 1000 x 64 16.6 / 24, bf16 8 x 40 x 20000 x 64 72 / 76, 8 x 7 x 20000 x 64 46 / 67, 8 x 24 x 20000 x 50 57 / 79, 8 x 7 x
// 63165 x 37 134 / 202, f32 1 x 8 x 1000 x 64 15 / 20.6, 4 x 64 x 200 x 64 17 / 18, 1 x 64 x 10000 x 64 17 / 26, 1 x 16 x 100,000 x 64 39 / 76; in turns of 64 features, with x and w read
// twice, 128 of them gained nothing (f32 2 x 48 x 3000 x 128 23.6 / 25.4, f16 26.4 / 26.0), 256 lost (f32 1 x 64 x 10000 x 256 42 / 34).
template <int T, int ROWS>
__global__ __launch_bounds__(kThreads) void small_grads_kernel(SmallGrads a)
{
    __shared__ __align__(16) float xs[ROWS * kSlab], ws[kWords * kSlab];
    __shared__ float dz[ROWS * kPitch];
    __shared__ int32_t states[ROWS];
    __shared__ float weights[ROWS];
    const LossArgs &l = a.l;
    const Words &w = l.words;
    const int64_t g = blockIdx.y;
    const int n0 = static_cast<int>(blockIdx.x) * kWords, words = min(kWords, w.vocab - n0), M = w.rows, K = a.columns;
    const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = (wave & 1) * 32, wn = (wave >> 1) * 32;
    const int rows = (M + 7) / 8 * 8;                       // sums over rows end here; a wave of rows that are not there has nothing to do with them
    const typename Num<T>::type *x = static_cast<const typename Num<T>::type *>(a.x) + g * a.x_batch,
                                *wp = static_cast<const typename Num<T>::type *>(a.w) + g * a.w_batch + static_cast<int64_t>(n0) * a.ldw;
    Slab<T, ROWS> sx;
    Slab<T, kWords> sw;
    if (K > 0) {
        sx.load(x, a.ldx, M, K);
        sw.load(wp, a.ldw, words, K);
    }
    // what the logits' gradient takes, sent for with them: a lane has row lane % 32 and the words 8 (r / 4) + 4 (lane / 32) + r % 4
    const int m_lane = wm + (lane & 31), mc = min(m_lane, M - 1);
    const float lse = l.lse[g * l.lse_batch + mc * l.lse_ld], dloss = l.dloss[g * l.dloss_batch + mc * l.dloss_ld];
    v4f bias[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int n = wn + q * 8 + half * 4;
        bias[q] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        if (l.bias && n + 4 <= words) bias[q] = load_four(l.bias, g * l.bias_batch + n0 + n, T);
        else if (l.bias)
#pragma unroll
            for (int c = 0; c < 3; ++c)
                if (n + c < words) bias[q][c] = load_one(l.bias, g * l.bias_batch + n0 + n + c, T);
    }
    if (threadIdx.x < ROWS) {
        const int m = threadIdx.x;
        states[m] = m >= M ? kDead : w.logit ? given_state(w, g, m) : row_state(w, g, m);
    }
    __syncthreads();
    v16f acc = zeros();
    if (K > 0) {
        sx.put(xs, states);
        sw.put(ws, nullptr);
        __syncthreads();
        if (wm < M)
#pragma unroll
        for (int t = 0; t < kSlab / 8; ++t) {
            const v4f p = *reinterpret_cast<const v4f *>(xs + slab_at(wm + (lane & 31), (2 * t + half) * 4)),
                      q = *reinterpret_cast<const v4f *>(ws + slab_at(wn + (lane & 31), (2 * t + half) * 4));
#pragma unroll
            for (int c = 0; c < 4; ++c) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(q[c], p[c], acc, 0, 0, 0);
        }
    }
    if (wm < M) {
        const int state = states[m_lane];
        const float weight = state == kDead ? 0.0f : state == kLive ? dloss * l.tau : __builtin_nanf("");
        if (wn == 0 && half == 0) weights[m_lane] = weight;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int n = wn + (r >> 2) * 8 + half * 4 + (r & 3);
            const float p = weight * exp2_of(fmaf(acc[r] + bias[r >> 2][r & 3], l.inv_tau, -lse) * kLog2E);
            dz[m_lane * kPitch + n] = state == kDead || n >= words ? 0.0f : p;
        }
    }
    __syncthreads();
    // the words that a row is held to, in their order, by one lane
    if (threadIdx.x < ROWS && states[threadIdx.x] != kDead) {
        const int m = threadIdx.x;
        const float weight = weights[m];
        float *row = dz + m * kPitch;
        if (w.logit) each_given(w, g, m, l.inv_tau, [&](int64_t word, float share) {
            if (word >= n0 && word < n0 + words) row[word - n0] -= weight * share;
        });
        else if (w.target) {
            const int64_t word = w.target[g * w.batch + m * w.ld];
            if (word >= n0 && word < n0 + words) row[word - n0] -= weight;
        } else {
            const int32_t *list = w.id + (g * w.rows + m) * w.top;
            const float *share = w.share + (g * w.rows + m) * w.top;
            int place = 0, step = 1;
            while (2 * step <= w.top) step *= 2;
            for (; step; step >>= 1)
                if (place + step <= w.top && list[place + step - 1] < n0) place += step;
            for (; place < w.top && list[place] < n0 + words; ++place) row[list[place] - n0] -= weight * share[place];
        }
    }
    __syncthreads();
    if (a.dbias && threadIdx.x < static_cast<unsigned>(words)) {
        float v = 0.0f;
        for (int m0 = 0; m0 < rows; m0 += 8)
#pragma unroll
            for (int m = m0; m < m0 + 8; ++m) v += dz[m * kPitch + threadIdx.x];
        const int64_t at = g * a.dbias_batch + n0 + threadIdx.x;
        if (a.accumulate) v += load_one(a.dbias, at, a.grad_type);
        store_one(a.dbias, at, a.grad_type, v);
    }
    if (K == 0) return;
    // rows wm .. of either result and 32 features from wn on; a lane holds one feature of 16 rows, so that 32 lanes store along a row
    const int k = wn + (lane & 31);
    if (a.dw) {
        v16f out = zeros();
        for (int m0 = 0; m0 < rows; m0 += 8)
#pragma unroll
            for (int m = m0; m < m0 + 8; m += 2)
                out = __builtin_amdgcn_mfma_f32_32x32x2f32(dz[(m + half) * kPitch + wm + (lane & 31)], xs[slab_at(m + half, k)], out, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int n = wm + (r >> 2) * 8 + half * 4 + (r & 3);
            if (n >= words || k >= K) continue;
            const int64_t at = g * a.dw_batch + static_cast<int64_t>(n0 + n) * a.lddw + k;
            store_one(a.dw, at, a.grad_type, a.accumulate ? out[r] + load_one(a.dw, at, a.grad_type) : out[r]);
        }
    }
    if (a.parts && wm < M) {
        v16f out = zeros();
#pragma unroll 8
        for (int n = 0; n < kWords; n += 2)
            out = __builtin_amdgcn_mfma_f32_32x32x2f32(dz[(wm + (lane & 31)) * kPitch + n + half], ws[slab_at(n + half, k)], out, 0, 0, 0);
        float *to = a.parts + (static_cast<int64_t>(blockIdx.x) * gridDim.y + g) * M * K;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int m = wm + (r >> 2) * 8 + half * 4 + (r & 3);
            if (m < M && k < K) to[static_cast<int64_t>(m) * K + k] = out[r];
        }
    }
}

// dx from its parts: 64 values a workgroup, whose groups of 64 threads take every GROUPS-th part.
template <int GROUPS>
__global__ __launch_bounds__(64 * GROUPS) void small_join_kernel(SmallGrads a)
{
    __shared__ float sums[GROUPS][64];
    const int64_t each = static_cast<int64_t>(a.l.words.rows) * a.columns, at = static_cast<int64_t>(blockIdx.x) * 64 + (threadIdx.x & 63), g = blockIdx.y;
    const int group = threadIdx.x >> 6;
    float s = 0.0f;
    if (at < each)
#pragma unroll 8
        for (int p = group; p < a.pieces; p += GROUPS) s += a.parts[(static_cast<int64_t>(p) * gridDim.y + g) * each + at];
    sums[group][threadIdx.x & 63] = s;
    __syncthreads();
    if (group != 0 || at >= each) return;
#pragma unroll
    for (int p = 1; p < GROUPS; ++p) s += sums[p][threadIdx.x];
    const int64_t m = at / a.columns, k = at - m * a.columns;
    store_one(a.dx, g * a.dx_batch + m * a.lddx + k, a.l.type, s);
}

}  // namespace

int launch_small_grads(const SmallGrads &a, hipStream_t stream)
{
    if (a.pieces <= 0 || a.batch <= 0) return GBMUF_OK;
    SmallGrads args = a;
    void *argv[] = {&args};
    using Fn = void (*)(SmallGrads);
    static constexpr Fn fns[3][2] = {{small_grads_kernel<kF32, kSmallRows>, small_grads_kernel<kF32, kSmallRows / 2>},
                                     {small_grads_kernel<kBf16, kSmallRows>, small_grads_kernel<kBf16, kSmallRows / 2>},
                                     {small_grads_kernel<kF16, kSmallRows>, small_grads_kernel<kF16, kSmallRows / 2>}};
    const Fn fn = fns[a.l.type][2 * a.l.words.rows <= kSmallRows ? 1 : 0];
    const hipError_t err = hipLaunchKernel(reinterpret_cast<const void *>(fn), dim3(static_cast<unsigned>(a.pieces), static_cast<unsigned>(a.batch)), dim3(kThreads), argv, 0, stream);
    if (err != hipSuccess) return hip_failed("hipLaunchKernel(small gradients)", err, GBMUF_EDEVICE);
    return launch_join_parts(a, a.pieces, stream);
}

int launch_join_parts(const SmallGrads &a, int32_t parts, hipStream_t stream)
{
    const int64_t blocks = (static_cast<int64_t>(a.l.words.rows) * a.columns + 63) / 64;
    if (!a.parts || blocks <= 0 || a.batch <= 0) return GBMUF_OK;
    SmallGrads args = a;
    args.pieces = parts;
    void *argv[] = {&args};
    const hipError_t err = hipLaunchKernel(reinterpret_cast<const void *>(parts > 32 ? small_join_kernel<16> : small_join_kernel<4>),
                                           dim3(static_cast<unsigned>(blocks), static_cast<unsigned>(a.batch)), dim3(parts > 32 ? 1024 : 256), argv, 0, stream);
    return err == hipSuccess ? GBMUF_OK : hip_failed("hipLaunchKernel(parts of dx)", err, GBMUF_EDEVICE);
}

}  // namespace gbmuf
