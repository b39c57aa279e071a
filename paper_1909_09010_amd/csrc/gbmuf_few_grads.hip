// gbmuf_few_grads.hip -- gradients of losses of up to 8 rows against any vocabulary: w is read from memory once, and dw written once.
#include "gbmuf_few.h"

namespace gbmuf {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;

template <int T, int C>
__device__ __forceinline__ void read_columns(const void *p, int64_t i, int left, float (&v)[C])
{
    using N = typename Num<T>::type;
    typedef N Piece __attribute__((ext_vector_type(C), aligned(sizeof(N))));
    const N *from = static_cast<const N *>(p) + i;
    if (left >= C) {
        const Piece r = *reinterpret_cast<const Piece *>(from);
#pragma unroll
        for (int c = 0; c < C; ++c) v[c] = static_cast<float>(r[c]);
    } else {
#pragma unroll
        for (int c = 0; c < C; ++c) v[c] = c < left ? static_cast<float>(from[c]) : 0.0f;
    }
}

template <int T, int C>
__device__ __forceinline__ void write_columns(void *p, int64_t i, int left, const float (&v)[C])
{
    using N = typename Num<T>::type;
    typedef N Piece __attribute__((ext_vector_type(C), aligned(sizeof(N))));
    N *to = static_cast<N *>(p) + i;
    if (left >= C) {
        Piece r;
#pragma unroll
        for (int c = 0; c < C; ++c) r[c] = static_cast<N>(v[c]);
        *reinterpret_cast<Piece *>(to) = r;
    } else {
#pragma unroll
        for (int c = 0; c < C; ++c)
            if (c < left) to[c] = static_cast<N>(v[c]);
    }
}

// A workgroup takes every gridDim.x-th piece of 64, 32 or 16 words for all rows.  The logits of a piece come from matrix instructions as in few_sums; their gradient
// stays in LDS, [word][row].  Then threads take C columns each of a word's row, which is in the L2 by now: dw's values are ROWS products with the thread's
// columns of x, dx's sums go on in registers over all pieces: 2 ROWS C multiply-adds a word and thread, 0.1 us a word of 1024 columns and CU for 8 rows, where
// its 4 KB read and 4 KB written take 0.32 at 6.5 TB/s.  `lanes` threads have a word's columns, the others further words.  Bound by w's way from memory.  us, this /
// the routes of more rows: 2 x 1 x 54538 x 241 78 / 142, 1 x 8 x 50000 x 1024 154 / 207, 9 x 6 x 5250 x 74 32 / 42, 1 x 1 x 2368 x 256 12.5 / 28, 1 x 3 x 300 x 700 16
// / 32.  16 rows are short of registers.  Values of w and dw are of type T and D.
template <int T, int D, int ROWS, int kWords>
__global__ __launch_bounds__(kThreads, 2) void few_grads_kernel(SmallGrads a, int32_t lanes)
{
    constexpr int C = 4, kTilesN = kWords / 16, kPitch = kWords + 4;
    constexpr int kStep = T == kF32 ? 16 : 32, kUnroll = 8 / kTilesN, kAhead = 4;
    constexpr size_t kBytes = sizeof(typename Num<T>::type);
    __shared__ __align__(16) float part[kWaves][16 * kPitch];
    __shared__ __align__(16) float dz[kWords][ROWS];
    const LossArgs &l = a.l;
    const Words &w = l.words;
    const int64_t g = blockIdx.y;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, M = w.rows, K = a.columns, V = w.vocab;
    const char *wp = static_cast<const char *>(a.w) + g * a.w_batch * kBytes;

    // a thread's columns of the rows that count
    const int groups = kThreads / lanes, group = static_cast<int>(threadIdx.x) / lanes, k_mine = static_cast<int>(threadIdx.x) % lanes * C, left = K - k_mine;
    float x[ROWS][C], dx[ROWS][C];
#pragma unroll
    for (int m = 0; m < ROWS; ++m) {
        const bool is = m < M && left > 0 && row_state(w, g, m) != kDead;
#pragma unroll
        for (int c = 0; c < C; ++c) x[m][c] = dx[m][c] = 0.0f;
        if (is) read_columns<T, C>(a.x, g * a.x_batch + m * a.ldx + k_mine, left, x[m]);
    }
    // what the row of the logits that a thread finishes brings along
    const int m_z = static_cast<int>(threadIdx.x) / (kWords / 4), mc = min(m_z, M - 1), state = m_z < M ? row_state(w, g, mc) : kDead;
    const float weight = row_weight(l, g, mc, state), lse = l.lse[g * l.lse_batch + mc * l.lse_ld];
    const char *xs = static_cast<const char *>(a.x) + (g * a.x_batch + min(lane & 15, M - 1) * a.ldx) * kBytes;

    for (int piece_n = blockIdx.x; piece_n < a.pieces; piece_n += gridDim.x) {
        const int n0 = piece_n * kWords, words = min(kWords, V - n0);
        // z of 16 rows and 64 words, the waves sharing the sum over k
        const char *ws[kTilesN];
        v4f acc[kTilesN];
#pragma unroll
        for (int j = 0; j < kTilesN; ++j) {
            ws[j] = wp + static_cast<int64_t>(min(n0 + j * 16 + (lane & 15), V - 1)) * a.ldw * kBytes;
            acc[j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        }
        for (int k0 = wave * kStep * kUnroll; k0 < K; k0 += kWaves * kStep * kUnroll) {
            v4u xv[kUnroll], wv[kUnroll][kTilesN];
            const int k = k0 + (lane >> 4) * (kStep / 4);
            if (k0 + kStep * kUnroll <= K) {
#pragma unroll
                for (int u = 0; u < kUnroll; ++u) {
                    xv[u] = *reinterpret_cast<const v4u_any *>(xs + (k + u * kStep) * kBytes);
#pragma unroll
                    for (int j = 0; j < kTilesN; ++j) wv[u][j] = *reinterpret_cast<const v4u_any *>(ws[j] + (k + u * kStep) * kBytes);
                }
            } else {
#pragma unroll
                for (int u = 0; u < kUnroll; ++u) {
                    xv[u] = piece<T>(xs, k + u * kStep, K);
#pragma unroll
                    for (int j = 0; j < kTilesN; ++j) wv[u][j] = piece<T>(ws[j], k + u * kStep, K);
                }
            }
#pragma unroll
            for (int u = 0; u < kUnroll; ++u)
#pragma unroll
                for (int j = 0; j < kTilesN; ++j) acc[j] = product<T>(wv[u][j], xv[u], acc[j]);
        }
#pragma unroll
        for (int j = 0; j < kTilesN; ++j) *reinterpret_cast<v4f *>(&part[wave][(lane & 15) * kPitch + j * 16 + (lane >> 4) * 4]) = acc[j];
        __syncthreads();
        // a thread has 4 words of one row
        if (m_z < ROWS) {
            const int at = static_cast<int>(threadIdx.x) % (kWords / 4) * 4;
            v4f z = *reinterpret_cast<const v4f *>(&part[0][m_z * kPitch + at]);
#pragma unroll
            for (int v = 1; v < kWaves; ++v) z += *reinterpret_cast<const v4f *>(&part[v][m_z * kPitch + at]);
            float d[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const bool is = state != kDead && at + c < words;
                const float b = l.bias && at + c < words ? load_one(l.bias, g * l.bias_batch + n0 + at + c, T) : 0.0f;
                d[c] = is ? weight * exp2_of(fmaf(z[c] + b, l.inv_tau, -lse) * kLog2E) : 0.0f;
            }
            const auto take = [&](int64_t word, float share) {
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (word == n0 + at + c) d[c] -= weight * share;
            };
            if (state != kDead) {
                if (w.target) take(w.target[g * w.batch + mc * w.ld], 1.0f);
                else {
                    const int32_t *list = w.id + (g * w.rows + mc) * w.top;
                    const float *share = w.share + (g * w.rows + mc) * w.top;
                    int place = 0, step = 1;
                    while (2 * step <= w.top) step *= 2;
                    for (; step; step >>= 1)
                        if (place + step <= w.top && list[place + step - 1] < n0 + at) place += step;
                    for (; place < w.top && list[place] < n0 + min(at + 4, words); ++place) take(list[place], share[place]);
                }
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) dz[at + c][m_z] = d[c];
        }
        __syncthreads();
        if (a.dbias && threadIdx.x < static_cast<unsigned>(words)) {
            float v = 0.0f;
#pragma unroll
            for (int m = 0; m < ROWS; ++m) v += dz[threadIdx.x][m];
            const int64_t at = g * a.dbias_batch + n0 + threadIdx.x;
            if (a.accumulate) v += load_one(a.dbias, at, D);
            store_one(a.dbias, at, D, v);
        }
        if (left > 0)
            for (int n = group; n < words; n += kAhead * groups) {
                float v[kAhead][C], was[kAhead][C];
                // words behind the last are read as the last one
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    const int64_t row = n0 + min(n + u * groups, words - 1);
                    if (a.parts) read_columns<T, C>(wp, row * a.ldw + k_mine, left, v[u]);
                    if (a.dw && a.accumulate) read_columns<D, C>(a.dw, g * a.dw_batch + row * a.lddw + k_mine, left, was[u]);
                }
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    const int word = n + u * groups;
                    if (word >= words) continue;
                    float out[C], d[ROWS];
#pragma unroll
                    for (int m = 0; m < ROWS; ++m) d[m] = dz[word][m];
#pragma unroll
                    for (int c = 0; c < C; ++c) out[c] = 0.0f;
#pragma unroll
                    for (int m = 0; m < ROWS; ++m)
#pragma unroll
                        for (int c = 0; c < C; ++c) {
                            out[c] = fmaf(d[m], x[m][c], out[c]);
                            if (a.parts) dx[m][c] = fmaf(d[m], v[u][c], dx[m][c]);
                        }
                    if (a.dw) {
                        if (a.accumulate)
#pragma unroll
                            for (int c = 0; c < C; ++c) out[c] += was[u][c];
                        write_columns<D, C>(a.dw, g * a.dw_batch + static_cast<int64_t>(n0 + word) * a.lddw + k_mine, left, out);
                    }
                }
            }
        __syncthreads();                                   // dz and the parts of z are the next piece's
    }
    if (!a.parts || left <= 0) return;
    float *to = a.parts + ((static_cast<int64_t>(blockIdx.x) * groups + group) * gridDim.y + g) * M * K;
#pragma unroll
    for (int m = 0; m < ROWS; ++m)
        if (m < M) write_columns<kF32, C>(to, static_cast<int64_t>(m) * K + k_mine, left, dx[m]);
}

}  // namespace

// Threads for a word's columns, 4 each.
int few_grads_lanes(int64_t K)
{
    int lanes = 16;
    while (lanes < kThreads && lanes * 4 < K) lanes *= 2;
    return lanes;
}

int launch_few_grads(const SmallGrads &a, int32_t workgroups, hipStream_t stream)
{
    if (a.pieces <= 0 || a.batch <= 0) return GBMUF_OK;
    SmallGrads args = a;
    int32_t lanes = few_grads_lanes(a.columns);
    void *argv[] = {&args, &lanes};
    using Fn = void (*)(SmallGrads, int32_t);
    // [type][gradients in f32][more than 4 rows][pieces of 64, 32, 16 words]
#define GBMUF_FEW(T, D) \
    {{few_grads_kernel<T, D, 4, 64>, few_grads_kernel<T, D, 4, 32>, few_grads_kernel<T, D, 4, 16>}, \
     {few_grads_kernel<T, D, 8, 64>, few_grads_kernel<T, D, 8, 32>, few_grads_kernel<T, D, 8, 16>}}
    static constexpr Fn fns[3][2][2][3] = {{{}, GBMUF_FEW(kF32, kF32)}, {GBMUF_FEW(kBf16, kBf16), GBMUF_FEW(kBf16, kF32)}, {GBMUF_FEW(kF16, kF16), GBMUF_FEW(kF16, kF32)}};
#undef GBMUF_FEW
    const void *fn = reinterpret_cast<const void *>(fns[a.l.type][a.grad_type == kF32 ? 1 : 0][a.l.words.rows > 4 ? 1 : 0][a.words == 64 ? 0 : a.words == 32 ? 1 : 2]);
    const hipError_t err = hipLaunchKernel(fn, dim3(static_cast<unsigned>(workgroups), static_cast<unsigned>(a.batch)), dim3(kThreads), argv, 0, stream);
    return err == hipSuccess ? GBMUF_OK : hip_failed("hipLaunchKernel(few rows' gradients)", err, GBMUF_EDEVICE);
}

}  // namespace gbmuf
