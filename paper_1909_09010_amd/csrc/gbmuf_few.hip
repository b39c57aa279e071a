// gbmuf_few.hip -- the forward product for few rows: what answering takes, token by token.
#include "gbmuf_few.h"

namespace gbmuf {
namespace {

// A workgroup takes 16 NT rows of w for all rows of x (up to 16 MT); its waves share the sum over k in turns of UNROLL steps.  Bound by the reading of w: 8 x
// 50,000 x 1024 bf16, w out of HBM, 21.6 us, 4.75 TB/s (twice the steps under way 21.7, streamed loads 23.6).
template <int T, int MT, int NT, int WAVES>
__device__ __forceinline__ void few_sums(const DirectArgs &a, float (&part)[WAVES][MT * 16 * (NT * 16 + 4)])
{
    constexpr int kStep = T == kF32 ? 16 : 32, kUnroll = MT * NT <= 2 ? 4 : 2;        // values of k that a wave's load of 16 bytes a lane covers
    const int64_t g = blockIdx.y;
    const int n0 = static_cast<int>(blockIdx.x) * NT * 16, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    constexpr size_t kBytes = sizeof(typename Num<T>::type);
    const char *xs[MT], *ws[NT];
#pragma unroll
    for (int i = 0; i < MT; ++i) xs[i] = static_cast<const char *>(a.a.p) + (g * a.a.batch + min(i * 16 + (lane & 15), a.t.M - 1) * a.a.ld) * kBytes;
#pragma unroll
    for (int j = 0; j < NT; ++j) ws[j] = static_cast<const char *>(a.b.p) + (g * a.b.batch + min(n0 + j * 16 + (lane & 15), a.t.N - 1) * a.b.ld) * kBytes;
    v4f acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    for (int k0 = wave * kStep * kUnroll; k0 < a.K; k0 += WAVES * kStep * kUnroll) {
        v4u x[kUnroll][MT], w[kUnroll][NT];
        const int k = k0 + (lane >> 4) * (kStep / 4);
        if (k0 + kStep * kUnroll <= a.K) {
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
#pragma unroll
                for (int j = 0; j < NT; ++j) w[u][j] = *reinterpret_cast<const v4u_any *>(ws[j] + (k + u * kStep) * kBytes);
#pragma unroll
                for (int i = 0; i < MT; ++i) x[u][i] = *reinterpret_cast<const v4u_any *>(xs[i] + (k + u * kStep) * kBytes);
            }
        } else {
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
#pragma unroll
                for (int j = 0; j < NT; ++j) w[u][j] = piece<T>(ws[j], k + u * kStep, a.K);
#pragma unroll
                for (int i = 0; i < MT; ++i) x[u][i] = piece<T>(xs[i], k + u * kStep, a.K);
            }
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = product<T>(w[u][j], x[u][i], acc[i][j]);
    }
    // a lane holds, of row lane % 16 of x, the columns 4 (lane / 16) + 0 .. 3
    constexpr int kPitch = NT * 16 + 4;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) *reinterpret_cast<v4f *>(&part[wave][(i * 16 + (lane & 15)) * kPitch + j * 16 + (lane >> 4) * 4]) = acc[i][j];
    __syncthreads();
}

// The sums of four columns from n on of row m.
template <int NT, int WAVES, int N>
__device__ __forceinline__ v4f few_joined(const float (&part)[WAVES][N], int m, int n)
{
    constexpr int kPitch = NT * 16 + 4;
    v4f s = *reinterpret_cast<const v4f *>(&part[0][m * kPitch + n]);
#pragma unroll
    for (int v = 1; v < WAVES; ++v) s += *reinterpret_cast<const v4f *>(&part[v][m * kPitch + n]);
    return s;
}

template <int T, int MT, int NT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void few_kernel(DirectArgs a)
{
    __shared__ __align__(16) float part[WAVES][MT * 16 * (NT * 16 + 4)];
    few_sums<T, MT, NT, WAVES>(a, part);
    const int64_t g = blockIdx.y;
    const int n0 = static_cast<int>(blockIdx.x) * NT * 16;
    for (int at = threadIdx.x; at < MT * 16 * NT * 4; at += 64 * WAVES) {
        const int m = at / (NT * 4), n = at % (NT * 4) * 4;
        if (m >= a.t.M || n0 + n >= a.t.N) continue;
        finish(a.e, g, m, n0 + n, a.t.N - n0 - n, few_joined<NT, WAVES>(part, m, n));
    }
}

// The same sums as logits: of every row the tile's part of the softmax statistics, from the 4 NT lanes that hold the row, and the logits of its words.
template <int T, int MT, int NT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void loss_few_kernel(DirectArgs a, LossArgs l)
{
    __shared__ __align__(16) float part[WAVES][MT * 16 * (NT * 16 + 4)];
    few_sums<T, MT, NT, WAVES>(a, part);
    const int64_t g = blockIdx.y;
    const int n0 = static_cast<int>(blockIdx.x) * NT * 16;
    const float scale = l.inv_tau * kLog2E;
    const Words &w = l.words;
    for (int at = threadIdx.x; at < MT * 16 * NT * 4; at += 64 * WAVES) {
        const int m = at / (NT * 4), n = n0 + at % (NT * 4) * 4, left = a.t.N - n;
        if (m >= a.t.M) continue;                           // all lanes of the row
        v4f z = few_joined<NT, WAVES>(part, m, n - n0);
#pragma unroll
        for (int c = 0; c < 4; ++c) z[c] = c < left ? z[c] + (l.bias ? load_one(l.bias, g * l.bias_batch + n + c, T) : 0.0f) : -__builtin_inff();
        float most = fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3]));
#pragma unroll
        for (int d = 1; d < NT * 4; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
        const float from = fabsf(most) < __builtin_inff() ? most : 0.0f;
        float s = 0.0f;
#pragma unroll
        for (int c = 0; c < 4; ++c) s += exp2_of((z[c] - from) * scale);
#pragma unroll
        for (int d = 1; d < NT * 4; d *= 2) s += __shfl_xor(s, d);
        if (n == n0) l.parts[(g * l.part_tiles + blockIdx.x) * w.rows + m] = float2{most, s};
        const int64_t row = g * w.rows + m;
        const auto logit = [&](int64_t word) {
            const int c = static_cast<int>(word - n);
            return c == 0 ? z[0] : c == 1 ? z[1] : c == 2 ? z[2] : z[3];
        };
        const int end = min(n + 4, a.t.N);
        if (w.target) {
            const int64_t *words = w.target + g * w.batch + m * w.ld;
            for (int j = 0; j < w.top; ++j) {
                const int64_t word = words[j];
                if (word >= n && word < end) l.at[row * w.top + j] = logit(word);
            }
        } else {
            const int32_t *list = w.id + row * w.top;
            int place = 0, step = 1;
            while (2 * step <= w.top) step *= 2;
            for (; step; step >>= 1)
                if (place + step <= w.top && list[place + step - 1] < n) place += step;
            for (; place < w.top && list[place] < end; ++place) l.at[row * w.top + place] = logit(list[place]);
        }
    }
}

// form 0: few tiles, 16 waves; 1: 16 rows of w a workgroup; 2, 3: 32, 64 rows.  What no call takes is nullptr: f32 of more than 32 rows against many outputs
// goes to tiles.
template <int T>
void (*pick(int mt, int form))(DirectArgs)
{
    using Fn = void (*)(DirectArgs);
    static constexpr Fn one[] = {few_kernel<T, 1, 1, 16>, few_kernel<T, 1, 1, 4>, few_kernel<T, 1, 2, 4>, nullptr};
    if (mt == 1) return one[form];
    if constexpr (T == kF32) {
        static constexpr Fn more[2][4] = {{few_kernel<T, 2, 1, 16>, few_kernel<T, 2, 1, 4>, few_kernel<T, 2, 2, 4>, nullptr},
                                          {few_kernel<T, 4, 1, 16>, few_kernel<T, 4, 1, 4>, nullptr, nullptr}};
        return more[mt == 4][form];
    } else {
        static constexpr Fn more[2][4] = {{few_kernel<T, 2, 1, 16>, few_kernel<T, 2, 1, 4>, nullptr, few_kernel<T, 2, 4, 4>},
                                          {few_kernel<T, 4, 1, 16>, few_kernel<T, 4, 1, 4>, nullptr, few_kernel<T, 4, 4, 4>}};
        return more[mt == 4][form];
    }
}

template <int T>
void (*pick_loss(int mt, int form))(DirectArgs, LossArgs)
{
    using Fn = void (*)(DirectArgs, LossArgs);
    static constexpr Fn one[] = {loss_few_kernel<T, 1, 1, 16>, loss_few_kernel<T, 1, 1, 4>, loss_few_kernel<T, 1, 2, 4>, nullptr};
    if (mt == 1) return one[form];
    if constexpr (T == kF32) {
        static constexpr Fn more[2][4] = {{loss_few_kernel<T, 2, 1, 16>, loss_few_kernel<T, 2, 1, 4>, loss_few_kernel<T, 2, 2, 4>, nullptr},
                                          {loss_few_kernel<T, 4, 1, 16>, loss_few_kernel<T, 4, 1, 4>, nullptr, nullptr}};
        return more[mt == 4][form];
    } else {
        static constexpr Fn more[2][4] = {{loss_few_kernel<T, 2, 1, 16>, loss_few_kernel<T, 2, 1, 4>, nullptr, loss_few_kernel<T, 2, 4, 4>},
                                          {loss_few_kernel<T, 4, 1, 16>, loss_few_kernel<T, 4, 1, 4>, nullptr, loss_few_kernel<T, 4, 4, 4>}};
        return more[mt == 4][form];
    }
}

// Which kernel a call takes, and how many rows of w a workgroup of it.
struct Form {
    int mt, form, rows;
};

Form form_of(const DirectArgs &a, int32_t type)
{
    const int mt = a.t.M <= 16 ? 1 : a.t.M <= 32 ? 2 : 4;
    const int64_t narrow = (a.t.N + 15) / 16;
    // A workgroup that takes more rows of w reads x less often.  us for 50,000 rows of 1024, 16 / 32 / 64 rows a workgroup: bf16, 8 rows of x 22 / 20 /
    // 21, 20 rows 31 / 25 / 23, 64 rows 60 / 41 / 35; f32, 8 rows 48 / 47 / 46, 20 rows 72 / 57 / 64 (64 rows 131 / 112 / 108: tiles
    // take 90).  Few workgroups share long sums between 16 waves.
    const bool many = narrow * a.t.batch >= 2048, widest = mt == 4 || (mt == 2 && type != kF32);
    const int form = many ? (widest ? 3 : 2) : narrow * a.t.batch < 256 && a.K >= 1024 ? 0 : 1;
    return Form{mt, form, form == 3 ? 64 : form == 2 ? 32 : 16};
}

}  // namespace

int launch_few(const DirectArgs &a, int32_t type, hipStream_t stream)
{
    if (a.t.M <= 0 || a.t.N <= 0 || a.t.batch <= 0) return GBMUF_OK;
    const Form f = form_of(a, type);
    const int64_t blocks = (a.t.N + f.rows - 1) / f.rows;
    const auto fn = type == kF32 ? pick<kF32>(f.mt, f.form) : type == kBf16 ? pick<kBf16>(f.mt, f.form) : pick<kF16>(f.mt, f.form);
    DirectArgs args = a;
    void *argv[] = {&args};
    const hipError_t err = hipLaunchKernel(reinterpret_cast<const void *>(fn), dim3(static_cast<unsigned>(blocks), static_cast<unsigned>(a.t.batch)),
                                           dim3(f.form == 0 ? 1024 : 256), argv, 0, stream);
    return err == hipSuccess ? GBMUF_OK : hip_failed("hipLaunchKernel(few rows)", err, GBMUF_EDEVICE);
}

int few_columns(const DirectArgs &a, int32_t type) { return form_of(a, type).rows; }

int launch_loss_few(const DirectArgs &a, const LossArgs &l, int32_t type, hipStream_t stream)
{
    if (a.t.M <= 0 || a.t.N <= 0 || a.t.batch <= 0) return GBMUF_OK;
    const Form f = form_of(a, type);
    const int64_t blocks = (a.t.N + f.rows - 1) / f.rows;
    const auto fn = type == kF32 ? pick_loss<kF32>(f.mt, f.form) : type == kBf16 ? pick_loss<kBf16>(f.mt, f.form) : pick_loss<kF16>(f.mt, f.form);
    DirectArgs args = a;
    LossArgs loss = l;
    void *argv[] = {&args, &loss};
    const hipError_t err = hipLaunchKernel(reinterpret_cast<const void *>(fn), dim3(static_cast<unsigned>(blocks), static_cast<unsigned>(a.t.batch)),
                                           dim3(f.form == 0 ? 1024 : 256), argv, 0, stream);
    return err == hipSuccess ? GBMUF_OK : hip_failed("hipLaunchKernel(few rows' logits)", err, GBMUF_EDEVICE);
}

}  // namespace gbmuf
