// gbmuf_few.hip -- the forward product for few rows: what answering takes, token by token.
#include "gbmuf_values.h"

namespace gbmuf {
namespace {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v4u_any __attribute__((ext_vector_type(4), aligned(2)));

// 16 bytes of a row from value k on: 4 f32 or 8 16-bit values; zeros from K on.
template <int T>
__device__ __forceinline__ v4u piece(const void *row, int k, int K)
{
    using N = typename Num<T>::type;
    constexpr int kValues = 16 / static_cast<int>(sizeof(N));
    const N *p = static_cast<const N *>(row) + k;
    if (k + kValues <= K) return *reinterpret_cast<const v4u_any *>(p);
    uint32_t v[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int c = 0; c < kValues; ++c)
        if (k + c < K) {
            if constexpr (T == kF32) v[c] = __float_as_uint(p[c]);
            else v[c >> 1] |= static_cast<uint32_t>(__builtin_bit_cast(uint16_t, p[c])) << (16 * (c & 1));
        }
    return v4u{v[0], v[1], v[2], v[3]};
}

// acc += w x' over the 4 (f32) or 8 (16-bit) k of each of the four lane groups
template <int T>
__device__ __forceinline__ v4f product(v4u w, v4u x, v4f acc)
{
    if constexpr (T == kF32) {
#pragma unroll
        for (int c = 0; c < 4; ++c) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[c]), __uint_as_float(x[c]), acc, 0, 0, 0);
        return acc;
    } else if constexpr (T == kBf16) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, w), __builtin_bit_cast(v8bf, x), acc, 0, 0, 0);
    } else {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, w), __builtin_bit_cast(v8h, x), acc, 0, 0, 0);
    }
}

// A workgroup takes 16 NT rows of w for all rows of x (up to 16 MT); its waves share the sum over k in turns of UNROLL steps.  Bound by the reading of w: 8 x
// 50,000 x 1024 bf16, w out of HBM, 21.6 us, 4.75 TB/s (twice the steps under way 21.7, streamed loads 23.6).
template <int T, int MT, int NT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void few_kernel(DirectArgs a)
{
    constexpr int kStep = T == kF32 ? 16 : 32, kUnroll = MT * NT <= 2 ? 4 : 2;        // values of k that a wave's load of 16 bytes a lane covers
    __shared__ __align__(16) float part[WAVES][MT * 16 * (NT * 16 + 4)];
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
    for (int at = threadIdx.x; at < MT * 16 * NT * 4; at += 64 * WAVES) {
        const int m = at / (NT * 4), n = at % (NT * 4) * 4;
        if (m >= a.t.M || n0 + n >= a.t.N) continue;
        v4f s = *reinterpret_cast<const v4f *>(&part[0][m * kPitch + n]);
#pragma unroll
        for (int v = 1; v < WAVES; ++v) s += *reinterpret_cast<const v4f *>(&part[v][m * kPitch + n]);
        finish(a.e, g, m, n0 + n, a.t.N - n0 - n, s);
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

}  // namespace

int launch_few(const DirectArgs &a, int32_t type, hipStream_t stream)
{
    if (a.t.M <= 0 || a.t.N <= 0 || a.t.batch <= 0) return GBMUF_OK;
    const int mt = a.t.M <= 16 ? 1 : a.t.M <= 32 ? 2 : 4;
    const int64_t narrow = (a.t.N + 15) / 16;
    // A workgroup that takes more rows of w reads x less often.  us for 50,000 rows of 1024, 16 / 32 / 64 rows a workgroup: bf16, 8 rows of x 22 / 20 /
    // 21, 20 rows 31 / 25 / 23, 64 rows 60 / 41 / 35; f32, 8 rows 48 / 47 / 46, 20 rows 72 / 57 / 64 (64 rows 131 / 112 / 108: tiles
    // take 90).  Few workgroups share long sums between 16 waves.
    const bool many = narrow * a.t.batch >= 2048, widest = mt == 4 || (mt == 2 && type != kF32);
    const int form = many ? (widest ? 3 : 2) : narrow * a.t.batch < 256 && a.K >= 1024 ? 0 : 1;
    const int rows = form == 3 ? 64 : form == 2 ? 32 : 16;
    const int64_t blocks = (a.t.N + rows - 1) / rows;
    const auto fn = type == kF32 ? pick<kF32>(mt, form) : type == kBf16 ? pick<kBf16>(mt, form) : pick<kF16>(mt, form);
    DirectArgs args = a;
    void *argv[] = {&args};
    const hipError_t err = hipLaunchKernel(reinterpret_cast<const void *>(fn), dim3(static_cast<unsigned>(blocks), static_cast<unsigned>(a.t.batch)),
                                           dim3(form == 0 ? 1024 : 256), argv, 0, stream);
    return err == hipSuccess ? GBMUF_OK : hip_failed("hipLaunchKernel(few rows)", err, GBMUF_EDEVICE);
}

}  // namespace gbmuf
