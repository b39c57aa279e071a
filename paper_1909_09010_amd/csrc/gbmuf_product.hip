// gbmuf_product.hip -- matrix products on gfx950's matrix cores for the local half: out = a b' over 16-bit numbers.
#include "gbmuf_values.h"

namespace gbmuf {
namespace {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

constexpr int kStep = 64;                                  // 16-bit words of a row per step: one 128-byte line

template <int T>
__device__ __forceinline__ v16f mfma(v4u a, v4u b, v16f c)
{
    if constexpr (T == kBf16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
}

// Stages R rows of one step in LDS: 128 bytes a row, the 16-byte chunk c of row r at place c ^ (r & 7), so that the 32 rows
// that a matrix instruction reads lie in all banks.  Whole steps go from global memory to LDS directly, 1 KB a wave and
// instruction, which writes lane by lane: the lanes fetch the chunk that belongs at their place.  A last step that is not whole goes
// through registers, zeros behind the end.
template <int R, int THREADS>
struct Stage {
    static constexpr int kPass = THREADS / 8, kPasses = R / kPass;
    const uint16_t *row[kPasses];
    int chunk[kPasses];

    __device__ __forceinline__ void init(const uint16_t *base, int64_t ld, int first, int count)
    {
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            const int r = i * kPass + static_cast<int>(threadIdx.x >> 3);
            row[i] = base + static_cast<int64_t>(min(first + r, count - 1)) * ld;        // rows behind the last are read as the last one
            chunk[i] = (static_cast<int>(threadIdx.x & 7) ^ (r & 7)) * 8;
        }
    }

    __device__ __forceinline__ void load(uint16_t *lds, int k0, int K) const
    {
        if (k0 + kStep <= K) {
#pragma unroll
            for (int i = 0; i < kPasses; ++i) {
                uint16_t *to = lds + (i * kPass + static_cast<int>(threadIdx.x >> 6) * 8) * kStep;
                __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) void *)(row[i] + k0 + chunk[i]),
                                                 (__attribute__((address_space(3))) void *)to, 16, 0, 0);
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            uint32_t v[4] = {0u, 0u, 0u, 0u};
            const int left = K - (k0 + chunk[i]);
#pragma unroll
            for (int c = 0; c < 8; ++c)
                if (c < left) v[c >> 1] |= static_cast<uint32_t>(row[i][k0 + chunk[i] + c]) << (16 * (c & 1));
            const int r = i * kPass + static_cast<int>(threadIdx.x >> 3);
            *reinterpret_cast<v4u *>(lds + r * kStep + (threadIdx.x & 7) * 8) = v4u{v[0], v[1], v[2], v[3]};
        }
    }
};

__device__ __forceinline__ v4u chunk_of(const uint16_t *lds, int row, int chunk)
{
    return *reinterpret_cast<const v4u *>(lds + row * kStep + ((chunk ^ (row & 7)) * 8));
}

// One tile of TM x TN, WM x WN waves.
template <int T, bool SPLIT, int TM, int TN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void product_kernel(ProductArgs a)
{
    constexpr int THREADS = 64 * WM * WN, FM = TM / WM / 32, FN = TN / WN / 32;
    __shared__ __align__(1024) uint16_t lds[2][(TM + TN) * kStep];

    const int per = a.tiles_m * a.tiles_n;
    int id = static_cast<int>(blockIdx.x);
    const int split = id / (per * a.batch);
    id -= split * per * a.batch;
    const int g = id / per;
    id -= g * per;
    const int m0 = (id % a.tiles_m) * TM, n0 = (id / a.tiles_m) * TN;

    const int all = (a.K + kStep - 1) / kStep, first = split * a.steps, last = min(first + a.steps, all);
    Stage<TM, THREADS> sa;
    Stage<TN, THREADS> sb;
    sa.init(a.a + g * a.a_batch, a.lda, m0, a.M);
    sb.init(a.b + g * a.b_batch, a.ldb, n0, a.N);

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wm = (wave % WM) * (TM / WM), wn = (wave / WM) * (TN / WN);
    v16f acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

    if (first < last) {
        sa.load(lds[0], first * kStep, a.K);
        sb.load(lds[0] + TM * kStep, first * kStep, a.K);
    }
    __syncthreads();
    for (int s = first; s < last; ++s) {
        const uint16_t *now = lds[(s - first) & 1];
        uint16_t *next = lds[(s - first + 1) & 1];
        if (s + 1 < last) {
            sa.load(next, (s + 1) * kStep, a.K);
            sb.load(next + TM * kStep, (s + 1) * kStep, a.K);
        }
        const uint16_t *la = now + wm * kStep, *lb = now + (TM + wn) * kStep;
#pragma unroll
        for (int k = 0; k < (SPLIT ? 2 : 4); ++k) {
            v4u x[SPLIT ? 2 : 1][FM], w[SPLIT ? 2 : 1][FN];
#pragma unroll
            for (int p = 0; p < (SPLIT ? 2 : 1); ++p) {
                const int c = p * 4 + k * 2 + (lane >> 5);
#pragma unroll
                for (int i = 0; i < FM; ++i) x[p][i] = chunk_of(la, i * 32 + (lane & 31), c);
#pragma unroll
                for (int j = 0; j < FN; ++j) w[p][j] = chunk_of(lb, j * 32 + (lane & 31), c);
            }
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    acc[i][j] = mfma<T>(w[0][j], x[0][i], acc[i][j]);
                    if constexpr (SPLIT) {
                        acc[i][j] = mfma<T>(w[1][j], x[0][i], acc[i][j]);
                        acc[i][j] = mfma<T>(w[0][j], x[1][i], acc[i][j]);
                    }
                }
        }
        __syncthreads();
    }

    // The tile leaves through LDS, 32 rows of every wave at a time, so that a wave's loads and stores follow rows.  A lane holds, of row
    // lane % 32, the columns 8 (r / 4) + 4 (lane / 32) + r % 4.
    constexpr int kRows = WM * 32, kPitch = TN + 4;
    static_assert(kRows * kPitch * 4 <= sizeof(lds), "a pass fits the stages");
    float *out = reinterpret_cast<float *>(&lds[0][0]);
#pragma unroll
    for (int i = 0; i < FM; ++i) {
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<v4f *>(out + ((wave % WM) * 32 + (lane & 31)) * kPitch + wn + j * 32 + 8 * q + 4 * (lane >> 5)) =
                    v4f{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        __syncthreads();
        for (int at = threadIdx.x; at < kRows * (TN / 4); at += THREADS) {
            const int row = at / (TN / 4), n = n0 + at % (TN / 4) * 4, m = m0 + row / 32 * (TM / WM) + i * 32 + row % 32;
            if (m >= a.M || n >= a.N) continue;
            const int left = a.N - n;
            v4f v = *reinterpret_cast<const v4f *>(out + row * kPitch + (n - n0));
            if constexpr (SPLIT) {
                const int em = row_exponent(a.a_max[g * a.a_max_batch + m]);
                const uint32_t *top = a.b_max + g * a.b_max_batch + n;
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (c < left) v[c] = ldexpf(v[c], em + row_exponent(top[c]));
            }
            if (a.splits > 1) {
                float *to = a.partial + ((static_cast<int64_t>(split) * a.batch + g) * a.M + m) * a.N + n;
                if (left >= 4) store4<kPlain>(to, v);
                else
                    for (int c = 0; c < 3; ++c)
                        if (c < left) to[c] = v[c];
            } else {
                finish(a.e, g, m, n, left, v);
            }
        }
        __syncthreads();
    }
}

// Joins the parts of sums that were split, in their order.
__global__ __launch_bounds__(256) void join_kernel(JoinArgs a)
{
    const int64_t all = a.M * a.N * a.batch, fours = (a.N + 3) / 4, work = fours * a.M * a.batch;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < work; i += static_cast<int64_t>(gridDim.x) * 256) {
        const int64_t row = i / fours, n = (i - row * fours) * 4, g = row / a.M;
        const int left = static_cast<int>(min(a.N - n, int64_t{4}));
        const float *from = a.partial + row * a.N + n;
        v4f s = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int p = 0; p < a.splits; ++p, from += all) {
            if (left == 4) s += load4<kPlain>(from);
            else
                for (int c = 0; c < 3; ++c)
                    if (c < left) s[c] += from[c];
        }
        finish(a.e, g, row - g * a.M, n, left, s);
    }
}

}  // namespace

int launch_product(const ProductArgs &a, int32_t type, hipStream_t stream)
{
    if (a.M <= 0 || a.N <= 0 || a.batch <= 0) return GBMUF_OK;
    const int64_t blocks = static_cast<int64_t>(a.tiles_m) * a.tiles_n * a.batch * a.splits;
    if (blocks > 0x7fffffffLL / 256) return GBMUF_EUNSUPPORTED;
    ProductArgs args = a;
    void *argv[] = {&args};
    using Fn = void (*)(ProductArgs);
    const Fn fn = type == kF32   ? product_kernel<kF16, true, 128, 128, 2, 2>
                  : type == kF16 ? product_kernel<kF16, false, 128, 128, 2, 2>
                                 : product_kernel<kBf16, false, 128, 128, 2, 2>;
    const hipError_t err = hipLaunchKernel(reinterpret_cast<const void *>(fn), dim3(static_cast<unsigned>(blocks)), dim3(256), argv, 0, stream);
    return err == hipSuccess ? GBMUF_OK : hip_failed("hipLaunchKernel(product)", err, GBMUF_EDEVICE);
}

int launch_join(const JoinArgs &a, hipStream_t stream)
{
    const int64_t all = (a.N + 3) / 4 * a.M * a.batch;
    if (all <= 0) return GBMUF_OK;
    JoinArgs args = a;
    void *argv[] = {&args};
    const int64_t blocks = (all + 255) / 256;
    const hipError_t err = hipLaunchKernel(reinterpret_cast<const void *>(join_kernel), dim3(static_cast<unsigned>(blocks < 65536 ? blocks : 65536)),
                                           dim3(256), argv, 0, stream);
    return err == hipSuccess ? GBMUF_OK : hip_failed("hipLaunchKernel(join)", err, GBMUF_EDEVICE);
}

}  // namespace gbmuf
