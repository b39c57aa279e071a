// gbmuf_layout.hip -- what products need laid out first: rows of 16-bit numbers along the axis that is summed over, whole steps
// long, taken apart into two f16 numbers where the source is f32; and, in the backward, dz = dy * act'(z) and its column sums.
#include "gbmuf_values.h"

namespace gbmuf {
namespace {

constexpr int kT = kLayTile;

__device__ __forceinline__ float value_at(const LayArgs &a, int64_t g, int r, int c)
{
    float v = load_one(a.src, g * a.batch_stride + r * a.ld + c, a.type);
    if (a.act) v *= slope(load_one(a.pre, g * a.p_batch + r * a.ldp + c, a.type), a.act);
    return v;
}

// Largest magnitudes of rows and columns, and sums of columns over the tile's rows.  Magnitudes compare as integers, and a maximum does not depend on
// the order of the atomics.
__global__ __launch_bounds__(256) void stats_kernel(LayArgs a)
{
    __shared__ float sums[4][kT];
    __shared__ uint32_t top[4][kT];
    const int tiles_c = (a.C + kT - 1) / kT, tiles_r = (a.R + kT - 1) / kT;
    int id = static_cast<int>(blockIdx.x);
    const int64_t g = id / (tiles_c * tiles_r);
    id -= static_cast<int>(g) * tiles_c * tiles_r;
    const int tr = id / tiles_c, r0 = tr * kT, c = id % tiles_c * kT + static_cast<int>(threadIdx.x & 63), wave = threadIdx.x >> 6;
    float s = 0.0f;
    uint32_t most = 0;
    for (int i = 0; i < kT / 4; ++i) {
        const int r = r0 + i * 4 + wave;
        const float v = r < a.R && c < a.C ? value_at(a, g, r, c) : 0.0f;
        s += v;
        const uint32_t bits = __float_as_uint(v) & 0x7fffffffu;
        most = max(most, bits);
        if (a.row_max) {
            uint32_t m = bits;
            for (int d = 32; d; d >>= 1) m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), d)));
            if ((threadIdx.x & 63) == 0 && r < a.R && m) atomicMax(a.row_max + g * a.R + r, m);
        }
    }
    sums[wave][threadIdx.x & 63] = s;
    top[wave][threadIdx.x & 63] = most;
    __syncthreads();
    if (wave != 0 || c >= a.C) return;
    const int t = threadIdx.x;
    if (a.col_max) {
        const uint32_t m = max(max(top[0][t], top[1][t]), max(top[2][t], top[3][t]));
        if (m) atomicMax(a.col_max + g * a.C + c, m);
    }
    if (a.col_sums) a.col_sums[(g * tiles_r + tr) * a.C + c] = (sums[0][t] + sums[1][t]) + (sums[2][t] + sums[3][t]);
}

// The two f16 numbers of a value that its row's exponent has scaled.
__device__ __forceinline__ void take_apart(float v, uint16_t &lead, uint16_t &trail)
{
    const _Float16 h = static_cast<_Float16>(v);
    const float f = static_cast<float>(h);
    const _Float16 l = fabsf(f) <= 65504.0f ? static_cast<_Float16>(v - f) : static_cast<_Float16>(0.0f);
    lead = __builtin_bit_cast(uint16_t, h);
    trail = __builtin_bit_cast(uint16_t, l);
}

__device__ __forceinline__ uint16_t word_of(float v, int32_t type)
{
    return type == kBf16 ? __builtin_bit_cast(uint16_t, static_cast<__bf16>(v)) : __builtin_bit_cast(uint16_t, static_cast<_Float16>(v));
}

typedef uint32_t v4u __attribute__((ext_vector_type(4)));

// One row's 8 values from `at` on, at place k of the packed row.
template <class At>
__device__ __forceinline__ void write8(uint16_t *row, int k, int32_t type, uint32_t max_bits, At at)
{
    uint16_t w[8], t[8];
    if (type == kF32) {
        const int e = -row_exponent(max_bits);
        for (int i = 0; i < 8; ++i) take_apart(ldexpf(at(i), e), w[i], t[i]);
        uint16_t *to = row + (k >> 5) * 64 + (k & 31);
        *reinterpret_cast<v4u *>(to) = __builtin_bit_cast(v4u, w);
        *reinterpret_cast<v4u *>(to + 32) = __builtin_bit_cast(v4u, t);
    } else {
        for (int i = 0; i < 8; ++i) w[i] = word_of(at(i), type);
        *reinterpret_cast<v4u *>(row + k) = __builtin_bit_cast(v4u, w);
    }
}

__global__ __launch_bounds__(256) void lay_kernel(LayArgs a)
{
    __shared__ float tile[kT][kT + 1];
    const int tiles_c = (a.C + kT - 1) / kT, tiles_r = (a.R + kT - 1) / kT;
    int id = static_cast<int>(blockIdx.x);
    const int64_t g = id / (tiles_c * tiles_r);
    id -= static_cast<int>(g) * tiles_c * tiles_r;
    const int r0 = id / tiles_c * kT, c0 = id % tiles_c * kT;
    for (int i = 0; i < kT / 4; ++i) {
        const int r = i * 4 + static_cast<int>(threadIdx.x >> 6), c = threadIdx.x & 63;
        float v = 0.0f;
        if (r0 + r < a.R && c0 + c < a.C) {
            v = value_at(a, g, r0 + r, c0 + c);
            if (a.dz) store_one(a.dz, g * a.dz_batch + (r0 + r) * a.dz_ld + c0 + c, a.type, v);
        }
        tile[r][c] = v;
    }
    __syncthreads();
    const int room = a.type == kF32 ? 32 : 64;             // packed rows are whole multiples of this many values
    if (a.plain)
        for (int j = threadIdx.x; j < kT * 8; j += 256) {
            const int r = j >> 3, c = (j & 7) * 8;
            if (r0 + r >= a.R || c0 + c >= (a.C + room - 1) / room * room) continue;
            write8(a.plain + g * a.plain_batch + static_cast<int64_t>(r0 + r) * a.plain_ld, c0 + c, a.type,
                   a.row_max ? a.row_max[g * a.R + r0 + r] : 0u, [&](int i) { return tile[r][c + i]; });
        }
    if (a.trans)
        for (int j = threadIdx.x; j < kT * 8; j += 256) {
            const int c = j & 63, r = (j >> 6) * 8;
            if (c0 + c >= a.C || r0 + r >= (a.R + room - 1) / room * room) continue;
            write8(a.trans + g * a.trans_batch + static_cast<int64_t>(c0 + c) * a.trans_ld, r0 + r, a.type,
                   a.col_max ? a.col_max[g * a.C + c0 + c] : 0u, [&](int i) { return tile[r + i][c]; });
        }
}

__global__ __launch_bounds__(256) void column_sums_kernel(SumArgs a)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (i >= static_cast<int64_t>(a.C) * a.batch) return;
    const int64_t g = i / a.C, c = i - g * a.C;
    float s = 0.0f;
    for (int t = 0; t < a.tiles; ++t) s += a.sums[(g * a.tiles + t) * a.C + c];
    if (a.accumulate) s += load_one(a.out, g * a.out_batch + c, a.type);
    store_one(a.out, g * a.out_batch + c, a.type, s);
}

__global__ __launch_bounds__(256) void zero_kernel(uint32_t *p, int64_t words)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (i < words) p[i] = 0u;
}

template <class Args>
int launch_256(void (*fn)(Args), const Args &a, int64_t blocks, const char *what, hipStream_t stream)
{
    if (blocks <= 0) return GBMUF_OK;
    if (blocks > 0x7fffffffLL / 256) return GBMUF_EUNSUPPORTED;
    Args args = a;
    void *argv[] = {&args};
    const hipError_t err = hipLaunchKernel(reinterpret_cast<const void *>(fn), dim3(static_cast<unsigned>(blocks)), dim3(256), argv, 0, stream);
    return err == hipSuccess ? GBMUF_OK : hip_failed(what, err, GBMUF_EDEVICE);
}

int64_t lay_blocks(const LayArgs &a)
{
    return static_cast<int64_t>((a.C + kT - 1) / kT) * ((a.R + kT - 1) / kT) * a.batch;
}

}  // namespace

int launch_stats(const LayArgs &a, hipStream_t stream) { return launch_256(stats_kernel, a, lay_blocks(a), "hipLaunchKernel(stats)", stream); }
int launch_lay(const LayArgs &a, hipStream_t stream) { return launch_256(lay_kernel, a, lay_blocks(a), "hipLaunchKernel(lay out)", stream); }

int launch_column_sums(const SumArgs &a, hipStream_t stream)
{
    return launch_256(column_sums_kernel, a, (static_cast<int64_t>(a.C) * a.batch + 255) / 256, "hipLaunchKernel(column sums)", stream);
}

int launch_zero(uint32_t *p, int64_t words, hipStream_t stream)
{
    if (words <= 0) return GBMUF_OK;
    const int64_t blocks = (words + 255) / 256;
    if (blocks > 0x7fffffffLL / 256) return GBMUF_EUNSUPPORTED;
    void *argv[] = {&p, &words};
    const hipError_t err = hipLaunchKernel(reinterpret_cast<const void *>(zero_kernel), dim3(static_cast<unsigned>(blocks)), dim3(256), argv, 0, stream);
    return err == hipSuccess ? GBMUF_OK : hip_failed("hipLaunchKernel(zero)", err, GBMUF_EDEVICE);
}

}  // namespace gbmuf
