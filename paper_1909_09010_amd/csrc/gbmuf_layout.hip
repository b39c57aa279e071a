// gbmuf_layout.hip -- what products need laid out first: f32 values taken apart into two f16 numbers, in rows along the axis that is summed over;
// 16-bit matrices whose rows do not lie on 16 bytes; and, in the backward, dz = dy * act'(z) and its column sums.
#include "gbmuf_values.h"

namespace gbmuf {
namespace {

constexpr int kT = kLayTile;

// More workgroups than a grid's first dimension holds lie in two; the last row's surplus has nothing to do.
constexpr int64_t kGridRow = 1 << 22;
__device__ __forceinline__ int block_number() { return static_cast<int>(blockIdx.y * gridDim.x + blockIdx.x); }

// The source that workgroup `block` works on, and its number among that source's.
__device__ __forceinline__ const LayArgs &source_of(const LaySet &set, int &block)
{
    int i = 0;
    while (i + 1 < set.n && block >= set.first[i + 1]) ++i;
    block -= set.first[i];
    return set.a[i];
}

// Up to 8 values (r, c) .. of a source, zeros behind the row's end.
template <int T>
__device__ __forceinline__ Eight row_read(const void *p, int64_t at, int left)
{
    if (left >= 8) return read8<T>(p, at);
    Eight e{};
#pragma unroll
    for (int c = 0; c < 8; ++c)
        if (c < left) e.v[c >> 2][c & 3] = load_one(p, at + c, T);
    return e;
}

template <int T>
__device__ __forceinline__ void row_write(void *p, int64_t at, int left, const Eight &e)
{
    if (left >= 8) return write8<T>(p, at, e);
#pragma unroll
    for (int c = 0; c < 8; ++c)
        if (c < left) store_one(p, at + c, T, e.v[c >> 2][c & 3]);
}

// ---------------------------------------------------------------------------------------
// 16-bit sources: rows at aligned places with zeros behind them, dz on the way, and its column sums.  A workgroup takes kT rows of
// 256 columns, a thread 8 columns of every eighth row.  Bound by HBM: one reading (two with an activation) and one writing.
// dz is rounded to the type here, since that is what the 16-bit matrix instructions take: against 64 bits the gradients of 4 x 5120 x 8192 x 1024 bf16 with tanh are off by 0.0023 of their
// size where products of the f32 dz, rounded at the end alike, are off by 0.0017.  A second product with what the rounding leaves would double the products' time.
// ---------------------------------------------------------------------------------------
template <int T>
__global__ __launch_bounds__(256) void copy_kernel(LaySet set)
{
    int id = block_number();
    if (id >= set.first[set.n]) return;
    const LayArgs &a = source_of(set, id);
    __shared__ float sums[8][256];
    const int width = a.plain ? static_cast<int>(a.plain_ld) : a.C;        // zeros up to the end of the copy's rows
    const int tiles_c = (width + 255) / 256, tiles_r = (a.R + kT - 1) / kT;
    const int64_t g = id / (tiles_c * tiles_r);
    id -= static_cast<int>(g) * tiles_c * tiles_r;
    const int tr = id / tiles_c, c0 = id % tiles_c * 256, c = c0 + static_cast<int>(threadIdx.x & 31) * 8, left = a.C - c;
    const int end = min((tr + 1) * kT, a.R);
    Eight total{};
    if (c < width)
        for (int r = tr * kT + static_cast<int>(threadIdx.x >> 5); r < end; r += 8) {
            Eight v = row_read<T>(a.src, g * a.batch_stride + r * a.ld + c, left);
            if (a.act) v = slope8(v, row_read<T>(a.pre, g * a.p_batch + r * a.ldp + c, left), a.act);
            total.v[0] += v.v[0];
            total.v[1] += v.v[1];
            if (a.dz) row_write<T>(a.dz, g * a.dz_batch + r * a.dz_ld + c, left, v);
            if (a.plain) write8<T>(a.plain, g * a.plain_batch + r * a.plain_ld + c, v);
        }
    if (!a.col_sums) return;
    float *mine = &sums[threadIdx.x >> 5][(threadIdx.x & 31) * 8];
    *reinterpret_cast<v4f *>(mine) = total.v[0];
    *reinterpret_cast<v4f *>(mine + 4) = total.v[1];
    __syncthreads();
    const int t = threadIdx.x;
    if (c0 + t >= a.C) return;
    float s = sums[0][t];
#pragma unroll
    for (int i = 1; i < 8; ++i) s += sums[i][t];
    a.col_sums[(g * tiles_r + tr) * a.C + c0 + t] = s;
}

// ---------------------------------------------------------------------------------------
// f32 sources, taken apart.
// ---------------------------------------------------------------------------------------
// The two f16 numbers of a value that its row's exponent has scaled.  An infinity is +-1 and, trailing, itself: of the three products with another
// value's two numbers that leaves the infinity that is due, also with another infinity, and NaN where the other's leading number is 0.
__device__ __forceinline__ void take_apart(float v, uint16_t &lead, uint16_t &trail)
{
    const _Float16 h = static_cast<_Float16>(v);
    const float f = static_cast<float>(h);
    const bool finite = fabsf(f) <= 65504.0f;
    const _Float16 l = finite ? static_cast<_Float16>(v - f) : h;
    lead = __builtin_bit_cast(uint16_t, finite ? h : static_cast<_Float16>(copysignf(1.0f, v)));
    trail = __builtin_bit_cast(uint16_t, l);
}

typedef uint32_t v4u __attribute__((ext_vector_type(4)));

// Eight values at place k of a packed row.
__device__ __forceinline__ void write_apart(uint16_t *row, int k, int exponent, const Eight &v)
{
    uint16_t w[8], t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) take_apart(ldexpf(v.v[i >> 2][i & 3], -exponent), w[i], t[i]);
    uint16_t *to = row + (k >> 5) * 64 + (k & 31);
    *reinterpret_cast<v4u *>(to) = __builtin_bit_cast(v4u, w);
    *reinterpret_cast<v4u *>(to + 32) = __builtin_bit_cast(v4u, t);
}

// The bits of a finite value's magnitude, which compare as integers.  Infinities and NaN have no part in their row's exponent.
__device__ __forceinline__ uint32_t magnitude(float v)
{
    const uint32_t m = __float_as_uint(v) & 0x7fffffffu;
    return m < 0x7f800000u ? m : 0u;
}

__device__ __forceinline__ uint32_t magnitude(const Eight &v)
{
    uint32_t m = 0;
#pragma unroll
    for (int c = 0; c < 8; ++c) m = max(m, magnitude(v.v[c >> 2][c & 3]));
    return m;
}

// Rows of up to 512 N values, a wave each, which holds its row in registers: read once, its largest magnitude found, taken apart and written
// once.
template <int N>
__global__ __launch_bounds__(256) void rows_kernel(LaySet set)
{
    int id = block_number();
    if (id >= set.first[set.n]) return;
    const LayArgs &a = source_of(set, id);
    const int64_t row = static_cast<int64_t>(id) * 4 + (threadIdx.x >> 6);
    if (row >= static_cast<int64_t>(a.R) * a.batch) return;
    const int64_t g = row / a.R, r = row - g * a.R;
    const int lane = threadIdx.x & 63, width = static_cast<int>(a.plain_ld / 2);
    const int64_t from = g * a.batch_stride + r * a.ld;
    Eight v[N];
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = (i * 64 + lane) * 8;
        v[i] = row_read<kF32>(a.src, from + c, a.C - c);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) most = max(most, magnitude(v[i]));
#pragma unroll
    for (int d = 32; d; d >>= 1) most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), d)));
    if (lane == 0) a.row_max[g * a.R + r] = most;
    uint16_t *to = a.plain + g * a.plain_batch + r * a.plain_ld;
    const int e = row_exponent(most);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = (i * 64 + lane) * 8;
        if (c < width) write_apart(to, c, e, v[i]);
    }
}

// A tile of kT x kT values in LDS, from a workgroup of 256: 8 columns a thread.
__device__ __forceinline__ void read_tile(const LayArgs &a, int64_t g, int r0, int c0, float (*tile)[kT + 1], bool copy)
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = i * 32 + static_cast<int>(threadIdx.x >> 3), c = static_cast<int>(threadIdx.x & 7) * 8;
        const int left = r0 + r < a.R ? a.C - c0 - c : 0;
        Eight v = row_read<kF32>(a.src, g * a.batch_stride + (r0 + r) * a.ld + c0 + c, left);
        if (a.act) v = slope8(v, row_read<kF32>(a.pre, g * a.p_batch + (r0 + r) * a.ldp + c0 + c, left), a.act);
        if (copy && a.dz) row_write<kF32>(a.dz, g * a.dz_batch + (r0 + r) * a.dz_ld + c0 + c, left, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) tile[r][c + k] = v.v[k >> 2][k & 3];
    }
    __syncthreads();
}

// Largest magnitudes of rows and columns, and sums of columns over the tile's rows.  A maximum does not depend on the order of the atomics.
__global__ __launch_bounds__(256) void stats_kernel(LaySet set)
{
    int id = block_number();
    if (id >= set.first[set.n]) return;
    const LayArgs &a = source_of(set, id);
    __shared__ float tile[kT][kT + 1];
    const int tiles_c = (a.C + kT - 1) / kT, tiles_r = (a.R + kT - 1) / kT;
    const int64_t g = id / (tiles_c * tiles_r);
    id -= static_cast<int>(g) * tiles_c * tiles_r;
    const int tr = id / tiles_c, r0 = tr * kT, c0 = id % tiles_c * kT;
    read_tile(a, g, r0, c0, tile, false);
    // four threads for a row (column): 16 values each
    const int line = threadIdx.x >> 2, part = (threadIdx.x & 3) * 16;
    if (a.row_max) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) m = max(m, magnitude(tile[line][part + i]));
        m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 1)));
        m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 2)));
        if (part == 0 && r0 + line < a.R && m) atomicMax(a.row_max + g * a.R + r0 + line, m);
    }
    if (a.col_max || a.col_sums) {
        uint32_t m = 0;
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float v = tile[part + i][line];
            m = max(m, magnitude(v));
            s += v;
        }
        m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 1)));
        m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 2)));
        s += __shfl_xor(s, 1);
        s += __shfl_xor(s, 2);
        if (part == 0 && c0 + line < a.C) {
            if (a.col_max && m) atomicMax(a.col_max + g * a.C + c0 + line, m);
            if (a.col_sums) a.col_sums[(g * tiles_r + tr) * a.C + c0 + line] = s;
        }
    }
}

// The copies along rows and along columns from one reading.
__global__ __launch_bounds__(256) void lay_kernel(LaySet set)
{
    int id = block_number();
    if (id >= set.first[set.n]) return;
    const LayArgs &a = source_of(set, id);
    __shared__ float tile[kT][kT + 1];
    const int tiles_c = (a.C + kT - 1) / kT, tiles_r = (a.R + kT - 1) / kT;
    const int64_t g = id / (tiles_c * tiles_r);
    id -= static_cast<int>(g) * tiles_c * tiles_r;
    const int r0 = id / tiles_c * kT, c0 = id % tiles_c * kT;
    read_tile(a, g, r0, c0, tile, true);
    if (a.plain)
#pragma unroll
        for (int j = threadIdx.x; j < kT * 8; j += 256) {
            const int r = j >> 3, c = (j & 7) * 8;
            if (r0 + r >= a.R || c0 + c >= static_cast<int>(a.plain_ld / 2)) continue;
            Eight v;
#pragma unroll
            for (int k = 0; k < 8; ++k) v.v[k >> 2][k & 3] = tile[r][c + k];
            write_apart(a.plain + g * a.plain_batch + static_cast<int64_t>(r0 + r) * a.plain_ld, c0 + c, row_exponent(a.row_max[g * a.R + r0 + r]), v);
        }
    if (a.trans)
#pragma unroll
        for (int j = threadIdx.x; j < kT * 8; j += 256) {
            const int c = j >> 3, r = (j & 7) * 8;         // 8 threads follow a packed row
            if (c0 + c >= a.C || r0 + r >= static_cast<int>(a.trans_ld / 2)) continue;
            Eight v;
#pragma unroll
            for (int k = 0; k < 8; ++k) v.v[k >> 2][k & 3] = tile[r + k][c];
            write_apart(a.trans + g * a.trans_batch + static_cast<int64_t>(c0 + c) * a.trans_ld, r0 + r, row_exponent(a.col_max[g * a.C + c0 + c]), v);
        }
}

// 64 columns a workgroup, whose four waves take every fourth tile's sums.
__global__ __launch_bounds__(256) void column_sums_kernel(SumArgs a)
{
    __shared__ float part[4][64];
    const int blocks = (a.C + 63) / 64, wave = threadIdx.x >> 6, g = block_number() / blocks, c = (block_number() - g * blocks) * 64 + static_cast<int>(threadIdx.x & 63);
    if (g >= a.batch) return;
    const float *from = a.sums + static_cast<int64_t>(g) * a.tiles * a.C + min(c, a.C - 1);
    float s = 0.0f;
#pragma unroll 8
    for (int t = wave; t < a.tiles; t += 4) s += from[static_cast<int64_t>(t) * a.C];
    part[wave][threadIdx.x & 63] = s;
    __syncthreads();
    if (wave != 0 || c >= a.C) return;
    const int i = threadIdx.x;
    s = (part[0][i] + part[1][i]) + (part[2][i] + part[3][i]);
    if (a.factor) s *= a.factor[g];
    if (a.accumulate) s += load_one(a.out, g * a.out_batch + c, a.type);
    store_one(a.out, g * a.out_batch + c, a.type, s);
}

__global__ __launch_bounds__(256) void zero_kernel(uint32_t *p, int64_t words)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (i < words) p[i] = 0u;
}

dim3 grid_of(int64_t blocks)
{
    const int64_t across = blocks < kGridRow ? blocks : kGridRow;
    return dim3(static_cast<unsigned>(across), static_cast<unsigned>((blocks + across - 1) / across));
}

int64_t tiles_over(int64_t rows, int64_t columns, int64_t wide, int64_t batch) { return (columns + wide - 1) / wide * ((rows + kT - 1) / kT) * batch; }

// One launch over the workgroups of all sources; blocks_of(l): how many l takes.
template <class BlocksOf>
int launch_set(void (*fn)(LaySet), const LaySet &set, BlocksOf blocks_of, const char *what, hipStream_t stream)
{
    LaySet s{};
    int64_t blocks = 0;
    for (int i = 0; i < set.n; ++i) {
        const int64_t n = blocks_of(set.a[i]);
        if (n <= 0) continue;
        s.first[s.n] = static_cast<int32_t>(blocks);
        s.add(set.a[i]);
        blocks += n;
    }
    if (blocks <= 0) return GBMUF_OK;
    if (blocks > 0x7fffffffLL - kGridRow) return GBMUF_EUNSUPPORTED;
    s.first[s.n] = static_cast<int32_t>(blocks);
    void *argv[] = {&s};
    const hipError_t err = hipLaunchKernel(reinterpret_cast<const void *>(fn), grid_of(blocks), dim3(256), argv, 0, stream);
    return err == hipSuccess ? GBMUF_OK : hip_failed(what, err, GBMUF_EDEVICE);
}

}  // namespace

int launch_stats(const LaySet &set, hipStream_t stream)
{
    return launch_set(stats_kernel, set, [](const LayArgs &a) { return tiles_over(a.R, a.C, kT, a.batch); }, "hipLaunchKernel(stats)", stream);
}

int launch_lay(const LaySet &set, hipStream_t stream)
{
    return launch_set(lay_kernel, set, [](const LayArgs &a) { return tiles_over(a.R, a.C, kT, a.batch); }, "hipLaunchKernel(lay out)", stream);
}

int launch_rows(const LaySet &set, hipStream_t stream)
{
    int32_t longest = 0;
    for (int i = 0; i < set.n; ++i) longest = set.a[i].C > longest ? set.a[i].C : longest;
    return launch_set(longest <= 1024 ? rows_kernel<2> : longest <= 2048 ? rows_kernel<4> : rows_kernel<8>, set,
                      [](const LayArgs &a) { return (static_cast<int64_t>(a.R) * a.batch + 3) / 4; }, "hipLaunchKernel(rows)", stream);
}

int launch_copy(const LaySet &set, hipStream_t stream)
{
    if (set.n == 0) return GBMUF_OK;
    return launch_set(set.a[0].type == kBf16 ? copy_kernel<kBf16> : copy_kernel<kF16>, set,
                      [](const LayArgs &a) { return tiles_over(a.R, a.plain ? a.plain_ld : a.C, 256, a.batch); }, "hipLaunchKernel(copy)", stream);
}

int launch_column_sums(const SumArgs &a, hipStream_t stream)
{
    const int64_t blocks = static_cast<int64_t>((a.C + 63) / 64) * a.batch;
    if (blocks <= 0) return GBMUF_OK;
    if (blocks > 0x7fffffffLL - kGridRow) return GBMUF_EUNSUPPORTED;
    SumArgs args = a;
    void *argv[] = {&args};
    const hipError_t err = hipLaunchKernel(reinterpret_cast<const void *>(column_sums_kernel), grid_of(blocks), dim3(256), argv, 0, stream);
    return err == hipSuccess ? GBMUF_OK : hip_failed("hipLaunchKernel(column sums)", err, GBMUF_EDEVICE);
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
