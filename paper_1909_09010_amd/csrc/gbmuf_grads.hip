// gbmuf_grads.hip -- the gradients of K workers: norms, clipping, and the local update of Algorithm 1.
#include "gbmuf_device.h"
#include "gbmuf_values.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

namespace gbmuf {
namespace {

struct GradTensor {              // on the device
    char *p;
    int64_t cols, ld;            // ld == cols where rows follow each other
    int64_t offset;              // of the first value among the worker's parameters
    int32_t worker, type;
    int64_t rows;
};

// One workgroup's share: values [start, start + n) of a tensor, counted row by row.  The tensor's own description is in it: what a workgroup waits
// for before its first load is one load from this list.
struct GradTile {
    GradTensor t;
    int64_t start;
    int32_t n, tensor;
};
static_assert(sizeof(GradTile) == 64, "half a cache line");

// Workgroups take 16 KB each, 4096 values of f32 or 8192 of 16-bit numbers: all loads are under way before the first value is used.  Clipping, Adagrad's
// step of 16 x 19.8 M f32, us: tiles of 1 K 843, 1592; 2 K 712, 1527; 4 K 674, 1503; 8 K 692, 1510; 32 K 709, 1515.  The norm of 16 x 19.8 M bf16: 4 K 130,
// 8 K 115.  Handles that make less than 1024 workgroups take half as much, down to 1024 values, as long as no worker has more tiles than a workgroup has
// threads, which lets the kernel after the norm join its sums: the step of 4 x 100,000 bf16, clipped, 12.6 with 8 K, 7.1 with 1 K, 7.7 with 512.
// Above what the caches hold bound by HBM, and by how its pages are met: accesses are streamed, which keeps neighbours together on their way, and a CU holds few workgroups at a
// time, by LDS that they declare and do not use, so that what is in flight is one short moving range.  us, the norm, clipping in place and Adagrad's step
// with it in blocks, 16 x 19.8 M f32: plain accesses 209, 682, 1505; streamed 189, 620, 1401; and 6, 3, 3 workgroups a CU 183, 585, 1385 (4 for all 190, 592,
// 1402; 3 for all 235, 626, 1425).  The norm reads 6.9 TB/s, clipping moves 6.5, the step alone 5.3.
// Which of the two goes by the bytes that a call's arrays cover.  us plain / streamed: clipping into others 16 x 2 M f32 and 16 x 4 M bf16 (244 MB) 60 / 64 and 61 / 64,
// 16 x 3 M and 16 x 6 M (366 MB) 94 / 91 and 95 / 91; in place 16 x 4 M f32 and 16 x 8 M bf16 (244 MB) 117 / 122 and 116 / 121, 16 x 6 M and 16 x 12 M (366 MB) 184 / 179 and
// 183 / 179; Adagrad in rows 16 x 1.5 M f32 (275 MB) 94 / 100, 16 x 2 M bf16 (305 MB) 112 / 120, 16 x 2 M f32 (366 MB) 137 / 131, 16 x 3 M bf16 (458 MB) 182 / 168; SGD
// 16 x 2 M f32 (244 MB) 83 / 88, 16 x 3 M (366 MB) 131 / 127, bf16 (366 MB) 134 / 140, 16 x 6 M bf16 (549 MB) 212 / 204.  The norm alone, which leaves
// nothing to find: 8 x 2 M bf16 (31 MB) 7.5 / 7.9, 16 x 1.5 M bf16 (46 MB) 11.7 / 10.3, 8 x 2 M f32 (61 MB) 13.3 / 12.0.  (MB of 2^20.)
constexpr int kThreads = 256, kTile = 4096, kJoinThreads = 1024;
constexpr int64_t kCached = 320 << 20, kReadOnce = 40 << 20;       // bytes: of the calls that write, of the norm alone
constexpr int64_t kManyTiles = 1024, kLeastTile = 1024;            // workgroups, values
constexpr int kSixPerCu = 24 * 128, kThreePerCu = 50 * 128;        // doubles of LDS

__device__ __forceinline__ int64_t grad_at(const GradTensor &t, int64_t i)
{
    if (t.ld == t.cols) return i;
    const int64_t r = i / t.cols;
    return i + r * (t.ld - t.cols);
}

// V values side by side: 16 bytes of f32 or of 16-bit numbers an instruction and lane, so that a wave's cover whole lines.
template <int V>
struct Some {
    float v[V];
};

template <int T, int V>
struct Piece {                   // at any address that the type allows
    typedef typename Num<T>::type type __attribute__((ext_vector_type(V), aligned(sizeof(typename Num<T>::type))));
};

template <bool S, int T, int V>
__device__ __forceinline__ Some<V> read_some(const void *p, int64_t i)
{
    const auto at = reinterpret_cast<const typename Piece<T, V>::type *>(static_cast<const typename Num<T>::type *>(p) + i);
    const typename Piece<T, V>::type x = S ? __builtin_nontemporal_load(at) : *at;
    Some<V> r;
#pragma unroll
    for (int c = 0; c < V; ++c) r.v[c] = static_cast<float>(x[c]);
    return r;
}

template <bool S, int T, int V>
__device__ __forceinline__ void write_some(void *p, int64_t i, const Some<V> &r)
{
    const auto at = reinterpret_cast<typename Piece<T, V>::type *>(static_cast<typename Num<T>::type *>(p) + i);
    typename Piece<T, V>::type x;
#pragma unroll
    for (int c = 0; c < V; ++c) x[c] = static_cast<typename Num<T>::type>(r.v[c]);
    if constexpr (S) __builtin_nontemporal_store(x, at);
    else *at = x;
}

// The tile's values, V at a time that lie side by side in the tensor: U times V are loaded, load(i), before the first are used, use(i, what was
// loaded); one(i) for single values.
template <int V, int U, class Load, class Use, class One>
__device__ __forceinline__ void each(const GradTile &tile, Load load, Use use, One one)
{
    const GradTensor &t = tile.t;
    constexpr int kAll = kThreads * V;
    if (t.ld == t.cols) {
        int32_t k = static_cast<int32_t>(threadIdx.x) * V;
        for (; k + (U - 1) * kAll + V <= tile.n; k += U * kAll) {
            decltype(load(tile.start)) v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = load(tile.start + k + u * kAll);
#pragma unroll
            for (int u = 0; u < U; ++u) use(tile.start + k + u * kAll, v[u]);
        }
        for (; k < tile.n; k += kAll) {
            if (k + V <= tile.n) use(tile.start + k, load(tile.start + k));
            else
                for (int32_t c = k; c < tile.n; ++c) one(tile.start + c);
        }
        return;
    }
    for (int32_t k = static_cast<int32_t>(threadIdx.x) * V; k < tile.n; k += kAll) {
        const int64_t i = tile.start + k;
        if (k + V <= tile.n && i % t.cols + V <= t.cols) use(i, load(i));
        else
            for (int32_t c = k; c < min(k + V, tile.n); ++c) one(tile.start + c);
    }
}

// The sum over a workgroup of THREADS, four waves at a time: more waves of zeros do not change it.
template <int THREADS>
__device__ __forceinline__ double block_sum(double s, double *lds)
{
    for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int i = 0; i < THREADS / 64; i += 4) s += (lds[i] + lds[i + 1]) + (lds[i + 2] + lds[i + 3]);
    return s;
}

template <bool S, int T>
__device__ __forceinline__ double tile_squares(const GradTile &tile)
{
    const GradTensor &t = tile.t;
    double s = 0.0;
    const auto add = [&](float v) { s = fma(static_cast<double>(v), static_cast<double>(v), s); };
    constexpr int V = T == kF32 ? 4 : 8;
    each<V, 4>(tile, [&](int64_t i) { return read_some<S, T, V>(t.p, grad_at(t, i)); },
            [&](int64_t, const Some<V> &v) {
#pragma unroll
                for (int c = 0; c < V; ++c) add(v.v[c]);
            },
            [&](int64_t i) { add(load_one(t.p, grad_at(t, i), T)); });
    return s;
}

template <bool S>
__global__ __launch_bounds__(kThreads) void norm_kernel(const GradTile *tiles, double *partial)
{
    __shared__ double lds[S ? kSixPerCu : 4];
    const GradTile tile = tiles[blockIdx.x];
    double s = tile.t.type == kF32 ? tile_squares<S, kF32>(tile) : tile.t.type == kBf16 ? tile_squares<S, kBf16>(tile) : tile_squares<S, kF16>(tile);
    s = block_sum<kThreads>(s, lds);
    if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

// A worker's norm from its tiles' sums, by a whole workgroup.
template <int THREADS>
__device__ __forceinline__ float join_norm(const double *partial, const int32_t *first, int32_t worker, double *lds)
{
    double s = 0.0;
    const int32_t end = first[worker + 1];
#pragma unroll 8
    for (int32_t i = first[worker] + static_cast<int32_t>(threadIdx.x); i < end; i += THREADS) s += partial[i];
    return static_cast<float>(sqrt(block_sum<THREADS>(s, lds)));
}

__global__ __launch_bounds__(kJoinThreads) void norm_join_kernel(const double *partial, const int32_t *first, float *norms)
{
    __shared__ double lds[kJoinThreads / 64];
    const float norm = join_norm<kJoinThreads>(partial, first, static_cast<int32_t>(blockIdx.x), lds);
    if (threadIdx.x == 0) norms[blockIdx.x] = norm;
}

// Where the norms are for the kernel after: joined already (partial nullptr), or to be joined by every workgroup for itself, which saves a
// launch where a worker has few tiles; that of the worker's first tile writes it.
struct Norms {
    float *norms;
    const double *partial;
    const int32_t *first;
};

__device__ __forceinline__ float norm_of(const Norms &n, int32_t worker, int32_t tile, double *lds)
{
    if (!n.partial) return n.norms[worker];
    const float norm = join_norm<kThreads>(n.partial, n.first, worker, lds);
    if (threadIdx.x == 0 && tile == n.first[worker]) n.norms[worker] = norm;
    return norm;
}

__device__ __forceinline__ float clip_factor(float norm, float most) { return norm <= most || most == INFINITY ? 1.0f : most / norm; }

// A product rounded to f32, whatever follows: without the barrier a product that f16 takes one by one becomes v_fma_mixlo_f16, which rounds the exact
// product once, to other bits than those of the values taken side by side, and makes +0 of -0.
__device__ __forceinline__ float times(float v, float f)
{
    float p = v * f;
    asm("" : "+v"(p));
    return p;
}

template <bool S, int T, int D>
__device__ __forceinline__ void clip_tile(const GradTile &tile, const GradTensor &d, float f)
{
    const GradTensor &t = tile.t;
    constexpr int V = T == kF32 || D == kF32 ? 4 : 8;
    each<V, 4>(tile, [&](int64_t i) { return read_some<S, T, V>(t.p, grad_at(t, i)); },
            [&](int64_t i, Some<V> v) {
#pragma unroll
                for (int c = 0; c < V; ++c) v.v[c] = times(v.v[c], f);
                if (d.ld == d.cols || i % d.cols + V <= d.cols) write_some<S, D, V>(d.p, grad_at(d, i), v);
                else
#pragma unroll
                    for (int c = 0; c < V; ++c) store_one(d.p, grad_at(d, i + c), D, v.v[c]);
            },
            [&](int64_t i) { store_one(d.p, grad_at(d, i), D, times(load_one(t.p, grad_at(t, i), T), f)); });
}

template <bool S, int T>
__device__ __forceinline__ void clip_to(const GradTile &tile, const GradTensor &d, float f)
{
    if (d.type == kF32) clip_tile<S, T, kF32>(tile, d, f);
    else if (d.type == kBf16) clip_tile<S, T, kBf16>(tile, d, f);
    else clip_tile<S, T, kF16>(tile, d, f);
}

// Tiles are taken from the last to the first: what the norm read last is still in the caches.
template <bool S>
__global__ __launch_bounds__(kThreads) void clip_kernel(const GradTile *tiles, const GradTensor *to, Norms norms, float most, int32_t in_place)
{
    __shared__ double lds[S ? kThreePerCu : 4];
    const int32_t number = static_cast<int32_t>(gridDim.x - 1 - blockIdx.x);
    const GradTile tile = tiles[number];
    const GradTensor d = to[tile.tensor];
    const float f = clip_factor(norm_of(norms, tile.t.worker, number, lds), most);
    if (in_place && f == 1.0f) return;                     // nothing changes
    if (tile.t.type == kF32) clip_to<S, kF32>(tile, d, f);
    else if (tile.t.type == kBf16) clip_to<S, kBf16>(tile, d, f);
    else clip_to<S, kF16>(tile, d, f);
}

struct StepArgs {
    const GradTile *tiles;
    Norms norms;                 // norms.norms nullptr: no clipping
    float *theta, *sums;         // sums nullptr: SGD
    Placement at, sums_at;
    float rate, eps, most;
    int32_t skip_nonfinite;
};

// The update rounds every multiply and add by itself, like the rest of the method.
__device__ __forceinline__ void update(float &theta, float &h, float g, const StepArgs &a)
{
    if (a.sums) {
        h = h + g * g;
        theta = theta - a.rate * g / (sqrtf(h) + a.eps);
    } else {
        theta = theta - a.rate * g;
    }
}

struct StepFour {
    Some<4> g, theta, h;
};

template <bool S, int T>
__device__ __forceinline__ void step_tile(const GradTile &tile, float f, const StepArgs &a)
{
    const GradTensor &t = tile.t;
    float *theta = a.theta + t.worker * a.at.stride;
    float *sums = a.sums ? a.sums + t.worker * a.sums_at.stride : nullptr;
    const auto one = [&](int64_t i) {
        const float g = load_one(t.p, grad_at(t, i), T) * f;
        const int64_t e = t.offset + i;
        float *p = theta + placed(a.at, e), *q = sums ? sums + placed(a.sums_at, e) : nullptr;
        float h = q ? *q : 0.0f, v = *p;
        update(v, h, g, a);
        *p = v;
        if (q) *q = h;
    };
    // four parameters that a block's edge parts are taken one by one
    const auto together = [&](int64_t e) { return ((e ^ (e + 3)) >> a.at.logB) == 0 && (!sums || ((e ^ (e + 3)) >> a.sums_at.logB) == 0); };
    each<4, 4>(tile,
            [&](int64_t i) {
                StepFour s{};
                const int64_t e = t.offset + i;
                if (!together(e)) return s;
                s.g = read_some<S, T, 4>(t.p, grad_at(t, i));
                s.theta = read_some<S, kF32, 4>(theta, placed(a.at, e));
                if (sums) s.h = read_some<S, kF32, 4>(sums, placed(a.sums_at, e));
                return s;
            },
            [&](int64_t i, StepFour s) {
                const int64_t e = t.offset + i;
                if (!together(e)) {
                    for (int c = 0; c < 4; ++c) one(i + c);
                    return;
                }
#pragma unroll
                for (int c = 0; c < 4; ++c) update(s.theta.v[c], s.h.v[c], s.g.v[c] * f, a);
                write_some<S, kF32, 4>(theta, placed(a.at, e), s.theta);
                if (sums) write_some<S, kF32, 4>(sums, placed(a.sums_at, e), s.h);
            },
            one);
}

template <bool S>
__global__ __launch_bounds__(kThreads) void step_kernel(StepArgs a)
{
    __shared__ double lds[S ? kThreePerCu : 4];
    const int32_t number = static_cast<int32_t>(gridDim.x - 1 - blockIdx.x);       // as clip_kernel
    const GradTile tile = a.tiles[number];
    float f = 1.0f;
    if (a.norms.norms) {
        const float norm = norm_of(a.norms, tile.t.worker, number, lds);
        if (a.skip_nonfinite && !(norm < INFINITY)) return;
        f = clip_factor(norm, a.most);
    }
    if (tile.t.type == kF32) step_tile<S, kF32>(tile, f, a);
    else if (tile.t.type == kBf16) step_tile<S, kBf16>(tile, f, a);
    else step_tile<S, kF16>(tile, f, a);
}

}  // namespace
}  // namespace gbmuf

using namespace gbmuf;

struct gbmuf_grads_s {
    int32_t workers = 0;
    int device = -1;
    int64_t n_tiles = 0, reach = 0;              // reach: end of the last tensor among a worker's parameters
    int64_t values = 0, bytes = 0;               // of all tensors
    bool few = false;                            // every worker has tiles, one for a thread at most
    std::vector<GradTensor> tensors;             // by worker, in the order of the list
    GradTensor *d_tensors = nullptr;
    GradTile *d_tiles = nullptr;
    int32_t *d_first = nullptr;                  // [workers + 1]: first tile of every worker
    double *d_partial = nullptr;
};

namespace {

void free_grads(gbmuf_grads_s &g)
{
    for (void *p : {static_cast<void *>(g.d_tensors), static_cast<void *>(g.d_tiles), static_cast<void *>(g.d_first), static_cast<void *>(g.d_partial)})
        if (p) (void)hipFree(p);
}

template <class T>
int to_device(T **dst, const T *src, size_t n)
{
    if (n == 0) return GBMUF_OK;
    hipError_t err = hipMalloc(reinterpret_cast<void **>(dst), n * sizeof(T));
    if (err != hipSuccess) return hip_failed("hipMalloc(gradient tables)", err, err == hipErrorOutOfMemory ? GBMUF_ENOMEM : GBMUF_EDEVICE);
    if (!src) return GBMUF_OK;
    err = hipMemcpy(*dst, src, n * sizeof(T), hipMemcpyHostToDevice);
    return err == hipSuccess ? GBMUF_OK : hip_failed("hipMemcpy(gradient tables)", err, GBMUF_EDEVICE);
}

int make_grads(gbmuf_grads_s &h, const gbmuf_grads_desc_t &d)
{
    const size_t n = static_cast<size_t>(d.n_tensors);
    h.workers = d.workers;
    std::vector<int64_t> next(static_cast<size_t>(d.workers), 0);
    std::vector<GradTensor> list(n);
    for (size_t i = 0; i < n; ++i) {
        const gbmuf_grad_tensor_t &t = d.tensors[i];
        if (t.worker < 0 || t.worker >= d.workers || t.dtype < GBMUF_F32 || t.dtype > GBMUF_F16 || t.rows < 0 || t.cols < 0 || t.offset < -1)
            return GBMUF_EINVAL;
        if (t.rows > 1 && t.row_stride < t.cols) return GBMUF_EINVAL;
        if (t.rows > 0 && t.cols > (static_cast<int64_t>(1) << 48) / t.rows) return GBMUF_EUNSUPPORTED;
        if (t.rows > 1 && static_cast<double>(t.rows) * static_cast<double>(t.row_stride) > 0x1p48) return GBMUF_EINVAL;     // no place overflows
        const int64_t count = t.rows * t.cols;
        if (count > 0 && (!t.data || reinterpret_cast<uintptr_t>(t.data) % type_bytes(t.dtype) != 0)) return GBMUF_EINVAL;
        int64_t &at = next[static_cast<size_t>(t.worker)];
        const int64_t offset = t.offset < 0 ? at : t.offset;
        if (offset > (static_cast<int64_t>(1) << 48)) return GBMUF_EUNSUPPORTED;
        at = offset + count;
        list[i] = GradTensor{static_cast<char *>(t.data), t.cols, t.rows > 1 ? t.row_stride : t.cols, offset, t.worker, t.dtype, t.rows};
        if (count > 0) h.reach = std::max(h.reach, at);
    }
    std::stable_sort(list.begin(), list.end(), [](const GradTensor &a, const GradTensor &b) { return a.worker < b.worker; });
    h.tensors = list;
    std::sort(list.begin(), list.end(), [](const GradTensor &a, const GradTensor &b) { return a.worker != b.worker ? a.worker < b.worker : a.offset < b.offset; });
    const GradTensor *before = nullptr;                    // places of one worker's tensors are apart
    for (const GradTensor &t : list) {
        if (t.rows * t.cols == 0) continue;
        if (before && before->worker == t.worker && before->offset + before->rows * before->cols > t.offset) return GBMUF_EINVAL;
        before = &t;
    }
    int64_t size = 2 * kTile;                              // one size for a handle: f32 anywhere in it takes the smaller
    for (const GradTensor &t : h.tensors) {
        if (t.type == kF32) size = kTile;
        h.values += t.rows * t.cols;
        h.bytes += t.rows * t.cols * static_cast<int64_t>(type_bytes(t.type));
    }
    int64_t most = 0;                                      // of one worker
    const auto count_tiles = [&](int64_t of) {
        int64_t all = 0;
        std::fill(next.begin(), next.end(), 0);
        for (const GradTensor &t : h.tensors) {
            const int64_t n = (t.rows * t.cols + of - 1) / of;
            all += n;
            next[static_cast<size_t>(t.worker)] += n;
        }
        most = *std::max_element(next.begin(), next.end());
        return all;
    };
    while (size > kLeastTile && count_tiles(size) < kManyTiles && count_tiles(size / 2) >= 0 && most <= kThreads) size /= 2;
    std::vector<GradTile> tiles;
    std::vector<int32_t> first(static_cast<size_t>(d.workers) + 1, 0);
    const int64_t count = count_tiles(size);
    if (count > 0x7fffffffLL / kThreads) return GBMUF_EUNSUPPORTED;
    tiles.reserve(static_cast<size_t>(count));
    for (size_t i = 0; i < h.tensors.size(); ++i) {
        const int64_t all = h.tensors[i].rows * h.tensors[i].cols;
        for (int64_t s = 0; s < all; s += size) tiles.push_back(GradTile{h.tensors[i], s, static_cast<int32_t>(std::min(size, all - s)), static_cast<int32_t>(i)});
        first[static_cast<size_t>(h.tensors[i].worker) + 1] = static_cast<int32_t>(tiles.size());
    }
    for (size_t w = 1; w < first.size(); ++w) first[w] = std::max(first[w], first[w - 1]);
    h.n_tiles = count;
    h.few = true;
    for (size_t w = 0; w + 1 < first.size(); ++w) h.few = h.few && first[w + 1] > first[w] && first[w + 1] - first[w] <= kThreads;
    int devices = 0;
    hipError_t err = hipGetDeviceCount(&devices);
    if (err != hipSuccess || devices < 1) return GBMUF_OK;  // host-side checks work without a GPU; the calls say EDEVICE
    if ((err = hipGetDevice(&h.device)) != hipSuccess) return hip_failed("hipGetDevice", err, GBMUF_EDEVICE);
    int rc = to_device(&h.d_tensors, h.tensors.data(), h.tensors.size());
    if (rc == GBMUF_OK) rc = to_device(&h.d_tiles, tiles.data(), tiles.size());
    if (rc == GBMUF_OK) rc = to_device(&h.d_first, first.data(), first.size());
    if (rc == GBMUF_OK) rc = to_device<double>(&h.d_partial, nullptr, tiles.size());
    return rc;
}

int check_grads_device(const gbmuf_grads_s *g)
{
    if (g->device < 0) return hip_failed("no GPU when the handle was made", hipErrorNoDevice, GBMUF_EDEVICE);
    int now = -1;
    const hipError_t err = hipGetDevice(&now);
    if (err != hipSuccess) return hip_failed("hipGetDevice", err, GBMUF_EDEVICE);
    return now == g->device ? GBMUF_OK : hip_failed("another GPU than the handle's is current", hipErrorInvalidDevice, GBMUF_EDEVICE);
}

int launch(const void *fn, int64_t blocks, void **argv, const char *what, hipStream_t stream, int threads = kThreads)
{
    if (blocks <= 0) return GBMUF_OK;
    const hipError_t err = hipLaunchKernel(fn, dim3(static_cast<unsigned>(blocks)), dim3(static_cast<unsigned>(threads)), argv, 0, stream);
    return err == hipSuccess ? GBMUF_OK : hip_failed(what, err, GBMUF_EDEVICE);
}

// The tiles' sums, and the norms unless the kernel after this one joins them (joined not nullptr).
int enqueue_norm(const gbmuf_grads_s *g, float *norms, Norms *joined, bool streamed, hipStream_t stream)
{
    const GradTile *tiles = g->d_tiles;
    double *partial = g->d_partial;
    const int32_t *first = g->d_first;
    void *a1[] = {&tiles, &partial}, *a2[] = {&partial, &first, &norms};
    const int rc = launch(reinterpret_cast<const void *>(streamed ? norm_kernel<true> : norm_kernel<false>), g->n_tiles, a1, "hipLaunchKernel(norm)", stream);
    if (rc != GBMUF_OK) return rc;
    if (joined) *joined = Norms{norms, g->few ? partial : nullptr, first};
    if (joined && g->few) return GBMUF_OK;
    return launch(reinterpret_cast<const void *>(norm_join_kernel), g->workers, a2, "hipLaunchKernel(norm join)", stream, kJoinThreads);
}

// Where the arrays of a step lie.
int place(const gbmuf_state_t &s, int64_t K, int64_t P, Placement *at, int64_t *extent)
{
    if (reinterpret_cast<uintptr_t>(s.theta) % 4 != 0) return GBMUF_EINVAL;
    const int64_t B = s.block_floats;
    constexpr int64_t kMost = static_cast<int64_t>(1) << 48;       // floats: what any memory holds, and no product below overflows
    if (P > kMost || s.worker_stride > kMost || s.block_stride > kMost) return GBMUF_EINVAL;
    if (B > 0 && static_cast<double>(P) / static_cast<double>(B) * static_cast<double>(s.block_stride) > static_cast<double>(kMost)) return GBMUF_EINVAL;
    if (B == 0) {
        if (s.worker_stride < P) return GBMUF_EINVAL;
        *at = Placement{s.worker_stride, 0, 62, 0};
        *extent = (K - 1) * s.worker_stride + P;
        return GBMUF_OK;
    }
    if (B < 4 || (B & (B - 1)) != 0 || B > (static_cast<int64_t>(1) << 30) || s.worker_stride < B) return GBMUF_EINVAL;
    if (s.block_stride < (K - 1) * s.worker_stride + B) return GBMUF_EINVAL;
    int32_t lg = 0;
    while ((static_cast<int64_t>(1) << lg) < B) ++lg;
    *at = Placement{s.worker_stride, s.block_stride - B, lg, 0};
    const int64_t blocks = (P + B - 1) / B;
    *extent = blocks > 0 ? (blocks - 1) * s.block_stride + (K - 1) * s.worker_stride + B : 0;
    return GBMUF_OK;
}

// Whether rows (blocks) of two placements of the same kind lie side by side, or their ranges apart.
bool apart(const gbmuf_state_t &a, int64_t extent_a, const gbmuf_state_t &b, int64_t extent_b, int64_t K, int64_t P)
{
    const float *x = a.theta, *y = b.theta;
    if (x + extent_a <= y || y + extent_b <= x) return true;
    if (a.block_floats != b.block_floats || a.worker_stride != b.worker_stride || a.block_stride != b.block_stride) return false;
    const int64_t d = x < y ? y - x : x - y;               // equal strides: pieces repeat alike
    const int64_t piece = a.block_floats ? a.block_floats : P;
    const auto inside = [&](int64_t len, int64_t step) { return step > 0 && d % step >= len && d % step + len <= step; };
    if (a.block_floats) return inside((K - 1) * a.worker_stride + piece, a.block_stride) ||
                               (inside(piece, a.worker_stride) && a.block_stride % a.worker_stride == 0);
    return inside(piece, a.worker_stride);
}

}  // namespace

extern "C" {

int gbmuf_grads_create(gbmuf_grads_t **out, const gbmuf_grads_desc_t *desc)
{
    if (!out) return GBMUF_EINVAL;
    *out = nullptr;
    if (!desc || desc->struct_size < sizeof(gbmuf_grads_desc_t) || desc->workers < 1 || desc->n_tensors < 0) return GBMUF_EINVAL;
    if (desc->n_tensors > 0 && !desc->tensors) return GBMUF_EINVAL;
    if (desc->workers > GBMUF_MAX_K || desc->n_tensors > 0x7fffffffLL) return GBMUF_EUNSUPPORTED;
    gbmuf_grads_s *h = new (std::nothrow) gbmuf_grads_s;
    if (!h) return GBMUF_ENOMEM;
    int rc = GBMUF_OK;
    try {
        rc = make_grads(*h, *desc);
    } catch (const std::bad_alloc &) {
        rc = GBMUF_ENOMEM;
    } catch (const std::length_error &) {
        rc = GBMUF_ENOMEM;
    }
    if (rc != GBMUF_OK) {
        free_grads(*h);
        delete h;
        return rc;
    }
    *out = h;
    return GBMUF_OK;
}

int gbmuf_grads_destroy(gbmuf_grads_t *grads)
{
    if (!grads) return GBMUF_OK;
    int rc = GBMUF_OK;
    if (grads->device >= 0) {
        if (hipDeviceSynchronize() != hipSuccess) rc = GBMUF_EDEVICE;
        free_grads(*grads);
    }
    delete grads;
    return rc;
}

int gbmuf_grad_norm(const gbmuf_grads_t *grads, float *norms, void *stream)
{
    if (!grads || !norms) return GBMUF_EINVAL;
    const int rc = check_grads_device(grads);
    return rc != GBMUF_OK ? rc : enqueue_norm(grads, norms, nullptr, grads->bytes > kReadOnce, static_cast<hipStream_t>(stream));
}

int gbmuf_grad_clip(const gbmuf_grads_t *src, const gbmuf_grads_t *dst, float max_norm, float *norms, void *stream)
{
    if (!src || !dst || !norms || !(max_norm >= 0.0f)) return GBMUF_EINVAL;
    if (src != dst) {
        if (src->workers != dst->workers || src->tensors.size() != dst->tensors.size()) return GBMUF_EINVAL;
        for (size_t i = 0; i < src->tensors.size(); ++i) {
            const GradTensor &a = src->tensors[i], &b = dst->tensors[i];
            if (a.worker != b.worker || a.rows * a.cols != b.rows * b.cols) return GBMUF_EINVAL;
        }
    }
    int rc = check_grads_device(src);
    if (rc != GBMUF_OK || (rc = check_grads_device(dst)) != GBMUF_OK) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    Norms n{};
    const bool streamed = src->bytes + (src == dst ? 0 : dst->bytes) > kCached;
    if ((rc = enqueue_norm(src, norms, &n, streamed, s)) != GBMUF_OK) return rc;
    const GradTile *tiles = src->d_tiles;
    const GradTensor *to = dst->d_tensors;
    int32_t in_place = src == dst ? 1 : 0;
    void *argv[] = {&tiles, &to, &n, &max_norm, &in_place};
    return launch(reinterpret_cast<const void *>(streamed ? clip_kernel<true> : clip_kernel<false>), src->n_tiles, argv, "hipLaunchKernel(clip)", s);
}

int gbmuf_local_step(const gbmuf_grads_t *grads, const gbmuf_step_desc_t *desc, const gbmuf_state_t *theta, const gbmuf_state_t *sums, float *norms,
                     void *stream)
{
    if (!grads || !desc || desc->struct_size < sizeof(gbmuf_step_desc_t) || !theta || !theta->theta) return GBMUF_EINVAL;
    if (desc->P < 0 || grads->reach > desc->P) return GBMUF_EINVAL;
    if (desc->rate != desc->rate || !(desc->eps >= 0.0f) || !(desc->max_norm >= 0.0f)) return GBMUF_EINVAL;
    const bool clip = desc->max_norm < INFINITY || desc->skip_nonfinite != 0;
    if (clip && !norms) return GBMUF_EINVAL;
    StepArgs a{};
    int64_t extent = 0, extent_sums = 0;
    int rc = place(*theta, grads->workers, desc->P, &a.at, &extent);
    if (rc != GBMUF_OK) return rc;
    if (sums) {
        if (!sums->theta) return GBMUF_EINVAL;
        if ((rc = place(*sums, grads->workers, desc->P, &a.sums_at, &extent_sums)) != GBMUF_OK) return rc;
        if (!apart(*theta, extent, *sums, extent_sums, grads->workers, desc->P)) return GBMUF_EINVAL;
        a.sums = sums->theta;
    }
    if ((rc = check_grads_device(grads)) != GBMUF_OK) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool streamed = grads->bytes + grads->values * (sums ? 8 : 4) > kCached;
    if (norms && (rc = enqueue_norm(grads, norms, clip ? &a.norms : nullptr, streamed, s)) != GBMUF_OK) return rc;
    a.tiles = grads->d_tiles;
    a.theta = theta->theta;
    a.rate = desc->rate; a.eps = desc->eps; a.most = desc->max_norm; a.skip_nonfinite = desc->skip_nonfinite;
    void *argv[] = {&a};
    return launch(reinterpret_cast<const void *>(streamed ? step_kernel<true> : step_kernel<false>), grads->n_tiles, argv, "hipLaunchKernel(local step)", s);
}

}  // extern "C"
