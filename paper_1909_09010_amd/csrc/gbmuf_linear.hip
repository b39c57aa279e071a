// gbmuf_linear.hip -- entry points of the products with a model's matrices: checks, workspace, and which kernels run.
#include "gbmuf_local.h"

#include "../../include/gbmuf.h"

#include <algorithm>
#include <initializer_list>
#include <numeric>

namespace gbmuf {
namespace {

constexpr int64_t kLargest = 0x7fffffff;
constexpr double kMostTiles = 1 << 21;       // of 128 x 128 results or operands: four of 64 x 64 each are what a grid of 256 threads holds
constexpr int64_t kStepWords = 64;
constexpr int64_t kCached = 128 << 20;        // bytes

// ---------------------------------------------------------------------------------------
// Checks
// ---------------------------------------------------------------------------------------
struct Extent {                  // bytes that a matrix covers
    uintptr_t at = 0;
    int64_t rows = 0, row = 0, ld = 0;           // rows of `row` bytes, ld apart
    int64_t batch = 0, stride = 0;               // matrices, stride apart
    int64_t matrix() const { return (rows - 1) * ld + row; }
    int64_t all() const { return (batch - 1) * stride + matrix(); }
    bool none() const { return at == 0 || rows <= 0 || row <= 0 || batch <= 0; }
};

Extent extent(const gbmuf_matrix_t &m, int64_t rows, int64_t cols, int64_t batch, int32_t type)
{
    const int64_t b = static_cast<int64_t>(type_bytes(type));
    Extent e;
    e.at = reinterpret_cast<uintptr_t>(m.data);
    constexpr int64_t kMost = static_cast<int64_t>(1) << 52;       // more is refused below
    e.rows = rows; e.row = cols * b; e.ld = rows > 1 ? std::min(m.ld, kMost) * b : 0;
    e.batch = batch; e.stride = batch > 1 ? std::min(m.batch_stride, kMost) * b : 0;
    return e;
}

// Pieces of `len` bytes, `step` apart, from a and from b, of which none of a meets one of b: so it is where the pieces of both lie side by
// side in every step.
bool side_by_side(uintptr_t a, int64_t len_a, uintptr_t b, int64_t len_b, int64_t step)
{
    if (step <= 0) return false;
    const int64_t d = b >= a ? static_cast<int64_t>((b - a) % static_cast<uintptr_t>(step))
                             : (step - static_cast<int64_t>((a - b) % static_cast<uintptr_t>(step))) % step;
    return d >= len_a && d + len_b <= step;
}

// Whether two matrices may share bytes.  Apart are: ranges that do not meet; matrices, or else rows, that lie side by side in every
// stretch of a length that divides all steps between them.
bool overlap(const Extent &a, const Extent &b)
{
    if (a.none() || b.none()) return false;
    if (a.at + a.all() <= b.at || b.at + b.all() <= a.at) return false;
    const int64_t matrices = std::gcd(a.stride, b.stride), rows = std::gcd(matrices, std::gcd(a.ld, b.ld));
    return !side_by_side(a.at, a.matrix(), b.at, b.matrix(), matrices) && !side_by_side(a.at, a.row, b.at, b.row, rows);
}

// Nothing spans more than 2^48 elements, and no product of strides and sizes overflows.
bool valid_input(const gbmuf_matrix_t &m, const Extent &e, int32_t type)
{
    if (m.ld < 0 || m.batch_stride < 0) return false;
    if (static_cast<double>(e.rows) * static_cast<double>(e.ld) + static_cast<double>(e.batch) * static_cast<double>(e.stride) > 0x1p48 * 4.0) return false;
    if (e.rows <= 0 || e.row <= 0 || e.batch <= 0) return true;
    return m.data && reinterpret_cast<uintptr_t>(m.data) % type_bytes(type) == 0;
}

// an output's elements are all apart: row after row and matrix after matrix, or the workers' rows inside each row's step
bool valid_output(const gbmuf_matrix_t &m, const Extent &e, int32_t type)
{
    if (!valid_input(m, e, type)) return false;
    if (e.none()) return true;
    const bool rows_apart = e.rows <= 1 || e.ld >= e.row, matrices_apart = e.batch <= 1 || e.stride >= e.matrix();
    const bool inside = e.stride >= e.row && (e.rows <= 1 || e.ld >= (e.batch - 1) * e.stride + e.row);
    return rows_apart && (matrices_apart || inside);
}

bool too_many_tiles(int64_t rows, int64_t cols, int64_t batch)
{
    return static_cast<double>((rows + 127) / 128) * static_cast<double>((cols + 127) / 128) * static_cast<double>(batch) >= kMostTiles;
}

int check_desc(const gbmuf_linear_desc_t *d)
{
    if (!d || d->struct_size < sizeof(gbmuf_linear_desc_t)) return GBMUF_EINVAL;
    if (d->dtype < GBMUF_F32 || d->dtype > GBMUF_F16 || d->activation < GBMUF_ACT_NONE || d->activation > GBMUF_ACT_TANH) return GBMUF_EINVAL;
    if (d->residual < GBMUF_RESIDUAL_NONE || d->residual > GBMUF_RESIDUAL_AFTER) return GBMUF_EINVAL;
    if (d->batch < 0 || d->rows < 0 || d->out_features < 0 || d->in_features < 0) return GBMUF_EINVAL;
    if (d->batch > 65535 || d->rows > kLargest / 2 - 64 || d->out_features > kLargest / 2 - 64 || d->in_features > kLargest / 2 - 64) return GBMUF_EUNSUPPORTED;
    const int64_t M = d->rows, N = d->out_features, K = d->in_features;
    if (too_many_tiles(M, N, d->batch) || too_many_tiles(M, K, d->batch) || too_many_tiles(N, K, d->batch)) return GBMUF_EUNSUPPORTED;
    return GBMUF_OK;
}

// Asked once: a process has a GPU or has none.
int check_device()
{
    static const hipError_t status = [] {
        int n = 0;
        const hipError_t err = hipGetDeviceCount(&n);
        return err == hipSuccess && n < 1 ? hipErrorNoDevice : err;
    }();
    return status == hipSuccess ? GBMUF_OK : hip_failed("hipGetDeviceCount", status, GBMUF_EDEVICE);
}

// ---------------------------------------------------------------------------------------
// Workspace: the same calls count it and hand it out.
// ---------------------------------------------------------------------------------------
struct Space {
    char *base;
    int64_t used = 0;
    template <class T>
    T *take(int64_t n)
    {
        T *p = reinterpret_cast<T *>(base + used);
        used += (n * static_cast<int64_t>(sizeof(T)) + 255) / 256 * 256;
        return p;
    }
};

// One operand of a product: rows of 16-bit words along the axis that is summed over.
struct Operand {
    const uint16_t *p = nullptr;
    int64_t ld = 0, batch = 0;
    uint32_t *max = nullptr;     // split
    int64_t max_batch = 0;
    bool whole = false;          // zeros follow up to the end of the last step
    bool across = false;         // [k][row]
};

bool lies_well(const gbmuf_matrix_t &m)
{
    return reinterpret_cast<uintptr_t>(m.data) % 16 == 0 && m.ld % 8 == 0 && m.batch_stride % 8 == 0;
}

// How a product's tiles go to workgroups: rounds of `slots` workgroups work at a time, and where the last one is far from full, the sums of its
// tiles are cut so that it is, in parts of 8 steps at least.  round: time of a step of a full round.
struct Cut {
    int tile = 0;
    Tiles t{};
    int64_t partial = 0;         // floats
    double cost = 0.0;
};

Cut cut(int tile, int64_t M, int64_t N, int64_t batch, int64_t steps, int64_t slots, double round)
{
    Cut c;
    c.tile = tile;
    c.t.M = static_cast<int32_t>(M); c.t.N = static_cast<int32_t>(N); c.t.batch = static_cast<int32_t>(batch);
    c.t.tiles_m = static_cast<int32_t>((M + tile - 1) / tile);
    c.t.tiles_n = static_cast<int32_t>((N + tile - 1) / tile);
    const int64_t tiles = static_cast<int64_t>(c.t.tiles_m) * c.t.tiles_n * batch, rest = tiles % slots;
    c.t.whole = static_cast<int32_t>(tiles);
    c.t.splits = 1;
    c.t.steps = static_cast<int32_t>(std::max<int64_t>(steps, 1));
    c.cost = static_cast<double>((tiles + slots - 1) / slots * steps) * round;
    const int64_t most = rest > 0 ? std::min<int64_t>({slots / rest, steps / 8, 64}) : 1;
    if (most < 2) return c;
    const int64_t each = (steps + most - 1) / most, splits = (steps + each - 1) / each, partial = rest * splits * tile * tile;
    // another launch, and writing and reading the parts at 4 TB/s
    const double cost = static_cast<double>(tiles / slots * steps + each) * round + 3.0 + static_cast<double>(partial) * 8.0 / 4e6;
    if (cost >= c.cost) return c;
    c.t.whole = static_cast<int32_t>(tiles - rest);
    c.t.splits = static_cast<int32_t>(splits);
    c.t.steps = static_cast<int32_t>(each);
    c.partial = partial;
    c.cost = cost;
    return c;
}

// Tiles of 256 x 256, one a CU, or of 128 x 128, two a CU.  us for a step of a round: 8192 x 8192 x 8192 bf16 take 886 us in 4 rounds of 128
// steps, and 1088 us in 8.  Tiles of 256 / of 128, us, * what is taken, workers x rows x out x in: forward bf16 1 x 2048 x 2048 x 2048 44 / 29*, 1 x 4096 x 4096 x 1024 39* / 46,
// 8 x 700 x 2600 x 656 62 / 47*, 4 x 1024 x 4096 x 1024 38* / 45, 8 x 5120 x 8192 x 512 430* / 498; f32 16 x 512 x 1024 x 512 64 / 52*, 16 x 5120 x 512 x 2048 736* / 754,
// 1 x 5120 x 10000 x 512 222* / 192; gradients bf16 1 x 4096 x 4096 x 1024 126 / 117*, 8 x 700 x 2600 x 656 115 / 97*, 4 x 5120 x 8192 x 1024 739* / 819; f32
// 8 x 1000 x 2048 x 400 226 / 199*.
Cut shape_of(int64_t M, int64_t N, int64_t K, int64_t batch, bool split_type)
{
    const int64_t steps = packed_words(K, split_type) / kStepWords;
    const Cut wide = cut(256, M, N, batch, steps, 256, 1.73), small = cut(128, M, N, batch, steps, 512, 1.06);
    return wide.cost <= small.cost ? wide : small;
}

int run_product(const Operand &a, const Operand &b, int64_t K, int32_t type, const Epilogue &e, const Cut &c, float *partial, hipStream_t stream)
{
    ProductArgs p{};
    p.a = a.p; p.b = b.p; p.lda = a.ld; p.ldb = b.ld; p.a_batch = a.batch; p.b_batch = b.batch;
    p.a_max = a.max; p.b_max = b.max; p.a_max_batch = a.max_batch; p.b_max_batch = b.max_batch;
    p.across = (a.across ? 1 : 0) | (b.across ? 2 : 0);
    p.K = static_cast<int32_t>(a.whole && b.whole && !p.across ? packed_words(K, type == kF32) : K);
    p.t = c.t;
    p.t.partial = partial;
    p.e = e;
    const int rc = launch_product(p, type, c.tile, stream);
    return rc != GBMUF_OK ? rc : launch_join(JoinArgs{p.t, c.tile, 0, e}, stream);
}

LayArgs source(const gbmuf_matrix_t &m, int64_t R, int64_t C, int32_t batch, int32_t type)
{
    LayArgs l{};
    l.src = m.data; l.ld = m.ld; l.batch_stride = m.batch_stride;
    l.R = static_cast<int32_t>(R); l.C = static_cast<int32_t>(C);
    l.batch = m.batch_stride == 0 ? std::min(batch, 1) : batch;        // what workers share is laid out once
    l.type = type;
    return l;
}

// Places of a packed copy of R rows of C values for `batch` workers (l.batch of them are written).
Operand packed(Space &space, int64_t R, int64_t C, int32_t batch, int32_t written, bool split, uint32_t *max)
{
    Operand o;
    o.ld = packed_words(C, split);
    o.p = space.take<uint16_t>(static_cast<int64_t>(batch) * R * o.ld);
    o.batch = written < batch ? 0 : R * o.ld;
    o.max = max;
    o.max_batch = written < batch ? 0 : R;
    o.whole = true;
    return o;
}

// values: of all workers
Epilogue into(const gbmuf_matrix_t &m, int64_t values, int32_t type)
{
    Epilogue e{};
    e.y = m.data; e.ldy = m.ld; e.y_batch = m.batch_stride; e.type = type;
    e.streamed = values * static_cast<int64_t>(type_bytes(type)) > kCached ? 1 : 0;
    return e;
}

// ---------------------------------------------------------------------------------------
// Products straight from where the matrices lie.
// ---------------------------------------------------------------------------------------
Source source_of(const gbmuf_matrix_t &m)
{
    Source s{};
    s.p = m.data; s.ld = m.ld; s.batch = m.batch_stride;
    return s;
}

DirectArgs direct_args(const Source &a, const Source &b, int64_t K, const Cut &c, const Epilogue &e)
{
    DirectArgs d{};
    d.a = a; d.b = b;
    d.K = static_cast<int32_t>(K);
    d.t = c.t;
    d.e = e;
    return d;
}

// Forward, tiles of 64 x 64: the sums are cut (where `may_cut`) where there are fewer tiles than CUs and they are long.  A step is 0.43 us of a CU's f32
// matrix instructions.
Cut direct_cut(int64_t M, int64_t N, int64_t K, int64_t batch, bool may_cut)
{
    const int64_t steps = (K + 31) / 32, tiles = (M + 63) / 64 * ((N + 63) / 64) * batch;
    return cut(64, M, N, batch, steps, may_cut && tiles < 256 ? 256 : std::max<int64_t>(tiles, 1), 0.5);
}

// Gradients: dx's sums are usually the longer ones, and a workgroup that shares its CU with others takes 1.2 us a step or more.  Sums that would last as
// long as the matrix instructions of both products at their rate, or longer, are cut to last half of that (us, f32: 4 x 128 x 2600 x 650, 82 steps of 88 tiles and
// 4 of 1804, 79 in two parts, 65 in four, 62 in eight; 8 x 128 x 2600 x 650 152 whole, 124 in two, 105 in four; 11 x 16 x 28173 x 942, 881 steps of 165 tiles and one
// of 72,765, 1890 in two, 1324 in four; 16 x 128 x 512 x 512, 16 steps of 256 tiles and 4 of 1024, 34 whole, 40 in two), but not into more than 64 parts
// for that (1 x 64 x 200,000 x 64 141 in 64, 87 in 358, 116 in 716).
Cut chain_cut(int64_t M, int64_t N, int64_t K, int64_t batch, const Cut &other)
{
    const int64_t steps = (K + 31) / 32, tiles = (M + 63) / 64 * ((N + 63) / 64) * batch;
    Cut c = cut(64, M, N, batch, steps, std::max<int64_t>(tiles, 1), 0.5);
    const int64_t all = tiles * steps + static_cast<int64_t>(other.t.whole) * other.t.steps;
    int64_t parts = tiles > 0 ? steps * 256 * 14 / (5 * (all + 1)) : 1;
    if (parts >= 2) parts = std::min(steps / 8, std::max(parts, std::min<int64_t>(2 * parts, 64)));
    if (parts < 2) return c;
    const int64_t each = (steps + parts - 1) / parts, splits = (steps + each - 1) / each;
    c.t.whole = 0;
    c.t.splits = static_cast<int32_t>(splits);
    c.t.steps = static_cast<int32_t>(each);
    c.partial = tiles * splits * 64 * 64;
    return c;
}

// Whether f32 arithmetic on the matrices as they lie is faster than laying them out for the 16-bit instructions, which costs launches and passes
// over them.  Both are estimated, in us: as they lie, by the steps of 64 x 64 x 32, of which the chip does 256 in 0.43 at best; laid out, by the launches, the values
// that are laid out and the operations.  As they lie / laid out, workers x rows x out x in:
//   forward f32: 1 x 200 x 1024 x 512 15 / 20, 4 x 200 x 1024 x 512 17 / 28, 8 x 250 x 1500 x 400 30 / 41, 8 x 128 x 2600 x 650 45 / 45 (with tanh and z
//     kept, operands in HBM before the call, 45 / 57), 8 x 250 x 2000 x 400 39 / 35, 4 x 512 x 1024 x 1024 46 / 41, 16 x 512 x 1024 x 512 83 / 51
//   gradients f32: 1 x 200 x 1024 x 512 16 / 42, 4 x 200 x 1024 x 512 32 / 50, 8 x 200 x 1024 x 512 53 / 60, 1 x 1000 x 1000 x 1000 64 / 64,
//     8 x 128 x 2600 x 650 105 / 117, 8 x 250 x 2000 x 400 99 / 86, 11 x 16 x 28173 x 942 1233 / 1714
//   gradients bf16: 1 x 200 x 1024 x 512 16 / 28, 8 x 128 x 400 x 400 22 / 26, 4 x 200 x 1024 x 512 34 / 30, 8 x 128 x 652 x 652 37 / 45,
//     16 x 16 x 10000 x 650 420 / 277, 1 x 3 x 31296 x 768 92 / 53
double steps_us(int64_t M, int64_t N, int64_t K, int64_t batch)
{
    return static_cast<double>((M + 63) / 64 * ((N + 63) / 64) * batch) * static_cast<double>((K + 31) / 32) * (0.43 / 256);
}

double products_us(const gbmuf_linear_desc_t &d)
{
    return 2.0 * d.batch * static_cast<double>(d.rows) * static_cast<double>(d.out_features) * static_cast<double>(d.in_features) *
           (d.dtype == GBMUF_F32 ? 3.0 : 1.0) / 0.9e9;
}

bool takes_direct_forward(const gbmuf_linear_desc_t &d)
{
    if (d.dtype != GBMUF_F32) return false;
    const double values = 1e-6 * d.batch * static_cast<double>(d.rows + d.out_features) * static_cast<double>(d.in_features);
    return 9.0 + 1.4 * steps_us(d.rows, d.out_features, d.in_features, d.batch) <= 18.0 + 1.5 * values + products_us(d);
}

// What up to 64 rows take.  The kernel for few rows reads each matrix once in one launch, but for more than 16 rows of one the matrix cores (f32) or
// the readings of x are what it waits for, where there are many outputs.  us, few rows / tiles of f32 / of 16 bits, 1024 to 50,000 outputs: f32, 20
// rows 57 / - / -, 64 rows 108 / 90 / -; bf16, 8 rows 20 / - / 22, 20 rows 25 / - / 22, 64 rows 41 / - / 23 (without copies, where rows lie on 16 bytes).
enum class Few { kNo, kAlways, kUnlessAligned, kDirect };
Few few_of(const gbmuf_linear_desc_t &d)
{
    if (d.rows > kFewRows) return Few::kNo;
    const int64_t tiles = (d.out_features + 127) / 128 * d.batch;
    if (d.rows <= 16 || tiles < 256) return Few::kAlways;
    if (d.dtype == GBMUF_F32) return d.rows > 32 ? Few::kDirect : Few::kAlways;
    return Few::kUnlessAligned;
}

// What a gradient of 16-bit types takes as it lies: matrices whose rows lie on 16 bytes and are whole pieces of that.
bool as_it_lies(const gbmuf_matrix_t &m, int64_t cols) { return lies_well(m) && cols % 8 == 0; }

bool takes_direct_backward(const gbmuf_linear_desc_t &d, const gbmuf_linear_grad_io_t &io)
{
    const bool split = d.dtype == GBMUF_F32;
    const double M = static_cast<double>(d.rows), N = static_cast<double>(d.out_features), K = static_cast<double>(d.in_features);
    const bool dx = io.dx.data, dw = io.dw.data;
    double values = 0.0;                                   // that are laid out
    if (split) values = M * N * ((dx ? 1 : 0) + (dw ? 1 : 0)) + (dx ? N * K : 0.0) + (dw ? M * K : 0.0);
    else values = (d.activation || !as_it_lies(io.dy, d.out_features) ? M * N : 0.0) + (dx && !as_it_lies(io.w, d.in_features) ? N * K : 0.0) +
                  (dw && !as_it_lies(io.x, d.in_features) ? M * K : 0.0);
    const double steps = (dx ? steps_us(d.rows, d.in_features, d.out_features, d.batch) : 0.0) +
                         (dw ? steps_us(d.out_features, d.in_features, d.rows, d.batch) : 0.0);
    const double laid = (split ? 38.0 : 28.0) + (split ? 3e-6 : 2e-6) * d.batch * values + ((dx ? 1 : 0) + (dw ? 1 : 0)) * products_us(d);
    return 10.0 + 2.2 * steps <= laid;
}

// ---------------------------------------------------------------------------------------
// Forward.  io nullptr: only count the workspace, for matrices that lie as badly as can be.
// ---------------------------------------------------------------------------------------
int forward(const gbmuf_linear_desc_t &d, const gbmuf_linear_io_t *io, Space &space, hipStream_t stream)
{
    const int64_t M = d.rows, N = d.out_features, K = d.in_features;
    const int32_t G = d.batch, type = d.dtype;
    const bool split = type == kF32;
    const gbmuf_matrix_t none{};
    Epilogue e{};
    if (io) {
        e = into(io->y, G * M * N, type);
        e.pre = io->pre.data; e.ldp = io->pre.ld; e.p_batch = io->pre.batch_stride;
        e.bias = io->bias.data; e.bias_batch = io->bias.batch_stride;
        e.res = io->residual.data; e.ldr = io->residual.ld; e.r_batch = io->residual.batch_stride;
        e.act = d.activation; e.place = d.residual;
    }
    const Few few = few_of(d);
    const bool is_few = few == Few::kAlways || (few == Few::kUnlessAligned && io && !(lies_well(io->x) && lies_well(io->w)));
    if (is_few || takes_direct_forward(d) || few == Few::kDirect) {
        const Cut c = direct_cut(M, N, K, G, !is_few);
        DirectArgs f = direct_args(source_of(io ? io->x : none), source_of(io ? io->w : none), K, c, e);
        if (is_few) return io ? launch_few(f, type, stream) : GBMUF_OK;
        f.t.partial = space.take<float>(c.partial);
        if (!io) return GBMUF_OK;
        const int rc = launch_direct_forward(f, stream);
        return rc != GBMUF_OK ? rc : launch_join(JoinArgs{f.t, 64, 0, e}, stream);
    }
    const Cut s = shape_of(M, N, K, G, split);
    float *partial = space.take<float>(s.partial);
    uint32_t *max = space.take<uint32_t>(split ? G * (M + N) : 0);
    const gbmuf_matrix_t &xm = io ? io->x : none, &wm = io ? io->w : none;
    const LayArgs lx = source(xm, M, K, G, type), lw = source(wm, N, K, G, type);
    Operand x{static_cast<const uint16_t *>(xm.data), xm.ld, xm.batch_stride, nullptr, 0, false, false};
    Operand w{static_cast<const uint16_t *>(wm.data), wm.ld, wm.batch_stride, nullptr, 0, false, false};
    const bool may_lay = few == Few::kNo, lay_x = split || (may_lay && (!io || !lies_well(xm))), lay_w = split || (may_lay && (!io || !lies_well(wm)));
    if (lay_x) x = packed(space, M, K, G, lx.batch, split, max);
    if (lay_w) w = packed(space, N, K, G, lw.batch, split, max + G * M);
    if (!io) return GBMUF_OK;
    int rc = GBMUF_OK;
    if (split && !(K > 0 && K <= kLongestRow) && (rc = launch_zero(max, G * (M + N), stream)) != GBMUF_OK) return rc;
    LaySet set;
    for (int i = 0; i < 2; ++i) {
        if (!(i == 0 ? lay_x : lay_w)) continue;
        LayArgs l = i == 0 ? lx : lw;
        const Operand &o = i == 0 ? x : w;
        l.row_max = o.max;
        l.plain = const_cast<uint16_t *>(o.p); l.plain_ld = o.ld; l.plain_batch = o.batch;
        set.add(l);
    }
    if (!split) rc = launch_copy(set, stream);
    else if (K > 0 && K <= kLongestRow) rc = launch_rows(set, stream);
    else if ((rc = launch_stats(set, stream)) == GBMUF_OK) rc = launch_lay(set, stream);
    if (rc != GBMUF_OK) return rc;
    return run_product(x, w, K, type, e, s, partial, stream);
}

// ---------------------------------------------------------------------------------------
// Backward
// ---------------------------------------------------------------------------------------
// dw's epilogue
Epilogue weight_grad(const gbmuf_linear_desc_t &d, const gbmuf_matrix_t &m, int32_t type)
{
    Epilogue e = into(m, d.batch * d.out_features * d.in_features, type);
    if (d.accumulate) { e.place = GBMUF_RESIDUAL_AFTER; e.res = m.data; e.ldr = m.ld; e.r_batch = m.batch_stride; }
    return e;
}

int backward_direct(const gbmuf_linear_desc_t &d, const gbmuf_linear_grad_io_t *io, Space &space, hipStream_t stream)
{
    const int64_t M = d.rows, N = d.out_features, K = d.in_features;
    const int32_t G = d.batch, type = d.dtype, grad_type = d.weight_grad_f32 ? kF32 : type;
    const gbmuf_linear_grad_io_t none{};
    const gbmuf_linear_grad_io_t &at = io ? *io : none;
    const bool dx = !io || io->dx.data, dw = !io || io->dw.data;
    Source z = source_of(at.dy);
    if (d.activation) { z.pre = at.pre.data; z.ldp = at.pre.ld; z.p_batch = at.pre.batch_stride; z.act = d.activation; }
    const Cut both = direct_cut(N, K, M, G, false), cw = direct_cut(N, dw ? K : 0, M, G, false);
    const Cut cx = chain_cut(M, dx ? K : 0, N, G, both);           // as for both products, so that the workspace is the same for one
    const Epilogue e = into(at.dx, G * M * K, type);
    DirectArgs px = direct_args(z, source_of(at.w), N, cx, e);
    DirectArgs pw = direct_args(z, source_of(at.x), M, cw, weight_grad(d, at.dw, grad_type));
    pw.e.streamed = 0;                                     // tiles of 64 columns: pieces of lines, which the caches join (11 x 16 x 28173 x 942 f32 1326 streamed, 1233 plain)
    px.t.partial = space.take<float>(cx.partial);
    if (!io) return GBMUF_OK;
    px.copy = at.dresidual.data; px.copy_ld = at.dresidual.ld; px.copy_batch = at.dresidual.batch_stride;
    pw.sums = at.dbias.data; pw.sums_batch = at.dbias.batch_stride; pw.sums_type = grad_type; pw.accumulate = d.accumulate;
    const int rc = launch_direct_backward(px, pw, type, stream);
    return rc != GBMUF_OK ? rc : launch_join(JoinArgs{px.t, 64, 0, e}, stream);
}

int sum_columns(const gbmuf_linear_desc_t &d, const gbmuf_matrix_t &out, const float *sums, int32_t type, hipStream_t stream)
{
    SumArgs a{};
    a.sums = sums; a.out = out.data; a.out_batch = out.batch_stride;
    a.C = static_cast<int32_t>(d.out_features); a.tiles = static_cast<int32_t>((d.rows + kLayTile - 1) / kLayTile);
    a.batch = d.batch; a.type = type; a.accumulate = d.accumulate;
    return launch_column_sums(a, stream);
}

// f32: dz, w and x are taken apart, along the axis of each product.
int backward_split(const gbmuf_linear_desc_t &d, const gbmuf_linear_grad_io_t *io, Space &space, hipStream_t stream)
{
    const int64_t M = d.rows, N = d.out_features, K = d.in_features;
    const int32_t G = d.batch;
    const gbmuf_linear_grad_io_t none{};
    const gbmuf_linear_grad_io_t &at = io ? *io : none;
    const bool dx = !io || at.dx.data, dw = !io || at.dw.data, db = !io || at.dbias.data, dr = at.dresidual.data;
    const Cut sx = shape_of(M, K, N, G, true), sw = shape_of(N, K, M, G, true);
    float *partial = space.take<float>(std::max(dx ? sx.partial : 0, dw ? sw.partial : 0));     // one product after the other
    float *sums = space.take<float>(db ? G * ((M + kLayTile - 1) / kLayTile) * N : 0);
    const int64_t n_max = G * (M + N + 2 * K);             // largest magnitudes: rows and columns of dz, columns of w and of x
    uint32_t *max = space.take<uint32_t>(n_max);

    // dz is a matrix for each worker even where dy is shared, since z may not be
    LayArgs lz = source(at.dy, M, N, G, kF32);
    if (d.activation) { lz.pre = at.pre.data; lz.ldp = at.pre.ld; lz.p_batch = at.pre.batch_stride; lz.act = d.activation; }
    if (d.activation || dr || db) lz.batch = G;
    const LayArgs lw = source(at.w, N, K, G, kF32), lx = source(at.x, M, K, G, kF32);
    Operand z, zt, wt, xt;
    if (dx) z = packed(space, M, N, G, lz.batch, true, max);
    if (dw) zt = packed(space, N, M, G, lz.batch, true, max + G * M);
    if (dx) wt = packed(space, K, N, G, lw.batch, true, max + G * (M + N));
    if (dw) xt = packed(space, K, M, G, lx.batch, true, max + G * (M + N + K));
    if (!io) return GBMUF_OK;

    int rc = launch_zero(max, n_max, stream);
    if (rc != GBMUF_OK) return rc;
    lz.row_max = dx ? z.max : nullptr;
    lz.col_max = dw ? zt.max : nullptr;
    lz.col_sums = db ? sums : nullptr;
    if (dx) { lz.plain = const_cast<uint16_t *>(z.p); lz.plain_ld = z.ld; lz.plain_batch = z.batch; }
    if (dw) { lz.trans = const_cast<uint16_t *>(zt.p); lz.trans_ld = zt.ld; lz.trans_batch = zt.batch; }
    lz.dz = at.dresidual.data; lz.dz_ld = at.dresidual.ld; lz.dz_batch = at.dresidual.batch_stride;
    LaySet stats, lay;
    if (dx || dw || db) stats.add(lz);
    if (dx || dw || dr) lay.add(lz);
    for (int i = 0; i < 2; ++i) {
        if (!(i == 0 ? dx : dw)) continue;
        LayArgs l = i == 0 ? lw : lx;
        const Operand &o = i == 0 ? wt : xt;
        l.col_max = o.max;
        l.trans = const_cast<uint16_t *>(o.p); l.trans_ld = o.ld; l.trans_batch = o.batch;
        stats.add(l);
        lay.add(l);
    }
    if ((rc = launch_stats(stats, stream)) != GBMUF_OK) return rc;
    if (db && (rc = sum_columns(d, at.dbias, sums, kF32, stream)) != GBMUF_OK) return rc;
    if ((rc = launch_lay(lay, stream)) != GBMUF_OK) return rc;
    if (dx && (rc = run_product(z, wt, N, kF32, into(at.dx, G * M * K, kF32), sx, partial, stream)) != GBMUF_OK) return rc;
    return dw ? run_product(zt, xt, M, kF32, weight_grad(d, at.dw, kF32), sw, partial, stream) : rc;
}

// bf16, f16: the products read w, x and dz across their rows where they need to, so that matrices whose rows lie on 16 bytes are taken as
// they are and the others copied to places that do.
int backward_16(const gbmuf_linear_desc_t &d, const gbmuf_linear_grad_io_t *io, Space &space, hipStream_t stream)
{
    const int64_t M = d.rows, N = d.out_features, K = d.in_features;
    const int32_t G = d.batch, type = d.dtype, grad_type = d.weight_grad_f32 ? kF32 : type;
    const gbmuf_linear_grad_io_t none{};
    const gbmuf_linear_grad_io_t &at = io ? *io : none;
    const bool dx = !io || at.dx.data, dw = !io || at.dw.data, db = !io || at.dbias.data, dr = at.dresidual.data;
    const Cut sx = shape_of(M, K, N, G, false), sw = shape_of(N, K, M, G, false);
    float *partial = space.take<float>(std::max(dx ? sx.partial : 0, dw ? sw.partial : 0));
    float *sums = space.take<float>(db ? G * ((M + kLayTile - 1) / kLayTile) * N : 0);

    LayArgs lz = source(at.dy, M, N, G, type);
    if (d.activation) { lz.pre = at.pre.data; lz.ldp = at.pre.ld; lz.p_batch = at.pre.batch_stride; lz.act = d.activation; }
    if (d.activation || dr || db) lz.batch = G;            // a matrix for each worker even where dy is shared
    const LayArgs lw = source(at.w, N, K, G, type), lx = source(at.x, M, K, G, type);
    const auto take = [&](const gbmuf_matrix_t &m, const LayArgs &l, bool copy) {
        if (copy) return packed(space, l.R, l.C, G, l.batch, false, nullptr);
        return Operand{static_cast<const uint16_t *>(m.data), m.ld, m.batch_stride, nullptr, 0, false, false};
    };
    const bool copy_z = (dx || dw) && (d.activation || !io || !as_it_lies(at.dy, N)), copy_w = dx && (!io || !as_it_lies(at.w, K)),
               copy_x = dw && (!io || !as_it_lies(at.x, K));
    const Operand z = take(at.dy, lz, copy_z);
    Operand w = take(at.w, lw, copy_w), x = take(at.x, lx, copy_x), zt = z;
    zt.across = w.across = x.across = true;
    if (!io) return GBMUF_OK;

    LaySet set;
    const auto add = [&](LayArgs l, const Operand &o, bool copy) {
        if (copy) { l.plain = const_cast<uint16_t *>(o.p); l.plain_ld = o.ld; l.plain_batch = o.batch; }
        set.add(l);
    };
    lz.col_sums = db ? sums : nullptr;
    lz.dz = at.dresidual.data; lz.dz_ld = at.dresidual.ld; lz.dz_batch = at.dresidual.batch_stride;
    if (copy_z || db || dr) add(lz, z, copy_z);
    if (copy_w) add(lw, w, true);
    if (copy_x) add(lx, x, true);
    int rc = launch_copy(set, stream);
    if (rc == GBMUF_OK && db) rc = sum_columns(d, at.dbias, sums, grad_type, stream);
    if (rc == GBMUF_OK && dx) rc = run_product(z, w, N, type, into(at.dx, G * M * K, type), sx, partial, stream);
    if (rc == GBMUF_OK && dw) rc = run_product(zt, x, M, type, weight_grad(d, at.dw, grad_type), sw, partial, stream);
    return rc;
}

int backward_laid(const gbmuf_linear_desc_t &d, const gbmuf_linear_grad_io_t *io, Space &space, hipStream_t stream)
{
    return d.dtype == GBMUF_F32 ? backward_split(d, io, space, stream) : backward_16(d, io, space, stream);
}

// dz goes along with dx and its column sums with dw: what is asked for without those takes the other way.
int backward(const gbmuf_linear_desc_t &d, const gbmuf_linear_grad_io_t &io, Space &space, hipStream_t stream)
{
    const bool sums = !io.dbias.data || (io.dw.data && d.in_features > 0), copy = !io.dresidual.data || (io.dx.data && d.in_features > 0);
    return takes_direct_backward(d, io) && sums && copy ? backward_direct(d, &io, space, stream) : backward_laid(d, &io, space, stream);
}

int64_t forward_bytes(const gbmuf_linear_desc_t &d)
{
    Space space{nullptr};
    (void)forward(d, nullptr, space, nullptr);
    return space.used;
}

int64_t backward_bytes(const gbmuf_linear_desc_t &d)
{
    Space direct{nullptr}, laid{nullptr};
    (void)backward_direct(d, nullptr, direct, nullptr);
    (void)backward_laid(d, nullptr, laid, nullptr);
    return std::max(direct.used, laid.used);
}

int check_workspace(const void *workspace, int64_t have, int64_t need, std::initializer_list<const Extent *> matrices)
{
    if (need == 0) return GBMUF_OK;
    if (!workspace || have < need || reinterpret_cast<uintptr_t>(workspace) % 256 != 0) return GBMUF_EINVAL;
    Extent space;
    space.at = reinterpret_cast<uintptr_t>(workspace);
    space.rows = space.batch = 1;
    space.row = need;
    for (const Extent *m : matrices)
        if (overlap(space, *m)) return GBMUF_EINVAL;
    return GBMUF_OK;
}

}  // namespace
}  // namespace gbmuf

using namespace gbmuf;

extern "C" {

int gbmuf_linear_workspace(const gbmuf_linear_desc_t *desc, int32_t backward_pass, int64_t *bytes)
{
    if (!bytes) return GBMUF_EINVAL;
    *bytes = 0;
    const int rc = check_desc(desc);
    if (rc != GBMUF_OK) return rc;
    *bytes = backward_pass ? backward_bytes(*desc) : forward_bytes(*desc);
    return GBMUF_OK;
}

int gbmuf_linear(const gbmuf_linear_desc_t *desc, const gbmuf_linear_io_t *io, void *workspace, int64_t workspace_bytes, void *stream)
{
    int rc = check_desc(desc);
    if (rc != GBMUF_OK) return rc;
    if (!io) return GBMUF_EINVAL;
    const int64_t M = desc->rows, N = desc->out_features, K = desc->in_features, G = desc->batch;
    const int32_t t = desc->dtype;
    const Extent x = extent(io->x, M, K, G, t), w = extent(io->w, N, K, G, t), b = extent(io->bias, 1, N, G, t),
                 r = extent(io->residual, M, N, G, t), y = extent(io->y, M, N, G, t), p = extent(io->pre, M, N, G, t);
    if (!valid_input(io->x, x, t) || !valid_input(io->w, w, t) || !valid_output(io->y, y, t)) return GBMUF_EINVAL;
    if (io->bias.data && !valid_input(io->bias, b, t)) return GBMUF_EINVAL;
    if (desc->residual != GBMUF_RESIDUAL_NONE && !valid_input(io->residual, r, t)) return GBMUF_EINVAL;
    if (io->pre.data && !valid_output(io->pre, p, t)) return GBMUF_EINVAL;
    for (const Extent *o : {&y, &p}) {
        if (overlap(*o, x) || overlap(*o, w) || overlap(*o, b)) return GBMUF_EINVAL;
        const bool in_place = o == &y && r.at == y.at && r.ld == y.ld && r.stride == y.stride;
        if (desc->residual != GBMUF_RESIDUAL_NONE && !in_place && overlap(*o, r)) return GBMUF_EINVAL;
    }
    if (overlap(y, p)) return GBMUF_EINVAL;
    int64_t need = 0;
    if ((rc = gbmuf_linear_workspace(desc, 0, &need)) != GBMUF_OK) return rc;
    if (M == 0 || N == 0 || G == 0) return GBMUF_OK;
    const Extent none, &res = desc->residual != GBMUF_RESIDUAL_NONE ? r : none;
    if ((rc = check_workspace(workspace, workspace_bytes, need, {&x, &w, &b, &res, &y, &p})) != GBMUF_OK) return rc;
    if ((rc = check_device()) != GBMUF_OK) return rc;
    Space space{static_cast<char *>(workspace)};
    return forward(*desc, io, space, static_cast<hipStream_t>(stream));
}

int gbmuf_linear_backward(const gbmuf_linear_desc_t *desc, const gbmuf_linear_grad_io_t *io, void *workspace, int64_t workspace_bytes,
                          void *stream)
{
    int rc = check_desc(desc);
    if (rc != GBMUF_OK) return rc;
    if (!io) return GBMUF_EINVAL;
    const int64_t M = desc->rows, N = desc->out_features, K = desc->in_features, G = desc->batch;
    const int32_t t = desc->dtype, gt = desc->weight_grad_f32 ? kF32 : t;
    const Extent x = extent(io->x, M, K, G, t), w = extent(io->w, N, K, G, t), z = extent(io->pre, M, N, G, t), dy = extent(io->dy, M, N, G, t);
    const Extent dx = extent(io->dx, M, K, G, t), dw = extent(io->dw, N, K, G, gt), db = extent(io->dbias, 1, N, G, gt),
                 dr = extent(io->dresidual, M, N, G, t);
    if (!valid_input(io->dy, dy, t) || (desc->activation && !valid_input(io->pre, z, t))) return GBMUF_EINVAL;
    if (io->dx.data && (!valid_input(io->w, w, t) || !valid_output(io->dx, dx, t))) return GBMUF_EINVAL;
    if (io->dw.data && (!valid_input(io->x, x, t) || !valid_output(io->dw, dw, gt))) return GBMUF_EINVAL;
    if (io->dbias.data && !valid_output(io->dbias, db, gt)) return GBMUF_EINVAL;
    if (io->dresidual.data && (desc->residual != GBMUF_RESIDUAL_BEFORE || !valid_output(io->dresidual, dr, t))) return GBMUF_EINVAL;
    const Extent *outs[] = {&dx, &dw, &db, &dr};
    for (int i = 0; i < 4; ++i) {
        if (overlap(*outs[i], dy) || (desc->activation && overlap(*outs[i], z))) return GBMUF_EINVAL;
        if ((io->dw.data && overlap(*outs[i], x)) || (io->dx.data && overlap(*outs[i], w))) return GBMUF_EINVAL;
        for (int j = 0; j < i; ++j)
            if (overlap(*outs[i], *outs[j])) return GBMUF_EINVAL;
    }
    int64_t need = 0;
    if ((rc = gbmuf_linear_workspace(desc, 1, &need)) != GBMUF_OK) return rc;
    if (G == 0) return GBMUF_OK;
    const Extent none, &pre = desc->activation ? z : none, &xs = io->dw.data ? x : none, &ws = io->dx.data ? w : none;
    if ((rc = check_workspace(workspace, workspace_bytes, need, {&xs, &ws, &pre, &dy, &dx, &dw, &db, &dr})) != GBMUF_OK) return rc;
    if ((rc = check_device()) != GBMUF_OK) return rc;
    Space space{static_cast<char *>(workspace)};
    return backward(*desc, *io, space, static_cast<hipStream_t>(stream));
}

}  // extern "C"
