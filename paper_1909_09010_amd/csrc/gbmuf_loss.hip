// gbmuf_loss.hip -- entry points of the losses over a vocabulary: checks, workspace, pieces, and which kernels run.
#include "gbmuf_products.h"

namespace gbmuf {
namespace {

// Both losses: cross entropy is held to one word a row, distillation to a list of them.
struct Loss {
    gbmuf_linear_desc_t linear;      // the logits' product, for the rules that products go by
    int32_t top;                     // 0: cross entropy
    int32_t weight_grad_f32, accumulate;
    float tau;
};

struct Inputs {
    gbmuf_matrix_t x, w, bias, target, teacher;
};

int check_desc(const gbmuf_loss_desc_t *d, bool distill, Loss &l)
{
    if (!d || d->struct_size < sizeof(gbmuf_loss_desc_t)) return GBMUF_EINVAL;
    if (d->dtype < GBMUF_F32 || d->dtype > GBMUF_F16 || d->batch < 0 || d->rows < 0 || d->vocab < 0 || d->in_features < 0) return GBMUF_EINVAL;
    if (distill ? d->top < 1 || !(d->temperature > 0.0f) || !(d->temperature < __builtin_inff()) : d->top != 0) return GBMUF_EINVAL;
    if (d->batch > 65535 || d->rows > kLargest / 2 - 64 || d->vocab > kLargest / 2 - 64 || d->in_features > kLargest / 2 - 64) return GBMUF_EUNSUPPORTED;
    const int64_t M = d->rows, N = d->vocab, K = d->in_features, G = d->batch;
    if (too_many_tiles(M, N, G) || too_many_tiles(M, K, G) || too_many_tiles(N, K, G) || d->top > kMostTop) return GBMUF_EUNSUPPORTED;
    if (static_cast<double>(M) * static_cast<double>(G) > (distill ? 0x1p25 : 0x1p28)) return GBMUF_EUNSUPPORTED;          // what launches over rows may have
    // lse is handed over in one f32, so that a probability is off by |lse| 2^-24: at 2^-10 logits of 64 leave it 8 bits.  The gradient is tau times a difference of two
    // probabilities, the loss tau^2 times one of logarithms, which cancel where student and teacher agree: at 2^10 they keep 14 and 4 bits.
    if (distill && !(d->temperature >= 0x1p-10f && d->temperature <= 0x1p10f)) return GBMUF_EUNSUPPORTED;
    l = Loss{};
    l.linear.struct_size = sizeof(l.linear);
    l.linear.dtype = d->dtype; l.linear.batch = d->batch;
    l.linear.rows = M; l.linear.out_features = N; l.linear.in_features = K;
    l.top = d->top;
    l.weight_grad_f32 = d->weight_grad_f32; l.accumulate = d->accumulate;
    l.tau = distill ? d->temperature : 1.0f;
    return GBMUF_OK;
}

// ---------------------------------------------------------------------------------------
// Pieces: what is laid out or written of a vocabulary at a time, of all workers, some of them or a part of one's words.
// ---------------------------------------------------------------------------------------
struct Pieces {
    int64_t workers, words;          // of a piece, at most
};

// bytes: of a word of one worker
Pieces pieces_of(int64_t G, int64_t V, int64_t bytes, int64_t most)
{
    const int64_t worker = std::max<int64_t>(V * bytes, 1);
    if (worker <= most) {
        const int64_t n = std::max<int64_t>(std::min(G, most / worker), 1), parts = (std::max<int64_t>(G, 1) + n - 1) / n;
        return Pieces{(std::max<int64_t>(G, 1) + parts - 1) / parts, std::max<int64_t>(V, 1)};           // as many workers in each
    }
    const int64_t n = (worker + most - 1) / most, words = ((V + n - 1) / n + 255) / 256 * 256;
    return Pieces{1, std::min(words, V)};
}

struct Piece {
    int64_t g, workers, v, words;
};

template <class F>
int each_piece(const Pieces &p, int64_t G, int64_t V, F f)
{
    for (int64_t g = 0; g < G; g += p.workers)
        for (int64_t v = 0; v < V; v += p.words) {
            const int rc = f(Piece{g, std::min(p.workers, G - g), v, std::min(p.words, V - v)});
            if (rc != GBMUF_OK) return rc;
        }
    return GBMUF_OK;
}

// A matrix from worker g and row r on.
gbmuf_matrix_t part(const gbmuf_matrix_t &m, int64_t g, int64_t r, int32_t type)
{
    gbmuf_matrix_t p = m;
    if (p.data) p.data = static_cast<char *>(m.data) + (g * m.batch_stride + r * m.ld) * static_cast<int64_t>(type_bytes(type));
    return p;
}

// A vector (ld unused) from worker g and element n on.
gbmuf_matrix_t vector_part(const gbmuf_matrix_t &m, int64_t g, int64_t n, int32_t type)
{
    gbmuf_matrix_t p = m;
    if (p.data) p.data = static_cast<char *>(m.data) + (g * m.batch_stride + n) * static_cast<int64_t>(type_bytes(type));
    return p;
}

// ---------------------------------------------------------------------------------------
// Words
// ---------------------------------------------------------------------------------------
// as_given: few rows' lists of few words need no order.
Words words_of(const Loss &l, const Inputs &in, bool as_given, Space &space)
{
    const gbmuf_matrix_t &target = in.target;
    const int64_t G = l.linear.batch, M = l.linear.rows;
    Words w{};
    w.top = 1;
    w.rows = static_cast<int32_t>(M);
    w.vocab = static_cast<int32_t>(l.linear.out_features);
    if (l.top == 0) {
        w.target = static_cast<const int64_t *>(target.data);
        w.ld = target.ld; w.batch = target.batch_stride;
        return w;
    }
    w.top = l.top;
    if (as_given) {
        w.target = static_cast<const int64_t *>(target.data);
        w.ld = target.ld; w.batch = target.batch_stride;
        w.logit = static_cast<const float *>(in.teacher.data);
        w.logit_ld = in.teacher.ld; w.logit_batch = in.teacher.batch_stride;
        return w;
    }
    w.id = space.take<int32_t>(G * M * l.top);
    w.share = space.take<float>(G * M * l.top);
    w.state = space.take<int32_t>(G * M);
    return w;
}

Words words_from(const Words &w, int64_t g)
{
    Words p = w;
    if (w.target) p.target += g * w.batch;
    else {
        const int64_t rows = g * w.rows;
        p.id += rows * w.top;
        p.share += rows * w.top;
        p.state += rows;
    }
    return p;
}

int order_words(const Loss &l, const Words &w, const Inputs &in, bool merge, hipStream_t stream)
{
    if (l.top == 0 || w.logit) return GBMUF_OK;
    TeacherArgs a{};
    a.id = static_cast<const int64_t *>(in.target.data); a.id_ld = in.target.ld; a.id_batch = in.target.batch_stride;
    a.logit = static_cast<const float *>(in.teacher.data); a.logit_ld = in.teacher.ld; a.logit_batch = in.teacher.batch_stride;
    a.out_id = const_cast<int32_t *>(w.id); a.out_share = const_cast<float *>(w.share); a.out_state = const_cast<int32_t *>(w.state);
    a.rows = w.rows; a.batch = l.linear.batch; a.top = w.top; a.vocab = w.vocab;
    a.inv_tau = 1.0f / l.tau;
    a.merge = merge ? 1 : 0;
    return launch_teacher(a, stream);
}

// Lists by window for tiles of `tile` rows, whose waves take half of them each.
WordLists lists_of(const Loss &l, const Words &w, int tile, bool shares, Space &space)
{
    WordLists lists{};
    if (l.top == 0) return lists;
    lists.block_rows = tile / 2;
    lists.blocks = (w.rows + lists.block_rows - 1) / lists.block_rows;
    lists.shift = 6;
    while ((static_cast<int64_t>(w.vocab) >> lists.shift) >= kMostWindows) ++lists.shift;
    lists.windows = (w.vocab >> lists.shift) + 1;
    const int64_t blocks = static_cast<int64_t>(l.linear.batch) * lists.blocks, n = blocks * lists.block_rows * w.top;
    lists.code = space.take<uint32_t>(n);
    lists.share = space.take<float>(shares ? n : 0);
    if (!shares) lists.share = nullptr;
    lists.starts = space.take<int32_t>(blocks * (lists.windows + 1));
    return lists;
}

WordLists lists_from(const WordLists &lists, const Words &w, int64_t g)
{
    WordLists p = lists;
    if (p.blocks == 0) return p;
    const int64_t n = g * p.blocks * p.block_rows * w.top;
    p.code += n;
    if (p.share) p.share += n;
    p.starts += g * p.blocks * (p.windows + 1);
    return p;
}

LossArgs loss_args(const Loss &l, const Inputs &in, const Words &w, const Piece &p)
{
    LossArgs a{};
    const gbmuf_matrix_t bias = vector_part(in.bias, p.g, p.v, l.linear.dtype);
    a.bias = bias.data; a.bias_batch = bias.batch_stride;
    a.words = words_from(w, p.g);
    a.type = l.linear.dtype;
    a.first = static_cast<int32_t>(p.v);
    a.inv_tau = 1.0f / l.tau; a.tau = l.tau;
    return a;
}

// Tiles of logits: of 256 x 256, one workgroup a CU, or of 128 x 128, two, as a product's, and how many of them a workgroup walks: as many as
// fill the rounds of the chip best.  us: a product's step, what leaving a tile takes, and what a workgroup pays before its first step.
Cut logits_shape(int64_t M, int64_t N, int64_t K, int64_t batch, bool split_type, bool backward)
{
    const int64_t steps = std::max<int64_t>(packed_words(K, split_type) / kStepWords, 1);
    Cut best;
    for (const int tile : {256, 128}) {
        if (split_type && tile == 256) continue;
        const bool wide = tile == 256;
        const int64_t rows = (M + tile - 1) / tile * batch, words = (N + tile - 1) / tile, slots = wide ? 256 : 512;
        const double each = static_cast<double>(steps) * (wide ? 1.73 : 1.06) + (wide ? 4.0 : 2.5) * (backward ? 2.0 : 1.0);
        for (int64_t walk = 1; walk <= std::min<int64_t>(words, 64); ++walk) {
            const int64_t groups = rows * ((words + walk - 1) / walk);
            const double cost = static_cast<double>((groups + slots - 1) / slots) * (static_cast<double>(walk) * each + 3.0);
            if (best.tile != 0 && cost >= best.cost) continue;
            best = Cut{};
            best.tile = tile;
            best.cost = cost;
            best.t.M = static_cast<int32_t>(M); best.t.N = static_cast<int32_t>(N); best.t.batch = static_cast<int32_t>(batch);
            best.t.tiles_m = static_cast<int32_t>((M + tile - 1) / tile);
            best.t.steps = static_cast<int32_t>(walk);
        }
    }
    best.t.splits = 1;
    best.t.tiles_n = static_cast<int32_t>(((N + best.tile - 1) / best.tile + best.t.steps - 1) / best.t.steps);
    best.t.whole = best.t.count();
    return best;
}

// The same tiles for fewer words or workers.
Cut same_shape(const Cut &c, int64_t N, int64_t batch)
{
    Cut s = c;
    s.t.N = static_cast<int32_t>(N); s.t.batch = static_cast<int32_t>(batch);
    s.t.tiles_n = static_cast<int32_t>(((N + c.tile - 1) / c.tile + c.t.steps - 1) / c.t.steps);
    s.t.whole = s.t.count();
    return s;
}

ProductArgs logits_args(const Operand &x, const Operand &w, int64_t K, int32_t type, const Cut &c)
{
    ProductArgs p{};
    p.a = x.p; p.b = w.p; p.lda = x.ld; p.ldb = w.ld; p.a_batch = x.batch; p.b_batch = w.batch;
    p.a_max = x.max; p.b_max = w.max; p.a_max_batch = x.max_batch; p.b_max_batch = w.max_batch;
    p.K = static_cast<int32_t>(type == kF32 || (x.whole && w.whole) ? packed_words(K, type == kF32) : K);
    p.t = c.t;
    return p;
}

Operand operand_of(const gbmuf_matrix_t &m)
{
    return Operand{static_cast<const uint16_t *>(m.data), m.ld, m.batch_stride, nullptr, 0, false, false};
}

// Lays out rows along their own axis: f32 taken apart with row maxima, 16-bit types copied.
int lay_rows(LayArgs l, const Operand &o, int64_t K, int32_t type, hipStream_t stream)
{
    if (type != kF32) {
        KeepArgs a{};
        a.words.rows = l.R;
        a.all = 1;
        a.x = l.src; a.ld = l.ld; a.batch_stride = l.batch_stride;
        a.out = const_cast<uint16_t *>(o.p); a.out_ld = o.ld;
        a.columns = l.C; a.batch = l.batch; a.type = type;
        return launch_keep(a, stream);
    }
    l.plain = const_cast<uint16_t *>(o.p); l.plain_ld = o.ld; l.plain_batch = o.batch;
    l.row_max = o.max;
    LaySet set;
    set.add(l);
    if (K > 0 && K <= kLongestRow) return launch_rows(set, stream);
    int rc = launch_zero(o.max, static_cast<int64_t>(l.R) * l.batch, stream);
    if (rc == GBMUF_OK) rc = launch_stats(set, stream);
    return rc == GBMUF_OK ? launch_lay(set, stream) : rc;
}

// ---------------------------------------------------------------------------------------
// Forward.  io nullptr: only count the workspace, for matrices that lie as those of `at` do.
// ---------------------------------------------------------------------------------------
constexpr int64_t kLaidBytes = 256 << 20;          // of w, at a time

int forward(const Loss &l, const Inputs &at, const gbmuf_loss_io_t *io, Space &space, hipStream_t stream)
{
    const gbmuf_linear_desc_t &d = l.linear;
    const int64_t M = d.rows, N = d.out_features, K = d.in_features;
    const int32_t G = d.batch, type = d.dtype;
    const bool split = type == kF32;
    const Few few = few_of(d);
    const bool is_few = few == Few::kAlways || (few == Few::kUnlessAligned && !(lies_well(at.x) && lies_well(at.w)));
    const bool direct = takes_direct_forward(d) || few == Few::kDirect;
    const Words words = words_of(l, at, is_few && l.top <= kFewWords, space);
    float *word_logits = space.take<float>(G * M * words.top);

    LossJoin j{};
    j.words = words;
    j.at = word_logits;
    j.batch = G;
    j.inv_tau = 1.0f / l.tau; j.tau = l.tau;
    if (io) {
        j.loss = static_cast<float *>(io->loss.data); j.loss_ld = io->loss.ld; j.loss_batch = io->loss.batch_stride;
        j.lse = static_cast<float *>(io->lse.data); j.lse_ld = io->lse.ld; j.lse_batch = io->lse.batch_stride;
    }
    const auto parts_of = [&](int64_t tiles) {
        j.tiles = static_cast<int32_t>(tiles);
        float2 *p = space.take<float2>(G * tiles * M);
        j.parts = p;
        return p;
    };
    int rc = GBMUF_OK;
    if (is_few || direct) {
        const Cut c = direct_cut(M, N, K, G, false);
        const DirectArgs f = direct_args(source_of(at.x), source_of(at.w), K, c, Epilogue{});
        const int columns = is_few ? few_columns(f, type) : 64;
        float2 *parts = parts_of((N + columns - 1) / columns);
        if (!io) return GBMUF_OK;
        if (!space.fits()) return GBMUF_EINVAL;
        LossArgs a = loss_args(l, at, words, Piece{0, G, 0, N});
        a.parts = parts; a.part_tiles = j.tiles;
        a.at = word_logits;
        if ((rc = order_words(l, words, at, false, stream)) != GBMUF_OK) return rc;
        rc = is_few ? launch_loss_few(f, a, type, stream) : launch_loss_direct(f, a, type, false, stream);
        return rc == GBMUF_OK ? launch_loss_join(j, stream) : rc;
    }
    // w is laid out a piece at a time, x once
    const bool may_lay = few == Few::kNo, lay_x = split || (may_lay && !lies_well(at.x)), lay_w = split || (may_lay && !lies_well(at.w));
    const Pieces pieces = lay_w ? pieces_of(G, N, packed_words(K, split) * 2, kLaidBytes) : Pieces{std::max(G, 1), std::max<int64_t>(N, 1)};
    const Cut shape = logits_shape(M, pieces.words, K, pieces.workers, split, false);
    const int64_t whole_pieces = N / pieces.words;
    float2 *parts = parts_of(whole_pieces * shape.t.tiles_n + same_shape(shape, N - whole_pieces * pieces.words, 1).t.tiles_n);
    const WordLists lists = lists_of(l, words, shape.tile, false, space);
    const LayArgs lx = source(at.x, M, K, G, type);
    Operand x = operand_of(at.x), w = operand_of(at.w);
    if (lay_x) x = packed(space, M, K, G, lx.batch, split, space.take<uint32_t>(split ? G * M : 0));
    if (lay_w) w = packed(space, pieces.words, K, static_cast<int32_t>(pieces.workers), static_cast<int32_t>(pieces.workers), split,
                          space.take<uint32_t>(split ? pieces.workers * pieces.words + 256 : 0));
    if (!io) return GBMUF_OK;
    if (!space.fits()) return GBMUF_EINVAL;
    if ((rc = order_words(l, words, at, false, stream)) != GBMUF_OK) return rc;
    if (lists.blocks > 0 && (rc = launch_word_lists(words, lists, G, stream)) != GBMUF_OK) return rc;
    if (lay_x && (rc = lay_rows(lx, x, K, type, stream)) != GBMUF_OK) return rc;
    rc = each_piece(pieces, G, N, [&](const Piece &p) {
        Operand px = x, pw = w;
        px.p += p.g * x.batch;
        if (px.max) px.max += p.g * x.max_batch;
        const gbmuf_matrix_t wm = part(at.w, p.g, p.v, type);
        if (lay_w) {
            const LayArgs lw = source(wm, p.words, K, static_cast<int32_t>(p.workers), type);
            pw.batch = lw.batch < p.workers ? 0 : p.words * w.ld;
            pw.max_batch = lw.batch < p.workers ? 0 : p.words;
            const int r = lay_rows(lw, pw, K, type, stream);
            if (r != GBMUF_OK) return r;
        } else pw = operand_of(wm);
        const Cut c = same_shape(shape, p.words, p.workers);
        LossArgs a = loss_args(l, at, words, p);
        a.lists = lists_from(lists, words, p.g);
        a.walk = c.t.steps;
        a.part_tiles = j.tiles;
        a.first_tile = static_cast<int32_t>(p.v / pieces.words) * shape.t.tiles_n;
        a.parts = parts + p.g * j.tiles * M;
        a.at = word_logits + p.g * M * words.top;
        return launch_vocab(logits_args(px, pw, K, type, c), a, type, shape.tile, false, stream);
    });
    return rc == GBMUF_OK ? launch_loss_join(j, stream) : rc;
}

// What any placement takes.  A w that lies well is taken whole, and one that does not in pieces, whose tiles go to workgroups otherwise: neither's parts are always the more.
int64_t forward_bytes(const Loss &l)
{
    const gbmuf_matrix_t well{}, badly{nullptr, 1, 0};
    const auto bytes = [&](const gbmuf_matrix_t &x, const gbmuf_matrix_t &w) {
        Space space{nullptr};
        (void)forward(l, Inputs{x, w, {}, {}, {}}, nullptr, space, nullptr);
        return space.used;
    };
    const int64_t most = bytes(badly, badly);
    switch (few_of(l.linear)) {
        case Few::kNo: return l.linear.dtype == kF32 ? most : std::max(most, bytes(badly, well));           // f32: however they lie
        case Few::kUnlessAligned: return std::max(most, bytes(well, well));
        default: return most;
    }
}

// ---------------------------------------------------------------------------------------
// Backward
// ---------------------------------------------------------------------------------------
// Bytes of dz, and what is laid out of it, at a time.  Fewer, larger launches: us by 256 / 512 / 768 / 1024 MB, bf16 8 x 5120 x 8197 x 512 (672 MB) 1532 / 1556 / 1421 /
// 1412, 2 x 5120 x 50000 x 1024 (1 GB) 3384 / 3180 / 3166 / 3312; f32 by 512 / 1024 / 1536 MB 8 x 700 x 10000 x 650 (720 MB) 1365 / 1260 / 1216.
constexpr int64_t kGradBytes = 768 << 20, kSplitGradBytes = 1536 << 20;

// dw's epilogue, for the words of a piece
Epilogue weight_grad(const Loss &l, const gbmuf_matrix_t &m, int64_t values, int32_t type)
{
    Epilogue e = into(m, values, type);
    if (l.accumulate) { e.place = GBMUF_RESIDUAL_AFTER; e.res = m.data; e.ldr = m.ld; e.r_batch = m.batch_stride; }
    return e;
}

LossArgs grad_args(const Loss &l, const Inputs &in, const gbmuf_loss_grad_io_t *io, const Words &w, const Piece &p)
{
    LossArgs a = loss_args(l, in, w, p);
    const gbmuf_matrix_t lse = part(io->lse, p.g, 0, kF32), dloss = part(io->dloss, p.g, 0, kF32);
    a.lse = static_cast<const float *>(lse.data); a.lse_ld = lse.ld; a.lse_batch = lse.batch_stride;
    a.dloss = static_cast<const float *>(dloss.data); a.dloss_ld = dloss.ld; a.dloss_batch = dloss.batch_stride;
    return a;
}

// Small sizes: dz in f32, then both products in f32 from where the matrices lie.
int backward_direct(const Loss &l, const Inputs *in, const gbmuf_loss_grad_io_t *io, Space &space, hipStream_t stream)
{
    const gbmuf_linear_desc_t &d = l.linear;
    const int64_t M = d.rows, N = d.out_features, K = d.in_features;
    const int32_t G = d.batch, type = d.dtype, grad_type = l.weight_grad_f32 ? kF32 : type;
    const Inputs none{};
    const Inputs &at = in ? *in : none;
    const gbmuf_loss_grad_io_t no_grads{};
    const gbmuf_loss_grad_io_t &out = io ? *io : no_grads;
    const bool dx = !io || out.dx.data, dw = !io || out.dw.data;
    const Words words = words_of(l, at, false, space);
    const int64_t ld = (N + 63) / 64 * 64;
    float *dz = space.take<float>(G * M * ld);
    int32_t *live = space.take<int32_t>(G * M);
    const Cut cz = direct_cut(M, N, K, G, false), both = direct_cut(N, K, M, G, false), cw = direct_cut(N, dw ? K : 0, M, G, false);
    const Cut cx = chain_cut(M, dx ? K : 0, N, G, both);
    float *partial = space.take<float>(cx.partial);
    if (!io) return GBMUF_OK;
    if (!space.fits()) return GBMUF_EINVAL;
    int rc = order_words(l, words, at, true, stream);
    if (rc != GBMUF_OK) return rc;
    LossArgs a = grad_args(l, at, io, words, Piece{0, G, 0, N});
    a.dz = dz; a.dz_ld = ld; a.dz_batch = M * ld;
    a.live = live;
    if ((rc = launch_loss_direct(direct_args(source_of(at.x), source_of(at.w), K, cz, Epilogue{}), a, type, true, stream)) != GBMUF_OK) return rc;
    Source z{};
    z.p = dz; z.ld = ld; z.batch = M * ld;
    const Epilogue e = into(out.dx, G * M * K, type);
    DirectArgs px = direct_args(z, source_of(at.w), N, cx, e);
    px.t.partial = partial;
    DirectArgs pw = direct_args(z, source_of(at.x), M, cw, weight_grad(l, out.dw, G * N * K, grad_type));
    pw.e.streamed = 0;
    pw.live = live; pw.live_batch = M;
    pw.sums = out.dbias.data; pw.sums_batch = out.dbias.batch_stride; pw.sums_type = grad_type; pw.accumulate = l.accumulate;
    rc = launch_loss_grads(px, pw, type, stream);
    return rc != GBMUF_OK ? rc : launch_join(JoinArgs{px.t, 64, 0, e}, stream);
}

// Up to 64 rows and features: all of a piece of the vocabulary in one workgroup, dx's parts joined by a second launch.
constexpr int64_t kSmallParts = 64 << 20;          // bytes of dx's parts
int64_t small_pieces(const gbmuf_linear_desc_t &d) { return (d.out_features + kSmallWords - 1) / kSmallWords; }
bool is_small(const gbmuf_linear_desc_t &d)
{
    return d.rows <= kSmallRows && d.rows > 0 && d.in_features <= kSmallColumns && d.out_features > 0 && small_pieces(d) <= 65535 &&
           static_cast<double>(small_pieces(d)) * d.batch * static_cast<double>(d.rows) * static_cast<double>(d.in_features) * 4.0 <= static_cast<double>(kSmallParts);
}

// Up to 8 rows: w is read from memory once, by workgroups that each walk pieces of the vocabulary; of 16-bit types while w is not more than 64 MB.  us, this / laid
// out: bf16 1 x 2 x 1000 x 256 18 / 25, 4 x 8 x 5000 x 512 41 / 48, 2 x 8 x 20000 x 304 61 / 56, f16 8 x 6 x 3000 x 301 42 / 59, bf16 1 x 8 x 30000 x 1024 82 / 91, 4 x 5 x 12800 x
// 832 156 / 99, 8 x 4 x 10000 x 640 164 / 110; f32 1 x 8 x 50000 x 1024 154 / 207.
// It ends at 1024 features, which 256 threads have of a word's row, 4 each: us, 1024 / 1028 or 1032 features: f32 1 x 8 x 50000 150 / 210, 2 x 3 x 5000 33 / 63, bf16 1 x 8 x 20000
// 65 / 73; a second turn over the columns is not built.
constexpr double kFewGradValues = 1 << 25;
bool is_few(const gbmuf_linear_desc_t &d)
{
    const double values = static_cast<double>(d.batch) * static_cast<double>(d.out_features) * static_cast<double>(d.in_features);
    return d.rows <= kFewGradRows && d.rows > 0 && d.in_features <= kFewGradColumns && d.out_features > 0 && (d.dtype == GBMUF_F32 || values <= kFewGradValues);
}
// Words of a piece: fewer where that makes work for more CUs.  us, 16 / 32 / 64: f32 1 x 3 x 300 x 700 16 / 21 / 32, bf16 2 x 5 x 1216 x 448 16 / 20 / 27, 1 x 8 x 5000 x 1024 27 / 31 /
// -, f32 9 x 6 x 1250 x 74 27 / 17.5 / -, bf16 1 x 8 x 10000 x 1024 43 / 40 / 57, 4 x 8 x 5000 x 512 - / 42 / 39, f16 8 x 6 x 3000 x 301 - / 47 / 41.
int64_t few_words(const gbmuf_linear_desc_t &d)
{
    const int64_t pieces = (d.out_features + 63) / 64 * d.batch;
    return pieces <= 80 ? 16 : pieces <= 256 ? 32 : 64;
}
int64_t few_pieces(const gbmuf_linear_desc_t &d) { return (d.out_features + few_words(d) - 1) / few_words(d); }
int64_t few_workgroups(const gbmuf_linear_desc_t &d) { return std::min<int64_t>(few_pieces(d), std::max<int64_t>(768 / std::max(d.batch, 1), 1)); }

int backward_few(const Loss &l, const Inputs *in, const gbmuf_loss_grad_io_t *io, Space &space, hipStream_t stream)
{
    const gbmuf_linear_desc_t &d = l.linear;
    const bool small = is_small(d);
    const int64_t M = d.rows, K = d.in_features, pieces = small ? small_pieces(d) : few_pieces(d), groups = few_workgroups(d), parts = small ? pieces : groups * (256 / few_grads_lanes(K));
    const int32_t G = d.batch, type = d.dtype;
    const Inputs none{};
    const Inputs &at = in ? *in : none;
    const Words words = words_of(l, at, in && small && l.top <= kFewWords, space);
    float *sums = space.take<float>(parts * G * M * K);
    if (!io) return GBMUF_OK;
    if (!space.fits()) return GBMUF_EINVAL;
    int rc = order_words(l, words, at, true, stream);
    if (rc != GBMUF_OK) return rc;
    SmallGrads a{};
    a.l = grad_args(l, at, io, words, Piece{0, G, 0, d.out_features});
    a.x = at.x.data; a.ldx = at.x.ld; a.x_batch = at.x.batch_stride;
    a.w = at.w.data; a.ldw = at.w.ld; a.w_batch = at.w.batch_stride;
    a.dx = io->dx.data; a.lddx = io->dx.ld; a.dx_batch = io->dx.batch_stride;
    a.dw = io->dw.data; a.lddw = io->dw.ld; a.dw_batch = io->dw.batch_stride;
    a.dbias = io->dbias.data; a.dbias_batch = io->dbias.batch_stride;
    a.parts = io->dx.data ? sums : nullptr;
    a.columns = static_cast<int32_t>(K); a.batch = G; a.pieces = static_cast<int32_t>(pieces);
    a.grad_type = l.weight_grad_f32 ? kF32 : type; a.accumulate = l.accumulate;
    if (small) return launch_small_grads(a, stream);
    a.words = static_cast<int32_t>(few_words(d));
    rc = launch_few_grads(a, static_cast<int32_t>(groups), stream);
    return rc == GBMUF_OK ? launch_join_parts(a, static_cast<int32_t>(parts), stream) : rc;
}

// Everything else: dz a piece at a time, in 16 bits or taken apart, and the products of the piece on the 16-bit matrix instructions.
// bf16 and f16 round dz to the type, scaled by dz_scale, since that is what the instructions take.  What it costs, root mean square against 64 bits of dx and dw, so / with dz in f32 and the
// results rounded alike: bf16 2 x 5120 x 50000 x 1024 0.22 / 0.17 %, with 64 words of a teacher 8 x 5120 x 8197 x 512 0.23 / 0.17 %; f16 8 x 699 x 10001 x 650 0.034 / 0.028 and 0.029 / 0.022 %.  A second number
// of 16 bits for what the rounding leaves would bring that back for both products once more: 2148 us beside 3104, 990 beside 1313, 358 beside 431.  A program that keeps logits in 16 bits rounds them as well.
int backward_laid(const Loss &l, const Inputs *in, const gbmuf_loss_grad_io_t *io, Space &space, hipStream_t stream)
{
    const gbmuf_linear_desc_t &d = l.linear;
    const int64_t M = d.rows, N = d.out_features, K = d.in_features;
    const int32_t G = d.batch, type = d.dtype, grad_type = l.weight_grad_f32 ? kF32 : type;
    const bool split = type == kF32;
    const Inputs none{};
    const Inputs &at = in ? *in : none;
    const gbmuf_loss_grad_io_t no_grads{};
    const gbmuf_loss_grad_io_t &out = io ? *io : no_grads;
    const bool dx = !io || out.dx.data, dw = !io || out.dw.data, db = !io || out.dbias.data;
    const Words words = words_of(l, at, false, space);

    // of a word: its dz (f32: and both layouts of it), w's row along k (f32) and, taken apart, along the words
    const int64_t word_bytes = split ? M * 12 + 128 + packed_words(K, true) * 2 + K * 4 : M * 2;
    const Pieces pieces = pieces_of(G, N, word_bytes, split ? kSplitGradBytes : kGradBytes);
    const int64_t PG = pieces.workers, PN = pieces.words, ld = (PN + 63) / 64 * 64;
    const bool copy_w = !split && (!io || !as_it_lies(at.w, K));
    const int64_t kept = packed_words(K, false);                 // columns of a row of x that is kept
    const Cut shape = logits_shape(M, PN, K, PG, split, true);
    const WordLists lists = lists_of(l, words, shape.tile, true, space);
    // the last workers or words may be fewer, and cut otherwise
    int64_t parts = 0;
    for (const int64_t workers : {PG, G % PG})
        for (const int64_t n : {PN, N % PN})
            if (workers > 0 && n > 0) parts = std::max({parts, shape_of(M, K, n, workers, split).partial, shape_of(n, K, M, workers, split).partial});
    float *partial = space.take<float>(parts);
    char *kept_x = space.take<char>(G * M * kept * static_cast<int64_t>(type_bytes(type)));
    float *most = space.take<float>(split ? 0 : G * (kMostParts + 1)), *factors = split ? nullptr : most + G * kMostParts;
    char *dz = space.take<char>(PG * M * ld * static_cast<int64_t>(type_bytes(type)));
    const bool several = PN < N;
    float *dx_sums = space.take<float>(several && !split ? PG * M * K : 0);
    float *sums = space.take<float>(db ? PG * 2 * ((M + 127) / 128) * PN : 0);         // of 64 rows, or of half a tile

    Operand x{reinterpret_cast<const uint16_t *>(kept_x), kept, M * kept, nullptr, 0, true, false}, w = operand_of(at.w), z, zt, wt, xt;
    uint32_t *max = nullptr, *dz_rows = nullptr, *w_rows = nullptr;
    if (split) {
        max = space.take<uint32_t>(PG * (2 * PN + K) + 256);    // of a piece: columns of dz, rows of w, up to the end of the last tile, and columns of w
        dz_rows = space.take<uint32_t>(G * M);
        uint32_t *x_max = space.take<uint32_t>(G * K);          // columns of x
        const int32_t workers = static_cast<int32_t>(PG);
        x = packed(space, M, K, G, G, true, space.take<uint32_t>(G * M));
        xt = packed(space, K, M, G, G, true, x_max);
        w = packed(space, PN, K, workers, workers, true, nullptr);
        wt = packed(space, K, PN, workers, workers, true, nullptr);
        z = packed(space, M, PN, workers, workers, true, dz_rows);
        zt = packed(space, PN, M, workers, workers, true, nullptr);
    } else if (copy_w) {
        w = packed(space, PN, K, static_cast<int32_t>(PG), static_cast<int32_t>(PG), false, nullptr);
    }
    if (!io) return GBMUF_OK;
    if (!space.fits()) return GBMUF_EINVAL;

    int rc = order_words(l, words, at, true, stream);
    if (rc != GBMUF_OK || (lists.blocks > 0 && (rc = launch_word_lists(words, lists, G, stream)) != GBMUF_OK)) return rc;
    KeepArgs keep{};
    keep.words = words;
    keep.x = at.x.data; keep.ld = at.x.ld; keep.batch_stride = at.x.batch_stride;
    keep.out = kept_x; keep.out_ld = kept;
    keep.columns = static_cast<int32_t>(K); keep.batch = G; keep.type = type;
    keep.dloss = static_cast<const float *>(out.dloss.data); keep.dloss_ld = out.dloss.ld; keep.dloss_batch = out.dloss.batch_stride;
    keep.tau = l.tau;
    keep.most_parts = static_cast<int32_t>(std::min<int64_t>((M + 2047) / 2048, kMostParts));
    keep.most = split || M == 0 ? nullptr : most;
    keep.row_max = dz_rows;
    if ((rc = launch_keep(keep, stream)) != GBMUF_OK) return rc;
    const gbmuf_matrix_t kept_m{kept_x, kept, M * kept};
    if (split) {
        const LayArgs lx = source(kept_m, M, K, G, kF32);
        if ((rc = lay_rows(lx, x, K, kF32, stream)) != GBMUF_OK) return rc;
        if (dw) {
            LayArgs t = lx;
            t.col_max = xt.max;
            t.trans = const_cast<uint16_t *>(xt.p); t.trans_ld = xt.ld; t.trans_batch = xt.batch;
            LaySet set;
            set.add(t);
            if ((rc = launch_zero(xt.max, G * K, stream)) != GBMUF_OK || (rc = launch_stats(set, stream)) != GBMUF_OK || (rc = launch_lay(set, stream)) != GBMUF_OK) return rc;
        }
    }
    return each_piece(pieces, G, N, [&](const Piece &p) {
        const int32_t workers = static_cast<int32_t>(p.workers);
        const int64_t pld = (p.words + 63) / 64 * 64;
        const gbmuf_matrix_t wm = part(at.w, p.g, p.v, type);
        Operand px = x, pw = w;
        px.p += p.g * x.batch;
        if (px.max) px.max += p.g * x.max_batch;
        int r = GBMUF_OK;
        Operand pwt = wt;
        if (split) {
            // w along k, for the logits, and along the words, for dx, from one reading after its maxima are known
            LayArgs lw = source(wm, p.words, K, workers, type);
            const bool shared = lw.batch < workers;
            uint32_t *columns = max + p.workers * p.words;
            w_rows = columns + p.workers * K;
            pw.batch = shared ? 0 : p.words * w.ld;
            pw.max = lw.row_max = w_rows; pw.max_batch = shared ? 0 : p.words;
            lw.plain = const_cast<uint16_t *>(pw.p); lw.plain_ld = pw.ld; lw.plain_batch = pw.batch;
            if (dx) {
                pwt.ld = packed_words(p.words, true);
                pwt.batch = shared ? 0 : K * pwt.ld;
                pwt.max = lw.col_max = columns; pwt.max_batch = shared ? 0 : K;
                lw.trans = const_cast<uint16_t *>(pwt.p); lw.trans_ld = pwt.ld; lw.trans_batch = pwt.batch;
            }
            LaySet set;
            set.add(lw);
            if ((r = launch_zero(max, p.workers * (2 * p.words + K), stream)) != GBMUF_OK || (r = launch_stats(set, stream)) != GBMUF_OK ||
                (r = launch_lay(set, stream)) != GBMUF_OK)
                return r;
        } else if (copy_w) {
            const LayArgs lw = source(wm, p.words, K, workers, type);
            pw.batch = lw.batch < workers ? 0 : p.words * w.ld;
            if ((r = lay_rows(lw, pw, K, type, stream)) != GBMUF_OK) return r;
        } else pw = operand_of(wm);

        const Cut c = same_shape(shape, p.words, workers);
        LossArgs a = grad_args(l, at, io, words, p);
        a.lists = lists_from(lists, words, p.g);
        a.walk = c.t.steps;
        a.dz = dz; a.dz_ld = pld; a.dz_batch = M * pld;
        a.streamed = p.workers * M * pld * static_cast<int64_t>(type_bytes(type)) > kCached ? 1 : 0;
        if (!split) {
            a.most = most + p.g * kMostParts; a.most_parts = keep.most_parts;
            a.factor = factors + p.g;
        }
        if (db) a.col_sums = sums;
        if (split && dw) a.col_max = max;
        if ((r = launch_vocab(logits_args(px, pw, K, type, c), a, type, c.tile, true, stream)) != GBMUF_OK) return r;

        const gbmuf_matrix_t dzm{dz, pld, M * pld}, pdx = part(out.dx, p.g, 0, type), pdw = part(out.dw, p.g, p.v, grad_type),
                             pdb = vector_part(out.dbias, p.g, p.v, grad_type);
        const float *factor = split || M == 0 ? nullptr : factors + p.g;         // M: else nobody writes it
        SumArgs s{};
        s.sums = sums; s.out = pdb.data; s.out_batch = pdb.batch_stride;
        s.C = static_cast<int32_t>(p.words); s.tiles = 2 * c.t.tiles_m;
        s.batch = workers; s.type = grad_type; s.accumulate = l.accumulate;
        s.factor = factor;

        Operand oz{reinterpret_cast<const uint16_t *>(dz), pld, M * pld, nullptr, 0, false, false}, ozt = oz, ow = pw, ox = px;
        if (split) {
            oz = z; ozt = zt; ow = pwt; ox = xt;
            oz.ld = packed_words(p.words, true); oz.batch = M * oz.ld; oz.max = dz_rows + p.g * M; oz.max_batch = M;
            ozt.batch = p.words * ozt.ld; ozt.max = max; ozt.max_batch = p.words;
            ox.p += p.g * xt.batch; ox.max += p.g * xt.max_batch;
            LayArgs lz = source(dzm, M, p.words, workers, kF32);
            lz.batch = workers;
            if (dx) {
                lz.row_max = oz.max;
                lz.plain = const_cast<uint16_t *>(oz.p); lz.plain_ld = oz.ld; lz.plain_batch = oz.batch;
            }
            if (dw) {
                lz.col_max = ozt.max;
                lz.trans = const_cast<uint16_t *>(ozt.p); lz.trans_ld = ozt.ld; lz.trans_batch = ozt.batch;
            }
            LaySet lay;
            if (dx || dw) lay.add(lz);
            if ((r = launch_lay(lay, stream)) != GBMUF_OK) return r;
        } else {
            ozt.across = ow.across = ox.across = true;
        }
        if (db && (r = launch_column_sums(s, stream)) != GBMUF_OK) return r;
        if (dx) {
            const gbmuf_matrix_t to = several && !split ? gbmuf_matrix_t{dx_sums, K, M * K} : pdx;
            const int32_t to_type = several ? kF32 : type;
            Epilogue e = into(to, p.workers * M * K, to_type);
            e.factor = factor;
            if (p.v > 0) { e.place = GBMUF_RESIDUAL_AFTER; e.res = to.data; e.ldr = to.ld; e.r_batch = to.batch_stride; }
            if ((r = run_product(oz, ow, p.words, type, e, shape_of(M, K, p.words, p.workers, split), partial, stream)) != GBMUF_OK) return r;
            if (several && !split && p.v + p.words == N) {
                CastArgs cast{};
                cast.from = dx_sums; cast.out = pdx.data; cast.ld = pdx.ld; cast.batch_stride = pdx.batch_stride;
                cast.rows = static_cast<int32_t>(M); cast.columns = static_cast<int32_t>(K); cast.batch = workers; cast.type = type;
                if ((r = launch_cast(cast, stream)) != GBMUF_OK) return r;
            }
        }
        if (!dw) return r;
        Epilogue e = weight_grad(l, pdw, p.workers * p.words * K, grad_type);
        e.factor = factor;
        return run_product(ozt, ox, M, type, e, shape_of(p.words, K, M, p.workers, split), partial, stream);
    });
}

// Small sizes, whose dz is small too.
constexpr int64_t kSmallGrads = 64 << 20;
bool may_be_direct(const gbmuf_linear_desc_t &d) { return d.batch * d.rows * (d.out_features + 63) * 4 <= kSmallGrads; }

// f32 laid out takes the logits' product as well, 40 us or so more.  Directly / laid out, us: f32 1 x 1000 x 1000 x 1000 83 / 123, 6 x 130 x 18188 x 294 430 / 475, 8 x
// 128 x 2600 x 650 145 / 189; bf16 4 x 100 x 1000 x 256 30 / 42, 4 x 200 x 1024 x 512 52 / 43, 1 x 327 x 16183 x 190 124 / 66.
// dw's sums over the rows are not cut there: f32 1 x 2000 x 300 x 1000 109 / 113, 1 x 5000 x 300 x 200 181 / 98, 6 x 4835 x 219 x 142 383 / 165.
constexpr int64_t kDirectRows = 2500;
// The column sums go along with dw: what is asked for without it takes the other way.
int backward(const Loss &l, const Inputs &in, const gbmuf_loss_grad_io_t &io, Space &space, hipStream_t stream)
{
    const gbmuf_linear_desc_t &d = l.linear;
    gbmuf_linear_grad_io_t g{};
    g.x = in.x; g.w = in.w; g.dx = io.dx; g.dw = io.dw; g.dbias = io.dbias;
    g.dy = gbmuf_matrix_t{nullptr, 64, 0};               // dz lies well
    const bool sums = !io.dbias.data || (io.dw.data && d.in_features > 0);
    if (is_small(d) || is_few(d)) return backward_few(l, &in, &io, space, stream);
    const bool direct = d.out_features == 0 || (may_be_direct(d) && sums && d.rows <= kDirectRows && takes_direct_backward(d, g, d.dtype == GBMUF_F32 ? 40.0 : 0.0));
    return direct ? backward_direct(l, &in, &io, space, stream) : backward_laid(l, &in, &io, space, stream);
}

int64_t workspace_bytes(const Loss &l, bool back)
{
    if (!back) return forward_bytes(l);
    Space laid{nullptr}, direct{nullptr}, small{nullptr};
    (void)backward_laid(l, nullptr, nullptr, laid, nullptr);
    if (may_be_direct(l.linear)) (void)backward_direct(l, nullptr, nullptr, direct, nullptr);
    if (is_small(l.linear) || is_few(l.linear)) (void)backward_few(l, nullptr, nullptr, small, nullptr);
    return std::max({laid.used, direct.used, small.used});
}

// ---------------------------------------------------------------------------------------
// Checks
// ---------------------------------------------------------------------------------------
struct Extents {
    Extent x, w, bias, target, teacher;
};

bool valid_inputs(const Loss &l, const Inputs &in, Extents &e)
{
    const gbmuf_linear_desc_t &d = l.linear;
    const int64_t M = d.rows, N = d.out_features, K = d.in_features, G = d.batch, T = l.top;
    const int32_t t = d.dtype;
    e.x = extent(in.x, M, K, G, t); e.w = extent(in.w, N, K, G, t); e.bias = extent(in.bias, 1, N, G, t);
    e.target = extent(in.target, M, T ? T : 1, G, kI64);
    if (T) e.teacher = extent(in.teacher, M, T, G, kF32);
    return valid_input(in.x, e.x, t) && valid_input(in.w, e.w, t) && (!in.bias.data || valid_input(in.bias, e.bias, t)) && valid_input(in.target, e.target, kI64) &&
           (!T || valid_input(in.teacher, e.teacher, kF32));
}

bool meets_inputs(const Extent &o, const Extents &e)
{
    return overlap(o, e.x) || overlap(o, e.w) || overlap(o, e.bias) || overlap(o, e.target) || overlap(o, e.teacher);
}

int run_forward(const gbmuf_loss_desc_t *desc, const gbmuf_loss_io_t *io, void *workspace, int64_t workspace_bytes_, void *stream, bool distill)
{
    Loss l;
    int rc = check_desc(desc, distill, l);
    if (rc != GBMUF_OK) return rc;
    if (!io) return GBMUF_EINVAL;
    const int64_t M = l.linear.rows, G = l.linear.batch;
    const Inputs in{io->x, io->w, io->bias, io->target, io->teacher};
    Extents e;
    if (!valid_inputs(l, in, e)) return GBMUF_EINVAL;
    const Extent loss = extent(io->loss, M, 1, G, kF32), lse = extent(io->lse, M, 1, G, kF32);
    if (!valid_output(io->loss, loss, kF32) || (io->lse.data && !valid_output(io->lse, lse, kF32))) return GBMUF_EINVAL;
    if (meets_inputs(loss, e) || meets_inputs(lse, e) || overlap(loss, lse)) return GBMUF_EINVAL;
    if (M == 0 || G == 0) return GBMUF_OK;
    if ((rc = check_workspace(workspace, workspace_bytes_, workspace_bytes(l, false), {&e.x, &e.w, &e.bias, &e.target, &e.teacher, &loss, &lse})) != GBMUF_OK) return rc;
    if ((rc = check_device()) != GBMUF_OK) return rc;
    Space space{static_cast<char *>(workspace), workspace_bytes_};
    return forward(l, in, io, space, static_cast<hipStream_t>(stream));
}

int run_backward(const gbmuf_loss_desc_t *desc, const gbmuf_loss_grad_io_t *io, void *workspace, int64_t workspace_bytes_, void *stream, bool distill)
{
    Loss l;
    int rc = check_desc(desc, distill, l);
    if (rc != GBMUF_OK) return rc;
    if (!io) return GBMUF_EINVAL;
    const int64_t M = l.linear.rows, N = l.linear.out_features, K = l.linear.in_features, G = l.linear.batch;
    const int32_t t = l.linear.dtype, gt = l.weight_grad_f32 ? kF32 : t;
    const Inputs in{io->x, io->w, io->bias, io->target, io->teacher};
    Extents e;
    if (!valid_inputs(l, in, e)) return GBMUF_EINVAL;
    const Extent lse = extent(io->lse, M, 1, G, kF32), dloss = extent(io->dloss, M, 1, G, kF32);
    if (!valid_input(io->lse, lse, kF32) || !valid_input(io->dloss, dloss, kF32)) return GBMUF_EINVAL;
    const Extent dx = extent(io->dx, M, K, G, t), dw = extent(io->dw, N, K, G, gt), db = extent(io->dbias, 1, N, G, gt);
    if ((io->dx.data && !valid_output(io->dx, dx, t)) || (io->dw.data && !valid_output(io->dw, dw, gt)) || (io->dbias.data && !valid_output(io->dbias, db, gt)))
        return GBMUF_EINVAL;
    const Extent *outs[] = {&dx, &dw, &db};
    for (int i = 0; i < 3; ++i) {
        if (meets_inputs(*outs[i], e) || overlap(*outs[i], lse) || overlap(*outs[i], dloss)) return GBMUF_EINVAL;
        for (int j = 0; j < i; ++j)
            if (overlap(*outs[i], *outs[j])) return GBMUF_EINVAL;
    }
    if (G == 0) return GBMUF_OK;
    const int64_t need = workspace_bytes(l, true);
    if ((rc = check_workspace(workspace, workspace_bytes_, need, {&e.x, &e.w, &e.bias, &e.target, &e.teacher, &lse, &dloss, &dx, &dw, &db})) != GBMUF_OK) return rc;
    if ((rc = check_device()) != GBMUF_OK) return rc;
    if (!io->dx.data && !io->dw.data && !io->dbias.data) return GBMUF_OK;
    Space space{static_cast<char *>(workspace), workspace_bytes_};
    return backward(l, in, *io, space, static_cast<hipStream_t>(stream));
}

}  // namespace
}  // namespace gbmuf

using namespace gbmuf;

extern "C" {

int gbmuf_loss_workspace(const gbmuf_loss_desc_t *desc, int32_t backward_pass, int64_t *bytes)
{
    if (!bytes) return GBMUF_EINVAL;
    *bytes = 0;
    Loss l;
    const int rc = check_desc(desc, desc && desc->struct_size >= sizeof(gbmuf_loss_desc_t) && desc->top != 0, l);
    if (rc != GBMUF_OK) return rc;
    *bytes = workspace_bytes(l, backward_pass != 0);
    return GBMUF_OK;
}

int gbmuf_cross_entropy(const gbmuf_loss_desc_t *desc, const gbmuf_loss_io_t *io, void *workspace, int64_t workspace_bytes, void *stream)
{
    return run_forward(desc, io, workspace, workspace_bytes, stream, false);
}

int gbmuf_cross_entropy_backward(const gbmuf_loss_desc_t *desc, const gbmuf_loss_grad_io_t *io, void *workspace, int64_t workspace_bytes, void *stream)
{
    return run_backward(desc, io, workspace, workspace_bytes, stream, false);
}

int gbmuf_distill(const gbmuf_loss_desc_t *desc, const gbmuf_loss_io_t *io, void *workspace, int64_t workspace_bytes, void *stream)
{
    return run_forward(desc, io, workspace, workspace_bytes, stream, true);
}

int gbmuf_distill_backward(const gbmuf_loss_desc_t *desc, const gbmuf_loss_grad_io_t *io, void *workspace, int64_t workspace_bytes, void *stream)
{
    return run_backward(desc, io, workspace, workspace_bytes, stream, true);
}

}  // extern "C"
