// gbmuf_linear.hip -- entry points of the products with a model's matrices: checks, workspace, and which kernels run.
#include "gbmuf_products.h"

namespace gbmuf {
namespace {

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
