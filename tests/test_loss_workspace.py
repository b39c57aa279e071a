"""What calls of the losses take of their workspace, held against what the query says.  The entry points' own host code, compiled with launches that run
nothing: each looks where its kernel would read and write, over random descriptions and placements."""
import os
import subprocess

import pytest

from paper_1909_09010_amd import build

PROGRAM = r"""
#include "gbmuf_loss.hip"
#include <random>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

namespace {

// Addresses of matrices lie below the workspace's, far apart; nothing is behind the workspace.
constexpr uintptr_t kSpace = uintptr_t{1} << 56;
int64_t have = 0, reached = 0;
const char *worst = "";
long launches = 0;

// n bytes from p on, if p is the workspace's
void uses(const void *p, int64_t n, const char *what)
{
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    if (at < kSpace || n <= 0) return;
    const int64_t end = static_cast<int64_t>(at - kSpace) + n;
    if (end > reached) {
        reached = end;
        worst = what;
    }
}

// `batch` matrices of rows of `row` values
void matrix(const void *p, int64_t batch, int64_t stride, int64_t rows, int64_t ld, int64_t row, int64_t bytes, const char *what)
{
    if (batch > 0 && rows > 0 && row > 0) uses(p, ((batch - 1) * stride + (rows - 1) * ld + row) * bytes, what);
}

void see_words(const gbmuf::Words &w, int64_t batch)
{
    const int64_t rows = batch * w.rows;
    uses(w.id, rows * w.top * 4, "words");
    uses(w.share, rows * w.top * 4, "shares");
    uses(w.state, rows * 4, "states");
}

void tiles(const gbmuf::Tiles &t, int tile)
{
    if (t.splits > 1) uses(t.partial, static_cast<int64_t>(t.rest()) * t.splits * tile * tile * 4, "parts of tiles");
}

// along: dz lies along the sum, else across it
void direct(const gbmuf::DirectArgs &a, bool along)
{
    tiles(a.t, 64);
    matrix(a.a.p, a.t.batch, a.a.batch, along ? a.t.M : a.K, a.a.ld, along ? a.K : a.t.M, 4, "dz");
    uses(a.live, a.t.batch * a.live_batch * 4, "live");
}

void see_lists(const gbmuf::WordLists &l, const gbmuf::Words &w, int64_t batch)
{
    const int64_t n = batch * l.blocks * l.block_rows * w.top;
    uses(l.code, n * 4, "codes");
    uses(l.share, n * 4, "shares of codes");
    uses(l.starts, batch * l.blocks * (l.windows + 1) * 4, "starts");
}

void laid(const gbmuf::LaySet &set, bool write)
{
    for (int i = 0; i < set.n; ++i) {
        const gbmuf::LayArgs &a = set.a[i];
        matrix(a.src, a.batch, a.batch_stride, a.R, a.ld, a.C, 4, "what is laid out");
        uses(a.row_max, static_cast<int64_t>(a.batch) * a.R * 4, "rows' largest");
        uses(a.col_max, static_cast<int64_t>(a.batch) * a.C * 4, "columns' largest");
        if (!write) continue;
        matrix(a.plain, a.batch, a.plain_batch, a.R, a.plain_ld, a.plain_ld, 2, "rows laid out");
        matrix(a.trans, a.batch, a.trans_batch, a.C, a.trans_ld, a.trans_ld, 2, "columns laid out");
    }
    ++launches;
}

void operand(const uint16_t *p, int64_t batch, int64_t stride, int64_t rows, int64_t ld, int64_t K, const uint32_t *max, int64_t max_batch, int64_t max_rows)
{
    matrix(p, batch, stride, rows, ld, K, 2, "an operand");
    if (max) matrix(max, batch, max_batch, 1, 0, max_rows, 4, "an operand's largest");
}

}  // namespace

namespace gbmuf {

int hip_failed(const char *, hipError_t, int status) { return status; }

int launch_product(const ProductArgs &a, int32_t, int tile, hipStream_t)
{
    ++launches;
    const Tiles &t = a.t;
    tiles(t, tile);
    const bool ax = a.across & 1, bx = a.across & 2;
    operand(a.a, t.batch, a.a_batch, ax ? a.K : t.M, a.lda, ax ? t.M : a.K, a.a_max, a.a_max_batch, t.M);
    operand(a.b, t.batch, a.b_batch, bx ? a.K : t.N, a.ldb, bx ? t.N : a.K, a.b_max, a.b_max_batch, t.N);
    matrix(a.e.y, t.batch, a.e.y_batch, t.M, a.e.ldy, t.N, type_bytes(a.e.type), "a product");
    uses(a.e.factor, t.batch * 4, "factors");
    return GBMUF_OK;
}
int launch_join(const JoinArgs &a, hipStream_t) { ++launches; tiles(a.t, a.tile); return GBMUF_OK; }
int launch_rows(const LaySet &s, hipStream_t) { laid(s, true); return GBMUF_OK; }
int launch_stats(const LaySet &s, hipStream_t) { laid(s, false); return GBMUF_OK; }
int launch_lay(const LaySet &s, hipStream_t) { laid(s, true); return GBMUF_OK; }
int launch_copy(const LaySet &s, hipStream_t) { laid(s, true); return GBMUF_OK; }
int launch_few(const DirectArgs &, int32_t, hipStream_t) { abort(); }
int launch_direct_forward(const DirectArgs &, hipStream_t) { abort(); }
int launch_direct_backward(const DirectArgs &, const DirectArgs &, int32_t, hipStream_t) { abort(); }
int launch_column_sums(const SumArgs &a, hipStream_t)
{
    ++launches;
    uses(a.sums, static_cast<int64_t>(a.batch) * a.tiles * a.C * 4, "sums of columns");
    return GBMUF_OK;
}
int launch_vocab(const ProductArgs &a, const LossArgs &l, int32_t type, int tile, bool backward, hipStream_t)
{
    ++launches;
    const Tiles &t = a.t;
    if (t.count() <= 0) return GBMUF_OK;
    const int64_t edge = type == kF32 ? (static_cast<int64_t>(t.N) + tile - 1) / tile * tile : t.N;       // scales are read up to the tile's end
    operand(a.a, t.batch, a.a_batch, t.M, a.lda, a.K, a.a_max, a.a_max_batch, t.M);
    operand(a.b, t.batch, a.b_batch, t.N, a.ldb, a.K, a.b_max, a.b_max_batch, edge);
    see_words(l.words, t.batch);
    if (l.lists.blocks > 0) see_lists(l.lists, l.words, t.batch);
    if (!backward) {
        uses(l.parts, ((t.batch - 1) * static_cast<int64_t>(l.part_tiles) + l.first_tile + t.tiles_n) * l.words.rows * 8, "parts of rows");
        if (l.first_tile + t.tiles_n > l.part_tiles) reached = INT64_MAX, worst = "a part that no row has";
        uses(l.at, t.batch * static_cast<int64_t>(l.words.rows) * l.words.top * 4, "words' logits");
    } else {
        matrix(l.dz, t.batch, l.dz_batch, t.M, l.dz_ld, l.dz_ld, type_bytes(type), "dz");
        uses(l.col_sums, static_cast<int64_t>(t.batch) * t.tiles_m * 2 * t.N * 4, "sums of columns");
        uses(l.col_max, static_cast<int64_t>(t.batch) * t.N * 4, "columns' largest");
        uses(l.factor, t.batch * 4, "factors");
        uses(l.most, ((t.batch - 1) * kMostParts + l.most_parts) * 4, "largest weights");
    }
    return GBMUF_OK;
}
int launch_loss_few(const DirectArgs &a, const LossArgs &l, int32_t type, hipStream_t)
{
    ++launches;
    see_words(l.words, a.t.batch);
    const int64_t columns = few_columns(a, type), n = (a.t.N + columns - 1) / columns;
    if (n != l.part_tiles) reached = INT64_MAX, worst = "a part that no row has";
    uses(l.parts, a.t.batch * n * l.words.rows * 8, "parts of rows");
    uses(l.at, a.t.batch * static_cast<int64_t>(l.words.rows) * l.words.top * 4, "words' logits");
    return GBMUF_OK;
}
int launch_loss_direct(const DirectArgs &a, const LossArgs &l, int32_t, bool backward, hipStream_t)
{
    ++launches;
    see_words(l.words, a.t.batch);
    if (backward) {
        matrix(l.dz, a.t.batch, l.dz_batch, a.t.M, l.dz_ld, l.dz_ld, 4, "dz");
        uses(l.live, a.t.batch * static_cast<int64_t>(l.words.rows) * 4, "live");
        return GBMUF_OK;
    }
    if (a.t.tiles_n != l.part_tiles) reached = INT64_MAX, worst = "a part that no row has";
    uses(l.parts, a.t.batch * static_cast<int64_t>(l.part_tiles) * l.words.rows * 8, "parts of rows");
    uses(l.at, a.t.batch * static_cast<int64_t>(l.words.rows) * l.words.top * 4, "words' logits");
    return GBMUF_OK;
}
int launch_loss_grads(const DirectArgs &dx, const DirectArgs &dw, int32_t, hipStream_t) { ++launches; direct(dx, true); direct(dw, false); return GBMUF_OK; }
int launch_small_grads(const SmallGrads &a, hipStream_t stream) { ++launches; see_words(a.l.words, a.batch); return launch_join_parts(a, a.pieces, stream); }
int launch_few_grads(const SmallGrads &a, int32_t, hipStream_t) { ++launches; see_words(a.l.words, a.batch); return GBMUF_OK; }
int launch_join_parts(const SmallGrads &a, int32_t parts, hipStream_t)
{
    ++launches;
    uses(a.parts, static_cast<int64_t>(parts) * a.batch * a.l.words.rows * a.columns * 4, "parts of dx");
    return GBMUF_OK;
}
int launch_teacher(const TeacherArgs &a, hipStream_t)
{
    ++launches;
    const int64_t rows = static_cast<int64_t>(a.rows) * a.batch;
    uses(a.out_id, rows * a.top * 4, "words");
    uses(a.out_share, rows * a.top * 4, "shares");
    uses(a.out_state, rows * 4, "states");
    return GBMUF_OK;
}
int launch_word_lists(const Words &w, const WordLists &l, int32_t batch, hipStream_t) { ++launches; see_words(w, batch); see_lists(l, w, batch); return GBMUF_OK; }
int launch_loss_join(const LossJoin &a, hipStream_t)
{
    ++launches;
    see_words(a.words, a.batch);
    uses(a.parts, static_cast<int64_t>(a.batch) * a.tiles * a.words.rows * 8, "parts of rows");
    uses(a.at, static_cast<int64_t>(a.batch) * a.words.rows * a.words.top * 4, "words' logits");
    return GBMUF_OK;
}
int launch_keep(const KeepArgs &a, hipStream_t)
{
    ++launches;
    const int64_t rows = static_cast<int64_t>(a.words.rows) * a.batch;
    if (!a.all) see_words(a.words, a.batch);
    uses(a.out, rows * a.out_ld * type_bytes(a.type), "rows that are kept");
    uses(a.row_max, rows * 4, "rows' largest");
    if (a.most) uses(a.most, static_cast<int64_t>(a.batch) * kMostParts * 4, "largest weights");
    return GBMUF_OK;
}
int launch_cast(const CastArgs &a, hipStream_t) { ++launches; uses(a.from, static_cast<int64_t>(a.batch) * a.rows * a.columns * 4, "sums of dx"); return GBMUF_OK; }
int launch_zero(uint32_t *p, int64_t words, hipStream_t) { ++launches; uses(p, words * 4, "zeros"); return GBMUF_OK; }

}  // namespace gbmuf

extern "C" hipError_t hipGetDeviceCount(int *n) { *n = 1; return hipSuccess; }

namespace {

struct Lies {
    bool well, shared;
};

// A matrix of its own, whose rows lie on 16 bytes or do not.
gbmuf_matrix_t place(int number, int64_t rows, int64_t cols, int64_t batch, int64_t bytes, Lies lies)
{
    gbmuf_matrix_t m{};
    const int64_t ld = lies.well ? (cols + 15) / 16 * 16 : cols + 1 - (cols & 1);       // odd
    m.data = reinterpret_cast<void *>((static_cast<uintptr_t>(number) << 50) + (lies.well ? 0 : bytes));
    m.ld = ld;
    m.batch_stride = lies.shared ? 0 : rows * ld + (lies.well ? 0 : 1);
    return m;
}

struct Call {
    int64_t G, M, V, K, top;
    int32_t dtype;
    bool backward, dx, dw, db, f32_grads, accumulate;
    Lies x, w;
};

int failed = 0;
long accepted = 0;

void run(const Call &c)
{
    gbmuf_loss_desc_t d{};
    d.struct_size = sizeof(d);
    d.dtype = c.dtype; d.batch = static_cast<int32_t>(c.G); d.top = static_cast<int32_t>(c.top);
    d.weight_grad_f32 = c.f32_grads; d.accumulate = c.accumulate;
    d.temperature = 2.0f;
    d.rows = c.M; d.vocab = c.V; d.in_features = c.K;
    if (gbmuf_loss_workspace(&d, c.backward, &have) != GBMUF_OK) return;
    const int64_t b = c.dtype == GBMUF_F32 ? 4 : 2, gb = c.f32_grads ? 4 : b, T = c.top ? c.top : 1;
    const Lies well{true, false};
    reached = 0;
    worst = "";
    void *space = reinterpret_cast<void *>(kSpace);
    const gbmuf_matrix_t x = place(1, c.M, c.K, c.G, b, c.x), w = place(2, c.V, c.K, c.G, b, c.w), bias = place(3, 1, c.V, c.G, b, well),
                         target = place(4, c.M, T, c.G, 8, well), teacher = place(5, c.M, T, c.G, 4, well), lse = place(6, c.M, 1, c.G, 4, well),
                         loss = place(7, c.M, 1, c.G, 4, well);
    int rc;
    if (!c.backward) {
        gbmuf_loss_io_t io{x, w, bias, target, c.top ? teacher : gbmuf_matrix_t{}, loss, lse};
        rc = (c.top ? gbmuf_distill : gbmuf_cross_entropy)(&d, &io, space, have, nullptr);
    } else {
        gbmuf_loss_grad_io_t io{x, w, bias, target, c.top ? teacher : gbmuf_matrix_t{}, lse, loss, {}, {}, {}};
        if (c.dx) io.dx = place(8, c.M, c.K, c.G, b, well);
        if (c.dw) io.dw = place(9, c.V, c.K, c.G, gb, well);
        if (c.db) io.dbias = place(10, 1, c.V, c.G, gb, well);
        rc = (c.top ? gbmuf_distill_backward : gbmuf_cross_entropy_backward)(&d, &io, space, have, nullptr);
    }
    ++accepted;
    if (rc == GBMUF_OK && reached <= have) return;
    if (++failed <= 20)
        printf("%s type %d, %ld x %ld x %ld x %ld, top %ld, x %s%s, w %s%s: status %d, %s end %ld bytes behind the %ld\n", c.backward ? "backward" : "forward", c.dtype,
               static_cast<long>(c.G), static_cast<long>(c.M), static_cast<long>(c.V), static_cast<long>(c.K), static_cast<long>(c.top), c.x.well ? "well" : "badly",
               c.x.shared ? " shared" : "", c.w.well ? "well" : "badly", c.w.shared ? " shared" : "", rc, worst, static_cast<long>(reached - have), static_cast<long>(have));
}

}  // namespace

int main(int argc, char **argv)
{
    if (argc == 8) {                      // one size, however it lies
        for (int i = 0; i < 32; ++i)
            run(Call{atoll(argv[2]), atoll(argv[3]), atoll(argv[4]), atoll(argv[5]), atoll(argv[6]), atoi(argv[7]), argv[1][0] == 'b', true, true, true, false, false,
                     {(i & 1) != 0, (i & 2) != 0}, {(i & 4) != 0, (i & 8) != 0}});
    } else {
        std::mt19937_64 random(atoll(argv[2]));
        const auto unit = [&] { return static_cast<double>(random() >> 11) * 0x1p-53; };
        const auto log = [&](double most) { return static_cast<int64_t>(exp(unit() * ::log(most))); };
        const auto coin = [&](double p) { return unit() < p; };
        for (long i = atoll(argv[1]); i > 0; --i) {
            Call c{};
            c.G = log(70.0); c.M = log(4e6); c.V = log(3e5); c.K = log(9000.0);
            if (coin(0.3)) c.M = log(100.0);
            c.top = coin(0.5) ? 0 : log(1025.0);
            c.dtype = static_cast<int32_t>(random() % 3);
            c.backward = coin(0.5);
            c.dx = coin(0.7); c.dw = coin(0.7); c.db = coin(0.7);
            c.f32_grads = coin(0.5); c.accumulate = coin(0.5);
            c.x = {coin(0.5), coin(0.2)}; c.w = {coin(0.5), coin(0.2)};
            run(c);
        }
    }
    printf("%ld calls, %ld launches, %d short\n", accepted, launches, failed);
    return failed ? 1 : 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    at = tmp_path_factory.mktemp("workspace")
    src, exe = at / "workspace.cpp", at / "workspace"
    src.write_text(PROGRAM)
    pkg = os.path.dirname(build.CSRC)
    subprocess.run(["g++", "-std=c++17", "-O2", "-D__HIP_PLATFORM_AMD__", "-I", build.CSRC, "-I/opt/rocm/include", "-o", str(exe), "-x", "c++", str(src), "-x", "none",
                    "-L" + pkg, "-lgbmuf", "-Wl,-rpath," + pkg, "-Wl,-rpath,/opt/rocm/lib"], check=True)
    return str(exe)


def holds(program, *args):
    got = subprocess.run([program, *map(str, args)], capture_output=True, text=True)
    assert got.returncode == 0, got.stdout[-4000:] + got.stderr[-2000:]
    return got.stdout


@pytest.mark.parametrize("seed", range(4))
def test_no_call_takes_more_than_the_query_says(program, seed):
    calls = int(holds(program, 60000, seed).split()[0])
    assert calls > 15000


# 16-bit w that fits no piece of what is laid out at a time, and walks fewer tiles where it is taken as it lies; workers, rows, words, features, the teacher's words
@pytest.mark.parametrize("size", [(13, 77558, 7703, 2632, 0), (2, 128542, 20177, 7200, 0), (15, 48994, 13551, 4616, 0), (4, 176334, 45503, 4357, 8),
                                  (1, 300, 70000, 2050, 0), (2, 64, 50000, 4096, 3), (3, 65, 50000, 4096, 17)])
@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_wide_matrices_however_they_lie(program, size, dtype):
    for backward in "fb":
        holds(program, backward, *size, dtype)


@pytest.mark.gpu
def test_a_wide_forward_stays_in_its_workspace():
    """bf16: as many parts as a w has that is taken as it lies, x laid out behind them; the bits are those of an x that lies well."""
    import torch
    from paper_1909_09010_amd import binding as B
    G, M, V, K = 13, 77558, 7703, 2632
    dev, t = "cuda:0", torch.bfloat16
    g = torch.Generator(device=dev).manual_seed(5)
    buf = torch.empty(G * M * K + 1, dtype=t, device=dev)
    crooked = buf[1:].view(G, M, K)
    for x in crooked:
        x.normal_(generator=g)
    w = torch.empty(G, V, K, dtype=t, device=dev).normal_(std=2 * K ** -0.5, generator=g)
    target = torch.randint(0, V, (G, M), generator=g, device=dev)
    op = B.CrossEntropy(M, V, K, G, t)
    need = op.workspace_bytes()
    ws = torch.empty(need + (1 << 26), dtype=torch.uint8, device=dev)
    ws[need:] = 17
    out = []
    for x in (crooked, crooked.clone()):
        loss = torch.empty(G, M, device=dev)
        op.forward(op.forward_io(x, w, target, loss), ws[:need])
        out.append(loss)
    torch.cuda.synchronize()
    assert torch.equal(*out) and torch.isfinite(out[0]).all()
    assert (ws[need:] == 17).all()
