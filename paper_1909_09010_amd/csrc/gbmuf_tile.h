// gbmuf_tile.h -- how a tile of sums that 32 x 32 matrix instructions hold leaves a workgroup.
#pragma once

#include "gbmuf_values.h"

namespace gbmuf {
namespace {

typedef float v16f __attribute__((ext_vector_type(16)));

// Tile number id: down 8 tiles, then the next column, which keeps what workgroups side by side read small.
struct TileAt {
    int64_t g;
    int tm, tn;
};
__device__ __forceinline__ TileAt tile_at(const Tiles &t, int id)
{
    const int per = t.tiles_m * t.tiles_n;
    TileAt at;
    at.g = id / per;
    id -= static_cast<int>(at.g) * per;
    const int band = id / (8 * t.tiles_n), rows = min(8, t.tiles_m - band * 8), in = id - band * 8 * t.tiles_n;
    at.tm = band * 8 + in % rows;
    at.tn = in / rows;
    return at;
}

// What workgroup b does.
struct Share {
    TileAt at;
    int first, last;         // steps [first, last)
    float *part;             // a split tile's: where its part goes, row by row
};
template <int TM, int TN>
__device__ __forceinline__ Share share_of(const Tiles &t, int b, int all)
{
    // workgroups go to the 8 XCDs in turns: each XCD takes a stretch of tiles, whose operands its L2 holds
    const auto stretch = [](int i, int n) { return i < n / 8 * 8 ? (i & 7) * (n / 8) + (i >> 3) : i; };
    if (b < t.whole) return Share{tile_at(t, stretch(b, t.whole)), 0, all, nullptr};
    const int rest = t.rest(), i = stretch(b - t.whole, rest * t.splits), split = i / rest, tile = i - split * rest;
    Share s{tile_at(t, t.whole + tile), split * t.steps, min((split + 1) * t.steps, all), nullptr};
    if (t.splits > 1) s.part = t.partial + static_cast<int64_t>(i) * (TM * TN);
    return s;
}

// LDS that leave() needs: 32 rows of every wave's columns.
template <int TM, int TN, int WM, int WN>
constexpr size_t leave_bytes() { return static_cast<size_t>(WM) * WN * 32 * (TN / WN + 4) * sizeof(float); }

// A tile of TM x TN by WM x WN waves leaves through LDS, so that a wave's loads and stores follow rows: 128 bytes of a row of 16-bit results
// for 8 lanes.  Every wave turns its own part around, 32 rows at a time, in its own piece of LDS, whose accesses stay in order
// without a wait: all waves have to be past what LDS held before, and meet no more.  A lane holds, of row lane % 32 of acc[i][j], the columns 8 (r / 4)
// + 4 (lane / 32) + r % 4; afterwards 8 columns side by side, whose bias and scales it loads once.  (Tiles turned around by the
// whole workgroup, row by row, cost 7 us where these cost 2: bf16, 256 x 256.)
template <int TM, int TN, int WM, int WN, bool SPLIT, class Args>
__device__ __forceinline__ void leave(const v16f (&acc)[TM / WM / 32][TN / WN / 32], void *lds, const Args &a, const Share &share)
{
    const int64_t g = share.at.g;
    const int m0 = share.at.tm * TM, n0 = share.at.tn * TN, M = a.t.M, N = a.t.N;
    constexpr int FM = TM / WM / 32, FN = TN / WN / 32, kColumns = TN / WN, kPitch = kColumns + 4, kLanes = kColumns / 8, kTogether = 64 / kLanes,
                  kTurns = 32 / kTogether;
    static_assert(FM == 1 || FM == 2 || FM == 4, "the cases below");
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float *out = static_cast<float *>(lds) + wave * 32 * kPitch;
    const int column = lane % kLanes * 8, first = lane / kLanes, n = n0 + (wave / WM) * kColumns + column, left = N - n;
    const int mw = m0 + (wave % WM) * (TM / WM) + first;
    const Epilogue &e = a.e;
    const bool parts = share.part != nullptr, simple = !e.act && !e.pre;
    Eight bias{};
    int scale[SPLIT ? 8 : 1];
    if (left >= 8 && e.bias && !parts) bias = load_eight(e.bias, g * e.bias_batch + n, e.type);
    if constexpr (SPLIT)
#pragma unroll
        for (int c = 0; c < 8; ++c) scale[c] = row_exponent(a.b_max[g * a.b_max_batch + min(n + c, N - 1)]);
    const auto put = [&](const v16f (&rows)[FN]) {
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<v4f *>(out + (lane & 31) * kPitch + j * 32 + 8 * q + 4 * (lane >> 5)) =
                    v4f{rows[j][4 * q], rows[j][4 * q + 1], rows[j][4 * q + 2], rows[j][4 * q + 3]};
    };
    const auto get = [&](int k) {
        const float *from = out + (first + k * kTogether) * kPitch + column;
        return Eight{{*reinterpret_cast<const v4f *>(from), *reinterpret_cast<const v4f *>(from + 4)}};
    };
    const float factor = !SPLIT && e.factor && !parts ? e.factor[g] : 1.0f;
    const auto scaled = [&](Eight z, uint32_t row_bits) {
        if constexpr (!SPLIT) {
            z.v[0] *= factor;
            z.v[1] *= factor;
        }
        if constexpr (SPLIT) {
            const int em = row_exponent(row_bits);
#pragma unroll
            for (int c = 0; c < 8; ++c) z.v[c >> 2][c & 3] = ldexpf(z.v[c >> 2][c & 3], em + scale[c]);
        }
        z.v[0] += bias.v[0];
        z.v[1] += bias.v[1];
        return z;
    };
#pragma unroll 1
    for (int i = 0; i < FM; ++i) {                         // one copy of what follows: only the registers that are put differ
        const auto m_of = [&](int k) { return mw + i * 32 + k * kTogether; };
        uint32_t top[SPLIT ? kTurns : 1];
        if constexpr (SPLIT)
#pragma unroll
            for (int k = 0; k < kTurns; ++k) top[k] = a.a_max[g * a.a_max_batch + min(m_of(k), M - 1)];
        const auto fetch = [&](int k) { return load_eight(e.res, g * e.r_batch + min(m_of(k), M - 1) * e.ldr + n, e.type); };
        Eight r[kTurns] = {};
        if (e.place && !parts && left >= 8 && simple) {
#pragma unroll
            for (int k = 0; k < kTurns; ++k) r[k] = fetch(k);
        }
        if (i == 0) put(acc[0]);
        if constexpr (FM > 1)
            if (i == 1) put(acc[1]);
        if constexpr (FM > 2) {
            if (i == 2) put(acc[2]);
            if (i == 3) put(acc[3]);
        }
        if (parts) {                                       // as they are, the whole tile
#pragma unroll
            for (int k = 0; k < kTurns; ++k) write8<kF32>(share.part, static_cast<int64_t>(m_of(k) - m0) * TN + (n - n0), scaled(get(k), top[SPLIT ? k : 0]));
        } else if (left >= 8 && simple) {
            Eight z[kTurns];
#pragma unroll
            for (int k = 0; k < kTurns; ++k) z[k] = get(k);
#pragma unroll
            for (int k = 0; k < kTurns; ++k) {
                z[k] = scaled(z[k], top[SPLIT ? k : 0]);
                z[k].v[0] += r[k].v[0];
                z[k].v[1] += r[k].v[1];
                if (m_of(k) < M) store_result(e, e.y, g * e.y_batch + m_of(k) * e.ldy + n, z[k]);
            }
        } else if (left >= 8) {
            // two rows at a time (with tanh 430 us where one took 446, bf16, 4 x 5120 x 8192 x 1024; four do not fit the registers)
#pragma unroll 1
            for (int k0 = 0; k0 < kTurns; k0 += 2) {
                Eight z[2], q[2] = {};
                const auto m = [&](int u) { return mw + i * 32 + (k0 + u) * kTogether; };
                if (e.place)
#pragma unroll
                    for (int u = 0; u < 2; ++u) q[u] = fetch(k0 + u);
                const auto add = [&] {
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        z[u].v[0] += q[u].v[0];
                        z[u].v[1] += q[u].v[1];
                    }
                };
                const auto store = [&](void *to, int64_t batch, int64_t ld) {
#pragma unroll
                    for (int u = 0; u < 2; ++u)
                        if (m(u) < M) store_result(e, to, g * batch + m(u) * ld + n, z[u]);
                };
#pragma unroll
                for (int u = 0; u < 2; ++u) z[u] = get(k0 + u);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    uint32_t bits = top[0];
                    if constexpr (SPLIT)
#pragma unroll
                        for (int t = 1; t < kTurns; ++t) bits = k0 + u == t ? top[t] : bits;
                    z[u] = scaled(z[u], bits);
                }
                if (e.place == GBMUF_RESIDUAL_BEFORE) add();
                if (e.pre) store(e.pre, e.p_batch, e.ldp);
                activate_all(z, e.act);
                if (e.place == GBMUF_RESIDUAL_AFTER) add();
                store(e.y, e.y_batch, e.ldy);
            }
        } else if (left > 0) {                             // the last columns of a matrix: 4, and what is left
#pragma unroll 1
            for (int k = 0; k < kTurns * 2; ++k) {
                const int m = m_of(k >> 1), c0 = (k & 1) * 4, rest = left - c0;
                if (m >= M || rest <= 0) continue;
                v4f v = *reinterpret_cast<const v4f *>(out + (first + (k >> 1) * kTogether) * kPitch + column + c0);
                if constexpr (SPLIT) {
                    const int em = row_exponent(a.a_max[g * a.a_max_batch + m]);
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (c < rest) v[c] = ldexpf(v[c], em + row_exponent(a.b_max[g * a.b_max_batch + n + c0 + c]));
                }
                finish(e, g, m, n + c0, rest, v);
            }
        }
    }
}

}  // namespace
}  // namespace gbmuf
