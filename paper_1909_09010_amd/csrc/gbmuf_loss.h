// gbmuf_loss.h -- what follows a tile of logits that 32 x 32 matrix instructions hold, where rows are held to words: a row's part of the
// softmax statistics, or the logits' gradient.  The logits themselves never leave the workgroup.
#pragma once

#include "gbmuf_tile.h"

namespace gbmuf {
namespace {

constexpr float kLog2E = 1.44269504f;

__device__ __forceinline__ float exp2_of(float v) { return __builtin_amdgcn_exp2f(v); }

// What row m of worker g counts: kDead, kLive, or kBad where it names a word that the vocabulary does not have.
__device__ __forceinline__ int row_state(const Words &w, int64_t g, int m)
{
    if (!w.target) return w.state[g * w.rows + m];
    const int64_t t = w.target[g * w.batch + m * w.ld];
    return t < 0 ? kDead : t < w.vocab ? kLive : kBad;
}

// The words of a row as the teacher gives them, by one lane: f(word, share) for those that are there, in their order.
template <class F>
__device__ __forceinline__ void each_given(const Words &w, int64_t g, int m, float inv_tau, F f)
{
    const int64_t *ids = w.target + g * w.batch + m * w.ld;
    const float *logits = w.logit + g * w.logit_batch + m * w.logit_ld;
    const float inf = __builtin_inff();
    float most = -inf, total = 0.0f;
    for (int j = 0; j < w.top; ++j)
        if (ids[j] >= 0) most = fmaxf(most, logits[j]);
    const float from = most == -inf ? 0.0f : most;
    const auto term = [&](int j) { return ids[j] >= 0 && logits[j] != -inf ? expf((logits[j] - from) * inv_tau) : 0.0f; };
    for (int j = 0; j < w.top; ++j) total += term(j);
    for (int j = 0; j < w.top; ++j)
        if (ids[j] >= 0 && logits[j] != -inf) f(ids[j], term(j) / total);
}

__device__ __forceinline__ int given_state(const Words &w, int64_t g, int m)
{
    const int64_t *ids = w.target + g * w.batch + m * w.ld;
    const float *logits = w.logit + g * w.logit_batch + m * w.logit_ld;
    int state = kDead;
    for (int j = 0; j < w.top; ++j)
        if (ids[j] >= 0 && logits[j] != -__builtin_inff()) state = max(state, static_cast<int>(ids[j] < w.vocab ? kLive : kBad));
    return state;
}

// d loss / d logit of a row, up to what the row is held to: a row that does not count has none, whatever its dloss.
__device__ __forceinline__ float row_weight(const LossArgs &a, int64_t g, int m, int state)
{
    const float d = a.dloss[g * a.dloss_batch + m * a.dloss_ld] * a.tau;
    return state == kDead ? 0.0f : state == kLive ? d : __builtin_nanf("");
}

// Maximum of WIDTH neighbouring lanes.
template <int WIDTH>
__device__ __forceinline__ float max_of(float v)
{
#pragma unroll
    for (int d = 1; d < WIDTH; d *= 2) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}

// What 16-bit dz, no value of which exceeds the worker's largest weight, is multiplied with, and 1 / that: f16's range is filled from above, so that what a row has
// below 2^-39 of that weight is nothing; and -weight, which every row's own word has nearly, is a number of the type.  As it is, equal weights (1 / rows) would all be
// rounded the same way, by up to half a unit, and so would be the gradients: by 0.3 % for 895 rows in bf16.
template <int T>
__device__ __forceinline__ float2 dz_scale(float most)
{
    if (!(most > 0.0f)) return float2{1.0f, 1.0f};
    const int e = ilogbf(most), s = max(-112, min(126, (T == kF16 ? 14 : 0) - e));
    const float part = ldexpf(most, -e);                   // 1 .. 2
    return float2{ldexpf(1.0f / part, s), ldexpf(part, -s)};
}

// Two parts of a softmax's sum: (largest logit, sum of exp of the logits less that, or of themselves where that is infinite).
__device__ __forceinline__ float2 join_stats(float2 a, float2 b, float scale)
{
    const float most = fmaxf(a.x, b.x), inf = __builtin_inff(), from = fabsf(most) < inf ? most : 0.0f;
    const auto part = [&](float2 p) { return fabsf(p.x) < inf ? p.y * exp2_of((p.x - from) * scale) : p.y; };
    return float2{most, part(a) + part(b)};
}

// LDS of leave_loss: 32 rows of every wave's columns, and a row's statistics of every wave beside each other.
template <int TM, int TN, int WM, int WN>
constexpr size_t loss_bytes() { return leave_bytes<TM, TN, WM, WN>() + static_cast<size_t>(TM) * WN * sizeof(float2); }

// The wave's own LDS accesses are done in their order; this keeps the compiler to it.
__device__ __forceinline__ void in_order()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
}

// A tile of TM x TN logits by WM x WN waves; all waves are past what LDS held before.  A lane holds, of row lane % 32 of acc[i][j], the columns
// 8 (r / 4) + 4 (lane / 32) + r % 4, so that what belongs to a row is a lane's own, and its sums need one exchange between the two
// halves of the wave.  Words whose logits or shares are wanted are few (64 of 8197 words: 1 in 2 lanes and tile): their rows go through LDS, where a lane
// finds any column, only where the wave has one.
// Forward: (largest logit, sum of exp of the others less that) of every row of the tile, and the logits of the row's words.
// Backward: dz = weight (exp(z / tau - lse) - share) in f32, through LDS so that stores follow rows; its column sums go along with dw.
template <int TM, int TN, int WM, int WN, bool BACKWARD>
__device__ __forceinline__ void leave_loss(v16f (&acc)[TM / WM / 32][TN / WN / 32], void *lds, const Tiles &t, const LossArgs &a, const TileAt &tile)
{
    constexpr int FM = TM / WM / 32, FN = TN / WN / 32, kColumns = TN / WN, kPitch = kColumns + 4;
    const int64_t g = tile.g;
    const int M = t.M, N = t.N, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    const int m_wave = tile.tm * TM + (wave % WM) * (TM / WM), n_wave = tile.tn * TN + (wave / WM) * kColumns;
    const bool whole = n_wave + kColumns <= N;
    float *out = static_cast<float *>(lds) + wave * 32 * kPitch;
    float2 *stats = reinterpret_cast<float2 *>(static_cast<char *>(lds) + leave_bytes<TM, TN, WM, WN>());
    const auto row_of = [&](int i) { return m_wave + i * 32 + (lane & 31); };

    v4f bias[FN][4];
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int n = n_wave + j * 32 + q * 8 + half * 4;
            const int64_t at = g * a.bias_batch + n;
            v4f b = {0.0f, 0.0f, 0.0f, 0.0f};
            if (a.bias) {
                if (whole) b = load_four(a.bias, at, a.type);
                else
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (n + c < N) b[c] = load_one(a.bias, at + c, a.type);
            }
            bias[j][q] = b;
        }

    // the words of each of the lane's rows: where the list of them reaches this wave's columns
    const int lo = a.first + n_wave, hi = a.first + min(n_wave + kColumns, N);
    const Words &w = a.words;
    int place[FM], word[FM], state[FM];
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const int m = min(row_of(i), M - 1);
        state[i] = kLive;
        if (BACKWARD) state[i] = row_of(i) < M ? row_state(w, g, m) : kDead;
        place[i] = 0;
        word[i] = kNoWord;
        if (w.target) {
            const int64_t at = w.target[g * w.batch + m * w.ld];
            word[i] = at >= lo && at < hi && row_of(i) < M ? static_cast<int>(at) : kNoWord;
        }
    }
    const auto list = [&](int i) { return w.id + (g * w.rows + min(row_of(i), M - 1)) * w.top; };
    if (!w.target) {
        int step = 1;
        while (2 * step <= w.top) step *= 2;
        for (; step; step >>= 1)
#pragma unroll
            for (int i = 0; i < FM; ++i)
                if (place[i] + step <= w.top && list(i)[place[i] + step - 1] < lo) place[i] += step;
#pragma unroll
        for (int i = 0; i < FM; ++i)
            if (place[i] < w.top && row_of(i) < M) {
                word[i] = list(i)[place[i]];
                word[i] = word[i] < hi ? word[i] : kNoWord;
            }
    }
    const auto next = [&](int i) {                          // the row's next word in these columns
        int n = kNoWord;
        if (!w.target && ++place[i] < w.top) {
            n = list(i)[place[i]];
            n = n < hi ? n : kNoWord;
        }
        word[i] = n;
    };
    const auto put = [&](const v16f (&rows)[FN]) {
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<v4f *>(out + (lane & 31) * kPitch + j * 32 + 8 * q + 4 * half) =
                    v4f{rows[j][4 * q], rows[j][4 * q + 1], rows[j][4 * q + 2], rows[j][4 * q + 3]};
    };

    const float scale = a.inv_tau * kLog2E;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const int m = row_of(i), mc = min(m, M - 1);
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] += bias[j][r >> 2][r & 3];
        if (!whole)
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (n_wave + j * 32 + (r >> 2) * 8 + half * 4 + (r & 3) >= N) acc[i][j][r] = -__builtin_inff();
        if constexpr (!BACKWARD) {
            float most = acc[i][0][0];
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) most = fmaxf(most, acc[i][j][r]);
            most = fmaxf(most, __shfl_xor(most, 32));
            // from an infinite logit nothing is taken away: it makes the sum infinite, or is nothing of it
            const float from = fabsf(most) < __builtin_inff() ? most : 0.0f;
            float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) sum[r & 3] += exp2_of((acc[i][j][r] - from) * scale);
            float s = (sum[0] + sum[1]) + (sum[2] + sum[3]);
            s += __shfl_xor(s, 32);
            if (half == 0) stats[(wave / WM) * TM + (wave % WM) * (TM / WM) + i * 32 + lane] = float2{most, s};
            if (__any(word[i] != kNoWord)) {
                in_order();
                put(acc[i]);
                in_order();
                float *to = a.at + (g * w.rows + mc) * w.top;
                while (word[i] != kNoWord) {
                    if (half == 0) to[place[i]] = out[(lane & 31) * kPitch + word[i] - lo];
                    next(i);
                }
                in_order();
            }
        } else {
            constexpr int kLanes = kColumns / 8, kTogether = 64 / kLanes, kTurns = 32 / kTogether;
            const float lse = a.lse[g * a.lse_batch + mc * a.lse_ld];
            const float weight = row_weight(a, g, mc, state[i]);
            if (a.live && tile.tn == 0 && wave / WM == 0 && half == 0 && m < M) a.live[g * w.rows + m] = state[i];
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float p = weight * exp2_of(fmaf(acc[i][j][r], a.inv_tau, -lse) * kLog2E);
                    acc[i][j][r] = state[i] == kDead ? 0.0f : p;
                }
            in_order();
            put(acc[i]);
            in_order();
            while (word[i] != kNoWord) {                    // in the list's order, by one lane
                if (half == 0) {
                    float *at = out + (lane & 31) * kPitch + word[i] - lo;
                    const float share = w.target ? 1.0f : w.share[(g * w.rows + mc) * w.top + place[i]];
                    if (state[i] != kDead) *at -= weight * share;
                }
                next(i);
            }
            in_order();
            const int column = lane % kLanes * 8, first = lane / kLanes, n = n_wave + column;
#pragma unroll
            for (int k = 0; k < kTurns; ++k) {
                const float *from = out + (first + k * kTogether) * kPitch + column;
                const Eight z{{*reinterpret_cast<const v4f *>(from), *reinterpret_cast<const v4f *>(from + 4)}};
                const int row = m_wave + i * 32 + first + k * kTogether;
                if (row < M && n < a.dz_ld) write8<kF32>(a.dz, g * a.dz_batch + row * a.dz_ld + n, z);
            }
            in_order();
        }
    }
}

// A tile's statistics, joined over its waves side by side; for all THREADS of the workgroup, which have met since.
template <int TM, int TN, int WM, int WN, int THREADS>
__device__ __forceinline__ void store_parts(const void *lds, const Tiles &t, const LossArgs &a, const TileAt &tile)
{
    const float2 *stats = reinterpret_cast<const float2 *>(static_cast<const char *>(lds) + leave_bytes<TM, TN, WM, WN>());
    for (int r = threadIdx.x; r < TM; r += THREADS) {
        const int m = tile.tm * TM + r;
        if (m >= t.M) continue;
        float2 s = stats[r];
#pragma unroll
        for (int v = 1; v < WN; ++v) s = join_stats(s, stats[v * TM + r], a.inv_tau * kLog2E);
        a.parts[(tile.g * a.part_tiles + a.first_tile + tile.tn) * a.words.rows + m] = s;
    }
}

}  // namespace
}  // namespace gbmuf
