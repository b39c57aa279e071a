// gbmuf_vocab.hip -- logits of many rows against a large vocabulary on gfx950's matrix cores, and what losses make of them: out = a b' is never
// written.
#include "gbmuf_loss.h"
#include "gbmuf_stage.h"

namespace gbmuf {
namespace {

// 32 x 32 values of a wave on their way between lanes that hold a row and lanes that hold 8 columns: the 16-byte chunk c of row r at place
// c ^ ((r / 2) & 7), so that 16 lanes meet all banks both ways.
typedef uint32_t v4u_any __attribute__((ext_vector_type(4), aligned(4)));
constexpr float kPlain = 65536.0f;       // up to here the rounding of what an exponent subtracts is a small one
constexpr int kScratch = 32 * 32;
__device__ __forceinline__ int scratch_at(int r, int c) { return r * 32 + (((c >> 2) ^ ((r >> 1) & 7)) << 2) + (c & 3); }

// Keeps what two branches end with from becoming one, with everything that either computes done for both.
template <int N>
__device__ __forceinline__ void apart() { asm volatile("; %0" ::"n"(N)); }

// Sends R rows of one step to LDS as Stage does.  Where the rows are is worked out for every step from one address a lane: Stage's addresses, kept over the
// steps of all tiles beside statistics and sums, would go to memory and back.
template <int R, int THREADS>
struct Sender {
    static constexpr int kPass = THREADS / 8, kPasses = R / kPass;
    static_assert(kPass % 16 == 0, "a thread's chunk lies at the same place in every pass");
    const uint16_t *base;        // of the matrix
    int64_t ld;
    int first, count;

    // whatever is derived from this number is derived anew
    __device__ __forceinline__ static int thread()
    {
        int t = threadIdx.x;
        asm volatile("" : "+v"(t));
        return t;
    }
    __device__ __forceinline__ static int chunk(int t) { return ((t & 7) ^ ((t >> 4) & 7)) * 8; }

    // rows behind the last are read as the last one
    __device__ __forceinline__ void load(uint16_t *lds, int k0) const
    {
        const int t = thread(), r = t >> 3;
        const uint16_t *at = base + k0 + chunk(t);
        uint16_t *to = lds + static_cast<int>(threadIdx.x >> 6) * 8 * kStep;
        const auto send = [&](int i, const uint16_t *from) {
            __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) void *)from,
                                             (__attribute__((address_space(3))) void *)(to + i * kPass * kStep), 16, 0, 0);
        };
        if (first + R <= count) {
            at += static_cast<int64_t>(first + r) * ld;
#pragma unroll
            for (int i = 0; i < kPasses; ++i) send(i, at + i * kPass * ld);
        } else {
#pragma unroll
            for (int i = 0; i < kPasses; ++i) send(i, at + static_cast<int64_t>(min(first + r + i * kPass, count - 1)) * ld);
        }
    }

    __device__ __forceinline__ void load_rest(uint16_t *lds, int k0, int K) const
    {
        const int t = thread(), r = t >> 3, left = K - (k0 + chunk(t));
#pragma unroll 1
        for (int i = 0; i < kPasses; ++i) {
            uint32_t v[4] = {0u, 0u, 0u, 0u};
            const uint16_t *from = base + static_cast<int64_t>(min(first + r + i * kPass, count - 1)) * ld + k0 + chunk(t);
            if (left >= 8) {                               // rows lie on 16 bytes
                const v4u all = *reinterpret_cast<const v4u *>(from);
                for (int c = 0; c < 4; ++c) v[c] = all[c];
            } else {
#pragma unroll
                for (int c = 0; c < 7; ++c)
                    if (c < left) v[c >> 1] |= static_cast<uint32_t>(from[c]) << (16 * (c & 1));
            }
            *reinterpret_cast<v4u *>(lds + (i * kPass + r) * kStep + (t & 7) * 8) = v4u{v[0], v[1], v[2], v[3]};
        }
    }
};

// A workgroup takes one block of TM rows and walks `walk` tiles of TN words, as one stream of steps: while a tile is left the first two steps of the
// next are on their way, so that only the arithmetic of leaving is paid.  Everything that a row needs is a lane's own (leave_loss): its statistics
// stay in registers over all of the tiles, and lse and weight are loaded once.
// Forward, per logit: a maximum, a multiply-add, an exponential and an addition.  Backward: a multiply-add, an exponential, a product, a choice of 0 in rows that do not
// count, whose logits may be no numbers (0.3 %: 2 x 5120 x 50000 x 1024 bf16 3134 us, 3124 without), and its way through LDS to where a row's 16 bytes leave together.
// Bounds: the steps, and what leaving a tile takes between them, when the matrix cores wait: a tile of 256 x 256 bf16 has steps of 1.73 us and leaves in 3.5 us
// forward, so that 512 features are 8 steps and a fifth of leaving.  A whole call, bf16 8 x 5120 x 8197 x 512: 362 us, 0.95 PFLOP/s where large products reach
// 1.31.  Tiles of 128 have two workgroups on a CU, one's leaving beside the other's steps, but twice the LDS reads a product: the caller's rule compares rounds
// of both.  f32, taken apart into two f16, has tiles of 128 only: those of 256 leave too few registers for the statistics (8 x 700 x 10000 x 650: 436 us, 333).
// Backward the stores share the way to memory with the steps' operands: dz of 8 x 5120 x 8197 x 512 bf16 takes 555 to 585 us, without them 460.  Registers read back from memory
// behind the stores, or a load among them, cost 40; one half of all rows' 128 bytes before the other 30 to 50, with a third more written to memory.
template <int T, bool SPLIT, int TM, int TN, int WM, int WN, bool BACKWARD, bool LISTS>
__global__ __launch_bounds__(64 * WM * WN, 2) void vocab_kernel(ProductArgs a, LossArgs l)
{
    constexpr int THREADS = 64 * WM * WN, FM = TM / WM / 32, FN = TN / WN / 32, kColumns = TN / WN, kTurns = SPLIT ? 2 : 4;
    __shared__ __align__(1024) uint16_t lds[2][(TM + TN) * kStep];
    __shared__ __align__(16) float scratches[WM * WN][kScratch];
    static_assert(sizeof(float2) * TM * WN <= sizeof(lds), "the rows' statistics take the stages' place");
    const Share share = share_of<TM, TN>(a.t, static_cast<int>(blockIdx.x), 0);
    const int64_t g = share.at.g;
    const int M = a.t.M, N = a.t.N, m0 = share.at.tm * TM, tiles = (N + TN - 1) / TN, first = share.at.tn * l.walk, last = min(first + l.walk, tiles);
    const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = (wave % WM) * (TM / WM), wn = (wave / WM) * kColumns;
    const Words &w = l.words;
    float *scratch = scratches[wave];

    // the stream of steps
    const int full = a.K / kStep, steps = (a.K + kStep - 1) / kStep;
    const Sender<TM, THREADS> sa{a.a + g * a.a_batch, a.lda, m0, M};
    int send_tile = steps > 0 ? first : last, send_step = 0, t = 0;
    const auto send = [&](uint16_t *to) {
        if (send_tile >= last) return;
        const Sender<TN, THREADS> sb{a.b + g * a.b_batch, a.ldb, send_tile * TN, N};
        if (send_step < full) {
            sa.load(to, send_step * kStep);
            sb.load(to + TM * kStep, send_step * kStep);
        } else {
            sa.load_rest(to, send_step * kStep, a.K);
            sb.load_rest(to + TM * kStep, send_step * kStep, a.K);
        }
        if (++send_step == steps) {
            send_step = 0;
            ++send_tile;
        }
    };
    send(lds[0]);

    // what a row brings along
    const float scale = l.inv_tau * kLog2E;
    float2 sigma{1.0f, 1.0f};
    if constexpr (BACKWARD && !SPLIT) {
        sigma = dz_scale<T>(max_of<64>(lane < l.most_parts ? l.most[g * kMostParts + lane] : 0.0f));
        if (share.at.tm == 0 && share.at.tn == 0 && threadIdx.x == 0) l.factor[g] = sigma.y;
    }
    float2 stats[FM];                                     // forward: as join_stats has them, of the lane's own columns
    float weight[FM], p_weight[FM], lse[FM];              // backward
    int32_t target[LISTS ? 1 : FM];
    bool near[FM], dead[FM];
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const int m = m0 + wm + i * 32 + (lane & 31), mc = min(m, M - 1);
        stats[i] = float2{-__builtin_inff(), 0.0f};
        if constexpr (!LISTS) {
            const int64_t word = w.target[g * w.batch + mc * w.ld];
            target[i] = m < M && word < w.vocab ? static_cast<int32_t>(word < 0 ? -1 : word) : -1;
        }
        if constexpr (BACKWARD) {
            const int state = m < M ? row_state(w, g, mc) : kDead;
            weight[i] = row_weight(l, g, mc, state) * sigma.x;
            dead[i] = state == kDead;
            const float n = dead[i] ? 0.0f : l.lse[g * l.lse_batch + mc * l.lse_ld];
            near[i] = fabsf(n) <= kPlain;
            lse[i] = near[i] ? n * kLog2E : n;
            p_weight[i] = near[i] ? weight[i] * exp2_of(-fmaf(n, kLog2E, -lse[i])) : weight[i];       // what the product rounded away
        }
    }

    // the logits' sums begin with the bias: a lane has one column's, loaded before anything of the tile before is stored -- a load is waited for together with
    // the stores before it
    static_assert(kColumns == 64, "a lane has a column");
    float bias = 0.0f;
    const auto load_bias = [&](int tile, int lane) {
        const int n = tile * TN + wn + lane;
        if constexpr (!SPLIT) bias = l.bias && n < N ? load_one(l.bias, g * l.bias_batch + n, T) : 0.0f;
    };
    load_bias(first, lane);

    meet<true>();
    send(lds[1]);
    constexpr int kReads = (SPLIT ? 2 : 1) * (FM + FN), kMfmas = (SPLIT ? 3 : 1) * FM * FN;
    for (int tile = first; tile < last; ++tile) {
        v16f acc[FM][FN];
        int begin = 0, entries = 0;                         // of the list of the wave's rows and columns
        if constexpr (LISTS)
            if (m0 + wm < M && tile * TN + wn < N) {
                const int32_t *starts = l.lists.starts + (g * l.lists.blocks + (m0 + wm) / (TM / WM)) * (l.lists.windows + 1) + ((l.first + tile * TN + wn) >> l.lists.shift);
                begin = starts[0];
                entries = starts[1] - begin;
            }
        if constexpr (!SPLIT) {
            in_order();
            scratch[threadIdx.x & 63] = bias;
            in_order();
        }
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const v4f from = SPLIT ? v4f{0.0f, 0.0f, 0.0f, 0.0f} : *reinterpret_cast<const v4f *>(scratch + j * 32 + q * 8 + half * 4);
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int c = 0; c < 4; ++c) acc[i][j][4 * q + c] = from[c];
            }
        Turn<T, SPLIT, TM, TN, FM, FN, 0> turn[2];
        if (steps > 0) turn[0].template load<0>(lds[t & 1], wm, wn);
        for (int s = 0; s < steps; ++s, ++t) {
            uint16_t *now = lds[t & 1], *next = lds[(t + 1) & 1];
            repeat<kTurns - 1>([&](auto k) {
                turn[(k + 1) & 1].template load<k + 1>(now, wm, wn);
                turn[k & 1].multiply(acc);
                interleave<kReads, kMfmas>();
                __builtin_amdgcn_sched_barrier(0);
            });
            // the stores of the tile before are not waited for here: what this step's waves read next arrived before they were sent
            if (BACKWARD && s == 0 && tile > first) meet<false>();
            else meet<true>();
            send(now);
            turn[0].template load<0>(next, wm, wn);         // of a tile's last step: not used
            turn[(kTurns - 1) & 1].multiply(acc);
            interleave<kReads, kMfmas>();
            __builtin_amdgcn_sched_barrier(0);
        }

        // what leaving derives from the lane is derived anew for every tile: kept over the steps, it would take the registers of the sums
        int lane = threadIdx.x & 63;
        asm volatile("" : "+v"(lane));
        const int half = lane >> 5;
        if (tile + 1 < last) load_bias(tile + 1, lane);
        const int n_wave = tile * TN + wn, lo = l.first + n_wave, hi = l.first + min(n_wave + kColumns, N);
        const bool whole = n_wave + kColumns <= N;
        const int left = N - n_wave - half * 4;             // columns from the lane's first on
        // words of the wave's rows among its columns, kHeld lanes' of them at hand; a code's column among the wave's, its row among a fragment's
        constexpr int kHeld = 2;
        uint32_t entry[kHeld] = {};
        float entry_share[kHeld] = {};
        const uint32_t *codes = nullptr;
        const float *shares = nullptr;
        const int window = lo & ((1 << l.lists.shift) - 1);            // where the wave's columns begin in theirs
        const uint32_t none = static_cast<uint32_t>(window + kColumns) << 17;         // no column of the wave's, past 2^15 too
        if constexpr (LISTS) {
            const int64_t at = (g * l.lists.blocks + (m0 + wm) / (TM / WM)) * (TM / WM) * w.top + begin;
            codes = l.lists.code + at;
            shares = l.lists.share + at;
#pragma unroll
            for (int k = 0; k < kHeld; ++k) {
                entry[k] = none;
                if (k * 64 + lane >= entries) continue;
                entry[k] = codes[k * 64 + lane];
                if (BACKWARD) entry_share[k] = shares[k * 64 + lane];
            }
        }
        const auto column_of = [&](uint32_t code) { return static_cast<int>(code >> 17) - window; };
        const auto row_in = [&](uint32_t code) { return static_cast<int>(code >> 10) & 31; };
        const auto in_fragment = [&](uint32_t code, int i, int j) { return (static_cast<int>(code >> 15) & 3) == i && column_of(code) >> 5 == j; };
        const auto put = [&](const v16f &rows) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<v4f *>(scratch + scratch_at(lane & 31, 8 * q + 4 * half)) = v4f{rows[4 * q], rows[4 * q + 1], rows[4 * q + 2], rows[4 * q + 3]};
        };

        if constexpr (SPLIT) {
            int em[FM];
#pragma unroll
            for (int i = 0; i < FM; ++i) em[i] = row_exponent(a.a_max[g * a.a_max_batch + min(m0 + wm + i * 32 + (lane & 31), M - 1)]);
            const float *from = static_cast<const float *>(l.bias) + g * l.bias_batch;
            const uint32_t *tops = a.b_max + g * a.b_max_batch;            // up to the end of the last tile, whatever lies behind N
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                v4f b[4];
                v4u e[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int n = n_wave + j * 32 + q * 8 + half * 4;
                    b[q] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
                    e[q] = *reinterpret_cast<const v4u_any *>(tops + n);
                    const int rest = left - (j * 32 + q * 8);
                    if (l.bias && rest >= 4) b[q] = read4<kF32>(from, n);
                    else if (l.bias) {
                        if (rest > 0) b[q][0] = from[n];
                        if (rest > 1) b[q][1] = from[n + 1];
                        if (rest > 2) b[q][2] = from[n + 2];
                    }
                }
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[i][j][r] = ldexpf(acc[i][j][r], em[i] + row_exponent(e[r >> 2][r & 3])) + b[r >> 2][r & 3];
            }
        }
        const auto cut = [&](int i, int j) {               // words behind the last
            if (!whole)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (j * 32 + (r >> 2) * 8 + (r & 3) >= left) acc[i][j][r] = -__builtin_inff();
        };
        const auto word_of = [&](int i) {                  // a row's word among the wave's columns
            if constexpr (LISTS) return -1;
            else return target[i] >= lo && target[i] < hi ? target[i] - lo : -1;
        };
        if constexpr (!BACKWARD) {
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                const int row0 = m0 + wm + i * 32, m = row0 + (lane & 31), column = word_of(i);
#pragma unroll
                for (int j = 0; j < FN; ++j) cut(i, j);
                float most = acc[i][0][0];
#pragma unroll
                for (int j = 0; j < FN; ++j)
#pragma unroll
                    for (int r = 0; r < 16; ++r) most = fmaxf(most, acc[i][j][r]);
                // sums of 2^(z scale - from), from = most scale rounded; afterwards less most scale itself.  Rows far from 0 have a sum of their own: from an
                // infinite logit nothing is taken away, it makes the sum infinite, or is nothing of it
                const bool near = fabsf(most * scale) <= kPlain;
                const float from = near ? most * scale : fabsf(most) < __builtin_inff() ? most : 0.0f;
                float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                if (__all(near)) {
#pragma unroll
                    for (int j = 0; j < FN; ++j)
#pragma unroll
                        for (int r = 0; r < 16; ++r) sum[r & 3] += exp2_of(fmaf(acc[i][j][r], scale, -from));
                    apart<0>();
                } else {
#pragma unroll
                    for (int j = 0; j < FN; ++j)
#pragma unroll
                        for (int r = 0; r < 16; ++r) sum[r & 3] += exp2_of(near ? fmaf(acc[i][j][r], scale, -from) : (acc[i][j][r] - from) * scale);
                    apart<1>();
                }
                sum[0] = (sum[0] + sum[1]) + (sum[2] + sum[3]);
                if (near) sum[0] *= exp2_of(-fmaf(most, scale, -from));
                stats[i] = join_stats(stats[i], float2{most, sum[0]}, scale);
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    if constexpr (LISTS) {
                        if (!__any(in_fragment(entry[0], i, j) || in_fragment(entry[1], i, j)) && entries <= 64 * kHeld) continue;
                        in_order();
                        put(acc[i][j]);
                        in_order();
                        const auto leave = [&](uint32_t code) {
                            if (in_fragment(code, i, j))
                                l.at[(g * w.rows + row0 + row_in(code)) * w.top + (code & 1023)] = scratch[scratch_at(row_in(code), column_of(code) & 31)];
                        };
#pragma unroll
                        for (int k = 0; k < kHeld; ++k) leave(entry[k]);
                        for (int e = 64 * kHeld + lane; e < entries; e += 64) {
                            leave(codes[e]);
                            __builtin_amdgcn_s_waitcnt(0x0f70);            // vmcnt(0), as below
                        }
                    } else if (__any(column >> 5 == j)) {
                        in_order();
                        put(acc[i][j]);
                        in_order();
                        if (column >> 5 == j && half == 0) l.at[g * w.rows + m] = scratch[scratch_at(lane, column & 31)];
                    }
                }
            }
        } else {
            // both halves of a row's 128 bytes one after the other; no load between the stores, which it would wait for
            const int from = lane >> 2, eight = (lane & 3) * 8;             // what a lane stores: rows `from` and 16 on, 8 columns; 4 lanes a row
            v4f total[FN][2], top[SPLIT ? FN : 1][2];
            Eight z[2];
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                total[j][0] = total[j][1] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
                if (SPLIT) top[j][0] = top[j][1] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
            }
            const auto store = [&](int i, int j) {
                const int n = n_wave + j * 32 + eight;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int row = m0 + wm + i * 32 + k * 16 + from;
                    total[j][0] += z[k].v[0];
                    total[j][1] += z[k].v[1];
                    if constexpr (SPLIT)
#pragma unroll
                        for (int c = 0; c < 8; ++c) top[j][c >> 2][c & 3] = fmaxf(top[j][c >> 2][c & 3], fabsf(z[k].v[c >> 2][c & 3]));
                    if (row >= M || n >= l.dz_ld) continue;
                    const int64_t at = g * l.dz_batch + row * l.dz_ld + n;
                    if (l.streamed) write8<SPLIT ? kF32 : T, true>(l.dz, at, z[k]);
                    else write8<SPLIT ? kF32 : T>(l.dz, at, z[k]);
                }
            };
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                const int column = word_of(i);
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    cut(i, j);
                    if (__all(near[i])) {
#pragma unroll
                        for (int r = 0; r < 16; ++r) acc[i][j][r] = dead[i] ? 0.0f : p_weight[i] * exp2_of(fmaf(acc[i][j][r], scale, -lse[i]));
                        apart<0>();
                    } else {
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const float z = acc[i][j][r];
                            acc[i][j][r] = dead[i] ? 0.0f : p_weight[i] * exp2_of(near[i] ? fmaf(z, scale, -lse[i]) : fmaf(z, l.inv_tau, -lse[i]) * kLog2E);
                        }
                        apart<1>();
                    }
                    in_order();
                    put(acc[i][j]);
                    in_order();
                    if constexpr (LISTS) {
                        const auto take = [&](uint32_t code, float part, float of) {
                            if (in_fragment(code, i, j)) scratch[scratch_at(row_in(code), column_of(code) & 31)] -= of * part;
                        };
#pragma unroll
                        for (int k = 0; k < kHeld; ++k)
                            if (__any(in_fragment(entry[k], i, j))) take(entry[k], entry_share[k], __shfl(weight[i], row_in(entry[k])));
                        for (int e = 64 * kHeld; e < entries; e += 64) {           // all lanes: a row's weight is another lane's
                            const uint32_t code = e + lane < entries ? codes[e + lane] : none;
                            take(code, code == none ? 0.0f : shares[e + lane], __shfl(weight[i], row_in(code)));
                            // vmcnt(0): else it would be waited for, with the stores, wherever its registers are used next, also when nothing was loaded
                            __builtin_amdgcn_s_waitcnt(0x0f70);
                        }
                        in_order();
                    } else if (__any(column >> 5 == j)) {
                        if (column >> 5 == j && half == 0) scratch[scratch_at(lane, column & 31)] -= weight[i];
                        in_order();
                    }
                    // what was read of the columns before leaves while these come back
                    if (i + j == 0) __builtin_amdgcn_s_waitcnt(0x0f70);        // vmcnt(0): the next tile's first two steps are here
                    else store(j == 0 ? i - 1 : i, j == 0 ? FN - 1 : j - 1);
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int r = k * 16 + from;
                        z[k] = Eight{{*reinterpret_cast<const v4f *>(scratch + scratch_at(r, eight)), *reinterpret_cast<const v4f *>(scratch + scratch_at(r, eight + 4))}};
                    }
                }
            }
            store(FM - 1, FN - 1);
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                // a lane's column of what 16 groups of lanes have of all columns
                const int n = n_wave + j * 32 + lane;
                const auto gather = [&](const v4f (&part)[2], auto join) {
                    in_order();
                    *reinterpret_cast<v4f *>(scratch + from * 32 + eight) = part[0];
                    *reinterpret_cast<v4f *>(scratch + from * 32 + eight + 4) = part[1];
                    in_order();
                    float v = scratch[half * 8 * 32 + (lane & 31)];
#pragma unroll
                    for (int k = 1; k < 8; ++k) v = join(v, scratch[(half * 8 + k) * 32 + (lane & 31)]);
                    in_order();
                    return join(v, __shfl_xor(v, 32));
                };
                if (l.col_sums) {
                    const float v = gather(total[j], [](float x, float y) { return x + y; });
                    if (half == 0 && n < N) l.col_sums[((g * a.t.tiles_m + share.at.tm) * WM + wave % WM) * N + n] = v;
                }
                if constexpr (SPLIT)
                    if (l.col_max) {
                        const uint32_t v = __float_as_uint(gather(top[j], [](float x, float y) { return fmaxf(x, y); }));
                        if (half == 0 && n < N && v) atomicMax(l.col_max + g * N + n, v);
                    }
            }
        }
    }
    if constexpr (!BACKWARD) {
        // nothing of the stages is read any more
        float2 *all = reinterpret_cast<float2 *>(&lds[0][0]);
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const float2 other{__shfl_xor(stats[i].x, 32), __shfl_xor(stats[i].y, 32)};
            const float2 s = join_stats(stats[i], other, scale);
            if (half == 0) all[(wave / WM) * TM + wm + i * 32 + lane] = s;
        }
        __syncthreads();
        for (int r = threadIdx.x; r < TM; r += THREADS) {
            if (m0 + r >= M) continue;
            float2 s = all[r];
#pragma unroll
            for (int v = 1; v < WN; ++v) s = join_stats(s, all[v * TM + r], scale);
            l.parts[(g * l.part_tiles + l.first_tile + share.at.tn) * w.rows + m0 + r] = s;
        }
    }
}

}  // namespace

int launch_vocab(const ProductArgs &a, const LossArgs &l, int32_t type, int tile, bool backward, hipStream_t stream)
{
    if (a.t.count() <= 0) return GBMUF_OK;
    ProductArgs args = a;
    LossArgs loss = l;
    void *argv[] = {&args, &loss};
    using Fn = void (*)(ProductArgs, LossArgs);
#define GBMUF_VOCAB(T, SPLIT, TILE, WN, BACKWARD) \
    {vocab_kernel<T, SPLIT, TILE, TILE, 2, WN, BACKWARD, false>, vocab_kernel<T, SPLIT, TILE, TILE, 2, WN, BACKWARD, true>}
    // [type][backward][tile][lists]
    static constexpr Fn fns[3][2][2][2] = {
        {{GBMUF_VOCAB(kF16, true, 128, 2, false), {}}, {GBMUF_VOCAB(kF16, true, 128, 2, true), {}}},
        {{GBMUF_VOCAB(kBf16, false, 128, 2, false), GBMUF_VOCAB(kBf16, false, 256, 4, false)}, {GBMUF_VOCAB(kBf16, false, 128, 2, true), GBMUF_VOCAB(kBf16, false, 256, 4, true)}},
        {{GBMUF_VOCAB(kF16, false, 128, 2, false), GBMUF_VOCAB(kF16, false, 256, 4, false)}, {GBMUF_VOCAB(kF16, false, 128, 2, true), GBMUF_VOCAB(kF16, false, 256, 4, true)}}};
#undef GBMUF_VOCAB
    const hipError_t err = hipLaunchKernel(reinterpret_cast<const void *>(fns[type][backward ? 1 : 0][tile == 256 ? 1 : 0][l.lists.blocks > 0 ? 1 : 0]),
                                           dim3(static_cast<unsigned>(a.t.blocks())), dim3(tile == 256 ? 512 : 256), argv, 0, stream);
    return err == hipSuccess ? GBMUF_OK : hip_failed("hipLaunchKernel(logits)", err, GBMUF_EDEVICE);
}

}  // namespace gbmuf
