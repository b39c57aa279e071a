// gbmuf_rows.hip -- what losses do row by row: a teacher's words put in order, losses from the parts of their logits, the rows of x that count.
#include "gbmuf_loss.h"

namespace gbmuf {
namespace {

// More workgroups than a grid's first dimension holds lie in two; the last row's surplus has nothing to do.
constexpr int64_t kGridRow = 1 << 22;
__device__ __forceinline__ int64_t block_number() { return static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x; }
dim3 grid_of(int64_t blocks)
{
    const int64_t across = blocks < kGridRow ? blocks : kGridRow;
    return dim3(static_cast<unsigned>(across), static_cast<unsigned>((blocks + across - 1) / across));
}

// Sum of WIDTH neighbouring lanes.
template <int WIDTH>
__device__ __forceinline__ float sum_of(float v)
{
#pragma unroll
    for (int d = 1; d < WIDTH; d *= 2) v += __shfl_xor(v, d);
    return v;
}

// ---------------------------------------------------------------------------------------
// A teacher's words.  One wave a row: the shares are a softmax over the words that are there (id not negative, logit not -infinity), and the words are
// sorted by a bitonic network in LDS, the place in the teacher's list behind the word, so that equal words keep their order and every
// key is another.
// ---------------------------------------------------------------------------------------
template <int MOST>
__global__ __launch_bounds__(256) void teacher_kernel(TeacherArgs a, int32_t padded)
{
    __shared__ uint64_t keys[4][MOST];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t all = static_cast<int64_t>(a.rows) * a.batch, at = block_number() * 4 + wave, row = at < all ? at : all - 1;
    const int64_t g = row / a.rows, i = row - g * a.rows;
    const int64_t *id = a.id + g * a.id_batch + i * a.id_ld;
    const float *logit = a.logit + g * a.logit_batch + i * a.logit_ld;
    uint64_t *key = keys[wave];
    const float inf = __builtin_inff();
    float most = -inf;
    int state = kDead;
    for (int j = lane; j < padded; j += 64) {
        int32_t word = kNoWord;
        if (j < a.top) {
            const int64_t v = id[j];
            const float l = logit[j];
            if (v >= 0 && l != -inf) {
                word = v < a.vocab ? static_cast<int32_t>(v) : a.vocab;          // behind every word that there is
                most = fmaxf(most, l);
                state = max(state, v < a.vocab ? kLive : kBad);
            }
        }
        key[j] = (static_cast<uint64_t>(static_cast<uint32_t>(word)) << 32) | static_cast<uint32_t>(j);
    }
    most = max_of<64>(most);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) state = max(state, __shfl_xor(state, d));
    const float from = most == -inf ? 0.0f : most;
    float total = 0.0f;
    for (int j = lane; j < a.top; j += 64)
        if (static_cast<int32_t>(key[j] >> 32) != kNoWord) total += expf((logit[j] - from) * a.inv_tau);
    total = sum_of<64>(total);
    __syncthreads();
    for (int size = 2; size <= padded; size *= 2)
        for (int d = size / 2; d; d /= 2) {
            for (int p = lane; p < padded / 2; p += 64) {
                const int lo = (p / d) * 2 * d + p % d, hi = lo + d;
                const uint64_t x = key[lo], y = key[hi];
                if ((x > y) == ((lo & size) == 0)) {
                    key[lo] = y;
                    key[hi] = x;
                }
            }
            __syncthreads();
        }
    if (at >= all) return;
    for (int p = lane; p < a.top; p += 64) {
        const uint64_t k = key[p];
        const int32_t word = static_cast<int32_t>(k >> 32);
        const auto share_of = [&](uint64_t x) { return expf((logit[static_cast<uint32_t>(x)] - from) * a.inv_tau) / total; };
        float share = word == kNoWord ? 0.0f : share_of(k);
        if (a.merge && word != kNoWord) {
            if (p > 0 && static_cast<int32_t>(key[p - 1] >> 32) == word) share = 0.0f;
            else
                for (int q = p + 1; q < a.top && static_cast<int32_t>(key[q] >> 32) == word; ++q) share += share_of(key[q]);
        }
        a.out_id[row * a.top + p] = word;
        a.out_share[row * a.top + p] = share;
    }
    if (lane == 0) a.out_state[row] = state;
}

// The value of the lane whose number differs in bit D: by the vector unit's own lane exchanges up to 8, which LDS's take four times as long for.
template <int D>
__device__ __forceinline__ uint32_t lane_xor(uint32_t v)
{
    const int x = static_cast<int>(v);
    if constexpr (D == 1) return __builtin_amdgcn_update_dpp(x, x, 0xb1, 0xf, 0xf, false);             // quad_perm 1 0 3 2
    if constexpr (D == 2) return __builtin_amdgcn_update_dpp(x, x, 0x4e, 0xf, 0xf, false);             // quad_perm 2 3 0 1
    // row_shl 4 for the lanes without the bit, row_shr 4 for those with it
    if constexpr (D == 4) return __builtin_amdgcn_update_dpp(__builtin_amdgcn_update_dpp(x, x, 0x104, 0xf, 0x5, false), x, 0x114, 0xf, 0xa, false);
    if constexpr (D == 8) return __builtin_amdgcn_update_dpp(x, x, 0x128, 0xf, 0xf, false);            // row_ror 8
    return __shfl_xor(x, D);
}

template <int SIZE, int D>
__device__ __forceinline__ void sort_step(uint32_t &key, int lane)
{
    const uint32_t other = lane_xor<D>(key), less = min(key, other), more = max(key, other);
    key = ((lane & D) == 0) == ((lane & SIZE) == 0) ? less : more;
    if constexpr (D > 1) sort_step<SIZE, D / 2>(key, lane);
}

// The same for up to 64 words of a vocabulary below 2^25: a lane has one, and the key is the word and the lane, in 32 bits.
constexpr int kShortTop = 64, kShortVocab = 1 << 25;
__global__ __launch_bounds__(256) void short_teacher_kernel(TeacherArgs a)
{
    const int lane = threadIdx.x & 63;
    const int64_t row = block_number() * 4 + (threadIdx.x >> 6);
    if (row >= static_cast<int64_t>(a.rows) * a.batch) return;
    const int64_t g = row / a.rows, i = row - g * a.rows;
    const float inf = __builtin_inff();
    int64_t v = -1;
    float logit = -inf;
    if (lane < a.top) {
        v = a.id[g * a.id_batch + i * a.id_ld + lane];
        logit = a.logit[g * a.logit_batch + i * a.logit_ld + lane];
    }
    const bool there = v >= 0 && logit != -inf;
    const bool any = __any(there), bad = __any(there && v >= a.vocab);
    uint32_t key = (!there ? 0xffffffc0u : static_cast<uint32_t>(v < a.vocab ? v : a.vocab) << 6) | static_cast<uint32_t>(lane);
    const float most = max_of<64>(there ? logit : -inf), from = most == -inf ? 0.0f : most;
    float share = there ? expf((logit - from) * a.inv_tau) : 0.0f;
    share /= sum_of<64>(share);
    if (!there) share = 0.0f;
    sort_step<2, 1>(key, lane);
    sort_step<4, 2>(key, lane);
    sort_step<8, 4>(key, lane);
    sort_step<16, 8>(key, lane);
    sort_step<32, 16>(key, lane);
    sort_step<64, 32>(key, lane);
    share = __shfl(share, static_cast<int>(key & 63));
    const int word = key >= 0xffffffc0u ? kNoWord : static_cast<int>(key >> 6);
    if (a.merge) {
        const int before = __shfl_up(word, 1);
        const bool again = lane > 0 && word != kNoWord && before == word;
        if (__any(again)) {
            float all = share;
            for (int d = 1; d < 64; ++d) {
                const int w = __shfl_down(word, d);
                const float s = __shfl_down(share, d);
                if (lane + d < 64 && w == word) all += s;
            }
            share = again ? 0.0f : all;
        }
        if (word == kNoWord) share = 0.0f;
    }
    if (lane < a.top) {
        a.out_id[row * a.top + lane] = word;
        a.out_share[row * a.top + lane] = share;
    }
    if (lane == 0) a.out_state[row] = bad ? kBad : any ? kLive : kDead;
}

// ---------------------------------------------------------------------------------------
// Lists of words by window: a workgroup takes the lists of a block of rows, counts the words of each window, and puts them there.  Within a window they lie in no
// certain order, which no result depends on: no two are the same word of the same row.
// ---------------------------------------------------------------------------------------
constexpr int kListThreads = 1024;           // 8 x 5120 rows of 64 words, without shares / with them: 18 / 30 us; 256 threads, an entry at a time, 46 / 67
__global__ __launch_bounds__(kListThreads) void word_lists_kernel(Words w, WordLists l)
{
    __shared__ int32_t count[kMostWindows];
    __shared__ int32_t sums[kListThreads / 64];
    const int64_t g = blockIdx.x / l.blocks;
    const int block = static_cast<int>(blockIdx.x % l.blocks), m0 = block * l.block_rows, rows = min(l.block_rows, w.rows - m0), n = rows * w.top;
    const int64_t first = (g * w.rows + m0) * w.top, out = static_cast<int64_t>(blockIdx.x) * l.block_rows * w.top;
    const int32_t *id = w.id + first;
    const float *share = w.share + first;
    int32_t *starts = l.starts + static_cast<int64_t>(blockIdx.x) * (l.windows + 1);
    for (int i = threadIdx.x; i < l.windows; i += kListThreads) count[i] = 0;
    __syncthreads();
    // kBatch entries of a thread at a time, all sent for before the first is looked at: f(word or kNoWord, share, e, p of each)
    constexpr int kBatch = 4;
    const auto each = [&](auto with_shares, auto f) {
        for (int first_e = threadIdx.x; first_e < n; first_e += kBatch * kListThreads) {
            int word[kBatch], before[kBatch], place[kBatch];
            float part[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {              // entries behind the last are read as the last one
                const int e = min(first_e + u * kListThreads, n - 1);
                word[u] = id[e];
                before[u] = id[max(e - 1, 0)];
                if (with_shares) part[u] = share[e];
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const int e = first_e + u * kListThreads;
                place[u] = e % w.top;
                if (e >= n || word[u] >= w.vocab || (place[u] != 0 && before[u] == word[u])) word[u] = kNoWord;
            }
            f(word, part, place, first_e);
        }
    };
    each(std::false_type{}, [&](const int (&word)[kBatch], const float (&)[kBatch], const int (&)[kBatch], int) {
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
            if (word[u] != kNoWord) atomicAdd(&count[word[u] >> l.shift], 1);
    });
    __syncthreads();
    // where each window begins: a thread's windows lie side by side
    const int per = (l.windows + kListThreads - 1) / kListThreads, from = threadIdx.x * per, to = min(from + per, l.windows);
    int mine = 0;
    for (int i = from; i < to; ++i) mine += count[i];
    int before = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int v = __shfl_up(before, d);
        if (static_cast<int>(threadIdx.x & 63) >= d) before += v;
    }
    if ((threadIdx.x & 63) == 63) sums[threadIdx.x >> 6] = before;
    __syncthreads();
    for (int v = 0; v < static_cast<int>(threadIdx.x >> 6); ++v) before += sums[v];
    int at = before - mine;
    for (int i = from; i < to; ++i) {
        const int c = count[i];
        starts[i] = at;
        count[i] = at;
        at += c;
    }
    if (threadIdx.x == kListThreads - 1) starts[l.windows] = before;
    __syncthreads();
    const auto put = [&](const int (&word)[kBatch], const float (&part)[kBatch], const int (&p)[kBatch], int first_e) {
        int to_place[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) to_place[u] = word[u] != kNoWord ? atomicAdd(&count[word[u] >> l.shift], 1) : 0;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (word[u] == kNoWord) continue;
            const uint32_t row = static_cast<uint32_t>((first_e + u * kListThreads) / w.top);
            l.code[out + to_place[u]] = static_cast<uint32_t>(word[u] & ((1 << l.shift) - 1)) << 17 | row << 10 | static_cast<uint32_t>(p[u]);
            if (l.share) l.share[out + to_place[u]] = part[u];
        }
    };
    if (l.share) each(std::true_type{}, put);
    else each(std::false_type{}, put);
}

// ---------------------------------------------------------------------------------------
// Losses.  A workgroup takes ROWS rows: 256 / ROWS threads share the parts of a row, side by side in memory with its neighbours', and then its words.
// ---------------------------------------------------------------------------------------
template <int ROWS>
__global__ __launch_bounds__(256) void loss_join_kernel(LossJoin a)
{
    constexpr int kThreads = 256 / ROWS;
    __shared__ float2 shared[4][ROWS];
    const Words &w = a.words;
    const uint32_t block = static_cast<uint32_t>(block_number()), blocks = static_cast<uint32_t>(w.rows + ROWS - 1) / ROWS;
    const int64_t g = block / blocks;
    if (g >= a.batch) return;
    const int m0 = static_cast<int>(block % blocks) * ROWS;
    const float inf = __builtin_inff(), scale = a.inv_tau * kLog2E;
    {
        const int r = threadIdx.x % ROWS, m = min(m0 + r, w.rows - 1);
        const float2 *from = a.parts + g * a.tiles * w.rows + m;
        float2 s = {-inf, 0.0f};
#pragma unroll 4
        for (int t = threadIdx.x / ROWS; t < a.tiles; t += kThreads) s = join_stats(s, from[static_cast<int64_t>(t) * w.rows], scale);
#pragma unroll
        for (int d = ROWS; d < 64; d *= 2) s = join_stats(s, float2{__shfl_xor(s.x, d), __shfl_xor(s.y, d)}, scale);
        if (static_cast<int>(threadIdx.x & 63) < ROWS) shared[threadIdx.x >> 6][r] = s;
        __syncthreads();
    }
    const int r = threadIdx.x / kThreads, first = threadIdx.x % kThreads, m = m0 + r;
    const bool inside = m < w.rows;
    float2 stats = shared[0][r];
#pragma unroll
    for (int v = 1; v < 4; ++v) stats = join_stats(stats, shared[v][r], scale);
    const float lse = (fabsf(stats.x) < inf ? stats.x * a.inv_tau : 0.0f) + logf(stats.y);
    const int64_t row = g * w.rows + m;
    int state = inside && !w.logit ? row_state(w, g, m) : kDead;
    float loss = 0.0f;
    if (w.logit) {
        // a few words as the teacher gives them: the first threads of the row have one each
        const int j = min(first, w.top - 1);
        const int64_t i = min(m, w.rows - 1), word = w.target[g * w.batch + i * w.ld + j];
        const float logit = w.logit[g * w.logit_batch + i * w.logit_ld + j];
        const bool there = inside && first < w.top && word >= 0 && logit != -inf;
        constexpr int kLanes = kThreads < 64 ? kThreads : 64;
        const float most = max_of<kLanes>(there ? logit : -inf), e = there ? expf((logit - (most == -inf ? 0.0f : most)) * a.inv_tau) : 0.0f;
        const float share = e / sum_of<kLanes>(e);
        state = static_cast<int>(max_of<kLanes>(static_cast<float>(!there ? kDead : word < w.vocab ? kLive : kBad)));
        if (there && word < w.vocab && share != 0.0f) loss = share * (logf(share) - fmaf(a.at[row * w.top + j], a.inv_tau, -lse));
        loss = sum_of<kLanes>(loss) * (a.tau * a.tau);
    } else if (w.target) loss = state == kLive ? lse - a.at[row] : 0.0f;
    else {
        if (state == kLive)
            for (int j = first; j < w.top; j += kThreads) {
                const int64_t at = row * w.top + j;
                const float share = w.share[at];
                // nothing is lost by a word that the teacher gives no share
                if (w.id[at] == kNoWord || share == 0.0f) continue;
                int64_t one = at;                           // a word's logit stands at its first place
                while (one > row * w.top && w.id[one - 1] == w.id[at]) --one;
                loss += share * (logf(share) - fmaf(a.at[one], a.inv_tau, -lse));
            }
        loss = sum_of<(kThreads < 64 ? kThreads : 64)>(loss);
        if constexpr (kThreads > 64) {
            __shared__ float waves[4];
            if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = loss;
            __syncthreads();
            loss = 0.0f;
            for (int v = 0; v < kThreads / 64; ++v) loss += waves[r * (kThreads / 64) + v];
        }
        loss *= a.tau * a.tau;
    }
    if (!inside || first != 0) return;
    const float bad = __builtin_nanf("");
    a.loss[g * a.loss_batch + m * a.loss_ld] = state == kBad ? bad : loss;
    if (a.lse) a.lse[g * a.lse_batch + m * a.lse_ld] = state == kBad ? bad : state == kDead ? 0.0f : lse;
}

// ---------------------------------------------------------------------------------------
// Rows of x: zeros where a row does not count, whatever it holds, since 0 times that is not always 0.  8 columns a thread.  The last workgroups, where
// `most` is wanted, `most_parts` for each worker, find the largest finite weight of rows that count.
// ---------------------------------------------------------------------------------------
template <int T>
__global__ __launch_bounds__(256) void keep_kernel(KeepArgs a, int64_t copies)
{
    const int64_t block = block_number();
    if (block < copies) {
        const int64_t id = block * 256 + threadIdx.x, all = static_cast<int64_t>(a.words.rows) * a.batch;
        const uint32_t per_row = static_cast<uint32_t>(a.out_ld / 8), rows = static_cast<uint32_t>(a.words.rows);
        int64_t row, g;
        if (copies < 1 << 23) {                             // 32 bits hold every number: a division of 64 takes as long as the copy of 16 bytes
            const uint32_t r = static_cast<uint32_t>(id) / per_row;
            row = r;
            g = r / rows;
        } else {
            row = id / per_row;
            g = row / rows;
        }
        if (row >= all) return;
        const int c = static_cast<int>(id - row * per_row) * 8, left = a.columns - c;
        const int64_t from = g * a.batch_stride + (row - g * a.words.rows) * a.ld + c;
        const int m = static_cast<int>(row - g * a.words.rows), state = a.all ? kLive : row_state(a.words, g, m);
        if (a.row_max && c == 0) {
            const float d = fabsf(a.dloss[g * a.dloss_batch + m * a.dloss_ld] * a.tau);
            a.row_max[row] = state != kDead && d < __builtin_inff() ? __float_as_uint(d) : 0u;
        }
        Eight v{};
        if (state != kDead) {
            // a row's last values are read together with what follows in the matrix, where it does
            if (m * a.ld + c + 8 <= (a.words.rows - 1) * a.ld + a.columns) {
                v = read8<T>(a.x, from);
#pragma unroll
                for (int k = 0; k < 8; ++k) v.v[k >> 2][k & 3] = k < left ? v.v[k >> 2][k & 3] : 0.0f;
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (k < left) v.v[k >> 2][k & 3] = load_one(a.x, from + k, T);
            }
        }
        write8<T>(a.out, row * a.out_ld + c, v);
        return;
    }
    if (!a.most) return;
    const int64_t of = block - copies, g = of / a.most_parts;
    if (g >= a.batch) return;
    const int part = static_cast<int>(of - g * a.most_parts), rows = a.words.rows;
    __shared__ float waves[4];
    float most = 0.0f;
    for (int64_t first = part * 256; first < rows; first += a.most_parts * 256 * 8)
#pragma unroll
        for (int k = 0; k < 8; ++k) {                       // rows behind the last are read as the last one
            const int m = static_cast<int>(min(first + k * a.most_parts * 256 + static_cast<int>(threadIdx.x), static_cast<int64_t>(rows - 1)));
            const float d = fabsf(a.dloss[g * a.dloss_batch + m * a.dloss_ld] * a.tau);
            if (row_state(a.words, g, m) == kLive && d < __builtin_inff()) most = fmaxf(most, d);
        }
    most = max_of<64>(most);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = most;
    __syncthreads();
    if (threadIdx.x == 0) a.most[g * kMostParts + part] = fmaxf(fmaxf(waves[0], waves[1]), fmaxf(waves[2], waves[3]));
}

__global__ __launch_bounds__(256) void cast_kernel(CastArgs a)
{
    const int64_t id = block_number() * 256 + threadIdx.x, per_row = (a.columns + 7) / 8, row = id / per_row;
    if (row >= static_cast<int64_t>(a.rows) * a.batch) return;
    const int c = static_cast<int>(id - row * per_row) * 8, left = a.columns - c;
    const int64_t g = row / a.rows, to = g * a.batch_stride + (row - g * a.rows) * a.ld + c, from = row * a.columns + c;
    if (left >= 8) return store_eight(a.out, to, a.type, read8<kF32>(a.from, from));
    for (int k = 0; k < left; ++k) store_one(a.out, to + k, a.type, a.from[from + k]);
}

}  // namespace

int launch_teacher(const TeacherArgs &a, hipStream_t stream)
{
    const int64_t blocks = (static_cast<int64_t>(a.rows) * a.batch + 3) / 4;
    if (blocks <= 0) return GBMUF_OK;
    TeacherArgs args = a;
    int32_t padded = 1;
    while (padded < a.top) padded *= 2;
    void *argv[] = {&args, &padded};
    const void *fn = a.top <= kShortTop && a.vocab < kShortVocab ? reinterpret_cast<const void *>(short_teacher_kernel) : reinterpret_cast<const void *>(padded <= 128 ? teacher_kernel<128> : teacher_kernel<kMostTop>);
    const hipError_t err = hipLaunchKernel(fn, grid_of(blocks), dim3(256), argv, 0, stream);
    return err == hipSuccess ? GBMUF_OK : hip_failed("hipLaunchKernel(teacher)", err, GBMUF_EDEVICE);
}

int launch_word_lists(const Words &w, const WordLists &l, int32_t batch, hipStream_t stream)
{
    const int64_t blocks = static_cast<int64_t>(l.blocks) * batch;
    if (blocks <= 0) return GBMUF_OK;
    if (blocks > 0x7fffffffLL / kListThreads) return GBMUF_EUNSUPPORTED;
    Words words = w;
    WordLists lists = l;
    void *argv[] = {&words, &lists};
    const hipError_t err = hipLaunchKernel(reinterpret_cast<const void *>(word_lists_kernel), dim3(static_cast<unsigned>(blocks)), dim3(kListThreads), argv, 0, stream);
    return err == hipSuccess ? GBMUF_OK : hip_failed("hipLaunchKernel(lists of words)", err, GBMUF_EDEVICE);
}

// Few rows: more threads for the parts of each.
int launch_loss_join(const LossJoin &a, hipStream_t stream)
{
    if (a.words.rows <= 0 || a.batch <= 0) return GBMUF_OK;
    const int64_t all = static_cast<int64_t>(a.words.rows) * a.batch;
    const int rows = a.words.rows <= 2 || all <= 256 ? 1 : all <= 4096 || a.words.logit ? 4 : 32;
    const int64_t blocks = static_cast<int64_t>((a.words.rows + rows - 1) / rows) * a.batch;
    LossJoin args = a;
    void *argv[] = {&args};
    const auto fn = rows == 1 ? loss_join_kernel<1> : rows == 4 ? loss_join_kernel<4> : loss_join_kernel<32>;
    const hipError_t err = hipLaunchKernel(reinterpret_cast<const void *>(fn), grid_of(blocks), dim3(256), argv, 0, stream);
    return err == hipSuccess ? GBMUF_OK : hip_failed("hipLaunchKernel(losses)", err, GBMUF_EDEVICE);
}

int launch_keep(const KeepArgs &a, hipStream_t stream)
{
    int64_t copies = (static_cast<int64_t>(a.words.rows) * a.batch * (a.out_ld / 8) + 255) / 256;
    const int64_t blocks = copies + (a.most ? static_cast<int64_t>(a.batch) * a.most_parts : 0);
    if (blocks <= 0) return GBMUF_OK;
    KeepArgs args = a;
    void *argv[] = {&args, &copies};
    const auto fn = a.type == kF32 ? keep_kernel<kF32> : a.type == kBf16 ? keep_kernel<kBf16> : keep_kernel<kF16>;
    const hipError_t err = hipLaunchKernel(reinterpret_cast<const void *>(fn), grid_of(blocks), dim3(256), argv, 0, stream);
    return err == hipSuccess ? GBMUF_OK : hip_failed("hipLaunchKernel(rows of x)", err, GBMUF_EDEVICE);
}

int launch_cast(const CastArgs &a, hipStream_t stream)
{
    const int64_t blocks = (static_cast<int64_t>(a.rows) * a.batch * ((a.columns + 7) / 8) + 255) / 256;
    if (blocks <= 0) return GBMUF_OK;
    CastArgs args = a;
    void *argv[] = {&args};
    const hipError_t err = hipLaunchKernel(reinterpret_cast<const void *>(cast_kernel), grid_of(blocks), dim3(256), argv, 0, stream);
    return err == hipSuccess ? GBMUF_OK : hip_failed("hipLaunchKernel(cast)", err, GBMUF_EDEVICE);
}

}  // namespace gbmuf
