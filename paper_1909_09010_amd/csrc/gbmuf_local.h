// gbmuf_local.h -- types shared by the local half's sources: products (gbmuf_product.hip), what is laid out for them
// (gbmuf_layout.hip), their entry points (gbmuf_linear.hip) and the gradients of workers (gbmuf_grads.hip).
#pragma once

#include "gbmuf_internal.h"

namespace gbmuf {

enum : int32_t { kF32 = 0, kBf16 = 1, kF16 = 2, kI64 = 3 };          // = GBMUF_F32 .., and the words of rows
constexpr size_t type_bytes(int32_t t) { return t == kI64 ? 8 : t == kF32 ? 4 : 2; }

// What is done with a sum s of products: z = s + bias (+ r), y = act(z) (+ r).
struct Epilogue {
    void *y, *pre;           // pre nullptr: not wanted
    const void *bias, *res;
    int64_t ldy, y_batch, ldp, p_batch, bias_batch, ldr, r_batch;
    int32_t act, place;      // GBMUF_ACT_*, GBMUF_RESIDUAL_*
    int32_t type;            // of all of them
    int32_t streamed;        // y is more than the caches hold
    const float *factor;     // [g] of the sums, or nullptr
};

// Which tiles of a result there are and how workgroups take them: the first `whole` tiles one each, and the sum over k of every other one
// goes to `splits` workgroups of `steps` steps each, whose parts lie [split][tile - whole][row][column].
struct Tiles {
    int32_t M, N, batch;
    int32_t tiles_m, tiles_n;
    int32_t whole, splits, steps;
    float *partial;
    __host__ __device__ int32_t count() const { return tiles_m * tiles_n * batch; }
    __host__ __device__ int32_t rest() const { return count() - whole; }
    __host__ __device__ int32_t blocks() const { return whole + rest() * splits; }
};

// out[g][m][n] = sum over k of a[g][m][k] * b[g][n][k], in 16-bit numbers whose k are contiguous.  Split: a row holds, for every 32
// k, their 32 leading parts and then their 32 trailing parts, and `k` counts both; a_max and b_max hold the bits of the largest finite magnitude of
// every row before the row was scaled.
struct ProductArgs {
    const uint16_t *a, *b;
    int64_t lda, ldb, a_batch, b_batch;
    const uint32_t *a_max, *b_max;
    int64_t a_max_batch, b_max_batch;
    int32_t K;               // 16-bit words
    int32_t across;          // 16-bit types: bit 0, 1: a (b) is [k][m] ([k][n]) with rows lda (ldb) apart, whole pieces of 8 columns
    Tiles t;                 // steps of 64 words
    Epilogue e;
};

// A matrix as it lies, with the slope of an activation at `pre` as a factor of every value where act is one.
struct Source {
    const void *p, *pre;
    int64_t ld, batch, ldp, p_batch;
    int32_t act, reserved;
};

// out[g][m][n] = sum over k of a(m, k) * b(n, k) in f32 arithmetic, straight from where the matrices lie; the form of a kernel says whether k or
// m (n) is what lies side by side.
struct DirectArgs {
    Source a, b;
    int32_t K;
    int32_t reserved;
    Tiles t;                 // steps of 32 values
    Epilogue e;
    const int32_t *live;     // [g][k]: b's values at k count as 0 where this is 0, whatever they are (gradients of losses); or nullptr
    int64_t live_batch;
    void *copy;              // a itself (dz), of the matrices' type, or nullptr
    int64_t copy_ld, copy_batch;
    void *sums;              // sums[g][m] (+)= sum over k of a(m, k), or nullptr; no tile is split
    int64_t sums_batch;
    int32_t sums_type, accumulate;
};

// The sums of the parts of split tiles, and what is done with them.
struct JoinArgs {
    Tiles t;
    int32_t tile, reserved;  // 64, 128 or 256
    Epilogue e;
};

// A source matrix R x C of `type`, with the slope of the activation at `pre` as a factor where there is one, and what is written of it.
// launch_copy: 16-bit types, plain, dz and col_sums.  launch_rows: f32 of up to kLongestRow columns, plain and row_max from one reading.
// launch_stats and launch_lay: f32, row_max, col_max and col_sums from a first reading, plain, trans and dz from a second.
struct LayArgs {
    const void *src, *pre;
    int64_t ld, batch_stride, ldp, p_batch;
    int32_t R, C, batch;
    int32_t type, act;       // act: GBMUF_ACT_NONE = no factor
    // any of these nullptr
    uint32_t *row_max, *col_max;          // [batch][R], [batch][C]: bits of the largest finite magnitude, zeroed before launch_stats
    float *col_sums;                      // [batch][row tiles][C]
    uint16_t *plain, *trans;              // rows of R (C) values along C (R), in 16 bits or taken apart; their whole length is written
    int64_t plain_ld, plain_batch, trans_ld, trans_batch;
    void *dz;                             // the product with the slope itself, of `type`
    int64_t dz_ld, dz_batch;
};
constexpr int kLayTile = 64, kLongestRow = 4096;

// Up to three sources of one type, laid out by one launch: those of one product or of a layer's gradients.
struct LaySet {
    LayArgs a[3];
    int32_t first[4];            // first workgroup of each, and how many there are, set by the launch
    int32_t n = 0;
    int32_t reserved = 0;
    void add(const LayArgs &l) { a[n++] = l; }
};

struct SumArgs {             // out[g][c] (+)= sum over t of sums[g][t][c]
    const float *sums;
    void *out;
    int64_t out_batch;
    int32_t C, tiles, batch, type, accumulate;
    const float *factor;     // [g] of the sums, or nullptr
};

// The words that rows are held to.  target: one of them each, negative where a row does not count.  Else lists of `top`: words in ascending order, kNoWord
// behind the last, and the share of each; or, of few rows and up to kFewWords, as the teacher gives them: target and logit.
enum : int32_t { kDead = 0, kLive = 1, kBad = 2 };         // what a row counts; kBad: it names a word that the vocabulary does not have
constexpr int32_t kNoWord = 0x7fffffff;
struct Words {
    const int64_t *target;
    int64_t ld, batch;
    const int32_t *id;       // [g][row][top], and share
    const float *share;
    const int32_t *state;    // [g][row]
    const float *logit;
    int64_t logit_ld, logit_batch;
    int32_t top;             // 1 where there is one word a row
    int32_t rows, vocab;     // of a worker, whole
};
constexpr int kFewWords = 16;

// The words of lists by where they meet a tile of logits: for every block of block_rows rows the words of each window of 64 << shift, one behind the
// other, as codes: 15 bits of place in the window, 7 of row in the block, 10 of place in the row's list; a word that a row has more than once is there once.
// starts: [g][block][windows + 1].
struct WordLists {
    uint32_t *code;
    int32_t *starts;
    float *share;            // nullptr: not wanted
    int32_t blocks, block_rows, windows, shift;          // shift: log2 of a window
};
constexpr int kMostWindows = 8192;         // of at most 2^15 words: 2^28, more than calls may have

// What is done with logits z = s + bias of the words `first` .. of the vocabulary.
struct LossArgs {
    const void *bias;        // of `type`, or nullptr
    int64_t bias_batch;
    Words words;
    int32_t type;
    int32_t first;
    float inv_tau, tau;
    WordLists lists;         // of tiles of many rows; code nullptr: rows have one word each
    int32_t walk, most_parts; // walk: tiles of logits that a workgroup takes one after the other
    // forward: parts[g][part][row], counted over the vocabulary from first_tile on, and z of the rows' words, at[g][row][top]
    float2 *parts;
    float *at;
    int32_t part_tiles, first_tile;
    // backward: dz[g][row][column], f32 or of 16-bit types (launch_vocab), rows dz_ld apart, whole pieces of 8 up to there
    const float *lse, *dloss;
    int64_t lse_ld, lse_batch, dloss_ld, dloss_batch;
    const float *most;       // 16-bit types, [g][kMostParts]: largest weights of most_parts parts of a worker's rows, or nullptr
    float *factor;           // out, [g]: 1 / what dz is multiplied with for that
    void *dz;
    int64_t dz_ld, dz_batch;
    int32_t streamed;        // dz is more than the caches hold
    int32_t reserved;
    float *col_sums;         // launch_vocab, [g][parts of 64 or 128 rows][column], or nullptr
    uint32_t *col_max;       // the same, f32, [g][column]: bits of the largest magnitude, zero before; or nullptr
    int32_t *live;           // launch_loss_direct, out: [g][row], or nullptr
};

// A teacher's words of every row, as it gives them, made lists of Words.
struct TeacherArgs {
    const int64_t *id;
    const float *logit;
    int64_t id_ld, id_batch, logit_ld, logit_batch;
    int32_t *out_id, *out_state;
    float *out_share;
    int32_t rows, batch, top, vocab;
    float inv_tau;
    int32_t merge;           // a word that a row has more than once has all of its shares at the first place
};

// Losses from their parts.
struct LossJoin {
    Words words;
    const float2 *parts;
    const float *at;
    float *loss, *lse;       // lse nullptr: not wanted
    int64_t loss_ld, loss_batch, lse_ld, lse_batch;
    int32_t tiles, batch;
    float inv_tau, tau;
};

// Rows of x that count, at aligned places with zeros behind them, zeros in place of the others; and for 16-bit types the largest weight of parts of a worker's rows.
constexpr int kMostParts = 64;
struct KeepArgs {
    Words words;
    const void *x;
    int64_t ld, batch_stride;
    void *out;               // [batch][rows][out_ld]
    int64_t out_ld;
    int32_t columns, batch, type;
    int32_t all;             // every row counts: words is not looked at but for its rows
    const float *dloss;
    int64_t dloss_ld, dloss_batch;
    float tau;
    int32_t most_parts;
    float *most;             // [batch][kMostParts], or nullptr
    uint32_t *row_max;       // [batch][rows]: bits of what no value of the row's dz exceeds; or nullptr
};

// Gradients of few rows: small_grads_kernel, and few_grads_kernel for more columns.
constexpr int kFewGradRows = 8, kFewGradColumns = 1024;
constexpr int kSmallRows = 64, kSmallColumns = 64, kSmallWords = 64;       // words of a piece of the vocabulary
struct SmallGrads {
    LossArgs l;              // words, bias, lse and dloss
    const void *x, *w;
    int64_t ldx, x_batch, ldw, w_batch;
    void *dx, *dw, *dbias;   // any of them nullptr; of l.type, dw and dbias of grad_type
    int64_t lddx, dx_batch, lddw, dw_batch, dbias_batch;
    float *parts;            // [piece][worker][row][column] of dx, or nullptr
    int32_t columns, batch, pieces, grad_type, accumulate;
    int32_t words;           // of a piece, few_grads_kernel: 64, 32 or 16
};

struct CastArgs {            // out = from, [batch][rows][columns]
    const float *from;
    void *out;
    int64_t ld, batch_stride;
    int32_t rows, columns, batch, type;
};

// values of a packed row of n numbers, in 16-bit words: whole steps of 64
constexpr int64_t packed_words(int64_t n, bool split) { return split ? (n + 31) / 32 * 64 : (n + 63) / 64 * 64; }

int launch_product(const ProductArgs &a, int32_t type, int tile, hipStream_t stream);   // tile: 128 or 256
int launch_few(const DirectArgs &a, int32_t type, hipStream_t stream);
constexpr int kFewRows = 64;
int launch_direct_forward(const DirectArgs &a, hipStream_t stream);          // f32, tiles of 64 x 64
int launch_direct_backward(const DirectArgs &dx, const DirectArgs &dw, int32_t type, hipStream_t stream);
int launch_join(const JoinArgs &a, hipStream_t stream);
int launch_copy(const LaySet &set, hipStream_t stream);
int launch_rows(const LaySet &set, hipStream_t stream);
int launch_stats(const LaySet &set, hipStream_t stream);
int launch_lay(const LaySet &set, hipStream_t stream);
int launch_column_sums(const SumArgs &a, hipStream_t stream);
int launch_vocab(const ProductArgs &a, const LossArgs &l, int32_t type, int tile, bool backward, hipStream_t stream);
int launch_loss_few(const DirectArgs &a, const LossArgs &l, int32_t type, hipStream_t stream);
int few_columns(const DirectArgs &a, int32_t type);        // of a tile of launch_loss_few
int launch_loss_direct(const DirectArgs &a, const LossArgs &l, int32_t type, bool backward, hipStream_t stream);
int launch_loss_grads(const DirectArgs &dx, const DirectArgs &dw, int32_t type, hipStream_t stream);   // dz in f32
int launch_small_grads(const SmallGrads &a, hipStream_t stream);
int launch_few_grads(const SmallGrads &a, int32_t workgroups, hipStream_t stream);
int few_grads_lanes(int64_t K);
int launch_join_parts(const SmallGrads &a, int32_t parts, hipStream_t stream);
int launch_teacher(const TeacherArgs &a, hipStream_t stream);
int launch_word_lists(const Words &w, const WordLists &l, int32_t batch, hipStream_t stream);
int launch_loss_join(const LossJoin &a, hipStream_t stream);
int launch_keep(const KeepArgs &a, hipStream_t stream);
int launch_cast(const CastArgs &a, hipStream_t stream);
constexpr int kMostTop = 1024;
int launch_zero(uint32_t *p, int64_t words, hipStream_t stream);

}  // namespace gbmuf
