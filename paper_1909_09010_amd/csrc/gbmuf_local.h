// gbmuf_local.h -- types shared by the local half's sources: products (gbmuf_product.hip), what is laid out for them
// (gbmuf_layout.hip), their entry points (gbmuf_linear.hip) and the gradients of workers (gbmuf_grads.hip).
#pragma once

#include "gbmuf_internal.h"

namespace gbmuf {

enum : int32_t { kF32 = 0, kBf16 = 1, kF16 = 2 };          // = GBMUF_F32 ..
constexpr size_t type_bytes(int32_t t) { return t == kF32 ? 4 : 2; }

// What is done with a sum s of products: z = s + bias (+ r), y = act(z) (+ r).
struct Epilogue {
    void *y, *pre;           // pre nullptr: not wanted
    const void *bias, *res;
    int64_t ldy, y_batch, ldp, p_batch, bias_batch, ldr, r_batch;
    int32_t act, place;      // GBMUF_ACT_*, GBMUF_RESIDUAL_*
    int32_t type;            // of all of them
    int32_t streamed;        // y is more than the caches hold
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
int launch_zero(uint32_t *p, int64_t words, hipStream_t stream);

}  // namespace gbmuf
