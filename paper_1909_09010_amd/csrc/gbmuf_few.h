// gbmuf_few.h -- matrix instructions on 16 rows of each operand, straight from where they lie.
#pragma once

#include "gbmuf_loss.h"

namespace gbmuf {
namespace {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v4u_any __attribute__((ext_vector_type(4), aligned(2)));

// 16 bytes of a row from value k on: 4 f32 or 8 16-bit values; zeros from K on.
template <int T>
__device__ __forceinline__ v4u piece(const void *row, int k, int K)
{
    using N = typename Num<T>::type;
    constexpr int kValues = 16 / static_cast<int>(sizeof(N));
    const N *p = static_cast<const N *>(row) + k;
    if (k + kValues <= K) return *reinterpret_cast<const v4u_any *>(p);
    uint32_t v[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int c = 0; c < kValues; ++c)
        if (k + c < K) {
            if constexpr (T == kF32) v[c] = __float_as_uint(p[c]);
            else v[c >> 1] |= static_cast<uint32_t>(__builtin_bit_cast(uint16_t, p[c])) << (16 * (c & 1));
        }
    return v4u{v[0], v[1], v[2], v[3]};
}

// acc += w x' over the 4 (f32) or 8 (16-bit) k of each of the four lane groups
template <int T>
__device__ __forceinline__ v4f product(v4u w, v4u x, v4f acc)
{
    if constexpr (T == kF32) {
#pragma unroll
        for (int c = 0; c < 4; ++c) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[c]), __uint_as_float(x[c]), acc, 0, 0, 0);
        return acc;
    } else if constexpr (T == kBf16) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, w), __builtin_bit_cast(v8bf, x), acc, 0, 0, 0);
    } else {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, w), __builtin_bit_cast(v8h, x), acc, 0, 0, 0);
    }
}

}  // namespace
}  // namespace gbmuf
