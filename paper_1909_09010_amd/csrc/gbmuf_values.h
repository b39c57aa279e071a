// gbmuf_values.h -- device code shared by the local half: number formats, activations, what follows a sum of products.
#pragma once

#include "gbmuf_device.h"
#include "gbmuf_local.h"

#include "../../include/gbmuf.h"

namespace gbmuf {
namespace {

template <int T> struct Num;
template <> struct Num<kF32> { using type = float; };
template <> struct Num<kBf16> { using type = __bf16; };
template <> struct Num<kF16> { using type = _Float16; };

template <int T> struct Four;    // four values, at any address that their type allows
template <> struct Four<kF32> { typedef float type __attribute__((ext_vector_type(4), aligned(4))); };
template <> struct Four<kBf16> { typedef __bf16 type __attribute__((ext_vector_type(4), aligned(2))); };
template <> struct Four<kF16> { typedef _Float16 type __attribute__((ext_vector_type(4), aligned(2))); };

template <int T>
__device__ __forceinline__ v4f read4(const void *p, int64_t i)
{
    const typename Four<T>::type v = *reinterpret_cast<const typename Four<T>::type *>(static_cast<const typename Num<T>::type *>(p) + i);
    return v4f{static_cast<float>(v[0]), static_cast<float>(v[1]), static_cast<float>(v[2]), static_cast<float>(v[3])};
}

template <int T>
__device__ __forceinline__ void write4(void *p, int64_t i, v4f v)
{
    using N = typename Num<T>::type;
    typename Four<T>::type r;
    for (int c = 0; c < 4; ++c) r[c] = static_cast<N>(v[c]);
    *reinterpret_cast<typename Four<T>::type *>(static_cast<N *>(p) + i) = r;
}

__device__ __forceinline__ float load_one(const void *p, int64_t i, int32_t type)
{
    if (type == kF32) return static_cast<const float *>(p)[i];
    if (type == kBf16) return static_cast<float>(static_cast<const __bf16 *>(p)[i]);
    return static_cast<float>(static_cast<const _Float16 *>(p)[i]);
}

__device__ __forceinline__ void store_one(void *p, int64_t i, int32_t type, float v)
{
    if (type == kF32) static_cast<float *>(p)[i] = v;
    else if (type == kBf16) static_cast<__bf16 *>(p)[i] = static_cast<__bf16>(v);
    else static_cast<_Float16 *>(p)[i] = static_cast<_Float16>(v);
}

__device__ __forceinline__ float activate(float z, int32_t act)
{
    switch (act) {
        case GBMUF_ACT_RELU: return z > 0.0f ? z : z != z ? z : 0.0f;
        case GBMUF_ACT_GELU: return 0.5f * z * erfcf(-0.70710678118654752f * z);     // 1 + erf(x) = erfc(-x), which keeps its bits where it is small
        case GBMUF_ACT_SILU: return z / (1.0f + expf(-z));
        case GBMUF_ACT_SIGMOID: return 1.0f / (1.0f + expf(-z));
        case GBMUF_ACT_TANH: return tanhf(z);
        default: return z;
    }
}

// act'(z)
__device__ __forceinline__ float slope(float z, int32_t act)
{
    switch (act) {
        case GBMUF_ACT_RELU: return z > 0.0f ? 1.0f : z != z ? z : 0.0f;
        case GBMUF_ACT_GELU:
            return 0.5f * erfcf(-0.70710678118654752f * z) + z * 0.39894228040143268f * expf(-0.5f * z * z);
        case GBMUF_ACT_SILU: {
            const float p = 1.0f / (1.0f + expf(-z)), q = 1.0f / (1.0f + expf(z));
            return p + z * p * q;
        }
        case GBMUF_ACT_SIGMOID: {                                  // e / (1 + e)^2, which does not cancel
            const float e = expf(-fabsf(z)), d = 1.0f + e;
            return e / (d * d);
        }
        case GBMUF_ACT_TANH: {
            const float e = expf(-2.0f * fabsf(z)), d = 1.0f + e;
            return 4.0f * e / (d * d);
        }
        default: return 1.0f;
    }
}

__device__ __forceinline__ v4f load_four(const void *p, int64_t i, int32_t type)
{
    return type == kF32 ? read4<kF32>(p, i) : type == kBf16 ? read4<kBf16>(p, i) : read4<kF16>(p, i);
}

__device__ __forceinline__ void store_four(void *p, int64_t i, int32_t type, v4f v)
{
    if (type == kF32) write4<kF32>(p, i, v);
    else if (type == kBf16) write4<kBf16>(p, i, v);
    else write4<kF16>(p, i, v);
}

// What follows the sums of `left` of four elements side by side (m, n) ..: vectors where there are four, at any alignment.
__device__ __forceinline__ void finish(const Epilogue &e, int64_t g, int64_t m, int64_t n, int left, v4f z)
{
    const bool four = left >= 4;
    const auto load = [&](const void *p, int64_t i) {
        if (four) return load_four(p, i, e.type);
        v4f v = {0.0f, 0.0f, 0.0f, 0.0f};
        v[0] = load_one(p, i, e.type);
        if (left > 1) v[1] = load_one(p, i + 1, e.type);
        if (left > 2) v[2] = load_one(p, i + 2, e.type);
        return v;
    };
    const auto store = [&](void *p, int64_t i, v4f v) {
        if (four) return store_four(p, i, e.type, v);
        store_one(p, i, e.type, v[0]);
        if (left > 1) store_one(p, i + 1, e.type, v[1]);
        if (left > 2) store_one(p, i + 2, e.type, v[2]);
    };
    if (e.bias) z += load(e.bias, g * e.bias_batch + n);
    v4f r = {0.0f, 0.0f, 0.0f, 0.0f};
    if (e.place) r = load(e.res, g * e.r_batch + m * e.ldr + n);
    if (e.place == GBMUF_RESIDUAL_BEFORE) z += r;
    if (e.pre) store(e.pre, g * e.p_batch + m * e.ldp + n, z);
    if (e.act)
        for (int c = 0; c < 4; ++c) z[c] = activate(z[c], e.act);
    if (e.place == GBMUF_RESIDUAL_AFTER) z += r;
    store(e.y, g * e.y_batch + m * e.ldy + n, z);
}

struct Eight {
    v4f v[2];
};

template <int T>
__device__ __forceinline__ Eight read8(const void *p, int64_t i)
{
    if constexpr (T == kF32) return Eight{{read4<T>(p, i), read4<T>(p, i + 4)}};
    typedef typename Num<T>::type N8 __attribute__((ext_vector_type(8), aligned(2)));
    const N8 r = *reinterpret_cast<const N8 *>(static_cast<const typename Num<T>::type *>(p) + i);
    Eight e;
#pragma unroll
    for (int c = 0; c < 8; ++c) e.v[c >> 2][c & 3] = static_cast<float>(r[c]);
    return e;
}

template <int T>
__device__ __forceinline__ void write8(void *p, int64_t i, const Eight &e)
{
    using N = typename Num<T>::type;
    if constexpr (T == kF32) {
        write4<T>(p, i, e.v[0]);
        write4<T>(p, i + 4, e.v[1]);
    } else {
        typedef N N8 __attribute__((ext_vector_type(8), aligned(2)));
        N8 r;
#pragma unroll
        for (int c = 0; c < 8; ++c) r[c] = static_cast<N>(e.v[c >> 2][c & 3]);
        *reinterpret_cast<N8 *>(static_cast<N *>(p) + i) = r;
    }
}

__device__ __forceinline__ Eight load_eight(const void *p, int64_t i, int32_t type)
{
    return type == kF32 ? read8<kF32>(p, i) : type == kBf16 ? read8<kBf16>(p, i) : read8<kF16>(p, i);
}

__device__ __forceinline__ void store_eight(void *p, int64_t i, int32_t type, const Eight &v)
{
    if (type == kF32) write8<kF32>(p, i, v);
    else if (type == kBf16) write8<kBf16>(p, i, v);
    else write8<kF16>(p, i, v);
}

__device__ __forceinline__ Eight activate8(Eight z, int32_t act)
{
    const auto all = [&](auto f) {
#pragma unroll
        for (int c = 0; c < 8; ++c) z.v[c >> 2][c & 3] = f(z.v[c >> 2][c & 3]);
    };
    switch (act) {
        case GBMUF_ACT_RELU: all([](float v) { return activate(v, GBMUF_ACT_RELU); }); break;
        case GBMUF_ACT_GELU: all([](float v) { return activate(v, GBMUF_ACT_GELU); }); break;
        case GBMUF_ACT_SILU: all([](float v) { return activate(v, GBMUF_ACT_SILU); }); break;
        case GBMUF_ACT_SIGMOID: all([](float v) { return activate(v, GBMUF_ACT_SIGMOID); }); break;
        case GBMUF_ACT_TANH: all([](float v) { return activate(v, GBMUF_ACT_TANH); }); break;
        default: break;
    }
    return z;
}

// What follows 8 sums side by side, of which `left` are the matrix's.
__device__ __forceinline__ void finish8(const Epilogue &e, int64_t g, int64_t m, int64_t n, int left, Eight z)
{
    if (left < 8) {
        finish(e, g, m, n, left, z.v[0]);
        if (left > 4) finish(e, g, m, n + 4, left - 4, z.v[1]);
        return;
    }
    const auto add = [&](const Eight &o) {
        z.v[0] += o.v[0];
        z.v[1] += o.v[1];
    };
    Eight r{};
    if (e.place) r = load_eight(e.res, g * e.r_batch + m * e.ldr + n, e.type);
    if (e.bias) add(load_eight(e.bias, g * e.bias_batch + n, e.type));
    if (e.place == GBMUF_RESIDUAL_BEFORE) add(r);
    if (e.pre) store_eight(e.pre, g * e.p_batch + m * e.ldp + n, e.type, z);
    z = activate8(z, e.act);
    if (e.place == GBMUF_RESIDUAL_AFTER) add(r);
    store_eight(e.y, g * e.y_batch + m * e.ldy + n, e.type, z);
}

// v times the slope at z
__device__ __forceinline__ Eight slope8(Eight v, const Eight &z, int32_t act)
{
    const auto all = [&](auto f) {
#pragma unroll
        for (int c = 0; c < 8; ++c) v.v[c >> 2][c & 3] *= f(z.v[c >> 2][c & 3]);
    };
    switch (act) {
        case GBMUF_ACT_RELU: all([](float t) { return slope(t, GBMUF_ACT_RELU); }); break;
        case GBMUF_ACT_GELU: all([](float t) { return slope(t, GBMUF_ACT_GELU); }); break;
        case GBMUF_ACT_SILU: all([](float t) { return slope(t, GBMUF_ACT_SILU); }); break;
        case GBMUF_ACT_SIGMOID: all([](float t) { return slope(t, GBMUF_ACT_SIGMOID); }); break;
        case GBMUF_ACT_TANH: all([](float t) { return slope(t, GBMUF_ACT_TANH); }); break;
        default: break;
    }
    return v;
}

// The exponent of a scaled row of a split matrix: values are taken times 2^-row_exponent, the largest lies in [2^14, 2^15)
// then.  bits: of the largest magnitude (infinity and NaN count as the largest finite exponent).
__device__ __forceinline__ int row_exponent(uint32_t bits)
{
    const int e = static_cast<int>(bits >> 23);
    return (e > 254 ? 254 : e < 1 ? 1 : e) - 127 - 14;
}

}  // namespace
}  // namespace gbmuf
