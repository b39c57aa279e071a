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

// e^x for x <= 0, within 2 units: 2^(x / ln 2), the quotient in two parts, of which the second is put in as 1 + r ln 2.  Nothing is left of it below -200.
// With it and the reciprocal instruction (1 unit) a logistic function takes 14 instructions, where expf and a division that rounds exactly take 27.  An
// epilogue's activation is done while the CU does nothing else: 4 x 5120 x 8192 x 1024 bf16, us without one 365, with relu 375, silu 410 (expf: 468),
// sigmoid 403 (458), tanh 430 (468), gelu 465 (545); its gradients with silu 825 (918), gelu 860 (966).
__device__ __forceinline__ float exp_below(float x)
{
    x = x < -200.0f ? -200.0f : x;
    const float t = x * 1.44269504f, r = fmaf(x, 1.92596299e-8f, fmaf(x, 1.44269504f, -t));
    return __builtin_amdgcn_exp2f(t) * fmaf(r, 0.69314718f, 1.0f);
}

__device__ __forceinline__ float logistic(float z)
{
    const float e = exp_below(-fabsf(z));
    return (z < 0.0f ? e : 1.0f) * __builtin_amdgcn_rcpf(1.0f + e);
}

// e = e^(-z^2 / 2), and the normal distribution's mass below z, half of erfc(-z / sqrt 2), which keeps its bits where it is small.  erfc(x) for x >= 0 is
// e^(-x^2) t p(t) with t = 1 / (1 + 0.4 x), p the polynomial of degree 9 nearest to e^(x^2) erfc(x) / t (by weighted least squares over
// 0 <= x <= 14: 1.8e-8 of it; nothing is left of e beyond).
struct Normal {
    float e, below;
};

__device__ __forceinline__ Normal normal(float z)
{
    float a = fabsf(z);
    a = a > 30.0f ? 30.0f : a;
    const float q = a * a, t = __builtin_amdgcn_rcpf(fmaf(a, 0.28284271f, 1.0f));
    Normal n;
    n.e = exp_below(-0.5f * q) * fmaf(fmaf(a, a, -q), -0.5f, 1.0f);
    float p = -0.0231016371f;
    const float c[] = {0.163407043f, -0.419151694f, 0.44375214f, -0.200491488f, 0.228449017f, 0.144222796f, 0.21192804f, 0.225295693f, 0.225690126f};
#pragma unroll
    for (int i = 0; i < 9; ++i) p = fmaf(p, t, c[i]);
    const float half = 0.5f * (p * t * n.e);
    n.below = z < 0.0f ? half : 1.0f - half;
    return n;
}

__device__ __forceinline__ float activate(float z, int32_t act)
{
    switch (act) {
        case GBMUF_ACT_RELU: return z > 0.0f ? z : z != z ? z : 0.0f;
        case GBMUF_ACT_GELU: return z * normal(z).below;
        case GBMUF_ACT_SILU: return z * logistic(z);
        case GBMUF_ACT_SIGMOID: return logistic(z);
        case GBMUF_ACT_TANH: {                                     // (1 - e) / (1 + e), or where that cancels Taylor's polynomial, to z^9
            const float e = exp_below(-2.0f * fabsf(z)), q = z * z;
            const float near = fmaf(q, fmaf(q, fmaf(q, fmaf(q, 62.0f / 2835.0f, -17.0f / 315.0f), 2.0f / 15.0f), -1.0f / 3.0f), 1.0f) * z;
            return fabsf(z) < 0.25f ? near : copysignf((1.0f - e) * __builtin_amdgcn_rcpf(1.0f + e), z);
        }
        default: return z;
    }
}

// act'(z)
__device__ __forceinline__ float slope(float z, int32_t act)
{
    switch (act) {
        case GBMUF_ACT_RELU: return z > 0.0f ? 1.0f : z != z ? z : 0.0f;
        case GBMUF_ACT_GELU: {
            const Normal n = normal(z);
            return n.below + z * 0.39894228f * n.e;
        }
        case GBMUF_ACT_SILU: {
            const float e = exp_below(-fabsf(z)), d = __builtin_amdgcn_rcpf(1.0f + e);
            return (z < 0.0f ? e : 1.0f) * d + z * (e * d * d);
        }
        case GBMUF_ACT_SIGMOID: {                                  // e / (1 + e)^2, which does not cancel
            const float e = exp_below(-fabsf(z)), d = __builtin_amdgcn_rcpf(1.0f + e);
            return e * d * d;
        }
        case GBMUF_ACT_TANH: {
            const float e = exp_below(-2.0f * fabsf(z)), d = __builtin_amdgcn_rcpf(1.0f + e);
            return 4.0f * e * d * d;
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

template <int T, bool STREAMED = false>
__device__ __forceinline__ void write8(void *p, int64_t i, const Eight &e)
{
    using N = typename Num<T>::type;
    constexpr int V = T == kF32 ? 4 : 8;
    typedef N Piece __attribute__((ext_vector_type(V), aligned(sizeof(N))));
#pragma unroll
    for (int k = 0; k < 8; k += V) {
        Piece r;
#pragma unroll
        for (int c = 0; c < V; ++c) r[c] = static_cast<N>(e.v[(k + c) >> 2][(k + c) & 3]);
        Piece *to = reinterpret_cast<Piece *>(static_cast<N *>(p) + i + k);
        if constexpr (STREAMED) __builtin_nontemporal_store(r, to);
        else *to = r;
    }
}

__device__ __forceinline__ Eight load_eight(const void *p, int64_t i, int32_t type)
{
    return type == kF32 ? read8<kF32>(p, i) : type == kBf16 ? read8<kBf16>(p, i) : read8<kF16>(p, i);
}

template <bool STREAMED = false>
__device__ __forceinline__ void store_eight(void *p, int64_t i, int32_t type, const Eight &v)
{
    if (type == kF32) write8<kF32, STREAMED>(p, i, v);
    else if (type == kBf16) write8<kBf16, STREAMED>(p, i, v);
    else write8<kF16, STREAMED>(p, i, v);
}

// An epilogue's y or pre.  Streamed, where that is more than the caches hold, it leaves them to the operands: 8 x 5120 x 8192 x 512 bf16 (671 MB) 469 us
// plain, 411 streamed, x 8197, whose rows end inside lines, 517 and 469.
__device__ __forceinline__ void store_result(const Epilogue &e, void *p, int64_t i, const Eight &v)
{
    if (e.streamed) store_eight<true>(p, i, e.type, v);
    else store_eight(p, i, e.type, v);
}

template <int N>
__device__ __forceinline__ void activate_all(Eight (&z)[N], int32_t act)
{
    const auto all = [&](auto f) {
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int c = 0; c < 8; ++c) z[k].v[c >> 2][c & 3] = f(z[k].v[c >> 2][c & 3]);
    };
    switch (act) {
        case GBMUF_ACT_RELU: all([](float v) { return activate(v, GBMUF_ACT_RELU); }); break;
        case GBMUF_ACT_GELU: all([](float v) { return activate(v, GBMUF_ACT_GELU); }); break;
        case GBMUF_ACT_SILU: all([](float v) { return activate(v, GBMUF_ACT_SILU); }); break;
        case GBMUF_ACT_SIGMOID: all([](float v) { return activate(v, GBMUF_ACT_SIGMOID); }); break;
        case GBMUF_ACT_TANH: all([](float v) { return activate(v, GBMUF_ACT_TANH); }); break;
        default: break;
    }
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
    if (e.pre) store_result(e, e.pre, g * e.p_batch + m * e.ldp + n, z);
    Eight one[1] = {z};
    activate_all(one, e.act);
    z = one[0];
    if (e.place == GBMUF_RESIDUAL_AFTER) add(r);
    store_result(e, e.y, g * e.y_batch + m * e.ldy + n, z);
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
// then.  bits: of the largest finite magnitude.
__device__ __forceinline__ int row_exponent(uint32_t bits)
{
    const int e = static_cast<int>(bits >> 23);
    return (e < 1 ? 1 : e) - 127 - 14;
}

}  // namespace
}  // namespace gbmuf
