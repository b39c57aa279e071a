// gbmuf_stage.h -- operands of 16-bit numbers staged in LDS for gfx950's matrix cores, and the turns of a step that multiply them.
#pragma once

#include "gbmuf_tile.h"

#include <type_traits>

namespace gbmuf {
namespace {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

constexpr int kStep = 64;                                  // 16-bit words of a row per step: one 128-byte line

template <int T>
__device__ __forceinline__ v16f mfma(v4u a, v4u b, v16f c)
{
    if constexpr (T == kBf16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
}

// Stages R rows of one step in LDS: 128 bytes a row, the 16-byte chunk c of row r at place c ^ ((r / 2) & 7), so that 16 rows
// lie in all 64 banks, as a matrix instruction's operands are read (c ^ (r & 7): half of the LDS cycles were conflicts).  Whole steps go from global memory to LDS directly, 1 KB a wave and
// instruction, which writes lane by lane: the lanes fetch the chunk that belongs at their place.  A last step that is not whole goes
// through registers, zeros behind the end.
template <int R, int THREADS>
struct Stage {
    static constexpr int kPass = THREADS / 8, kPasses = R / kPass;
    const uint16_t *row[kPasses];

    __device__ __forceinline__ static int chunk(int i)
    {
        const int r = i * kPass + static_cast<int>(threadIdx.x >> 3);
        return (static_cast<int>(threadIdx.x & 7) ^ ((r >> 1) & 7)) * 8;
    }

    __device__ __forceinline__ void init(const uint16_t *base, int64_t ld, int first, int count)
    {
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            const int r = i * kPass + static_cast<int>(threadIdx.x >> 3);
            row[i] = base + static_cast<int64_t>(min(first + r, count - 1)) * ld + chunk(i);   // rows behind the last are read as the last one
        }
    }

    __device__ __forceinline__ void load(uint16_t *lds, int k0) const
    {
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            uint16_t *to = lds + (i * kPass + static_cast<int>(threadIdx.x >> 6) * 8) * kStep;
            __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) void *)(row[i] + k0),
                                             (__attribute__((address_space(3))) void *)to, 16, 0, 0);
        }
    }

    __device__ __forceinline__ void load_rest(uint16_t *lds, int k0, int K) const
    {
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            uint32_t v[4] = {0u, 0u, 0u, 0u};
            const int left = K - (k0 + chunk(i));
            if (left >= 8) {                               // rows lie on 16 bytes
                const v4u all = *reinterpret_cast<const v4u *>(row[i] + k0);
#pragma unroll
                for (int c = 0; c < 4; ++c) v[c] = all[c];
            } else {
#pragma unroll
                for (int c = 0; c < 7; ++c)
                    if (c < left) v[c >> 1] |= static_cast<uint32_t>(row[i][k0 + c]) << (16 * (c & 1));
            }
            const int r = i * kPass + static_cast<int>(threadIdx.x >> 3);
            *reinterpret_cast<v4u *>(lds + r * kStep + (threadIdx.x & 7) * 8) = v4u{v[0], v[1], v[2], v[3]};
        }
    }
};

__device__ __forceinline__ v4u chunk_of(const uint16_t *lds, int row, int chunk)
{
    return *reinterpret_cast<const v4u *>(lds + row * kStep + ((chunk ^ ((row >> 1) & 7)) * 8));
}

// The same for an operand whose k lie across its rows: a step is 64 rows of R columns, the 16-byte chunk c of row k at place c ^ ((k & 3) << 2), so
// that 4 rows of 32 columns lie in all banks.  The transposing load hands 16 lanes the 4 x 16 values that their addresses cover, a column of 4 k each.
template <int R, int THREADS>
struct StageAcross {
    static constexpr int kChunks = R / 8, kPass = THREADS / kChunks, kPasses = kStep / kPass;
    static_assert(kPass % 4 == 0, "every pass places its chunks alike");
    const uint16_t *row[kPasses];
    int64_t ld;

    __device__ __forceinline__ static int row_of() { return static_cast<int>(threadIdx.x) / kChunks; }

    // columns behind the last whole piece are read as that piece: their results are dropped
    __device__ __forceinline__ void init(const uint16_t *base, int64_t stride, int first, int count)
    {
        ld = stride;
        const int c = first + ((static_cast<int>(threadIdx.x) % kChunks) ^ ((row_of() & 3) << 2)) * 8;
#pragma unroll
        for (int i = 0; i < kPasses; ++i) row[i] = base + static_cast<int64_t>(i * kPass + row_of()) * stride + min(c, (count - 1) / 8 * 8);
    }

    __device__ __forceinline__ void load(uint16_t *lds, int k0) const
    {
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            uint16_t *to = lds + (i * THREADS + static_cast<int>(threadIdx.x >> 6) * 64) * 8;
            __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) void *)(row[i] + k0 * ld),
                                             (__attribute__((address_space(3))) void *)to, 16, 0, 0);
        }
    }

    __device__ __forceinline__ void load_rest(uint16_t *lds, int k0, int K) const
    {
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            v4u v = {0u, 0u, 0u, 0u};
            if (k0 + i * kPass + row_of() < K) v = *reinterpret_cast<const v4u *>(row[i] + k0 * ld);
            *reinterpret_cast<v4u *>(lds + (i * THREADS + static_cast<int>(threadIdx.x)) * 8) = v;
        }
    }
};

// Where a lane's pieces of the columns first .. first + 31 lie in a stage, in bytes, for its first k of turn 0.
template <int R>
__device__ __forceinline__ uint32_t column_place(int first)
{
    const int lane = threadIdx.x & 63, p = lane & 15, k = (lane >> 5) * 8 + (p >> 2), c = first + ((lane >> 4) & 1) * 16 + (p & 3) * 4;
    return static_cast<uint32_t>(k * R + (((c >> 3) ^ ((k & 3) << 2)) << 3) + (c & 4)) * 2;
}

// 8 k of a lane's column of each of N = 2, 4 or 6 fragments: four k at AT, four more 4 rows on.  One piece of assembly, with its wait: before
// a transposing load that the compiler knows, it waits for every load on its way to LDS, and with that for the whole next step (4 x 8192 x 1024 over 5120
// bf16 406 us).
#define GBMUF_READ(lo, hi, at, k, k4) "ds_read_b64_tr_b16 %" #lo ", %" #at " offset:%" #k "\n\tds_read_b64_tr_b16 %" #hi ", %" #at " offset:%" #k4 "\n\t"
#define GBMUF_TO(i) "=&v"(lo[i]), "=&v"(hi[i])
template <int AT, int ROW>
__device__ __forceinline__ void read_columns(const uint32_t (&at)[2], uint64_t (&lo)[2], uint64_t (&hi)[2])
{
    asm volatile(GBMUF_READ(0, 1, 4, 6, 7) GBMUF_READ(2, 3, 5, 6, 7) "s_waitcnt lgkmcnt(0)"
                 : GBMUF_TO(0), GBMUF_TO(1)
                 : "v"(at[0]), "v"(at[1]), "n"(AT), "n"(AT + 4 * ROW)
                 : "memory");
}
template <int AT, int ROW>
__device__ __forceinline__ void read_columns(const uint32_t (&at)[4], uint64_t (&lo)[4], uint64_t (&hi)[4])
{
    asm volatile(GBMUF_READ(0, 1, 8, 12, 13) GBMUF_READ(2, 3, 9, 12, 13) GBMUF_READ(4, 5, 10, 12, 13) GBMUF_READ(6, 7, 11, 12, 13) "s_waitcnt lgkmcnt(0)"
                 : GBMUF_TO(0), GBMUF_TO(1), GBMUF_TO(2), GBMUF_TO(3)
                 : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "n"(AT), "n"(AT + 4 * ROW)
                 : "memory");
}
template <int AT, int ROW>
__device__ __forceinline__ void read_columns(const uint32_t (&at)[6], uint64_t (&lo)[6], uint64_t (&hi)[6])
{
    asm volatile(GBMUF_READ(0, 1, 12, 18, 19) GBMUF_READ(2, 3, 13, 18, 19) GBMUF_READ(4, 5, 14, 18, 19) GBMUF_READ(6, 7, 15, 18, 19)
                     GBMUF_READ(8, 9, 16, 18, 19) GBMUF_READ(10, 11, 17, 18, 19) "s_waitcnt lgkmcnt(0)"
                 : GBMUF_TO(0), GBMUF_TO(1), GBMUF_TO(2), GBMUF_TO(3), GBMUF_TO(4), GBMUF_TO(5)
                 : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "v"(at[4]), "v"(at[5]), "n"(AT), "n"(AT + 4 * ROW)
                 : "memory");
}
#undef GBMUF_READ
#undef GBMUF_TO

// What a wave needs of a step for one turn of matrix instructions: 16 of the 64 words of its rows (SPLIT: 16 leading and the 16
// trailing parts).  m and n: the wave's first row of a and of b.
template <int T, bool SPLIT, int TM, int TN, int FM, int FN, int ACROSS>
struct Turn {
    static constexpr int kParts = SPLIT ? 2 : 1;
    v4u x[kParts][FM], w[kParts][FN];

    template <int TURN>
    __device__ __forceinline__ void load(const uint16_t *lds, int m, int n)
    {
        const int lane = threadIdx.x & 63;
        const uint16_t *la = lds, *lb = lds + TM * kStep;
#pragma unroll
        for (int p = 0; p < kParts; ++p) {
            const int c = p * 4 + TURN * 2 + (lane >> 5);
            if constexpr (!(ACROSS & 2))
#pragma unroll
                for (int j = 0; j < FN; ++j) w[p][j] = chunk_of(lb, n + j * 32 + (lane & 31), c);
            if constexpr (!(ACROSS & 1))
#pragma unroll
                for (int i = 0; i < FM; ++i) x[p][i] = chunk_of(la, m + i * 32 + (lane & 31), c);
        }
        if constexpr (ACROSS != 0) {
            static_assert(ACROSS == 2 || (ACROSS == 3 && TM == TN), "b across its rows, or both");
            constexpr int N = FN + (ACROSS & 1 ? FM : 0);
            const uint32_t stage = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const uint16_t *)lds));
            uint32_t at[N];
            uint64_t lo[N], hi[N];
#pragma unroll
            for (int j = 0; j < FN; ++j) at[j] = stage + TM * kStep * 2 + column_place<TN>(n + j * 32);
#pragma unroll
            for (int i = FN; i < N; ++i) at[i] = stage + column_place<TM>(m + (i - FN) * 32);
            read_columns<TURN * 16 * TN * 2, TN * 2>(at, lo, hi);
            const auto joined = [&](int i) {
                return v4u{static_cast<uint32_t>(lo[i]), static_cast<uint32_t>(lo[i] >> 32), static_cast<uint32_t>(hi[i]), static_cast<uint32_t>(hi[i] >> 32)};
            };
#pragma unroll
            for (int j = 0; j < FN; ++j) w[0][j] = joined(j);
#pragma unroll
            for (int i = FN; i < N; ++i) x[0][i - FN] = joined(i);
        }
    }

    __device__ __forceinline__ void multiply(v16f (&acc)[FM][FN]) const
    {
#pragma unroll
        for (int p = 0; p < (SPLIT ? 3 : 1); ++p)          // lead lead, trail lead, lead trail
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i][j] = mfma<T>(w[p == 1 ? 1 : 0][j], x[p == 2 ? 1 : 0][i], acc[i][j]);
    }
};

// Spreads READS loads of LDS evenly between MFMAS matrix instructions.
template <int READS, int MFMAS, int I = 0>
__device__ __forceinline__ void interleave()
{
    if constexpr (I < MFMAS) {
        constexpr int n = (I + 1) * READS / MFMAS - I * READS / MFMAS;
        if constexpr (n > 0) __builtin_amdgcn_sched_group_barrier(0x100, n, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        interleave<READS, MFMAS, I + 1>();
    }
}

// f(0), f(1) .. f(N - 1), the numbers known to the compiler
template <int N, class F>
__device__ __forceinline__ void repeat(F f)
{
    if constexpr (N > 0) {
        repeat<N - 1>(f);
        f(std::integral_constant<int, N - 1>{});
    }
}

// The waves meet, everything that they read of LDS at hand and (MEMORY) everything on its way to LDS there.  The wait is one that the compiler sees: it does
// not wait for what was read before once more, together with what is read next.
template <bool MEMORY>
__device__ __forceinline__ void meet()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(MEMORY ? 0x0070 : 0xc07f);  // vmcnt(0) lgkmcnt(0), or the latter alone
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

}  // namespace
}  // namespace gbmuf
