// Tiles of rows for the matrix cores (km_adapter.hip, km_group.hip): operand
// chunks, their moves to LDS and the transposing reads from it (km_places.h: where
// they lie).
#pragma once

#include <type_traits>

#include "km_ops.h"
#include "km_places.h"

namespace km {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

#define KM_LDS __attribute__((address_space(3)))
#define KM_GLOBAL __attribute__((address_space(1)))

// Where a lane reads past the end of a row or of the rows: 16 zero bytes.
__device__ __align__(16) const uint32_t zero_chunk[4] = {0, 0, 0, 0};

// 16-byte operand chunks: E elements of one row (or column) along the
// contraction.  A 64-lane operand is 16 rows x 4 chunks; mma adds the product
// of two, D[m][n] += sum_k first[m][k] second[n][k], lane l holding rows m =
// 4 (l / 16) + 0..3 of column n = l % 16.  float32 takes four 16x16x4 steps.
template <class T>
struct Mma;
template <>
struct Mma<__bf16> {
    static constexpr int E = 8;
    static __device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c,
                                                       0, 0, 0);
    }
};
template <>
struct Mma<_Float16> {
    static constexpr int E = 8;
    static __device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0,
                                                      0, 0);
    }
};
template <>
struct Mma<float> {
    static constexpr int E = 4;
    static __device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
        const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], c, 0, 0, 0);
        return c;
    }
};

// Elements at positions k0 .. k0 + E of a row of K >= 1 elements, `stride`
// apart, zero past its end.  Without branches, so that a lane's loads are in
// flight together: past the end the row's first elements are read.
template <class T>
__device__ __forceinline__ u32x4 chunk_guarded(const T* row, int64_t k0, int64_t K, int64_t stride = 1) {
    constexpr int E = Mma<T>::E;
    Vec<T, E> v;
#pragma unroll
    for (int e = 0; e < E; ++e) v.e[e] = row[(k0 + e < K ? k0 + e : 0) * stride];
#pragma unroll
    for (int e = 0; e < E; ++e) v.e[e] = k0 + e < K ? v.e[e] : (T)0.0f;
    return __builtin_bit_cast(u32x4, v);
}
__device__ __forceinline__ u32x4 only_if(bool in, u32x4 v) {
    u32x4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = in ? v[i] : 0u;
    return o;
}
// The same for rows that can be read 16 bytes at a time (K a multiple of E):
// past the end the zero bytes are read, so that nothing waits for the load.
template <class T>
__device__ __forceinline__ u32x4 chunk_aligned(const T* row, int64_t k0, int64_t K, bool in = true) {
    return *(in && k0 < K ? reinterpret_cast<const u32x4*>(row + k0) : reinterpret_cast<const u32x4*>(zero_chunk));
}
template <class T>
__device__ __forceinline__ u32x4 chunk(const T* row, int64_t k0, int64_t K, bool aligned) {
    return aligned ? chunk_aligned(row, k0, K) : chunk_guarded(row, k0, K);   // `aligned` is uniform
}

// 16 bytes of a row from element k0 on, zero past its K elements, at any address.
// One value of four words: as elements, the compiler would load both branches' so.
template <class T>
__device__ __forceinline__ u32x4 chunk_any(const T* row, int64_t k0, int64_t K) {
    constexpr int E = 16 / (int)sizeof(T);
    if (k0 + E <= K) {
        u32x4 v;
        __builtin_memcpy(&v, row + k0, 16);
        return v;
    }
    Vec<T, E> v;
#pragma unroll
    for (int e = 0; e < E; ++e) v.e[e] = row[k0 + e < K ? k0 + e : 0];
#pragma unroll
    for (int e = 0; e < E; ++e) v.e[e] = k0 + e < K ? v.e[e] : (T)0.0f;
    return __builtin_bit_cast(u32x4, v);
}

// Four consecutive results, col0 .. of a row of P.
template <class T>
__device__ __forceinline__ void store4(T* row, int64_t col0, int64_t P, f32x4 v, bool aligned) {
    if (aligned && col0 + 4 <= P) {
        Vec<T, 4> o;
#pragma unroll
        for (int i = 0; i < 4; ++i) o.e[i] = from_f32<T>(v[i]);
        *reinterpret_cast<Vec<T, 4>*>(row + col0) = o;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (col0 + i < P) row[col0 + i] = from_f32<T>(v[i]);
    }
}

// One asynchronous 16-byte move a lane from `src` to LDS base + 16 lane.
__device__ __forceinline__ void load_lds16(const void* src, char* wave_base) {
    __builtin_amdgcn_global_load_lds((const KM_GLOBAL void*)src, (KM_LDS void*)wave_base, 16, 0, 0);
}

__device__ __forceinline__ int64_t row_of(const int32_t* order, int64_t place) { return order ? order[place] : place; }

// Operand of 16 columns c0 .. along rows k0 + 0 .. of a tile whose rows are the
// contraction (CPR chunks a row).  The swizzle is the same k0 rows further (a
// multiple of a matrix step), so `at` (tr_lane) is a lane's place for k0 = 0.
template <class T, int CPR>
__device__ __forceinline__ int tr_lane(int c0, int lane) {
    const int li = lane & 15, g = lane >> 4;
    if constexpr (sizeof(T) == 2) {
        const int k = g * 8 + (li >> 2), ch = c0 / 8 + ((li & 3) >> 1);
        return (k * CPR + swz_tr<T, CPR>(k, ch)) * 16 + (li & 1) * 8;
    } else {
        const int k = g * 4, c = c0 + li;
        return (k * CPR + swz_tr<T, CPR>(k, c / 4)) * 16 + (c & 3) * 4;
    }
}
template <class T, int CPR>
__device__ __forceinline__ u32x4 read_tr(const char* tile, int k0, int at) {
    if constexpr (sizeof(T) == 2) {
        s16x4 v[2];
#pragma unroll
        for (int t = 0; t < 2; ++t)
            v[t] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((KM_LDS s16x4*)(tile + at + (k0 + 4 * t) * CPR * 16));
        struct Two { s16x4 a, b; } w{v[0], v[1]};
        return __builtin_bit_cast(u32x4, w);
    } else {
        u32x4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = *reinterpret_cast<const uint32_t*>(tile + at + (k0 + j) * CPR * 16);
        return v;
    }
}

// The same for N operands (1, 2 or 4) at the places `at`, `k0` rows in, where
// loads to LDS are on their way: the compiler would let the transposing read
// wait for all of them (it cannot tell that they go elsewhere), so 16-bit
// operands are read and waited for in one piece here.
template <int OFF, int STEP>
__device__ __forceinline__ void tr_wait(u32x4 (&v)[1], const uint32_t (&p)[1]) {
    uint64_t x[2];
    asm volatile("ds_read_b64_tr_b16 %0, %2 offset:%3\n\t"
                 "ds_read_b64_tr_b16 %1, %2 offset:%4\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(x[0]), "=&v"(x[1])
                 : "v"(p[0]), "n"(OFF), "n"(OFF + STEP)
                 : "memory");
    struct Two { uint64_t a, b; };
    v[0] = __builtin_bit_cast(u32x4, Two{x[0], x[1]});
}
template <int OFF, int STEP>
__device__ __forceinline__ void tr_wait(u32x4 (&v)[2], const uint32_t (&p)[2]) {
    uint64_t x[4];
    asm volatile("ds_read_b64_tr_b16 %0, %4 offset:%6\n\t"
                 "ds_read_b64_tr_b16 %1, %4 offset:%7\n\t"
                 "ds_read_b64_tr_b16 %2, %5 offset:%6\n\t"
                 "ds_read_b64_tr_b16 %3, %5 offset:%7\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3])
                 : "v"(p[0]), "v"(p[1]), "n"(OFF), "n"(OFF + STEP)
                 : "memory");
    struct Two { uint64_t a, b; };
#pragma unroll
    for (int i = 0; i < 2; ++i) v[i] = __builtin_bit_cast(u32x4, Two{x[2 * i], x[2 * i + 1]});
}
template <int OFF, int STEP>
__device__ __forceinline__ void tr_wait(u32x4 (&v)[4], const uint32_t (&p)[4]) {
    uint64_t x[8];
    asm volatile("ds_read_b64_tr_b16 %0, %8 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %1, %8 offset:%13\n\t"
                 "ds_read_b64_tr_b16 %2, %9 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %3, %9 offset:%13\n\t"
                 "ds_read_b64_tr_b16 %4, %10 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %5, %10 offset:%13\n\t"
                 "ds_read_b64_tr_b16 %6, %11 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %7, %11 offset:%13\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]),
                   "=&v"(x[7])
                 : "v"(p[0]), "v"(p[1]), "v"(p[2]), "v"(p[3]), "n"(OFF), "n"(OFF + STEP)
                 : "memory");
    struct Two { uint64_t a, b; };
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __builtin_bit_cast(u32x4, Two{x[2 * i], x[2 * i + 1]});
}
template <class T, int CPR, int K0, int N>
__device__ __forceinline__ void read_tr_wait(u32x4 (&v)[N], const char* tile, const int (&at)[N]) {
    if constexpr (sizeof(T) == 2) {
        uint32_t p[N];
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = (uint32_t)(uintptr_t)(KM_LDS const char*)(tile + at[i]);
        tr_wait<K0 * CPR * 16, 4 * CPR * 16>(v, p);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = read_tr<T, CPR>(tile, K0, at[i]);
    }
}

}  // namespace

}  // namespace km
