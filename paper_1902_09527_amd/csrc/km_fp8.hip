// Rows in 8-bit floating point with a power of two for each 128 elements:
//   a = the block's largest finite magnitude,
//   e = max(-126, the least whole number with a <= 448 2^e),  byte e + 127,
//   q = x 2^-e rounded to the nearest e4m3 value (ties to even),
// 448 = 1.75 2^8 being the largest e4m3 value, so no finite value overflows; what
// is not finite becomes NaN and does not count for a.  x 2^-e is exact in float32
// (or below half of the least e4m3 value), so q is rounded once.
//
// 16 lanes share a block, 8 elements each (the maximum over a row of 16 lanes is four
// cross-lane moves), four blocks of a lane in flight.  Bound by the memory's rate:
// 16,383 x 4100 bf16, 41 us, 5.1 TB/s.  Back from 8 bits a lane takes one block at a
// time: to bf16 37 us (5.5 TB/s), to float32 95 (3.5).
#include <math.h>

#include "km_tile.h"

namespace km {

namespace {

constexpr int kBlock = 128;
constexpr int kLanes = 16, kEach = kBlock / kLanes;   // lanes of a block, elements of a lane

// Elements c .. c + 8 of a row of d, zero past its end, at any address.
template <class T>
__device__ __forceinline__ void row_get(const T* row, int64_t c, int64_t d, T (&v)[kEach]) {
    if (c + kEach <= d) {
        __builtin_memcpy(v, row + c, sizeof(v));
    } else {
#pragma unroll
        for (int e = 0; e < kEach; ++e) v[e] = row[c + e < d ? c + e : 0];
#pragma unroll
        for (int e = 0; e < kEach; ++e) v[e] = c + e < d ? v[e] : (T)0.0f;
    }
}
template <class T>
__device__ __forceinline__ void row_put(T* row, int64_t c, int64_t d, const T (&v)[kEach]) {
    if (c + kEach <= d) {
        __builtin_memcpy(row + c, v, sizeof(v));
    } else {
#pragma unroll
        for (int e = 0; e < kEach; ++e)
            if (c + e < d) row[c + e] = v[e];
    }
}

template <int CTRL>
__device__ __forceinline__ uint32_t max_dpp(uint32_t v) {
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xf, 0xf, false);
    return v > o ? v : o;
}

struct QuantArgs {
    const void* X;
    int64_t ldx, n;
    int32_t d, nb;
    uint8_t *Q, *E;
    int64_t ldq;      // bytes a row of Q
    int32_t dq;       // values written a row: d, or more (zeros past d)
};

template <class T>
__global__ __launch_bounds__(256) void k_quantize(QuantArgs A) {
    constexpr int UN = 4, kUnits = 256 / kLanes;   // blocks in flight a lane; side by side
    const int64_t total = A.n * A.nb, step = (int64_t)gridDim.x * kUnits;
    const int l = threadIdx.x % kLanes;
    for (int64_t u0 = (int64_t)blockIdx.x * kUnits + threadIdx.x / kLanes; u0 < total; u0 += UN * step) {
        T x[UN][kEach];
        int64_t row[UN];
        int32_t b[UN];
#pragma unroll
        for (int y = 0; y < UN; ++y) {
            const int64_t u = u0 + y * step < total ? u0 + y * step : u0;
            row[y] = u / A.nb;
            b[y] = (int32_t)(u - row[y] * A.nb);
            row_get(static_cast<const T*>(A.X) + row[y] * A.ldx, (int64_t)b[y] * kBlock + l * kEach, A.d, x[y]);
        }
#pragma unroll
        for (int y = 0; y < UN; ++y) {
            if (u0 + y * step >= total) break;
            float v[kEach];
            uint32_t most = 0;
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                v[e] = to_f32(x[y][e]);
                const uint32_t bits = __builtin_bit_cast(uint32_t, v[e]) & 0x7fffffff;
                const bool fin = bits < 0x7f800000;
                v[e] = fin ? v[e] : NAN;
                most = fin && bits > most ? bits : most;
            }
            most = max_dpp<0xb1>(most);
            most = max_dpp<0x4e>(most);
            most = max_dpp<0x141>(most);
            most = max_dpp<0x140>(most);
            // The exponent, one more above 1.75 times a power of two.
            int byte = (int)((most + 0x1fffff) >> 23) - 8;
            byte = byte > 1 ? byte : 1;
            const float scale = __builtin_bit_cast(float, (uint32_t)(254 - byte) << 23);
            uint32_t w[kEach / 4];
#pragma unroll
            for (int e = 0; e < kEach; e += 4) {
                int q = __builtin_amdgcn_cvt_pk_fp8_f32(v[e] * scale, v[e + 1] * scale, 0, false);
                w[e / 4] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[e + 2] * scale, v[e + 3] * scale, q, true);
            }
            uint8_t o[kEach];
            __builtin_memcpy(o, w, sizeof(o));
            row_put(A.Q + row[y] * A.ldq, (int64_t)b[y] * kBlock + l * kEach, A.dq, o);
            if (l == 0) A.E[row[y] * A.nb + b[y]] = (uint8_t)byte;
        }
    }
}

template <class T>
__global__ __launch_bounds__(256) void k_dequantize(QuantArgs A, T* out) {
    constexpr int kUnits = 256 / kLanes;
    const int64_t total = A.n * A.nb, step = (int64_t)gridDim.x * kUnits;
    const int l = threadIdx.x % kLanes;
    for (int64_t u = (int64_t)blockIdx.x * kUnits + threadIdx.x / kLanes; u < total; u += step) {
        const int64_t row = u / A.nb, b = u - row * A.nb, c = b * kBlock + l * kEach;
        uint8_t q[kEach];
        row_get(A.Q + row * A.ldq, c, A.d, q);
        const int byte = A.E[u];
        uint32_t w[kEach / 4];
        __builtin_memcpy(w, q, sizeof(w));
        T o[kEach];
        auto stands = [&](float v) { return from_f32<T>(byte < 255 ? ldexpf(v, byte - 127) : NAN); };
#pragma unroll
        for (int e = 0; e < kEach / 4; ++e) {
            o[4 * e] = stands(__builtin_amdgcn_cvt_f32_fp8(w[e], 0));
            o[4 * e + 1] = stands(__builtin_amdgcn_cvt_f32_fp8(w[e], 1));
            o[4 * e + 2] = stands(__builtin_amdgcn_cvt_f32_fp8(w[e], 2));
            o[4 * e + 3] = stands(__builtin_amdgcn_cvt_f32_fp8(w[e], 3));
        }
        row_put(out + row * A.d, c, A.d, o);
    }
}

unsigned quant_blocks(int64_t units, int each) {
    const int64_t b = (units + 16 * each - 1) / (16 * each);
    return (unsigned)(b < 1 ? 1 : b < 8192 ? b : 8192);
}

}  // namespace

hipError_t launch_quantize(const void* X, int64_t ldx, int64_t n, int32_t d, int type, uint8_t* Q, int64_t ldq,
                           int32_t dq, uint8_t* E, hipStream_t s) {
    if (n == 0) return hipSuccess;
    QuantArgs A{X, ldx, n, d, (d + kBlock - 1) / kBlock, Q, E, ldq, dq};
    const dim3 g(quant_blocks(n * A.nb, 4)), b(256);
    if (type == kF32) hipLaunchKernelGGL((k_quantize<float>), g, b, 0, s, A);
    else if (type == kBF16) hipLaunchKernelGGL((k_quantize<__bf16>), g, b, 0, s, A);
    else hipLaunchKernelGGL((k_quantize<_Float16>), g, b, 0, s, A);
    return hipGetLastError();
}

hipError_t launch_dequantize(const uint8_t* Q, const uint8_t* E, int64_t n, int32_t d, int type, void* X,
                             hipStream_t s) {
    if (n == 0) return hipSuccess;
    QuantArgs A{nullptr, 0, n, d, (d + kBlock - 1) / kBlock, const_cast<uint8_t*>(Q), const_cast<uint8_t*>(E), d, d};
    const dim3 g(quant_blocks(n * A.nb, 1)), b(256);
    if (type == kF32) hipLaunchKernelGGL((k_dequantize<float>), g, b, 0, s, A, static_cast<float*>(X));
    else if (type == kBF16) hipLaunchKernelGGL((k_dequantize<__bf16>), g, b, 0, s, A, static_cast<__bf16*>(X));
    else hipLaunchKernelGGL((k_dequantize<_Float16>), g, b, 0, s, A, static_cast<_Float16*>(X));
    return hipGetLastError();
}

}  // namespace km
