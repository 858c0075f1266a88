// The norm over many tensors, g = sqrt(sum of all squares), and the tensors
// scaled to a limit of it: t min(1, limit / g).
//
// Squares are formed and added in float64 (a float32 square overflows from 1.8e19
// and vanishes below 1e-23), by blocks whose sums are added in order.  The
// tensors' places come as kernel arguments, kNormMost or kScaleMost a launch, so
// that a captured launch needs no memory of the host.  The second pass adds the
// blocks' sums again in every block, which is less than a launch of its own; it
// goes backwards, so that what the first pass read last and the last-level cache
// still holds is read first.
//
// Bound by the memory's rate: 16 bytes a lane, at any address.
#include <math.h>

#include "km_tile.h"

namespace km {

namespace {

constexpr int kNormMost = 165, kScaleMost = 120;   // tensors a launch: under 4 KB of arguments
constexpr int kThreads = 256;
constexpr int kClipUnroll = 4;                    // loads in flight a lane

struct NormSet {
    struct {
        const void* p;
        int64_t n;
        int32_t first, type;   // first block, row type
    } t[kNormMost];
    int32_t count, blocks, step;   // step: elements a block
    double* part;
};
struct ScaleSet {
    struct {
        const void* p;
        void* q;
        int64_t n;
        int32_t first, type;
    } t[kScaleMost];
    int32_t count, blocks, step, parts;
    const double* part;   // of all tensors
    double limit;
    float* norm;          // written by the first block of a launch, or null
};

// The tensor of a block: the last whose first block is not behind it.
template <class S>
__device__ __forceinline__ int tensor_of(const S& A, int block) {
    int lo = 0, hi = A.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (A.t[mid].first <= block) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ double block_sum(double v, double* s) {
#pragma unroll
    for (int o = 32; o > 0; o /= 2) v += __shfl_xor(v, o);
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    v = (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
    return v;
}

template <class T>
__device__ __forceinline__ double squares(const T* p, int64_t a, int64_t b) {
    constexpr int E = 16 / (int)sizeof(T);
    double sum = 0.0;
    const int64_t whole = a + (b - a) / (kThreads * E * kClipUnroll) * (kThreads * E * kClipUnroll);
    for (int64_t i = a + threadIdx.x * E; i < whole; i += kThreads * E * kClipUnroll) {
        Vec<T, E> v[kClipUnroll];
#pragma unroll
        for (int y = 0; y < kClipUnroll; ++y) __builtin_memcpy(&v[y], p + i + y * kThreads * E, 16);
#pragma unroll
        for (int y = 0; y < kClipUnroll; ++y)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const double x = (double)to_f32(v[y].e[e]);
                sum = fma(x, x, sum);
            }
    }
    for (int64_t i = whole + threadIdx.x; i < b; i += kThreads) {
        const double x = (double)to_f32(p[i]);
        sum = fma(x, x, sum);
    }
    return sum;
}

__global__ __launch_bounds__(kThreads) void k_clip_norm(NormSet A) {
    __shared__ double s[4];
    const int t = tensor_of(A, blockIdx.x);
    const int64_t a = (int64_t)(blockIdx.x - A.t[t].first) * A.step, n = A.t[t].n, b = a + A.step < n ? a + A.step : n;
    double v;
    if (A.t[t].type == kF32) v = squares(static_cast<const float*>(A.t[t].p), a, b);
    else if (A.t[t].type == kBF16) v = squares(static_cast<const __bf16*>(A.t[t].p), a, b);
    else v = squares(static_cast<const _Float16*>(A.t[t].p), a, b);
    v = block_sum(v, s);
    if (threadIdx.x == 0) A.part[blockIdx.x] = v;
}

__device__ __forceinline__ double all_parts(const double* part, int n, double* s) {
    double v = 0.0;
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += kThreads) v += part[i];
    return sqrt(block_sum(v, s));
}

__global__ __launch_bounds__(kThreads) void k_clip_total(const double* part, int n, float* norm) {
    __shared__ double s[4];
    const double g = all_parts(part, n, s);
    if (threadIdx.x == 0) *norm = (float)g;
}

template <class T>
__device__ __forceinline__ void scaled(const T* p, T* q, int64_t a, int64_t b, float f) {
    constexpr int E = 16 / (int)sizeof(T);
    const int64_t whole = a + (b - a) / (kThreads * E * kClipUnroll) * (kThreads * E * kClipUnroll);
    for (int64_t i = a + threadIdx.x * E; i < whole; i += kThreads * E * kClipUnroll) {
        Vec<T, E> v[kClipUnroll];
#pragma unroll
        for (int y = 0; y < kClipUnroll; ++y) __builtin_memcpy(&v[y], p + i + y * kThreads * E, 16);
#pragma unroll
        for (int y = 0; y < kClipUnroll; ++y) {
#pragma unroll
            for (int e = 0; e < E; ++e) v[y].e[e] = from_f32<T>(to_f32(v[y].e[e]) * f);
            __builtin_memcpy(q + i + y * kThreads * E, &v[y], 16);
        }
    }
    for (int64_t i = whole + threadIdx.x; i < b; i += kThreads) q[i] = from_f32<T>(to_f32(p[i]) * f);
}

__global__ __launch_bounds__(kThreads) void k_clip_scale(ScaleSet A) {
    __shared__ double s[4];
    const double g = all_parts(A.part, A.parts, s);
    if (A.norm && blockIdx.x == 0 && threadIdx.x == 0) *A.norm = (float)g;
    // A norm that is not finite leaves the tensors as they are.
    const float f = g > A.limit && g < INFINITY ? (float)(A.limit / g) : 1.0f;
    const int block = A.blocks - 1 - (int)blockIdx.x, t = tensor_of(A, block);
    const auto& e = A.t[t];
    if (f == 1.0f && e.p == e.q) return;
    const int64_t a = (int64_t)(block - e.first) * A.step, b = a + A.step < e.n ? a + A.step : e.n;
    if (e.type == kF32) scaled(static_cast<const float*>(e.p), static_cast<float*>(e.q), a, b, f);
    else if (e.type == kBF16) scaled(static_cast<const __bf16*>(e.p), static_cast<__bf16*>(e.q), a, b, f);
    else scaled(static_cast<const _Float16*>(e.p), static_cast<_Float16*>(e.q), a, b, f);
}

static_assert(sizeof(NormSet) <= 4096 && sizeof(ScaleSet) <= 4096, "");

}  // namespace

ClipShape clip_shape(const int64_t* sizes, int32_t count) {
    ClipShape L{};
    int64_t total = 0;
    for (int32_t i = 0; i < count; ++i) total += sizes[i];
    // Some 8 blocks a compute unit, none below 4096 elements.
    L.step = 4096;
    while (L.step < (1 << 30) && total / L.step > 4096) L.step *= 2;
    for (int32_t i = 0; i < count; ++i) L.parts += (sizes[i] + L.step - 1) / L.step;
    L.bytes = ((size_t)L.parts * 8 + 255) / 256 * 256;
    if (L.bytes == 0) L.bytes = 256;
    return L;
}

hipError_t launch_clip_norm(const void* const* p, const int64_t* sizes, const int32_t* types, int32_t count,
                            const ClipShape& L, double* part, hipStream_t s) {
    int64_t done = 0;
    NormSet A{};
    A.step = L.step;
    for (int32_t i = 0; i <= count; ++i) {
        if (A.count == kNormMost || (i == count && A.count > 0)) {
            A.part = part + done;
            hipLaunchKernelGGL(k_clip_norm, dim3((unsigned)A.blocks), dim3(kThreads), 0, s, A);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            done += A.blocks;
            A.count = A.blocks = 0;
        }
        if (i == count || sizes[i] == 0) continue;
        auto& t = A.t[A.count++];
        t.p = p[i];
        t.n = sizes[i];
        t.type = types[i];
        t.first = A.blocks;
        A.blocks += (int32_t)((sizes[i] + L.step - 1) / L.step);
    }
    return hipSuccess;
}

hipError_t launch_clip_total(const ClipShape& L, const double* part, float* norm, hipStream_t s) {
    hipLaunchKernelGGL(k_clip_total, dim3(1), dim3(kThreads), 0, s, part, (int)L.parts, norm);
    return hipGetLastError();
}

hipError_t launch_clip_scale(const void* const* p, void* const* q, const int64_t* sizes, const int32_t* types,
                             int32_t count, const ClipShape& L, const double* part, double limit, float* norm,
                             hipStream_t s) {
    ScaleSet A{};
    A.step = L.step;
    A.part = part;
    A.parts = (int32_t)L.parts;
    A.limit = limit;
    A.norm = norm;
    for (int32_t i = count - 1; i >= -1; --i) {   // the last tensors first, as in a launch
        if (A.count == kScaleMost || (i < 0 && A.count > 0)) {
            hipLaunchKernelGGL(k_clip_scale, dim3((unsigned)A.blocks), dim3(kThreads), 0, s, A);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            A.count = A.blocks = 0;
            A.norm = nullptr;
        }
        if (i < 0 || sizes[i] == 0) continue;
        auto& t = A.t[A.count++];
        t.p = p[i];
        t.q = q[i];
        t.n = sizes[i];
        t.type = types[i];
        t.first = A.blocks;
        A.blocks += (int32_t)((sizes[i] + L.step - 1) / L.step);
    }
    return hipSuccess;
}

}  // namespace km
