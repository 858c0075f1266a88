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
// Bound by the memory's rate: 16 bytes a lane.  Tensors lie at any address (views
// of a flat buffer): a block's range begins where 16 bytes are aligned, so the loads
// are.  400M bf16 at odd places: 183 us for the norm and 278 for the scaled values,
// 5.2 TB/s over both (201 and 322 with loads at any address).
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

// Elements of block i of a tensor of n at p: `step` of them, but that every block
// after the first begins at a multiple of 16 bytes, and `head` elements of the first
// are before one.
struct Range {
    int64_t a, head, b;
};
template <class T>
__device__ __forceinline__ Range range_of(const void* p, int64_t n, int64_t i, int64_t step) {
    const int64_t h = (int64_t)((16 - (uintptr_t)p % 16) % 16 / sizeof(T));
    const int64_t a = i == 0 ? 0 : h + i * step, b = h + (i + 1) * step;
    const int64_t end = b < n ? b : n, head = i == 0 ? h : a;
    return Range{a < n ? a : n, head < end ? head : end, end};
}

template <class T>
__device__ __forceinline__ double squares(const T* p, const Range& r) {
    constexpr int E = 16 / (int)sizeof(T);
    double sum = 0.0;
    auto one = [&](int64_t i) {
        const double x = (double)to_f32(p[i]);
        sum = fma(x, x, sum);
    };
    const int64_t whole = r.head + (r.b - r.head) / (kThreads * E * kClipUnroll) * (kThreads * E * kClipUnroll);
    for (int64_t i = r.head + threadIdx.x * E; i < whole; i += kThreads * E * kClipUnroll) {
        Vec<T, E> v[kClipUnroll];
#pragma unroll
        for (int y = 0; y < kClipUnroll; ++y) v[y] = *reinterpret_cast<const Vec<T, E>*>(p + i + y * kThreads * E);
#pragma unroll
        for (int y = 0; y < kClipUnroll; ++y)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const double x = (double)to_f32(v[y].e[e]);
                sum = fma(x, x, sum);
            }
    }
    for (int64_t i = r.a + threadIdx.x; i < r.head; i += kThreads) one(i);
    for (int64_t i = whole + threadIdx.x; i < r.b; i += kThreads) one(i);
    return sum;
}

__global__ __launch_bounds__(kThreads) void k_clip_norm(NormSet A) {
    __shared__ double s[4];
    const int t = tensor_of(A, blockIdx.x);
    const void* p = A.t[t].p;
    const int64_t i = blockIdx.x - A.t[t].first, n = A.t[t].n;
    double v;
    if (A.t[t].type == kF32) v = squares(static_cast<const float*>(p), range_of<float>(p, n, i, A.step));
    else if (A.t[t].type == kBF16) v = squares(static_cast<const __bf16*>(p), range_of<__bf16>(p, n, i, A.step));
    else v = squares(static_cast<const _Float16*>(p), range_of<_Float16>(p, n, i, A.step));
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

// The outputs' addresses may be aligned otherwise than the tensors': their stores are
// at any address.
template <class T>
__device__ __forceinline__ void scaled(const void* from, void* to, int64_t n, int64_t block, int64_t step, float f) {
    constexpr int E = 16 / (int)sizeof(T);
    const T* p = static_cast<const T*>(from);
    T* q = static_cast<T*>(to);
    const Range r = range_of<T>(from, n, block, step);
    auto one = [&](int64_t i) { q[i] = from_f32<T>(to_f32(p[i]) * f); };
    const int64_t whole = r.head + (r.b - r.head) / (kThreads * E * kClipUnroll) * (kThreads * E * kClipUnroll);
    for (int64_t i = r.head + threadIdx.x * E; i < whole; i += kThreads * E * kClipUnroll) {
        Vec<T, E> v[kClipUnroll];
#pragma unroll
        for (int y = 0; y < kClipUnroll; ++y) v[y] = *reinterpret_cast<const Vec<T, E>*>(p + i + y * kThreads * E);
#pragma unroll
        for (int y = 0; y < kClipUnroll; ++y) {
#pragma unroll
            for (int e = 0; e < E; ++e) v[y].e[e] = from_f32<T>(to_f32(v[y].e[e]) * f);
            __builtin_memcpy(q + i + y * kThreads * E, &v[y], 16);
        }
    }
    for (int64_t i = r.a + threadIdx.x; i < r.head; i += kThreads) one(i);
    for (int64_t i = whole + threadIdx.x; i < r.b; i += kThreads) one(i);
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
    const int64_t i = block - e.first;
    if (e.type == kF32) scaled<float>(e.p, e.q, e.n, i, A.step, f);
    else if (e.type == kBF16) scaled<__bf16>(e.p, e.q, e.n, i, A.step, f);
    else scaled<_Float16>(e.p, e.q, e.n, i, A.step, f);
}

static_assert(sizeof(NormSet) <= 4096 && sizeof(ScaleSet) <= 4096, "");

}  // namespace

ClipShape clip_shape(const int64_t* sizes, int32_t count) {
    ClipShape L{};
    int64_t total = 0;
    for (int32_t i = 0; i < count; ++i) total += sizes[i];
    // Blocks of at least 4096 elements.  Some 2048 sums, which every block of the
    // second pass adds again; more blocks there (800 MB: 1024 blocks 320 us, 16384
    // 296).
    auto step = [&](int64_t blocks) {
        const int64_t v = (total / blocks + 4095) / 4096 * 4096;
        return (int32_t)(v < 4096 ? 4096 : v < (1 << 30) ? v : 1 << 30);
    };
    L.step = step(2048);
    L.scale_step = step(16384);
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
    A.step = L.scale_step;
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
        A.blocks += (int32_t)((sizes[i] + L.scale_step - 1) / L.scale_step);
    }
    return hipSuccess;
}

}  // namespace km
