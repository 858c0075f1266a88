// Layer norm of the rows: y = (x - mu) rs g + b with rs = 1 / sqrt(v + eps),
// v the mean square deviation, and its gradients
//   dx = rs (h - mean(h) - xh mean(h xh)),  h = dy g,  xh = (x - mu) rs,
//   dg = sum_rows dy xh,  db = sum_rows dy.
//
// A row stays in registers between the sum and the squared deviations, so it
// is read once and the variance is formed from deviations (no difference of
// large sums).  All arithmetic is float32.  L lanes share a row, each lane
// owning the same columns of every row, so the backward pass keeps its share
// of dg and db in registers over all rows of a block; a second kernel adds the
// blocks' sums in a fixed order.  Rows too wide for the registers are read
// again from cache.  Bound by the memory's rate.
#include "km_ops.h"

namespace km {

namespace {

constexpr int kNormThreads = 256;

// Sum over the L lanes of a row.  L = 256: over the block, through LDS; the
// caller alternates between two slots so that one barrier a sum is enough.
template <int L>
__device__ __forceinline__ float row_sum(float v, float (*s)[4], int slot) {
    if constexpr (L <= 64) {
        return group_sum<L>(v);
    } else {
        v = group_sum<64>(v);
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) s[slot][wave] = v;
        __syncthreads();
        return (s[slot][0] + s[slot][1]) + (s[slot][2] + s[slot][3]);
    }
}

__device__ __forceinline__ float param_at(const void* p, int f32, int type, int64_t i) {
    if (f32 || type == kF32) return static_cast<const float*>(p)[i];
    if (type == kBF16) return (float)static_cast<const __bf16*>(p)[i];
    return (float)static_cast<const _Float16*>(p)[i];
}

template <class T>
constexpr int type_of() {
    return sizeof(T) == 4 ? kF32 : __is_same(T, __bf16) ? kBF16 : kF16;
}

// R steps of V elements a lane: d <= L R V.
template <class T, int V, int L, int R>
__global__ __launch_bounds__(kNormThreads) void k_norm_fwd(NormArgs A) {
    using W = Vec<T, V>;
    __shared__ float s_red[2][4];
    const int l = threadIdx.x % L, nv = A.d / V;
    const float dim = (float)A.d;
    constexpr int TY = type_of<T>();
    const int64_t step = (int64_t)gridDim.x * (kNormThreads / L);
    for (int64_t i = (int64_t)blockIdx.x * (kNormThreads / L) + threadIdx.x / L; i < A.n; i += step) {
        const W* __restrict__ x = reinterpret_cast<const W*>(static_cast<const T*>(A.X) + i * A.ldx);
        W* y = reinterpret_cast<W*>(static_cast<T*>(A.Y) + i * A.d);
        W v[R];
        float sum = 0.0f;
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (l + r * L < nv) {
                v[r] = x[l + r * L];
#pragma unroll
                for (int e = 0; e < V; ++e) sum += to_f32(v[r].e[e]);
            }
        const float mu = row_sum<L>(sum, s_red, 0) / dim;
        float sq = 0.0f;
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (l + r * L < nv)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float t = to_f32(v[r].e[e]) - mu;
                    sq = fmaf(t, t, sq);
                }
        const float rs = 1.0f / sqrtf(row_sum<L>(sq, s_red, 1) / dim + A.eps);
        if (l == 0) {
            A.mean[i] = mu;
            A.rstd[i] = rs;
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (l + r * L < nv) {
                W o;
                const int64_t c = (int64_t)(l + r * L) * V;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float g = A.gamma ? param_at(A.gamma, A.param_f32, TY, c + e) : 1.0f;
                    const float b = A.beta ? param_at(A.beta, A.param_f32, TY, c + e) : 0.0f;
                    o.e[e] = from_f32<T>(fmaf((to_f32(v[r].e[e]) - mu) * rs, g, b));
                }
                y[l + r * L] = o;
            }
    }
}

// Rows wider than the registers: a block a row, read three times (twice from cache).
template <class T, int V>
__global__ __launch_bounds__(kNormThreads) void k_norm_fwd_wide(NormArgs A) {
    using W = Vec<T, V>;
    __shared__ float s_red[2][4];
    const int nv = A.d / V;
    const float dim = (float)A.d;
    constexpr int TY = type_of<T>();
    for (int64_t i = blockIdx.x; i < A.n; i += gridDim.x) {
        const W* __restrict__ x = reinterpret_cast<const W*>(static_cast<const T*>(A.X) + i * A.ldx);
        W* y = reinterpret_cast<W*>(static_cast<T*>(A.Y) + i * A.d);
        float sum = 0.0f, sq = 0.0f;
#pragma unroll 4
        for (int c = threadIdx.x; c < nv; c += kNormThreads) {
            const W v = x[c];
#pragma unroll
            for (int e = 0; e < V; ++e) sum += to_f32(v.e[e]);
        }
        const float mu = row_sum<256>(sum, s_red, 0) / dim;
#pragma unroll 4
        for (int c = threadIdx.x; c < nv; c += kNormThreads) {
            const W v = x[c];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float t = to_f32(v.e[e]) - mu;
                sq = fmaf(t, t, sq);
            }
        }
        const float rs = 1.0f / sqrtf(row_sum<256>(sq, s_red, 1) / dim + A.eps);
        if (threadIdx.x == 0) {
            A.mean[i] = mu;
            A.rstd[i] = rs;
        }
#pragma unroll 2
        for (int c = threadIdx.x; c < nv; c += kNormThreads) {
            const W v = x[c];
            W o;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const int64_t q = (int64_t)c * V + e;
                const float g = A.gamma ? param_at(A.gamma, A.param_f32, TY, q) : 1.0f;
                const float b = A.beta ? param_at(A.beta, A.param_f32, TY, q) : 0.0f;
                o.e[e] = from_f32<T>(fmaf((to_f32(v.e[e]) - mu) * rs, g, b));
            }
            y[c] = o;
        }
    }
}

template <class T, int V, int L, int R>
__global__ __launch_bounds__(kNormThreads) void k_norm_bwd(NormArgs A) {
    using W = Vec<T, V>;
    __shared__ float s_red[2][4];
    constexpr int TY = type_of<T>(), kGroups = kNormThreads / L;
    const int l = threadIdx.x % L, nv = A.d / V;
    const float dim = (float)A.d;
    float g[R][V], dg[R][V], db[R][V];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            dg[r][e] = db[r][e] = 0.0f;
            const int64_t c = (int64_t)(l + r * L) * V + e;
            g[r][e] = A.gamma && l + r * L < nv ? param_at(A.gamma, A.param_f32, TY, c) : 1.0f;
        }
    const int64_t step = (int64_t)gridDim.x * kGroups;
    for (int64_t i = (int64_t)blockIdx.x * kGroups + threadIdx.x / L; i < A.n; i += step) {
        const W* __restrict__ x = reinterpret_cast<const W*>(static_cast<const T*>(A.X) + i * A.ldx);
        const W* __restrict__ y = reinterpret_cast<const W*>(static_cast<const T*>(A.dY) + i * A.lddy);
        W* dx = reinterpret_cast<W*>(static_cast<T*>(A.dX) + i * A.d);
        const float mu = A.mean[i], rs = A.rstd[i];
        W vx[R], vy[R];
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (l + r * L < nv) {
                vx[r] = x[l + r * L];
                vy[r] = y[l + r * L];
            }
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (l + r * L < nv)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float xh = (to_f32(vx[r].e[e]) - mu) * rs, dy = to_f32(vy[r].e[e]);
                    const float h = dy * g[r][e];
                    s1 += h;
                    s2 = fmaf(h, xh, s2);
                    dg[r][e] = fmaf(dy, xh, dg[r][e]);
                    db[r][e] += dy;
                }
        s1 = row_sum<L>(s1, s_red, 0) / dim;
        s2 = row_sum<L>(s2, s_red, 1) / dim;
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (l + r * L < nv) {
                W o;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float xh = (to_f32(vx[r].e[e]) - mu) * rs;
                    const float h = to_f32(vy[r].e[e]) * g[r][e];
                    o.e[e] = from_f32<T>(rs * (h - s1 - xh * s2));
                }
                dx[l + r * L] = o;
            }
    }
    if (!A.part) return;
    // The block's share: the groups of lanes that own the same columns are
    // added in group order.
    extern __shared__ float s_part[];   // (kGroups - 1) x 2 x R V L, none for one group
    float* out = A.part + (int64_t)blockIdx.x * 2 * A.d;
    constexpr int kCols = R * V * L;
    const int grp = threadIdx.x / L;
    if constexpr (kGroups > 1) {
        if (grp > 0) {
            float* m = s_part + (int64_t)(grp - 1) * 2 * kCols;
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    m[(r * V + e) * L + l] = dg[r][e];
                    m[kCols + (r * V + e) * L + l] = db[r][e];
                }
        }
        __syncthreads();
        if (grp > 0) return;
        for (int q = 0; q < kGroups - 1; ++q) {
            const float* m = s_part + (int64_t)q * 2 * kCols;
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    dg[r][e] += m[(r * V + e) * L + l];
                    db[r][e] += m[kCols + (r * V + e) * L + l];
                }
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (l + r * L < nv)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const int64_t c = (int64_t)(l + r * L) * V + e;
                out[c] = dg[r][e];
                out[A.d + c] = db[r][e];
            }
}

// Wide rows: a block a row; its sums of dg and db stay in its own row of
// part, each column owned by one lane.
template <class T, int V>
__global__ __launch_bounds__(kNormThreads) void k_norm_bwd_wide(NormArgs A) {
    using W = Vec<T, V>;
    __shared__ float s_red[2][4];
    constexpr int TY = type_of<T>();
    const int nv = A.d / V;
    const float dim = (float)A.d;
    float* out = A.part ? A.part + (int64_t)blockIdx.x * 2 * A.d : nullptr;
    bool first = true;
    for (int64_t i = blockIdx.x; i < A.n; i += gridDim.x, first = false) {
        const W* __restrict__ x = reinterpret_cast<const W*>(static_cast<const T*>(A.X) + i * A.ldx);
        const W* __restrict__ y = reinterpret_cast<const W*>(static_cast<const T*>(A.dY) + i * A.lddy);
        W* dx = reinterpret_cast<W*>(static_cast<T*>(A.dX) + i * A.d);
        const float mu = A.mean[i], rs = A.rstd[i];
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll 2
        for (int c = threadIdx.x; c < nv; c += kNormThreads) {
            const W vx = x[c], vy = y[c];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const int64_t q = (int64_t)c * V + e;
                const float g = A.gamma ? param_at(A.gamma, A.param_f32, TY, q) : 1.0f;
                const float xh = (to_f32(vx.e[e]) - mu) * rs, dy = to_f32(vy.e[e]), h = dy * g;
                s1 += h;
                s2 = fmaf(h, xh, s2);
                if (out) {
                    out[q] = first ? dy * xh : fmaf(dy, xh, out[q]);
                    out[A.d + q] = first ? dy : out[A.d + q] + dy;
                }
            }
        }
        s1 = row_sum<256>(s1, s_red, 0) / dim;
        s2 = row_sum<256>(s2, s_red, 1) / dim;
#pragma unroll 2
        for (int c = threadIdx.x; c < nv; c += kNormThreads) {
            const W vx = x[c], vy = y[c];
            W o;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const int64_t q = (int64_t)c * V + e;
                const float g = A.gamma ? param_at(A.gamma, A.param_f32, TY, q) : 1.0f;
                const float xh = (to_f32(vx.e[e]) - mu) * rs, h = to_f32(vy.e[e]) * g;
                o.e[e] = from_f32<T>(rs * (h - s1 - xh * s2));
            }
            dx[c] = o;
        }
    }
}

// dg and db: 64 columns a block, 4 waves take every fourth row of part.
__global__ __launch_bounds__(256) void k_norm_sums(NormArgs A) {
    __shared__ float s[2][4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = blockIdx.x * 64 + lane;
    float g = 0.0f, b = 0.0f;
    if (c < A.d) {
#pragma unroll 4
        for (int r = wave; r < A.blocks; r += 4) {
            g += A.part[(int64_t)r * 2 * A.d + c];
            b += A.part[(int64_t)r * 2 * A.d + A.d + c];
        }
    }
    s[0][wave][lane] = g;
    s[1][wave][lane] = b;
    __syncthreads();
    if (wave == 0 && c < A.d) {
        if (A.dgamma) A.dgamma[c] = (s[0][0][lane] + s[0][1][lane]) + (s[0][2][lane] + s[0][3][lane]);
        if (A.dbeta) A.dbeta[c] = (s[1][0][lane] + s[1][1][lane]) + (s[1][2][lane] + s[1][3][lane]);
    }
}

// Lanes a row and steps a lane by the row's vectors.
struct Shape {
    int L, R;
};
Shape norm_shape(int nv) {
    if (nv <= 8) return {8, 1};
    if (nv <= 32) return {32, 1};
    if (nv <= 64) return {64, 1};
    if (nv <= 128) return {64, 2};
    if (nv <= 256) return {64, 4};
    if (nv <= 512) return {256, 2};
    if (nv <= 1024) return {256, 4};
    return {256, 0};
}

int bwd_blocks(int64_t n, int nv) {
    const int64_t groups = kNormThreads / norm_shape(nv).L, b = (n + 8 * groups - 1) / (8 * groups);
    return (int)(b < 1 ? 1 : b > 512 ? 512 : b);
}

template <class T, int V, int L, int R>
hipError_t norm_go(const NormArgs& A, bool bwd, hipStream_t s) {
    const int groups = kNormThreads / L;
    if (bwd) {
        const size_t lds = A.part && groups > 1 ? (size_t)(groups - 1) * 2 * R * V * L * 4 : 0;
        hipLaunchKernelGGL((k_norm_bwd<T, V, L, R>), dim3((unsigned)A.blocks), dim3(kNormThreads), lds, s, A);
    } else {
        int64_t b = (A.n + groups - 1) / groups;
        if (b > 32768) b = 32768;
        hipLaunchKernelGGL((k_norm_fwd<T, V, L, R>), dim3((unsigned)b), dim3(kNormThreads), 0, s, A);
    }
    return hipGetLastError();
}

template <class T, int V>
hipError_t norm_vec(const NormArgs& A, bool bwd, hipStream_t s) {
    const Shape S = norm_shape(A.d / V);
    if (S.L == 8) return norm_go<T, V, 8, 1>(A, bwd, s);
    if (S.L == 32) return norm_go<T, V, 32, 1>(A, bwd, s);
    if (S.L == 64 && S.R == 1) return norm_go<T, V, 64, 1>(A, bwd, s);
    if (S.L == 64 && S.R == 2) return norm_go<T, V, 64, 2>(A, bwd, s);
    if (S.L == 64 && S.R == 4) return norm_go<T, V, 64, 4>(A, bwd, s);
    if (S.R == 2) return norm_go<T, V, 256, 2>(A, bwd, s);
    if (S.R == 4) return norm_go<T, V, 256, 4>(A, bwd, s);
    if (bwd) {
        hipLaunchKernelGGL((k_norm_bwd_wide<T, V>), dim3((unsigned)A.blocks), dim3(kNormThreads), 0, s, A);
    } else {
        const int64_t b = A.n < 32768 ? A.n : 32768;
        hipLaunchKernelGGL((k_norm_fwd_wide<T, V>), dim3((unsigned)b), dim3(kNormThreads), 0, s, A);
    }
    return hipGetLastError();
}

template <class T>
hipError_t norm_type(NormArgs& A, bool bwd, hipStream_t s) {
    bool vec = rows_vec16(A.X, A.ldx, A.d, sizeof(T));
    if (bwd)
        vec = vec && rows_vec16(A.dY, A.lddy, A.d, sizeof(T)) && rows_vec16(A.dX, A.d, A.d, sizeof(T));
    else
        vec = vec && rows_vec16(A.Y, A.d, A.d, sizeof(T));
    constexpr int V = 16 / (int)sizeof(T);
    A.blocks = bwd_blocks(A.n, vec ? A.d / V : A.d);
    return vec ? norm_vec<T, V>(A, bwd, s) : norm_vec<T, 1>(A, bwd, s);
}

hipError_t norm_any(NormArgs& A, bool bwd, int type, hipStream_t s) {
    if (type == kF32) return norm_type<float>(A, bwd, s);
    if (type == kBF16) return norm_type<__bf16>(A, bwd, s);
    return norm_type<_Float16>(A, bwd, s);
}

}  // namespace

// Blocks of the backward pass: at least 8 rows a group of lanes where there
// are that many, and at most 512.
int norm_bwd_max_blocks(int64_t n, int32_t d, int type) {
    const int a = bwd_blocks(n, d), b = bwd_blocks(n, (int)(d * row_type_bytes(type) / 16));
    return a > b ? a : b;
}

hipError_t launch_norm_fwd(NormArgs A, int type, hipStream_t s) {
    return A.n == 0 ? hipSuccess : norm_any(A, false, type, s);
}

hipError_t launch_norm_bwd(NormArgs A, int type, hipStream_t s) {
    if (A.n > 0) {
        hipError_t e = norm_any(A, true, type, s);
        if (e != hipSuccess) return e;
    }
    if (!A.dgamma && !A.dbeta) return hipSuccess;
    // No rows: blocks is 0 and the sums are zeros.
    hipLaunchKernelGGL(k_norm_sums, dim3((unsigned)((A.d + 63) / 64)), dim3(256), 0, s, A);
    return hipGetLastError();
}

}  // namespace km
