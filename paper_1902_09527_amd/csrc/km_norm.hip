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
// blocks' sums in a fixed order.  Rows too wide for the registers of 1024 lanes
// are read again from cache, and dg and db take a pass over columns.
//
// Bound by the memory's rate.  8192 x 4096 bf16: forward 23 us (5.9 TB/s),
// backward 44 (4.6) and sums 5; 1,000,003 x 250 float32 (two elements a lane):
// forward 450 us (4.5 TB/s), backward 593 to 630 (4.8 to 5.1) and sums 5.
#include "km_ops.h"

namespace km {

namespace {

constexpr int kNormThreads = 256;

// Rows after which a lane's sums of dg and db are added to its totals: the
// rounding errors of a sum grow with its terms, so a lane's n rows cost those of
// kFold + n / kFold terms (1,000,003 x 250 float32, 490 rows a lane: dg off by
// 2.0e-7 of its norm, 4.4e-7 in one sum; the time is the same).
constexpr int kFold = 32;
// The totals of 1024 lanes, or of 32 columns a lane and more, are kept in LDS: in
// registers they would leave half as many waves on the chip, or none of the
// registers that the next row is loaded to.
template <int V, int L, int R>
constexpr bool kFoldLds = L == 1024 || R * V >= 32;

// Threads of a block whose rows have L lanes each.
constexpr int norm_threads(int L) { return L > kNormThreads ? L : kNormThreads; }

// Sum over the L lanes of a row.  L >= 256: over the block, through LDS; the
// caller alternates between two slots so that one barrier a sum is enough.
template <int L>
__device__ __forceinline__ float row_sum(float v, float (*s)[16], int slot) {
    if constexpr (L <= 64) {
        return group_sum<L>(v);
    } else {
        v = group_sum<64>(v);
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) s[slot][wave] = v;
        __syncthreads();
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < L / 64; w += 4)
            sum += (s[slot][w] + s[slot][w + 1]) + (s[slot][w + 2] + s[slot][w + 3]);
        return sum;
    }
}

// V consecutive parameters (of type P) from column c; `fill` where there are
// none.  V > 1: c is a multiple of V and p 16-byte aligned.
template <class P, int V>
__device__ __forceinline__ void params(const void* p, int64_t c, float fill, float* out) {
    constexpr int S = V * sizeof(P) > 16 ? 16 / (int)sizeof(P) : V;
    if (!p) {
#pragma unroll
        for (int e = 0; e < V; ++e) out[e] = fill;
        return;
    }
#pragma unroll
    for (int q = 0; q < V / S; ++q) {
        const Vec<P, S> v = *reinterpret_cast<const Vec<P, S>*>(static_cast<const P*>(p) + c + q * S);
#pragma unroll
        for (int e = 0; e < S; ++e) out[q * S + e] = to_f32(v.e[e]);
    }
}

// R steps of V elements a lane: d <= L R V.
template <class T, class P, int V, int L, int R>
__global__ __launch_bounds__(norm_threads(L)) void k_norm_fwd(NormArgs A) {
    using W = Vec<T, V>;
    __shared__ float s_red[2][16];
    const int l = threadIdx.x % L, nv = A.d / V;
    const float dim = (float)A.d;
    float g[R][V], b[R][V];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const bool in = l + r * L < nv;
        params<P, V>(in ? A.gamma : nullptr, (int64_t)(l + r * L) * V, 1.0f, g[r]);
        params<P, V>(in ? A.beta : nullptr, (int64_t)(l + r * L) * V, 0.0f, b[r]);
    }
    constexpr int kGroups = norm_threads(L) / L;
    const int64_t step = (int64_t)gridDim.x * kGroups;
    int64_t i = (int64_t)blockIdx.x * kGroups + threadIdx.x / L;
    // The next row's loads are in flight while a row is worked on.
    W nx[R];
    auto fetch = [&](int64_t q) {
        const W* __restrict__ x = reinterpret_cast<const W*>(static_cast<const T*>(A.X) + q * A.ldx);
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (l + r * L < nv) nx[r] = x[l + r * L];
    };
    if (i < A.n) fetch(i);
    for (; i < A.n; i += step) {
        W* y = reinterpret_cast<W*>(static_cast<T*>(A.Y) + i * A.d);
        W v[R];
#pragma unroll
        for (int r = 0; r < R; ++r) v[r] = nx[r];
        if (i + step < A.n) fetch(i + step);
        float sum = 0.0f;
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (l + r * L < nv)
#pragma unroll
                for (int e = 0; e < V; ++e) sum += to_f32(v[r].e[e]);
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
#pragma unroll
                for (int e = 0; e < V; ++e)
                    o.e[e] = from_f32<T>(fmaf((to_f32(v[r].e[e]) - mu) * rs, g[r][e], b[r][e]));
                y[l + r * L] = o;
            }
    }
}

// Rows wider than the registers: a block a row, read three times (twice from cache).
template <class T, class P, int V>
__global__ __launch_bounds__(kNormThreads) void k_norm_fwd_wide(NormArgs A) {
    using W = Vec<T, V>;
    __shared__ float s_red[2][16];
    const int nv = A.d / V;
    const float dim = (float)A.d;
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
            float g[V], b[V];
            params<P, V>(A.gamma, (int64_t)c * V, 1.0f, g);
            params<P, V>(A.beta, (int64_t)c * V, 0.0f, b);
#pragma unroll
            for (int e = 0; e < V; ++e) o.e[e] = from_f32<T>(fmaf((to_f32(v.e[e]) - mu) * rs, g[e], b[e]));
            y[c] = o;
        }
    }
}

template <class T, class P, int V, int L, int R>
__global__ __launch_bounds__(norm_threads(L)) void k_norm_bwd(NormArgs A) {
    using W = Vec<T, V>;
    __shared__ float s_red[2][16];
    constexpr int kGroups = norm_threads(L) / L;
    const int l = threadIdx.x % L, nv = A.d / V;
    const float dim = (float)A.d;
    float g[R][V], dg[R][V], db[R][V];
    // Totals of dg and db: a lane's own, or its place in LDS, and that of its group.
    constexpr bool kLds = kFoldLds<V, L, R>;
    constexpr int kCols = R * V * L;
    extern __shared__ float s_part[];   // groups (kLds) or groups - 1 times 2 kCols; none without part
    const int grp = threadIdx.x / L;
    float tg[kLds ? 1 : R][V], tb[kLds ? 1 : R][V];
    auto place = [&](int q, int r, int e) { return s_part + q * 2 * kCols + (r * V + e) * L + l; };
#pragma unroll
    for (int r = 0; r < R; ++r) {
        params<P, V>(l + r * L < nv ? A.gamma : nullptr, (int64_t)(l + r * L) * V, 1.0f, g[r]);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            dg[r][e] = db[r][e] = 0.0f;
            if constexpr (!kLds) tg[r][e] = tb[r][e] = 0.0f;
        }
    }
    bool folded = false;
    auto fold = [&]() {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                if constexpr (kLds) {
                    place(grp, r, e)[0] = folded ? place(grp, r, e)[0] + dg[r][e] : dg[r][e];
                    place(grp, r, e)[kCols] = folded ? place(grp, r, e)[kCols] + db[r][e] : db[r][e];
                } else {
                    tg[r][e] += dg[r][e];
                    tb[r][e] += db[r][e];
                }
                dg[r][e] = db[r][e] = 0.0f;
                if (kLds && e % 4 == 3) __builtin_amdgcn_sched_barrier(0);   // few registers at a time
            }
        folded = true;
    };
    int rows = 0;
    const int64_t step = (int64_t)gridDim.x * kGroups;
    int64_t i = (int64_t)blockIdx.x * kGroups + threadIdx.x / L;
    // The next row's loads are in flight while a row is worked on.
    W nx[R], ny[R];
    float nmu = 0.0f, nrs = 0.0f;
    auto fetch = [&](int64_t q) {
        const W* __restrict__ x = reinterpret_cast<const W*>(static_cast<const T*>(A.X) + q * A.ldx);
        const W* __restrict__ y = reinterpret_cast<const W*>(static_cast<const T*>(A.dY) + q * A.lddy);
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (l + r * L < nv) {
                nx[r] = x[l + r * L];
                ny[r] = y[l + r * L];
            }
        nmu = A.mean[q];
        nrs = A.rstd[q];
    };
    if (i < A.n) fetch(i);
    for (; i < A.n; i += step) {
        W* dx = reinterpret_cast<W*>(static_cast<T*>(A.dX) + i * A.d);
        const float mu = nmu, rs = nrs;
        W vx[R], vy[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            vx[r] = nx[r];
            vy[r] = ny[r];
        }
        if (i + step < A.n) fetch(i + step);
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
        if (++rows == kFold && A.part) {
            fold();
            rows = 0;
        }
    }
    if (!A.part) return;
    constexpr bool kOwn = kLds && kGroups == 1;   // the last sums have not to go through LDS
    if constexpr (!kOwn) fold();
    // The block's share: the groups of lanes that own the same columns are
    // added in group order.
    float* out = A.part + (int64_t)blockIdx.x * 2 * A.d;
    constexpr int kOthers = kLds ? 0 : 1;   // the first group's place of the others'
    if constexpr (kGroups > 1) {
        if constexpr (!kLds) {
            if (grp > 0)
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        place(grp - 1, r, e)[0] = tg[r][e];
                        place(grp - 1, r, e)[kCols] = tb[r][e];
                    }
        }
        __syncthreads();
        if (grp > 0) return;
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (l + r * L < nv)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float sg = kOwn && !folded ? 0.0f : kLds ? place(0, r, e)[0] : tg[kLds ? 0 : r][e];
                float sb = kOwn && !folded ? 0.0f : kLds ? place(0, r, e)[kCols] : tb[kLds ? 0 : r][e];
                if constexpr (kOwn) {
                    sg += dg[r][e];
                    sb += db[r][e];
                }
                for (int q = 1; q < kGroups; ++q) {
                    sg += place(q - kOthers, r, e)[0];
                    sb += place(q - kOthers, r, e)[kCols];
                }
                const int64_t c = (int64_t)(l + r * L) * V + e;
                out[c] = sg;
                out[A.d + c] = sb;
            }
}

// Wider rows: a block a row, read twice (once from cache); dg and db apart.
template <class T, class P, int V>
__global__ __launch_bounds__(kNormThreads) void k_norm_bwd_wide(NormArgs A) {
    using W = Vec<T, V>;
    __shared__ float s_red[2][16];
    const int nv = A.d / V;
    const float dim = (float)A.d;
    for (int64_t i = blockIdx.x; i < A.n; i += gridDim.x) {
        const W* __restrict__ x = reinterpret_cast<const W*>(static_cast<const T*>(A.X) + i * A.ldx);
        const W* __restrict__ y = reinterpret_cast<const W*>(static_cast<const T*>(A.dY) + i * A.lddy);
        W* dx = reinterpret_cast<W*>(static_cast<T*>(A.dX) + i * A.d);
        const float mu = A.mean[i], rs = A.rstd[i];
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll 4
        for (int c = threadIdx.x; c < nv; c += kNormThreads) {
            const W vx = x[c], vy = y[c];
            float g[V];
            params<P, V>(A.gamma, (int64_t)c * V, 1.0f, g);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float xh = (to_f32(vx.e[e]) - mu) * rs, h = to_f32(vy.e[e]) * g[e];
                s1 += h;
                s2 = fmaf(h, xh, s2);
            }
        }
        s1 = row_sum<256>(s1, s_red, 0) / dim;
        s2 = row_sum<256>(s2, s_red, 1) / dim;
#pragma unroll 2
        for (int c = threadIdx.x; c < nv; c += kNormThreads) {
            const W vx = x[c], vy = y[c];
            W o;
            float g[V];
            params<P, V>(A.gamma, (int64_t)c * V, 1.0f, g);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float xh = (to_f32(vx.e[e]) - mu) * rs, h = to_f32(vy.e[e]) * g[e];
                o.e[e] = from_f32<T>(rs * (h - s1 - xh * s2));
            }
            dx[c] = o;
        }
    }
}

// Shares of dg and db for the wider rows: V columns a lane, blockIdx.y's run of
// rows (A.blocks of them), its sums in registers and written once.  Two reads
// more of the rows: backward of 8192 x 16384 float32 619 us (1100 with sums
// updated in memory row by row; 337 at a copy's rate).
template <class T, int V>
__global__ __launch_bounds__(kNormThreads) void k_norm_cols(NormArgs A) {
    using W = Vec<T, V>;
    const int nv = A.d / V, c = blockIdx.x * kNormThreads + threadIdx.x;
    if (c >= nv) return;
    const int64_t per = (A.n + A.blocks - 1) / A.blocks, i0 = blockIdx.y * per;
    const int64_t i1 = i0 + per < A.n ? i0 + per : A.n;
    float tg[V], tb[V];
#pragma unroll
    for (int e = 0; e < V; ++e) tg[e] = tb[e] = 0.0f;
    for (int64_t q = i0; q < i1; q += kFold) {
        const int64_t q1 = q + kFold < i1 ? q + kFold : i1;
        float dg[V], db[V];
#pragma unroll
        for (int e = 0; e < V; ++e) dg[e] = db[e] = 0.0f;
#pragma unroll 4
        for (int64_t i = q; i < q1; ++i) {
            const W vx = reinterpret_cast<const W*>(static_cast<const T*>(A.X) + i * A.ldx)[c];
            const W vy = reinterpret_cast<const W*>(static_cast<const T*>(A.dY) + i * A.lddy)[c];
            const float mu = A.mean[i], rs = A.rstd[i];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float dy = to_f32(vy.e[e]);
                dg[e] = fmaf(dy, (to_f32(vx.e[e]) - mu) * rs, dg[e]);
                db[e] += dy;
            }
        }
#pragma unroll
        for (int e = 0; e < V; ++e) {
            tg[e] += dg[e];
            tb[e] += db[e];
        }
    }
    float* out = A.part + (int64_t)blockIdx.y * 2 * A.d + (int64_t)c * V;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        out[e] = tg[e];
        out[A.d + e] = tb[e];
    }
}

// dg (blockIdx.y = 0) and db: 64 columns a block, 16 waves take every 16th
// row of part; their sums are added in wave order.
__global__ __launch_bounds__(1024) void k_norm_sums(NormArgs A) {
    __shared__ float s[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = blockIdx.x * 64 + lane;
    float* out = blockIdx.y ? A.dbeta : A.dgamma;
    if (!out) return;
    float sum = 0.0f;
    if (c < A.d) {
        const float* p = A.part + (blockIdx.y ? A.d : 0) + c;
#pragma unroll 8
        for (int r = wave; r < A.blocks; r += 16) sum += p[(int64_t)r * 2 * A.d];
    }
    s[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && c < A.d) {
        sum = 0.0f;
#pragma unroll
        for (int w = 0; w < 16; ++w) sum += s[w][lane];
        out[c] = sum;
    }
}

// Lanes a row and steps a lane by the row's vectors.
struct Shape {
    int L, R;
};
// Beyond 1024 vectors a row is a block's of 1024 lanes where that pays (both
// sides measured): backward of 18587 x 11456 bf16 286 us (1827 a row read
// twice), forward 210 (289); 16384 x 2050 bf16, two elements a lane: backward
// 71 us (232), but forward 65 (43 read three times).
Shape norm_shape(int nv, int V, bool bwd) {
    if (nv <= 8) return {8, 1};
    if (nv <= 32) return {32, 1};
    if (nv <= 64) return {64, 1};
    if (nv <= 128) return {64, 2};
    if (nv <= 256) return {64, 4};
    if (nv <= 512) return {256, 2};
    if (nv <= 1024) return {256, 4};
    if (nv <= 2048 && (bwd || V > 2)) return {1024, 2};
    // 16 bytes a lane have no room for more of a row.
    if (nv <= 4096 && V <= 2 && bwd) return {1024, 4};
    return {256, 0};
}

// Blocks of the backward pass: two rows a group of lanes where the rows are
// few, and at most 512 (each writes its sums of dg and db). Fewer vectors a
// row never make more blocks.
int bwd_blocks(int64_t n, int nv) {
    const int L = norm_shape(nv, 1, true).L;   // V matters from 256 lanes on only, where a block has one row anyhow
    const int64_t groups = norm_threads(L) / L, b = (n + 2 * groups - 1) / (2 * groups);
    return (int)(b < 1 ? 1 : b > 512 ? 512 : b);
}

template <class T, class P, int V, int L, int R>
hipError_t norm_go(const NormArgs& A, bool bwd, hipStream_t s) {
    constexpr int kThreads = norm_threads(L), groups = kThreads / L;
    if (bwd) {
        const size_t lds = A.part ? (size_t)(kFoldLds<V, L, R> ? groups : groups - 1) * 2 * R * V * L * 4 : 0;
        if (lds > 60 * 1024) {   // beyond what a kernel has without asking
            const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&k_norm_bwd<T, P, V, L, R>),
                                                     hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
            if (e != hipSuccess) return e;
        }
        hipLaunchKernelGGL((k_norm_bwd<T, P, V, L, R>), dim3((unsigned)A.blocks), dim3(kThreads), lds, s, A);
    } else {
        // At most 2048 blocks (8 a compute unit): gamma and beta are loaded once a block.
        int64_t b = (A.n + groups - 1) / groups;
        if (b > 2048) b = 2048;
        hipLaunchKernelGGL((k_norm_fwd<T, P, V, L, R>), dim3((unsigned)b), dim3(kThreads), 0, s, A);
    }
    return hipGetLastError();
}

template <class T, class P, int V>
hipError_t norm_vec(const NormArgs& A, bool bwd, hipStream_t s) {
    const Shape S = norm_shape(A.d / V, V, bwd);
    if (S.L == 8) return norm_go<T, P, V, 8, 1>(A, bwd, s);
    if (S.L == 32) return norm_go<T, P, V, 32, 1>(A, bwd, s);
    if (S.L == 64 && S.R == 1) return norm_go<T, P, V, 64, 1>(A, bwd, s);
    if (S.L == 64 && S.R == 2) return norm_go<T, P, V, 64, 2>(A, bwd, s);
    if (S.L == 64 && S.R == 4) return norm_go<T, P, V, 64, 4>(A, bwd, s);
    if (S.L == 256 && S.R == 2) return norm_go<T, P, V, 256, 2>(A, bwd, s);
    if (S.L == 256 && S.R == 4) return norm_go<T, P, V, 256, 4>(A, bwd, s);
    if (S.L == 1024 && S.R == 2) return norm_go<T, P, V, 1024, 2>(A, bwd, s);
    if constexpr (V <= 2)
        if (S.L == 1024) return norm_go<T, P, V, 1024, 4>(A, bwd, s);
    if (bwd) {
        const int64_t b = A.n < 32768 ? A.n : 32768;
        hipLaunchKernelGGL((k_norm_bwd_wide<T, P, V>), dim3((unsigned)b), dim3(kNormThreads), 0, s, A);
        if (A.part)
            hipLaunchKernelGGL((k_norm_cols<T, V>),
                               dim3((unsigned)((A.d / V + kNormThreads - 1) / kNormThreads), (unsigned)A.blocks),
                               dim3(kNormThreads), 0, s, A);
    } else {
        const int64_t b = A.n < 32768 ? A.n : 32768;
        hipLaunchKernelGGL((k_norm_fwd_wide<T, P, V>), dim3((unsigned)b), dim3(kNormThreads), 0, s, A);
    }
    return hipGetLastError();
}

// 16 bytes a lane where the rows allow it, else two elements, else one.
template <class T, class P>
hipError_t norm_type(NormArgs& A, bool bwd, hipStream_t s) {
    constexpr int E = (int)sizeof(T), V = 16 / E;
    auto fits = [&](int bytes) {
        bool ok = rows_vec(A.X, A.ldx, A.d, E, bytes);
        if (bwd)
            ok = ok && rows_vec(A.dY, A.lddy, A.d, E, bytes) && rows_vec(A.dX, A.d, A.d, E, bytes);
        else
            ok = ok && rows_vec(A.Y, A.d, A.d, E, bytes);
        const int pb = bytes / E * (int)sizeof(P) < 16 ? bytes / E * (int)sizeof(P) : 16;   // one parameter load
        return ok && ((uintptr_t)A.gamma | (uintptr_t)A.beta) % pb == 0;
    };
    const int v = fits(16) ? V : fits(2 * E) ? 2 : 1;
    A.blocks = bwd_blocks(A.n, A.d / v);
    if (v == V) return norm_vec<T, P, V>(A, bwd, s);
    return v == 2 ? norm_vec<T, P, 2>(A, bwd, s) : norm_vec<T, P, 1>(A, bwd, s);
}

hipError_t norm_any(NormArgs& A, bool bwd, int type, hipStream_t s) {
    if (type == kF32) return norm_type<float, float>(A, bwd, s);
    if (type == kBF16) return A.param_f32 ? norm_type<__bf16, float>(A, bwd, s) : norm_type<__bf16, __bf16>(A, bwd, s);
    return A.param_f32 ? norm_type<_Float16, float>(A, bwd, s) : norm_type<_Float16, _Float16>(A, bwd, s);
}

}  // namespace

int norm_bwd_max_blocks(int64_t n, int32_t d) { return bwd_blocks(n, d); }

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
    hipLaunchKernelGGL(k_norm_sums, dim3((unsigned)((A.d + 63) / 64), 2), dim3(1024), 0, s, A);
    return hipGetLastError();
}

}  // namespace km
