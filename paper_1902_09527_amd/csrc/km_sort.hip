// Rows sorted by cluster and back.
//
// The plan is a stable counting sort of the n m slots by cluster (empty slots
// last): up to kSortRankMax slots in one block, more in passes over digits of
// the cluster index (one pass for up to kSortBins - 1 clusters): a histogram
// per tile, its prefix sums over the tiles, and the scatter, which ranks the
// slots of a tile wave by wave in their order.  No result depends on the
// order in which blocks or lanes run.
//
// The row movers are one pass over the rows each, in slot order: a row is
// read once and written to the places of its slots (gather, gradient of
// combine), or its slots' rows are read and their weighted sum is written
// (combine, gradient of gather).  They are bound by the memory's rate.
#include "km_ops.h"

namespace km {

namespace {

__device__ __forceinline__ int key_of(int id, int k) { return (unsigned)id < (unsigned)k ? id : k; }

// Up to kSortRankMax slots: the place of slot p is the number of slots with a
// smaller (key, p), counted against keys in LDS.  (N / 64) N comparisons of a
// wave: 4 us at 1024 slots, one launch instead of three.
__global__ __launch_bounds__(kSortRankMax) void k_sort_rank(SortArgs A) {
    __shared__ __align__(16) int s_key[kSortRankMax];
    __shared__ int s_sorted[kSortRankMax];
    const int p = threadIdx.x, N = A.N, k = A.k;
    const int key = p < N ? key_of(A.ids[p], k) : INT_MAX;
    s_key[p] = key;
    __syncthreads();
    if (p < N) {
        int place = 0;
        const int N4 = (N + 3) & ~3;   // blockDim is a multiple of 64: the padding holds INT_MAX
#pragma unroll 4
        for (int q = 0; q < N4; q += 4) {
            const int4 o = *reinterpret_cast<const int4*>(s_key + q);
            place += (o.x < key || (o.x == key && q < p)) ? 1 : 0;
            place += (o.y < key || (o.y == key && q + 1 < p)) ? 1 : 0;
            place += (o.z < key || (o.z == key && q + 2 < p)) ? 1 : 0;
            place += (o.w < key || (o.w == key && q + 3 < p)) ? 1 : 0;
        }
        s_sorted[place] = key;
        A.order[place] = p;
        A.pos[p] = place;
        A.sorted_ids[place] = key < k ? key : -1;
    }
    __syncthreads();
    for (int64_t c = p; c <= k; c += blockDim.x) {   // offsets[c]: slots with a key below c
        int lo = 0, hi = N;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (s_sorted[mid] < c) lo = mid + 1; else hi = mid;
        }
        A.offsets[c] = lo;
    }
}

// One counting pass: the digit of an item is (key >> shift) & (2^bits - 1);
// with a single pass the key itself.  idx: the items' order so far (null: the
// slots' own).
struct Pass {
    const int32_t* idx;
    int32_t* out;          // order after this pass
    uint32_t* hist;        // tiles x bins: counts, then their prefix over the tiles
    uint32_t* tot;         // bins: totals
    int32_t bins, shift, mask, rounds, bits, last, single;
    int64_t tiles;
};

__device__ __forceinline__ int digit_of(const SortArgs& A, const Pass& P, int item) {
    return (key_of(A.ids[item], A.k) >> P.shift) & P.mask;
}

__global__ __launch_bounds__(kSortThreads) void k_sort_hist(SortArgs A, Pass P) {
    __shared__ uint32_t s_hist[kSortBins];
    for (int b = threadIdx.x; b < P.bins; b += kSortThreads) s_hist[b] = 0;
    __syncthreads();
    const int64_t t0 = (int64_t)blockIdx.x * kSortThreads * P.rounds;
    for (int r = 0; r < P.rounds; ++r) {
        const int64_t i = t0 + (int64_t)r * kSortThreads + threadIdx.x;
        if (i < A.N) atomicAdd(&s_hist[digit_of(A, P, P.idx ? P.idx[i] : (int)i)], 1u);   // counts: order is no matter
    }
    __syncthreads();
    uint32_t* h = P.hist + (int64_t)blockIdx.x * P.bins;
    for (int b = threadIdx.x; b < P.bins; b += kSortThreads) h[b] = s_hist[b];
}

// Prefix sums over the tiles, 64 digit values a block: 16 waves take a run of
// tiles each, lanes the digit values.
__global__ __launch_bounds__(1024) void k_sort_scan(Pass P) {
    __shared__ uint32_t s_sum[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int b = blockIdx.x * 64 + lane;
    const int64_t per = (P.tiles + 15) / 16, t0 = wave * per, t1 = t0 + per < P.tiles ? t0 + per : P.tiles;
    uint32_t sum = 0;
    if (b < P.bins) {
#pragma unroll 8
        for (int64_t t = t0; t < t1; ++t) sum += P.hist[t * P.bins + b];
    }
    s_sum[wave][lane] = sum;
    __syncthreads();
    uint32_t run = 0, all = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
        if (w == wave) run = all;
        all += s_sum[w][lane];
    }
    if (b >= P.bins) return;
    if (wave == 0) P.tot[b] = all;
#pragma unroll 4
    for (int64_t t = t0; t < t1; ++t) {
        const uint32_t v = P.hist[t * P.bins + b];
        P.hist[t * P.bins + b] = run;
        run += v;
    }
}

__global__ __launch_bounds__(kSortThreads) void k_sort_scatter(SortArgs A, Pass P) {
    extern __shared__ uint32_t s_place[];   // waves x bins: next place of each digit value, per wave
    __shared__ uint32_t s_wave[kSortWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, bins = P.bins;
    for (int b = tid; b < kSortWaves * bins; b += kSortThreads) s_place[b] = 0;
    __syncthreads();
    // A wave's items are consecutive, 64 a round.
    const int64_t w0 = ((int64_t)blockIdx.x * kSortWaves + wave) * 64 * P.rounds;
    uint32_t* mine = s_place + wave * bins;
    for (int r = 0; r < P.rounds; ++r) {
        const int64_t i = w0 + r * 64 + lane;
        if (i < A.N) atomicAdd(&mine[digit_of(A, P, P.idx ? P.idx[i] : (int)i)], 1u);
    }
    __syncthreads();
    // Exclusive sums of the totals over the digit values, 4 values a thread.
    constexpr int kPer = kSortBins / kSortThreads;
    uint32_t v[kPer], own = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int b = tid * kPer + j;
        v[j] = b < bins ? P.tot[b] : 0;
        own += v[j];
    }
    uint32_t inc = own;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t up = __shfl_up(inc, o);
        if (lane >= o) inc += up;
    }
    if (lane == 63) s_wave[wave] = inc;
    __syncthreads();
    uint32_t base = inc - own;
    for (int w = 0; w < wave; ++w) base += s_wave[w];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int b = tid * kPer + j;
        if (b < bins) {
            if (P.single && blockIdx.x == 0) A.offsets[b] = (int32_t)base;   // bins = k + 1: one pass only
            uint32_t at = base + P.hist[(int64_t)blockIdx.x * bins + b];
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) {
                const uint32_t c = s_place[w * bins + b];
                s_place[w * bins + b] = at;
                at += c;
            }
            base += v[j];
        }
    }
    __syncthreads();
    // Places: lanes of a round with the same digit value take consecutive
    // ones in lane order; the lowest of them moves the counter.
    for (int r = 0; r < P.rounds; ++r) {
        const int64_t i = w0 + r * 64 + lane;
        const bool in = i < A.N;
        const int item = in ? (P.idx ? P.idx[i] : (int)i) : 0;
        const int key = in ? key_of(A.ids[item], A.k) : 0;
        const int dg = in ? (key >> P.shift) & P.mask : 0;
        uint64_t same = __ballot(in);
        for (int b = 0; b < P.bits; ++b) {
            const bool bit = (dg >> b) & 1;
            const uint64_t set = __ballot(bit);
            same &= bit ? set : ~set;
        }
        const int lead = __ffsll((unsigned long long)same) - 1;
        uint32_t at = 0;
        if (in && lane == lead) at = atomicAdd(&mine[dg], (uint32_t)__popcll(same));
        at = __shfl(at, in ? lead : 0);
        if (in) {
            at += (uint32_t)__popcll(same & ((1ull << lane) - 1));
            P.out[at] = item;
            if (P.last) {
                A.pos[item] = (int32_t)at;
                A.sorted_ids[at] = key < A.k ? key : -1;
            }
        }
    }
}

// offsets after several passes: the first place whose key is not below c.
__global__ __launch_bounds__(256) void k_sort_offsets(SortArgs A) {
    for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c <= A.k; c += (int64_t)gridDim.x * 256) {
        int32_t lo = 0, hi = A.N;
        while (lo < hi) {
            const int32_t mid = lo + (hi - lo) / 2;
            if (key_of(A.sorted_ids[mid], A.k) < c) lo = mid + 1; else hi = mid;
        }
        A.offsets[c] = lo;
    }
}

}  // namespace

SortShape sort_shape(int64_t N, int32_t k) {
    SortShape S{};
    S.bytes = 256;
    if (N <= kSortRankMax) return S;
    int kbits = 1;
    while (kbits < 31 && ((int64_t)1 << kbits) <= k) ++kbits;   // keys are 0..k
    int most = 0;
    while ((1 << (most + 1)) <= kSortBins) ++most;
    S.passes = k < kSortBins ? 1 : (kbits + most - 1) / most;
    S.bits = (kbits + S.passes - 1) / S.passes;
    // Tiles of 2048 slots while they are few (more blocks), then longer ones
    // (the histograms stay small beside the slots).
    int64_t rounds = N / ((int64_t)kSortThreads * 512);
    S.rounds = (int)(rounds < 4 ? 4 : rounds > 64 ? 64 : rounds);
    const int64_t tile = (int64_t)kSortThreads * S.rounds;
    S.tiles = (N + tile - 1) / tile;
    const int64_t bins = S.passes == 1 ? (int64_t)k + 1 : (int64_t)1 << S.bits;
    auto up = [](size_t b) { return (b + 255) / 256 * 256; };
    S.off_hist = 0;
    S.off_tot = up((size_t)S.tiles * bins * 4);
    S.off_idx = S.off_tot + up((size_t)bins * 4);
    S.bytes = S.off_idx + (S.passes > 1 ? up((size_t)N * 4) : 0);
    return S;
}

hipError_t launch_sort_plan(const SortArgs& A, const SortShape& S, char* ws, hipStream_t s) {
    if (S.passes == 0) {
        const int threads = A.N < 1 ? 64 : (A.N + 63) / 64 * 64;
        hipLaunchKernelGGL(k_sort_rank, dim3(1), dim3(threads), 0, s, A);
        return hipGetLastError();
    }
    // Passes alternate between the workspace's order and A.order and end in A.order.
    int32_t* tmp = reinterpret_cast<int32_t*>(ws + S.off_idx);
    const int32_t* in = nullptr;
    for (int q = 0; q < S.passes; ++q) {
        Pass P{};
        P.idx = in;
        P.out = (S.passes - 1 - q) % 2 == 0 ? A.order : tmp;
        P.hist = reinterpret_cast<uint32_t*>(ws + S.off_hist);
        P.tot = reinterpret_cast<uint32_t*>(ws + S.off_tot);
        P.single = S.passes == 1;
        P.bins = P.single ? A.k + 1 : 1 << S.bits;
        P.shift = q * S.bits;
        P.mask = (1 << S.bits) - 1;
        P.bits = S.bits;
        P.rounds = S.rounds;
        P.tiles = S.tiles;
        P.last = q == S.passes - 1;
        hipLaunchKernelGGL(k_sort_hist, dim3((unsigned)S.tiles), dim3(kSortThreads), 0, s, A, P);
        hipLaunchKernelGGL(k_sort_scan, dim3((unsigned)((P.bins + 63) / 64)), dim3(1024), 0, s, P);
        hipLaunchKernelGGL(k_sort_scatter, dim3((unsigned)S.tiles), dim3(kSortThreads),
                           (size_t)kSortWaves * P.bins * 4, s, A, P);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        in = P.out;
    }
    if (S.passes > 1) {
        const int64_t b = ((int64_t)A.k + 256) / 256;
        hipLaunchKernelGGL(k_sort_offsets, dim3((unsigned)(b < 4096 ? b : 4096)), dim3(256), 0, s, A);
    }
    return hipGetLastError();
}

// --------------------------------------------------------------------------
// Row movers.  L lanes (a power of two up to 64) share a row, V elements a
// lane and step.

namespace {

constexpr int kMoveThreads = 256;

template <class T, int V, int L>
__global__ __launch_bounds__(kMoveThreads) void k_gather(MoveArgs A) {
    using W = Vec<T, V>;
    const int l = threadIdx.x % L, nv = A.d / V;
    const int32_t used = *A.used;
    const int64_t step = (int64_t)gridDim.x * (kMoveThreads / L);
    for (int64_t i = (int64_t)blockIdx.x * (kMoveThreads / L) + threadIdx.x / L; i < A.n; i += step) {
        const W* __restrict__ x = reinterpret_cast<const W*>(static_cast<const T*>(A.src) + i * A.ld);
        const int32_t* __restrict__ pos = A.pos + i * A.m;
        for (int c = l; c < nv; c += 4 * L) {
            W v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (c + u * L < nv) v[u] = x[c + u * L];
            for (int j = 0; j < A.m; ++j) {
                const int32_t p = pos[j];
                W* y = reinterpret_cast<W*>(static_cast<T*>(A.dst) + (int64_t)p * A.d);
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (c + u * L < nv) y[c + u * L] = p < used ? v[u] : W{};
            }
        }
    }
}

// Y[i] = sum_j w[i,j] Z[pos[i,j]] over the slots in use, in float32, j ascending.
template <class T, int V, int L>
__global__ __launch_bounds__(kMoveThreads) void k_combine(MoveArgs A) {
    using W = Vec<T, V>;
    const int l = threadIdx.x % L, nv = A.d / V;
    const int32_t used = *A.used;
    const int64_t step = (int64_t)gridDim.x * (kMoveThreads / L);
    for (int64_t i = (int64_t)blockIdx.x * (kMoveThreads / L) + threadIdx.x / L; i < A.n; i += step) {
        const int32_t* __restrict__ pos = A.pos + i * A.m;
        W* y = reinterpret_cast<W*>(static_cast<T*>(A.dst) + i * A.d);
        for (int c = l; c < nv; c += 4 * L) {
            float acc[4][V] = {};
            for (int j = 0; j < A.m; ++j) {
                const int32_t p = pos[j];
                if (p >= used) continue;
                const W* __restrict__ z = reinterpret_cast<const W*>(static_cast<const T*>(A.src) + (int64_t)p * A.ld);
                const float w = A.w ? A.w[i * A.m + j] : 1.0f;
                W v[4];
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (c + u * L < nv) v[u] = z[c + u * L];
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (c + u * L < nv)
#pragma unroll
                        for (int e = 0; e < V; ++e) acc[u][e] = fmaf(w, to_f32(v[u].e[e]), acc[u][e]);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (c + u * L < nv) {
                    W o;
#pragma unroll
                    for (int e = 0; e < V; ++e) o.e[e] = from_f32<T>(acc[u][e]);
                    y[c + u * L] = o;
                }
        }
    }
}

// dZ[pos] = w dY[i] (zero rows for empty slots), dw[i,j] = <dY[i], Z[pos]>.
template <class T, int V, int L>
__global__ __launch_bounds__(kMoveThreads) void k_combine_bwd(MoveArgs A) {
    using W = Vec<T, V>;
    const int l = threadIdx.x % L, nv = A.d / V;
    const int32_t used = *A.used;
    const int64_t step = (int64_t)gridDim.x * (kMoveThreads / L);
    for (int64_t i = (int64_t)blockIdx.x * (kMoveThreads / L) + threadIdx.x / L; i < A.n; i += step) {
        const W* __restrict__ g = reinterpret_cast<const W*>(static_cast<const T*>(A.src) + i * A.ld);
        for (int j = 0; j < A.m; ++j) {   // dY[i] comes from cache after the first slot
            const int64_t q = i * A.m + j;
            const int32_t p = A.pos[q];
            const bool in = p < used;
            const float w = A.w ? A.w[q] : 1.0f;
            const W* __restrict__ z = reinterpret_cast<const W*>(static_cast<const T*>(A.src2) + (int64_t)p * A.ld2);
            W* dz = reinterpret_cast<W*>(static_cast<T*>(A.dst) + (int64_t)p * A.d);
            float dot = 0.0f;
            for (int c = l; c < nv; c += 4 * L) {
                W a[4], b[4];
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (c + u * L < nv && in) {
                        a[u] = g[c + u * L];
                        if (A.dw) b[u] = z[c + u * L];
                    }
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (c + u * L < nv) {
                        W o{};
                        if (in)
#pragma unroll
                            for (int e = 0; e < V; ++e) {
                                const float x = to_f32(a[u].e[e]);
                                o.e[e] = from_f32<T>(w * x);
                                if (A.dw) dot = fmaf(x, to_f32(b[u].e[e]), dot);
                            }
                        dz[c + u * L] = o;
                    }
            }
            if (A.dw) {
                dot = group_sum<L>(dot);
                if (l == 0) A.dw[q] = dot;
            }
        }
    }
}

enum Mover { kGather, kCombine, kCombineBwd };

template <class T, int V, int L>
hipError_t move_go(const MoveArgs& A, Mover mv, hipStream_t s) {
    const int64_t per = kMoveThreads / L;
    int64_t blocks = (A.n + per - 1) / per;
    if (blocks > 65536) blocks = 65536;
    const dim3 g((unsigned)blocks), b(kMoveThreads);
    switch (mv) {
        case kGather: hipLaunchKernelGGL((k_gather<T, V, L>), g, b, 0, s, A); break;
        case kCombine: hipLaunchKernelGGL((k_combine<T, V, L>), g, b, 0, s, A); break;
        default: hipLaunchKernelGGL((k_combine_bwd<T, V, L>), g, b, 0, s, A); break;
    }
    return hipGetLastError();
}

template <class T, int V>
hipError_t move_lanes(const MoveArgs& A, Mover mv, hipStream_t s) {
    const int nv = A.d / V;
    if (nv <= 4) return move_go<T, V, 4>(A, mv, s);
    if (nv <= 16) return move_go<T, V, 16>(A, mv, s);
    return move_go<T, V, 64>(A, mv, s);
}

template <class T>
hipError_t move_type(const MoveArgs& A, Mover mv, hipStream_t s) {
    bool vec = rows_vec16(A.src, A.ld, A.d, sizeof(T)) && rows_vec16(A.dst, A.d, A.d, sizeof(T));
    if (A.src2) vec = vec && rows_vec16(A.src2, A.ld2, A.d, sizeof(T));
    if (vec) return move_lanes<T, 16 / (int)sizeof(T)>(A, mv, s);
    return move_lanes<T, 1>(A, mv, s);
}

hipError_t move_any(const MoveArgs& A, Mover mv, int type, hipStream_t s) {
    if (A.n == 0) return hipSuccess;
    if (type == kF32) return move_type<float>(A, mv, s);
    if (type == kBF16) return move_type<__bf16>(A, mv, s);
    return move_type<_Float16>(A, mv, s);
}

}  // namespace

hipError_t launch_sort_gather(const MoveArgs& A, int type, hipStream_t s) { return move_any(A, kGather, type, s); }
hipError_t launch_sort_combine(const MoveArgs& A, int type, hipStream_t s) { return move_any(A, kCombine, type, s); }
hipError_t launch_sort_combine_bwd(const MoveArgs& A, int type, hipStream_t s) {
    return move_any(A, kCombineBwd, type, s);
}

}  // namespace km
