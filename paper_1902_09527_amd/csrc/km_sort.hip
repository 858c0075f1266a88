// Rows sorted by cluster and back.
//
// The plan is a stable counting sort of the n m slots by cluster (empty slots
// last): up to kSortRankMax slots by comparing, more in passes over digits of
// the cluster index (one pass for up to kSortBins - 1 clusters): a histogram
// per tile, its prefix sums over the tiles, and the scatter, which ranks the
// slots of a tile wave by wave in their order.  No result depends on the
// order in which blocks or lanes run.
//
// Measured: 32 slots 4.0 us; 1M slots of 100 clusters 26 us (histogram 4,
// prefixes 6.6, scatter 15), 2M of 1000 56 us (8, 8.5, 39); bound by launches
// and latency, and by the scatter's pieces of lines.
//
// The row movers are one pass over the rows each, in slot order: a row is
// read once and written to the places of its slots (gather, gradient of
// combine), or its slots' rows are read and their weighted sum is written
// (combine, gradient of gather).  They are bound by the memory's rate: 2M x
// 256 float32 rows 773 us out and 778 us back (5.3 TB/s of rows read and
// written; a large copy reaches 4.8), 16,382 x 2048 bf16 rows 31 us for the
// gradients of combine (5.4 TB/s).
#include <type_traits>

#include "km_ops.h"

namespace km {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Clusters up to which the ranking counts the offsets too.
constexpr int kSortRankOffsets = 1 << 13;

__device__ __forceinline__ int key_of(int id, int k) { return (unsigned)id < (unsigned)k ? id : k; }

// Up to kSortRankMax slots: the place of slot p is the number of slots with a
// smaller (key, p), and offsets[c] the number with a key below c, so both are
// one kind of item: 64 of them a block, one a lane, whose waves share the slots
// in chunks of 64 (broadcast from LDS, a wave's own part).  All slots of a chunk
// come before an item of equal key, or all after it, but for the item's own
// chunk: one comparison a slot.  (N + k) N / 64 comparisons of a wave over the
// chip, one launch instead of three: 4.0 us at 1 to 64 slots, 5.0 at 1024, 8.6
// at 4096 and 13.4 at 8192, where the three of a counting pass take 10 to 13 us
// (and 5 more of the host) at any of these; two passes (more than 4095 clusters)
// 25 us.
__global__ __launch_bounds__(1024) void k_sort_rank(SortArgs A, int slot_blocks) {
    __shared__ __align__(16) int s_key[16][64];
    __shared__ int s_count[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int N = A.N, k = A.k, own = blockIdx.x;
    const bool slots = own < slot_blocks;
    const int64_t p = slots ? (int64_t)own * 64 + lane : (int64_t)(own - slot_blocks) * 64 + lane;   // slot or cluster
    int key = INT_MAX;
    if (!slots) key = p <= k ? (int)p : k;
    else if (p < N) key = key_of(A.ids[p], k);
    const int chunks = (N + 63) / 64;
    int count = 0;
    auto load = [&](int c) { return c < chunks && c * 64 + lane < N ? key_of(A.ids[c * 64 + lane], k) : INT_MAX; };
    int next = load(wave);
    for (int c = wave; c < chunks; c += waves) {
        __builtin_amdgcn_wave_barrier();   // a wave's own: its reads of the last chunk come first
        s_key[wave][lane] = next;
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        next = load(c + waves);
        const int4* o4 = reinterpret_cast<const int4*>(s_key[wave]);
        if (slots && c == own) {
#pragma unroll 4
            for (int q = 0; q < 16; ++q) {
                const int4 o = o4[q];
                count += o.x < key || (o.x == key && q * 4 < lane);
                count += o.y < key || (o.y == key && q * 4 + 1 < lane);
                count += o.z < key || (o.z == key && q * 4 + 2 < lane);
                count += o.w < key || (o.w == key && q * 4 + 3 < lane);
            }
        } else {
            const int below = key + (slots && c < own && key < INT_MAX ? 1 : 0);   // k + 1 at most
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                const int4 o = o4[q];
                count += o.x < below;
                count += o.y < below;
                count += o.z < below;
                count += o.w < below;
            }
        }
    }
    s_count[wave][lane] = count;
    __syncthreads();
    if (wave != 0) return;
    for (int w = 1; w < waves; ++w) count += s_count[w][lane];
    if (!slots) {
        if (p <= k) A.offsets[p] = count;
    } else if (p < N) {
        A.order[count] = (int)p;
        A.pos[p] = count;
        A.sorted_ids[count] = key < k ? key : -1;
    }
}

// One counting pass: the digit of an item is (key >> shift) & (2^bits - 1);
// with a single pass the key itself.  idx: the items' order so far (null: the
// slots' own).  A tile is kSortThreads RO items, a wave's items consecutive
// (64 RO of them), RO a lane; all of a lane's keys are loaded at once.
struct Pass {
    const int32_t* idx;
    int32_t* out;          // order after this pass
    uint32_t* hist;        // tiles x bins: counts, then their prefix over the tiles
    uint32_t* tot;         // bins: totals
    int32_t bins, shift, mask, bits, last, single;
    int64_t tiles;
};

// The items of a lane and their keys (item -1: past the end).
template <int RO>
__device__ __forceinline__ void load_items(const SortArgs& A, const Pass& P, int64_t tile, int32_t* item,
                                           int32_t* key) {
    const int64_t w0 = (tile * kSortWaves + (threadIdx.x >> 6)) * 64 * RO + (threadIdx.x & 63);
#pragma unroll
    for (int r = 0; r < RO; ++r) {
        const int64_t i = w0 + r * 64;
        item[r] = i < A.N ? (P.idx ? P.idx[i] : (int32_t)i) : -1;
    }
#pragma unroll
    for (int r = 0; r < RO; ++r) key[r] = item[r] >= 0 ? key_of(A.ids[item[r]], A.k) : 0;
}

template <int RO>
__global__ __launch_bounds__(kSortThreads) void k_sort_hist(SortArgs A, Pass P) {
    __shared__ uint32_t s_hist[kSortBins];
    int32_t item[RO], key[RO];
    load_items<RO>(A, P, blockIdx.x, item, key);
    for (int b = threadIdx.x; b < P.bins; b += kSortThreads) s_hist[b] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < RO; ++r)
        if (item[r] >= 0) atomicAdd(&s_hist[(key[r] >> P.shift) & P.mask], 1u);   // counts: order is no matter
    __syncthreads();
    uint32_t* h = P.hist + (int64_t)blockIdx.x * P.bins;
    for (int b = threadIdx.x; b < P.bins; b += kSortThreads) h[b] = s_hist[b];
}

// Prefix sums over the tiles, 16 digit values a block: its 64 groups of 16
// lanes take a run of tiles each.
__global__ __launch_bounds__(1024) void k_sort_scan(Pass P) {
    __shared__ uint32_t s_sum[64][16];
    const int lane = threadIdx.x & 15, seg = threadIdx.x >> 4;
    const int b = blockIdx.x * 16 + lane;
    const int64_t per = (P.tiles + 63) / 64, t0 = seg * per, t1 = t0 + per < P.tiles ? t0 + per : P.tiles;
    uint32_t sum = 0;
    if (b < P.bins) {
#pragma unroll 8
        for (int64_t t = t0; t < t1; ++t) sum += P.hist[t * P.bins + b];
    }
    s_sum[seg][lane] = sum;
    __syncthreads();
    if (b >= P.bins) return;
    uint32_t run = 0, all = 0;
#pragma unroll 16
    for (int w = 0; w < 64; ++w) {
        if (w == seg) run = all;
        all += s_sum[w][lane];
    }
    if (seg == 0) P.tot[b] = all;
#pragma unroll 8
    for (int64_t t = t0; t < t1; ++t) {
        const uint32_t v = P.hist[t * P.bins + b];
        P.hist[t * P.bins + b] = run;
        run += v;
    }
}

// A tile writes a few places of every cluster, next to those of the tiles
// beside it.  Blocks are dealt over 8 XCDs with an L2 each, so an XCD takes
// consecutive tiles: their pieces of a line meet in one L2 instead of going to
// memory one by one (2M slots, 1000 clusters: 50 us without, the pieces of 16
// bytes written as whole lines).
template <int RO>
__global__ __launch_bounds__(kSortThreads) void k_sort_scatter(SortArgs A, Pass P) {
    extern __shared__ uint32_t s_place[];   // waves x bins: next place of each digit value, per wave
    __shared__ uint32_t s_wave[kSortWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, bins = P.bins;
    const int64_t share = (P.tiles + 7) / 8, tile = blockIdx.x % 8 * share + blockIdx.x / 8;
    if (tile >= P.tiles) return;   // the grid is 8 share blocks
    // The tile's prefixes and the totals, kPer values a thread.
    constexpr int kPer = kSortBins / kSortThreads;
    uint32_t v[kPer], before[kPer], own = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int b = tid * kPer + j;
        v[j] = b < bins ? P.tot[b] : 0;
        before[j] = b < bins ? P.hist[tile * bins + b] : 0;
        own += v[j];
    }
    int32_t item[RO], key[RO];
    load_items<RO>(A, P, tile, item, key);
    for (int b = tid; b < kSortWaves * bins; b += kSortThreads) s_place[b] = 0;
    __syncthreads();
    uint32_t* mine = s_place + wave * bins;
#pragma unroll
    for (int r = 0; r < RO; ++r)
        if (item[r] >= 0) atomicAdd(&mine[(key[r] >> P.shift) & P.mask], 1u);
    // Exclusive sums of the totals over the digit values.
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
            if (P.single && tile == 0) A.offsets[b] = (int32_t)base;   // bins = k + 1: one pass only
            uint32_t at = base + before[j];
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
#pragma unroll
    for (int r = 0; r < RO; ++r) {
        const bool in = item[r] >= 0;
        const int dg = (key[r] >> P.shift) & P.mask;
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
            P.out[at] = item[r];
            if (P.last) {
                A.pos[item[r]] = (int32_t)at;
                A.sorted_ids[at] = key[r] < A.k ? key[r] : -1;
            }
        }
    }
}

// offsets after several passes, or of very many clusters: the first place
// whose key is not below c.
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

hipError_t sort_offsets(const SortArgs& A, hipStream_t s) {
    const int64_t b = ((int64_t)A.k + 256) / 256;
    hipLaunchKernelGGL(k_sort_offsets, dim3((unsigned)(b < 4096 ? b : 4096)), dim3(256), 0, s, A);
    return hipGetLastError();
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
    // Short tiles while they are few (more blocks), then longer ones (the
    // histograms stay small beside the slots).
    S.rounds = N <= (1 << 18) ? 2 : N <= (1 << 20) ? 4 : N <= (1 << 22) ? 8 : 16;
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
        const bool apart = A.k > kSortRankOffsets;   // offsets by search, over the chip
        const int chunks = (A.N + 63) / 64, waves = chunks < 1 ? 1 : chunks < 16 ? chunks : 16;
        const int blocks = chunks + (apart ? 0 : A.k / 64 + 1);
        if (blocks > 0) hipLaunchKernelGGL(k_sort_rank, dim3(blocks), dim3(64 * waves), 0, s, A, chunks);
        hipError_t e = hipGetLastError();
        return e == hipSuccess && apart ? sort_offsets(A, s) : e;
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
        P.tiles = S.tiles;
        P.last = q == S.passes - 1;
        const dim3 g((unsigned)S.tiles), g8((unsigned)((S.tiles + 7) / 8 * 8)), t(kSortThreads);
        const size_t lds = (size_t)kSortWaves * P.bins * 4;
        if (lds > 60 * 1024) {   // beyond what a kernel has without asking
            hipError_t e = hipSuccess;
            auto raise = [&](auto* kernel) {
                e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                                        kSortWaves * kSortBins * 4);
            };
            if (S.rounds == 2) raise(k_sort_scatter<2>);
            else if (S.rounds == 4) raise(k_sort_scatter<4>);
            else if (S.rounds == 8) raise(k_sort_scatter<8>);
            else raise(k_sort_scatter<16>);
            if (e != hipSuccess) return e;
        }
#define KM_SORT(K, G, LDS)                                                                 \
    do {                                                                                 \
        if (S.rounds == 2) hipLaunchKernelGGL((K<2>), G, t, LDS, s, A, P);               \
        else if (S.rounds == 4) hipLaunchKernelGGL((K<4>), G, t, LDS, s, A, P);          \
        else if (S.rounds == 8) hipLaunchKernelGGL((K<8>), G, t, LDS, s, A, P);          \
        else hipLaunchKernelGGL((K<16>), G, t, LDS, s, A, P);                            \
    } while (0)
        KM_SORT(k_sort_hist, g, 0);
        hipLaunchKernelGGL(k_sort_scan, dim3((unsigned)((P.bins + 15) / 16)), dim3(1024), 0, s, P);
        KM_SORT(k_sort_scatter, g8, lds);
#undef KM_SORT
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        in = P.out;
    }
    return S.passes > 1 ? sort_offsets(A, s) : hipSuccess;
}

// --------------------------------------------------------------------------
// Row movers.  L lanes (a power of two up to 64) share a row, V elements a
// lane and step.

namespace {

constexpr int kMoveThreads = 256;

// Rows of up to L vectors (CU = 1) go four at a time, wider ones in four
// vectors a lane (CU = 4), so that four loads of a lane are in flight.
template <class R, int L, int CU>
__global__ __launch_bounds__(kMoveThreads) void k_gather(MoveArgs A, int nv, int64_t ld) {
    constexpr int RU = 4 / CU;
    const int l = threadIdx.x % L;
    const int32_t used = *A.used;
    const R* __restrict__ src = static_cast<const R*>(A.src);
    R* dst = static_cast<R*>(A.dst);
    const int64_t step = (int64_t)gridDim.x * (kMoveThreads / L) * RU;
    for (int64_t i0 = ((int64_t)blockIdx.x * (kMoveThreads / L) + threadIdx.x / L) * RU; i0 < A.n; i0 += step) {
        for (int c = l; c < nv; c += CU * L) {
            R v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int64_t i = i0 + u / CU;
                const int cc = c + u % CU * L;
                if (i < A.n && cc < nv) v[u] = src[i * ld + cc];
            }
            for (int j = 0; j < A.m; ++j) {
                int32_t p[RU];
#pragma unroll
                for (int r = 0; r < RU; ++r) p[r] = i0 + r < A.n ? A.pos[(i0 + r) * A.m + j] : 0;
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int cc = c + u % CU * L;
                    if (i0 + u / CU < A.n && cc < nv)
                        dst[(int64_t)p[u / CU] * nv + cc] = p[u / CU] < used ? v[u] : R{};
                }
            }
        }
    }
}

// Y[i] = sum_j w[i,j] Z[pos[i,j]] over the slots in use, in float32, j ascending.
template <class T, int V, int L, int CU>
__global__ __launch_bounds__(kMoveThreads) void k_combine(MoveArgs A) {
    using W = Vec<T, V>;
    constexpr int RU = 4 / CU;
    const int l = threadIdx.x % L, nv = A.d / V;
    const int32_t used = *A.used;
    const int64_t step = (int64_t)gridDim.x * (kMoveThreads / L) * RU;
    for (int64_t i0 = ((int64_t)blockIdx.x * (kMoveThreads / L) + threadIdx.x / L) * RU; i0 < A.n; i0 += step) {
        for (int c = l; c < nv; c += CU * L) {
            float acc[4][V] = {};
            for (int j = 0; j < A.m; ++j) {
                int32_t p[RU];
                float w[RU];
#pragma unroll
                for (int r = 0; r < RU; ++r) {
                    const bool in = i0 + r < A.n;
                    p[r] = in ? A.pos[(i0 + r) * A.m + j] : used;
                    w[r] = in && A.w ? A.w[(i0 + r) * A.m + j] : 1.0f;
                }
                W v[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int cc = c + u % CU * L;
                    if (p[u / CU] < used && cc < nv)
                        v[u] = reinterpret_cast<const W*>(static_cast<const T*>(A.src) + (int64_t)p[u / CU] * A.ld)[cc];
                }
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (p[u / CU] < used && c + u % CU * L < nv)
#pragma unroll
                        for (int e = 0; e < V; ++e) acc[u][e] = fmaf(w[u / CU], to_f32(v[u].e[e]), acc[u][e]);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int cc = c + u % CU * L;
                if (i0 + u / CU < A.n && cc < nv) {
                    W o;
#pragma unroll
                    for (int e = 0; e < V; ++e) o.e[e] = from_f32<T>(acc[u][e]);
                    reinterpret_cast<W*>(static_cast<T*>(A.dst) + (i0 + u / CU) * A.d)[cc] = o;
                }
            }
        }
    }
}

// dZ[pos] = w dY[i] (zero rows for empty slots), dw[i,j] = <dY[i], Z[pos]>.
// A group of lanes takes one slot's row at a time, RU slots with CU = 1.
template <class T, int V, int L, int CU>
__global__ __launch_bounds__(kMoveThreads) void k_combine_bwd(MoveArgs A) {
    using W = Vec<T, V>;
    constexpr int RU = 4 / CU;
    const int l = threadIdx.x % L, nv = A.d / V;
    const int32_t used = *A.used;
    const int64_t slots = A.n * A.m, step = (int64_t)gridDim.x * (kMoveThreads / L) * RU;
    for (int64_t q0 = ((int64_t)blockIdx.x * (kMoveThreads / L) + threadIdx.x / L) * RU; q0 < slots; q0 += step) {
        int32_t p[RU];
        int64_t i[RU];
        float w[RU], dot[RU];
#pragma unroll
        for (int r = 0; r < RU; ++r) {
            const bool in = q0 + r < slots;
            p[r] = in ? A.pos[q0 + r] : 0;
            w[r] = in && A.w ? A.w[q0 + r] : 1.0f;
            i[r] = A.m == 1 ? q0 + r : (q0 + r) / A.m;
            dot[r] = 0.0f;
        }
        for (int c = l; c < nv; c += CU * L) {
            W a[4], b[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int r = u / CU, cc = c + u % CU * L;
                if (q0 + r < slots && cc < nv && p[r] < used) {
                    a[u] = reinterpret_cast<const W*>(static_cast<const T*>(A.src) + i[r] * A.ld)[cc];
                    if (A.dw)
                        b[u] = reinterpret_cast<const W*>(static_cast<const T*>(A.src2) + (int64_t)p[r] * A.ld2)[cc];
                }
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int r = u / CU, cc = c + u % CU * L;
                if (q0 + r < slots && cc < nv) {
                    W* dz = reinterpret_cast<W*>(static_cast<T*>(A.dst) + (int64_t)p[r] * A.d) + cc;
                    if (p[r] < used) {
                        W o;
#pragma unroll
                        for (int e = 0; e < V; ++e) {
                            const float x = to_f32(a[u].e[e]);
                            o.e[e] = from_f32<T>(w[r] * x);
                            if (A.dw) dot[r] = fmaf(x, to_f32(b[u].e[e]), dot[r]);
                        }
                        *dz = o;
                    } else {
                        *dz = W{};
                    }
                }
            }
        }
        if (A.dw) {
#pragma unroll
            for (int r = 0; r < RU; ++r) {
                const float sum = group_sum<L>(dot[r]);
                if (l == 0 && q0 + r < slots) A.dw[q0 + r] = sum;
            }
        }
    }
}

dim3 move_grid(int64_t rows, int per) {
    const int64_t blocks = (rows + per - 1) / per;
    return dim3((unsigned)(blocks > 65536 ? 65536 : blocks));
}

// Lanes a row: the fewest that take it in one vector each, 64 for wider rows.
template <class F>
hipError_t by_lanes(int nv, F&& go) {
    using std::integral_constant;
    if (nv <= 4) go(integral_constant<int, 4>{}, integral_constant<int, 1>{});
    else if (nv <= 8) go(integral_constant<int, 8>{}, integral_constant<int, 1>{});
    else if (nv <= 16) go(integral_constant<int, 16>{}, integral_constant<int, 1>{});
    else if (nv <= 32) go(integral_constant<int, 32>{}, integral_constant<int, 1>{});
    else if (nv <= 64) go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    else go(integral_constant<int, 64>{}, integral_constant<int, 4>{});
    return hipGetLastError();
}

// gather moves words of 16, 4 or 2 bytes, whatever they hold.
template <class R>
hipError_t gather_words(const MoveArgs& A, size_t es, hipStream_t s) {
    const int nv = (int)(A.d * es / sizeof(R));
    const int64_t ld = A.ld * (int64_t)es / (int64_t)sizeof(R);
    return by_lanes(nv, [&](auto l, auto cu) {
        constexpr int L = decltype(l)::value, CU = decltype(cu)::value;
        hipLaunchKernelGGL((k_gather<R, L, CU>), move_grid(A.n, kMoveThreads / L * (4 / CU)), dim3(kMoveThreads), 0, s,
                           A, nv, ld);
    });
}

template <class T, int V, bool BWD>
hipError_t combine_lanes(const MoveArgs& A, hipStream_t s) {
    return by_lanes(A.d / V, [&](auto l, auto cu) {
        constexpr int L = decltype(l)::value, CU = decltype(cu)::value, per = kMoveThreads / L * (4 / CU);
        if constexpr (BWD)
            hipLaunchKernelGGL((k_combine_bwd<T, V, L, CU>), move_grid(A.n * A.m, per), dim3(kMoveThreads), 0, s, A);
        else
            hipLaunchKernelGGL((k_combine<T, V, L, CU>), move_grid(A.n, per), dim3(kMoveThreads), 0, s, A);
    });
}

// 16 bytes a lane where the rows allow it, else two elements, else one.
template <class T, bool BWD>
hipError_t combine_type(const MoveArgs& A, hipStream_t s) {
    constexpr int E = (int)sizeof(T);
    auto fits = [&](int bytes) {
        return rows_vec(A.src, A.ld, A.d, E, bytes) && rows_vec(A.dst, A.d, A.d, E, bytes) &&
               (!A.src2 || rows_vec(A.src2, A.ld2, A.d, E, bytes));
    };
    if (fits(16)) return combine_lanes<T, 16 / E, BWD>(A, s);
    if (fits(2 * E)) return combine_lanes<T, 2, BWD>(A, s);
    return combine_lanes<T, 1, BWD>(A, s);
}

template <bool BWD>
hipError_t combine_any(const MoveArgs& A, int type, hipStream_t s) {
    if (A.n == 0) return hipSuccess;
    if (type == kF32) return combine_type<float, BWD>(A, s);
    if (type == kBF16) return combine_type<__bf16, BWD>(A, s);
    return combine_type<_Float16, BWD>(A, s);
}

}  // namespace

hipError_t launch_sort_gather(const MoveArgs& A, int type, hipStream_t s) {
    if (A.n == 0) return hipSuccess;
    const size_t es = row_type_bytes(type);
    auto fits = [&](int bytes) {
        return rows_vec(A.src, A.ld, A.d, es, bytes) && rows_vec(A.dst, A.d, A.d, es, bytes);
    };
    if (fits(16)) return gather_words<u32x4>(A, es, s);
    if (fits(4)) return gather_words<uint32_t>(A, es, s);
    return gather_words<uint16_t>(A, es, s);
}
hipError_t launch_sort_combine(const MoveArgs& A, int type, hipStream_t s) { return combine_any<false>(A, type, s); }
hipError_t launch_sort_combine_bwd(const MoveArgs& A, int type, hipStream_t s) {
    return combine_any<true>(A, type, s);
}

}  // namespace km
