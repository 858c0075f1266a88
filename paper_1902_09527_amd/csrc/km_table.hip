// Rows of a table by their ids, scaled, and the table's gradient:
//   y_i = s T[id_i],  dT[c] = s sum over the slots of id c of dy.
//
// The gradient goes by the sorted plan, so that no sum depends on the order of
// atomics.  The places are cut into chunks of kTableChunk, whatever their ids, and
// the lanes of a row sum a chunk's rows in order, writing an id's sum where its
// places end.  An id that began before a chunk or goes on behind it leaves a float32
// part there (a chunk has two places for them), and a second kernel adds the parts
// of such ids in order.  So every lane's chain of loads that wait for one another is
// the same few, be the ids even or one of them everything.
//
// Bound by the memory's rate: 16 bytes a lane, rows at any address.  Gradient of
// 16,384 rows of 1024 bf16 for 50,000 ids: 22 us (6.2 TB/s, most of it zeros) and 9 of
// the join; of 1M rows of 32 float32 for 100 ids: 23 and 6 us.
#include "km_tile.h"

namespace km {

namespace {

constexpr int64_t kStreamBytes = 32 << 20;   // results of more go past the caches

// A lane's 16 bytes of a row of d elements.
template <class T>
using Part = Vec<T, 16 / (int)sizeof(T)>;

template <bool STREAM, class T, int E>
__device__ __forceinline__ void part_put(T* row, int64_t c, int64_t d, const float (&v)[E]) {
    Vec<T, E> o;
#pragma unroll
    for (int e = 0; e < E; ++e) o.e[e] = from_f32<T>(v[e]);
    if (c + E <= d) {
        if constexpr (STREAM && sizeof(o) == 16) {
            typedef u32x4 __attribute__((aligned(2))) any4;
            __builtin_nontemporal_store(__builtin_bit_cast(u32x4, o), reinterpret_cast<any4*>(row + c));
        } else {
            __builtin_memcpy(row + c, &o, sizeof(o));
        }
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (c + e < d) row[c + e] = o.e[e];
    }
}

// A row is taken by 2^A.lanes lanes, 16 bytes each, in A.slices slices: unit u is
// slice u % slices of row u / slices.  Divisions by a row's width would cost more than
// the row (50,000 rows of 1024 bf16 written: 46 us with them, 30 without).
struct Unit {
    int64_t row, col;
};
template <int E>
__device__ __forceinline__ Unit unit_at(const TableArgs& A, int64_t u) {
    int64_t row = u, slice = 0;
    if (A.slices > 1) {
        row = u / A.slices;
        slice = u - row * A.slices;
    }
    return Unit{row, ((slice << A.lanes) + (threadIdx.x & ((1 << A.lanes) - 1))) * E};
}

template <class T, bool STREAM>
__global__ __launch_bounds__(256) void k_table_fwd(TableArgs A) {
    constexpr int E = 16 / (int)sizeof(T), UN = 4;
    const int64_t total = A.n * A.slices, step = (int64_t)gridDim.x << (8 - A.lanes);
    for (int64_t u0 = ((int64_t)blockIdx.x << (8 - A.lanes)) + (threadIdx.x >> A.lanes); u0 < total; u0 += UN * step) {
        Unit u[UN];
        int id[UN];
        u32x4 v[UN];
#pragma unroll
        for (int y = 0; y < UN; ++y) {
            u[y] = unit_at<E>(A, u0 + y * step < total ? u0 + y * step : u0);
            id[y] = A.ids[u[y].row];
        }
#pragma unroll
        for (int y = 0; y < UN; ++y)
            if (u[y].col < A.d)
                v[y] = chunk_any(static_cast<const T*>(A.table) + ((unsigned)id[y] < (unsigned)A.k ? id[y] : 0) * A.ld,
                                 u[y].col, A.d);
#pragma unroll
        for (int y = 0; y < UN; ++y) {
            if (u0 + y * step >= total) break;
            if (u[y].col >= A.d) continue;
            float o[E];
            const bool in = (unsigned)id[y] < (unsigned)A.k;
            const Part<T> x = __builtin_bit_cast(Part<T>, v[y]);
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = in ? to_f32(x.e[e]) * A.scale : 0.0f;
            part_put<STREAM>(static_cast<T*>(A.out) + u[y].row * A.d, u[y].col, A.d, o);
        }
    }
}

// --------------------------------------------------------------------------

// Rows of ids without slots: zeros.
template <class T>
__device__ __forceinline__ void no_slots(const TableArgs& A, int64_t block, int64_t blocks) {
    constexpr int E = 16 / (int)sizeof(T), UN = 4;
    const int64_t total = (int64_t)A.k * A.slices, step = blocks << (8 - A.lanes);
    for (int64_t at = (block << (8 - A.lanes)) + (threadIdx.x >> A.lanes); at < total; at += UN * step) {
        Unit u[UN];
        bool none[UN];
#pragma unroll
        for (int y = 0; y < UN; ++y) {
            u[y] = unit_at<E>(A, at + y * step < total ? at + y * step : at);
            none[y] = A.offsets[u[y].row] == A.offsets[u[y].row + 1];
        }
        const float zero[E] = {};
#pragma unroll
        for (int y = 0; y < UN; ++y)
            if (none[y] && u[y].col < A.d) part_put<true>(static_cast<T*>(A.out) + u[y].row * A.d, u[y].col, A.d, zero);
    }
}

// Unit `at`: a chunk's slice.
template <class T>
__device__ __forceinline__ void chunk_sums(const TableArgs& A, int64_t at) {
    constexpr int E = 16 / (int)sizeof(T), UN = 4;
    const int64_t used = A.offsets[A.k];
    const Unit u = unit_at<E>(A, at);
    const int64_t p0 = u.row * kTableChunk;
    if (p0 >= used || u.col >= A.d) return;
    const int64_t p1 = p0 + kTableChunk < used ? p0 + kTableChunk : used;
    const int before = p0 > 0 ? A.sids[p0 - 1] : -1, behind = p1 < used ? A.sids[p1] : -1;
    int32_t id[UN], row[UN];
    auto ask = [&](int64_t p) {
#pragma unroll
        for (int q = 0; q < UN; ++q) {
            const int64_t x = p + q < p1 ? p + q : p1 - 1;
            id[q] = A.sids[x];
            row[q] = A.order[x];
        }
    };
    int c = before;         // the id that is summed
    bool began = false;     // in this chunk
    float sum[E] = {};
    auto done = [&](bool ended) {
        if (began && ended) {
            float o[E];
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = sum[e] * A.scale;
            part_put<true>(static_cast<T*>(A.out) + (int64_t)c * A.d, u.col, A.d, o);
        } else {
            part_put<false>(A.part + (2 * u.row + began) * A.d, u.col, A.d, sum);
        }
    };
    ask(p0);
    bool some = false;   // places of c in this chunk
    for (int64_t p = p0; p < p1; p += UN) {
        u32x4 w[UN];
        int32_t is[UN];
#pragma unroll
        for (int q = 0; q < UN; ++q) {
            w[q] = chunk_any(static_cast<const T*>(A.dY) + (int64_t)row[q] * A.ld, u.col, A.d);
            is[q] = id[q];
        }
        if (p + UN < p1) ask(p + UN);
#pragma unroll
        for (int q = 0; q < UN; ++q) {
            if (p + q >= p1) break;
            if (is[q] != c) {
                if (some) done(true);
                c = is[q];
                began = true;
#pragma unroll
                for (int e = 0; e < E; ++e) sum[e] = 0.0f;
            }
            some = true;
            const Part<T> x = __builtin_bit_cast(Part<T>, w[q]);
#pragma unroll
            for (int e = 0; e < E; ++e) sum[e] += to_f32(x.e[e]);
        }
    }
    done(behind != c);
}

template <class T>
__global__ __launch_bounds__(256) void k_table_bwd(TableArgs A) {
    if (blockIdx.x < A.chunk_blocks)
        chunk_sums<T>(A, ((int64_t)blockIdx.x << (8 - A.lanes)) + (threadIdx.x >> A.lanes));
    else
        no_slots<T>(A, blockIdx.x - A.chunk_blocks, gridDim.x - A.chunk_blocks);
}

// Ids whose places lie in several chunks: the sum of their parts in order, L lanes a
// column each taking every L-th.  A block tests A.tests ids, or chunks that an id
// begins in and goes on behind (by_chunk), a thread each, and adds those it finds.
template <class T, int L>
__global__ __launch_bounds__(256) void k_table_join(TableArgs A) {
    constexpr int kCols = 256 / L;
    __shared__ float s_sum[L][kCols + 1];
    __shared__ int s_found[257];
    if (threadIdx.x == 0) s_found[0] = 0;
    __syncthreads();
    const int64_t i = (int64_t)blockIdx.x * A.tests + threadIdx.x;
    if ((int)threadIdx.x < A.tests) {
        int c = -1;
        if (!A.by_chunk) {
            if (i < A.k) c = (int)i;
        } else {
            const int64_t p1 = (i + 1) * kTableChunk;
            if (p1 < A.offsets[A.k]) {
                c = A.sids[p1];
                if (A.sids[p1 - 1] != c || A.offsets[c] / kTableChunk != i) c = -1;
            }
        }
        if (c >= 0) {
            const int first = A.offsets[c], last = A.offsets[c + 1];
            if (last > first && first / kTableChunk != (last - 1) / kTableChunk) s_found[1 + atomicAdd(s_found, 1)] = c;
        }
    }
    __syncthreads();
    // This block's columns.
    const int width = (int)((A.d + gridDim.y - 1) / gridDim.y), lo = (int)blockIdx.y * width;
    const int hi = lo + width < A.d ? lo + width : A.d;
    const int found = s_found[0], cols = hi > lo ? hi - lo : 0;
    // The ids of few parts: a lane a column of one.  In whatever order: each has a sum of
    // its own.
    constexpr int kFewParts = 8;
    for (int x = threadIdx.x; x < found * cols; x += 256) {
        const int c = s_found[1 + x / cols], col = lo + x % cols, first = A.offsets[c], last = A.offsets[c + 1];
        const int64_t b = first / kTableChunk;
        const int more = (int)((last - 1) / kTableChunk - b);   // chunks after the first
        if (more > kFewParts) continue;
        float sum = A.part[(2 * b + 1) * A.d + col];
        for (int q = 1; q <= more; ++q) sum += A.part[2 * (b + q) * A.d + col];
        static_cast<T*>(A.out)[(int64_t)c * A.d + col] = from_f32<T>(sum * A.scale);
    }
    const int l = threadIdx.x % kCols, y = threadIdx.x / kCols;
    for (int f = 0; f < found; ++f) {
        const int c = s_found[1 + f], first = A.offsets[c], last = A.offsets[c + 1];
        const int64_t b = first / kTableChunk, more = (last - 1) / kTableChunk - b;
        if (more <= kFewParts) continue;
        for (int col0 = lo; col0 < hi; col0 += kCols) {
            const int col = col0 + l < hi ? col0 + l : hi - 1;
            float sum = y == 0 ? A.part[(2 * b + 1) * A.d + col] : 0.0f;
#pragma unroll 8
            for (int64_t q = 1 + y; q <= more; q += L) sum += A.part[2 * (b + q) * A.d + col];
            s_sum[y][l] = sum;
            __syncthreads();
            if (y == 0 && col0 + l < hi) {
                float all = 0.0f;
#pragma unroll
                for (int q = 0; q < L; ++q) all += s_sum[q][l];
                static_cast<T*>(A.out)[(int64_t)c * A.d + col] = from_f32<T>(all * A.scale);
            }
            __syncthreads();
        }
    }
}

// Blocks whose lanes take `units` units, four each, or as many as are of use.
unsigned some_blocks(int64_t units, int lanes) {
    const int64_t b = ((units << lanes) + 1023) / 1024;
    return (unsigned)(b < 1 ? 1 : b < 16384 ? b : 16384);
}

template <class T>
hipError_t forward_t(TableArgs A, const TableShape& L, hipStream_t s) {
    A.lanes = L.lanes;
    A.slices = L.slices;
    // Few rows: a unit a lane, all at once.
    const int64_t units = A.n * A.slices, few = (units << A.lanes) <= 256 * 1024 ? 4 : 1;
    const dim3 g(some_blocks(units * few, A.lanes)), b(256);
    if (A.n * A.d * (int64_t)sizeof(T) > kStreamBytes) hipLaunchKernelGGL((k_table_fwd<T, true>), g, b, 0, s, A);
    else hipLaunchKernelGGL((k_table_fwd<T, false>), g, b, 0, s, A);
    return hipGetLastError();
}

template <class T>
hipError_t backward_t(TableArgs A, const TableShape& L, hipStream_t s) {
    A.lanes = L.lanes;
    A.slices = L.slices;
    const int64_t rows = 256 >> L.lanes;   // of a block
    A.chunk_blocks = (uint32_t)((L.chunks * L.slices + rows - 1) / rows);
    hipLaunchKernelGGL((k_table_bwd<T>), dim3(A.chunk_blocks + some_blocks((int64_t)A.k * L.slices, L.lanes)), dim3(256),
                       0, s, A);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || L.chunks < 2) return e;
    // The fewer of ids and chunks, up to 256 tests a block while there are 1024 blocks.
    A.by_chunk = L.chunks < A.k;
    const int64_t all = A.by_chunk ? L.chunks : A.k, tests = all / 1024;
    A.tests = (int32_t)(tests < 1 ? 1 : tests < 256 ? tests : 256);
    const unsigned gx = (unsigned)((all + A.tests - 1) / A.tests);
    if (A.d < 256) {
        hipLaunchKernelGGL((k_table_join<T, 32>), dim3(gx, (unsigned)((A.d + 7) / 8)), dim3(256), 0, s, A);
    } else {
        const int64_t gy = (A.d + 63) / 64;
        hipLaunchKernelGGL((k_table_join<T, 4>), dim3(gx, (unsigned)(gy < 64 ? gy : 64)), dim3(256), 0, s, A);
    }
    return hipGetLastError();
}

}  // namespace

TableShape table_shape(int64_t n, int32_t d, int type) {
    TableShape L{};
    const int e = type == kF32 ? 4 : 8;
    const int64_t per = ((int64_t)d + e - 1) / e;
    while (L.lanes < 8 && (1 << L.lanes) < per) ++L.lanes;
    L.slices = (int32_t)((per + 255) / 256);
    L.chunks = (n + kTableChunk - 1) / kTableChunk;
    L.bytes = ((size_t)L.chunks * 2 * d * 4 + 255) / 256 * 256;
    if (L.bytes == 0) L.bytes = 256;
    return L;
}

hipError_t launch_table_fwd(const TableArgs& A, int type, hipStream_t s) {
    if (A.n == 0) return hipSuccess;
    const TableShape L = table_shape(A.n, A.d, type);
    if (type == kF32) return forward_t<float>(A, L, s);
    if (type == kBF16) return forward_t<__bf16>(A, L, s);
    return forward_t<_Float16>(A, L, s);
}

hipError_t launch_table_bwd(const TableArgs& A, const TableShape& L, int type, hipStream_t s) {
    if (type == kF32) return backward_t<float>(A, L, s);
    if (type == kBF16) return backward_t<__bf16>(A, L, s);
    return backward_t<_Float16>(A, L, s);
}

}  // namespace km
