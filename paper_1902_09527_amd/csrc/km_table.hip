// Rows of a table by their ids, scaled, and the table's gradient:
//   y_i = s T[id_i],  dT[c] = s sum over the slots of id c of dy.
//
// The gradient goes by the sorted plan, so that no sum depends on the order of
// atomics.  Ids of few slots are summed by the lanes of their row.  Of an id with
// more, the places are cut into fixed chunks, whose float32 sums are joined in
// order.  A chunk is a block, and an id of many slots may begin in one chunk,
// cover others and end in a last one: every chunk has two places for what it
// cannot finish, the part of an id that began before it and of one that goes on
// behind it.
//
// Bound by the memory's rate: 16 bytes a lane, rows at any address.
#include "km_tile.h"

namespace km {

namespace {

// A lane's 16 bytes of a row of d elements.
template <class T>
using Part = Vec<T, 16 / (int)sizeof(T)>;

template <class T>
__device__ __forceinline__ Part<T> part_get(const T* row, int64_t c, int64_t d) {
    constexpr int E = 16 / (int)sizeof(T);
    Part<T> v;
    if (c + E <= d) {
        __builtin_memcpy(&v, row + c, 16);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v.e[e] = row[c + e < d ? c + e : 0];
    }
    return v;
}
template <class T, int E>
__device__ __forceinline__ void part_put(T* row, int64_t c, int64_t d, const float (&v)[E]) {
    Vec<T, E> o;
#pragma unroll
    for (int e = 0; e < E; ++e) o.e[e] = from_f32<T>(v[e]);
    if (c + E <= d) {
        __builtin_memcpy(row + c, &o, sizeof(o));
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (c + e < d) row[c + e] = o.e[e];
    }
}

template <class T>
__global__ __launch_bounds__(256) void k_table_fwd(TableArgs A) {
    constexpr int E = 16 / (int)sizeof(T), UN = 4;
    const int64_t per = (A.d + E - 1) / E, total = A.n * per, step = (int64_t)gridDim.x * 256;
    for (int64_t i0 = (int64_t)blockIdx.x * 256 + threadIdx.x; i0 < total; i0 += UN * step) {
        int64_t row[UN], col[UN];
        int id[UN];
        Part<T> v[UN];
#pragma unroll
        for (int y = 0; y < UN; ++y) {
            const int64_t i = i0 + y * step < total ? i0 + y * step : i0;
            row[y] = i / per;
            col[y] = (i - row[y] * per) * E;
            id[y] = A.ids[row[y]];
        }
#pragma unroll
        for (int y = 0; y < UN; ++y)
            v[y] = part_get(static_cast<const T*>(A.table) + ((unsigned)id[y] < (unsigned)A.k ? id[y] : 0) * A.ld, col[y],
                            A.d);
#pragma unroll
        for (int y = 0; y < UN; ++y) {
            if (i0 + y * step >= total) break;
            float o[E];
            const bool in = (unsigned)id[y] < (unsigned)A.k;
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = in ? to_f32(v[y].e[e]) * A.scale : 0.0f;
            part_put(static_cast<T*>(A.out) + row[y] * A.d, col[y], A.d, o);
        }
    }
}

// --------------------------------------------------------------------------

// By a lane an id and 16 bytes of its row: ids of at most kTableShort slots.
template <class T>
__device__ __forceinline__ void short_ids(const TableArgs& A, int64_t block, int64_t blocks) {
    constexpr int E = 16 / (int)sizeof(T), UN = 4;
    const int64_t per = (A.d + E - 1) / E, total = A.k * per, step = blocks * 256;
    for (int64_t i0 = block * 256 + threadIdx.x; i0 < total; i0 += UN * step) {
        int64_t c[UN], col[UN];
        int a[UN], b[UN];
#pragma unroll
        for (int y = 0; y < UN; ++y) {
            const int64_t i = i0 + y * step < total ? i0 + y * step : i0;
            c[y] = i / per;
            col[y] = (i - c[y] * per) * E;
            a[y] = A.offsets[c[y]];
            b[y] = A.offsets[c[y] + 1];
        }
        // The first slot of each is on its way before the others are.
        int64_t row[UN];
#pragma unroll
        for (int y = 0; y < UN; ++y) row[y] = b[y] > a[y] && b[y] - a[y] <= kTableShort ? A.order[a[y]] : -1;
        Part<T> v[UN];
#pragma unroll
        for (int y = 0; y < UN; ++y)
            if (row[y] >= 0) v[y] = part_get(static_cast<const T*>(A.dY) + row[y] * A.ld, col[y], A.d);
#pragma unroll
        for (int y = 0; y < UN; ++y) {
            if (i0 + y * step >= total) break;
            const int count = b[y] - a[y];
            if (count > kTableShort) continue;
            float sum[E];
#pragma unroll
            for (int e = 0; e < E; ++e) sum[e] = count > 0 ? to_f32(v[y].e[e]) : 0.0f;
            for (int p = a[y] + 1; p < b[y]; p += UN) {
                Part<T> w[UN];
#pragma unroll
                for (int q = 0; q < UN; ++q)
                    w[q] = part_get(static_cast<const T*>(A.dY) + (int64_t)A.order[p + q < b[y] ? p + q : p] * A.ld, col[y],
                                    A.d);
#pragma unroll
                for (int q = 0; q < UN; ++q)
                    if (p + q < b[y])
#pragma unroll
                        for (int e = 0; e < E; ++e) sum[e] += to_f32(w[q].e[e]);
            }
#pragma unroll
            for (int e = 0; e < E; ++e) sum[e] *= A.scale;
            part_put(static_cast<T*>(A.out) + c[y] * A.d, col[y], A.d, sum);
        }
    }
}

// Ids of more slots, by chunks of A.chunk places: 2^A.lanes lanes share a row's
// slice, the other lanes of a block take other rows.
template <class T>
__device__ __forceinline__ void long_ids(const TableArgs& A, int64_t block, float (*s_sum)[16 / sizeof(T) + 1],
                                         int* s_runs) {
    constexpr int E = 16 / (int)sizeof(T), UN = 8;
    const int lanes = 1 << A.lanes, groups = 256 >> A.lanes, slices = A.slices;
    const int64_t b = block / slices;
    const int slice = (int)(block - b * slices), l = threadIdx.x & (lanes - 1), group = threadIdx.x >> A.lanes;
    const int64_t col = ((int64_t)slice * lanes + l) * E, used = A.offsets[A.k];
    const int64_t p0 = b * A.chunk, p1 = p0 + A.chunk < used ? p0 + A.chunk : used;
    // Where the ids of many slots begin in this chunk.
    if (threadIdx.x == 0) s_runs[0] = 0;
    __syncthreads();
    for (int64_t p = p0 + threadIdx.x; p < p1; p += 256) {
        const int c = A.sids[p];
        if (p > p0 && A.sids[p - 1] == c) continue;
        if (A.offsets[c + 1] - A.offsets[c] > kTableShort) s_runs[1 + atomicAdd(s_runs, 1)] = (int)(p - p0);
    }
    __syncthreads();
    const int runs = s_runs[0];
    for (int r = 0; r < runs; ++r) {   // in whatever order: each has a sum of its own
        const int64_t p = p0 + s_runs[1 + r];
        const int c = A.sids[p], first = A.offsets[c], last = A.offsets[c + 1];
        const int64_t end = last < p1 ? last : p1;
        float sum[E] = {};
        if (col < A.d) {
            for (int64_t q0 = p + group; q0 < end; q0 += UN * groups) {
                int64_t row[UN];
#pragma unroll
                for (int y = 0; y < UN; ++y) row[y] = A.order[q0 + y * groups < end ? q0 + y * groups : q0];
                Part<T> w[UN];
#pragma unroll
                for (int y = 0; y < UN; ++y) w[y] = part_get(static_cast<const T*>(A.dY) + row[y] * A.ld, col, A.d);
#pragma unroll
                for (int y = 0; y < UN; ++y)
                    if (q0 + y * groups < end)
#pragma unroll
                        for (int e = 0; e < E; ++e) sum[e] += to_f32(w[y].e[e]);
            }
        }
        // The groups' sums, halves added in turn.
#pragma unroll
        for (int e = 0; e < E; ++e) s_sum[threadIdx.x][e] = sum[e];
        __syncthreads();
        for (int h = groups / 2; h > 0; h /= 2) {
            if (group < h)
#pragma unroll
                for (int e = 0; e < E; ++e) s_sum[threadIdx.x][e] += s_sum[threadIdx.x + h * lanes][e];
            __syncthreads();
        }
        if (group == 0 && col < A.d) {
            if (first >= p0 && last <= p1) {
#pragma unroll
                for (int e = 0; e < E; ++e) sum[e] = s_sum[threadIdx.x][e] * A.scale;
                part_put(static_cast<T*>(A.out) + (int64_t)c * A.d, col, A.d, sum);
            } else {
                float* part = A.part + (2 * b + (first >= p0)) * A.d;
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (col + e < A.d) part[col + e] = s_sum[threadIdx.x][e];
            }
        }
        __syncthreads();
    }
}

template <class T>
__global__ __launch_bounds__(256) void k_table_bwd(TableArgs A) {
    __shared__ float s_sum[256][16 / sizeof(T) + 1];
    __shared__ int s_runs[1 + kTableChunk / kTableShort + 2];   // runs of a chunk: all but the ends' are whole
    if (blockIdx.x < A.long_blocks) long_ids<T>(A, blockIdx.x, s_sum, s_runs);
    else short_ids<T>(A, blockIdx.x - A.long_blocks, gridDim.x - A.long_blocks);
}

// An id that begins in chunk blockIdx.x and goes on behind it: the sum of its
// parts in order, 16 lanes a column each taking every 16th.
template <class T>
__global__ __launch_bounds__(256) void k_table_join(TableArgs A) {
    __shared__ float s_sum[16][17];
    const int64_t b = blockIdx.x, p0 = b * A.chunk, p1 = p0 + A.chunk;
    const int64_t used = A.offsets[A.k];
    if (p1 >= used) return;
    const int c = A.sids[p1 - 1], first = A.offsets[c], last = A.offsets[c + 1];
    if (first < p0 || last <= p1 || last - first <= kTableShort) return;
    const int64_t behind = (last - 1) / A.chunk - b;   // chunks after this one
    const int l = threadIdx.x & 15, y = threadIdx.x >> 4;
    for (int64_t col0 = (int64_t)blockIdx.y * 16; col0 < A.d; col0 += (int64_t)gridDim.y * 16) {
        const int64_t col = col0 + l < A.d ? col0 + l : A.d - 1;
        float sum = y == 0 ? A.part[(2 * b + 1) * A.d + col] : 0.0f;
#pragma unroll 8
        for (int64_t q = 1 + y; q <= behind; q += 16) sum += A.part[2 * (b + q) * A.d + col];
        s_sum[y][l] = sum;
        __syncthreads();
        if (y == 0 && col0 + l < A.d) {
            float all = 0.0f;
#pragma unroll
            for (int q = 0; q < 16; ++q) all += s_sum[q][l];
            static_cast<T*>(A.out)[(int64_t)c * A.d + col] = from_f32<T>(all * A.scale);
        }
        __syncthreads();
    }
}

unsigned some_blocks(int64_t lanes, int64_t most) {
    const int64_t b = (lanes + 255) / 256;
    return (unsigned)(b < 1 ? 1 : b < most ? b : most);
}

template <class T>
hipError_t forward_t(const TableArgs& A, hipStream_t s) {
    constexpr int E = 16 / (int)sizeof(T);
    const int64_t chunks = A.n * ((A.d + E - 1) / E);
    hipLaunchKernelGGL((k_table_fwd<T>), dim3(some_blocks((chunks + 3) / 4, 16384)), dim3(256), 0, s, A);
    return hipGetLastError();
}

template <class T>
hipError_t backward_t(TableArgs A, const TableShape& L, hipStream_t s) {
    constexpr int E = 16 / (int)sizeof(T);
    A.chunk = L.chunk;
    A.lanes = L.lanes;
    A.slices = L.slices;
    A.long_blocks = (uint32_t)(L.chunks * L.slices);
    const int64_t parts = (int64_t)A.k * ((A.d + E - 1) / E);
    hipLaunchKernelGGL((k_table_bwd<T>), dim3(A.long_blocks + some_blocks((parts + 3) / 4, 16384)), dim3(256), 0, s, A);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || L.chunks < 2) return e;
    const int64_t gy = (A.d + 15) / 16;
    hipLaunchKernelGGL((k_table_join<T>), dim3((unsigned)L.chunks, (unsigned)(gy < 64 ? gy : 64)), dim3(256), 0, s, A);
    return hipGetLastError();
}

}  // namespace

TableShape table_shape(int64_t n, int32_t d, int type) {
    TableShape L{};
    const int e = type == kF32 ? 4 : 8;
    const int64_t per = ((int64_t)d + e - 1) / e;
    while (L.lanes < 8 && (1 << L.lanes) < per) ++L.lanes;
    L.slices = (int32_t)((per + 255) / 256);
    // Four rounds of a block's rows in flight.
    const int rows = 4 * 8 * (256 >> L.lanes);
    L.chunk = rows < 64 ? 64 : rows > kTableChunk ? kTableChunk : rows;
    L.chunks = (n + L.chunk - 1) / L.chunk;
    L.bytes = ((size_t)L.chunks * 2 * d * 4 + 255) / 256 * 256;
    if (L.bytes == 0) L.bytes = 256;
    return L;
}

hipError_t launch_table_fwd(const TableArgs& A, int type, hipStream_t s) {
    if (A.n == 0) return hipSuccess;
    if (type == kF32) return forward_t<float>(A, s);
    if (type == kBF16) return forward_t<__bf16>(A, s);
    return forward_t<_Float16>(A, s);
}

hipError_t launch_table_bwd(const TableArgs& A, const TableShape& L, int type, hipStream_t s) {
    if (type == kF32) return backward_t<float>(A, L, s);
    if (type == kBF16) return backward_t<__bf16>(A, L, s);
    return backward_t<_Float16>(A, L, s);
}

}  // namespace km
