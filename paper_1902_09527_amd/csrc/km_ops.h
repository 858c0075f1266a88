// Shared by the operators of a layer conditioned on clusters (km_sort.hip,
// km_norm.hip, km_adapter.hip) and their entry points (km_ops.hip).  The
// public interface is include/kmeans_ops.h.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace km {

// Row types; the values are KM_F32, KM_BF16, KM_F16 of kmeans_ops.h.
enum RowType { kF32 = 0, kBF16 = 1, kF16 = 2 };
constexpr int kF8 = 3;   // e4m3 values with a scale for each 128 (in the grouped products alone)

inline size_t row_type_bytes(int t) { return t == kF32 ? 4 : t == kF8 ? 1 : 2; }

// V elements moved by one load or store.
template <class T, int V>
struct alignas(sizeof(T) * V) Vec {
    T e[V];
};

template <class T>
__device__ __forceinline__ float to_f32(T v) {
    return (float)v;
}
// Rounds to nearest even; the only rounding of a result.
template <class T>
__device__ __forceinline__ T from_f32(float v) {
    return (T)v;
}

// Sum over groups of W consecutive lanes (W a power of two up to 64), the
// same value in every lane of a group.  Cross-lane moves within the vector
// unit, no LDS: quads by permutation, 8 and 16 lanes by mirroring (the parts
// are uniform by then), 32 and 64 by swapping rows.
template <int CTRL>
__device__ __forceinline__ float add_dpp(float v) {
    const int i = __builtin_bit_cast(int, v);
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(i, i, CTRL, 0xf, 0xf, false));
}
template <int W>
__device__ __forceinline__ float group_sum(float v) {
    if constexpr (W >= 2) v = add_dpp<0xb1>(v);    // quad_perm 1,0,3,2
    if constexpr (W >= 4) v = add_dpp<0x4e>(v);    // quad_perm 2,3,0,1
    if constexpr (W >= 8) v = add_dpp<0x141>(v);   // row_half_mirror
    if constexpr (W >= 16) v = add_dpp<0x140>(v);  // row_mirror
    if constexpr (W >= 32) {
        const uint32_t i = __builtin_bit_cast(uint32_t, v);
        const auto r = __builtin_amdgcn_permlane16_swap(i, i, false, false);
        v = __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
    }
    if constexpr (W >= 64) {
        const uint32_t i = __builtin_bit_cast(uint32_t, v);
        const auto r = __builtin_amdgcn_permlane32_swap(i, i, false, false);
        v = __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
    }
    return v;
}

// Whether rows at p with row stride ld (elements of es bytes) and width d can
// be moved `bytes` at a time.
inline bool rows_vec(const void* p, int64_t ld, int64_t d, size_t es, int bytes) {
    return (uintptr_t)p % bytes == 0 && (ld * (int64_t)es) % bytes == 0 && (d * (int64_t)es) % bytes == 0;
}
inline bool rows_vec16(const void* p, int64_t ld, int64_t d, size_t es) { return rows_vec(p, ld, d, es, 16); }

// Error text and device checks of km_capi.hip, for km_ops.hip (km_host.hip).
int ops_hip_error(hipError_t e, const char* what);
int ops_error(int status, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
int ops_check_range(const void* p, size_t bytes, int device, const char* what);

// ---- rows sorted by cluster and back (km_sort.hip)

constexpr int64_t kSortRankMax = 6144;   // slots up to which they are ranked by comparing
constexpr int kSortBins = 4096;          // most digit values of a counting pass
constexpr int kSortThreads = 512;
constexpr int kSortWaves = kSortThreads / 64;

// How N slots with keys 0..k are sorted: passes over digits of `bits` bits,
// tiles of kSortThreads * rounds slots.  passes = 0: ranked by comparing.
struct SortShape {
    int passes, bits, rounds;
    int64_t tiles;
    size_t off_hist, off_tot, off_idx, bytes;   // workspace segments
};
SortShape sort_shape(int64_t N, int32_t k);

struct SortArgs {
    const int32_t* ids;
    int32_t N, k;
    int32_t *order, *pos, *sorted_ids, *offsets;
};
hipError_t launch_sort_plan(const SortArgs& A, const SortShape& S, char* ws, hipStream_t s);

// Rows to and from their sorted places.  A slot is in use where its place is
// below offsets[k] (= *used).
struct MoveArgs {
    const int32_t* pos;    // n x m places
    const int32_t* used;   // slots in use
    int64_t n;
    int32_t m, d;
    const void *src, *src2;   // gather: X; combine: Z; backward: dY and Z
    int64_t ld, ld2;
    void* dst;                // gather: Xs; combine: Y; backward: dZ (contiguous rows)
    const float* w;           // n x m weights, or null (ones)
    float* dw;                // backward: n x m, or null
};
hipError_t launch_sort_gather(const MoveArgs& A, int type, hipStream_t s);
hipError_t launch_sort_combine(const MoveArgs& A, int type, hipStream_t s);
hipError_t launch_sort_combine_bwd(const MoveArgs& A, int type, hipStream_t s);

// ---- layer norm (km_norm.hip)

struct NormArgs {
    const void *X, *dY;
    int64_t ldx, lddy, n;
    int32_t d;
    const void *gamma, *beta;   // d values or null (ones, zeros)
    int32_t param_f32;          // their type: float32, else the rows'
    float eps;
    void *Y, *dX;               // contiguous rows
    float *mean, *rstd;         // written forward, read backward
    float *dgamma, *dbeta;      // d values or null
    float* part;                // backward: blocks x 2 x d partial sums
    int32_t blocks;             // backward: rows of part (set by the launch)
};
int norm_bwd_max_blocks(int64_t n, int32_t d);   // most rows of part that the backward pass writes
hipError_t launch_norm_fwd(NormArgs A, int type, hipStream_t s);
hipError_t launch_norm_bwd(NormArgs A, int type, hipStream_t s);

// ---- shared projection with cluster adapters (km_adapter.hip)

constexpr int kAdapterFew = 64;       // rows up to which the forward pass takes the form for few rows
constexpr int kAdapterMaxRank = 128;

struct AdapterArgs {
    const void *X, *dY;
    int64_t ldx, lddy, n;
    int32_t di, dout, k, r;
    const void *W, *A, *B;
    const int32_t* ids;                         // clusters of the rows (forward, few rows, no plan)
    const int32_t *order, *sids, *offsets;      // the plan; order null: rows are in its order
    const float* scale;                         // k, or null (ones)
    void *Y, *H;                                // H: read backward
    void *dX, *dA, *dB;
};
// The shared product: tiles of `tile` x `tile`, its contraction in `splits` parts.
struct MainShape {
    int32_t tile, splits;
};
struct AdapterShape {
    MainShape main;
    int32_t rp;          // elements a row of the inner products, as the matrix cores take them
    int32_t few;         // forward: few rows
    int32_t pad_i, pad_o;   // din and dout padded to 16 bytes
    int32_t chunk;       // backward: rows a chunk
    int64_t max_items, part_a;   // part_a: float32 values of dA's partial sums
    size_t off_x, off_w, off_y, off_split, off_s, off_shift, off_count, off_items, off_first, off_part, bytes;   // workspace segments
};
AdapterShape adapter_shape(int64_t n, int32_t di, int32_t dout, int32_t k, int32_t r, int type, bool backward);
hipError_t launch_adapter_forward(const AdapterArgs& D, char* ws, const AdapterShape& L, int type, hipStream_t s);
hipError_t launch_adapter_backward(const AdapterArgs& D, char* ws, const AdapterShape& L, int type, hipStream_t s);

// ---- products grouped by cluster (km_group.hip)

constexpr int kGroupFew = 64;   // rows up to which the forward pass takes the form for few rows

struct GroupItem {
    int32_t c, p0, p1, slot;   // places p0 .. p1 of cluster c; slot: partial sum to write, -1: the result itself
};
struct GroupArgs {
    const void *X, *dY;
    int64_t ldx, lddy, n;
    int32_t di, dout, k;
    const void* W;                            // k x dout x di
    const uint8_t *XE, *WE;                   // 8 bits: the scales' bytes
    const int32_t *order, *sids, *offsets;    // the plan; order null: rows are in its order
    void *Y, *dX, *dW;                        // dX, dW: either may be null
};
// A list of items of at most `size` places.
struct GroupList {
    int32_t size;
    int64_t max_items;
    size_t off_count, off_items, off_first;   // workspace segments
};
struct GroupShape {
    int32_t few, grad_tile;
    int32_t splits, any_splits, any_tile;   // parts of the contraction; those and the tile at any addresses
    GroupList rows, cuts;
    size_t off_split, off_part, bytes;
};
int64_t group_items(int64_t n, int32_t k, int32_t size);   // most items that n places are cut into
GroupShape group_shape(int64_t n, int32_t di, int32_t dout, int32_t k, int type, bool backward);
hipError_t launch_group_forward(const GroupArgs& D, char* ws, const GroupShape& L, int type, int out_type,
                                hipStream_t s);
hipError_t launch_group_backward(const GroupArgs& D, char* ws, const GroupShape& L, int type, hipStream_t s);

// ---- rows in 8 bits (km_fp8.hip)

// Q: n rows of dq >= d values (zeros past d), ldq bytes apart; E: a byte for each 128.
hipError_t launch_quantize(const void* X, int64_t ldx, int64_t n, int32_t d, int type, uint8_t* Q, int64_t ldq,
                           int32_t dq, uint8_t* E, hipStream_t s);
hipError_t launch_dequantize(const uint8_t* Q, const uint8_t* E, int64_t n, int32_t d, int type, void* X,
                             hipStream_t s);

// ---- rows of a table (km_table.hip)

constexpr int kTableChunk = 32;   // places of a chunk

struct TableArgs {
    const int32_t* ids;                       // forward
    const int32_t *order, *sids, *offsets;    // backward: the plan
    const void *table, *dY;
    int64_t ld, n;                            // of table or dY; slots
    int32_t d, k;
    float scale;
    void* out;                                // rows, or the table's gradient
    float* part;                              // backward: chunks x 2 x d
    int32_t lanes, slices;                    // set by the launch: log2 of the lanes of a row's slice; slices
    int32_t tests, by_chunk;                  // backward, as the following
    uint32_t chunk_blocks;
};
struct TableShape {
    int32_t lanes, slices;
    int64_t chunks;
    size_t bytes;
};
TableShape table_shape(int64_t n, int32_t d, int type);
hipError_t launch_table_fwd(const TableArgs& A, int type, hipStream_t s);
hipError_t launch_table_bwd(const TableArgs& A, const TableShape& L, int type, hipStream_t s);

// ---- the norm over many tensors (km_clip.hip)

struct ClipShape {
    int32_t step, scale_step;   // elements a block, of the first and the second pass
    int64_t parts;              // blocks of the first pass
    size_t bytes;
};
ClipShape clip_shape(const int64_t* sizes, int32_t count);
hipError_t launch_clip_norm(const void* const* p, const int64_t* sizes, const int32_t* types, int32_t count,
                            const ClipShape& L, double* part, hipStream_t s);
hipError_t launch_clip_total(const ClipShape& L, const double* part, float* norm, hipStream_t s);
// norm may be null (a call without tensors of any element).
hipError_t launch_clip_scale(const void* const* p, void* const* q, const int64_t* sizes, const int32_t* types,
                             int32_t count, const ClipShape& L, const double* part, double limit, float* norm,
                             hipStream_t s);

}  // namespace km
