// Where the 16-byte chunks of an operand's tile lie, in memory and in LDS: plain
// arithmetic, that the host checks against a matrix's end as the kernels use it.
#pragma once

#include <stdint.h>

#ifdef __HIPCC__
#define KM_BOTH __host__ __device__ __forceinline__
#else
#define KM_BOTH inline
#endif

namespace km {

// Chunk position of a stage's rows in LDS: rows are 128 bytes, so 16 rows read
// at one chunk index fall on all 64 banks once.
KM_BOTH int swz(int row, int c) { return c ^ ((row >> 1) & 7); }

KM_BOTH int swz4(int row, int c) { return c ^ ((row >> 2) & 3); }   // rows of 64 bytes

// The same for tiles that hold the contraction along their rows (TR): 16-bit
// tiles are read 4 rows x 16 columns at a time, float32 by columns.
template <class T, int CPR>
KM_BOTH int swz_tr(int k, int c) {
    const int m = sizeof(T) == 2 ? ((k & 3) | ((k >> 3) & 1) << 2) << 1 : ((k >> 2) & 3) << 2;
    return c ^ (m & (CPR - 1));
}

// A stage of such a tile of a K x P matrix: 128 bytes of rows by TN columns, dealt in
// chunks to NT threads.  A thread's chunk i is kDown rows below its chunk i - 1.
template <class T, int TN, int NT>
struct TrStage {
    static constexpr int E = 16 / (int)sizeof(T), CPR = TN / E, BK = 128 / (int)sizeof(T), kDown = NT / CPR;
    static constexpr int N = BK / kDown;   // chunks of a thread
    static_assert(kDown % 8 == 0, "16 rows swizzle alike: two places a thread, of even and odd chunks");

    // The first column of the tile at bn: the last tile of a width that TN does not divide
    // moves left until it is whole, so that nothing is read past a row's end (past the
    // last row's that is past the matrix).  It and its neighbour then give the same
    // values twice.  Where P is of whole chunks, so is what it moves to.
    static KM_BOTH int first(int bn, int P) { return P >= TN && bn > P - TN ? P - TN : bn; }
    // Stages from the first on that have no chunk past an end.
    static KM_BOTH int whole(int K, int P) { return P >= TN ? K / BK : 0; }

    static KM_BOTH int row(int i, int tid) { return i * kDown + tid / CPR; }   // of the stage
    static KM_BOTH int column(int i, int tid) { return swz_tr<T, CPR>(row(i, tid), tid % CPR) * E; }   // of the tile
    // Whether chunk i of stage k has its place in the matrix, the tile beginning at bn.
    static KM_BOTH bool in(int i, int tid, int k, int bn, int K, int P) {
        return k * BK + row(i, tid) < K && bn + column(i, tid) < P;
    }
    // Its bytes from the stage's first row in the tile's first column: those of the rows
    // above chunk i, and `behind`, the same for all even and for all odd chunks.
    static KM_BOTH uint64_t above(int i, uint32_t row_bytes) { return (uint64_t)(i * kDown) * row_bytes; }
    static KM_BOTH uint32_t behind(int i, int tid, uint32_t row_bytes) {
        return (uint32_t)(tid / CPR) * row_bytes + (uint32_t)column(i, tid) * (uint32_t)sizeof(T);
    }
};

}  // namespace km
