// Products grouped by cluster, with ragged sizes: for the rows of cluster c
//   y = W_c x,  dx = W_c^T dy,  dW_c = sum dy x^T,
// in float32, bfloat16 and float16, and y with both operands in 8-bit floating
// point, a power of two for each 128 elements along the contraction.
//
// Rows are taken in cluster order (places).  A list of row tiles, none of which
// spans two clusters, is made on the device from the plan's offsets, so nothing
// has to know the sizes on the host: the grid is the most tiles that n rows of k
// clusters can have, and blocks past the list's end do nothing.  dW contracts
// over a cluster's places; long clusters are cut into chunks where there are few
// tiles, and the chunks' float32 sums are joined in order.
//
// Sums are float32 (matrix-core accumulators); a result is rounded once.
#include <limits.h>
#include <math.h>

#include "km_tile.h"

namespace km {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// What an operand of R rows (or columns) by 64 bytes of the contraction is for a
// lane, and the product of two: D[m][n] += sum_k first[m][k] second[n][k].  A
// lane holds runs of four m of its column n = lane % R.
// The results' type O matters for 8 bits alone.
template <class T, class O>
struct Op {
    static constexpr int R = 16, E = Mma<T>::E;
    using Acc = f32x4;
    struct Frag {
        u32x4 v;
    };
    static __device__ __forceinline__ int chunk(int lane) { return lane >> 4; }   // of a row's 4 chunks of 64 bytes
    static __device__ __forceinline__ Frag read(const char* buf, int at) {
        return {*reinterpret_cast<const u32x4*>(buf + at)};
    }
    static __device__ __forceinline__ Acc mma(const Frag& a, const Frag& b, Acc c, int, int) {
        return Mma<T>::mma(a.v, b.v, c);
    }
    static constexpr int kRuns = 1;
    static __device__ __forceinline__ int run(int, int lane) { return (lane >> 4) * 4; }   // first m of run j
};
// e4m3 values: 64 of a row, two chunks a lane.  The scale of 64 elements comes as
// a byte (2^(byte - 127)) of the lane's row; a matrix step takes one for each 32.
// The step adds its products to float32 accumulators, but of each 8 consecutive
// ones it drops the bits more than 13 below the largest one's exponent m (measured,
// one pair of products at a time; the step without scales does too): less than 2^-10
// 2^m of the 8, 1.3e-5 of the norm for products of 4096 normal values.  A bfloat16
// result's own rounding is 2^-9 of it or more, a float16 one's 2^-12, so a float16
// result of very uneven products may be two roundings off; the e4m3 operands were
// rounded by 2^-4 before.  It is taken for both because it is the 8-bit rate: products
// that keep float32 (the next form, for float32 results) are bfloat16's at best, and
// there 2.5 times as long (16,380 rows, 10 clusters, 4096 to 8192: 1440 us, 570).
template <class O>
struct Op<uint8_t, O> {
    static constexpr int R = 32, E = 16;
    using Acc = f32x16;
    struct Frag {
        u32x4 v, w;
    };
    static __device__ __forceinline__ int chunk(int lane) { return (lane >> 5) * 2; }
    static __device__ __forceinline__ Frag read(const char* buf, int at) {
        // The second chunk is the first's neighbour: bit 4 of the swizzled place.
        return {*reinterpret_cast<const u32x4*>(buf + at), *reinterpret_cast<const u32x4*>(buf + (at ^ 16))};
    }
    static __device__ __forceinline__ Acc mma(const Frag& a, const Frag& b, Acc c, int sa, int sb) {
        return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(__builtin_bit_cast(i32x8, a),
                                                               __builtin_bit_cast(i32x8, b), c, 0, 0, 0, sa, 0, sb);
    }
    static constexpr int kRuns = 4;
    static __device__ __forceinline__ int run(int j, int lane) { return j * 8 + (lane >> 5) * 4; }
};

// Eight e4m3 values as bfloat16, which holds them exactly; NaN under a byte of 255.
__device__ __forceinline__ u32x4 widen(uint32_t lo, uint32_t hi, int byte) {
    const float scale = byte == 255 ? INFINITY : 1.0f;
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    struct Four {
        bf16x2 v[4];
    } o{{__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false),
         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true),
         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false),
         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true)}};
    return __builtin_bit_cast(u32x4, o);
}
// e4m3 values with float32 results: widened to bfloat16, whose products and sums
// keep float32.  A chunk is the operand of two steps.  The powers of two go to the
// sums of a block (add_scaled): values times theirs may lie outside of bfloat16, the
// products' being in range, and its matrix steps lose what lies below 2^-126.
template <>
struct Op<uint8_t, float> {
    static constexpr int R = 16, E = 16;
    using Acc = f32x4;
    struct Frag {
        u32x4 v;
    };
    static __device__ __forceinline__ int chunk(int lane) { return lane >> 4; }
    static __device__ __forceinline__ Frag read(const char* buf, int at) {
        return {*reinterpret_cast<const u32x4*>(buf + at)};
    }
    struct Wide {
        u32x4 v[2];
    };
    static __device__ __forceinline__ Wide wide(const Frag& a, int byte) {
        return {{widen(a.v[0], a.v[1], byte), widen(a.v[2], a.v[3], byte)}};
    }
    static __device__ __forceinline__ Acc mma(const Wide& a, const Wide& b, Acc c) {
        return Mma<__bf16>::mma(a.v[1], b.v[1], Mma<__bf16>::mma(a.v[0], b.v[0], c));
    }
    // v times the powers of its first operand's rows (bytes a) and its second's (b).
    static __device__ __forceinline__ void add_scaled(Acc& c, const Acc& v, const int (&a)[4], int b) {
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] += __builtin_ldexpf(v[i], a[i] + b - 254);
    }
    static constexpr int kRuns = 1;
    static __device__ __forceinline__ int run(int, int lane) { return (lane >> 4) * 4; }
};

// 8 bits with float32 results: widened operands take the registers of the larger
// tiles, so there is one form at any address (16,380 rows, 10 clusters, 4096 to 8192:
// 1.44 to 1.51 ms; four clusters of 2000 rows, 2001 to 2003: 123 us).
template <class T, class O>
constexpr bool kWide = sizeof(T) == 1 && sizeof(O) == 4;

// --------------------------------------------------------------------------
// Lists of row tiles and of chunks.

// What to list: `size` places at most an item, none of two clusters.
struct ListArgs {
    const int32_t* offsets;
    int32_t k, size;
    int32_t* count;
    GroupItem* items;
    int32_t *first, *num;   // per cluster: first partial slot, items; null: not wanted
};

// A block a list.  In order of the clusters.  3 us for 16 clusters, 5 for 64 and two
// lists: a launch's own time, that neither the plan nor the host could save.  A
// cluster's items are written by one lane: 20 us for 100,000 rows in one cluster, 650
// for a million rows of 64 columns in one (15,625 items).
__global__ __launch_bounds__(1024) void k_gr_list(ListArgs A0, ListArgs A1) {
    const ListArgs& A = blockIdx.x ? A1 : A0;
    __shared__ int s[2][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int items = 0, slots = 0;   // so far
    for (int c0 = 0; c0 < A.k; c0 += 1024) {
        const int c = c0 + tid;
        const int a = c < A.k ? A.offsets[c] : 0, b = c < A.k ? A.offsets[c + 1] : 0;
        const int ni = (b - a + A.size - 1) / A.size, ns = ni > 1 ? ni : 0;
        int xi = ni, xs = ns;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int ui = __shfl_up(xi, o), us = __shfl_up(xs, o);
            if (lane >= o) xi += ui, xs += us;
        }
        if (lane == 63) s[0][wave] = xi, s[1][wave] = xs;
        __syncthreads();
        int bi = items, bs = slots;
        for (int w = 0; w < 16; ++w) {
            if (w < wave) bi += s[0][w], bs += s[1][w];
            items += s[0][w];
            slots += s[1][w];
        }
        bi += xi - ni;
        bs += xs - ns;
        if (c < A.k) {
            if (A.num) {
                A.first[c] = bs;
                A.num[c] = ni;
            }
            for (int q = 0; q < ni; ++q) {
                const int p = a + q * A.size;
                A.items[bi + q] = GroupItem{c, p, b - p < A.size ? b : p + A.size, A.num && ni > 1 ? bs + q : -1};
            }
        }
        __syncthreads();
    }
    if (tid == 0) A.count[0] = items;
}

// --------------------------------------------------------------------------
// Results.

// Four consecutive results, col0 .. of a row of P, at any address.
template <class O>
__device__ __forceinline__ void put4(O* row, int64_t col0, int64_t P, f32x4 v) {
    Vec<O, 4> o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o.e[i] = from_f32<O>(v[i]);
    if (col0 + 4 <= P) {
        __builtin_memcpy(row + col0, &o, sizeof(o));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (col0 + i < P) row[col0 + i] = o.e[i];
    }
}

struct Two {
    uint32_t a, b;
};
template <class O>
__device__ __forceinline__ Two pack4(f32x4 v) {
    Vec<O, 4> x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x.e[i] = from_f32<O>(v[i]);
    return __builtin_bit_cast(Two, x);
}
// The odd halves (rows of 16 or 32 lanes) of p against the even ones of q.
template <int W>
__device__ __forceinline__ void swap_rows(uint32_t& p, uint32_t& q) {
    if constexpr (W == 16) {
        const auto s = __builtin_amdgcn_permlane16_swap(p, q, false, false);
        p = s[0], q = s[1];
    } else {
        const auto s = __builtin_amdgcn_permlane32_swap(p, q, false, false);
        p = s[0], q = s[1];
    }
}
__device__ __forceinline__ uint32_t other_half16(uint32_t v) {   // of lane + 8 in its 16
    return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x128, 0xf, 0xf, false);   // row_ror:8
}
// 16 bytes to column col of a row of P, at any address.  STREAM: past the caches.
template <bool STREAM, class O>
__device__ __forceinline__ void put8(O* row, int64_t col, int64_t P, u32x4 o) {
    if (col + 8 <= P) {
        typedef u32x4 __attribute__((aligned(2))) any4;
        if constexpr (STREAM) __builtin_nontemporal_store(o, reinterpret_cast<any4*>(row + col));
        else __builtin_memcpy(row + col, &o, 16);
    } else {
        const Vec<O, 8> e = __builtin_bit_cast(Vec<O, 8>, o);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i < P) row[col + i] = e.e[i];
    }
}

// A wave's results of one operand of rows (Q::R of them) and FC of columns, from
// column col0 on.  row(r): where row r of the operand goes, null: nowhere.  In 16
// bits the lanes exchange parts first, so that 16 rows of 64 bytes are written at
// once, or (LINES) 8 of 128, past the caches; every lane of the wave calls it.
template <class Q, class O, bool LINES, int FC, class F>
__device__ __forceinline__ void put_rows(const typename Q::Acc (&acc)[FC], int64_t col0, int64_t P, int lane, F&& row) {
    auto part = [&](int h, int j) {
        f32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = acc[h][j * 4 + i];
        return v;
    };
    if constexpr (sizeof(O) == 2 && FC * Q::R == 64) {
        // x[s][i], y[s][i]: the first and last 32 columns of 16 rows, lane l holding
        // row l % 16, eight columns from at on.
        const int g = lane >> 4, li = lane & 15, at = (g & 1) * 16 + (g >> 1) * 8;
        constexpr int S = Q::R / 16;
        uint32_t x[S][4], y[S][4];
        if constexpr (Q::R == 16) {
#pragma unroll
            for (int h = 0; h < 4; h += 2) {
                Two p = pack4<O>(part(h, 0)), q = pack4<O>(part(h + 1, 0));
                swap_rows<16>(p.a, q.a);
                swap_rows<16>(p.b, q.b);
                uint32_t* o = h == 0 ? x[0] : y[0];
                o[0] = p.a, o[1] = p.b, o[2] = q.a, o[3] = q.b;
            }
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t z[2][4];
#pragma unroll
                for (int j = 0; j < 4; j += 2) {
                    Two p = pack4<O>(part(h, j)), q = pack4<O>(part(h, j + 1));
                    swap_rows<32>(p.a, q.a);
                    swap_rows<32>(p.b, q.b);
                    uint32_t* o = z[j / 2];
                    o[0] = p.a, o[1] = p.b, o[2] = q.a, o[3] = q.b;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    swap_rows<16>(z[0][i], z[1][i]);
                    (h == 0 ? x : y)[0][i] = z[0][i];
                    (h == 0 ? x : y)[S - 1][i] = z[1][i];
                }
            }
        }
        if constexpr (!LINES) {
#pragma unroll
            for (int s = 0; s < S; ++s) {
                O* p = row(s * 16 + li);
                if (!p) continue;
                put8<false>(p, col0 + at, P, u32x4{x[s][0], x[s][1], x[s][2], x[s][3]});
                put8<false>(p, col0 + at + 32, P, u32x4{y[s][0], y[s][1], y[s][2], y[s][3]});
            }
            return;
        }
        const bool low = li < 8;
        const int64_t col = col0 + at + (low ? 0 : 32);
#pragma unroll
        for (int s = 0; s < S; ++s) {
            u32x4 o[2];   // rows 0 .. 7, 8 .. 15
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t t = other_half16(low ? y[s][i] : x[s][i]);
                o[0][i] = low ? x[s][i] : t;
                o[1][i] = low ? t : y[s][i];
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                O* p = row(s * 16 + i * 8 + (li & 7));
                if (p) put8<true>(p, col, P, o[i]);
            }
        }
    } else {
        O* p = row(lane % Q::R);
        if (!p) return;
#pragma unroll
        for (int h = 0; h < FC; ++h)
#pragma unroll
            for (int j = 0; j < Q::kRuns; ++j) put4(p, col0 + h * Q::R + Q::run(j, lane), P, part(h, j));
    }
}

// --------------------------------------------------------------------------
// Y[row] = V_c U[row], V = W_c (P x K) forward, W_c^T (W_c is K x P) with TR.

struct MainArgs {
    const void* U;
    int64_t ldu, n;
    const void* W;
    const uint8_t *UE, *WE;   // 8 bits: a byte for each 128 elements of a row, nb a row
    const int32_t *order, *count, *used;   // used: places of clusters
    const GroupItem* items;
    void* Y;
    int32_t K, P, nb;
    int32_t tn;               // tiles of columns
    int32_t splits, share;    // parts of the contraction, stages of one; more than one part: sums to part
    float* part;              // splits x n x P, by place
};

// A block's place among all of a grid's: a launch has fewer than 2^32 threads in a
// dimension, so grids of a block a tile may have two (many_blocks).
__device__ __forceinline__ uint32_t block_at() { return blockIdx.y * gridDim.x + blockIdx.x; }

// Rows of no cluster: zeros, by all blocks, a wave a row.
template <class O>
__device__ __forceinline__ void zero_rows(const MainArgs& A, int waves) {
    constexpr int E = 16 / (int)sizeof(O);
    const int64_t step = (int64_t)gridDim.x * gridDim.y * waves;
    for (int64_t p = A.used[0] + (int64_t)block_at() * waves + (threadIdx.x >> 6); p < A.n; p += step) {
        O* y = static_cast<O*>(A.Y) + row_of(A.order, p) * A.P;
        for (int64_t col = (threadIdx.x & 63) * E; col < A.P; col += 64 * E) {
            const u32x4 zero{0, 0, 0, 0};
            if (col + E <= A.P) {
                __builtin_memcpy(y + col, &zero, 16);
            } else {
                for (int i = 0; col + i < A.P; ++i) y[col + i] = from_f32<O>(0.0f);
            }
        }
    }
}

// What the two forms share: a tile is TM places x TN columns, WR x WC waves; the
// contraction goes in stages of 128 bytes a row.  Rows of a tile are dealt to its
// waves in kParts turns, so that a tile of few rows leaves out the products of the
// turns past them.
template <class T, class O, int TM, int TN, int WR, int WC>
struct Geo {
    using P = Op<T, O>;
    static constexpr int E = P::E, R = P::R, KS = 4 * E, BK = 2 * KS, NT = 64 * WR * WC;
    static constexpr int FR = TM / WR / R, FC = TN / WC / R;
    static constexpr int NU = TM * 8 / NT, NW = TN * 8 / NT, CPR = TN / E;
    static constexpr int kStage = (TM + TN) * 128;
    static constexpr int kParts = FR < 4 ? FR : 4, FP = FR / kParts;   // turns, and a wave's operands of one
    static constexpr int kTurn = FP * R * WR;                          // rows of a turn
    static_assert(FR % kParts == 0 && NT % 128 == 0, "");
    // The tile's row of operand f, but for the lane's.
    static __device__ __forceinline__ int row(int f, int wr) { return f / FP * kTurn + wr * (FP * R) + f % FP * R; }
};

// An item of the list, which nothing writes while a product runs: by way of the
// scalar unit.
__device__ __forceinline__ GroupItem item_at(const GroupItem* items, int64_t i) {
    typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
    const i32x4 v = *reinterpret_cast<const __attribute__((address_space(4))) i32x4*>((uintptr_t)(items + i));
    return GroupItem{v[0], v[1], v[2], v[3]};
}

// A tile of the list: places p0 .. of cluster c, columns bn .. , stages k0 .. of the
// contraction (part `split`).
struct Tile {
    int c, p0, rows, bn, split, k0;
};
// A tile's parts, then down 4 row tiles before the next columns.
template <class T, int TN, int NT, bool TR>
__device__ __forceinline__ Tile tile_at(const MainArgs& A, int items, int u) {
    const int t = u / A.splits, split = u - t * A.splits;
    const int group = 4 * A.tn, grp = t / group, m0 = grp * 4, in = t - grp * group;
    const int gm = items - m0 < 4 ? items - m0 : 4;
    const GroupItem it = item_at(A.items, m0 + in % gm);
    const int bn = in / gm * TN;
    return Tile{it.c, it.p0, it.p1 - it.p0, TR ? TrStage<T, TN, NT>::first(bn, A.P) : bn, split, split * A.share};
}

constexpr int kWindow = 8;   // 8 bits: stages whose scales are in LDS at once, twice

// Blocks stay and take tile after tile.  The stages of all of a block's tiles are
// one sequence: two of them are in LDS, and the next tile's first ones are on their
// way while the last ones of a tile are multiplied and its results are written.
//
// Tiles of 256 x 256 in 8 waves (one block a compute unit: 128 KB of LDS), 128 x 128
// (two) or 64 x 64 (four): the larger reads less for a product, the smaller has less
// past a cluster's end (main_choice has the times).  Bound by the matrix cores where
// clusters are long: four clusters of 4096 rows, 4096 x 4096 bf16, 475 us (1160
// TFLOP/s; one of them by the library 1459), 8 bits 246 us (2240).  16 skewed clusters
// of 16,384 rows, 4096 x 4096 f16, are 4.4 rounds of tiles for 4, and take 565 to 585 us.  By the
// memory where they are short: 64 clusters, 2048 x 2048 bf16, 193 us, 4.0 TB/s.
template <class T, class O, int TM, int TN, int WR, int WC, bool TR>
__global__ __launch_bounds__(64 * WR * WC, TM == 64 ? 4 : 2) void k_gr_main(MainArgs A) {
    using G = Geo<T, O, TM, TN, WR, WC>;
    using P = typename G::P;
    constexpr bool F8 = sizeof(T) == 1;
    constexpr int E = G::E, R = G::R, KS = G::KS, BK = G::BK, NT = G::NT, FR = G::FR, FC = G::FC, NU = G::NU, NW = G::NW;
    constexpr int CPR = G::CPR, kStage = G::kStage, kParts = G::kParts, FP = G::FP, kTurn = G::kTurn;
    static_assert(!F8 || NT >= TM + TN, "");
    extern __shared__ __align__(16) char s_tiles[];
    char* s_scale = s_tiles + 2 * kStage;   // 8 bits: [2][TM + TN][kWindow]
    int32_t* s_rows = reinterpret_cast<int32_t*>(s_scale + (F8 ? 2 * kWindow * (TM + TN) : 0));   // [3][TM]
    const int tid = threadIdx.x, lane = tid & 63, li = lane % R;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wr = wave / WC, wc = wave % WC;

    // Consecutive tiles go to one XCD (blocks are dealt over 8).
    const int items = __builtin_amdgcn_readfirstlane(A.count[0]);
    const int tiles = items * A.tn * A.splits, per = (tiles + 7) / 8, step = gridDim.x / 8;
    const int x0 = (blockIdx.x % 8) * per, x1 = x0 + per < tiles ? x0 + per : tiles;
    int t = x0 + blockIdx.x / 8;
    if (t < x1) {
        const int nk = A.share < 2 ? 2 : A.share;   // stages past the last are of zeros
        // Where a thread's chunks of the next stage come from: bases that move on with
        // the stages, the thread's places behind them being fixed (below 4 GB, as the
        // host sees to).
        const char *ub = nullptr, *wb = nullptr;
        uint32_t uo[NU], wo[TR ? 2 : NW];   // TR: of even and odd chunks
        int lk = 0, whole = 0, bn_load = 0;   // that stage, the stages without a chunk past an end, and its columns
        const int uc = swz(tid / 8, tid % 8) * E;   // NT / 8 rows further on the swizzle is the same
        const uint32_t es = sizeof(T), ldub = (uint32_t)A.ldu * es, ldwb = (uint32_t)(TR ? A.P : A.K) * es;
        using S = TrStage<T, TN, NT>;   // TR
        // The rows of a tile, a thread each, by way of LDS (rows past the last: not stored).
        auto fetch_row = [&](const Tile& q) {
            return tid < TM ? (int32_t)row_of(A.order, q.p0 + (tid < q.rows ? tid : q.rows - 1)) : 0;
        };
        auto point = [&](const Tile& q, const int32_t* rows) {
            ub = static_cast<const char*>(A.U) + (A.order ? 0 : (int64_t)q.p0 * A.ldu * es) + (int64_t)q.k0 * 128;
#pragma unroll
            for (int i = 0; i < NU; ++i)
                uo[i] = (uint32_t)(rows[(i * NT + tid) / 8] - (A.order ? 0 : q.p0)) * ldub + uc * es;
            const char* const W = static_cast<const char*>(A.W) + (int64_t)q.c * A.K * A.P * es;
            if constexpr (TR) {
                wb = W + (int64_t)q.bn * es + (int64_t)q.k0 * BK * ldwb;
#pragma unroll
                for (int i = 0; i < 2; ++i) wo[i] = S::behind(i, tid, ldwb);
            } else {
                wb = W + (int64_t)q.bn * ldwb + (int64_t)q.k0 * 128;
                const int last = A.P - 1 - q.bn;   // columns past it: not stored
#pragma unroll
                for (int i = 0; i < NW; ++i) {
                    const int col = (i * NT + tid) / 8;
                    wo[i] = (uint32_t)(col < last ? col : last) * ldwb + uc * es;
                }
            }
            bn_load = q.bn;
            lk = q.k0;
            if constexpr (TR) whole = S::whole(A.K, A.P);
            else whole = A.K / BK;
        };
        // Chunk i (of NU + NW a thread) of the next stage to LDS; guard: it may lie past an end.
        auto load = [&](int i, char* buf, bool guard) {
            const char* src;
            bool in = true;
            char* to = buf + (i * NT + wave * 64) * 16;   // W's chunks follow U's
            if (i < NU) {
                src = ub + uo[i];
                if (guard) in = lk * BK + uc < A.K;
            } else if constexpr (TR) {
                src = wb + S::above(i - NU, ldwb) + wo[(i - NU) % 2];
                if (guard) in = S::in(i - NU, tid, lk, bn_load, A.K, A.P);
            } else {
                src = wb + wo[i - NU];
                if (guard) in = lk * BK + uc < A.K;
            }
            load_lds16(in ? (const void*)src : (const void*)zero_chunk, to);
        };
        auto load_part = [&](int q, char* buf) {   // of kParts
            constexpr int N = NU + NW;
            if (lk < whole) {
#pragma unroll
                for (int i = q * N / kParts; i < (q + 1) * N / kParts; ++i) load(i, buf, false);
            } else {
#pragma unroll
                for (int i = q * N / kParts; i < (q + 1) * N / kParts; ++i) load(i, buf, true);
            }
            if (q == kParts - 1) {
                ub += 128;
                wb += TR ? (int64_t)BK * ldwb : 128;
                ++lk;
            }
        };
        // 8 bits: the scales of window w of this thread's row of tile q, to registers
        // and from there to LDS.
        uint32_t sv[2] = {0, 0};
        auto fetch_scales = [&](const Tile& q, const int32_t* rows, int w) {
            if constexpr (F8) {
                w += q.k0 / kWindow;   // a part is of whole windows
                const int64_t col = q.bn + tid - TM < A.P ? q.bn + tid - TM : A.P - 1;
                const uint8_t* e = (tid < TM ? A.UE + (int64_t)rows[tid < TM ? tid : 0] * A.nb
                                             : A.WE + ((int64_t)q.c * A.P + col) * A.nb) + w * kWindow;
                const int left = A.nb - w * kWindow;
                if (left >= kWindow) {
                    __builtin_memcpy(sv, e, 8);
                } else {
                    sv[0] = sv[1] = 0x7f7f7f7f;
#pragma unroll
                    for (int x = 0; x < kWindow - 1; ++x)
                        if (x < left) sv[x / 4] = (sv[x / 4] & ~(0xffu << x % 4 * 8)) | (uint32_t)e[x] << x % 4 * 8;
                }
            }
        };
        int window = 0;   // the one in use
        auto put_scales = [&](int b) {
            if constexpr (F8)
                if (tid < TM + TN) __builtin_memcpy(s_scale + (b * (TM + TN) + tid) * kWindow, sv, 8);
        };

        Tile cur = tile_at<T, TN, NT, TR>(A, items, t);
        {
            const int32_t row = fetch_row(cur);
            if (tid < TM) s_rows[tid] = row;
            __syncthreads();
        }
        point(cur, s_rows);
        fetch_scales(cur, s_rows, 0);
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int q = 0; q < kParts; ++q) load_part(q, s_tiles + kt * kStage);
        put_scales(0);

        typename P::Acc acc[FR][FC];
        auto clear = [&]() {
#pragma unroll
            for (int f = 0; f < FR; ++f)
#pragma unroll
                for (int h = 0; h < FC; ++h)
#pragma unroll
                    for (int i = 0; i < 4 * P::kRuns; ++i) acc[f][h][i] = 0.0f;
        };
        // A lane's places in a stage; the second half of a row is 64 bytes off (one
        // bit of the swizzled chunk).
        const int ua = (G::row(0, wr) + li) * 128 + swz(li, P::chunk(lane)) * 16;
        int wa[TR ? FC : 1];
        if constexpr (TR) {
#pragma unroll
            for (int h = 0; h < FC; ++h) wa[h] = TM * 128 + tr_lane<T, CPR>(wc * (TN / WC) + h * 16, lane);
        } else {
            wa[0] = TM * 128 + (wc * (TN / WC) + li) * 128 + swz(li, P::chunk(lane)) * 16;
        }
        // Operands: the rows' are replaced in place, each as soon as its products are
        // under way; the columns' are held twice.
        struct Cols {
            typename P::Frag v[FC];
        };
        typename P::Frag rf[FR];
        uint32_t sa[F8 ? FC : 1], sb[F8 ? FR : 1];   // 8 bits: the scales of four stages, this one's lowest
        auto read_row = [&](int f, const char* buf, int s) {
            rf[f] = P::read(buf, (ua ^ (s * 64)) + (f / FP * kTurn + f % FP * R) * 128);
        };
        auto read_cols = [&](Cols& C, const char* buf, int s) {
            if constexpr (TR) {
                u32x4 v[FC];
                if (s == 0) read_tr_wait<T, CPR, 0>(v, buf, wa);
                else read_tr_wait<T, CPR, KS>(v, buf, wa);
#pragma unroll
                for (int h = 0; h < FC; ++h) C.v[h].v = v[h];
            } else {
#pragma unroll
                for (int h = 0; h < FC; ++h) C.v[h] = P::read(buf, (wa[0] ^ (s * 64)) + h * (R * 128));
            }
        };
        auto read_scales = [&](int kt) {
            if constexpr (F8) {
                if (kt % 4 == 0) {
                    const char* s = s_scale + window * (TM + TN) * kWindow + kt % kWindow;
#pragma unroll
                    for (int h = 0; h < FC; ++h)
                        sa[h] = *reinterpret_cast<const uint32_t*>(s + (TM + wc * (TN / WC) + h * R + li) * kWindow);
#pragma unroll
                    for (int f = 0; f < FR; ++f)
                        sb[f] = *reinterpret_cast<const uint32_t*>(s + (G::row(f, wr) + li) * kWindow);
                } else {
#pragma unroll
                    for (int h = 0; h < FC; ++h) sa[h] >>= 8;
#pragma unroll
                    for (int f = 0; f < FR; ++f) sb[f] >>= 8;
                }
            }
        };
        int live = 0;
        // Loads of a stage, reads of a half stage and the products of the one before
        // are issued in turns, so that the matrix cores do not wait for either: the
        // products of C; C2 and the rows' operands read from buf2 (half s2); the next
        // stage loaded into bufl, if not null.
        auto half = [&](const Cols& C, Cols& C2, const char* buf2, int s2, char* bufl) {
#pragma unroll
            for (int q = 0; q < kParts; ++q) {
                if (bufl) load_part(q, bufl);
                if (!TR && q == 0) read_cols(C2, buf2, s2);
                if (q < live) {
#pragma unroll
                    for (int f = q * FP; f < (q + 1) * FP; ++f)
#pragma unroll
                        for (int h = 0; h < FC; ++h)
                            acc[f][h] = P::mma(C.v[h], rf[f], acc[f][h], (int)sa[F8 ? h : 0], (int)sb[F8 ? f : 0]);
                }
#pragma unroll
                for (int f = q * FP; f < (q + 1) * FP; ++f) read_row(f, buf2, s2);
                __builtin_amdgcn_sched_barrier(0);
                if (TR && q == 0) {   // while the first products are at work
                    read_cols(C2, buf2, s2);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        };
        // Every wave's reads of one stage and its loads of the next have ended.
        auto turn = [&]() {
            __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0) lgkmcnt(0)
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
        Cols C0, C1;
        turn();
#pragma unroll
        for (int f = 0; f < FR; ++f) read_row(f, s_tiles, 0);
        read_cols(C0, s_tiles, 0);
        // Rows of three tiles are in LDS: a wave may write the next tile's while another
        // still reads those of the tile before this one.
        for (int at = 0, slot = 0, ahead = 1;; slot = ahead, ahead = ahead == 2 ? 0 : ahead + 1) {
            const bool more = t + step < x1;
            Tile next = cur;
            int32_t row = 0;
            if (more) {
                next = tile_at<T, TN, NT, TR>(A, items, t + step);
                row = fetch_row(next);
            }
            live = (cur.rows + kTurn - 1) / kTurn;
            clear();
            for (int kt = 0; kt < nk; ++kt, at ^= 1) {
                char* here = s_tiles + at * kStage;
                const char* there = s_tiles + (at ^ 1) * kStage;
                read_scales(kt);
                half(C0, C1, here, 1, nullptr);
                if (kt == 0 && more && tid < TM) s_rows[ahead * TM + tid] = row;
                if constexpr (F8) {
                    // The scales of the next window, asked for a stage before (the next
                    // tile's: with its pointers), go to LDS in the last stage of this one.
                    const bool last = kt + 1 == nk;
                    if (last ? more : (kt + 1) % kWindow == 0) put_scales(window ^= 1);
                }
                turn();
                __builtin_amdgcn_sched_barrier(0);
                if (kt + 2 == nk && more) point(next, s_rows + ahead * TM);
                if constexpr (F8) {
                    if (kt + 2 == nk ? more : (kt + 2) % kWindow == 0 && kt + 2 < nk) {
                        const bool mine = kt + 2 < nk;
                        fetch_scales(mine ? cur : next, s_rows + (mine ? slot : ahead) * TM,
                                     mine ? (kt + 2) / kWindow : 0);
                    }
                }
                // After the last stage the reads are of what the buffer held before, and are not used.
                half(C1, C0, there, 0, kt + 2 < nk || more ? here : nullptr);
            }
#pragma unroll
            for (int f = 0; f < FR; ++f) {
                const int r0 = G::row(f, wr);
                const int64_t col = cur.bn + wc * (TN / WC);
                // Lines of 128 bytes take registers that the largest tile does not have.
                if (TM == 256 || A.splits == 1)
                    put_rows<P, O, TM == 128>(acc[f], col, A.P, lane, [&](int r) {
                        return r0 + r < cur.rows ? static_cast<O*>(A.Y) + (int64_t)s_rows[slot * TM + r0 + r] * A.P
                                                 : nullptr;
                    });
                else if constexpr (TM < 256)   // the largest tile is for products of many
                    put_rows<P, float, false>(acc[f], col, A.P, lane, [&](int r) {
                        return r0 + r < cur.rows ? A.part + (cur.split * A.n + cur.p0 + r0 + r) * A.P : nullptr;
                    });
            }
            if (!more) break;
            t += step;
            cur = next;
        }
    }
    if (A.splits == 1) zero_rows<O>(A, WR * WC);
}

// The same at any address: a tile a block, a stage in registers while the one
// before it is multiplied.  Stages of whole chunks are loaded with no test, the
// others chunk by chunk to their buffer (both in registers would spill).  Eight
// clusters of 512 rows, 1001 to 1003 bf16: 34 us, 33 at 1024 to 1024.
template <class T, class O, int TM, int TN, int WR, int WC, bool TR>
__global__ __launch_bounds__(64 * WR * WC, (kWide<T, O> && TM == 64 ? 4 : 1)) void k_gr_any(MainArgs A) {
    using G = Geo<T, O, TM, TN, WR, WC>;
    using P = typename G::P;
    constexpr bool F8 = sizeof(T) == 1;
    constexpr int E = G::E, R = G::R, KS = G::KS, BK = G::BK, NT = G::NT, FR = G::FR, FC = G::FC, NU = G::NU, NW = G::NW;
    constexpr int CPR = G::CPR, kStage = G::kStage, kParts = G::kParts, FP = G::FP, kTurn = G::kTurn;
    constexpr int kScales = 16;   // 8 bits: stages whose scales are in LDS
    extern __shared__ __align__(16) char s_tiles[];
    uint8_t* s_scale = reinterpret_cast<uint8_t*>(s_tiles + 2 * kStage);   // 8 bits: [TM + TN][kScales]
    int32_t* s_rows = reinterpret_cast<int32_t*>(s_tiles + 2 * kStage + (F8 ? kScales * (TM + TN) : 0));
    const int tid = threadIdx.x, lane = tid & 63, li = lane % R;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wr = wave / WC, wc = wave % WC;
    const int items = __builtin_amdgcn_readfirstlane(A.count[0]);
    const uint32_t block = block_at();
    const int64_t tiles = (int64_t)items * A.tn * A.splits, per = (tiles + 7) / 8, t = block % 8 * per + block / 8;
    if (block / 8 < per && t < tiles) {
        const Tile q = tile_at<T, TN, NT, TR>(A, items, (int)t);
        const int all = (A.K + BK - 1) / BK, end = q.k0 + A.share < all ? q.k0 + A.share : all;
        const int live = (q.rows + kTurn - 1) / kTurn;
        const int64_t ldw = TR ? A.P : A.K;
        const T* const W = static_cast<const T*>(A.W) + (int64_t)q.c * A.K * A.P;
        for (int r = tid; r < TM; r += NT) s_rows[r] = (int32_t)row_of(A.order, q.p0 + (r < q.rows ? r : q.rows - 1));
        __syncthreads();
        const int uc = swz(tid / 8, tid % 8) * E;
        // Where chunk i of a stage (NU + NW a thread) begins: its row, at stage 0.
        auto from = [&](int i) -> const T* {
            const int x = i * NT + tid;
            if (i < NU) return static_cast<const T*>(A.U) + (int64_t)s_rows[x / 8] * A.ldu;
            const int y = x - NU * NT;
            if constexpr (TR) return W + (int64_t)(y / CPR) * ldw;
            return W + (q.bn + y / 8 < A.P ? q.bn + y / 8 : A.P - 1) * ldw;
        };
        const T* p[NU + NW];
#pragma unroll
        for (int i = 0; i < NU + NW; ++i) {
            p[i] = from(i);
            if (TR && i >= NU) {
                const int y = (i - NU) * NT + tid;
                p[i] += (int64_t)q.k0 * BK * ldw + q.bn + swz_tr<T, CPR>(y / CPR, y % CPR) * E;
            } else {
                p[i] += (int64_t)q.k0 * BK + uc;
            }
        }
        // Stages without a chunk past the contraction's end or the last column.
        int whole;
        if constexpr (TR) whole = TrStage<T, TN, NT>::whole(A.K, A.P);
        else whole = A.K / BK;
        typedef u32x4 __attribute__((aligned(1))) any4;
        u32x4 v[NU + NW];
        bool held = false;   // the stage is in v, else in its buffer already
        auto fetch = [&](int kt, char* buf) {
            held = kt < whole;
            if (held) {
#pragma unroll
                for (int i = 0; i < NU + NW; ++i) {
                    v[i] = *reinterpret_cast<const any4*>(p[i]);
                    p[i] += TR && i >= NU ? (int64_t)BK * ldw : BK;
                }
                return;
            }
#pragma unroll 1
            for (int i = 0; i < NU + NW; ++i) {
                u32x4 o;
                if (!TR || i < NU) {
                    o = chunk_any(from(i), (int64_t)kt * BK + uc, A.K);
                } else {
                    const int y = (i - NU) * NT + tid, kk = y / CPR;
                    const bool in = kt * BK + kk < A.K;
                    o = only_if(in, chunk_any(in ? from(i) + (int64_t)kt * BK * ldw : W,
                                              q.bn + swz_tr<T, CPR>(kk, y % CPR) * E, A.P));
                }
                *reinterpret_cast<u32x4*>(buf + (i * NT + tid) * 16) = o;
            }
        };

        // 8 bits: the scales of the stages from k0 on, a row a thread.
        auto scales = [&](int k0) {
            if constexpr (F8) {
                for (int r = tid; r < TM + TN; r += NT) {
                    const uint8_t* e;
                    if (r < TM) {
                        e = A.UE + row_of(A.order, q.p0 + (r < q.rows ? r : q.rows - 1)) * A.nb;
                    } else {
                        const int64_t col = q.bn + r - TM < A.P ? q.bn + r - TM : A.P - 1;
                        e = A.WE + ((int64_t)q.c * A.P + col) * A.nb;
                    }
#pragma unroll
                    for (int x = 0; x < kScales; ++x)
                        if (k0 + x < A.nb) s_scale[r * kScales + x] = e[k0 + x];
                }
            }
        };
        typename P::Acc acc[FR][FC];
#pragma unroll
        for (int f = 0; f < FR; ++f)
#pragma unroll
            for (int h = 0; h < FC; ++h)
#pragma unroll
                for (int i = 0; i < 4 * P::kRuns; ++i) acc[f][h][i] = 0.0f;
        const int ua = (G::row(0, wr) + li) * 128 + swz(li, P::chunk(lane)) * 16;
        int wa[TR ? FC : 1];
        if constexpr (TR) {
#pragma unroll
            for (int h = 0; h < FC; ++h) wa[h] = TM * 128 + tr_lane<T, CPR>(wc * (TN / WC) + h * 16, lane);
        } else {
            wa[0] = TM * 128 + (wc * (TN / WC) + li) * 128 + swz(li, P::chunk(lane)) * 16;
        }
        scales(q.k0);
        int at = 0;
        fetch(q.k0, s_tiles);
        for (int kt = q.k0; kt < end; ++kt, at ^= 1) {
            char* buf = s_tiles + at * kStage;
            if (held) {
#pragma unroll
                for (int i = 0; i < NU + NW; ++i) *reinterpret_cast<u32x4*>(buf + (i * NT + tid) * 16) = v[i];
            }
            __syncthreads();
            if (kt + 1 < end) fetch(kt + 1, s_tiles + (at ^ 1) * kStage);
            int sa[F8 ? FC : 1], sb[F8 ? FR : 1];
            if constexpr (F8) {
                const uint8_t* cols = s_scale + (TM + wc * (TN / WC)) * kScales + (kt - q.k0) % kScales;
#pragma unroll
                for (int h = 0; h < FC; ++h) sa[h] = cols[(h * R + li) * kScales];
#pragma unroll
                for (int f = 0; f < FR; ++f) sb[f] = s_scale[(G::row(f, wr) + li) * kScales + (kt - q.k0) % kScales];
                if constexpr (kWide<T, O>) {   // a stage is a block
                    typename P::Wide a[2][FC];
                    int sr[FC][4];   // of the columns of a lane's results
#pragma unroll
                    for (int h = 0; h < FC; ++h) {
#pragma unroll
                        for (int s = 0; s < 2; ++s)
                            a[s][h] = P::wide(P::read(buf, (wa[0] ^ (s * 64)) + h * (R * 128)), sa[h]);
#pragma unroll
                        for (int i = 0; i < 4; ++i) sr[h][i] = cols[(h * R + P::run(0, lane) + i) * kScales];
                    }
#pragma unroll
                    for (int f = 0; f < FR; ++f) {
                        if (f / FP >= live) continue;
                        typename P::Wide b[2];
#pragma unroll
                        for (int s = 0; s < 2; ++s)
                            b[s] = P::wide(P::read(buf, (ua ^ (s * 64)) + (f / FP * kTurn + f % FP * R) * 128), sb[f]);
#pragma unroll
                        for (int h = 0; h < FC; ++h) {
                            typename P::Acc v{0, 0, 0, 0};
#pragma unroll
                            for (int s = 0; s < 2; ++s) v = P::mma(a[s][h], b[s], v);
                            P::add_scaled(acc[f][h], v, sr[h], sb[f]);
                        }
                    }
                }
            }
            if constexpr (!kWide<T, O>) {
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    typename P::Frag b[FR], a[FC];
#pragma unroll
                    for (int f = 0; f < FR; ++f) b[f] = P::read(buf, (ua ^ (s * 64)) + (f / FP * kTurn + f % FP * R) * 128);
                    if constexpr (TR) {
                        u32x4 x[FC];
                        if (s == 0) read_tr_wait<T, CPR, 0>(x, buf, wa);
                        else read_tr_wait<T, CPR, KS>(x, buf, wa);
#pragma unroll
                        for (int h = 0; h < FC; ++h) a[h].v = x[h];
                    } else {
#pragma unroll
                        for (int h = 0; h < FC; ++h) a[h] = P::read(buf, (wa[0] ^ (s * 64)) + h * (R * 128));
                    }
#pragma unroll
                    for (int p = 0; p < kParts; ++p) {
                        if (p >= live) continue;
#pragma unroll
                        for (int f = p * FP; f < (p + 1) * FP; ++f)
#pragma unroll
                            for (int h = 0; h < FC; ++h)
                                acc[f][h] = P::mma(a[h], b[f], acc[f][h], sa[F8 ? h : 0], sb[F8 ? f : 0]);
                    }
                }
            }
            if (F8 && (kt + 1 - q.k0) % kScales == 0 && kt + 1 < end) {
                __syncthreads();
                scales(kt + 1);
            }
        }
#pragma unroll
        for (int f = 0; f < FR; ++f) {
            const int r0 = G::row(f, wr);
            const int64_t col = q.bn + wc * (TN / WC);
            if (A.splits == 1)
                put_rows<P, O, false>(acc[f], col, A.P, lane, [&](int r) {
                    return r0 + r < q.rows ? static_cast<O*>(A.Y) + (int64_t)s_rows[r0 + r] * A.P : nullptr;
                });
            else
                put_rows<P, float, false>(acc[f], col, A.P, lane, [&](int r) {
                    return r0 + r < q.rows ? A.part + (q.split * A.n + q.p0 + r0 + r) * A.P : nullptr;
                });
        }
    }
    if (A.splits == 1) zero_rows<O>(A, WR * WC);
}

// The parts of the contraction, added in order: a block a place and 1024 columns.
// Bound by the parts' bytes, which the last-level cache holds where there are parts.
template <class O>
__global__ __launch_bounds__(256) void k_gr_sum(MainArgs A) {
    const int64_t place = blockIdx.x, col = ((int64_t)blockIdx.y * 256 + threadIdx.x) * 4, step = A.n * A.P;
    if (col >= A.P) return;
    f32x4 v{0, 0, 0, 0};
    if (place < A.used[0]) {
        const float* p = A.part + place * A.P + col;
        if (col + 4 <= A.P) {
#pragma unroll 4
            for (int q = 0; q < A.splits; ++q) {
                f32x4 x;
                __builtin_memcpy(&x, p + q * step, 16);
                v += x;
            }
        } else {
            for (int q = 0; q < A.splits; ++q)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (col + i < A.P) v[i] += p[q * step + i];
        }
    }
    put4(static_cast<O*>(A.Y) + row_of(A.order, place) * A.P, col, A.P, v);
}

// --------------------------------------------------------------------------
// dW_c = sum over c's places of V[row] U[row]^T: both operands hold the
// contraction along their rows and are read transposed.

struct GradArgs {
    const void *U, *V;       // X (P wide) and dY (Q wide)
    int64_t ldu, ldv;
    const int32_t *order, *count;
    const GroupItem* items;
    const int32_t *first, *num;
    void* out;               // k x Q x P
    float* part;             // slots x Q x P
    int32_t k, P, Q;
    int32_t tq, tp;          // tiles
};

// An item's tile: V's columns from bm, U's from bn.
struct GradTile {
    int c, p0, p1, slot, bm, bn;
};
template <int TM, int TN>
__device__ __forceinline__ GradTile grad_tile_at(const GradArgs& A, int64_t t) {
    const int each = A.tq * A.tp;
    const int64_t item = t / each;
    const GroupItem it = item_at(A.items, item);
    // Down 4 tiles of V's columns before the next of U's.
    const int in = (int)(t - item * each), group = 4 * A.tp, grp = in / group, m0 = grp * 4, at = in - grp * group;
    const int gm = A.tq - m0 < 4 ? A.tq - m0 : 4;
    return GradTile{it.c, it.p0, it.p1, it.slot, (m0 + at % gm) * TM, at / gm * TN};
}
// The j-th tile of an XCD: eight consecutive ones go to one, the next eight to the
// next, so that all share the tiles of a long cluster.
__device__ __forceinline__ int64_t grad_index(int64_t j, uint32_t block) { return (j / 8 * 8 + block % 8) * 8 + j % 8; }

template <class T, int TM, int TN, int WR, int WC>
__device__ __forceinline__ void grad_put(const GradArgs& A, const GradTile& q,
                                         const f32x4 (&acc)[TM / WR / 16][TN / WC / 16], int wr, int wc, int lane) {
    const int64_t slot = q.slot < 0 ? q.c : q.slot, col = q.bn + wc * (TN / WC);
#pragma unroll
    for (int f = 0; f < TM / WR / 16; ++f) {
        const int64_t r0 = q.bm + wr * (TM / WR) + f * 16;
        auto to = [&](auto* out) {
            return [=, &A](int r) { return r0 + r < A.Q ? out + (slot * A.Q + r0 + r) * A.P : nullptr; };
        };
        if (q.slot < 0) put_rows<Op<T, T>, T, true>(acc[f], col, A.P, lane, to(static_cast<T*>(A.out)));
        else put_rows<Op<T, T>, float, false>(acc[f], col, A.P, lane, to(A.part));
    }
}

// Blocks stay and take tile after tile, two stages of 128 bytes a column being on
// their way or in LDS, as in k_gr_main: a tile has few stages where clusters are
// short, and what it starts and ends with is what they would wait for.
//
// Bound by its loads' and stores' latency: 16,384 rows in 64 skewed clusters, 2048 x
// 2048 bf16, 327 us (403 MB read, 537 written, 2.9 TB/s; 219 with no results
// written); four clusters of 4096, 4096 x 4096, 600 us (915 TFLOP/s).  Tiles of 128
// x 128, two a compute unit, took 385 us for the 327: twice the reads.  They stay for
// small weights, whose tiles would not fill the chip.
template <class T, int TM, int TN, int WR, int WC>
__global__ __launch_bounds__(64 * WR * WC, 2) void k_gr_grad(GradArgs A) {
    constexpr int E = Mma<T>::E, KS = 4 * E, BK = 2 * KS, NT = 64 * WR * WC, es = sizeof(T);
    constexpr int FR = TM / WR / 16, FC = TN / WC / 16;
    constexpr int CPR = TM / E, kDown = NT / CPR, N = BK / kDown;   // chunks a place; places from one chunk of a
                                                                    // thread to its next; a thread's of a stage
    constexpr int kStage = (TM + TN) * 128;
    static_assert(TM == TN && FR % 4 == 0 && FC % 2 == 0 && kDown % 8 == 0, "");
    extern __shared__ __align__(16) char s_tiles[];   // two stages: V, then U
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wr = wave / WC, wc = wave % WC;
    const int64_t tiles = (int64_t)__builtin_amdgcn_readfirstlane(A.count[0]) * A.tq * A.tp, step = gridDim.x / 8;
    int64_t j = blockIdx.x / 8;
    if (grad_index(j, blockIdx.x) >= tiles) return;
    // This tile and the three after it (of no places where there are none).
    auto tile = [&](int64_t x) {
        const int64_t t = grad_index(x, blockIdx.x);
        return t < tiles ? grad_tile_at<TM, TN>(A, t) : GradTile{0, 0, 0, 0, 0, 0};
    };
    GradTile q0 = tile(j), q1 = tile(j + step), q2 = tile(j + 2 * step), q3 = tile(j + 3 * step);

    // The next stage to load: places lp .. of tile L, the ahead-th after this one.
    GradTile L = q0;
    int lp = L.p0, ahead = 0;
    int32_t row[N];
    const int kk = tid / CPR;
    // The column of even and odd chunks (16 places further on the swizzle is the same).
    const uint32_t colb[2] = {(uint32_t)swz_tr<T, CPR>(kk, tid % CPR) * 16,
                              (uint32_t)swz_tr<T, CPR>(kDown + kk, tid % CPR) * 16};
    const uint32_t ldub = (uint32_t)A.ldu * es, ldvb = (uint32_t)A.ldv * es;
    auto rows = [&]() {   // of that stage, behind the bases of load()
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int p = lp + i * kDown + kk < L.p1 ? lp + i * kDown + kk : L.p0;
            row[i] = A.order ? A.order[p] : p - L.p0;
        }
    };
    auto load = [&](char* buf) {
        const int64_t base = A.order ? 0 : L.p0;
        const char* v = static_cast<const char*>(A.V) + (base * A.ldv + L.bm) * es;
        const char* u = static_cast<const char*>(A.U) + (base * A.ldu + L.bn) * es;
        char* to = buf + wave * 1024;
        if (lp + BK <= L.p1 && L.bm + TM <= A.Q && L.bn + TN <= A.P) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                load_lds16(v + (uint32_t)((uint32_t)row[i] * ldvb + colb[i % 2]), to + i * (NT * 16));
#pragma unroll
            for (int i = 0; i < N; ++i)
                load_lds16(u + (uint32_t)((uint32_t)row[i] * ldub + colb[i % 2]), to + TM * 128 + i * (NT * 16));
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const bool in = lp + i * kDown + kk < L.p1;
                const int c = (int)colb[i % 2] / es;
                const char* a = v + (uint32_t)((uint32_t)row[i] * ldvb + colb[i % 2]);
                const char* b = u + (uint32_t)((uint32_t)row[i] * ldub + colb[i % 2]);
                load_lds16(in && L.bm + c < A.Q ? (const void*)a : (const void*)zero_chunk, to + i * (NT * 16));
                load_lds16(in && L.bn + c < A.P ? (const void*)b : (const void*)zero_chunk, to + TM * 128 + i * (NT * 16));
            }
        }
        lp += BK;
        if (lp >= L.p1) {
            ++ahead;
            auto pick = [&](int a, int b, int c) { return ahead == 1 ? a : ahead == 2 ? b : c; };
            L = GradTile{pick(q1.c, q2.c, q3.c),    pick(q1.p0, q2.p0, q3.p0), pick(q1.p1, q2.p1, q3.p1),
                         pick(q1.slot, q2.slot, q3.slot), pick(q1.bm, q2.bm, q3.bm), pick(q1.bn, q2.bn, q3.bn)};
            lp = L.p0;
        }
        if (L.p1 > L.p0) rows();
    };
    rows();
    load(s_tiles);
    if (L.p1 > L.p0) load(s_tiles + kStage);
    int va[FR], ua[FC];
#pragma unroll
    for (int f = 0; f < FR; ++f) va[f] = tr_lane<T, CPR>(wr * (TM / WR) + f * 16, lane);
#pragma unroll
    for (int h = 0; h < FC; ++h) ua[h] = TM * 128 + tr_lane<T, CPR>(wc * (TN / WC) + h * 16, lane);
    auto turn = [&]() {
        __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0) lgkmcnt(0)
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    turn();
    for (int at = 0;;) {
        f32x4 acc[FR][FC];
#pragma unroll
        for (int f = 0; f < FR; ++f)
#pragma unroll
            for (int h = 0; h < FC; ++h) acc[f][h] = f32x4{0, 0, 0, 0};
        for (int p = q0.p0; p < q0.p1; p += BK, at ^= 1) {
            char* buf = s_tiles + at * kStage;
            auto half = [&](auto s) {
                constexpr int K0 = decltype(s)::value;
                u32x4 a[FC];
#pragma unroll
                for (int h = 0; h < FC; h += 2) {
                    u32x4 v[2];
                    const int q[2] = {ua[h], ua[h + 1]};
                    read_tr_wait<T, CPR, K0>(v, buf, q);
                    a[h] = v[0], a[h + 1] = v[1];
                }
#pragma unroll
                for (int f = 0; f < FR; f += 4) {
                    u32x4 b[4];
                    const int q[4] = {va[f], va[f + 1], va[f + 2], va[f + 3]};
                    read_tr_wait<T, CPR, K0>(b, buf, q);
                    if (K0 != 0 && f + 4 == FR) {
                        // All of the stage is in registers or multiplied: once every wave is
                        // here, and the next stage has landed, the one behind it may come.
                        turn();
                        if (L.p1 > L.p0) load(buf);
                        __builtin_amdgcn_sched_barrier(0);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int h = 0; h < FC; ++h) acc[f + i][h] = Mma<T>::mma(a[h], b[i], acc[f + i][h]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
            half(std::integral_constant<int, 0>{});
            half(std::integral_constant<int, KS>{});
        }
        grad_put<T, TM, TN, WR, WC>(A, q0, acc, wr, wc, lane);
        if (q1.p1 <= q1.p0) break;
        j += step;
        q0 = q1, q1 = q2, q2 = q3;
        q3 = tile(j + 3 * step);
        --ahead;
    }
}

// The same at any address: a tile a block, a stage in registers while the one
// before it is multiplied.  Eight clusters of 512 rows, 1001 x 1003 bf16: 53 us, 44
// at 1024 x 1024 with k_gr_grad.
template <class T, int TM, int TN, int WR, int WC>
__global__ __launch_bounds__(64 * WR * WC, 2) void k_gr_grad_any(GradArgs A) {
    constexpr int E = Mma<T>::E, KS = 4 * E, BK = 2 * KS, NT = 64 * WR * WC;
    constexpr int FR = TM / WR / 16, FC = TN / WC / 16;
    constexpr int CPR = TM / E, N = BK * CPR / NT;
    constexpr int kStage = (TM + TN) * 128;
    static_assert(TM == TN && FR % 4 == 0 && FC % 4 == 0, "");
    extern __shared__ __align__(16) char s_tiles[];   // two stages: V, then U
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wr = wave / WC, wc = wave % WC;
    const uint32_t block = block_at();
    const int64_t tiles = (int64_t)__builtin_amdgcn_readfirstlane(A.count[0]) * A.tq * A.tp;
    const int64_t t = grad_index(block / 8, block);
    if (t >= tiles) return;
    GradTile q = grad_tile_at<TM, TN>(A, t);
    // The last tile of a width that TM does not divide moves left until it is whole: it and
    // its neighbour then write the same values.
    const bool wide = A.Q >= TM && A.P >= TN;
    if (wide) {
        q.bm = q.bm < A.Q - TM ? q.bm : A.Q - TM;
        q.bn = q.bn < A.P - TN ? q.bn : A.P - TN;
    }
    int32_t row[N];   // of the next stage to load; behind the last, the first once more
    auto rows = [&](int p) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int x = p + (i * NT + tid) / CPR;
            row[i] = (int32_t)row_of(A.order, x < q.p1 ? x : q.p0);
        }
    };
    typedef u32x4 __attribute__((aligned(1))) any4;
    u32x4 v[2 * N];   // wide: the stage on its way, else it goes to its buffer at once
    auto load = [&](int p, char* buf) {
        if (wide) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int x = i * NT + tid, c = swz_tr<T, CPR>(x / CPR, x % CPR) * E;
                v[i] = *reinterpret_cast<const any4*>(static_cast<const T*>(A.V) + row[i] * A.ldv + (q.bm + c));
                v[N + i] = *reinterpret_cast<const any4*>(static_cast<const T*>(A.U) + row[i] * A.ldu + (q.bn + c));
            }
            return;
        }
#pragma unroll 1
        for (int i = 0; i < 2 * N; ++i) {
            const bool first = i < N;
            const int x = (first ? i : i - N) * NT + tid, k = x / CPR, c = swz_tr<T, CPR>(k, x % CPR) * E;
            const bool in = p + k < q.p1;
            const int64_t r = row_of(A.order, in ? p + k : q.p0);
            const u32x4 o = first ? chunk_any(static_cast<const T*>(A.V) + r * A.ldv, q.bm + c, A.Q)
                                  : chunk_any(static_cast<const T*>(A.U) + r * A.ldu, q.bn + c, A.P);
            *reinterpret_cast<u32x4*>(buf + (first ? 0 : TM * 128) + x * 16) = only_if(in, o);
        }
    };
    int va[FR], ua[FC];
#pragma unroll
    for (int f = 0; f < FR; ++f) va[f] = tr_lane<T, CPR>(wr * (TM / WR) + f * 16, lane);
#pragma unroll
    for (int h = 0; h < FC; ++h) ua[h] = TM * 128 + tr_lane<T, CPR>(wc * (TN / WC) + h * 16, lane);
    f32x4 acc[FR][FC];
#pragma unroll
    for (int f = 0; f < FR; ++f)
#pragma unroll
        for (int h = 0; h < FC; ++h) acc[f][h] = f32x4{0, 0, 0, 0};
    rows(q.p0);
    load(q.p0, s_tiles);
    rows(q.p0 + BK);
    int at = 0;
    for (int p = q.p0; p < q.p1; p += BK, at ^= 1) {
        char* buf = s_tiles + at * kStage;
        if (wide) {
#pragma unroll
            for (int i = 0; i < 2 * N; ++i) {
                const int x = i % N * NT + tid;
                *reinterpret_cast<u32x4*>(buf + (i < N ? 0 : TM * 128) + x * 16) = only_if(p + x / CPR < q.p1, v[i]);
            }
        }
        __syncthreads();
        if (p + BK < q.p1) {
            load(p + BK, s_tiles + (at ^ 1) * kStage);
            rows(p + 2 * BK);
        }
        auto half = [&](auto s) {
            constexpr int K0 = decltype(s)::value;
            u32x4 a[FC];
            read_tr_wait<T, CPR, K0>(a, buf, ua);
#pragma unroll
            for (int f = 0; f < FR; f += 4) {
                u32x4 b[4];
                const int y[4] = {va[f], va[f + 1], va[f + 2], va[f + 3]};
                read_tr_wait<T, CPR, K0>(b, buf, y);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int h = 0; h < FC; ++h) acc[f + i][h] = Mma<T>::mma(a[h], b[i], acc[f + i][h]);
            }
        };
        half(std::integral_constant<int, 0>{});
        half(std::integral_constant<int, KS>{});
    }
    grad_put<T, TM, TN, WR, WC>(A, q, acc, wr, wc, lane);
}

// Clusters of no chunk: zeros; of several: the sum of their parts in order.  16
// bytes a lane, past the caches.  4 us where there is nothing to join.
template <class T>
__global__ __launch_bounds__(256) void k_gr_join(GradArgs A) {
    constexpr int E = 16 / (int)sizeof(T);
    const int64_t size = (int64_t)A.Q * A.P, step = (int64_t)gridDim.x * 256 * E;
    const int64_t first = ((int64_t)blockIdx.x * 256 + threadIdx.x) * E;
    for (int c = blockIdx.y; c < A.k; c += gridDim.y) {
        const int num = A.num[c];
        if (num == 1) continue;
        const float* part = A.part + A.first[c] * size;
        T* out = static_cast<T*>(A.out) + c * size;
        for (int64_t i = first; i < size; i += step) {
            float v[E] = {};
            if (i + E <= size) {
#pragma unroll 4
                for (int q = 0; q < num; ++q) {
                    float x[E];
                    __builtin_memcpy(x, part + q * size + i, sizeof(x));
#pragma unroll
                    for (int e = 0; e < E; ++e) v[e] += x[e];
                }
                Vec<T, E> o;
#pragma unroll
                for (int e = 0; e < E; ++e) o.e[e] = from_f32<T>(v[e]);
                typedef u32x4 __attribute__((aligned(2))) any4;
                __builtin_nontemporal_store(__builtin_bit_cast(u32x4, o), reinterpret_cast<any4*>(out + i));
            } else {
                for (int e = 0; i + e < size; ++e) {
                    float x = 0.0f;
                    for (int q = 0; q < num; ++q) x += part[q * size + i + e];
                    out[i + e] = from_f32<T>(x);
                }
            }
        }
    }
}

// --------------------------------------------------------------------------
// Few rows, forward: the time is that of reading the experts in use once.

struct FewArgs {
    const void* U;
    int64_t ldu;
    const void* W;
    const uint8_t *UE, *WE;
    const int32_t *order, *sids, *offsets;
    void* Y;
    int32_t n, k, K, P, nb;
};

// 16 columns and the places of one cluster a block, from the place blockIdx.y on
// if a cluster starts there; its NWAVE waves share the contraction, some four steps
// each.  No list and no workspace: one launch.  48 rows of 4096, 100 clusters, 4096
// columns in 8 bits: 128 us, the rate of a copy; 48 rows of 48 such clusters f16 296 us
// (5.4 TB/s), float32 620 (5.2), 8 bits 171 and with float32 results 191; 32 rows of
// 1024, 8 clusters, bf16: 7 us.
template <class T, class O>
struct FewOp {
    static constexpr int kBytes = 16;   // of a row a lane and step
    using Frag = typename Op<T, O>::Frag;
    static __device__ __forceinline__ f32x4 mma(const Frag& a, const Frag& b, f32x4 c, int sa, int sb) {
        return Op<T, O>::mma(a, b, c, sa, sb);
    }
};
template <class O>
struct FewOp<uint8_t, O> {
    static constexpr int kBytes = 32;
    using Frag = typename Op<uint8_t, O>::Frag;
    static __device__ __forceinline__ f32x4 mma(const Frag& a, const Frag& b, f32x4 c, int sa, int sb) {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(__builtin_bit_cast(i32x8, a),
                                                                __builtin_bit_cast(i32x8, b), c, 0, 0, 0, sa, 0, sb);
    }
};
template <>
struct FewOp<uint8_t, float> {
    static constexpr int kBytes = 16;
    using Q = Op<uint8_t, float>;
    using Frag = Q::Frag;
    // The products of B steps of one block, with the bytes of the lane's column and row.
    template <int B>
    static __device__ __forceinline__ void add(f32x4& c, const Frag* a, const Frag (&b)[B], int sa, int sb) {
        f32x4 v{0, 0, 0, 0};
#pragma unroll
        for (int z = 0; z < B; ++z) v = Q::mma(Q::wide(a[z], sa), Q::wide(b[z], sb), v);
        int cols[4];   // the lane's results are of four other columns
#pragma unroll
        for (int i = 0; i < 4; ++i) cols[i] = __shfl(sa, (threadIdx.x & 48) + Q::run(0, threadIdx.x & 63) + i);
        Q::add_scaled(c, v, cols, sb);
    }
};

template <class T, class O, bool AL, int NWAVE, int RF>
__device__ __forceinline__ void few_block(const FewArgs& A, int c, int p0, int rows, f32x4 (*s_red)[4][64]) {
    using P = FewOp<T, O>;
    constexpr bool F8 = sizeof(T) == 1;
    constexpr int EL = P::kBytes / (int)sizeof(T), KS = 4 * EL;   // elements a lane, of a step
    constexpr int UN = (RF <= 2 ? 4 : 2) / (F8 && RF == 4 ? 2 : AL ? 1 : 2);
    const int lane = threadIdx.x & 63, g = lane >> 4, li = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t col0 = (int64_t)blockIdx.x * 16;
    const int64_t col = (int64_t)c * A.P + (col0 + li < A.P ? col0 + li : A.P - 1);   // columns past P: not stored
    const T* w = static_cast<const T*>(A.W) + col * A.K;
    const uint8_t* we = F8 ? A.WE + col * A.nb : nullptr;
    const T* x[RF];
    const uint8_t* xe[RF];
#pragma unroll
    for (int f = 0; f < RF; ++f) {
        const int r = f * 16 + li;
        const int64_t row = row_of(A.order, p0 + (r < rows ? r : rows - 1));
        x[f] = static_cast<const T*>(A.U) + row * A.ldu;
        if constexpr (F8) xe[f] = A.UE + row * A.nb;
    }
    f32x4 acc[RF];
#pragma unroll
    for (int f = 0; f < RF; ++f) acc[f] = f32x4{0, 0, 0, 0};
    auto get = [&](const T* row, int64_t k0) {
        typename P::Frag o;
        if constexpr (AL) {
            o.v = *(k0 < A.K ? reinterpret_cast<const u32x4*>(row + k0) : reinterpret_cast<const u32x4*>(zero_chunk));
            if constexpr (P::kBytes == 32)
                o.w = *(k0 + 16 < A.K ? reinterpret_cast<const u32x4*>(row + k0 + 16)
                                      : reinterpret_cast<const u32x4*>(zero_chunk));
        } else {
            o.v = chunk_any(row, k0, A.K);
            if constexpr (P::kBytes == 32) o.w = chunk_any(row, k0 + 16, A.K);
        }
        return o;
    };
    const int steps = (A.K + KS - 1) / KS;
    for (int s = wave * UN; s < steps; s += NWAVE * UN) {   // steps past the last are of zeros
        typename P::Frag a[UN], b[UN][RF];
        int sa[UN], sb[UN][RF];
#pragma unroll
        for (int y = 0; y < UN; ++y) {
            const int64_t k0 = (int64_t)(s + y) * KS + g * EL;
            a[y] = get(w, k0);
#pragma unroll
            for (int f = 0; f < RF; ++f) b[y][f] = get(x[f], k0);
            if constexpr (F8) {   // KS: 64 or 128
                const int at = (s + y) / (128 / KS), e = at < A.nb ? at : 0;
                sa[y] = we[e];
#pragma unroll
                for (int f = 0; f < RF; ++f) sb[y][f] = xe[f][e];
            }
        }
        __builtin_amdgcn_sched_barrier(0);   // all of them are issued before the first is waited for
        if constexpr (kWide<T, O>) {
            constexpr int B = UN % 2 == 0 ? 2 : 1;   // two steps are a block
#pragma unroll
            for (int y = 0; y < UN; y += B)
#pragma unroll
                for (int f = 0; f < RF; ++f) {
                    typename P::Frag rows[B];
#pragma unroll
                    for (int z = 0; z < B; ++z) rows[z] = b[y + z][f];
                    P::add(acc[f], a + y, rows, sa[y], sb[y][f]);
                }
        } else {
#pragma unroll
            for (int y = 0; y < UN; ++y)
#pragma unroll
                for (int f = 0; f < RF; ++f) acc[f] = P::mma(a[y], b[y][f], acc[f], F8 ? sa[y] : 0, F8 ? sb[y][f] : 0);
        }
    }
    // The waves' sums: the upper half's to the lower half, then in order.
    constexpr int H = NWAVE / 2;
    if (wave >= H)
#pragma unroll
        for (int q = 0; q < RF; ++q) s_red[wave - H][q][lane] = acc[q];
    __syncthreads();
    if (wave < H)
#pragma unroll
        for (int q = 0; q < RF; ++q) s_red[wave][q][lane] += acc[q];
    __syncthreads();
    for (int q = wave; q < RF; q += NWAVE) {
        const int r = q * 16 + li;
        if (r >= rows) continue;
        f32x4 v{0, 0, 0, 0};
#pragma unroll
        for (int y = 0; y < H; ++y) v += s_red[y][q][lane];
        put4(static_cast<O*>(A.Y) + row_of(A.order, p0 + r) * A.P, col0 + g * 4, A.P, v);
    }
}

template <class T, class O, bool AL, int NWAVE>
__global__ __launch_bounds__(64 * NWAVE, 4) void k_gr_few(FewArgs A) {
    __shared__ f32x4 s_red[NWAVE / 2][4][64];
    const int p = blockIdx.y, c = __builtin_amdgcn_readfirstlane(A.sids[p]);
    if (p > 0 && A.sids[p - 1] == c) return;   // not the first place of its cluster
    if (c < 0) {                               // rows of no cluster
        const int64_t col0 = (int64_t)blockIdx.x * 16;
        for (int q = threadIdx.x; q < (A.n - p) * 16; q += 64 * NWAVE)
            if (col0 + q % 16 < A.P)
                static_cast<O*>(A.Y)[row_of(A.order, p + q / 16) * A.P + col0 + q % 16] = from_f32<O>(0.0f);
        return;
    }
    const int rows = __builtin_amdgcn_readfirstlane(A.offsets[c + 1]) - p;
    if (rows <= 16) few_block<T, O, AL, NWAVE, 1>(A, c, p, rows, s_red);
    else if (rows <= 32) few_block<T, O, AL, NWAVE, 2>(A, c, p, rows, s_red);
    else few_block<T, O, AL, NWAVE, 4>(A, c, p, rows, s_red);
}

// --------------------------------------------------------------------------
// Launches

template <class K>
hipError_t raise_lds(K* kernel, int bytes) {
    return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

constexpr int kCus = 256;

// A grid of at least `blocks` blocks, which block_at numbers; of 2^20 in the first
// dimension where they are more (512 threads of a block: 2^29).
dim3 many_blocks(int64_t blocks) {
    constexpr int64_t kMost = 1 << 20;
    if (blocks <= kMost) return dim3((unsigned)blocks);
    return dim3((unsigned)kMost, (unsigned)((blocks + kMost - 1) / kMost));
}

// Stages of one of `splits` parts of `all` stages: whole windows of scales in 8 bits.
int part_stages(int all, int splits, bool f8) {
    const int share = (all + splits - 1) / splits;
    return splits > 1 && f8 ? (share + 7) / 8 * 8 : share;
}

bool a16(const void* p) { return ((uintptr_t)p & 15) == 0; }

template <class T, class O, int TM, int TN, int WR, int WC, bool TR>
hipError_t main_tile(MainArgs A, int64_t max_items, hipStream_t s) {
    A.tn = (A.P + TN - 1) / TN;
    constexpr int lds = 2 * (TM + TN) * 128 + (sizeof(T) == 1 ? 2 * kWindow * (TM + TN) : 0) + 3 * TM * 4;
    static_assert(lds <= 160 * 1024, "");
    if (lds > 65536) {
        const hipError_t e = raise_lds(k_gr_main<T, O, TM, TN, WR, WC, TR>, lds);
        if (e != hipSuccess) return e;
    }
    // As many blocks as the chip holds at once.
    const int64_t tiles = (max_items * A.tn * A.splits + 7) / 8 * 8, most = kCus * (TM == 256 ? 1 : TM == 128 ? 2 : 4);
    hipLaunchKernelGGL((k_gr_main<T, O, TM, TN, WR, WC, TR>), dim3((unsigned)(tiles < most ? tiles : most)),
                       dim3(64 * WR * WC), lds, s, A);
    return hipGetLastError();
}

template <class T, class O, int TM, int TN, int WR, int WC, bool TR>
hipError_t any_tile(MainArgs A, int64_t max_items, hipStream_t s) {
    A.tn = (A.P + TN - 1) / TN;
    constexpr int lds = 2 * (TM + TN) * 128 + (sizeof(T) == 1 ? 16 * (TM + TN) : 0) + TM * 4;
    if (lds > 65536) {
        const hipError_t e = raise_lds(k_gr_any<T, O, TM, TN, WR, WC, TR>, lds);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((k_gr_any<T, O, TM, TN, WR, WC, TR>), many_blocks((max_items * A.tn * A.splits + 7) / 8 * 8),
                       dim3(64 * WR * WC), lds, s, A);
    return hipGetLastError();
}

// Whether k_gr_main can take rows of K (ld apart) and weights: 16 bytes at a time,
// places behind its bases below 4 GB.
template <class T>
bool main_ok(const void* U, int64_t ld, int64_t n, int64_t K, const void* W, int64_t w, const int32_t* order) {
    const int64_t es = sizeof(T), most = (int64_t)1 << 32;
    return rows_vec16(U, ld, K, es) && w * es % 16 == 0 && a16(W) && (order ? n : 256) * ld * es < most &&
           256 * w * es < most;
}

// A product's tiles and parts as the launch takes them: those of any addresses where
// rows or weights cannot be read 16 bytes at a time.
struct MainPlan {
    GroupList list;
    int32_t splits;
};
MainPlan main_plan(const GroupArgs& D, const GroupShape& L, bool al) {
    MainPlan M{L.rows, al ? L.splits : L.any_splits};
    if (!al) M.list.size = L.any_tile;
    M.list.max_items = group_items(D.n, D.k, M.list.size);
    return M;
}

template <class T, class O, bool TR>
hipError_t main_go(MainArgs A, const MainPlan& M, bool al, hipStream_t s) {
    const int64_t items = M.list.max_items;
    const int bk = 128 / (int)sizeof(T), all = (A.K + bk - 1) / bk;
    A.splits = M.splits;
    A.share = part_stages(all, M.splits, sizeof(T) == 1);
    hipError_t e;
    if constexpr (kWide<T, O>) {
        e = M.list.size == 128 ? any_tile<T, O, 128, 128, 2, 2, TR>(A, items, s)
                               : any_tile<T, O, 64, 64, 2, 2, TR>(A, items, s);
    } else {
        if (!al && M.list.size == 128) e = any_tile<T, O, 128, 128, 2, 2, TR>(A, items, s);
        else if (!al) e = any_tile<T, O, 64, 64, 2, 2, TR>(A, items, s);
        else if (M.list.size == 256) e = main_tile<T, O, 256, 256, 2, 4, TR>(A, items, s);
        else if (M.list.size == 128) e = main_tile<T, O, 128, 128, 2, 2, TR>(A, items, s);
        else e = main_tile<T, O, 64, 64, 2, 2, TR>(A, items, s);
    }
    if (e != hipSuccess || A.splits == 1) return e;
    hipLaunchKernelGGL((k_gr_sum<O>), dim3((unsigned)A.n, (unsigned)((A.P + 1023) / 1024)), dim3(256), 0, s, A);
    return hipGetLastError();
}

ListArgs list_args(const GroupArgs& D, const GroupList& L, char* ws, bool cut) {
    ListArgs A{};
    A.offsets = D.offsets;
    A.k = D.k;
    A.size = L.size;
    A.count = reinterpret_cast<int32_t*>(ws + L.off_count);
    A.items = reinterpret_cast<GroupItem*>(ws + L.off_items);
    if (cut) {
        A.first = reinterpret_cast<int32_t*>(ws + L.off_first);
        A.num = A.first + D.k;
    }
    return A;
}

// The lists that are wanted (not null): row tiles and chunks.
hipError_t lists_go(const GroupArgs& D, const GroupList* rows, const GroupList* cuts, char* ws, hipStream_t s) {
    const ListArgs R = rows ? list_args(D, *rows, ws, false) : list_args(D, *cuts, ws, true);
    const ListArgs C = cuts ? list_args(D, *cuts, ws, true) : R;
    hipLaunchKernelGGL(k_gr_list, dim3(rows && cuts ? 2 : 1), dim3(1024), 0, s, R, C);
    return hipGetLastError();
}

template <class T, class O>
hipError_t forward_t(const GroupArgs& D, char* ws, const GroupShape& L, hipStream_t s) {
    if (L.few) {
        const bool al = rows_vec16(D.X, D.ldx, D.di, sizeof(T)) && D.di % (16 / (int)sizeof(T)) == 0 && a16(D.W);
        FewArgs F{};
        F.U = D.X;
        F.ldu = D.ldx;
        F.W = D.W;
        F.UE = D.XE;
        F.WE = D.WE;
        F.order = D.order;
        F.sids = D.sids;
        F.offsets = D.offsets;
        F.Y = D.Y;
        F.n = (int32_t)D.n;
        F.k = D.k;
        F.K = D.di;
        F.P = D.dout;
        F.nb = (D.di + 127) / 128;
        const dim3 g((unsigned)((D.dout + 15) / 16), (unsigned)D.n);
        const int steps = (int)(((int64_t)D.di * sizeof(T) + 4 * FewOp<T, O>::kBytes - 1) / (4 * FewOp<T, O>::kBytes));
        auto go = [&](auto waves) {
            constexpr int W = decltype(waves)::value;
            if (al) hipLaunchKernelGGL((k_gr_few<T, O, true, W>), g, dim3(64 * W), 0, s, F);
            else hipLaunchKernelGGL((k_gr_few<T, O, false, W>), g, dim3(64 * W), 0, s, F);
        };
        if (steps <= 16) go(std::integral_constant<int, 4>{});
        else if (steps <= 64) go(std::integral_constant<int, 8>{});
        else go(std::integral_constant<int, sizeof(T) == 1 ? 8 : 16>{});   // 8 bits: registers
        return hipGetLastError();
    }
    const bool al = !kWide<T, O> && main_ok<T>(D.X, D.ldx, D.n, D.di, D.W, D.di, D.order);
    const MainPlan plan = main_plan(D, L, al);
    const hipError_t e = lists_go(D, &plan.list, nullptr, ws, s);
    if (e != hipSuccess) return e;
    const ListArgs Q = list_args(D, plan.list, ws, false);
    MainArgs M{};
    M.U = D.X;
    M.ldu = D.ldx;
    M.W = D.W;
    M.UE = D.XE;
    M.WE = D.WE;
    M.order = D.order;
    M.count = Q.count;
    M.items = Q.items;
    M.used = D.offsets + D.k;
    M.n = D.n;
    M.Y = D.Y;
    M.K = D.di;
    M.P = D.dout;
    M.nb = (D.di + 127) / 128;
    M.part = reinterpret_cast<float*>(ws + L.off_split);
    return main_go<T, O, false>(M, plan, al, s);
}

template <class T, int TILE, int WC>
hipError_t grad_tile(GradArgs A, int64_t max_items, bool al, hipStream_t s) {
    A.tq = (A.Q + TILE - 1) / TILE;
    A.tp = (A.P + TILE - 1) / TILE;
    constexpr int lds = 2 * 2 * TILE * 128;
    const int64_t tiles = (max_items * A.tq * A.tp + 63) / 64 * 64, most = kCus * (TILE == 256 ? 1 : 2);
    if (al) {
        if (lds > 65536) {
            const hipError_t e = raise_lds(k_gr_grad<T, TILE, TILE, 2, WC>, lds);
            if (e != hipSuccess) return e;
        }
        hipLaunchKernelGGL((k_gr_grad<T, TILE, TILE, 2, WC>), dim3((unsigned)(tiles < most ? tiles : most)),
                           dim3(128 * WC), lds, s, A);
    } else {
        hipLaunchKernelGGL((k_gr_grad_any<T, 128, 128, 2, 2>), many_blocks(tiles), dim3(256), 2 * 2 * 128 * 128, s, A);
    }
    return hipGetLastError();
}

// Whether k_gr_grad can take rows of d, ld apart: 16 bytes at a time, places behind
// its bases below 4 GB.
template <class T>
bool grad_ok(const void* U, int64_t ld, int64_t n, int64_t d, const int32_t* order, int64_t size) {
    const int64_t es = sizeof(T);
    return rows_vec16(U, ld, d, es) && (order ? n : size) * ld * es < (int64_t)1 << 32;
}

template <class T>
hipError_t backward_t(const GroupArgs& D, char* ws, const GroupShape& L, hipStream_t s) {
    const bool al = main_ok<T>(D.dY, D.lddy, D.n, D.dout, D.W, D.di, D.order);   // dX
    const MainPlan plan = main_plan(D, L, al);
    const bool want = D.dX && D.n > 0;
    hipError_t e = want || D.dW ? lists_go(D, want ? &plan.list : nullptr, D.dW ? &L.cuts : nullptr, ws, s) : hipSuccess;
    if (e != hipSuccess) return e;
    if (want) {
        const ListArgs Q = list_args(D, plan.list, ws, false);
        MainArgs M{};
        M.U = D.dY;
        M.ldu = D.lddy;
        M.W = D.W;
        M.order = D.order;
        M.count = Q.count;
        M.items = Q.items;
        M.used = D.offsets + D.k;
        M.n = D.n;
        M.Y = D.dX;
        M.K = D.dout;
        M.P = D.di;
        M.part = reinterpret_cast<float*>(ws + L.off_split);
        e = main_go<T, T, true>(M, plan, al, s);
        if (e != hipSuccess) return e;
    }
    if (D.dW) {
        const ListArgs Q = list_args(D, L.cuts, ws, true);
        GradArgs G{};
        G.U = D.X;
        G.ldu = D.ldx;
        G.V = D.dY;
        G.ldv = D.lddy;
        G.order = D.order;
        G.count = Q.count;
        G.items = Q.items;
        G.first = Q.first;
        G.num = Q.num;
        G.out = D.dW;
        G.part = reinterpret_cast<float*>(ws + L.off_part);
        G.k = D.k;
        G.P = D.di;
        G.Q = D.dout;
        if (L.cuts.max_items > 0) {
            const bool whole = grad_ok<T>(D.X, D.ldx, D.n, D.di, D.order, L.cuts.size) &&
                               grad_ok<T>(D.dY, D.lddy, D.n, D.dout, D.order, L.cuts.size);
            if (whole && L.grad_tile == 256) e = grad_tile<T, 256, 4>(G, L.cuts.max_items, true, s);
            else e = grad_tile<T, 128, 2>(G, L.cuts.max_items, whole, s);
            if (e != hipSuccess) return e;
        }
        // Some 16 blocks a compute unit: most clusters have one chunk, which is no work here.
        const int64_t gy = D.k < 1024 ? D.k : 1024, wide = ((int64_t)D.dout * D.di + 2047) / 2048, gx = 4096 / gy;
        hipLaunchKernelGGL((k_gr_join<T>), dim3((unsigned)(wide < gx ? wide : gx), (unsigned)gy), dim3(256), 0, s, G);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

namespace {

// The tile and the parts of the contraction of a product, by an estimate of its time
// (`met` clusters have rows; main: k_gr_main, else k_gr_any).
struct MainChoice {
    int32_t tile, splits;
};
MainChoice main_choice(int64_t n, int64_t met, int32_t K, int32_t P, int type, bool main) {
    const int es = (int)row_type_bytes(type), all = (K + 128 / es - 1) / (128 / es);
    const int i = type == kF32 ? 1 : type == kF8 ? 2 : 0;
    // A compute unit holds `held` tiles at once.  A stage of as many takes `busy` us on
    // a chip at work, and no stage less than `alone`; measured with 64 to 16,384 rows
    // of 256 to 4096 (16-bit, float32 and 8-bit rows).  A tile starts and ends in the
    // time of `edge` stages (too little for float32 tiles of 64 with few stages: 100,003
    // rows of 256 to 256 are estimated at 94 us and take 142).
    struct Kind {
        int tile, held;
        double busy[3], alone[3], edge[3];
    };
    const Kind kinds[3] = {{256, 1, {1.65, 7.2, 1.75}, {1.05, 7.0, 1.1}, {3.5, 1.0, 5.5}},
                           {128, 2, {1.15, 3.3, 1.15}, {0.85, 1.7, 0.85}, {2.5, 1.0, 2.2}},
                           {64, 4, {0.96, 1.55, 0.85}, {0.6, 0.6, 0.5}, {2.0, 1.0, 2.0}}};
    // At any address blocks come as others end: no round is waited for, and a stage's time
    // grows from `alone` with the tiles that share a compute unit (1001 to 1003 columns
    // in bf16, 8 clusters of 512: 34 us with tiles of 128, 37 with 64; 2001 to 2003, 4 of
    // 2000: 131 and 206; 3001 to 301, 100 of 30: 92 and 46).
    const Kind anywhere[2] = {{128, 2, {1.6, 5.2, 2.1}, {1.55, 2.6, 1.9}, {3.0, 3.0, 3.0}},
                              {64, 4, {1.4, 1.9, 1.8}, {0.65, 1.1, 1.0}, {3.0, 3.0, 3.0}}};
    MainChoice best{128, 1};
    double least = 0;
    for (int q = 0; q < (main ? 3 : 2); ++q) {
        const Kind& k = main ? kinds[q] : anywhere[q];
        // A cluster's last tile is half full, and none has less than one.
        double items = (double)n / k.tile + 0.5 * met;
        if (items < met) items = (double)met;
        for (int splits = 1; splits <= 16 && (splits == 1 || (k.tile < 256 && all / splits >= 4)); splits *= 2) {
            const int share = part_stages(all, splits, type == kF8);
            if (splits > 1 && share * (splits - 1) >= all) continue;   // no part without a stage
            const double tiles = items * ((P + k.tile - 1) / k.tile) * splits, rounds = tiles / (kCus * k.held);
            double stage = tiles <= kCus ? k.alone[i] : k.busy[i];
            if (!main && tiles > kCus && rounds < 1)
                stage = k.alone[i] + (k.busy[i] - k.alone[i]) * (tiles / kCus - 1) / (k.held - 1);
            // Small tiles make up for each other's waits.
            const bool flows = k.tile == 64 || !main;
            double t = (flows && rounds > 1 ? rounds + 0.5 : ceil(rounds)) * stage * (share + k.edge[i]);
            if (splits > 1) t += 6 + (double)splits * n * P * 8 / 4e6;   // sums at 4 TB/s, and a launch
            if (least == 0 || t < least) {
                least = t;
                best = MainChoice{k.tile, splits};
            }
        }
    }
    return best;
}

}  // namespace

// Most items of up to `size` places that n places of k clusters are cut into.
int64_t group_items(int64_t n, int32_t k, int32_t size) { return n / size + (k < n ? k : n); }

GroupShape group_shape(int64_t n, int32_t di, int32_t dout, int32_t k, int type, bool backward) {
    GroupShape L{};
    size_t o = 0;
    auto take = [&](size_t b) {
        const size_t at = o;
        o += (b + 255) / 256 * 256;
        return at;
    };
    L.few = !backward && n <= kGroupFew;
    const int64_t met = k < n ? k : n;   // most clusters with rows
    if (!L.few) {
        const int32_t K = backward ? dout : di, P = backward ? di : dout;
        const MainChoice main = main_choice(n, met, K, P, type, true), any = main_choice(n, met, K, P, type, false);
        L.rows.size = main.tile;
        L.splits = main.splits;
        L.any_splits = any.splits;
        L.any_tile = any.tile;
        const int most = L.splits > L.any_splits ? L.splits : L.any_splits;
        L.off_split = take(most > 1 ? (size_t)most * n * P * 4 : 0);
        L.rows.max_items = group_items(n, k, 64);   // 64: the least size of a tile
        L.rows.off_count = take(4);
        L.rows.off_items = take((size_t)L.rows.max_items * sizeof(GroupItem));
    }
    if (backward) {
        const int64_t big = (((int64_t)di + 255) / 256) * (((int64_t)dout + 255) / 256);
        L.grad_tile = big * met >= 128 ? 256 : 128;
        const int64_t each = L.grad_tile == 256 ? big : (((int64_t)di + 127) / 128) * (((int64_t)dout + 127) / 128);
        // Chunks that give the chip some two rounds of blocks.
        int64_t size = n * each / 512;
        size = size < 256 ? 256 : (size + 63) / 64 * 64;
        L.cuts.size = (int32_t)(size < INT32_MAX / 2 ? size : INT32_MAX / 2);
        const int64_t cuts = n / L.cuts.size;
        L.cuts.max_items = group_items(n, k, L.cuts.size);
        L.cuts.off_count = take(4);
        L.cuts.off_items = take((size_t)L.cuts.max_items * sizeof(GroupItem));
        L.cuts.off_first = take((size_t)k * 8);
        // A cluster of several chunks has one that is not full: at most 2 cuts partial sums.
        L.off_part = take((size_t)(2 * cuts) * di * dout * 4);
    }
    L.bytes = o > 0 ? o : 256;
    return L;
}

hipError_t launch_group_forward(const GroupArgs& D, char* ws, const GroupShape& L, int type, int out_type,
                                hipStream_t s) {
    if (D.n == 0) return hipSuccess;
    if (type == kF8) {
        if (out_type == kF32) return forward_t<uint8_t, float>(D, ws, L, s);
        if (out_type == kBF16) return forward_t<uint8_t, __bf16>(D, ws, L, s);
        return forward_t<uint8_t, _Float16>(D, ws, L, s);
    }
    if (type == kF32) return forward_t<float, float>(D, ws, L, s);
    if (type == kBF16) return forward_t<__bf16, __bf16>(D, ws, L, s);
    return forward_t<_Float16, _Float16>(D, ws, L, s);
}

hipError_t launch_group_backward(const GroupArgs& D, char* ws, const GroupShape& L, int type, hipStream_t s) {
    if (type == kF32) return backward_t<float>(D, ws, L, s);
    if (type == kBF16) return backward_t<__bf16>(D, ws, L, s);
    return backward_t<_Float16>(D, ws, L, s);
}

}  // namespace km
