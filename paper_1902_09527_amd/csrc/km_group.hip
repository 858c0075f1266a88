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
// ones it drops the bits more than 13 below the largest one's exponent (measured,
// one pair of products at a time): 1.3e-5 of the norm of products of 4096 normal
// values.  That is below a hundredth of a bfloat16 result's own rounding and a
// tenth of a float16 one's; float32 results take the next form.
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

// Eight e4m3 values times 2^(byte - 127) as bfloat16, which holds them exactly.
__device__ __forceinline__ u32x4 widen(uint32_t lo, uint32_t hi, int byte) {
    const float scale = __builtin_bit_cast(float, byte > 0 ? (uint32_t)byte << 23 : 0x400000u);
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
// keep float32.  A chunk is the operand of two steps.
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
    static __device__ __forceinline__ Acc mma(const Frag& a, const Frag& b, Acc c, int sa, int sb) {
#pragma unroll
        for (int i = 0; i < 4; i += 2)
            c = Mma<__bf16>::mma(widen(a.v[i], a.v[i + 1], sa), widen(b.v[i], b.v[i + 1], sb), c);
        return c;
    }
    static constexpr int kRuns = 1;
    static __device__ __forceinline__ int run(int, int lane) { return (lane >> 4) * 4; }
};

// 16 bytes of a row from element k0 on, zero past its K elements, at any address.
template <class T>
__device__ __forceinline__ u32x4 chunk_any(const T* row, int64_t k0, int64_t K) {
    constexpr int E = 16 / (int)sizeof(T);
    if (k0 + E <= K) {
        u32x4 v;
        __builtin_memcpy(&v, row + k0, 16);
        return v;
    }
    Vec<T, E> v;
#pragma unroll
    for (int e = 0; e < E; ++e) v.e[e] = row[k0 + e < K ? k0 + e : 0];
#pragma unroll
    for (int e = 0; e < E; ++e) v.e[e] = k0 + e < K ? v.e[e] : (T)0.0f;
    return __builtin_bit_cast(u32x4, v);
}

// --------------------------------------------------------------------------
// Lists of row tiles and of chunks.

// What to list: `size` places at most an item, none of two clusters.
struct ListArgs {
    const int32_t* offsets;
    int32_t n, k, size;
    int32_t* count;
    GroupItem* items;
    int32_t *first, *num;   // per cluster: first partial slot, items; null: not wanted, and
                            // the places of no cluster are listed too, as cluster -1
};

// A block a list.  In order of the clusters.
__global__ __launch_bounds__(1024) void k_gr_list(ListArgs A0, ListArgs A1) {
    const ListArgs& A = blockIdx.x ? A1 : A0;
    __shared__ int s[2][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int items = 0, slots = 0;   // so far
    const int end = A.num ? A.k : A.k + 1;
    for (int c0 = 0; c0 < end; c0 += 1024) {
        const int c = c0 + tid;
        const int a = c < end ? A.offsets[c] : 0, b = c < A.k ? A.offsets[c + 1] : c < end ? A.n : 0;
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
        if (c < end) {
            if (A.num) {
                A.first[c] = bs;
                A.num[c] = ni;
            }
            for (int q = 0; q < ni; ++q) {
                const int p = a + q * A.size;
                A.items[bi + q] =
                    GroupItem{c < A.k ? c : -1, p, b - p < A.size ? b : p + A.size, A.num && ni > 1 ? bs + q : -1};
            }
        }
        __syncthreads();
    }
    if (tid == 0) A.count[0] = items;
}

// --------------------------------------------------------------------------
// Y[row] = V_c U[row], V = W_c (P x K) forward, W_c^T (W_c is K x P) with TR.

struct MainArgs {
    const void* U;
    int64_t ldu;
    const void* W;
    const uint8_t *UE, *WE;   // 8 bits: a byte for each 128 elements of a row, nb a row
    const int32_t *order, *count;
    const GroupItem* items;
    void* Y;
    int32_t K, P, nb, y4;     // y4: Y can be written 4 elements at a time
    int32_t tn;               // tiles of columns
};

constexpr int kWindow = 32;   // stages whose scales are in LDS

// A tile is TM places x TN columns, WR x WC waves; the contraction goes in stages
// of 128 bytes a row, NS of them in LDS.  Rows of a tile are dealt to its waves in
// kParts turns, so that a tile of few rows leaves out the products of the turns
// past them.
template <class T, class O, int TM, int TN, int WR, int WC, int NS, bool TR, bool AL>
__global__ __launch_bounds__(64 * WR * WC) void k_gr_main(MainArgs A) {
    using P = Op<T, O>;
    constexpr bool F8 = sizeof(T) == 1;
    constexpr int E = P::E, R = P::R, KS = 4 * E, BK = 2 * KS, NT = 64 * WR * WC;
    constexpr int FR = TM / WR / R, FC = TN / WC / R;
    constexpr int NU = TM * 8 / NT, NW = TN * 8 / NT, CPR = TN / E;
    constexpr int kStage = (TM + TN) * 128;
    constexpr int kParts = FR < 4 ? FR : 4, FP = FR / kParts;   // turns, and a wave's operands of one
    constexpr int kTurn = FP * R * WR;                          // rows of a turn
    static_assert(FR % kParts == 0 && NT % 128 == 0, "");
    extern __shared__ __align__(16) char s_tiles[];
    uint8_t* s_scale = reinterpret_cast<uint8_t*>(s_tiles + NS * kStage);   // 8 bits: [kWindow][TM + TN]
    int32_t* s_rows = reinterpret_cast<int32_t*>(s_tiles + NS * kStage + (F8 ? kWindow * (TM + TN) : 0));
    const int tid = threadIdx.x, lane = tid & 63, li = lane % R;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wr = wave / WC, wc = wave % WC;

    // Consecutive tiles go to one XCD (blocks are dealt over 8), down 4 row tiles
    // before the next columns.
    const int items = __builtin_amdgcn_readfirstlane(A.count[0]);
    const int64_t tiles = (int64_t)items * A.tn, per = (tiles + 7) / 8;
    const int64_t t = (blockIdx.x % 8) * per + blockIdx.x / 8;
    if (blockIdx.x / 8 >= per || t >= tiles) return;
    const int64_t grp = t / (4 * (int64_t)A.tn), m0 = grp * 4;
    const int gm = items - m0 < 4 ? (int)(items - m0) : 4;
    const int64_t in_grp = t - grp * 4 * A.tn;
    const GroupItem it = A.items[m0 + in_grp % gm];
    const int64_t bn = in_grp / gm * TN;
    const int c = __builtin_amdgcn_readfirstlane(it.c), p0 = __builtin_amdgcn_readfirstlane(it.p0);
    const int rows = __builtin_amdgcn_readfirstlane(it.p1) - p0;
    O* const Y = static_cast<O*>(A.Y);
    if (c < 0) {   // rows of no cluster
        for (int q = tid; q < rows * TN; q += NT) {
            const int64_t col = bn + q % TN;
            if (col < A.P) Y[row_of(A.order, p0 + q / TN) * A.P + col] = from_f32<O>(0.0f);
        }
        return;
    }
    const int nk = (A.K + BK - 1) / BK, live = (rows + kTurn - 1) / kTurn;
    const int64_t ldw = TR ? A.P : A.K;
    const T* const W = static_cast<const T*>(A.W) + (int64_t)c * A.K * A.P;

    // Where a thread's chunks of a stage come from: pointers that move on with the
    // stages (AL), the place in the stage being fixed.
    const T* up[NU];
    const T* wp[NW];
    const int uc = swz(tid / 8, tid % 8) * E;   // NT / 8 rows further on the swizzle is the same
#pragma unroll
    for (int i = 0; i < NU; ++i) {
        const int r = (i * NT + tid) / 8;
        const int64_t row = row_of(A.order, p0 + (r < rows ? r : rows - 1));   // past the last: not stored
        up[i] = static_cast<const T*>(A.U) + row * A.ldu + (AL ? uc : 0);
        if (tid % 8 == 0) s_rows[r] = (int32_t)row;
    }
#pragma unroll
    for (int i = 0; i < NW; ++i) {
        const int q = i * NT + tid;
        if constexpr (TR) {
            wp[i] = W + (int64_t)(q / CPR) * ldw + (AL ? bn + swz_tr<T, CPR>(q / CPR, q % CPR) * E : 0);
        } else {
            const int64_t col = bn + q / 8 < A.P ? bn + q / 8 : A.P - 1;   // past the last: not stored
            wp[i] = W + col * ldw + (AL ? uc : 0);
        }
    }
    // Stages without a chunk past the contraction's end or the last column.
    const int whole = !TR || bn + TN <= A.P ? A.K / BK : 0;

    // Chunk i of stage kt (of NU + NW a thread) to LDS; guard: it may lie past an end.
    auto load = [&](int i, int kt, char* buf, bool guard) {
        if (i < NU) {
            const void* src = !guard || kt * BK + uc < A.K ? (const void*)up[i] : (const void*)zero_chunk;
            load_lds16(src, buf + (i * NT + wave * 64) * 16);
            up[i] += BK;
            return;
        }
        i -= NU;
        const int q = i * NT + tid;
        char* wb = buf + TM * 128;
        if constexpr (TR) {
            const int kk = q / CPR;
            const bool in = !guard || (kt * BK + kk < A.K && bn + swz_tr<T, CPR>(kk, q % CPR) * E < A.P);
            load_lds16(in ? (const void*)wp[i] : (const void*)zero_chunk, wb + (i * NT + wave * 64) * 16);
            wp[i] += BK * ldw;
        } else {
            const void* src = !guard || kt * BK + uc < A.K ? (const void*)wp[i] : (const void*)zero_chunk;
            load_lds16(src, wb + (i * NT + wave * 64) * 16);
            wp[i] += BK;
        }
    };
    // The same through registers, at any address.
    auto fetch = [&](int i, int kt) -> u32x4 {
        if (i < NU) return chunk_any(up[i], (int64_t)kt * BK + uc, A.K);
        i -= NU;
        if constexpr (TR) {
            const int q = i * NT + tid, kk = q / CPR;
            const bool in = kt * BK + kk < A.K;
            return only_if(in, chunk_any(in ? wp[i] + (int64_t)kt * BK * ldw : W,
                                         bn + swz_tr<T, CPR>(kk, q % CPR) * E, A.P));
        } else {
            return chunk_any(wp[i], (int64_t)kt * BK + uc, A.K);
        }
    };

    // 8 bits: the scales of the stages from k0 on, a row a thread.
    auto scales = [&](int k0) {
        if constexpr (F8) {
            for (int r = tid; r < TM + TN; r += NT) {
                const uint8_t* e;
                if (r < TM) {
                    e = A.UE + row_of(A.order, p0 + (r < rows ? r : rows - 1)) * A.nb;
                } else {
                    const int64_t col = bn + r - TM < A.P ? bn + r - TM : A.P - 1;
                    e = A.WE + ((int64_t)c * A.P + col) * A.nb;
                }
                const int left = A.nb - k0 < kWindow ? A.nb - k0 : kWindow;
                uint8_t v[kWindow];
                if (left == kWindow) {
                    __builtin_memcpy(v, e + k0, kWindow);
                } else {
#pragma unroll
                    for (int q = 0; q < kWindow; ++q) v[q] = e[k0 + (q < left ? q : 0)];
                }
#pragma unroll
                for (int q = 0; q < kWindow; ++q) s_scale[q * (TM + TN) + r] = v[q];
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

    // A lane's places in a stage; the second half of a row is 64 bytes off (one bit
    // of the swizzled chunk).
    auto tile_row = [&](int f) { return f / FP * kTurn + wr * (FP * R) + f % FP * R + li; };
    const int ua = tile_row(0) * 128 + swz(li, P::chunk(lane)) * 16;
    int wa[TR ? FC : 1];
    if constexpr (TR) {
#pragma unroll
        for (int h = 0; h < FC; ++h) wa[h] = TM * 128 + tr_lane<T, CPR>(wc * (TN / WC) + h * 16, lane);
    } else {
        wa[0] = TM * 128 + (wc * (TN / WC) + li) * 128 + swz(li, P::chunk(lane)) * 16;
    }
    struct Frags {
        typename P::Frag b[FR], a[FC];
    };
    int sa[F8 ? FC : 1], sb[F8 ? FR : 1];   // 8 bits: the stage's scales
    // Operand i of half s of a stage: first the columns' (TR: read_cols), then the rows'.
    auto read = [&](Frags& F, int i, const char* buf, int s) {
        if (i < FC) {
            if constexpr (!TR) F.a[i] = P::read(buf, (wa[0] ^ (s * 64)) + i * (R * 128));
        } else {
            const int f = i - FC;
            F.b[f] = P::read(buf, (ua ^ (s * 64)) + (f / FP * kTurn + f % FP * R) * 128);
        }
    };
    auto read_cols = [&](Frags& F, const char* buf, int s) {
        if constexpr (TR) {
            u32x4 v[FC];
            if (s == 0) read_tr_wait<T, CPR, 0>(v, buf, wa);
            else read_tr_wait<T, CPR, KS>(v, buf, wa);
#pragma unroll
            for (int h = 0; h < FC; ++h) F.a[h].v = v[h];
        }
    };
    auto read_scales = [&](int kt) {
        if constexpr (F8) {
            const uint8_t* s = s_scale + kt % kWindow * (TM + TN);
#pragma unroll
            for (int h = 0; h < FC; ++h) sa[h] = s[TM + wc * (TN / WC) + h * R + li];
#pragma unroll
            for (int f = 0; f < FR; ++f) sb[f] = s[tile_row(f)];
        }
    };
    auto products = [&](const Frags& F, int q) {
        if (q >= live) return;
#pragma unroll
        for (int f = q * FP; f < (q + 1) * FP; ++f)
#pragma unroll
            for (int h = 0; h < FC; ++h)
                acc[f][h] = P::mma(F.a[h], F.b[f], acc[f][h], sa[F8 ? h : 0], sb[F8 ? f : 0]);
    };

    if constexpr (!AL) {
        // One stage in registers while the one before is multiplied.
        u32x4 v[NU + NW];
        scales(0);
#pragma unroll
        for (int i = 0; i < NU + NW; ++i) v[i] = fetch(i, 0);
        for (int kt = 0; kt < nk; ++kt) {
            char* buf = s_tiles + kt % NS * kStage;
#pragma unroll
            for (int i = 0; i < NU + NW; ++i) *reinterpret_cast<u32x4*>(buf + (i * NT + tid) * 16) = v[i];
            __syncthreads();
            if (kt + 1 < nk) {
#pragma unroll
                for (int i = 0; i < NU + NW; ++i) v[i] = fetch(i, kt + 1);
            }
            read_scales(kt);
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                Frags F;
#pragma unroll
                for (int i = 0; i < FR + FC; ++i) read(F, i, buf, s);
                read_cols(F, buf, s);
#pragma unroll
                for (int q = 0; q < kParts; ++q) products(F, q);
            }
            if (F8 && (kt + 1) % kWindow == 0 && kt + 1 < nk) {
                __syncthreads();
                scales(kt + 1);
            }
        }
    } else {
        auto load_all = [&](int kt, char* buf) {
#pragma unroll
            for (int i = 0; i < NU + NW; ++i) load(i, kt, buf, kt >= whole);
        };
#pragma unroll
        for (int kt = 0; kt < NS; ++kt)
            if (kt < nk) load_all(kt, s_tiles + kt * kStage);
        scales(0);
        // Operands are read from LDS half a stage ahead of their products, and a
        // stage is loaded while the one before it is multiplied.  The barrier of a
        // stage stands between its two halves of products, when the second half's
        // operands are in registers, and loads, reads and products are issued in
        // turns, so that the matrix cores do not wait for either.
        // The products of F; F2 read from buf2 (half s2); kl >= 0: stage kl loaded into bufl.
        auto half = [&](const Frags& F, Frags& F2, const char* buf2, int s2, int kl, char* bufl, bool guard) {
#pragma unroll
            for (int q = 0; q < kParts; ++q) {
                if (kl >= 0) {
#pragma unroll
                    for (int i = q * (NU + NW) / kParts; i < (q + 1) * (NU + NW) / kParts; ++i) load(i, kl, bufl, guard);
                }
#pragma unroll
                for (int i = q * (FR + FC) / kParts; i < (q + 1) * (FR + FC) / kParts; ++i) read(F2, i, buf2, s2);
                products(F, q);
                __builtin_amdgcn_sched_barrier(0);
                if (TR && q == 0) {   // while the first products are at work
                    read_cols(F2, buf2, s2);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        };
        // This wave's operands have arrived (F2 of the half before).
        auto arrived = [&]() { __builtin_amdgcn_s_waitcnt(0xc07f); };   // lgkmcnt(0)
        // Every wave's reads of one stage and its loads of the next have ended; the
        // loads of the stages behind that one (kBehind) may be on their way.
        constexpr int kBehind = (NS - 2) * (NU + NW);
        static_assert(kBehind < 64, "");
        auto turn = [&](bool all) {
            if (all) __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0) lgkmcnt(0)
            else __builtin_amdgcn_s_waitcnt(0x0070 | (kBehind & 15) | (kBehind >> 4) << 14);
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
        Frags F0, F1;
        turn(true);
#pragma unroll
        for (int i = 0; i < FR + FC; ++i) read(F0, i, s_tiles, 0);
        read_cols(F0, s_tiles, 0);
        int at = 0;   // the stage's place in the ring
        auto stage = [&](int kt, bool last) {
            char* cur = s_tiles + at * kStage;
            at = at + 1 == NS ? 0 : at + 1;
            const char* nxt = s_tiles + at * kStage;
            read_scales(kt);
            arrived();
            __builtin_amdgcn_sched_barrier(0);
            half(F0, F1, cur, 1, -1, cur, false);
            turn(last);
            __builtin_amdgcn_sched_barrier(0);
            // Every wave has the scales of this stage in registers: the window may move on.
            if (F8 && (kt + 1) % kWindow == 0 && kt + 1 < nk) {
                scales(kt + 1);
                __syncthreads();
            }
            // After the last stage the reads are of what the buffer held before, and are not used.
            half(F1, F0, nxt, 0, !last ? kt + NS : kt + NS < nk ? kt + NS : -1, cur, last);
        };
        int kt = 0;
        for (; kt + NS < whole && kt + NS < nk; ++kt) stage(kt, false);
        for (; kt < nk; ++kt) stage(kt, true);
    }

#pragma unroll
    for (int f = 0; f < FR; ++f) {
        const int r = tile_row(f);
        if (r >= rows) continue;
        O* y = Y + (int64_t)s_rows[r] * A.P;
#pragma unroll
        for (int h = 0; h < FC; ++h)
#pragma unroll
            for (int j = 0; j < P::kRuns; ++j) {
                f32x4 v;
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = acc[f][h][j * 4 + i];
                store4(y, bn + wc * (TN / WC) + h * R + P::run(j, lane), A.P, v, A.y4);
            }
    }
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
    int32_t k, P, Q, o4;
    int32_t tq, tp;          // tiles
};

template <class T, int TM, int TN, int WR, int WC, bool AL>
__global__ __launch_bounds__(64 * WR * WC) void k_gr_grad(GradArgs A) {
    constexpr int E = Mma<T>::E, KS = 4 * E, BK = 2 * KS, NT = 64 * WR * WC;
    constexpr int FR = TM / WR / 16, FC = TN / WC / 16;
    constexpr int CM = TM / E, CN = TN / E;               // chunks a place of V and of U
    constexpr int NV = BK * CM / NT, NU = BK * CN / NT;   // chunks a thread of a stage
    constexpr int kStage = (TM + TN) * 128;
    static_assert(FR % 4 == 0 && FC % 2 == 0, "");
    extern __shared__ __align__(16) char s_tiles[];       // two stages: V, then U
    const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, li = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wr = wave / WC, wc = wave % WC;
    const int items = __builtin_amdgcn_readfirstlane(A.count[0]);
    const int64_t each = (int64_t)A.tq * A.tp, tiles = items * each, per = (tiles + 7) / 8;
    const int64_t t = (blockIdx.x % 8) * per + blockIdx.x / 8;
    if (blockIdx.x / 8 >= per || t >= tiles) return;
    const GroupItem it = A.items[t / each];
    // Down 4 tiles of V's columns before the next of U's.
    const int64_t in = t % each, grp = in / (4 * (int64_t)A.tp), m0 = grp * 4;
    const int gm = A.tq - m0 < 4 ? (int)(A.tq - m0) : 4;
    const int64_t in_grp = in - grp * 4 * A.tp;
    const int64_t bm = (m0 + in_grp % gm) * TM, bn = in_grp / gm * TN;
    const int p1 = it.p1;

    int64_t vr[NV], ur[NU];   // rows of the next stage to load
    auto rows = [&](int p) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int q = p + (i * NT + tid) / CM;
            vr[i] = row_of(A.order, q < p1 ? q : it.p0);
        }
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int q = p + (i * NT + tid) / CN;
            ur[i] = row_of(A.order, q < p1 ? q : it.p0);
        }
    };
    // Where chunk i of V (v) or U comes from, and whether it is there.
    auto chunk_of = [&](bool v, int i, int p, const T*& row, int64_t& col) {
        const int q = i * NT + tid, cpr = v ? CM : CN, kk = q / cpr;
        row = v ? static_cast<const T*>(A.V) + vr[i] * A.ldv : static_cast<const T*>(A.U) + ur[i] * A.ldu;
        col = (v ? bm + swz_tr<T, CM>(kk, q % CM) * E : bn + swz_tr<T, CN>(kk, q % CN) * E);
        return p + kk < p1;
    };
    u32x4 held[AL ? 1 : NV + NU];
    auto load = [&](int p, char* buf) {
#pragma unroll
        for (int i = 0; i < NV + NU; ++i) {
            const bool v = i < NV;
            const T* row;
            int64_t col;
            const bool in = chunk_of(v, v ? i : i - NV, p, row, col);
            const int64_t width = v ? A.Q : A.P;
            if constexpr (AL)
                load_lds16(in && col < width ? (const void*)(row + col) : (const void*)zero_chunk,
                           buf + (v ? 0 : TM * 128) + ((v ? i : i - NV) * NT + wave * 64) * 16);
            else
                held[i] = only_if(in, chunk_any(row, col, width));
        }
    };
    auto put = [&](char* buf) {
        if constexpr (!AL)
#pragma unroll
            for (int i = 0; i < NV + NU; ++i)
                *reinterpret_cast<u32x4*>(buf + (i < NV ? 0 : TM * 128) + ((i < NV ? i : i - NV) * NT + tid) * 16) =
                    held[i];
    };
    int va[FR], ua[FC];
#pragma unroll
    for (int f = 0; f < FR; ++f) va[f] = tr_lane<T, CM>(wr * (TM / WR) + f * 16, lane);
#pragma unroll
    for (int h = 0; h < FC; ++h) ua[h] = TM * 128 + tr_lane<T, CN>(wc * (TN / WC) + h * 16, lane);
    f32x4 acc[FR][FC];
#pragma unroll
    for (int f = 0; f < FR; ++f)
#pragma unroll
        for (int h = 0; h < FC; ++h) acc[f][h] = f32x4{0, 0, 0, 0};

    int at = 0;
    rows(it.p0);
    load(it.p0, s_tiles);
    rows(it.p0 + BK);
    put(s_tiles);
    for (int p = it.p0; p < p1; p += BK, at ^= 1) {
        const char* buf = s_tiles + at * kStage;
        char* other = s_tiles + (at ^ 1) * kStage;
        // The stage has landed, and every wave is done with the other buffer.
        __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0) lgkmcnt(0)
        __syncthreads();
        if (p + BK < p1) {
            load(p + BK, other);
            rows(p + 2 * BK);
        }
        __builtin_amdgcn_sched_barrier(0);
        auto half = [&](auto s) {
            constexpr int K0 = decltype(s)::value;
            u32x4 a[FC];
#pragma unroll
            for (int h = 0; h < FC; h += 2) {
                u32x4 v[2];
                const int q[2] = {ua[h], ua[h + 1]};
                read_tr_wait<T, CN, K0>(v, buf, q);
                a[h] = v[0], a[h + 1] = v[1];
            }
#pragma unroll
            for (int f = 0; f < FR; f += 4) {
                u32x4 b[4];
                const int q[4] = {va[f], va[f + 1], va[f + 2], va[f + 3]};
                read_tr_wait<T, CM, K0>(b, buf, q);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int h = 0; h < FC; ++h) acc[f + i][h] = Mma<T>::mma(a[h], b[i], acc[f + i][h]);
            }
        };
        half(std::integral_constant<int, 0>{});
        half(std::integral_constant<int, KS>{});
        if (p + BK < p1) put(other);
    }
    const int64_t slot = it.slot < 0 ? it.c : it.slot;
#pragma unroll
    for (int f = 0; f < FR; ++f) {
        const int64_t q = bm + wr * (TM / WR) + f * 16 + li;
        if (q >= A.Q) continue;
        const int64_t at_row = (slot * A.Q + q) * A.P;
#pragma unroll
        for (int h = 0; h < FC; ++h) {
            const int64_t col = bn + wc * (TN / WC) + h * 16 + g * 4;
            if (it.slot < 0) store4(static_cast<T*>(A.out) + at_row, col, A.P, acc[f][h], A.o4);
            else store4(A.part + at_row, col, A.P, acc[f][h], A.P % 4 == 0);
        }
    }
}

// Clusters of no chunk: zeros; of several: the sum of their parts in order.
template <class T>
__global__ __launch_bounds__(256) void k_gr_join(GradArgs A) {
    const int64_t size = (int64_t)A.Q * A.P, step = (int64_t)gridDim.x * 1024;
    const bool by4 = A.o4 && size % 4 == 0;
    for (int c = blockIdx.y; c < A.k; c += gridDim.y) {
        const int num = A.num[c];
        if (num == 1) continue;
        const float* part = A.part + A.first[c] * size;
        T* out = static_cast<T*>(A.out) + c * size;
        for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < size; i += step) {
            f32x4 v{0, 0, 0, 0};
            if (by4) {
#pragma unroll 4
                for (int q = 0; q < num; ++q) v += *reinterpret_cast<const f32x4*>(part + q * size + i);
            } else {
                for (int q = 0; q < num; ++q)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (i + e < size) v[e] += part[q * size + i + e];
            }
            store4(out, i, size, v, by4);
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
    int32_t n, k, K, P, nb, y4;
};

// 16 columns and the places of one cluster a block, from the place blockIdx.y on
// if a cluster starts there; its 16 waves share the contraction.
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
    using Frag = Op<uint8_t, float>::Frag;
    static __device__ __forceinline__ f32x4 mma(const Frag& a, const Frag& b, f32x4 c, int sa, int sb) {
        return Op<uint8_t, float>::mma(a, b, c, sa, sb);
    }
};

template <class T, class O, bool AL, int RF>
__device__ __forceinline__ void few_block(const FewArgs& A, int c, int p0, int rows, f32x4 (*s_red)[4][64]) {
    using P = FewOp<T, O>;
    constexpr bool F8 = sizeof(T) == 1;
    constexpr int EL = P::kBytes / (int)sizeof(T), KS = 4 * EL, NWAVE = 16;   // elements a lane, of a step
    constexpr int UN = !AL ? 1 : RF <= 2 ? 4 : 2;
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
#pragma unroll
        for (int y = 0; y < UN; ++y)
#pragma unroll
            for (int f = 0; f < RF; ++f) acc[f] = P::mma(a[y], b[y][f], acc[f], F8 ? sa[y] : 0, F8 ? sb[y][f] : 0);
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
    if (wave < RF) {
        const int r = wave * 16 + li;
        if (r >= rows) return;
        f32x4 v{0, 0, 0, 0};
#pragma unroll
        for (int y = 0; y < H; ++y) v += s_red[y][wave][lane];
        store4(static_cast<O*>(A.Y) + row_of(A.order, p0 + r) * A.P, col0 + g * 4, A.P, v, A.y4);
    }
}

template <class T, class O, bool AL>
__global__ __launch_bounds__(1024) void k_gr_few(FewArgs A) {
    __shared__ f32x4 s_red[8][4][64];
    const int p = blockIdx.y, c = __builtin_amdgcn_readfirstlane(A.sids[p]);
    if (p > 0 && A.sids[p - 1] == c) return;   // not the first place of its cluster
    if (c < 0) {                               // rows of no cluster
        const int64_t col0 = (int64_t)blockIdx.x * 16;
        for (int q = threadIdx.x; q < (A.n - p) * 16; q += 1024)
            if (col0 + q % 16 < A.P)
                static_cast<O*>(A.Y)[row_of(A.order, p + q / 16) * A.P + col0 + q % 16] = from_f32<O>(0.0f);
        return;
    }
    const int rows = __builtin_amdgcn_readfirstlane(A.offsets[c + 1]) - p;
    if (rows <= 16) few_block<T, O, AL, 1>(A, c, p, rows, s_red);
    else if (rows <= 32) few_block<T, O, AL, 2>(A, c, p, rows, s_red);
    else few_block<T, O, AL, 4>(A, c, p, rows, s_red);
}

// --------------------------------------------------------------------------
// Launches

template <class K>
hipError_t raise_lds(K* kernel, int bytes) {
    return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

template <class T, class O, int TM, int TN, int WR, int WC, int NS, bool TR, bool AL>
hipError_t main_tile(MainArgs A, int64_t max_items, hipStream_t s) {
    A.tn = (A.P + TN - 1) / TN;
    constexpr int lds = NS * (TM + TN) * 128 + (sizeof(T) == 1 ? kWindow * (TM + TN) : 0) + TM * 4;
    static_assert(lds <= 160 * 1024, "");
    if (lds > 65536) {
        const hipError_t e = raise_lds(k_gr_main<T, O, TM, TN, WR, WC, NS, TR, AL>, lds);
        if (e != hipSuccess) return e;
    }
    const int64_t tiles = max_items * A.tn;
    hipLaunchKernelGGL((k_gr_main<T, O, TM, TN, WR, WC, NS, TR, AL>), dim3((unsigned)((tiles + 7) / 8 * 8)),
                       dim3(64 * WR * WC), lds, s, A);
    return hipGetLastError();
}

// 8 bits with float32 results: widened operands take the registers of the larger
// tiles, so there is one form at any address.
template <class T, class O>
constexpr bool kWide = sizeof(T) == 1 && sizeof(O) == 4;

template <class T, class O, bool TR>
hipError_t main_go(const MainArgs& A, const GroupList& L, bool al, hipStream_t s) {
    if constexpr (kWide<T, O>) {
        return main_tile<T, O, 128, 128, 2, 2, 2, TR, false>(A, L.max_items, s);
    } else {
    if (!al) return main_tile<T, O, 128, 128, 2, 2, 2, TR, false>(A, L.max_items, s);
    if (L.size == 256) return main_tile<T, O, 256, 256, 2, 4, 2, TR, true>(A, L.max_items, s);
    return main_tile<T, O, 64, 64, 2, 2, 2, TR, true>(A, L.max_items, s);
    }
}

// The list of row tiles as the launch takes it: tiles of 128 rows where rows or
// weights cannot be read 16 bytes at a time.
GroupList row_list(const GroupArgs& D, GroupList L, bool al) {
    if (!al) L.size = 128;
    L.max_items = group_items(D.n, D.k, L.size) + 1;   // one list more: rows of no cluster
    return L;
}

bool a16(const void* p) { return ((uintptr_t)p & 15) == 0; }

template <class T>
bool rows16(const void* p, int64_t ld, int64_t d) {
    return rows_vec16(p, ld, d, sizeof(T));
}

ListArgs list_args(const GroupArgs& D, const GroupList& L, char* ws, bool cut) {
    ListArgs A{};
    A.offsets = D.offsets;
    A.n = (int32_t)D.n;
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
    const bool al = rows16<T>(D.X, D.ldx, D.di) && D.di % (16 / (int)sizeof(T)) == 0 && a16(D.W);
    const int32_t y4 = D.dout % 4 == 0 && a16(D.Y);
    if (L.few) {
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
        F.y4 = y4;
        const dim3 g((unsigned)((D.dout + 15) / 16), (unsigned)D.n), b(1024);
        if (al) hipLaunchKernelGGL((k_gr_few<T, O, true>), g, b, 0, s, F);
        else hipLaunchKernelGGL((k_gr_few<T, O, false>), g, b, 0, s, F);
        return hipGetLastError();
    }
    const GroupList rows = row_list(D, L.rows, al && !kWide<T, O>);
    const hipError_t e = lists_go(D, &rows, nullptr, ws, s);
    if (e != hipSuccess) return e;
    const ListArgs Q = list_args(D, rows, ws, false);
    MainArgs M{};
    M.U = D.X;
    M.ldu = D.ldx;
    M.W = D.W;
    M.UE = D.XE;
    M.WE = D.WE;
    M.order = D.order;
    M.count = Q.count;
    M.items = Q.items;
    M.Y = D.Y;
    M.K = D.di;
    M.P = D.dout;
    M.nb = (D.di + 127) / 128;
    M.y4 = y4;
    return main_go<T, O, false>(M, rows, al, s);
}

template <class T, int TM, int TN, int WR, int WC, bool AL>
hipError_t grad_tile(GradArgs A, int64_t max_items, hipStream_t s) {
    A.tq = (A.Q + TM - 1) / TM;
    A.tp = (A.P + TN - 1) / TN;
    constexpr int lds = 2 * (TM + TN) * 128;
    if (lds > 65536) {
        const hipError_t e = raise_lds(k_gr_grad<T, TM, TN, WR, WC, AL>, lds);
        if (e != hipSuccess) return e;
    }
    const int64_t tiles = max_items * A.tq * A.tp;
    hipLaunchKernelGGL((k_gr_grad<T, TM, TN, WR, WC, AL>), dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(64 * WR * WC), lds,
                       s, A);
    return hipGetLastError();
}

template <class T>
hipError_t backward_t(const GroupArgs& D, char* ws, const GroupShape& L, hipStream_t s) {
    constexpr int E = Mma<T>::E;
    const bool y16 = rows16<T>(D.dY, D.lddy, D.dout), x16 = rows16<T>(D.X, D.ldx, D.di);
    const bool al = y16 && D.di % E == 0 && a16(D.W);   // dX
    const GroupList rows = row_list(D, L.rows, al);
    const bool want = D.dX && D.n > 0;
    hipError_t e = want || D.dW ? lists_go(D, want ? &rows : nullptr, D.dW ? &L.cuts : nullptr, ws, s) : hipSuccess;
    if (e != hipSuccess) return e;
    if (want) {
        const ListArgs Q = list_args(D, rows, ws, false);
        MainArgs M{};
        M.U = D.dY;
        M.ldu = D.lddy;
        M.W = D.W;
        M.order = D.order;
        M.count = Q.count;
        M.items = Q.items;
        M.Y = D.dX;
        M.K = D.dout;
        M.P = D.di;
        M.y4 = D.di % 4 == 0 && a16(D.dX);
        e = main_go<T, T, true>(M, rows, al, s);
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
        G.o4 = D.di % 4 == 0 && a16(D.dW);
        if (L.cuts.max_items > 0) {
            if (!(x16 && y16)) e = grad_tile<T, 128, 128, 2, 2, false>(G, L.cuts.max_items, s);
            else if (L.grad_tile == 256) e = grad_tile<T, 256, 256, 2, 4, true>(G, L.cuts.max_items, s);
            else e = grad_tile<T, 128, 128, 2, 2, true>(G, L.cuts.max_items, s);
            if (e != hipSuccess) return e;
        }
        const int64_t gx = ((int64_t)D.dout * D.di + 1023) / 1024;
        hipLaunchKernelGGL((k_gr_join<T>), dim3((unsigned)(gx < 1024 ? gx : 1024), (unsigned)(D.k < 1024 ? D.k : 1024)),
                           dim3(256), 0, s, G);
        e = hipGetLastError();
    }
    return e;
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
        const int64_t tall = (n + 255) / 256, wide = ((backward ? di : dout) + 255) / 256;
        L.rows.size = n >= 64 * met && tall * wide >= 64 ? 256 : 64;
        L.rows.max_items = group_items(n, k, 64) + 1;   // 64: the least size of a tile
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
