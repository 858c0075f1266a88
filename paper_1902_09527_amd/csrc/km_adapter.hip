// A shared projection with one low-rank adapter per cluster:
//   h = A_c x,  y = W x + s_c B_c h,
// and its gradients for rows and adapters (W is frozen):
//   g = s_c B_c^T dy,  dx = W^T dy + A_c^T g,
//   dA_c = sum g x^T,  dB_c = s_c sum dy h^T  over the cluster's rows.
//
// Rows are taken in cluster order (places), so a tile of rows meets few
// clusters.  The inner products (h, g) are formed first: they are r wide, and
// one pass over the rows forms them.  The shared product is a tiled matrix
// product over the places whose contraction continues past the shared width
// with the r inner products against each cluster's adapter: the adapter's
// term costs r more steps of the same accumulators and no pass over the
// results.  The adapters' gradients contract over a cluster's rows; long
// clusters are cut into chunks whose float32 sums are joined in order.
//
// Sums are float32 (matrix-core accumulators), and s h and g keep their float32
// values between the two products: as an operand of the 16-bit matrix cores such
// a value v is two, v rounded and the remainder rounded (16 bits together in
// bfloat16, 22 in float16), and float16's narrow exponents are met by a power of
// two that is taken out first and multiplied back into the float32 product.  H
// is rounded once, as the result that it is, and dB is the product with that H.
#include <limits.h>
#include <math.h>

#include "km_tile.h"

namespace km {

namespace {

// S, the inner products that the second product takes: per place and step of 16
// indexes of r the 16 values (float32), or their 16 upper and 16 lower parts
// (16 bits), which meet the same 16 of the adapter; zero past r.
constexpr int kStep = 16;
template <class T>
constexpr int kStepElems = sizeof(T) == 2 ? 2 * kStep : kStep;
template <class T>
constexpr bool kShifted = std::is_same_v<T, _Float16>;

// The power of two that is taken out of float16 parts, m the largest finite
// magnitude among their values: m is left between 2^14 and 2^15, so the two parts
// of v are off by at most 2^-22 |v| + 2^-39 m.
__device__ __forceinline__ int f16_shift(float m) {
    const int e = __builtin_amdgcn_frexp_expf(m);
    return (e > -100 ? e : -100) - 15;
}
__device__ __forceinline__ float finite_max(float m, float v) { return fmaxf(m, fabsf(v) < INFINITY ? fabsf(v) : 0.0f); }

// Consecutive values of a step (`step`: its first element), from index i on.
// The lower part of what is not finite is nothing.
template <class T, int N>
__device__ __forceinline__ void put_step(T* step, int i, const float (&v)[N], int shift) {
    Vec<T, N> hi, lo;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float x = kShifted<T> ? ldexpf(v[e], -shift) : v[e];
        hi.e[e] = from_f32<T>(x);
        if constexpr (sizeof(T) == 2) {
            const float up = to_f32(hi.e[e]);
            lo.e[e] = fabsf(up) < INFINITY ? from_f32<T>(x - up) : (T)0.0f;
        }
    }
    *reinterpret_cast<Vec<T, N>*>(step + i) = hi;
    if constexpr (sizeof(T) == 2) *reinterpret_cast<Vec<T, N>*>(step + kStep + i) = lo;
}

// --------------------------------------------------------------------------
// Chunks of clusters, for the adapters' gradients.

struct Item {
    int32_t c, p0, p1, slot;   // places p0 .. p1 of cluster c; slot: partial sum to write, -1: the result itself
};

// Chunks of every cluster, in order.
struct ListArgs {
    const int32_t* offsets;
    int32_t k, chunk;
    int32_t* count;      // items
    Item* items;
    int32_t *first, *num;   // per cluster: first partial slot, chunks (0: empty)
};

// By a block of 256 threads; s: 8 words of LDS.
__device__ __forceinline__ void list_chunks(const ListArgs& A, int* s) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int items = 0, slots = 0;   // so far
    for (int c0 = 0; c0 < A.k; c0 += 256) {
        const int c = c0 + tid;
        const int a = c < A.k ? A.offsets[c] : 0, b = c < A.k ? A.offsets[c + 1] : 0;
        const int ni = (b - a + A.chunk - 1) / A.chunk, ns = ni > 1 ? ni : 0;
        int xi = ni, xs = ns;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int ui = __shfl_up(xi, o), us = __shfl_up(xs, o);
            if (lane >= o) xi += ui, xs += us;
        }
        if (lane == 63) s[wave] = xi, s[4 + wave] = xs;
        __syncthreads();
        int bi = items, bs = slots;
        for (int w = 0; w < 4; ++w) {
            if (w < wave) bi += s[w], bs += s[4 + w];
            items += s[w];
            slots += s[4 + w];
        }
        bi += xi - ni;
        bs += xs - ns;
        if (c < A.k) {
            A.first[c] = bs;
            A.num[c] = ni;
            for (int q = 0; q < ni; ++q) {
                const int p = a + q * A.chunk;
                A.items[bi + q] = Item{c, p, b - p < A.chunk ? b : p + A.chunk, ni > 1 ? bs + q : -1};
            }
        }
        __syncthreads();
    }
    if (tid == 0) A.count[0] = items;
}

// --------------------------------------------------------------------------
// Inner products: S[place] = s_c Q_c u (in steps, rp elements a place) and, if H
// is not null, H[row] = Q_c u.  16 places a block; its four waves
// share the contraction, their sums are added in wave order through LDS.
// TR = false: Q_c is r x K (rows along the contraction); true: K x r, brought
// through LDS, a wave's own part, and read transposed.  The clusters of a block
// follow one another.  Bound by the latency of its few rounds of loads: 8192 x
// 2048 bf16, 64 clusters, r = 16: 18 us forward, 15 backward (the rows are 7 us
// of memory time); 16384 x 4096 float16, r = 32: 66 to 73 us.
struct InnerArgs {
    const void* U;
    int64_t ldu;
    const void* Q;
    const int32_t *order, *sids, *offsets;
    const float* scale;
    void *S, *H;
    int32_t* shift;   // float16: per place and step
    int64_t n;
    int32_t K, r, rp, u16, q16, h4;   // u16 / q16: rows of U / Q can be read 16 bytes at a time; h4: H written by fours
};

template <class T, int RF, bool TR, bool AL, bool QAL>
__global__ __launch_bounds__(256) void k_ad_inner(InnerArgs A, ListArgs L) {
    constexpr int E = Mma<T>::E, KS = 4 * E, VPR = RF * 16 / E;
    constexpr int UN = RF <= 2 ? 4 : RF == 4 ? 2 : 1;   // steps of a wave in flight
    constexpr int NQ = (KS * VPR + 63) / 64;            // chunks a lane of one step's K x r operand
    __shared__ f32x4 s_red[4][RF][64];
    __shared__ __align__(16) char s_q[TR ? 4 : 1][TR ? UN * KS * VPR * 16 : 16];
    if (TR && blockIdx.x == gridDim.x - 1) {   // one more block: the chunks of the adapters' gradients
        list_chunks(L, reinterpret_cast<int*>(s_q));
        return;
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, li = lane & 15;
    const int64_t p0 = (int64_t)blockIdx.x * 16;
    const int64_t place = p0 + li;
    const bool in = place < A.n;
    const int mine = in ? A.sids[place] : -1;
    const int64_t row = in ? row_of(A.order, place) : 0;
    const T* u = static_cast<const T*>(A.U) + row * A.ldu;
    const int steps = (A.K + KS - 1) / KS, steps_r = (A.r + kStep - 1) / kStep;
    int c = __builtin_amdgcn_readfirstlane(A.sids[p0]);
    while (c >= 0) {
        f32x4 acc[RF];
#pragma unroll
        for (int j = 0; j < RF; ++j) acc[j] = f32x4{0, 0, 0, 0};
        const T* q = static_cast<const T*>(A.Q) + (int64_t)c * A.r * A.K;
        for (int s = wave * UN; s < steps; s += 4 * UN) {   // steps past the last are of zeros
            u32x4 b[UN];
#pragma unroll
            for (int x = 0; x < UN; ++x) {
                const int64_t k0 = (int64_t)(s + x) * KS + g * E;
                b[x] = AL ? chunk_aligned(u, k0, A.K) : chunk_guarded(u, k0, A.K);
            }
            if constexpr (TR) {
                u32x4 v[UN][NQ];
#pragma unroll
                for (int x = 0; x < UN; ++x)
#pragma unroll
                    for (int y = 0; y < NQ; ++y) {
                        const int z = y * 64 + lane, kk = z / VPR;
                        const int64_t k = (int64_t)(s + x) * KS + kk;
                        if constexpr (QAL)
                            v[x][y] = chunk_aligned(q + k * A.r, z % VPR * E, A.r, k < A.K);
                        else
                            v[x][y] = only_if(k < A.K, chunk_guarded(q + (k < A.K ? k : 0) * A.r, z % VPR * E, A.r));
                    }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int x = 0; x < UN; ++x)
#pragma unroll
                    for (int y = 0; y < NQ; ++y) {
                        const int z = y * 64 + lane, kk = z / VPR;
                        if (kk < KS)
                            *reinterpret_cast<u32x4*>(s_q[wave] + ((x * KS + kk) * VPR + swz_tr<T, VPR>(kk, z % VPR)) * 16) =
                                v[x][y];
                    }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // the wave's own part of LDS
#pragma unroll
                for (int x = 0; x < UN; ++x)
#pragma unroll
                    for (int j = 0; j < RF; ++j)
                        acc[j] = Mma<T>::mma(read_tr<T, VPR>(s_q[wave], x * KS, tr_lane<T, VPR>(j * 16, lane)), b[x],
                                             acc[j]);
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            } else {
                u32x4 a[UN][RF];
#pragma unroll
                for (int x = 0; x < UN; ++x)
#pragma unroll
                    for (int j = 0; j < RF; ++j) {
                        const int rr = j * 16 + li;   // rows past r give results that are not kept
                        const T* src = q + (int64_t)(rr < A.r ? rr : 0) * A.K;
                        const int64_t k0 = (int64_t)(s + x) * KS + g * E;
                        a[x][j] = QAL ? chunk_aligned(src, k0, A.K) : chunk_guarded(src, k0, A.K);
                    }
                __builtin_amdgcn_sched_barrier(0);   // all of them are issued before the first is waited for
#pragma unroll
                for (int x = 0; x < UN; ++x)
#pragma unroll
                    for (int j = 0; j < RF; ++j) acc[j] = Mma<T>::mma(a[x][j], b[x], acc[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < RF; ++j) s_red[wave][j][lane] = acc[j];
        __syncthreads();
        const float sc = A.scale ? A.scale[c] : 1.0f;
        for (int j = wave; j < steps_r; j += 4) {
            f32x4 v = (s_red[0][j][lane] + s_red[1][j][lane]) + (s_red[2][j][lane] + s_red[3][j][lane]);
            const int r0 = j * kStep + g * 4;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (r0 + i >= A.r) v[i] = 0.0f;
            const float w[4] = {v[0] * sc, v[1] * sc, v[2] * sc, v[3] * sc};
            int shift = 0;
            if constexpr (kShifted<T>) {
                float m = 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i) m = finite_max(m, w[i]);
                m = fmaxf(m, __shfl_xor(m, 16));
                shift = f16_shift(fmaxf(m, __shfl_xor(m, 32)));
            }
            if (mine == c) {
                if (A.H) store4(static_cast<T*>(A.H) + row * A.r, r0, A.r, v, A.h4);
                put_step(static_cast<T*>(A.S) + place * A.rp + j * kStepElems<T>, g * 4, w, shift);
                if (kShifted<T> && g == 0) A.shift[place * steps_r + j] = shift;
            }
        }
        __syncthreads();
        const int64_t next = A.offsets[c + 1];
        c = next < p0 + 16 && next < A.n ? __builtin_amdgcn_readfirstlane(A.sids[next]) : -1;
    }
    if (in && mine < 0)   // rows in no cluster
        for (int j = wave; j < steps_r; j += 4) {
            if (A.H) store4(static_cast<T*>(A.H) + row * A.r, j * kStep + g * 4, A.r, f32x4{0, 0, 0, 0}, A.h4);
            put_step(static_cast<T*>(A.S) + place * A.rp + j * kStepElems<T>, g * 4, {0.0f, 0.0f, 0.0f, 0.0f}, 0);
            if (kShifted<T> && g == 0) A.shift[place * steps_r + j] = 0;
        }
}

// --------------------------------------------------------------------------
// The shared product over places with the adapters' term:
//   Y[row] = V u + Q_c S[place],  V = W (P x K) forward, W^T (W is K x P) with TR.
// A tile is TM places x TN columns, WR x WC waves; the contraction goes in
// stages of 128 bytes a row, loaded to LDS (NS stages) while the one before is
// used.
//
// 256 x 256 with 8 waves: the most products a byte loaded that registers and
// LDS hold (128 accumulators a lane, 128 KB of stages).  16384 x 4096 x 8192
// float16: 880 to 1006 us by the clock the card keeps (1.09 to 1.25 PFLOP/s; the
// library's product alone 813 us); 8192 x 2048 x 2048 bf16: 64 us forward, 64 to
// 67 backward (1.03 to 1.07 PFLOP/s; library 54), of which some 15 us are a
// tile's start and end.  The matrix cores are busy 66 % of a clock that falls to
// 1.7 GHz under this load: half of the stage loads taken out saves 8 %, L2 hits
// for all of them 6 %, so it is the card's power that is left to save.
// float32, 100,003 x 256 x 256: 143 to 150 us (90 TFLOP/s; 8 stages a tile).
struct MainArgs {
    const void* U;
    int64_t ldu;
    const void *W, *Q, *S;
    const int32_t* shift;   // float16: per place and step of S
    const int32_t *order, *sids;
    void* Y;
    int64_t n;
    int32_t K, P, r, rp, q16, y4, y16;   // y4 / y16: Y can be written 4 elements / 16 bytes at a time
    int32_t tm, tn;   // tiles
    int64_t ldw;      // row stride of W
    int32_t splits;   // parts of the contraction, a block each; more than one: sums to part
    float* part;      // splits x n x P, by place
};

template <class T, int TM, int TN, int WR, int WC, int NS, bool TR, bool AL>
__global__ __launch_bounds__(64 * WR * WC) void k_ad_main(MainArgs A) {
    constexpr int E = Mma<T>::E, KS = 4 * E, BK = 2 * KS, NT = 64 * WR * WC;
    constexpr int FR = TM / WR / 16, FC = TN / WC / 16;
    constexpr int NU = TM * 8 / NT, NW = TN * 8 / NT, CPR = TN / E;
    constexpr int kStage = (TM + TN) * 128;
    constexpr int kLaterShifts = TM / WR < 64 ? 64 : TM / WR;   // a wave's, whole loads
    // A ring of NS stages: TM rows of U, then TN rows (TR: BK rows) of W; then the
    // first step of the places' inner products, their rows and clusters; float16:
    // the powers of two of the first step, and of a later one by wave.
    extern __shared__ __align__(16) char s_tiles[];
    char* s_inner = s_tiles + NS * kStage;
    int32_t* s_rows = reinterpret_cast<int32_t*>(s_inner + TM * 64);
    int32_t* s_ids = s_rows + TM;
    int32_t* s_shift = s_ids + TM;
    const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, li = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wr = wave / WC, wc = wave % WC;

    // Consecutive tiles go to one XCD (blocks are dealt over 8), down 4 tiles
    // of places before the next columns.
    const int64_t tiles = (int64_t)A.tm * A.tn * A.splits, per = (tiles + 7) / 8;
    int64_t t = (blockIdx.x % 8) * per + blockIdx.x / 8;
    if (blockIdx.x / 8 >= per || t >= tiles) return;
    // This block's stages k_first .. of the contraction.
    const int all = (A.K + BK - 1) / BK, share = (all + A.splits - 1) / A.splits, split = (int)(t % A.splits);
    t /= A.splits;
    const int k_first = split * share, nk = all - k_first < share ? all - k_first : share;   // >= 1, as the host sees to
    const int64_t grp = t / (4 * (int64_t)A.tn), m0 = grp * 4;
    const int gm = A.tm - m0 < 4 ? (int)(A.tm - m0) : 4;
    const int64_t in_grp = t - grp * 4 * A.tn;
    const int64_t bm = (m0 + in_grp % gm) * TM, bn = in_grp / gm * TN;
    const int64_t w0 = bm + wr * (TM / WR), cb = bn + wc * (TN / WC);

    // Where a thread's chunks of a stage come from: pointers that move on with
    // the stages (AL), the place in the stage being fixed.
    const T* up[NU];
    const T* wp[NW];
    const int uc = swz(tid / 8, tid % 8) * E;   // NT / 8 rows further on the swizzle is the same
    static_assert(NT % 128 == 0, "");
#pragma unroll
    for (int i = 0; i < NU; ++i) {
        int64_t place = bm + (i * NT + tid) / 8;
        if (place >= A.n) place = A.n - 1;   // not stored
        const int64_t row = row_of(A.order, place);
        up[i] = static_cast<const T*>(A.U) + row * A.ldu + uc + (int64_t)k_first * BK;
        if (tid % 8 == 0) {
            s_rows[(i * NT + tid) / 8] = (int32_t)row;
            s_ids[(i * NT + tid) / 8] = A.sids[place];
            if constexpr (kShifted<T>) s_shift[(i * NT + tid) / 8] = A.shift[place * (A.rp / KS)];
        }
    }
#pragma unroll
    for (int i = 0; i < NW; ++i) {
        const int q = i * NT + tid;
        if constexpr (TR) {
            const int kk = q / CPR;
            wp[i] = static_cast<const T*>(A.W) + ((int64_t)k_first * BK + kk) * A.ldw + bn + swz_tr<T, CPR>(kk, q % CPR) * E;
        } else {
            int64_t col = bn + q / 8;
            if (col >= A.P) col = A.P - 1;   // not stored
            wp[i] = static_cast<const T*>(A.W) + col * A.ldw + uc + (int64_t)k_first * BK;
        }
    }
    // Stages (of this block) without a chunk past the contraction's end or the last column.
    const int k_left = A.K - k_first * BK, whole = !TR || bn + TN <= A.P ? k_left / BK : 0;

    // Chunk i of stage kt (of NU + NW a thread) to LDS; guard: it may lie past an end.
    auto load = [&](int i, int kt, char* buf, bool guard) {
        if (i < NU) {
            if constexpr (AL) {
                const void* src = !guard || kt * BK + uc < k_left ? (const void*)up[i] : (const void*)zero_chunk;
                load_lds16(src, buf + (i * NT + wave * 64) * 16);
                up[i] += BK;
            } else {
                *reinterpret_cast<u32x4*>(buf + (i * NT + tid) * 16) =
                    chunk_guarded(up[i] - uc, (int64_t)kt * BK + uc, k_left);
            }
            return;
        }
        i -= NU;
        const int q = i * NT + tid;
        char* wb = buf + TM * 128;
        if constexpr (TR) {
            const int kk = q / CPR;
            const int64_t col = bn + swz_tr<T, CPR>(kk, q % CPR) * E;
            if constexpr (AL) {
                const bool in = !guard || (kt * BK + kk < k_left && col < A.P);
                load_lds16(in ? (const void*)wp[i] : (const void*)zero_chunk, wb + (i * NT + wave * 64) * 16);
                wp[i] += BK * A.ldw;
            } else {
                const int64_t k = (int64_t)(k_first + kt) * BK + kk;
                *reinterpret_cast<u32x4*>(wb + q * 16) = only_if(
                    k < A.K, chunk_guarded(static_cast<const T*>(A.W) + (k < A.K ? k : 0) * A.ldw, col, A.P));
            }
        } else {
            if constexpr (AL) {
                const void* src = !guard || kt * BK + uc < k_left ? (const void*)wp[i] : (const void*)zero_chunk;
                load_lds16(src, wb + (i * NT + wave * 64) * 16);
                wp[i] += BK;
            } else {
                *reinterpret_cast<u32x4*>(wb + q * 16) = chunk_guarded(wp[i] - uc, (int64_t)kt * BK + uc, k_left);
            }
        }
    };
    auto load_all = [&](int kt, char* buf) {
#pragma unroll
        for (int i = 0; i < NU + NW; ++i) load(i, kt, buf, kt >= whole);
    };

#pragma unroll
    for (int kt = 0; kt < NS; ++kt)
        if (kt < nk) load_all(kt, s_tiles + kt * kStage);
#pragma unroll
    for (int i = 0; i < TM * 4 / NT; ++i) {
        const int q = i * NT + tid;
        const int64_t place = bm + q / 4 < A.n ? bm + q / 4 : A.n - 1;
        load_lds16(static_cast<const T*>(A.S) + place * A.rp + q % 4 * E, s_inner + (i * NT + wave * 64) * 16);
    }

    f32x4 acc[FR][FC];
#pragma unroll
    for (int f = 0; f < FR; ++f)
#pragma unroll
        for (int h = 0; h < FC; ++h) acc[f][h] = f32x4{0, 0, 0, 0};

    // A lane's places in a stage; the second half of a row is 64 bytes off
    // (one bit of the swizzled chunk), 16 rows are 2048 bytes.
    const int ua = (wr * (TM / WR) + li) * 128 + swz(li, g) * 16;
    int wa[TR ? FC : 1];
    if constexpr (TR) {
#pragma unroll
        for (int h = 0; h < FC; ++h) wa[h] = TM * 128 + tr_lane<T, CPR>(wc * (TN / WC) + h * 16, lane);
    } else {
        wa[0] = TM * 128 + (wc * (TN / WC) + li) * 128 + swz(li, g) * 16;
    }
    struct Frags {
        u32x4 b[FR], a[FC];
    };
    // Operand i of half s of a stage: first the columns' (TR: read_cols), then the rows'.
    auto read = [&](Frags& F, int i, const char* buf, int s) {
        if (i < FC) {
            if constexpr (!TR) F.a[i] = *reinterpret_cast<const u32x4*>(buf + (wa[0] ^ (s * 64)) + i * 2048);
        } else {
            F.b[i - FC] = *reinterpret_cast<const u32x4*>(buf + (ua ^ (s * 64)) + (i - FC) * 2048);
        }
    };
    auto read_cols = [&](Frags& F, const char* buf, int s) {
        if constexpr (TR) {
            if (s == 0) read_tr_wait<T, CPR, 0>(F.a, buf, wa);
            else read_tr_wait<T, CPR, KS>(F.a, buf, wa);
        }
    };

    // Operands are read from LDS half a stage ahead of their products, and a
    // stage is loaded while the one before it is multiplied.  The barrier of a
    // stage stands between its two halves of products, when the second half's
    // operands are in registers, and loads, reads and products are issued in
    // turns (kParts of each), so that the matrix cores do not wait for either.
    constexpr int kParts = FR % 4 == 0 && (FR + FC) % 4 == 0 ? 4 : 2;
    constexpr int kLoads = (NU + NW) / kParts, kReads = (FR + FC) / kParts;
    static_assert((NU + NW) % kParts == 0 && (FR + FC) % kParts == 0 && FR % kParts == 0, "");
    // The products of F; F2 read from buf2 (half s2); kl >= 0: stage kl loaded into bufl.
    auto half = [&](const Frags& F, Frags& F2, const char* buf2, int s2, int kl, char* bufl, bool guard) {
#pragma unroll
        for (int q = 0; q < kParts; ++q) {
            if (kl >= 0) {
#pragma unroll
                for (int i = 0; i < kLoads; ++i) load(q * kLoads + i, kl, bufl, guard);
            }
#pragma unroll
            for (int i = 0; i < kReads; ++i) read(F2, q * kReads + i, buf2, s2);
#pragma unroll
            for (int f = q * (FR / kParts); f < (q + 1) * (FR / kParts); ++f)
#pragma unroll
                for (int h = 0; h < FC; ++h) acc[f][h] = Mma<T>::mma(F.a[h], F.b[f], acc[f][h]);
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
        arrived();
        __builtin_amdgcn_sched_barrier(0);
        half(F0, F1, cur, 1, -1, cur, false);
        turn(last);
        __builtin_amdgcn_sched_barrier(0);
        // After the last stage the reads are of what the buffer held before, and are not used.
        half(F1, F0, nxt, 0, !last ? kt + NS : kt + NS < nk ? kt + NS : -1, cur, last);
    };
    int kt = 0;
    for (; kt + NS < whole && kt + NS < nk; ++kt) stage(kt, false);
    for (; kt + 1 < nk; ++kt) stage(kt, true);

    // The adapters' operand of one cluster and step of r (16 bits: twice, for the
    // upper and the lower parts of the inner products), the wave's CN columns, to its part of the buffer of the stage before the last (two
    // places in turn).  The first is loaded beside the last stage.
    constexpr int CN = TN / WC;
    char* s_q = s_tiles + (at == 0 ? NS - 1 : at - 1) * kStage + wave * (2 * CN * 64);
    static_assert(WR * WC * 2 * CN * 64 <= kStage, "");
    auto fetch = [&](int c, int k0, int buf) {
        char* to = s_q + buf * CN * 64;
        if (A.q16) {
#pragma unroll
            for (int i = 0; i < CN * 4 / 64; ++i) {
                const int q = i * 64 + lane;
                const T* src;
                bool in;
                if constexpr (TR) {
                    const int kk = q / (CN / E), rr = k0 + kk % kStep;
                    const int64_t col = cb + swz_tr<T, CN / E>(kk, q % (CN / E)) * E;
                    in = rr < A.r && col < A.P;
                    src = static_cast<const T*>(A.Q) + ((int64_t)c * A.r + rr) * A.P + col;
                } else {
                    const int64_t col = cb + q / 4;
                    const int rr = k0 + swz4(q / 4, q % 4) * E % kStep;
                    in = col < A.P && rr < A.r;
                    src = static_cast<const T*>(A.Q) + ((int64_t)c * A.P + col) * A.r + rr;
                }
                load_lds16(in ? (const void*)src : (const void*)zero_chunk, to + i * 1024);
            }
        } else {
#pragma unroll 1
            for (int q = lane; q < CN * 4; q += 64) {
                u32x4 v;
                if constexpr (TR) {
                    const int kk = q / (CN / E), rr = k0 + kk % kStep;
                    v = only_if(rr < A.r,
                                chunk_guarded(static_cast<const T*>(A.Q) + ((int64_t)c * A.r + (rr < A.r ? rr : 0)) * A.P,
                                              cb + swz_tr<T, CN / E>(kk, q % (CN / E)) * E, A.P));
                } else {
                    const int64_t col = cb + q / 4 < A.P ? cb + q / 4 : 0;   // columns past P are not stored
                    v = chunk_guarded(static_cast<const T*>(A.Q) + ((int64_t)c * A.P + col) * A.r,
                                      k0 + swz4(q / 4, q % 4) * E % kStep, A.r);
                }
                *reinterpret_cast<u32x4*>(to + q * 16) = v;
            }
        }
    };
    // The adapters' term belongs to the first part of the contraction.  It goes
    // over the steps of r, and in each over the clusters of the wave's places
    // (which are in cluster order, -1 last).  The first two operands:
    constexpr int RM = TM / WR;
    int c_first = -1, c_second = -1;
    if (w0 < A.n && split == 0) {
        const int* ids = s_ids + (w0 - bm);
        c_first = __builtin_amdgcn_readfirstlane(ids[0]);
#pragma unroll
        for (int i = (RM + 63) / 64 - 1; i >= 0; --i) {
            const int at = i * 64 + lane, id = at < RM && w0 + at < A.n ? ids[at] : -1;
            const uint64_t m = __ballot(id > c_first);
            if (m) c_second = __builtin_amdgcn_readlane(id, __builtin_ctzll(m));
        }
    }
    int k_second = 0;
    if (c_second < 0 && A.r > kStep) c_second = c_first, k_second = kStep;
    if (c_first >= 0) fetch(c_first, 0, 0);
    if (c_second >= 0) fetch(c_second, k_second, 1);
    char* s_later = s_tiles + at * kStage + wave * (RM * 64);   // in the last stage's buffer
    static_assert(TM * WC * 64 <= kStage, "");
    stage(kt, true);
    // The wave's inner products of a later step, to its part of the last stage's
    // buffer, which no wave reads any more.  The second step's are on their way
    // during the first.
    constexpr int kLater = RM / 16 + (kShifted<T> ? (RM + 63) / 64 : 0), kOperand = CN * 4 / 64;
    auto fetch_later = [&](int k0) {
#pragma unroll
        for (int i = 0; i < RM / 16; ++i) {
            const int q = i * 64 + lane;
            const int64_t place = w0 + q / 4 < A.n ? w0 + q / 4 : A.n - 1;
            load_lds16(static_cast<const T*>(A.S) + place * A.rp + k0 / kStep * KS + q % 4 * E, s_later + i * 1024);
        }
        if constexpr (kShifted<T>) {
#pragma unroll
            for (int i = 0; i < (RM + 63) / 64; ++i) {
                const int64_t place = w0 + i * 64 + lane < A.n ? w0 + i * 64 + lane : A.n - 1;
                __builtin_amdgcn_global_load_lds((const KM_GLOBAL void*)(A.shift + place * (A.rp / KS) + k0 / kStep),
                                                 (KM_LDS void*)(s_shift + TM + wave * kLaterShifts + i * 64), 4, 0, 0);
            }
        }
    };
    if (c_first >= 0 && A.r > kStep) fetch_later(kStep);

    // A lane keeps the sum only where its place is of the cluster, so that nothing
    // of one cluster's adapter reaches another's rows.  The next two operands are
    // on their way during the products of one.
    int mine[FR];
#pragma unroll
    for (int f = 0; f < FR; ++f) mine[f] = w0 + f * 16 + li < A.n ? s_ids[w0 - bm + f * 16 + li] : -1;
    auto after = [&](int& c, int& k0) {   // the next cluster and step; c = -1: none
        int next = -1;
#pragma unroll
        for (int f = FR - 1; f >= 0; --f) {
            const uint64_t m = __ballot(mine[f] > c);
            if (m) next = __builtin_amdgcn_readlane(mine[f], __builtin_ctzll(m));
        }
        c = next;
        if (next < 0 && (k0 += kStep) < A.r) c = c_first;
    };
    const char* s_b = s_inner + (w0 - bm) * 64;
    const int32_t* s_e = s_shift + (w0 - bm);
    bool first = true;
    for (int buf = 0, c = c_first, k0 = 0, next = c_second, k_next = k_second; c >= 0; buf ^= 1, first = false) {
        // This operand is in the wave's own part of LDS (and the inner products of
        // its step, which were asked for before the operand that follows it); what
        // was asked for later may be on its way.
        if (!A.q16) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        else if (first && A.r > kStep) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kOperand + kLater) : "memory");
        else if (next >= 0) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kOperand) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        u32x4 a[FC];
        const char* q = s_q + buf * CN * 64;
        if constexpr (TR) {
            int qa[FC];
#pragma unroll
            for (int h = 0; h < FC; ++h) qa[h] = tr_lane<T, CN / E>(h * 16, lane);
            read_tr_wait<T, CN / E, 0>(a, q, qa);
        } else {
#pragma unroll
            for (int h = 0; h < FC; ++h)
                a[h] = *reinterpret_cast<const u32x4*>(q + ((h * 16 + li) * 4 + swz4(li, g)) * 16);
        }
        int c_after = next, k_after = k_next;
        if (next >= 0) after(c_after, k_after);
        if (c_after >= 0) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // read before it is overwritten
            fetch(c_after, k_after, buf);
        }
#pragma unroll
        for (int f = 0; f < FR; ++f) {
            const bool is = mine[f] == c;
            if (!__ballot(is)) continue;
            const u32x4 b = *reinterpret_cast<const u32x4*>(s_b + (f * 16 + li) * 64 + g * 16);
            float two = 1.0f;
            if constexpr (kShifted<T>) two = ldexpf(1.0f, s_e[f * 16 + li]);
#pragma unroll
            for (int h = 0; h < FC; ++h) {
                f32x4 d = Mma<T>::mma(a[h], b, kShifted<T> ? f32x4{0, 0, 0, 0} : acc[f][h]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (kShifted<T>) d[i] = fmaf(d[i], two, acc[f][h][i]);
                    acc[f][h][i] = is ? d[i] : acc[f][h][i];
                }
            }
        }
        if (next >= 0 && k_next != k0) {   // on to the next step's inner products
            s_b = s_later;
            s_e = s_shift + TM + wave * kLaterShifts;
            if (k_next > kStep) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                fetch_later(k_next);
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            }
        }
        c = next;
        k0 = k_next;
        next = c_after;
        k_next = k_after;
    }

    // 16-bit results go through LDS so that 128 consecutive bytes of a row are
    // written at once (a lane holds 8): 8 rows an instruction, or one where rows
    // are not 16-byte aligned.
    if constexpr (sizeof(T) == 2 && CN == 64) {
        static_assert(RM * 128 * WR * WC <= NS * kStage, "");
        if (A.splits == 1) {    // the same for the whole grid
            __syncthreads();    // every wave is done with the stages and operands
            char* own = s_tiles + wave * (RM * 128);
#pragma unroll
            for (int f = 0; f < FR; ++f)
#pragma unroll
                for (int h = 0; h < FC; ++h) {
                    Vec<T, 4> o;
#pragma unroll
                    for (int i = 0; i < 4; ++i) o.e[i] = from_f32<T>(acc[f][h][i]);
                    const int row = f * 16 + li, ch = h * 2 + (g >> 1);
                    *reinterpret_cast<Vec<T, 4>*>(own + row * 128 + ((ch ^ (row & 7)) * 16) + (g & 1) * 8) = o;
                }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (!A.y16) {
                for (int row = 0; row < RM && w0 + row < A.n; ++row)
                    if (cb + lane < A.P)
                        static_cast<T*>(A.Y)[(int64_t)s_rows[w0 - bm + row] * A.P + cb + lane] =
                            *reinterpret_cast<const T*>(own + row * 128 + ((lane >> 3) ^ (row & 7)) * 16 + (lane & 7) * 2);
                return;
            }
            const int64_t col = cb + lane % 8 * 8;
#pragma unroll
            for (int i = 0; i < RM / 8; ++i) {
                const int row = i * 8 + lane / 8;
                const u32x4 v = *reinterpret_cast<const u32x4*>(own + row * 128 + ((lane % 8) ^ (row & 7)) * 16);
                if (w0 + row < A.n && col < A.P)
                    *reinterpret_cast<u32x4*>(static_cast<T*>(A.Y) + (int64_t)s_rows[w0 - bm + row] * A.P + col) = v;
            }
            return;
        }
    }
#pragma unroll
    for (int f = 0; f < FR; ++f) {
        const int64_t place = w0 + f * 16 + li;
        if (place >= A.n) continue;
        if (A.splits > 1) {
            float* y = A.part + ((int64_t)split * A.n + place) * A.P;
#pragma unroll
            for (int h = 0; h < FC; ++h) store4(y, cb + h * 16 + g * 4, A.P, acc[f][h], A.P % 4 == 0);
            continue;
        }
        T* y = static_cast<T*>(A.Y) + (int64_t)s_rows[place - bm] * A.P;
#pragma unroll
        for (int h = 0; h < FC; ++h) store4(y, cb + h * 16 + g * 4, A.P, acc[f][h], A.y4);
    }
}

// The parts of the contraction, added in order: a block a place and 1024 columns.
template <class T>
__global__ __launch_bounds__(256) void k_ad_sum(MainArgs A) {
    const int64_t place = blockIdx.x, col = ((int64_t)blockIdx.y * 256 + threadIdx.x) * 4;
    if (col >= A.P) return;
    T* y = static_cast<T*>(A.Y) + row_of(A.order, place) * A.P;
    const float* p = A.part + place * A.P + col;
    const int64_t step = A.n * A.P;
    f32x4 v{0, 0, 0, 0};
    if (A.P % 4 == 0) {
#pragma unroll 4
        for (int q = 0; q < A.splits; ++q) v += *reinterpret_cast<const f32x4*>(p + q * step);
    } else {
        for (int q = 0; q < A.splits; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (col + i < A.P) v[i] += p[q * step + i];
    }
    store4(y, col, A.P, v, A.y4);
}

// --------------------------------------------------------------------------
// Few rows, forward: the time is that of reading W (and the adapters) once.

struct FewArgs {
    const void* X;
    int64_t ldx;
    const void *W, *A, *B;
    const int32_t *order, *cl;   // cl: the cluster of every place (a plan's), or of every row (order null)
    const float* scale;
    void *S, *H, *Y;             // S: in steps; forward of few rows: float32, n x r
    int32_t* shift;              // float16: per place and step
    int64_t ldw;                 // row stride of W
    int32_t n, K, P, r, k, x16, q16, y4;
};

// The inner products of a place and step, a lane each of 16 (any others idle).
template <class T>
__device__ __forceinline__ void put_lanes(T* S, int32_t* shift, int64_t step, int i, float v) {
    int e = 0;
    if constexpr (kShifted<T>) {
        float m = finite_max(0.0f, v);
#pragma unroll
        for (int o = 1; o < kStep; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
        e = f16_shift(m);
        if (i == 0) shift[step] = e;
    }
    put_step(S + step * kStepElems<T>, i, {v}, e);
}

// h: a wave a (place, index), its lanes along the row.  STEP: a block of 16
// waves a place and step, for S in steps.
template <class T, bool STEP>
__global__ __launch_bounds__(STEP ? 1024 : 256) void k_ad_few_inner(FewArgs A) {
    constexpr int E = Mma<T>::E, kWaves = STEP ? kStep : 4;
    __shared__ float s_sum[kStep];
    const int lane = threadIdx.x & 63, wide = STEP ? (A.r + kStep - 1) / kStep * kStep : A.r;
    const int64_t w = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
    if (w >= (int64_t)A.n * wide) return;   // STEP: none, the grid is n wide / 16 blocks
    const int p = (int)(w / wide), j = (int)(w % wide);
    const int c = A.cl[p];
    const int64_t row = row_of(A.order, p);
    float sum = 0.0f;
    const bool in = (unsigned)c < (unsigned)A.k && j < A.r;
    if (in) {
        const T* x = static_cast<const T*>(A.X) + row * A.ldx;
        const T* a = static_cast<const T*>(A.A) + ((int64_t)c * A.r + j) * A.K;
        if (A.x16) {
#pragma unroll 4
            for (int k0 = lane * E; k0 < A.K; k0 += 64 * E) {
                const Vec<T, E> u = *reinterpret_cast<const Vec<T, E>*>(x + k0);
                const Vec<T, E> v = *reinterpret_cast<const Vec<T, E>*>(a + k0);
#pragma unroll
                for (int e = 0; e < E; ++e) sum = fmaf(to_f32(u.e[e]), to_f32(v.e[e]), sum);
            }
        } else {
#pragma unroll 4
            for (int k0 = lane; k0 < A.K; k0 += 64) sum = fmaf(to_f32(x[k0]), to_f32(a[k0]), sum);
        }
    }
    sum = group_sum<64>(sum);
    if (lane == 0) {
        if (j < A.r) static_cast<T*>(A.H)[row * A.r + j] = from_f32<T>(sum);
        const float s = in ? sum * (A.scale ? A.scale[c] : 1.0f) : 0.0f;
        if constexpr (STEP) s_sum[j % kStep] = s;
        else static_cast<float*>(A.S)[w] = s;
    }
    if constexpr (STEP) {
        __syncthreads();
        const int i = threadIdx.x;
        if (i < kStep) put_lanes(static_cast<T*>(A.S), A.shift, blockIdx.x, i, s_sum[i]);
    }
}


// g: a block a (place, 16 indexes), its threads along the contraction, a row
// of B_c each.  One more block lists the chunks.
template <class T>
__global__ __launch_bounds__(256) void k_ad_few_inner_t(FewArgs A, ListArgs L) {
    constexpr int E = Mma<T>::E;
    __shared__ float s_sum[4][16];
    if (blockIdx.x == gridDim.x - 1) {
        list_chunks(L, reinterpret_cast<int*>(s_sum));
        return;
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, jc = (A.r + kStep - 1) / kStep;
    const int p = (int)(blockIdx.x / jc), j0 = (int)(blockIdx.x % jc) * 16;
    const int c = A.cl[p];
    float acc[16] = {};
    if (c >= 0) {
        const T* x = static_cast<const T*>(A.X) + row_of(A.order, p) * A.ldx;
        const T* b = static_cast<const T*>(A.B) + (int64_t)c * A.K * A.r;
#pragma unroll 2
        for (int k = threadIdx.x; k < A.K; k += 256) {
            const float u = to_f32(x[k]);
#pragma unroll
            for (int q = 0; q < 16 / E; ++q) {
                const Vec<T, E> v = __builtin_bit_cast(
                    Vec<T, E>, A.q16 ? chunk_aligned(b + (int64_t)k * A.r, j0 + q * E, A.r)
                                     : chunk_guarded(b + (int64_t)k * A.r, j0 + q * E, A.r));
#pragma unroll
                for (int e = 0; e < E; ++e) acc[q * E + e] = fmaf(u, to_f32(v.e[e]), acc[q * E + e]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        acc[i] = group_sum<64>(acc[i]);
        if (lane == 0) s_sum[wave][i] = acc[i];
    }
    __syncthreads();
    const int i = threadIdx.x;
    if (i < 16) {
        const bool in = c >= 0 && j0 + i < A.r;
        const float s = (s_sum[0][i] + s_sum[1][i]) + (s_sum[2][i] + s_sum[3][i]);
        put_lanes(static_cast<T*>(A.S), A.shift, blockIdx.x, i, in ? s * (A.scale ? A.scale[c] : 1.0f) : 0.0f);
    }
}

// y: 16 columns a block, its 16 waves share the contraction; RF x 16 places.
// 48 rows of 4096 x 4096 bf16: 20 us (W once at the memory's rate: 7; every
// block reads all rows of X, 100 MB from L2), 1 row of 1024 x 1024: 4.7 us.  32
// columns a block halve that traffic but fill half of the chip: 26 us.
template <class T, int RF, bool AL>
__global__ __launch_bounds__(1024) void k_ad_few_main(FewArgs A) {
    constexpr int E = Mma<T>::E, KS = 4 * E, UN = AL ? 4 : 1, NWAVE = 16;
    __shared__ f32x4 s_red[NWAVE / 2][RF][64];
    const int lane = threadIdx.x & 63, g = lane >> 4, li = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t col0 = (int64_t)blockIdx.x * 16;
    const T* w = static_cast<const T*>(A.W) + (col0 + li < A.P ? col0 + li : A.P - 1) * A.ldw;   // columns past P: not stored
    const T* x[RF];
#pragma unroll
    for (int f = 0; f < RF; ++f) {
        const int p = f * 16 + li < A.n ? f * 16 + li : A.n - 1;
        x[f] = static_cast<const T*>(A.X) + row_of(A.order, p) * A.ldx;
    }
    f32x4 acc[RF];
#pragma unroll
    for (int f = 0; f < RF; ++f) acc[f] = f32x4{0, 0, 0, 0};
    const int steps = (A.K + KS - 1) / KS;
    for (int s = wave * UN; s < steps; s += NWAVE * UN) {   // steps past the last are of zeros
        u32x4 a[UN], b[UN][RF];
#pragma unroll
        for (int y = 0; y < UN; ++y) {
            const int64_t k0 = (int64_t)(s + y) * KS + g * E;
            a[y] = AL ? chunk_aligned(w, k0, A.K) : chunk_guarded(w, k0, A.K);
#pragma unroll
            for (int f = 0; f < RF; ++f) b[y][f] = AL ? chunk_aligned(x[f], k0, A.K) : chunk_guarded(x[f], k0, A.K);
        }
        __builtin_amdgcn_sched_barrier(0);   // all of them are issued before the first is waited for
#pragma unroll
        for (int y = 0; y < UN; ++y)
#pragma unroll
            for (int f = 0; f < RF; ++f) acc[f] = Mma<T>::mma(a[y], b[y][f], acc[f]);
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
        const int p = q * 16 + li;
        if (p >= A.n) continue;
        f32x4 v{0, 0, 0, 0};
#pragma unroll
        for (int y = 0; y < H; ++y) v += s_red[y][q][lane];
        const int c = A.cl[p];
        const int64_t o0 = col0 + g * 4;
        if ((unsigned)c < (unsigned)A.k) {
            const float* s = static_cast<const float*>(A.S) + (int64_t)p * A.r;
            const T* b[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                b[i] = static_cast<const T*>(A.B) + ((int64_t)c * A.P + (o0 + i < A.P ? o0 + i : 0)) * A.r;
            if (A.q16) {
                for (int j = 0; j < A.r; j += E) {
                    Vec<T, E> t[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) t[i] = *reinterpret_cast<const Vec<T, E>*>(b[i] + j);
#pragma unroll
                    for (int e = 0; e < E; ++e)
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[i] = fmaf(s[j + e], to_f32(t[i].e[e]), v[i]);
                }
            } else {
                for (int j = 0; j < A.r; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = fmaf(s[j], to_f32(b[i][j]), v[i]);
            }
        }
        store4(static_cast<T*>(A.Y) + row_of(A.order, p) * A.P, o0, A.P, v, A.y4);
    }
}

// --------------------------------------------------------------------------
// Gradients of the adapters: out_c = sum over the cluster's places of
// U[row] V[place or row]^T, U wide (P), V r wide.

struct GradArgs {
    const void* U;
    int64_t ldu;
    const void* V;           // dA: S, by place, in steps; dB: H, by row
    int64_t ldv;
    const int32_t* shift;    // float16, dA: per place and step
    const int32_t* order;
    const float* scale;      // per cluster, or null
    const int32_t* count;
    const Item* items;
    const int32_t *first, *num;
    void* out;               // WF: k x r x P, else k x P x r
    float* part;             // slots x r x P, each as out
    int32_t k, P, r, v16, o4, tiles;   // o4: out written by fours
};

// Bound by the latency of a chunk's stages: 8192 x 2048 bf16, 64 clusters, r =
// 16: 25 us for both gradients (rows: 14 us of memory time); 100,003 x 256
// float32: 57 us (43).  The two parts of S take twice the LDS of one: beyond r =
// 64 a compute unit has one block instead of two (8192 x 2048 float16, r = 128:
// the whole backward pass 235 us, 206 with g rounded to float16).
//
// 128 columns a block, 32 a wave; stages of 2 KS places, loaded while the one
// before is multiplied (the skinny operand through registers).  WF: the wide
// operand comes first (lanes hold four consecutive columns: dA), else second
// (four consecutive indexes of r: dB).
//
// dA's skinny operand is S: RF steps, in 16 bits of two operands each.  In
// float16 one power of two, the largest of the item's places, is taken out of all.
template <class T, int RF>
constexpr int kSkinny = RF * kStepElems<T> * 8 * Mma<T>::E * (int)sizeof(T);   // bytes of a stage

template <class T, int RF, bool WF, bool AL>
__device__ __forceinline__ void grad_block(const GradArgs& A, char (*s_u)[32 * 512], char (*s_v)[kSkinny<T, RF>]) {
    constexpr int E = Mma<T>::E, KS = 4 * E, BK = 2 * KS, TC = 128, CPR = TC / E;
    constexpr int VW = WF ? kStepElems<T> : 16, VPR = RF * VW / E;   // elements of 16 indexes, chunks a place
    constexpr int NU = BK * CPR / 256, NV = (BK * VPR + 255) / 256;
    constexpr bool kShift = WF && kShifted<T>;
    static_assert(BK * CPR * 16 == 32 * 512 && BK * VPR * 16 <= kSkinny<T, RF>, "");
    const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, li = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t total = (int64_t)A.count[0] * A.tiles;
    for (int64_t w = blockIdx.x; w < total; w += gridDim.x) {
        const Item it = A.items[w / A.tiles];
        const int64_t bc = (w % A.tiles) * TC;
        int64_t ur[NU], vr[NV];   // rows of the next stage to load
        u32x4 v[NV];
        int most = 0, ve[kShift ? NV : 1];
        const int steps = (A.r + kStep - 1) / kStep;
        if constexpr (kShift) {
            __shared__ int s_max[4];
            const int32_t* p = A.shift + (int64_t)it.p0 * steps;
            const int64_t size = (int64_t)(it.p1 - it.p0) * steps;
            most = INT_MIN;
            for (int64_t i = tid; i < size; i += 256) most = p[i] > most ? p[i] : most;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int other = __shfl_xor(most, o);
                most = other > most ? other : most;
            }
            if (lane == 0) s_max[wave] = most;
            __syncthreads();
#pragma unroll
            for (int q = 0; q < 4; ++q) most = s_max[q] > most ? s_max[q] : most;
        }
        auto rows = [&](int64_t p0) {
#pragma unroll
            for (int i = 0; i < NU; ++i) {
                const int64_t p = p0 + (i * 256 + tid) / CPR;
                ur[i] = row_of(A.order, p < it.p1 ? p : it.p0);
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int64_t p = p0 + (i * 256 + tid) / VPR, q = p < it.p1 ? p : it.p0;
                vr[i] = WF ? q : row_of(A.order, q);
            }
        };
        auto load = [&](int64_t p0, int buf) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int q = i * 256 + tid;
                const bool in = p0 + q / VPR < it.p1;
                const T* src = static_cast<const T*>(A.V) + vr[i] * A.ldv;
                if constexpr (WF) v[i] = only_if(in, chunk_aligned(src, q % VPR * E, A.ldv));
                else v[i] = only_if(in, chunk(src, q % VPR * E, A.r, A.v16));
                if constexpr (kShift) {
                    const int step = q % VPR * E / VW;
                    ve[i] = A.shift[vr[i] * steps + (step < steps ? step : 0)];
                }
            }
#pragma unroll
            for (int i = 0; i < NU; ++i) {
                const int q = i * 256 + tid, kk = q / CPR;
                const int64_t col = bc + swz_tr<T, CPR>(kk, q % CPR) * E;
                const bool in = p0 + kk < it.p1;
                const T* src = static_cast<const T*>(A.U) + ur[i] * A.ldu;
                if constexpr (AL)
                    load_lds16(in && col < A.P ? (const void*)(src + col) : (const void*)zero_chunk,
                               s_u[buf] + (i * 256 + wave * 64) * 16);
                else
                    *reinterpret_cast<u32x4*>(s_u[buf] + q * 16) = only_if(in, chunk_guarded(src, col, A.P));
            }
        };
        auto put = [&](int buf) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int q = i * 256 + tid, kk = q / VPR;
                if constexpr (kShift) {
                    Vec<T, E> x = __builtin_bit_cast(Vec<T, E>, v[i]);
#pragma unroll
                    for (int e = 0; e < E; ++e) x.e[e] = from_f32<T>(ldexpf(to_f32(x.e[e]), ve[i] - most));
                    v[i] = __builtin_bit_cast(u32x4, x);
                }
                if (kk < BK) *reinterpret_cast<u32x4*>(s_v[buf] + (kk * VPR + swz_tr<T, VPR>(kk, q % VPR)) * 16) = v[i];
            }
        };
        const int ua[2] = {tr_lane<T, CPR>(wave * 32, lane), tr_lane<T, CPR>(wave * 32 + 16, lane)};
        f32x4 acc[2][RF];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < RF; ++j) acc[h][j] = f32x4{0, 0, 0, 0};
        int buf = 0;
        rows(it.p0);
        load(it.p0, 0);
        rows(it.p0 + BK);
        put(0);
        for (int64_t p = it.p0; p < it.p1; p += BK, buf ^= 1) {
            // The stage has landed, and every wave is done with the other buffer.
            __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0) lgkmcnt(0)
            __syncthreads();
            if (p + BK < it.p1) {
                load(p + BK, buf ^ 1);
                rows(p + 2 * BK);
            }
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                u32x4 a[2];
                if (s == 0) read_tr_wait<T, CPR, 0>(a, s_u[buf], ua);
                else read_tr_wait<T, CPR, KS>(a, s_u[buf], ua);
                constexpr int all = RF * VW / 16, N = all < 4 ? all : 4;   // skinny operands, four at a time
#pragma unroll
                for (int j = 0; j < all; j += N) {
                    u32x4 b[N];
                    int at[N];
#pragma unroll
                    for (int i = 0; i < N; ++i) at[i] = tr_lane<T, VPR>((j + i) * 16, lane);
                    if (s == 0) read_tr_wait<T, VPR, 0>(b, s_v[buf], at);
                    else read_tr_wait<T, VPR, KS>(b, s_v[buf], at);
#pragma unroll
                    for (int i = 0; i < N; ++i)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            f32x4& d = acc[h][(j + i) * 16 / VW];
                            d = WF ? Mma<T>::mma(a[h], b[i], d) : Mma<T>::mma(b[i], a[h], d);
                        }
                }
            }
            if (p + BK < it.p1) put(buf ^ 1);
        }
        __syncthreads();   // both buffers are free for the next item
        const float sc = A.scale ? A.scale[it.c] : 1.0f;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < RF; ++j) {
                const int64_t cw = bc + wave * 32 + h * 16;
                const int64_t slot = it.slot < 0 ? it.c : it.slot;
                // WF: row rr of r, columns 4 g ..;  else row = column li, indexes 4 g ..
                const int64_t rr = WF ? j * 16 + li : cw + li, x0 = WF ? cw + g * 4 : j * 16 + g * 4;
                const int64_t rows_ = WF ? A.r : A.P, width = WF ? A.P : A.r;
                if (rr >= rows_) continue;
                const int64_t at = (slot * rows_ + rr) * width;
                f32x4 o = acc[h][j] * sc;
                if constexpr (kShift)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[i] = ldexpf(o[i], most);
                if (it.slot < 0) store4(static_cast<T*>(A.out) + at, x0, width, o, A.o4);
                else store4(A.part + at, x0, width, o, width % 4 == 0);
            }
    }
}

// dA (blockIdx.y = 0) and dB.
template <class T, int RF, bool AL>
__global__ __launch_bounds__(256) void k_ad_grad(GradArgs A, GradArgs B) {
    __shared__ __align__(16) char s_u[2][32 * 512];
    __shared__ __align__(16) char s_v[2][kSkinny<T, RF>];
    if (blockIdx.y == 0)
        grad_block<T, RF, true, AL>(A, s_u, s_v);
    else
        grad_block<T, RF, false, AL>(B, s_u, s_v);
}

// Clusters of no chunk: zeros; of several: the sum of their parts in order.
// dA: blockIdx.z = 0, dB: 1.
template <class T>
__global__ __launch_bounds__(256) void k_ad_join(GradArgs A, GradArgs B) {
    const GradArgs& G = blockIdx.z ? B : A;
    const int64_t size = (int64_t)G.r * G.P;
    for (int c = blockIdx.y; c < G.k; c += gridDim.y) {
        const int num = G.num[c];
        if (num == 1) continue;
        const float* part = G.part + G.first[c] * size;
        T* out = static_cast<T*>(G.out) + c * size;
        for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < size; i += (int64_t)gridDim.x * 256) {
            float sum = 0.0f;
#pragma unroll 4
            for (int q = 0; q < num; ++q) sum += part[q * size + i];
            out[i] = from_f32<T>(sum);
        }
    }
}

// --------------------------------------------------------------------------
// Rows of a width that is no multiple of 16 bytes, copied with zeros up to one:
// the tiles' loads then move 16 bytes.  A thread a chunk.
template <class T>
__global__ __launch_bounds__(256) void k_ad_pad(const T* src, int64_t ld, int64_t rows, int32_t d, T* dst, int32_t dp) {
    constexpr int E = Mma<T>::E;
    const int64_t per = dp / E, total = rows * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256)
        *reinterpret_cast<u32x4*>(dst + i * E) = chunk_guarded(src + i / per * ld, i % per * E, d);
}

// --------------------------------------------------------------------------
// Launches

template <class T>
hipError_t pad_rows(const void* src, int64_t ld, int64_t rows, int32_t d, char* dst, int32_t dp, hipStream_t s) {
    const int64_t blocks = (rows * (dp / Mma<T>::E) + 255) / 256;
    hipLaunchKernelGGL((k_ad_pad<T>), dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, s,
                       static_cast<const T*>(src), ld, rows, d, reinterpret_cast<T*>(dst), dp);
    return hipGetLastError();
}

// The operands' 16 x rf indexes of r: 1, 2, 4 or 8.
template <class F>
void by_rank(int rf, F&& go) {
    using std::integral_constant;
    if (rf == 1) go(integral_constant<int, 1>{});
    else if (rf == 2) go(integral_constant<int, 2>{});
    else if (rf <= 4) go(integral_constant<int, 4>{});
    else go(integral_constant<int, 8>{});
}

template <class T, bool TR>
hipError_t inner_go(const InnerArgs& A, const ListArgs& L, hipStream_t s) {
    const dim3 g((unsigned)((A.n + 15) / 16) + (TR ? 1 : 0)), b(256);
    const int rf = (A.r + 15) / 16;
    auto go = [&](auto j) {
        constexpr int RF = decltype(j)::value;
        if (A.u16 && A.q16) hipLaunchKernelGGL((k_ad_inner<T, RF, TR, true, true>), g, b, 0, s, A, L);
        else if (A.u16) hipLaunchKernelGGL((k_ad_inner<T, RF, TR, true, false>), g, b, 0, s, A, L);
        else hipLaunchKernelGGL((k_ad_inner<T, RF, TR, false, false>), g, b, 0, s, A, L);
    };
    by_rank(rf, go);
    return hipGetLastError();
}

template <class K>
hipError_t raise_lds(K* kernel, int bytes) {
    return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

template <class T, int TM, int TN, int WR, int WC, int NS, bool TR, bool AL>
hipError_t main_tile(MainArgs A, hipStream_t s) {
    A.tm = (int)((A.n + TM - 1) / TM);
    A.tn = (A.P + TN - 1) / TN;
    constexpr int RM = TM / WR;   // float16: the powers of two of a step, and of a later one by wave
    constexpr int lds = NS * (TM + TN) * 128 + TM * 72 + (kShifted<T> ? (TM + WR * WC * (RM < 64 ? 64 : RM)) * 4 : 0);
    static_assert(lds <= 160 * 1024, "");
    if (lds > 65536) {
        const hipError_t e = raise_lds(k_ad_main<T, TM, TN, WR, WC, NS, TR, AL>, lds);
        if (e != hipSuccess) return e;
    }
    const int64_t tiles = (int64_t)A.tm * A.tn * A.splits;
    hipLaunchKernelGGL((k_ad_main<T, TM, TN, WR, WC, NS, TR, AL>), dim3((unsigned)((tiles + 7) / 8 * 8)),
                       dim3(64 * WR * WC), lds, s, A);
    if (A.splits > 1)
        hipLaunchKernelGGL((k_ad_sum<T>), dim3((unsigned)A.n, (unsigned)((A.P + 1023) / 1024)), dim3(256), 0, s, A);
    return hipGetLastError();
}

template <class T, bool TR>
hipError_t main_go(const MainArgs& A, const MainShape& M, bool al, hipStream_t s) {
    if (!al) return main_tile<T, 64, 64, 2, 2, 2, TR, false>(A, s);
    if (M.tile == 256) return main_tile<T, 256, 256, 2, 4, 2, TR, true>(A, s);
    if (M.tile == 128) return main_tile<T, 128, 128, 2, 4, 4, TR, true>(A, s);
    return main_tile<T, 64, 64, 2, 2, 2, TR, true>(A, s);
}

template <class T>
hipError_t grad_go(const GradArgs& A, const GradArgs& B, bool al, int64_t max_items, hipStream_t s) {
    int64_t blocks = max_items * (A.tiles > B.tiles ? A.tiles : B.tiles);
    if (blocks > 65536) blocks = 65536;
    if (blocks < 1) blocks = 1;
    by_rank((A.r + 15) / 16, [&](auto j) {
        constexpr int RF = decltype(j)::value;
        const dim3 g((unsigned)blocks, 2), b(256);
        if (al) hipLaunchKernelGGL((k_ad_grad<T, RF, true>), g, b, 0, s, A, B);
        else hipLaunchKernelGGL((k_ad_grad<T, RF, false>), g, b, 0, s, A, B);
    });
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t size = (int64_t)A.r * (A.P > B.P ? A.P : B.P), gx = (size + 1023) / 1024;
    hipLaunchKernelGGL((k_ad_join<T>), dim3((unsigned)(gx < 1024 ? gx : 1024), (unsigned)(A.k < 128 ? A.k : 128), 2),
                       dim3(256), 0, s, A, B);
    return hipGetLastError();
}

// Rows up to which the inner products are formed a wave a row and index: the
// 16-row blocks of k_ad_inner take a block's clusters one after the other, and
// there are too few of them (128 rows of 4096, 32 clusters: 50 us).
constexpr int kFewInner = 1024;

bool a16(const void* p) { return ((uintptr_t)p & 15) == 0; }

template <class T>
hipError_t forward_t(const AdapterArgs& D, char* ws, const AdapterShape& L, hipStream_t s) {
    constexpr int E = Mma<T>::E;
    const bool x16 = rows_vec16(D.X, D.ldx, D.di, sizeof(T)) && a16(D.W) && a16(D.A);
    const bool y4 = D.dout % 4 == 0 && a16(D.Y);
    hipError_t e;
    MainArgs M{};
    M.U = D.X;
    M.ldu = D.ldx;
    M.W = D.W;
    M.ldw = D.di;
    M.Q = D.B;
    M.S = ws + L.off_s;
    M.shift = reinterpret_cast<const int32_t*>(ws + L.off_shift);
    M.order = D.order;
    M.sids = D.sids;
    M.Y = D.Y;
    M.n = D.n;
    M.K = D.di;
    M.P = D.dout;
    M.r = D.r;
    M.rp = L.rp;
    M.q16 = D.r % E == 0 && a16(D.B);
    M.y4 = y4;
    M.y16 = D.dout % E == 0 && a16(D.Y);
    M.splits = L.main.splits;
    M.part = reinterpret_cast<float*>(ws + L.off_split);
    bool u16 = x16;
    if (L.pad_i != D.di) {
        if ((e = pad_rows<T>(D.X, D.ldx, D.n, D.di, ws + L.off_x, L.pad_i, s)) != hipSuccess) return e;
        if ((e = pad_rows<T>(D.W, D.di, D.dout, D.di, ws + L.off_w, L.pad_i, s)) != hipSuccess) return e;
        M.U = ws + L.off_x;
        M.W = ws + L.off_w;
        M.ldu = M.ldw = L.pad_i;
        u16 = true;
    }
    if (L.few || D.n <= kFewInner) {
        FewArgs F{};
        F.X = D.X;
        F.ldx = D.ldx;
        F.W = D.W;
        F.A = D.A;
        F.B = D.B;
        F.order = D.order;
        F.cl = D.sids ? D.sids : D.ids;
        F.scale = D.scale;
        F.S = ws + L.off_s;
        F.H = D.H;
        F.Y = D.Y;
        F.n = (int32_t)D.n;
        F.K = D.di;
        F.P = D.dout;
        F.r = D.r;
        F.k = D.k;
        F.x16 = x16;
        F.y4 = y4;
        F.q16 = M.q16;
        F.shift = reinterpret_cast<int32_t*>(ws + L.off_shift);
        if (!L.few) {
            const unsigned steps = (unsigned)((D.r + kStep - 1) / kStep);
            hipLaunchKernelGGL((k_ad_few_inner<T, true>), dim3((unsigned)D.n * steps), dim3(1024), 0, s, F);
            if ((e = hipGetLastError()) != hipSuccess) return e;
            return main_go<T, false>(M, L.main, u16, s);
        }
        hipLaunchKernelGGL((k_ad_few_inner<T, false>), dim3((unsigned)((D.n * D.r + 3) / 4)), dim3(256), 0, s, F);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        F.X = M.U;
        F.ldx = M.ldu;
        F.W = M.W;
        F.ldw = M.ldw;
        auto go = [&](auto f) {
            constexpr int RF = decltype(f)::value;
            const dim3 g((unsigned)((D.dout + 15) / 16)), b(1024);
            if (u16) hipLaunchKernelGGL((k_ad_few_main<T, RF, true>), g, b, 0, s, F);
            else hipLaunchKernelGGL((k_ad_few_main<T, RF, false>), g, b, 0, s, F);
        };
        if (D.n <= 16) go(std::integral_constant<int, 1>{});
        else if (D.n <= 32) go(std::integral_constant<int, 2>{});
        else if (D.n <= 48) go(std::integral_constant<int, 3>{});
        else go(std::integral_constant<int, 4>{});
        return hipGetLastError();
    }
    InnerArgs I{};
    I.U = M.U;
    I.ldu = M.ldu;
    I.Q = D.A;
    I.order = D.order;
    I.sids = D.sids;
    I.offsets = D.offsets;
    I.scale = D.scale;
    I.S = ws + L.off_s;
    I.shift = reinterpret_cast<int32_t*>(ws + L.off_shift);
    I.H = D.H;
    I.n = D.n;
    I.K = D.di;
    I.r = D.r;
    I.rp = L.rp;
    I.u16 = u16;
    I.q16 = x16;
    I.h4 = D.r % 4 == 0 && a16(D.H);
    if ((e = inner_go<T, false>(I, ListArgs{}, s)) != hipSuccess) return e;
    return main_go<T, false>(M, L.main, u16, s);
}

template <class T>
hipError_t backward_t(const AdapterArgs& D, char* ws, const AdapterShape& L, hipStream_t s) {
    constexpr int E = Mma<T>::E;
    bool dy16 = rows_vec16(D.dY, D.lddy, D.dout, sizeof(T)), x16 = rows_vec16(D.X, D.ldx, D.di, sizeof(T));
    bool w16 = D.di % E == 0 && a16(D.W);
    hipError_t e;
    char* S = ws + L.off_s;
    int32_t* shift = reinterpret_cast<int32_t*>(ws + L.off_shift);
    const void *dY = D.dY, *X = D.X, *W = D.W;
    int64_t lddy = D.lddy, ldx = D.ldx, ldw = D.di;
    if (D.n > 0 && L.pad_o != D.dout) {
        if ((e = pad_rows<T>(dY, lddy, D.n, D.dout, ws + L.off_y, L.pad_o, s)) != hipSuccess) return e;
        dY = ws + L.off_y;
        lddy = L.pad_o;
        dy16 = true;
    }
    if (D.n > 0 && L.pad_i != D.di) {
        if ((e = pad_rows<T>(X, ldx, D.n, D.di, ws + L.off_x, L.pad_i, s)) != hipSuccess) return e;
        if ((e = pad_rows<T>(W, ldw, D.dout, D.di, ws + L.off_w, L.pad_i, s)) != hipSuccess) return e;
        X = ws + L.off_x;
        W = ws + L.off_w;
        ldx = ldw = L.pad_i;
        x16 = w16 = true;
    }
    ListArgs Q{};
    Q.offsets = D.offsets;
    Q.k = D.k;
    Q.chunk = L.chunk;
    Q.count = reinterpret_cast<int32_t*>(ws + L.off_count);
    Q.items = reinterpret_cast<Item*>(ws + L.off_items);
    Q.first = reinterpret_cast<int32_t*>(ws + L.off_first);
    Q.num = Q.first + D.k;
    InnerArgs I{};
    I.U = dY;
    I.ldu = lddy;
    I.Q = D.B;
    I.order = D.order;
    I.sids = D.sids;
    I.offsets = D.offsets;
    I.scale = D.scale;
    I.S = S;
    I.shift = shift;
    I.n = D.n;
    I.K = D.dout;
    I.r = D.r;
    I.rp = L.rp;
    I.u16 = dy16;
    I.q16 = D.r % E == 0 && a16(D.B);
    if (D.n <= kFewInner) {
        FewArgs F{};
        F.X = dY;
        F.ldx = lddy;
        F.B = D.B;
        F.order = D.order;
        F.cl = D.sids;
        F.scale = D.scale;
        F.S = S;
        F.shift = shift;
        F.n = (int32_t)D.n;
        F.K = D.dout;
        F.r = D.r;
        F.k = D.k;
        F.q16 = I.q16;
        hipLaunchKernelGGL((k_ad_few_inner_t<T>), dim3((unsigned)(D.n * ((D.r + kStep - 1) / kStep) + 1)), dim3(256), 0, s,
                           F, Q);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    } else if ((e = inner_go<T, true>(I, Q, s)) != hipSuccess) {
        return e;
    }
    if (D.n > 0) {
        MainArgs M{};
        M.U = dY;
        M.ldu = lddy;
        M.W = W;
        M.ldw = ldw;
        M.Q = D.A;
        M.S = S;
        M.shift = shift;
        M.order = D.order;
        M.sids = D.sids;
        M.Y = D.dX;
        M.n = D.n;
        M.K = D.dout;
        M.P = D.di;
        M.r = D.r;
        M.rp = L.rp;
        M.y4 = D.di % 4 == 0 && a16(D.dX);
        M.y16 = D.di % E == 0 && a16(D.dX);
        M.q16 = D.di % E == 0 && a16(D.A);
        M.splits = L.main.splits;
        M.part = reinterpret_cast<float*>(ws + L.off_split);
        if ((e = main_go<T, true>(M, L.main, dy16 && w16, s)) != hipSuccess) return e;
    }
    GradArgs G{};
    G.order = D.order;
    G.count = Q.count;
    G.items = Q.items;
    G.first = Q.first;
    G.num = Q.num;
    G.k = D.k;
    G.r = D.r;
    G.part = reinterpret_cast<float*>(ws + L.off_part);
    G.U = X;
    G.ldu = ldx;
    G.V = S;
    G.ldv = L.rp;
    G.shift = shift;
    G.out = D.dA;
    G.P = D.di;
    G.tiles = (D.di + 127) / 128;
    G.o4 = D.di % 4 == 0 && a16(D.dA);
    GradArgs B = G;
    B.U = dY;
    B.ldu = lddy;
    B.V = D.H;
    B.ldv = D.r;
    B.v16 = D.r % E == 0 && a16(D.H);
    B.scale = D.scale;
    B.out = D.dB;
    B.P = D.dout;
    B.tiles = (D.dout + 127) / 128;
    B.o4 = D.r % 4 == 0 && a16(D.dB);
    // Two halves of the partial sums' segment.
    B.part = G.part + L.part_a;
    return grad_go<T>(G, B, x16 && dy16, L.max_items, s);
}

}  // namespace

namespace {

// The tile and the parts of the contraction of an n x P product over K, by an
// estimate of its time.  Unit: a 64 x 64 tile's stage by itself on a compute
// unit.  256 and 128 wide tiles take a compute unit each, four of 64 share one
// and make up for each other's waits.  Measured at 4096^3, a flop of the three
// costs 1 : 1.4 : 1.9 in 16 bits and 1 : 1.04 : 1.13 in float32; a tile's start
// and end cost about `edge` of its stages.  Parts of the contraction keep the
// chip busy where there are few tiles, and cost the float32 sums they write
// and a launch.
MainShape main_shape(int64_t n, int32_t K, int32_t P, int type) {
    const bool f32 = type == kF32;
    const int all = (K + (f32 ? 31 : 63)) / (f32 ? 32 : 64);
    const double us = f32 ? 0.48 : 0.122;   // a unit
    const struct {
        int tile, slots;
        double work, cost16, cost32, edge16, edge32;
    } kinds[3] = {{256, 256, 16, 1.0, 1.0, 4, 1}, {128, 256, 4, 1.4, 1.04, 12, 3}, {64, 1024, 4, 1.9, 1.13, 4, 1}};
    MainShape best{64, 1};
    double least = 0;
    for (const auto& k : kinds)
        for (int splits = 1; splits <= 8 && splits <= all; splits *= 2) {
            const double tiles = (double)((n + k.tile - 1) / k.tile) * ((P + k.tile - 1) / k.tile) * splits;
            double rounds = tiles / k.slots;
            if (k.tile == 64) rounds = rounds < 0.25 ? 0.75 : rounds + 0.5;
            else rounds = ceil(rounds);
            double t = rounds * k.work * (f32 ? k.cost32 : k.cost16) *
                       ((all + splits - 1) / splits + (f32 ? k.edge32 : k.edge16));
            if (splits > 1) t += (6 + (double)splits * n * P * 8 / 4e6) / us;
            if (least == 0 || t < least) {
                least = t;
                best = MainShape{k.tile, splits};
            }
        }
    const int share = (all + best.splits - 1) / best.splits;
    best.splits = (all + share - 1) / share;   // no part without a stage
    return best;
}

}  // namespace

AdapterShape adapter_shape(int64_t n, int32_t di, int32_t dout, int32_t k, int32_t r, int type, bool backward) {
    AdapterShape L{};
    const int ks = type == kF32 ? 16 : 32;
    const int steps = (r + kStep - 1) / kStep;
    L.rp = steps * ks;
    L.few = !backward && n <= kAdapterFew;
    auto up = [](size_t b) { return (b + 255) / 256 * 256; };
    size_t o = 0;
    auto take = [&](size_t b) {
        const size_t at = o;
        o += up(b);
        return at;
    };
    L.main = main_shape(n, backward ? dout : di, backward ? di : dout, type);
    L.off_split = take(!L.few && L.main.splits > 1 ? (size_t)L.main.splits * n * (backward ? di : dout) * 4 : 0);
    // Copies of rows whose width is no multiple of 16 bytes.
    const int e = ks / 4;
    const size_t es = row_type_bytes(type);
    L.pad_i = (di + e - 1) / e * e;
    L.pad_o = (dout + e - 1) / e * e;
    // Few rows: element loads cost a wave about 3 ns an element of its rows and
    // columns (48 rows of 4097: 147 us, 58 with the copies), the copies two
    // launches and W's traffic at 3 TB/s (1 row of 4097: 36 us without, 41 with).
    if (L.few && 0.003 * di * ((n + 15) / 16 + 1) < 7 + 2.0 * dout * di * es / 3e6) L.pad_i = di;
    const bool ci = L.pad_i != di, co = backward && L.pad_o != dout;
    L.off_x = take(ci ? (size_t)n * L.pad_i * es : 0);
    L.off_w = take(ci ? (size_t)dout * L.pad_i * es : 0);
    L.off_y = take(co ? (size_t)n * L.pad_o * es : 0);
    L.off_s = take(L.few ? (size_t)n * r * 4 : (size_t)n * L.rp * es);
    L.off_shift = take(type == kF16 && !L.few ? (size_t)n * steps * 4 : 0);
    if (backward) {
        // Chunks long enough that their float32 sums are a small part of the
        // rows read, and at most 256 or so of them.
        const int64_t part = (n / 256 + 63) / 64 * 64;
        L.chunk = 16 * r > 512 ? 16 * r : 512;
        if (part > L.chunk) L.chunk = (int32_t)part;
        // A chunk is a block's run of stages, some 1.5 us each: shorter ones while
        // the blocks do not fill the chip twice over (4000 x 256 float32, 8
        // clusters: gradients 45 us without, 30 with; 8192 x 1024 bf16, r = 64:
        // 90 and 80).  64 rows or twice the blocks only add partial sums (8192 x
        // 512 bf16, r = 8: 34 us so, 38 then).
        const int64_t tiles = ((int64_t)di + 127) / 128 + ((int64_t)dout + 127) / 128;
        while (L.chunk > 128 && L.chunk > 4 * r && (n / L.chunk + (k < n ? k : n)) * tiles < 512) L.chunk /= 2;
        const int64_t cuts = n / L.chunk;
        L.max_items = cuts + (k < n ? k : n);
        // A cluster of several chunks has one that is not full: at most 2 cuts partial sums.
        const int64_t slots = 2 * cuts;
        L.off_count = take(4);
        L.off_items = take((size_t)L.max_items * sizeof(Item));
        L.off_first = take((size_t)k * 8);
        L.part_a = slots * r * di;
        L.off_part = take((size_t)(L.part_a + slots * r * dout) * 4);
    }
    L.bytes = o > 0 ? o : 256;
    return L;
}

hipError_t launch_adapter_forward(const AdapterArgs& D, char* ws, const AdapterShape& L, int type, hipStream_t s) {
    if (D.n == 0) return hipSuccess;
    if (type == kF32) return forward_t<float>(D, ws, L, s);
    if (type == kBF16) return forward_t<__bf16>(D, ws, L, s);
    return forward_t<_Float16>(D, ws, L, s);
}

hipError_t launch_adapter_backward(const AdapterArgs& D, char* ws, const AdapterShape& L, int type, hipStream_t s) {
    if (type == kF32) return backward_t<float>(D, ws, L, s);
    if (type == kBF16) return backward_t<__bf16>(D, ws, L, s);
    return backward_t<_Float16>(D, ws, L, s);
}

}  // namespace km
