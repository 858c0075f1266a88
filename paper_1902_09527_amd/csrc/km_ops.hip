// C-ABI entry points of the operators of a layer conditioned on clusters:
// argument checks, workspace layouts and launches.  The declarations and
// their contracts are in include/kmeans_ops.h.
#include <math.h>

#include "kmeans_ops.h"
#include "km_ops.h"

namespace {

bool type_ok(int32_t t) { return t == KM_F32 || t == KM_BF16 || t == KM_F16; }

// n rows of d elements, ld apart: sizes that stay within 63-bit byte offsets
// (and widths within 32-bit column indexes).
constexpr int64_t kMostColumns = (int64_t)1 << 28;
bool rows_ok(int64_t n, int64_t d, int64_t ld) {
    return n >= 0 && d >= 1 && d <= kMostColumns && ld >= d && (n == 0 || ld <= (INT64_MAX / 16) / n);
}

// Checks arrays against the current device; the first refusal is kept.
struct Checks {
    int dev = 0, rc = KM_OK;
    Checks() {
        const hipError_t e = hipGetDevice(&dev);
        if (e != hipSuccess) rc = km::ops_hip_error(e, "hipGetDevice");
    }
    void array(const void* p, size_t bytes, const char* what) {
        if (rc == KM_OK && bytes > 0) rc = km::ops_check_range(p, bytes, dev, what);
    }
    void rows(const void* p, int64_t n, int64_t d, int64_t ld, int32_t type, const char* what) {
        if (n > 0) array(p, (size_t)((n - 1) * ld + d) * km::row_type_bytes(type), what);
    }
};

int bad(const char* what) { return km::ops_error(KM_ERR_INVALID_ARG, "%s", what); }

int workspace_ok(const void* ws, size_t have, size_t need) {
    if (!ws || have < need || ((uintptr_t)ws & 255))
        return km::ops_error(KM_ERR_INVALID_ARG, "workspace: %zu bytes, 256-byte aligned, needed", need);
    return KM_OK;
}

int done(hipError_t e, const char* what) { return e == hipSuccess ? KM_OK : km::ops_hip_error(e, what); }

bool slots_ok(int64_t n, int32_t m, int32_t k) {
    return n >= 0 && m >= 1 && k >= 1 && k < INT32_MAX && n <= INT32_MAX / (int64_t)m;
}

// What the row movers share.
int move_args(km::MoveArgs& A, int64_t n, int32_t m, int32_t k, int32_t d, int32_t type, const int32_t* pos,
              const int32_t* offsets) {
    if (!slots_ok(n, m, k)) return bad("n >= 0, m >= 1, 1 <= k < 2^31 - 1 and n m < 2^31 needed");
    if (d < 1 || !type_ok(type)) return bad("d >= 1 and a type of KM_F32, KM_BF16 or KM_F16 needed");
    if (n > 0 && (!pos || !offsets)) return bad("pos or offsets is null");
    A = km::MoveArgs{};
    A.pos = pos;
    A.used = offsets ? offsets + k : nullptr;
    A.n = n;
    A.m = m;
    A.d = d;
    return KM_OK;
}

void check_plan(Checks& C, const km::MoveArgs& A, int32_t k, const int32_t* offsets) {
    C.array(A.pos, (size_t)A.n * A.m * 4, "pos");
    C.array(offsets, (size_t)(k + (int64_t)1) * 4, "offsets");
}

}  // namespace

extern "C" {

size_t kmeans_sort_workspace_bytes(int64_t n, int32_t m, int32_t k) {
    return slots_ok(n, m, k) ? km::sort_shape(n * m, k).bytes : 0;
}

int kmeans_sort_plan(const int32_t* ids, int64_t n, int32_t m, int32_t k, int32_t* order, int32_t* pos,
                     int32_t* sorted_ids, int32_t* offsets, void* workspace, size_t workspace_bytes,
                     void* hip_stream) {
    if (!slots_ok(n, m, k)) return bad("n >= 0, m >= 1, 1 <= k < 2^31 - 1 and n m < 2^31 needed");
    if (!offsets || (n > 0 && (!ids || !order || !pos || !sorted_ids))) return bad("null array");
    const km::SortShape S = km::sort_shape(n * m, k);
    int rc = workspace_ok(workspace, workspace_bytes, S.bytes);
    if (rc != KM_OK) return rc;
    Checks C;
    const size_t b = (size_t)n * m * 4;
    C.array(ids, b, "ids");
    C.array(order, b, "order");
    C.array(pos, b, "pos");
    C.array(sorted_ids, b, "sorted_ids");
    C.array(offsets, (size_t)(k + (int64_t)1) * 4, "offsets");
    C.array(workspace, S.bytes, "workspace");
    if (C.rc != KM_OK) return C.rc;
    km::SortArgs A{ids, (int32_t)(n * m), k, order, pos, sorted_ids, offsets};
    return done(km::launch_sort_plan(A, S, static_cast<char*>(workspace), static_cast<hipStream_t>(hip_stream)),
                "kmeans_sort_plan");
}

int kmeans_sort_gather(const void* X, int64_t ldx, int64_t n, int32_t m, int32_t k, int32_t d, int32_t type,
                       const int32_t* pos, const int32_t* offsets, void* Xs, void* hip_stream) {
    km::MoveArgs A;
    int rc = move_args(A, n, m, k, d, type, pos, offsets);
    if (rc != KM_OK) return rc;
    if (!rows_ok(n, d, ldx) || !rows_ok(n * m, d, d)) return bad("ldx >= d needed, and sizes within 63 bits");
    if (n == 0) return KM_OK;
    if (!X || !Xs) return bad("X or Xs is null");
    Checks C;
    check_plan(C, A, k, offsets);
    C.rows(X, n, d, ldx, type, "X");
    C.rows(Xs, n * m, d, d, type, "Xs");
    if (C.rc != KM_OK) return C.rc;
    A.src = X;
    A.ld = ldx;
    A.dst = Xs;
    return done(km::launch_sort_gather(A, type, static_cast<hipStream_t>(hip_stream)), "kmeans_sort_gather");
}

int kmeans_sort_combine(const void* Z, int64_t ldz, int64_t n, int32_t m, int32_t k, int32_t d, int32_t type,
                        const int32_t* pos, const int32_t* offsets, const float* w, void* Y, void* hip_stream) {
    km::MoveArgs A;
    int rc = move_args(A, n, m, k, d, type, pos, offsets);
    if (rc != KM_OK) return rc;
    if (!rows_ok(n * m, d, ldz) || !rows_ok(n, d, d)) return bad("ldz >= d needed, and sizes within 63 bits");
    if (n == 0) return KM_OK;
    if (!Z || !Y) return bad("Z or Y is null");
    Checks C;
    check_plan(C, A, k, offsets);
    C.rows(Z, n * m, d, ldz, type, "Z");
    C.rows(Y, n, d, d, type, "Y");
    if (w) C.array(w, (size_t)n * m * 4, "w");
    if (C.rc != KM_OK) return C.rc;
    A.src = Z;
    A.ld = ldz;
    A.dst = Y;
    A.w = w;
    return done(km::launch_sort_combine(A, type, static_cast<hipStream_t>(hip_stream)), "kmeans_sort_combine");
}

int kmeans_sort_combine_backward(const void* dY, int64_t lddy, const void* Z, int64_t ldz, int64_t n, int32_t m,
                                 int32_t k, int32_t d, int32_t type, const int32_t* pos, const int32_t* offsets,
                                 const float* w, void* dZ, float* dw, void* hip_stream) {
    km::MoveArgs A;
    int rc = move_args(A, n, m, k, d, type, pos, offsets);
    if (rc != KM_OK) return rc;
    if (!rows_ok(n, d, lddy) || (dw && !rows_ok(n * m, d, ldz)) || !rows_ok(n * m, d, d))
        return bad("lddy >= d and ldz >= d needed, and sizes within 63 bits");
    if (n == 0) return KM_OK;
    if (!dY || !dZ || (dw && !Z)) return bad("dY, Z or dZ is null");
    Checks C;
    check_plan(C, A, k, offsets);
    C.rows(dY, n, d, lddy, type, "dY");
    C.rows(dZ, n * m, d, d, type, "dZ");
    if (w) C.array(w, (size_t)n * m * 4, "w");
    if (dw) {
        C.rows(Z, n * m, d, ldz, type, "Z");
        C.array(dw, (size_t)n * m * 4, "dw");
    }
    if (C.rc != KM_OK) return C.rc;
    A.src = dY;
    A.ld = lddy;
    A.src2 = dw ? Z : nullptr;
    A.ld2 = ldz;
    A.dst = dZ;
    A.w = w;
    A.dw = dw;
    return done(km::launch_sort_combine_bwd(A, type, static_cast<hipStream_t>(hip_stream)),
                "kmeans_sort_combine_backward");
}

int kmeans_norm_forward(const void* X, int64_t ldx, int64_t n, int32_t d, int32_t type, const void* gamma,
                        const void* beta, int32_t param_f32, float eps, void* Y, float* mean, float* rstd,
                        void* hip_stream) {
    if (!type_ok(type)) return bad("a type of KM_F32, KM_BF16 or KM_F16 needed");
    if (!rows_ok(n, d, ldx)) return bad("n >= 0, d >= 1, ldx >= d needed, and sizes within 63 bits");
    if (!(eps >= 0.0f) || !isfinite(eps)) return bad("eps is negative or not finite");
    if (n == 0) return KM_OK;
    if (!X || !Y || !mean || !rstd) return bad("X, Y, mean or rstd is null");
    Checks C;
    const size_t pb = (size_t)d * (param_f32 ? 4 : km::row_type_bytes(type));
    C.rows(X, n, d, ldx, type, "X");
    C.rows(Y, n, d, d, type, "Y");
    C.array(mean, (size_t)n * 4, "mean");
    C.array(rstd, (size_t)n * 4, "rstd");
    if (gamma) C.array(gamma, pb, "gamma");
    if (beta) C.array(beta, pb, "beta");
    if (C.rc != KM_OK) return C.rc;
    km::NormArgs A{};
    A.X = X;
    A.ldx = ldx;
    A.n = n;
    A.d = d;
    A.gamma = gamma;
    A.beta = beta;
    A.param_f32 = param_f32 != 0;
    A.eps = eps;
    A.Y = Y;
    A.mean = mean;
    A.rstd = rstd;
    return done(km::launch_norm_fwd(A, type, static_cast<hipStream_t>(hip_stream)), "kmeans_norm_forward");
}

size_t kmeans_norm_workspace_bytes(int64_t n, int32_t d, int32_t type) {
    if (!type_ok(type) || !rows_ok(n, d, d)) return 0;
    const size_t b = (size_t)km::norm_bwd_max_blocks(n, d) * 2 * d * 4;
    return (b + 255) / 256 * 256;
}

int kmeans_norm_backward(const void* dY, int64_t lddy, const void* X, int64_t ldx, int64_t n, int32_t d,
                         int32_t type, const float* mean, const float* rstd, const void* gamma, int32_t param_f32,
                         void* dX, float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes,
                         void* hip_stream) {
    if (!type_ok(type)) return bad("a type of KM_F32, KM_BF16 or KM_F16 needed");
    if (!rows_ok(n, d, ldx) || !rows_ok(n, d, lddy))
        return bad("n >= 0, d >= 1, ldx >= d, lddy >= d needed, and sizes within 63 bits");
    if (n > 0 && (!dY || !X || !mean || !rstd || !dX)) return bad("dY, X, mean, rstd or dX is null");
    const bool sums = dgamma || dbeta;
    const size_t need = kmeans_norm_workspace_bytes(n, d, type);
    if (sums) {
        const int rc = workspace_ok(workspace, workspace_bytes, need);
        if (rc != KM_OK) return rc;
    }
    Checks C;
    C.rows(dY, n, d, lddy, type, "dY");
    C.rows(X, n, d, ldx, type, "X");
    C.rows(dX, n, d, d, type, "dX");
    C.array(mean, (size_t)n * 4, "mean");
    C.array(rstd, (size_t)n * 4, "rstd");
    if (gamma) C.array(gamma, (size_t)d * (param_f32 ? 4 : km::row_type_bytes(type)), "gamma");
    if (dgamma) C.array(dgamma, (size_t)d * 4, "dgamma");
    if (dbeta) C.array(dbeta, (size_t)d * 4, "dbeta");
    if (sums) C.array(workspace, need, "workspace");
    if (C.rc != KM_OK) return C.rc;
    km::NormArgs A{};
    A.X = X;
    A.ldx = ldx;
    A.dY = dY;
    A.lddy = lddy;
    A.n = n;
    A.d = d;
    A.gamma = gamma;
    A.param_f32 = param_f32 != 0;
    A.mean = const_cast<float*>(mean);
    A.rstd = const_cast<float*>(rstd);
    A.dX = dX;
    A.dgamma = dgamma;
    A.dbeta = dbeta;
    A.part = sums ? static_cast<float*>(workspace) : nullptr;
    return done(km::launch_norm_bwd(A, type, static_cast<hipStream_t>(hip_stream)), "kmeans_norm_backward");
}

// Forward workspace: the operator's own, then a plan where none is given.
struct AdapterPlan {
    km::SortShape sort;
    size_t order, pos, sids, offsets, ws, bytes;
};
static AdapterPlan adapter_plan(int64_t n, int32_t k, size_t at) {
    AdapterPlan P{};
    auto take = [&](size_t b) {
        const size_t here = at;
        at += (b + 255) / 256 * 256;
        return here;
    };
    P.sort = km::sort_shape(n, k);
    P.order = take((size_t)n * 4);
    P.pos = take((size_t)n * 4);
    P.sids = take((size_t)n * 4);
    P.offsets = take(((size_t)k + 1) * 4);
    P.ws = take(P.sort.bytes);
    P.bytes = at;
    return P;
}

static int adapter_sizes(int64_t n, int32_t din, int32_t dout, int32_t k, int32_t r, int32_t type) {
    if (!slots_ok(n, 1, k) || din < 1 || dout < 1 || r < 1 || !type_ok(type))
        return bad("n, din, dout, k, r or type out of range");
    if (n > (int64_t)1 << 27 || din > 1 << 24 || dout > 1 << 24)   // the kernels' grids and 32-bit stage counts
        return km::ops_error(KM_ERR_UNSUPPORTED, "more than 2^27 rows or 2^24 columns");
    if (r > km::kAdapterMaxRank)
        return km::ops_error(KM_ERR_UNSUPPORTED, "adapters have a rank of at most %d", km::kAdapterMaxRank);
    if (!rows_ok(n, din, din) || !rows_ok(n, dout, dout) || !rows_ok(dout, din, din) ||
        !rows_ok((int64_t)k * r, din, din) || !rows_ok((int64_t)k * r, dout, dout))
        return bad("sizes within 63 bits needed");
    return KM_OK;
}

size_t kmeans_adapter_workspace_bytes(int64_t n, int32_t din, int32_t dout, int32_t k, int32_t r, int32_t type,
                                      int32_t backward) {
    if (adapter_sizes(n, din, dout, k, r, type) != KM_OK) return 0;
    const km::AdapterShape L = km::adapter_shape(n, din, dout, k, r, type, backward != 0);
    return backward || L.few ? L.bytes : adapter_plan(n, k, L.bytes).bytes;
}

int kmeans_adapter_tile(int64_t n, int32_t din, int32_t dout, int32_t k, int32_t r, int32_t type, int32_t backward,
                        int32_t* tile, int32_t* splits) {
    const int rc = adapter_sizes(n, din, dout, k, r, type);
    if (rc != KM_OK) return rc;
    if (!tile || !splits) return bad("tile or splits is null");
    const km::AdapterShape L = km::adapter_shape(n, din, dout, k, r, type, backward != 0);
    *tile = L.few ? 0 : L.main.tile;
    *splits = L.few ? 1 : L.main.splits;
    return KM_OK;
}

int kmeans_adapter_forward(const void* X, int64_t ldx, int64_t n, int32_t din, int32_t dout, int32_t k, int32_t r,
                           int32_t type, const void* W, const void* A, const void* B, const float* scale,
                           const int32_t* ids, const int32_t* order, const int32_t* sorted_ids,
                           const int32_t* offsets, void* Y, void* H, void* workspace, size_t workspace_bytes,
                           void* hip_stream) {
    int rc = adapter_sizes(n, din, dout, k, r, type);
    if (rc != KM_OK) return rc;
    if (!rows_ok(n, din, ldx)) return bad("ldx >= din needed, and sizes within 63 bits");
    if (!W || !A || !B) return bad("W, A or B is null");
    if (n > 0 && (!X || !Y || !H)) return bad("X, Y or H is null");
    const bool plan = sorted_ids || offsets || order;
    if (n > 0 && (plan ? (!sorted_ids || !offsets) : !ids)) return bad("ids, or sorted_ids and offsets, needed");
    const km::AdapterShape L = km::adapter_shape(n, din, dout, k, r, type, false);
    const AdapterPlan P = adapter_plan(n, k, L.bytes);
    const size_t need = plan || L.few ? L.bytes : P.bytes;
    if ((rc = workspace_ok(workspace, workspace_bytes, need)) != KM_OK) return rc;
    if (n == 0) return KM_OK;
    const size_t es = km::row_type_bytes(type);
    Checks C;
    C.rows(X, n, din, ldx, type, "X");
    C.array(W, (size_t)din * dout * es, "W");
    C.array(A, (size_t)k * r * din * es, "A");
    C.array(B, (size_t)k * r * dout * es, "B");
    if (scale) C.array(scale, (size_t)k * 4, "scale");
    if (plan) {
        if (order) C.array(order, (size_t)n * 4, "order");
        C.array(sorted_ids, (size_t)n * 4, "sorted_ids");
        C.array(offsets, ((size_t)k + 1) * 4, "offsets");
    } else {
        C.array(ids, (size_t)n * 4, "ids");
    }
    C.array(Y, (size_t)n * dout * es, "Y");
    C.array(H, (size_t)n * r * es, "H");
    C.array(workspace, need, "workspace");
    if (C.rc != KM_OK) return C.rc;
    char* ws = static_cast<char*>(workspace);
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    km::AdapterArgs D{};
    D.X = X;
    D.ldx = ldx;
    D.n = n;
    D.di = din;
    D.dout = dout;
    D.k = k;
    D.r = r;
    D.W = W;
    D.A = A;
    D.B = B;
    D.ids = ids;
    D.order = order;
    D.sids = sorted_ids;
    D.offsets = offsets;
    D.scale = scale;
    D.Y = Y;
    D.H = H;
    if (!plan && !L.few) {
        auto at = [&](size_t o) { return reinterpret_cast<int32_t*>(ws + o); };
        const km::SortArgs S{ids, (int32_t)n, k, at(P.order), at(P.pos), at(P.sids), at(P.offsets)};
        const hipError_t e = km::launch_sort_plan(S, P.sort, ws + P.ws, st);
        if (e != hipSuccess) return km::ops_hip_error(e, "kmeans_adapter_forward");
        D.order = S.order;
        D.sids = S.sorted_ids;
        D.offsets = S.offsets;
    }
    return done(km::launch_adapter_forward(D, ws, L, type, st), "kmeans_adapter_forward");
}

int kmeans_adapter_backward(const void* dY, int64_t lddy, const void* X, int64_t ldx, const void* H, int64_t n,
                            int32_t din, int32_t dout, int32_t k, int32_t r, int32_t type, const void* W,
                            const void* A, const void* B, const float* scale, const int32_t* order,
                            const int32_t* sorted_ids, const int32_t* offsets, void* dX, void* dA, void* dB,
                            void* workspace, size_t workspace_bytes, void* hip_stream) {
    int rc = adapter_sizes(n, din, dout, k, r, type);
    if (rc != KM_OK) return rc;
    if (!rows_ok(n, din, ldx) || !rows_ok(n, dout, lddy)) return bad("ldx >= din and lddy >= dout needed");
    if (!W || !A || !B || !offsets || !dA || !dB) return bad("W, A, B, offsets, dA or dB is null");
    if (n > 0 && (!dY || !X || !H || !dX || !sorted_ids)) return bad("dY, X, H, dX or sorted_ids is null");
    const km::AdapterShape L = km::adapter_shape(n, din, dout, k, r, type, true);
    if ((rc = workspace_ok(workspace, workspace_bytes, L.bytes)) != KM_OK) return rc;
    const size_t es = km::row_type_bytes(type);
    Checks C;
    C.rows(dY, n, dout, lddy, type, "dY");
    C.rows(X, n, din, ldx, type, "X");
    C.array(H, (size_t)n * r * es, "H");
    C.array(W, (size_t)din * dout * es, "W");
    C.array(A, (size_t)k * r * din * es, "A");
    C.array(B, (size_t)k * r * dout * es, "B");
    if (scale) C.array(scale, (size_t)k * 4, "scale");
    if (order) C.array(order, (size_t)n * 4, "order");
    C.array(sorted_ids, (size_t)n * 4, "sorted_ids");
    C.array(offsets, ((size_t)k + 1) * 4, "offsets");
    C.array(dX, (size_t)n * din * es, "dX");
    C.array(dA, (size_t)k * r * din * es, "dA");
    C.array(dB, (size_t)k * r * dout * es, "dB");
    C.array(workspace, L.bytes, "workspace");
    if (C.rc != KM_OK) return C.rc;
    km::AdapterArgs D{};
    D.dY = dY;
    D.lddy = lddy;
    D.X = X;
    D.ldx = ldx;
    D.H = const_cast<void*>(H);
    D.n = n;
    D.di = din;
    D.dout = dout;
    D.k = k;
    D.r = r;
    D.W = W;
    D.A = A;
    D.B = B;
    D.scale = scale;
    D.order = order;
    D.sids = sorted_ids;
    D.offsets = offsets;
    D.dX = dX;
    D.dA = dA;
    D.dB = dB;
    return done(km::launch_adapter_backward(D, static_cast<char*>(workspace), L, type,
                                            static_cast<hipStream_t>(hip_stream)),
                "kmeans_adapter_backward");
}

}  // extern "C"
