// C ABI of the expert layer: argument validation on the host, then the HIP
// launchers. Nothing is enqueued when validation fails.
#include <math.h>
#include <stdint.h>

#include <initializer_list>

#include "base.h"
#include "internal.hpp"

namespace {

constexpr int64_t kMaxExperts = 2048;
constexpr int64_t kMaxChoices = 64;      // experts a token
constexpr int64_t kMaxNorm = 16384;      // elements of a row held in registers
constexpr int64_t kMaxDim = (int64_t)1 << 20;

bool aligned(const void *p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

int hip_status(hipError_t e) { return e == hipSuccess ? BASE_OK : BASE_ERR_HIP; }

bool overlap(const void *a, int64_t an, const void *b, int64_t bn) {
    if (a == nullptr || b == nullptr) return false;
    const char *pa = static_cast<const char *>(a);
    const char *pb = static_cast<const char *>(b);
    return pa < pb + bn && pb < pa + an;
}

// Overlap other than being the same matrix.
bool partly(const void *a, const void *b, int64_t n) { return a != b && overlap(a, n, b, n); }

struct Span {
    const void *at;
    int64_t bytes;
};

// Whether an output overlaps an input or another output. (Those that may be an input are
// looked at with partly, and are not among its `in`.)
bool clash(std::initializer_list<Span> out, std::initializer_list<Span> in) {
    for (const Span *a = out.begin(); a != out.end(); ++a) {
        if (a->bytes == 0) continue;
        for (const Span *b = a + 1; b != out.end(); ++b)
            if (b->bytes != 0 && overlap(a->at, a->bytes, b->at, b->bytes)) return true;
        for (const Span &b : in)
            if (overlap(a->at, a->bytes, b.at, b.bytes)) return true;
    }
    return false;
}

int64_t size_of(int dtype) { return dtype == BASE_BF16 ? 2 : 4; }

int check_dtype(int dtype) {
    return dtype == BASE_BF16 || dtype == BASE_F32 ? BASE_OK : BASE_ERR_UNSUPPORTED_DTYPE;
}

// T tokens, k choices, rows of d.
int check_moves(int64_t T, int64_t k, int64_t d, int dtype) {
    if (T <= 0 || k <= 0 || d <= 0 || d % 8 != 0) return BASE_ERR_INVALID_ARG;
    if (check_dtype(dtype) != BASE_OK) return BASE_ERR_UNSUPPORTED_DTYPE;
    if (T > INT32_MAX || k > kMaxChoices || T * k > INT32_MAX || d > kMaxDim) return BASE_ERR_RANGE;
    return BASE_OK;
}

int check_route(int64_t T, int64_t E, int64_t k) {
    if (T <= 0 || E <= 0 || k <= 0) return BASE_ERR_INVALID_ARG;
    if (T > INT32_MAX || E > kMaxExperts || k > kMaxChoices || T * k > INT32_MAX)
        return BASE_ERR_RANGE;
    return BASE_OK;
}

int check_norm(const int32_t *perm, int64_t x_rows, int64_t k, const int32_t *offsets, int64_t N,
               int64_t E, int64_t d, int dtype) {
    if (N <= 0 || E <= 0 || d <= 0 || d % 8 != 0 || x_rows <= 0 || k <= 0)
        return BASE_ERR_INVALID_ARG;
    if (offsets == nullptr && E != 1) return BASE_ERR_INVALID_ARG;
    if (perm == nullptr && (x_rows != N || k != 1)) return BASE_ERR_INVALID_ARG;
    if (check_dtype(dtype) != BASE_OK) return BASE_ERR_UNSUPPORTED_DTYPE;
    if (N > INT32_MAX || x_rows > INT32_MAX || k > INT32_MAX || E > kMaxExperts || d > kMaxNorm)
        return BASE_ERR_RANGE;
    if (!aligned(perm, 4) || !aligned(offsets, 4)) return BASE_ERR_INVALID_ARG;
    return BASE_OK;
}

int check_linear(int64_t N, int64_t E, int64_t K, int64_t O, int dtype) {
    if (N <= 0 || E <= 0 || K <= 0 || O <= 0 || K % 8 != 0 || O % 8 != 0)
        return BASE_ERR_INVALID_ARG;
    if (check_dtype(dtype) != BASE_OK) return BASE_ERR_UNSUPPORTED_DTYPE;
    if (N > INT32_MAX || E > kMaxExperts || K > kMaxDim || O > kMaxDim) return BASE_ERR_RANGE;
    return BASE_OK;
}

// The workspace of a product, as far as it is used, and whether it is there.
Span used(int product, int64_t N, int64_t E, int64_t K, int64_t O, int dtype,
          const void *workspace) {
    return {workspace,
            (int64_t)base::linear_workspace_size(product, N, E, K, O, dtype == BASE_BF16)};
}
bool there(const Span &ws, size_t bytes) {
    return ws.bytes == 0 ||
           (ws.at != nullptr && bytes >= (size_t)ws.bytes && aligned(ws.at, 256));
}

}  // namespace

extern "C" {

size_t base_topk_workspace_size(int64_t T, int64_t E, int64_t k) {
    if (check_route(T, E, k) != BASE_OK) return 0;
    return base::topk_workspace_size(T, E, k);
}

int base_topk_assign(const float *S, int64_t T, int64_t E, int64_t k, int32_t *assign,
                     float *scores, int32_t *perm, int32_t *slots, int32_t *offsets,
                     void *workspace, size_t workspace_bytes, void *stream) {
    if (S == nullptr || assign == nullptr || perm == nullptr || slots == nullptr ||
        offsets == nullptr)
        return BASE_ERR_INVALID_ARG;
    if (const int st = check_route(T, E, k)) return st;
    if (k > E) return BASE_ERR_INVALID_ARG;
    if (!aligned(S, 16) || !aligned(assign, 4) || !aligned(scores, 4) || !aligned(perm, 4) ||
        !aligned(slots, 4) || !aligned(offsets, 4))
        return BASE_ERR_INVALID_ARG;
    if (workspace == nullptr || workspace_bytes < base::topk_workspace_size(T, E, k) ||
        !aligned(workspace, 256))
        return BASE_ERR_WORKSPACE;
    const int64_t pairs = T * k * 4;
    if (clash({{assign, pairs}, {scores, pairs}, {perm, pairs}, {slots, pairs}, {offsets, (E + 1) * 4},
               {workspace, (int64_t)base::topk_workspace_size(T, E, k)}},
              {{S, T * E * 4}}))
        return BASE_ERR_INVALID_ARG;
    return hip_status(base::launch_topk(S, T, E, k, assign, scores, perm, slots, offsets, workspace,
                                        static_cast<hipStream_t>(stream)));
}

int base_sort_by_expert(const int32_t *assign, int64_t T, int64_t E, int64_t k, int32_t *perm,
                        int32_t *slots, int32_t *offsets, void *workspace, size_t workspace_bytes,
                        void *stream) {
    if (assign == nullptr || perm == nullptr || slots == nullptr || offsets == nullptr)
        return BASE_ERR_INVALID_ARG;
    if (const int st = check_route(T, E, k)) return st;
    if (!aligned(assign, 4) || !aligned(perm, 4) || !aligned(slots, 4) || !aligned(offsets, 4))
        return BASE_ERR_INVALID_ARG;
    if (workspace == nullptr || workspace_bytes < base::topk_workspace_size(T, E, k) ||
        !aligned(workspace, 256))
        return BASE_ERR_WORKSPACE;
    const int64_t pairs = T * k * 4;
    if (clash({{perm, pairs}, {slots, pairs}, {offsets, (E + 1) * 4},
               {workspace, (int64_t)base::topk_workspace_size(T, E, k)}},
              {{assign, pairs}}))
        return BASE_ERR_INVALID_ARG;
    return hip_status(base::launch_topk(nullptr, T, E, k, const_cast<int32_t *>(assign), nullptr,
                                        perm, slots, offsets, workspace,
                                        static_cast<hipStream_t>(stream)));
}

int base_dispatch(const void *in, const float *weights, const int32_t *slots, void *out, int64_t T,
                  int64_t k, int64_t d, int dtype, void *stream) {
    if (in == nullptr || slots == nullptr || out == nullptr) return BASE_ERR_INVALID_ARG;
    if (const int st = check_moves(T, k, d, dtype)) return st;
    if (!aligned(in, 16) || !aligned(out, 16) || !aligned(weights, 4) || !aligned(slots, 4))
        return BASE_ERR_INVALID_ARG;
    const int64_t row = d * size_of(dtype);
    if (clash({{out, T * k * row}}, {{in, T * row}, {weights, T * k * 4}, {slots, T * k * 4}}))
        return BASE_ERR_INVALID_ARG;
    return hip_status(base::launch_dispatch(in, weights, slots, out, T, k, d, dtype == BASE_BF16,
                                            static_cast<hipStream_t>(stream)));
}

int base_combine(const void *F, const float *weights, const int32_t *slots, const void *residual,
                 void *out, int64_t T, int64_t k, int64_t d, int dtype, void *stream) {
    if (F == nullptr || slots == nullptr || out == nullptr) return BASE_ERR_INVALID_ARG;
    if (const int st = check_moves(T, k, d, dtype)) return st;
    if (!aligned(F, 16) || !aligned(out, 16) || !aligned(residual, 16) || !aligned(weights, 4) ||
        !aligned(slots, 4))
        return BASE_ERR_INVALID_ARG;
    const int64_t row = d * size_of(dtype);
    if (clash({{out, T * row}}, {{F, T * k * row}, {weights, T * k * 4}, {slots, T * k * 4}}) ||
        partly(out, residual, T * row))
        return BASE_ERR_INVALID_ARG;
    return hip_status(base::launch_combine(F, weights, slots, residual, out, T, k, d,
                                           dtype == BASE_BF16, static_cast<hipStream_t>(stream)));
}

int base_combine_backward(const void *dY, const void *F, const float *weights,
                          const int32_t *slots, void *dF, float *dweights, int64_t T, int64_t k,
                          int64_t d, int dtype, void *stream) {
    if (dY == nullptr || F == nullptr || weights == nullptr || slots == nullptr || dF == nullptr ||
        dweights == nullptr)
        return BASE_ERR_INVALID_ARG;
    if (const int st = check_moves(T, k, d, dtype)) return st;
    if (!aligned(dY, 16) || !aligned(F, 16) || !aligned(dF, 16) || !aligned(weights, 4) ||
        !aligned(slots, 4) || !aligned(dweights, 4))
        return BASE_ERR_INVALID_ARG;
    const int64_t row = d * size_of(dtype);
    if (clash({{dF, T * k * row}, {dweights, T * k * 4}},
              {{dY, T * row}, {F, T * k * row}, {weights, T * k * 4}, {slots, T * k * 4}}))
        return BASE_ERR_INVALID_ARG;
    return hip_status(base::launch_combine_backward(dY, F, weights, slots, dF, dweights, T, k, d,
                                                    dtype == BASE_BF16,
                                                    static_cast<hipStream_t>(stream)));
}

int base_expert_norm(const void *x, const int32_t *perm, int64_t x_rows, int64_t k,
                     const void *weight, const void *bias, const int32_t *offsets, void *y,
                     float *mean, float *rstd, int64_t N, int64_t E, int64_t d, double eps,
                     int dtype, void *stream) {
    if (x == nullptr || weight == nullptr || y == nullptr || mean == nullptr || rstd == nullptr)
        return BASE_ERR_INVALID_ARG;
    if (const int st = check_norm(perm, x_rows, k, offsets, N, E, d, dtype)) return st;
    if (!(eps >= 0.0) || !isfinite(eps)) return BASE_ERR_INVALID_ARG;
    if (!aligned(x, 16) || !aligned(weight, 16) || !aligned(bias, 16) || !aligned(y, 16) ||
        !aligned(mean, 4) || !aligned(rstd, 4))
        return BASE_ERR_INVALID_ARG;
    const int64_t row = d * size_of(dtype);
    if (clash({{y, N * row}, {mean, N * 4}, {rstd, N * 4}},
              {{x, x_rows * row}, {perm, N * 4}, {weight, E * row}, {bias, E * row},
               {offsets, (E + 1) * 4}}))
        return BASE_ERR_INVALID_ARG;
    return hip_status(base::launch_norm(x, perm, x_rows, k, weight, bias, offsets, y, mean, rstd, N,
                                        E, d, eps, dtype == BASE_BF16,
                                        static_cast<hipStream_t>(stream)));
}

size_t base_expert_norm_workspace_size(int64_t N, int64_t E, int64_t d) {
    if (N <= 0 || E <= 0 || d <= 0 || d % 8 != 0 || N > INT32_MAX || E > kMaxExperts ||
        d > kMaxNorm)
        return 0;
    return base::norm_workspace_size(N, E, d);
}

int base_expert_norm_backward(const void *dy, const void *x, const int32_t *perm, int64_t x_rows,
                              int64_t k, const void *weight, const float *mean, const float *rstd,
                              const int32_t *offsets, const void *residual, void *dx,
                              float *dweight, float *dbias, int64_t N, int64_t E, int64_t d,
                              int dtype, void *workspace, size_t workspace_bytes, void *stream) {
    if (dy == nullptr || x == nullptr || weight == nullptr || mean == nullptr || rstd == nullptr ||
        dx == nullptr || dweight == nullptr)
        return BASE_ERR_INVALID_ARG;
    if (const int st = check_norm(perm, x_rows, k, offsets, N, E, d, dtype)) return st;
    if (!aligned(dy, 16) || !aligned(x, 16) || !aligned(weight, 16) || !aligned(mean, 4) ||
        !aligned(rstd, 4) || !aligned(residual, 16) || !aligned(dx, 16) || !aligned(dweight, 4) ||
        !aligned(dbias, 4))
        return BASE_ERR_INVALID_ARG;
    const int64_t row = d * size_of(dtype);
    if (overlap(dx, N * row, x, x_rows * row) || partly(dx, dy, N * row) ||
        partly(dx, residual, N * row))
        return BASE_ERR_INVALID_ARG;
    if (workspace == nullptr || workspace_bytes < base::norm_workspace_size(N, E, d) ||
        !aligned(workspace, 256))
        return BASE_ERR_WORKSPACE;
    const Span ws = {workspace, (int64_t)base::norm_workspace_size(N, E, d)};
    const Span dw = {dweight, E * d * 4}, db = {dbias, E * d * 4};
    if (clash({{dx, N * row}, dw, db, ws},
              {{x, x_rows * row}, {perm, N * 4}, {weight, E * row}, {mean, N * 4}, {rstd, N * 4},
               {offsets, (E + 1) * 4}}) ||
        clash({dw, db, ws}, {{dy, N * row}, {residual, N * row}}))
        return BASE_ERR_INVALID_ARG;
    return hip_status(base::launch_norm_backward(dy, x, perm, x_rows, k, weight, mean, rstd, offsets,
                                                 residual, dx, dweight, dbias, N, E, d,
                                                 dtype == BASE_BF16, workspace,
                                                 static_cast<hipStream_t>(stream)));
}

size_t base_expert_linear_workspace_size(int product, int64_t N, int64_t E, int64_t K, int64_t O,
                                         int dtype) {
    if (product < BASE_PRODUCT_Y || product > BASE_PRODUCT_DW) return 0;
    if (check_linear(N, E, K, O, dtype) != BASE_OK) return 0;
    return base::linear_workspace_size(product, N, E, K, O, dtype == BASE_BF16);
}

int base_expert_linear_tile(int product, int64_t N, int64_t E, int64_t K, int64_t O, int dtype,
                            int32_t *rows, int32_t *cols, int32_t *parts) {
    if (rows == nullptr || cols == nullptr || parts == nullptr || product < BASE_PRODUCT_Y ||
        product > BASE_PRODUCT_DW)
        return BASE_ERR_INVALID_ARG;
    if (const int st = check_linear(N, E, K, O, dtype)) return st;
    base::linear_tile(product, N, E, K, O, dtype == BASE_BF16, rows, cols, parts);
    return BASE_OK;
}

int base_expert_linear(const void *x, const void *w, const void *bias, const void *residual,
                       const int32_t *offsets, void *y, int64_t N, int64_t E, int64_t K, int64_t O,
                       int relu, int dtype, void *workspace, size_t workspace_bytes,
                       void *stream) {
    if (x == nullptr || w == nullptr || offsets == nullptr || y == nullptr)
        return BASE_ERR_INVALID_ARG;
    if (const int st = check_linear(N, E, K, O, dtype)) return st;
    if (relu != 0 && relu != 1) return BASE_ERR_INVALID_ARG;
    if (!aligned(x, 16) || !aligned(w, 16) || !aligned(bias, 16) || !aligned(residual, 16) ||
        !aligned(y, 16) || !aligned(offsets, 4))
        return BASE_ERR_INVALID_ARG;
    const int64_t sz = size_of(dtype);
    const Span ws = used(BASE_PRODUCT_Y, N, E, K, O, dtype, workspace);
    if (clash({{y, N * O * sz}, ws},
              {{x, N * K * sz}, {w, E * O * K * sz}, {bias, E * O * sz}, {offsets, (E + 1) * 4}}) ||
        clash({ws}, {{residual, N * O * sz}}) || partly(y, residual, N * O * sz))
        return BASE_ERR_INVALID_ARG;
    if (!there(ws, workspace_bytes)) return BASE_ERR_WORKSPACE;
    return hip_status(base::launch_linear(x, w, bias, residual, offsets, y, N, E, K, O, relu,
                                          dtype == BASE_BF16, workspace,
                                          static_cast<hipStream_t>(stream)));
}

int base_expert_linear_dx(const void *dy, const void *w, const void *relu_of,
                          const int32_t *offsets, void *dx, int64_t N, int64_t E, int64_t K,
                          int64_t O, int dtype, void *workspace, size_t workspace_bytes,
                          void *stream) {
    if (dy == nullptr || w == nullptr || offsets == nullptr || dx == nullptr)
        return BASE_ERR_INVALID_ARG;
    if (const int st = check_linear(N, E, K, O, dtype)) return st;
    if (!aligned(dy, 16) || !aligned(w, 16) || !aligned(relu_of, 16) || !aligned(dx, 16) ||
        !aligned(offsets, 4))
        return BASE_ERR_INVALID_ARG;
    const int64_t sz = size_of(dtype);
    const Span ws = used(BASE_PRODUCT_DX, N, E, K, O, dtype, workspace);
    if (clash({{dx, N * K * sz}, ws},
              {{dy, N * O * sz}, {w, E * O * K * sz}, {offsets, (E + 1) * 4}}) ||
        clash({ws}, {{relu_of, N * K * sz}}) || partly(dx, relu_of, N * K * sz))
        return BASE_ERR_INVALID_ARG;
    if (!there(ws, workspace_bytes)) return BASE_ERR_WORKSPACE;
    return hip_status(base::launch_linear_dx(dy, w, relu_of, offsets, dx, N, E, K, O,
                                             dtype == BASE_BF16, workspace,
                                             static_cast<hipStream_t>(stream)));
}

int base_expert_linear_dw(const void *dy, const void *x, const int32_t *offsets, float *dw,
                          float *db, int64_t N, int64_t E, int64_t K, int64_t O, int dtype,
                          void *workspace, size_t workspace_bytes, void *stream) {
    if (dy == nullptr || x == nullptr || offsets == nullptr || dw == nullptr)
        return BASE_ERR_INVALID_ARG;
    if (const int st = check_linear(N, E, K, O, dtype)) return st;
    if (!aligned(dy, 16) || !aligned(x, 16) || !aligned(dw, 16) || !aligned(db, 16) ||
        !aligned(offsets, 4))
        return BASE_ERR_INVALID_ARG;
    const int64_t sz = size_of(dtype);
    const Span ws = used(BASE_PRODUCT_DW, N, E, K, O, dtype, workspace);
    if (clash({{dw, E * O * K * 4}, {db, E * O * 4}, ws},
              {{dy, N * O * sz}, {x, N * K * sz}, {offsets, (E + 1) * 4}}))
        return BASE_ERR_INVALID_ARG;
    if (!there(ws, workspace_bytes)) return BASE_ERR_WORKSPACE;
    return hip_status(base::launch_linear_dw(dy, x, offsets, dw, db, N, E, K, O,
                                             dtype == BASE_BF16, workspace,
                                             static_cast<hipStream_t>(stream)));
}

}  // extern "C"
