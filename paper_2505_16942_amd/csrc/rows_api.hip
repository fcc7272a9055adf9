// Host side of the row operators declared in include/corr.h: argument checks, the workspace's layout and the order of kernels.
#include "checks.h"
#include "rows_internal.h"
#include "corr_bench.h"

namespace {

constexpr int64_t MAX_ROWS = 1LL << 30, MAX_COLS = 1LL << 21, MAX_ELEMENTS = 1LL << 36;

corr_status check_linear(corr_dtype type, corr_activation act, int64_t M, int64_t N, int64_t K) {
    if (!known(type) || !known(act) || M < 0 || N <= 0 || K <= 0) return CORR_ERR_INVALID_ARG;
    if (M > MAX_ROWS || N > MAX_COLS || K > MAX_COLS || M * N > MAX_ELEMENTS || M * K > MAX_ELEMENTS || N * K > MAX_ELEMENTS) return CORR_ERR_UNSUPPORTED;
    return CORR_OK;
}
// rows of an odd number of 16-bit elements (or an odd number apart) are copied to rows that start on 16-byte borders
bool packed(corr_dtype t, int64_t cols, int64_t stride) { return t != CORR_TYPE_F32 && ((cols | stride) & 1); }
int64_t up8(int64_t n) { return (n + 7) & ~7LL; }

struct LinearLayout { size_t x, w, part, total; bool pack_x, pack_w; ProductPlan plan; };
LinearLayout linear_layout(corr_dtype t, int64_t M, int64_t N, int64_t K, int64_t x_stride) {
    LinearLayout l = {};
    Carver c;
    l.plan = product_plan(t, 0, 0, (int)M, (int)N, (int)K);
    l.pack_x = l.plan.tile && packed(t, K, x_stride);
    l.pack_w = l.plan.tile && packed(t, K, K);
    l.x = c.take(l.pack_x ? (size_t)M * up8(K) * 2 : 0);
    l.w = c.take(l.pack_w ? (size_t)N * up8(K) * 2 : 0);
    l.part = c.take(product_part_bytes(l.plan, (int)M, (int)N));
    l.total = c.used;
    return l;
}

struct BackwardLayout { size_t x, w, dz, dz_lo, part, sums, total; bool pack_x, pack_w, own_dz, two; int parts; };
BackwardLayout backward_layout(corr_dtype t, corr_activation act, int64_t M, int64_t N, int64_t K, int64_t x_stride, int64_t dy_stride, bool fine = false) {
    BackwardLayout l = {};
    Carver c;
    l.pack_x = packed(t, K, x_stride);
    l.pack_w = packed(t, K, K);
    l.own_dz = act != CORR_ACT_NONE || packed(t, N, dy_stride);
    l.two = fine || (t == CORR_TYPE_F16 && act != CORR_ACT_NONE && act != CORR_ACT_RELU);      // d_y itself, or zero, needs no second part
    l.x = c.take(l.pack_x ? (size_t)M * up8(K) * 2 : 0);
    l.w = c.take(l.pack_w ? (size_t)N * up8(K) * 2 : 0);
    l.dz = c.take(l.own_dz ? (size_t)M * up8(N) * corr_elem_bytes(t) : 0);
    l.dz_lo = c.take(l.two ? (size_t)M * up8(N) * 2 : 0);
    const size_t px = product_part_bytes(product_plan(t, 0, 1, (int)M, (int)K, (int)N), (int)M, (int)K);
    const size_t pw = product_part_bytes(product_plan(t, 1, 1, (int)N, (int)K, (int)M), (int)N, (int)K);
    l.part = c.take(px > pw ? px : pw);
    l.parts = slope_parts(M);
    l.sums = c.take((size_t)l.parts * N * 4);
    l.total = c.used;
    return l;
}

// d_x = dz w and d_w = dz^T x, each if wanted.
hipError_t gradient_products(corr_dtype type, const BackwardLayout& l, const void* dz, int64_t ld_dz, const void* x, int64_t x_stride, const void* w,
                             void* d_x, void* d_w, int64_t M, int64_t N, int64_t K, char* ws, hipStream_t s) {
    hipError_t e = launch_pack16({x, x_stride, ws + l.x, up8(K), l.pack_x && d_w ? M : 0, K}, {w, K, ws + l.w, up8(K), l.pack_w && d_x ? N : 0, K}, s);
    ProductArgs p = {};
    p.type = type; p.act = CORR_ACT_NONE;
    p.a = dz; p.lda = ld_dz;
    if (l.two) p.a_lo = ws + l.dz_lo;
    p.part = reinterpret_cast<float*>(ws + l.part);
    if (d_x && e == hipSuccess) {
        p.b = w; p.ldb = K; p.b_rows = 1;
        if (l.pack_w) { p.b = ws + l.w; p.ldb = up8(K); }
        p.M = (int)M; p.N = (int)K; p.K = (int)N;
        p.y = d_x; p.ldy = K;
        e = launch_product(p, s);
    }
    if (d_w && e == hipSuccess) {
        p.b = x; p.ldb = x_stride; p.a_rows = p.b_rows = 1;
        if (l.pack_x) { p.b = ws + l.x; p.ldb = up8(K); }
        p.M = (int)N; p.N = (int)K; p.K = (int)M;
        p.y = d_w; p.ldy = K;
        e = launch_product(p, s);
    }
    return e;
}

corr_status check_gated(corr_dtype type, corr_activation act, int64_t M, int64_t N, int64_t K) {
    return N > MAX_COLS ? CORR_ERR_UNSUPPORTED : check_linear(type, act, M, 2 * N, K);
}
// dz is always a matrix of its own, and in two parts for fp16, and for bf16 where that costs nothing: rounded once, it adds as much error as the result's own
// rounding does (M x K -> 2 x N in one part and in two, us: 32 x 64 -> 2 x 64 25 and 25, 8 x 256 -> 2 x 1024 29 and 27; 300 x 64 -> 2 x 512 29 and 42, 1000 x 256 ->
// 2 x 512 34 and 53, 129600 x 256 -> 2 x 512 349 and 572).
BackwardLayout gated_backward_layout(corr_dtype t, int64_t M, int64_t N, int64_t K, int64_t x_stride) {
    return backward_layout(t, CORR_ACT_SILU, M, 2 * N, K, x_stride, 2 * N, t == CORR_TYPE_BF16 && M * (N < K ? N : K) <= 2048);
}

corr_status check_norm(const corr_residual_norm_args* a) {
    if (!a || !known(a->stream_type) || !known(a->type) || !known(a->gate_act) || !known(a->post) || !known(a->pre)) return CORR_ERR_INVALID_ARG;
    if (a->stream_type != a->type && a->stream_type != CORR_TYPE_F32) return CORR_ERR_INVALID_ARG;
    if (a->rows < 0 || a->cols <= 0 || !(a->eps > 0.f)) return CORR_ERR_INVALID_ARG;
    if (a->rows > MAX_ROWS || a->cols > 16384) return CORR_ERR_UNSUPPORTED;
    if (a->rows && (!a->h || a->h_stride < a->cols)) return CORR_ERR_INVALID_ARG;
    if (a->y ? a->y_stride < a->cols : (a->gate || a->scale || a->post != CORR_NORM_NONE || a->h_scale != 1.f)) return CORR_ERR_INVALID_ARG;
    if (a->gate && a->gate_stride < a->cols) return CORR_ERR_INVALID_ARG;
    if (a->h_stride > MAX_ROWS || (a->y && a->y_stride > MAX_ROWS) || (a->gate && a->gate_stride > MAX_ROWS)) return CORR_ERR_UNSUPPORTED;
    if (a->post == CORR_NORM_NONE && (a->post_weight || a->post_bias)) return CORR_ERR_INVALID_ARG;
    if (a->pre == CORR_NORM_NONE && (a->pre_weight || a->pre_bias)) return CORR_ERR_INVALID_ARG;
    const int es = corr_elem_bytes(a->stream_type), et = corr_elem_bytes(a->type);
    if (!on(a->h, es) || !on(a->y, et) || !on(a->gate, et)) return CORR_ERR_INVALID_ARG;
    for (const float* v : {a->scale, a->post_weight, a->post_bias, a->pre_weight, a->pre_bias}) if (!on(v, 4)) return CORR_ERR_INVALID_ARG;
    return CORR_OK;
}
// Absent matrices have no strides to look at.
corr_residual_norm_args plain(const corr_residual_norm_args& a) {
    corr_residual_norm_args b = a;
    if (!b.y) b.y_stride = 0;
    if (!b.gate) { b.gate_stride = 0; b.gate_act = CORR_ACT_NONE; }
    return b;
}

hipError_t launch_norm(const NormArgs& n, hipStream_t s) {
#define PAIR(S, T, name) if (n.a.stream_type == CORR_TYPE_##S && n.a.type == CORR_TYPE_##T) return launch_residual_norm_##name(n, s);
    NORM_PAIRS(PAIR)
#undef PAIR
    return hipErrorInvalidValue;
}
hipError_t launch_norm_backward(const NormArgs& n, hipStream_t s) {
#define PAIR(S, T, name) if (n.a.stream_type == CORR_TYPE_##S && n.a.type == CORR_TYPE_##T) return launch_residual_norm_backward_##name(n, s);
    NORM_PAIRS(PAIR)
#undef PAIR
    return hipErrorInvalidValue;
}

}  // namespace

// Workgroups of the gradient's kernel, each with a part of the column sums: as many as the compute units hold at a time (`full`: sums of all
// five vectors take registers), and none without a row (residual_norm.hip: `per` is the most rows that a workgroup has at a time).
int norm_backward_parts(int64_t rows, int64_t cols, bool full) {
    const int64_t per = cols <= 64 ? 32 : cols <= 128 ? 16 : cols <= 256 ? 8 : cols <= 512 ? 4 : 1;
    const int64_t units = cols <= 512 ? (full ? 2 : 3) : cols <= 1024 ? (full ? 4 : 6) : cols <= 2048 ? (full ? 2 : 3) : 1;
    const int64_t most = 256 * units, need = (rows + per - 1) / per;
    return (int)(need < most ? need : most);
}

extern "C" {

size_t corr_linear_workspace_bytes(corr_dtype type, int64_t M, int64_t N, int64_t K, int64_t x_stride) {
    if (check_linear(type, CORR_ACT_NONE, M, N, K) != CORR_OK || M == 0) return 0;
    return linear_layout(type, M, N, K, x_stride).total;
}

corr_status corr_linear(corr_dtype type, corr_activation act, const void* x, int64_t x_stride, const void* w, const float* bias,
                        const void* residual, int64_t residual_stride, void* preact, void* y, int64_t y_stride,
                        int64_t M, int64_t N, int64_t K, void* workspace, size_t workspace_bytes, void* stream) {
    corr_status st = check_linear(type, act, M, N, K);
    if (st != CORR_OK) return st;
    if (M == 0) return CORR_OK;
    if (!x || !w || !y || x_stride < K || y_stride < N || (residual && residual_stride < N)) return CORR_ERR_INVALID_ARG;
    if (x_stride > MAX_COLS || y_stride > MAX_COLS || (residual && residual_stride > MAX_COLS)) return CORR_ERR_UNSUPPORTED;
    const int es = corr_elem_bytes(type);
    if (!on(x, 4) || !on(w, 4) || !on(bias, 4) || !on(residual, es) || !on(preact, es) || !on(y, es)) return CORR_ERR_INVALID_ARG;
    const LinearLayout l = linear_layout(type, M, N, K, x_stride);
    if (l.total && (!workspace || workspace_bytes < l.total || !on(workspace, 16))) return CORR_ERR_INVALID_ARG;
    const Range out[] = {range(y, M, N, y_stride, es), range(preact, M, N, N, es), range(l.total ? workspace : nullptr, 1, (int64_t)l.total, 0, 1)};
    const Range in[] = {range(x, M, K, x_stride, es), range(w, N, K, K, es), range(bias, 1, N, N, 4)};
    if (any_overlap(out, in)) return CORR_ERR_INVALID_ARG;
    const Range res = range(residual, M, N, residual_stride, es);
    const bool in_place = residual == y && residual_stride == y_stride;
    if ((!in_place && overlap(res, out[0])) || overlap(res, out[1]) || overlap(res, out[2])) return CORR_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    char* const ws = static_cast<char*>(workspace);
    hipError_t e = hipSuccess;
    ProductArgs p = {};
    p.type = type; p.act = act;
    p.a = x; p.lda = x_stride;
    p.b = w; p.ldb = K;
    p.M = (int)M; p.N = (int)N; p.K = (int)K;
    e = launch_pack16({x, x_stride, ws + l.x, up8(K), l.pack_x ? M : 0, K}, {w, K, ws + l.w, up8(K), l.pack_w ? N : 0, K}, s);
    if (l.pack_x) { p.a = ws + l.x; p.lda = up8(K); }
    if (l.pack_w) { p.b = ws + l.w; p.ldb = up8(K); }
    p.bias = bias; p.res = residual; p.ld_res = residual_stride; p.pre = preact; p.y = y; p.ldy = y_stride;
    p.part = reinterpret_cast<float*>(ws + l.part);
    if (e == hipSuccess) e = launch_product(p, s);
    return e == hipSuccess ? CORR_OK : CORR_ERR_HIP;
}

size_t corr_linear_backward_workspace_bytes(corr_dtype type, corr_activation act, int64_t M, int64_t N, int64_t K,
                                            int64_t x_stride, int64_t d_y_stride) {
    if (check_linear(type, act, M, N, K) != CORR_OK || M == 0) return 0;
    return backward_layout(type, act, M, N, K, x_stride, d_y_stride).total;
}

corr_status corr_linear_backward(corr_dtype type, corr_activation act, const void* x, int64_t x_stride, const void* w,
                                 const void* preact, const void* d_y, int64_t d_y_stride, void* d_x, void* d_w, float* d_bias,
                                 int64_t M, int64_t N, int64_t K, void* workspace, size_t workspace_bytes, void* stream) {
    corr_status st = check_linear(type, act, M, N, K);
    if (st != CORR_OK) return st;
    const int es = corr_elem_bytes(type);
    if (!on(d_x, es) || !on(d_w, es) || !on(d_bias, 4)) return CORR_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e = hipSuccess;
    if (M == 0) {
        e = launch_zero(d_w, (size_t)N * K * es, s);
        if (e == hipSuccess) e = launch_zero(d_bias, (size_t)N * 4, s);
        return e == hipSuccess ? CORR_OK : CORR_ERR_HIP;
    }
    if (!d_y || (d_w && !x) || (d_x && !w) || (act != CORR_ACT_NONE && !preact)) return CORR_ERR_INVALID_ARG;
    if ((d_w && x_stride < K) || d_y_stride < N) return CORR_ERR_INVALID_ARG;
    if (x_stride > MAX_COLS || d_y_stride > MAX_COLS) return CORR_ERR_UNSUPPORTED;
    if (!on(x, 4) || !on(w, 4) || !on(preact, es) || !on(d_y, 4)) return CORR_ERR_INVALID_ARG;
    const BackwardLayout l = backward_layout(type, act, M, N, K, x_stride, d_y_stride);
    if (!workspace || workspace_bytes < l.total || !on(workspace, 16)) return CORR_ERR_INVALID_ARG;
    const Range out[] = {range(d_x, M, K, K, es), range(d_w, N, K, K, es), range(d_bias, 1, N, N, 4), range(workspace, 1, (int64_t)l.total, 0, 1)};
    const Range in[] = {range(d_w ? x : nullptr, M, K, x_stride, es), range(d_x ? w : nullptr, N, K, K, es),
                        range(act != CORR_ACT_NONE ? preact : nullptr, M, N, N, es), range(d_y, M, N, d_y_stride, es)};
    if (any_overlap(out, in)) return CORR_ERR_INVALID_ARG;
    char* const ws = static_cast<char*>(workspace);
    const void* dz = d_y;
    int64_t ld_dz = d_y_stride;
    float* const sums = d_bias ? reinterpret_cast<float*>(ws + l.sums) : nullptr;
    if (l.own_dz && (d_x || d_w)) { dz = ws + l.dz; ld_dz = up8(N); }
    if (dz != d_y || sums) {
        e = launch_slope(type, act, d_y, d_y_stride, preact, dz == d_y ? nullptr : ws + l.dz, dz == d_y || !l.two ? nullptr : ws + l.dz_lo, up8(N),
                         sums, M, (int)N, s);
        if (sums && e == hipSuccess) {
            const ColumnSums o = {{d_bias, nullptr, nullptr, nullptr, nullptr}};
            e = launch_column_sums(sums, l.parts, 1, (int)N, o, s);
        }
    }
    if (e == hipSuccess) e = gradient_products(type, l, dz, ld_dz, x, x_stride, w, d_x, d_w, M, N, K, ws, s);
    return e == hipSuccess ? CORR_OK : CORR_ERR_HIP;
}

size_t corr_gated_linear_workspace_bytes(corr_dtype type, int64_t M, int64_t N, int64_t K, int64_t x_stride) {
    if (check_gated(type, CORR_ACT_NONE, M, N, K) != CORR_OK || M == 0) return 0;
    return linear_layout(type, M, 2 * N, K, x_stride).total;
}

corr_status corr_gated_linear(corr_dtype type, corr_activation act, const void* x, int64_t x_stride, const void* w, const float* bias,
                              void* preact, void* y, int64_t y_stride, int64_t M, int64_t N, int64_t K,
                              void* workspace, size_t workspace_bytes, void* stream) {
    corr_status st = check_gated(type, act, M, N, K);
    if (st != CORR_OK) return st;
    if (M == 0) return CORR_OK;
    if (!x || !w || !y || x_stride < K || y_stride < N) return CORR_ERR_INVALID_ARG;
    if (x_stride > MAX_COLS || y_stride > MAX_COLS) return CORR_ERR_UNSUPPORTED;
    const int es = corr_elem_bytes(type);
    if (!on(x, 4) || !on(w, 4) || !on(bias, 4) || !on(preact, es) || !on(y, es)) return CORR_ERR_INVALID_ARG;
    const LinearLayout l = linear_layout(type, M, 2 * N, K, x_stride);
    if (l.total && (!workspace || workspace_bytes < l.total || !on(workspace, 16))) return CORR_ERR_INVALID_ARG;
    const Range out[] = {range(y, M, N, y_stride, es), range(preact, M, 2 * N, 2 * N, es), range(l.total ? workspace : nullptr, 1, (int64_t)l.total, 0, 1)};
    const Range in[] = {range(x, M, K, x_stride, es), range(w, 2 * N, K, K, es), range(bias, 1, 2 * N, 2 * N, 4)};
    if (any_overlap(out, in)) return CORR_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    char* const ws = static_cast<char*>(workspace);
    ProductArgs p = {};
    p.type = type; p.act = act; p.gated = 1;
    p.a = x; p.lda = x_stride;
    p.b = w; p.ldb = K;
    p.M = (int)M; p.N = (int)N; p.K = (int)K;
    hipError_t e = launch_pack16({x, x_stride, ws + l.x, up8(K), l.pack_x ? M : 0, K}, {w, K, ws + l.w, up8(K), l.pack_w ? 2 * N : 0, K}, s);
    if (l.pack_x) { p.a = ws + l.x; p.lda = up8(K); }
    if (l.pack_w) { p.b = ws + l.w; p.ldb = up8(K); }
    p.bias = bias; p.pre = preact; p.y = y; p.ldy = y_stride;
    p.part = reinterpret_cast<float*>(ws + l.part);
    if (e == hipSuccess) e = launch_product(p, s);
    return e == hipSuccess ? CORR_OK : CORR_ERR_HIP;
}

size_t corr_gated_linear_backward_workspace_bytes(corr_dtype type, int64_t M, int64_t N, int64_t K, int64_t x_stride) {
    if (check_gated(type, CORR_ACT_NONE, M, N, K) != CORR_OK || M == 0) return 0;
    return gated_backward_layout(type, M, N, K, x_stride).total;
}

corr_status corr_gated_linear_backward(corr_dtype type, corr_activation act, const void* x, int64_t x_stride, const void* w,
                                       const void* preact, const void* d_y, int64_t d_y_stride, void* d_x, void* d_w, float* d_bias,
                                       int64_t M, int64_t N, int64_t K, void* workspace, size_t workspace_bytes, void* stream) {
    corr_status st = check_gated(type, act, M, N, K);
    if (st != CORR_OK) return st;
    const int es = corr_elem_bytes(type);
    if (!on(d_x, es) || !on(d_w, es) || !on(d_bias, 4)) return CORR_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e = hipSuccess;
    if (M == 0) {
        e = launch_zero(d_w, (size_t)2 * N * K * es, s);
        if (e == hipSuccess) e = launch_zero(d_bias, (size_t)2 * N * 4, s);
        return e == hipSuccess ? CORR_OK : CORR_ERR_HIP;
    }
    if (!d_y || !preact || (d_w && !x) || (d_x && !w) || (d_w && x_stride < K) || d_y_stride < N) return CORR_ERR_INVALID_ARG;
    if (x_stride > MAX_COLS || d_y_stride > MAX_COLS) return CORR_ERR_UNSUPPORTED;
    if (!on(x, 4) || !on(w, 4) || !on(preact, es) || !on(d_y, es)) return CORR_ERR_INVALID_ARG;
    const BackwardLayout l = gated_backward_layout(type, M, N, K, x_stride);
    if (!workspace || workspace_bytes < l.total || !on(workspace, 16)) return CORR_ERR_INVALID_ARG;
    const Range out[] = {range(d_x, M, K, K, es), range(d_w, 2 * N, K, K, es), range(d_bias, 1, 2 * N, 2 * N, 4),
                         range(workspace, 1, (int64_t)l.total, 0, 1)};
    const Range in[] = {range(d_w ? x : nullptr, M, K, x_stride, es), range(d_x ? w : nullptr, 2 * N, K, K, es),
                        range(preact, M, 2 * N, 2 * N, es), range(d_y, M, N, d_y_stride, es)};
    if (any_overlap(out, in)) return CORR_ERR_INVALID_ARG;
    if (!d_x && !d_w && !d_bias) return CORR_OK;
    char* const ws = static_cast<char*>(workspace);
    float* const sums = d_bias ? reinterpret_cast<float*>(ws + l.sums) : nullptr;
    e = launch_slope_gated(type, act, d_y, d_y_stride, preact, d_x || d_w ? ws + l.dz : nullptr, l.two ? ws + l.dz_lo : nullptr, up8(2 * N), sums,
                           M, (int)N, s);
    if (sums && e == hipSuccess) {
        const ColumnSums o = {{d_bias, nullptr, nullptr, nullptr, nullptr}};
        e = launch_column_sums(sums, l.parts, 1, (int)(2 * N), o, s);
    }
    if (e == hipSuccess) e = gradient_products(type, l, ws + l.dz, up8(2 * N), x, x_stride, w, d_x, d_w, M, 2 * N, K, ws, s);
    return e == hipSuccess ? CORR_OK : CORR_ERR_HIP;
}

corr_status corr_debug_linear_tile(corr_dtype type, int product, int64_t M, int64_t N, int64_t K, int* tile_rows, int* tile_cols, int* splits) {
    if (!tile_rows || !tile_cols || !splits || M <= 0 || check_linear(type, CORR_ACT_NONE, M, N, K) != CORR_OK) return CORR_ERR_INVALID_ARG;
    ProductPlan p;
    switch (product) {
        case CORR_PRODUCT_Y: p = product_plan(type, 0, 0, (int)M, (int)N, (int)K); break;
        case CORR_PRODUCT_DX: p = product_plan(type, 0, 1, (int)M, (int)K, (int)N); break;
        case CORR_PRODUCT_DW: p = product_plan(type, 1, 1, (int)N, (int)K, (int)M); break;
        default: return CORR_ERR_INVALID_ARG;
    }
    product_tile(p, *tile_rows, *tile_cols);
    *splits = p.splits;
    return CORR_OK;
}

corr_status corr_debug_gated_tile(corr_dtype type, int64_t M, int64_t N, int64_t K, int* tile_rows, int* tile_cols, int* splits) {
    if (!tile_rows || !tile_cols || !splits || M <= 0 || check_gated(type, CORR_ACT_NONE, M, N, K) != CORR_OK) return CORR_ERR_INVALID_ARG;
    gated_tile(type, (int)M, (int)N, (int)K, *tile_rows, *tile_cols, *splits);
    return CORR_OK;
}

corr_status corr_residual_norm(const corr_residual_norm_args* a, void* h_out, void* n_out, void* stream) {
    corr_status st = check_norm(a);
    if (st != CORR_OK) return st;
    const int es = corr_elem_bytes(a->stream_type), et = corr_elem_bytes(a->type);
    if ((a->pre == CORR_NORM_NONE) != !n_out || (!h_out && !n_out) || (h_out && !a->y)) return CORR_ERR_INVALID_ARG;
    if (!on(h_out, es) || !on(n_out, et)) return CORR_ERR_INVALID_ARG;
    if (a->rows == 0) return CORR_OK;
    const int64_t R = a->rows, C = a->cols;
    const bool in_place = h_out == a->h && a->h_stride == C;
    const Range out[] = {range(h_out, R, C, C, es), range(n_out, R, C, C, et)};
    const Range in[] = {range(in_place ? nullptr : a->h, R, C, a->h_stride, es), range(a->y, R, C, a->y_stride, et),
                        range(a->gate, R, C, a->gate_stride, et)};
    if (any_overlap(out, in) || overlap(out[1], range(a->h, R, C, a->h_stride, es))) return CORR_ERR_INVALID_ARG;
    for (const float* v : {a->scale, a->post_weight, a->post_bias, a->pre_weight, a->pre_bias})
        for (const Range& o : out) if (overlap(o, range(v, 1, C, C, 4))) return CORR_ERR_INVALID_ARG;
    NormArgs n = {};
    n.a = plain(*a);
    n.h_out = h_out; n.n_out = n_out;
    return launch_norm(n, static_cast<hipStream_t>(stream)) == hipSuccess ? CORR_OK : CORR_ERR_HIP;
}

size_t corr_residual_norm_backward_workspace_bytes(int64_t rows, int64_t cols) {
    if (rows <= 0 || cols <= 0 || rows > MAX_ROWS || cols > 16384) return 0;
    return ((size_t)norm_backward_parts(rows, cols, false) * 5 * cols * 4 + 255) & ~(size_t)255;
}

corr_status corr_residual_norm_backward(const corr_residual_norm_args* a, const void* d_h_out, const void* d_n_out,
                                        void* d_h, void* d_y, void* d_gate, float* d_scale, float* d_post_weight,
                                        float* d_post_bias, float* d_pre_weight, float* d_pre_bias,
                                        void* workspace, size_t workspace_bytes, void* stream) {
    corr_status st = check_norm(a);
    if (st != CORR_OK) return st;
    const int64_t R = a->rows, C = a->cols;
    const int es = corr_elem_bytes(a->stream_type), et = corr_elem_bytes(a->type);
    if ((!d_h_out && !d_n_out && R) || (d_n_out && a->pre == CORR_NORM_NONE)) return CORR_ERR_INVALID_ARG;
    if ((d_y && !a->y) || (d_gate && !a->gate) || (d_scale && !a->scale) || (d_post_weight && !a->post_weight) || (d_post_bias && !a->post_bias) ||
        (d_pre_weight && !a->pre_weight) || (d_pre_bias && !a->pre_bias)) return CORR_ERR_INVALID_ARG;
    if (!on(d_h_out, es) || !on(d_n_out, et) || !on(d_h, es) || !on(d_y, et) || !on(d_gate, et)) return CORR_ERR_INVALID_ARG;
    const ColumnSums sums = {{d_scale, d_post_weight, d_post_bias, d_pre_weight, d_pre_bias}};
    bool wanted = false;
    for (float* v : sums.out) { wanted |= v != nullptr; if (!on(v, 4)) return CORR_ERR_INVALID_ARG; }
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (R == 0) return !wanted || launch_column_sums(nullptr, 0, 5, (int)C, sums, s) == hipSuccess ? CORR_OK : CORR_ERR_HIP;
    const size_t need = corr_residual_norm_backward_workspace_bytes(R, C);
    if (wanted && (!workspace || workspace_bytes < need || !on(workspace, 16))) return CORR_ERR_INVALID_ARG;
    const Range out[] = {range(d_h, R, C, C, es), range(d_y, R, C, C, et), range(d_gate, R, C, C, et), range(d_scale, 1, C, C, 4),
                         range(d_post_weight, 1, C, C, 4), range(d_post_bias, 1, C, C, 4), range(d_pre_weight, 1, C, C, 4),
                         range(d_pre_bias, 1, C, C, 4), range(wanted ? workspace : nullptr, 1, (int64_t)need, 0, 1)};
    const Range in[] = {range(a->h, R, C, a->h_stride, es), range(a->y, R, C, a->y_stride, et), range(a->gate, R, C, a->gate_stride, et),
                        range(d_h_out, R, C, C, es), range(d_n_out, R, C, C, et), range(a->scale, 1, C, C, 4), range(a->post_weight, 1, C, C, 4),
                        range(a->post_bias, 1, C, C, 4), range(a->pre_weight, 1, C, C, 4), range(a->pre_bias, 1, C, C, 4)};
    if (any_overlap(out, in)) return CORR_ERR_INVALID_ARG;
    NormArgs n = {};
    n.a = plain(*a);
    n.d_h_out = d_h_out; n.d_n_out = d_n_out;
    n.d_h = d_h; n.d_y = d_y; n.d_gate = d_gate;
    n.part = wanted ? static_cast<float*>(workspace) : nullptr;
    n.parts = norm_backward_parts(R, C, a->type == CORR_TYPE_F32 || a->scale || a->post_bias || a->pre_bias);
    hipError_t e = launch_norm_backward(n, s);
    // vectors of a norm that d_n_out does not reach have no sums of their own
    if (e == hipSuccess && wanted) e = launch_column_sums(n.part, n.parts, 5, (int)C, sums, s);
    return e == hipSuccess ? CORR_OK : CORR_ERR_HIP;
}

}  // extern "C"
