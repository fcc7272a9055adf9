// Host side of the operators on maps declared in include/corr.h: argument checks, the workspace's layout and the order of kernels.
#include "attention.h"
#include "checks.h"
#include "group_norm.h"

namespace {

constexpr int64_t MAX_LENGTH = 1LL << 30, MAX_STRIDE = 1LL << 21, MAX_ITEM = 1LL << 40, MAX_ELEMENTS = 1LL << 36;

// ---- attention
corr_status check_sizes(corr_dtype type, int64_t B, int64_t Lq, int64_t Lk, int64_t H, int64_t HK, int64_t D) {
    if (!known(type) || B < 0 || Lq < 0 || Lk < 0 || H <= 0 || HK <= 0 || D <= 0 || H % HK) return CORR_ERR_INVALID_ARG;
    if (D % 8 || D > 256 || H > 128 || B > 1 << 20 || B * HK > 1 << 20 || Lq > MAX_LENGTH || Lk > MAX_LENGTH) return CORR_ERR_UNSUPPORTED;
    if (Lq * (H / HK) > MAX_LENGTH || B * H * D * Lq > MAX_ELEMENTS || B * HK * D * Lk > MAX_ELEMENTS) return CORR_ERR_UNSUPPORTED;
    return CORR_OK;
}
struct Strided { const void* p; int64_t item, row, head, L, H; };
corr_status check_strided(const corr_attention_args* a, const Strided& x) {
    if (!x.L || !a->B) return CORR_OK;
    if (!x.p || x.item < 0 || x.row < 0 || x.head < 0) return CORR_ERR_INVALID_ARG;
    if (x.item > MAX_ITEM || x.row > MAX_STRIDE || x.head > MAX_STRIDE) return CORR_ERR_UNSUPPORTED;
    if (!on(x.p, 4) || (a->type != CORR_TYPE_F32 && ((x.item | x.row | x.head) & 1))) return CORR_ERR_INVALID_ARG;
    return CORR_OK;
}
Strided q_of(const corr_attention_args* a) { return {a->q, a->q_item, a->q_row, a->q_head, a->Lq, a->H}; }
Strided k_of(const corr_attention_args* a) { return {a->k, a->k_item, a->k_row, a->k_head, a->Lk, a->HK}; }
Strided v_of(const corr_attention_args* a) { return {a->v, a->v_item, a->v_row, a->v_head, a->Lk, a->HK}; }
Range range(const corr_attention_args* a, const Strided& x) {
    if (!x.L || !a->B || !x.p) return {0, 0, 0, 0};
    const int64_t last = (a->B - 1) * x.item + (x.L - 1) * x.row + (x.H - 1) * x.head + a->D;
    return {(uintptr_t)x.p, (uintptr_t)x.p + (uintptr_t)last * corr_elem_bytes(a->type), 0, 0};
}
corr_status check_attention(const corr_attention_args* a) {
    if (!a) return CORR_ERR_INVALID_ARG;
    corr_status st = check_sizes(a->type, a->B, a->Lq, a->Lk, a->H, a->HK, a->D);
    for (const Strided& x : {q_of(a), k_of(a), v_of(a)}) if (st == CORR_OK) st = check_strided(a, x);
    if (st != CORR_OK) return st;
    if (!(a->scale > 0.f && a->scale <= 0x1p127f) || !on(a->k_lengths, 4)) return CORR_ERR_INVALID_ARG;      // scale log2 e is finite
    return CORR_OK;
}
AttentionArgs kernel_args(const corr_attention_args* a) {
    AttentionArgs k = {};
    k.q = a->q; k.q_item = a->q_item; k.q_row = a->q_row; k.q_head = a->q_head;
    k.k = a->k; k.k_item = a->k_item; k.k_row = a->k_row; k.k_head = a->k_head;
    k.v = a->v; k.v_item = a->v_item; k.v_row = a->v_row; k.v_head = a->v_head;
    k.B = (int)a->B; k.Lq = (int)a->Lq; k.Lk = (int)a->Lk; k.HK = (int)a->HK; k.per = (int)(a->H / a->HK); k.D = (int)a->D;
    k.rows = k.Lq * k.per;
    k.scale = a->scale; k.k_lengths = a->k_lengths; k.key_mask = a->key_mask;
    return k;
}
// a launch has fewer than 2^32 threads
bool too_many(const AttentionPlan& p, int64_t B, int64_t HK) { return (int64_t)p.tiles * p.splits * B * HK * p.waves >= 1LL << 26; }

struct AttentionLayout { AttentionPlan plan; size_t o, ml, k3, v3, total; };
AttentionLayout attention_layout(corr_dtype t, int64_t B, int64_t Lq, int64_t Lk, int64_t H, int64_t HK, int64_t D) {
    AttentionLayout l = {};
    Carver c;
    l.plan = attention_plan(t, PASS_FORWARD, (int)B, (int)Lq, (int)Lk, (int)HK, (int)(H / HK), (int)D);
    const size_t rows = l.plan.splits > 1 ? (size_t)l.plan.splits * B * H * Lq : 0;
    l.o = c.take(rows * D * 4);
    l.ml = c.take(rows * 8);
    const size_t planes = l.plan.planes ? (size_t)B * Lk * HK * D * 6 : 0;
    l.k3 = c.take(planes);
    l.v3 = c.take(planes);
    l.total = c.used;
    return l;
}
struct GradientLayout { AttentionPlan q, kv; size_t aux, part_q, part_k, part_v, k3, v3, q3, o3, total; };
GradientLayout gradient_layout(corr_dtype t, int64_t B, int64_t Lq, int64_t Lk, int64_t H, int64_t HK, int64_t D) {
    GradientLayout l = {};
    Carver c;
    const int per = (int)(H / HK);
    l.q = attention_plan(t, PASS_DQ, (int)B, (int)Lq, (int)Lk, (int)HK, per, (int)D);
    l.kv = attention_plan(t, PASS_DKV, (int)B, (int)Lq, (int)Lk, (int)HK, per, (int)D);
    l.aux = c.take((size_t)B * HK * attention_aux_rows((int)(Lq * per)) * 8);
    l.part_q = c.take(l.q.splits > 1 ? (size_t)l.q.splits * B * Lq * H * D * 4 : 0);
    const size_t keys = l.kv.splits > 1 ? (size_t)l.kv.splits * B * Lk * HK * D * 4 : 0;
    l.part_k = c.take(keys);
    l.part_v = c.take(keys);
    const size_t key_planes = l.q.planes ? (size_t)B * Lk * HK * D * 6 : 0, row_planes = l.kv.planes ? (size_t)B * Lq * H * D * 6 : 0;
    l.k3 = c.take(key_planes);
    l.v3 = c.take(key_planes);
    l.q3 = c.take(row_planes);
    l.o3 = c.take(row_planes);
    l.total = c.used;
    return l;
}

// ---- group norm
corr_status check_group_norm(corr_dtype type, corr_activation act, int64_t B, int64_t P, int64_t C, int64_t G) {
    if (!known(type) || !known(act) || B < 0 || P < 0 || C <= 0 || G <= 0 || C % G) return CORR_ERR_INVALID_ARG;
    if (C > 16384 || B > 65535 || B * C > 1 << 23 || P > MAX_LENGTH || B * P > MAX_LENGTH) return CORR_ERR_UNSUPPORTED;
    return CORR_OK;
}
struct GroupNormLayout { GroupNormArgs args; size_t part, sums, stats, total; };
GroupNormLayout group_norm_layout(corr_dtype type, int64_t B, int64_t P, int64_t C, int64_t G, bool gradient) {
    GroupNormLayout l = {};
    Carver c;
    l.args.type = type;
    l.args.B = (int)B; l.args.P = P; l.args.C = (int)C; l.args.G = (int)G;
    group_norm_plan(l.args, gradient);
    l.part = c.take((size_t)B * l.args.parts * C * 8);
    if (gradient) l.sums = c.take((size_t)B * C * 8);
    else l.stats = c.take((size_t)B * G * 8);            // where the caller keeps none
    l.total = c.used;
    return l;
}

}  // namespace

extern "C" {

size_t corr_group_norm_workspace_bytes(corr_dtype type, int64_t B, int64_t P, int64_t C, int64_t G) {
    if (check_group_norm(type, CORR_ACT_NONE, B, P, C, G) != CORR_OK || !B || !P) return 0;
    return group_norm_layout(type, B, P, C, G, false).total;
}

corr_status corr_group_norm(corr_dtype type, corr_activation act, const void* x, int64_t x_stride, const float* weight, const float* bias,
                            float eps, float* stats, void* y, int64_t B, int64_t P, int64_t C, int64_t G,
                            void* workspace, size_t workspace_bytes, void* stream) {
    corr_status st = check_group_norm(type, act, B, P, C, G);
    if (st != CORR_OK) return st;
    if (!(eps > 0.f) || !on(stats, 4) || !on(weight, 4) || !on(bias, 4)) return CORR_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (!B || !P) return launch_zero(stats, (size_t)B * G * 8, s) == hipSuccess ? CORR_OK : CORR_ERR_HIP;
    const int es = corr_elem_bytes(type);
    if (!x || !y || x_stride < C || !on(x, es) || !on(y, es)) return CORR_ERR_INVALID_ARG;
    if (x_stride > MAX_STRIDE) return CORR_ERR_UNSUPPORTED;
    const GroupNormLayout l = group_norm_layout(type, B, P, C, G, false);
    if (!workspace || workspace_bytes < l.total || !on(workspace, 16)) return CORR_ERR_INVALID_ARG;
    const bool in_place = y == x && x_stride == C;
    const Range outs[] = {range(y, B * P, C, C, es), range(stats, 1, B * G * 2, 0, 4), range(workspace, 1, (int64_t)l.total, 0, 1)};
    const Range in[] = {range(in_place ? nullptr : x, B * P, C, x_stride, es), range(weight, 1, C, 0, 4), range(bias, 1, C, 0, 4)};
    if (any_overlap(outs, in)) return CORR_ERR_INVALID_ARG;
    GroupNormArgs a = l.args;
    char* const ws = static_cast<char*>(workspace);
    a.act = act; a.eps = eps;
    a.x = x; a.x_stride = x_stride; a.weight = weight; a.bias = bias; a.y = y;
    a.stats = stats ? stats : reinterpret_cast<float*>(ws + l.stats);
    a.part = reinterpret_cast<float*>(ws + l.part);
    return launch_group_norm(a, s) == hipSuccess ? CORR_OK : CORR_ERR_HIP;
}

size_t corr_group_norm_backward_workspace_bytes(corr_dtype type, int64_t B, int64_t P, int64_t C, int64_t G) {
    if (check_group_norm(type, CORR_ACT_NONE, B, P, C, G) != CORR_OK || !B || !P) return 0;
    return group_norm_layout(type, B, P, C, G, true).total;
}

corr_status corr_group_norm_backward(corr_dtype type, corr_activation act, const void* x, int64_t x_stride, const float* stats,
                                     const float* weight, const float* bias, const void* d_y, int64_t d_y_stride,
                                     void* d_x, float* d_weight, float* d_bias, int64_t B, int64_t P, int64_t C, int64_t G,
                                     void* workspace, size_t workspace_bytes, void* stream) {
    corr_status st = check_group_norm(type, act, B, P, C, G);
    if (st != CORR_OK) return st;
    const int es = corr_elem_bytes(type);
    if (!on(d_x, es) || !on(d_weight, 4) || !on(d_bias, 4)) return CORR_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (!B || !P) {
        hipError_t e = launch_zero(d_weight, (size_t)C * 4, s);
        if (e == hipSuccess) e = launch_zero(d_bias, (size_t)C * 4, s);
        return e == hipSuccess ? CORR_OK : CORR_ERR_HIP;
    }
    if (!x || !stats || !d_y || x_stride < C || d_y_stride < C || !on(x, es) || !on(d_y, es) || !on(stats, 4) || !on(weight, 4) || !on(bias, 4))
        return CORR_ERR_INVALID_ARG;
    if (x_stride > MAX_STRIDE || d_y_stride > MAX_STRIDE) return CORR_ERR_UNSUPPORTED;
    const GroupNormLayout l = group_norm_layout(type, B, P, C, G, true);
    if (!workspace || workspace_bytes < l.total || !on(workspace, 16)) return CORR_ERR_INVALID_ARG;
    const Range outs[] = {range(d_x, B * P, C, C, es), range(d_weight, 1, C, 0, 4), range(d_bias, 1, C, 0, 4),
                          range(workspace, 1, (int64_t)l.total, 0, 1)};
    const Range in[] = {range(x, B * P, C, x_stride, es), range(d_y, B * P, C, d_y_stride, es), range(stats, 1, B * G * 2, 0, 4),
                        range(weight, 1, C, 0, 4), range(bias, 1, C, 0, 4)};
    if (any_overlap(outs, in)) return CORR_ERR_INVALID_ARG;
    GroupNormArgs a = l.args;
    char* const ws = static_cast<char*>(workspace);
    a.act = act;
    a.x = x; a.x_stride = x_stride; a.weight = weight; a.bias = bias; a.stats = const_cast<float*>(stats);
    a.d_y = d_y; a.d_y_stride = d_y_stride; a.d_x = d_x; a.d_weight = d_weight; a.d_bias = d_bias;
    a.part = reinterpret_cast<float*>(ws + l.part);
    a.sums = reinterpret_cast<float*>(ws + l.sums);
    return launch_group_norm_backward(a, s) == hipSuccess ? CORR_OK : CORR_ERR_HIP;
}

size_t corr_attention_workspace_bytes(corr_dtype type, int64_t B, int64_t Lq, int64_t Lk, int64_t H, int64_t HK, int64_t D) {
    if (check_sizes(type, B, Lq, Lk, H, HK, D) != CORR_OK || !B || !Lq) return 0;
    return attention_layout(type, B, Lq, Lk, H, HK, D).total;
}

corr_status corr_attention(const corr_attention_args* a, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    corr_status st = check_attention(a);
    if (st != CORR_OK) return st;
    if (!a->B || !a->Lq) return CORR_OK;
    const int es = corr_elem_bytes(a->type);
    if (!out || !on(out, es) || !on(lse, 4)) return CORR_ERR_INVALID_ARG;
    const AttentionLayout l = attention_layout(a->type, a->B, a->Lq, a->Lk, a->H, a->HK, a->D);
    if (too_many(l.plan, a->B, a->HK)) return CORR_ERR_UNSUPPORTED;
    if (l.total && (!workspace || workspace_bytes < l.total || !on(workspace, 16))) return CORR_ERR_INVALID_ARG;
    const int64_t rows = a->B * a->Lq * a->H;
    const Range outs[] = {range(out, 1, rows * a->D, 0, es), range(lse, 1, rows, 0, 4), range(l.total ? workspace : nullptr, 1, (int64_t)l.total, 0, 1)};
    const Range in[] = {range(a, q_of(a)), range(a, k_of(a)), range(a, v_of(a)), range(a->k_lengths, 1, a->B, 0, 4),
                        range(a->key_mask, a->Lk ? 1 : 0, a->B * a->Lk, 0, 1)};
    if (any_overlap(outs, in)) return CORR_ERR_INVALID_ARG;
    AttentionArgs k = kernel_args(a);
    k.out = out; k.lse = lse;
    char* const ws = static_cast<char*>(workspace);
    k.part_o = reinterpret_cast<float*>(ws + l.o); k.part_ml = reinterpret_cast<float*>(ws + l.ml);
    k.k3 = ws + l.k3; k.v3 = ws + l.v3;
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e = hipErrorInvalidValue;
#define TYPE(T, name) if (a->type == CORR_TYPE_##T) e = launch_attention_##name(k, l.plan, s);
    ATTENTION_TYPES(TYPE)
#undef TYPE
    return e == hipSuccess ? CORR_OK : CORR_ERR_HIP;
}

size_t corr_attention_backward_workspace_bytes(corr_dtype type, int64_t B, int64_t Lq, int64_t Lk, int64_t H, int64_t HK, int64_t D) {
    if (check_sizes(type, B, Lq, Lk, H, HK, D) != CORR_OK || !B || !Lq || !Lk) return 0;
    return gradient_layout(type, B, Lq, Lk, H, HK, D).total;
}

corr_status corr_attention_backward(const corr_attention_args* a, const void* out, const float* lse, const void* d_out,
                                    void* d_q, void* d_k, void* d_v, void* workspace, size_t workspace_bytes, void* stream) {
    corr_status st = check_attention(a);
    if (st != CORR_OK) return st;
    const int es = corr_elem_bytes(a->type);
    if (!d_k != !d_v || !on(d_q, es) || !on(d_k, es) || !on(d_v, es)) return CORR_ERR_INVALID_ARG;
    if (!a->B || (!d_q && !d_k)) return CORR_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int64_t rows = a->B * a->Lq * a->H, keys = a->B * a->Lk * a->HK;
    hipError_t e = hipSuccess;
    if (!rows || !keys) {
        e = launch_zero(d_q, (size_t)rows * a->D * es, s);
        if (e == hipSuccess) e = launch_zero(d_k, (size_t)keys * a->D * es, s);
        if (e == hipSuccess) e = launch_zero(d_v, (size_t)keys * a->D * es, s);
        return e == hipSuccess ? CORR_OK : CORR_ERR_HIP;
    }
    if (!out || !lse || !d_out || !on(out, es) || !on(lse, 4) || !on(d_out, 4)) return CORR_ERR_INVALID_ARG;
    const GradientLayout l = gradient_layout(a->type, a->B, a->Lq, a->Lk, a->H, a->HK, a->D);
    if (too_many(l.q, a->B, a->HK) || too_many(l.kv, a->B, a->HK)) return CORR_ERR_UNSUPPORTED;
    if (!workspace || workspace_bytes < l.total || !on(workspace, 16)) return CORR_ERR_INVALID_ARG;
    const Range outs[] = {range(d_q, 1, rows * a->D, 0, es), range(d_k, 1, keys * a->D, 0, es), range(d_v, 1, keys * a->D, 0, es),
                          range(workspace, 1, (int64_t)l.total, 0, 1)};
    const Range in[] = {range(a, q_of(a)), range(a, k_of(a)), range(a, v_of(a)), range(a->k_lengths, 1, a->B, 0, 4),
                        range(a->key_mask, 1, a->B * a->Lk, 0, 1), range(out, 1, rows * a->D, 0, es), range(lse, 1, rows, 0, 4),
                        range(d_out, 1, rows * a->D, 0, es)};
    if (any_overlap(outs, in)) return CORR_ERR_INVALID_ARG;
    AttentionArgs k = kernel_args(a);
    char* const ws = static_cast<char*>(workspace);
    k.o = out; k.saved_lse = lse; k.d_out = d_out;
    k.aux = reinterpret_cast<float*>(ws + l.aux);
    k.part_q = reinterpret_cast<float*>(ws + l.part_q);
    k.part_k = reinterpret_cast<float*>(ws + l.part_k);
    k.part_v = reinterpret_cast<float*>(ws + l.part_v);
    k.k3 = ws + l.k3; k.v3 = ws + l.v3; k.q3 = ws + l.q3; k.o3 = ws + l.o3;
    k.d_q = d_q; k.d_k = d_k; k.d_v = d_v;
    e = hipErrorInvalidValue;
#define TYPE(T, name) if (a->type == CORR_TYPE_##T) e = launch_attention_backward_##name(k, l.q, l.kv, s);
    ATTENTION_TYPES(TYPE)
#undef TYPE
    return e == hipSuccess ? CORR_OK : CORR_ERR_HIP;
}

}  // extern "C"
