// Launchers of attention.hip (one object per type), called by maps_api.hip after its checks.
#pragma once
#include "rows.h"

// A key head is read by `per` query heads: a pair (item, key head) has rows = Lq * per rows, row r being query r / per of head
// hk * per + r % per, so that shared heads meet in one tile.
struct AttentionArgs {
    const void *q, *k, *v;
    int64_t q_item, q_row, q_head, k_item, k_row, k_head, v_item, v_row, v_head;      // elements
    int B, Lq, Lk, HK, per, rows, D;
    float scale;
    const int* k_lengths; const uint8_t* key_mask;
    void* out; float* lse;                 // [B][Lq][HK * per][D]; [B][HK * per][Lq] or null
    void *k3, *v3, *q3, *o3;                // fp32: three bf16 planes of k and v, q and d_out, [3][B][L][H][D] each
    float* part_o; float* part_ml;         // splits > 1: [splits][B * HK][rows][D] sums, [..][2] {exponent of two, sum}
    // gradient
    const void* o; const float* saved_lse; const void* d_out;
    float* aux;                            // [2][B * HK][rows up to a multiple of 64]: lse log2 e (less LIFT; 2 lse of far rows), sum of d_out out
    void *d_q, *d_k, *d_v;                 // each may be null (d_k and d_v together)
    float *part_q, *part_k, *part_v;       // splits > 1: [splits] of the gradient's elements
};
// How a call is cut up: `tile` rows (keys) a workgroup of `waves` waves, `splits` shares of `share` keys (rows) each.
// `planes`: fp32 tiles come from three planes that are made first.
// `two`: 16-bit weights and dS in two parts, and one block of rows (keys) a wave.
struct AttentionPlan { int waves, blocks, tile, tiles, splits, share; bool planes, two; };
enum AttentionPass { PASS_FORWARD = 0, PASS_DQ, PASS_DKV };
AttentionPlan attention_plan(corr_dtype t, AttentionPass pass, int B, int Lq, int Lk, int HK, int per, int D);
__host__ __device__ static inline int attention_aux_rows(int rows) { return (rows + 63) & ~63; }

#define ATTENTION_TYPES(X) X(F32, f32) X(BF16, bf16) X(F16, f16)
#define CORR_DECLARE_ATTENTION(T, name)                                                                \
    hipError_t launch_attention_##name(const AttentionArgs& a, const AttentionPlan& p, hipStream_t s); \
    hipError_t launch_attention_backward_##name(const AttentionArgs& a, const AttentionPlan& pq, const AttentionPlan& pk, hipStream_t s);
ATTENTION_TYPES(CORR_DECLARE_ATTENTION)
#undef CORR_DECLARE_ATTENTION
