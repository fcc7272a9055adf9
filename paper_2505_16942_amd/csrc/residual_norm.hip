// Norms before and after a block, with the block's gate, its scale and the residual, and their gradient:
//   p = norm1(y) w1 + b1,   t = alpha h + s act(g) p   (h_out),   n = norm2(t) w2 + b2.
// A row's elements stay in the registers of G threads from its only load to its only store; the next row's are on their way
// meanwhile.  Sums over a row go through the lanes of a wave and, for rows that need more than a wave, LDS.  Means and squares in
// fp32; the layer norm subtracts the mean before it squares.  The gradient makes the forward pass's row again from the
// forward pass's inputs (as many bytes as reading saved ones) and keeps the sums over rows of its columns in registers from row to row.
#include "rows_internal.h"

namespace {

enum { V_SCALE, V_W1, V_B1, V_W2, V_B2, VECTORS };

template <int CTRL> __device__ __forceinline__ float dpp(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, false));
}
// Sum over aligned groups of W lanes, in every lane: neighbours, pairs, quads and eights by lane permutations inside the add,
// 16 and 32 lanes by exchanging rows of the wave with itself.
template <int W> __device__ __forceinline__ float lane_sum(float x) {
    if constexpr (W >= 2) x += dpp<0xB1>(x);             // quad_perm 1 0 3 2
    if constexpr (W >= 4) x += dpp<0x4E>(x);             // quad_perm 2 3 0 1
    if constexpr (W >= 8) x += dpp<0x141>(x);            // row_half_mirror
    if constexpr (W >= 16) x += dpp<0x140>(x);           // row_mirror
    // (the casts matter: __builtin_bit_cast of a vector's element takes its first)
    if constexpr (W >= 32) {
        const unsigned u = __builtin_bit_cast(unsigned, x);
        const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        x = __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
    }
    if constexpr (W >= 64) {
        const unsigned u = __builtin_bit_cast(unsigned, x);
        const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        x = __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
    }
    return x;
}
// Sums over the G threads of a row.  Waves of one row add up in LDS (two buffers in turn: a wave may be one sum ahead of
// another, never two).
template <int G>
struct RowSum {
    float2* lds;
    int turn;
    __device__ __forceinline__ float2 operator()(float x, float y) {
        x = lane_sum<(G < 64 ? G : 64)>(x);
        y = lane_sum<(G < 64 ? G : 64)>(y);
        if constexpr (G > 64) {
            constexpr int WAVES = G / 64;
            float2* const b = lds + (turn ^= 1) * WAVES;
            if ((threadIdx.x & 63) == 0) b[threadIdx.x >> 6] = make_float2(x, y);
            __syncthreads();
            const float2 v = b[threadIdx.x % WAVES];
            x = lane_sum<WAVES>(v.x);
            y = lane_sum<WAVES>(v.y);
        }
        return make_float2(x, y);
    }
    __device__ __forceinline__ float operator()(float x) {
        if constexpr (G > 64) return (*this)(x, 0.f).x;
        else return lane_sum<G>(x);
    }
};

// E elements of a row per thread, in pieces of V = 8: piece q of thread j begins at column (q * G + j) * V.  RAGGED: rows that start
// on their elements' borders alone and may end inside a piece; then the last piece is the row's last eight columns, some of which
// another thread has too: both compute and store the same, and sums over the row count them once (in()).
constexpr int V = 8;
template <class T, bool RAGGED> struct Piece { typedef typename RowVec<T, V>::value value; typedef value type __attribute__((aligned(RAGGED ? sizeof(T) : 16))); };
template <class T, int E> struct Raw { typename RowVec<T, V>::value v[E / V]; };
template <int G, int E, bool RAGGED>
struct Cols {
    int j, C;
    __device__ __forceinline__ int at(int piece) const { return (piece * G + j) * V; }
    __device__ __forceinline__ bool has(int piece) const { return at(piece) < C; }
    __device__ __forceinline__ int start(int piece) const { return RAGGED ? min(at(piece), C - V) : at(piece); }
    __device__ __forceinline__ bool in(int e) const {
        const int q = e / V;
        return has(q) && (!RAGGED || (C < V ? e % V < C : start(q) + e % V >= at(q)));
    }
    static constexpr bool CHOSEN = RAGGED || G >= 1024;  // the widest kernels spill less with it
    __device__ __forceinline__ bool counts(int e) const { return !CHOSEN || in(e); }
    __device__ __forceinline__ bool stays(int e) const { return CHOSEN || has(e / V); }
    template <class T> __device__ __forceinline__ void ask(const T* row, Raw<T, E>& r) const {
#pragma unroll
        for (int q = 0; q < E / V; ++q) {
            r.v[q] = {};
            if (!has(q)) continue;
            if (!RAGGED || C >= V) r.v[q] = *reinterpret_cast<const typename Piece<T, RAGGED>::type*>(row + start(q));
            else
#pragma unroll
                for (int e = 0; e < V; ++e) if (e < C) r.v[q][e] = row[e];
        }
    }
    template <class T> __device__ __forceinline__ void open(const Raw<T, E>& r, float (&v)[E]) const {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = (float)r.v[e / V][e % V];
    }
    template <class T> __device__ __forceinline__ void load(const T* row, float (&v)[E]) const {
        Raw<T, E> r;
        ask(row, r);
        open(r, v);
    }
    // OWN: of columns that two threads have, only the one's that counts them (sums that are read again)
    template <bool OWN = false, class T> __device__ __forceinline__ void store(T* row, const float (&v)[E]) const {
#pragma unroll
        for (int q = 0; q < E / V; ++q) {
            if (!has(q)) continue;
            typename Piece<T, RAGGED>::value x;
#pragma unroll
            for (int e = 0; e < V; ++e) x[e] = (T)v[q * V + e];
            if (OWN && RAGGED && start(q) < at(q)) {
#pragma unroll
                for (int e = 0; e < V; ++e) if (in(q * V + e)) row[max(start(q), 0) + e] = x[e];
            } else if (!RAGGED || C >= V) *reinterpret_cast<typename Piece<T, RAGGED>::type*>(row + start(q)) = x;
            else
#pragma unroll
                for (int e = 0; e < V; ++e) if (e < C) row[e] = x[e];
        }
    }
    // a vector of parameters; `none` where there is none
    __device__ __forceinline__ void vector(const float* p, float none, float (&v)[E]) const {
        if (p) load<float>(p, v);
        else
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = none;
    }
};
constexpr int threads_of(int G) { return G < 128 ? 256 : G; }

// Sums over a row count a column once: ragged rows say which thread does (counts()); in others what lies past the end is zero and
// stays it (stays()), which takes fewer instructions (129600 x 256 bf16 gradient: 141 -> 118 us, with fewer workgroups).
// v becomes the normalised row; returns 1 / its spread (1 for CORR_NORM_NONE).
template <int G, int E, bool RAGGED>
__device__ __forceinline__ float normalise(int kind, float (&v)[E], const Cols<G, E, RAGGED>& c, float inv, float eps, RowSum<G>& sum) {
    if (kind == CORR_NORM_NONE) return 1.f;
    if (kind == CORR_NORM_LAYER) {
        float m = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) m += c.counts(e) ? v[e] : 0.f;
        const float mean = sum(m) * inv;
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = c.stays(e) ? v[e] - mean : 0.f;
    }
    float q = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) q = c.counts(e) ? fmaf(v[e], v[e], q) : q;
    const float rho = 1.f / sqrtf(sum(q) * inv + eps);
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] *= rho;
    return rho;
}
// q, the gradient of the normalised row `hat`, becomes the gradient of the row.
template <int G, int E, bool RAGGED>
__device__ __forceinline__ void normalise_back(int kind, float (&q)[E], const float (&hat)[E], float rho, const Cols<G, E, RAGGED>& c, float inv,
                                               RowSum<G>& sum) {
    if (kind == CORR_NORM_NONE) return;
    float a = 0.f, b = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) a = c.counts(e) ? fmaf(q[e], hat[e], a) : a;
    if (kind == CORR_NORM_LAYER) {
#pragma unroll
        for (int e = 0; e < E; ++e) b += c.counts(e) ? q[e] : 0.f;
        const float2 s = sum(a, b);
        a = s.x * inv;
        b = s.y * inv;
#pragma unroll
        for (int e = 0; e < E; ++e) q[e] = c.stays(e) ? rho * (q[e] - b - hat[e] * a) : 0.f;
    } else {
        a = sum(a) * inv;
#pragma unroll
        for (int e = 0; e < E; ++e) q[e] = rho * (q[e] - hat[e] * a);
    }
}

template <class S, class T, bool RAGGED, int G, int E>
__global__ __launch_bounds__(threads_of(G)) void residual_norm_kernel(NormArgs n) {
    constexpr int GROUPS = threads_of(G) / G;
    constexpr bool KEEP = G < 1024, AHEAD = E <= V;      // vectors stay in registers from row to row; the next row is asked for early
    __shared__ float2 lds[G > 64 ? 2 * (G / 64) : 1];
    const corr_residual_norm_args& a = n.a;
    const Cols<G, E, RAGGED> c = {(int)threadIdx.x % G, (int)a.cols};
    const float inv = 1.f / (float)a.cols;
    RowSum<G> sum = {lds, 0};
    float s[E], w1[E], b1[E], w2[E], b2[E];
    if (KEEP) {
        c.vector(a.scale, 1.f, s);
        c.vector(a.post_weight, 1.f, w1); c.vector(a.post_bias, 0.f, b1);
        c.vector(a.pre_weight, 1.f, w2); c.vector(a.pre_bias, 0.f, b2);
    }
    Raw<S, E> rh;
    Raw<T, E> ry, rg;
    auto ask = [&](int64_t r) {
        if (r >= a.rows) return;
        c.ask((const S*)a.h + r * a.h_stride, rh);
        if (a.y) c.ask((const T*)a.y + r * a.y_stride, ry);
        if (a.gate) c.ask((const T*)a.gate + r * a.gate_stride, rg);
    };
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    int64_t r = (int64_t)blockIdx.x * GROUPS + threadIdx.x / G;
    if (AHEAD) ask(r);
    for (; r < a.rows; r += step) {
        float t[E], p[E], g[E];
        if (AHEAD) {
            c.open(rh, t);
            if (a.y) c.open(ry, p);
            if (a.gate) c.open(rg, g);
            ask(r + step);
        } else {
            if (a.y) c.load((const T*)a.y + r * a.y_stride, p);
            if (a.gate) c.load((const T*)a.gate + r * a.gate_stride, g);
        }
        if (a.y) {
            normalise(a.post, p, c, inv, a.eps, sum);
            if (!KEEP) c.vector(a.post_weight, 1.f, w1);
#pragma unroll
            for (int e = 0; e < E; ++e) p[e] *= w1[e];
            if (!KEEP) c.vector(a.post_bias, 0.f, w1);
#pragma unroll
            for (int e = 0; e < E; ++e) p[e] += KEEP ? b1[e] : w1[e];
            if (!KEEP) c.vector(a.scale, 1.f, w1);
#pragma unroll
            for (int e = 0; e < E; ++e) p[e] *= KEEP ? s[e] : w1[e];
            if (a.gate) {
                row_act_all(a.gate_act, g);
#pragma unroll
                for (int e = 0; e < E; ++e) p[e] *= g[e];
            }
            if (!AHEAD) c.load((const S*)a.h + r * a.h_stride, t);
#pragma unroll
            for (int e = 0; e < E; ++e) t[e] = fmaf(a.h_scale, t[e], p[e]);
            // in place, a wave may not write what another still has to read of this row
            if (RAGGED && G > 64 && n.h_out == a.h) __syncthreads();
            if (n.h_out) c.store((S*)n.h_out + r * a.cols, t);
        } else if (!AHEAD) c.load((const S*)a.h + r * a.h_stride, t);
        if (a.pre != CORR_NORM_NONE) {
            normalise(a.pre, t, c, inv, a.eps, sum);
            if (!KEEP) c.vector(a.pre_weight, 1.f, w2);
#pragma unroll
            for (int e = 0; e < E; ++e) t[e] *= w2[e];
            if (!KEEP) c.vector(a.pre_bias, 0.f, w2);
#pragma unroll
            for (int e = 0; e < E; ++e) t[e] += KEEP ? b2[e] : w2[e];
            c.store((T*)n.n_out + r * a.cols, t);
        }
    }
}

// FULL: sums for all five vectors; else for the two weights alone (no scale, no biases), which leaves registers.  Rows of a
// thousand threads (more than 4096 columns) leave few: the normalised y waits in LDS, and vectors and the gate are read again.
// Past 8192 columns there are none for the columns' sums: they are added up in the workgroup's own part, in memory.
template <class S, class T, bool RAGGED, bool FULL, int G, int E>
__global__ __launch_bounds__(threads_of(G)) void residual_norm_backward_kernel(NormArgs n) {
    constexpr int GROUPS = threads_of(G) / G;
    constexpr bool TIGHT = G >= 1024, IN_MEMORY = TIGHT && E > V, AHEAD = !TIGHT, KEEP = !TIGHT && (G <= 256 || !FULL);
    __shared__ float2 lds[G > 64 ? 2 * (G / 64) : 1];
    __shared__ float join[GROUPS > 1 ? (GROUPS - 1) * G * E : TIGHT ? G * E : 1];      // also where the normalised y waits
    const corr_residual_norm_args& a = n.a;
    const Cols<G, E, RAGGED> c = {(int)threadIdx.x % G, (int)a.cols};
    const int group = threadIdx.x / G;
    const float inv = 1.f / (float)a.cols;
    RowSum<G> sum = {lds, 0};
    float s[E], w1[E], b1[E], w2[E];
    if (KEEP) {
        c.vector(a.post_weight, 1.f, w1); c.vector(a.pre_weight, 1.f, w2);
        if (FULL) { c.vector(a.scale, 1.f, s); c.vector(a.post_bias, 0.f, b1); }
    }
    // the branch p = hat w1 + b1 of normalised y in place of it
    auto branch = [&](float (&v)[E]) {
        if (!KEEP) c.vector(a.post_weight, 1.f, w1);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] *= w1[e];
        if (FULL && a.post_bias) {
            if (!KEEP) c.vector(a.post_bias, 0.f, b1);
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] += b1[e];
        }
    };
    auto scaled = [&](float (&v)[E]) {
        if (!FULL || !a.scale) return;
        if (!KEEP) c.vector(a.scale, 1.f, s);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] *= s[e];
    };
    float* const part = n.part ? n.part + (int64_t)blockIdx.x * VECTORS * a.cols : nullptr;
    float acc[IN_MEMORY ? 1 : VECTORS][E] = {};
    bool first = true;
    auto add = [&](int v, auto value) {                  // value(e), summed over rows
        if constexpr (IN_MEMORY) {
            if (!part) return;
            float x[E] = {};
            float* const row = part + (int64_t)v * a.cols;
            if (!first) c.load(row, x);
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] += value(e);
            c.template store<true>(row, x);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) acc[v][e] += value(e);
        }
    };
    Raw<S, E> rh, rdh;
    Raw<T, E> ry, rg, rdn;
    auto ask = [&](int64_t r) {
        if (r >= a.rows) return;
        c.ask((const S*)a.h + r * a.h_stride, rh);
        if (a.y) c.ask((const T*)a.y + r * a.y_stride, ry);
        if (a.gate) c.ask((const T*)a.gate + r * a.gate_stride, rg);
        if (n.d_n_out) c.ask((const T*)n.d_n_out + r * a.cols, rdn);
        if (n.d_h_out) c.ask((const S*)n.d_h_out + r * a.cols, rdh);
    };
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    int64_t r = (int64_t)blockIdx.x * GROUPS + group;
    if (AHEAD) ask(r);
    for (; r < a.rows; r += step) {
        float t[E], p[E], g[E], D[E], x[E];              // p: normalised y; x: act(g); g: act'(g); t: the normalised row, and scratch
        Raw<S, E> now_dh = rdh;
        Raw<T, E> now_dn = rdn;
        float rho1 = 1.f;
        if (AHEAD) {
            c.open(rh, t);
            if (a.y) c.open(ry, p);
            if (a.gate) c.open(rg, g);
            ask(r + step);
        } else {
            if (a.y) c.load((const T*)a.y + r * a.y_stride, p);
            if (a.gate) c.load((const T*)a.gate + r * a.gate_stride, g);
        }
        if (a.gate) {
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = g[e];
            row_act_all(a.gate_act, x);
            if (!TIGHT) row_slope_all(a.gate_act, g);
        }
        if (a.y) {
            rho1 = normalise(a.post, p, c, inv, a.eps, sum);
            float u[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                u[e] = p[e];
                if (TIGHT) join[e * G + c.j] = p[e];
            }
            branch(u);
            if (a.gate) {
#pragma unroll
                for (int e = 0; e < E; ++e) u[e] *= x[e];
            }
            scaled(u);
            if (!AHEAD) c.load((const S*)a.h + r * a.h_stride, t);
#pragma unroll
            for (int e = 0; e < E; ++e) t[e] = fmaf(a.h_scale, t[e], u[e]);
        } else if (!AHEAD) c.load((const S*)a.h + r * a.h_stride, t);
        if (n.d_n_out) {
            const float rho2 = normalise(a.pre, t, c, inv, a.eps, sum);
            if (AHEAD) c.open(now_dn, D);
            else c.load((const T*)n.d_n_out + r * a.cols, D);
            if (a.pre_weight) add(V_W2, [&](int e) { return D[e] * t[e]; });
            if (FULL && a.pre_bias) add(V_B2, [&](int e) { return D[e]; });
            if (!KEEP) c.vector(a.pre_weight, 1.f, w2);
#pragma unroll
            for (int e = 0; e < E; ++e) D[e] *= w2[e];
            normalise_back(a.pre, D, t, rho2, c, inv, sum);
            if (n.d_h_out) {
                if (AHEAD) c.open(now_dh, t);
                else c.load((const S*)n.d_h_out + r * a.cols, t);
#pragma unroll
                for (int e = 0; e < E; ++e) D[e] += t[e];
            }
        } else {
            if (AHEAD) c.open(now_dh, D);
            else c.load((const S*)n.d_h_out + r * a.cols, D);
            if (IN_MEMORY && first) {                    // nothing reaches these: zeros
                add(V_W2, [](int) { return 0.f; });
                add(V_B2, [](int) { return 0.f; });
            }
        }
        if (n.d_h) {
            const float alpha = a.y ? a.h_scale : 1.f;
#pragma unroll
            for (int e = 0; e < E; ++e) t[e] = alpha * D[e];
            c.store((S*)n.d_h + r * a.cols, t);
        }
        if (a.y) {
            if (TIGHT) {
                if (a.gate) {
                    c.load((const T*)a.gate + r * a.gate_stride, g);
#pragma unroll
                    for (int e = 0; e < E; ++e) x[e] = g[e];
                    row_act_all(a.gate_act, x);
                    row_slope_all(a.gate_act, g);
                }
#pragma unroll
                for (int e = 0; e < E; ++e) p[e] = join[e * G + c.j];
            }
            // D becomes the gradient of act(g) p, then of p, then of the normalised y
            if ((FULL && a.scale) || n.d_gate) {
#pragma unroll
                for (int e = 0; e < E; ++e) t[e] = p[e];
                branch(t);
#pragma unroll
                for (int e = 0; e < E; ++e) t[e] *= D[e];
                if (FULL && a.scale) {
                    if (a.gate) add(V_SCALE, [&](int e) { return t[e] * x[e]; });
                    else add(V_SCALE, [&](int e) { return t[e]; });
                }
                if (n.d_gate) {
                    scaled(t);
#pragma unroll
                    for (int e = 0; e < E; ++e) t[e] *= g[e];
                    c.store((T*)n.d_gate + r * a.cols, t);
                }
            }
            scaled(D);
            if (a.gate) {
#pragma unroll
                for (int e = 0; e < E; ++e) D[e] *= x[e];
            }
            if (a.post_weight) add(V_W1, [&](int e) { return D[e] * p[e]; });
            if (FULL && a.post_bias) add(V_B1, [&](int e) { return D[e]; });
            if (a.post_weight) {
                if (!KEEP) c.vector(a.post_weight, 1.f, w1);
#pragma unroll
                for (int e = 0; e < E; ++e) D[e] *= w1[e];
            }
            normalise_back(a.post, D, p, rho1, c, inv, sum);
            if (n.d_y) c.store((T*)n.d_y + r * a.cols, D);
        }
        first = false;
    }
    if (!part) return;
    if constexpr (!IN_MEMORY) {
#pragma unroll
        for (int v = 0; v < VECTORS; ++v) {
            if (!FULL && v != V_W1 && v != V_W2) continue;
            if constexpr (GROUPS > 1) {
                __syncthreads();
                if (group) {
#pragma unroll
                    for (int e = 0; e < E; ++e) join[((group - 1) * E + e) * G + c.j] = acc[v][e];
                }
                __syncthreads();
                if (!group)
                    for (int o = 0; o < GROUPS - 1; ++o)
#pragma unroll
                        for (int e = 0; e < E; ++e) acc[v][e] += join[(o * E + e) * G + c.j];
            }
            if (!group) c.store(part + (int64_t)v * a.cols, acc[v]);
        }
    }
}

template <class S, class T, bool BACK, bool FULL, bool RAGGED, int G, int E>
void run(const NormArgs& n, hipStream_t s) {
    constexpr int THREADS = threads_of(G), GROUPS = THREADS / G;
    if constexpr (BACK) hipLaunchKernelGGL((residual_norm_backward_kernel<S, T, RAGGED, FULL, G, E>), dim3(n.parts), dim3(THREADS), 0, s, n);
    else {
        const int64_t need = (n.a.rows + GROUPS - 1) / GROUPS, most = 2048 * 256 / THREADS;
        hipLaunchKernelGGL((residual_norm_kernel<S, T, RAGGED, G, E>), dim3((unsigned)(need < most ? need : most)), dim3(THREADS), 0, s, n);
    }
}
template <class S, class T, bool BACK, bool FULL, bool RAGGED>
void by_cols(const NormArgs& n, hipStream_t s) {
    const int64_t C = n.a.cols;
    if (C <= 64) run<S, T, BACK, FULL, RAGGED, 8, 8>(n, s);
    else if (C <= 128) run<S, T, BACK, FULL, RAGGED, 16, 8>(n, s);
    else if (C <= 256) run<S, T, BACK, FULL, RAGGED, 32, 8>(n, s);
    else if (C <= 512) run<S, T, BACK, FULL, RAGGED, 64, 8>(n, s);
    else if (C <= 1024) run<S, T, BACK, FULL, RAGGED, 128, 8>(n, s);
    else if (C <= 2048) run<S, T, BACK, FULL, RAGGED, 256, 8>(n, s);
    else if (C <= 4096) run<S, T, BACK, FULL, RAGGED, 512, 8>(n, s);
    else if (C <= 8192) run<S, T, BACK, FULL, RAGGED, 1024, 8>(n, s);
    else run<S, T, BACK, FULL, RAGGED, 1024, 16>(n, s);
}
template <class S, class T, bool BACK, bool FULL>
hipError_t by_border(const NormArgs& n, hipStream_t s) {
    const corr_residual_norm_args& a = n.a;
    const uintptr_t all = (uintptr_t)a.h | (uintptr_t)a.y | (uintptr_t)a.gate | (uintptr_t)a.scale | (uintptr_t)a.post_weight |
                          (uintptr_t)a.post_bias | (uintptr_t)a.pre_weight | (uintptr_t)a.pre_bias | (uintptr_t)n.h_out | (uintptr_t)n.n_out |
                          (uintptr_t)n.d_h_out | (uintptr_t)n.d_n_out | (uintptr_t)n.d_h | (uintptr_t)n.d_y | (uintptr_t)n.d_gate;
    if ((all & 15) == 0 && ((a.cols | a.h_stride | a.y_stride | a.gate_stride) & (V - 1)) == 0) by_cols<S, T, BACK, FULL, false>(n, s);
    else by_cols<S, T, BACK, FULL, true>(n, s);
    return hipGetLastError();
}
template <class S, class T>
hipError_t forward(const NormArgs& n, hipStream_t s) { return by_border<S, T, false, true>(n, s); }
template <class S, class T>
hipError_t backward(const NormArgs& n, hipStream_t s) {
    return n.a.scale || n.a.post_bias || n.a.pre_bias ? by_border<S, T, true, true>(n, s) : by_border<S, T, true, false>(n, s);
}

}  // namespace

// This file is compiled once for each pair of types (CORR_NORM_PAIR, in NORM_PAIRS' order).
#if CORR_NORM_PAIR == 0
#define S float
#define T float
#define NAME(f) f##_f32_f32
#elif CORR_NORM_PAIR == 1
#define S float
#define T __bf16
#define NAME(f) f##_f32_bf16
#elif CORR_NORM_PAIR == 2
#define S float
#define T _Float16
#define NAME(f) f##_f32_f16
#elif CORR_NORM_PAIR == 3
#define S __bf16
#define T __bf16
#define NAME(f) f##_bf16_bf16
#else
#define S _Float16
#define T _Float16
#define NAME(f) f##_f16_f16
#endif
hipError_t NAME(launch_residual_norm)(const NormArgs& n, hipStream_t s) { return forward<S, T>(n, s); }
hipError_t NAME(launch_residual_norm_backward)(const NormArgs& n, hipStream_t s) { return backward<S, T>(n, s); }
