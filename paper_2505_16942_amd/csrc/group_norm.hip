// Norm over the channels of a group and all pixels of an item, with an activation, channels last, and its gradient.
// Bound by bytes: the forward pass reads x twice (for the statistics, which need all of a group, and for y) and writes y once, the gradient reads x and
// d_y twice.  2 x 518400 x 256 in 32 groups, bf16 (265 MB an item: no cache holds it): 346 us, of that statistics 140 (while the last result leaves the
// memory-side cache) and y 191 (5.5 TB/s), 4.6 TB/s over three passes, a copy's rate.  Gradient of 2 x 129600 x 128 in 8 groups, bf16: 85 us, sums 38
// (3.6 TB/s), d_x 41 (4.9 TB/s).  Small ones are launches: 4 x 7285 x 96 in 32, fp32: gradient 24 us in three of 10, 6 and 11.
#include <algorithm>
#include <type_traits>
#include "matrix.h"
#include "group_norm.h"

namespace {

constexpr int THREADS = 256, JOIN_THREADS = 1024;
inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// A thread has V neighbouring channels (16 bytes of them) and every rt-th row of its workgroup's share; ct threads stand beside each other.
template <int V> struct Columns {
    int ct, rt, c, r0, left;
    __device__ __forceinline__ Columns(int C, int ct_) : ct(ct_), rt(THREADS / ct_) {
        c = (blockIdx.x * ct + threadIdx.x % ct) * V;
        r0 = threadIdx.x / ct;
        left = C - c;
    }
};
template <int V> int threads_across(int C) {
    int ct = 1;
    while (ct < THREADS && ct * V < C) ct *= 2;
    return ct;
}

// Half the difference of two values, which no finite ones overflow.
__device__ __forceinline__ float half_apart(float x, float y) { return 0.5f * x - 0.5f * y; }
// n values with mean and sum of squares about it, and m more: Chan, Golub and LeVeque's rule, which cancels nothing however large the mean is
__device__ __forceinline__ void merge(float n, float& mean, float& square, float m, float mean2, float square2) {
    if (m == 0.f) return;
    const float d = half_apart(mean2, mean), f = m / (n + m);
    mean = fmaf(d, 2.f * f, mean);
    square += square2 + d * (4.f * n * f) * d;
}
// A first mean, of values times their shares of one, is off by the roundings of sums as large as the values; the shares of what the values differ from it
// put that right, and make a constant's mean that constant.  (Differences from one of the values instead would have the roundings of that one, however far
// it lies from the others.)  Rounded past the largest value it would be infinite; NaN and infinities come back with the differences.
__device__ __forceinline__ float finite(float mean) { return fminf(fmaxf(mean, -3.4028235e38f), 3.4028235e38f); }

// U rows of a thread's V channels as they are stored, rt rows apart.
template <class T, int V, int U> struct Chunk {
    typename Some<T, V>::type x[U];
    __device__ __forceinline__ void load_row(int u, const T* q, int left) {
        if (left >= V) x[u] = *reinterpret_cast<const typename Some<T, V>::type*>(q);
        else
#pragma unroll
            for (int e = 0; e < V; ++e) x[u][e] = e < left ? q[e] : (T)0.f;
    }
    __device__ __forceinline__ void load(const T* p, int64_t step, int left) {
#pragma unroll
        for (int u = 0; u < U; ++u) load_row(u, p + u * step, left);
    }
    __device__ __forceinline__ void load_first(const T* p, int64_t step, int left, int rows) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u < rows) load_row(u, p + u * step, left);
            else x[u] = typename Some<T, V>::type{};
        }
    }
    __device__ __forceinline__ void get(int u, float (&v)[V]) const {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = (float)x[u][e];
    }
};
// The workgroup's rows of N matrices, U rows a thread at a time, the next on their way: f(chunks, first row, how many of the U).  Whole chunks are
// loaded without a question, the rest at the end.
template <class T, int V, int U, int N, class F>
__device__ __forceinline__ void each_chunk(const T* const (&p)[N], const int64_t (&stride)[N], int rows, int r0, int rt, int left, F f) {
    Chunk<T, V, U> next[N];
    const int whole = rows / (U * rt);
    const T* at[N];
#pragma unroll
    for (int i = 0; i < N; ++i) at[i] = p[i] + r0 * stride[i];
    const int rest = min(U, max(0, (rows - whole * U * rt - r0 + rt - 1) / rt));
    auto ask = [&](int k) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (k < whole) next[i].load(at[i], rt * stride[i], left);
            else next[i].load_first(at[i], rt * stride[i], left, rest);
            at[i] += U * rt * stride[i];
        }
    };
    ask(0);
    for (int k = 0; k < whole; ++k) {
        Chunk<T, V, U> now[N];
#pragma unroll
        for (int i = 0; i < N; ++i) now[i] = next[i];
        ask(k + 1);
        f(now, r0 + k * U * rt, std::integral_constant<int, U>{});
    }
    if (rest) f(next, r0 + whole * U * rt, rest);
}

// Means and squares of every channel over the workgroup's rows, U rows at a time from registers, the next U on their way.
template <class T, int V>
__global__ __launch_bounds__(THREADS) void stats_kernel(GroupNormArgs a, int ct) {
    constexpr int U = 8;
    __shared__ float means[V][THREADS], squares[V][THREADS];
    const Columns<V> at(a.C, ct);
    const int64_t lo = blockIdx.y * a.share, hi = min(a.P, lo + a.share), item = blockIdx.z * a.P;
    const int rows = (int)(hi - lo);
    float mean[V] = {}, square[V] = {}, n = 0.f;
    if (at.left > 0)
        each_chunk<T, V, U, 1>({(const T*)a.x + at.c + (item + lo) * a.x_stride}, {a.x_stride}, rows, at.r0, at.rt, at.left, [&](auto& now, int, auto many) {
            if constexpr (!std::is_same<decltype(many), int>::value) {
                const float f = (float)U / (n + U), nf = n * f;
                float s[V], q[V] = {};
                // in pairs, which are exact for equal values
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    float two[U / 2];
#pragma unroll
                    for (int u = 0; u < U / 2; ++u) two[u] = fmaf((float)now[0].x[2 * u][e], 1.f / U, (float)now[0].x[2 * u + 1][e] * (1.f / U));
#pragma unroll
                    for (int step = 1; step < U / 2; step *= 2)
#pragma unroll
                        for (int u = 0; u + step < U / 2; u += 2 * step) two[u] += two[u + step];
                    s[e] = two[0];
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int e = 0; e < V; ++e) { const float d = (float)now[0].x[u][e] - s[e]; q[e] = fmaf(d, d, q[e]); }
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float d = half_apart(s[e], mean[e]);
                    mean[e] = fmaf(d, 2.f * f, mean[e]);
                    square[e] += fmaf(d * (4.f * nf), d, q[e]);
                }
                n += U;
            } else {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (u >= many) break;
#pragma unroll
                    for (int e = 0; e < V; ++e) merge(n, mean[e], square[e], 1.f, (float)now[0].x[u][e], 0.f);
                    n += 1.f;
                }
            }
        });
    // threads r0 and r0 + half meet; both counts follow from the rows
    auto count = [&](int r0, int step) { return rows > r0 ? (float)((rows - r0 + step - 1) / step) : 0.f; };
#pragma unroll
    for (int e = 0; e < V; ++e) { means[e][threadIdx.x] = mean[e]; squares[e][threadIdx.x] = square[e]; }
    for (int half = at.rt / 2; half; half /= 2) {
        __syncthreads();
        if (at.r0 < half) {
            const float m = count(at.r0 + half, 2 * half);
            const int other = threadIdx.x + half * ct;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                merge(n, mean[e], square[e], m, means[e][other], squares[e][other]);
                means[e][threadIdx.x] = mean[e];
                squares[e][threadIdx.x] = square[e];
            }
            n = count(at.r0, half);
        }
    }
    if (at.r0 == 0)
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (e < at.left) {
                float* const p = a.part + 2 * ((int64_t)(blockIdx.z * a.parts + blockIdx.y) * a.C + at.c + e);
                p[0] = mean[e];
                p[1] = square[e];
            }
}

// the sum over a workgroup of WAVES waves, the same in every thread
template <int WAVES> __device__ __forceinline__ float sum_all(float x, float* room) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d);
    __syncthreads();                                     // the last sum has been read
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = x;
    __syncthreads();
    x = room[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) x += room[w];
    return x;
}

// A group's parts: mean and 1 / spread.  One workgroup a group and item, or several after each other.  The parts' means are averaged first, in two goes,
// and the squares taken about that.
constexpr int MOST_GROUPS = 1 << 20;                     // workgroups: a launch has fewer than 2^32 threads
template <int WAVES, int HELD_PARTS>
__global__ __launch_bounds__(64 * WAVES) void finish_stats_kernel(GroupNormArgs a) {
    __shared__ float room[WAVES];
    const int width = a.C / a.G, all = a.parts * width;
    const float n = (float)a.P * (float)width;
    for (int at = blockIdx.x; at < a.B * a.G; at += gridDim.x) {
        const int g = at % a.G, b = at / a.G;
        const float* const part = a.part + 2 * ((int64_t)b * a.parts * a.C + g * width);
        auto load = [&](int i, float& mean, float& square, float& rows) {
            const int p = (unsigned)i / (unsigned)width;
            const float* const q = part + 2 * ((int64_t)p * a.C + (i - p * width));
            mean = q[0];
            square = q[1];
            rows = (float)min(a.share, a.P - p * a.share);
        };
        // a thread's first parts stay in its registers; any more are read in each go
        float m[HELD_PARTS], q[HELD_PARTS], rows[HELD_PARTS];
#pragma unroll
        for (int j = 0; j < HELD_PARTS; ++j) {
            const int i = threadIdx.x + j * 64 * WAVES;
            m[j] = q[j] = rows[j] = 0.f;
            if (i < all) load(i, m[j], q[j], rows[j]);
        }
        auto each = [&](auto f) {
#pragma unroll
            for (int j = 0; j < HELD_PARTS; ++j) if (rows[j] > 0.f) f(m[j], q[j], rows[j]);
            for (int i = threadIdx.x + HELD_PARTS * 64 * WAVES; i < all; i += 64 * WAVES) {
                float mean, square, rows;
                load(i, mean, square, rows);
                f(mean, square, rows);
            }
        };
        float mean = 0.f, rest = 0.f, square = 0.f;
        each([&](float x, float, float r) { mean = fmaf(x, r / n, mean); });
        mean = finite(sum_all<WAVES>(mean, room));
        each([&](float x, float, float r) { rest = fmaf(half_apart(x, mean), 2.f * (r / n), rest); });
        mean += sum_all<WAVES>(rest, room);
        each([&](float x, float y, float r) { const float d = x - mean; square += fmaf(r * d, d, y); });
        square = sum_all<WAVES>(square, room);
        if (threadIdx.x == 0) {
            const float rho = 1.f / sqrtf(square / n + a.eps);
            a.stats[2 * at] = rho == 0.f ? 0.f : mean;   // squares past the largest value: a difference from the mean may be as well
            a.stats[2 * at + 1] = rho;
        }
    }
}

// mean, 1 / spread, weight and bias of a thread's channels
template <int V> struct Channels { float mean[V], rho[V], w[V], b[V]; };
template <int V>
__device__ __forceinline__ void load_channels(const GroupNormArgs& a, int item, int c, Channels<V>& k) {
    const int width = a.C / a.G;
    int g = c / width, next = (g + 1) * width;            // the group, and where the next begins
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int ch = min(c + e, a.C - 1);
        if (ch >= next) { ++g; next += width; }
        const float* const s = a.stats + 2 * ((int64_t)item * a.G + g);
        k.mean[e] = s[0];
        k.rho[e] = s[1];
        k.w[e] = a.weight ? a.weight[ch] : 1.f;
        k.b[e] = a.bias ? a.bias[ch] : 0.f;
    }
}

template <class T, int V, int ACT>
__global__ __launch_bounds__(THREADS) void apply_kernel(GroupNormArgs a, int ct) {
    constexpr int U = 4;
    const Columns<V> at(a.C, ct);
    if (at.left <= 0) return;
    // the last rows that the statistics were made from are nearest
    const int b = gridDim.z - 1 - blockIdx.z;
    const int64_t lo = (gridDim.y - 1 - blockIdx.y) * a.share, hi = min(a.P, lo + a.share), item = b * a.P;
    Channels<V> k;
    load_channels(a, b, at.c, k);
#pragma unroll
    for (int e = 0; e < V; ++e) k.w[e] *= k.rho[e];
    T* const y = (T*)a.y + at.c + (item + lo) * a.C;
    each_chunk<T, V, U, 1>({(const T*)a.x + at.c + (item + lo) * a.x_stride}, {a.x_stride}, (int)(hi - lo), at.r0, at.rt, at.left, [&](auto& now, int r, auto many) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u >= many) break;
            float v[V];
            now[0].get(u, v);
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = row_act(ACT, fmaf(v[e] - k.mean[e], k.w[e], k.b[e]));
            store_some<T, V>(y + (int64_t)(r + u * at.rt) * a.C, v, at.left, a.past);
        }
    });
}

// ---- gradient.  hat = (x - mean) rho, z = hat w + b, dz = d_y act'(z).
template <int ACT, int V>
__device__ __forceinline__ void slopes(const Channels<V>& k, float (&x)[V], float (&g)[V]) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
        x[e] = (x[e] - k.mean[e]) * k.rho[e];
        if (ACT != CORR_ACT_NONE) g[e] *= row_act_slope(ACT, fmaf(x[e], k.w[e], k.b[e]));
    }
}
// Sums over the workgroup's rows of dz hat and dz, channel by channel.
template <class T, int V, int ACT>
__global__ __launch_bounds__(THREADS) void sums_kernel(GroupNormArgs a, int ct) {
    constexpr int U = 4;
    __shared__ float first[V][THREADS], second[V][THREADS];
    const Columns<V> at(a.C, ct);
    const int64_t lo = blockIdx.y * a.share, hi = min(a.P, lo + a.share), item = blockIdx.z * a.P;
    float hats[V] = {}, ones[V] = {};
    if (at.left > 0) {
        Channels<V> k;
        load_channels(a, blockIdx.z, at.c, k);
        each_chunk<T, V, U, 2>({(const T*)a.x + at.c + (item + lo) * a.x_stride, (const T*)a.d_y + at.c + (item + lo) * a.d_y_stride}, {a.x_stride, a.d_y_stride},
                               (int)(hi - lo), at.r0, at.rt, at.left, [&](auto& now, int, auto many) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (u >= many) break;
                float v[V], g[V];
                now[0].get(u, v);
                now[1].get(u, g);
                slopes<ACT>(k, v, g);
#pragma unroll
                for (int e = 0; e < V; ++e) { hats[e] = fmaf(g[e], v[e], hats[e]); ones[e] += g[e]; }
            }
        });
    }
#pragma unroll
    for (int e = 0; e < V; ++e) { first[e][threadIdx.x] = hats[e]; second[e][threadIdx.x] = ones[e]; }
    for (int half = at.rt / 2; half; half /= 2) {
        __syncthreads();
        if (at.r0 < half)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                first[e][threadIdx.x] = hats[e] += first[e][threadIdx.x + half * ct];
                second[e][threadIdx.x] = ones[e] += second[e][threadIdx.x + half * ct];
            }
    }
    if (at.r0 == 0 && at.left > 0) {
        float* const p = a.part + (int64_t)(blockIdx.z * a.parts + blockIdx.y) * 2 * a.C + at.c;
        store_some<float, V>(p, hats, at.left);
        store_some<float, V>(p + a.C, ones, at.left);
    }
}
// The parts of an item added in order: 16 channels a workgroup, 64 shares of the parts; `items` of them, whose sum is the vectors' gradient if they
// are all.  The shares are added in pairs: one after the other they made most of the sums' error (4 x 7285 x 96 fp32, 2-norm:
// d_weight 1.8e-7 -> 1.4e-7, d_bias 2.0e-7 -> 1.2e-7).
__device__ __forceinline__ float sum8(const float* p) {      // of a column of 16
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = p[16 * i];
    return ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
}
__global__ __launch_bounds__(JOIN_THREADS) void join_kernel(GroupNormArgs a, int items) {
    constexpr int SHARES = JOIN_THREADS / 16;
    __shared__ float sums[SHARES][16];
    const int col = threadIdx.x & 15, share = threadIdx.x >> 4, c = blockIdx.x * 16 + col;
    float all = 0.f;
    for (int b = blockIdx.z * items; b < (blockIdx.z + 1) * items; ++b) {
        const float* const p = a.part + ((int64_t)b * a.parts * 2 + blockIdx.y) * a.C + c;
        float sum = 0.f;
        if (c < a.C)
#pragma unroll 4
            for (int i = share; i < a.parts; i += SHARES) sum += p[(int64_t)i * 2 * a.C];
        __syncthreads();                                 // the last item's sums have been read
        sums[share][col] = sum;
        __syncthreads();
        const bool last = share == 0 && c < a.C;
        if (share < 8) sum = sum8(&sums[share * 8][col]);
        __syncthreads();
        if (share < 8) sums[share][col] = sum;
        __syncthreads();
        if (!last) continue;
        sum = sum8(&sums[0][col]);
        a.sums[((int64_t)b * 2 + blockIdx.y) * a.C + c] = sum;
        all += sum;
    }
    float* const out = blockIdx.y ? a.d_bias : a.d_weight;
    if (items == a.B && out && share == 0 && c < a.C) out[c] = all;
}
// d_x = rho (w dz - S1 / n - hat S2 / n), S1 and S2 the group's sums of w dz and w dz hat, which every workgroup adds up for its columns.
template <class T, int V, int ACT>
__global__ __launch_bounds__(THREADS) void dx_kernel(GroupNormArgs a, int ct) {
    constexpr int U = 4;
    __shared__ float s1[THREADS * V], s2[THREADS * V];       // of the channels from the first column's group on: groups of this workgroup's columns
    const Columns<V> at(a.C, ct);
    const int width = a.C / a.G, c0 = blockIdx.x * ct * V, c1 = min(a.C, c0 + ct * V), g0 = c0 / width, groups = (c1 - 1) / width - g0 + 1;
    const int b = gridDim.z - 1 - blockIdx.z;                // the last rows first, as above
    const float* const sums = a.sums + (int64_t)b * 2 * a.C;
    const float by = 1.f / ((float)a.P * (float)width);
    // 2^k neighbouring threads a group, as many as there are
    int team = 64;
    while (team > 1 && (team > width || groups * team > THREADS)) team /= 2;
    for (int g = threadIdx.x / team; g < (groups + THREADS / team - 1) / (THREADS / team) * (THREADS / team); g += THREADS / team) {
        float x = 0.f, y = 0.f;
        if (g < groups)
            for (int c = (g0 + g) * width + threadIdx.x % team; c < (g0 + g + 1) * width; c += team) {
                const float w = a.weight ? a.weight[c] : 1.f;
                x = fmaf(w, sums[a.C + c], x);
                y = fmaf(w, sums[c], y);
            }
        for (int s = 1; s < team; s *= 2) { x += __shfl_xor(x, s); y += __shfl_xor(y, s); }
        if (g < groups && threadIdx.x % team == 0) { s1[g] = x * by; s2[g] = y * by; }
    }
    __syncthreads();
    if (at.left <= 0) return;
    const int64_t lo = (gridDim.y - 1 - blockIdx.y) * a.share, hi = min(a.P, lo + a.share), item = b * a.P;
    Channels<V> k;
    load_channels(a, b, at.c, k);
    float m1[V], m2[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int g = min(at.c + e, a.C - 1) / width - g0;
        m1[e] = s1[g];
        m2[e] = s2[g];
    }
    T* const out = (T*)a.d_x + at.c + (item + lo) * a.C;
    each_chunk<T, V, U, 2>({(const T*)a.x + at.c + (item + lo) * a.x_stride, (const T*)a.d_y + at.c + (item + lo) * a.d_y_stride}, {a.x_stride, a.d_y_stride},
                           (int)(hi - lo), at.r0, at.rt, at.left, [&](auto& now, int r, auto many) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u >= many) break;
            float v[V], g[V];
            now[0].get(u, v);
            now[1].get(u, g);
            slopes<ACT>(k, v, g);
#pragma unroll
            for (int e = 0; e < V; ++e) g[e] = k.rho[e] * (fmaf(k.w[e], g[e], -m1[e]) - v[e] * m2[e]);
            store_some<T, V>(out + (int64_t)(r + u * at.rt) * a.C, g, at.left, a.past);
        }
    });
}

// ---- small maps: a workgroup has a group of an item in its registers and reads it once; one launch where the kernels above are three and four.  A
// thread has V neighbouring channels (`across` threads have the group's) of up to PIECES pixels.
constexpr int HELD_THREADS = 1024, PIECES = 8;
struct Held {
    int across, q, pixel, step, c, left;                 // c: the thread's first channel; left: of its group from there on
    __device__ __forceinline__ Held(const GroupNormArgs& a, int V, int across_) : across(across_) {
        const int width = a.C / a.G;
        q = threadIdx.x % across;
        pixel = threadIdx.x / across;
        step = HELD_THREADS / across;
        c = blockIdx.x % a.G * width + q * V;
        left = width - q * V;
    }
};
template <class T, int V, int ACT>
__global__ __launch_bounds__(HELD_THREADS) void held_kernel(GroupNormArgs a, int across) {
    __shared__ float room[HELD_THREADS / 64];
    const Held at(a, V, across);
    const int b = blockIdx.x / a.G;
    const T* const x = (const T*)a.x + (b * a.P + at.pixel) * a.x_stride + at.c;
    Chunk<T, V, PIECES> k;
    const float by = 1.f / ((float)a.P * (float)(a.C / a.G));
#pragma unroll
    for (int j = 0; j < PIECES; ++j) if (at.pixel + j * at.step < a.P) k.load_row(j, x + j * at.step * a.x_stride, at.left);
    float w[V], bias[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        w[e] = a.weight && e < at.left ? a.weight[at.c + e] : 1.f;
        bias[e] = a.bias && e < at.left ? a.bias[at.c + e] : 0.f;
    }
    float mean = 0.f, rest = 0.f, square = 0.f;
#pragma unroll
    for (int j = 0; j < PIECES; ++j)
        if (at.pixel + j * at.step < a.P)
#pragma unroll
            for (int e = 0; e < V; ++e) if (e < at.left) mean = fmaf((float)k.x[j][e], by, mean);
    mean = finite(sum_all<HELD_THREADS / 64>(mean, room));
#pragma unroll
    for (int j = 0; j < PIECES; ++j)
        if (at.pixel + j * at.step < a.P)
#pragma unroll
            for (int e = 0; e < V; ++e) if (e < at.left) rest = fmaf(half_apart((float)k.x[j][e], mean), 2.f * by, rest);
    mean += sum_all<HELD_THREADS / 64>(rest, room);
#pragma unroll
    for (int j = 0; j < PIECES; ++j)
        if (at.pixel + j * at.step < a.P)
#pragma unroll
            for (int e = 0; e < V; ++e) if (e < at.left) { const float d = (float)k.x[j][e] - mean; square = fmaf(d, d, square); }
    const float rho = 1.f / sqrtf(sum_all<HELD_THREADS / 64>(square, room) * by + a.eps);
    if (rho == 0.f) mean = 0.f;                          // as above
    if (a.stats && threadIdx.x == 0) { a.stats[2 * blockIdx.x] = mean; a.stats[2 * blockIdx.x + 1] = rho; }
    T* const y = (T*)a.y + (b * a.P + at.pixel) * a.C + at.c;
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
        if (at.pixel + j * at.step >= a.P) break;
        float v[V];
        k.get(j, v);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = row_act(ACT, fmaf(v[e] - mean, rho * w[e], bias[e]));
        store_some<T, V>(y + (int64_t)j * at.step * a.C, v, at.left);
    }
}
template <class T, int V, int ACT>
__global__ __launch_bounds__(HELD_THREADS) void held_backward_kernel(GroupNormArgs a, int across) {
    __shared__ float sums[2][V][HELD_THREADS / 64][8];   // of a wave's threads that have the same channels
    __shared__ float total[2][8 * V];
    const Held at(a, V, across);
    const int b = blockIdx.x / a.G, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, width = a.C / a.G;
    const float by = 1.f / ((float)a.P * (float)width);
    const T* const x = (const T*)a.x + (b * a.P + at.pixel) * a.x_stride + at.c;
    const T* const d = (const T*)a.d_y + (b * a.P + at.pixel) * a.d_y_stride + at.c;
    Chunk<T, V, PIECES> kx, kd;
#pragma unroll
    for (int j = 0; j < PIECES; ++j)
        if (at.pixel + j * at.step < a.P) {
            kx.load_row(j, x + j * at.step * a.x_stride, at.left);
            kd.load_row(j, d + j * at.step * a.d_y_stride, at.left);
        }
    Channels<V> k;
    const float mean = a.stats[2 * blockIdx.x], rho = a.stats[2 * blockIdx.x + 1];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        k.mean[e] = mean;
        k.rho[e] = rho;
        k.w[e] = a.weight && e < at.left ? a.weight[at.c + e] : 1.f;
        k.b[e] = a.bias && e < at.left ? a.bias[at.c + e] : 0.f;
    }
    float hats[V] = {}, ones[V] = {};
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
        if (at.pixel + j * at.step >= a.P) break;
        float v[V], g[V];
        kx.get(j, v);
        kd.get(j, g);
        slopes<ACT>(k, v, g);
#pragma unroll
        for (int e = 0; e < V; ++e) { hats[e] = fmaf(g[e], v[e], hats[e]); ones[e] += g[e]; }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
        for (int s = across; s < 64; s *= 2) { hats[e] += __shfl_xor(hats[e], s); ones[e] += __shfl_xor(ones[e], s); }
        if (lane < across) { sums[0][e][wave][lane] = hats[e]; sums[1][e][wave][lane] = ones[e]; }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * across * V; i += HELD_THREADS) {
        const int which = i / (across * V), c = i % (across * V);
        float sum = 0.f;
        if (c < width) {
            for (int w = 0; w < HELD_THREADS / 64; ++w) sum += sums[which][c % V][w][c / V];
            const int ch = blockIdx.x % a.G * width + c;
            a.sums[((int64_t)b * 2 + which) * a.C + ch] = sum;
            float* const out = which ? a.d_bias : a.d_weight;
            if (a.B == 1 && out) out[ch] = sum;
            if (a.weight) sum *= a.weight[ch];
        }
        total[which][c] = sum;
    }
    __syncthreads();
    if (!a.d_x) return;
    float s1 = 0.f, s2 = 0.f;
    for (int c = 0; c < width; ++c) { s2 += total[0][c]; s1 += total[1][c]; }
    s1 *= by;
    s2 *= by;
    T* const out = (T*)a.d_x + (b * a.P + at.pixel) * a.C + at.c;
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
        if (at.pixel + j * at.step >= a.P) break;
        float v[V], g[V];
        kx.get(j, v);
        kd.get(j, g);
        slopes<ACT>(k, v, g);
#pragma unroll
        for (int e = 0; e < V; ++e) g[e] = rho * (fmaf(k.w[e], g[e], -s1) - v[e] * s2);
        store_some<T, V>(out + (int64_t)j * at.step * a.C, g, at.left);
    }
}

// f(act) with the activation as a constant: chosen inside the kernels' loops it costs them their order of loads
template <class F> void with_act(int act, F f) {
    switch (act) {
        case CORR_ACT_RELU: f(std::integral_constant<int, CORR_ACT_RELU>{}); break;
        case CORR_ACT_GELU: f(std::integral_constant<int, CORR_ACT_GELU>{}); break;
        case CORR_ACT_GELU_TANH: f(std::integral_constant<int, CORR_ACT_GELU_TANH>{}); break;
        case CORR_ACT_SILU: f(std::integral_constant<int, CORR_ACT_SILU>{}); break;
        case CORR_ACT_SIGMOID: f(std::integral_constant<int, CORR_ACT_SIGMOID>{}); break;
        default: f(std::integral_constant<int, CORR_ACT_NONE>{});
    }
}
template <class T, int V>
hipError_t forward(const GroupNormArgs& a, hipStream_t s) {
    if (a.held) {
        with_act(a.act, [&](auto act) { hipLaunchKernelGGL((held_kernel<T, V, decltype(act)::value>), dim3(a.B * a.G), dim3(HELD_THREADS), 0, s, a, a.held); });
        return hipGetLastError();
    }
    const int ct = threads_across<V>(a.C);
    const dim3 grid((unsigned)cdiv(a.C, ct * V), a.parts, a.B);
    hipLaunchKernelGGL((stats_kernel<T, V>), grid, dim3(THREADS), 0, s, a, ct);
    const dim3 groups((unsigned)std::min(a.B * a.G, MOST_GROUPS));
    // few parts: one wave (64 x 64 x 512 in 512 groups bf16, the whole call: 146 -> 26 us)
    const int all = a.parts * (a.C / a.G);
    if (all <= 64) hipLaunchKernelGGL((finish_stats_kernel<1, 1>), groups, dim3(64), 0, s, a);
    else if (all <= JOIN_THREADS) hipLaunchKernelGGL((finish_stats_kernel<JOIN_THREADS / 64, 1>), groups, dim3(JOIN_THREADS), 0, s, a);
    else hipLaunchKernelGGL((finish_stats_kernel<JOIN_THREADS / 64, 8>), groups, dim3(JOIN_THREADS), 0, s, a);
    const hipError_t e = hipGetLastError();              // without statistics there is no result
    if (e != hipSuccess) return e;
    with_act(a.act, [&](auto act) { hipLaunchKernelGGL((apply_kernel<T, V, decltype(act)::value>), grid, dim3(THREADS), 0, s, a, ct); });
    return hipGetLastError();
}
// Few items' sums follow each other in one launch.
bool joined_at_once(const GroupNormArgs& a) { return a.B == 1 || (a.B <= 4 && !a.held); }
template <class T, int V>
void backward(const GroupNormArgs& a, hipStream_t s) {
    if (a.held) {
        with_act(a.act, [&](auto act) { hipLaunchKernelGGL((held_backward_kernel<T, V, decltype(act)::value>), dim3(a.B * a.G), dim3(HELD_THREADS), 0, s, a, a.held); });
        return;
    }
    const int ct = threads_across<V>(a.C);
    const dim3 grid((unsigned)cdiv(a.C, ct * V), a.parts, a.B);
    with_act(a.act, [&](auto act) { hipLaunchKernelGGL((sums_kernel<T, V, decltype(act)::value>), grid, dim3(THREADS), 0, s, a, ct); });
    const int items = joined_at_once(a) ? a.B : 1;
    hipLaunchKernelGGL(join_kernel, dim3((a.C + 15) / 16, 2, a.B / items), dim3(JOIN_THREADS), 0, s, a, items);
    if (a.d_x) with_act(a.act, [&](auto act) { hipLaunchKernelGGL((dx_kernel<T, V, decltype(act)::value>), grid, dim3(THREADS), 0, s, a, ct); });
}

}  // namespace

// Shares for four workgroups on every compute unit, of eight rows a thread at least; none where a group stays in a workgroup's registers.
void group_norm_plan(GroupNormArgs& a, bool gradient) {
    const int V = a.type == CORR_TYPE_F32 ? 4 : 8, ct = V == 4 ? threads_across<4>(a.C) : threads_across<8>(a.C), rt = THREADS / ct;
    const int64_t across = cdiv(a.C, ct * V) * a.B, want = cdiv(1024, across), most = cdiv(a.P, 8 * rt);
    int64_t parts = want < most ? want : most;
    if (parts < 1) parts = 1;
    a.share = cdiv(a.P, parts);
    a.parts = (int)cdiv(a.P, a.share);
    // a result larger than a quarter of the memory-side cache goes past the caches
    a.past = (int64_t)a.B * a.P * a.C * corr_elem_bytes(a.type) >= (64 << 20);
    // In registers: little data, whose rows' pieces of 16 bytes cost whole lines (2 x 2852 x 64 in 8 groups fp16: 16.5 -> 11 us, gradient 23 -> 19, the host's part
    // of that about 9; 2 x 2852 x 256 in 32 bf16: 17 -> 13, gradient 24.2 and 23.6; but 16 x 1000 x 256: 18 -> 20 and 24 -> 40, 64 x 2048 x 256: 51 -> 131).
    const int64_t across_group = a.C / a.G / V, pieces = a.P * across_group;
    const bool whole = a.C / a.G % V == 0 && across_group <= 8 && (across_group & (across_group - 1)) == 0;
    a.held = whole && pieces <= HELD_THREADS * PIECES && pieces * a.B * a.G <= (gradient ? 1 << 17 : 1 << 18) ? (int)across_group : 0;
}
hipError_t launch_group_norm(const GroupNormArgs& a, hipStream_t s) {
    return a.type == CORR_TYPE_F32 ? forward<float, 4>(a, s) : a.type == CORR_TYPE_BF16 ? forward<__bf16, 8>(a, s) : forward<_Float16, 8>(a, s);
}
hipError_t launch_group_norm_backward(const GroupNormArgs& a, hipStream_t s) {
    if (a.type == CORR_TYPE_F32) backward<float, 4>(a, s);
    else if (a.type == CORR_TYPE_BF16) backward<__bf16, 8>(a, s);
    else backward<_Float16, 8>(a, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || joined_at_once(a) || (!a.d_weight && !a.d_bias)) return e;
    const ColumnSums o = {{a.d_weight, a.d_bias, nullptr, nullptr, nullptr}};
    return launch_column_sums(a.sums, a.B, 2, a.C, o, s);
}
