// Products of rows with weights: y = act(x w^T + bias) + residual, and the two products of its gradient.
#include <type_traits>
#include "matrix.h"
#include "rows_internal.h"

namespace {

enum Tile { TILE_FEW = 0, TILE_64, TILE_128, TILE_256, TILE_ROWS };
inline int cdiv(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// The part of an operand that one workgroup reads: `at` moves with the k loop, `left` bytes of the matrix lie from there on
// (offsets inside one step stay below 2^31: the callers limit row strides).
struct Window {
    const unsigned char* at;
    int64_t left, step;
    __device__ __forceinline__ unsigned size() const {     // by halves: whole 64-bit comparisons would go to the vector unit
        const int hi = (int)(left >> 32);
        const unsigned lo = (unsigned)left;
        return hi < 0 ? 0 : hi > 0 || lo > 0x7ffffff0u ? 0x7ffffff0u : lo;
    }
    __device__ __forceinline__ i32x4 rsrc() const {
        const uint64_t p = (uint64_t)at;
        return i32x4{__builtin_amdgcn_readfirstlane((int)p), __builtin_amdgcn_readfirstlane((int)(p >> 32) & 0xffff),
                     __builtin_amdgcn_readfirstlane((int)size()), 0x00020000};
    }
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer() const {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(at), 0, __builtin_amdgcn_readfirstlane((int)size()), 0x00020000);
    }
    __device__ __forceinline__ void next() { at += step; left -= step; }
};
// rows r0 .. of a [rows][ld] matrix with k contiguous, from k0 on; or of a [K][ld] matrix with the rows contiguous
template <bool ROWS, int ES, int BK>
__device__ __forceinline__ Window window(const void* p, int64_t ld, int rows, int K, int r0, int k0) {
    Window w;
    w.at = (const unsigned char*)p + ((ROWS ? (int64_t)k0 * ld + r0 : (int64_t)r0 * ld + k0)) * ES;
    w.left = ROWS ? ((int64_t)(K - 1 - k0) * ld + (rows - r0)) * ES : ((int64_t)(rows - 1 - r0) * ld + (K - k0)) * ES;
    w.left = (w.left + 3) & ~(int64_t)3;                 // whole words: odd lengths come in rows that are padded
    w.step = (ROWS ? (int64_t)BK * ld : BK) * ES;
    return w;
}

// Which tile and split workgroup w takes.  Workgroup w runs on XCD w % 8: each XCD gets a run of consecutive pieces of work; a split's tiles
// follow each other, and tiles are numbered in panels of eight columns, so that the 32 pieces an XCD works on at a time share
// operands in its L2.
__device__ __forceinline__ void tile_of(int w, int tm, int tn, int splits, int& m, int& n, int& split) {
    const int T = tm * tn, all = T * splits, q = all >> 3, r = all & 7, x = w & 7;
    int t = x * q + min(x, r) + (w >> 3);
    split = t / T;
    t -= split * T;
    const int per = 8 * tm, panel = t / per, in = t - panel * per, wide = min(8, tn - 8 * panel);
    m = in / wide;
    n = 8 * panel + in - m * wide;
}

// ---- epilogue
// V elements of row m from column n on
template <class T, int V>
__device__ __forceinline__ void finish(const ProductArgs& g, float (&v)[V], const float (&bias)[V], int m, int n) {
    const int left = g.N - n;
    if (m >= g.M || left <= 0) return;
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] += bias[e];
    if (g.pre) store_some<T, V>((T*)g.pre + (int64_t)m * g.N + n, v, left, g.past);
    row_act_all(g.act, v);
    if (g.res) {
        float r[V];
        load_some<T, V>((const T*)g.res + (int64_t)m * g.ld_res + n, r, left);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] += r[e];
    }
    store_some<T, V>((T*)g.y + (int64_t)m * g.ldy + n, v, left, g.past);
}
template <int V>
__device__ __forceinline__ void load_bias(const ProductArgs& g, float (&bias)[V], int n) {
#pragma unroll
    for (int e = 0; e < V; ++e) bias[e] = g.bias && n + e < g.N ? g.bias[n + e] : 0.f;
}
// Gated: V elements of both halves.  g.N columns of y; bias and pre have 2 N, the gate's first.
template <class T, int V>
__device__ __forceinline__ void store_gated(const ProductArgs& g, float (&gate)[V], const float (&up)[V], int m, int n) {
    const int left = g.N - n;
    if (m >= g.M || left <= 0) return;
    if (g.pre) {
        T* const z = (T*)g.pre + (int64_t)m * 2 * g.N + n;
        store_some<T, V>(z, gate, left, g.past);
        store_some<T, V>(z + g.N, up, left, g.past);
    }
    row_act_all(g.act, gate);
#pragma unroll
    for (int e = 0; e < V; ++e) gate[e] *= up[e];
    store_some<T, V>((T*)g.y + (int64_t)m * g.ldy + n, gate, left, g.past);
}
template <class T, int V>
__device__ __forceinline__ void finish_gated(const ProductArgs& g, float (&gate)[V], float (&up)[V], const float (&bias)[2][V], int m, int n) {
#pragma unroll
    for (int e = 0; e < V; ++e) { gate[e] += bias[0][e]; up[e] += bias[1][e]; }
    store_gated<T, V>(g, gate, up, m, n);
}
template <int V>
__device__ __forceinline__ void load_gated_bias(const ProductArgs& g, float (&bias)[2][V], int n) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
        bias[0][e] = g.bias && n + e < g.N ? g.bias[n + e] : 0.f;
        bias[1][e] = g.bias && n + e < g.N ? g.bias[g.N + n + e] : 0.f;
    }
}
// A wave's FN x FM blocks of 16 x 16 (rows of the instruction's first operand are n: a lane has four consecutive n of one m), 16 rows
// of C at a time by way of LDS, so that a lane gets 16 bytes of a row and eight (16) lanes a whole 128-byte line or more.  Straight from
// the registers, in pieces of 8 bytes and one activation after the other, the widening product at 1080p took 95 us.
template <int FN> constexpr int box_floats() { return 16 * (16 * FN + 4); }
template <class T, int FM, int FN>
__device__ __forceinline__ void finish_wave(const ProductArgs& g, f32x4 (&acc)[FN][FM], float* box, int m0, int n0, int lane, int split, int splits) {
    constexpr int LD = 16 * FN + 4;
    const int lr = lane & 15, lg = lane >> 4;
    auto by_rows = [&](auto width, auto f) {
        constexpr int V = decltype(width)::value, LANES = 16 * FN / V, ROWS = 64 / LANES;
        const int c = lane % LANES * V, r0 = lane / LANES;
#pragma unroll
        for (int j = 0; j < FM; ++j) {
#pragma unroll
            for (int i = 0; i < FN; ++i) *reinterpret_cast<f32x4*>(box + lr * LD + 16 * i + 4 * lg) = acc[i][j];
            asm volatile("" ::: "memory");               // one wave: its LDS accesses are done in order
#pragma unroll
            for (int r = r0; r < 16; r += ROWS) {
                float v[V];
#pragma unroll
                for (int e = 0; e < V; e += 4) {
                    const f32x4 x = *reinterpret_cast<const f32x4*>(box + r * LD + c + e);
                    v[e] = x[0]; v[e + 1] = x[1]; v[e + 2] = x[2]; v[e + 3] = x[3];
                }
                f(v, m0 + 16 * j + r, n0 + c);
            }
            asm volatile("" ::: "memory");
        }
    };
    if (splits > 1) {
        by_rows(std::integral_constant<int, 4>{}, [&](float (&v)[4], int m, int n) {
            if (m < g.M && n < g.N) store_some<float, 4>(g.part + ((int64_t)split * g.M + m) * g.N + n, v, g.N - n);
        });
    } else {
        constexpr int V = 16 / sizeof(T);
        float bias[V];
        load_bias(g, bias, n0 + lane % (16 * FN / V) * V);
        by_rows(std::integral_constant<int, V>{}, [&](float (&v)[V], int m, int n) { finish<T, V>(g, v, bias, m, n); });
    }
}

// Gated: even blocks of columns are the gate's, odd ones the other half's of the same columns of y, from column n0 on.
template <class T, int FM, int FN>
__device__ __forceinline__ void finish_gated_wave(const ProductArgs& g, f32x4 (&acc)[FN][FM], float* box, int m0, int n0, int lane, int split, int splits) {
    constexpr int LD = 16 * FN + 4;
    const int lr = lane & 15, lg = lane >> 4;
    auto by_rows = [&](auto width, auto f) {
        constexpr int V = decltype(width)::value, LANES = 8 * FN / V, ROWS = 64 / LANES;
        const int c = lane % LANES * V, r0 = lane / LANES, at = c / 16 * 32 + c % 16;
#pragma unroll
        for (int j = 0; j < FM; ++j) {
#pragma unroll
            for (int i = 0; i < FN; ++i) *reinterpret_cast<f32x4*>(box + lr * LD + 16 * i + 4 * lg) = acc[i][j];
            asm volatile("" ::: "memory");               // one wave: its LDS accesses are done in order
#pragma unroll
            for (int r = r0; r < 16; r += ROWS) {
                float v[2][V];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < V; e += 4) {
                        const f32x4 x = *reinterpret_cast<const f32x4*>(box + r * LD + at + 16 * h + e);
                        v[h][e] = x[0]; v[h][e + 1] = x[1]; v[h][e + 2] = x[2]; v[h][e + 3] = x[3];
                    }
                f(v, m0 + 16 * j + r, n0 + c);
            }
            asm volatile("" ::: "memory");
        }
    };
    if (splits > 1) {
        by_rows(std::integral_constant<int, 4>{}, [&](float (&v)[2][4], int m, int n) {
            if (m >= g.M || n >= g.N) return;
            float* const p = g.part + ((int64_t)split * g.M + m) * 2 * g.N + n;
            store_some<float, 4>(p, v[0], g.N - n);
            store_some<float, 4>(p + g.N, v[1], g.N - n);
        });
    } else {
        constexpr int V = 16 / sizeof(T);
        float bias[2][V];
        load_gated_bias(g, bias, n0 + lane % (8 * FN / V) * V);
        by_rows(std::integral_constant<int, V>{}, [&](float (&v)[2][V], int m, int n) { finish_gated<T, V>(g, v[0], v[1], bias, m, n); });
    }
}

// Gated: row r of a tile of weights is row in_half(r) of the gate's weights or (second_half(r)) of the other half's, in turns of 16, so that a
// lane's blocks 2 i and 2 i + 1 belong to the same columns of y.
__device__ __forceinline__ int in_half(int r) { return (r >> 5) * 16 + (r & 15); }
__device__ __forceinline__ int second_half(int r) { return r >> 4 & 1; }

// ------------------------------------------------------------------------------------------------ 16-bit operands
// A workgroup makes BM x BN elements in steps of BK k.  Tiles lie in LDS as they are stored, in two halves that take turns: while
// one is multiplied, the next step's 16-byte pieces land in the other.
//   k contiguous:    rows of 2 BK bytes, piece p of row r at p ^ (r & 7) (BK = 32: p ^ (r / 2 & 3))
//   rows contiguous: BK k-rows of 2 R bytes, 32-byte block c of row k at c ^ turn(k); read by the transposing LDS load
// so that neither the rows of a fragment nor the k of a transposed one meet in a bank (LDS conflict cycles: 1 in 900).
// 8192^3 bf16 with residual: 0.89 to 1.0 ms, 1.1 to 1.24 PFLOP/s, bound by the matrix cores under the card's power limit.  Short sums are
// bound by bytes and by the turns of a tile (load, multiply, store): 32400 x 256 -> 1024, gelu, preact: 50 us, 149 MB.  A third stage in LDS and
// orders of k that differ from tile to tile made no difference.
template <int R> __device__ __forceinline__ int turn(int k) {
    return R >= 128 ? (k & 3) | ((k >> 3) & 1) << 2 : (k & 3) ^ ((k >> 3) & 1);
}
// piece p of row r of BK elements: where it lies
template <int BK> __device__ __forceinline__ int place(int r, int p) { return BK == 64 ? p ^ (r & 7) : p ^ (r >> 1 & 3); }
template <bool ROWS, int R, int WAVES, int BK, bool GATED = false>
struct Loader16 {
    static constexpr int PIECES = R * BK * 2 / (1024 * WAVES);
    unsigned voff[PIECES];
    __device__ __forceinline__ void plan(int wave, int lane, int64_t ld) {
#pragma unroll
        for (int q = 0; q < PIECES; ++q) {
            const int p = (q * WAVES + wave) * 1024 + lane * 16;
            if constexpr (ROWS) {
                const int k = p / (2 * R), piece = (p % (2 * R)) >> 4;
                voff[q] = (unsigned)(k * ld * 2) + ((((piece >> 1) ^ turn<R>(k)) << 1) | (piece & 1)) * 16;
            } else {
                const int row = p / (2 * BK), piece = (p >> 4) % (BK / 8);
                voff[q] = (unsigned)((GATED ? in_half(row) : row) * ld * 2) + place<BK>(row, piece) * 16;
            }
        }
    }
    __device__ __forceinline__ void issue(const Window& w, unsigned lds, int wave) const {
        const i32x4 rsrc = w.rsrc();
#pragma unroll
        for (int q = 0; q < PIECES; ++q) dma16(rsrc, lds + (q * WAVES + wave) * 1024, voff[q]);
    }
    // a load's 1024 bytes are rows of one half
    __device__ __forceinline__ void issue(const Window& gate, const Window& up, unsigned lds, int wave) const {
        const i32x4 one = gate.rsrc(), two = up.rsrc();
#pragma unroll
        for (int q = 0; q < PIECES; ++q)
            dma16(second_half((q * WAVES + wave) * (512 / BK)) ? two : one, lds + (q * WAVES + wave) * 1024, voff[q]);
    }
};
// F fragments of 16 rows from row `base` on: lane (lr, lg) holds k = 8 lg .. + 7 of a row of 32 k.
template <class T, bool ROWS, int R, int F, int BK>
struct Reader16 {
    unsigned off[ROWS ? F : 2];
    __device__ __forceinline__ void plan(int base, int lr, int lg) {
        if constexpr (ROWS) {
#pragma unroll
            for (int i = 0; i < F; ++i) {
                const int k = 8 * lg + (lr >> 2);
                off[i] = k * (2 * R) + (((base >> 4) + i) ^ turn<R>(k)) * 32 + (lr & 3) * 8;
            }
        } else {
            off[0] = (base + lr) * (2 * BK) + place<BK>(lr, lg) * 16;
            off[1] = off[0] ^ 64;
        }
    }
    __device__ __forceinline__ typename Frag<T>::type get(lds_byte* tile, int i, int ks) const {
        if constexpr (ROWS) {
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(tile + off[i] + ks * 32 * 2 * R));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(tile + off[i] + (ks * 32 + 4) * 2 * R));
            return __builtin_bit_cast(typename Frag<T>::type, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            return *(__attribute__((address_space(3))) typename Frag<T>::type*)(tile + off[ks] + i * 32 * BK);
        }
    }
};
// Elements from k = left on are taken out: what lies behind a row's end belongs to the next row.
template <class V>
__device__ __forceinline__ V keep_first(V v, int left) {
    u32x4 u = __builtin_bit_cast(u32x4, v);
#pragma unroll
    for (int d = 0; d < 4; ++d) u[d] &= left >= 2 * d + 2 ? 0xffffffffu : left == 2 * d + 1 ? 0xffffu : 0u;
    return __builtin_bit_cast(V, u);
}

// TWO: the first operand is in two parts (rows_internal.h), multiplied one after the other, the low one first: twice the matrix work and twice the
// loads (fp16, and bf16 gradients of few gated elements; fp16 gradients with silu, and with relu: 14570 x 243 -> 126: 51 and 41 us; 32400 x 256 -> 1024: 153 and 104; 4096^3: 503 and
// 265).  A sum of the low part's products that is not finite says that an element of the second operand is not, or (bf16; fp16's values
// cannot overflow it) that the high part's sum is not either: then the high part alone gives what the whole would.
// GATED: the second operand's rows come in turns from its two halves of g.N (BN / 2 columns of y a tile), so that a lane's sums have both factors of
// the same columns and the sums need no memory: 14400 x 320 -> 2 x 1280 bf16 with silu and preact 51 us (120 MB), 14570 x 256 -> 2 x 682 fp32
// with gelu 65 us (157 TFLOP/s), bound as the products without a gate.
template <class T, bool AR, bool BR, int BM, int BN, int WM, int WN, int BK, bool TWO, bool GATED = false>
__global__ __launch_bounds__(64 * WM * WN, BK == 32 ? 4 : 2) void product16_kernel(ProductArgs g, int tm, int tn, int splits, int steps_per) {
    constexpr int WAVES = WM * WN, TM = BM / WM, TN = BN / WN, FM = TM / 16, FN = TN / 16;
    constexpr int A_BYTES = BM * BK * 2, HALF = (BM + BN) * BK * 2;
    __shared__ __align__(1024) unsigned char smem[2 * HALF];
    lds_byte* const lds = (lds_byte*)smem;
    const unsigned lds_at = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)lds);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lr = lane & 15, lg = lane >> 4;
    int mt, nt, split;
    tile_of(blockIdx.x, tm, tn, splits, mt, nt, split);
    const int m0 = mt * BM, n0 = nt * (GATED ? BN / 2 : BN);
    const int k0 = split * steps_per * 64, k_left = min(g.K - k0, steps_per * 64);
    const int whole = k_left / BK, tail = k_left % BK, steps = whole + (tail != 0);
    Window wa = window<AR, 2, BK>(TWO ? g.a_lo : g.a, g.lda, g.M, g.K, m0, k0), wb = window<BR, 2, BK>(g.b, g.ldb, g.N, g.K, n0, k0);
    Window wu = wb;
    if constexpr (GATED) wu.at += (int64_t)g.N * g.ldb * 2;
    Loader16<AR, BM, WAVES, BK> la;
    Loader16<BR, BN, WAVES, BK, GATED> lb;
    la.plan(wave, lane, g.lda);
    lb.plan(wave, lane, g.ldb);
    const int wm = (wave % WM) * TM, wn = (wave / WM) * TN;
    Reader16<T, AR, BM, FM, BK> ra;
    Reader16<T, BR, BN, FN, BK> rb;
    ra.plan(wm, lr, lg);
    rb.plan(wn, lr, lg);
    f32x4 acc[FN][FM] = {};
    auto ask = [&](int half) {
        la.issue(wa, lds_at + half * HALF, wave);
        if constexpr (GATED) { lb.issue(wb, wu, lds_at + half * HALF + A_BYTES, wave); wu.next(); }
        else lb.issue(wb, lds_at + half * HALF + A_BYTES, wave);
        wa.next(); wb.next();
    };
    // A wave past the result's borders only helps to load (129600 x 256 -> 324: 52 -> 49 us).  Loads stay ahead of a step's products where k
    // is contiguous (129600 x 320 -> 256: 43 -> 35 us; 8192^3 with residual: 915 and 922); where the rows are, mixed is better (129600 x 324 x 256: 40 and 42).
    const bool busy = AR || (n0 + (GATED ? wn / 2 : wn) < g.N && m0 + wm < g.M);
    auto multiply = [&](int half, auto last) {
        if constexpr (!AR) __builtin_amdgcn_sched_barrier(0);
        if (!busy) return;
        lds_byte* const ta = lds + half * HALF;
        lds_byte* const tb = ta + A_BYTES;
#pragma unroll
        for (int ks = 0; ks < BK / 32; ++ks) {
            typename Frag<T>::type fa[FM], fb[FN];
#pragma unroll
            for (int j = 0; j < FM; ++j) fa[j] = ra.get(ta, j, ks);
#pragma unroll
            for (int i = 0; i < FN; ++i) fb[i] = rb.get(tb, i, ks);
            if constexpr (decltype(last)::value) {
                const int left = tail - ks * 32 - lg * 8;
#pragma unroll
                for (int j = 0; j < FM; ++j) if (!AR) fa[j] = keep_first(fa[j], left);
#pragma unroll
                for (int i = 0; i < FN; ++i) if (!BR) fb[i] = keep_first(fb[i], left);
            }
#pragma unroll
            for (int i = 0; i < FN; ++i)
#pragma unroll
                for (int j = 0; j < FM; ++j) acc[i][j] = mma(fb[i], fa[j], acc[i][j]);
        }
    };
    auto pass = [&] {
        ask(0);
        for (int t = 0; t < whole; ++t) {
            arrive_all();
            if (t + 1 < steps) ask((t + 1) & 1);
            multiply(t & 1, std::false_type{});
        }
        if (tail) {
            arrive_all();
            multiply(whole & 1, std::true_type{});
        }
    };
    auto scale = [&](float by) {
#pragma unroll
        for (int i = 0; i < FN; ++i)
#pragma unroll
            for (int j = 0; j < FM; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] = fabsf(acc[i][j][e]) < INFINITY ? acc[i][j][e] * by : 0.f;
    };
    if constexpr (TWO) {
        pass();
        scale(1.f / LOW_PART<T>);
        wa = window<AR, 2, BK>(g.a, g.lda, g.M, g.K, m0, k0);
        wb = window<BR, 2, BK>(g.b, g.ldb, g.N, g.K, n0, k0);
        arrive_all();                                    // the tiles have been read
    }
    pass();
    if constexpr (TWO) {
#pragma unroll
        for (int i = 0; i < FN; ++i)
#pragma unroll
            for (int j = 0; j < FM; ++j) acc[i][j] *= 1.f / HIGH_PART<T>;
    }
    __syncthreads();                                     // the tiles have been read
    if constexpr (GATED) {
        if (busy) finish_gated_wave<T, FM, FN>(g, acc, (float*)smem + wave * box_floats<FN>(), m0 + wm, n0 + wn / 2, lane, split, splits);
    } else if (busy) finish_wave<T, FM, FN>(g, acc, (float*)smem + wave * box_floats<FN>(), m0 + wm, n0 + wn, lane, split, splits);
}

// ------------------------------------------------------------------------------------------------ gated, short k
// Where k is short a tile's loads, products and stores each wait for the others. Here rows stay: a wave holds its 16 FM rows of x, at most 32 KS k of
// them, in registers as second operands, and the weights pass by in chunks of 32 columns of y (both halves: 64 rows of w) in two buffers of LDS that
// take turns. A block's row 4 lg + e is the chunk's column 8 lg + 4 c + e (c: which of two blocks), so that a lane's sums are eight columns of one row in
// both halves and go to memory from the registers. Two chunks are stored together, for whole lines of 128 bytes (one by one, 32400 x 256 -> 2 x 1024 bf16
// with silu and preact took 73 us, 129600 x 256 -> 2 x 512 with gelu and preact 148), and have the next chunk's products to leave.
// In tiles (tiles of 128 x 256 above) and here, us: 32400 x 256 -> 2 x 1024 with preact 80 and 62, without 67 and 53; 129600 x 256 -> 2 x 512 160 and 120 (464 MB, 3.9
// TB/s), 117 and 86; 129600 x 128 -> 2 x 256 64 and 57, 48 and 38. With a preact bound by stores, else by the LDS reads of weights (27 us of 86 at their
// peak; 64 rows a wave would halve them but spill with two chunks of results) and the activation.
// as dma16, four bytes a lane
__device__ __forceinline__ void dma4(i32x4 rsrc, unsigned lds, unsigned voff) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds"
                 :: "s"(lds), "v"(voff), "s"(rsrc) : "memory");
}
constexpr unsigned NOWHERE = 0x7ffffff8u;                // beyond any resource's size
template <class T, int FM, int WAVES, int KS>
__global__ __launch_bounds__(64 * WAVES, WAVES / 2) void short_gated_kernel(ProductArgs g, int tm, int parts, int per) {
    constexpr int ROW = KS * 64, HALF = 64 * ROW, LOADS = HALF / (1024 * WAVES), IN_HALF = HALF / 2048;
    typedef typename Frag<T>::type F;
    __shared__ __align__(1024) unsigned char smem[2 * HALF];
    __shared__ __align__(256) float bias[2][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lr = lane & 15, lg = lane >> 4;
    // an XCD takes all chunks of the rows that it takes
    const int turn = blockIdx.x >> 3, mt = turn / parts * 8 + (blockIdx.x & 7), part = turn % parts;
    if (mt >= tm) return;
    const int chunks = (g.N + 31) >> 5, lo = part * per, hi = min(chunks, lo + per);
    const int m0 = (mt * WAVES + wave) * 16 * FM;
    Window wg = window<false, 2, 32>(g.b, g.ldb, g.N, g.K, 32 * lo, 0), wu = wg;
    wg.step = wu.step = 64 * g.ldb;
    wu.at += (int64_t)g.N * g.ldb * 2;
    unsigned voff[LOADS];
#pragma unroll
    for (int q = 0; q < LOADS; ++q) {
        const int p = (q * WAVES + wave) * 64 + lane, r = p / (4 * KS) & 31, piece = (p % (4 * KS)) ^ ((r & 3) | (r >> 3 & 1) << 2);
        voff[q] = 8 * piece < g.K ? (unsigned)(r * g.ldb * 2) + piece * 16 : NOWHERE;
    }
    const i32x4 rb = {__builtin_amdgcn_readfirstlane((int)(uint64_t)g.bias), __builtin_amdgcn_readfirstlane((int)((uint64_t)g.bias >> 32) & 0xffff),
                      g.bias ? 8 * g.N : 0, 0x00020000};
    const unsigned lds_at = (unsigned)(uintptr_t)(lds_byte*)smem, bias_at = (unsigned)(uintptr_t)(lds_byte*)bias;
    int asked = 32 * lo;
    auto ask = [&](int half) {
        const i32x4 one = wg.rsrc(), two = wu.rsrc();
#pragma unroll
        for (int q = 0; q < LOADS; ++q)
            dma16(q * WAVES + wave >= IN_HALF ? two : one, lds_at + half * HALF + (q * WAVES + wave) * 1024, voff[q]);
        if (wave == 0) {
            const int n = asked + (lane & 31);
            dma4(rb, bias_at + half * 256, n < g.N ? (unsigned)(n + (lane >> 5) * g.N) * 4 : NOWHERE);
        }
        wg.next(); wu.next(); asked += 32;
    };
    ask(0);
    F x[KS][FM];
#pragma unroll
    for (int j = 0; j < FM; ++j) {
        const T* const row = (const T*)g.a + (int64_t)min(m0 + 16 * j + lr, g.M - 1) * g.lda;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const int k = 32 * s + 8 * lg;
            const F v = __builtin_bit_cast(F, *reinterpret_cast<const typename Some<T, 8>::type*>(row + (k < g.K ? k : 0)));
            x[s][j] = k < g.K ? v : F{};
        }
    }
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int j = 0; j < FM; ++j) asm volatile("" : "+v"(x[s][j]));
    arrive_all();
    if (lo + 1 < hi) ask(1);
    const int row_at = (8 * (lr >> 2) + (lr & 3)) * ROW, even = row_at + ((lg ^ (lr & 7)) << 4), odd = row_at + (((4 + lg) ^ (lr & 7)) << 4);
    typedef typename Some<T, 8>::type Row8;
    Row8 held[FM][3];                                    // the first chunk of two, to go with the second one's as whole lines
    auto chunk = [&](int c, auto turn) {
        constexpr int half = decltype(turn)::value;
        const unsigned char* const tile = smem + half * HALF;
        f32x4 acc[4][FM];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const f32x4 v = *reinterpret_cast<const f32x4*>(&bias[half][(b >> 1) * 32 + 8 * lg + 4 * (b & 1)]);
#pragma unroll
            for (int j = 0; j < FM; ++j) acc[b][j] = v;
        }
        auto weights = [&](F (&w)[4], int s) {
#pragma unroll
            for (int b = 0; b < 4; ++b)
                w[b] = *reinterpret_cast<const F*>(tile + (s & 1 ? odd : even) + (s >> 1) * 128 + (b & 1) * 4 * ROW + (b >> 1) * 32 * ROW);
        };
        F w[2][4];
        weights(w[0], 0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            if (s + 1 < KS) weights(w[(s + 1) & 1], s + 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int j = 0; j < FM; ++j) acc[b][j] = mma(w[s & 1][b], x[s][j], acc[b][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
        arrive_all();                                    // the next chunk is there, and this one has been read
        if (c + 2 < hi) ask(half);
        const bool both = half ? 32 * c + 32 <= g.N : c + 1 < hi && 32 * c + 64 <= g.N;
        const int n = 32 * c + 8 * lg;
#pragma unroll
        for (int j = 0; j < FM; ++j) {
            const int m = m0 + 16 * j + lr;
            float gate[8], up[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) { gate[e] = acc[e >> 2][j][e & 3]; up[e] = acc[2 + (e >> 2)][j][e & 3]; }
            if (!both) { store_gated<T, 8>(g, gate, up, m, n); continue; }
            Row8 v[3];
#pragma unroll
            for (int e = 0; e < 8; ++e) { v[1][e] = (T)gate[e]; v[2][e] = (T)up[e]; }
            row_act_all(g.act, gate);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[0][e] = (T)(gate[e] * up[e]);
            if constexpr (!half) {
#pragma unroll
                for (int i = 0; i < 3; ++i) held[j][i] = v[i];
            } else if (m < g.M) {
                auto store = [&](T* to, int i) {
                    Row8* const one = reinterpret_cast<Row8*>(to - 32); Row8* const two = reinterpret_cast<Row8*>(to);
                    if (g.past) { __builtin_nontemporal_store(held[j][i], one); __builtin_nontemporal_store(v[i], two); }
                    else { *one = held[j][i]; *two = v[i]; }
                };
                store((T*)g.y + (int64_t)m * g.ldy + n, 0);
                if (g.pre) {
                    T* const z = (T*)g.pre + (int64_t)m * 2 * g.N + n;
                    store(z, 1); store(z + g.N, 2);
                }
            }
        }
    };
    for (int c = lo; c < hi; c += 2) {
        chunk(c, std::integral_constant<int, 0>{});
        if (c + 1 < hi) chunk(c + 1, std::integral_constant<int, 1>{});
    }
}

// ------------------------------------------------------------------------------------------------ fp32 operands
// An fp32 value is the sum of three bf16 values; the six of the nine partial products that reach 2^-24 are accumulated in
// fp32.  Steps of 32 k: the thread that loads four elements splits them and writes them to three planes in LDS, the next step's on
// their way into registers meanwhile.
//   k contiguous:    rows of 64 bytes, piece p of row r at p ^ (r / 2 & 3)
//   rows contiguous: as for 16 bits, 32 k-rows
// 4096^3: 0.61 ms = 225 TFLOP/s, 1.35 PFLOP/s of bf16 products: the library's rate.  Short sums add their stores to that, one after the other:
// 518400 x 1024 -> 256 is 1290 us of products and 109 of stores, 1399 in all; x 324 -> 256: 438 and 109, 600 to 710 us (as the clock falls under
// sustained work: 1.8 GHz, matrix instructions in 43 % of the cycles, splitting in 28 %).  Without loads that took 531 us, with one
// product of six 472.  Two workgroups a compute unit; a third spills (838 us), and so does a second set of loads on their way.
template <bool ROWS, int R, int NT, bool GATED = false>
struct Loader32 {
    static constexpr int PIECES = R * 8 / NT;
    unsigned voff[PIECES], dst[PIECES];
    f32x4 x[PIECES];
    int k[PIECES];
    __device__ __forceinline__ void plan(int tid, int64_t ld) {
#pragma unroll
        for (int q = 0; q < PIECES; ++q) {
            const int p = q * NT + tid;
            if constexpr (ROWS) {
                const int kr = p / (R / 4), c = p % (R / 4);
                k[q] = kr;
                voff[q] = (unsigned)(kr * ld * 4) + c * 16;
                dst[q] = kr * 2 * R + (((c >> 2) ^ turn<R>(kr)) << 5) + (c & 3) * 8;
            } else {
                const int row = p >> 3, c = p & 7;
                k[q] = c * 4;
                voff[q] = (unsigned)((GATED ? in_half(row) : row) * ld * 4) + c * 16;
                dst[q] = row * 64 + (((c >> 1) ^ (row >> 1 & 3)) << 4) + (c & 1) * 8;
            }
        }
    }
    __device__ __forceinline__ void ask(const Window& w) {
        const __amdgpu_buffer_rsrc_t r = w.buffer();
#pragma unroll
        for (int q = 0; q < PIECES; ++q)
            x[q] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)voff[q], 0, 0));
    }
    // a wave's 64 pieces are eight rows of one half
    __device__ __forceinline__ void ask(const Window& gate, const Window& up, int wave) {
#pragma unroll
        for (int q = 0; q < PIECES; ++q) {
            const __amdgpu_buffer_rsrc_t r = second_half((q * NT / 64 + wave) * 8) ? up.buffer() : gate.buffer();
            x[q] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)voff[q], 0, 0));
        }
    }
    __device__ __forceinline__ void cut(int left) {      // the last step of rows with k contiguous
        if constexpr (!ROWS) {
#pragma unroll
            for (int q = 0; q < PIECES; ++q)
#pragma unroll
                for (int e = 0; e < 4; ++e) if (k[q] + e >= left) x[q][e] = 0.f;
        }
    }
    __device__ __forceinline__ void split(unsigned char* plane0) const {
#pragma unroll
        for (int q = 0; q < PIECES; ++q) {
            f32x2 lo = {x[q][0], x[q][1]}, hi = {x[q][2], x[q][3]};
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                const bf16x2 cl = __builtin_convertvector(lo, bf16x2), ch = __builtin_convertvector(hi, bf16x2);
                *reinterpret_cast<u32x2*>(plane0 + p * (R * 64) + dst[q]) = u32x2{__builtin_bit_cast(unsigned, cl), __builtin_bit_cast(unsigned, ch)};
                if (p < 2) {
                    lo -= __builtin_convertvector(cl, f32x2);
                    hi -= __builtin_convertvector(ch, f32x2);
                }
            }
        }
    }
};
template <bool ROWS, int R, int F>
struct Reader32 {
    unsigned off[ROWS ? F : 1];
    __device__ __forceinline__ void plan(int base, int lr, int lg) {
        if constexpr (ROWS) {
#pragma unroll
            for (int i = 0; i < F; ++i) {
                const int k = 8 * lg + (lr >> 2);
                off[i] = k * (2 * R) + (((base >> 4) + i) ^ turn<R>(k)) * 32 + (lr & 3) * 8;
            }
        } else off[0] = (base + lr) * 64 + ((lg ^ (lr >> 1 & 3)) << 4);
    }
    __device__ __forceinline__ bf16x8 get(lds_byte* plane, int i) const {
        if constexpr (ROWS) {
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(plane + off[i]));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(plane + off[i] + 4 * 2 * R));
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else return *(__attribute__((address_space(3))) bf16x8*)(plane + off[0] + i * 1024);
    }
};

template <bool AR, bool BR, int BM, int BN, int WM, int WN, bool GATED = false>
__global__ __launch_bounds__(64 * WM * WN, 2) void product32_kernel(ProductArgs g, int tm, int tn, int splits, int steps_per) {
    constexpr int NT = 64 * WM * WN, TM = BM / WM, TN = BN / WN, FM = TM / 16, FN = TN / 16;
    constexpr int PA = BM * 64, PB = BN * 64;
    __shared__ __align__(1024) unsigned char smem[3 * (PA + PB)];
    lds_byte* const lds = (lds_byte*)smem;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lr = lane & 15, lg = lane >> 4;
    int mt, nt, split;
    tile_of(blockIdx.x, tm, tn, splits, mt, nt, split);
    const int m0 = mt * BM, n0 = nt * (GATED ? BN / 2 : BN);
    const int k0 = split * steps_per * 32, k_left = min(g.K - k0, steps_per * 32), steps = (k_left + 31) >> 5;
    Window wa = window<AR, 4, 32>(g.a, g.lda, g.M, g.K, m0, k0), wb = window<BR, 4, 32>(g.b, g.ldb, g.N, g.K, n0, k0);
    Window wu = wb;
    if constexpr (GATED) wu.at += (int64_t)g.N * g.ldb * 4;
    Loader32<AR, BM, NT> la;
    Loader32<BR, BN, NT, GATED> lb;
    la.plan(tid, g.lda);
    lb.plan(tid, g.ldb);
    const int wm = (wave % WM) * TM, wn = (wave / WM) * TN;
    Reader32<AR, BM, FM> ra;
    Reader32<BR, BN, FN> rb;
    ra.plan(wm, lr, lg);
    rb.plan(wn, lr, lg);
    f32x4 acc[FN][FM] = {};
    auto ask = [&] {
        la.ask(wa);
        if constexpr (GATED) lb.ask(wb, wu, wave);
        else lb.ask(wb);
    };
    ask();
    auto step = [&](auto last) {
        if constexpr (decltype(last)::value) { la.cut(k_left - 32 * (steps - 1)); lb.cut(k_left - 32 * (steps - 1)); }
        __syncthreads();                                 // the last step's fragments have been read
        la.split(smem); lb.split(smem + 3 * PA);
        if constexpr (!decltype(last)::value) {
            wa.next(); wb.next();
            if constexpr (GATED) wu.next();
            ask();
        }
        __syncthreads();
        bf16x8 fa[3][FM], fb[3][FN];
#pragma unroll
        for (int p = 0; p < 3; ++p) {
#pragma unroll
            for (int i = 0; i < FN; ++i) fb[p][i] = rb.get(lds + 3 * PA + p * PB, i);
#pragma unroll
            for (int j = 0; j < FM; ++j) fa[p][j] = ra.get(lds + p * PA, j);
        }
        // small products first
        constexpr int QA[6] = {2, 0, 1, 1, 0, 0}, QB[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
        for (int q = 0; q < 6; ++q)
#pragma unroll
            for (int i = 0; i < FN; ++i)
#pragma unroll
                for (int j = 0; j < FM; ++j) acc[i][j] = mma(fb[QB[q]][i], fa[QA[q]][j], acc[i][j]);
    };
    for (int t = 0; t + 1 < steps; ++t) step(std::false_type{});
    step(std::true_type{});                              // the only one that can be short
    // An infinity, a NaN or a value beyond bf16's range has no three parts (its remainder is infinity - infinity): what is
    // not finite here is taken from fp32 instructions instead, one k of a row per lane.
    float none = 0.f;                                    // NaN if any sum is not finite (past the borders anything may lie)
    auto column = [&](int i) { return n0 + (GATED ? in_half(wn + 16 * i) : wn + 16 * i); };
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
        for (int j = 0; j < FM; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                none = fmaf(m0 + wm + 16 * j + lr < g.M && column(i) + 4 * lg + e < g.N ? acc[i][j][e] : 0.f, 0.f, none);
    if (__any(none != 0.f)) {
        const float* const A = (const float*)g.a;
        const float* const B = (const float*)g.b;
        for (int i = 0; i < FN; ++i)
            for (int j = 0; j < FM; ++j) {
                f32x4 plain = {};
                const int64_t m = min(m0 + wm + 16 * j + lr, g.M - 1), n = min(column(i) + lr, g.N - 1) + (GATED && (i & 1) ? g.N : 0);
                for (int k = 0; k < k_left; k += 4) {
                    float xa = 0.f, xb = 0.f;
                    if (k + lg < k_left) {
                        const int64_t kk = k0 + k + lg;
                        xa = A[AR ? kk * g.lda + m : m * g.lda + kk];
                        xb = B[BR ? kk * g.ldb + n : n * g.ldb + kk];
                    }
                    plain = __builtin_amdgcn_mfma_f32_16x16x4f32(xb, xa, plain, 0, 0, 0);
                }
#pragma unroll
                for (int ii = 0; ii < FN; ++ii)
#pragma unroll
                    for (int jj = 0; jj < FM; ++jj)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (ii == i && jj == j && !(fabsf(acc[ii][jj][e]) < INFINITY)) acc[ii][jj][e] = plain[e];
            }
    }
    __syncthreads();                                     // the planes have been read
    if constexpr (GATED) finish_gated_wave<float, FM, FN>(g, acc, (float*)smem + wave * box_floats<FN>(), m0 + wm, n0 + wn / 2, lane, split, splits);
    else finish_wave<float, FM, FN>(g, acc, (float*)smem + wave * box_floats<FN>(), m0 + wm, n0 + wn, lane, split, splits);
}

// ------------------------------------------------------------------------------------------------ few rows
// Up to 16 MT rows: every weight is read once, straight into the matrix instruction's fragments.  A workgroup makes 16 columns
// of C; its waves take turns along k and add up in LDS.  Bound by the weights' bytes: 1 x 4096 -> 16384 bf16: 22 us, 6.1 TB/s (weights that
// lie in the memory-side cache; 28 from memory).
template <class T>
__device__ __forceinline__ typename Frag<T>::type few_load(const T* p, int left) {       // 8 elements, zeros from `left` on
    if (left >= 8) return *reinterpret_cast<const typename Some<T, 8>::type*>(p);
    typename Frag<T>::type v = {};
#pragma unroll
    for (int e = 0; e < 8; ++e) if (e < left) v[e] = p[e];
    return v;
}
// The waves' sums in their order, and the epilogue.
template <class T, int WAVES, int MT, bool GATED>
__device__ __forceinline__ void few_finish(const ProductArgs& g, f32x4 (&sums)[WAVES][GATED ? 2 * MT : MT][64], int wave, int lane, int n0) {
    const int lr = lane & 15, lg = lane >> 4;
    for (int j = wave; j < MT; j += WAVES) {
        f32x4 x = sums[0][j][lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) x += sums[w][j][lane];
        float v[4] = {x[0], x[1], x[2], x[3]};
        if constexpr (GATED) {
            x = sums[0][MT + j][lane];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) x += sums[w][MT + j][lane];
            float up[4] = {x[0], x[1], x[2], x[3]}, bias[2][4];
            load_gated_bias(g, bias, n0 + 4 * lg);
            finish_gated<T, 4>(g, v, up, bias, 16 * j + lr, n0 + 4 * lg);
        } else {
            float bias[4];
            load_bias(g, bias, n0 + 4 * lg);
            finish<T, 4>(g, v, bias, 16 * j + lr, n0 + 4 * lg);
        }
    }
}
// GATED: 16 columns of both halves, as MT more sums.
template <class T, int WAVES, int MT, bool GATED = false>
__global__ __launch_bounds__(64 * WAVES) void few_rows16_kernel(ProductArgs g) {
    constexpr int H = GATED ? 2 : 1;
    __shared__ f32x4 sums[WAVES][H * MT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lr = lane & 15, lg = lane >> 4;
    const int n0 = blockIdx.x * 16, n = n0 + lr;
    const T* W[H];
#pragma unroll
    for (int h = 0; h < H; ++h) W[h] = (const T*)g.b + ((int64_t)min(n, g.N - 1) + (int64_t)h * g.N) * g.ldb;
    const T* X[MT];
#pragma unroll
    for (int j = 0; j < MT; ++j) X[j] = (const T*)g.a + (int64_t)min(16 * j + lr, g.M - 1) * g.lda;
    f32x4 acc[H * MT] = {};
    constexpr int U = H * MT == 1 ? 4 : 2;               // 32 k each
    int k = wave * 32 * U + lg * 8;
    for (; k - lg * 8 + 32 * U <= g.K; k += WAVES * 32 * U) {
        typename Frag<T>::type w[U][H], x[U][MT];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < H; ++h) w[u][h] = few_load<T>(W[h] + k + 32 * u, 8);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < MT; ++j) x[u][j] = few_load<T>(X[j] + k + 32 * u, 8);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < H; ++h)
#pragma unroll
                for (int j = 0; j < MT; ++j) acc[h * MT + j] = mma(w[u][h], x[u][j], acc[h * MT + j]);
    }
    for (int u = 0; u < U; ++u, k += 32) {               // the one wave whose turn the last, shorter stretch is
        if (k - lg * 8 >= g.K) break;
#pragma unroll
        for (int h = 0; h < H; ++h) {
            const typename Frag<T>::type w = few_load<T>(W[h] + k, g.K - k);
#pragma unroll
            for (int j = 0; j < MT; ++j) acc[h * MT + j] = mma(w, few_load<T>(X[j] + k, g.K - k), acc[h * MT + j]);
        }
    }
#pragma unroll
    for (int j = 0; j < H * MT; ++j) sums[wave][j][lane] = acc[j];
    __syncthreads();
    few_finish<T, WAVES, MT, GATED>(g, sums, wave, lane, n0);
}
// fp32: v_mfma_f32_16x16x4_f32, whose four k are the same element of four lanes' 16 bytes.
__device__ __forceinline__ f32x4 few_load32(const float* p, int left) {
    if (left >= 4) return *reinterpret_cast<const Some<float, 4>::type*>(p);
    f32x4 v = {};
#pragma unroll
    for (int e = 0; e < 4; ++e) if (e < left) v[e] = p[e];
    return v;
}
template <int WAVES, int MT, bool GATED = false>
__global__ __launch_bounds__(64 * WAVES) void few_rows32_kernel(ProductArgs g) {
    constexpr int H = GATED ? 2 : 1;
    __shared__ f32x4 sums[WAVES][H * MT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lr = lane & 15, lg = lane >> 4;
    const int n0 = blockIdx.x * 16, n = n0 + lr;
    const float* W[H];
#pragma unroll
    for (int h = 0; h < H; ++h) W[h] = (const float*)g.b + ((int64_t)min(n, g.N - 1) + (int64_t)h * g.N) * g.ldb;
    const float* X[MT];
#pragma unroll
    for (int j = 0; j < MT; ++j) X[j] = (const float*)g.a + (int64_t)min(16 * j + lr, g.M - 1) * g.lda;
    f32x4 acc[H * MT] = {};
    constexpr int U = H * MT == 1 ? 4 : 2;               // 16 k each
    int k = wave * 16 * U + lg * 4;
    for (; k - lg * 4 + 16 * U <= g.K; k += WAVES * 16 * U) {
        f32x4 w[U][H], x[U][MT];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < H; ++h) w[u][h] = few_load32(W[h] + k + 16 * u, 4);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < MT; ++j) x[u][j] = few_load32(X[j] + k + 16 * u, 4);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int h = 0; h < H; ++h)
#pragma unroll
                    for (int j = 0; j < MT; ++j)
                        acc[h * MT + j] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[u][h][e], x[u][j][e], acc[h * MT + j], 0, 0, 0);
    }
    for (int u = 0; u < U; ++u, k += 16) {
        if (k - lg * 4 >= g.K) break;
#pragma unroll
        for (int h = 0; h < H; ++h) {
            const f32x4 w = few_load32(W[h] + k, g.K - k);
#pragma unroll
            for (int j = 0; j < MT; ++j) {
                const f32x4 x = few_load32(X[j] + k, g.K - k);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[h * MT + j] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[e], x[e], acc[h * MT + j], 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < H * MT; ++j) sums[wave][j][lane] = acc[j];
    __syncthreads();
    few_finish<float, WAVES, MT, GATED>(g, sums, wave, lane, n0);
}

// ------------------------------------------------------------------------------------------------ splits, packing, slopes
// The splits' sums, then the epilogue.  LANES threads take turns at a quad's splits (in a fixed order: the sum has the same bits on every
// call), so that few outputs with many splits still keep enough loads on their way.
template <class T, int LANES>
__global__ __launch_bounds__(256) void join_kernel(ProductArgs g, int splits) {
    __shared__ f32x4 sums[LANES > 1 ? 256 : 1];
    constexpr int QUADS = 256 / LANES;
    const int quads = (g.N + 3) >> 2, lane = threadIdx.x / QUADS, slot = threadIdx.x % QUADS;
    const int64_t total = (int64_t)g.M * quads, plane = (int64_t)g.M * g.N, q = (int64_t)blockIdx.x * QUADS + slot;
    const int64_t m = q / quads;
    const int n = (int)(q - m * quads) * 4;
    f32x4 x = {};
    if (q < total) {
        const float* p = g.part + m * g.N + n + lane * plane;
#pragma unroll 4
        for (int s = lane; s < splits; s += LANES, p += LANES * plane) {
            float v[4];
            load_some<float, 4>(p, v, g.N - n);
            x += f32x4{v[0], v[1], v[2], v[3]};
        }
    }
    if constexpr (LANES > 1) {
        sums[threadIdx.x] = x;
        __syncthreads();
        if (lane) return;
#pragma unroll
        for (int l = 1; l < LANES; ++l) x += sums[l * QUADS + slot];
    }
    if (q >= total) return;
    float v[4] = {x[0], x[1], x[2], x[3]}, bias[4];
    load_bias(g, bias, n);
    finish<T, 4>(g, v, bias, (int)m, n);
}
// Gated: the two halves' sums.
template <class T>
__global__ __launch_bounds__(256) void join_gated_kernel(ProductArgs g, int splits) {
    const int quads = (g.N + 3) >> 2;
    const int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x, m = q / quads, plane = (int64_t)g.M * 2 * g.N;
    if (m >= g.M) return;
    const int n = (int)(q - m * quads) * 4;
    const float* p = g.part + m * 2 * g.N + n;
    float sum[2][4] = {}, bias[2][4];
#pragma unroll 4
    for (int s = 0; s < splits; ++s, p += plane) {
        float v[4], w[4];
        load_some<float, 4>(p, v, g.N - n);
        load_some<float, 4>(p + g.N, w, g.N - n);
#pragma unroll
        for (int e = 0; e < 4; ++e) { sum[0][e] += v[e]; sum[1][e] += w[e]; }
    }
    load_gated_bias(g, bias, n);
    finish_gated<T, 4>(g, sum[0], sum[1], bias, (int)m, n);
}
template <class T>
void join(const ProductArgs& g, const ProductPlan& p, hipStream_t s) {
    if (g.gated) {
        hipLaunchKernelGGL((join_gated_kernel<T>), dim3((unsigned)(((int64_t)g.M * ((g.N + 3) / 4) + 255) / 256)), dim3(256), 0, s, g, p.splits);
        return;
    }
    const int64_t quads = (int64_t)g.M * ((g.N + 3) / 4);
    if (p.splits >= 8) hipLaunchKernelGGL((join_kernel<T, 8>), dim3((unsigned)((quads + 31) / 32)), dim3(256), 0, s, g, p.splits);
    else hipLaunchKernelGGL((join_kernel<T, 1>), dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, s, g, p.splits);
}

// Rows to 16-byte borders, zeros behind their ends, of two matrices in one launch: eight elements a thread.
__global__ __launch_bounds__(256) void pack16_kernel(Pack16 one, Pack16 two) {
    const int64_t ones = one.rows * (one.ld_dst / 8), all = ones + two.rows * (two.ld_dst / 8);
    for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < all; k += (int64_t)gridDim.x * 256) {
        const Pack16& p = k < ones ? one : two;
        const int64_t i = k < ones ? k : k - ones;
        const int pieces = (int)(p.ld_dst / 8);
        const int64_t r = all < (1LL << 31) ? (int64_t)((unsigned)i / (unsigned)pieces) : i / pieces;
        const int c = (int)(i - r * pieces) * 8;
        const uint16_t* const src = (const uint16_t*)p.src + r * p.ld_src + c;
        u32x4 x;
        if (c + 8 <= p.cols) x = __builtin_bit_cast(u32x4, *reinterpret_cast<const Some<short, 8>::type*>(src));
        else
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                const unsigned lo = c + 2 * d < p.cols ? src[2 * d] : 0, hi = c + 2 * d + 1 < p.cols ? src[2 * d + 1] : 0;
                x[d] = lo | hi << 16;
            }
        *reinterpret_cast<u32x4*>((uint16_t*)p.dst + i * 8) = x;
    }
}

// dz = dy act'(z) and its column sums in one pass.  A thread has V columns and every RT-th row of its workgroup's share, two at a time; the sums
// over rows meet in LDS.  Bound by bytes: 32400 x 1024 fp32: 74 us, 5.4 TB/s; 129600 x 256 bf16: 42 us, 4.7 TB/s.  dz is rounded to the
// operands' type because the matrix cores take it so; the sums add what was not rounded.  bf16: once; the rounding is as large as that of the
// results, whose error grows to sqrt 2 times theirs alone.  fp16 holds dz in two parts where an activation shapes it (`dz_lo`):
// with one, a small d_y times a small slope would lose its digits below 6e-5 and vanish below 3e-8, fp16's largest times gelu's 1.13 would
// overflow, and half of the results would not be the nearest fp16 values (with two: 1 in 1000).
constexpr int SLOPE_THREADS = 256;
template <class T, int V>
__global__ __launch_bounds__(SLOPE_THREADS) void slope_kernel(int act, const T* __restrict__ dy, int64_t ld_dy, const T* __restrict__ z,
                                                             T* __restrict__ dz, T* __restrict__ dz_lo, int64_t ld_dz, float* __restrict__ part,
                                                             int64_t M, int N, int ct, int64_t rows_per) {
    __shared__ float sums[SLOPE_THREADS][V];
    const int tid = threadIdx.x, c = tid % ct, rt = SLOPE_THREADS / ct, r0 = tid / ct;
    const int n = (blockIdx.x * ct + c) * V, left = N - n;
    const int64_t lo = (int64_t)blockIdx.y * rows_per, hi = min(M, lo + rows_per);
    float sum[V] = {};
    if (left > 0) {
        for (int64_t m = lo + r0; m < hi; m += 2 * rt) {
            const bool two = m + rt < hi;
            float v[2][V], s[2][V];
            load_some<T, V>(dy + m * ld_dy + n, v[0], left);
            if (act != CORR_ACT_NONE) load_some<T, V>(z + m * N + n, s[0], left);
            if (two) {
                load_some<T, V>(dy + (m + rt) * ld_dy + n, v[1], left);
                if (act != CORR_ACT_NONE) load_some<T, V>(z + (m + rt) * N + n, s[1], left);
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (u && !two) break;
                if (act != CORR_ACT_NONE) {
                    row_slope_all(act, s[u]);
#pragma unroll
                    for (int e = 0; e < V; ++e) v[u][e] *= s[u][e];
                }
#pragma unroll
                for (int e = 0; e < V; ++e) sum[e] += v[u][e];
                if constexpr (std::is_same<T, _Float16>::value) if (dz_lo) {
                    float lo[V];
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float x = HIGH_PART<T> * v[u][e], d = x - (float)(T)x;
                        lo[e] = d == d ? LOW_PART<T> * d : 0.f;         // an infinity or NaN is in the high part
                        v[u][e] = x;
                    }
                    store_some<T, V>(dz_lo + (m + u * rt) * ld_dz + n, lo, left);
                }
                if (dz) store_some<T, V>(dz + (m + u * rt) * ld_dz + n, v[u], left);
            }
        }
    }
    if (!part) return;
#pragma unroll
    for (int e = 0; e < V; ++e) sums[tid][e] = sum[e];
    __syncthreads();
    if (r0 == 0 && left > 0) {
        for (int r = 1; r < rt; ++r)
#pragma unroll
            for (int e = 0; e < V; ++e) sum[e] += sums[r * ct + c][e];
        store_some<float, V>(part + (int64_t)blockIdx.y * N + n, sum, left);
    }
}

// Gated: dz of both halves, [M][2 N]: d_y up act'(gate) and d_y act(gate), rounded as above (two parts where dz_lo is there), and their column sums.  fp16's
// parts hold values up to 1.3e5.  Bound by bytes: 129600 x 512 bf16 with gelu: 146 us, 663 MB, 4.5 TB/s.
template <class T, int V>
__global__ __launch_bounds__(SLOPE_THREADS) void slope_gated_kernel(int act, const T* __restrict__ dy, int64_t ld_dy, const T* __restrict__ z,
                                                                   T* __restrict__ dz, T* __restrict__ dz_lo, int64_t ld_dz, float* __restrict__ part,
                                                                   int64_t M, int N, int ct, int64_t rows_per) {
    __shared__ float sums[2][SLOPE_THREADS][V];
    const int tid = threadIdx.x, c = tid % ct, rt = SLOPE_THREADS / ct, r0 = tid / ct;
    const int n = (blockIdx.x * ct + c) * V, left = N - n;
    const int64_t lo = (int64_t)blockIdx.y * rows_per, hi = min(M, lo + rows_per);
    float sum[2][V] = {};
    if (left > 0)
        for (int64_t m = lo + r0; m < hi; m += rt) {
            float d[2][V], gate[V], up[V];
            load_some<T, V>(dy + m * ld_dy + n, d[0], left);
            load_some<T, V>(z + m * 2 * N + n, gate, left);
            load_some<T, V>(z + m * 2 * N + N + n, up, left);
            float slope[V];
#pragma unroll
            for (int e = 0; e < V; ++e) slope[e] = gate[e];
            row_act_all(act, gate);
            row_slope_all(act, slope);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                d[1][e] = d[0][e] * gate[e];
                d[0][e] = d[0][e] * slope[e] * up[e];    // in this order: of the two, only up can be large
                sum[0][e] += d[0][e];
                sum[1][e] += d[1][e];
            }
            if (!dz) continue;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t to = m * ld_dz + h * N + n;
                if constexpr (sizeof(T) == 2) if (dz_lo) {
                    float lo_part[V];
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float x = HIGH_PART<T> * d[h][e], r = x - (float)(T)x;
                        lo_part[e] = fabsf(r) < INFINITY ? LOW_PART<T> * r : 0.f;       // an infinity or NaN is in the high part
                        d[h][e] = x;
                    }
                    store_some<T, V>(dz_lo + to, lo_part, left);
                }
                store_some<T, V>(dz + to, d[h], left);
            }
        }
    if (!part) return;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < V; ++e) sums[h][tid][e] = sum[h][e];
    __syncthreads();
    if (r0 == 0 && left > 0) {
        for (int r = 1; r < rt; ++r)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < V; ++e) sum[h][e] += sums[h][r * ct + c][e];
#pragma unroll
        for (int h = 0; h < 2; ++h) store_some<float, V>(part + (int64_t)blockIdx.y * 2 * N + h * N + n, sum[h], left);
    }
}

template <class T, bool AR, bool BR, int BM, int BN, int WM, int WN, int BK>
void run16(const ProductArgs& g, const ProductPlan& p, hipStream_t s) {
    if constexpr (!AR && !BR) {
        if (g.gated) {
            const int tm = cdiv(g.M, BM), tn = cdiv(g.N, BN / 2);
            hipLaunchKernelGGL((product16_kernel<T, AR, BR, BM, BN, WM, WN, BK, false, true>), dim3(tm * tn * p.splits), dim3(64 * WM * WN), 0, s, g, tm, tn, p.splits, p.steps);
            return;
        }
    }
    const int tm = cdiv(g.M, BM), tn = cdiv(g.N, BN);
    if constexpr (BR) {
        if (g.a_lo) {
            hipLaunchKernelGGL((product16_kernel<T, AR, BR, BM, BN, WM, WN, BK, true>), dim3(tm * tn * p.splits), dim3(64 * WM * WN), 0, s, g, tm, tn, p.splits, p.steps);
            return;
        }
    }
    hipLaunchKernelGGL((product16_kernel<T, AR, BR, BM, BN, WM, WN, BK, false>), dim3(tm * tn * p.splits), dim3(64 * WM * WN), 0, s, g, tm, tn, p.splits, p.steps);
}
template <class T, bool AR, bool BR>
void run16(const ProductArgs& g, const ProductPlan& p, hipStream_t s) {
    if (p.tile == TILE_256) run16<T, AR, BR, 256, 256, 2, 4, 64>(g, p, s);
    else if (p.tile == TILE_128) run16<T, AR, BR, 128, 128, 2, 2, 64>(g, p, s);
    else if (p.tile == TILE_ROWS) run16<T, AR, BR, 128, 256, 2, 4, 32>(g, p, s);
    else run16<T, AR, BR, 64, 64, 2, 2, 64>(g, p, s);
}
template <class T>
void few16(const ProductArgs& g, hipStream_t s) {
    const dim3 grid(cdiv(g.N, 16));
    if (g.gated) {
        if (g.M <= 16) hipLaunchKernelGGL((few_rows16_kernel<T, 8, 1, true>), grid, dim3(512), 0, s, g);
        else hipLaunchKernelGGL((few_rows16_kernel<T, 8, 2, true>), grid, dim3(512), 0, s, g);
        return;
    }
#define FEW16(WAVES, MT) hipLaunchKernelGGL((few_rows16_kernel<T, WAVES, MT>), grid, dim3(64 * WAVES), 0, s, g)
    const bool narrow = g.N <= 4096;
    if (g.M <= 16) { if (narrow) FEW16(8, 1); else FEW16(4, 1); }
    else { if (narrow) FEW16(8, 2); else FEW16(4, 2); }
#undef FEW16
}
template <class T>
void product16(const ProductArgs& g, const ProductPlan& p, hipStream_t s) {
    if (p.tile == TILE_FEW) few16<T>(g, s);
    else if (!g.a_rows && !g.b_rows) run16<T, false, false>(g, p, s);
    else if (!g.a_rows) run16<T, false, true>(g, p, s);
    else run16<T, true, true>(g, p, s);
    if (p.splits > 1) join<T>(g, p, s);
}
template <bool AR, bool BR>
void run32(const ProductArgs& g, const ProductPlan& p, hipStream_t s) {
    if constexpr (!AR && !BR) {
        if (g.gated) {
            const int edge = p.tile == TILE_64 ? 64 : 128, tm = cdiv(g.M, edge), tn = cdiv(g.N, edge / 2);
            if (edge == 64) hipLaunchKernelGGL((product32_kernel<AR, BR, 64, 64, 2, 2, true>), dim3(tm * tn * p.splits), dim3(256), 0, s, g, tm, tn, p.splits, p.steps);
            else hipLaunchKernelGGL((product32_kernel<AR, BR, 128, 128, 2, 2, true>), dim3(tm * tn * p.splits), dim3(256), 0, s, g, tm, tn, p.splits, p.steps);
            return;
        }
    }
    if (p.tile == TILE_64) {
        const int tm = cdiv(g.M, 64), tn = cdiv(g.N, 64);
        hipLaunchKernelGGL((product32_kernel<AR, BR, 64, 64, 2, 2>), dim3(tm * tn * p.splits), dim3(256), 0, s, g, tm, tn, p.splits, p.steps);
    } else {
        const int tm = cdiv(g.M, 128), tn = cdiv(g.N, 128);
        hipLaunchKernelGGL((product32_kernel<AR, BR, 128, 128, 2, 2>), dim3(tm * tn * p.splits), dim3(256), 0, s, g, tm, tn, p.splits, p.steps);
    }
}
void product32(const ProductArgs& g, const ProductPlan& p, hipStream_t s) {
    if (p.tile == TILE_FEW) {
        const dim3 grid(cdiv(g.N, 16));
        if (g.gated && g.M <= 16) hipLaunchKernelGGL((few_rows32_kernel<8, 1, true>), grid, dim3(512), 0, s, g);
        else if (g.gated) hipLaunchKernelGGL((few_rows32_kernel<8, 2, true>), grid, dim3(512), 0, s, g);
        else if (g.M <= 16) hipLaunchKernelGGL((few_rows32_kernel<8, 1>), grid, dim3(512), 0, s, g);
        else hipLaunchKernelGGL((few_rows32_kernel<8, 2>), grid, dim3(512), 0, s, g);
    } else if (!g.a_rows && !g.b_rows) run32<false, false>(g, p, s);
    else if (!g.a_rows) run32<false, true>(g, p, s);
    else run32<true, true>(g, p, s);
    if (p.splits > 1) join<float>(g, p, s);
}

}  // namespace

ProductPlan product_plan(corr_dtype type, int a_rows, int b_rows, int M, int N, int K) {
    const bool wide = type == CORR_TYPE_F32;
    const int bk = wide ? 32 : 64, all = cdiv(K, bk);
    ProductPlan p = {TILE_64, 1, all};
    // Few rows: weights straight into the fragments, no joins.  A workgroup walks along all of k, so that a long k goes to tiles and splits
    // instead (16 x 16384 -> 1024 bf16: 30 us, 11 in tiles; x 1024 -> 1024: 4.4 and 7.1), unless there are columns for every compute unit and
    // the weights' bytes are what counts (1 x 16384 -> 16384 bf16: 110 and 143; 8 x 4096 -> 16384 fp32: 52 and 81).
    const bool few = wide ? K <= 2048 || N >= 4096 : K <= 2048 || (M <= 8 && K <= 4096) || (M <= 16 && (int64_t)N * K >= 1 << 27);
    if (M <= 32 && few && !a_rows && !b_rows) { p.tile = TILE_FEW; return p; }
    int64_t tiles = (int64_t)cdiv(M, 64) * cdiv(N, 64);
    const int64_t t128 = (int64_t)cdiv(M, 128) * cdiv(N, 128), t256 = (int64_t)cdiv(M, 256) * cdiv(N, 256);
    const int64_t trows = (int64_t)cdiv(M, 128) * cdiv(N, 256);
    // Tiles of 128 x 256 in steps of 32 k, 16 waves a compute unit, where there is little to multiply for every element that is stored:
    // 259200 x 128 -> 256: 44 us, 55 in tiles of 256; 32400 x 256 -> 1024 with gelu and preact: 44 and 50; 129600 x 324 -> 256: 45 and 46,
    // with gelu and preact 57 and 62.  Past the memory-side cache (256 MB; a preact is not counted) steps of whole pieces of 64 bytes only, and
    // a shorter k: 518400 x 324 -> 256: 240 us, 200 to 218 in tiles of 256; x 240: 183 and 160; x 352: 202 and 189; x 256: 135 and 141.
    // Tiles of 256 read operands half as often, but one workgroup fills a compute unit: for products that give every unit one, and
    // that do not make them multiply much more (129600 x 384 -> 324: 63 us in tiles of 128, 69 in 256; 259200 x 384 -> 256: 110 and 90).
    // Tiles of 128 if they, or their splits, give 320 workgroups (5704 x 4096 -> 1024 fp16: 58 us, 77 in tiles of 64), else tiles of 64
    // (2048 x 1024 -> 256 fp32: 18 us, 24 in tiles of 128; 2852 x 1024 -> 256 fp16: 12.7 and 14.8).
    // Splits have eight steps or more; joining them costs about 4 us, as much as 16 steps of 16-bit tiles of 64 (2852 x 1024 -> 256: 7.5 us
    // whole, 11.4 in two) or six of fp32.
    const int most = all >= 32 || wide ? max(1, all / 8) : 1;
    const bool large = !wide && t256 >= 256 && t256 * 4 <= t128 * 1.25, cached = (int64_t)M * (K + N) * 2 <= 192 << 20;
    if (!wide && K <= (cached ? 352 : 256) && N > 128 && trows >= 512 && (cached || K % 32 == 0 || !large)) { p.tile = TILE_ROWS; tiles = trows; }
    else if (large) { p.tile = TILE_256; tiles = t256; }
    else if (t128 * max((int64_t)1, min((int64_t)most, 512 / t128)) >= 320) { p.tile = TILE_128; tiles = t128; }
    // workgroups for two (tiles of 64: four) on every compute unit
    const int64_t want = p.tile == TILE_256 ? 256 : p.tile == TILE_64 ? 1024 : 512;
    if (tiles < want / 2) {
        const int splits = (int)min((int64_t)most, want / tiles);
        p.steps = cdiv(all, splits);
        p.splits = cdiv(all, p.steps);
    }
    return p;
}

void product_tile(const ProductPlan& p, int& rows, int& cols) {
    rows = p.tile == TILE_256 ? 256 : p.tile == TILE_64 ? 64 : p.tile == TILE_FEW ? 0 : 128;
    cols = p.tile == TILE_256 || p.tile == TILE_ROWS ? 256 : p.tile == TILE_128 ? 128 : p.tile == TILE_64 ? 64 : 16;
}

namespace {
constexpr int SHORT_FM = 2, SHORT_WAVES = 4, SHORT_ROWS = 16 * SHORT_FM * SHORT_WAVES, SHORT_SLOTS = 512;      // two workgroups a compute unit
// Whole pieces of k, and seven chunks for every workgroup that fits at a time (bf16 with silu and preact, tiles and here: 14570 x 256 -> 2 x 1024 38 and 34 us, 57600 x
// 128 -> 2 x 256 32 and 27; below: 14570 x 256 -> 2 x 384 18 and 22, 8192 x 256 -> 2 x 1024 20 and 22).  An XCD takes every eighth 128 rows, so the rows have to be 16 times that many and
// leave no more than one place idle beside 15 taken ones (k = 256, the same product of rows and columns, here and tiles: 1 x 114688 162 and 29, 1000 x 14336 30 and 26,
// 2048 x 7168 26 and 26, 2500 x 5760 36 and 26, 4096 x 3584 24 and 26, 9300 x 1600 27 and 26, 10000 x 1472 24 and 26).
bool short_rows(const ProductArgs& g) {
    const int64_t tm = cdiv(g.M, SHORT_ROWS);
    return g.gated && g.type != CORR_TYPE_F32 && g.K <= 256 && g.K % 8 == 0 && tm * cdiv(g.N, 32) >= 7 * SHORT_SLOTS && tm >= 16 && 8 * cdiv(tm, 8) * 15 <= 16 * tm;
}
template <class T>
void short_gated(const ProductArgs& g, hipStream_t s) {
    const int tm = cdiv(g.M, SHORT_ROWS), chunks = cdiv(g.N, 32);
    int per = 0;
    int64_t best = INT64_MAX;
    for (int p = 1; p <= min(chunks, 32); ++p) {          // rounds of workgroups, times two chunks at a time and about one for the rows
        const int some = 2 * cdiv(chunks, 2 * p);
        const int64_t cost = ((int64_t)tm * cdiv(chunks, some) + SHORT_SLOTS - 1) / SHORT_SLOTS * (some + 1);
        if (cost < best) { best = cost; per = some; }
    }
    const int parts = cdiv(chunks, per);
    const dim3 grid(8 * cdiv(tm, 8) * parts), threads(64 * SHORT_WAVES);
    if (g.K <= 128) hipLaunchKernelGGL((short_gated_kernel<T, SHORT_FM, SHORT_WAVES, 4>), grid, threads, 0, s, g, tm, parts, per);
    else hipLaunchKernelGGL((short_gated_kernel<T, SHORT_FM, SHORT_WAVES, 8>), grid, threads, 0, s, g, tm, parts, per);
}
}  // namespace

void gated_tile(corr_dtype type, int M, int N, int K, int& rows, int& cols, int& splits) {
    ProductArgs g = {};
    g.type = type; g.gated = 1; g.M = M; g.N = N; g.K = K;
    const ProductPlan p = product_plan(type, 0, 0, M, 2 * N, K);
    product_tile(p, rows, cols);
    splits = p.splits;
    if (short_rows(g)) { rows = SHORT_ROWS; cols = 64; splits = 1; }
}

hipError_t launch_product(const ProductArgs& args, hipStream_t s) {
    ProductArgs g = args;
    const ProductPlan p = product_plan(g.type, g.a_rows, g.b_rows, g.M, g.gated ? 2 * g.N : g.N, g.K);
    // A result larger than half of the memory-side cache goes past the caches, so that the operands stay in them (259200 x 1024 -> 128
    // bf16: 137 -> 119 us); whole lines only (rows of 648 bytes: 43 -> 46 us).
    const int64_t row = g.ldy * corr_elem_bytes(g.type);
    g.past = (int64_t)g.M * row >= (128 << 20) && row % 64 == 0 && ((uintptr_t)g.y & 63) == 0;
    if (short_rows(g)) {
        if (g.type == CORR_TYPE_BF16) short_gated<__bf16>(g, s);
        else short_gated<_Float16>(g, s);
        return hipGetLastError();
    }
    if (g.type == CORR_TYPE_F32) product32(g, p, s);
    else if (g.type == CORR_TYPE_BF16) product16<__bf16>(g, p, s);
    else product16<_Float16>(g, p, s);
    return hipGetLastError();
}

hipError_t launch_pack16(const Pack16& one, const Pack16& two, hipStream_t s) {
    const int64_t total = one.rows * (one.ld_dst / 8) + two.rows * (two.ld_dst / 8);
    if (!total) return hipSuccess;
    const int64_t blocks = (total + 255) / 256;
    hipLaunchKernelGGL(pack16_kernel, dim3((unsigned)(blocks < 1 << 20 ? blocks : 1 << 20)), dim3(256), 0, s, one, two);
    return hipGetLastError();
}

int slope_parts(int64_t M) { return (int)min((int64_t)1024, max((int64_t)1, (M + 31) / 32)); }

namespace {
template <class T, int V>
void slope(int act, const void* dy, int64_t ld_dy, const void* z, void* dz, void* dz_lo, int64_t ld_dz, float* part, int64_t M, int N, hipStream_t s) {
    int ct = 1;
    while (ct < SLOPE_THREADS && ct * V < N) ct *= 2;
    const int parts = slope_parts(M);
    const int64_t per = (M + parts - 1) / parts;
    hipLaunchKernelGGL((slope_kernel<T, V>), dim3(cdiv(N, ct * V), parts), dim3(SLOPE_THREADS), 0, s, act, (const T*)dy, ld_dy, (const T*)z,
                       (T*)dz, (T*)dz_lo, ld_dz, part, M, N, ct, per);
}
}  // namespace

hipError_t launch_slope(corr_dtype t, int act, const void* dy, int64_t ld_dy, const void* z, void* dz, void* dz_lo, int64_t ld_dz,
                        float* part, int64_t M, int N, hipStream_t s) {
    if (t == CORR_TYPE_F32) slope<float, 4>(act, dy, ld_dy, z, dz, dz_lo, ld_dz, part, M, N, s);
    else if (t == CORR_TYPE_BF16) slope<__bf16, 8>(act, dy, ld_dy, z, dz, dz_lo, ld_dz, part, M, N, s);
    else slope<_Float16, 8>(act, dy, ld_dy, z, dz, dz_lo, ld_dz, part, M, N, s);
    return hipGetLastError();
}

namespace {
template <class T, int V>
void slope_gated(int act, const void* dy, int64_t ld_dy, const void* z, void* dz, void* dz_lo, int64_t ld_dz, float* part, int64_t M, int N, hipStream_t s) {
    int ct = 1;
    while (ct < SLOPE_THREADS && ct * V < N) ct *= 2;
    const int parts = slope_parts(M);
    hipLaunchKernelGGL((slope_gated_kernel<T, V>), dim3(cdiv(N, ct * V), parts), dim3(SLOPE_THREADS), 0, s, act, (const T*)dy, ld_dy, (const T*)z,
                       (T*)dz, (T*)dz_lo, ld_dz, part, M, N, ct, (M + parts - 1) / parts);
}
}  // namespace

hipError_t launch_slope_gated(corr_dtype t, int act, const void* dy, int64_t ld_dy, const void* z, void* dz, void* dz_lo, int64_t ld_dz,
                              float* part, int64_t M, int N, hipStream_t s) {
    if (t == CORR_TYPE_F32) slope_gated<float, 4>(act, dy, ld_dy, z, dz, dz_lo, ld_dz, part, M, N, s);
    else if (t == CORR_TYPE_BF16) slope_gated<__bf16, 8>(act, dy, ld_dy, z, dz, dz_lo, ld_dz, part, M, N, s);
    else slope_gated<_Float16, 8>(act, dy, ld_dy, z, dz, dz_lo, ld_dz, part, M, N, s);
    return hipGetLastError();
}
