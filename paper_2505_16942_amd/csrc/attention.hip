// Attention of one map's rows to another's: o = softmax(scale q k^T) v per head, and its gradient.  Compiled once per type
// (CORR_ATTENTION_TYPE: 0 fp32, 1 bf16, 2 fp16).
#include <type_traits>
#include "matrix.h"
#include "attention.h"

namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.69314718055994531f;
constexpr unsigned PAST = 0x80000000u;      // an offset past every resource's end: the load into LDS writes zeros
constexpr unsigned RANGE = 0x7ffffff0u;
inline int cdiv(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// ---- how products are made.  A fragment is one matrix instruction's operand: 32 k, lane (lr, lg) = (lane & 15, lane >> 4) holds row lr and 8 of them.
// `straight`: a tile's row, along the row.  `turned`: one of its columns, along 32 of its rows; these are taken in the order in which a product's result
// lies in its lanes (rows 4 lg + e and 16 + 4 lg + e), so that the scores are the next product's operand without leaving their lanes.  Tiles lie in
// LDS in rows of DP 16-bit elements, 16-byte piece p of row r at slot(r, p), which spreads both kinds of read over the banks.
// (LDS has 256 bytes of banks.  A 16-byte read serves lanes 0-3, 12-15, 20-27 at a time, and so on; the transposing one 32 neighbours: from 128 elements
// on rows r and 12 + r (4 + r and 8 + r), r < 4, have neighbouring pieces.)
template <int DP> __device__ __forceinline__ int slot(int row, int piece) {
    return piece ^ (DP == 32 ? row >> 1 & 3 : DP == 64 ? row & 7 : ((row ^ (row >> 1 & 4)) & 7) << 1 | (row >> 3 & 1));
}
template <class F, int DP> __device__ __forceinline__ F read_straight(lds_byte* tile, int row, int t, int lg) {
    return *(__attribute__((address_space(3))) F*)(tile + row * 2 * DP + slot<DP>(row, 4 * t + lg) * 16);
}
template <class F, int DP> __device__ __forceinline__ F read_turned(lds_byte* tile, int row0, int db, int lr, int lg) {
    const int r = row0 + 4 * lg + (lr >> 2), piece = 2 * db + ((lr & 3) >> 1);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(tile + r * 2 * DP + slot<DP>(r, piece) * 16 + (lr & 1) * 8));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(tile + (r + 16) * 2 * DP + slot<DP>(r + 16, piece) * 16 + (lr & 1) * 8));
    return __builtin_bit_cast(F, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}
constexpr int FK = 32;
template <class T> struct Num {
    typedef typename Frag<T>::type F;
    template <int DP, int ROWS> static __device__ __forceinline__ F straight(lds_byte* tile, int row, int t, int lg) { return read_straight<F, DP>(tile, row, t, lg); }
    template <int DP, int ROWS> static __device__ __forceinline__ F turned(lds_byte* tile, int row0, int db, int lr, int lg) {
        return read_turned<F, DP>(tile, row0, db, lr, lg);
    }
    static __device__ __forceinline__ F pack(const f32x4* x) {
        F f;
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = (T)x[e >> 2][e & 3];
        return f;
    }
    // what pack() left out
    static __device__ __forceinline__ F rest(const f32x4* x, const F& high) {
        F f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float r = x[e >> 2][e & 3] - (float)high[e];
            f[e] = (T)(fabsf(r) < INFINITY ? r : 0.f);
        }
        return f;
    }
    // Weights, none of which is negative, in two parts: rounded towards zero, and what that left out and a trace more, so that an infinity of the other
    // operand is multiplied by two parts above zero and stays one.
    static __device__ __forceinline__ F pack_under(const f32x4* x) {
        if constexpr (std::is_same<T, __bf16>::value) {
            u32x4 u;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                u[e] = __float_as_uint(x[e >> 1][2 * (e & 1)]) >> 16 | (__float_as_uint(x[e >> 1][2 * (e & 1) + 1]) & 0xffff0000u);
            return __builtin_bit_cast(F, u);
        } else {
            u32x4 u;
#pragma unroll
            for (int e = 0; e < 4; ++e) u[e] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_pkrtz(x[e >> 1][2 * (e & 1)], x[e >> 1][2 * (e & 1) + 1]));
            return __builtin_bit_cast(F, u);
        }
    }
    static __device__ __forceinline__ F rest_over(const f32x4* x, const F& high) {
        F f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float w = x[e >> 2][e & 3], r = w - (float)high[e];
            f[e] = (T)(std::is_same<T, __bf16>::value ? fmaf(w, 0x1p-30f, r) : r + fminf(w, 0x1p-24f));
        }
        return f;
    }
    static __device__ __forceinline__ f32x4 times(const F& a, const F& b, f32x4 c) { return mma(a, b, c); }
    // the transposed product, bit by bit what times(b, a) makes
    static __device__ __forceinline__ f32x4 times_back(const F& a, const F& b, f32x4 c) { return mma(a, b, c); }
    // elements d .. d + 7 of row `p`, zeros behind D or without a row
    static __device__ __forceinline__ F load(const T* p, int d, int D, bool there) {
        F f = {};
        if (there && d < D) f = *reinterpret_cast<const typename Some<T, 8>::type*>(p + d);
        return f;
    }
};
// fp32: three bf16 parts an element and the six of nine partial products that reach 2^-24, as in the row operators' products: 2.7 times the rate of
// the fp32 instruction.  A tile is three planes.
struct Parts { bf16x8 p[3]; };
__device__ __forceinline__ void split4(f32x4 x, u32x2 (&parts)[3]) {
    f32x2 lo = {x[0], x[1]}, hi = {x[2], x[3]};
#pragma unroll
    for (int p = 0; p < 3; ++p) {
        const bf16x2 cl = __builtin_convertvector(lo, bf16x2), ch = __builtin_convertvector(hi, bf16x2);
        parts[p] = u32x2{__builtin_bit_cast(unsigned, cl), __builtin_bit_cast(unsigned, ch)};
        if (p < 2) {
            lo -= __builtin_convertvector(cl, f32x2);
            hi -= __builtin_convertvector(ch, f32x2);
        }
    }
}
template <> struct Num<float> {
    typedef Parts F;
    template <int DP, int ROWS> static __device__ __forceinline__ F straight(lds_byte* tile, int row, int t, int lg) {
        F f;
#pragma unroll
        for (int p = 0; p < 3; ++p) f.p[p] = read_straight<bf16x8, DP>(tile + p * ROWS * 2 * DP, row, t, lg);
        return f;
    }
    template <int DP, int ROWS> static __device__ __forceinline__ F turned(lds_byte* tile, int row0, int db, int lr, int lg) {
        F f;
#pragma unroll
        for (int p = 0; p < 3; ++p) f.p[p] = read_turned<bf16x8, DP>(tile + p * ROWS * 2 * DP, row0, db, lr, lg);
        return f;
    }
    static __device__ __forceinline__ F pack(const f32x4* x) {
        u32x2 one[3], two[3];
        split4(x[0], one);
        split4(x[1], two);
        F f;
#pragma unroll
        for (int p = 0; p < 3; ++p) f.p[p] = __builtin_bit_cast(bf16x8, u32x4{one[p][0], one[p][1], two[p][0], two[p][1]});
        return f;
    }
    static __device__ __forceinline__ f32x4 times(const F& a, const F& b, f32x4 c) {
        constexpr int QA[6] = {2, 0, 1, 1, 0, 0}, QB[6] = {0, 2, 1, 0, 1, 0};      // small products first
#pragma unroll
        for (int q = 0; q < 6; ++q) c = mma(a.p[QA[q]], b.p[QB[q]], c);
        return c;
    }
    static __device__ __forceinline__ f32x4 times_back(const F& a, const F& b, f32x4 c) {
        constexpr int QA[6] = {0, 2, 1, 0, 1, 0}, QB[6] = {2, 0, 1, 1, 0, 0};
#pragma unroll
        for (int q = 0; q < 6; ++q) c = mma(a.p[QA[q]], b.p[QB[q]], c);
        return c;
    }
    static __device__ __forceinline__ F load(const float* p, int d, int D, bool there) {
        f32x4 x[2] = {};
        if (there && d < D) {
            x[0] = *reinterpret_cast<const Some<float, 4>::type*>(p + d);
            x[1] = *reinterpret_cast<const Some<float, 4>::type*>(p + d + 4);
        }
        return pack(x);
    }
};
// fp32 whose tiles come from three planes that were made before (split_kernel): they land in LDS by themselves, as 16-bit ones do.
struct Planes;
template <> struct Num<Planes> : Num<float> {};
template <class T> struct Elem { typedef T type; };
template <> struct Elem<Planes> { typedef float type; };
template <class T> constexpr bool F32 = std::is_same<typename Elem<T>::type, float>::value;
// Weights as a product's operand.  fp16's normal values begin at 6e-5, below which a softmax over many keys lies: they are held 2^14 times as
// large (at most 2^(14 + SLACK)), and the results divided by that.
template <class T> constexpr float LIFT = std::is_same<T, _Float16>::value ? 14.f : 0.f;

// The sums are rescaled only when a score passes the reference by more than 2^SLACK, which their types hold: fp16 up to 2^(14 + 1.75), the others as they
// like.  Of a wave's 32 rows some row's largest score grows in nearly every second of 200 tiles.
template <class T> constexpr float SLACK = std::is_same<T, _Float16>::value ? 1.75f : 8.f;

// Scores far from zero.  The exponent s c - m c is one rounding of the exact product less a rounded m c.  That rounding is common to the row and divides out,
// but it grows with m: past 2^21 it takes the quarter of a bit that fp16 has left above SLACK, past 2^31 fp32's range.  A workgroup with a row of |m c|
// above FAR (a rounding of 2^-8) walks over its keys once more with the exponent (s - m) c, m its largest score.  In the one walk that others need, a
// subtraction under a condition took 50 registers more and a workgroup of three from each compute unit.  (2 x 14400 x 14400 x 2 x 64 bf16 with all rows far: 290 ->
// 515 us; the gradient's rows 379 -> 427, keys 522 -> 668.)
constexpr float FAR = 65536.f;
// The gradient's P = e^(s - lse) has what lse log2 e is rounded by.  Workgroups with a row of |lse| from FAR_LSE on (1e-5 there) take the difference before the
// factor, of s scale rounded as the forward pass rounds it into lse, so that a key which has all of a row's weight has 1.  What is left is lse's own rounding.
constexpr float FAR_LSE = 256.f;
__device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.f : m; }
// x scale - y in two roundings
__device__ __forceinline__ float less(float x, float scale, float y) {
#pragma clang fp contract(off)
    const float p = x * scale;
    return p - y;
}
// a score's weight: `low` is the row's lse log2 e - LIFT, where far its lse
template <class T, bool FAR_ROWS> __device__ __forceinline__ float power(float s, float scale, float c, float low) {
    if constexpr (!FAR_ROWS) return __builtin_amdgcn_exp2f(fmaf(s, c, -low));
    const float x = less(s, scale, low);
    return __builtin_amdgcn_exp2f(fmaf(x > 0.f ? 0.f : x, LOG2E, LIFT<T>));
}

// rows (keys) of a tile in LDS: 64, or 32 for longer heads: from 64 elements on for one wave and for fp32's planes, from 128 on for fp32, at 256 for the rest
template <class T, int DP, int WAVES> constexpr int tile_rows() {
    return DP <= (WAVES == 1 || std::is_same<T, Planes>::value ? 32 : std::is_same<T, float>::value ? 64 : 128) ? 64 : 32;
}

// the largest (sum) over the four lanes that share lane & 15
struct Both { float one, two; };
__device__ __forceinline__ Both swap16(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return {__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ __forceinline__ Both swap32(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return {__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ __forceinline__ float lanes_max(float x) {
    const Both a = swap16(x), b = swap32(fmaxf(a.one, a.two));
    return fmaxf(b.one, b.two);
}
__device__ __forceinline__ float lanes_sum(float x) {
    const Both a = swap16(x), b = swap32(a.one + a.two);
    return b.one + b.two;
}

// ---- tiles
// A tile of ROWS rows of a strided array, D of DP elements each, on its way into LDS: `ask` starts it, `land` brings what was asked for to its place
// (one call of the workgroup for both tiles).  16 bits: straight into LDS, in one of two places that take turns.
__device__ __forceinline__ i32x4 resource(const void* p) {
    const uint64_t u = (uint64_t)p;
    return i32x4{__builtin_amdgcn_readfirstlane((int)u), __builtin_amdgcn_readfirstlane((int)(u >> 32) & 0xffff), (int)RANGE, 0x00020000};
}
template <class T, int DP, int ROWS, int WAVES>
struct Tile {
    static constexpr int BYTES = ROWS * DP * 2, PLACES = 2, PIECES = BYTES / (1024 * WAVES);
    static_assert(BYTES % (1024 * WAVES) == 0 && PIECES > 0, "whole loads of 1024 bytes for every wave");
    int row[PIECES];
    unsigned col[PIECES];                    // byte offset inside the row, or PAST behind its end
    __device__ __forceinline__ void plan(int wave, int lane, int D) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int at = (i * WAVES + wave) * 1024 + lane * 16;
            row[i] = at / (DP * 2);
            const int piece = slot<DP>(row[i], at / 16 % (DP / 8));         // an involution
            col[i] = piece * 8 < D ? piece * 16 : PAST;
        }
    }
    // offset(row): the byte offset of a row from p on, PAST if it does not count
    template <class O> __device__ __forceinline__ void ask(const T* p, unsigned lds, int wave, O offset) {
        const i32x4 rsrc = resource(p);
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const unsigned at = offset(row[i]);
            dma16(rsrc, lds + (i * WAVES + wave) * 1024, at == PAST || col[i] == PAST ? PAST : at + col[i]);
        }
    }
};
// fp32: through registers, where an element's three parts are made; one place.
template <int DP, int ROWS, int WAVES>
struct Tile<float, DP, ROWS, WAVES> {
    static constexpr int PLANE = ROWS * DP * 2, BYTES = 3 * PLANE, PLACES = 1, PIECES = ROWS * DP / (256 * WAVES);
    f32x4 x[PIECES];
    int lane_, D_;
    __device__ __forceinline__ void plan(int wave, int lane, int D) { lane_ = wave * 64 + lane; D_ = D; }
    template <class O> __device__ __forceinline__ void ask(const float* p, unsigned, int, O offset) {
        const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(p), 0, (int)RANGE, 0x00020000);
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int at = i * WAVES * 64 + lane_, row = at / (DP / 4), d = at % (DP / 4) * 4;
            const unsigned to = offset(row);
            x[i] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, (int)(to == PAST || d >= D_ ? PAST : to + d * 4), 0, 0));
        }
    }
    __device__ __forceinline__ void store(unsigned char* tile) const {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int at = i * WAVES * 64 + lane_, row = at / (DP / 4), d = at % (DP / 4) * 4;
            u32x2 parts[3];
            split4(x[i], parts);
#pragma unroll
            for (int q = 0; q < 3; ++q)
                *reinterpret_cast<u32x2*>(tile + q * PLANE + row * 2 * DP + slot<DP>(row, d >> 3) * 16 + (d & 4) * 2) = parts[q];
        }
    }
};
// Planes: two places where they are 24 KB together, else one, whose loads start when the last tiles have been read.
template <int DP, int ROWS, int WAVES>
struct Tile<Planes, DP, ROWS, WAVES> : Tile<__bf16, DP, ROWS, WAVES> {
    typedef Tile<__bf16, DP, ROWS, WAVES> Plane;
    static constexpr int BYTES = 3 * Plane::BYTES, PLACES = BYTES <= 12288 ? 2 : 1;
    template <class O> __device__ __forceinline__ void ask(const __bf16* p, int64_t plane, unsigned lds, int wave, O offset) {
#pragma unroll
        for (int q = 0; q < 3; ++q) Plane::ask(p + q * plane, lds + q * Plane::BYTES, wave, offset);
    }
};
template <class L> struct Late { static constexpr bool value = false; };
template <int DP, int ROWS, int WAVES> struct Late<Tile<Planes, DP, ROWS, WAVES>> { static constexpr bool value = Tile<Planes, DP, ROWS, WAVES>::PLACES == 1; };

template <class L> __device__ __forceinline__ void land(const L& one, const L& two, unsigned char* smem) {
    if constexpr (L::PLACES == 2 || Late<L>::value) arrive_all();
    else {
        __syncthreads();                                 // the last tiles have been read
        one.store(smem);
        two.store(smem + L::BYTES);
        __syncthreads();
    }
}
// Which keys of a tile count: those before the item's length (and the share's end) whose mask byte is not zero.
struct Keys {
    const uint8_t* mask;                     // of this item, or null
    int end;
    __device__ __forceinline__ unsigned byte(int k0, int lane) const { return mask && k0 + lane < end ? mask[k0 + lane] : 0u; }
    __device__ __forceinline__ uint64_t bits(int k0, int n, unsigned byte) const {
        const int left = min(end - k0, n);
        uint64_t w = left <= 0 ? 0 : ~0ull >> (64 - left);
        if (mask) w &= __ballot(byte != 0);
        return w;
    }
};
template <class T> __device__ __forceinline__ Keys keys_of(const AttentionArgs& a, int b) {
    Keys k;
    k.end = a.Lk;
    if (a.k_lengths) k.end = max(0, min(a.Lk, __builtin_amdgcn_readfirstlane(a.k_lengths[b])));
    k.mask = a.key_mask ? a.key_mask + (int64_t)b * a.Lk : nullptr;
    return k;
}
// Tiles of a head follow each other, and so meet its keys at about the same time on every XCD.  Runs of a head's tiles on one XCD would leave XCDs
// idle whose items are short.
struct Place { int b, hk, bh, tile, split; };
// Rows of one head of k or v from some key on: of the caller's array, or of the planes.
template <class T> struct Source {
    const T* p; int64_t row;
    template <class L> __device__ __forceinline__ void ask(L& load, int first, unsigned to, int wave, uint64_t bits) const {
        const unsigned step = (unsigned)(row * (int)sizeof(T));
        load.ask(p + first * row, to, wave, [&](int r) { return (bits >> r) & 1 ? r * step : PAST; });
    }
};
template <> struct Source<Planes> {
    const __bf16* p; int64_t row, plane;
    template <class L> __device__ __forceinline__ void ask(L& load, int first, unsigned to, int wave, uint64_t bits) const {
        const unsigned step = (unsigned)(row * 2);
        load.ask(p + first * row, plane, to, wave, [&](int r) { return (bits >> r) & 1 ? r * step : PAST; });
    }
};
template <class T>
__device__ __forceinline__ Source<T> source(const void* p, const void* planes, int64_t item, int64_t row, int64_t head, const AttentionArgs& a, const Place& at, int first) {
    if constexpr (std::is_same<T, Planes>::value) {
        const int64_t dense = (int64_t)a.HK * a.D;
        return {(const __bf16*)planes + ((int64_t)at.b * a.Lk + first) * dense + at.hk * a.D, dense, a.B * a.Lk * dense};
    } else return {(const T*)p + at.b * item + at.hk * head + first * row, row};
}
__device__ __forceinline__ Place place_of(const AttentionArgs& a, int tiles, int splits) {
    const int n = blockIdx.x;
    Place p;
    p.tile = n % tiles;
    const int m = n / tiles;
    p.split = m % splits;
    p.bh = m / splits;
    p.b = p.bh / a.HK;
    p.hk = p.bh - p.b * a.HK;
    return p;
}
__device__ __forceinline__ void query_of(const AttentionArgs& a, int r, int& q, int& g) {
    q = a.per == 1 ? r : (int)((unsigned)r / (unsigned)a.per);
    g = r - q * a.per;
}

// ---- forward.  One pass over the keys with a running reference m (the largest score, or a little less) and sum l of each row: o = sum e^(s - m) v / sum
// e^(s - m), rescaled when m moves.  S^T = K Q^T in tiles of 16 keys x 16 rows: a lane has four keys of one row, so that a row's maximum is a lane's own and
// two exchanges away, and the weights are the operand of O^T = V^T P^T as they lie.  Weights are rounded once to the operands' type (their sum is
// not): the matrix cores take them so, and it makes the result's error sqrt 2 times its own rounding's (bf16: 2.3e-3 in the 2-norm, 1.7e-3).
// Four waves of 16 QB rows share tiles of keys and values that land in LDS while the last ones are multiplied.  With two blocks a wave a fragment that
// is read once is multiplied twice.  1 x 32400 x 32400, 2 heads of 128, bf16: 1090 us, 985 TFLOP/s, matrix instructions in 40 % of the cycles, the vector unit (an
// exponential, fma, maximum, sum and half a rounding an element) in most others: a wave's two kinds of work alternate, and a compute unit holds
// eight waves.  2 x 14400 x 14400, 2 heads of 64: 282 us, 750 TFLOP/s: the vector unit, about 80 % of the cycles with
// the exponentials' turns.  fp32's six products: 2 x 2852 x 7285, 4 heads of
// 64: 232 us, 183 TFLOP/s (1.1 PFLOP/s of bf16).
// One row of 8 query heads on 2 key heads, 8 x 32768 keys of ragged lengths (157 MB), bf16, one wave a workgroup, 74 shares: 38 us from memory, 4.1 TB/s
// (28 from the memory-side cache), and 8 for their join; 110 or 172 shares make no difference.
template <class T, int DP, int WAVES, int QB, bool TWO = false>
__global__ __launch_bounds__(64 * WAVES, WAVES == 1 || (DP == 256 && F32<T>) ? 1 : 2) void forward_kernel(AttentionArgs a, int tiles, int splits, int share) {
    typedef Num<T> N;
    typedef typename Elem<T>::type E;
    typedef typename N::F F;
    constexpr int KT = tile_rows<T, DP, WAVES>(), KB = KT / 16, CH = DP / FK, DB = DP / 16;
    typedef Tile<T, DP, KT, WAVES> Load;
    __shared__ __align__(1024) unsigned char smem[2 * Load::PLACES * Load::BYTES];
    lds_byte* const lds = (lds_byte*)smem;
    const unsigned lds_at = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)lds);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lr = lane & 15, lg = lane >> 4;
    const Place at = place_of(a, tiles, splits);
    Keys keys = keys_of<T>(a, at.b);
    const int k_lo = at.split * share;
    keys.end = min(keys.end, k_lo + share);
    const int steps = keys.end > k_lo ? (keys.end - k_lo + KT - 1) / KT : 0;
    const Source<T> from_k = source<T>(a.k, a.k3, a.k_item, a.k_row, a.k_head, a, at, k_lo), from_v = source<T>(a.v, a.v3, a.v_item, a.v_row, a.v_head, a, at, k_lo);
    const int r0 = (at.tile * WAVES + wave) * 16 * QB;
    F fq[QB][CH];
#pragma unroll
    for (int j = 0; j < QB; ++j) {
        const int r = r0 + 16 * j + lr;
        int q, g;
        query_of(a, r, q, g);
        const E* p = (const E*)a.q + at.b * a.q_item + (at.hk * a.per + g) * a.q_head + q * a.q_row;
#pragma unroll
        for (int t = 0; t < CH; ++t) fq[j][t] = N::load(p, t * FK + lg * 8, a.D, r < a.rows);
    }
    Load load_k, load_v;
    load_k.plan(wave, lane, a.D);
    load_v.plan(wave, lane, a.D);
    auto ask = [&](int t, uint64_t bits) {
        const unsigned to = lds_at + t % Load::PLACES * 2 * Load::BYTES;
        from_k.ask(load_k, t * KT, to, wave, bits);
        from_v.ask(load_v, t * KT, to + Load::BYTES, wave, bits);
    };
    const float c = a.scale * LOG2E;
    float slack = SLACK<T> / c;
    f32x4 o[DB][QB] = {};
    // a weight is 2^(s c + k), in the second walk 2^((s - m) c + LIFT)
    float m[QB], k[QB], l[QB];
    bool far = false;
#pragma unroll
    for (int j = 0; j < QB; ++j) { m[j] = -INFINITY; k[j] = LIFT<T>; l[j] = 0.f; }
    // FROM_M: m is known
    auto walk = [&](auto from_m) {
        constexpr bool FROM_M = decltype(from_m)::value;
        uint64_t bits = 0;
        unsigned byte = 0;
        if (steps) {
            bits = keys.bits(k_lo, KT, keys.byte(k_lo, lane));
            if (bits && !Late<Load>::value) ask(0, bits);
            byte = keys.byte(k_lo + KT, lane);
        }
        for (int t = 0; t < steps; ++t) {
            if constexpr (Late<Load>::value) {
                __syncthreads();
                if (bits) ask(t, bits);
            }
            land(load_k, load_v, smem);
            uint64_t next = 0;
            if (t + 1 < steps) {
                next = keys.bits(k_lo + (t + 1) * KT, KT, byte);
                if (next && !Late<Load>::value) ask(t + 1, next);
                byte = keys.byte(k_lo + (t + 2) * KT, lane);
            }
            if (bits) {
                lds_byte* const tk = lds + t % Load::PLACES * 2 * Load::BYTES;
                lds_byte* const tv = tk + Load::BYTES;
                f32x4 s[QB][KB] = {};
#pragma unroll
                for (int h = 0; h < CH; ++h)
#pragma unroll
                    for (int i = 0; i < KB; ++i) {
                        const F f = N::template straight<DP, KT>(tk, 16 * i + lr, h, lg);
#pragma unroll
                        for (int j = 0; j < QB; ++j) s[j][i] = N::times(f, fq[j][h], s[j][i]);
                    }
                if (bits != ~0ull >> (64 - KT)) {
                    const uint64_t mine = bits >> (4 * lg);
#pragma unroll
                    for (int i = 0; i < KB; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
#pragma unroll
                            for (int j = 0; j < QB; ++j) s[j][i][e] = (mine >> (16 * i + e)) & 1 ? s[j][i][e] : -INFINITY;
                }
                if constexpr (!FROM_M) {
                    bool grew = false;
                    float top[QB];
#pragma unroll
                    for (int j = 0; j < QB; ++j) {
                        float x = s[j][0][0];
#pragma unroll
                        for (int i = 0; i < KB; ++i)
#pragma unroll
                            for (int e = 0; e < 4; ++e) x = fmaxf(x, s[j][i][e]);
                        top[j] = lanes_max(x);
                        grew |= top[j] - m[j] > slack;
                    }
                    if (__any(grew)) {
                        bool past = false;
#pragma unroll
                        for (int j = 0; j < QB; ++j) {
                            const bool first = m[j] == -INFINITY;
                            m[j] = fmaxf(m[j], top[j]);
                            const float now = fmaf(-reference(m[j]), c, LIFT<T>), by = first ? 0.f : __builtin_amdgcn_exp2f(now - k[j]);
                            k[j] = now;
                            past |= !(fabsf(now) <= FAR) && m[j] < INFINITY;       // an infinite score is NaN either way
                            l[j] *= by;
#pragma unroll
                            for (int d = 0; d < DB; ++d) o[d][j] *= by;
                        }
                        if (__any(past)) { far = true; slack = 0.f; }
                    }
                }
#pragma unroll
                for (int j = 0; j < QB; ++j)
#pragma unroll
                    for (int i = 0; i < KB; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            s[j][i][e] = __builtin_amdgcn_exp2f(FROM_M ? fmaf(s[j][i][e] - reference(m[j]), c, LIFT<T>) : fmaf(s[j][i][e], c, k[j]));
                            l[j] += s[j][i][e];
                        }
#pragma unroll
                for (int i = 0; i < KB; i += 2) {
                    F fp[QB], lp[QB];
#pragma unroll
                    for (int j = 0; j < QB; ++j) {
                        if constexpr (TWO) {
                            fp[j] = N::pack_under(&s[j][i]);
                            lp[j] = N::rest_over(&s[j][i], fp[j]);
                        } else fp[j] = N::pack(&s[j][i]);
                    }
#pragma unroll
                    for (int d = 0; d < DB; ++d) {
                        const F f = N::template turned<DP, KT>(tv, 16 * i, d, lr, lg);
#pragma unroll
                        for (int j = 0; j < QB; ++j) {
                            if constexpr (TWO) o[d][j] = N::times(f, lp[j], o[d][j]);
                            o[d][j] = N::times(f, fp[j], o[d][j]);
                        }
                    }
                }
            }
            bits = next;
        }
    };
    walk(std::false_type{});
    if (__syncthreads_or(far)) {
        far = true;
#pragma unroll
        for (int j = 0; j < QB; ++j) {
            l[j] = 0.f;
#pragma unroll
            for (int d = 0; d < DB; ++d) o[d][j] = f32x4{};
        }
        walk(std::true_type{});
    }
#pragma unroll
    for (int j = 0; j < QB; ++j) {
        const float sum = lanes_sum(l[j]);
        const int r = r0 + 16 * j + lr;
        if (r >= a.rows) continue;
        int q, g;
        query_of(a, r, q, g);
        const int head = at.hk * a.per + g;
        const float ref = reference(m[j]), lift = far ? LIFT<T> : fmaf(ref, c, k[j]);       // the power of two that weights at the reference have
        if (splits > 1) {
            const float by = __builtin_amdgcn_exp2f(-lift);
            const int64_t row = ((int64_t)at.split * a.B * a.HK + at.bh) * a.rows + r;
#pragma unroll
            for (int d = 0; d < DB; ++d)
                if (16 * d + 4 * lg < a.D) *reinterpret_cast<f32x4*>(a.part_o + row * a.D + 16 * d + 4 * lg) = o[d][j] * by;
            if (lg == 0) { a.part_ml[2 * row] = ref; a.part_ml[2 * row + 1] = sum * by; }
            continue;
        }
        const float by = sum == 0.f ? 0.f : 1.f / sum;
        E* const p = (E*)a.out + (((int64_t)at.b * a.Lq + q) * a.HK * a.per + head) * a.D;
#pragma unroll
        for (int d = 0; d < DB; ++d) {
            const float v[4] = {o[d][j][0] * by, o[d][j][1] * by, o[d][j][2] * by, o[d][j][3] * by};
            if (16 * d + 4 * lg < a.D) store_some<E, 4>(p + 16 * d + 4 * lg, v, 4);
        }
        if (a.lse && lg == 0)
            a.lse[((int64_t)at.b * a.HK * a.per + head) * a.Lq + q] = sum == 0.f ? -INFINITY : less(ref, a.scale, (lift - log2f(sum)) * LN2);
    }
}

// The splits' sums of a row, brought to one reference.  `across` threads have four elements each; `shares` of them take turns at the splits, in a
// fixed order.
template <class T, int THREADS>
__global__ __launch_bounds__(THREADS) void forward_join_kernel(AttentionArgs a, int splits, int across, int shares) {
    __shared__ f32x4 sums[THREADS];
    __shared__ float tops[THREADS], totals[THREADS];
    const int tid = threadIdx.x, team = across * shares, lane = tid % across, share = tid / across % shares, d = 4 * lane;
    const int64_t all = (int64_t)a.B * a.HK * a.rows, row = (int64_t)blockIdx.x * (THREADS / team) + tid / team;
    const float c = a.scale * LOG2E;
    float top = -INFINITY, sum = 0.f;
    f32x4 x = {};
    if (row < all && d < a.D) {
        const float* ml = a.part_ml + 2 * (share * all + row);
        const float* o = a.part_o + (share * all + row) * a.D + d;
#pragma unroll 4
        for (int s = share; s < splits; s += shares, ml += 2 * shares * all, o += shares * all * a.D) {
            const float m = ml[0], l = ml[1];
            const f32x4 v = *reinterpret_cast<const f32x4*>(o);
            if (l == 0.f) continue;
            const float now = fmaxf(top, m), was = __builtin_amdgcn_exp2f((top - now) * c), is = __builtin_amdgcn_exp2f((m - now) * c);
            sum = sum * was + l * is;
            x = x * was + v * is;
            top = now;
        }
    }
    if (shares > 1) {
        tops[tid] = top; totals[tid] = sum; sums[tid] = x;
        __syncthreads();
        if (share) return;
        for (int i = 1; i < shares; ++i) {
            const int other = tid + i * across;
            if (totals[other] == 0.f) continue;
            const float now = fmaxf(top, tops[other]), was = __builtin_amdgcn_exp2f((top - now) * c), is = __builtin_amdgcn_exp2f((tops[other] - now) * c);
            sum = sum * was + totals[other] * is;
            x = x * was + sums[other] * is;
            top = now;
        }
    }
    if (row >= all || d >= a.D) return;
    const int bh = (int)(row / a.rows), r = (int)(row - (int64_t)bh * a.rows), b = bh / a.HK, hk = bh - b * a.HK;
    int q, g;
    query_of(a, r, q, g);
    const int head = hk * a.per + g;
    const float by = sum == 0.f ? 0.f : 1.f / sum;
    const float v[4] = {x[0] * by, x[1] * by, x[2] * by, x[3] * by};
    store_some<T, 4>((T*)a.out + (((int64_t)b * a.Lq + q) * a.HK * a.per + head) * a.D + d, v, 4);
    if (a.lse && lane == 0) a.lse[((int64_t)b * a.HK * a.per + head) * a.Lq + q] = sum == 0.f ? -INFINITY : less(top, a.scale, -log2f(sum) * LN2);
}

// ---- gradient.  With P = exp(s - lse) and delta = sum over d of d_out out: dV = P^T dO, dS = P (dO V^T - delta), dQ = scale dS K,
// dK = scale dS^T Q.  Rows' sums meet in one workgroup and keys' sums in another, so scores are computed twice (seven products for five) and nothing
// is added by atomics: the same bits on every call.  2 x 14400 x 14400, 2 heads of 64, bf16: rows 378 us, keys 522 (seven products: 830 TFLOP/s), matrix
// instructions in a third of the cycles, the vector unit in six tenths; in fp16 460 and 618, with the powers of two of dS.
// delta, and lse in powers of two (less LIFT: the weights are 2^LIFT times as large), in the order of rows; rows behind the last have a weight of zero.  A far
// row has 2 lse there, which is larger than any of the others.
template <class T>
__global__ __launch_bounds__(256) void delta_kernel(AttentionArgs a, int aux_rows) {
    const int lane = threadIdx.x & 15;
    const int64_t all = (int64_t)a.B * a.HK * aux_rows;
    for (int64_t row = (int64_t)blockIdx.x * 16 + threadIdx.x / 16; row < all; row += (int64_t)gridDim.x * 16) {      // 16 lanes a row
        const int bh = (int)(row / aux_rows), r = (int)(row - (int64_t)bh * aux_rows), b = bh / a.HK, hk = bh - b * a.HK;
        float sum = 0.f, low = INFINITY;
        if (r < a.rows) {
            int q, g;
            query_of(a, r, q, g);
            const int head = hk * a.per + g;
            const int64_t at = (((int64_t)b * a.Lq + q) * a.HK * a.per + head) * a.D;
            for (int d = 8 * lane; d < a.D; d += 128) {
                float x[8], y[8];
                load_some<T, 8>((const T*)a.o + at + d, x, 8);
                load_some<T, 8>((const T*)a.d_out + at + d, y, 8);
#pragma unroll
                for (int e = 0; e < 8; ++e) sum = fmaf(x[e], y[e], sum);
            }
            const float lse = a.saved_lse[((int64_t)b * a.HK * a.per + head) * a.Lq + q];
            low = lse == -INFINITY ? INFINITY : fabsf(lse) < FAR_LSE ? lse * LOG2E - LIFT<T> : 2.f * lse;      // a row without a key: no weight
        }
#pragma unroll
        for (int x = 1; x < 16; x *= 2) sum += __shfl_xor(sum, x);
        if (lane == 0) { a.aux[row] = low; a.aux[all + row] = low == INFINITY ? 0.f : sum; }
    }
}

__device__ __forceinline__ bool far_row(float low) { return fabsf(low) >= 2.f * FAR_LSE && low != INFINITY; }
__device__ __forceinline__ bool far_row(f32x4 low) { return far_row(low[0]) || far_row(low[1]) || far_row(low[2]) || far_row(low[3]); }
// lse of any row, infinity where it has no key
template <class T> __device__ __forceinline__ float row_lse(float low) { return fabsf(low) >= 2.f * FAR_LSE ? 0.5f * low : (low + LIFT<T>) * LN2; }

// dS as a product's operand.  bf16 has fp32's range: rounded once.  fp16 would lose what is small: a row's (key's) elements are held
// times a power of two that brings the largest so far to 2^13 .. 2^15, and the sums follow when it changes.  The elements come 2^LIFT times as large, as the
// weights in them.
template <class T, int N> struct Lifted {
    static constexpr bool ON = std::is_same<T, _Float16>::value;
    float by[N];
    __device__ __forceinline__ Lifted() {
#pragma unroll
        for (int j = 0; j < N; ++j) by[j] = 0x1p46f;
    }
    // x: the tile's elements, [N][X] quads
    template <int X, int DB> __device__ __forceinline__ void lift(f32x4 (&x)[N][X], f32x4 (&sums)[DB][N]) {
        if constexpr (ON) {
#pragma unroll
            for (int j = 0; j < N; ++j) {
                float top = 0.f;
#pragma unroll
                for (int i = 0; i < X; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) top = fmaxf(top, fabsf(x[j][i][e]));
                top = lanes_max(top);
                const bool grow = top * by[j] > 32768.f && top < INFINITY;
                if (__any(grow)) {
                    const float now = grow ? __builtin_amdgcn_ldexpf(1.f, 14 - __builtin_amdgcn_frexp_expf(top)) : by[j], to = now / by[j];
                    by[j] = now;
#pragma unroll
                    for (int d = 0; d < DB; ++d) sums[d][j] *= to;
                }
#pragma unroll
                for (int i = 0; i < X; ++i) x[j][i] *= by[j];
            }
        }
    }
    __device__ __forceinline__ float back(int j) const { return ON ? 1.f / (16384.f * by[j]) : 1.f; }
};

template <class T, int DP, int QB, bool TWO = false>
__global__ __launch_bounds__(256, DP == 256 && (F32<T> || TWO) ? 1 : 2) void dq_kernel(AttentionArgs a, int tiles, int splits, int share) {
    typedef Num<T> N;
    typedef typename Elem<T>::type E;
    typedef typename N::F F;
    constexpr int KT = tile_rows<T, DP, 4>(), CH = DP / FK, DB = DP / 16, PB = 2;
    // The sums of dO V^T begin at -delta, four registers more a row and one instruction less an element: 2 x 14400 x 14400 x 2 x 64 bf16: 387 -> 375 us; fp16's
    // powers of two and heads of 256 leave no registers for it (478 -> 511, 430 -> 442).
    constexpr bool FROM = !Lifted<T, QB>::ON && DP <= 128;
    typedef Tile<T, DP, KT, 4> Load;
    __shared__ __align__(1024) unsigned char smem[2 * Load::PLACES * Load::BYTES];
    lds_byte* const lds = (lds_byte*)smem;
    const unsigned lds_at = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)lds);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lr = lane & 15, lg = lane >> 4;
    const Place at = place_of(a, tiles, splits);
    Keys keys = keys_of<T>(a, at.b);
    const int k_lo = at.split * share;
    keys.end = min(keys.end, k_lo + share);
    const int steps = keys.end > k_lo ? (keys.end - k_lo + KT - 1) / KT : 0;
    const Source<T> from_k = source<T>(a.k, a.k3, a.k_item, a.k_row, a.k_head, a, at, k_lo), from_v = source<T>(a.v, a.v3, a.v_item, a.v_row, a.v_head, a, at, k_lo);
    const int r0 = (at.tile * 4 + wave) * 16 * QB;
    F fq[QB][CH], fo[QB][CH];
    float low[QB], delta[QB];
#pragma unroll
    for (int j = 0; j < QB; ++j) {
        const int r = r0 + 16 * j + lr;
        const bool there = r < a.rows;
        int q, g;
        query_of(a, r, q, g);
        const int head = at.hk * a.per + g;
        const E* p = (const E*)a.q + at.b * a.q_item + head * a.q_head + q * a.q_row;
        const E* w = (const E*)a.d_out + (((int64_t)at.b * a.Lq + q) * a.HK * a.per + head) * a.D;
#pragma unroll
        for (int t = 0; t < CH; ++t) {
            fq[j][t] = N::load(p, t * FK + lg * 8, a.D, there);
            fo[j][t] = N::load(w, t * FK + lg * 8, a.D, there);
        }
        const int aux_rows = attention_aux_rows(a.rows);
        const float* const aux = a.aux + (int64_t)at.bh * aux_rows + r;
        low[j] = there ? aux[0] : INFINITY;
        delta[j] = there ? aux[(int64_t)a.B * a.HK * aux_rows] : 0.f;
    }
    Load load_k, load_v;
    load_k.plan(wave, lane, a.D);
    load_v.plan(wave, lane, a.D);
    auto ask = [&](int t, uint64_t bits) {
        const unsigned to = lds_at + t % Load::PLACES * 2 * Load::BYTES;
        from_k.ask(load_k, t * KT, to, wave, bits);
        from_v.ask(load_v, t * KT, to + Load::BYTES, wave, bits);
    };
    bool some_far = false;
#pragma unroll
    for (int j = 0; j < QB; ++j) some_far |= far_row(low[j]);
    const bool far = __syncthreads_or(some_far);
    if (far)
#pragma unroll
        for (int j = 0; j < QB; ++j) low[j] = row_lse<T>(low[j]);
    const float c = a.scale * LOG2E;
    f32x4 dq[DB][QB] = {};
    Lifted<T, QB> lifted;
    auto walk = [&](auto is_far) {
        constexpr bool IS_FAR = decltype(is_far)::value;
        uint64_t bits = 0;
        unsigned byte = 0;
        if (steps) {
            bits = keys.bits(k_lo, KT, keys.byte(k_lo, lane));
            if (bits && !Late<Load>::value) ask(0, bits);
            byte = keys.byte(k_lo + KT, lane);
        }
        for (int t = 0; t < steps; ++t) {
            if constexpr (Late<Load>::value) {
                __syncthreads();
                if (bits) ask(t, bits);
            }
            land(load_k, load_v, smem);
            uint64_t next = 0;
            if (t + 1 < steps) {
                next = keys.bits(k_lo + (t + 1) * KT, KT, byte);
                if (next && !Late<Load>::value) ask(t + 1, next);
                byte = keys.byte(k_lo + (t + 2) * KT, lane);
            }
            if (bits) {
                lds_byte* const tk = lds + t % Load::PLACES * 2 * Load::BYTES;
                lds_byte* const tv = tk + Load::BYTES;
                const bool some = bits != ~0ull >> (64 - KT);
                const uint64_t mine = bits >> (4 * lg);
#pragma unroll
                for (int kk = 0; kk < KT / FK; ++kk) {
                    f32x4 s[QB][PB] = {}, dp[QB][PB] = {};
                    if constexpr (FROM)
#pragma unroll
                        for (int j = 0; j < QB; ++j)
#pragma unroll
                            for (int i = 0; i < PB; ++i) dp[j][i] = f32x4{-delta[j], -delta[j], -delta[j], -delta[j]};
#pragma unroll
                    for (int h = 0; h < CH; ++h)
#pragma unroll
                        for (int i = 0; i < PB; ++i) {
                            const F f = N::template straight<DP, KT>(tk, FK * kk + 16 * i + lr, h, lg);
                            const F w = N::template straight<DP, KT>(tv, FK * kk + 16 * i + lr, h, lg);
#pragma unroll
                            for (int j = 0; j < QB; ++j) {
                                s[j][i] = N::times(f, fq[j][h], s[j][i]);
                                dp[j][i] = N::times(w, fo[j][h], dp[j][i]);
                            }
                        }
#pragma unroll
                    for (int j = 0; j < QB; ++j)
#pragma unroll
                        for (int i = 0; i < PB; ++i)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float p = power<T, IS_FAR>(s[j][i][e], a.scale, c, low[j]);
                                dp[j][i][e] = p * (FROM ? dp[j][i][e] : dp[j][i][e] - delta[j]);
                                if (some) dp[j][i][e] = (mine >> (FK * kk + 16 * i + e)) & 1 ? dp[j][i][e] : 0.f;
                            }
                    lifted.lift(dp, dq);
                    F fs[QB], ls[QB];
#pragma unroll
                    for (int j = 0; j < QB; ++j) {
                        fs[j] = N::pack(dp[j]);
                        if constexpr (TWO) ls[j] = N::rest(dp[j], fs[j]);
                    }
#pragma unroll
                    for (int d = 0; d < DB; ++d) {
                        const F f = N::template turned<DP, KT>(tk, FK * kk, d, lr, lg);
#pragma unroll
                        for (int j = 0; j < QB; ++j) {
                            if constexpr (TWO) dq[d][j] = N::times(f, ls[j], dq[d][j]);
                            dq[d][j] = N::times(f, fs[j], dq[d][j]);
                        }
                    }
                }
            }
            bits = next;
        }
    };
    if (far) walk(std::true_type{});
    else walk(std::false_type{});
#pragma unroll
    for (int j = 0; j < QB; ++j) {
        const int r = r0 + 16 * j + lr;
        if (r >= a.rows) continue;
        int q, g;
        query_of(a, r, q, g);
        const int64_t row = (((int64_t)at.b * a.Lq + q) * a.HK * a.per + at.hk * a.per + g) * a.D;
        const float by = lifted.back(j) * a.scale;
#pragma unroll
        for (int d = 0; d < DB; ++d) {
            if (16 * d + 4 * lg >= a.D) continue;
            const float v[4] = {dq[d][j][0] * by, dq[d][j][1] * by, dq[d][j][2] * by, dq[d][j][3] * by};
            if (splits > 1) store_some<float, 4>(a.part_q + (int64_t)at.split * a.B * a.Lq * a.HK * a.per * a.D + row + 16 * d + 4 * lg, v, 4);
            else store_some<E, 4>((E*)a.d_q + row + 16 * d + 4 * lg, v, 4);
        }
    }
}

// A workgroup has 64 KB keys in its waves' registers (KB blocks of 16 a wave) and goes over the rows of the query heads that read them.  S = Q K^T here: a lane has four rows
// of one key.  A key that does not count has sums of its own, which are not stored.
template <class T, int DP, int KB, bool TWO = false>
__global__ __launch_bounds__(256, DP == 256 ? 1 : 2) void dkv_kernel(AttentionArgs a, int tiles, int splits, int share) {
    typedef Num<T> N;
    typedef typename Elem<T>::type E;
    typedef typename N::F F;
    constexpr int RT = tile_rows<T, DP, 4>(), CH = DP / FK, DB = DP / 16, PB = 2;
    typedef Tile<T, DP, RT, 4> Load;
    __shared__ __align__(1024) unsigned char smem[2 * Load::PLACES * Load::BYTES];
    __shared__ int answers[4];                           // of the waves: 1, a key counts; 2, a row is far
    lds_byte* const lds = (lds_byte*)smem;
    const unsigned lds_at = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)lds);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lr = lane & 15, lg = lane >> 4;
    const Place at = place_of(a, tiles, splits);
    const Keys keys = keys_of<T>(a, at.b);
    const int k0 = (at.tile * 4 + wave) * 16 * KB, r_lo = at.split * share, r_hi = min(a.rows, r_lo + share);
    const int aux_rows = attention_aux_rows(a.rows);
    const float* const lows = a.aux + (int64_t)at.bh * aux_rows;
    const float* const deltas = lows + (int64_t)a.B * a.HK * aux_rows;
    // whether a row of the share is far: the first rows' answer comes with the keys
    const f32x4 first = r_lo + 4 * tid < r_hi ? *reinterpret_cast<const f32x4*>(lows + r_lo + 4 * tid) : f32x4{};
    bool some_far = false;
#pragma unroll 8
    for (int r = r_lo + 4 * (tid + 256); r < r_hi; r += 4 * 256) some_far |= far_row(*reinterpret_cast<const f32x4*>(lows + r));
    F fk[KB][CH], fv[KB][CH];
    bool counts[KB];
    bool any = false;
#pragma unroll
    for (int j = 0; j < KB; ++j) {
        const int k = k0 + 16 * j + lr;
        counts[j] = k < keys.end && (!keys.mask || keys.mask[k]);
        any |= counts[j];
        const E* p = (const E*)a.k + at.b * a.k_item + at.hk * a.k_head + k * a.k_row;
        const E* w = (const E*)a.v + at.b * a.v_item + at.hk * a.v_head + k * a.v_row;
#pragma unroll
        for (int t = 0; t < CH; ++t) {
            fk[j][t] = N::load(p, t * FK + lg * 8, a.D, counts[j]);
            fv[j][t] = N::load(w, t * FK + lg * 8, a.D, counts[j]);
        }
    }
    const int mine = (__any(any) ? 1 : 0) | (__any(some_far || far_row(first)) ? 2 : 0);
    if (lane == 0) answers[wave] = mine;
    __syncthreads();
    const int answer = __builtin_amdgcn_readfirstlane(answers[0] | answers[1] | answers[2] | answers[3]);
    const int steps = answer & 1 ? (r_hi - r_lo + RT - 1) / RT : 0;
    const bool far = answer & 2;
    const int64_t o_row = (int64_t)a.HK * a.per * a.D;
    Load load_q, load_o;
    load_q.plan(wave, lane, a.D);
    load_o.plan(wave, lane, a.D);
    auto ask = [&](int t) {
        const unsigned to = lds_at + t % Load::PLACES * 2 * Load::BYTES;
        const int r0 = r_lo + t * RT;
        int q0, g0;
        query_of(a, r0, q0, g0);
        auto rows = [&](int row, int head, int es) {     // byte offsets of rows from query q0 on
            return [=, &a](int i) {
                int q, g;
                query_of(a, r0 + i, q, g);
                return r0 + i < r_hi ? (unsigned)(((q - q0) * row + g * head) * es) : PAST;
            };
        };
        const int64_t dense = ((int64_t)at.b * a.Lq + q0) * o_row + (int64_t)at.hk * a.per * a.D;
        if constexpr (std::is_same<T, Planes>::value) {
            const int64_t plane = (int64_t)a.B * a.Lq * o_row;
            load_q.ask((const __bf16*)a.q3 + dense, plane, to, wave, rows((int)o_row, a.D, 2));
            load_o.ask((const __bf16*)a.o3 + dense, plane, to + Load::BYTES, wave, rows((int)o_row, a.D, 2));
        } else {
            load_q.ask((const T*)a.q + at.b * a.q_item + (int64_t)at.hk * a.per * a.q_head + q0 * a.q_row, to, wave, rows((int)a.q_row, (int)a.q_head, sizeof(T)));
            load_o.ask((const T*)a.d_out + dense, to + Load::BYTES, wave, rows((int)o_row, a.D, sizeof(T)));
        }
    };
    const float c = a.scale * LOG2E;
    f32x4 dk[DB][KB] = {}, dv[DB][KB] = {};
    Lifted<T, KB> lifted;
    auto walk = [&](auto is_far) {
        constexpr bool IS_FAR = decltype(is_far)::value;
        if (steps && !Late<Load>::value) ask(0);
        for (int t = 0; t < steps; ++t) {
            if constexpr (Late<Load>::value) {
                __syncthreads();
                ask(t);
            }
            land(load_q, load_o, smem);
            if (t + 1 < steps && !Late<Load>::value) ask(t + 1);
            lds_byte* const tq = lds + t % Load::PLACES * 2 * Load::BYTES;
            lds_byte* const to = tq + Load::BYTES;
#pragma unroll
            for (int kk = 0; kk < RT / FK; ++kk) {
                f32x4 low[PB], delta[PB];
#pragma unroll
                for (int i = 0; i < PB; ++i) {               // share and tiles are multiples of 16, and so is the array's length
                    const int r = r_lo + t * RT + FK * kk + 16 * i + 4 * lg;
                    low[i] = f32x4{INFINITY, INFINITY, INFINITY, INFINITY};
                    delta[i] = f32x4{};
                    if (r < r_hi) {
                        low[i] = *reinterpret_cast<const f32x4*>(lows + r);
                        delta[i] = *reinterpret_cast<const f32x4*>(deltas + r);
                    }
                    if constexpr (IS_FAR)
#pragma unroll
                        for (int e = 0; e < 4; ++e) low[i][e] = row_lse<T>(low[i][e]);
                }
                f32x4 s[KB][PB] = {}, dp[KB][PB] = {};
#pragma unroll
                for (int h = 0; h < CH; ++h)
#pragma unroll
                    for (int i = 0; i < PB; ++i) {
                        const F f = N::template straight<DP, RT>(tq, FK * kk + 16 * i + lr, h, lg);
                        const F w = N::template straight<DP, RT>(to, FK * kk + 16 * i + lr, h, lg);
#pragma unroll
                        for (int j = 0; j < KB; ++j) {
                            s[j][i] = IS_FAR ? N::times_back(f, fk[j][h], s[j][i]) : N::times(f, fk[j][h], s[j][i]);
                            dp[j][i] = N::times(w, fv[j][h], dp[j][i]);
                        }
                    }
                // products and weights one after the other: 50 spilled registers less (2 x 1000 x 1000 x 4 x 256 fp32: 185 -> 153 us)
                if constexpr (F32<T> && DP == 256) __builtin_amdgcn_sched_barrier(0);
                F fp[KB], fs[KB], lp[KB], ls[KB];
#pragma unroll
                for (int j = 0; j < KB; ++j) {
#pragma unroll
                    for (int i = 0; i < PB; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float p = power<T, IS_FAR>(s[j][i][e], a.scale, c, low[i][e]);
                            dp[j][i][e] = p * (dp[j][i][e] - delta[i][e]);
                            s[j][i][e] = p;
                        }
                    if constexpr (TWO) {
                        fp[j] = N::pack_under(s[j]);
                        lp[j] = N::rest_over(s[j], fp[j]);
                    } else fp[j] = N::pack(s[j]);
                }
                lifted.lift(dp, dk);
#pragma unroll
                for (int j = 0; j < KB; ++j) {
                    fs[j] = N::pack(dp[j]);
                    if constexpr (TWO) ls[j] = N::rest(dp[j], fs[j]);
                }
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    const F f = N::template turned<DP, RT>(to, FK * kk, d, lr, lg);
                    const F w = N::template turned<DP, RT>(tq, FK * kk, d, lr, lg);
#pragma unroll
                    for (int j = 0; j < KB; ++j) {
                        if constexpr (TWO) {
                            dv[d][j] = N::times(f, lp[j], dv[d][j]);
                            dk[d][j] = N::times(w, ls[j], dk[d][j]);
                        }
                        dv[d][j] = N::times(f, fp[j], dv[d][j]);
                        dk[d][j] = N::times(w, fs[j], dk[d][j]);
                    }
                }
            }
        }
    };
    if (far) walk(std::true_type{});
    else walk(std::false_type{});
    const int64_t all = (int64_t)a.B * a.Lk * a.HK * a.D;
#pragma unroll
    for (int j = 0; j < KB; ++j) {
        const int k = k0 + 16 * j + lr;
        if (k >= a.Lk) continue;
        const int64_t row = (((int64_t)at.b * a.Lk + k) * a.HK + at.hk) * a.D;
        const float bk = lifted.back(j) * a.scale, bv = LIFT<T> ? 1.f / 16384.f : 1.f;
#pragma unroll
        for (int d = 0; d < DB; ++d) {
            if (16 * d + 4 * lg >= a.D) continue;
            float x[4], y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = counts[j] ? dk[d][j][e] * bk : 0.f;
                y[e] = counts[j] ? dv[d][j][e] * bv : 0.f;
            }
            const int64_t to = row + 16 * d + 4 * lg;
            if (splits > 1) {
                store_some<float, 4>(a.part_k + at.split * all + to, x, 4);
                store_some<float, 4>(a.part_v + at.split * all + to, y, 4);
            } else {
                store_some<E, 4>((E*)a.d_k + to, x, 4);
                store_some<E, 4>((E*)a.d_v + to, y, 4);
            }
        }
    }
}

// The splits' parts of a gradient, added in their order.
template <class T>
__global__ __launch_bounds__(256) void sum_kernel(const float* one, const float* two, T* to_one, T* to_two, int64_t quads, int splits) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= quads) return;
    const float* p = (blockIdx.y ? two : one) + 4 * i;
    f32x4 x = {};
#pragma unroll 4
    for (int s = 0; s < splits; ++s) x += *reinterpret_cast<const f32x4*>(p + s * quads * 4);
    const float v[4] = {x[0], x[1], x[2], x[3]};
    store_some<T, 4>((blockIdx.y ? to_two : to_one) + 4 * i, v, 4);
}

// fp32 arrays' three planes, [3][B][L][H][D] each: four elements a thread.  A pair of arrays in one launch.
struct Pair { const float* p; int64_t item, row, head; __bf16* to; };
__global__ __launch_bounds__(256) void split_kernel(Pair one, Pair two, int L, int H, int D, int64_t quads) {
    const Pair& x = blockIdx.y ? two : one;
    const int across = D / 4;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < quads; i += (int64_t)gridDim.x * 256) {
        const int64_t n = i / across, r = n / H;
        const int d = (int)(i - n * across) * 4, h = (int)(n - r * H), b = (int)(r / L);
        const Some<float, 4>::type v = *reinterpret_cast<const Some<float, 4>::type*>(x.p + b * x.item + (r - (int64_t)b * L) * x.row + h * x.head + d);
        u32x2 parts[3];
        split4(f32x4{v[0], v[1], v[2], v[3]}, parts);
#pragma unroll
        for (int q = 0; q < 3; ++q) *reinterpret_cast<u32x2*>(x.to + (q * quads + i) * 4) = parts[q];
    }
}
inline unsigned blocks_of(int64_t n) { return (unsigned)(n < 1 << 20 ? n : 1 << 20); }
void split(const Pair& one, const Pair& two, int B, int L, int H, int D, hipStream_t s) {
    const int64_t quads = (int64_t)B * L * H * (D / 4);
    hipLaunchKernelGGL(split_kernel, dim3(blocks_of((quads + 255) / 256), 2), dim3(256), 0, s, one, two, L, H, D, quads);
}

// Where two blocks of 16 rows (keys) a wave fit its registers: keys of heads of 128 would spill 75 (1 x 32400 x 32400 x 2 x 128 bf16: 4060 us, with one block
// 2600; all registers of a wave: 2800 to 2900), fp32's of 64 77.
constexpr bool two_fit(AttentionPass pass, bool f32, int DP) { return DP <= (pass != PASS_DKV ? (f32 ? 64 : 128) : f32 ? 32 : 64); }
// Few rows take one wave a workgroup.
constexpr bool one_fits(bool f32, int DP) { return !f32 || DP <= 128; }

template <class T, int DP>
void forward_pass(const AttentionArgs& a, const AttentionPlan& p, hipStream_t s) {
    const dim3 grid(p.tiles * p.splits * a.B * a.HK);
    if constexpr (!F32<T>) if (p.two) {
        hipLaunchKernelGGL((forward_kernel<T, DP, 4, 1, true>), grid, dim3(256), 0, s, a, p.tiles, p.splits, p.share);
        return;
    }
    if (p.blocks == 1) hipLaunchKernelGGL((forward_kernel<T, DP, 4, 1>), grid, dim3(256), 0, s, a, p.tiles, p.splits, p.share);
    else if constexpr (two_fit(PASS_FORWARD, F32<T>, DP)) hipLaunchKernelGGL((forward_kernel<T, DP, 4, 2>), grid, dim3(256), 0, s, a, p.tiles, p.splits, p.share);
}
template <class T, int DP>
void dq_pass(const AttentionArgs& a, const AttentionPlan& p, hipStream_t s) {
    const dim3 grid(p.tiles * p.splits * a.B * a.HK);
    if constexpr (!F32<T>) if (p.two) {
        hipLaunchKernelGGL((dq_kernel<T, DP, 1, true>), grid, dim3(256), 0, s, a, p.tiles, p.splits, p.share);
        return;
    }
    if (p.blocks == 1) hipLaunchKernelGGL((dq_kernel<T, DP, 1>), grid, dim3(256), 0, s, a, p.tiles, p.splits, p.share);
    else if constexpr (two_fit(PASS_DQ, F32<T>, DP)) hipLaunchKernelGGL((dq_kernel<T, DP, 2>), grid, dim3(256), 0, s, a, p.tiles, p.splits, p.share);
}
template <class T, int DP>
void dkv_pass(const AttentionArgs& a, const AttentionPlan& p, hipStream_t s) {
    const dim3 grid(p.tiles * p.splits * a.B * a.HK);
    if constexpr (!F32<T>) if (p.two) {
        hipLaunchKernelGGL((dkv_kernel<T, DP, 1, true>), grid, dim3(256), 0, s, a, p.tiles, p.splits, p.share);
        return;
    }
    if (p.blocks == 1) hipLaunchKernelGGL((dkv_kernel<T, DP, 1>), grid, dim3(256), 0, s, a, p.tiles, p.splits, p.share);
    else if constexpr (two_fit(PASS_DKV, F32<T>, DP)) hipLaunchKernelGGL((dkv_kernel<T, DP, 2>), grid, dim3(256), 0, s, a, p.tiles, p.splits, p.share);
}
void split_keys(const AttentionArgs& a, hipStream_t s) {
    split({(const float*)a.k, a.k_item, a.k_row, a.k_head, (__bf16*)a.k3}, {(const float*)a.v, a.v_item, a.v_row, a.v_head, (__bf16*)a.v3}, a.B, a.Lk, a.HK, a.D, s);
}
template <class T, int DP>
hipError_t forward(const AttentionArgs& a, const AttentionPlan& p, hipStream_t s) {
    bool done = false;
    if constexpr (F32<T>) if (p.planes) {
        split_keys(a, s);
        forward_pass<Planes, DP>(a, p, s);
        done = true;
    }
    if constexpr (one_fits(F32<T>, DP)) if (p.waves == 1) {
        hipLaunchKernelGGL((forward_kernel<T, DP, 1, 1, !F32<T>>), dim3(p.tiles * p.splits * a.B * a.HK), dim3(64), 0, s, a, p.tiles, p.splits, p.share);
        done = true;
    }
    if (!done) forward_pass<T, DP>(a, p, s);
    if (p.splits > 1) {
        int across = 2, shares = 1;
        while (4 * across < a.D) across *= 2;
        const int threads = p.splits >= 32 ? 1024 : 256;
        while (2 * shares * across <= threads && 4 * shares <= p.splits) shares *= 2;
        const dim3 grid(cdiv((int64_t)a.B * a.HK * a.rows, threads / (across * shares)));
        if (threads == 1024) hipLaunchKernelGGL((forward_join_kernel<T, 1024>), grid, dim3(1024), 0, s, a, p.splits, across, shares);
        else hipLaunchKernelGGL((forward_join_kernel<T, 256>), grid, dim3(256), 0, s, a, p.splits, across, shares);
    }
    return hipGetLastError();
}
template <class T, int DP>
hipError_t backward(const AttentionArgs& a, const AttentionPlan& pq, const AttentionPlan& pk, hipStream_t s) {
    const int aux_rows = attention_aux_rows(a.rows);
    hipLaunchKernelGGL(delta_kernel<T>, dim3(blocks_of(((int64_t)a.B * a.HK * aux_rows + 15) / 16)), dim3(256), 0, s, a, aux_rows);
    if (a.d_q) {
        bool done = false;
        if constexpr (F32<T>) if (pq.planes) {
            split_keys(a, s);
            dq_pass<Planes, DP>(a, pq, s);
            done = true;
        }
        if (!done) dq_pass<T, DP>(a, pq, s);
        if (pq.splits > 1) {
            const int64_t quads = (int64_t)a.B * a.Lq * a.HK * a.per * a.D / 4;
            hipLaunchKernelGGL(sum_kernel<T>, dim3(cdiv(quads, 256)), dim3(256), 0, s, a.part_q, a.part_q, (T*)a.d_q, (T*)a.d_q, quads, pq.splits);
        }
    }
    if (a.d_k) {
        bool done = false;
        if constexpr (F32<T>) if (pk.planes) {
            const int H = a.HK * a.per;
            const int64_t row = (int64_t)H * a.D;
            split({(const float*)a.q, a.q_item, a.q_row, a.q_head, (__bf16*)a.q3}, {(const float*)a.d_out, a.Lq * row, row, a.D, (__bf16*)a.o3}, a.B, a.Lq, H, a.D, s);
            dkv_pass<Planes, DP>(a, pk, s);
            done = true;
        }
        if (!done) dkv_pass<T, DP>(a, pk, s);
        if (pk.splits > 1) {
            const int64_t quads = (int64_t)a.B * a.Lk * a.HK * a.D / 4;
            hipLaunchKernelGGL(sum_kernel<T>, dim3(cdiv(quads, 256), 2), dim3(256), 0, s, a.part_k, a.part_v, (T*)a.d_k, (T*)a.d_v, quads, pk.splits);
        }
    }
    return hipGetLastError();
}
#define BY_LENGTH(f, T, ...) a.D <= 32 ? f<T, 32>(__VA_ARGS__) : a.D <= 64 ? f<T, 64>(__VA_ARGS__) : a.D <= 128 ? f<T, 128>(__VA_ARGS__) : f<T, 256>(__VA_ARGS__)

}  // namespace

#if CORR_ATTENTION_TYPE == 0
hipError_t launch_attention_f32(const AttentionArgs& a, const AttentionPlan& p, hipStream_t s) { return BY_LENGTH(forward, float, a, p, s); }
hipError_t launch_attention_backward_f32(const AttentionArgs& a, const AttentionPlan& pq, const AttentionPlan& pk, hipStream_t s) { return BY_LENGTH(backward, float, a, pq, pk, s); }

// What a call costs, in multiples of the time that a compute unit with all the workgroups it holds at a time (`held`) takes for a whole one: rounds
// of them, the last one with fewer, which use the unit less well (2 x 2852 x 7285 x 4 x 64 fp32, 360 workgroups: forward 373 us, in two shares
// 263, in three 294; 1 x 14400 x 14400 x 256 bf16, 225: 314 in two, 417 in three, 329 in four).
namespace {
double rounds(int64_t groups, int held) {
    const int64_t whole = groups / (256 * held), rest = groups - whole * 256 * held, n = (rest + 255) / 256;
    const double use[] = {1, held == 1 ? 1. : held == 2 ? .65 : .6, held == 2 ? 1. : .85, 1, 1};
    return whole * held + n / use[n];
}
// as the kernels' registers and LDS allow
int held_at_once(bool f32, AttentionPass pass, int pad, int blocks) {
    if (pad == 256) return f32 || pass == PASS_DKV ? 1 : 2;
    if (pad == 128) return f32 && pass == PASS_FORWARD ? 3 : 2;
    if (f32) return blocks == 2 && pass == (pad == 64 ? PASS_DQ : PASS_DKV) ? 2 : 3;
    return pad == 32 || blocks == 1 ? 4 : pass == PASS_DKV ? 2 : 3;
}
}  // namespace

// Rows of a workgroup: 16 in one wave where there are no more (shares of the keys for five on every compute unit), else 64, or 128 in two blocks of 16
// a wave.  Shares of the long axis, of four tiles at least, where they make the rounds of workgroups fuller by more than their join costs (about
// 4 us and the sums' way to memory and back).
AttentionPlan attention_plan(corr_dtype t, AttentionPass pass, int B, int Lq, int Lk, int HK, int per, int D) {
    const int pad = D <= 32 ? 32 : D <= 64 ? 64 : D <= 128 ? 128 : 256;
    const bool f32 = t == CORR_TYPE_F32;
    const int rows = Lq * per, along = pass == PASS_DKV ? Lk : rows, over = pass == PASS_DKV ? rows : Lk, most = over > 256 ? cdiv(over, 256) : 1;
    const int64_t heads = (int64_t)B * HK;
    AttentionPlan p;
    p.waves = pass == PASS_FORWARD && along <= 16 && one_fits(f32, pad) ? 1 : 4;
    p.blocks = 1;
    // Rounded once, weights and dS add as much error as the result's own rounding does; a second part takes that away at half the products again.  It is there where
    // launches and loads are what takes the time (bf16, 4 heads of 64, keys 2852; forward, rows' and keys' gradient in one part and in two, us: 512 rows and heads 14.9
    // 20.7 20.6 and 15.2 21.1 20.6; 2800: 18.9 21.9 25.8 and 20.0 21.6 29.2; 11408: 27.5 33.8 43 and 32.3 39.7 54; 28800, 7200 keys: 88 117 150 and 125 159 240; 8 x
    // 32768 keys, one row: 74 and 77), and for the gradients of few keys, of which the same holds.
    p.two = !f32 && (p.waves == 1 || heads * rows <= 512 || (pass == PASS_DKV && heads * Lk <= 64));
    // Planes are made once a call and read by every tile of rows: from 2048 rows on (2852 x 2852 x 4 x 32: 51 us, 53 without; 7200 x 7200 x 2 x 32: 102 and
    // 117; 256 x 20000 x 2 x 128: 71 and 51).
    p.planes = f32 && p.waves == 4 && along >= 2048;
    int splits = 1;
    if (p.waves == 1) {
        const int64_t want = heads > 0 ? (1280 + heads - 1) / heads : 1;
        const int finest = over > 64 ? cdiv(over, 64) : 1;
        splits = (int)(want < finest ? want : finest);
    } else {
        const int products = pass == PASS_FORWARD ? 2 : pass == PASS_DQ ? 3 : 4;
        // products a microsecond of one compute unit, and the bytes that the join moves in one
        const double rate = (f32 ? pad == 32 ? 140e6 : 190e6 : pad == 32 ? 450e6 : 700e6) / 256, bytes = 4e6;
        double best = 1e30;
        for (int blocks = 1; blocks <= (two_fit(pass, f32, pad) && !p.two ? 2 : 1); ++blocks) {
            const int64_t groups = cdiv(along, 64 * blocks) * heads;
            const int held = held_at_once(f32, pass, pad, blocks);
            // one block a wave reads its tiles for half as many products
            const double one = (blocks == 1 ? pass == PASS_DKV ? 1.2 : 1.05 : 1.) * 2. * products * 64 * blocks * over * (double)pad / rate;
            for (int s = 1; s <= most && (s == 1 || groups * (s - 1) < 2048); ++s) {
                const double join = s == 1 ? 0 : 4 + 8. * s * heads * along * D * (pass == PASS_DKV ? 2 : 1) / bytes;
                const double cost = rounds(groups * s, held) * one / s + join;
                if (cost < best) { best = cost; splits = s; p.blocks = blocks; }
            }
        }
    }
    p.tile = 16 * p.waves * p.blocks;
    p.tiles = cdiv(along, p.tile);
    p.share = over > 0 ? (cdiv(over, splits) + 63) & ~63 : 64;
    p.splits = over > 0 ? cdiv(over, p.share) : 1;
    return p;
}
#elif CORR_ATTENTION_TYPE == 1
hipError_t launch_attention_bf16(const AttentionArgs& a, const AttentionPlan& p, hipStream_t s) { return BY_LENGTH(forward, __bf16, a, p, s); }
hipError_t launch_attention_backward_bf16(const AttentionArgs& a, const AttentionPlan& pq, const AttentionPlan& pk, hipStream_t s) { return BY_LENGTH(backward, __bf16, a, pq, pk, s); }
#else
hipError_t launch_attention_f16(const AttentionArgs& a, const AttentionPlan& p, hipStream_t s) { return BY_LENGTH(forward, _Float16, a, p, s); }
hipError_t launch_attention_backward_f16(const AttentionArgs& a, const AttentionPlan& pq, const AttentionPlan& pk, hipStream_t s) { return BY_LENGTH(backward, _Float16, a, pq, pk, s); }
#endif
