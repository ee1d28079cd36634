// Linear attention with a decay for each head,
//     S[t] = exp(g[t]) S[t-1] + k[t]^T v[t],   y[t] = scale q[t] S[t],
// and its gradients.  A chunk of C steps is taken at once: with b the running sum of g inside the chunk and S the state in front,
//     y_i = scale exp(b_i) q_i S + sum_{j <= i} A_ij v_j,   A_ij = scale exp(b_i - b_j) (q_i . k_j),
//     S'  = exp(b_C) S + sum_j exp(b_C - b_j) k_j^T v_j,
// matrix products all of them.  Every factor is the exponential of a difference of sums (held as two floats, made in double), never a
// quotient of exponentials, so nothing overflows that the states do not, and is multiplied in as its root, twice, so that of a large number
// what is left stays.  A decay of zero ends a document: factors across it are zeros by selection, not by multiplication, whatever is
// on its other side.  Nothing else forgets: a product of decays that leaves nothing of a number is not zero itself (its root is 2^-126 at the
// least), and an infinity or NaN in a state stays.
//
// A workgroup walks chunks in their order with the state in registers, 16 columns a wave (the backward pass in the other order with the
// state's gradient).  Where heads are too few to fill the card, a sequence is cut into segments: a walk that makes states only, a
// scan over the segments' ends, and the walk itself.  The state's products take the factor of k or q as three bf16 parts, so that states
// are sums of fp32 products in bf16 calls too; what is rounded to bf16 is A and the copies of S that are multiplied.
//
// Measured (MI355X, 8192 steps x 32 heads of 128 x 128, bf16): ends 43 us, scan 12, walk 88 (110-120 with marks), gradients' ends 44, backward
// walk 235.  The bytes of the walk are 268 MB, 48 us; what bounds it is issue: vector instructions 58% busy, LDS 50%, matrix cores 23%, of
// waves that do the same phase between barriers; 42% of LDS's cycles are bank conflicts (rows 272 bytes apart begin 4 banks after one
// another, and a turned read takes 8 banks from each of four rows).  On the way: loads ahead of a chunk that waited for branches or for spilled
// addresses cost half of a chunk's time (162 -> 90 us), places in vector registers spilled (backward 406 -> 228).  The walk with marks still
// spills 15 registers (15 of the 216 MB it writes).  Tried without gain: 4 waves of 32 columns, rows 32 bytes further apart in LDS (more
// conflicts), two blocks of 16 rows at once, 2 chunks a segment.  Roots of factors instead of factors, large states looked for and E's diagonal
// apart took the backward walk from 222 to 235 us and the others 1-3% up.
//
// A product mixes rows, and a zero times an infinity is none: a chunk that holds anything not finite, or so large that a product on the
// way could become so, or decays far above one, or that meets a state with so large a number, is taken a row at a time, by the formulas as
// they stand.  (Infinities and NaN in a state need not be looked for: products keep them in their row and column.)  The backward pass makes
// the states of such a chunk again from its mark for every step, a number of updates that grows with the square of the chunk: where all chunks
// are of this kind, 8192 x 32 heads of 128 take 4.1 ms forward and 107 ms backward.
#include <string.h>

#include <cmath>
#include <type_traits>

#include "hy_common.hpp"
#include "hy_launch.hpp"
#include "hy_scan.hpp"

namespace hy {

namespace {

typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t* lds_quad_t;

constexpr float kForgets = -87.3f;  // exp of less is below the smallest normal number
constexpr double kLog2E = 1.4426950408889634074;
// Of a chunk that is taken at once: bits by which decays above one may grow a state, and what numbers (times a scale above one) stay
// below, so that products of two numbers, a factor and a sum over 128 are finite: 24 + 2 * 46 + 7 < 127; and what the states' numbers
// stay below, so that those of a state and the other's gradient are, and of one with a number of the chunk: 2 * 56 + 14 < 127.
constexpr float kMostGrowth = 24.0f, kMostNumber = 0x1p46f, kMostState = 0x1p56f;

// A factor exp2(d) as its root r = exp2(d / 2), multiplied in twice: growth beyond the range of one factor is left to the products it is in,
// and a root is zero for a reset alone (2^-252 of the largest number is below 2^-124).
__device__ __forceinline__ float half_factor(float d) {
    const float x = 0.5f * d;
    return __builtin_amdgcn_exp2f(x > 127.0f ? 127.0f : x < -126.0f ? -126.0f : x);  // (of NaN: NaN)
}
__device__ __forceinline__ float step_factor(float g) { return g < kForgets ? 0.0f : half_factor((float)((double)g * kLog2E)); }
__device__ __forceinline__ float scaled(float x, float half) { return half == 0.0f ? 0.0f : x * half * half; }

// Eight numbers of a row of an operand: k = 8 lq + e of a block of 32 (lane: li = lane % 16, lq = lane / 16), or in the order of
// accumulators ("turned"), k = 16 (e / 4) + 4 lq + e % 4.  A product's result has in lane (li, lq), register r, row 4 lq + r of its
// first operand and row li of the second.
template <typename T>
struct Frag;
template <>
struct Frag<BF16> {
    bf16x8_t x;
};
template <>
struct Frag<F32> {
    float x[8];
};

__device__ __forceinline__ void multiply(f32x4_t& acc, const Frag<BF16>& a, const Frag<BF16>& b) {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.x, b.x, acc, 0, 0, 0);
}
__device__ __forceinline__ void multiply(f32x4_t& acc, const Frag<F32>& a, const Frag<F32>& b) {
#pragma unroll
    for (int e = 0; e < 8; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a.x[e], b.x[e], acc, 0, 0, 0);
}

template <typename T>
using Elem = std::conditional_t<std::is_same_v<T, F32>, float, uint16_t>;

// Steps of a chunk: what LDS holds of them.
template <typename T>
constexpr int kChunk = T::kBytes == 2 ? 64 : 32;

// Rows of D numbers in LDS and their distance: 16 bytes more than they take, so that 16 rows at a column spread over the banks.
template <typename T, int D>
constexpr int kPitch = D + 16 / T::kBytes;

__device__ __forceinline__ Frag<BF16> frag_of(const float (&f)[8], BF16) {
    Words<4> w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w.w[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
    return Frag<BF16>{__builtin_bit_cast(bf16x8_t, w)};
}
__device__ __forceinline__ Frag<F32> frag_of(const float (&f)[8], F32) {
    Frag<F32> r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r.x[i] = f[i];
    return r;
}
__device__ __forceinline__ void floats_of(const Frag<BF16>& a, float (&f)[8]) {
    const Words<4> w = __builtin_bit_cast(Words<4>, a.x);
#pragma unroll
    for (int i = 0; i < 4; ++i) f[2 * i] = bf16_lo(w.w[i]), f[2 * i + 1] = bf16_hi(w.w[i]);
}
__device__ __forceinline__ void floats_of(const Frag<F32>& a, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = a.x[i];
}

// Row `row`, k from `k0`.
template <int PITCH>
__device__ __forceinline__ Frag<BF16> row_frag(const uint16_t* t, int row, int k0, int lq) {
    return Frag<BF16>{*reinterpret_cast<const bf16x8_t*>(t + row * PITCH + k0 + 8 * lq)};
}
template <int PITCH>
__device__ __forceinline__ Frag<F32> row_frag(const float* t, int row, int k0, int lq) {
    Frag<F32> r;
    const float4 *p = reinterpret_cast<const float4*>(t + row * PITCH + k0 + 8 * lq), a = p[0], b = p[1];
    r.x[0] = a.x, r.x[1] = a.y, r.x[2] = a.z, r.x[3] = a.w, r.x[4] = b.x, r.x[5] = b.y, r.x[6] = b.z, r.x[7] = b.w;
    return r;
}
template <int PITCH>
__device__ __forceinline__ Frag<BF16> turned_row_frag(const uint16_t* t, int row, int k0, int lq) {
    const uint2 a = *reinterpret_cast<const uint2*>(t + row * PITCH + k0 + 4 * lq), b = *reinterpret_cast<const uint2*>(t + row * PITCH + k0 + 16 + 4 * lq);
    return Frag<BF16>{__builtin_bit_cast(bf16x8_t, make_uint4(a.x, a.y, b.x, b.y))};
}
template <int PITCH>
__device__ __forceinline__ Frag<F32> turned_row_frag(const float* t, int row, int k0, int lq) {
    Frag<F32> r;
    const float4 a = *reinterpret_cast<const float4*>(t + row * PITCH + k0 + 4 * lq), b = *reinterpret_cast<const float4*>(t + row * PITCH + k0 + 16 + 4 * lq);
    r.x[0] = a.x, r.x[1] = a.y, r.x[2] = a.z, r.x[3] = a.w, r.x[4] = b.x, r.x[5] = b.y, r.x[6] = b.z, r.x[7] = b.w;
    return r;
}
// Columns of a tile as rows of an operand: lane li has column `c0` + li, k = rows from
// k0 in the plain order.  bf16: LDS turns 4 x 16 numbers at a time; lane l of 16 says where row l / 4 has its columns 4 (l % 4) and
// gets column l.
template <int PITCH>
__device__ __forceinline__ Frag<BF16> column_frag(const uint16_t* t, int k0, int c0, int li, int lq) {
    const uint16_t* p = t + (k0 + 8 * lq + li / 4) * PITCH + c0 + 4 * (li % 4);
    const s16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_quad_t)p), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_quad_t)(p + 4 * PITCH));
    const uint2 ua = __builtin_bit_cast(uint2, a), ub = __builtin_bit_cast(uint2, b);
    return Frag<BF16>{__builtin_bit_cast(bf16x8_t, make_uint4(ua.x, ua.y, ub.x, ub.y))};
}
template <int PITCH>
__device__ __forceinline__ Frag<F32> column_frag(const float* t, int k0, int c0, int li, int lq) {
    const float* p = t + (k0 + 8 * lq) * PITCH + c0 + li;
    Frag<F32> r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r.x[e] = p[e * PITCH];
    return r;
}

// Four results next to each other in LDS.
__device__ __forceinline__ void put4(uint16_t* p, const f32x4_t& v) { *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])); }
__device__ __forceinline__ void put4(float* p, const f32x4_t& v) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }

// acc += first (x) (f as fp32 numbers): of bf16 products f is three parts, which make its 24 bits.
__device__ __forceinline__ void multiply_wide(f32x4_t& acc, const Frag<BF16>& a, const Frag<BF16> (&f)[3]) {
    multiply(acc, a, f[2]);
    multiply(acc, a, f[1]);
    multiply(acc, a, f[0]);
}
__device__ __forceinline__ void multiply_wide(f32x4_t& acc, const Frag<F32>& a, const Frag<F32> (&f)[1]) { multiply(acc, a, f[0]); }
template <typename T>
constexpr int kParts = T::kBytes == 2 ? 3 : 1;
__device__ __forceinline__ void wide_frag(float (&f)[8], Frag<BF16> (&o)[3]) {
#pragma unroll
    for (int x = 0; x < 3; ++x) {
        o[x] = frag_of(f, BF16{});
        if (x == 2) break;
        float part[8];
        floats_of(o[x], part);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] -= part[e];  // (numbers, all of them: chunks with others are not taken at once)
    }
}
__device__ __forceinline__ void wide_frag(float (&f)[8], Frag<F32> (&o)[1]) { o[0] = frag_of(f, F32{}); }

// Where a tensor's rows are: [B, L, heads, d], channels contiguous.
struct Rows {
    const char* p;
    int64_t batch, step, head;  // bytes
    int32_t d, wide;            // wide: 8 numbers from a multiple of 8 on can be moved by 16 bytes, and rows of a chunk are near
};

// What a chunk's steps do to a state, in LDS: halves of the sums of log2 decays up to and with a step (two floats), the last step up to and with it
// that forgets (-1: none), roots of the factors from the chunk's start to behind a step, from behind it to the end, and of the whole.
template <int C>
struct Decays {
    float hi[C], lo[C];
    int32_t forgot[C];
    float from_start[C], to_end[C];
    float whole;
    double sum;
};

// A wave makes them; lane t has step t.  g: its log decay (0 behind the last step).  Whether the chunk can be taken at once.
template <int C>
__device__ __forceinline__ bool make_decays(Decays<C>& s, float g, int lane) {
    const bool forgets = g < kForgets, inside = lane < C;
    bool fine = fabsf(g) < INFINITY || forgets;
    if (__builtin_amdgcn_ballot_w64(g > 0.0f && inside) != 0)
        fine &= of_lane(wave_upto(g > 0.0f && inside ? g * (float)kLog2E : 0.0f), kWave - 1) <= kMostGrowth;
    const double b = wave_upto(forgets || !inside ? 0.0 : (double)g * kLog2E);
    const unsigned long long all = __builtin_amdgcn_ballot_w64(forgets && inside), upto = all & (~0ull >> (63 - lane));
    const int forgot = upto ? 63 - __builtin_clzll(upto) : -1, last = all ? 63 - __builtin_clzll(all) : -1;
    const double end = of_lane(b, kWave - 1);
    const float hi = (float)b;
    if (inside) {
        s.hi[lane] = 0.5f * hi, s.lo[lane] = 0.5f * (float)(b - (double)hi), s.forgot[lane] = forgot;
        s.from_start[lane] = forgot < 0 ? half_factor(hi) : 0.0f;
        s.to_end[lane] = lane >= last ? half_factor((float)(end - b)) : 0.0f;
    }
    if (lane == 0) {
        s.whole = last < 0 ? half_factor((float)end) : 0.0f;
        s.sum = last < 0 ? end : -INFINITY;
    }
    return fine;
}

// C rows of a chunk on their way to a tile in LDS: loaded a chunk ahead.  What lies behind the n-th row and the d-th number is loaded from
// elsewhere in them and becomes zeros in LDS, so that no load waits for a branch (16000 cycles of a chunk's 36000 before).
template <typename T, int C, int D, int NT>
struct Ahead {
    static constexpr int kPerRow = D / 8, kRows = NT / kPerRow, kEach = C > kRows ? C / kRows : 1, W = T::kBytes == 2 ? 4 : 8;
    static constexpr bool kIdle = kRows > C;  // lanes behind the last row load another's and put nothing
    static_assert(NT % kPerRow == 0 && (kIdle || C % kRows == 0), "a lane has the same columns of every kRows-th row");
    Words<W> r[kEach];

    __device__ __forceinline__ void load_one(int i, const char* p) {
        const Words<4> a = load_words<4>(p);
#pragma unroll
        for (int j = 0; j < 4; ++j) r[i].w[j] = a.w[j];
        if constexpr (W == 8) {
            const Words<4> b = load_words<4>(p + 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) r[i].w[4 + j] = b.w[j];
        }
    }
    // n: 1 at least.  (One path: where two of them load the same registers, a load waits for those before it.)
    __device__ __forceinline__ void load(const Rows& x, const char* from, int n, int c0) {
        if (!x.wide) return;
        const uint32_t me = (uint32_t)fresh((int)threadIdx.x), row0 = me / kPerRow, step = (uint32_t)x.step;
        const int c = c0 + (int)(me % kPerRow) * 8;
        const uint32_t at = (uint32_t)(c < x.d ? c : 0) * T::kBytes;
#pragma unroll
        for (int i = 0; i < kEach; ++i) load_one(i, from + (min(row0 + i * kRows, (uint32_t)n - 1) * step + at));
    }
    // Whether all are below `most` (bits of a float).  Rows that cannot be moved by 16 bytes are loaded here, number by number.
    __device__ __forceinline__ bool put(Elem<T>* tile, uint32_t most, const Rows& x, const char* from, int n, int c0) {
        typedef uint16_t pair_t __attribute__((ext_vector_type(2)));
        pair_t pairs = {0, 0};
        uint32_t one = 0;
        const uint32_t me = (uint32_t)fresh((int)threadIdx.x), row0 = me / kPerRow, c = me % kPerRow * 8;
        if (!x.wide) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const char* p = from + (int64_t)min(row0 + i * kRows, (uint32_t)n - 1) * x.step;
                uint32_t f[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int at = c0 + (int)c + j;
                    const char* pj = p + (int64_t)(at < x.d ? at : 0) * T::kBytes;
                    if constexpr (W == 8) f[j] = *reinterpret_cast<const uint32_t*>(pj);
                    else f[j] = *reinterpret_cast<const uint16_t*>(pj);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (c0 + (int)c + j >= x.d) f[j] = 0;
                    if constexpr (W == 8) r[i].w[j] = f[j];
                    else r[i].w[j / 2] = j % 2 ? r[i].w[j / 2] | f[j] << 16 : f[j];
                }
            }
        }
        if (n < C || c0 + D > x.d) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const bool in = row0 + i * kRows < (uint32_t)n && c0 + (int)c < x.d;
#pragma unroll
                for (int j = 0; j < W; ++j) r[i].w[j] = in ? r[i].w[j] : 0;
            }
        }
        Elem<T>* const to = tile + row0 * kPitch<T, D> + c;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            if (kIdle && row0 >= C) continue;
#pragma unroll
            for (int j = 0; j < W; ++j) {
                if constexpr (W == 4) pairs = __builtin_elementwise_max(pairs, __builtin_bit_cast(pair_t, r[i].w[j] & 0x7fff7fffu));
                else one = max(one, r[i].w[j] & 0x7fffffffu);
            }
#pragma unroll
            for (int j = 0; j < W; j += 4) {
                const Words<4> o{{r[i].w[j], r[i].w[j + 1], r[i].w[j + 2], r[i].w[j + 3]}};
                store_words<4>(to + i * kRows * kPitch<T, D> + j * (4 / T::kBytes), o);
            }
        }
        if constexpr (W == 4) return max(pairs[0], pairs[1]) < most >> 16;
        return one < most;
    }
};

template <typename T>
__device__ __forceinline__ float unpacked(const typename Pack<T, 1>::Raw& r) {
    float f[1];
    Pack<T, 1>::unpack(r, f);
    return f[0];
}
template <typename T>
__device__ __forceinline__ float number(const char* p) { return unpacked<T>(Pack<T, 1>::load(p)); }

struct LaArgs {
    Rows q, k, v, g, dy;  // (g: head is not looked at)
    const float *state_in, *dstate_out;
    char *y, *marks, *dv;
    const char* marks_in;
    float *state_out, *dstate_in;
    void *dq, *dk;         // of T, or the heads' shares in fp32
    void* dg;              // of T, or the tiles' shares in fp32
    float* ends;           // states (and their gradients) at the segments' ends: [segment][head and tile][DK DV], and their log2 decays
    double* sums;
    int64_t L, chunks, each;  // chunks of a segment
    int32_t H, group, dk_, dv_, tiles, segments, finer;  // finer: segments of the ends for one of the walk
    float scale;
    uint32_t most;  // numbers of chunks that are taken at once are below, as bits of a float
};

// A head, a tile of its columns and a segment: the workgroup's.
struct Place {
    int64_t b, item;  // item: (b H + h) tiles + tile
    int32_t h, hk, tile, segment;
};
__device__ __forceinline__ int32_t uniform(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ Place place_of(const LaArgs& a, uint32_t i) {
    Place p;  // (all below 2^31, and kept in scalar registers: pointers made of them are, too)
    const uint32_t n = (uint32_t)a.segments, item = (uint32_t)uniform((int32_t)(i / n)), bh = (uint32_t)uniform((int32_t)(item / (uint32_t)a.tiles));
    p.segment = uniform((int32_t)(i % n));
    p.item = item;
    p.tile = uniform((int32_t)(item % (uint32_t)a.tiles));
    p.h = uniform((int32_t)(bh % (uint32_t)a.H));
    p.b = uniform((int32_t)(bh / (uint32_t)a.H));
    p.hk = uniform(p.h / a.group);
    return p;
}

// max(most, |a|, |b|), NaN left out.
__device__ __forceinline__ float larger(float most, float a, float b) { return fmaxf(fmaxf(most, fabsf(a)), fabsf(b)); }

// The state of a wave: DK rows by 16 columns, in 16 x 16 pieces, as results of (rows of k) x (columns of v): lane (li, lq) has column li,
// rows 16 i + 4 lq + r of piece i.
template <int DT>
struct State {
    f32x4_t s[DT];

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < DT; ++i) s[i] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    }
    // from / to [dk][dv] numbers of a head; c: the lane's column (all loads first: one that waits for a branch waits for memory, 32 times
    // in a row)
    __device__ __forceinline__ void load(const float* p, int dk, int dv, int c, int lq) {
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) s[i][r] = p[(int64_t)min(16 * i + 4 * lq + r, dk - 1) * dv + min(c, dv - 1)];
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (16 * i + 4 * lq + r >= dk || c >= dv) s[i][r] = 0.0f;
    }
    __device__ __forceinline__ void store(float* p, int dk, int dv, int c, int lq) const {
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int d = 16 * i + 4 * lq + r;
                if (d < dk && c < dv) p[(int64_t)d * dv + c] = s[i][r];
            }
    }
    // the library's own order: pieces, then lanes
    __device__ __forceinline__ void load_own(const float* p, int lane) {
#pragma unroll
        for (int i = 0; i < DT; ++i) s[i] = *reinterpret_cast<const f32x4_t*>(p + (i * kWave + lane) * 4);
    }
    __device__ __forceinline__ void store_own(float* p, int lane) const {
#pragma unroll
        for (int i = 0; i < DT; ++i) *reinterpret_cast<f32x4_t*>(p + (i * kWave + lane) * 4) = s[i];
    }
    __device__ __forceinline__ void decay(float half) {
        half = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(half)));
        const float factor = half * half;
        if (half > 0x1p-63f) {
#pragma unroll
            for (int i = 0; i < DT; ++i) s[i] *= factor;
        } else if (half != 0.0f) {
#pragma unroll
            for (int i = 0; i < DT; ++i) s[i] = s[i] * half * half;
        } else {
            clear();  // (of infinities, too)
        }
    }
    // Whether a number of it is too large for products (not an infinity or NaN).
    __device__ __forceinline__ bool large() const {
        float most = 0.0f;
#pragma unroll
        for (int i = 0; i < DT; ++i) most = larger(larger(most, s[i][0], s[i][1]), s[i][2], s[i][3]);
        if (__builtin_amdgcn_ballot_w64(most >= kMostState) == 0) return false;
        const uint32_t from = __float_as_uint(kMostState), all = __float_as_uint(INFINITY) - from;
        uint32_t least = all;  // how far above the limit; numbers below it are far above infinity
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) least = min(least, (__float_as_uint(s[i][r]) & 0x7fffffffu) - from);
        return least < all;
    }
    __device__ __forceinline__ void decay_step(float half) {
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) s[i][r] = scaled(s[i][r], half);
    }
    // One step by itself: s = r r s + a[d] b[c] of `dk` by `dv` numbers.
    template <typename T>
    __device__ __forceinline__ void step(float half, const char* a, const char* b, float scale, int dk, int dv, int c, int lq) {
        const float bc = c < dv ? number<T>(b + (int64_t)c * T::kBytes) * scale : 0.0f;
#pragma unroll
        for (int i = 0; i < DT; ++i) {
            const int d0 = 16 * i + fresh(4 * lq);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int d = d0 + r;
                if (d < dk && c < dv) s[i][r] = fmaf(number<T>(a + (int64_t)d * T::kBytes), bc, scaled(s[i][r], half));
            }
        }
    }
    // sum over d of a[d] s[d][c], in every lane that has the column
    template <typename T>
    __device__ __forceinline__ float product(const char* a, int dk, int lq) const {
        float y = 0.0f;
#pragma unroll
        for (int i = 0; i < DT; ++i) {
            const int d0 = 16 * i + fresh(4 * lq);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int d = d0 + r;
                if (d < dk) y = fmaf(number<T>(a + (int64_t)d * T::kBytes), s[i][r], y);
            }
        }
        y += __shfl_xor(y, 16, kWave);
        return y + __shfl_xor(y, 32, kWave);
    }
};

// States as marks: of T, the same order.
template <typename T>
__device__ __forceinline__ void store_mark(char* p, const f32x4_t& v) {
    const float f[4] = {v[0], v[1], v[2], v[3]};
    Pack<T, 4>::store(p, Pack<T, 4>::pack(f));
}
template <typename T>
__device__ __forceinline__ f32x4_t load_mark(const char* p) {
    float f[4];
    Pack<T, 4>::unpack(Pack<T, 4>::load(p), f);
    return f32x4_t{f[0], f[1], f[2], f[3]};
}

// s += first^T (x) weighted second over the chunk's rows: rows of `a` become the state's rows, columns of `b` its columns, of which
// the wave has `mine` in `fb`; `half` are the roots of the rows' factors.
template <typename T, int DK, int DT, int KB>
__device__ __forceinline__ void add_rows(State<DT>& s, const Elem<T>* a, const Frag<T> (&fb)[KB], const float* half, float scale, int li, int lq) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
        Frag<T> parts[kParts<T>];
        float f[8];
        floats_of(fb[kb], f);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float h = half[32 * kb + 8 * lq + e];
            f[e] = f[e] * (h * scale) * h;  // (numbers, all of them: nothing to select)
        }
        wide_frag(f, parts);
#pragma unroll
        for (int i = 0; i < DT; ++i) multiply_wide(s.s[i], column_frag<kPitch<T, DK>>(a, 32 * kb, 16 * i, li, lq), parts);
    }
}
// The columns of a tile that a wave has, 32 rows at a time.
template <typename T, int PITCH, int KB>
__device__ __forceinline__ void own_columns(Frag<T> (&f)[KB], const Elem<T>* tile, int c0, int li, int lq) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) f[kb] = column_frag<PITCH>(tile, 32 * kb, c0, li, lq);
}
__device__ __forceinline__ double with_sum(double sum, double more) {
    return sum == -INFINITY || more == -INFINITY ? -INFINITY : sum + more;  // (nothing undoes a reset, NaN neither)
}
__device__ __forceinline__ double step_sum(float g) { return g < kForgets ? -INFINITY : (double)g * kLog2E; }

// ---- states at the segments' ends by themselves, of segments that have another behind them; BACK: the states' gradients at their
// beginnings, from the end on, of rows of q and columns of dy.

template <typename T, int DK, int DV, bool BACK>
__global__ __launch_bounds__(DV * 4, T::kBytes == 2 && DV == 128 ? 4 : 2) void la_ends_walk_kernel(LaArgs a) {
    constexpr int C = kChunk<T>, NT = DV * 4, KB = C / 32, DT = DK / 16;
    constexpr int PV = kPitch<T, DV>;
    __shared__ __attribute__((aligned(16))) Elem<T> tile_a[C * kPitch<T, DK>];
    __shared__ __attribute__((aligned(16))) Elem<T> tile_b[C * PV];
    __shared__ Decays<C> decays;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, li = lane % 16, lq = lane / 16;
    const Place at = place_of(a, blockIdx.x);
    if (at.segment == (BACK ? 0 : a.segments - 1)) return;
    const Rows &ra = BACK ? a.q : a.k, &rb = BACK ? a.dy : a.v;
    const char *ap = ra.p + at.b * ra.batch + at.hk * ra.head, *bp = rb.p + at.b * rb.batch + at.h * rb.head;
    const char* gp = a.g.p + at.b * a.g.batch + (int64_t)at.h * T::kBytes;
    const int c0 = at.tile * DV, cw = w * 16;  // the tile's columns, the wave's in it
    const int64_t head_state = (at.b * a.H + at.h) * a.dk_ * a.dv_, items = uniform((int32_t)(gridDim.x / (uint32_t)a.segments));
    const float scale = BACK ? a.scale : 1.0f;
    State<DT> S;
    if (!BACK && at.segment == 0 && a.state_in) S.load(a.state_in + head_state, a.dk_, a.dv_, c0 + cw + li, lq);
    else if (BACK && at.segment == a.segments - 1 && a.dstate_out) S.load(a.dstate_out + head_state, a.dk_, a.dv_, c0 + cw + li, lq);
    else S.clear();
    const int64_t first = at.segment * a.each, last = first + a.each < a.chunks ? first + a.each : a.chunks;
    double sum = 0.0;
    Ahead<T, C, DK, NT> next_a;
    Ahead<T, C, DV, NT> next_b;
    typename Pack<T, 1>::Raw next_g{};  // (64 lines of memory: the waves' that need it)
    auto steps = [&](int64_t x) { return a.L - x * C < C ? (int)(a.L - x * C) : C; };
    auto load = [&](int64_t x) {
        const int64_t t = x * C;
        const int n = steps(x);
        next_a.load(ra, ap + t * ra.step, n, 0);
        next_b.load(rb, bp + t * rb.step, n, c0);
        if (w == 0) next_g = Pack<T, 1>::load(gp + (t + min(lane, n - 1)) * a.g.step);
    };
    load(BACK ? last - 1 : first);
    for (int64_t y = first; y < last; ++y) {
        const int64_t x = BACK ? last - 1 - (y - first) : y;
        __syncthreads();  // nobody reads the chunk before any more
        bool fine = next_a.put(tile_a, a.most, ra, ap + x * C * ra.step, steps(x), 0);
        fine &= next_b.put(tile_b, a.most, rb, bp + x * C * rb.step, steps(x), c0);
        if (w == 0) fine &= make_decays<C>(decays, lane < steps(x) ? unpacked<T>(next_g) : 0.0f, lane);
        const bool at_once = !__syncthreads_or(!fine);
        if (y + 1 < last) load(BACK ? x - 1 : x + 1);
        if (at_once) {
            const int part = fresh(lane), li = part % 16, lq = part / 16;
            Frag<T> fb[KB];
            own_columns<T, PV>(fb, tile_b, cw, li, lq);
            S.decay(decays.whole);
            add_rows<T, DK>(S, tile_a, fb, BACK ? decays.from_start : decays.to_end, scale, li, lq);
            sum = with_sum(sum, decays.sum);
        } else {
            for (int i = 0, n = steps(x); i < n; ++i) {
                const int part = fresh(lane), li = part % 16, lq = part / 16;
                const int64_t t = x * C + (BACK ? n - 1 - i : i);
                const float g = number<T>(gp + t * a.g.step), half = step_factor(g);
                // (what goes back has its step's decay behind it, of what the step adds too)
                S.template step<T>(BACK ? 1.0f : half, ap + t * ra.step, bp + t * rb.step, scale, a.dk_, a.dv_, c0 + cw + li, lq);
                if constexpr (BACK) S.decay_step(half);
                sum = with_sum(sum, step_sum(g));
            }
        }
    }
    S.store_own(a.ends + (at.segment * items + at.item) * (DK * DV) + w * (DK * 16), lane);
    if (threadIdx.x == 0) a.sums[at.segment * items + at.item] = sum;
}

// ---- the walk forward: outputs, marks and the last state

template <typename T, int DK, int DV>
struct WalkLds {
    static constexpr int C = kChunk<T>;
    Elem<T> k[C * kPitch<T, DK>], v[C * kPitch<T, DV>], q[C * kPitch<T, DK>], a[C * kPitch<T, C>];
    Decays<C> d;
};

template <typename T, int DK, int DV, bool MARKS>
__global__ __launch_bounds__(DV * 4, T::kBytes == 2 && DV == 128 ? 4 : 2) void la_walk_kernel(LaArgs a) {
    constexpr int C = kChunk<T>, NW = DV / 16, NT = NW * kWave, IT = C / 16, KB = C / 32, DT = DK / 16;
    constexpr int PK = kPitch<T, DK>, PV = kPitch<T, DV>, PA = kPitch<T, C>;
    __shared__ __attribute__((aligned(16))) WalkLds<T, DK, DV> s;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, li = lane % 16, lq = lane / 16;
    const Place at = place_of(a, blockIdx.x);
    const char *kp = a.k.p + at.b * a.k.batch + at.hk * a.k.head, *vp = a.v.p + at.b * a.v.batch + at.h * a.v.head;
    const char *qp = a.q.p + at.b * a.q.batch + at.hk * a.q.head, *gp = a.g.p + at.b * a.g.batch + (int64_t)at.h * T::kBytes;
    const int c0 = at.tile * DV, cw = w * 16;  // the tile's columns, the wave's in it
    const int64_t head_state = (at.b * a.H + at.h) * a.dk_ * a.dv_, items = uniform((int32_t)(gridDim.x / (uint32_t)a.segments));
    State<DT> S;
    if (at.segment > 0) S.load_own(a.ends + ((at.segment - 1) * items + at.item) * (DK * DV) + w * (DK * 16), lane);
    else if (a.state_in) S.load(a.state_in + head_state, a.dk_, a.dv_, c0 + cw + li, lq);
    else S.clear();
    for (int i = threadIdx.x; i < C * PA; i += NT) s.a[i] = 0;  // (blocks above the diagonal are read, as zeros)
    const int64_t first = at.segment * a.each, last = first + a.each < a.chunks ? first + a.each : a.chunks;
    Ahead<T, C, DK, NT> next_q, next_k;
    Ahead<T, C, DV, NT> next_v;
    typename Pack<T, 1>::Raw next_g{};  // (64 lines of memory: the waves' that need it)
    auto steps = [&](int64_t x) { return a.L - x * C < C ? (int)(a.L - x * C) : C; };
    auto load = [&](int64_t x) {
        const int64_t t = x * C;
        const int n = steps(x);
        next_k.load(a.k, kp + t * a.k.step, n, 0);
        next_q.load(a.q, qp + t * a.q.step, n, 0);
        next_v.load(a.v, vp + t * a.v.step, n, c0);
        if (w == 0) next_g = Pack<T, 1>::load(gp + (t + min(lane, n - 1)) * a.g.step);
    };
    load(first);
    for (int64_t x = first; x < last; ++x) {
        if constexpr (MARKS) {
            char* const m = a.marks + ((at.item * a.chunks + x) * (DK * DV) + w * (DK * 16)) * T::kBytes;
            const int part = fresh(lane);
#pragma unroll
            for (int i = 0; i < DT; ++i) store_mark<T>(m + (i * kWave + part) * 4 * T::kBytes, S.s[i]);
        }
        const int64_t t = x * C;
        const int n = steps(x);
        __syncthreads();  // nobody reads the chunk before any more
        bool fine = next_k.put(s.k, a.most, a.k, kp + t * a.k.step, n, 0);
        fine &= next_q.put(s.q, a.most, a.q, qp + t * a.q.step, n, 0);
        fine &= next_v.put(s.v, a.most, a.v, vp + t * a.v.step, n, c0);
        if (w == 0) fine &= make_decays<C>(s.d, lane < n ? unpacked<T>(next_g) : 0.0f, lane);
        fine &= !S.large();
        const bool at_once = !__syncthreads_or(!fine);
        if (x + 1 < last) load(x + 1);
        if (!at_once) {
            for (int i = 0; i < n; ++i) {
                const int part = fresh(lane), li = part % 16, lq = part / 16;
                const int64_t u = t + i;
                S.template step<T>(step_factor(number<T>(gp + u * a.g.step)), kp + u * a.k.step, vp + u * a.v.step, 1.0f, a.dk_, a.dv_, c0 + cw + li, lq);
                const int c = c0 + cw + li;
                const float one[1] = {S.template product<T>(qp + u * a.q.step, a.dk_, lq) * a.scale};
                if (lq == 0 && c < a.dv_) Pack<T, 1>::store(a.y + (((at.b * a.L + u) * a.H + at.h) * a.dv_ + c) * T::kBytes, Pack<T, 1>::pack(one));
            }
            continue;
        }
        // A below the diagonal, a block of 16 x 16 a wave at a time
        constexpr int kBlocks = IT * (IT + 1) / 2;
#pragma unroll 1
        for (int y = 0; y < (kBlocks + NW - 1) / NW; ++y) {
            const int part = fresh(lane), li = part % 16, lq = part / 16;  // (addresses of one phase at a time)
            const int block = y * NW + w;
            if (block >= kBlocks) break;
            int it = 0;
            while ((it + 1) * (it + 2) / 2 <= block) ++it;
            const int jt = block - it * (it + 1) / 2;
            f32x4_t p = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int kb = 0; kb < DK / 32; ++kb)
                multiply(p, row_frag<PK>(s.k, 16 * jt + li, 32 * kb, lq), row_frag<PK>(s.q, 16 * it + li, 32 * kb, lq));
            const int i = 16 * it + li, j0 = 16 * jt + 4 * lq, forgot = s.d.forgot[i];
            const float hi = s.d.hi[i], lo = s.d.lo[i];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float half = __builtin_amdgcn_exp2f((hi - s.d.hi[j0 + r]) + (lo - s.d.lo[j0 + r]));
                p[r] = j0 + r <= i && j0 + r >= forgot ? p[r] * (half * a.scale) * half : 0.0f;
            }
            put4(s.a + i * PA + j0, p);
        }
        Frag<T> fv[KB];
        {
            const int part = fresh(lane), li = part % 16, lq = part / 16;
            own_columns<T, PV>(fv, s.v, cw, li, lq);
        }
        Frag<T> fs[DK / 32];  // the state as an operand
#pragma unroll
        for (int y = 0; y < DK / 32; ++y) {
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = S.s[2 * y + e / 4][e % 4];
            fs[y] = frag_of(f, T{});
        }
        char* const y_rows = a.y + ((at.b * a.L + t) * a.H + at.h) * a.dv_ * T::kBytes;
        const uint32_t v_row = (uint32_t)a.H * (uint32_t)a.dv_ * T::kBytes;
        __syncthreads();  // A is there
#pragma unroll 1
        for (int it = 0; it < IT; ++it) {
            const int part = fresh(lane), li = part % 16, lq = part / 16;
            const int i = 16 * it + li;
            f32x4_t o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int y = 0; y < DK / 32; ++y) multiply(o, fs[y], turned_row_frag<PK>(s.q, i, 32 * y, lq));
            const float half = s.d.from_start[i], first = half * a.scale;
#pragma unroll
            for (int r = 0; r < 4; ++r) o[r] = half == 0.0f ? 0.0f : o[r] * first * half;
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                if (kb > it / 2) break;
                multiply(o, fv[kb], row_frag<PA>(s.a, i, 32 * kb, lq));
            }
            const int c = c0 + cw + 4 * lq;
            if (i < n && c < a.dv_) {
                char* const to = y_rows + (uint64_t)(uint32_t)i * v_row + (uint32_t)c * T::kBytes;
                const float f[4] = {o[0], o[1], o[2], o[3]};
                if (a.dv_ % 4 == 0) {
                    Pack<T, 4>::store(to, Pack<T, 4>::pack(f));
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (c + r < a.dv_) {
                            const float one[1] = {f[r]};
                            Pack<T, 1>::store(to + r * T::kBytes, Pack<T, 1>::pack(one));
                        }
                }
            }
        }
        S.decay(s.d.whole);
        {
            const int part = fresh(lane), li = part % 16, lq = part / 16;
            add_rows<T, DK>(S, s.k, fv, s.d.to_end, 1.0f, li, lq);
        }
    }
    if (at.segment == a.segments - 1 && a.state_out) S.store(a.state_out + head_state, a.dk_, a.dv_, c0 + cw + li, lq);
}

// Ends of segments made by themselves -> ends of everything up to them (BACK: from them on): e[s] += decay of s * e[s - 1].
template <bool BACK>
__global__ __launch_bounds__(256) void la_ends_kernel(float* ends, const double* sums, int64_t items, int32_t size, int32_t segments) {
    constexpr int kAtOnce = 8;
    const int64_t n = items * (size / 4);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t item = i / (size / 4);
        float4 e = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int x0 = 0; x0 < segments - 1; x0 += kAtOnce) {  // (nothing comes behind the last)
            float4 own[kAtOnce];
            double d[kAtOnce];
#pragma unroll
            for (int y = 0; y < kAtOnce; ++y) {
                const int x = x0 + y < segments - 1 ? x0 + y : segments - 2, at = BACK ? segments - 1 - x : x;
                own[y] = reinterpret_cast<const float4*>(ends)[at * n + i];
                d[y] = sums[at * items + item];
            }
#pragma unroll
            for (int y = 0; y < kAtOnce; ++y) {
                const int x = x0 + y, at = BACK ? segments - 1 - x : x;
                if (x >= segments - 1) break;
                const float half = d[y] == -INFINITY ? 0.0f : half_factor((float)d[y]);
                e.x = scaled(e.x, half) + own[y].x, e.y = scaled(e.y, half) + own[y].y;
                e.z = scaled(e.z, half) + own[y].z, e.w = scaled(e.w, half) + own[y].w;
                reinterpret_cast<float4*>(ends)[at * n + i] = e;
            }
        }
    }
}

// ---- the backward walk

template <typename T, int DK, int DV>
struct BwdLds {
    static constexpr int C = kChunk<T>, NW = DV / 16, PK = kPitch<T, DK>;
    // the state in front of the chunk and the gradient of that behind it, turned; fp32: one after the other in one place
    static constexpr bool kTwo = T::kBytes == 2;
    Elem<T> q[C * PK], k[C * PK], v[C * kPitch<T, DV>], dy[C * kPitch<T, DV>];
    Elem<T> a[C * kPitch<T, C>], e[C * kPitch<T, C>];  // A and its gradient's part for q and k, this below its diagonal
    float self[C];                                     // and on it
    Elem<T> s[DV * PK], m[kTwo ? DV * PK : 1];
    float near[DK / 16][C], far[DK / 16][C];  // shares of the log decays' gradients
    float both[NW];                           // <S, M>
    Decays<C> d;
};
static_assert(sizeof(BwdLds<BF16, 128, 128>) <= 160 * 1024 && sizeof(BwdLds<F32, 128, 128>) <= 160 * 1024, "what a compute unit has");

// Sum over the lanes li + 16, + 32, + 48.
__device__ __forceinline__ float over_quarters(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
// Sum over 16 lanes next to each other, in the last of them.
__device__ __forceinline__ float over_columns(float x) {
    x += moved<0x111, 0xf>(x);
    x += moved<0x112, 0xf>(x);
    x += moved<0x114, 0xf>(x);
    return x + moved<0x118, 0xf>(x);
}
template <typename T>
__device__ __forceinline__ f32x4_t four(const Elem<T>* p) {
    float f[4];
    Pack<T, 4>::unpack(Pack<T, 4>::load(p), f);
    return f32x4_t{f[0], f[1], f[2], f[3]};
}
__device__ __forceinline__ float dot(const f32x4_t& a, const f32x4_t& b) { return fmaf(a[0], b[0], fmaf(a[1], b[1], fmaf(a[2], b[2], a[3] * b[3]))); }

// For every chunk, from what lies in LDS and M in registers: A and E below the diagonal; dv = to_end k M + A^T dy;
// dq = from_start scale dy S^T + E k; dk = to_end v M^T + E^T q; and M itself.  dg needs no products of its own: the pairs of steps on both
// sides of a decay are what q . dq and k . dk add up to on both sides of it, but for what a step says to itself (E's diagonal, kept apart: it
// reaches over no decay, and would leave its rounding where the decays leave little).  160 KB of LDS leave room for one workgroup of 8 waves on a
// compute unit: vector instructions 43% busy, LDS 37% (of which 42% are conflicts), matrix cores 13%.  dq and dk of heads that share q and k go to shares in fp32 and are
// summed afterwards in a fixed order (32768 steps, 16 heads of 64 x 128 by four: 25 us each).
template <typename T, int DK, int DV, bool SHARES>
__global__ __launch_bounds__(DV * 4, 2) void la_bwd_kernel(LaArgs a) {
    using Lds = BwdLds<T, DK, DV>;
    constexpr int C = kChunk<T>, NW = DV / 16, NT = NW * kWave, IT = C / 16, KB = C / 32, DT = DK / 16, VB = DV / 32;
    constexpr int PK = kPitch<T, DK>, PV = kPitch<T, DV>, PA = kPitch<T, C>;
    __shared__ __attribute__((aligned(16))) Lds s;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, li = lane % 16, lq = lane / 16;
    const Place at = place_of(a, blockIdx.x);
    const char *kp = a.k.p + at.b * a.k.batch + at.hk * a.k.head, *vp = a.v.p + at.b * a.v.batch + at.h * a.v.head;
    const char *qp = a.q.p + at.b * a.q.batch + at.hk * a.q.head, *dyp = a.dy.p + at.b * a.dy.batch + at.h * a.dy.head;
    const char* gp = a.g.p + at.b * a.g.batch + (int64_t)at.h * T::kBytes;
    const int c0 = at.tile * DV, cw = w * 16;
    const int64_t items = uniform((int32_t)(gridDim.x / (uint32_t)a.segments)), head_state = (at.b * a.H + at.h) * a.dk_ * a.dv_;
    const int own = w * (DK * 16) + lane * 4;  // this lane's numbers in states of the library's own order, piece by piece
    constexpr int kStep = kWave * 4;
    State<DT> M;  // the gradient of the state behind the chunk
    if (at.segment < a.segments - 1) {
        const float* p = a.ends + ((int64_t)(at.segment + 1) * a.finer * items + at.item) * (DK * DV) + own;
#pragma unroll
        for (int i = 0; i < DT; ++i) M.s[i] = *reinterpret_cast<const f32x4_t*>(p + i * kStep);
    } else if (a.dstate_out) {
        M.load(a.dstate_out + head_state, a.dk_, a.dv_, c0 + cw + li, lq);
    } else {
        M.clear();
    }
    for (int i = threadIdx.x; i < C * PA; i += NT) s.a[i] = 0, s.e[i] = 0;  // (blocks above the diagonal are read, as zeros)
    const int64_t first = at.segment * a.each, last = first + a.each < a.chunks ? first + a.each : a.chunks;
    const int64_t heads_qk = a.H / a.group, rows_all = items / a.tiles / a.H * a.L;  // B L
    const int64_t share = SHARES ? ((int64_t)(at.h % a.group) * a.tiles + at.tile) * (rows_all * heads_qk * a.dk_) : 0;

    // `count` numbers of a row of dq or dk from d on: row i of those from step t on
    using O = std::conditional_t<SHARES, F32, T>;
    const uint32_t k_row = (uint32_t)heads_qk * (uint32_t)a.dk_ * O::kBytes, v_row = (uint32_t)a.H * (uint32_t)a.dv_ * T::kBytes;
    auto give = [&](void* base, int64_t t, int i, int d, const float* v, auto count) {
        constexpr int N = decltype(count)::value;
        if (d >= a.dk_) return;
        char* p = static_cast<char*>(base) + (share + ((at.b * a.L + t) * heads_qk + at.hk) * a.dk_) * O::kBytes;
        p += (uint64_t)(uint32_t)i * k_row + (uint32_t)d * O::kBytes;
        if (N > 1 && a.dk_ % 4 == 0) {
            float f[N];
#pragma unroll
            for (int r = 0; r < N; ++r) f[r] = v[r];
            Pack<O, N>::store(p, Pack<O, N>::pack(f));
        } else {
#pragma unroll
            for (int r = 0; r < N; ++r)
                if (d + r < a.dk_) {
                    const float one[1] = {v[r]};
                    Pack<O, 1>::store(p + r * O::kBytes, Pack<O, 1>::pack(one));
                }
        }
    };
    auto give_four = [&](void* base, int64_t t, int i, int d, const f32x4_t& v) {
        const float f[4] = {v[0], v[1], v[2], v[3]};
        give(base, t, i, d, f, std::integral_constant<int, 4>{});
    };
    auto give_decay = [&](int64_t t, float x) {
        const float one[1] = {x};
        const int64_t e = (at.b * a.L + t) * a.H + at.h;
        if (a.tiles > 1) static_cast<float*>(a.dg)[at.tile * (rows_all * a.H) + e] = x;
        else Pack<T, 1>::store(static_cast<char*>(a.dg) + e * T::kBytes, Pack<T, 1>::pack(one));
    };
    auto dv_row = [&](int64_t t) { return a.dv + ((at.b * a.L + t) * a.H + at.h) * a.dv_ * T::kBytes; };
    auto steps = [&](int64_t x) { return a.L - x * C < C ? (int)(a.L - x * C) : C; };

    Ahead<T, C, DK, NT> next_q, next_k;
    Ahead<T, C, DV, NT> next_v, next_dy;
    typename Pack<T, 4>::Raw next_s[DT];
    typename Pack<T, 1>::Raw next_g{};  // (64 lines of memory: the waves' that need it)
    float g_now = 0.0f;
    auto load = [&](int64_t x) {
        const int64_t t = x * C;
        const int n = steps(x);
        next_q.load(a.q, qp + t * a.q.step, n, 0);
        next_k.load(a.k, kp + t * a.k.step, n, 0);
        next_v.load(a.v, vp + t * a.v.step, n, c0);
        next_dy.load(a.dy, dyp + t * a.dy.step, n, c0);
        const char* p = a.marks_in + ((at.item * a.chunks + x) * (DK * DV) + own) * T::kBytes;
#pragma unroll
        for (int i = 0; i < DT; ++i) next_s[i] = Pack<T, 4>::load(p + i * kStep * T::kBytes);
        if (w == 0 || w == NW - 1) next_g = Pack<T, 1>::load(gp + (t + min(lane, n - 1)) * a.g.step);
    };
    // The last wave's: gradients of the log decays of a chunk that was taken at once.  Pairs of steps on both sides of decay t: those
    // with an earlier step in front of the chunk and a later one behind it; those with a later one behind it; of those inside the
    // chunk or with an earlier step in front of it, all whose later step is from t on less those whose earlier step is, too.
    int64_t done = -1;
    auto give_decays = [&]() {
        if (done < 0 || w != NW - 1) return;
        double near = 0.0, far = 0.0, both = 0.0;
        if (lane < C) {
#pragma unroll
            for (int y = 0; y < DT; ++y) near += (double)s.near[y][lane], far += (double)s.far[y][lane];
        }
#pragma unroll
        for (int y = 0; y < NW; ++y) both += (double)s.both[y];
        double before = __shfl_up(wave_upto(far), 1, kWave);  // (not the sum with its own less its own, which may be all there is)
        if (lane == 0) before = 0.0;
        // (from behind: what is not finite stays in front of itself)
        const int turn = kWave - 1 - lane;
        const double from = __shfl(wave_upto((double)__shfl(near, turn, kWave)), turn, kWave);
        const int64_t t = done * C + lane;
        if (lane < steps(done)) give_decay(t, g_now < kForgets ? 0.0f : (float)(from + before + both));
    };
    load(last - 1);
    for (int64_t x = last - 1; x >= first; --x) {
        const int64_t t = x * C;
        const int n = steps(x);
        __syncthreads();  // nobody reads the chunk behind any more
        give_decays();
        bool fine = next_q.put(s.q, a.most, a.q, qp + t * a.q.step, n, 0);
        fine &= next_k.put(s.k, a.most, a.k, kp + t * a.k.step, n, 0);
        fine &= next_v.put(s.v, a.most, a.v, vp + t * a.v.step, n, c0);
        fine &= next_dy.put(s.dy, a.most, a.dy, dyp + t * a.dy.step, n, c0);
        {
            Elem<T>* p = s.s + (cw + li) * PK + 4 * lq;
#pragma unroll
            for (int i = 0; i < DT; ++i) {
                store_words<Pack<T, 4>::kWords>(p + 16 * i, next_s[i]);
                if constexpr (Lds::kTwo) put4(s.m + (cw + li) * PK + 16 * i + 4 * lq, M.s[i]);
            }
        }
        g_now = lane < n ? unpacked<T>(next_g) : 0.0f;
        if (w == 0) fine &= make_decays<C>(s.d, g_now, lane);
        float both = 0.0f;  // <S, M>
        {
            State<DT> S;
#pragma unroll
            for (int i = 0; i < DT; ++i) {
                float f[4];
                Pack<T, 4>::unpack(next_s[i], f);
#pragma unroll
                for (int r = 0; r < 4; ++r) S.s[i][r] = f[r], both = fmaf(f[r], M.s[i][r], both);
            }
            fine &= !M.large() && !S.large();
        }
        both = wave_upto(both);
        const bool at_once = !__syncthreads_or(!fine);
        if (lane == kWave - 1) s.both[w] = scaled(both, s.d.whole);
        if (x > first) load(x - 1);
        done = -1;
        if (!at_once) {
            float *const sum_q = reinterpret_cast<float*>(s.q), *const sum_k = reinterpret_cast<float*>(s.k);
            const char* mark = a.marks_in + ((at.item * a.chunks + x) * (DK * DV) + own) * T::kBytes;
            for (int i = n - 1; i >= 0; --i) {
                const int part = fresh(lane), li = part % 16, lq = part / 16, c = c0 + cw + li;
                const int64_t u = t + i;
                State<DT> S;
#pragma unroll
                for (int y = 0; y < DT; ++y) S.s[y] = load_mark<T>(mark + y * kStep * T::kBytes);
                for (int64_t z = t; z < u; ++z)
                    S.template step<T>(step_factor(number<T>(gp + z * a.g.step)), kp + z * a.k.step, vp + z * a.v.step, 1.0f, a.dk_, a.dv_, c0 + cw + li, lq);
                const float half = step_factor(number<T>(gp + u * a.g.step));
                M.template step<T>(1.0f, qp + u * a.q.step, dyp + u * a.dy.step, a.scale, a.dk_, a.dv_, c0 + cw + li, lq);
                float both = 0.0f;
                if (half != 0.0f)
#pragma unroll
                    for (int y = 0; y < DT; ++y)
#pragma unroll
                        for (int r = 0; r < 4; ++r) both = fmaf(scaled(S.s[y][r], half), M.s[y][r], both);
                S.template step<T>(half, kp + u * a.k.step, vp + u * a.v.step, 1.0f, a.dk_, a.dv_, c0 + cw + li, lq);
                const float dv[1] = {M.template product<T>(kp + u * a.k.step, a.dk_, lq)};
                const float dyc = c < a.dv_ ? number<T>(dyp + u * a.dy.step + (int64_t)c * T::kBytes) * a.scale : 0.0f;
                const float vc = c < a.dv_ ? number<T>(vp + u * a.v.step + (int64_t)c * T::kBytes) : 0.0f;
                if (lq == 0 && c < a.dv_) Pack<T, 1>::store(dv_row(u) + c * T::kBytes, Pack<T, 1>::pack(dv));
                __syncthreads();  // the step behind has been given
                both = of_lane(wave_upto(both), kWave - 1);
                if (lane == 0) s.both[w] = both;
#pragma unroll
                for (int y = 0; y < DT; ++y) {
                    const int d0 = 16 * y + fresh(4 * lq);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {  // (columns behind the last add nothing)
                        const float fq = over_columns(c < a.dv_ ? S.s[y][r] * dyc : 0.0f), fk = over_columns(c < a.dv_ ? M.s[y][r] * vc : 0.0f);
                        if (li == 15) sum_q[w * DK + d0 + r] = fq, sum_k[w * DK + d0 + r] = fk;
                    }
                }
                __syncthreads();
                const int d = threadIdx.x;
                if (d < DK) {
                    float fq[1] = {0.0f}, fk[1] = {0.0f};
                    for (int y = 0; y < NW; ++y) fq[0] += sum_q[y * DK + d], fk[0] += sum_k[y * DK + d];
                    give(a.dq, u, 0, d, fq, std::integral_constant<int, 1>{});
                    give(a.dk, u, 0, d, fk, std::integral_constant<int, 1>{});
                }
                if (threadIdx.x == 0) {
                    float f = 0.0f;
                    for (int y = 0; y < NW; ++y) f += s.both[y];
                    give_decay(u, f);
                }
                M.decay_step(half);
            }
            continue;
        }
        done = x;
        // A, and its gradient's part E_ij = scale exp(b_i - b_j) (dy_i . v_j)
        constexpr int kBlocks = IT * (IT + 1) / 2;
#pragma unroll 1
        for (int y = 0; y < (kBlocks + NW - 1) / NW; ++y) {
            const int part = fresh(lane), li = part % 16, lq = part / 16;  // (addresses of one phase at a time)
            const int block = y * NW + w;
            if (block >= kBlocks) break;
            int it = 0;
            while ((it + 1) * (it + 2) / 2 <= block) ++it;
            const int jt = block - it * (it + 1) / 2;
            f32x4_t p = {0.0f, 0.0f, 0.0f, 0.0f}, e = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int kb = 0; kb < DK / 32; ++kb)
                multiply(p, row_frag<PK>(s.k, 16 * jt + li, 32 * kb, lq), row_frag<PK>(s.q, 16 * it + li, 32 * kb, lq));
#pragma unroll
            for (int kb = 0; kb < VB; ++kb)
                multiply(e, row_frag<PV>(s.v, 16 * jt + li, 32 * kb, lq), row_frag<PV>(s.dy, 16 * it + li, 32 * kb, lq));
            const int i = 16 * it + li, j0 = 16 * jt + 4 * lq, forgot = s.d.forgot[i];
            const float hi = s.d.hi[i], lo = s.d.lo[i];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const bool in = j0 + r <= i && j0 + r >= forgot;
                const float half = __builtin_amdgcn_exp2f((hi - s.d.hi[j0 + r]) + (lo - s.d.lo[j0 + r])), first = half * a.scale;
                p[r] = in ? p[r] * first * half : 0.0f;
                e[r] = in ? e[r] * first * half : 0.0f;
            }
            if (it == jt)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (j0 + r == i) s.self[i] = e[r], e[r] = 0.0f;
            put4(s.a + i * PA + j0, p);
            put4(s.e + i * PA + j0, e);
        }
        // dv of the wave's columns from M in registers
        f32x4_t dv[IT];
        {
            const int part = fresh(lane), li = part % 16, lq = part / 16;
            Frag<T> fm[DK / 32];
#pragma unroll
            for (int y = 0; y < DK / 32; ++y) {
                float f[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = M.s[2 * y + e / 4][e % 4];
                fm[y] = frag_of(f, T{});
            }
#pragma unroll
            for (int jt = 0; jt < IT; ++jt) {
                dv[jt] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int y = 0; y < DK / 32; ++y) multiply(dv[jt], fm[y], turned_row_frag<PK>(s.k, 16 * jt + li, 32 * y, lq));
                const float half = s.d.to_end[16 * jt + li];
#pragma unroll
                for (int r = 0; r < 4; ++r) dv[jt][r] = scaled(dv[jt][r], half);
            }
        }
        __syncthreads();  // A and E are there
        Frag<T> fdy[KB];
        {
            const int part = fresh(lane), li = part % 16, lq = part / 16;
            own_columns<T, PV>(fdy, s.dy, cw, li, lq);
        }
#pragma unroll
        for (int jt = 0; jt < IT; ++jt) {
            const int part = fresh(lane), li = part % 16, lq = part / 16;
#pragma unroll
            for (int kb = jt / 2; kb < KB; ++kb) multiply(dv[jt], fdy[kb], column_frag<PA>(s.a, 32 * kb, 16 * jt, li, lq));
            const int j = 16 * jt + li, c = c0 + cw + 4 * lq;
            if (j < n && c < a.dv_) {
                const float f[4] = {dv[jt][0], dv[jt][1], dv[jt][2], dv[jt][3]};
                char* p = dv_row(t) + (uint64_t)(uint32_t)j * v_row + (uint32_t)c * T::kBytes;
                if (a.dv_ % 4 == 0) {
                    Pack<T, 4>::store(p, Pack<T, 4>::pack(f));
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (c + r < a.dv_) {
                            const float one[1] = {f[r]};
                            Pack<T, 1>::store(p + r * T::kBytes, Pack<T, 1>::pack(one));
                        }
                }
            }
        }
        // dq and dk: a wave has blocks of 16 rows, every NW / kBand-th, by 16 numbers of every kBand-th
        constexpr int kBand = NW < DT ? NW : DT, kRows = (IT * kBand + NW - 1) / NW;
        float near[DT / kBand][kRows];
#pragma unroll
        for (int y = 0; y < DT / kBand; ++y) {
            const int part = fresh(lane), li = part % 16, lq = part / 16;
            const int dt = y * kBand + w % kBand;
            Frag<T> fs[VB], fk[KB];
#pragma unroll
            for (int kb = 0; kb < VB; ++kb) fs[kb] = column_frag<PK>(s.s, 32 * kb, 16 * dt, li, lq);
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) fk[kb] = column_frag<PK>(s.k, 32 * kb, 16 * dt, li, lq);
#pragma unroll
            for (int z = 0; z < kRows; ++z) {
                const int it = z * (NW / kBand) + w / kBand, i = 16 * it + li;
                if (it >= IT) continue;
                f32x4_t o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int kb = 0; kb < VB; ++kb) multiply(o, fs[kb], row_frag<PV>(s.dy, i, 32 * kb, lq));
                const float half = s.d.from_start[i], first = half * a.scale;
#pragma unroll
                for (int r = 0; r < 4; ++r) o[r] = half == 0.0f ? 0.0f : o[r] * first * half;
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
                    if (kb <= it / 2) multiply(o, fk[kb], row_frag<PA>(s.e, i, 32 * kb, lq));
                near[y][z] = dot(four<T>(s.q + i * PK + 16 * dt + 4 * lq), o);
                o += s.self[i] * four<T>(s.k + i * PK + 16 * dt + 4 * lq);
                if (i < n) give_four(a.dq, t, i, 16 * dt + 4 * lq, o);
                __builtin_amdgcn_sched_barrier(0);  // (blocks side by side need more registers than there are)
            }
        }
        if constexpr (!Lds::kTwo) {
            __syncthreads();  // S has been read
#pragma unroll
            for (int i = 0; i < DT; ++i) put4(s.s + (cw + li) * PK + 16 * i + 4 * lq, M.s[i]);
            __syncthreads();
        }
        const Elem<T>* const sm_t = Lds::kTwo ? s.m : s.s;
#pragma unroll
        for (int y = 0; y < DT / kBand; ++y) {
            const int part = fresh(lane), li = part % 16, lq = part / 16;
            const int dt = y * kBand + w % kBand;
            Frag<T> fm[VB], fq[KB];
#pragma unroll
            for (int kb = 0; kb < VB; ++kb) fm[kb] = column_frag<PK>(sm_t, 32 * kb, 16 * dt, li, lq);
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) fq[kb] = column_frag<PK>(s.q, 32 * kb, 16 * dt, li, lq);
#pragma unroll
            for (int z = 0; z < kRows; ++z) {
                const int jt = z * (NW / kBand) + w / kBand, j = 16 * jt + li;
                if (jt >= IT) continue;
                f32x4_t o = {0.0f, 0.0f, 0.0f, 0.0f}, o2 = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int kb = 0; kb < VB; ++kb) multiply(o, fm[kb], row_frag<PV>(s.v, j, 32 * kb, lq));
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
                    if (kb >= jt / 2) multiply(o2, fq[kb], column_frag<PA>(s.e, 32 * kb, 16 * jt, li, lq));
                const float half = s.d.to_end[j];
#pragma unroll
                for (int r = 0; r < 4; ++r) o[r] = scaled(o[r], half);
                const f32x4_t k4 = four<T>(s.k + j * PK + 16 * dt + 4 * lq);
                const float far = over_quarters(dot(k4, o)), less = over_quarters(near[y][z] - dot(k4, o2));
                if (lq == 0) s.far[dt][j] = far, s.near[dt][j] = less;
                o += o2 + s.self[j] * four<T>(s.q + j * PK + 16 * dt + 4 * lq);
                if (j < n) give_four(a.dk, t, j, 16 * dt + 4 * lq, o);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        M.decay(s.d.whole);
        {
            const int part = fresh(lane), li = part % 16, lq = part / 16;
            add_rows<T, DK>(M, s.q, fdy, s.d.from_start, a.scale, li, lq);
        }
    }
    __syncthreads();
    give_decays();
    if (at.segment == 0 && a.dstate_in) M.store(a.dstate_in + head_state, a.dk_, a.dv_, c0 + cw + li, lq);
}

// out[r][d] = sum over the shares: heads that share a row of q and k, and tiles of their columns; [share][rows].
template <typename T, int VEC>
__global__ __launch_bounds__(256) void la_shares_kernel(const float* shares, void* out, int64_t n, int32_t count) {
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * VEC; i < n; i += (int64_t)gridDim.x * 256 * VEC) {
        float sum[VEC] = {};
        for (int x = 0; x < count; ++x) {
            float f[VEC];
            Pack<F32, VEC>::unpack(Pack<F32, VEC>::load_nt(shares + x * n + i), f);
#pragma unroll
            for (int j = 0; j < VEC; ++j) sum[j] += f[j];
        }
        Pack<T, VEC>::store(static_cast<char*>(out) + i * T::kBytes, Pack<T, VEC>::pack(sum));
    }
}

__global__ __launch_bounds__(256) void la_copy_kernel(const float* from, float* to, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) to[i] = from ? from[i] : 0.0f;
}

// ---- one token: the state, read and written, is what it costs (64 x 32 heads of 128 x 128: 268 MB in 50 us).  A workgroup has 4 CL columns
// of a head's state (VEC = 1: CL), a lane VEC of them in every (256 / CL)-th row.
struct StepArgs {
    const char *q, *k, *v, *g;
    char* y;
    float* state;
    int32_t H, group, dk, dv, slices;
    float scale;
};
template <typename T, int CL, int VEC, bool STREAM>
__global__ __launch_bounds__(256) void la_step_kernel(StepArgs a) {
    constexpr int kRows = 256 / CL;
    __shared__ float sum[kRows][CL * VEC];
    const int cl = threadIdx.x % CL, row = threadIdx.x / CL;
    const int64_t bh = blockIdx.x / (uint32_t)a.slices, b = bh / a.H;
    const int h = (int)(bh % a.H), c = ((int)(blockIdx.x % (uint32_t)a.slices) * CL + cl) * VEC;
    const int64_t qk = (b * (a.H / a.group) + h / a.group) * a.dk;
    const float half = step_factor(number<T>(a.g + bh * T::kBytes));
    float v[VEC] = {}, y[VEC] = {};
    if (c < a.dv) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) v[j] = number<T>(a.v + (bh * a.dv + c + j) * T::kBytes);
        float* const p = a.state + bh * a.dk * a.dv + c;
#pragma unroll 8
        for (int d = row; d < a.dk; d += kRows) {
            float s[VEC];
            Pack<F32, VEC>::unpack(STREAM ? Pack<F32, VEC>::load_nt(p + (int64_t)d * a.dv) : Pack<F32, VEC>::load(p + (int64_t)d * a.dv), s);
            const float k = number<T>(a.k + (qk + d) * T::kBytes), q = number<T>(a.q + (qk + d) * T::kBytes);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                s[j] = scaled(s[j], half) + k * v[j];
                y[j] = fmaf(q, s[j], y[j]);
            }
            Pack<F32, VEC>::store(p + (int64_t)d * a.dv, Pack<F32, VEC>::pack(s));
        }
    }
#pragma unroll
    for (int j = 0; j < VEC; ++j) sum[row][cl * VEC + j] = y[j];
    __syncthreads();
    const int i = threadIdx.x, at = (int)(blockIdx.x % (uint32_t)a.slices) * (CL * VEC) + i;
    if (i < CL * VEC && at < a.dv) {
        float f = 0.0f;
#pragma unroll
        for (int r = 0; r < kRows; ++r) f += sum[r][i];
        const float one[1] = {f * a.scale};
        Pack<T, 1>::store(a.y + (bh * a.dv + at) * T::kBytes, Pack<T, 1>::pack(one));
    }
}

// ---- sizes

int chunk_of(const LaShape& s) { return s.dtype == HY_F32 ? kChunk<F32> : kChunk<BF16>; }
int64_t chunks_of(const LaShape& s) { return (s.L + chunk_of(s) - 1) / chunk_of(s); }
int tile_rows(const LaShape& s) { return s.dk > 64 ? 128 : 64; }     // DK
int tile_columns(const LaShape& s) { return s.dv > 64 ? 128 : 64; }  // DV
int64_t tiles_of(const LaShape& s) { return (s.dv + tile_columns(s) - 1) / tile_columns(s); }
int64_t items_of(const LaShape& s) { return s.B * s.H * tiles_of(s); }
int64_t state_size(const LaShape& s) { return (int64_t)tile_rows(s) * tile_columns(s); }

// Segments of a sequence, so that `want` workgroups are there, of 4 chunks at the least (2: the same time where heads are few).
struct Cut {
    int64_t segments, each;
};
Cut cut(const LaShape& s, int64_t want) {
    const int64_t chunks = chunks_of(s), items = items_of(s);
    int64_t n = (want + items - 1) / items;
    if (n > (chunks + 3) / 4) n = (chunks + 3) / 4;
    if (n < 1) n = 1;
    const int64_t each = (chunks + n - 1) / n;
    return Cut{(chunks + each - 1) / each, each};
}
constexpr int64_t kForwardGroups = 512, kBackwardGroups = 256;

int64_t ends_bytes(const LaShape& s, const Cut& c) {
    return c.segments > 1 ? c.segments * items_of(s) * (state_size(s) * 4 + 8) : 0;
}
int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }

Rows rows_of(const void* p, const LaShape& s, int which, int64_t d) {
    const int64_t e = s.dtype == HY_F32 ? 4 : 2;
    const int64_t* st = s.stride[which];
    const bool wide = d % 8 == 0 && reinterpret_cast<uintptr_t>(p) % 16 == 0 && st[0] * e % 16 == 0 && st[1] * e % 16 == 0 && st[2] * e % 16 == 0 &&
                      st[1] < (INT64_C(1) << 24);  // (a chunk's rows within 2^32 bytes)
    return Rows{static_cast<const char*>(p), st[0] * e, st[1] * e, st[2] * e, (int32_t)d, wide};
}

LaArgs args_of(const LaPtrs& p, const LaShape& s) {
    LaArgs a{};
    a.q = rows_of(p.q, s, kLaQ, s.dk), a.k = rows_of(p.k, s, kLaK, s.dk), a.v = rows_of(p.v, s, kLaV, s.dv);
    a.g = rows_of(p.g, s, kLaG, 1), a.dy = rows_of(p.dy, s, kLaDy, s.dv);
    a.state_in = p.state_in, a.dstate_out = p.dstate_out;
    a.y = static_cast<char*>(p.y), a.state_out = p.state_out, a.dstate_in = p.dstate_in;
    a.L = s.L, a.chunks = chunks_of(s);
    a.H = (int32_t)s.H, a.group = s.group, a.dk_ = (int32_t)s.dk, a.dv_ = (int32_t)s.dv, a.tiles = (int32_t)tiles_of(s);
    a.scale = (float)s.scale;
    const float most = fabsf(a.scale) <= 1.0f ? kMostNumber : kMostNumber / fabsf(a.scale);  // (NaN: none is below)
    static_assert(sizeof(most) == sizeof(a.most), "its bits");
    if (most > 0.0f) memcpy(&a.most, &most, sizeof most);
    return a;
}

// f<T, DK, DV>
template <typename F>
hy_status by_tile(const LaShape& s, F&& f) {
    using std::integral_constant;
    auto columns = [&](auto t, auto dk) {
        return tile_columns(s) == 128 ? f(t, dk, integral_constant<int, 128>{}) : f(t, dk, integral_constant<int, 64>{});
    };
    auto rows = [&](auto t) { return tile_rows(s) == 128 ? columns(t, integral_constant<int, 128>{}) : columns(t, integral_constant<int, 64>{}); };
    return s.dtype == HY_F32 ? rows(F32{}) : rows(BF16{});
}

hy_status scan_ends(const LaArgs& a, const LaShape& s, bool back, hipStream_t st) {
    const int64_t items = items_of(s);
    const dim3 grid(workgroups_for(items * (state_size(s) / 4), 256, 256));
    return back ? launch_kernel(la_ends_kernel<true>, grid, dim3(256), st, a.ends, static_cast<const double*>(a.sums), items, (int32_t)state_size(s), a.segments)
                : launch_kernel(la_ends_kernel<false>, grid, dim3(256), st, a.ends, static_cast<const double*>(a.sums), items, (int32_t)state_size(s), a.segments);
}

// The forward walk.
hy_status walk(LaArgs a, const LaShape& s, const Cut& c, void* ws, hipStream_t st) {
    const int64_t items = items_of(s);
    a.segments = (int32_t)c.segments, a.each = c.each;
    a.ends = static_cast<float*>(ws), a.sums = reinterpret_cast<double*>(static_cast<float*>(ws) + c.segments * items * state_size(s));
    const dim3 grid((uint32_t)(items * c.segments));
    if (c.segments > 1) {
        hy_status rc = by_tile(s, [&](auto t, auto dk, auto dv) {
            return launch_kernel(la_ends_walk_kernel<decltype(t), decltype(dk)::value, decltype(dv)::value, false>, grid, dim3(decltype(dv)::value * 4), st, a);
        });
        if (rc == HY_OK) rc = scan_ends(a, s, false, st);
        if (rc != HY_OK) return rc;
    }
    return by_tile(s, [&](auto t, auto dk, auto dv) {
        using T = decltype(t);
        constexpr int DK = decltype(dk)::value, DV = decltype(dv)::value;
        return a.marks ? launch_kernel(la_walk_kernel<T, DK, DV, true>, grid, dim3(DV * 4), st, a)
                       : launch_kernel(la_walk_kernel<T, DK, DV, false>, grid, dim3(DV * 4), st, a);
    });
}

// Workspace of the backward call: segments' ends, shares of dq and dk, shares of dg, and marks, if the caller has none.
struct BwdParts {
    Cut cut, walk_cut, ends_cut;
    int32_t finer;  // segments that the gradients' ends are walked in, for each of the backward walk's
    int64_t ends, shares, dg, marks, y, all;  // bytes
    int32_t count;
};
BwdParts bwd_parts(const LaShape& s, bool with_marks) {
    BwdParts b{};
    b.cut = cut(s, kBackwardGroups), b.walk_cut = cut(s, kForwardGroups);
    // The walk of the ends has room for two workgroups on a compute unit where the backward walk has one: halves of its segments
    // (8192 x 32 heads of 128: 53 us in 8 segments of 16 chunks).
    b.finer = b.cut.segments > 1 && b.cut.each >= 8 ? 2 : 1;
    if (b.finer == 2) {
        const int64_t chunks = chunks_of(s), each = (b.cut.each + 1) / 2 * 2;
        b.cut = Cut{(chunks + each - 1) / each, each};
        b.ends_cut = Cut{(chunks + each / 2 - 1) / (each / 2), each / 2};
    } else {
        b.ends_cut = b.cut;
    }
    b.count = (int32_t)(s.group * tiles_of(s));
    b.ends = up16(ends_bytes(s, b.ends_cut));
    if (!with_marks && ends_bytes(s, b.walk_cut) > b.ends) b.ends = up16(ends_bytes(s, b.walk_cut));
    b.shares = b.count > 1 ? up16(b.count * s.B * s.L * (s.H / s.group) * s.dk * 4) : 0;
    b.dg = tiles_of(s) > 1 ? up16(tiles_of(s) * s.B * s.L * s.H * 4) : 0;
    b.marks = with_marks ? 0 : up16(la_marks_bytes(s));
    b.y = with_marks ? 0 : up16(s.B * s.L * s.H * s.dv * (s.dtype == HY_F32 ? 4 : 2));
    b.all = b.ends + 2 * b.shares + b.dg + b.marks + b.y;
    return b;
}

}  // namespace

bool la_served(const LaShape& s) {
    const int64_t most = INT64_C(1) << 23;
    if (s.dk > 128 || s.H > INT32_MAX || s.dv > INT32_MAX) return false;
    if (s.B == 0 || s.H == 0 || s.dv == 0 || s.L == 0) return true;
    const int64_t tiles = (s.dv + 63) / 64, chunks = (s.L + 63) / 64;
    return s.B < most && s.H < most && tiles < most && chunks < most && s.B * s.H < most && s.B * s.H * tiles < most && s.B * s.H * tiles * chunks < most;
}

int64_t la_marks_bytes(const LaShape& s) { return items_of(s) * chunks_of(s) * state_size(s) * (s.dtype == HY_F32 ? 4 : 2); }

int64_t la_fwd_workspace_bytes(const LaShape& s) { return ends_bytes(s, cut(s, kForwardGroups)); }

int64_t la_bwd_workspace_bytes(const LaShape& s, bool marks) { return bwd_parts(s, marks).all; }

hy_status launch_la_fwd(const LaPtrs& p, const LaShape& s, void* ws, hipStream_t st) {
    if (s.L == 0) {
        const int64_t n = s.B * s.H * s.dk * s.dv;
        return launch_kernel(la_copy_kernel, dim3(workgroups_for(n, 256, 256)), dim3(256), st, p.state_in, p.state_out, n);
    }
    LaArgs a = args_of(p, s);
    a.marks = static_cast<char*>(p.marks);
    return walk(a, s, cut(s, kForwardGroups), ws, st);
}

hy_status launch_la_bwd(const LaPtrs& p, const LaShape& s, void* ws, hipStream_t st) {
    if (s.L == 0) {
        const int64_t n = s.B * s.H * s.dk * s.dv;
        return launch_kernel(la_copy_kernel, dim3(workgroups_for(n, 256, 256)), dim3(256), st, p.dstate_out, p.dstate_in, n);
    }
    const BwdParts b = bwd_parts(s, p.marks_in != nullptr);
    char* const base = static_cast<char*>(ws);
    char *const shares_q = base + b.ends, *const shares_k = shares_q + b.shares, *const shares_g = shares_k + b.shares;
    char *const marks = shares_g + b.dg, *const y = marks + b.marks;
    LaArgs a = args_of(p, s);
    a.marks_in = static_cast<const char*>(p.marks_in);
    if (!a.marks_in) {
        LaArgs f = a;
        f.marks = marks, f.y = y, f.state_out = nullptr;
        const hy_status rc = walk(f, s, b.walk_cut, base, st);
        if (rc != HY_OK) return rc;
        a.marks_in = marks;
    }
    const int64_t items = items_of(s);
    a.segments = (int32_t)b.cut.segments, a.each = b.cut.each, a.finer = b.finer;
    a.ends = reinterpret_cast<float*>(base), a.sums = reinterpret_cast<double*>(a.ends + b.ends_cut.segments * items * state_size(s));
    a.dv = static_cast<char*>(p.dv);
    a.dq = b.count > 1 ? shares_q : p.dq, a.dk = b.count > 1 ? shares_k : p.dk, a.dg = b.dg > 0 ? shares_g : p.dg;
    const dim3 grid((uint32_t)(items * b.cut.segments));
    hy_status rc = HY_OK;
    if (b.cut.segments > 1) {
        LaArgs f = a;
        f.segments = (int32_t)b.ends_cut.segments, f.each = b.ends_cut.each;
        const dim3 ends_grid((uint32_t)(items * b.ends_cut.segments));
        rc = by_tile(s, [&](auto t, auto dk, auto dv) {
            return launch_kernel(la_ends_walk_kernel<decltype(t), decltype(dk)::value, decltype(dv)::value, true>, ends_grid, dim3(decltype(dv)::value * 4), st, f);
        });
        if (rc == HY_OK) rc = scan_ends(f, s, true, st);
        if (rc != HY_OK) return rc;
    }
    rc = by_tile(s, [&](auto t, auto dk, auto dv) {
        using T = decltype(t);
        constexpr int DK = decltype(dk)::value, DV = decltype(dv)::value;
        return b.count > 1 ? launch_kernel(la_bwd_kernel<T, DK, DV, true>, grid, dim3(DV * 4), st, a)
                           : launch_kernel(la_bwd_kernel<T, DK, DV, false>, grid, dim3(DV * 4), st, a);
    });
    auto reduce = [&](const void* from, void* to, int64_t n, int32_t count) {
        const float* f = static_cast<const float*>(from);
        auto sums = [&](auto t, auto vec) {
            constexpr int VEC = decltype(vec)::value;
            return launch_kernel(la_shares_kernel<decltype(t), VEC>, dim3(workgroups_for(n, 256 * VEC, 256)), dim3(256), st, f, to, n, count);
        };
        using std::integral_constant;
        const bool fours = n % 4 == 0 && (reinterpret_cast<uintptr_t>(to) | reinterpret_cast<uintptr_t>(from)) % 16 == 0;
        if (s.dtype == HY_F32) return fours ? sums(F32{}, integral_constant<int, 4>{}) : sums(F32{}, integral_constant<int, 1>{});
        return fours ? sums(BF16{}, integral_constant<int, 4>{}) : sums(BF16{}, integral_constant<int, 1>{});
    };
    const int64_t nqk = s.B * s.L * (s.H / s.group) * s.dk;
    if (rc == HY_OK && b.count > 1) rc = reduce(shares_q, p.dq, nqk, b.count);
    if (rc == HY_OK && b.count > 1) rc = reduce(shares_k, p.dk, nqk, b.count);
    if (rc == HY_OK && b.dg > 0) rc = reduce(shares_g, p.dg, s.B * s.L * s.H, (int32_t)tiles_of(s));
    return rc;
}

hy_status launch_la_step(const LaPtrs& p, const LaShape& s, hipStream_t st) {
    StepArgs a{};
    a.q = static_cast<const char*>(p.q), a.k = static_cast<const char*>(p.k), a.v = static_cast<const char*>(p.v);
    a.g = static_cast<const char*>(p.g), a.y = static_cast<char*>(p.y), a.state = p.state_out;
    a.H = (int32_t)s.H, a.group = s.group, a.dk = (int32_t)s.dk, a.dv = (int32_t)s.dv, a.scale = (float)s.scale;
    const bool fours = s.dv % 4 == 0;
    const int64_t heads = s.B * s.H;
    // 128 columns of a head a workgroup, 32 where that leaves compute units idle
    auto run = [&](auto t, auto cl, auto vec, auto stream) {
        constexpr int CL = decltype(cl)::value, VEC = decltype(vec)::value;
        a.slices = (int32_t)((s.dv + CL * VEC - 1) / (CL * VEC));
        return launch_kernel(la_step_kernel<decltype(t), CL, VEC, decltype(stream)::value>, dim3((uint32_t)(heads * a.slices)), dim3(256), st, a);
    };
    auto by = [&](auto t) {
        using std::integral_constant;
        if (!fours) return run(t, integral_constant<int, 32>{}, integral_constant<int, 1>{}, std::false_type{});
        if (heads < 512) return run(t, integral_constant<int, 8>{}, integral_constant<int, 4>{}, std::false_type{});
        // States that the other layers' push out of the memory-side cache (256 MiB) between two tokens are read as a stream: 64 x 32 of
        // 128 x 128 (128 MiB) with another such state between two tokens 50 us instead of 55, with none 51 instead of 41.
        const bool large = heads * s.dk * s.dv * 4 >= INT64_C(1) << 26;
        return large ? run(t, integral_constant<int, 32>{}, integral_constant<int, 4>{}, std::true_type{})
                     : run(t, integral_constant<int, 32>{}, integral_constant<int, 4>{}, std::false_type{});
    };
    return s.dtype == HY_F32 ? by(F32{}) : by(BF16{});
}

}  // namespace hy
