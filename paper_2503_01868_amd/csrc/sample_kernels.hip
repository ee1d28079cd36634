// The next token of every row of logits: temperature, top-k, top-p, min-p, and a draw by a given random number.
//
// Nothing is sorted.  Logits are compared as whole numbers in their order ("keys", 16 bits of a bf16 number, 32 of an fp32 one).  What
// top-k and top-p keep is everything above one key and the first few words at it: the key is found by its digits, 11 bits at a time,
// from counts (top-k) or sums of weights (top-p) of the words with each digit, in LDS.  The sums of top-p are whole multiples of
// 2^-61 of all weights' sum or less, so that atomic additions give the same bits in any order: each weight is rounded to one, and a sum of
// V words is off by V 2^-62 of it at most (1e-15 for a list of 4096, 3e-14 for 131072 words).  The sums that the draw goes by are in
// double, in a fixed order: a lane's words, a wave by halves, pieces of 64 lanes in the order of the vocabulary.  The weights are exp in
// double, for the words in question alone, off by some 3e-16 of themselves for each unit of their exponent.
//
// A workgroup takes a row.  Where few words can be chosen at all (a small vocabulary, min_p alone, a top_k up to half of a list: 2048, or 1024 of
// more rows than compute units), those are gathered into a list in LDS, in the order of the vocabulary, and everything else happens there: a
// border that lies below enough of the largest logits is taken from every fourth piece of the row, and one pass over the row gathers what
// is above it.  Otherwise the row is read again, a piece at a time: for every digit, for words at the border, for the sums of the draw.
//
// Measured (MI355X): 512 rows of 131072 fp32 words 85-88 us, of which reading them once and a quarter is 60; where they are read again, 551 us with
// top-p alone and 204 with a temperature alone; the largest logit alone 68.  64 rows of 65536 bf16 words 32 us on 64 compute units: 2 for the
// settings, 2 for the border's pieces, 6 for the gathering, 3 and 5 for the borders of top-k and top-p, and the launch (114 where they were read
// again); with top-p alone 128.  One row of 512 words 9 us, half of it in the two borders (22).
#include <type_traits>

#include "hy_common.hpp"
#include "hy_launch.hpp"
#include "hy_scan.hpp"

namespace hy {

namespace {

constexpr int kDigit = 11, kBins = 1 << kDigit;
constexpr int kMostBlocks = 512;  // runs of words whose weights are summed
constexpr int kTable = 64;
constexpr int kEach = 4;             // words of a list that a lane has at most
constexpr int kMostPieces = 4096;    // pieces of a row that a list is gathered from
constexpr int kAhead = 4;            // pieces that a wave loads at once
constexpr int kGroups = 4;           // largest logits that a lane keeps
constexpr int kPart = 4;             // a border is looked for in every kPart-th piece
constexpr int64_t kUnits = 256;      // compute units

// 2^(i / 64), rounded once
__device__ const double kPowers[kTable] = {
    0x1.0000000000000p+0, 0x1.02c9a3e778061p+0, 0x1.059b0d3158574p+0, 0x1.0874518759bc8p+0,
    0x1.0b5586cf9890fp+0, 0x1.0e3ec32d3d1a2p+0, 0x1.11301d0125b51p+0, 0x1.1429aaea92de0p+0,
    0x1.172b83c7d517bp+0, 0x1.1a35beb6fcb75p+0, 0x1.1d4873168b9aap+0, 0x1.2063b88628cd6p+0,
    0x1.2387a6e756238p+0, 0x1.26b4565e27cddp+0, 0x1.29e9df51fdee1p+0, 0x1.2d285a6e4030bp+0,
    0x1.306fe0a31b715p+0, 0x1.33c08b26416ffp+0, 0x1.371a7373aa9cbp+0, 0x1.3a7db34e59ff7p+0,
    0x1.3dea64c123422p+0, 0x1.4160a21f72e2ap+0, 0x1.44e086061892dp+0, 0x1.486a2b5c13cd0p+0,
    0x1.4bfdad5362a27p+0, 0x1.4f9b2769d2ca7p+0, 0x1.5342b569d4f82p+0, 0x1.56f4736b527dap+0,
    0x1.5ab07dd485429p+0, 0x1.5e76f15ad2148p+0, 0x1.6247eb03a5585p+0, 0x1.6623882552225p+0,
    0x1.6a09e667f3bcdp+0, 0x1.6dfb23c651a2fp+0, 0x1.71f75e8ec5f74p+0, 0x1.75feb564267c9p+0,
    0x1.7a11473eb0187p+0, 0x1.7e2f336cf4e62p+0, 0x1.82589994cce13p+0, 0x1.868d99b4492edp+0,
    0x1.8ace5422aa0dbp+0, 0x1.8f1ae99157736p+0, 0x1.93737b0cdc5e5p+0, 0x1.97d829fde4e50p+0,
    0x1.9c49182a3f090p+0, 0x1.a0c667b5de565p+0, 0x1.a5503b23e255dp+0, 0x1.a9e6b5579fdbfp+0,
    0x1.ae89f995ad3adp+0, 0x1.b33a2b84f15fbp+0, 0x1.b7f76f2fb5e47p+0, 0x1.bcc1e904bc1d2p+0,
    0x1.c199bdd85529cp+0, 0x1.c67f12e57d14bp+0, 0x1.cb720dcef9069p+0, 0x1.d072d4a07897cp+0,
    0x1.d5818dcfba487p+0, 0x1.da9e603db3285p+0, 0x1.dfc97337b9b5fp+0, 0x1.e502ee78b3ff6p+0,
    0x1.ea4afa2a490dap+0, 0x1.efa1bee615a27p+0, 0x1.f50765b6e4540p+0, 0x1.fa7c1819e90d8p+0,
};

struct SampleArgs {
    SamplePtrs p;
    SampleAll all;
    int64_t N, stride;
    int32_t V, run;  // pieces of 64 lanes in a run of words
};

__device__ __forceinline__ uint32_t key_of(float z, int bits) {
    z = z != z ? -INFINITY : z + 0.0f;  // (and no zero below another)
    const uint32_t w = __float_as_uint(z);
    return (w & 0x80000000u ? ~w : w | 0x80000000u) >> (32 - bits);
}
__device__ __forceinline__ float logit_of(uint32_t key, int bits) {
    const uint32_t w = key << (32 - bits);
    // (the digits that a bf16 key has lost are ones where the number is negative)
    return __uint_as_float(w & 0x80000000u ? w & 0x7fffffffu : ~(w | ((bits < 32 ? 1u << (32 - bits) : 1u) - 1u)));
}

// exp(x) for x <= 0: 2^(k / 64) from a table and a power series for what is left, |r| <= ln 2 / 128: the first term left out, r^6 / 720, is
// below 2^-53 / 3.
__device__ __forceinline__ double exp_of(double x, const double* table) {
    if (!(x > -746.0)) return 0.0;  // (the smallest number is exp(-744.4))
    const double k = __builtin_rint(x * (kTable / 0.693147180559945309417));
    double r = fma(k, -0.693147180559945309417 / kTable, x);
    r = fma(k, -2.3190468138462995584e-17 / kTable, r);  // ln 2 behind its 53 bits
    double p = fma(r, 1.0 / 120, 1.0 / 24);
    p = fma(p, r, 1.0 / 6);
    p = fma(p, r, 0.5);
    p = fma(p * r, r, r);
    const int n = (int)k;
    const double t = table[n & (kTable - 1)];
    return ldexp(fma(t, p, t), n >> 6);
}

// Weights as whole numbers: multiples of 2^-unit.  `sum` is all weights' sum, 1 at least (twice as much would do): below 2^62 altogether.
__device__ __forceinline__ int unit_of(double sum) { return 61 - ((int)(__builtin_bit_cast(unsigned long long, sum) >> 52) - 1023); }
__device__ __forceinline__ unsigned long long whole(double weight, int unit) { return (unsigned long long)__builtin_rint(ldexp(weight, unit)); }

template <typename X>
__device__ __forceinline__ X wave_total(X x) {
    return of_lane(wave_upto(x), kWave - 1);
}

template <int NT>
struct Lds {
    double table[kTable];
    union {
        uint32_t count[kBins];
        unsigned long long weight[kBins];
        double block[kMostBlocks];
        uint32_t piece[kMostPieces];
    };
    uint32_t key[NT * kEach], word[NT * kEach];  // the list
    unsigned long long wave[3][NT / kWave];
    unsigned long long above, inside, total;
    int32_t bin, at, last;
    uint32_t listed, low, high;
};

// Sums over the workgroup, `upto` with the lanes in front.  `turn` walks over three places, so that one barrier is enough.
template <int NT, typename X>
__device__ __forceinline__ X block_upto(Lds<NT>& s, X x, X& total, int& turn) {
    X* const at = reinterpret_cast<X*>(s.wave[turn]);
    static_assert(sizeof(X) <= sizeof(s.wave[0][0]), "a place for every wave");
    turn = turn == 2 ? 0 : turn + 1;
    const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave;
    const X upto = wave_upto(x);
    if (lane == kWave - 1) at[w] = upto;
    __syncthreads();
    X before = 0;
    total = 0;
#pragma unroll
    for (int j = 0; j < NT / kWave; ++j) {
        if (j == w) before = total;
        total += at[j];
    }
    total = of_lane(total, 0);
    return before + upto;
}
template <int NT>
__device__ __forceinline__ uint32_t block_max(Lds<NT>& s, uint32_t x, int& turn) {
    uint32_t* const at = reinterpret_cast<uint32_t*>(s.wave[turn]);
    turn = turn == 2 ? 0 : turn + 1;
#pragma unroll
    for (int d = kWave / 2; d > 0; d /= 2) x = max(x, (uint32_t)__shfl_xor(x, d, kWave));
    if (threadIdx.x % kWave == 0) at[threadIdx.x / kWave] = x;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < NT / kWave; ++j) x = max(x, at[j]);
    return of_lane(x, 0);
}

// A row's words, wave by wave and piece by piece.  Pieces begin where 16 bytes do: the first has `pad` places in front of the row.
template <typename T, int NT>
struct Row {
    static constexpr int VEC = 16 / T::kBytes, kPiece = VEC * kWave, kBits = T::kBytes * 8, kWaves = NT / kWave;
    const char* from;
    int32_t V, run, pad;
    int lane, w;

    __device__ __forceinline__ int32_t pieces_all() const { return (V + pad + kPiece - 1) / kPiece; }
    __device__ __forceinline__ int32_t first_of(int32_t piece) const { return piece * kPiece + lane * VEC - pad; }
    __device__ __forceinline__ bool has(int32_t i) const { return (uint32_t)i < (uint32_t)V; }
    __device__ __forceinline__ Words<4> fetch(int32_t i) const {
        if (i >= 0 && i + VEC <= V) return load_words<4>(from + (int64_t)i * T::kBytes);
        float f[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            float one[1] = {-INFINITY};
            if (has(i + e)) Pack<T, 1>::unpack(Pack<T, 1>::load(from + (int64_t)(i + e) * T::kBytes), one);
            f[e] = one[0];
        }
        return Pack<T, VEC>::pack(f);
    }
    // f(piece, logits): of all pieces of this wave, in the order of runs
    template <typename F>
    __device__ __forceinline__ void pieces(F&& f) const {
        const int32_t all = pieces_all();
        for (int32_t b = w * run; b < all; b += kWaves * run)
            for (int32_t x = b; x < b + run && x < all; ++x) {
                float z[VEC];
                uint32_t key[VEC];
                Pack<T, VEC>::unpack(fetch(first_of(x)), z);
#pragma unroll
                for (int e = 0; e < VEC; ++e) key[e] = key_of(z[e], kBits);
                f(x, key);
            }
    }
    // f(piece, logits): of this wave's share of every `part`-th piece
    template <typename F>
    __device__ __forceinline__ void spread(int32_t part, F&& f) const {
        const int32_t all = pieces_all(), step = kWaves * part;
        for (int32_t b = w * part; b < all; b += step * kAhead) {
            const int32_t last = b + (kAhead - 1) * step;
            Words<4> r[kAhead];
            if ((b > 0 || pad == 0) && (int64_t)(last + 1) * kPiece - pad <= V) {
#pragma unroll
                for (int j = 0; j < kAhead; ++j) r[j] = load_words<4>(from + (int64_t)first_of(b + j * step) * T::kBytes);
            } else {
#pragma unroll
                for (int j = 0; j < kAhead; ++j) r[j] = fetch(first_of(min(b + j * step, all)));
            }
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                float z[VEC];
                Pack<T, VEC>::unpack(r[j], z);
                if (b + j * step < all) f(b + j * step, z);
            }
        }
    }
    // f(index, key): of every word
    template <typename F>
    __device__ __forceinline__ void words(F&& f) const {
        pieces([&](int32_t piece, const uint32_t(&key)[VEC]) {
            const int32_t i = first_of(piece);
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (has(i + e)) f(i + e, key[e]);
        });
    }
};

// The highest bin up to which, from the top, the amounts add up to `need` (of all bins, one from which they do exist): LDS has it
// in bin, what is in higher bins in `above`, its own amount in `inside` and the amount of all bins in `total`.
template <int NT, typename X>
__device__ __forceinline__ void find_bin(Lds<NT>& s, const X* bins, unsigned long long need, int& turn) {
    constexpr int kOwn = kBins / NT;
    X mine = 0;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) mine += bins[kBins - 1 - (threadIdx.x * kOwn + j)];
    X total;
    const X upto = block_upto<NT, X>(s, mine, total, turn);
    unsigned long long above = upto - mine;
    if (threadIdx.x == NT - 1) s.total = total;
    if (above < need && need <= upto) {
        for (int j = 0; j < kOwn; ++j) {
            const int b = kBins - 1 - ((int)threadIdx.x * kOwn + j);
            const unsigned long long here = bins[b];
            if (need <= above + here) {
                s.bin = b, s.above = above, s.inside = here;
                break;
            }
            above += here;
        }
    }
    __syncthreads();
}

// Of the keys in [lo, hi], those from the highest on whose amounts add up to `need`: keys above `least`, and of those at it `need`
// more (all: every one).  The first round takes words by their distance from the largest, in equal steps down to the least, which
// parts a row's words better than the digits of their keys do: few are in one step, and mostly one round is enough; the next go by the
// keys in the step that is reached.  `most`: rounds after which what is reached is taken whole.
struct Border {
    uint32_t least;
    unsigned long long need;
    bool all;
};
template <int NT, int BITS, typename X, int E, typename F>
__device__ __forceinline__ Border find_border(Lds<NT>& s, X* bins, const uint32_t (&key)[E], F&& amount, uint32_t lo, uint32_t hi,
                                              unsigned long long need, int most, int& turn) {
    const float z_hi = logit_of(hi, BITS), wide = z_hi - logit_of(lo, BITS), step = (kBins - 1) / wide;
    bool even = wide > 0.0f && wide < INFINITY && step < INFINITY;
    int shift = 0;
    for (;;) {
        const int width = hi > lo ? 32 - __builtin_clz(hi - lo) : 0;
        shift = width > kDigit ? width - kDigit : 0;
        auto bin_of = [&](uint32_t k) {
            return even ? kBins - 1 - min((int)((z_hi - logit_of(k, BITS)) * step), kBins - 1) : (int)((k - lo) >> shift);
        };
        for (int j = threadIdx.x; j < kBins; j += NT) bins[j] = 0;
        if (threadIdx.x == 0) s.low = ~0u, s.high = 0;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (key[e] < lo || key[e] > hi) continue;
            const X x = amount(e);
            if (x > 0) atomicAdd(&bins[bin_of(key[e])], x);
        }
        __syncthreads();
        find_bin<NT>(s, bins, need, turn);
        const int bin = of_lane(s.bin, 0);
        need -= of_lane(s.above, 0);
        const bool all = of_lane(s.inside, 0) == need;
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (key[e] >= lo && key[e] <= hi && bin_of(key[e]) == bin) {
                atomicMin(&s.low, key[e]);
                atomicMax(&s.high, key[e]);
            }
        __syncthreads();
        lo = of_lane(s.low, 0), hi = of_lane(s.high, 0);
        if (all || lo == hi || --most == 0) return Border{lo, need, all};
        even = false;
        __syncthreads();  // (the next round's beginning)
    }
}

// What the settings of a row are.
struct Settings {
    double scale, top_p, min_p, u;  // scale: 1 / temperature
    int32_t top_k;

    // What the running sum has to pass.  (Sums are added in several orders, so that one may pass another by its rounding.)
    __device__ __forceinline__ double want(double sum) const { return u < 1.0 ? u * sum : INFINITY; }
};

// The choice among the listed words: a lane has `each` of them, in the order of the vocabulary, as keys (0: none).
template <int NT, int BITS>
__device__ __forceinline__ void choose_listed(const SampleArgs& a, Lds<NT>& s, int64_t n, uint32_t (&key)[kEach], const int32_t (&word)[kEach],
                                              uint32_t lo, uint32_t top, int32_t listed, const Settings& set, int& turn) {
    auto drop = [&](const Border& b) {
        uint32_t mine = 0, total;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            if (key[e] < b.least) key[e] = 0;
            mine += key[e] == b.least;
        }
        if (b.all) return;
        int64_t left = (int64_t)b.need - (int64_t)(block_upto<NT, uint32_t>(s, mine, total, turn) - mine);
#pragma unroll
        for (int e = 0; e < kEach; ++e)
            if (key[e] == b.least && --left < 0) key[e] = 0;
    };
    uint32_t least = lo;
    if (set.top_k >= 1 && set.top_k < listed) {
        const Border b = find_border<NT, BITS>(s, s.count, key, [](int) { return 1u; }, lo, top, (unsigned long long)set.top_k, INT32_MAX, turn);
        drop(b);
        least = b.least;
    }
    const double z_top = logit_of(top, BITS);
    const uint32_t none = key_of(-INFINITY, BITS);
    auto weight = [&](uint32_t x) -> double {
        if (x == top) return 1.0;
        if (x <= none) return 0.0;
        return exp_of(((double)logit_of(x, BITS) - z_top) * set.scale, s.table);
    };
    double w[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) w[e] = key[e] ? weight(key[e]) : 0.0;
    if (set.top_p < 1.0) {
        double some = 0.0, sum;
#pragma unroll
        for (int e = 0; e < kEach; ++e) some += w[e];
        block_upto<NT, double>(s, some, sum, turn);
        const int unit = unit_of(sum);
        unsigned long long mine = 0, total;
#pragma unroll
        for (int e = 0; e < kEach; ++e) mine += whole(w[e], unit);
        block_upto<NT, unsigned long long>(s, mine, total, turn);
        const double most = set.top_p > 0.0 ? __builtin_ceil(set.top_p * (double)total) : 1.0;
        unsigned long long need = most < 1.0 ? 1 : (unsigned long long)most;
        if (need > total) need = total;
        Border b = find_border<NT, BITS>(s, s.weight, key, [&](int e) { return whole(w[e], unit); }, least, top, need, INT32_MAX, turn);
        if (!b.all) {
            const unsigned long long one = whole(weight(b.least), unit);
            b.need = one > 0 ? (b.need + one - 1) / one : 1;
        }
        drop(b);
    }
    double mine = 0.0, sum;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        if (key[e] == 0 || !(w[e] >= set.min_p || key[e] == top)) w[e] = 0.0;
        mine += w[e];
    }
    if (threadIdx.x == 0) s.at = INT32_MAX, s.last = -1;
    double here = block_upto<NT, double>(s, mine, sum, turn) - mine;
    const double want = set.want(sum);
    int32_t hit = INT32_MAX, last = -1;
    double hit_weight = 0.0, last_weight = 0.0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        here += w[e];
        if (w[e] > 0.0) {
            last = word[e], last_weight = w[e];
            if (hit == INT32_MAX && here > want) hit = word[e], hit_weight = w[e];
        }
    }
    if (hit != INT32_MAX) atomicMin(&s.at, hit);
    if (last >= 0) atomicMax(&s.last, last);
    __syncthreads();
    const bool none_hit = s.at == INT32_MAX;
    if (none_hit ? last >= 0 && last == s.last : hit == s.at) {
        a.p.token[n] = none_hit ? last : hit;
        if (a.p.prob) a.p.prob[n] = (float)((none_hit ? last_weight : hit_weight) / sum);
    }
    __syncthreads();
}

template <typename T, int NT>
__global__ __launch_bounds__(NT, NT == 512 ? 4 : 1) void sample_kernel(SampleArgs a) {
    using R = Row<T, NT>;
    constexpr int kBits = R::kBits, kPiece = R::kPiece, VEC = R::VEC, kMostList = NT * kEach;
    constexpr bool kLong = NT > 256;  // (else all words are a list)
    __shared__ __attribute__((aligned(16))) Lds<NT> s;
    const int lane = threadIdx.x % kWave, w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    int turn = 0;
    if (threadIdx.x < kTable) s.table[threadIdx.x] = kPowers[threadIdx.x];
    const uint32_t none = key_of(-INFINITY, kBits);
    for (int64_t n = blockIdx.x; n < a.N; n += gridDim.x) {
        R row;
        row.from = static_cast<const char*>(a.p.logits) + n * a.stride * T::kBytes;
        row.V = a.V, row.run = a.run, row.lane = lane, row.w = w;
        row.pad = (int32_t)(reinterpret_cast<uintptr_t>(row.from) % 16) / T::kBytes;

        double T_n = a.p.temperature ? (double)a.p.temperature[n] : a.all.temperature;
        double top_p = a.p.top_p ? (double)a.p.top_p[n] : a.all.top_p, min_p = a.p.min_p ? (double)a.p.min_p[n] : a.all.min_p;
        double u = a.p.u[n];
        if (T_n != T_n) T_n = 1.0;
        if (top_p != top_p) top_p = 1.0;
        if (min_p != min_p) min_p = 0.0;
        if (!(u > 0.0)) u = 0.0;
        // (the same for all lanes: in scalar registers)
        T_n = of_lane(T_n, 0), top_p = of_lane(top_p, 0), min_p = of_lane(min_p, 0), u = of_lane(u, 0);
        const int32_t top_k = of_lane(a.p.top_k ? a.p.top_k[n] : a.all.top_k, 0);
        const Settings set{of_lane(1.0 / T_n, 0), top_p, min_p, u, top_k};
        __syncthreads();  // (the row before)

        uint32_t key[kEach], top = 0, from = none, listed = 0;  // the list's words, its least key and the largest, how many
        int32_t word[kEach];
        if (a.V <= kMostList && T_n > 0.0) {  // all words are the list
            const int32_t each = (a.V + NT - 1) / NT;
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                word[e] = (int32_t)threadIdx.x * each + e;
                key[e] = 0;
                if (e < each && word[e] < a.V) {
                    float z[1];
                    Pack<T, 1>::unpack(Pack<T, 1>::load(row.from + (int64_t)word[e] * T::kBytes), z);
                    key[e] = key_of(z[0], kBits);
                }
                top = max(top, key[e]);
            }
            top = block_max<NT>(s, top, turn);
            if (top != none) {  // (of those that have a weight)
                uint32_t low = ~0u, mine = 0;
#pragma unroll
                for (int e = 0; e < kEach; ++e) {
                    if (key[e] <= none) key[e] = 0;
                    else low = min(low, key[e]), ++mine;
                }
                from = ~block_max<NT>(s, ~low, turn);
                block_upto<NT, uint32_t>(s, mine, listed, turn);
            }
        } else if (kLong && T_n > 0.0) {
            // A list of words that has all that can be chosen.  With top_k, those from a border on that lies below enough of the
            // largest logits that the lanes see in every fourth piece: should too few words be there, or too many, the border is
            // taken from all pieces, of as many different words as top_k.  Without top_k and top_p, min_p is a border by itself.
            const int32_t all = row.pieces_all();
            const bool few = top_k >= 1 && top_k <= kMostList / 2 && top_k < a.V;
            const bool near = (top_k < 1 || top_k >= a.V) && top_p >= 1.0 && min_p > 0.0;
            int32_t part = few && all >= kPart * R::kWaves ? kPart : 1;
            for (;; part = 1) {
                float m[kGroups];
#pragma unroll
                for (int e = 0; e < kGroups; ++e) m[e] = -INFINITY;
                row.spread(part, [&](int32_t, const float(&z)[VEC]) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) m[e % kGroups] = fmaxf(m[e % kGroups], z[e]);
                });
                uint32_t first[kGroups], low = ~0u;
                top = 0;
#pragma unroll
                for (int e = 0; e < kGroups; ++e) first[e] = key_of(m[e], kBits), top = max(top, first[e]), low = min(low, first[e]);
                top = block_max<NT>(s, top, turn);
                from = none;
                if (top != none && all <= kMostPieces) {
                    if (few) {
                        const int32_t need = part == 1 ? top_k : top_k * 21 / 64 + 16;  // (1.3 quarters, and 16)
                        low = ~block_max<NT>(s, ~low, turn);
                        from = find_border<NT, kBits>(s, s.count, first, [](int) { return 1u; }, low, top, (unsigned long long)need, 2, turn).least;
                    } else if (near) {
                        // (a weight this near to min_p may round to it)
                        const double z = logit_of(top, kBits), d = fmax(0.0, -T_n * log(min_p)) + T_n * 0x1p-50, t = z - d - 1e-6 * (fabs(z) + d);
                        const float f = (float)t;  // (the margin is more than this rounds)
                        from = f == f ? min(key_of(f, kBits), top) : top;
                    }
                }
                if (from > none) {
                    const float least = logit_of(from, kBits);
                    __syncthreads();
                    for (int j = threadIdx.x; j < kMostPieces; j += NT) s.piece[j] = 0;
                    if (threadIdx.x == 0) s.listed = 0;
                    __syncthreads();
                    // lanes' pieces that have such words, then the words of those
                    row.spread(1, [&](int32_t piece, const float(&z)[VEC]) {
                        float most = z[0];
#pragma unroll
                        for (int e = 1; e < VEC; ++e) most = fmaxf(most, z[e]);
                        const unsigned long long hits = __builtin_amdgcn_ballot_w64(most >= least);
                        if (hits == 0) return;
                        uint32_t base = 0;
                        if (lane == 0) {
                            const uint32_t c = __builtin_popcountll(hits);
                            base = atomicAdd(&s.listed, c);
                            s.piece[piece] = base << 7 | c;
                        }
                        base = __builtin_amdgcn_readfirstlane(base);
                        const uint32_t at = __builtin_amdgcn_mbcnt_hi((uint32_t)(hits >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)hits, base));
                        if (most >= least && at < kMostList) s.word[at] = (uint32_t)(row.first_of(piece) + row.pad);
                    });
                    __syncthreads();
                    const uint32_t found = s.listed;
                    if (found <= kMostList) {
                        // pieces came in any order: how far each one's have to move
                        constexpr int kOwn = kMostPieces / NT;
                        uint32_t mine = 0, total;
#pragma unroll
                        for (int j = 0; j < kOwn; ++j) mine += s.piece[threadIdx.x * kOwn + j] & 127;
                        uint32_t before = block_upto<NT, uint32_t>(s, mine, total, turn) - mine;
#pragma unroll
                        for (int j = 0; j < kOwn; ++j) {
                            const uint32_t x = s.piece[threadIdx.x * kOwn + j];
                            s.piece[threadIdx.x * kOwn + j] = before - (x >> 7);
                            before += x & 127;
                        }
                        __syncthreads();
#pragma unroll
                        for (int e = 0; e < kEach; ++e) {
                            const uint32_t i = e * NT + threadIdx.x;
                            if (i < found) s.key[i + s.piece[s.word[i] / kPiece]] = s.word[i];
                        }
                        __syncthreads();
                        const uint32_t each = (found + NT - 1) / NT;
                        Words<4> r[kEach];
                        int32_t at[kEach];
                        mine = 0;
#pragma unroll
                        for (int e = 0; e < kEach; ++e) {
                            const uint32_t i = threadIdx.x * each + e;
                            at[e] = a.V;
                            if ((uint32_t)e < each && i < found) at[e] = (int32_t)s.key[i] - row.pad;
                            if (at[e] < a.V) r[e] = row.fetch(at[e]);
                        }
#pragma unroll
                        for (int e = 0; e < kEach; ++e) {
                            if (at[e] >= a.V) continue;
                            float z[VEC];
                            Pack<T, VEC>::unpack(r[e], z);
#pragma unroll
                            for (int j = 0; j < VEC; ++j) mine += z[j] >= least;
                        }
                        before = block_upto<NT, uint32_t>(s, mine, total, turn) - mine;
                        if (total <= kMostList && (part == 1 || total >= (uint32_t)top_k)) {
                            listed = total;
#pragma unroll
                            for (int e = 0; e < kEach; ++e) {
                                if (at[e] >= a.V) continue;
                                float z[VEC];
                                Pack<T, VEC>::unpack(r[e], z);
#pragma unroll
                                for (int j = 0; j < VEC; ++j)
                                    if (z[j] >= least) s.key[before] = key_of(z[j], kBits), s.word[before++] = (uint32_t)(at[e] + j);
                            }
                        }
                    }
                    __syncthreads();
                }
                if (listed > 0 || part == 1) break;
            }
            if (listed > 0) {
                const uint32_t each = (listed + NT - 1) / NT;
                uint32_t most = 0;
#pragma unroll
                for (int e = 0; e < kEach; ++e) {
                    const uint32_t i = threadIdx.x * each + e;
                    const bool in = (uint32_t)e < each && i < listed;
                    key[e] = in ? s.key[i] : 0, word[e] = in ? (int32_t)s.word[i] : 0;
                    most = max(most, key[e]);
                }
                top = block_max<NT>(s, most, turn);
            }
        }
        from = of_lane(from, 0), top = of_lane(top, 0), listed = of_lane(listed, 0);
        if (listed > 0) {
            choose_listed<NT, kBits>(a, s, n, key, word, from, top, (int32_t)listed, set, turn);
            continue;
        }

        // the largest logit and the lowest index that has it
        unsigned long long best = (unsigned long long)top << 32;
        if (!(T_n > 0.0)) {
            row.words([&](int32_t i, uint32_t key) {
                const unsigned long long x = (unsigned long long)key << 32 | (uint32_t)~i;
                best = x > best ? x : best;
            });
#pragma unroll
            for (int d = kWave / 2; d > 0; d /= 2) {
                const unsigned long long x = __shfl_xor(best, d, kWave);
                best = x > best ? x : best;
            }
            if (lane == 0) s.wave[0][w] = best;
            __syncthreads();
            for (int j = 0; j < NT / kWave; ++j) best = s.wave[0][j] > best ? s.wave[0][j] : best;
            top = (uint32_t)(best >> 32);
        }
        const double z_top = logit_of(top, kBits);
        if (top == none || !(T_n > 0.0)) {
            if (threadIdx.x == 0) {
                a.p.token[n] = top == none ? -1 : (int64_t)(uint32_t)~(uint32_t)best;
                if (a.p.prob) a.p.prob[n] = top == none ? 0.0f : 1.0f;
            }
            continue;
        }
        if constexpr (!kLong) continue;
        const double scale = set.scale;
        auto weight = [&](uint32_t key) -> double {
            if (key == top) return 1.0;
            if (key == none) return 0.0;
            return exp_of(((double)logit_of(key, kBits) - z_top) * scale, s.table);
        };
        int unit = 0;
        if (top_p < 1.0) {  // (the sum of all weights in fp32, to some bits: only its size is asked for)
            float mine = 0.0f, sum;
            const float most = (float)z_top, slope = (float)(scale * 1.4426950408889634074);
            row.spread(1, [&](int32_t, const float(&z)[VEC]) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float x = (z[e] - most) * slope;
                    mine += z[e] == most ? 1.0f : x > -100.0f ? __builtin_amdgcn_exp2f(x) : 0.0f;  // (NaN: none)
                }
            });
            block_upto<NT, float>(s, mine, sum, turn);
            unit = unit_of((double)sum);
        }
        auto whole_weight = [&](uint32_t key) { return whole(weight(key), unit); };

        // kept: keys above `least`, and the first `ties` words of those at it (-1: all)
        uint32_t least = 0;
        int64_t ties = -1;
        if (top_k >= 1 && top_k < a.V) {
            unsigned long long need = top_k;
            uint32_t prefix = 0;
            for (int low = kBits; low > 0;) {  // the digits above bit `low` are known
                const int next = low > kDigit ? low - kDigit : 0;
                for (int j = threadIdx.x; j < kBins; j += NT) s.count[j] = 0;
                __syncthreads();
                row.words([&](int32_t, uint32_t key) {
                    if (low == kBits || key >> low == prefix) atomicAdd(&s.count[(key >> next) & ((1u << (low - next)) - 1)], 1u);
                });
                __syncthreads();
                find_bin<NT>(s, s.count, need, turn);
                prefix = prefix << (low - next) | (uint32_t)s.bin;
                need -= s.above;
                low = next;
                if (s.inside == need) {  // all that begin like this
                    least = prefix << low;
                    need = 0;
                    break;
                }
            }
            if (need > 0) least = prefix, ties = (int64_t)need;
            __syncthreads();
        }
        if (top_p < 1.0) {
            unsigned long long need = 0;
            uint32_t prefix = 0;
            for (int low = kBits; low > 0;) {
                const int next = low > kDigit ? low - kDigit : 0;
                for (int j = threadIdx.x; j < kBins; j += NT) s.weight[j] = 0;
                __syncthreads();
                row.words([&](int32_t, uint32_t key) {
                    if (key < least || (key == least && ties >= 0) || (low < kBits && key >> low != prefix)) return;
                    const unsigned long long x = whole_weight(key);
                    if (x > 0) atomicAdd(&s.weight[(key >> next) & ((1u << (low - next)) - 1)], x);
                });
                if (threadIdx.x == 0 && ties >= 0 && (low == kBits || least >> low == prefix))
                    atomicAdd(&s.weight[(least >> next) & ((1u << (low - next)) - 1)], ties * whole_weight(least));
                __syncthreads();
                if (low == kBits) {
                    find_bin<NT>(s, s.weight, 1, turn);  // (for the sum of all)
                    const double most = top_p > 0.0 ? __builtin_ceil(top_p * (double)s.total) : 1.0;
                    need = most < 1.0 ? 1 : (unsigned long long)most;
                    if (need > s.total) need = s.total;
                    __syncthreads();
                }
                find_bin<NT>(s, s.weight, need, turn);
                prefix = prefix << (low - next) | (uint32_t)s.bin;
                need -= s.above;
                low = next;
                if (s.inside == need && (prefix << low) > least) {
                    least = prefix << low, ties = -1;
                    need = 0;
                    break;
                }
                __syncthreads();
            }
            if (need > 0) {
                const unsigned long long each = whole_weight(prefix);
                const unsigned long long some = each > 0 ? (need + each - 1) / each : 1;
                if (prefix == least && ties >= 0) ties = (int64_t)some < ties ? (int64_t)some : ties;
                else ties = (int64_t)some;
                least = prefix;
            }
            __syncthreads();
        }

        // where the `ties`-th word at `least` is
        int32_t last_tie = a.V;
        if (ties >= 0) {
            for (int j = threadIdx.x; j < kMostBlocks; j += NT) s.count[j] = 0;
            if (threadIdx.x == 0) s.at = a.V;
            __syncthreads();
            row.pieces([&](int32_t piece, const uint32_t(&key)[VEC]) {
                uint32_t c = 0;
#pragma unroll
                for (int e = 0; e < VEC; ++e) c += key[e] == least && row.has(row.first_of(piece) + e);
                if (__builtin_amdgcn_ballot_w64(c > 0) == 0) return;
                c = wave_total(c);
                if (lane == 0) s.count[piece / a.run] += c;  // a run is one wave's
            });
            __syncthreads();
            if (w == 0) {
                uint32_t mine = 0;
                constexpr int kOwn = kMostBlocks / kWave;
                for (int j = 0; j < kOwn; ++j) mine += s.count[lane * kOwn + j];
                uint32_t before = wave_upto(mine) - mine;
                for (int j = 0; j < kOwn; ++j) {
                    const uint32_t here = s.count[lane * kOwn + j];
                    if (before < ties && ties <= before + here) s.bin = lane * kOwn + j, s.above = before;
                    before += here;
                }
            }
            __syncthreads();
            if (w == 0) {  // the run, a piece at a time
                int64_t left = ties - (int64_t)s.above;
                const int32_t run = s.bin, all = row.pieces_all();
                for (int32_t x = run * a.run; x < (run + 1) * a.run && x < all && left > 0; ++x) {
                    float z[VEC];
                    Pack<T, VEC>::unpack(row.fetch(row.first_of(x)), z);
                    uint32_t c = 0;
                    for (int e = 0; e < VEC; ++e) c += row.has(row.first_of(x) + e) && key_of(z[e], kBits) == least;
                    const uint32_t upto = wave_upto(c);
                    if (upto - c < left && left <= upto) {
                        int64_t mine = left - (upto - c);
                        for (int e = 0; e < VEC; ++e)
                            if (row.has(row.first_of(x) + e) && key_of(z[e], kBits) == least && --mine == 0) s.at = row.first_of(x) + e;
                    }
                    left -= of_lane(upto, kWave - 1);
                }
            }
            __syncthreads();
            last_tie = s.at;
        }

        // the kept weights of every run
        auto kept = [&](int32_t i, uint32_t key) -> double {
            if (!row.has(i) || key < least || (key == least && i > last_tie)) return 0.0;
            const double x = weight(key);
            return x >= min_p || key == top ? x : 0.0;
        };
        for (int j = threadIdx.x; j < kMostBlocks; j += NT) s.block[j] = 0.0;
        __syncthreads();
        {
            double mine = 0.0;
            row.pieces([&](int32_t piece, const uint32_t(&key)[VEC]) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) mine += kept(row.first_of(piece) + e, key[e]);
                if ((piece + 1) % a.run == 0 || piece + 1 == row.pieces_all()) {
                    if (__builtin_amdgcn_ballot_w64(mine > 0.0) != 0) {
                        const double x = wave_total(mine);
                        if (lane == 0 && piece / a.run < kMostBlocks) s.block[piece / a.run] = x;
                    }
                    mine = 0.0;
                }
            });
        }
        __syncthreads();
        if (w == 0) {
            constexpr int kOwn = kMostBlocks / kWave;
            double mine = 0.0;
            for (int j = 0; j < kOwn; ++j) mine += s.block[lane * kOwn + j];
            const double upto = wave_upto(mine);
            const double sum = of_lane(upto, kWave - 1), want = set.want(sum);
            // the first run up to which there is more than `want`, else the last one that has something
            double before = upto - mine;
            int32_t run = -1, last = -1;
            double at_run = 0.0, at_last = 0.0;
            for (int j = 0; j < kOwn; ++j) {
                const double here = s.block[lane * kOwn + j];
                if (here > 0.0) {
                    last = lane * kOwn + j, at_last = before;
                    if (run < 0 && before + here > want) run = last, at_run = before;
                }
                before += here;
            }
            unsigned long long who = __builtin_amdgcn_ballot_w64(run >= 0);
            if (who != 0) {
                const int l = __builtin_ctzll(who);
                run = __shfl(run, l, kWave), at_run = __shfl(at_run, l, kWave);
            } else {
                const int l = 63 - __builtin_clzll(__builtin_amdgcn_ballot_w64(last >= 0));
                run = __shfl(last, l, kWave), at_run = __shfl(at_last, l, kWave);
            }
            // in the run: the first word up to which there is more, else the last one with a weight
            int32_t token = -1, spare = -1;
            double chosen = 0.0, spare_weight = 0.0, upto_here = at_run;
            const int32_t all = row.pieces_all();
            for (int32_t x = run * a.run; x < (run + 1) * a.run && x < all && token < 0; ++x) {
                float z[VEC];
                double f[VEC], c = 0.0;
                Pack<T, VEC>::unpack(row.fetch(row.first_of(x)), z);
                for (int e = 0; e < VEC; ++e) c += f[e] = kept(row.first_of(x) + e, key_of(z[e], kBits));
                const double upto = wave_upto(c);
                double here = upto_here + (upto - c);
                int32_t mine = -1, my_last = -1;
                double fm = 0.0, fl = 0.0;
                for (int e = 0; e < VEC; ++e) {
                    here += f[e];
                    if (f[e] > 0.0) {
                        my_last = row.first_of(x) + e, fl = f[e];
                        if (mine < 0 && here > want) mine = my_last, fm = f[e];
                    }
                }
                who = __builtin_amdgcn_ballot_w64(mine >= 0);
                if (who != 0) {
                    const int l = __builtin_ctzll(who);
                    token = __shfl(mine, l, kWave), chosen = __shfl(fm, l, kWave);
                }
                who = __builtin_amdgcn_ballot_w64(my_last >= 0);
                if (who != 0) {
                    const int l = 63 - __builtin_clzll(who);
                    spare = __shfl(my_last, l, kWave), spare_weight = __shfl(fl, l, kWave);
                }
                upto_here += of_lane(upto, kWave - 1);
            }
            if (token < 0) token = spare, chosen = spare_weight;
            if (lane == 0) {
                a.p.token[n] = token;
                if (a.p.prob) a.p.prob[n] = (float)(chosen / sum);
            }
        }
        __syncthreads();
    }
}

template <typename T, int NT>
hy_status run(SampleArgs a, hipStream_t st) {
    constexpr int kPiece = Row<T, NT>::kPiece;
    const int64_t pieces = ((int64_t)a.V + Row<T, NT>::VEC - 1 + kPiece - 1) / kPiece;  // (wherever the row begins)
    a.run = (int32_t)((pieces + kMostBlocks - 1) / kMostBlocks);
    return launch_kernel(sample_kernel<T, NT>, dim3(workgroups_for(a.N, 1, NT)), dim3(NT), st, a);
}

template <typename T>
hy_status by_size(const SampleArgs& a, hipStream_t st) {
    // more rows than compute units: two workgroups share one, so that one reads while the other chooses
    if (a.V <= 256 * kEach) return run<T, 256>(a, st);
    return a.N > kUnits ? run<T, 512>(a, st) : run<T, 1024>(a, st);
}

}  // namespace

hy_status launch_sample(const SamplePtrs& p, const SampleAll& all, int64_t N, int64_t V, int64_t stride, int32_t dtype, hipStream_t st) {
    const SampleArgs a{p, all, N, stride, (int32_t)V, 1};
    return dtype == HY_F32 ? by_size<F32>(a, st) : by_size<BF16>(a, st);
}

}  // namespace hy
