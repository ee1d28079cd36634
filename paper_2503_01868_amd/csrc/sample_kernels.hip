// The next token of every row of logits: temperature, top-k, top-p, min-p, and a draw by a given random number.
//
// Nothing is sorted.  Logits are compared as whole numbers in their order ("keys", 16 bits of a bf16 number, 32 of an fp32 one).  What
// top-k and top-p keep is everything above one key and the first few words at it: the key is found by its digits, 11 bits at a time,
// from counts (top-k) or sums of weights (top-p) of the words with each digit, in LDS.  The sums of top-p are whole multiples of
// the smallest weight that matters, so that atomic additions give the same bits in any order; the sums that the draw goes by are in
// double, in a fixed order: a lane's words, a wave by halves, pieces of 64 lanes in the order of the vocabulary.  The weights are exp in
// double, for the words in question alone: a border between two words is that of the definition but for some 1e-15.
//
// A workgroup takes a row, and reads it again for every one of these passes.
#include <type_traits>

#include "hy_common.hpp"
#include "hy_launch.hpp"

namespace hy {

namespace {

constexpr int kDigit = 11, kBins = 1 << kDigit;
constexpr int kMostBlocks = 512;  // runs of words whose weights are summed
constexpr int kTable = 64;

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

// exp(x) for x <= 0: 2^(k / 64) from a table and a power series for what is left, |r| <= ln 2 / 128: the first term left out is below
// 2^-53 / 10.
__device__ __forceinline__ double exp_of(double x, const double* table) {
    if (!(x > -708.0)) return 0.0;
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

template <typename X>
__device__ __forceinline__ X wave_total(X x) {
#pragma unroll
    for (int d = kWave / 2; d > 0; d /= 2) x += __shfl_xor(x, d, kWave);
    return x;
}
template <typename X>
__device__ __forceinline__ X wave_upto(X x, int lane) {
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const X y = __shfl_up(x, d, kWave);
        if (lane >= d) x += y;
    }
    return x;
}

template <int NT>
struct Lds {
    double table[kTable];
    union {
        uint32_t count[kBins];
        unsigned long long weight[kBins];
        double block[kMostBlocks];
    };
    unsigned long long wave[NT / kWave];
    unsigned long long above, inside, total;
    int32_t bin, at;
    double before, sum;
};

// A row's words, wave by wave and piece by piece.
template <typename T, int NT>
struct Row {
    static constexpr int VEC = 16 / T::kBytes, kPiece = VEC * kWave, kBits = T::kBytes * 8;
    const char* from;
    int32_t V, run;
    bool whole;  // its pieces begin where 16 bytes do
    int lane, w;

    __device__ __forceinline__ Words<4> fetch(int64_t i) const {
        if (whole && i + VEC <= V) return load_words<4>(from + i * T::kBytes);
        float f[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            float one[1] = {-INFINITY};
            if (i + e < V) Pack<T, 1>::unpack(Pack<T, 1>::load(from + (i + e) * T::kBytes), one);
            f[e] = one[0];
        }
        return Pack<T, VEC>::pack(f);
    }
    __device__ __forceinline__ int64_t first_of(int32_t piece) const { return (int64_t)piece * kPiece + lane * VEC; }
    // f(piece, keys): of all pieces of this wave
    template <typename F>
    __device__ __forceinline__ void pieces(F&& f) const {
        const int32_t all = (V + kPiece - 1) / kPiece;
        for (int32_t b = w * run; b < all; b += NT / kWave * run)
            for (int32_t x = b; x < b + run && x < all; ++x) {
                float z[VEC];
                uint32_t key[VEC];
                Pack<T, VEC>::unpack(fetch(first_of(x)), z);
#pragma unroll
                for (int e = 0; e < VEC; ++e) key[e] = key_of(z[e], kBits);
                f(x, key);
            }
    }
    // f(index, key): of every word
    template <typename F>
    __device__ __forceinline__ void words(F&& f) const {
        pieces([&](int32_t piece, const uint32_t(&key)[VEC]) {
            const int64_t i = first_of(piece);
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (i + e < V) f((int32_t)(i + e), key[e]);
        });
    }
};

// The highest bin up to which, from the top, the amounts add up to `need` (of all bins, one from which they do exist): LDS has it
// in bin, what is in higher bins in `above`, its own amount in `inside` and the amount of all bins in `total`.
template <int NT, typename X>
__device__ __forceinline__ void find_bin(Lds<NT>& s, const X* bins, unsigned long long need) {
    constexpr int kEach = kBins / NT;
    const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave;
    unsigned long long mine = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) mine += bins[kBins - 1 - (threadIdx.x * kEach + j)];
    unsigned long long upto = wave_upto(mine, lane);
    if (lane == kWave - 1) s.wave[w] = upto;
    __syncthreads();
    for (int j = 0; j < w; ++j) upto += s.wave[j];
    unsigned long long above = upto - mine;
    if (threadIdx.x == NT - 1) s.total = upto;
    if (above < need && need <= upto) {
        for (int j = 0; j < kEach; ++j) {
            const int b = kBins - 1 - ((int)threadIdx.x * kEach + j);
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

template <typename T, int NT>
__global__ __launch_bounds__(NT) void sample_kernel(SampleArgs a) {
    using R = Row<T, NT>;
    constexpr int kBits = R::kBits, kPiece = R::kPiece, VEC = R::VEC, kWaves = NT / kWave;
    __shared__ Lds<NT> s;
    const int lane = threadIdx.x % kWave, w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    if (threadIdx.x < kTable) s.table[threadIdx.x] = exp2(threadIdx.x / (double)kTable);
    for (int64_t n = blockIdx.x; n < a.N; n += gridDim.x) {
        R row;
        row.from = static_cast<const char*>(a.p.logits) + n * a.stride * T::kBytes;
        row.V = a.V, row.run = a.run, row.lane = lane, row.w = w;
        row.whole = (reinterpret_cast<uintptr_t>(row.from) & 15) == 0;

        // the largest logit and the lowest index that has it
        unsigned long long best = 0;
        row.words([&](int32_t i, uint32_t key) {
            const unsigned long long x = (unsigned long long)key << 32 | (uint32_t)~i;
            best = x > best ? x : best;
        });
#pragma unroll
        for (int d = kWave / 2; d > 0; d /= 2) {
            const unsigned long long x = __shfl_xor(best, d, kWave);
            best = x > best ? x : best;
        }
        __syncthreads();  // (the row before)
        if (lane == 0) s.wave[w] = best;
        __syncthreads();
        for (int j = 0; j < kWaves; ++j) best = s.wave[j] > best ? s.wave[j] : best;
        const uint32_t top = (uint32_t)(best >> 32);
        const double z_top = logit_of(top, kBits);
        const uint32_t none = key_of(-INFINITY, kBits);

        double T_n = a.p.temperature ? (double)a.p.temperature[n] : a.all.temperature;
        double top_p = a.p.top_p ? (double)a.p.top_p[n] : a.all.top_p, min_p = a.p.min_p ? (double)a.p.min_p[n] : a.all.min_p;
        const int32_t top_k = a.p.top_k ? a.p.top_k[n] : a.all.top_k;
        double u = a.p.u[n];
        if (T_n != T_n) T_n = 1.0;
        if (top_p != top_p) top_p = 1.0;
        if (min_p != min_p) min_p = 0.0;
        if (!(u > 0.0)) u = 0.0;
        if (top == none || !(T_n > 0.0)) {
            if (threadIdx.x == 0) {
                a.p.token[n] = top == none ? -1 : (int64_t)(uint32_t)~(uint32_t)best;
                if (a.p.prob) a.p.prob[n] = top == none ? 0.0f : 1.0f;
            }
            __syncthreads();
            continue;
        }
        const double scale = 1.0 / T_n;
        auto weight = [&](uint32_t key) -> double {
            if (key == top) return 1.0;
            if (key == none) return 0.0;
            return exp_of(((double)logit_of(key, kBits) - z_top) * scale, s.table);
        };
        // (sums of V weights of at most 2^unit stay below 2^63)
        const int unit = 62 - (32 - __builtin_clz((uint32_t)a.V));
        auto whole_weight = [&](uint32_t key) { return (unsigned long long)ldexp(weight(key), unit); };

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
                find_bin<NT>(s, s.count, need);
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
                    find_bin<NT>(s, s.weight, 1);  // (for the sum of all)
                    const double most = top_p > 0.0 ? __builtin_ceil(top_p * (double)s.total) : 1.0;
                    need = most < 1.0 ? 1 : (unsigned long long)most;
                    if (need > s.total) need = s.total;
                    __syncthreads();
                }
                find_bin<NT>(s, s.weight, need);
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
        const int32_t runs = (int32_t)(((int64_t)a.V + (int64_t)kPiece * a.run - 1) / ((int64_t)kPiece * a.run));
        if (ties >= 0) {
            for (int j = threadIdx.x; j < kMostBlocks; j += NT) s.count[j] = 0;
            if (threadIdx.x == 0) s.at = a.V;
            __syncthreads();
            row.pieces([&](int32_t piece, const uint32_t(&key)[VEC]) {
                uint32_t c = 0;
#pragma unroll
                for (int e = 0; e < VEC; ++e) c += key[e] == least && row.first_of(piece) + e < a.V;
                if (__builtin_amdgcn_ballot_w64(c > 0) == 0) return;
                c = wave_total(c);
                if (lane == 0) s.count[piece / a.run] += c;  // a run is one wave's
            });
            __syncthreads();
            if (w == 0) {
                uint32_t mine = 0;
                constexpr int kEach = kMostBlocks / kWave;
                for (int j = 0; j < kEach; ++j) mine += s.count[lane * kEach + j];
                uint32_t before = wave_upto(mine, lane) - mine;
                for (int j = 0; j < kEach; ++j) {
                    const uint32_t here = s.count[lane * kEach + j];
                    if (before < ties && ties <= before + here) s.bin = lane * kEach + j, s.above = before;
                    before += here;
                }
            }
            __syncthreads();
            if (w == 0) {  // the run, a piece at a time
                int64_t left = ties - (int64_t)s.above;
                const int32_t run = s.bin, all = (a.V + kPiece - 1) / kPiece;
                for (int32_t x = run * a.run; x < (run + 1) * a.run && x < all && left > 0; ++x) {
                    float z[VEC];
                    Pack<T, VEC>::unpack(row.fetch(row.first_of(x)), z);
                    uint32_t c = 0;
                    for (int e = 0; e < VEC; ++e) c += row.first_of(x) + e < a.V && key_of(z[e], kBits) == least;
                    const uint32_t upto = wave_upto(c, lane);
                    if (upto - c < left && left <= upto) {
                        int64_t mine = left - (upto - c);
                        for (int e = 0; e < VEC; ++e)
                            if (row.first_of(x) + e < a.V && key_of(z[e], kBits) == least && --mine == 0) s.at = (int32_t)row.first_of(x) + e;
                    }
                    left -= __shfl(upto, kWave - 1, kWave);
                }
            }
            __syncthreads();
            last_tie = s.at;
        }

        // the kept weights of every run
        auto kept = [&](int32_t i, uint32_t key) -> double {
            if (i >= a.V || key < least || (key == least && i > last_tie)) return 0.0;
            const double x = weight(key);
            return x >= min_p || key == top ? x : 0.0;
        };
        for (int j = threadIdx.x; j < kMostBlocks; j += NT) s.block[j] = 0.0;
        __syncthreads();
        {
            double mine = 0.0;
            row.pieces([&](int32_t piece, const uint32_t(&key)[VEC]) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) mine += kept((int32_t)(row.first_of(piece) + e), key[e]);
                if ((piece + 1) % a.run == 0 || piece + 1 == (a.V + kPiece - 1) / kPiece) {
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
            constexpr int kEach = kMostBlocks / kWave;
            double mine = 0.0;
            for (int j = 0; j < kEach; ++j) mine += s.block[lane * kEach + j];
            const double upto = wave_upto(mine, lane);
            const double sum = __shfl(upto, kWave - 1, kWave), want = u * sum;
            // the first run up to which there is more than `want`, else the last one that has something
            double before = upto - mine;
            int32_t run = -1, last = -1;
            double at_run = 0.0, at_last = 0.0;
            for (int j = 0; j < kEach; ++j) {
                const double here = s.block[lane * kEach + j];
                if (here > 0.0) {
                    last = lane * kEach + j, at_last = before;
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
            const int32_t all = (a.V + kPiece - 1) / kPiece;
            for (int32_t x = run * a.run; x < (run + 1) * a.run && x < all && token < 0; ++x) {
                float z[VEC];
                double f[VEC], c = 0.0;
                Pack<T, VEC>::unpack(row.fetch(row.first_of(x)), z);
                for (int e = 0; e < VEC; ++e) c += f[e] = kept((int32_t)(row.first_of(x) + e), key_of(z[e], kBits));
                const double upto = wave_upto(c, lane);
                double here = upto_here + (upto - c);
                int32_t mine = -1, my_last = -1;
                double fm = 0.0, fl = 0.0;
                for (int e = 0; e < VEC; ++e) {
                    here += f[e];
                    if (f[e] > 0.0) {
                        my_last = (int32_t)(row.first_of(x) + e), fl = f[e];
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
                upto_here += __shfl(upto, kWave - 1, kWave);
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
    const int64_t pieces = (a.V + kPiece - 1) / kPiece;
    a.run = (int32_t)((pieces + kMostBlocks - 1) / kMostBlocks);
    return launch_kernel(sample_kernel<T, NT>, dim3(workgroups_for(a.N, 1, NT)), dim3(NT), st, a);
}

template <typename T>
hy_status by_size(const SampleArgs& a, hipStream_t st) {
    return a.V * T::kBytes <= 256 * 16 ? run<T, 256>(a, st) : run<T, 1024>(a, st);
}

}  // namespace

hy_status launch_sample(const SamplePtrs& p, const SampleAll& all, int64_t N, int64_t V, int64_t stride, int32_t dtype, hipStream_t st) {
    const SampleArgs a{p, all, N, stride, (int32_t)V, 1};
    return dtype == HY_F32 ? by_size<F32>(a, st) : by_size<BF16>(a, st);
}

}  // namespace hy
