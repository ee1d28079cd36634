// One AdamW step over the tensors of a model in one launch:
//     m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,  p = p (1 - lr wd) - c1 m / (c2 sqrt(v) + eps),
// c1 = lr / (1 - b1^t), c2 = 1 / sqrt(1 - b2^t).  Every element is read once and written once: the bytes are what it costs.
//
// A workgroup takes a chunk of kChunk elements of one tensor, which a table in device memory tells it; its waves take blocks of
// 256, four neighbouring elements a lane.  With 8-bit states a block is also what shares a scale, so that its largest magnitude
// is a matter of one wave.  m and the root r of v are held as e4m3 values (448 at the most): r and not v, whose range is twice
// as wide in the exponent.  An r that is not zero is held as at least the smallest e4m3 value: the step divides by it.
// The products and sums are rounded one by one (no fused multiply-add): the 8-bit values depend on every bit in front of the
// rounding, and so they can be checked against any other program that follows the formulas.
//
// Measured: 34 million bf16 parameters with masters and fp32 states 155-158 us, 6.0 TB/s; 202 million with 8-bit states 563 us, 5.8
// TB/s, where vector instructions are 92% busy besides (the rounding one by one, the blocks' largest magnitudes).
#include "hy_common.hpp"
#include "hy_launch.hpp"

namespace hy {

namespace {

constexpr int kPer = 4;                               // elements of a lane
constexpr int kBlock = kAdamwBlock;                   // of a wave at a time
constexpr int kWaves = kAdamwThreads / kWave;
constexpr int kBlocks = kAdamwChunk / kBlock / kWaves;  // of a wave
static_assert(kPer * kWave == kBlock, "a wave takes a block");

struct AdamwArgs {
    const AdamwEntry* entries;
    const int32_t* owner;
    const float* grad_scale;
    float lr, beta1, keep1, beta2, keep2, c1, c2, eps;
};

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
    for (int d = kWave / 2; d > 0; d /= 2) x = fmaxf(x, __shfl_xor(x, d, kWave));
    return x;
}

// Four elements at p + i, as many as `n` of them exist; 0 for the others.
template <typename T>
__device__ __forceinline__ typename Pack<T, kPer>::Raw take(const void* p, int64_t i, int n, bool whole) {
    const char* at = static_cast<const char*>(p) + i * T::kBytes;
    if (whole) return Pack<T, kPer>::load_nt(at);
    float f[kPer] = {};
#pragma unroll
    for (int j = 0; j < kPer; ++j)
        if (j < n) {
            float one[1];
            Pack<T, 1>::unpack(Pack<T, 1>::load(at + j * T::kBytes), one);
            f[j] = one[0];
        }
    return Pack<T, kPer>::pack(f);
}
template <typename T>
__device__ __forceinline__ void give(void* p, int64_t i, int n, bool whole, const float (&f)[kPer]) {
    char* at = static_cast<char*>(p) + i * T::kBytes;
    if (whole) {
        Pack<T, kPer>::store_nt(at, Pack<T, kPer>::pack(f));
        return;
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j)
        if (j < n) {
            const float one[1] = {f[j]};
            Pack<T, 1>::store(at + j * T::kBytes, Pack<T, 1>::pack(one));
        }
}
// Four e4m3 values in a word.
__device__ __forceinline__ uint32_t take8(const void* p, int64_t i, int n, bool whole) {
    const uint8_t* at = static_cast<const uint8_t*>(p) + i;
    if (whole) return __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(at));
    uint32_t w = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j)
        if (j < n) w |= (uint32_t)at[j] << 8 * j;
    return w;
}
__device__ __forceinline__ void give8(void* p, int64_t i, int n, bool whole, uint32_t w) {
    uint8_t* at = static_cast<uint8_t*>(p) + i;
    if (whole) {
        __builtin_nontemporal_store(w, reinterpret_cast<uint32_t*>(at));
        return;
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j)
        if (j < n) at[j] = (uint8_t)(w >> 8 * j);
}
__device__ __forceinline__ void widen8(uint32_t w, float scale, float (&f)[kPer]) {
    f[0] = __builtin_amdgcn_cvt_f32_fp8(w, 0) * scale;
    f[1] = __builtin_amdgcn_cvt_f32_fp8(w, 1) * scale;
    f[2] = __builtin_amdgcn_cvt_f32_fp8(w, 2) * scale;
    f[3] = __builtin_amdgcn_cvt_f32_fp8(w, 3) * scale;
}
// The block's values as e4m3 and their scale.  What is not finite takes no part in the scale and is held as NaN.
template <bool ROOT>
__device__ __forceinline__ uint32_t narrow8(const float (&f)[kPer], float* scale) {
#pragma clang fp contract(off)
    constexpr float kTop = 448.0f, kTiny = 0x1p-100f, kLeast = 0x1p-9f;
    float top = 0.0f;
#pragma unroll
    for (int j = 0; j < kPer; ++j) top = fmaxf(top, fabsf(f[j]) < INFINITY ? fabsf(f[j]) : 0.0f);
    top = wave_max(top);
    const bool some = top >= kTiny;
    const float up = some ? kTop / top : 0.0f;
    *scale = some ? top * (1.0f / kTop) : 0.0f;
    float y[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        y[j] = f[j] * up;
        if (ROOT && some && f[j] > 0.0f) y[j] = fmaxf(y[j], kLeast);
        if (fabsf(f[j]) == INFINITY) y[j] = NAN;
    }
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
}

template <typename P, typename G, bool MASTER, bool NARROW>
__global__ __launch_bounds__(kWaves * kWave) void adamw_kernel(AdamwArgs a) {
#pragma clang fp contract(off)
    const AdamwEntry e = a.entries[a.owner[blockIdx.x]];
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int64_t first = ((int64_t)blockIdx.x - e.first_chunk) * kAdamwChunk + w * (kBlocks * kBlock);
    const float gs = a.grad_scale ? *a.grad_scale : 1.0f;
    const float shrink = 1.0f - a.lr * e.weight_decay;
    using PP = std::conditional_t<MASTER, F32, P>;  // what the step is taken on
    const void* from = MASTER ? (const void*)e.master : e.param;

    typename Pack<PP, kPer>::Raw rp[kBlocks];
    typename Pack<G, kPer>::Raw rg[kBlocks];
    Words<4> rm[kBlocks], rv[kBlocks];
    uint32_t cm[kBlocks], cv[kBlocks];
    float sm[kBlocks], sv[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
        const int64_t i = first + b * kBlock + lane * kPer;
        const int64_t left = e.count - i;
        const int n = left < 0 ? 0 : left < kPer ? (int)left : kPer;
        const bool whole = n == kPer && e.aligned;
        rp[b] = take<PP>(from, i, n, whole);
        rg[b] = take<G>(e.grad, i, n, whole);
        if constexpr (NARROW) {
            const bool there = first + b * kBlock < e.count;
            const int64_t s = first / kBlock + b;
            cm[b] = take8(e.exp_avg, i, n, whole);
            cv[b] = take8(e.exp_avg_sq, i, n, whole);
            sm[b] = there ? e.avg_scale[s] : 0.0f;
            sv[b] = there ? e.sq_scale[s] : 0.0f;
        } else {
            rm[b] = take<F32>(e.exp_avg, i, n, whole);
            rv[b] = take<F32>(e.exp_avg_sq, i, n, whole);
        }
    }
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
        const int64_t i = first + b * kBlock + lane * kPer;
        const int64_t left = e.count - i;
        const int n = left < 0 ? 0 : left < kPer ? (int)left : kPer;
        const bool whole = n == kPer && e.aligned;
        float p[kPer], g[kPer], m[kPer], v[kPer], r[kPer];
        Pack<PP, kPer>::unpack(rp[b], p);
        Pack<G, kPer>::unpack(rg[b], g);
        if constexpr (NARROW) {
            widen8(cm[b], sm[b], m);
            widen8(cv[b], sv[b], v);
#pragma unroll
            for (int j = 0; j < kPer; ++j) v[j] *= v[j];
        } else {
            Pack<F32, kPer>::unpack(rm[b], m);
            Pack<F32, kPer>::unpack(rv[b], v);
        }
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const float gj = g[j] * gs;
            m[j] = m[j] * a.beta1 + gj * a.keep1;
            v[j] = v[j] * a.beta2 + gj * gj * a.keep2;
            r[j] = sqrtf(v[j]);
            p[j] = p[j] * shrink - m[j] * a.c1 / (r[j] * a.c2 + a.eps);
        }
        if constexpr (MASTER) give<F32>(e.master, i, n, whole, p);
        give<P>(e.param, i, n, whole, p);
        if constexpr (NARROW) {
            float tm, tv;
            const uint32_t wm = narrow8<false>(m, &tm), wv = narrow8<true>(r, &tv);
            give8(e.exp_avg, i, n, whole, wm);
            give8(e.exp_avg_sq, i, n, whole, wv);
            if (lane == 0 && n > 0) {
                const int64_t s = first / kBlock + b;
                e.avg_scale[s] = tm;
                e.sq_scale[s] = tv;
            }
        } else {
            give<F32>(e.exp_avg, i, n, whole, m);
            give<F32>(e.exp_avg_sq, i, n, whole, v);
        }
    }
}

template <typename P, typename G, bool MASTER>
hy_status run(const AdamwArgs& a, int64_t chunks, int32_t bits, hipStream_t st) {
    const dim3 grid((uint32_t)chunks), block(kWaves * kWave);
    return bits == 8 ? launch_kernel(adamw_kernel<P, G, MASTER, true>, grid, block, st, a)
                     : launch_kernel(adamw_kernel<P, G, MASTER, false>, grid, block, st, a);
}

template <typename G>
hy_status by_param(const AdamwArgs& a, const AdamwShape& s, hipStream_t st) {
    if (s.param == HY_F32) return run<F32, G, false>(a, s.chunks, s.bits, st);
    return s.master ? run<BF16, G, true>(a, s.chunks, s.bits, st) : run<BF16, G, false>(a, s.chunks, s.bits, st);
}

}  // namespace

hy_status launch_adamw(const AdamwEntry* entries, const int32_t* owner, const float* grad_scale, const AdamwHyper& h,
                       const AdamwShape& s, hipStream_t st) {
    AdamwArgs a{};
    a.entries = entries, a.owner = owner, a.grad_scale = grad_scale;
    a.lr = (float)h.lr, a.beta1 = (float)h.beta1, a.beta2 = (float)h.beta2, a.eps = (float)h.eps;
    a.keep1 = (float)(1.0 - h.beta1), a.keep2 = (float)(1.0 - h.beta2);
    a.c1 = (float)(h.lr / h.bias1), a.c2 = (float)(1.0 / h.bias2_root);
    return s.grad == HY_F32 ? by_param<F32>(a, s, st) : by_param<BF16>(a, s, st);
}

}  // namespace hy
