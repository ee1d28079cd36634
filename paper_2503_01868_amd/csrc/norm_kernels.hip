// Root-mean-square norm of rows with the residual's addition in front, and its gradients:
//     h = x + r (rounded),  rstd = 1 / sqrt(mean h^2 + eps),  y = h rstd w
//     dx = dh + rstd (w dy - h rstd^2 mean(w dy h)),  dw = sum over rows of dy h rstd
// Every element is read once and written once: the bytes are what it costs.  A row stays in the registers of the lanes that share
// it (a wave, 4 waves or 16: TPR lanes with N pieces of 16 bytes each) between its sum and its output; rows that do not fit are
// read again, from the sum just written where there is one.  Sums run over a lane's elements, the lanes of a wave by halves, and the
// waves in their order, whatever the timing.  8192 rows of 4096 bf16 numbers with the residual (MI355X): forward 46-54 us, 8-bit output 45-49
// (268 and 235 MB; a large copy moves 5.6 TB/s), gradients 41-43 and 4 for the sum of dw's shares.
#include <type_traits>

#include "hy_common.hpp"
#include "hy_launch.hpp"

namespace hy {

namespace {

constexpr float kTop = 448.0f, kTiny = 0x1p-100f;  // of e4m3; rows below it are zeros
constexpr int kReduceColumns = 64, kReduceGroups = 16;

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
    for (int d = kWave / 2; d > 0; d /= 2) x += __shfl_xor(x, d, kWave);
    return x;
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
    for (int d = kWave / 2; d > 0; d /= 2) x = fmaxf(x, __shfl_xor(x, d, kWave));
    return x;
}

// Sum and maximum over the TPR lanes of a row.  `turn` alternates between two places, so that one barrier is enough.
template <int TPR, bool MAX>
__device__ __forceinline__ void over_row(float& sum, float& top, float (*lds)[2][TPR / kWave], int turn) {
    sum = wave_sum(sum);
    if constexpr (MAX) top = wave_max(top);
    if constexpr (TPR > kWave) {
        const int w = threadIdx.x / kWave;
        if (threadIdx.x % kWave == 0) {
            lds[turn][0][w] = sum;
            if constexpr (MAX) lds[turn][1][w] = top;
        }
        __syncthreads();
        sum = 0.0f;
        top = 0.0f;
#pragma unroll
        for (int i = 0; i < TPR / kWave; ++i) {
            sum += lds[turn][0][i];
            if constexpr (MAX) top = fmaxf(top, lds[turn][1][i]);
        }
    }
}

struct NormArgs {
    NormPtrs p;
    int64_t N, D, x_stride, r_stride;
    float eps, inverse;  // 1 / D
};

// The VEC numbers of piece i of a row, zeros behind its end.
template <typename T, int VEC>
__device__ __forceinline__ void piece(const char* row, int64_t i, int64_t D, float (&f)[VEC]) {
    if (i * VEC < D) {
        Pack<T, VEC>::unpack(Pack<T, VEC>::load(row + i * VEC * T::kBytes), f);
    } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) f[j] = 0.0f;
    }
}
template <typename T, int VEC>
__device__ __forceinline__ void piece_nt(const char* row, int64_t i, int64_t D, float (&f)[VEC]) {
    if (i * VEC < D) {
        Pack<T, VEC>::unpack(Pack<T, VEC>::load_nt(row + i * VEC * T::kBytes), f);
    } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) f[j] = 0.0f;
    }
}

__device__ __forceinline__ uint32_t two_e4m3(float a, float b, float up) {
    a = fabsf(a) == INFINITY ? NAN : a * up;
    b = fabsf(b) == INFINITY ? NAN : b * up;
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xffffu;
}
template <int VEC>
__device__ __forceinline__ void store_e4m3(void* row, int64_t i, const float (&u)[VEC], float up) {
    uint8_t* at = static_cast<uint8_t*>(row) + i * VEC;
    if constexpr (VEC == 1) {
        *at = (uint8_t)two_e4m3(u[0], 0.0f, up);
    } else {
        uint32_t w[VEC / 4];
#pragma unroll
        for (int j = 0; j < VEC / 4; ++j) w[j] = two_e4m3(u[4 * j], u[4 * j + 1], up) | two_e4m3(u[4 * j + 2], u[4 * j + 3], up) << 16;
        Words<VEC / 4> o;
#pragma unroll
        for (int j = 0; j < VEC / 4; ++j) o.w[j] = w[j];
        store_words<VEC / 4>(at, o);
    }
}

// h of piece i: x, plus the residual and rounded to T if there is one.  Streaming loads: 8192 x 4096 to 8 bits 51 -> 45 us a call.
template <typename T, int VEC>
__device__ __forceinline__ void sum_piece(const NormArgs& a, int64_t n, int64_t i, float (&h)[VEC]) {
    const char* x = static_cast<const char*>(a.p.x) + n * a.x_stride * T::kBytes;
    piece_nt<T, VEC>(x, i, a.D, h);
    if (a.p.residual) {
        float r[VEC];
        piece_nt<T, VEC>(static_cast<const char*>(a.p.residual) + n * a.r_stride * T::kBytes, i, a.D, r);
#pragma unroll
        for (int j = 0; j < VEC; ++j) h[j] += r[j];
        Pack<T, VEC>::unpack(Pack<T, VEC>::pack(h), h);
    }
}

template <typename T, int VEC, int TPR, int N, bool EIGHT, bool LONG>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void norm_kernel(NormArgs a) {
#pragma clang fp contract(off)
    constexpr int kRows = TPR < 256 ? 256 / TPR : 1;  // rows of a workgroup
    __shared__ float lds[2][2][TPR / kWave];
    const int lane = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    const int64_t pieces = (a.D + VEC - 1) / VEC;
    int turn = 0;
    for (int64_t n = (int64_t)blockIdx.x * kRows + sub; n < a.N; n += (int64_t)gridDim.x * kRows, turn ^= 1) {
        char* const total = static_cast<char*>(a.p.h) + n * a.D * T::kBytes;
        float h[N][VEC];
        float sum = 0.0f, top = 0.0f;
        auto take = [&](int64_t i, float (&f)[VEC]) {
            sum_piece<T, VEC>(a, n, i, f);
            if (a.p.h && i < pieces) Pack<T, VEC>::store(total + i * VEC * T::kBytes, Pack<T, VEC>::pack(f));
#pragma unroll
            for (int j = 0; j < VEC; ++j) sum = fmaf(f[j], f[j], sum);
            if constexpr (EIGHT) {
                float w[VEC];
                if (a.p.w) piece<T, VEC>(static_cast<const char*>(a.p.w), i, a.D, w);
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float u = a.p.w ? f[j] * w[j] : f[j];
                    top = fmaxf(top, fabsf(u) < INFINITY ? fabsf(u) : 0.0f);
                }
            }
        };
        if constexpr (LONG) {
            for (int64_t i = lane; i < pieces; i += TPR) take(i, h[0]);
        } else {
#pragma unroll
            for (int x = 0; x < N; ++x) take(x * TPR + lane, h[x]);
        }
        over_row<TPR, EIGHT>(sum, top, lds, turn);
        const float rstd = 1.0f / sqrtf(sum * a.inverse + a.eps);
        const bool some = top >= kTiny;
        const float up = some ? kTop / top : 0.0f;
        if (lane == 0) {
            if (a.p.rstd) a.p.rstd[n] = rstd;
            if constexpr (EIGHT) a.p.y_scale[n] = some ? top * (1.0f / kTop) * rstd : 0.0f * rstd;
        }
        auto give = [&](int64_t i, const float (&f)[VEC]) {
            if (i >= pieces) return;
            float w[VEC], y[VEC];
            if (a.p.w) piece<T, VEC>(static_cast<const char*>(a.p.w), i, a.D, w);
            if constexpr (EIGHT) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) y[j] = a.p.w ? f[j] * w[j] : f[j];
                store_e4m3<VEC>(static_cast<char*>(a.p.y) + n * a.D, i, y, up);
            } else {
#pragma unroll
                for (int j = 0; j < VEC; ++j) y[j] = a.p.w ? f[j] * rstd * w[j] : f[j] * rstd;
                Pack<T, VEC>::store(static_cast<char*>(a.p.y) + (n * a.D + i * VEC) * T::kBytes, Pack<T, VEC>::pack(y));
            }
        };
        if constexpr (LONG) {
            for (int64_t i = lane; i < pieces; i += TPR) {
                if (a.p.h) piece<T, VEC>(total, i, a.D, h[0]);  // what this lane has just written
                else sum_piece<T, VEC>(a, n, i, h[0]);
                give(i, h[0]);
            }
        } else {
#pragma unroll
            for (int x = 0; x < N; ++x) give(x * TPR + lane, h[x]);
        }
    }
}

// A workgroup (TPR = 64: each wave) keeps its share of dw in registers over all its rows and leaves it in the workspace.  Rows that do
// not fit keep it there (LONG: the workspace begins as zeros, which every lane sets for its own pieces).
template <typename T, int VEC, int TPR, int N, bool LONG>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void norm_bwd_kernel(NormArgs a, float* partial) {
    constexpr int kRows = TPR < 256 ? 256 / TPR : 1;
    __shared__ float lds[2][2][TPR / kWave];
    const int lane = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    const int64_t pieces = (a.D + VEC - 1) / VEC, group = (int64_t)blockIdx.x * kRows + sub;
    const char *w = static_cast<const char*>(a.p.w), *dh = static_cast<const char*>(a.p.dh);
    float* const mine = partial ? partial + group * a.D : nullptr;
    float dw[LONG ? 1 : N][VEC] = {};
    if (LONG && partial)
        for (int64_t i = lane; i < pieces; i += TPR)
#pragma unroll
            for (int j = 0; j < VEC; ++j) mine[i * VEC + j] = 0.0f;
    int turn = 0;
    if constexpr (LONG) {
        for (int64_t n = group; n < a.N; n += (int64_t)gridDim.x * kRows, turn ^= 1) {
            const char *hrow = static_cast<const char*>(a.p.h) + n * a.D * T::kBytes, *dyrow = static_cast<const char*>(a.p.dy) + n * a.D * T::kBytes;
            const float rstd = a.p.rstd[n];
            float h[VEC], dy[VEC], fw[VEC];
            float sum = 0.0f, none = 0.0f;
            for (int64_t i = lane; i < pieces; i += TPR) {
                piece_nt<T, VEC>(hrow, i, a.D, h);
                piece_nt<T, VEC>(dyrow, i, a.D, dy);
                if (partial)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) mine[i * VEC + j] = fmaf(dy[j] * h[j], rstd, mine[i * VEC + j]);
                if (w) piece<T, VEC>(w, i, a.D, fw);
#pragma unroll
                for (int j = 0; j < VEC; ++j) sum = fmaf(w ? dy[j] * fw[j] : dy[j], h[j], sum);
            }
            over_row<TPR, false>(sum, none, lds, turn);
            const float c = sum * a.inverse * (rstd * rstd);
            for (int64_t i = lane; i < pieces; i += TPR) {
                float o[VEC], more[VEC] = {};
                piece<T, VEC>(hrow, i, a.D, h);
                piece<T, VEC>(dyrow, i, a.D, dy);
                if (w) piece<T, VEC>(w, i, a.D, fw);
                if (dh) piece_nt<T, VEC>(dh + n * a.D * T::kBytes, i, a.D, more);
#pragma unroll
                for (int j = 0; j < VEC; ++j) o[j] = fmaf(rstd, (w ? dy[j] * fw[j] : dy[j]) - h[j] * c, more[j]);
                Pack<T, VEC>::store(static_cast<char*>(a.p.dx) + (n * a.D + i * VEC) * T::kBytes, Pack<T, VEC>::pack(o));
            }
        }
        return;
    }
    // A row's numbers are on their way while the row before is summed: 8192 rows of 4096 bf16 numbers 90 us without it.
    using Raw = typename Pack<T, VEC>::Raw;
    Raw next_h[N], next_dy[N], next_dh[N], raw_w[N];
    float next_rstd = 0.0f;
    const int64_t step = (int64_t)gridDim.x * kRows;
    auto load = [&](int64_t n) {
        const int64_t row = n * a.D;
#pragma unroll
        for (int x = 0; x < N; ++x) {
            const int64_t i = x * TPR + lane;
            if (i >= pieces) continue;
            next_h[x] = Pack<T, VEC>::load_nt(static_cast<const char*>(a.p.h) + (row + i * VEC) * T::kBytes);
            next_dy[x] = Pack<T, VEC>::load_nt(static_cast<const char*>(a.p.dy) + (row + i * VEC) * T::kBytes);
            if (dh) next_dh[x] = Pack<T, VEC>::load_nt(dh + (row + i * VEC) * T::kBytes);
        }
        next_rstd = a.p.rstd[n];
    };
    if (w)
#pragma unroll
        for (int x = 0; x < N; ++x)
            if (x * TPR + lane < pieces) raw_w[x] = Pack<T, VEC>::load(w + (int64_t)(x * TPR + lane) * VEC * T::kBytes);
    if (group < a.N) load(group);
    for (int64_t n = group; n < a.N; n += step, turn ^= 1) {
        const float rstd = next_rstd;
        Raw rh[N], rdy[N], rdh[N];
        float sum = 0.0f, none = 0.0f;
#pragma unroll
        for (int x = 0; x < N; ++x) rh[x] = next_h[x], rdy[x] = next_dy[x], rdh[x] = next_dh[x];
        if (n + step < a.N) load(n + step);
#pragma unroll
        for (int x = 0; x < N; ++x) {
            if (x * TPR + lane >= pieces) continue;
            float h[VEC], dy[VEC], fw[VEC];
            Pack<T, VEC>::unpack(rh[x], h);
            Pack<T, VEC>::unpack(rdy[x], dy);
            if (w) Pack<T, VEC>::unpack(raw_w[x], fw);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                dw[x][j] = fmaf(dy[j] * h[j], rstd, dw[x][j]);
                sum = fmaf(w ? dy[j] * fw[j] : dy[j], h[j], sum);
            }
        }
        over_row<TPR, false>(sum, none, lds, turn);
        const float c = sum * a.inverse * (rstd * rstd);
#pragma unroll
        for (int x = 0; x < N; ++x) {
            const int64_t i = x * TPR + lane;
            if (i >= pieces) continue;
            float h[VEC], dy[VEC], fw[VEC], more[VEC] = {}, o[VEC];
            Pack<T, VEC>::unpack(rh[x], h);
            Pack<T, VEC>::unpack(rdy[x], dy);
            if (w) Pack<T, VEC>::unpack(raw_w[x], fw);
            if (dh) Pack<T, VEC>::unpack(rdh[x], more);
#pragma unroll
            for (int j = 0; j < VEC; ++j) o[j] = fmaf(rstd, (w ? dy[j] * fw[j] : dy[j]) - h[j] * c, more[j]);
            Pack<T, VEC>::store(static_cast<char*>(a.p.dx) + (n * a.D + i * VEC) * T::kBytes, Pack<T, VEC>::pack(o));
        }
    }
    if constexpr (!LONG) {
        if (!partial) return;
#pragma unroll
        for (int x = 0; x < N; ++x) {
            const int64_t i = x * TPR + lane;
            if (i >= pieces) continue;
            if constexpr (VEC == 1) {
                mine[i] = dw[x][0];
            } else {
#pragma unroll
                for (int j = 0; j < VEC; j += 4)
                    *reinterpret_cast<float4*>(mine + i * VEC + j) = make_float4(dw[x][j], dw[x][j + 1], dw[x][j + 2], dw[x][j + 3]);
            }
        }
    }
}

// dw[d] = sum of the shares, 16 runs of them side by side and then the runs.
template <typename T>
__global__ __launch_bounds__(kReduceColumns* kReduceGroups) void norm_dw_kernel(const float* partial, void* dw, int64_t shares, int64_t D) {
    __shared__ float lds[kReduceGroups][kReduceColumns];
    const int c = threadIdx.x % kReduceColumns, g = threadIdx.x / kReduceColumns;
    const int64_t each = (shares + kReduceGroups - 1) / kReduceGroups, first = g * each, last = first + each < shares ? first + each : shares;
    for (int64_t d0 = (int64_t)blockIdx.x * kReduceColumns; d0 < D; d0 += (int64_t)gridDim.x * kReduceColumns) {
        const int64_t d = d0 + c;
        float sum = 0.0f;
        if (d < D) {
            int64_t s = first;
            for (; s + 8 <= last; s += 8) {
                float f[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = partial[(s + j) * D + d];
#pragma unroll
                for (int j = 0; j < 8; ++j) sum += f[j];
            }
            for (; s < last; ++s) sum += partial[s * D + d];
        }
        lds[g][c] = sum;
        __syncthreads();
        if (g == 0 && d < D) {
            sum = 0.0f;
#pragma unroll
            for (int j = 0; j < kReduceGroups; ++j) sum += lds[j][c];
            const float one[1] = {sum};
            Pack<T, 1>::store(static_cast<char*>(dw) + d * T::kBytes, Pack<T, 1>::pack(one));
        }
        __syncthreads();
    }
}

// Lanes of a row and its pieces in each.
template <typename F>
hy_status by_row(int64_t pieces, F&& f) {
    using std::integral_constant;
    if (pieces <= 64) return f(integral_constant<int, 64>{}, integral_constant<int, 1>{}, std::false_type{});
    if (pieces <= 128) return f(integral_constant<int, 64>{}, integral_constant<int, 2>{}, std::false_type{});
    if (pieces <= 256) return f(integral_constant<int, 256>{}, integral_constant<int, 1>{}, std::false_type{});
    if (pieces <= 512) return f(integral_constant<int, 256>{}, integral_constant<int, 2>{}, std::false_type{});
    if (pieces <= 1024) return f(integral_constant<int, 256>{}, integral_constant<int, 4>{}, std::false_type{});
    if (pieces <= 2048) return f(integral_constant<int, 1024>{}, integral_constant<int, 2>{}, std::false_type{});
    return f(integral_constant<int, 1024>{}, integral_constant<int, 1>{}, std::true_type{});
}

// Rows that begin where 16 bytes do and end with a whole piece are moved by 16 bytes, others by elements.
template <typename F>
hy_status by_type(int32_t dtype, bool wide, F&& f) {
    if (dtype == HY_F32) return wide ? f(F32{}, std::integral_constant<int, 4>{}) : f(F32{}, std::integral_constant<int, 1>{});
    return wide ? f(BF16{}, std::integral_constant<int, 8>{}) : f(BF16{}, std::integral_constant<int, 1>{});
}

bool wide_rows(const NormPtrs& p, const NormShape& s) {
    const int64_t vec = s.dtype == HY_F32 ? 4 : 8;
    const void* all[] = {p.x, p.residual, p.w, p.y, p.h, p.dy, p.dh, p.dx};
    for (const void* q : all)
        if (reinterpret_cast<uintptr_t>(q) % 16 != 0) return false;
    return s.D % vec == 0 && s.x_stride % vec == 0 && s.r_stride % vec == 0;
}

NormArgs norm_args(const NormPtrs& p, const NormShape& s) {
    return NormArgs{p, s.N, s.D, s.x_stride, s.r_stride, (float)s.eps, (float)(1.0 / (double)s.D)};
}

// Shares of dw: two workgroups for each compute unit, fewer rows than that a share each.
constexpr int64_t kShares = 512;
int64_t shares_of(int64_t N) { return N < kShares ? N : kShares; }

}  // namespace

int64_t norm_bwd_workspace_bytes(int64_t N, int64_t D) { return (shares_of(N) + 3) / 4 * 4 * D * 4; }

hy_status launch_norm_fwd(const NormPtrs& p, const NormShape& s, hipStream_t st) {
    const NormArgs a = norm_args(p, s);
    return by_type(s.dtype, wide_rows(p, s), [&](auto t, auto vec) {
        using T = decltype(t);
        constexpr int VEC = decltype(vec)::value;
        return by_row((s.D + VEC - 1) / VEC, [&](auto tpr, auto n, auto is_long) {
            constexpr int TPR = decltype(tpr)::value, N = decltype(n)::value, threads = TPR < 256 ? 256 : TPR;
            constexpr bool LONG = decltype(is_long)::value;
            const dim3 grid(workgroups_for(s.N, threads / TPR, threads)), block(threads);
            return p.y_scale ? launch_kernel(norm_kernel<T, VEC, TPR, N, true, LONG>, grid, block, st, a)
                             : launch_kernel(norm_kernel<T, VEC, TPR, N, false, LONG>, grid, block, st, a);
        });
    });
}

hy_status launch_norm_bwd(const NormPtrs& p, const NormShape& s, void* ws, hipStream_t st) {
    const NormArgs a = norm_args(p, s);
    float* const partial = p.dw ? static_cast<float*>(ws) : nullptr;
    int64_t shares = 0;
    const hy_status rc = s.N == 0 ? HY_OK : by_type(s.dtype, wide_rows(p, s), [&](auto t, auto vec) {
        using T = decltype(t);
        constexpr int VEC = decltype(vec)::value;
        return by_row((s.D + VEC - 1) / VEC, [&](auto tpr, auto n, auto is_long) {
            constexpr int TPR = decltype(tpr)::value, N = decltype(n)::value, threads = TPR < 256 ? 256 : TPR, rows = threads / TPR;
            const int64_t groups = (shares_of(s.N) + rows - 1) / rows;
            shares = groups * rows;
            return launch_kernel(norm_bwd_kernel<T, VEC, TPR, N, decltype(is_long)::value>, dim3((uint32_t)groups), dim3(threads), st, a, partial);
        });
    });
    if (rc != HY_OK || !p.dw) return rc;
    constexpr int threads = kReduceColumns * kReduceGroups;
    const dim3 grid(workgroups_for(s.D, kReduceColumns, threads));
    return s.dtype == HY_F32 ? launch_kernel(norm_dw_kernel<F32>, grid, dim3(threads), st, static_cast<const float*>(partial), p.dw, shares, s.D)
                             : launch_kernel(norm_dw_kernel<BF16>, grid, dim3(threads), st, static_cast<const float*>(partial), p.dw, shares, s.D);
}

}  // namespace hy
