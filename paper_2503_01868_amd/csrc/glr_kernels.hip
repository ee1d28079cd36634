// Gated linear recurrence: s[t] = a[t] s[t-1] + u[t], y[t] = q[t] s[t], a = exp(g), u = k v, and its gradients.
//
// The recurrence is linear, so a stretch of steps acts on the state before it as s -> A s + H with two numbers per channel,
// A the product of its a and H its result from zero.  Tiles of kGlrRows steps are summed up this way in parallel, a scan over
// the tiles' pairs gives each tile its incoming state (the "marks"), and the tile is walked from there.  The gradient runs
// the other way with the same A: with m[t] = dLoss/ds[t] and c[t] = a[t] m[t] (what a step hands to the one before it),
// m[t] = q[t] dy[t] + c[t+1], so a stretch takes c -> A c + C.
#include "hy_common.hpp"
#include "hy_launch.hpp"

namespace hy {

namespace {

constexpr int kWaves = 8;                      // waves of a workgroup, one after the other in time
constexpr int kRowsPerWave = kGlrRows / kWaves;

struct Src {
    const char* p;
    int64_t bstride, rstride;  // bytes between batch items and between rows
};

struct GlrArgs {
    Src q, k, v, g, dy;
    char *y, *dq, *dk, *dv, *dg;
    float* dg_parts;           // [B, L, D / part] fp32, where a group is summed up in parts
    const float* marks;        // [B, tiles, D] states before the tiles
    const float* rmarks;       // [B, tiles, D] c of the step after the tile
    float *A, *H;              // [B, tiles, D]
    int64_t L, D;
    int32_t tiles, ncb, group, part;  // part: channels of a group that a wave sums up (a power of two)
};

// VEC channels per lane; SHARED: both channels of a lane (or its only one) take the gate of their group.
template <typename T, int VEC, bool SHARED>
struct Io {
    using P = Pack<T, VEC>;
    using G = Pack<T, SHARED ? 1 : VEC>;
    static __device__ __forceinline__ void gates(const typename G::Raw& r, float (&a)[VEC]) {
        float f[SHARED ? 1 : VEC];
        G::unpack(r, f);
#pragma unroll
        for (int i = 0; i < VEC; ++i) a[i] = i == 0 || !SHARED ? expf(f[SHARED ? 0 : i]) : a[0];
    }
};

struct Place {
    int w, lane, tile;
    int64_t b, c, row0;   // row0: the wave's first step
    int rows;             // steps of the sequence that the wave has
    bool there;           // its channels exist
};

template <int VEC>
__device__ __forceinline__ Place place(const GlrArgs& a) {
    Place p;
    p.w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    p.lane = threadIdx.x % kWave;
    uint32_t i = blockIdx.x;
    const uint32_t cb = i % (uint32_t)a.ncb;
    i /= (uint32_t)a.ncb;
    p.tile = i % (uint32_t)a.tiles;
    p.b = i / (uint32_t)a.tiles;
    p.c = (int64_t)cb * (kWave * VEC) + p.lane * VEC;
    p.there = p.c < a.D;
    if (!p.there) p.c = 0;
    p.row0 = (int64_t)p.tile * kGlrRows + p.w * kRowsPerWave;
    const int64_t left = a.L - p.row0;
    p.rows = left < 0 ? 0 : left < kRowsPerWave ? (int)left : kRowsPerWave;
    return p;
}

// The wave's rows of a tensor; steps behind the last are the last one again (their values are not used).
template <typename PK>
__device__ __forceinline__ void load_rows(typename PK::Raw (&r)[kRowsPerWave], const Src& s, const GlrArgs& a, const Place& p,
                                          int64_t lane_bytes) {
    const char* base = s.p + p.b * s.bstride + lane_bytes;
#pragma unroll
    for (int i = 0; i < kRowsPerWave; ++i) {
        const int64_t t = p.row0 + i < a.L ? p.row0 + i : a.L - 1;
        r[i] = PK::load_nt(base + t * s.rstride);
    }
}

// What the waves before (or, REV, behind) wave w of a workgroup make of the state at the workgroup's edge.
template <int VEC, bool REV>
__device__ __forceinline__ void join(const float (&lA)[kWaves][kWave * VEC], const float (&lH)[kWaves][kWave * VEC], int w,
                                     int lane, float (&A)[VEC], float (&H)[VEC]) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) A[i] = 1.0f, H[i] = 0.0f;
    for (int x = REV ? kWaves - 1 : 0; REV ? x > w : x < w; x += REV ? -1 : 1)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const float xa = lA[x][lane * VEC + i];
            H[i] = fmaf(xa, H[i], lH[x][lane * VEC + i]);
            A[i] *= xa;
        }
}

// A and H (REV: C) of every tile.
template <typename T, int VEC, bool SHARED, bool REV>
__global__ __launch_bounds__(kWaves * kWave) void glr_sum_kernel(GlrArgs a) {
    using P = Pack<T, VEC>;
    using IO = Io<T, VEC, SHARED>;
    __shared__ float lA[kWaves][kWave * VEC], lH[kWaves][kWave * VEC];
    const Place p = place<VEC>(a);
    const int64_t at = p.c * T::kBytes, gat = p.c / a.group * T::kBytes;
    typename P::Raw x[kRowsPerWave], y[kRowsPerWave];
    typename IO::G::Raw g[kRowsPerWave];
    load_rows<P>(x, REV ? a.q : a.k, a, p, at);
    load_rows<P>(y, REV ? a.dy : a.v, a, p, at);
    load_rows<typename IO::G>(g, a.g, a, p, gat);
    float A[VEC], H[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) A[i] = 1.0f, H[i] = 0.0f;
#pragma unroll
    for (int j = 0; j < kRowsPerWave; ++j) {
        const int r = REV ? kRowsPerWave - 1 - j : j;
        if (r < p.rows) {
            float fx[VEC], fy[VEC], ga[VEC];
            P::unpack(x[r], fx);
            P::unpack(y[r], fy);
            IO::gates(g[r], ga);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                H[i] = REV ? ga[i] * fmaf(fx[i], fy[i], H[i]) : fmaf(ga[i], H[i], fx[i] * fy[i]);
                A[i] *= ga[i];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) lA[p.w][p.lane * VEC + i] = A[i], lH[p.w][p.lane * VEC + i] = H[i];
    __syncthreads();
    if (p.w == (REV ? 0 : kWaves - 1) && p.there) {
        float eA[VEC], eH[VEC];
        join<VEC, REV>(lA, lH, p.w, p.lane, eA, eH);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int64_t o = (p.b * a.tiles + p.tile) * a.D + p.c + i;
            a.A[o] = A[i] * eA[i];
            a.H[o] = fmaf(A[i], eH[i], H[i]);
        }
    }
}

// marks[b][tile][c]: the state before (REV: c behind) each tile; `out`: what comes out at the end.  A lane per channel.
template <bool REV>
__global__ __launch_bounds__(256) void glr_scan_kernel(const float* A, const float* H, const float* in, float* marks, float* out,
                                                       int64_t B, int64_t tiles, int64_t D) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= B * D) return;
    const int64_t b = i / D, c = i % D;
    float s = in ? in[i] : 0.0f;
    for (int64_t j = 0; j < tiles; ++j) {
        const int64_t o = (b * tiles + (REV ? tiles - 1 - j : j)) * D + c;
        marks[o] = s;
        s = fmaf(A[o], s, H[o]);
    }
    if (out) out[i] = s;
}

// y of every tile from the state before it.
template <typename T, int VEC, bool SHARED>
__global__ __launch_bounds__(kWaves * kWave) void glr_fwd_kernel(GlrArgs a) {
    using P = Pack<T, VEC>;
    using IO = Io<T, VEC, SHARED>;
    __shared__ float lA[kWaves][kWave * VEC], lH[kWaves][kWave * VEC];
    const Place p = place<VEC>(a);
    const int64_t at = p.c * T::kBytes, gat = p.c / a.group * T::kBytes;
    typename P::Raw q[kRowsPerWave], k[kRowsPerWave], v[kRowsPerWave];
    typename IO::G::Raw g[kRowsPerWave];
    load_rows<P>(k, a.k, a, p, at);
    load_rows<P>(v, a.v, a, p, at);
    load_rows<typename IO::G>(g, a.g, a, p, gat);
    load_rows<P>(q, a.q, a, p, at);
    float A[VEC], H[VEC], pa[kRowsPerWave][VEC], ph[kRowsPerWave][VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) A[i] = 1.0f, H[i] = 0.0f;
#pragma unroll
    for (int r = 0; r < kRowsPerWave; ++r) {
        float fk[VEC], fv[VEC], ga[VEC];
        P::unpack(k[r], fk);
        P::unpack(v[r], fv);
        IO::gates(g[r], ga);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            if (r < p.rows) {
                H[i] = fmaf(ga[i], H[i], fk[i] * fv[i]);
                A[i] *= ga[i];
            }
            pa[r][i] = A[i];
            ph[r][i] = H[i];
        }
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) lA[p.w][p.lane * VEC + i] = A[i], lH[p.w][p.lane * VEC + i] = H[i];
    __syncthreads();
    float S[VEC], eA[VEC], eH[VEC];
    join<VEC, false>(lA, lH, p.w, p.lane, eA, eH);
#pragma unroll
    for (int i = 0; i < VEC; ++i) S[i] = fmaf(eA[i], a.marks[(p.b * a.tiles + p.tile) * a.D + p.c + i], eH[i]);
    if (!p.there) return;
    char* yp = a.y + ((p.b * a.L + p.row0) * a.D + p.c) * T::kBytes;
#pragma unroll
    for (int r = 0; r < kRowsPerWave; ++r) {
        float fq[VEC];
        P::unpack(q[r], fq);
#pragma unroll
        for (int i = 0; i < VEC; ++i) fq[i] *= fmaf(pa[r][i], S[i], ph[r][i]);
        if (r < p.rows) P::store_nt(yp + (int64_t)r * a.D * T::kBytes, P::pack(fq));
    }
}

// dq, dk, dv, dg of every tile from the state before it and the gradient behind it.
template <typename T, int VEC, bool SHARED>
__global__ __launch_bounds__(kWaves * kWave) void glr_bwd_kernel(GlrArgs a) {
    using P = Pack<T, VEC>;
    using IO = Io<T, VEC, SHARED>;
    __shared__ float lA[kWaves][kWave * VEC], lH[kWaves][kWave * VEC], lC[kWaves][kWave * VEC];
    const Place p = place<VEC>(a);
    const int64_t at = p.c * T::kBytes, gat = p.c / a.group * T::kBytes;
    typename P::Raw q[kRowsPerWave], k[kRowsPerWave], v[kRowsPerWave], dy[kRowsPerWave];
    typename IO::G::Raw g[kRowsPerWave];
    load_rows<P>(k, a.k, a, p, at);
    load_rows<P>(v, a.v, a, p, at);
    load_rows<typename IO::G>(g, a.g, a, p, gat);
    load_rows<P>(q, a.q, a, p, at);
    load_rows<P>(dy, a.dy, a, p, at);
    float A[VEC], H[VEC], C[VEC], ga[kRowsPerWave][VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) A[i] = 1.0f, H[i] = 0.0f, C[i] = 0.0f;
#pragma unroll
    for (int r = 0; r < kRowsPerWave; ++r) {
        float fk[VEC], fv[VEC];
        P::unpack(k[r], fk);
        P::unpack(v[r], fv);
        IO::gates(g[r], ga[r]);
        if (r < p.rows)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                H[i] = fmaf(ga[r][i], H[i], fk[i] * fv[i]);
                A[i] *= ga[r][i];
            }
    }
#pragma unroll
    for (int r = kRowsPerWave - 1; r >= 0; --r) {
        float fq[VEC], fy[VEC];
        P::unpack(q[r], fq);
        P::unpack(dy[r], fy);
        if (r < p.rows)
#pragma unroll
            for (int i = 0; i < VEC; ++i) C[i] = ga[r][i] * fmaf(fq[i], fy[i], C[i]);
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const int o = p.lane * VEC + i;
        lA[p.w][o] = A[i], lH[p.w][o] = H[i], lC[p.w][o] = C[i];
    }
    __syncthreads();
    float S[VEC], R[VEC], eA[VEC], eH[VEC];
    const int64_t m0 = (p.b * a.tiles + p.tile) * a.D + p.c;
    join<VEC, false>(lA, lH, p.w, p.lane, eA, eH);
#pragma unroll
    for (int i = 0; i < VEC; ++i) S[i] = fmaf(eA[i], a.marks[m0 + i], eH[i]);
    join<VEC, true>(lA, lC, p.w, p.lane, eA, eH);
#pragma unroll
    for (int i = 0; i < VEC; ++i) R[i] = fmaf(eA[i], a.rmarks[m0 + i], eH[i]);

    const int64_t row = p.b * a.L + p.row0;
    const int64_t o0 = (row * a.D + p.c) * T::kBytes;
    float kept[kRowsPerWave][VEC];  // a[t] s[t-1]
#pragma unroll
    for (int r = 0; r < kRowsPerWave; ++r) {
        float fk[VEC], fv[VEC], fy[VEC];
        P::unpack(k[r], fk);
        P::unpack(v[r], fv);
        P::unpack(dy[r], fy);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            kept[r][i] = ga[r][i] * S[i];
            S[i] = fmaf(fk[i], fv[i], kept[r][i]);
            fy[i] *= S[i];
        }
        if (r < p.rows && p.there) P::store_nt(a.dq + o0 + (int64_t)r * a.D * T::kBytes, P::pack(fy));
    }
#pragma unroll
    for (int r = kRowsPerWave - 1; r >= 0; --r) {
        if (r >= p.rows) continue;  // the same for all lanes
        float fk[VEC], fv[VEC], fq[VEC], fy[VEC], dg[VEC];
        P::unpack(k[r], fk);
        P::unpack(v[r], fv);
        P::unpack(q[r], fq);
        P::unpack(dy[r], fy);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const float m = fmaf(fq[i], fy[i], R[i]);
            R[i] = ga[r][i] * m;
            dg[i] = p.there ? m * kept[r][i] : 0.0f;
            const float dk = m * fv[i];
            fv[i] = m * fk[i];
            fk[i] = dk;
        }
        const int64_t o = o0 + (int64_t)r * a.D * T::kBytes;
        if (p.there) {
            P::store_nt(a.dk + o, P::pack(fk));
            P::store_nt(a.dv + o, P::pack(fv));
        }
        if constexpr (!SHARED) {
            if (p.there) P::store_nt(a.dg + o, P::pack(dg));
        } else {
            // the part's lanes are neighbours: halving distances, the same order in every call
            float s = dg[0];
#pragma unroll
            for (int i = 1; i < VEC; ++i) s += dg[i];
            const int lanes = a.part / VEC;
            for (int d = lanes / 2; d > 0; d /= 2) s += __shfl_xor(s, d, kWave);
            if (p.there && p.lane % lanes == 0) {
                const float one[1] = {s};
                const int64_t n = (row + r) * (a.D / a.part) + p.c / a.part;
                if (a.part == a.group) Pack<T, 1>::store_nt(a.dg + n * T::kBytes, Pack<T, 1>::pack(one));
                else a.dg_parts[n] = s;
            }
        }
    }
}

// dg[row][n] = sum over the group's parts, in their order.
template <typename T>
__global__ __launch_bounds__(256) void glr_dg_kernel(const float* parts, char* dg, int64_t n, int32_t per) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    float s[1] = {0.0f};
    for (int32_t j = 0; j < per; ++j) s[0] += parts[i * per + j];
    Pack<T, 1>::store(dg + i * T::kBytes, Pack<T, 1>::pack(s));
}

// One step of every sequence: the state is updated where it is.
template <typename T, int VEC, bool SHARED>
__global__ __launch_bounds__(256) void glr_step_kernel(const char* q, const char* k, const char* v, const char* g, float* state,
                                                       char* y, int64_t n, int32_t group) {
    using P = Pack<T, VEC>;
    using IO = Io<T, VEC, SHARED>;
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * VEC;
    if (i >= n) return;
    const auto rq = P::load(q + i * T::kBytes), rk = P::load(k + i * T::kBytes), rv = P::load(v + i * T::kBytes);
    const auto rg = IO::G::load(g + i / group * T::kBytes);
    const auto rs = Pack<F32, VEC>::load(state + i);
    float fq[VEC], fk[VEC], fv[VEC], ga[VEC], s[VEC];
    P::unpack(rq, fq);
    P::unpack(rk, fk);
    P::unpack(rv, fv);
    IO::gates(rg, ga);
    Pack<F32, VEC>::unpack(rs, s);
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
        s[j] = fmaf(ga[j], s[j], fk[j] * fv[j]);
        fq[j] *= s[j];
    }
    Pack<F32, VEC>::store(state + i, Pack<F32, VEC>::pack(s));
    P::store(y + i * T::kBytes, P::pack(fq));
}

template <typename T, int VEC, bool SHARED>
struct Kernels {
    static hy_status forward(GlrArgs& a, const GlrPtrs& p, uint32_t grid, float* marks, int64_t B, hipStream_t st) {
        const dim3 g(grid), b(kWaves * kWave);
        hy_status rc = launch_kernel(glr_sum_kernel<T, VEC, SHARED, false>, g, b, st, a);
        if (rc == HY_OK)
            rc = launch_kernel(glr_scan_kernel<false>, dim3((uint32_t)((B * a.D + 255) / 256)), dim3(256), st, (const float*)a.A,
                               (const float*)a.H, p.state_in, marks, p.state_out, B, (int64_t)a.tiles, a.D);
        if (rc == HY_OK && p.y) rc = launch_kernel(glr_fwd_kernel<T, VEC, SHARED>, g, b, st, a);
        return rc;
    }
    static hy_status backward(GlrArgs& a, const GlrPtrs& p, uint32_t grid, float* rmarks, int64_t B, hipStream_t st) {
        const dim3 g(grid), b(kWaves * kWave);
        hy_status rc = launch_kernel(glr_sum_kernel<T, VEC, SHARED, true>, g, b, st, a);
        if (rc == HY_OK)
            rc = launch_kernel(glr_scan_kernel<true>, dim3((uint32_t)((B * a.D + 255) / 256)), dim3(256), st, (const float*)a.A,
                               (const float*)a.H, p.dstate_out, rmarks, p.dstate_in, B, (int64_t)a.tiles, a.D);
        if (rc == HY_OK) rc = launch_kernel(glr_bwd_kernel<T, VEC, SHARED>, g, b, st, a);
        return rc;
    }
    static hy_status step(const GlrPtrs& p, int64_t n, int32_t group, hipStream_t st) {
        const int64_t per = 256 * VEC;
        return launch_kernel(glr_step_kernel<T, VEC, SHARED>, dim3((uint32_t)((n + per - 1) / per)), dim3(256), st,
                             (const char*)p.q, (const char*)p.k, (const char*)p.v, (const char*)p.g, p.state_out, (char*)p.y, n,
                             group);
    }
};

template <typename F>
hy_status by_kind(hy_dtype dtype, bool pairs, bool shared, F f) {
    if (dtype == HY_F32) {
        if (pairs) return shared ? f(Kernels<F32, 2, true>{}) : f(Kernels<F32, 2, false>{});
        return shared ? f(Kernels<F32, 1, true>{}) : f(Kernels<F32, 1, false>{});
    }
    if (pairs) return shared ? f(Kernels<BF16, 2, true>{}) : f(Kernels<BF16, 2, false>{});
    return shared ? f(Kernels<BF16, 1, true>{}) : f(Kernels<BF16, 1, false>{});
}

int64_t tiles_of(const GlrShape& s) { return (s.L + kGlrRows - 1) / kGlrRows; }

// Two channels per lane need rows that begin where two elements do, and both channels in one group.
bool in_pairs(const GlrShape& s) {
    if (s.D % 2 != 0 || (s.group > 1 && s.group % 2 != 0) || s.odd_start) return false;
    for (int i = 0; i < 5; ++i)
        if (s.rstride[i] % 2 != 0 || s.bstride[i] % 2 != 0) {
            if (i == kGlrG && s.group > 1) continue;  // one gate at a time
            return false;
        }
    return true;
}

// The largest power of two that divides `group`, up to the `width` channels of a wave.
int32_t part_of(int32_t group, int32_t width) {
    int32_t part = 1;
    while (part < width && group % (2 * part) == 0) part *= 2;
    return part;
}

int64_t round16(int64_t n) { return (n + 15) / 16 * 16; }

GlrArgs args_of(const GlrPtrs& p, const GlrShape& s, int64_t* grid) {
    const int64_t e = s.dtype == HY_F32 ? 4 : 2;
    auto src = [&](const void* x, int i) { return Src{(const char*)x, s.bstride[i] * e, s.rstride[i] * e}; };
    GlrArgs a{};
    a.q = src(p.q, kGlrQ), a.k = src(p.k, kGlrK), a.v = src(p.v, kGlrV), a.g = src(p.g, kGlrG), a.dy = src(p.dy, kGlrDy);
    a.y = (char*)p.y, a.dq = (char*)p.dq, a.dk = (char*)p.dk, a.dv = (char*)p.dv, a.dg = (char*)p.dg;
    a.L = s.L, a.D = s.D, a.group = s.group;
    const int64_t width = in_pairs(s) ? 2 * kWave : kWave, tiles = tiles_of(s), ncb = (s.D + width - 1) / width;
    *grid = tiles <= INT32_MAX && ncb <= INT32_MAX && s.B <= INT32_MAX / tiles / ncb ? s.B * tiles * ncb : -1;
    a.tiles = (int32_t)tiles, a.ncb = (int32_t)ncb;
    a.part = part_of(s.group, (int32_t)width);
    return a;
}

// No steps: the state goes on as it is.
hy_status hand_on(const float* in, float* out, const GlrShape& s, hipStream_t st) {
    return launch_kernel(glr_scan_kernel<false>, dim3((uint32_t)((s.B * s.D + 255) / 256)), dim3(256), st, (const float*)nullptr,
                         (const float*)nullptr, in, (float*)nullptr, out, s.B, (int64_t)0, s.D);
}

}  // namespace

// A, H and the marks (where the caller does not take them).
int64_t glr_fwd_workspace_bytes(const GlrShape& s) { return 3 * round16(s.B * tiles_of(s) * s.D * 4); }

// The same (a fourth array for the states where no marks come in), and the parts of dg, as many as lanes of one channel have.
int64_t glr_bwd_workspace_bytes(const GlrShape& s, bool marks) {
    const int64_t n = round16(s.B * tiles_of(s) * s.D * 4);
    const int32_t part = part_of(s.group, kWave);
    return (marks ? 3 : 4) * n + (part == s.group ? 0 : s.B * s.L * (s.D / part) * 4);
}

hy_status launch_glr_fwd(const GlrPtrs& p, const GlrShape& s, void* ws, hipStream_t st) {
    if (s.L == 0) return hand_on(p.state_in, p.state_out, s, st);
    int64_t grid;
    GlrArgs a = args_of(p, s, &grid);
    if (grid < 0) return HY_ERR_UNSUPPORTED;
    const int64_t n = round16(s.B * tiles_of(s) * s.D * 4);
    char* w = static_cast<char*>(ws);
    a.A = (float*)w, a.H = (float*)(w + n);
    float* marks = p.marks_out ? p.marks_out : (float*)(w + 2 * n);
    a.marks = marks;
    return by_kind(s.dtype, in_pairs(s), s.group > 1,
                   [&](auto kernels) { return kernels.forward(a, p, (uint32_t)grid, marks, s.B, st); });
}

hy_status launch_glr_bwd(const GlrPtrs& p, const GlrShape& s, void* ws, hipStream_t st) {
    if (s.L == 0) return hand_on(p.dstate_out, p.dstate_in, s, st);
    int64_t grid;
    GlrArgs a = args_of(p, s, &grid);
    if (grid < 0) return HY_ERR_UNSUPPORTED;
    const int64_t n = round16(s.B * tiles_of(s) * s.D * 4);
    char* w = static_cast<char*>(ws);
    a.A = (float*)w, a.H = (float*)(w + n);
    float* rmarks = (float*)(w + 2 * n);
    a.rmarks = rmarks;
    w += 3 * n;
    hy_status rc = HY_OK;
    if (p.marks) {
        a.marks = p.marks;
    } else {
        float* marks = (float*)w;
        w += n;
        a.marks = marks;
        GlrPtrs f = p;  // the states alone
        f.y = nullptr, f.state_out = nullptr;
        rc = by_kind(s.dtype, in_pairs(s), s.group > 1,
                     [&](auto kernels) { return kernels.forward(a, f, (uint32_t)grid, marks, s.B, st); });
    }
    a.dg_parts = (float*)w;
    if (rc == HY_OK)
        rc = by_kind(s.dtype, in_pairs(s), s.group > 1,
                     [&](auto kernels) { return kernels.backward(a, p, (uint32_t)grid, rmarks, s.B, st); });
    if (rc == HY_OK && a.part != s.group) {
        const int64_t out = s.B * s.L * (s.D / s.group);
        if ((out + 255) / 256 > INT32_MAX) return HY_ERR_UNSUPPORTED;
        const dim3 g((uint32_t)((out + 255) / 256)), b(256);
        const float* parts = a.dg_parts;
        const int32_t per = s.group / a.part;
        rc = s.dtype == HY_F32 ? launch_kernel(glr_dg_kernel<F32>, g, b, st, parts, (char*)p.dg, out, per)
                               : launch_kernel(glr_dg_kernel<BF16>, g, b, st, parts, (char*)p.dg, out, per);
    }
    return rc;
}

hy_status launch_glr_step(const GlrPtrs& p, const GlrShape& s, hipStream_t st) {
    const int64_t n = s.B * s.D;
    if ((n + 255) / 256 > INT32_MAX) return HY_ERR_UNSUPPORTED;
    return by_kind(s.dtype, in_pairs(s), s.group > 1, [&](auto kernels) { return kernels.step(p, n, s.group, st); });
}

}  // namespace hy
