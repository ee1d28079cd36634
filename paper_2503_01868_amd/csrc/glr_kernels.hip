// Gated linear recurrence: s[t] = a[t] s[t-1] + u[t], y[t] = q[t] s[t], a = exp(g), u = k v, and its gradients.
//
// The recurrence is linear, so a stretch of steps acts on the state before it as s -> A s + H with two numbers per channel,
// A the product of its a and H its result from zero.  The gradient runs the other way with the same A: with m[t] = dLoss/ds[t]
// and c[t] = a[t] m[t] (what a step hands to the one before it), m[t] = q[t] dy[t] + c[t+1], so a stretch takes c -> A c + C.
//
// One pass: a workgroup loads a tile of kGlrRows steps by 64 or 128 channels into registers, each wave kRowsPerWave rows, sums
// it up, publishes (A, H), takes the state at its edge from the tiles before it (behind it, backward), publishes its own and
// writes the tile's results from the registers.  Every tensor is read and written once: that traffic is what bounds it.
//
// The edge: tile i needs s = A[i-1] (A[i-2] (...) + H[i-2]) + H[i-1].  A workgroup looks at kWindow tiles before it until one of
// them has published its state and all tiles between have published their sums, and applies those one by one.  That is the
// order a walk from the first tile has, wherever the look finds a state: results do not depend on timing.  A state travels up to
// kWindow tiles per exchange between compute units, so the exchanges are few against the tiles that are in flight.
// Without flags or fences: glr_unset_kernel fills the records with kUnset, a NaN that no value ever is (a producer that holds
// it stores the plain NaN); words are stored and loaded as atomics at device scope, and a record is there when none of its words
// is kUnset.  Tiles wait for tiles of lower launch index only, and for a bounded time: after kPolls looks the workgroup walks
// the sequence itself, by the same sums.
#include "hy_common.hpp"
#include "hy_launch.hpp"

namespace hy {

namespace {

constexpr int kWaves = 8;                      // waves of a workgroup, one after the other in time
constexpr int kRowsPerWave = kGlrRows / kWaves;
constexpr int kWindow = 2 * kWaves;
constexpr uint32_t kUnset = 0xffffdeadu;
constexpr int kPolls = 4096;

struct Src {
    const char* p;
    int64_t bstride, rstride;  // bytes between batch items and between rows
};

struct GlrArgs {
    Src q, k, v, g, dy;
    char *y, *dq, *dk, *dv, *dg;
    float* dg_parts;           // [B, L, D / part] fp32, where a group is summed up in parts
    const float* edge_in;      // [B, D]: the state before the first tile (the gradient behind the last), or null: zero
    float* edge_out;           // [B, D]: what comes out at the other end, or null
    const float* marks;        // [B, tiles, D] states before the tiles (backward)
    float* marks_out;          // forward, or null
    uint64_t* sums;            // [tiles, B, D]: (A, H) or (A, C) of the tiles, in the order of the walk
    uint32_t* states;          // [tiles, B, D]: the state behind (the c before) them
    int64_t B, L, D;
    int32_t tiles, ncb, group, part;  // part: channels of a group that a wave sums up (a power of two)
    int32_t polls;
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
    int w, lane;
    int order, tile;      // the tile's place in the walk and in the sequence
    int64_t b, c;
    bool there;           // its channels exist
};

// Launch order: tile by tile of the walk, in it all sequences and channels.
template <int VEC, bool REV>
__device__ __forceinline__ Place place(const GlrArgs& a) {
    Place p;
    p.w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    p.lane = threadIdx.x % kWave;
    uint32_t i = blockIdx.x;
    const uint32_t cb = i % (uint32_t)a.ncb;
    i /= (uint32_t)a.ncb;
    p.b = i % (uint32_t)a.B;
    p.order = i / (uint32_t)a.B;
    p.tile = REV ? a.tiles - 1 - p.order : p.order;
    p.c = (int64_t)cb * (kWave * VEC) + p.lane * VEC;
    p.there = p.c < a.D;
    if (!p.there) p.c = 0;
    return p;
}

struct Rows {
    int64_t first;
    int n;  // steps of the sequence that the wave has
};
__device__ __forceinline__ Rows rows_of(const GlrArgs& a, int tile, int w) {
    Rows r;
    r.first = (int64_t)tile * kGlrRows + w * kRowsPerWave;
    const int64_t left = a.L - r.first;
    r.n = left < 0 ? 0 : left < kRowsPerWave ? (int)left : kRowsPerWave;
    return r;
}

// The wave's rows of a tensor; steps behind the last are the last one again (their values are not used).
template <typename PK>
__device__ __forceinline__ void load_rows(typename PK::Raw (&r)[kRowsPerWave], const Src& s, const GlrArgs& a, const Place& p,
                                          const Rows& at, int64_t lane_bytes) {
    const char* base = s.p + p.b * s.bstride + lane_bytes;
#pragma unroll
    for (int i = 0; i < kRowsPerWave; ++i) {
        const int64_t t = at.first + i < a.L ? at.first + i : a.L - 1;
        r[i] = PK::load_nt(base + t * s.rstride);
    }
}

template <int VEC>
struct Shared {
    float A[kWaves][kWave * VEC], H[kWaves][kWave * VEC];            // of the waves
    float wA[kWindow][kWave * VEC], wH[kWindow][kWave * VEC];        // of the tiles in the window, nearest first; or, in wH,
    int32_t found[2][kWindow];                                       // their state.  0: nothing yet, 1: sums, 2: state
};

// What waves [0, w) (REV: (w, last]) of the workgroup make of the state at its edge; all of them with w = kWaves (REV: -1).
template <int VEC, bool REV>
__device__ __forceinline__ void join(const Shared<VEC>& s, int w, int lane, float (&A)[VEC], float (&H)[VEC]) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) A[i] = 1.0f, H[i] = 0.0f;
    for (int x = REV ? kWaves - 1 : 0; REV ? x > w : x < w; x += REV ? -1 : 1)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const float xa = s.A[x][lane * VEC + i];
            H[i] = fmaf(xa, H[i], s.H[x][lane * VEC + i]);
            A[i] *= xa;
        }
}

__device__ __forceinline__ uint32_t word_of(float x) {
    const uint32_t b = __float_as_uint(x);
    return b == kUnset ? 0x7fc00000u : b;
}

// x and y of the steps (k and v forward, q and dy backward) -> A and H (C) of the wave's rows, into LDS.
template <typename T, int VEC, bool SHARED, bool REV>
__device__ __forceinline__ void sum_rows(Shared<VEC>& s, const typename Pack<T, VEC>::Raw (&x)[kRowsPerWave],
                                         const typename Pack<T, VEC>::Raw (&y)[kRowsPerWave], const float (&ga)[kRowsPerWave][VEC],
                                         const Place& p, int n) {
    using P = Pack<T, VEC>;
    float A[VEC], H[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) A[i] = 1.0f, H[i] = 0.0f;
#pragma unroll
    for (int j = 0; j < kRowsPerWave; ++j) {
        const int r = REV ? kRowsPerWave - 1 - j : j;
        float fx[VEC], fy[VEC];
        P::unpack(x[r], fx);
        P::unpack(y[r], fy);
        if (r < n)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                H[i] = REV ? ga[r][i] * fmaf(fx[i], fy[i], H[i]) : fmaf(ga[r][i], H[i], fx[i] * fy[i]);
                A[i] *= ga[r][i];
            }
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) s.A[p.w][p.lane * VEC + i] = A[i], s.H[p.w][p.lane * VEC + i] = H[i];
}

// The wave's sums of any tile, row by row from memory: sum_rows' operations in few registers.
template <typename T, int VEC, bool SHARED, bool REV>
__device__ __forceinline__ void sum_tile(Shared<VEC>& s, const GlrArgs& a, const Place& p, int tile) {
    using P = Pack<T, VEC>;
    using IO = Io<T, VEC, SHARED>;
    const Rows at = rows_of(a, tile, p.w);
    const Src &sx = REV ? a.q : a.k, &sy = REV ? a.dy : a.v;
    float A[VEC], H[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) A[i] = 1.0f, H[i] = 0.0f;
#pragma unroll 1
    for (int j = 0; j < at.n; ++j) {
        const int64_t t = at.first + (REV ? at.n - 1 - j : j);
        float fx[VEC], fy[VEC], ga[VEC];
        P::unpack(P::load(sx.p + p.b * sx.bstride + t * sx.rstride + p.c * T::kBytes), fx);
        P::unpack(P::load(sy.p + p.b * sy.bstride + t * sy.rstride + p.c * T::kBytes), fy);
        IO::gates(IO::G::load(a.g.p + p.b * a.g.bstride + t * a.g.rstride + p.c / a.group * T::kBytes), ga);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            H[i] = REV ? ga[i] * fmaf(fx[i], fy[i], H[i]) : fmaf(ga[i], H[i], fx[i] * fy[i]);
            A[i] *= ga[i];
        }
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) s.A[p.w][p.lane * VEC + i] = A[i], s.H[p.w][p.lane * VEC + i] = H[i];
}

// The state at the tile's edge, with the waves' sums of the tile in LDS (and a barrier behind them); publishes the tile's own.
template <typename T, int VEC, bool SHARED, bool REV>
__device__ __forceinline__ void edge_of(Shared<VEC>& s, const GlrArgs& a, const Place& p, float (&S)[VEC]) {
    const int64_t per = a.B * a.D, here = p.b * a.D + p.c;
    float tA[VEC], tH[VEC];
    const bool last = p.order == a.tiles - 1;
    if (p.w == 0) {
        join<VEC, REV>(s, REV ? -1 : kWaves, p.lane, tA, tH);
        if (p.order > 0 && !last && p.there)
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                __hip_atomic_store(a.sums + p.order * per + here + i, word_of(tA[i]) | (uint64_t)word_of(tH[i]) << 32,
                                   __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) S[i] = a.edge_in ? a.edge_in[here + i] : 0.0f;
    if (p.order > 0) {
        int have[2] = {0, 0};
        int base = -1;  // the nearest tile whose state is there
        for (int look = 0; look < a.polls; ++look) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int slot = p.w + x * kWaves, of = p.order - 1 - slot;
                if (of >= 0 && have[x] < 2) {
                    uint32_t st[VEC];
                    uint64_t su[VEC];
                    bool state = true, sums = true;
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        st[i] = __hip_atomic_load(a.states + of * per + here + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                        su[i] = have[x] || of == 0 ? 0 : __hip_atomic_load(a.sums + of * per + here + i, __ATOMIC_RELAXED,
                                                                           __HIP_MEMORY_SCOPE_AGENT);
                        state = state && st[i] != kUnset;
                        sums = sums && (uint32_t)su[i] != kUnset && (uint32_t)(su[i] >> 32) != kUnset;
                    }
                    if (__all(state || !p.there)) {
                        have[x] = 2;
#pragma unroll
                        for (int i = 0; i < VEC; ++i) s.wH[slot][p.lane * VEC + i] = __uint_as_float(st[i]);
                    } else if (have[x] == 0 && of > 0 && __all(sums || !p.there)) {
                        have[x] = 1;
#pragma unroll
                        for (int i = 0; i < VEC; ++i) {
                            s.wA[slot][p.lane * VEC + i] = __uint_as_float((uint32_t)su[i]);
                            s.wH[slot][p.lane * VEC + i] = __uint_as_float((uint32_t)(su[i] >> 32));
                        }
                    }
                }
                if (p.lane == 0) s.found[look & 1][slot] = have[x];
            }
            __syncthreads();
            // every wave sees the same and decides the same
            base = -1;
            for (int x = 0; x < kWindow; ++x) {
                const int f = s.found[look & 1][x];
                if (f != 1) {
                    base = f == 2 ? x : -1;
                    break;
                }
            }
            if (base >= 0) break;
            __builtin_amdgcn_s_sleep(2);
        }
        if (base >= 0) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) S[i] = s.wH[base][p.lane * VEC + i];
            for (int x = base - 1; x >= 0; --x)
#pragma unroll
                for (int i = 0; i < VEC; ++i) S[i] = fmaf(s.wA[x][p.lane * VEC + i], S[i], s.wH[x][p.lane * VEC + i]);
        } else {
            float wA[VEC], wH[VEC];
            for (int x = 0; x < p.order; ++x) {
                __syncthreads();
                sum_tile<T, VEC, SHARED, REV>(s, a, p, REV ? a.tiles - 1 - x : x);
                __syncthreads();
                join<VEC, REV>(s, REV ? -1 : kWaves, p.lane, wA, wH);
#pragma unroll
                for (int i = 0; i < VEC; ++i) S[i] = fmaf(wA[i], S[i], wH[i]);
            }
            __syncthreads();
            sum_tile<T, VEC, SHARED, REV>(s, a, p, p.tile);  // the waves' sums again
            __syncthreads();
        }
    }
    if (p.w == 0 && p.there) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const float e = fmaf(tA[i], S[i], tH[i]);
            if (!last) __hip_atomic_store(a.states + p.order * per + here + i, word_of(e), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            else if (a.edge_out) a.edge_out[here + i] = e;
        }
    }
}

constexpr int kMarks = 4;  // 16-byte pieces per lane
__global__ __launch_bounds__(256) void glr_unset_kernel(uint4* rec, int64_t n) {
    const int64_t i0 = (int64_t)blockIdx.x * 256 * kMarks + threadIdx.x;
#pragma unroll
    for (int x = 0; x < kMarks; ++x)
        if (i0 + 256 * x < n) store_words<4>(rec + i0 + 256 * x, Words<4>{{kUnset, kUnset, kUnset, kUnset}});
}

// The state of sequences without steps goes on as it is.
__global__ __launch_bounds__(256) void glr_hand_on_kernel(const float* in, float* out, int64_t n) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < n) out[i] = in ? in[i] : 0.0f;
}

// Y: q comes in and y goes out; else the states alone.
template <typename T, int VEC, bool SHARED, bool Y>
__global__ __launch_bounds__(kWaves * kWave) void glr_fwd_kernel(GlrArgs a) {
    using P = Pack<T, VEC>;
    using IO = Io<T, VEC, SHARED>;
    __shared__ Shared<VEC> s;
    const Place p = place<VEC, false>(a);
    const Rows at = rows_of(a, p.tile, p.w);
    const int64_t lane_bytes = p.c * T::kBytes;
    typename P::Raw q[kRowsPerWave], k[kRowsPerWave], v[kRowsPerWave];
    typename IO::G::Raw g[kRowsPerWave];
    load_rows<P>(k, a.k, a, p, at, lane_bytes);
    load_rows<P>(v, a.v, a, p, at, lane_bytes);
    load_rows<typename IO::G>(g, a.g, a, p, at, p.c / a.group * T::kBytes);
    if constexpr (Y) load_rows<P>(q, a.q, a, p, at, lane_bytes);
    float ga[kRowsPerWave][VEC];
#pragma unroll
    for (int r = 0; r < kRowsPerWave; ++r) IO::gates(g[r], ga[r]);
    sum_rows<T, VEC, SHARED, false>(s, k, v, ga, p, at.n);
    __syncthreads();
    float S[VEC], eA[VEC], eH[VEC];
    edge_of<T, VEC, SHARED, false>(s, a, p, S);
    if (a.marks_out && p.w == 0 && p.there)
#pragma unroll
        for (int i = 0; i < VEC; ++i) a.marks_out[(p.b * a.tiles + p.tile) * a.D + p.c + i] = S[i];
    if (!Y || !p.there) return;
    join<VEC, false>(s, p.w, p.lane, eA, eH);
#pragma unroll
    for (int i = 0; i < VEC; ++i) S[i] = fmaf(eA[i], S[i], eH[i]);
    char* yp = a.y + ((p.b * a.L + at.first) * a.D + p.c) * T::kBytes;
#pragma unroll
    for (int r = 0; r < kRowsPerWave; ++r) {
        float fq[VEC], fk[VEC], fv[VEC];
        P::unpack(q[r], fq);
        P::unpack(k[r], fk);
        P::unpack(v[r], fv);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            S[i] = fmaf(ga[r][i], S[i], fk[i] * fv[i]);
            fq[i] *= S[i];
        }
        if (r < at.n) P::store_nt(yp + (int64_t)r * a.D * T::kBytes, P::pack(fq));
    }
}

// dq, dk, dv, dg of every tile from the state before it and the gradient behind it.
template <typename T, int VEC, bool SHARED>
__global__ __launch_bounds__(kWaves * kWave) void glr_bwd_kernel(GlrArgs a) {
    using P = Pack<T, VEC>;
    using IO = Io<T, VEC, SHARED>;
    __shared__ Shared<VEC> s;
    const Place p = place<VEC, true>(a);
    const Rows at = rows_of(a, p.tile, p.w);
    const int64_t lane_bytes = p.c * T::kBytes;
    typename P::Raw q[kRowsPerWave], k[kRowsPerWave], v[kRowsPerWave], dy[kRowsPerWave];
    typename IO::G::Raw g[kRowsPerWave];
    load_rows<P>(q, a.q, a, p, at, lane_bytes);
    load_rows<P>(dy, a.dy, a, p, at, lane_bytes);
    load_rows<typename IO::G>(g, a.g, a, p, at, p.c / a.group * T::kBytes);
    load_rows<P>(k, a.k, a, p, at, lane_bytes);
    load_rows<P>(v, a.v, a, p, at, lane_bytes);
    float ga[kRowsPerWave][VEC];
#pragma unroll
    for (int r = 0; r < kRowsPerWave; ++r) IO::gates(g[r], ga[r]);
    float S[VEC], R[VEC], eA[VEC], eH[VEC];
    sum_rows<T, VEC, SHARED, true>(s, q, dy, ga, p, at.n);
    __syncthreads();
    edge_of<T, VEC, SHARED, true>(s, a, p, R);
    join<VEC, true>(s, p.w, p.lane, eA, eH);
#pragma unroll
    for (int i = 0; i < VEC; ++i) R[i] = fmaf(eA[i], R[i], eH[i]);
    __syncthreads();
    sum_rows<T, VEC, SHARED, false>(s, k, v, ga, p, at.n);
    __syncthreads();
    join<VEC, false>(s, p.w, p.lane, eA, eH);
#pragma unroll
    for (int i = 0; i < VEC; ++i) S[i] = fmaf(eA[i], a.marks[(p.b * a.tiles + p.tile) * a.D + p.c + i], eH[i]);

    const int64_t row = p.b * a.L + at.first;
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
        if (r < at.n && p.there) P::store_nt(a.dq + o0 + (int64_t)r * a.D * T::kBytes, P::pack(fy));
    }
#pragma unroll
    for (int r = kRowsPerWave - 1; r >= 0; --r) {
        if (r >= at.n) continue;  // the same for all lanes
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
            float sum = dg[0];
#pragma unroll
            for (int i = 1; i < VEC; ++i) sum += dg[i];
            const int lanes = a.part / VEC;
            for (int d = lanes / 2; d > 0; d /= 2) sum += __shfl_xor(sum, d, kWave);
            if (p.there && p.lane % lanes == 0) {
                const float one[1] = {sum};
                const int64_t n = (row + r) * (a.D / a.part) + p.c / a.part;
                if (a.part == a.group) Pack<T, 1>::store_nt(a.dg + n * T::kBytes, Pack<T, 1>::pack(one));
                else a.dg_parts[n] = sum;
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
    static hy_status forward(const GlrArgs& a, uint32_t grid, hipStream_t st) {
        return a.y ? launch_kernel(glr_fwd_kernel<T, VEC, SHARED, true>, dim3(grid), dim3(kWaves * kWave), st, a)
                   : launch_kernel(glr_fwd_kernel<T, VEC, SHARED, false>, dim3(grid), dim3(kWaves * kWave), st, a);
    }
    static hy_status backward(const GlrArgs& a, uint32_t grid, hipStream_t st) {
        return launch_kernel(glr_bwd_kernel<T, VEC, SHARED>, dim3(grid), dim3(kWaves * kWave), st, a);
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
    a.B = s.B, a.L = s.L, a.D = s.D, a.group = s.group;
    const int64_t width = in_pairs(s) ? 2 * kWave : kWave, tiles = tiles_of(s), ncb = (s.D + width - 1) / width;
    *grid = tiles <= INT32_MAX && ncb <= INT32_MAX && s.B <= INT32_MAX / tiles / ncb ? s.B * tiles * ncb : -1;
    a.tiles = (int32_t)tiles, a.ncb = (int32_t)ncb;
    a.part = part_of(s.group, (int32_t)width);
    return a;
}

hy_status hand_on(const float* in, float* out, const GlrShape& s, hipStream_t st) {
    return launch_kernel(glr_hand_on_kernel, dim3((uint32_t)((s.B * s.D + 255) / 256)), dim3(256), st, in, out, s.B * s.D);
}

// Records of the tiles: none where a sequence is one tile.
int64_t record_bytes(const GlrShape& s) { return tiles_of(s) > 1 ? round16(s.B * tiles_of(s) * s.D * 12) : 0; }

hy_status take_records(GlrArgs& a, const GlrShape& s, void* ws, hipStream_t st) {
    const int64_t bytes = record_bytes(s), n = s.B * tiles_of(s) * s.D;
    a.sums = static_cast<uint64_t*>(ws);
    a.states = reinterpret_cast<uint32_t*>(a.sums + n);
    a.polls = tuning().glr_wait == 1 ? 0 : kPolls;
    if (bytes == 0) return HY_OK;
    const int64_t per = 256 * kMarks * 16;
    if ((bytes + per - 1) / per > INT32_MAX) return HY_ERR_UNSUPPORTED;
    return launch_kernel(glr_unset_kernel, dim3((uint32_t)((bytes + per - 1) / per)), dim3(256), st, static_cast<uint4*>(ws), bytes / 16);
}

}  // namespace

int64_t glr_fwd_workspace_bytes(const GlrShape& s) { return record_bytes(s); }

// Records, the states where no marks come in, and the parts of dg, as many as lanes of one channel have.
int64_t glr_bwd_workspace_bytes(const GlrShape& s, bool marks) {
    const int32_t part = part_of(s.group, kWave);
    return record_bytes(s) + (marks ? 0 : round16(s.B * tiles_of(s) * s.D * 4)) +
           (part == s.group ? 0 : s.B * s.L * (s.D / part) * 4);
}

hy_status launch_glr_fwd(const GlrPtrs& p, const GlrShape& s, void* ws, hipStream_t st) {
    if (s.L == 0) return hand_on(p.state_in, p.state_out, s, st);
    int64_t grid;
    GlrArgs a = args_of(p, s, &grid);
    if (grid < 0) return HY_ERR_UNSUPPORTED;
    a.edge_in = p.state_in, a.edge_out = p.state_out, a.marks_out = p.marks_out;
    hy_status rc = take_records(a, s, ws, st);
    if (rc != HY_OK) return rc;
    return by_kind(s.dtype, in_pairs(s), s.group > 1, [&](auto kernels) { return kernels.forward(a, (uint32_t)grid, st); });
}

hy_status launch_glr_bwd(const GlrPtrs& p, const GlrShape& s, void* ws, hipStream_t st) {
    if (s.L == 0) return hand_on(p.dstate_out, p.dstate_in, s, st);
    int64_t grid;
    GlrArgs a = args_of(p, s, &grid);
    if (grid < 0) return HY_ERR_UNSUPPORTED;
    char* rest = static_cast<char*>(ws) + record_bytes(s);
    a.marks = p.marks;
    if (!p.marks) {
        float* marks = reinterpret_cast<float*>(rest);
        rest += round16(s.B * tiles_of(s) * s.D * 4);
        GlrPtrs f = p;  // the states alone
        f.y = nullptr, f.state_out = nullptr, f.marks_out = marks;
        hy_status rc = launch_glr_fwd(f, s, ws, st);
        if (rc != HY_OK) return rc;
        a.marks = marks;
    }
    a.dg_parts = reinterpret_cast<float*>(rest);
    a.edge_in = p.dstate_out, a.edge_out = p.dstate_in;
    hy_status rc = take_records(a, s, ws, st);
    if (rc == HY_OK)
        rc = by_kind(s.dtype, in_pairs(s), s.group > 1, [&](auto kernels) { return kernels.backward(a, (uint32_t)grid, st); });
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
