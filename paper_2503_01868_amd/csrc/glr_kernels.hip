// Gated linear recurrence: s[t] = a[t] s[t-1] + u[t], y[t] = q[t] s[t], a = exp(g), u = k v, and its gradients.
//
// The recurrence is linear, so a stretch of steps acts on the state before it as s -> A s + H with two numbers per channel,
// A the product of its a and H its result from zero.  The gradient runs the other way with the same A: with m[t] = dLoss/ds[t]
// and c[t] = a[t] m[t] (what a step hands to the one before it), m[t] = q[t] dy[t] + c[t+1], so a stretch takes c -> A c + C.
//
// A is held as G = log A, the sum of the stretch's g: where g > 0, A may pass fp32's range over a stretch while the states stay
// within it, because they are small or zero.  A s is taken as R (R s), R = exp(G / 2): what it gives is in range whenever the
// product is.  A product with a decay or a state of zero is zero, whatever the other factor is (times0): a decay of zero forgets
// infinities and NaN too, and an infinite decay makes nothing of nothing.  G is -infinity exactly if a stretch has a decay of
// zero; other decays, however small their product, hand on what is not finite.
//
// One pass: a workgroup loads a tile of kGlrRows steps by 64 to 256 channels into registers, each of kWaves waves kRowsPerWave
// rows, sums it up, publishes (G, H), takes the state at its edge from the tiles before it (behind it, backward) and writes the
// tile's results from the registers.  Every tensor is read and written once: that traffic is what bounds it.
//
// The edge.  Tiles are grouped in blocks of kBlockTiles.  The state at the first tile of a block is that of the block before,
// taken through that block's joint (G, H); the state at a tile is its block's, taken through the joint sums of the tiles between.
// The last tile of a block publishes its joint sums and, once it has its own state, the next block's.  So a state is always the
// result of the same operations, wherever they are done: results do not depend on timing.  A tile reads the sums before it in
// its block, and the states and joint sums of the kBlocksBack blocks before, nearest first: a state travels 32 tiles per exchange
// between compute units (about 3 us).
// Without flags or fences: glr_unset_kernel fills the records with kUnset, a NaN that no value ever is (a producer that holds
// it stores the plain NaN); words are stored and loaded as atomics at device scope, and a record is there when none of its words
// is kUnset.  Tiles wait for tiles of lower launch index only, and for a bounded time: after kPolls looks the workgroup walks
// the sequence itself, by the same sums.
#include <algorithm>

#include "hy_common.hpp"
#include "hy_launch.hpp"

namespace hy {

namespace {

constexpr int kWaves = 8;                      // waves of a workgroup, one after the other in time
constexpr int kRowsPerWave = kGlrRows / kWaves;
constexpr int kBlockTiles = 8;
constexpr int kBlocksBack = 4;
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
    // records, in the order of the walk: (G, H) (backward: (G, C)) of the tiles [tiles, B, D] and of the blocks [blocks, B, D],
    // and the states at the blocks' first tiles [blocks, B, D]
    uint64_t *sums, *joint;
    uint32_t* states;
    int64_t B, L, D;
    int32_t tiles, ncb, group, part;  // part: channels of a group that a wave sums up (a power of two)
    int32_t polls;
};

// x * y, and 0 where either of them is 0.
extern "C" __device__ float glr_fmul_legacy(float, float) __asm("llvm.amdgcn.fmul.legacy");
__device__ __forceinline__ float times0(float x, float y) { return glr_fmul_legacy(x, y); }

// The decay of two stretches, as logarithms.
__device__ __forceinline__ float both(float G, float H) { return G == -INFINITY || H == -INFINITY ? -INFINITY : G + H; }

// R of a stretch: the power of two of a rounded product, in fp32 calls too (off by 6e-8 (2 + |G|) of itself; where G is far below zero,
// that is little of a state).  No product of decays that is not zero becomes zero (or forgets NaN): below 2^-245 it may as well be 2^-245.
__device__ __forceinline__ float root_of(float G) {
    const float r = __builtin_amdgcn_exp2f((G < -170.0f ? -170.0f : G) * 0.72134752f);
    return G == -INFINITY ? 0.0f : r;
}

// A s + H
__device__ __forceinline__ float through(float R, float s, float H) { return times0(R, times0(R, s)) + H; }

// The sum of the g of a lane's rows, and whether one of their decays is zero.
template <int N>
struct Logs {
    float sum[N];
    bool dead[N];
    __device__ __forceinline__ Logs() {
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i] = 0.0f, dead[i] = false;
    }
    __device__ __forceinline__ float get(int i) const { return dead[i] ? -INFINITY : sum[i]; }
};

// VEC channels per lane; SHARED: both channels of a lane (or its only one) take the gate of their group.
template <typename T, int VEC, bool SHARED>
struct Io {
    using P = Pack<T, VEC>;
    using G = Pack<T, SHARED ? 1 : VEC>;
    static constexpr int kGates = SHARED ? 1 : VEC;
    static __device__ __forceinline__ void gates(const typename G::Raw& r, float (&a)[VEC]) {
        float f[kGates];
        G::unpack(r, f);
#pragma unroll
        for (int i = 0; i < VEC; ++i) a[i] = i == 0 || !SHARED ? decay(f[SHARED ? 0 : i]) : a[0];
    }
    // there: the row exists
    static __device__ __forceinline__ void gates(const typename G::Raw& r, float (&a)[VEC], Logs<kGates>& logs, bool there = true) {
        float f[kGates];
        G::unpack(r, f);
        gates(r, a);
#pragma unroll
        for (int i = 0; i < kGates; ++i) {
            logs.sum[i] += there ? f[i] : 0.0f;
            logs.dead[i] = logs.dead[i] || (there && a[i] == 0.0f);
        }
    }
    // exp(g) of a step (stretches: root_of).  fp32 calls take the full function; for bf16 calls the power of two of the rounded
    // product is enough (6e-8 times 1 + |g| of a) and a tenth of the instructions: with the full function the vector ALUs were what
    // bounded the kernels.
    static __device__ __forceinline__ float decay(float g) {
        if constexpr (T::kBytes == 4) return expf(g);
        return __builtin_amdgcn_exp2f(g * 1.44269504f);
    }
};

struct Place {
    int w, lane;
    int order, tile;      // the tile's place in the walk and in the sequence
    int64_t b;            // (b, order, tile and w are the same in all lanes, and in scalar registers)
    uint32_t c;
    bool there;           // its channels exist
};

// Launch order: tile by tile of the walk, in it all sequences and channels.
template <int VEC, bool REV>
__device__ __forceinline__ Place place(const GlrArgs& a) {
    Place p;
    p.w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    p.lane = threadIdx.x % kWave;
    const uint32_t i = blockIdx.x / (uint32_t)a.ncb;
    const uint32_t cb = blockIdx.x - i * (uint32_t)a.ncb;
    p.order = __builtin_amdgcn_readfirstlane(i / (uint32_t)a.B);
    p.b = __builtin_amdgcn_readfirstlane(i - p.order * (uint32_t)a.B);
    p.tile = REV ? a.tiles - 1 - p.order : p.order;
    p.c = cb * (kWave * VEC) + p.lane * VEC;
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

// Buffer instructions, for their addresses: a base and a row's offset that all lanes share and 32 bits per lane, where a pointer per
// row would take two registers and two additions for every load in flight.  (Every offset is inside its tensor; the range check has nothing to do.)
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const char* base) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, -1, 0x00027000);
}
constexpr int kNt = 2;  // once-touched data, as in load_words_nt

template <typename PK>
__device__ __forceinline__ typename PK::Raw buffer_load(__amdgpu_buffer_rsrc_t b, uint32_t lane, uint32_t row) {
    typename PK::Raw r;
    if constexpr (PK::kBytes == 8) {
        const auto x = __builtin_amdgcn_raw_buffer_load_b64(b, lane, row, kNt);
        r.w[0] = x[0], r.w[1] = x[1];
    } else if constexpr (PK::kBytes == 4) {
        r.w[0] = __builtin_amdgcn_raw_buffer_load_b32(b, lane, row, kNt);
    } else {
        r.w[0] = __builtin_amdgcn_raw_buffer_load_b16(b, lane, row, kNt);
    }
    return r;
}
template <typename PK>
__device__ __forceinline__ void buffer_store(__amdgpu_buffer_rsrc_t b, uint32_t lane, uint32_t row, const typename PK::Raw& r) {
    if constexpr (PK::kBytes == 8) __builtin_amdgcn_raw_buffer_store_b64(u32x2_t{r.w[0], r.w[1]}, b, lane, row, kNt);
    else if constexpr (PK::kBytes == 4) __builtin_amdgcn_raw_buffer_store_b32(r.w[0], b, lane, row, kNt);
    else __builtin_amdgcn_raw_buffer_store_b16((uint16_t)r.w[0], b, lane, row, kNt);
}

// Rows stay as they were loaded while the workgroup waits: what has been computed from them before is computed again behind
// this point, where the compiler would keep it, in twice the registers.
template <typename R>
__device__ __forceinline__ void keep_raw(R (&r)[kRowsPerWave]) {
#pragma unroll
    for (int i = 0; i < kRowsPerWave; ++i)
#pragma unroll
        for (unsigned j = 0; j < sizeof(R) / 4; ++j) asm volatile("" : "+v"(r[i].w[j]));
}

// The wave's rows of a tensor; steps behind the last are the last one again (their values are not used).
template <typename PK>
__device__ __forceinline__ void load_rows(typename PK::Raw (&r)[kRowsPerWave], const Src& s, const GlrArgs& a, const Place& p,
                                          const Rows& at, uint32_t lane_bytes) {
    const int64_t first = at.n > 0 ? at.first : a.L - 1;
    const auto from = buffer_of(s.p + p.b * s.bstride + first * s.rstride);
    const uint32_t step = (uint32_t)s.rstride;
#pragma unroll
    for (int i = 0; i < kRowsPerWave; ++i) r[i] = buffer_load<PK>(from, lane_bytes, (i < at.n ? i : at.n > 0 ? at.n - 1 : 0) * step);
}

template <int VEC>
struct Shared {
    float G[kWaves][kWave * VEC], R[kWaves][kWave * VEC], H[kWaves][kWave * VEC];  // of the waves
    float S[kWave * VEC];                                  // the state at the tile's edge
    int32_t lost;                                          // no state came
};

// The state at its edge -> the one that wave w begins with: through waves [0, w) (REV: (w, last]) of the workgroup.
template <int VEC, bool REV>
__device__ __forceinline__ void join(const Shared<VEC>& s, int w, int lane, float (&S)[VEC]) {
#pragma unroll
    for (int y = 0; y < kWaves - 1; ++y) {
        const int x = REV ? kWaves - 1 - y : y;
        if (REV ? x <= w : x >= w) break;
#pragma unroll
        for (int i = 0; i < VEC; ++i) S[i] = through(s.R[x][lane * VEC + i], S[i], s.H[x][lane * VEC + i]);
    }
}

// G and H of the tile, for N channels from `slot` on; `together`: the waves whose sums are on their way from LDS at a time.
template <int VEC, bool REV, int together, int N>
__device__ __forceinline__ void join_all(const Shared<VEC>& s, int slot, float (&G)[N], float (&H)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) G[i] = 0.0f, H[i] = 0.0f;
#pragma unroll together
    for (int x = 0; x < kWaves; ++x) {
        const int w = REV ? kWaves - 1 - x : x;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            H[i] = through(s.R[w][slot + i], H[i], s.H[w][slot + i]);
            G[i] = both(G[i], s.G[w][slot + i]);
        }
    }
}

// f(r) for the wave's n rows, in their order or backwards; all of them without a test per row.
template <bool REV, typename F>
__device__ __forceinline__ void for_rows(int n, F f) {
    if (n == kRowsPerWave) {
#pragma unroll
        for (int j = 0; j < kRowsPerWave; ++j) f(REV ? kRowsPerWave - 1 - j : j);
    } else {
#pragma unroll
        for (int j = 0; j < kRowsPerWave; ++j) {
            const int r = REV ? kRowsPerWave - 1 - j : j;
            if (r < n) f(r);
        }
    }
}

__device__ __forceinline__ uint32_t word_of(float x) {
    const uint32_t b = __float_as_uint(x);
    return b == kUnset ? 0x7fc00000u : b;
}

// x and y of the steps (k and v forward, q and dy backward) -> H (C) of the wave's rows, into LDS.
template <typename T, int VEC, bool REV, typename Gates>
__device__ __forceinline__ void sum_rows(Shared<VEC>& s, const typename Pack<T, VEC>::Raw (&x)[kRowsPerWave],
                                         const typename Pack<T, VEC>::Raw (&y)[kRowsPerWave],
                                         const Place& p, int n, Gates gates) {
    using P = Pack<T, VEC>;
    float H[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) H[i] = 0.0f;
    for_rows<REV>(n, [&](int r) {
        float fx[VEC], fy[VEC], ga[VEC];
        P::unpack(x[r], fx);
        P::unpack(y[r], fy);
        gates(r, ga);
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            H[i] = REV ? times0(ga[i], fmaf(fx[i], fy[i], H[i])) : fmaf(fx[i], fy[i], times0(ga[i], H[i]));
    });
#pragma unroll
    for (int i = 0; i < VEC; ++i) s.H[p.w][p.lane * VEC + i] = H[i];
}
// And their G and R.
template <int VEC, int N>
__device__ __forceinline__ void put_logs(Shared<VEC>& s, const Place& p, const Logs<N>& logs) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const float G = logs.get(i % N);
        s.G[p.w][p.lane * VEC + i] = G, s.R[p.w][p.lane * VEC + i] = root_of(G);
    }
}

// The wave's sums of any tile, row by row from memory: the same operations in few registers.
template <typename T, int VEC, bool SHARED, bool REV>
__device__ __forceinline__ void sum_tile(Shared<VEC>& s, const GlrArgs& a, const Place& p, int tile) {
    using P = Pack<T, VEC>;
    using IO = Io<T, VEC, SHARED>;
    const Rows at = rows_of(a, tile, p.w);
    const Src &sx = REV ? a.q : a.k, &sy = REV ? a.dy : a.v;
    Logs<IO::kGates> logs;
    float H[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) H[i] = 0.0f;
#pragma unroll 1
    for (int j = 0; j < at.n; ++j) {
        const int64_t t = at.first + (REV ? at.n - 1 - j : j);
        float fx[VEC], fy[VEC], ga[VEC];
        P::unpack(P::load(sx.p + p.b * sx.bstride + t * sx.rstride + p.c * T::kBytes), fx);
        P::unpack(P::load(sy.p + p.b * sy.bstride + t * sy.rstride + p.c * T::kBytes), fy);
        IO::gates(IO::G::load(a.g.p + p.b * a.g.bstride + t * a.g.rstride + p.c / (uint32_t)a.group * T::kBytes), ga, logs);
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            H[i] = REV ? times0(ga[i], fmaf(fx[i], fy[i], H[i])) : fmaf(fx[i], fy[i], times0(ga[i], H[i]));
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) s.H[p.w][p.lane * VEC + i] = H[i];
    put_logs(s, p, logs);
}

// A record's words, as they are, and whether they are there.
__device__ __forceinline__ uint64_t peek(const uint64_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ uint32_t peek(const uint32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ bool is_set(uint64_t x) { return (uint32_t)x != kUnset && (uint32_t)(x >> 32) != kUnset; }
__device__ __forceinline__ bool is_set(uint32_t x) { return x != kUnset; }
__device__ __forceinline__ void publish(uint64_t* p, float G, float H) {
    __hip_atomic_store(p, word_of(G) | (uint64_t)word_of(H) << 32, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void publish(uint32_t* p, float s) {
    __hip_atomic_store(p, word_of(s), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float G_of(uint64_t x) { return __uint_as_float((uint32_t)x); }
__device__ __forceinline__ float H_of(uint64_t x) { return __uint_as_float((uint32_t)(x >> 32)); }

// Whether the tile's walk goes on behind its block.
__device__ __forceinline__ bool ends_block(const GlrArgs& a, const Place& p) {
    return p.order % kBlockTiles == kBlockTiles - 1 && p.order + 1 < a.tiles;
}

// One channel per lane, with the waves' sums in LDS: publishes the tile's sums, finds the state at its edge and leaves it in LDS;
// publishes what others need of it.  c: the channel, slot: its place in the workgroup.  Every look loads all that is missing.
template <int VEC, bool REV>
__device__ __forceinline__ void find_edge(Shared<VEC>& s, const GlrArgs& a, const Place& p, uint32_t c, bool there, int slot) {
    constexpr int BT = kBlockTiles - 1, BB = kBlocksBack;
    const int64_t per = a.B * a.D, here = p.b * a.D;  // (the same in all lanes; a lane's own part is c)
    const int block = p.order / kBlockTiles, inside = p.order % kBlockTiles;
    const bool ends = ends_block(a, p), last = p.order + 1 == a.tiles;
    float tile_G[1], tile_H[1];
    join_all<VEC, REV, 8>(s, slot, tile_G, tile_H);
    const float tG = tile_G[0], tH = tile_H[0];
    if (!last && inside < BT && there) publish(a.sums + (p.order * per + here) + c, tG, tH);
    float cG = 0.0f, cH = 0.0f, S = a.edge_in ? a.edge_in[here + c] : 0.0f;
    bool summed = inside == 0, found = block == 0;
    uint64_t jnt[BB];       // of block - i
    uint32_t have = 1;      // bits
    for (int look = 0; look < a.polls && !(summed && found); ++look) {
        // (looks take the memory's time from the tiles: without a pause 8192 x 4096 forward 82 us, backward 139; 81 and 131 with it)
        if (look > 0) __builtin_amdgcn_s_sleep(8);
        uint32_t at = c;
        asm volatile("" : "+v"(at));  // addresses are made when records are loaded, not kept over all looks
        uint64_t sum[BT];
        uint32_t st[BB];
        if (!summed)
#pragma unroll
            for (int i = 0; i < BT; ++i)
                if (i < inside) sum[i] = peek(a.sums + ((block * kBlockTiles + i) * per + here) + at);
        if (!found)
#pragma unroll
            for (int i = 0; i < BB; ++i) {
                if (i < block) st[i] = peek(a.states + ((block - i) * per + here) + at);
                if (i > 0 && i <= block && !(have >> i & 1)) jnt[i] = peek(a.joint + ((block - i) * per + here) + at);
            }
        if (!summed) {
            bool set = true;
#pragma unroll
            for (int i = 0; i < BT; ++i)
                if (i < inside) set = set && is_set(sum[i]);
            summed = __all(set || !there);
            if (summed) {
#pragma unroll
                for (int i = 0; i < BT; ++i)
                    if (i < inside) {
                        cH = through(root_of(G_of(sum[i])), cH, H_of(sum[i]));
                        cG = both(cG, G_of(sum[i]));
                    }
                if (ends && there) publish(a.joint + (block * per + here) + c, both(cG, tG), through(root_of(tG), cH, tH));
            }
        }
        if (!found) {
            // the nearest block whose state is there, with the joint sums from it to here
            int from = -1;
            bool way = true;
#pragma unroll
            for (int i = 0; i < BB; ++i) {
                if (i > 0 && i <= block && !(have >> i & 1) && __all(is_set(jnt[i]) || !there)) have |= 1u << i;
                way = way && (have >> i & 1);
                if (from < 0 && way && (i == block || (i < block && __all(is_set(st[i]) || !there)))) from = i;
            }
            if (from >= 0) {
                found = true;
#pragma unroll
                for (int i = BB - 1; i >= 0; --i) {
                    if (i == from && i < block) S = __uint_as_float(st[i]);
                    if (i > 0 && i <= from) S = through(root_of(G_of(jnt[i])), S, H_of(jnt[i]));
                }
            }
        }
    }
    if (!(summed && found)) {
        if (p.lane == 0) s.lost = 1;
        return;
    }
    const float tR = root_of(tG);
    if (ends && there) publish(a.states + ((block + 1) * per + here) + c, through(root_of(both(cG, tG)), S, through(tR, cH, tH)));
    S = through(root_of(cG), S, cH);
    s.S[slot] = S;
    if (last && a.edge_out && there) a.edge_out[here + c] = through(tR, S, tH);
}

// No state came in time: the workgroup walks the sequence up to its tile.  S: the state; the waves' sums are back in LDS.
template <typename T, int VEC, bool SHARED, bool REV>
__device__ __forceinline__ void walk(Shared<VEC>& s, const GlrArgs& a, const Place& p, float (&S)[VEC]) {
    const int64_t per = a.B * a.D, here = p.b * a.D + p.c;
    const int block = p.order / kBlockTiles;
    float tG[VEC], tH[VEC], cG[VEC], cH[VEC], B0[VEC];  // B0: the block's state
#pragma unroll
    for (int i = 0; i < VEC; ++i) B0[i] = a.edge_in ? a.edge_in[here + i] : 0.0f, cG[i] = 0.0f, cH[i] = 0.0f;
    for (int x = 0; x <= p.order; ++x) {
        if (x > 0 && x % kBlockTiles == 0)
#pragma unroll
            for (int i = 0; i < VEC; ++i) B0[i] = through(root_of(cG[i]), B0[i], cH[i]), cG[i] = 0.0f, cH[i] = 0.0f;
#pragma unroll
        for (int i = 0; i < VEC; ++i) S[i] = through(root_of(cG[i]), B0[i], cH[i]);
        __syncthreads();
        sum_tile<T, VEC, SHARED, REV>(s, a, p, REV ? a.tiles - 1 - x : x);
        __syncthreads();
        join_all<VEC, REV, 1>(s, p.lane * VEC, tG, tH);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            cH[i] = through(root_of(tG[i]), cH[i], tH[i]);
            cG[i] = both(cG[i], tG[i]);
        }
    }
    if (p.w != 0 || !p.there) return;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        tH[i] = through(root_of(tG[i]), S[i], tH[i]);
        B0[i] = through(root_of(cG[i]), B0[i], cH[i]);
    }
    if (ends_block(a, p))
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            publish(a.joint + block * per + here + i, cG[i], cH[i]);
            publish(a.states + (block + 1) * per + here + i, B0[i]);
        }
    if (a.edge_out && p.order + 1 == a.tiles)
#pragma unroll
        for (int i = 0; i < VEC; ++i) a.edge_out[here + i] = tH[i];
}

// With the waves' sums on their way to LDS: the state at the tile's edge.
template <typename T, int VEC, bool SHARED, bool REV>
__device__ __forceinline__ void edge_of(Shared<VEC>& s, const GlrArgs& a, const Place& p, float (&S)[VEC]) {
    if (threadIdx.x == 0) s.lost = 0;
    __syncthreads();
    if (p.w < VEC) {
        const uint32_t c0 = __builtin_amdgcn_readfirstlane(p.c);  // the workgroup's first channel (lane 0's exists)
        const int slot = p.w * kWave + p.lane;
        const bool there = c0 + slot < a.D;
        find_edge<VEC, REV>(s, a, p, there ? c0 + slot : 0, there, slot);
    }
    __syncthreads();
    if (s.lost) {
        walk<T, VEC, SHARED, REV>(s, a, p, S);
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) S[i] = s.S[p.lane * VEC + i];
    }
}

constexpr int kMarks = 4;  // 16-byte pieces per lane
__global__ __launch_bounds__(256) void glr_unset_kernel(uint4* rec, int64_t n) {
    for (int64_t i0 = (int64_t)blockIdx.x * 256 * kMarks + threadIdx.x; i0 < n; i0 += (int64_t)gridDim.x * 256 * kMarks)
#pragma unroll
        for (int x = 0; x < kMarks; ++x)
            if (i0 + 256 * x < n) store_words<4>(rec + i0 + 256 * x, Words<4>{{kUnset, kUnset, kUnset, kUnset}});
}

// The state of sequences without steps goes on as it is.
__global__ __launch_bounds__(256) void glr_hand_on_kernel(const float* in, float* out, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) out[i] = in ? in[i] : 0.0f;
}

// Y: q comes in and y goes out; else the states alone.  Bound by the bytes, and by the wait for the edge in launches of a few rounds:
// 8192 x 4096 bf16 76 us (4.4 TB/s of its tensors), 131072 x 1024 with a gate for 16 channels 265 us (4.1; the looks for the edge read
// 100 MB beside the inputs' 822), 3 x 5003 x 1000 fp32 61 us (4.1; rows of 4000 bytes end inside lines, a quarter is read twice).
template <typename T, int VEC, bool SHARED, bool Y>
__global__ __launch_bounds__(kWaves * kWave, 4) void glr_fwd_kernel(GlrArgs a) {
    using P = Pack<T, VEC>;
    using IO = Io<T, VEC, SHARED>;
    __shared__ Shared<VEC> s;
    const Place p = place<VEC, false>(a);
    const Rows at = rows_of(a, p.tile, p.w);
    const uint32_t lane_bytes = p.c * T::kBytes;
    typename P::Raw q[kRowsPerWave], k[kRowsPerWave], v[kRowsPerWave];
    typename IO::G::Raw g[kRowsPerWave];
    load_rows<P>(k, a.k, a, p, at, lane_bytes);
    load_rows<P>(v, a.v, a, p, at, lane_bytes);
    load_rows<typename IO::G>(g, a.g, a, p, at, p.c / (uint32_t)a.group * T::kBytes);
    if constexpr (Y) load_rows<P>(q, a.q, a, p, at, lane_bytes);
    Logs<IO::kGates> logs;
    sum_rows<T, VEC, false>(s, k, v, p, at.n, [&](int r, float(&ga)[VEC]) { IO::gates(g[r], ga, logs); });
    put_logs(s, p, logs);
    float S[VEC];
    edge_of<T, VEC, SHARED, false>(s, a, p, S);
    keep_raw(k);
    keep_raw(v);
    keep_raw(g);
    if (a.marks_out && p.w == 0 && p.there)
#pragma unroll
        for (int i = 0; i < VEC; ++i) a.marks_out[(p.b * a.tiles + p.tile) * a.D + p.c + i] = S[i];
    if (!Y || !p.there) return;
    join<VEC, false>(s, p.w, p.lane, S);
    const auto yp = buffer_of(a.y + (p.b * a.L + at.first) * a.D * T::kBytes);
    const uint32_t step = (uint32_t)a.D * T::kBytes;
    for_rows<false>(at.n, [&](int r) {
        float fq[VEC], fk[VEC], fv[VEC], ga[VEC];
        P::unpack(q[r], fq);
        P::unpack(k[r], fk);
        P::unpack(v[r], fv);
        IO::gates(g[r], ga);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            S[i] = fmaf(fk[i], fv[i], times0(ga[i], S[i]));
            fq[i] *= S[i];
        }
        buffer_store<P>(yp, lane_bytes, r * step, P::pack(fq));
    });
}

// The sum over runs of `lanes` (a power of two) neighbours, in each of them; the order is that of a tree from the nearest up.
__device__ __forceinline__ float sum_of_neighbours(float x, int lanes) {
#define HY_ADD_DPP(ctrl) x += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), ctrl, 0xf, 0xf, true))
    if (lanes >= 2) HY_ADD_DPP(0xb1);    // lane ^ 1
    if (lanes >= 4) HY_ADD_DPP(0x4e);    // lane ^ 2
    if (lanes >= 8) HY_ADD_DPP(0x141);   // the other half of 8 lanes, mirrored
    if (lanes >= 16) HY_ADD_DPP(0x140);  // the other half of 16
#undef HY_ADD_DPP
    if (lanes >= 32) x += __shfl_xor(x, 16, kWave);
    if (lanes >= 64) x += __shfl_xor(x, 32, kWave);
    return x;
}

// dq, dk, dv, dg of every tile from the state before it and the gradient behind it.  Two channels a lane: with four the rows that are
// held spill.  8192 x 4096 bf16 124 us (5.0 TB/s of 617 MB), 131072 x 1024 with a gate for 16 channels 520 us (3.7 TB/s of its tensors; the
// looks for the edge read 145 MB beside the inputs' 1099, and vector instructions fill half of it).
template <typename T, int VEC, bool SHARED>
__global__ __launch_bounds__(kWaves * kWave, 4) void glr_bwd_kernel(GlrArgs a) {
    using P = Pack<T, VEC>;
    using IO = Io<T, VEC, SHARED>;
    __shared__ Shared<VEC> s;
    const Place p = place<VEC, true>(a);
    const Rows at = rows_of(a, p.tile, p.w);
    const uint32_t lane_bytes = p.c * T::kBytes;
    typename P::Raw q[kRowsPerWave], k[kRowsPerWave], v[kRowsPerWave], dy[kRowsPerWave];
    typename IO::G::Raw g[kRowsPerWave];
    load_rows<P>(q, a.q, a, p, at, lane_bytes);
    load_rows<P>(dy, a.dy, a, p, at, lane_bytes);
    load_rows<typename IO::G>(g, a.g, a, p, at, p.c / (uint32_t)a.group * T::kBytes);
    load_rows<P>(k, a.k, a, p, at, lane_bytes);
    load_rows<P>(v, a.v, a, p, at, lane_bytes);
    float S[VEC], R[VEC], decay[kRowsPerWave][IO::kGates];
    Logs<IO::kGates> logs;
#pragma unroll
    for (int r = kRowsPerWave - 1; r >= 0; --r) {  // (a branch for whole tiles keeps later loads behind it)
        float ga[VEC];
        IO::gates(g[r], ga, logs, r < at.n);
#pragma unroll
        for (int i = 0; i < IO::kGates; ++i) decay[r][i] = ga[i];
    }
    put_logs(s, p, logs);
    auto gates = [&](int r, float(&ga)[VEC]) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) ga[i] = decay[r][SHARED ? 0 : i];
    };
    sum_rows<T, VEC, true>(s, q, dy, p, at.n, gates);
    edge_of<T, VEC, SHARED, true>(s, a, p, R);
    keep_raw(q);
    keep_raw(dy);
    join<VEC, true>(s, p.w, p.lane, R);
#pragma unroll
    for (int i = 0; i < VEC; ++i) S[i] = a.marks[(p.b * a.tiles + p.tile) * a.D + p.c + i];
    __syncthreads();
    sum_rows<T, VEC, false>(s, k, v, p, at.n, gates);
    __syncthreads();
    join<VEC, false>(s, p.w, p.lane, S);
    keep_raw(k);
    keep_raw(v);

    const int64_t row = p.b * a.L + at.first;
    const int64_t o0 = row * a.D * T::kBytes;
    const auto dq = buffer_of(a.dq + o0), dk = buffer_of(a.dk + o0), dv = buffer_of(a.dv + o0);
    const uint32_t step = (uint32_t)a.D * T::kBytes;
    float kept[kRowsPerWave][VEC];  // a[t] s[t-1]
    for_rows<false>(at.n, [&](int r) {
        float fk[VEC], fv[VEC], fy[VEC], ga[VEC];
        P::unpack(k[r], fk);
        P::unpack(v[r], fv);
        P::unpack(dy[r], fy);
        gates(r, ga);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            kept[r][i] = times0(ga[i], S[i]);
            S[i] = fmaf(fk[i], fv[i], kept[r][i]);
            fy[i] *= S[i];
        }
        if (p.there) buffer_store<P>(dq, lane_bytes, r * step, P::pack(fy));
    });
    for_rows<true>(at.n, [&](int r) {
        float fk[VEC], fv[VEC], fq[VEC], fy[VEC], dg[VEC], ga[VEC];
        gates(r, ga);
        P::unpack(k[r], fk);
        P::unpack(v[r], fv);
        P::unpack(q[r], fq);
        P::unpack(dy[r], fy);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const float m = fmaf(fq[i], fy[i], R[i]);
            R[i] = times0(ga[i], m);
            dg[i] = p.there ? times0(m, kept[r][i]) : 0.0f;
            const float mv = m * fv[i];
            fv[i] = m * fk[i];
            fk[i] = mv;
        }
        if (p.there) {
            buffer_store<P>(dk, lane_bytes, r * step, P::pack(fk));
            buffer_store<P>(dv, lane_bytes, r * step, P::pack(fv));
        }
        if constexpr (!SHARED) {
            if (p.there) buffer_store<P>(buffer_of(a.dg + o0), lane_bytes, r * step, P::pack(dg));
        } else {
            // the part's lanes are neighbours
            float sum = dg[0];
#pragma unroll
            for (int i = 1; i < VEC; ++i) sum += dg[i];
            const int lanes = a.part / VEC;
            sum = sum_of_neighbours(sum, lanes);
            if (p.there && p.lane % lanes == 0) {
                const float one[1] = {sum};
                const int64_t n = (row + r) * (a.D / a.part);
                const uint32_t m = p.c / (uint32_t)a.part;
                if (a.part == a.group) Pack<T, 1>::store_nt(a.dg + n * T::kBytes + m * T::kBytes, Pack<T, 1>::pack(one));
                else (a.dg_parts + n)[m] = sum;
            }
        }
    });
}

// dg[row][n] = sum over the group's parts, in their order.
template <typename T>
__global__ __launch_bounds__(256) void glr_dg_kernel(const float* parts, char* dg, int64_t n, int32_t per) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        float s[1] = {0.0f};
        for (int32_t j = 0; j < per; ++j) s[0] += parts[i * per + j];
        Pack<T, 1>::store(dg + i * T::kBytes, Pack<T, 1>::pack(s));
    }
}

// One step of every sequence: the state is updated where it is.  64 x 4096: 2.6 us, a launch's time.
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
        s[j] = fmaf(fk[j], fv[j], times0(ga[j], s[j]));
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
        if constexpr (VEC > 2) return HY_ERR_UNSUPPORTED;
        else
        return launch_kernel(glr_bwd_kernel<T, VEC, SHARED>, dim3(grid), dim3(kWaves * kWave), st, a);
    }
    static hy_status step(const GlrPtrs& p, int64_t n, int32_t group, hipStream_t st) {
        const int64_t per = 256 * VEC;
        return launch_kernel(glr_step_kernel<T, VEC, SHARED>, dim3((uint32_t)((n + per - 1) / per)), dim3(256), st,
                             (const char*)p.q, (const char*)p.k, (const char*)p.v, (const char*)p.g, p.state_out, (char*)p.y, n,
                             group);
    }
};

// Channels of a lane: 8 bytes of them where D, the group, every row and every start are multiples, and no more than the waves
// of a workgroup fill.  Rows of 512 bytes per workgroup stream 12% faster than rows of 256.
int vec_of(const GlrShape& s, int most) {
    int vec = std::min(most, s.dtype == HY_F32 ? 2 : 4);
    auto fits = [&](int n) {
        if (s.D % n != 0 || (s.group > 1 && s.group % n != 0) || s.start_align % n != 0) return false;
        for (int i = 0; i < 5; ++i)
            if ((s.rstride[i] % n != 0 || s.bstride[i] % n != 0) && (i != kGlrG || s.group == 1)) return false;  // (gates of
        return true;                                                                                           // groups: one by one)
    };
    while (vec > 1 && (!fits(vec) || kWave * vec / 2 >= s.D)) vec /= 2;
    return vec;
}

// Which lanes the backward has: its rows take a third more registers than the forward's.
constexpr int kBwdVec = 2;

template <typename F>
hy_status by_kind(const GlrShape& s, int vec, F f) {
    const bool shared = s.group > 1;
    if (s.dtype == HY_F32) {
        if (vec == 2) return shared ? f(Kernels<F32, 2, true>{}) : f(Kernels<F32, 2, false>{});
        return shared ? f(Kernels<F32, 1, true>{}) : f(Kernels<F32, 1, false>{});
    }
    if (vec == 4) return shared ? f(Kernels<BF16, 4, true>{}) : f(Kernels<BF16, 4, false>{});
    if (vec == 2) return shared ? f(Kernels<BF16, 2, true>{}) : f(Kernels<BF16, 2, false>{});
    return shared ? f(Kernels<BF16, 1, true>{}) : f(Kernels<BF16, 1, false>{});
}

int64_t tiles_of(const GlrShape& s) { return (s.L + kGlrRows - 1) / kGlrRows; }
int64_t blocks_of(const GlrShape& s) { return (tiles_of(s) + kBlockTiles - 1) / kBlockTiles; }

// The largest power of two that divides `group`, up to the `width` channels of a wave.
int32_t part_of(int32_t group, int32_t width) {
    int32_t part = 1;
    while (part < width && group % (2 * part) == 0) part *= 2;
    return part;
}

int64_t round16(int64_t n) { return (n + 15) / 16 * 16; }

GlrArgs args_of(const GlrPtrs& p, const GlrShape& s, int vec, int64_t* grid) {
    const int64_t e = s.dtype == HY_F32 ? 4 : 2;
    auto src = [&](const void* x, int i) { return Src{(const char*)x, s.bstride[i] * e, s.rstride[i] * e}; };
    GlrArgs a{};
    a.q = src(p.q, kGlrQ), a.k = src(p.k, kGlrK), a.v = src(p.v, kGlrV), a.g = src(p.g, kGlrG), a.dy = src(p.dy, kGlrDy);
    a.y = (char*)p.y, a.dq = (char*)p.dq, a.dk = (char*)p.dk, a.dv = (char*)p.dv, a.dg = (char*)p.dg;
    a.B = s.B, a.L = s.L, a.D = s.D, a.group = s.group;
    const int64_t width = vec * kWave, tiles = tiles_of(s), ncb = (s.D + width - 1) / width;
    // 32 bits address the rows of a wave
    bool near = s.D <= (INT64_C(1) << 26);
    for (int i = 0; i < 5; ++i) near = near && s.rstride[i] <= (INT64_C(1) << 26);
    *grid = near && s.B <= most_workgroups(kWaves * kWave) / tiles / ncb ? s.B * tiles * ncb : -1;
    a.tiles = (int32_t)tiles, a.ncb = (int32_t)ncb;
    a.part = part_of(s.group, (int32_t)width);
    return a;
}

hy_status hand_on(const float* in, float* out, const GlrShape& s, hipStream_t st) {
    return launch_kernel(glr_hand_on_kernel, dim3(workgroups_for(s.B * s.D, 256, 256)), dim3(256), st, in, out, s.B * s.D);
}

// Records of the tiles: none where a sequence is one tile.
int64_t record_bytes(const GlrShape& s) {
    return tiles_of(s) > 1 ? round16(s.B * s.D * (8 * tiles_of(s) + 12 * blocks_of(s))) : 0;
}

hy_status take_records(GlrArgs& a, const GlrShape& s, void* ws, hipStream_t st) {
    const int64_t bytes = record_bytes(s);
    a.sums = static_cast<uint64_t*>(ws);
    a.joint = a.sums + tiles_of(s) * s.B * s.D;
    a.states = reinterpret_cast<uint32_t*>(a.joint + blocks_of(s) * s.B * s.D);
    a.polls = tuning().glr_wait == 0 ? kPolls : tuning().glr_wait == 1 ? 0 : 1;
    if (bytes == 0) return HY_OK;
    return launch_kernel(glr_unset_kernel, dim3(workgroups_for(bytes / 16, 256 * kMarks, 256)), dim3(256), st, static_cast<uint4*>(ws),
                         bytes / 16);
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
    const int vec = vec_of(s, 4);
    GlrArgs a = args_of(p, s, vec, &grid);
    if (grid < 0) return HY_ERR_UNSUPPORTED;
    a.edge_in = p.state_in, a.edge_out = p.state_out, a.marks_out = p.marks_out;
    hy_status rc = take_records(a, s, ws, st);
    if (rc != HY_OK) return rc;
    return by_kind(s, vec, [&](auto kernels) { return kernels.forward(a, (uint32_t)grid, st); });
}

hy_status launch_glr_bwd(const GlrPtrs& p, const GlrShape& s, void* ws, hipStream_t st) {
    if (s.L == 0) return hand_on(p.dstate_out, p.dstate_in, s, st);
    int64_t grid;
    const int vec = vec_of(s, kBwdVec);
    GlrArgs a = args_of(p, s, vec, &grid);
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
        rc = by_kind(s, vec, [&](auto kernels) { return kernels.backward(a, (uint32_t)grid, st); });
    if (rc == HY_OK && a.part != s.group) {
        const int64_t out = s.B * s.L * (s.D / s.group);
        const dim3 g(workgroups_for(out, 256, 256)), b(256);
        const float* parts = a.dg_parts;
        const int32_t per = s.group / a.part;
        rc = s.dtype == HY_F32 ? launch_kernel(glr_dg_kernel<F32>, g, b, st, parts, (char*)p.dg, out, per)
                               : launch_kernel(glr_dg_kernel<BF16>, g, b, st, parts, (char*)p.dg, out, per);
    }
    return rc;
}

hy_status launch_glr_step(const GlrPtrs& p, const GlrShape& s, hipStream_t st) {
    const int64_t n = s.B * s.D;
    if ((n + 255) / 256 > most_workgroups(256)) return HY_ERR_UNSUPPORTED;
    return by_kind(s, vec_of(s, 4), [&](auto kernels) { return kernels.step(p, n, s.group, st); });
}

}  // namespace hy
