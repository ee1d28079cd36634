// Softmax cross entropy of z = x W^T over a vocabulary, and its gradients, without keeping z.
//
//     lse[n] = log sum_v exp z[n, v],  loss[n] = lse[n] - z[n, target[n]]
//     P[n, v] = dloss[n] (exp(z[n, v] - lse[n]) - [v = target[n]]),  dx = P W,  dW = P^T x
//
// Forward: a tile of z stays in registers; each of its rows leaves the largest value and the sum of exponentials below it, and
// a second kernel joins the tiles of a row.  Backward, for a piece of the vocabulary at a time: z again, P from it, and the two
// products.  The matrix products are what bounds it where rows are wide, 8 N V D operations; of narrow rows as much the bytes of P in
// both orders, 8 for a logit (8192 x 65536 bf16: 2.1 ms at D = 256, 2.9 at 512).
//
// bf16 operands enter the products as they are, with k contiguous in both of them: x and, but for few rows, the piece of W are
// transposed once, and P, rounded to bf16 in units of the largest |dloss|, is written in both orders.  fp32 calls multiply in parts,
// to fp32's precision, keep P in fp32, and read P and W across k where a product needs it.
//
// Measured, loss and gradients: 8192 x 65536 x 4096 bf16 14.1-14.7 ms (1.20-1.25 PFLOP/s, the four products at 1.15 to 1.3),
// 8192 x 512 x 4096 197 us (0.70 PFLOP/s: tiles of 128 x 128 on 256 compute units once, and 30 us of transposition);
// 1003 x 5003 x 1000 fp32 283 us (0.85 PFLOP/s of the six products of parts).  The loss alone, 8 x 65536 x 4096: 105 us, 5.1 TB/s.
#include <algorithm>

#include "hy_gemm.hpp"
#include "hy_launch.hpp"

namespace hy {

namespace {

// What an element of T is in a product: its bits.
template <typename T>
using Bits = std::conditional_t<T::kBytes == 4, uint32_t, uint16_t>;

// Rows of D bf16 numbers -> rows of `ld`, zeros behind them: rows that do not begin where 16 bytes do.
__global__ __launch_bounds__(256) void pack_kernel(const uint16_t* src, uint16_t* dst, int64_t rows, int64_t D, int64_t ld) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * ld; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / ld, c = i % ld;
        dst[i] = c < D ? src[r * D + c] : 0;
    }
}

// The largest weight of a row that takes part, by one workgroup.  P in this unit is -1 where a target is far from foreseen, which
// bf16 holds; as a multiple of 1 / N, say, all those would be rounded alike, and the errors of a sum over them would not cancel.
struct Unit {
    const float* dloss;
    float* unit;  // null: none is wanted
};
__device__ __forceinline__ void find_unit(const Unit& u, const int64_t* target, int64_t rows, int64_t V) {
    __shared__ float tops[256 / kWave];
    float top = 0.0f;
    constexpr int kTogether = 16;  // rows of a lane on their way together: one wait for 4096 of them
    for (int64_t m0 = threadIdx.x; m0 < rows; m0 += 256 * kTogether) {
        float d[kTogether];
        int64_t v[kTogether];
#pragma unroll
        for (int i = 0; i < kTogether; ++i) {
            const int64_t m = m0 + 256 * i < rows ? m0 + 256 * i : m0;
            d[i] = fabsf(u.dloss[m]);
            v[i] = target[m];
        }
#pragma unroll
        for (int i = 0; i < kTogether; ++i)
            if (v[i] >= 0 && v[i] < V && d[i] < INFINITY) top = fmaxf(top, d[i]);
    }
    for (int d = 32; d > 0; d /= 2) top = fmaxf(top, __shfl_xor(top, d, kWave));
    if (threadIdx.x % kWave == 0) tops[threadIdx.x / kWave] = top;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 256 / kWave; ++i) top = fmaxf(top, tops[i]);
        *u.unit = top > 0.0f ? top : 1.0f;
    }
}

// Rows of D numbers -> D rows of `ld` (a multiple of 64); zeros behind the last row, and for the rows whose target is none.
// Pieces of 64 x 64 through LDS, 16 bytes a lane.  The workgroups of the first row of the grid have nothing to turn: one finds the
// weights' unit.
template <typename T>
__global__ __launch_bounds__(256) void turn_kernel(const Bits<T>* src, Bits<T>* dst, int64_t rows, int64_t D, int64_t ld,
                                                   const int64_t* target, int64_t V, Unit unit) {
    if (unit.unit && blockIdx.y == 0) {
        if (blockIdx.x == 0) find_unit(unit, target, rows, V);
        return;
    }
    constexpr int kPer = 16 / T::kBytes, kLanes = 64 / kPer, kPitch = 64 + kPer;  // numbers of a lane, lanes of a row
    __shared__ __attribute__((aligned(16))) Bits<T> s[64][kPitch];
    const int64_t r0 = (int64_t)blockIdx.x * 64, c0 = (int64_t)(blockIdx.y - (unit.unit ? 1 : 0)) * 64;
    const int x = threadIdx.x % kLanes * kPer;
#pragma unroll
    for (int y = threadIdx.x / kLanes; y < 64; y += 256 / kLanes) {
        const int64_t r = r0 + y, c = c0 + x;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (r < rows && c < D && (!target || (target[r] >= 0 && target[r] < V))) {
            const Bits<T>* p = src + r * D + c;
            if (D % kPer == 0) {
                v = *reinterpret_cast<const uint4*>(p);
            } else {
                Bits<T> one[kPer];
#pragma unroll
                for (int i = 0; i < kPer; ++i) one[i] = c + i < D ? p[i] : 0;
                v = *reinterpret_cast<const uint4*>(one);
            }
        }
        *reinterpret_cast<uint4*>(&s[y][x]) = v;
    }
    __syncthreads();
#pragma unroll
    for (int y = threadIdx.x / kLanes; y < 64; y += 256 / kLanes) {
        if (c0 + y >= D) continue;
        Bits<T> one[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i) one[i] = s[x + i][y];
        *reinterpret_cast<uint4*>(dst + (c0 + y) * ld + r0 + x) = *reinterpret_cast<const uint4*>(one);
    }
}

struct XentArgs {
    GemmArgs g;
    const int64_t* target;
    int64_t V, v0;            // the vocabulary, and the first column of this piece
    // losses
    float2* part;             // [rows][tiles]: the largest value and the sum below it
    int64_t tiles, tile0;
    float* zt;                // [rows] the targets' values
    // gradients
    const float *lse, *dloss;
    const float* unit;        // dloss is taken in this unit (null: 1), and the products are taken back
    void *p, *pt;             // P [rows][p_ld], bf16 or fp32, and of bf16 its transpose [columns][pt_ld]
    int64_t p_ld, pt_ld;
    // products
    char* out;
    float* sum;               // the sum so far (not of the first piece)
    int64_t out_ld;
    bool first, last;
    float* split;             // [splits][rows][out_ld]: where a product's k is divided among workgroups
    int32_t splits;
};

// A row of a tile of P: its target's column, whether it takes part, lse and dloss.
struct RowNeeds {
    int32_t want, counts;
    float lse, weight;
};

// The target's column within a tile of `width` columns that begins at `first`; -1: it is none of them.
__device__ __forceinline__ int column_of(int64_t target, int64_t first, int width) {
    const int64_t c = target - first;
    return c >= 0 && c < width ? (int)c : -1;
}

// exp as a power of two: off by 6e-8 (1 + |x|) of itself, so what is small beside the sum it goes into may be off by more.  Losses
// take it in fp32 calls too: over the terms of a sum these errors average out to some 1e-7 of it, about lse's own rounding.
__device__ __forceinline__ float fast_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }

// Tiles in runs of a few rows of tiles, a run of neighbours for each XCD: what its workgroups share stays in its L2.
template <int BM, int BN>
__device__ __forceinline__ void tile_of(const GemmArgs& g, uint32_t index, int64_t* m0, int64_t* n0, uint32_t* tn) {
    constexpr uint32_t kRun = 8;
    const uint32_t i = xcd_contiguous(index, (uint32_t)g.mt * (uint32_t)g.nt);
    const uint32_t per = kRun * (uint32_t)g.nt, first = i / per * kRun;
    const uint32_t h = (uint32_t)g.mt - first < kRun ? (uint32_t)g.mt - first : kRun;
    *tn = i % per / h;
    *m0 = (int64_t)(first + i % per % h) * BM;
    *n0 = (int64_t)*tn * BN;
}

template <typename G, int BM, int BN, int MW, int NW>
__global__ __launch_bounds__(MW * NW * kWave) void loss_kernel(XentArgs a) {
    __shared__ __attribute__((aligned(16))) char lds[G::kLds + BM * 4];
    int* const wants = reinterpret_cast<int*>(lds + G::kLds);  // what the rows need, loaded in front of the product
    G t;
    int64_t m0, n0;
    uint32_t tn;
    tile_of<BM, BN>(a.g, blockIdx.x, &m0, &n0, &tn);
    const int cols = a.g.b.rows - n0 < BN ? (int)(a.g.b.rows - n0) : BN;  // of the piece: behind it are the next one's targets
    for (int row = threadIdx.x; row < BM; row += G::kThreads)
        wants[row] = m0 + row < a.g.a.rows ? column_of(a.target[m0 + row], a.v0 + n0, cols) : -1;
    t.run(lds, a.g, m0, n0, 0, (a.g.K + G::kStep - 1) / G::kStep);
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int wm = w % MW, wn = w / MW, li = lane % 16, lq = lane / 16;
    float2(*share)[NW] = reinterpret_cast<float2(*)[NW]>(lds);
    const int col0 = wn * G::WN + 4 * lq;
    __syncthreads();  // the tiles have been read
#pragma unroll
    for (int i = 0; i < G::MI; ++i) {
        const int row = wm * G::WM + i * 16 + li;
        const int64_t m = m0 + row;
        const int want = wants[row];
        float top = -INFINITY;
        if (cols < BN)
#pragma unroll
            for (int j = 0; j < G::NI; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (col0 + j * 16 + r >= cols) t.acc[i][j][r] = -INFINITY;
#pragma unroll
        for (int j = 0; j < G::NI; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (col0 + j * 16 + r == want) a.zt[m] = t.acc[i][j][r];
                top = fmaxf(top, t.acc[i][j][r]);
            }
        top = fmaxf(top, __shfl_xor(top, 16, kWave));
        top = fmaxf(top, __shfl_xor(top, 32, kWave));
        const float ref = top == -INFINITY ? 0.0f : top;
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < G::NI; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) sum += fast_exp(t.acc[i][j][r] - ref);
        sum += __shfl_xor(sum, 16, kWave);
        sum += __shfl_xor(sum, 32, kWave);
        if (lq == 0) share[row][wn] = make_float2(top, sum);
    }
    __syncthreads();
    for (int row = threadIdx.x; row < BM; row += G::kThreads) {
        if (m0 + row >= a.g.a.rows) continue;
        float top = -INFINITY, sum = 0.0f;
        for (int x = 0; x < NW; ++x) top = fmaxf(top, share[row][x].x);
        const float ref = top == -INFINITY ? 0.0f : top;
        for (int x = 0; x < NW; ++x) sum += share[row][x].y * fast_exp(share[row][x].x - ref);
        a.part[(m0 + row) * a.tiles + a.tile0 + tn] = make_float2(top, sum);
    }
}

// Few rows of fp32 x: the losses' part of kFewWords words and up to 16 NT rows per workgroup, bounded by the bytes of W, which go from
// memory to registers, become parts there and are multiplied.  The eight waves divide k; x comes from the caches.
constexpr int kFewWords = 64, kFewWaves = 8, kFewTiles = kFewWords / 16;

// Values k .. k + 7 of a row of D (a multiple of 4); zeros from D on.
__device__ __forceinline__ void few_load(float4 (&v)[2], const float* row, int64_t k, int64_t D) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
        v[i] = k + 4 * i < D ? *reinterpret_cast<const float4*>(row + k + 4 * i) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
}
template <int NT>
__global__ __launch_bounds__(kFewWaves * kWave) void few_kernel(const float* x, const float* w, const int64_t* target, float2* part, float* zt,
                                                                int64_t N, int64_t V, int64_t D, int64_t tiles) {
    constexpr int U = 2;  // steps of 32 k on their way together
    __shared__ f32x4_t sums[kFewWaves][kFewTiles * NT][kWave];
    __shared__ float2 tops[kFewTiles][16 * NT];
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, li = lane % 16, lq = lane / 16;
    const int64_t v0 = (int64_t)blockIdx.x * kFewWords;
    const float *wr[kFewTiles], *xr[NT];
#pragma unroll
    for (int i = 0; i < kFewTiles; ++i) wr[i] = w + std::min(v0 + i * 16 + li, V - 1) * D;
#pragma unroll
    for (int j = 0; j < NT; ++j) xr[j] = x + std::min((int64_t)(j * 16 + li), N - 1) * D;
    f32x4_t acc[kFewTiles][NT] = {};
    const int64_t steps = (D + 31) / 32, each = (steps + kFewWaves - 1) / kFewWaves;
    const int64_t end = std::min(steps, each * (wv + 1));
    for (int64_t s = each * wv; s < end; s += U) {
        float4 rw[U][kFewTiles][2], rx[U][NT][2];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t k = s + u < end ? (s + u) * 32 + lq * 8 : D;  // (from D on: zeros)
#pragma unroll
            for (int i = 0; i < kFewTiles; ++i) few_load(rw[u][i], wr[i], k, D);
#pragma unroll
            for (int j = 0; j < NT; ++j) few_load(rx[u][j], xr[j], k, D);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            uint4 fx[NT][3], fw[3];
#pragma unroll
            for (int j = 0; j < NT; ++j) parts_of(rx[u][j], fx[j]);
#pragma unroll
            for (int i = 0; i < kFewTiles; ++i) {
                parts_of(rw[u][i], fw);
#pragma unroll
                for (int j = 0; j < NT; ++j) {
#pragma unroll
                    for (int y = 0; y < kSplitProducts; ++y)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, fw[kSplitB[y]]),
                                                                            __builtin_bit_cast(bf16x8_t, fx[j][kSplitA[y]]), acc[i][j], 0, 0, 0);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kFewTiles; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) sums[wv][i * NT + j][lane] = acc[i][j];
    __syncthreads();
    // a wave joins the waves' shares of its pieces of 16 words by 16 rows: lane (li, lq) has row li, words 4 lq .. 4 lq + 3
    for (int piece = wv; piece < kFewTiles * NT; piece += kFewWaves) {
        const int i = piece / NT, j = piece % NT;
        f32x4_t z = sums[0][piece][lane];
        for (int y = 1; y < kFewWaves; ++y) z += sums[y][piece][lane];
        const int64_t m = j * 16 + li;
        const int want = m < N ? column_of(target[m], v0, kFewWords) : -1;
        float top = -INFINITY;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int word = i * 16 + 4 * lq + r;
            if (v0 + word >= V) z[r] = -INFINITY;
            else if (word == want) zt[m] = z[r];
            top = fmaxf(top, z[r]);
        }
        top = fmaxf(top, __shfl_xor(top, 16, kWave));
        top = fmaxf(top, __shfl_xor(top, 32, kWave));
        const float ref = top == -INFINITY ? 0.0f : top;
        float sum = 0.0f;
#pragma unroll
        for (int r = 0; r < 4; ++r) sum += fast_exp(z[r] - ref);
        sum += __shfl_xor(sum, 16, kWave);
        sum += __shfl_xor(sum, 32, kWave);
        if (lq == 0) tops[i][m] = make_float2(top, sum);
    }
    __syncthreads();
    const int m = threadIdx.x;
    if (m < 16 * NT && m < N) {
        float top = -INFINITY, sum = 0.0f;
        for (int i = 0; i < kFewTiles; ++i) top = fmaxf(top, tops[i][m].x);
        const float ref = top == -INFINITY ? 0.0f : top;
        for (int i = 0; i < kFewTiles; ++i) sum += tops[i][m].y * fast_exp(tops[i][m].x - ref);
        part[m * tiles + blockIdx.x] = make_float2(top, sum);
    }
}

// A wave joins the tiles of a row.
__global__ __launch_bounds__(256) void join_kernel(const float2* part, const float* zt, const int64_t* target, float* loss,
                                                   float* lse, int64_t rows, int64_t tiles, int64_t V) {
    const int64_t m = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
    const int lane = threadIdx.x % kWave;
    if (m >= rows) return;
    float top = -INFINITY, sum = 0.0f;
    for (int64_t i = lane; i < tiles; i += kWave) top = fmaxf(top, part[m * tiles + i].x);
    for (int d = 32; d > 0; d /= 2) top = fmaxf(top, __shfl_xor(top, d, kWave));
    const float ref = top == -INFINITY ? 0.0f : top;
    for (int64_t i = lane; i < tiles; i += kWave) {
        const float2 x = part[m * tiles + i];
        sum += x.y * expf(x.x - ref);
    }
    for (int d = 32; d > 0; d /= 2) sum += __shfl_xor(sum, d, kWave);
    if (lane == 0) {
        const float rest = logf(sum);
        lse[m] = ref + rest;
        // (lse less the target's value would lose what is small beside the largest value)
        loss[m] = target[m] >= 0 && target[m] < V ? (ref - zt[m]) + rest : 0.0f;
    }
}

// A wave's part of a result, rounded to bf16, to rows of `ld` (a multiple of 8) from (m0, n0) on, as far as there are `rows` and `cols`
// (a multiple of 8): through its own part of LDS, so that a row leaves in 16-byte pieces side by side.
template <typename G>
__device__ __forceinline__ void rows_out(const f32x4_t (&acc)[G::MI][G::NI], uint32_t* own, uint16_t* to, int64_t ld, int64_t m0, int64_t n0,
                                         int64_t rows, int64_t cols) {
    const int lane = threadIdx.x % kWave, li = lane % 16, lq = lane / 16;
    constexpr int kMask = G::WN / 8 < 8 ? G::WN / 8 - 1 : 7;  // pieces of 4 words trade places by row
#pragma unroll
    for (int i = 0; i < G::MI; ++i)
#pragma unroll
        for (int j = 0; j < G::NI; ++j) {
            const int row = i * 16 + li, piece = j * 2 + lq / 2;
            *reinterpret_cast<uint2*>(own + row * (G::WN / 2) + (piece ^ (row & kMask)) * 4 + lq % 2 * 2) =
                make_uint2(pack_bf16x2(acc[i][j][0], acc[i][j][1]), pack_bf16x2(acc[i][j][2], acc[i][j][3]));
        }
    constexpr int kLanes = G::WN / 8;
#pragma unroll
    for (int y = 0; y < G::WM; y += kWave / kLanes) {
        const int row = y + lane / kLanes, piece = lane % kLanes;
        const uint4 v = *reinterpret_cast<const uint4*>(own + row * (G::WN / 2) + (piece ^ (row & kMask)) * 4);
        const int64_t m = m0 + row, n = n0 + 8 * piece;
        if (m < rows && n < cols) *reinterpret_cast<uint4*>(to + m * ld + n) = v;
    }
}

template <typename T, typename G, int BM, int BN, int MW, int NW>
__global__ __launch_bounds__(MW * NW * kWave) void grad_kernel(XentArgs a) {
    __shared__ __attribute__((aligned(16))) char lds[G::kLds + BM * 16];
    // What the rows need, loaded in front of the product (a part of the same array: beside another one the compiler takes any
    // read from LDS for one of the loads into it, and waits).
    RowNeeds* const needs = reinterpret_cast<RowNeeds*>(lds + G::kLds);
    G t;
    int64_t m0, n0;
    uint32_t tn;
    tile_of<BM, BN>(a.g, blockIdx.x, &m0, &n0, &tn);
    for (int row = threadIdx.x; row < BM; row += G::kThreads) {
        const int64_t m = m0 + row < a.g.a.rows ? m0 + row : 0, v = a.target[m];
        needs[row] = RowNeeds{column_of(v, a.v0 + n0, BN), m0 + row < a.g.a.rows && v >= 0 && v < a.V, a.lse[m],
                              a.unit ? a.dloss[m] / *a.unit : a.dloss[m]};
    }
    t.run(lds, a.g, m0, n0, 0, (a.g.K + G::kStep - 1) / G::kStep);
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int wm = w % MW, wn = w / MW, li = lane % 16, lq = lane / 16;
    const int64_t rows = a.g.a.rows;
    const int cols = a.g.b.rows - n0 < BN ? (int)(a.g.b.rows - n0) : BN, col0 = wn * G::WN + 4 * lq;
#pragma unroll
    for (int i = 0; i < G::MI; ++i) {
        const RowNeeds need = needs[wm * G::WM + i * 16 + li];
#pragma unroll
        for (int j = 0; j < G::NI; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int col = col0 + j * 16 + r;
                const float z = t.acc[i][j][r] - need.lse;
                float p = T::kBytes == 4 ? expf(z) : fast_exp(z);
                if (col == need.want) p -= 1.0f;
                t.acc[i][j][r] = need.counts && col < cols ? need.weight * p : 0.0f;  // zeros, whatever is in the row
            }
    }
    if constexpr (T::kBytes == 4) {
        // 64 bytes of a row side by side
#pragma unroll
        for (int i = 0; i < G::MI; ++i)
#pragma unroll
            for (int j = 0; j < G::NI; ++j) {
                const int64_t m = m0 + wm * G::WM + i * 16 + li, n = n0 + col0 + j * 16;
                if (m < rows && n < a.p_ld) *reinterpret_cast<f32x4_t*>(static_cast<float*>(a.p) + m * a.p_ld + n) = t.acc[i][j];
            }
        return;
    }
    // Both orders go out through the wave's own part of LDS, so that a row leaves in 16-byte pieces side by side.  As they are in
    // the registers, four columns or one row at a time, they took a fifth of the kernel's time.
    constexpr int kT = G::WM / 2, kTMask = kT / 8 - 1;  // P^T: words of a row; pieces of 8 words trade places by row
    uint32_t* own = reinterpret_cast<uint32_t*>(lds) + w * (G::WM * G::WN / 2);
    __syncthreads();  // the tiles have been read
    {
#pragma unroll
        for (int i = 0; i < G::MI; ++i)
#pragma unroll
            for (int j = 0; j < G::NI; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    // columns 2 h and 2 h + 1 of this row and of its neighbour: an even lane takes the first of both rows, an odd
                    // one the second
                    const uint32_t mine = pack_bf16x2(t.acc[i][j][2 * h], t.acc[i][j][2 * h + 1]);
                    const uint32_t other = __builtin_amdgcn_update_dpp(0, mine, 0xb1, 0xf, 0xf, true);
                    const uint32_t both = li % 2 ? other >> 16 | (mine & 0xffff0000u) : (mine & 0xffffu) | other << 16;
                    const int row = j * 16 + 4 * lq + 2 * h + li % 2, word = i * 8 + li / 2;
                    own[row * kT + (word ^ ((((row >> 1 & 6) | (row & 1)) & kTMask) * 8))] = both;
                }
        constexpr int kTLanes = kT / 4;  // lanes of a row
#pragma unroll
        for (int y = 0; y < G::WN; y += kWave / kTLanes) {
            const int row = y + lane / kTLanes, word = lane % kTLanes * 4;
            const uint4 v = *reinterpret_cast<const uint4*>(own + row * kT + (word ^ ((((row >> 1 & 6) | (row & 1)) & kTMask) * 8)));
            const int64_t n = n0 + wn * G::WN + row, m = m0 + wm * G::WM + 2 * word;
            if (n < a.g.b.rows && m < a.pt_ld) *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.pt) + n * a.pt_ld + m) = v;
        }
        rows_out<G>(t.acc, own, static_cast<uint16_t*>(a.p), a.p_ld, m0 + wm * G::WM, n0 + wn * G::WN, rows, a.p_ld);
    }
}

// Up to four neighbouring elements of a product on their way out: a share of it; or with the sum so far, to the sum or to the
// result.  none: the row takes no part.
template <typename T>
__device__ __forceinline__ void finish(const XentArgs& a, float (&f)[4], int64_t at, int have, bool none, float* split, float unit) {
    const bool four = have == 4 && a.out_ld % 4 == 0;
    float* to = split ? split : a.last ? nullptr : a.sum;
    if (!split)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if (none) f[r] = 0.0f;
            if (!a.first && r < have) f[r] += a.sum[at + r];
        }
    if (!to)
#pragma unroll
        for (int r = 0; r < 4; ++r) f[r] *= unit;
    if (four) {
        if (to) Pack<F32, 4>::store(to + at, Pack<F32, 4>::pack(f));
        else Pack<T, 4>::store(a.out + at * T::kBytes, Pack<T, 4>::pack(f));
        return;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
        if (r < have) {
            const float one[1] = {f[r]};
            if (to) to[at + r] = f[r];
            else Pack<T, 1>::store(a.out + (at + r) * T::kBytes, Pack<T, 1>::pack(one));
        }
}

// out = A B^T, or its sum over pieces.
template <typename T, typename G, int BM, int BN, int MW, int NW>
__global__ __launch_bounds__(MW * NW * kWave) void product_kernel(XentArgs a) {
    __shared__ __attribute__((aligned(16))) char lds[G::kLds + BM * 4];
    int* const nones = reinterpret_cast<int*>(lds + G::kLds);
    G t;
    int64_t m0, n0;
    uint32_t tn;
    const uint32_t tiles = (uint32_t)a.g.mt * (uint32_t)a.g.nt, share = blockIdx.x / tiles;
    tile_of<BM, BN>(a.g, blockIdx.x - share * tiles, &m0, &n0, &tn);
    const int steps = (a.g.K + G::kStep - 1) / G::kStep;
    for (int row = threadIdx.x; row < BM; row += G::kThreads)
        nones[row] = a.target && m0 + row < a.g.a.rows && (a.target[m0 + row] < 0 || a.target[m0 + row] >= a.V);
    t.run(lds, a.g, m0, n0, (int)((int64_t)steps * share / a.splits), (int)((int64_t)steps * (share + 1) / a.splits));
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int wm = w % MW, wn = w / MW, li = lane % 16, lq = lane / 16;
    const float unit = a.unit ? *a.unit : 1.0f;
    float* split = a.splits > 1 ? a.split + share * a.g.a.rows * a.out_ld : nullptr;
    if constexpr (T::kBytes == 2)
        if (!split && a.first && a.last && a.out_ld % 8 == 0) {
            __syncthreads();  // the tiles have been read
#pragma unroll
            for (int i = 0; i < G::MI; ++i) {
                const bool none = nones[wm * G::WM + i * 16 + li];
#pragma unroll
                for (int j = 0; j < G::NI; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r) t.acc[i][j][r] = none ? 0.0f : t.acc[i][j][r] * unit;
            }
            rows_out<G>(t.acc, reinterpret_cast<uint32_t*>(lds) + w * (G::WM * G::WN / 2), reinterpret_cast<uint16_t*>(a.out), a.out_ld,
                        m0 + wm * G::WM, n0 + wn * G::WN, a.g.a.rows, a.g.b.rows);
            return;
        }
#pragma unroll
    for (int i = 0; i < G::MI; ++i) {
        const int64_t m = m0 + wm * G::WM + i * 16 + li;
        if (m >= a.g.a.rows) continue;
        const bool none = nones[m - m0];
#pragma unroll
        for (int j = 0; j < G::NI; ++j) {
            const int64_t n = n0 + wn * G::WN + j * 16 + 4 * lq, at = m * a.out_ld + n;
            const int have = a.g.b.rows - n < 4 ? (int)(a.g.b.rows - n) : 4;
            float f[4] = {t.acc[i][j][0], t.acc[i][j][1], t.acc[i][j][2], t.acc[i][j][3]};
            finish<T>(a, f, at, have, none, split, unit);
        }
    }
}

// The sum of a product's shares, in their order; four elements a lane.
template <typename T>
__global__ __launch_bounds__(256) void gather_kernel(XentArgs a) {
    const int64_t quads = (a.out_ld + 3) / 4, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= a.g.a.rows * quads) return;
    const int64_t m = i / quads, n = i % quads * 4, at = m * a.out_ld + n;
    const int have = a.out_ld - n < 4 ? (int)(a.out_ld - n) : 4;
    float f[4] = {};
    for (int s = 0; s < a.splits; ++s) {
        const float* p = a.split + s * a.g.a.rows * a.out_ld + at;
        if (have == 4 && a.out_ld % 4 == 0) {
            const float4 x = *reinterpret_cast<const float4*>(p);
            f[0] += x.x, f[1] += x.y, f[2] += x.z, f[3] += x.w;
        } else {
            for (int r = 0; r < have; ++r) f[r] += p[r];
        }
    }
    finish<T>(a, f, at, have, a.target && (a.target[m] < 0 || a.target[m] >= a.V), nullptr, a.unit ? *a.unit : 1.0f);
}

__global__ __launch_bounds__(256) void zero_kernel(char* p, int64_t bytes) {
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 2; i < bytes; i += (int64_t)gridDim.x * 512)
        *reinterpret_cast<uint16_t*>(p + i) = 0;
}

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
int64_t cut(int64_t n, int64_t by) { return (n + by - 1) / by; }

// How a problem is laid out.
struct Layout {
    bool packed;              // x and W are copied for the products (bf16 rows that do not begin where 16 bytes do)
    int64_t ld;               // of x and W in the products
    int64_t nt;               // N rounded up: the k of dW
    int64_t piece, pieces;    // columns of the vocabulary at a time
    int64_t sizes[2];         // of all pieces but the last, and of the last
};

constexpr int64_t kPieceBytes = INT64_C(512) << 20;  // of P and its transpose

Layout layout_of(const XentShape& s) {
    Layout l;
    const int64_t e = s.dtype == HY_F32 ? 4 : 2;
    l.packed = s.dtype == HY_BF16 && s.D % 8 != 0;
    l.ld = l.packed ? up(s.D, kGemmK) : s.D;
    l.nt = up(s.N, kGemmK);
    const int64_t most = std::min<int64_t>(std::max<int64_t>(1024, kPieceBytes / (2 * e * l.nt) / 256 * 256), 1 << 22);
    l.pieces = cut(s.V, most);
    l.piece = std::min(up(cut(s.V, l.pieces), 256), up(s.V, kGemmK));
    l.pieces = cut(s.V, l.piece);
    l.sizes[1] = s.V - (l.pieces - 1) * l.piece;
    l.sizes[0] = l.pieces > 1 ? l.piece : l.sizes[1];
    return l;
}

// Pieces of the workspace, in order.
struct Carver {
    uintptr_t at;  // (a number: sizes are found without a workspace)
    explicit Carver(void* ws) : at(reinterpret_cast<uintptr_t>(ws)) {}
    template <typename T>
    T* take(int64_t n) {
        const uintptr_t p = at;
        at += (uintptr_t)up(n * (int64_t)sizeof(T), 256);
        return reinterpret_cast<T*>(p);
    }
};

// Up to 32 rows of fp32 values that begin where 16 bytes do.
bool few_rows(const XentShape& s) { return s.dtype == HY_F32 && s.N <= 32 && s.D % 4 == 0 && cut(s.V, kFewWords) <= most_workgroups(kFewWaves * kWave); }

struct FwdSpace {
    uint16_t *x, *w;
    float2* part;
    float* zt;
    int64_t tiles;
    FwdSpace(const XentShape& s, const Layout& l, Carver& c) {
        const int64_t edge = s.N <= 64 ? 64 : 128;  // the narrowest tiles
        tiles = few_rows(s) ? cut(s.V, kFewWords) : (l.pieces - 1) * cut(l.sizes[0], edge) + cut(l.sizes[1], edge);
        x = l.packed ? c.take<uint16_t>(s.N * l.ld) : nullptr;
        w = l.packed ? c.take<uint16_t>(std::min(l.piece, s.V) * l.ld) : nullptr;
        part = c.take<float2>(s.N * tiles);
        zt = c.take<float>(s.N);
    }
};

GemmArgs product_of(const GemmOperand& a, const GemmOperand& b, int64_t K) {
    GemmArgs g{};
    g.a = a, g.b = b, g.K = (int32_t)K;
    return g;
}

// The logits of a piece of `cols` columns.
GemmArgs logits_of(const XentShape& s, const Layout& l, int64_t cols) {
    return product_of(GemmOperand{nullptr, l.ld, s.N}, GemmOperand{nullptr, l.ld, cols}, l.packed ? l.ld : s.D);
}

// Tiles of 256 x 256 (1.10 PFLOP/s at 8192 x 4096 x 4096) where they fill most of the chip and are more than a few steps long (60 rows
// against 60000 symbols of width 4096, dW's k of 64: 727 us a training step so, 710 in tiles of 128 x 128; the same at a k of 512,
// 3-7% more time at 1024); else of 128 x 128: four steps in
// LDS (0.85 PFLOP/s with one workgroup per compute unit, 8192 x 512 x 4096), or two, where more workgroups than compute units
// can share them.
enum class Tile { k256, k128Deep, k128, kFew32, kFew64, kWide, kAcross };
Tile tile_for(const GemmArgs& g) {
    if (cut(g.a.rows, 256) * cut(g.b.rows, 256) >= 192 && g.K > 256) return Tile::k256;
    return cut(g.a.rows, 128) * cut(g.b.rows, 128) <= 256 ? Tile::k128Deep : Tile::k128;
}
struct Edges {
    int64_t rows, cols;
};
Edges edges_of(Tile t) {
    switch (t) {
        case Tile::k256: return {256, 256};
        case Tile::kFew32: return {32, 64};
        case Tile::kFew64: return {64, 64};
        case Tile::kWide: return {128, 192};
        default: return {128, 128};
    }
}
// The logits of few rows are bounded by the bytes of W: narrow tiles with many steps on their way (8 x 65536 x 4096: 134 us in tiles of
// 256 x 256, 106 in tiles of 32 x 64).
Tile logit_tile(const GemmArgs& g) { return g.a.rows <= 32 ? Tile::kFew32 : g.a.rows <= 64 ? Tile::kFew64 : tile_for(g); }

// Whether HIP takes a workgroup for every tile (more than one only where tiles are few).
bool launchable(const GemmArgs& g, Tile tile) {
    const Edges e = edges_of(tile);
    return cut(g.a.rows, e.rows) <= most_workgroups(tile == Tile::kFew32 || tile == Tile::kFew64 ? 256 : 512) / cut(g.b.rows, e.cols);
}

template <typename F>
hy_status by_tile(XentArgs& a, Tile tile, F f) {
    const Edges e = edges_of(tile);
    const int64_t mt = cut(a.g.a.rows, e.rows), nt = cut(a.g.b.rows, e.cols);
    if (!launchable(a.g, tile)) return HY_ERR_UNSUPPORTED;
    a.g.mt = (int32_t)mt, a.g.nt = (int32_t)nt;
    return f(dim3((uint32_t)(mt * nt)));
}

// fp32 operands: one workgroup per compute unit has room in LDS, so tiles of 128 x 128, or of 128 x 192 where fewer rounds of them are
// less work for the busiest compute unit and k is not divided instead (1003 x 5003 x 1000: 320 tiles, or 216, a fifth
// less time).
Tile split_tile(const GemmArgs& g) {
    const int64_t square = cut(g.a.rows, 128) * cut(g.b.rows, 128), wide = cut(g.a.rows, 128) * cut(g.b.rows, 192);
    return square > 128 && 3 * cut(wide, 256) < 2 * cut(square, 256) ? Tile::kWide : Tile::k128;
}

template <typename T>
Tile logit_tile_for(const GemmArgs& g) {
    return T::kBytes == 2 ? logit_tile(g) : g.a.rows <= 64 ? Tile::kFew64 : split_tile(g);
}
template <typename T, bool TB>
Tile product_tile_for(const GemmArgs& g) {
    if (T::kBytes == 2) return TB ? Tile::kAcross : tile_for(g);
    return g.a.rows <= 64 || g.K <= 64 ? Tile::kFew64 : split_tile(g);
}

template <typename T>
hy_status losses(XentArgs& a, hipStream_t st) {
    const Tile tile = logit_tile_for<T>(a.g);
    return by_tile(a, tile, [&](dim3 grid) {
        if constexpr (T::kBytes == 4)
            switch (tile) {
                case Tile::kFew64: return launch_kernel(loss_kernel<GemmSplit<64, 64, 1, 4>, 64, 64, 1, 4>, grid, dim3(256), st, a);
                case Tile::kWide: return launch_kernel(loss_kernel<GemmSplit<128, 192, 2, 4>, 128, 192, 2, 4>, grid, dim3(512), st, a);
                default: return launch_kernel(loss_kernel<GemmSplit<128, 128, 2, 4>, 128, 128, 2, 4>, grid, dim3(512), st, a);
            }
        else
            switch (tile) {
                case Tile::k256: return launch_kernel(loss_kernel<Gemm<256, 256, 2, 4, 2>, 256, 256, 2, 4>, grid, dim3(512), st, a);
                case Tile::k128: return launch_kernel(loss_kernel<Gemm<128, 128, 2, 4, 2>, 128, 128, 2, 4>, grid, dim3(512), st, a);
                case Tile::k128Deep: return launch_kernel(loss_kernel<Gemm<128, 128, 2, 4, 4>, 128, 128, 2, 4>, grid, dim3(512), st, a);
                case Tile::kFew32: return launch_kernel(loss_kernel<Gemm<32, 64, 1, 4, 6>, 32, 64, 1, 4>, grid, dim3(256), st, a);
                default: return launch_kernel(loss_kernel<Gemm<64, 64, 1, 4, 4>, 64, 64, 1, 4>, grid, dim3(256), st, a);
            }
    });
}

template <typename T>
hy_status gradients(XentArgs& a, hipStream_t st) {
    const Tile tile = logit_tile_for<T>(a.g);
    return by_tile(a, tile, [&](dim3 grid) {
        if constexpr (T::kBytes == 4)
            switch (tile) {
                case Tile::kFew64: return launch_kernel(grad_kernel<T, GemmSplit<64, 64, 1, 4>, 64, 64, 1, 4>, grid, dim3(256), st, a);
                case Tile::kWide: return launch_kernel(grad_kernel<T, GemmSplit<128, 192, 2, 4>, 128, 192, 2, 4>, grid, dim3(512), st, a);
                default: return launch_kernel(grad_kernel<T, GemmSplit<128, 128, 2, 4>, 128, 128, 2, 4>, grid, dim3(512), st, a);
            }
        else
            switch (tile) {
                case Tile::kFew32: return launch_kernel(grad_kernel<T, Gemm<32, 64, 1, 4, 6>, 32, 64, 1, 4>, grid, dim3(256), st, a);
                case Tile::kFew64: return launch_kernel(grad_kernel<T, Gemm<64, 64, 1, 4, 4>, 64, 64, 1, 4>, grid, dim3(256), st, a);
                case Tile::k256: return launch_kernel(grad_kernel<T, Gemm<256, 256, 2, 4, 2>, 256, 256, 2, 4>, grid, dim3(512), st, a);
                case Tile::k128: return launch_kernel(grad_kernel<T, Gemm<128, 128, 2, 4, 2>, 128, 128, 2, 4>, grid, dim3(512), st, a);
                default: return launch_kernel(grad_kernel<T, Gemm<128, 128, 2, 4, 4>, 128, 128, 2, 4>, grid, dim3(512), st, a);
            }
    });
}

// Into how many shares a product's k is divided: where its tiles leave half of the compute units or more without work, as many as
// they hold, of at least 8 steps each (64 x 60000 x 256 bf16, dx in 16 shares or in up to 48: 112 us a training step or 83).
template <typename T, bool TB>
int32_t splits_for(const GemmArgs& g) {
    const Tile tile = product_tile_for<T, TB>(g);
    const Edges e = edges_of(tile);
    const int64_t tiles = cut(g.a.rows, e.rows) * cut(g.b.rows, e.cols), steps = g.K / (T::kBytes == 4 ? 32 : 64);
    const int64_t room = 256 * (tile == Tile::kFew64 ? 3 : tile == Tile::kAcross ? 2 : 1);  // workgroups that the chip holds
    if (2 * tiles > room || tile == Tile::k256) return 1;
    return (int32_t)std::max<int64_t>(1, std::min<int64_t>({room / tiles, steps / 8, room > 256 ? 48 : 16}));
}

// Whether dx is computed from W as it lies: fp32 always; bf16 where a turned copy would take longer than the product loses by
// operands that go through registers (a training step with and without the copy: 60 x 60000 x 4096 697 us and 478, 256 rows 885 and 684,
// 512 x 30000 x 4096 636 and 566, 1000 x 60000 x 1024 636 and 610; but 250 x 9000 x 2048 98 and 100, 250 x 1000 x 512 43 and 46).
template <typename T>
bool across(const XentShape& s) {
    return T::kBytes == 4 || s.N <= 128 || (s.N <= 1024 && s.V * s.D >= INT64_C(1) << 25);
}

// The two products of a piece of `cols` columns.  fp32: P lies turned where k runs over its rows.
template <typename T>
GemmArgs dw_product(const XentShape& s, const Layout& l, int64_t cols, const void* p = nullptr, const void* xt = nullptr) {
    if (T::kBytes == 4) return product_of(GemmOperand{p, up(cols, kGemmK), cols}, GemmOperand{xt, l.nt, s.D}, s.N);
    return product_of(GemmOperand{p, l.nt, cols}, GemmOperand{xt, l.nt, s.D}, up(s.N, 32));  // (what the tiles of P, of 32 rows at least, fill)
}
template <typename T>
GemmArgs dx_product(const XentShape& s, const Layout& l, int64_t cols, const void* p = nullptr, const void* w = nullptr) {
    const int64_t ld = up(cols, kGemmK);
    if (across<T>(s)) return product_of(GemmOperand{p, ld, s.N}, GemmOperand{w, l.ld, s.D}, cols);
    return product_of(GemmOperand{p, ld, s.N}, GemmOperand{w, ld, s.D}, ld);
}

template <typename T>
struct BwdSpace {
    uint16_t *x, *w;
    Bits<T> *xt, *wt, *p, *pt;
    float *sum, *split, *unit;
    BwdSpace(const XentShape& s, const Layout& l, Carver& c) {
        const int64_t piece = std::min(l.piece, s.V), ld = up(piece, kGemmK);
        x = l.packed ? c.take<uint16_t>(s.N * l.ld) : nullptr;
        w = l.packed ? c.take<uint16_t>(piece * l.ld) : nullptr;
        xt = c.take<Bits<T>>(s.D * l.nt);
        wt = !across<T>(s) ? c.take<Bits<T>>(s.D * ld) : nullptr;
        p = c.take<Bits<T>>(s.N * ld);
        pt = T::kBytes == 2 ? c.take<Bits<T>>(piece * l.nt) : nullptr;
        sum = l.pieces > 1 ? c.take<float>(s.N * s.D) : nullptr;
        int64_t most = 0;
        auto floats = [&](const GemmArgs& g, int32_t n) { return n > 1 ? n * g.a.rows * s.D : 0; };
        for (const int64_t cols : l.sizes) {
            const GemmArgs dw = dw_product<T>(s, l, cols), dx = dx_product<T>(s, l, cols);
            const int32_t dx_splits = across<T>(s) ? splits_for<T, true>(dx) : splits_for<T, false>(dx);
            most = std::max({most, floats(dw, splits_for<T, false>(dw)), floats(dx, dx_splits)});
        }
        split = c.take<float>(most);
        unit = c.take<float>(1);
    }
};

template <typename T, bool TA, bool TB>
hy_status product(XentArgs& a, float* split, hipStream_t st) {
    a.split = split;
    a.splits = splits_for<T, TB>(a.g);
    const Tile tile = product_tile_for<T, TB>(a.g);
    hy_status rc = by_tile(a, tile, [&](dim3 grid) {
        grid.x *= (uint32_t)a.splits;
        if constexpr (T::kBytes == 4)
            switch (tile) {
                case Tile::kFew64: return launch_kernel(product_kernel<T, GemmSplit<64, 64, 1, 4, TA, TB>, 64, 64, 1, 4>, grid, dim3(256), st, a);
                case Tile::kWide: return launch_kernel(product_kernel<T, GemmSplit<128, 192, 2, 4, TA, TB>, 128, 192, 2, 4>, grid, dim3(512), st, a);
                default: return launch_kernel(product_kernel<T, GemmSplit<128, 128, 2, 4, TA, TB>, 128, 128, 2, 4>, grid, dim3(512), st, a);
            }
        else if constexpr (TB)
            return launch_kernel(product_kernel<T, GemmAcross<128, 128, 2, 4>, 128, 128, 2, 4>, grid, dim3(512), st, a);
        else
            switch (tile) {
                case Tile::k256: return launch_kernel(product_kernel<T, Gemm<256, 256, 2, 4, 2>, 256, 256, 2, 4>, grid, dim3(512), st, a);
                case Tile::k128: return launch_kernel(product_kernel<T, Gemm<128, 128, 2, 4, 2>, 128, 128, 2, 4>, grid, dim3(512), st, a);
                default: return launch_kernel(product_kernel<T, Gemm<128, 128, 2, 4, 4>, 128, 128, 2, 4>, grid, dim3(512), st, a);
            }
    });
    if (rc != HY_OK || a.splits == 1) return rc;
    const int64_t lanes = a.g.a.rows * ((a.out_ld + 3) / 4);  // (of few tiles: far from the launch's limit)
    return launch_kernel(gather_kernel<T>, dim3((uint32_t)cut(lanes, 256)), dim3(256), st, a);
}

hy_status pack(const uint16_t* src, uint16_t* dst, int64_t rows, int64_t D, int64_t ld, hipStream_t st) {
    return launch_kernel(pack_kernel, dim3(workgroups_for(rows * ld, 256, 256)), dim3(256), st, src, dst, rows, D, ld);
}

template <typename T>
hy_status turn(const void* src, Bits<T>* dst, int64_t rows, int64_t D, int64_t ld, const int64_t* target, int64_t V, Unit unit,
               hipStream_t st) {
    return launch_kernel(turn_kernel<T>, dim3((uint32_t)cut(ld, 64), (uint32_t)(cut(D, 64) + (unit.unit ? 1 : 0))), dim3(256), st,
                         (const Bits<T>*)src, dst, rows, D, ld, target, V, unit);
}

// x, and the piece of W that begins at row v, as operands.
template <typename T>
hy_status operands(const XentPtrs& p, const XentShape& s, const Layout& l, uint16_t* x, uint16_t* w, int64_t v, GemmOperand* ox,
                   GemmOperand* ow, hipStream_t st) {
    const int64_t rows = std::min(l.piece, s.V - v);
    const char* piece = (const char*)p.w + v * s.D * T::kBytes;
    *ox = GemmOperand{l.packed ? x : p.x, l.ld, s.N};
    *ow = GemmOperand{l.packed ? (const void*)w : piece, l.ld, rows};
    if (!l.packed) return HY_OK;
    hy_status rc = v == 0 ? pack((const uint16_t*)p.x, x, s.N, s.D, l.ld, st) : HY_OK;
    if (rc == HY_OK) rc = pack((const uint16_t*)piece, w, rows, s.D, l.ld, st);
    return rc;
}

template <typename T>
hy_status forward(const XentPtrs& p, const XentShape& s, void* ws, hipStream_t st) {
    const Layout l = layout_of(s);
    Carver c(ws);
    FwdSpace f(s, l, c);
    XentArgs a{};
    a.target = p.target, a.V = s.V;
    a.part = f.part, a.zt = f.zt, a.tiles = f.tiles;
    if (few_rows(s)) {
        auto* const kernel = s.N <= 16 ? few_kernel<1> : few_kernel<2>;
        hy_status rc = launch_kernel(kernel, dim3((uint32_t)f.tiles), dim3(kFewWaves * kWave), st, (const float*)p.x, (const float*)p.w,
                                     p.target, f.part, f.zt, s.N, s.V, s.D, f.tiles);
        if (rc != HY_OK) return rc;
    } else {
        auto tiles = [&](int64_t cols) {
            const GemmArgs z = logits_of(s, l, cols);
            return cut(cols, edges_of(logit_tile_for<T>(z)).cols);
        };
        a.tiles = (l.pieces - 1) * tiles(l.sizes[0]) + tiles(l.sizes[1]);
        for (int64_t v = 0; v < s.V; v += l.piece) {
            a.g = logits_of(s, l, std::min(l.piece, s.V - v));
            hy_status rc = operands<T>(p, s, l, f.x, f.w, v, &a.g.a, &a.g.b, st);
            a.v0 = v;
            if (rc == HY_OK) rc = losses<T>(a, st);
            if (rc != HY_OK) return rc;
            a.tile0 += a.g.nt;
        }
    }
    return launch_kernel(join_kernel, dim3((uint32_t)cut(s.N, 4)), dim3(256), st, (const float2*)f.part, (const float*)f.zt, p.target,
                         p.loss, p.lse, s.N, a.tiles, s.V);
}

template <typename T>
hy_status backward(const XentPtrs& p, const XentShape& s, void* ws, hipStream_t st) {
    const Layout l = layout_of(s);
    Carver c(ws);
    BwdSpace<T> b(s, l, c);
    const float* unit = T::kBytes == 2 ? b.unit : nullptr;
    hy_status rc = turn<T>(p.x, b.xt, s.N, s.D, l.nt, p.target, s.V, Unit{p.dloss, T::kBytes == 2 ? b.unit : nullptr}, st);
    for (int64_t v = 0; rc == HY_OK && v < s.V; v += l.piece) {
        const int64_t cols = std::min(l.piece, s.V - v), ld = up(cols, kGemmK);
        constexpr bool kTurned = T::kBytes == 4;
        XentArgs a{};
        a.g.K = (int32_t)(l.packed ? l.ld : s.D);
        rc = operands<T>(p, s, l, b.x, b.w, v, &a.g.a, &a.g.b, st);
        const GemmOperand words = a.g.b;
        if (rc == HY_OK && !across<T>(s)) rc = turn<T>((const char*)p.w + v * s.D * T::kBytes, b.wt, cols, s.D, ld, nullptr, 0, Unit{}, st);
        a.target = p.target, a.V = s.V, a.v0 = v;
        a.lse = p.lse_in, a.dloss = p.dloss, a.unit = unit;
        a.p = b.p, a.p_ld = ld;
        a.pt = b.pt, a.pt_ld = l.nt;
        if (rc == HY_OK) rc = gradients<T>(a, st);
        XentArgs dw{};
        dw.g = dw_product<T>(s, l, cols, kTurned ? b.p : b.pt, b.xt);
        dw.out = (char*)p.dw + v * s.D * T::kBytes, dw.out_ld = s.D, dw.first = dw.last = true, dw.unit = unit;
        if (rc == HY_OK) rc = product<T, kTurned, false>(dw, b.split, st);
        XentArgs dx{};
        dx.g = dx_product<T>(s, l, cols, b.p, across<T>(s) ? words.p : b.wt);
        dx.out = (char*)p.dx, dx.out_ld = s.D, dx.sum = b.sum, dx.first = v == 0, dx.last = v + l.piece >= s.V, dx.unit = unit;
        dx.target = p.target, dx.V = s.V;
        if (rc == HY_OK) rc = across<T>(s) ? product<T, false, true>(dx, b.split, st) : product<T, false, T::kBytes == 4>(dx, b.split, st);
    }
    return rc;
}

// Row distances that a lane's 32-bit offsets within a tile reach, and a workgroup for every tile of every product of a piece (the
// last one may be narrower, and take other tiles).
template <typename T>
bool served_as(const XentShape& s, const Layout& l, bool backward) {
    for (const int64_t cols : l.sizes) {
        const GemmArgs z = logits_of(s, l, cols);
        if (!launchable(z, logit_tile_for<T>(z))) return false;
        if (!backward) continue;
        const GemmArgs dw = dw_product<T>(s, l, cols), dx = dx_product<T>(s, l, cols);
        if (!launchable(dw, product_tile_for<T, false>(dw))) return false;
        if (!launchable(dx, across<T>(s) ? product_tile_for<T, true>(dx) : product_tile_for<T, false>(dx))) return false;
    }
    return true;
}

}  // namespace

bool xent_served(const XentShape& s, bool backward) {
    constexpr int64_t kMost = 64 * 65533;  // (a row of workgroups more in turn_kernel's grid)
    if (s.N > kMost || s.D > kMost) return false;
    const Layout l = layout_of(s);
    return s.dtype == HY_F32 ? served_as<F32>(s, l, backward) : served_as<BF16>(s, l, backward);
}

int64_t xent_fwd_workspace_bytes(const XentShape& s) {
    const Layout l = layout_of(s);
    Carver c(nullptr);
    FwdSpace f(s, l, c);
    return (int64_t)c.at;
}

int64_t xent_bwd_workspace_bytes(const XentShape& s) {
    const Layout l = layout_of(s);
    Carver c(nullptr);
    if (s.dtype == HY_F32) BwdSpace<F32>(s, l, c);
    else BwdSpace<BF16>(s, l, c);
    return (int64_t)c.at;
}

hy_status launch_xent_fwd(const XentPtrs& p, const XentShape& s, void* ws, hipStream_t st) {
    return s.dtype == HY_F32 ? forward<F32>(p, s, ws, st) : forward<BF16>(p, s, ws, st);
}

hy_status launch_xent_bwd(const XentPtrs& p, const XentShape& s, void* ws, hipStream_t st) {
    if (s.N == 0) {  // no rows: nothing but zeros for the weights
        const int64_t bytes = s.V * s.D * (s.dtype == HY_F32 ? 4 : 2);
        return launch_kernel(zero_kernel, dim3(workgroups_for(bytes, 512, 256)), dim3(256), st, (char*)p.dw, bytes);
    }
    return s.dtype == HY_F32 ? backward<F32>(p, s, ws, st) : backward<BF16>(p, s, ws, st);
}

}  // namespace hy
