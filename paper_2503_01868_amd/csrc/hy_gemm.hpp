// Matrix products C[m][n] = sum_k A[m][k] B[n][k] on the matrix cores with fp32 sums: of bf16 numbers with k contiguous in both (Gemm) or
// with B k after k (GemmAcross), and of fp32 numbers in three bf16 parts each (GemmSplit).
#pragma once
#include <type_traits>

#include "hy_common.hpp"

namespace hy {

constexpr int kGemmK = 64;        // every operand made here has rows of a multiple

// Rows of bf16 numbers (Gemm) or of fp32 numbers (GemmSplit).
struct GemmOperand {
    const void* p;
    int64_t ld;          // elements between rows (between k's, where the operand lies turned)
    int64_t rows;
};

struct GemmArgs {
    GemmOperand a, b;
    int32_t K;           // what is behind a row's K numbers counts as zeros.  bf16: a multiple of 8, and rows begin where 16 bytes do
    int32_t mt, nt;      // tiles
};

__device__ uint4 gemm_zeros;  // (where the loads behind a tail go)

typedef __attribute__((address_space(3))) void* lds_ptr_t;
typedef const __attribute__((address_space(1))) void* global_ptr_t;

// A workgroup of MW x NW waves computes BM x BN; a wave BM / MW x BN / NW in 16 x 16 pieces.  Lane (li = lane % 16, lq =
// lane / 16) of a wave holds in acc[i][j][r] the sum of row 16 i + li and column 16 j + 4 lq + r of its part.
//
// STAGES steps of both tiles are in LDS or on their way there, straight from memory.  A step is two halves of 32 k: while the
// matrix cores work on one half, in registers, the other is read from LDS; the one barrier of a step says that the next step
// has arrived and that nobody reads this one any more.
template <int BM, int BN, int MW, int NW, int STAGES>
struct Gemm {
    static constexpr int kStep = 64;  // k of a step: 128 bytes of a row
    static constexpr int kWaves = MW * NW, kThreads = kWaves * kWave;
    static constexpr int WM = BM / MW, WN = BN / NW, MI = WM / 16, NI = WN / 16;
    static constexpr int kRowBytes = kStep * 2;
    static constexpr int kBytes = (BM + BN) * kRowBytes;  // of one step's tiles
    static constexpr int kLds = STAGES * kBytes;
    static constexpr int AL = BM * 8 / kThreads, BL = BN * 8 / kThreads;  // 16-byte pieces of a lane

    f32x4_t acc[MI][NI];

    // Rows of 128 bytes in LDS, the 16-byte pieces of row r at r * 128 + (piece ^ (r % 8)) * 16: the 16 lanes that read one
    // piece of 16 rows spread over all banks.  A wave's load fills 8 rows, so lane l fetches piece (l % 8) ^ (l / 8).
    // Steps [first, last).
    __device__ __forceinline__ void run(char* lds, const GemmArgs& g, int64_t m0, int64_t n0, int first, int last) {
        const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
        const int li = lane % 16, lq = lane / 16;
        uint32_t ao[AL], bo[BL];
        auto offset = [&](int i, int64_t first_row, const GemmOperand& x) {
            int64_t r = (i * kWaves + w) * 8 + lane / 8;
            if (first_row + r >= x.rows) r = x.rows - 1 - first_row;  // rows that do not exist: the last one again
            return (uint32_t)((r * x.ld + ((lane % 8) ^ (lane / 8)) * 8) * 2);
        };
#pragma unroll
        for (int i = 0; i < AL; ++i) ao[i] = offset(i, m0, g.a);
#pragma unroll
        for (int i = 0; i < BL; ++i) bo[i] = offset(i, n0, g.b);
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[i][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};

        const char *abase = (const char*)g.a.p + m0 * g.a.ld * 2, *bbase = (const char*)g.b.p + n0 * g.b.ld * 2;
        const int total = last - first, tail = g.K % kStep;
        int k = first;
        auto fetch = [&](int stage) {
            char* to = lds + stage * kBytes + w * 1024;
            const char *pa = abase + k * (kStep * 2), *pb = bbase + k * (kStep * 2);
            ++k;
            if (tail > 0 && k * kStep > g.K) {
                const bool beyond = ((lane % 8) ^ (lane / 8)) * 8 >= tail;
                const char* none = reinterpret_cast<const char*>(&gemm_zeros);
#pragma unroll
                for (int i = 0; i < AL; ++i)
                    __builtin_amdgcn_global_load_lds((global_ptr_t)(beyond ? none : pa + ao[i]), (lds_ptr_t)(to + i * kWaves * 1024), 16, 0, 0);
#pragma unroll
                for (int i = 0; i < BL; ++i)
                    __builtin_amdgcn_global_load_lds((global_ptr_t)(beyond ? none : pb + bo[i]),
                                                     (lds_ptr_t)(to + BM * kRowBytes + i * kWaves * 1024), 16, 0, 0);
                return;
            }
#pragma unroll
            for (int i = 0; i < AL; ++i)
                __builtin_amdgcn_global_load_lds((global_ptr_t)(pa + ao[i]), (lds_ptr_t)(to + i * kWaves * 1024), 16, 0, 0);
#pragma unroll
            for (int i = 0; i < BL; ++i)
                __builtin_amdgcn_global_load_lds((global_ptr_t)(pb + bo[i]), (lds_ptr_t)(to + BM * kRowBytes + i * kWaves * 1024), 16, 0, 0);
        };
        const int wm = w % MW, wn = w / MW;
        const char *ra = lds + (wm * WM + li) * kRowBytes, *rb = lds + (BM + wn * WN + li) * kRowBytes;
        const int piece[2] = {(lq ^ (li % 8)) * 16, ((4 + lq) ^ (li % 8)) * 16};
        struct Half {
            bf16x8_t a[MI], b[NI];
        };
        auto read = [&](Half& h, int stage, int half) {
            const int at = stage * kBytes + piece[half];
#pragma unroll
            for (int j = 0; j < NI; ++j) h.b[j] = *reinterpret_cast<const bf16x8_t*>(rb + at + j * 16 * kRowBytes);
#pragma unroll
            for (int i = 0; i < MI; ++i) h.a[i] = *reinterpret_cast<const bf16x8_t*>(ra + at + i * 16 * kRowBytes);
        };
        auto multiply = [&](const Half& h) {
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(h.b[j], h.a[i], acc[i][j], 0, 0, 0);
        };
        // Waits until all but the newest `steps` steps' loads of this wave have arrived and everything it reads from LDS has,
        // then for the other waves.  (s_waitcnt: vmcnt in bits 0-3 and 14-15, lgkmcnt 0 in bits 8-11)
        constexpr int kLoads = AL + BL;
        auto meet = [&](auto steps) {
            constexpr int n = decltype(steps)::value * kLoads;
            static_assert(n < 64, "vmcnt");
            __builtin_amdgcn_s_waitcnt((n & 15) | n >> 4 << 14 | 0x0070);
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
        Half h0, h1;
#pragma unroll
        for (int x = 0; x < STAGES; ++x)
            if (x < total) fetch(x);
        if (total >= STAGES) meet(std::integral_constant<int, STAGES - 1>{});
        else meet(std::integral_constant<int, 0>{});
        read(h0, 0, 0);
        int stage = 0;
        // The order of a half's instructions: a read from LDS (and, with them, a load into it) behind every few products, so
        // that neither waits for the other.  Masks: 8 products, 0x100 reads from LDS, 0x20 loads.
        auto weave = [&](auto loads) {
            constexpr int kReads = MI + NI, kProducts = MI * NI, kEach = kProducts / kReads;
#pragma unroll
            for (int x = 0; x < kReads; ++x) {
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                if constexpr (decltype(loads)::value) __builtin_amdgcn_sched_group_barrier(0x20, (kLoads + kReads - 1) / kReads, 0);
                __builtin_amdgcn_sched_group_barrier(8, kEach, 0);
            }
            __builtin_amdgcn_sched_group_barrier(8, kProducts - kEach * kReads, 0);
        };
        auto first_half = [&] {
            // h0 has had a whole multiply to arrive; said here, or the compiler waits for h1 too before it uses h0
            __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
            asm volatile("" ::: "memory");
            read(h1, stage, 1);
            multiply(h0);
            weave(std::false_type{});
            __builtin_amdgcn_sched_barrier(0);
        };
        auto second_half = [&](auto more) {
            const int next = stage == STAGES - 1 ? 0 : stage + 1;
            if constexpr (decltype(more)::value) fetch(stage);
            read(h0, next, 0);
            multiply(h1);
            weave(more);
            __builtin_amdgcn_sched_barrier(0);
            stage = next;
        };
        int t = 0;
        for (; t + STAGES < total; ++t) {
            first_half();
            meet(std::integral_constant<int, STAGES - 2>{});
            second_half(std::true_type{});
        }
        for (; t + 1 < total; ++t) {  // the last steps: nothing more to fetch
            first_half();
            meet(std::integral_constant<int, 0>{});
            second_half(std::false_type{});
        }
        first_half();
        multiply(h1);
    }
};

// The parts of an fp32 number, each in the upper half of a word: cut, not rounded, so that no part overflows.  All of an infinity
// is in the first part; a NaN is one in the second.  (An infinity meets the lower parts of the other factor too, and makes NaN where
// one of them is zero, that is, where 16 bits hold the factor.)
__device__ __forceinline__ void parts_of(float x, uint32_t (&part)[3]) {
    constexpr int kInfinite = 0x204;  // of either sign
    part[0] = __float_as_uint(x);
    const float head = __uint_as_float(part[0] & 0xffff0000u);
    const float rest = __builtin_amdgcn_classf(x, kInfinite) ? 0.0f : x - head;
    part[1] = __float_as_uint(rest);
    part[2] = __float_as_uint(rest - __uint_as_float(part[1] & 0xffff0000u));
}
// Eight of them as operands of a product.
__device__ __forceinline__ void parts_of(const float4 (&w)[2], uint4 (&f)[3]) {
    const float v[8] = {w[0].x, w[0].y, w[0].z, w[0].w, w[1].x, w[1].y, w[1].z, w[1].w};
    uint32_t o[4][3];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t a[3], b[3];
        parts_of(v[2 * i], a);
        parts_of(v[2 * i + 1], b);
#pragma unroll
        for (int x = 0; x < 3; ++x) o[i][x] = __builtin_amdgcn_perm(b[x], a[x], 0x07060302);  // the upper halves
    }
#pragma unroll
    for (int x = 0; x < 3; ++x) f[x] = make_uint4(o[0][x], o[1][x], o[2][x], o[3][x]);
}
// The products of parts that reach an fp32 product's 24 bits, the smallest first: the parts of one factor and of the other.
constexpr int kSplitProducts = 6;
constexpr int kSplitA[kSplitProducts] = {2, 0, 1, 1, 0, 0}, kSplitB[kSplitProducts] = {0, 2, 1, 0, 1, 0};

// The same for fp32 operands, to fp32's precision: a number is three bf16 numbers (8 bits each, the head, the middle and the
// tail of the 24), and a product the sum of six products of parts.  Numbers become parts once, between memory and LDS: a step's
// are fetched into registers two steps ahead and written to LDS as three planes of 64-byte rows (the 16-byte pieces of row r at
// piece ^ (r / 2 % 4)) one step ahead.  A part that is in a register serves two or three of the six products, so LDS is read half
// as often as for six products of planes.  An operand may lie turned in memory, k after k (TA, TB: its `rows` are then how many
// numbers it has for each k, and k's are `ld` apart): eight loads of a number each, neighbours in a wave, make a piece.
// 4000 x 8000 x 1024: 1.45 ms for the four products of a training step, 1.08 PFLOP/s of parts; the splitting takes as many issue
// slots as the products do.
template <int BM, int BN, int MW, int NW, bool TA = false, bool TB = false>
struct GemmSplit {
    static constexpr int kStep = 32;
    static constexpr int kWaves = MW * NW, kThreads = kWaves * kWave;
    static constexpr int WM = BM / MW, WN = BN / NW, MI = WM / 16, NI = WN / 16;
    static constexpr int kPlane = (BM + BN) * kStep * 2, kBytes = 3 * kPlane, kLds = 2 * kBytes;
    static constexpr int kPieces = ((BM + BN) * 4 + kThreads - 1) / kThreads;  // of 8 numbers, of a lane
    static constexpr int kPiecesA = BM * 4 / kThreads;
    static_assert(kPiecesA * kThreads == BM * 4 && BM % kWave == 0 && BN % kWave == 0, "a lane's pieces, and a wave's, are of one operand");

    f32x4_t acc[MI][NI];

    __device__ __forceinline__ void run(char* lds, const GemmArgs& g, int64_t m0, int64_t n0, int first, int last) {
        const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
        const int li = lane % 16, lq = lane / 16, wm = w % MW, wn = w / MW;
        const float* from[kPieces];  // the lane's row; of a turned operand, its beginning
        int to[kPieces], at[kPieces], row_at[kPieces];
#pragma unroll
        for (int x = 0; x < kPieces; ++x) {
            const bool b = x >= kPiecesA, turned = b ? TB : TA;
            const int edge = b ? BN : BM;
            int i = (x - (b ? kPiecesA : 0)) * kThreads + w * kWave;
            if (i >= edge * 4) i -= kThreads;  // none is left: those of the lane's last piece again
            const int row = turned ? i % edge + lane : (i + lane) / 4, piece = turned ? i / edge : lane % 4;
            const GemmOperand& o = b ? g.b : g.a;
            int64_t r = (b ? n0 : m0) + row;
            if (r >= o.rows) r = o.rows - 1;  // rows that do not exist: the last one again
            from[x] = static_cast<const float*>(o.p) + (turned ? 0 : r * o.ld);
            row_at[x] = (int)r;
            at[x] = piece * 8;
            to[x] = ((b ? BM : 0) + row) * (kStep * 2) + (piece ^ (row / 2 % 4)) * 16;
        }
        const bool fours = (TA || (g.a.ld % 4 == 0 && ((uintptr_t)g.a.p & 15) == 0)) &&
                           (TB || (g.b.ld % 4 == 0 && ((uintptr_t)g.b.p & 15) == 0));
        auto fetch = [&](float4 (&v)[kPieces][2], int step) {
            const bool whole = (step + 1) * kStep <= g.K;
            auto some = [&](auto full, auto wide) {
#pragma unroll
                for (int x = 0; x < kPieces; ++x) {
                    const int k0 = step * kStep + at[x];
                    float f[8];
                    if (x >= kPiecesA ? TB : TA) {
                        const int64_t ld = x >= kPiecesA ? g.b.ld : g.a.ld;
                        const float* const row = from[x] + k0 * ld;
#pragma unroll
                        for (int j = 0; j < 8; ++j) f[j] = full || k0 + j < g.K ? (row + j * ld)[row_at[x]] : 0.0f;
                    } else if (wide) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) v[x][h] = *reinterpret_cast<const float4*>(from[x] + k0 + 4 * h);
                        continue;
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j) f[j] = full || k0 + j < g.K ? from[x][k0 + j] : 0.0f;
                    }
                    v[x][0] = make_float4(f[0], f[1], f[2], f[3]);
                    v[x][1] = make_float4(f[4], f[5], f[6], f[7]);
                }
            };
            if (whole && fours) some(std::true_type{}, std::true_type{});
            else some(std::false_type{}, std::false_type{});
        };
        auto put = [&](const float4 (&v)[kPieces][2], int stage) {
#pragma unroll
            for (int x = 0; x < kPieces; ++x) {
                uint4 f[3];
                parts_of(v[x], f);
#pragma unroll
                for (int y = 0; y < 3; ++y) *reinterpret_cast<uint4*>(lds + stage * kBytes + y * kPlane + to[x]) = f[y];
            }
        };
        auto meet = [&] {  // what the waves have written to LDS is there; loads into registers stay on their way
            __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[i][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        const int piece = (lq ^ (li / 2 % 4)) * 16;
        const char *ra = lds + (wm * WM + li) * (kStep * 2) + piece, *rb = lds + (BM + wn * WN + li) * (kStep * 2) + piece;
        float4 v0[kPieces][2], v1[kPieces][2];
        fetch(v0, first);
        put(v0, 0);
        fetch(v0, first + 1);  // (behind K: zeros)
        meet();
        auto step = [&](int t, float4 (&next)[kPieces][2], float4 (&after)[kPieces][2]) {
            const int stage = (t - first) % 2;
            fetch(after, t + 2 < last ? t + 2 : last - 1);
            bf16x8_t fa[3][MI], fb[3][NI];
            auto read = [&](int pa, int pb) {
#pragma unroll
                for (int j = 0; j < NI; ++j) fb[pb][j] = *reinterpret_cast<const bf16x8_t*>(rb + stage * kBytes + pb * kPlane + j * 16 * kStep * 2);
#pragma unroll
                for (int i = 0; i < MI; ++i) fa[pa][i] = *reinterpret_cast<const bf16x8_t*>(ra + stage * kBytes + pa * kPlane + i * 16 * kStep * 2);
            };
            read(2, 0);  // in the order of their use
            read(0, 2);
            read(1, 1);
            put(next, stage ^ 1);  // (behind the last step: nobody reads it)
#pragma unroll
            for (int y = 0; y < kSplitProducts; ++y)
#pragma unroll
                for (int i = 0; i < MI; ++i)
#pragma unroll
                    for (int j = 0; j < NI; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[kSplitB[y]][j], fa[kSplitA[y]][i], acc[i][j], 0, 0, 0);
            // the parts are made between the products
            __builtin_amdgcn_sched_group_barrier(0x100, 3 * (MI + NI), 0);
#pragma unroll
            for (int y = 0; y < kSplitProducts * MI * NI; ++y) {
                __builtin_amdgcn_sched_group_barrier(8, 1, 0);
                __builtin_amdgcn_sched_group_barrier(2, 3, 0);
            }
            meet();
        };
        int t = first;
        for (; t + 1 < last; t += 2) {
            step(t, v0, v1);
            step(t + 1, v1, v0);
        }
        if (t < last) step(t, v0, v1);
    }
};

// The same of bf16 operands where B lies turned in memory, k after k (its `rows` are how many numbers it has for each k, an even
// distance `ld` apart from an address of a word): for few rows of A, where a turned copy would cost as much as the product.  Both
// go through registers, a step of 64 k at a time and two steps ahead; a lane takes two columns of 8 k, a word each, and puts them
// together.  LDS rows are Gemm's.  dx of 60 rows against 60000 symbols of width 4096, 491 MB of W: 139 us (3.5 TB/s; a turned copy
// alone 195).
template <int BM, int BN, int MW, int NW>
struct GemmAcross {
    static constexpr int kStep = 64;
    static constexpr int kWaves = MW * NW, kThreads = kWaves * kWave;
    static constexpr int WM = BM / MW, WN = BN / NW, MI = WM / 16, NI = WN / 16;
    static constexpr int kRowBytes = kStep * 2, kBytes = (BM + BN) * kRowBytes, kLds = 2 * kBytes;
    static constexpr int AL = BM * 8 / kThreads, BL = 8 / kWaves;  // pieces of 8 k of a lane: of a row; of two columns
    static_assert(AL * kThreads == BM * 8 && BL * kWaves == 8 && BN == 2 * kWave, "whole pieces, and a wave's are of the same 8 k");

    f32x4_t acc[MI][NI];

    struct Held {
        u32x4_t a[AL];
        uint32_t b[BL][8];
    };

    __device__ __forceinline__ void run(char* lds, const GemmArgs& g, int64_t m0, int64_t n0, int first, int last) {
        const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
        const int li = lane % 16, lq = lane / 16, wm = w % MW, wn = w / MW;
        const uint16_t* a_from[AL];
        int a_to[AL];
#pragma unroll
        for (int x = 0; x < AL; ++x) {
            const int i = x * kThreads + (int)threadIdx.x, row = i / 8, piece = i % 8;
            const int64_t r = m0 + row < g.a.rows ? m0 + row : g.a.rows - 1;  // rows that do not exist: the last one again
            a_from[x] = static_cast<const uint16_t*>(g.a.p) + r * g.a.ld + piece * 8;
            a_to[x] = row * kRowBytes + (piece ^ (row % 8)) * 16;
        }
        const int64_t pairs = (g.b.rows + 1) / 2, pair = n0 / 2 + lane;
        const uint32_t b_at = (uint32_t)(pair < pairs ? pair : pairs - 1);
        const int b_to = (BM + 2 * lane) * kRowBytes, b_row = 2 * lane % 8;
        auto fetch = [&](Held& h, int step) {
#pragma unroll
            for (int x = 0; x < AL; ++x) h.a[x] = *reinterpret_cast<const u32x4_t*>(a_from[x] + (int64_t)step * kStep);
            const char* const base = static_cast<const char*>(g.b.p) + (int64_t)step * kStep * g.b.ld * 2;
            const bool whole = (step + 1) * kStep <= g.K;
#pragma unroll
            for (int x = 0; x < BL; ++x)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int k = (x * kWaves + w) * 8 + j;
                    h.b[x][j] = whole || step * kStep + k < g.K ? reinterpret_cast<const uint32_t*>(base + k * g.b.ld * 2)[b_at] : 0u;
                }
        };
        auto put = [&](const Held& h, int stage) {
            char* const to = lds + stage * kBytes;
#pragma unroll
            for (int x = 0; x < AL; ++x) *reinterpret_cast<u32x4_t*>(to + a_to[x]) = h.a[x];
#pragma unroll
            for (int x = 0; x < BL; ++x)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t v[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = __builtin_amdgcn_perm(h.b[x][2 * j + 1], h.b[x][2 * j], c ? 0x07060302 : 0x05040100);
                    *reinterpret_cast<uint4*>(to + b_to + c * kRowBytes + ((x * kWaves + w) ^ (b_row + c)) * 16) = make_uint4(v[0], v[1], v[2], v[3]);
                }
        };
        auto meet = [&] {  // what the waves have written to LDS is there; loads into registers stay on their way
            __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[i][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        const char *ra = lds + (wm * WM + li) * kRowBytes, *rb = lds + (BM + wn * WN + li) * kRowBytes;
        Held h0, h1;
        fetch(h0, first);
        put(h0, 0);
        fetch(h0, first + 1 < last ? first + 1 : first);
        meet();
        auto step = [&](int t, Held& next, Held& after) {
            const int stage = (t - first) % 2;
            fetch(after, t + 2 < last ? t + 2 : last - 1);
            bf16x8_t fa[2][MI], fb[2][NI];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int piece = ((4 * h + lq) ^ (li % 8)) * 16 + stage * kBytes;
#pragma unroll
                for (int j = 0; j < NI; ++j) fb[h][j] = *reinterpret_cast<const bf16x8_t*>(rb + j * 16 * kRowBytes + piece);
#pragma unroll
                for (int i = 0; i < MI; ++i) fa[h][i] = *reinterpret_cast<const bf16x8_t*>(ra + i * 16 * kRowBytes + piece);
            }
            put(next, stage ^ 1);  // (behind the last step: nobody reads it)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < MI; ++i)
#pragma unroll
                    for (int j = 0; j < NI; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[h][j], fa[h][i], acc[i][j], 0, 0, 0);
            meet();
        };
        int t = first;
        for (; t + 1 < last; t += 2) {
            step(t, h0, h1);
            step(t + 1, h1, h0);
        }
        if (t < last) step(t, h0, h1);
    }
};

}  // namespace hy
