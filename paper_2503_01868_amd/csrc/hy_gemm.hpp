// Matrix products C[m][n] = sum_k A[m][k] B[n][k] on bf16 matrix cores with fp32 sums: both operands have k contiguous.
#pragma once
#include <type_traits>

#include "hy_common.hpp"

namespace hy {

constexpr int kGemmK = 64;        // k per step: 128 bytes of a row

// A matrix of bf16 rows; fp32 values are three planes (head, middle and tail bits).
struct GemmOperand {
    const uint16_t* p;
    int64_t ld, plane;   // elements between rows and between planes
    int64_t rows;
};

// One product: the sum over `segments` pairs of planes of products over K (a multiple of kGemmK).  tail > 0: the rows hold only
// K - kGemmK + tail numbers, a multiple of 8, and what is behind them counts as zeros.
struct GemmArgs {
    GemmOperand a, b;
    int32_t K, segments, tail;
    uint32_t aplanes, bplanes;  // the planes of segment i in bits 4 i .. 4 i + 3
    int32_t mt, nt;             // tiles
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
    static constexpr int kWaves = MW * NW, kThreads = kWaves * kWave;
    static constexpr int WM = BM / MW, WN = BN / NW, MI = WM / 16, NI = WN / 16;
    static constexpr int kRowBytes = kGemmK * 2;
    static constexpr int kBytes = (BM + BN) * kRowBytes;  // of one step's tiles
    static constexpr int kLds = STAGES * kBytes;
    static constexpr int AL = BM * 8 / kThreads, BL = BN * 8 / kThreads;  // 16-byte pieces of a lane

    f32x4_t acc[MI][NI];

    // Rows of 128 bytes in LDS, the 16-byte pieces of row r at r * 128 + (piece ^ (r % 8)) * 16: the 16 lanes that read one
    // piece of 16 rows spread over all banks.  A wave's load fills 8 rows, so lane l fetches piece (l % 8) ^ (l / 8).
    // Steps [first, last) of all segments' steps.
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

        const char *abase = (const char*)(g.a.p + m0 * g.a.ld), *bbase = (const char*)(g.b.p + n0 * g.b.ld);
        const int steps = g.K / kGemmK, total = last - first;
        int seg = first / steps, k = first - seg * steps;
        auto fetch = [&](int stage) {
            char* to = lds + stage * kBytes + w * 1024;
            const char* pa = abase + ((g.aplanes >> 4 * seg & 15) * g.a.plane + k * kGemmK) * 2;
            const char* pb = bbase + ((g.bplanes >> 4 * seg & 15) * g.b.plane + k * kGemmK) * 2;
            if (g.tail > 0 && k == steps - 1) {
                const bool beyond = ((lane % 8) ^ (lane / 8)) * 8 >= g.tail;
                const char* none = reinterpret_cast<const char*>(&gemm_zeros);
#pragma unroll
                for (int i = 0; i < AL; ++i)
                    __builtin_amdgcn_global_load_lds((global_ptr_t)(beyond ? none : pa + ao[i]), (lds_ptr_t)(to + i * kWaves * 1024), 16, 0, 0);
#pragma unroll
                for (int i = 0; i < BL; ++i)
                    __builtin_amdgcn_global_load_lds((global_ptr_t)(beyond ? none : pb + bo[i]),
                                                     (lds_ptr_t)(to + BM * kRowBytes + i * kWaves * 1024), 16, 0, 0);
                k = 0, ++seg;
                return;
            }
#pragma unroll
            for (int i = 0; i < AL; ++i)
                __builtin_amdgcn_global_load_lds((global_ptr_t)(pa + ao[i]), (lds_ptr_t)(to + i * kWaves * 1024), 16, 0, 0);
#pragma unroll
            for (int i = 0; i < BL; ++i)
                __builtin_amdgcn_global_load_lds((global_ptr_t)(pb + bo[i]), (lds_ptr_t)(to + BM * kRowBytes + i * kWaves * 1024), 16, 0, 0);
            if (++k == steps) k = 0, ++seg;
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

}  // namespace hy
