// Matrix products C[m][n] = sum_k A[m][k] B[n][k] on bf16 matrix cores with fp32 sums: both operands have k contiguous.
#pragma once
#include "hy_common.hpp"

namespace hy {

constexpr int kGemmK = 64;        // k per step: 128 bytes of a row

// A matrix of bf16 rows; fp32 values are three planes (head, middle and tail bits).
struct GemmOperand {
    const uint16_t* p;
    int64_t ld, plane;   // elements between rows and between planes
    int64_t rows;
};

// One product: the sum over `segments` pairs of planes of products over K (a multiple of kGemmK).
struct GemmArgs {
    GemmOperand a, b;
    int32_t K, segments;
    uint32_t aplanes, bplanes;  // the planes of segment i in bits 4 i .. 4 i + 3
    int32_t mt, nt;             // tiles
};

typedef __attribute__((address_space(3))) void* lds_ptr_t;
typedef const __attribute__((address_space(1))) void* global_ptr_t;

// A workgroup of MW x NW waves computes BM x BN; a wave BM / MW x BN / NW in 16 x 16 pieces.  Lane (li = lane % 16, lq =
// lane / 16) of a wave holds in acc[i][j][r] the sum of row 16 i + li and column 16 j + 4 lq + r of its part.
template <int BM, int BN, int MW, int NW>
struct Gemm {
    static constexpr int kWaves = MW * NW, kThreads = kWaves * kWave;
    static constexpr int WM = BM / MW, WN = BN / NW, MI = WM / 16, NI = WN / 16;
    static constexpr int kRowBytes = kGemmK * 2;
    static constexpr int kBytes = (BM + BN) * kRowBytes;  // of one step's tiles
    static constexpr int AL = BM * 8 / kThreads, BL = BN * 8 / kThreads;  // 16-byte pieces of a lane

    f32x4_t acc[MI][NI];

    // Rows of 128 bytes in LDS, the 16-byte pieces of row r at r * 128 + (piece ^ (r % 8)) * 16: the 16 lanes that read one
    // piece of 16 rows spread over all banks.  A wave's load fills 8 rows, so lane l fetches piece (l % 8) ^ (l / 8).
    __device__ __forceinline__ void run(char* lds, const GemmArgs& g, int64_t m0, int64_t n0) {
        const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
        const int li = lane % 16, lq = lane / 16;
        uint32_t ao[AL], bo[BL];
        auto offset = [&](int i, int64_t first, const GemmOperand& x) {
            int64_t r = (i * kWaves + w) * 8 + lane / 8;
            if (first + r >= x.rows) r = x.rows - 1 - first;  // rows that do not exist: the last one again
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
        const int steps = g.K / kGemmK, total = steps * g.segments;
        int seg = 0, k = 0;
        auto fetch = [&](char* to) {
            const char* pa = abase + ((g.aplanes >> 4 * seg & 15) * g.a.plane + k * kGemmK) * 2;
            const char* pb = bbase + ((g.bplanes >> 4 * seg & 15) * g.b.plane + k * kGemmK) * 2;
#pragma unroll
            for (int i = 0; i < AL; ++i)
                __builtin_amdgcn_global_load_lds((global_ptr_t)(pa + ao[i]), (lds_ptr_t)(to + (i * kWaves + w) * 1024), 16, 0, 0);
#pragma unroll
            for (int i = 0; i < BL; ++i)
                __builtin_amdgcn_global_load_lds((global_ptr_t)(pb + bo[i]), (lds_ptr_t)(to + BM * kRowBytes + (i * kWaves + w) * 1024),
                                                 16, 0, 0);
            if (++k == steps) k = 0, ++seg;
        };
        const int wm = w % MW, wn = w / MW;
        const int ra = (wm * WM + li) * kRowBytes, rb = BM * kRowBytes + (wn * WN + li) * kRowBytes;
        auto multiply = [&](const char* from) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int piece = ((s * 4 + lq) ^ (li % 8)) * 16;
                bf16x8_t fa[MI], fb[NI];
#pragma unroll
                for (int j = 0; j < NI; ++j) fb[j] = *reinterpret_cast<const bf16x8_t*>(from + rb + j * 16 * kRowBytes + piece);
#pragma unroll
                for (int i = 0; i < MI; ++i) fa[i] = *reinterpret_cast<const bf16x8_t*>(from + ra + i * 16 * kRowBytes + piece);
#pragma unroll
                for (int i = 0; i < MI; ++i)
#pragma unroll
                    for (int j = 0; j < NI; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j], fa[i], acc[i][j], 0, 0, 0);
            }
        };
        fetch(lds);
        for (int t = 0; t < total; ++t) {
            // the step's tiles have arrived, and every wave is done with the others
            __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
            __syncthreads();
            if (t + 1 < total) fetch(lds + (t + 1) % 2 * kBytes);
            multiply(lds + t % 2 * kBytes);
        }
    }
};

}  // namespace hy
