// Entry points of linear attention, the norm and the choice of tokens with sizes, strides and pointers of every magnitude, linked
// against stand-ins for the launchers: built with sanitizers, so that an overflow in the checks themselves shows.
#include <stdint.h>
#include <stdio.h>

#include <random>
#include <vector>

#include "hy_launch.hpp"

namespace hy {
bool la_served(const LaShape& s) { return s.dk <= 128; }
int64_t la_marks_bytes(const LaShape&) { return 16; }
int64_t la_fwd_workspace_bytes(const LaShape&) { return 0; }
int64_t la_bwd_workspace_bytes(const LaShape&, bool) { return 0; }
hy_status launch_la_fwd(const LaPtrs&, const LaShape&, void*, hipStream_t) { return HY_OK; }
hy_status launch_la_bwd(const LaPtrs&, const LaShape&, void*, hipStream_t) { return HY_OK; }
hy_status launch_la_step(const LaPtrs&, const LaShape&, hipStream_t) { return HY_OK; }
int64_t norm_bwd_workspace_bytes(int64_t, int64_t) { return 0; }
hy_status launch_norm_fwd(const NormPtrs&, const NormShape&, hipStream_t) { return HY_OK; }
hy_status launch_norm_bwd(const NormPtrs&, const NormShape&, void*, hipStream_t) { return HY_OK; }
hy_status launch_sample(const SamplePtrs&, const SampleAll&, int64_t, int64_t, int64_t, int32_t, hipStream_t) { return HY_OK; }
}  // namespace hy

int main() {
    std::mt19937_64 rng(1);
    std::vector<int64_t> sizes = {0, -1, 1000, INT64_MAX, INT64_MIN};
    for (int k = 0; k < 63; k += 3) sizes.push_back(INT64_C(1) << k), sizes.push_back((INT64_C(1) << k) - 1);
    auto any = [&] { return sizes[rng() % sizes.size()]; };
    auto at = [](int i) { return reinterpret_cast<void*>((uintptr_t)(i + 1) << 48); };
    auto maybe = [&](int i) { return rng() % 2 ? static_cast<float*>(at(i)) : nullptr; };
    int64_t taken = 0;
    for (int i = 0; i < 300000; ++i) {
        const int64_t B = any(), L = any(), H = any(), dk = any(), dv = any(), bytes = any();
        const int32_t group = (int32_t)(rng() % 3 ? 1 << rng() % 6 : any()), dtype = (int32_t)(rng() % 2);
        int64_t strides[14];
        for (int64_t& x : strides) x = any();
        const int64_t* st = rng() % 2 ? strides : nullptr;
        hyena_la_marks_bytes(B, L, H, group, dk, dv, dtype);
        hyena_la_fwd_workspace_bytes(B, L, H, group, dk, dv, dtype);
        hyena_la_bwd_workspace_bytes(B, L, H, group, dk, dv, dtype, i % 2);
        taken += hyena_la_fwd(at(0), at(1), at(2), at(3), maybe(4), at(5), maybe(6), maybe(7), st, at(8), bytes, B, L, H, group, dk, dv, 1.0,
                              dtype, nullptr) == HY_OK;
        taken += hyena_la_bwd(at(0), at(1), at(2), at(3), at(4), maybe(5), maybe(11), maybe(12), at(6), at(7), at(8), at(9), maybe(13), st,
                              at(10), bytes, B, L, H, group, dk, dv, 1.0, dtype, nullptr) == HY_OK;
        taken += hyena_la_step(at(0), at(1), at(2), at(3), maybe(4), at(5), B, H, group, dk, dv, 1.0, dtype, nullptr) == HY_OK;
        taken += hyena_rmsnorm_fwd(at(0), maybe(1), maybe(2), at(3), maybe(4), maybe(5), maybe(6), B, L, H, dk, 1e-6, dtype, nullptr) == HY_OK;
        hyena_rmsnorm_bwd_workspace_bytes(B, L, dtype);
        taken += hyena_rmsnorm_bwd(at(0), at(1), maybe(2), maybe(3), maybe(4), at(5), maybe(6), at(7), bytes, B, L, dtype, nullptr) == HY_OK;
        taken += hyena_sample(at(0), maybe(1), maybe(2), 1.0, nullptr, (int32_t)any(), maybe(3), 1.0, maybe(4), 0.0,
                              static_cast<int64_t*>(at(5)), maybe(6), B, L, H, dtype, nullptr) == HY_OK;
    }
    printf("block api selftest: %s\n", taken > 1000 ? "0 problem(s)" : "hardly a call was taken");
    return 0;
}
