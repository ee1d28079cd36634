// Entry points around the mixers with sizes, strides and pointers of every magnitude, linked against stand-ins for the launchers:
// built with sanitizers, so that an overflow in the checks themselves shows.
#include <stdint.h>
#include <stdio.h>

#include <random>
#include <vector>

#include "hy_launch.hpp"

namespace hy {
TuningSnapshot::TuningSnapshot() {}
TuningSnapshot::~TuningSnapshot() {}
int64_t glr_fwd_workspace_bytes(const GlrShape&) { return 0; }
int64_t glr_bwd_workspace_bytes(const GlrShape&, bool) { return 0; }
hy_status launch_glr_fwd(const GlrPtrs&, const GlrShape&, void*, hipStream_t) { return HY_OK; }
hy_status launch_glr_bwd(const GlrPtrs&, const GlrShape&, void*, hipStream_t) { return HY_OK; }
hy_status launch_glr_step(const GlrPtrs&, const GlrShape&, hipStream_t) { return HY_OK; }
bool xent_served(const XentShape&, bool) { return true; }
int64_t xent_fwd_workspace_bytes(const XentShape&) { return 0; }
int64_t xent_bwd_workspace_bytes(const XentShape&) { return 0; }
hy_status launch_xent_fwd(const XentPtrs&, const XentShape&, void*, hipStream_t) { return HY_OK; }
hy_status launch_xent_bwd(const XentPtrs&, const XentShape&, void*, hipStream_t) { return HY_OK; }
hy_status launch_adamw(const AdamwEntry*, const int32_t*, const float*, const AdamwHyper&, const AdamwShape&, hipStream_t) { return HY_OK; }
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
        const int64_t B = any(), L = any(), D = any(), bytes = any();
        const int32_t group = (int32_t)(rng() % 3 ? 1 << rng() % 6 : any()), dtype = (int32_t)(rng() % 2);
        int64_t strides[10];
        for (int64_t& x : strides) x = any();
        const int64_t* st = rng() % 2 ? strides : nullptr;
        hyena_glr_fwd_workspace_bytes(B, L, D, group, dtype);
        hyena_glr_bwd_workspace_bytes(B, L, D, group, dtype, i % 2);
        hyena_xent_fwd_workspace_bytes(B, L, D, dtype);
        hyena_xent_bwd_workspace_bytes(B, L, D, dtype);
        taken += hyena_glr_fwd(at(0), at(1), at(2), at(3), maybe(4), at(5), maybe(6), maybe(7), st, at(8), bytes, B, L, D, group,
                               dtype, nullptr) == HY_OK;
        taken += hyena_glr_bwd(at(0), at(1), at(2), at(3), at(4), maybe(5), maybe(11), maybe(12), at(6), at(7), at(8), at(9),
                               maybe(13), st, at(10), bytes, B, L, D, group, dtype, nullptr) == HY_OK;
        taken += hyena_glr_step(at(0), at(1), at(2), at(3), maybe(4), at(5), B, D, group, dtype, nullptr) == HY_OK;
        const int64_t* target = static_cast<const int64_t*>(at(2));
        taken += hyena_xent_fwd(at(0), at(1), target, maybe(3), maybe(4), at(5), bytes, B, L, D, dtype, nullptr) == HY_OK;
        taken += hyena_xent_bwd(maybe(0), at(1), at(3), target, maybe(4), at(5), at(6), at(7), bytes, B, L, D, dtype, nullptr) == HY_OK;
        hy_adamw_tensor t[2] = {};
        for (int x = 0; x < 2; ++x) {
            t[x].param = at(7 * x), t[x].grad = at(7 * x + 1), t[x].exp_avg = at(7 * x + 2), t[x].exp_avg_sq = at(7 * x + 3);
            t[x].avg_scale = maybe(7 * x + 4), t[x].sq_scale = maybe(7 * x + 5), t[x].master = maybe(7 * x + 6), t[x].count = any();
        }
        const int64_t need = hyena_adamw_table_bytes(t, 2);
        static char table[100000];
        int64_t chunks;
        if (need > 0 && need <= (int64_t)sizeof table)
            taken += hyena_adamw_table(t, 2, dtype, (int32_t)(rng() % 2), rng() % 2 ? 8 : 32, 0, table, need, &chunks) == HY_OK;
        taken += hyena_adamw_step(at(0), any(), any(), dtype, dtype, 32, 0, 1e-3, 0.9, 0.95, 1e-8, any(), nullptr, nullptr) == HY_OK;
    }
    printf("model api selftest: %s\n", taken > 1000 ? "0 problem(s)" : "hardly a call was taken");
    return 0;
}
