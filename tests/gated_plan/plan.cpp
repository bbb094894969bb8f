// Reads calls, "bf16 m d f d_out" each, and prints of each the tile of h, of y and its splits, of da and db, of the gradients and
// their splits (dx, dWg and dWu, dWd): the planner's own choices, and its workspaces' bytes.
#include <cstdio>

#include "gated_plan.hpp"

struct Call {
    int64_t m, d, f, d_out, ld_wg, ld_wu;
    bool bf16;
};

int main() {
    int bf16;
    long long m, d, f, o;
    while (std::scanf("%d %lld %lld %lld %lld", &bf16, &m, &d, &f, &o) == 5) {
        const Call c = {m, d, f, o, f, f, bf16 != 0};
        const gnnav::Plan a(c, false), b(c, true);
        std::printf("%d %d %d %d %d %d %d %d %zu %zu\n", a.gate, a.down, a.down_splits, b.dgate, b.grads, b.dx_splits, b.dw_splits, b.dd_splits, a.total, b.total);
    }
}
