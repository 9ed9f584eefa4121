// Launch rules of the mixture of experts that are decided on the host.
#include <cstdio>

#include "pivot_quant.h"

namespace pivot { void set_error(const char*, ...) {} }

using namespace pivot;

int main() {
    // eight down layers of 64x4096, the first pruned to nothing: seven eighths of 32 blocks in the mean
    std::vector<pivot_qfc_plan_t> layers(8);
    std::vector<const pivot_qfc_plan_t*> ps;
    for (int e = 0; e < 8; ++e) {
        const std::vector<uint8_t> mask(4 * 32, e > 0);
        pivot_qfc_desc d{64, 4096, 16, 128, 128, 0, 0, -1, 0};
        if (build_qfc_host(d, nullptr, 0, mask.data(), nullptr, nullptr, nullptr, layers[e].host) != PIVOT_OK) return 1;
        ps.push_back(&layers[e]);
    }
    if (moe_mean_blocks(ps) != 28) { std::printf("mean %d\n", moe_mean_blocks(ps)); return 1; }
    if (moe_mean_blocks({ps[0]}) != 0 || moe_mean_blocks({ps[1]}) != 32 || moe_mean_blocks({}) != 0) return 1;
    std::printf("all checks passed\n");
    return 0;
}
