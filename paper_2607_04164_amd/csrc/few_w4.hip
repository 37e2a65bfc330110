// The few-token layer with 4-bit weights (see few.h and w4.h).
#include "few.h"

namespace bmoe {

hipError_t launch_few_w4(const FewArgs& a, hipStream_t s) {
    auto stack = [&](const bmoe_matrix& m, int64_t rows, int K) {
        return w4_stack(m.w, m.scales, m.zeros, rows, K, a.w.group);
    };
    if (a.w.group == 32) return launch_few_t<FmtW4<32>>(a, stack, s);
    if (a.w.group == 64) return launch_few_t<FmtW4<64>>(a, stack, s);
    return launch_few_t<FmtW4<128>>(a, stack, s);
}

}  // namespace bmoe
