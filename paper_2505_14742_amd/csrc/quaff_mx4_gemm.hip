// Product of 4-bit microscaled operands, dense or grouped by expert, with the low-rank term of an adapter.
#include "quaff_group_few.h"

namespace quaff {

hipError_t launch_mx4_rows(const GroupArgs& g, hipStream_t stream) {
    if (g.t == 0) return hipSuccess;
    if (g.tile == 16) {
        ProfScope prof(K_MX4_GEMM, stream);
        return launch_group_few<kGroupMx4>(g, stream);
    }
    return launch_group_rows<true, false>(g, K_MX4_GEMM, stream);
}

}  // namespace quaff
