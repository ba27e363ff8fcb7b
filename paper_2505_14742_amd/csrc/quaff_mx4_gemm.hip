// Product of 4-bit microscaled operands, dense or grouped by expert, with the low-rank term of an adapter.
#include "quaff_group_few.h"

namespace quaff {

hipError_t launch_mx4_rows(const GroupArgs& g, hipStream_t stream) {
    if (g.t == 0) return hipSuccess;
    ProfScope prof(K_MX4_GEMM, stream);
    if (few_group_rows(g)) return launch_group_few<kGroupMx4>(g, stream);
    if (large_row_tiles(g)) return launch_group_rows<256, 256, 2, 4, 2, true, false>(g, stream);
    if (small_row_tiles(g)) return launch_group_rows<64, 64, 2, 2, 2, true, false>(g, stream);
    return launch_group_rows<128, 128, 2, 2, 2, true, false>(g, stream);
}

}  // namespace quaff
