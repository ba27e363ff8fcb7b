// Product of 4-bit microscaled operands, dense or grouped by expert, with the low-rank term of an adapter.
#include "quaff_group_gemm.h"

namespace quaff {

hipError_t launch_mx4_rows(const GroupArgs& g, hipStream_t stream) {
    if (g.t == 0) return hipSuccess;
    ProfScope prof(K_MX4_GEMM, stream);
    constexpr int BM = 128, BN = 128;
    const int64_t partial = g.offsets ? (g.n_groups < g.t ? g.n_groups : g.t) : 1;
    const int64_t tiles = (g.t / BM + partial) * ((g.N + BN - 1) / BN);
    if (tiles + 7 > 0x7fffffff) return hipErrorInvalidValue;
    group_rows_kernel<BM, BN, 2, 2, 2, true, false><<<dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(256), 0, stream>>>(g);
    return hipGetLastError();
}

}  // namespace quaff
