// Products grouped by expert in bf16 (forward, input gradient, weight gradient) and the check of their offsets.
#include "quaff_group_gemm.h"

namespace quaff {

// most row tiles that t rows in n_groups groups can have
static int64_t row_tiles(const GroupArgs& g, int bm) {
    const int64_t partial = g.offsets ? (g.n_groups < g.t ? g.n_groups : g.t) : 1;
    return g.t / bm + partial;
}

hipError_t launch_grouped_rows(const GroupArgs& g, bool b_transposed, hipStream_t stream) {
    if (g.t == 0) return hipSuccess;
    ProfScope prof(K_GROUPED, stream);
    constexpr int BM = 128, BN = 128;
    const int64_t tiles = row_tiles(g, BM) * ((g.N + BN - 1) / BN);
    if (tiles + 7 > 0x7fffffff) return hipErrorInvalidValue;
    const dim3 grid((unsigned)((tiles + 7) / 8 * 8)), block(256);
    if (b_transposed) group_rows_kernel<BM, BN, 2, 2, 2, false, true><<<grid, block, 0, stream>>>(g);
    else group_rows_kernel<BM, BN, 2, 2, 2, false, false><<<grid, block, 0, stream>>>(g);
    return hipGetLastError();
}

hipError_t launch_grouped_ragged(const GroupArgs& g, hipStream_t stream) {
    ProfScope prof(K_GROUPED, stream);
    constexpr int BM = 128, BN = 128;
    const int64_t tiles = (int64_t)((g.M + BM - 1) / BM) * ((g.N + BN - 1) / BN);
    if (tiles > 0x7fffffff) return hipErrorInvalidValue;
    group_ragged_kernel<BM, BN, 2, 2, 2><<<dim3((unsigned)tiles, g.n_groups), dim3(256), 0, stream>>>(g);
    return hipGetLastError();
}

__global__ void __launch_bounds__(256) check_group_offsets_kernel(const int64_t* offsets, int n, int64_t t, int32_t* result) {
    __shared__ int first_bad;
    if (threadIdx.x == 0) first_bad = n + 1;
    __syncthreads();
    for (int i = threadIdx.x; i <= n; i += 256) {
        const int64_t v = offsets[i];
        if (v < 0 || v > t || (i > 0 && v < offsets[i - 1])) atomicMin(&first_bad, i);
    }
    __syncthreads();
    if (threadIdx.x == 0) *result = first_bad > n ? 0 : 1 + first_bad;
}

hipError_t launch_check_group_offsets(const int64_t* offsets, int32_t n_groups, int64_t t, int32_t* result, hipStream_t stream) {
    ProfScope prof(K_GROUPED, stream);
    check_group_offsets_kernel<<<1, 256, 0, stream>>>(offsets, n_groups, t, result);
    return hipGetLastError();
}

}  // namespace quaff
