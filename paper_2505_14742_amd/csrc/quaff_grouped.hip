// Products grouped by expert in bf16 (forward, input gradient, weight gradient) and the check of their offsets.
#include "quaff_group_few.h"

namespace quaff {

hipError_t launch_grouped_rows(const GroupArgs& g, bool b_transposed, hipStream_t stream) {
    if (g.t == 0) return hipSuccess;
    ProfScope prof(K_GROUPED, stream);
    if (few_group_rows(g)) return b_transposed ? launch_group_few<kGroupKN, 4>(g, stream) : launch_group_few<kGroupNK, 1>(g, stream);
    if (large_row_tiles(g)) {
        if (b_transposed) return launch_group_rows<256, 256, 2, 4, 2, false, true>(g, stream);
        return launch_group_rows<256, 256, 2, 4, 2, false, false>(g, stream);
    }
    if (b_transposed) return launch_group_rows<128, 128, 2, 2, 2, false, true>(g, stream);
    return launch_group_rows<128, 128, 2, 2, 2, false, false>(g, stream);
}

hipError_t launch_grouped_ragged(const GroupArgs& g, hipStream_t stream) {
    ProfScope prof(K_GROUPED, stream);
    const int64_t large = (int64_t)((g.M + 255) / 256) * ((g.N + 255) / 256) * g.n_groups;
    if (large >= 256) return launch_group_ragged<256, 256, 2, 4, 2>(g, stream);
    return launch_group_ragged<128, 128, 2, 2, 2>(g, stream);
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
