// Products grouped by expert in bf16 (forward, input gradient, weight gradient) and the check of their offsets.
#include "quaff_group_few.h"

namespace quaff {

// Sum of the parts of the contraction, in order, for the rows of all groups (which lie one after the other)
__global__ void __launch_bounds__(256) group_join_kernel(GroupArgs g) {
    const int from = g.offsets ? group_bound(g.offsets, 0, g.t) : 0, to = g.offsets ? group_bound(g.offsets, g.n_groups, g.t) : g.t;
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    const int row = (int)(i / g.N), col = (int)(i - (int64_t)row * g.N);
    if (row < from || row >= to) return;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < g.k_parts; ++p) v += *reinterpret_cast<const f32x4*>(g.partial + (int64_t)p * g.t * g.N + i);
    v *= g.scale;
    const int64_t at = (int64_t)row * g.ldc + col;
    if (g.C16) {
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        *reinterpret_cast<bf16x4*>(g.C16 + at) = (bf16x4){(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
    } else {
        f32x4* c = reinterpret_cast<f32x4*>(g.C + at);
        *c = g.accumulate ? *c + v : v;
    }
}

hipError_t launch_group_join(const GroupArgs& g, hipStream_t stream) {
    group_join_kernel<<<dim3((unsigned)(((int64_t)g.t * g.N + 1023) / 1024)), dim3(256), 0, stream>>>(g);
    return hipGetLastError();
}

hipError_t launch_grouped_rows(const GroupArgs& g, bool b_transposed, hipStream_t stream) {
    if (g.t == 0) return hipSuccess;
    if (g.tile == 16) {
        ProfScope prof(K_GROUPED, stream);
        return b_transposed ? launch_group_few<kGroupKN>(g, stream) : launch_group_few<kGroupNK>(g, stream);
    }
    return b_transposed ? launch_group_rows<false, true>(g, K_GROUPED, stream) : launch_group_rows<false, false>(g, K_GROUPED, stream);
}

// Sum of the slabs of every group that has more than one, in their order; groups without rows get zeros.
__global__ void __launch_bounds__(256) group_reduce_kernel(GroupArgs g) {
    const int lane = threadIdx.x & 63, group = blockIdx.y;
    int first = 0, mine = 0;                                       // slabs of the groups before this one, and its own
    for (int base = 0; base <= group; base += 64) {
        int n = 0;
        if (base + lane <= group) {
            const int a = group_bound(g.offsets, base + lane, g.t), b = group_bound(g.offsets, base + lane + 1, g.t);
            n = b > a ? (b - a + g.slab - 1) / g.slab : 0;
        }
        if (base + lane == group) mine = n;
        else first += n;
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        first += __shfl_xor(first, off, 64);
        mine += __shfl_xor(mine, off, 64);
    }
    if (mine == 1) return;
    // (whatever the offsets are: no more than there is room for)
    const int most = g.t / g.slab + (g.n_groups < g.t ? g.n_groups : g.t);
    if (mine > most - first) mine = most - first;
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= g.c_group) return;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    const float* p = g.partial + (int64_t)first * g.c_group + i;
    for (int s = 0; s < mine; ++s) v += *reinterpret_cast<const f32x4*>(p + (int64_t)s * g.c_group);
    *reinterpret_cast<f32x4*>(g.C + (int64_t)group * g.c_group + i) = v;
}

hipError_t launch_grouped_ragged(const GroupArgs& g, hipStream_t stream) {
    hipError_t e;
    {
        ProfScope prof(K_GROUPED, stream);
        int bm, bn;
        group_ragged_tile(g.t, g.M, g.N, g.n_groups, &bm, &bn);
        if (bn == 32) e = launch_group_ragged<128, 32, 4, 1, 2>(g, stream);
        else if (bn == 64) e = launch_group_ragged<128, 64, 4, 1, 2>(g, stream);
        else if (bm == 32) e = launch_group_ragged<32, 128, 1, 4, 2>(g, stream);
        else if (bm == 64) e = launch_group_ragged<64, 128, 1, 4, 2>(g, stream);
        else if (bm == 256) e = launch_group_ragged<256, 256, 2, 4, 2>(g, stream);
        else e = launch_group_ragged<128, 128, 2, 2, 2>(g, stream);
    }
    if (e != hipSuccess || !g.slab) return e;
    ProfScope prof(K_GROUPED, stream);
    group_reduce_kernel<<<dim3((unsigned)((g.c_group + 1023) / 1024), g.n_groups), dim3(256), 0, stream>>>(g);
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
