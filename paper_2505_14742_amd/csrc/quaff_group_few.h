// Products grouped by expert where a group has few rows (single tokens through a layer, tokens spread over many experts): the weight is
// read once from memory, that is the whole cost.  A workgroup takes 16 rows of a group and 16 NB columns of its result; its
// wavefronts share the contraction (every fourth or sixteenth unit of it), so that a large part of the weight is in flight at once, and join their sums
// in LDS in a fixed order.  v_mfma_f32_16x16x32_bf16 and v_mfma_scale_f32_16x16x128_f8f6f4: lane = row or column (lane & 15) and
// one of four chunks of the contraction (lane >> 4), 16 bytes.
#pragma once
#include "quaff_group_gemm.h"

namespace quaff {

// Low-rank operands in LDS: T [16 x r] fp32 and the factor [16 columns x r] bf16, rows of 64 values (zeros beyond r) and a pad
constexpr int kFewTRow = 68 * 4, kFewLRow = 72 * 2, kFewT = 16 * kFewTRow, kFewL = 16 * kFewLRow;

// KIND: B is 4-bit [N x K], bf16 [N x K] or bf16 [K x N]
template <int KIND, int NB, int NW>
__global__ void __launch_bounds__(NW * 64) group_few_kernel(GroupArgs g) {
    constexpr int COLS = 16 * NB, NT = NW * 64;
    constexpr bool MX4 = KIND == kGroupMx4, KN = KIND == kGroupKN;
    // [K x N]: a wavefront's own 32 H contraction rows x COLS columns, four loads of 1 KiB for 32 of them
    static_assert(!KN || NB == 4, "whole lines of a contraction row");
    constexpr int H = NW > 4 ? 2 : 4, STAGE = KN ? H * 32 * COLS * 2 : 0, RED = 16 * COLS * 4;
    __shared__ __attribute__((aligned(1024))) int8_t lds_raw[(NW * STAGE > NW * RED ? NW * STAGE : NW * RED) + (MX4 ? kFewT + kFewL : 0)];
    GroupTile gt;
    if (!find_group_tile<1>(g.offsets, g.n_groups, g.t, 16, (g.N + COLS - 1) / COLS, gt)) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, q = lane >> 4, n0 = gt.tn * COLS;
    const int64_t row = gt.row0 + (n < gt.rows ? n : gt.rows - 1);
    const char* const pa = static_cast<const char*>(g.A) + row * g.lda + q * 16;
    const char* const pb = static_cast<const char*>(g.B) + (int64_t)gt.group * g.b_group;
    // The adapter's operands (NB = 1), 16 bytes of each to a thread: requested behind the first loads of the weight, so that they add no latency of their own
    // (168 groups of 7 rows, 512 -> 896 at rank 64, with loops over global memory at the end: 183 us, so 57)
    f32x4 tv = {0.f, 0.f, 0.f, 0.f};
    i32x4 lv = {0, 0, 0, 0};
    auto fetch_low_rank = [&] {
        if constexpr (MX4) {
            if (tid * 4 < gt.rows * g.r) {
                const f32x4* p = reinterpret_cast<const f32x4*>(g.T + (int64_t)gt.row0 * g.r) + tid;
#pragma unroll
                for (int part = 0; part < kMx4MaxParts; ++part)
                    if (part < g.t_parts) tv += p[(int64_t)part * g.t * g.r / 4];
            }
            // plain: 16 r values one after the other; [r x N]: two pieces of a row
            const uint16_t* const L = g.L + (int64_t)gt.group * g.N * g.r;
            if (tid * 8 < 16 * g.r)
                lv = *reinterpret_cast<const i32x4*>(g.l_rn ? L + (int64_t)(tid >> 1) * g.N + n0 + (tid & 1) * 8 : L + (int64_t)n0 * g.r + tid * 8);
        }
    };
    f32x4 acc[NB];
#pragma unroll
    for (int c = 0; c < NB; ++c) acc[c] = (f32x4){0.f, 0.f, 0.f, 0.f};
    if constexpr (!KN) {
        // a unit: 128 contraction bytes of every row, two loads
        constexpr int U = 4;                                                         // units requested at a time
        const int units = MX4 ? (g.K + 255) / 256 : (g.K + 63) / 64;
        const char* pw[NB];
        const uint8_t* ps[NB];
#pragma unroll
        for (int c = 0; c < NB; ++c) {
            const int col = n0 + c * 16 + n;
            pw[c] = pb + (int64_t)(col < g.N ? col : g.N - 1) * g.ldb + q * 16;
            if constexpr (MX4) ps[c] = g.SB + (int64_t)gt.group * g.sb_group + (int64_t)(col < g.N ? col : g.N - 1) * g.ld_scale;
        }
        const uint8_t* const pas = MX4 ? g.SA + row * g.ld_scale : nullptr;
        for (int u0 = wave; u0 < units; u0 += NW * U) {
            i32x4 w[U][NB][2], a[U][2];
            int sw[U][NB][2], sa[U][2];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int u = u0 + i * NW;
                if (u >= units) break;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const bool in = MX4 || u * 64 + h * 32 + q * 8 < g.K;          // (bf16: the contraction may end inside the unit)
                    const i32x4 zero = {0, 0, 0, 0};
                    a[i][h] = in ? *reinterpret_cast<const i32x4*>(pa + u * 128 + h * 64) : zero;
#pragma unroll
                    for (int c = 0; c < NB; ++c) w[i][c][h] = in ? *reinterpret_cast<const i32x4*>(pw[c] + u * 128 + h * 64) : zero;
                }
                if constexpr (MX4) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        sa[i][h] = *reinterpret_cast<const int*>(pas + u * 8 + h * 4);
#pragma unroll
                        for (int c = 0; c < NB; ++c) sw[i][c][h] = *reinterpret_cast<const int*>(ps[c] + u * 8 + h * 4);
                    }
                }
            }
            if (u0 == wave) fetch_low_rank();
#pragma unroll
            for (int i = 0; i < U; ++i) {
                if (u0 + i * NW >= units) break;
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int c = 0; c < NB; ++c) {
                        if constexpr (MX4) {
                            const i32x8 va = {a[i][h][0], a[i][h][1], a[i][h][2], a[i][h][3], 0, 0, 0, 0};
                            const i32x8 vb = {w[i][c][h][0], w[i][c][h][1], w[i][c][h][2], w[i][c][h][3], 0, 0, 0, 0};
                            acc[c] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(va, vb, acc[c], 4, 4, 0, (int)((uint32_t)sa[i][h] >> (8 * q)), 0,
                                                                                      (int)((uint32_t)sw[i][c][h] >> (8 * q)));
                        } else {
                            acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[i][h]), __builtin_bit_cast(bf16x8, w[i][c][h]),
                                                                             acc[c], 0, 0, 0);
                        }
                    }
            }
        }
        if (wave >= units) fetch_low_rank();
    } else {
        lds_i8* const st = (lds_i8*)lds_raw + wave * STAGE;
        const int units = (g.K + 32 * H - 1) / (32 * H);
        using S = GroupStage<COLS, true>;
        const int tr_row = q * 8 + (n >> 2);
        for (int u = wave; u < units; u += NW) {
            i32x4 a[H];
#pragma unroll
            for (int h = 0; h < H; ++h) {
                a[h] = (i32x4){0, 0, 0, 0};
                if ((u * H + h) * 32 + q * 8 < g.K) a[h] = *reinterpret_cast<const i32x4*>(pa + (u * H + h) * 64);
            }
#pragma unroll
            for (int i = 0; i < 4 * H; ++i) {
                int krow, byte;
                S::source(i, lane, krow, byte);
                const int k = u * 32 * H + krow;
                const bool in = k < g.K && n0 * 2 + byte < g.N * 2;
                dma_load_16<false>(in ? pb + (int64_t)k * g.ldb + n0 * 2 + byte : reinterpret_cast<const char*>(kZeroChunk), st + i * 1024);
            }
            QUAFF_WAIT_VMCNT(0);
#pragma unroll
            for (int h = 0; h < H; ++h)
#pragma unroll
                for (int c = 0; c < NB; ++c) {
                    const lds_i8* p = st + (h * 32 + tr_row) * S::RB + (((c >> 1) ^ S::swz(tr_row)) * 64) + (c & 1) * 32 + (n & 3) * 8;
                    union { i16x4 v[2]; i32x4 w; } f;
                    f.v[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)p);
                    f.v[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(p + 4 * S::RB));
                    acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[h]), __builtin_bit_cast(bf16x8, f.w), acc[c], 0, 0, 0);
                }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                   // read before the next unit arrives
        }
        __syncthreads();
    }
    if constexpr (MX4) {
        static_assert(NB == 1, "one block of columns");
        if (g.r) {
            lds_i8* const ts = (lds_i8*)lds_raw + NW * RED;
            lds_i8* const ls = ts + kFewT;
            if (tid < 256) {
                const int row = tid * 4 / g.r, at = tid * 4 % g.r;
                if (row < 16) *(lds_f32x4*)(ts + row * kFewTRow + at * 4) = tv;                     // (rows past the group's: zeros)
                for (int i = tid * 4 + 16 * g.r; i < 16 * 64; i += 1024) {                          // zeros beyond r
                    const int j = i - 16 * g.r, width = 64 - g.r;
                    *(lds_f32x4*)(ts + j / width * kFewTRow + (g.r + j % width) * 4) = (f32x4){0.f, 0.f, 0.f, 0.f};
                }
            }
            typedef __attribute__((address_space(3))) uint16_t lds_u16;
            if (tid * 8 < 16 * g.r) {
                if (g.l_rn) {
                    union { i32x4 v; uint16_t h[8]; } u{lv};
#pragma unroll
                    for (int e = 0; e < 8; ++e) *(lds_u16*)(ls + ((tid & 1) * 8 + e) * kFewLRow + (tid >> 1) * 2) = u.h[e];
                } else {
                    *(lds_i32x4*)(ls + tid * 8 / g.r * kFewLRow + tid * 8 % g.r * 2) = lv;
                }
            }
            for (int i = tid * 8 + 16 * g.r; i < 16 * 64; i += NT * 8) {
                const int j = i - 16 * g.r, width = 64 - g.r;
                *(lds_i32x4*)(ls + j / width * kFewLRow + (g.r + j % width) * 2) = (i32x4){0, 0, 0, 0};
            }
            __syncthreads();
            if (wave == 0)
                for (int k0 = 0; k0 < g.r; k0 += 32) {
                    const lds_i8* p = ts + n * kFewTRow + (k0 + q * 8) * 4;
                    const f32x4 x[2] = {*(const lds_f32x4*)p, *(const lds_f32x4*)(p + 16)};
                    const bf16x8 l = __builtin_bit_cast(bf16x8, *(const lds_i32x4*)(ls + n * kFewLRow + (k0 + q * 8) * 2));
                    i32x4 planes[3];
                    split_bf16(x, planes);
#pragma unroll
                    for (int p = 0; p < 3; ++p)
                        acc[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, planes[p]), l, acc[0], 0, 0, 0);
                }
        }
    }
    // accumulator register i of a 16 x 16 block: row 4 q + i, column n
    lds_f32* const red = (lds_f32*)lds_raw;
#pragma unroll
    for (int c = 0; c < NB; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) red[wave * (16 * COLS) + (4 * q + i) * COLS + c * 16 + n] = acc[c][i];
    __syncthreads();
    for (int i = tid; i < gt.rows * COLS; i += NT) {
        const int r = i / COLS, col = n0 + i % COLS;
        if (col >= g.N) continue;
        float v = red[i];
#pragma unroll
        for (int w = 1; w < NW; ++w) v += red[w * (16 * COLS) + i];
        if constexpr (!MX4) v *= g.scale;
        const int64_t at = (int64_t)(gt.row0 + r) * g.ldc + col;
        if (g.C16) g.C16[at] = __builtin_bit_cast(uint16_t, (__bf16)v);
        else g.C[at] = g.accumulate ? g.C[at] + v : v;
    }
}

template <int KIND, int NB, int NW>
static hipError_t launch_group_few_form(const GroupArgs& g, hipStream_t stream) {
    const int64_t tiles = group_row_tiles(g, 16) * ((g.N + 16 * NB - 1) / (16 * NB));
    if (tiles + 7 > 0x7fffffff) return hipErrorInvalidValue;
    group_few_kernel<KIND, NB, NW><<<dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(NW * 64), 0, stream>>>(g);
    return hipGetLastError();
}

// Plain weights: 16 columns a workgroup (32 take too many registers for the loads in flight: 16 rows x 4096 -> 11008 4-bit 12.6 us, so 15.0).
// [K x N]: sixteen wavefronts share a contraction where there is less than one workgroup per compute unit (1 x 4096 -> 4096: 16.5 us, so 13.7).
template <int KIND>
static hipError_t launch_group_few(const GroupArgs& g, hipStream_t stream) {
    if constexpr (KIND == kGroupKN) {
        const int64_t rows = group_row_tiles(g, 16);
        if (rows * ((g.N + 63) / 64) < kUnits) return launch_group_few_form<KIND, 4, 16>(g, stream);
        return launch_group_few_form<KIND, 4, 4>(g, stream);
    } else {
        return launch_group_few_form<KIND, 1, 4>(g, stream);
    }
}

}  // namespace quaff
