// Products grouped by expert: the rows of a batch lie group after group (offsets in device memory), every group has a weight
// of its own.  One kernel template for three products and two types:
//     rows    C[i, :] = sum_k A[i, k] B_g[k, :] for the rows i of group g   (forward, input gradient)
//     ragged  C_g = sum over the rows i of group g of A[i, :]^T B[i, :]      (weight gradient)
// bf16, or 4-bit floating point (E2M1) with one E8M0 scale per 32 contraction values; fp32 accumulation in both.
//
// Operand tiles stream global -> LDS with direct-to-LDS loads through a ring of stages of 128 contraction bytes per row (64
// bf16 or 256 4-bit values).  A fragment of v_mfma_f32_32x32x16_bf16 and of v_mfma_scale_f32_32x32x64_f8f6f4 is 16 bytes per
// lane in both types, so they share layout, loop and epilogue.
#pragma once
#include "quaff_gemm_dma.h"

namespace quaff {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
typedef __attribute__((address_space(3))) int lds_i32;

// One operand of a tile.  Plain: rows of the tile x contraction, contraction contiguous.  Transposed: contraction rows x
// columns of the tile (bf16 only), gathered with transposing LDS reads.
template <int ROWS, bool TR>
struct GroupStage {
    static constexpr int BYTES = ROWS * 128, LOADS = BYTES / 1024;
    static constexpr int RB = ROWS * 2;                         // transposed: bytes of a contraction row
    // Transposing reads of half a wavefront touch four contraction rows x 64 bytes; their 64-byte units are put in different
    // banks by xor with the row (rows of 128 bytes: two rows cover the banks; rows of 64: four do by themselves).
    __device__ static __forceinline__ int swz(int krow) { return RB >= 256 ? krow & 3 : RB == 128 ? (krow >> 1) & 1 : 0; }
    // What the lane's 16 bytes of 1 KiB load q hold: row and byte of the row (plain: tile row and contraction byte;
    // transposed: contraction row and column byte)
    __device__ static __forceinline__ void source(int q, int lane, int& row, int& byte) {
        if constexpr (!TR) {
            row = q * 8 + (lane >> 3);
            byte = ((lane & 7) ^ ((q * 4 + (lane >> 4)) & 7)) * 16;
        } else {
            constexpr int C16 = RB / 16;
            row = q * (64 / C16) + lane / C16;
            const int c = lane % C16;
            byte = (((c >> 2) ^ swz(row)) * 4 + (c & 3)) * 16;
        }
    }
};

// The row tiles of all groups, and the one this workgroup owns.  Workgroups are dealt to the eight XCDs round-robin; every
// XCD takes a contiguous eighth of the tiles, ordered in blocks of GM tile rows by all tile columns, so that the operand
// panels its compute units touch together are few.  The number of tiles is known here only: surplus workgroups return false.
struct GroupTile { int group, row0, rows, tm, tn; };

__device__ __forceinline__ int group_bound(const int64_t* offsets, int i, int t) {
    const int64_t v = offsets[i];
    return v < 0 ? 0 : v > t ? t : (int)v;
}

template <int BM, int GM>
__device__ __forceinline__ bool find_group_tile(const int64_t* offsets, int n_groups, int t, int tiles_n, GroupTile& out) {
    const int lane = threadIdx.x & 63;
    auto tiles_of = [&](int g, int& a, int& len) {
        a = len = 0;
        if (g < n_groups) {
            a = group_bound(offsets, g, t);
            const int b = group_bound(offsets, g + 1, t);
            len = b > a ? b - a : 0;
        }
        return (len + BM - 1) / BM;
    };
    int total = 0;
    if (!offsets) total = (t + BM - 1) / BM;
    else {
        for (int base = 0; base < n_groups; base += 64) {
            int a, len;
            total += tiles_of(base + lane, a, len);
        }
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) total += __shfl_xor(total, off, 64);
        total = __builtin_amdgcn_readfirstlane(total);
    }
    const int64_t all = (int64_t)total * tiles_n, per = (all + 7) / 8;
    const int64_t lin = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((int64_t)(blockIdx.x >> 3) >= per || lin >= all) return false;
    const int block = (int)(lin / ((int64_t)GM * tiles_n)), rest = (int)(lin - (int64_t)block * GM * tiles_n);
    const int rows = total - block * GM < GM ? total - block * GM : GM;
    out.tn = rest / rows;
    int tm = block * GM + rest % rows;
    if (!offsets) {
        out.group = 0;
        out.row0 = tm * BM;
        out.rows = t - out.row0 < BM ? t - out.row0 : BM;
        out.tm = tm;
        return true;
    }
    for (int base = 0; base < n_groups; base += 64) {
        int a, len;
        const int n = tiles_of(base + lane, a, len);
        int sum = n;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int up = __shfl_up(sum, off, 64);
            if (lane >= off) sum += up;
        }
        const uint64_t above = __ballot(sum > tm);
        if (above) {
            const int l = __builtin_ctzll(above);
            const int k = tm - (__builtin_amdgcn_readlane(sum, l) - __builtin_amdgcn_readlane(n, l));
            const int len_g = __builtin_amdgcn_readlane(len, l);
            out.group = base + l;
            out.row0 = __builtin_amdgcn_readlane(a, l) + k * BM;
            out.rows = len_g - k * BM < BM ? len_g - k * BM : BM;
            out.tm = k;
            return true;
        }
        tm -= __builtin_amdgcn_readlane(sum, 63);
    }
    return false;
}

// Operand tile of a workgroup, as the loader sees it
struct GroupOperand {
    const char* p;      // the tile's first row and first contraction byte (plain), or first contraction row and first column byte
    int64_t ld;         // bytes
    int rows;           // valid tile rows (columns of a transposed tile), at least 1
};

template <int BM, int BN, int WGM, int WGN, int NS, bool MX4, bool TA, bool TB>
struct GroupCfg {
    static constexpr int NW = WGM * WGN, NT = NW * 64;
    static constexpr int WM = BM / WGM, WN = BN / WGN, TM = WM / 32, TN = WN / 32;
    using SA = GroupStage<BM, TA>;
    using SB = GroupStage<BN, TB>;
    static constexpr int SCALE_BYTES = MX4 ? (BM + BN) * 8 : 0;         // eight scales of every row
    static constexpr int CODE_BYTES = SA::BYTES + SB::BYTES;
    static constexpr int STAGE_BYTES = CODE_BYTES + SCALE_BYTES;
    static constexpr int LOADS = CODE_BYTES / 1024, SLOADS = SCALE_BYTES / 256;
    static constexpr int LDS_BYTES = NS * STAGE_BYTES;
    static_assert(!MX4 || (!TA && !TB), "4-bit operands are contraction-contiguous");
    static_assert(LOADS % NW == 0, "whole rounds of loads");
    static_assert(LDS_BYTES <= 160 * 1024, "LDS of a compute unit");
};

// acc += A B over `stages` stages of the contraction.  bf16: k_valid contraction elements in all (a multiple of 8 where an
// operand is plain), chunks past the end are fetched as zeros; 4-bit rows are stored padded to whole stages.
template <class C, bool MX4, bool TA, bool TB, int BM, int BN, int WGN, int NS>
__device__ __forceinline__ void group_mainloop(const GroupOperand& a, const GroupOperand& b, const uint8_t* sa, const uint8_t* sb,
                                               int64_t lds_row, int stages, int k_valid, lds_i8* lds, int wave, int lane,
                                               f32x16 (&acc)[C::TM][C::TN]) {
    auto issue = [&](int kt, int s) {
        lds_i8* const st = lds + s * C::STAGE_BYTES;
#pragma unroll
        for (int j = 0; j < C::LOADS / C::NW; ++j) {
            const int q = j * C::NW + wave;
            const bool isA = q < C::SA::LOADS;
            int row, byte;
            const char* src;
            bool past;
            auto one = [&](const GroupOperand& o, auto stage, int qq, auto tr) {
                using S = decltype(stage);
                S::source(qq, lane, row, byte);
                if constexpr (!decltype(tr)::value) {
                    const int k = kt * 128 + byte;
                    past = !MX4 && k >= k_valid * 2;
                    src = o.p + (int64_t)(row < o.rows ? row : o.rows - 1) * o.ld + k;
                } else {
                    const int k = kt * 64 + row;
                    past = k >= k_valid || byte >= o.rows * 2;
                    src = o.p + (int64_t)k * o.ld + byte;
                }
            };
            if (isA) one(a, typename C::SA{}, q, std::integral_constant<bool, TA>{});
            else one(b, typename C::SB{}, q - C::SA::LOADS, std::integral_constant<bool, TB>{});
            if (past) src = reinterpret_cast<const char*>(kZeroChunk);
            dma_load_16<true>(src, st + q * 1024);
        }
        if constexpr (MX4) {
#pragma unroll
            for (int j = 0; j < (C::SLOADS + C::NW - 1) / C::NW; ++j) {
                const int q = j * C::NW + wave;
                if (q < C::SLOADS) {
                    // 32 rows x 8 bytes: lane = 2 row + half
                    int row = q * 32 + (lane >> 1);
                    const uint8_t* src;
                    if (row < BM) src = sa + (int64_t)(row < a.rows ? row : a.rows - 1) * lds_row;
                    else { row -= BM; src = sb + (int64_t)(row < b.rows ? row : b.rows - 1) * lds_row; }
                    dma_load_4<true>(src + kt * 8 + (lane & 1) * 4, st + C::CODE_BYTES + q * 256);
                }
            }
        }
    };
    const int wm = wave / WGN, wn = wave % WGN, r32 = lane & 31, half = lane >> 5;
    const int sw = (r32 >> 1) & 7;
    const int plain_off = r32 * 128 + (((MX4 ? half * 4 : half) ^ sw) * 16);
    const int tr_i = lane & 15, tr_row = (lane >> 5) * 8 + (tr_i >> 2), tr_in = ((lane >> 4) & 1) * 32 + (tr_i & 3) * 8;
    auto frag = [&](lds_i8* base, int blk, int ks, auto stage, auto tr) {
        if constexpr (!decltype(tr)::value) {
            return *(const lds_i32x4*)(base + blk * 4096 + (plain_off ^ (ks * (MX4 ? 16 : 32))));
        } else {
            using S = decltype(stage);
            lds_i8* p = base + (ks * 16 + tr_row) * S::RB + ((blk ^ S::swz(tr_row)) * 64) + tr_in;
            union { i16x4 h[2]; i32x4 v; } u;
            u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)p);
            u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(p + 4 * S::RB));
            return u.v;
        }
    };
    auto compute = [&](int s) {
        lds_i8* const st = lds + s * C::STAGE_BYTES;
        int xa[C::TM], xb[C::TN];
        if constexpr (MX4) {
#pragma unroll
            for (int i = 0; i < C::TM; ++i) xa[i] = *(const lds_i32*)(st + C::CODE_BYTES + (wm * C::WM + i * 32 + r32) * 8 + half * 4);
#pragma unroll
            for (int j = 0; j < C::TN; ++j) xb[j] = *(const lds_i32*)(st + C::CODE_BYTES + (BM + wn * C::WN + j * 32 + r32) * 8 + half * 4);
        }
        auto sub = [&](auto step) {
            constexpr int ks = decltype(step)::value;
            i32x4 fa[C::TM], fb[C::TN];
#pragma unroll
            for (int i = 0; i < C::TM; ++i) fa[i] = frag(st, wm * C::TM + i, ks, typename C::SA{}, std::integral_constant<bool, TA>{});
#pragma unroll
            for (int j = 0; j < C::TN; ++j) fb[j] = frag(st + C::SA::BYTES, wn * C::TN + j, ks, typename C::SB{}, std::integral_constant<bool, TB>{});
#pragma unroll
            for (int i = 0; i < C::TM; ++i)
#pragma unroll
                for (int j = 0; j < C::TN; ++j) {
                    if constexpr (MX4) {
                        const i32x8 va = {fa[i][0], fa[i][1], fa[i][2], fa[i][3], 0, 0, 0, 0};
                        const i32x8 vb = {fb[j][0], fb[j][1], fb[j][2], fb[j][3], 0, 0, 0, 0};
                        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(va, vb, acc[i][j], 4, 4, ks, xa[i], ks, xb[j]);
                    } else {
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fa[i]), __builtin_bit_cast(bf16x8, fb[j]),
                                                                            acc[i][j], 0, 0, 0);
                    }
                }
        };
        sub(std::integral_constant<int, 0>{});
        sub(std::integral_constant<int, 1>{});
        sub(std::integral_constant<int, 2>{});
        sub(std::integral_constant<int, 3>{});
    };
    static_assert(NS == 2, "two stages used in turn");
    if (stages > 0) issue(0, 0);
    for (int kt = 0; kt < stages; ++kt) {
        QUAFF_WAIT_VMCNT(0);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();                   // everyone's loads of this stage landed, and the other stage has been read
        asm volatile("" ::: "memory");
        if (kt + 1 < stages) issue(kt + 1, (kt + 1) & 1);
        compute(kt & 1);
    }
}

__device__ __forceinline__ uint16_t group_bf16(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }

// C rows/columns of accumulator register i of a 32 x 32 block: row (i & 3) + 8 (i >> 2) + 4 half, column lane & 31
template <class C, bool MX4>
__device__ __forceinline__ void group_store(const GroupArgs& g, f32x16 (&acc)[C::TM][C::TN], float* c, uint16_t* c16, int rows, int cols,
                                            int m0, int n0, int lane) {
    const float s = MX4 ? 1.0f : g.scale;
#pragma unroll
    for (int i = 0; i < C::TM; ++i)
#pragma unroll
        for (int j = 0; j < C::TN; ++j) {
            const int col = n0 + j * 32 + (lane & 31);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int row = m0 + i * 32 + (e & 3) + 8 * (e >> 2) + 4 * (lane >> 5);
                if (row < rows && col < cols) {
                    const int64_t at = (int64_t)row * g.ldc + col;
                    const float v = acc[i][j][e] * s;
                    if (c16) c16[at] = group_bf16(v);
                    else c[at] = g.accumulate ? c[at] + v : v;
                }
            }
        }
}

// Low-rank term: T as a pair of bf16 values (16 significant bits) times the group's bf16 factor
template <class C>
__device__ __forceinline__ void group_low_rank(const GroupArgs& g, const GroupTile& gt, f32x16 (&acc)[C::TM][C::TN], int m0, int n0, int lane) {
    const int r32 = lane & 31, half = lane >> 5;
    const uint16_t* L = g.L + (int64_t)gt.group * g.N * g.r;
    for (int k0 = 0; k0 < g.r; k0 += 16) {
        bf16x8 hi[C::TM], lo[C::TM], fb[C::TN];
#pragma unroll
        for (int i = 0; i < C::TM; ++i) {
            int row = m0 + i * 32 + r32;
            row = row < gt.rows ? row : gt.rows - 1;
            const f32x4* p = reinterpret_cast<const f32x4*>(g.T + (int64_t)(gt.row0 + row) * g.r + k0 + half * 8);
            const f32x4 x[2] = {p[0], p[1]};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float v = x[e >> 2][e & 3];
                hi[i][e] = (__bf16)v;
                lo[i][e] = (__bf16)(v - (float)hi[i][e]);
            }
        }
#pragma unroll
        for (int j = 0; j < C::TN; ++j) {
            int col = n0 + j * 32 + r32;
            col = col < g.N ? col : g.N - 1;
            if (g.l_rn) {
                union { uint16_t h[8]; bf16x8 v; } u;
#pragma unroll
                for (int e = 0; e < 8; ++e) u.h[e] = L[(int64_t)(k0 + half * 8 + e) * g.N + col];
                fb[j] = u.v;
            } else {
                fb[j] = *reinterpret_cast<const bf16x8*>(L + (int64_t)col * g.r + k0 + half * 8);
            }
        }
#pragma unroll
        for (int i = 0; i < C::TM; ++i)
#pragma unroll
            for (int j = 0; j < C::TN; ++j) {
                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(hi[i], fb[j], acc[i][j], 0, 0, 0);
                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lo[i], fb[j], acc[i][j], 0, 0, 0);
            }
    }
}

template <class C>
__device__ __forceinline__ void group_clear(f32x16 (&acc)[C::TM][C::TN]) {
#pragma unroll
    for (int i = 0; i < C::TM; ++i)
#pragma unroll
        for (int j = 0; j < C::TN; ++j) acc[i][j] = f32x16{};
}

template <int BM, int BN, int WGM, int WGN, int NS, bool MX4, bool TB>
__global__ void __launch_bounds__(WGM * WGN * 64) group_rows_kernel(GroupArgs g) {
    using C = GroupCfg<BM, BN, WGM, WGN, NS, MX4, false, TB>;
    __shared__ __attribute__((aligned(1024))) int8_t lds_raw[C::LDS_BYTES];
    GroupTile gt;
    if (!find_group_tile<BM, 8>(g.offsets, g.n_groups, g.t, (g.N + BN - 1) / BN, gt)) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int n0 = gt.tn * BN, cols = g.N - n0 < BN ? g.N - n0 : BN;
    GroupOperand a{static_cast<const char*>(g.A) + (int64_t)gt.row0 * g.lda, g.lda, gt.rows};
    GroupOperand b{static_cast<const char*>(g.B) + (int64_t)gt.group * g.b_group + (TB ? (int64_t)n0 * 2 : (int64_t)n0 * g.ldb), g.ldb, cols};
    const uint8_t* sa = MX4 ? g.SA + (int64_t)gt.row0 * g.ld_scale : nullptr;
    const uint8_t* sb = MX4 ? g.SB + (int64_t)gt.group * g.sb_group + (int64_t)n0 * g.ld_scale : nullptr;
    f32x16 acc[C::TM][C::TN];
    group_clear<C>(acc);
    group_mainloop<C, MX4, false, TB, BM, BN, WGN, NS>(a, b, sa, sb, g.ld_scale, (g.K + (MX4 ? 255 : 63)) / (MX4 ? 256 : 64), g.K,
                                                       (lds_i8*)lds_raw, wave, lane, acc);
    const int m0 = (wave / WGN) * C::WM, nw = (wave % WGN) * C::WN;
    if constexpr (MX4) if (g.r) group_low_rank<C>(g, gt, acc, m0, n0 + nw, lane);
    const int64_t at = (int64_t)gt.row0 * g.ldc + n0;
    group_store<C, MX4>(g, acc, g.C ? g.C + at : nullptr, g.C16 ? g.C16 + at : nullptr, gt.rows, cols, m0, nw, lane);
}

template <int BM, int BN, int WGM, int WGN, int NS>
__global__ void __launch_bounds__(WGM * WGN * 64) group_ragged_kernel(GroupArgs g) {
    using C = GroupCfg<BM, BN, WGM, WGN, NS, false, true, true>;
    __shared__ __attribute__((aligned(1024))) int8_t lds_raw[C::LDS_BYTES];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int tiles_n = (g.N + BN - 1) / BN;
    const int group = blockIdx.y, m0 = (blockIdx.x / tiles_n) * BM, n0 = (blockIdx.x % tiles_n) * BN;
    const int begin = group_bound(g.offsets, group, g.t), end = group_bound(g.offsets, group + 1, g.t);
    const int len = end > begin ? end - begin : 0;
    const int rows = g.M - m0 < BM ? g.M - m0 : BM, cols = g.N - n0 < BN ? g.N - n0 : BN;
    GroupOperand a{static_cast<const char*>(g.A) + (int64_t)begin * g.lda + (int64_t)m0 * 2, g.lda, rows};
    GroupOperand b{static_cast<const char*>(g.B) + (int64_t)begin * g.ldb + (int64_t)n0 * 2, g.ldb, cols};
    f32x16 acc[C::TM][C::TN];
    group_clear<C>(acc);
    group_mainloop<C, false, true, true, BM, BN, WGN, NS>(a, b, nullptr, nullptr, 0, (len + 63) / 64, len, (lds_i8*)lds_raw, wave, lane, acc);
    group_store<C, false>(g, acc, g.C + (int64_t)group * g.c_group + (int64_t)m0 * g.ldc + n0, nullptr, rows, cols, (wave / WGN) * C::WM,
                          (wave % WGN) * C::WN, lane);
}

}  // namespace quaff
