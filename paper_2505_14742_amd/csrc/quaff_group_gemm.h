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
#include <utility>

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
struct GroupTile {
    int group, row0, rows;      // its rows
    int tm, tn;                 // tile row among all tile rows, tile column
    int len;                    // rows of the whole group
    int quarter;                // -1: the whole tile
};

__device__ __forceinline__ int group_bound(const int64_t* offsets, int i, int t) {
    const int64_t v = offsets[i];
    return v < 0 ? 0 : v > t ? t : (int)v;
}

constexpr int kUnits = 256;             // compute units

// QUARTERS: the tiles that are left over from whole rounds of one tile per compute unit are dealt out in quarters (half the rows, half the
// columns; out.quarter 0 .. 3) where one round of quarters takes them (6000 rows in two groups, 2048 -> 5632, 16 tiles left: 182 us, so 160;
// with 104 or 176 left two and three rounds of quarters cost more than one of whole tiles: 238 -> 253 us, 142 -> 155).
template <int GM, bool QUARTERS = false>
__device__ __forceinline__ bool find_group_tile(const int64_t* offsets, int n_groups, int t, int BM, int tiles_n, GroupTile& out) {
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
    // (no more than the launch has workgroups for, whatever the offsets are; the launch keeps the product in 31 bits)
    const int most = t / BM + (offsets && n_groups < t ? n_groups : offsets ? t : 1);
    total = total < most ? total : most;
    uint32_t all = (uint32_t)total * tiles_n, id = blockIdx.x, first = 0;
    out.quarter = -1;
    if constexpr (QUARTERS) {
        const uint32_t whole = all / kUnits * kUnits, left = all - whole;
        if (id < whole) all = whole;
        else {
            first = whole;
            id -= whole;
            all = left;
            if (left <= kUnits / 4) {
                all = 4 * left;
                out.quarter = 0;
            }
        }
    }
    const uint32_t per = (all + 7) / 8, at = id >> 3;
    uint32_t lin = (id & 7) * per + at;
    if (at >= per || lin >= all) return false;
    if (QUARTERS && out.quarter == 0) {
        out.quarter = (int)(lin & 3);
        lin >>= 2;
    }
    lin += first;
    const uint32_t block = lin / ((uint32_t)GM * tiles_n), rest = lin - block * GM * tiles_n;
    const uint32_t rows = total - block * GM < GM ? total - block * GM : GM;
    out.tn = (int)(rest / rows);
    int tm = (int)(block * GM + rest % rows);
    out.tm = tm;
    if (!offsets) {
        out.group = 0;
        out.row0 = tm * BM;
        out.rows = t - out.row0 < BM ? t - out.row0 : BM;
        out.len = t;
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
            out.len = len_g;
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

template <int BM_, int BN_, int WGM_, int WGN_, int NS_, bool MX4_, bool TA_, bool TB_>
struct GroupCfg {
    // NS: stages of B in the ring; A has one more where the LDS has room for it
    static constexpr int BM = BM_, BN = BN_, WGN = WGN_, NS = NS_;
    static constexpr int NSA = NS_ + (!MX4_ && BM_ * BN_ >= 128 * 128 ? 1 : 0);
    static constexpr bool MX4 = MX4_, TA = TA_, TB = TB_;
    static constexpr int NW = WGM_ * WGN_, NT = NW * 64;
    static constexpr int WM = BM / WGM_, WN = BN / WGN_, TM = WM / 32, TN = WN / 32;
    using SA = GroupStage<BM, TA>;
    using SB = GroupStage<BN, TB>;
    static constexpr int B_AT = NSA * SA::BYTES, SCALES_AT = B_AT + NS * SB::BYTES;
    static constexpr int LA = SA::LOADS / NW, LB = SB::LOADS / NW;      // 1 KiB loads of a wavefront per stage
    static constexpr int LOADS = LA + LB;
    // Scales are fetched for four stages at a time, 32 bytes of every row in two pieces, into one of two buffers of their own: eight
    // bytes a stage would be as many requests to the L2 as the codes are
    static constexpr int SCALE_PIECE = (BM + BN) * 16, SCALE_BYTES = MX4 ? 2 * SCALE_PIECE : 0;
    static constexpr int SLOADS = SCALE_BYTES / 1024, LS = SLOADS / NW;
    static constexpr int LDS_BYTES = SCALES_AT + 2 * SCALE_BYTES;
    static_assert(!MX4 || (!TA && !TB), "4-bit operands are contraction-contiguous");
    static_assert(SA::LOADS % NW == 0 && SB::LOADS % NW == 0 && SLOADS % NW == 0, "whole rounds of loads");
    static_assert(LDS_BYTES <= 160 * 1024, "LDS of a compute unit");
    static_assert(!MX4 || (BM % 64 == 0 && BN % 64 == 0), "a scale load holds 64 rows of one operand");
    static_assert(NS == 2, "the waits count on two stages of B");
};

// (the compiler takes a pointer computed from a lookup among lanes for one that differs between them)
template <class T>
__device__ __forceinline__ const T* group_uniform(const T* p) {
    const uint64_t v = (uint64_t)p;
    return (const T*)(((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32) | (uint32_t)__builtin_amdgcn_readfirstlane((int)v));
}

// What a wavefront loads: byte offsets, from the operand's first byte of a stage, of its lanes' 16 bytes in every 1 KiB load
template <class C>
struct GroupLoads { uint32_t a[C::LA], b[C::LB], s[C::LS > 0 ? C::LS : 1]; };

template <int ROWS, bool TR, int N, int NW>
__device__ __forceinline__ void group_offsets(const GroupOperand& o, int wave, int lane, uint32_t (&off)[N]) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
        int row, byte;
        GroupStage<ROWS, TR>::source(j * NW + wave, lane, row, byte);
        // rows (columns) past the edge repeat valid ones and are never stored
        if constexpr (!TR) off[j] = (uint32_t)((row < o.rows ? row : o.rows - 1) * o.ld + byte);
        else off[j] = (uint32_t)(row * o.ld + (byte < o.rows * 2 ? byte : 0));
    }
}

// The stages as group_mainloop reads them.  Opaque to the compiler: a main loop with one caller is given the array's address in place of its
// parameter before it is inlined, the parameter's restrict is lost with it, and transposed reads wait for all loads in flight (8192 rows in eight
// uneven groups, 4096 -> 4096, forward: 338 us, so 289; 2048 x 5632 gradients of 16 groups: 314, so 292).
__device__ __forceinline__ const lds_i8* group_ring(const int8_t* lds) {
    const lds_i8* p = (const lds_i8*)lds;
    asm("" : "+s"(p));
    return p;
}

template <class F, int... I>
__device__ __forceinline__ void group_each(F& f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }

// acc += A B over `stages` stages of the contraction.  bf16: k_valid contraction elements in all (a multiple of 8 where an
// operand is plain), chunks past the end are fetched as zeros; 4-bit rows are stored padded to whole stages.
// The ring holds NS stages.  Fragments are double-buffered in registers; the barrier of a stage sits between the reads of its last
// sub-step and that sub-step's MFMAs, and the stage is refilled right behind it, so a load has a whole stage of time.
// `dma` and `rd` are the same memory; as separate restrict parameters they keep the compiler from ordering every LDS read behind all
// outstanding loads (the order is kept by the waits and barriers here).  `rd` comes from group_ring.
template <class C>
__device__ __forceinline__ void group_mainloop(GroupOperand a, GroupOperand b, const uint8_t* sa, const uint8_t* sb, int64_t ld_scale,
                                               int stages, int k_valid,
                                               lds_i8* __restrict__ dma, const lds_i8* __restrict__ rd, int wave, int lane,
                                               f32x16 (&acc)[C::TM][C::TN]) {
    constexpr int TM = C::TM, TN = C::TN, NS = C::NS;
    constexpr bool MX4 = C::MX4, TA = C::TA, TB = C::TB;
    if (stages <= 0) return;
    a.p = group_uniform(a.p);
    b.p = group_uniform(b.p);
    if constexpr (MX4) {
        sa = group_uniform(sa);
        sb = group_uniform(sb);
    }
    GroupLoads<C> ld;
    group_offsets<C::BM, TA, C::LA, C::NW>(a, wave, lane, ld.a);
    group_offsets<C::BN, TB, C::LB, C::NW>(b, wave, lane, ld.b);
    auto scale_load = [&](int j) { return j * C::NW + wave; };
    if constexpr (MX4) {
#pragma unroll
        for (int j = 0; j < C::LS; ++j) {
            // 64 rows of A, then of B, first the scales of the first two stages of four, then those of the others
            constexpr int half = C::SLOADS / 2;
            const int q = scale_load(j), piece = q >= half, row = (q - piece * half) * 64 + lane;
            const bool is_a = row < C::BM;
            const int r = is_a ? row : row - C::BM, rows = is_a ? a.rows : b.rows;
            ld.s[j] = (uint32_t)((r < rows ? r : rows - 1) * ld_scale + piece * 16);
        }
    }
    const int64_t step_a = TA ? 64 * a.ld : 128, step_b = TB ? 64 * b.ld : 128;
    const int full = MX4 ? stages : k_valid / 64;         // stages that need no zeros
    // zeros: the stage may reach past the end of the contraction (4-bit: the stage may be the last)
    auto issue_one = [&](int kt, int s, auto zeros, auto of_b) {
        constexpr bool B = decltype(of_b)::value, TR = B ? TB : TA;
        lds_i8* const st = dma + (B ? C::B_AT + s * C::SB::BYTES : s * C::SA::BYTES);
        const char* const p = B ? b.p + kt * step_b : a.p + kt * step_a;
        const int left = k_valid - kt * 64;
#pragma unroll
        for (int j = 0; j < (B ? C::LB : C::LA); ++j) {
            const int q = j * C::NW + wave;
            const char* src = p + (B ? ld.b[j] : ld.a[j]);
            if constexpr (decltype(zeros)::value && !MX4) {
                int row, byte;
                if constexpr (B) C::SB::source(q, lane, row, byte);
                else C::SA::source(q, lane, row, byte);
                if (TR ? row >= left : byte >= left * 2) src = reinterpret_cast<const char*>(kZeroChunk);
            }
            dma_load_16<false>(src, st + q * 1024);
        }
    };
    using No = std::false_type;
    using Yes = std::true_type;
    auto issue_a = [&](int kt, int s, auto zeros) { issue_one(kt < stages ? kt : stages - 1, s, zeros, No{}); };
    auto issue_b = [&](int kt, int s, auto zeros) { issue_one(kt < stages ? kt : stages - 1, s, zeros, Yes{}); };
    // scales of the four stages 4 group ...
    auto scale_piece = [&](int group, int j) {
        constexpr int half = C::SLOADS / 2;
        const int q = scale_load(j), piece = q >= half;
        const bool is_a = (q - piece * half) * 64 < C::BM;
        dma_load_16<false>((is_a ? sa : sb) + group * 32 + ld.s[j], dma + C::SCALES_AT + (group & 1) * C::SCALE_BYTES + q * 1024);
    };
    auto issue_scales = [&](int group) {
#pragma unroll
        for (int j = 0; j < C::LS; ++j) scale_piece(group, j);
    };
    // ... of which the contraction may have fewer: nothing behind a row's scales is read.  A last stage whose piece it has alone is
    // fetched in words, eight bytes after eight bytes.
    auto issue_last_scales = [&](int group) {
        if constexpr (MX4) {
#pragma unroll
            for (int j = 0; j < C::LS; ++j)
                if (group * 4 + (scale_load(j) >= C::SLOADS / 2 ? 3 : 1) < stages) scale_piece(group, j);
            if ((stages & 1) && stages - 1 >= group * 4 && stages - 1 < group * 4 + 4) {
                const int piece = ((stages - 1) >> 1) & 1;
                for (int q = wave; q < (C::BM + C::BN) / 32; q += C::NW) {
                    const int row = q * 32 + (lane >> 1);
                    const bool is_a = q * 32 < C::BM;
                    const int r = is_a ? row : row - C::BM, rows = is_a ? a.rows : b.rows;
                    dma_load_4<false>((is_a ? sa : sb) + (r < rows ? r : rows - 1) * ld_scale + (stages - 1) * 8 + (lane & 1) * 4,
                                      dma + C::SCALES_AT + (group & 1) * C::SCALE_BYTES + piece * C::SCALE_PIECE + q * 256);
                }
            }
        }
    };
    const int wm = wave / C::WGN, wn = wave % C::WGN, r32 = lane & 31, half = lane >> 5;
    // 4-bit: half a wavefront takes blocks 4 half + ks of the stage's eight, so that its four scales of a stage are one word
    const int plain_off = r32 * 128 + (((MX4 ? half * 4 : half) ^ ((r32 >> 1) & 7)) * 16);
    const int tr_i = lane & 15, tr_row = (lane >> 5) * 8 + (tr_i >> 2), tr_in = ((lane >> 4) & 1) * 32 + (tr_i & 3) * 8;
    auto frag = [&](const lds_i8* base, int blk, int ks, auto stage, auto tr) {
        if constexpr (!decltype(tr)::value) {
            return *(const lds_i32x4*)(base + blk * 4096 + (plain_off ^ (ks * (MX4 ? 16 : 32))));
        } else {
            using S = decltype(stage);
            const lds_i8* p = base + tr_row * S::RB + tr_in + ((blk ^ S::swz(tr_row)) * 64) + ks * 16 * S::RB;
            union { i16x4 h[2]; i32x4 v; } u;
            u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)p);
            u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(p + 4 * S::RB));
            return u.v;
        }
    };
    auto read_frags = [&](int s_a, int s_b, int ks, i32x4 (&fa)[TM], i32x4 (&fb)[TN]) {
        const lds_i8* const sta = rd + s_a * C::SA::BYTES;
        const lds_i8* const stb = rd + C::B_AT + s_b * C::SB::BYTES;
#pragma unroll
        for (int i = 0; i < TM; ++i) fa[i] = frag(sta, wm * TM + i, ks, typename C::SA{}, std::integral_constant<bool, TA>{});
#pragma unroll
        for (int j = 0; j < TN; ++j) fb[j] = frag(stb, wn * TN + j, ks, typename C::SB{}, std::integral_constant<bool, TB>{});
    };
    auto read_scales = [&](int kt, int (&xa)[TM], int (&xb)[TN], auto last) {
        if constexpr (MX4) {
            const lds_i8* st = rd + C::SCALES_AT + ((kt >> 2) & 1) * C::SCALE_BYTES + ((kt >> 1) & 1) * C::SCALE_PIECE;
            int row = 16;
            if (decltype(last)::value && kt == stages - 1 && (stages & 1)) row = 8;
            else st += (kt & 1) * 8;
            st += r32 * row + half * 4;
#pragma unroll
            for (int i = 0; i < TM; ++i) xa[i] = *(const lds_i32*)(st + (wm * C::WM + i * 32) * row);
#pragma unroll
            for (int j = 0; j < TN; ++j) xb[j] = *(const lds_i32*)(st + (C::BM + wn * C::WN + j * 32) * row);
        }
    };
    int xa[TM], xb[TN];
    auto mfmas = [&](const i32x4 (&fa)[TM], const i32x4 (&fb)[TN], auto step) {
        constexpr int ks = decltype(step)::value;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) {
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
    // issue order inside a sub-step: the reads of the next one follow the first half of the MFMAs, so that the wait at its top finds
    // them landed; direct loads follow the reads
    auto order = [&](auto extra_reads, auto loads) {
        constexpr int R = TM * (TA ? 2 : 1) + TN * (TB ? 2 : 1) + decltype(extra_reads)::value, MF = TM * TN, U = MF / 2 > 0 ? MF / 2 : 1, V = MF - U;
        constexpr int L = decltype(loads)::value;
        auto one = [&](auto u_) {
            constexpr int u = decltype(u_)::value;
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if constexpr (u < U) {
                constexpr int cnt = R * (u + 1) / U - R * u / U;
                if constexpr (cnt > 0) __builtin_amdgcn_sched_group_barrier(0x100, cnt, 0);
            } else if constexpr (L > 0) {
                constexpr int v = u - U, cnt = L * (v + 1) / V - L * v / V;
                if constexpr (cnt > 0) __builtin_amdgcn_sched_group_barrier(0x020, cnt, 0);
            }
        };
        group_each(one, std::make_integer_sequence<int, MF>{});
    };
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    using I2 = std::integral_constant<int, 2>;
    using I3 = std::integral_constant<int, 3>;
    // Order of the requests: scales, then for every stage B before A.  With a third stage of A the one wait of a stage leaves the last
    // request of A in flight: only half of a stage's bytes have one stage of time, the others two (8192^3, both operands plain: 851 us, so 808).
    issue_last_scales(0);
#pragma unroll
    for (int s = 0; s < C::NSA; ++s) {
        if (s < NS) issue_b(s, s, Yes{});
        issue_a(s, s, Yes{});
    }
    constexpr int LATE = (C::NSA - NS) * C::LA;                         // requests that may be in flight at a stage's wait
    QUAFF_WAIT_VMCNT((NS - 1) * (C::LA + C::LB) + LATE);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    int s = 0, s_a = 0;
    if (!MX4 && (wm * C::WM >= a.rows || wn * C::WN >= b.rows)) {
        // A wavefront whose part of the tile lies past the edge only fetches for the others: the same requests and barriers as below (8192 rows in eight
        // uneven groups, 4096 -> 4096: 355 us, so 347; 4-bit products gain nothing, their stages wait for the requests).
        for (int kt = 0; kt < stages; ++kt) {
            QUAFF_WAIT_VMCNT(LATE);
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            issue_b(kt + NS, s, Yes{});
            issue_a(kt + C::NSA, s_a, Yes{});
            s = s + 1 == NS ? 0 : s + 1;
            s_a = s_a + 1 == C::NSA ? 0 : s_a + 1;
        }
        QUAFF_WAIT_VMCNT(0);
        return;
    }
    i32x4 fa0[TM], fb0[TN], fa1[TM], fb1[TN];
    read_frags(0, 0, 0, fa0, fb0);
    read_scales(0, xa, xb, Yes{});
    auto stage = [&](int kt, auto zeros, auto with_scales) {
        const int next = s + 1 == NS ? 0 : s + 1, next_a = s_a + 1 == C::NSA ? 0 : s_a + 1;
        read_frags(s_a, s, 1, fa1, fb1);
        mfmas(fa0, fb0, I0{});
        order(I0{}, I0{});
        read_frags(s_a, s, 2, fa0, fb0);
        mfmas(fa1, fb1, I1{});
        order(I0{}, I0{});
        read_frags(s_a, s, 3, fa1, fb1);
        mfmas(fa0, fb0, I2{});
        order(I0{}, I0{});
        QUAFF_WAIT_VMCNT(LATE);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();                 // this stage has been read by everyone, the next one has landed
        asm volatile("" ::: "memory");
        int xa2[TM], xb2[TN];
        read_frags(next_a, next, 0, fa0, fb0);
        read_scales(kt + 1 < stages ? kt + 1 : kt, xa2, xb2, zeros);
        issue_b(kt + NS, s, zeros);
        issue_a(kt + C::NSA, s_a, zeros);
        constexpr bool SC = decltype(with_scales)::value;
        if constexpr (SC) issue_scales((kt + NS) >> 2);
        mfmas(fa1, fb1, I3{});
        order(std::integral_constant<int, MX4 ? TM + TN : 0>{}, std::integral_constant<int, C::LOADS + (SC ? C::LS : 0)>{});
#pragma unroll
        for (int i = 0; i < TM; ++i) xa[i] = xa2[i];
#pragma unroll
        for (int j = 0; j < TN; ++j) xb[j] = xb2[j];
        s = next;
        s_a = next_a;
    };
    // (copies of the loop body: a branch inside would keep loads and MFMAs apart)
    int kt = 0;
    if constexpr (MX4) {
        for (; kt + 8 <= stages; kt += 4) {
            stage(kt, No{}, No{});
            stage(kt + 1, No{}, No{});
            stage(kt + 2, No{}, Yes{});                  // requests stage kt + 4 and the scales of four more
            stage(kt + 3, No{}, No{});
        }
        if (kt + 4 < stages) issue_last_scales((kt >> 2) + 1);
        for (; kt < stages; ++kt) stage(kt, Yes{}, No{});
    } else {
        for (; kt < full - C::NSA; ++kt) stage(kt, No{}, No{});
        for (; kt < stages; ++kt) stage(kt, Yes{}, No{});
    }
    QUAFF_WAIT_VMCNT(0);
}

// The results of the largest tiles pass the L2 by (2048 x 5632 gradients of 16 groups: 307 us, so 285).  bf16 results of 4-bit products mostly gain
// (rows x contraction -> columns, kept in the L2 and so: 16384 x 1024 -> 8192 174 and 139 us, 4096 x 4096 -> 11008 139 and 128, 8192 rows of it 273 and
// 259), two of eight sizes lose (8192^3 329 and 346, 16384 x 2048 -> 5632 in eight groups 180 and 187).
template <class C, class T>
__device__ __forceinline__ void group_put(T v, T* p) {
    if constexpr (C::BM == 256) __builtin_nontemporal_store(v, p);
    else *p = v;
}

// Accumulator register e of a 32 x 32 block: row (e & 3) + 8 (e >> 2) + 4 half, column lane & 31.  A wavefront's fp32 store covers
// two rows x 128 bytes.  bf16: neighbouring lanes exchange values so that the even one holds columns c, c + 1 of register e and the odd
// one those of register e + 1 - half as many stores of four rows x 64 bytes.
// Whole tiles (FULL) store without comparisons.
template <class C, bool FULL>
__device__ __forceinline__ void group_store_tile(const GroupArgs& g, f32x16 (&acc)[C::TM][C::TN], float* c, uint16_t* c16, int rows, int cols,
                                                 int m0, int n0, int lane) {
    const int half4 = 4 * (lane >> 5), col = lane & 31;
    const float s = C::MX4 ? 1.0f : g.scale;
    if (c16) {
        const bool odd = lane & 1;
        const uint32_t at = (uint32_t)((half4 + odd) * g.ldc + col - odd) * 2;
        char* const base = reinterpret_cast<char*>(c16 + (int64_t)m0 * g.ldc + n0);
#pragma unroll
        for (int i = 0; i < C::TM; ++i)
#pragma unroll
            for (int j = 0; j < C::TN; ++j)
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const int row = i * 32 + (e & 3) + 8 * (e >> 2);
                    const float u = acc[i][j][e] * s, v = acc[i][j][e + 1] * s;
                    const float other = __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(odd ? u : v), 0xB1, 0xf, 0xf, true));
                    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
                    const bf16x2 pair = {(__bf16)(odd ? other : u), (__bf16)(odd ? v : other)};
                    if (FULL || (m0 + row + half4 + odd < rows && n0 + j * 32 + col < cols))
                        group_put<C>(__builtin_bit_cast(uint32_t, pair), reinterpret_cast<uint32_t*>(base + ((int64_t)row * g.ldc + j * 32) * 2 + at));
                }
        return;
    }
    const uint32_t at = (uint32_t)(half4 * g.ldc + col) * 4;
    char* const base = reinterpret_cast<char*>(c + (int64_t)m0 * g.ldc + n0);
#pragma unroll
    for (int i = 0; i < C::TM; ++i)
#pragma unroll
        for (int j = 0; j < C::TN; ++j) {
            if (g.accumulate) {                       // (all loads of a block before its stores)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int row = i * 32 + (e & 3) + 8 * (e >> 2);
                    float* p = reinterpret_cast<float*>(base + ((int64_t)row * g.ldc + j * 32) * 4 + at);
                    float old = 0.0f;
                    if (FULL || (m0 + row + half4 < rows && n0 + j * 32 + col < cols)) old = *p;
                    acc[i][j][e] = acc[i][j][e] * s + old;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] *= s;
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int row = i * 32 + (e & 3) + 8 * (e >> 2);
                if (FULL || (m0 + row + half4 < rows && n0 + j * 32 + col < cols))
                    group_put<C>(acc[i][j][e], reinterpret_cast<float*>(base + ((int64_t)row * g.ldc + j * 32) * 4 + at));
            }
        }
}

// c, c16: the tile's first element (one of them); m0, n0: the wavefront's part of the tile
template <class C>
__device__ __forceinline__ void group_store(const GroupArgs& g, f32x16 (&acc)[C::TM][C::TN], float* c, uint16_t* c16, int rows, int cols,
                                            int m0, int n0, int lane) {
    c = const_cast<float*>(group_uniform(c));
    c16 = const_cast<uint16_t*>(group_uniform(c16));
    if (m0 + C::WM <= rows && n0 + C::WN <= cols) group_store_tile<C, true>(g, acc, c, c16, rows, cols, m0, n0, lane);
    else if (m0 < rows && n0 < cols) group_store_tile<C, false>(g, acc, c, c16, rows, cols, m0, n0, lane);
}

// Eight fp32 values as three vectors of bf16 whose sum they are: eight of the 24 significant bits each.  The bits are cut off, not rounded,
// which keeps the largest values finite; the two differences are exact.  An infinity stays in the first (less itself it would be NaN).
__device__ __forceinline__ void split_bf16(const f32x4 (&x)[2], i32x4 (&out)[3]) {
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        uint32_t u[3][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float v = x[p >> 1][(p & 1) * 2 + h];
            u[0][h] = __float_as_uint(v);
            const float rest = __builtin_isinf(v) ? 0.0f : v - __uint_as_float(u[0][h] & 0xffff0000u);
            u[1][h] = __float_as_uint(rest);
            u[2][h] = __float_as_uint(rest - __uint_as_float(u[1][h] & 0xffff0000u));
        }
#pragma unroll
        for (int i = 0; i < 3; ++i) out[i][p] = (int)((u[i][1] & 0xffff0000u) | (u[i][0] >> 16));
    }
}

// Low-rank term: the sum of T's parts, all 24 bits of it as three bf16 values, times the group's bf16 factor.  Both go through the
// LDS that the main loop has left, in one round trip (fragments fetched from global memory one by one: 4096 x 4096 -> 11008 at rank 64
// 205 us, so 140 with a pair of 16 bits; in another run 150 with the pair, so 152).  Three planes of T and a plain factor have rows of 32, 64 or 128 bytes; 16-byte chunks swapped by row so
// that a fragment's reads are spread over the banks.
__device__ __forceinline__ int low_rank_slot(int stride, int row, int chunk) {
    const int per = 256 / stride, mask = stride / 16 - 1;                      // rows that cover all banks, chunks of a row
    return row * stride + ((chunk ^ ((row / per) & mask)) * 16);
}

template <class C>
__device__ __forceinline__ void group_low_rank(const GroupArgs& g, const GroupTile& gt, f32x16 (&acc)[C::TM][C::TN], int m0, int n0, int col0,
                                               int cols, lds_i8* lds, int lane) {
    const int r = g.r, tid = threadIdx.x;
    const int lb = r == 16 ? 32 : r == 32 ? 64 : 128;                           // bytes of a row
    constexpr int PLANE = C::BM * 128;
    lds_i8* const at = lds;
    lds_i8* const bt = lds + 3 * PLANE;
    static_assert(3 * PLANE + C::BN * 128 <= C::LDS_BYTES, "room for both operands");
    const uint16_t* const L = g.L + (int64_t)gt.group * g.N * r;
    using S = GroupStage<C::BN, true>;
    __syncthreads();                                                            // the main loop's stages have been read
    for (int i = tid; i < C::BN * r / 8; i += C::NT) {
        if (g.l_rn) {
            const int k = i / (C::BN / 8), c = i % (C::BN / 8);
            i32x4 v = {0, 0, 0, 0};
            if (c * 8 < cols) v = *reinterpret_cast<const i32x4*>(L + (int64_t)k * g.N + col0 + c * 8);
            *(lds_i32x4*)(bt + k * S::RB + (((c >> 2) ^ S::swz(k)) * 4 + (c & 3)) * 16) = v;
        } else {
            const int row = i / (r / 8), c = i % (r / 8);
            i32x4 v = {0, 0, 0, 0};
            if (row < cols) v = *reinterpret_cast<const i32x4*>(L + (int64_t)(col0 + row) * r + c * 8);
            *(lds_i32x4*)(bt + low_rank_slot(lb, row, c)) = v;
        }
    }
    for (int i = tid; i < C::BM * r / 8; i += C::NT) {
        const int row = i / (r / 8), c = i % (r / 8);
        f32x4 x[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
        if (row < gt.rows) {
            const f32x4* p = reinterpret_cast<const f32x4*>(g.T + (int64_t)(gt.row0 + row) * r + c * 8);
            for (int q = 0; q < g.t_parts; ++q, p += (int64_t)g.t * r / 4) {
                x[0] += p[0];
                x[1] += p[1];
            }
        }
        i32x4 planes[3];
        split_bf16(x, planes);
#pragma unroll
        for (int p = 0; p < 3; ++p) *(lds_i32x4*)(at + p * PLANE + low_rank_slot(lb, row, c)) = planes[p];
    }
    __syncthreads();
    const int r32 = lane & 31, half = lane >> 5;
    const int tr_i = lane & 15, tr_row = half * 8 + (tr_i >> 2), tr_in = ((lane >> 4) & 1) * 32 + (tr_i & 3) * 8;
    for (int k0 = 0; k0 < r; k0 += 16) {
        i32x4 fb[C::TN];
#pragma unroll
        for (int j = 0; j < C::TN; ++j) {
            if (g.l_rn) {
                const lds_i8* p = bt + (k0 + tr_row) * S::RB + ((((n0 >> 5) + j) ^ S::swz(tr_row)) * 64) + tr_in;
                union { i16x4 h[2]; i32x4 v; } u;
                u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)p);
                u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(p + 4 * S::RB));
                fb[j] = u.v;
            } else {
                fb[j] = *(const lds_i32x4*)(bt + low_rank_slot(lb, n0 + j * 32 + r32, k0 / 8 + half));
            }
        }
#pragma unroll
        for (int i = 0; i < C::TM; ++i) {
            const int row = m0 + i * 32 + r32;
            i32x4 fa[3];
#pragma unroll
            for (int p = 0; p < 3; ++p) fa[p] = *(const lds_i32x4*)(at + p * PLANE + low_rank_slot(lb, row, k0 / 8 + half));
#pragma unroll
            for (int p = 0; p < 3; ++p)
#pragma unroll
                for (int j = 0; j < C::TN; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fa[p]), __builtin_bit_cast(bf16x8, fb[j]), acc[i][j], 0, 0, 0);
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

// one tile: rows gt.row0 ... of gt.group, columns from n0 on
template <class C>
__device__ __forceinline__ void group_rows_tile(const GroupArgs& g, const GroupTile& gt, int n0, int8_t* lds_raw) {
    constexpr bool MX4 = C::MX4, TB = C::TB;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int cols = g.N - n0 < C::BN ? g.N - n0 : C::BN;
    GroupOperand a{static_cast<const char*>(g.A) + (int64_t)gt.row0 * g.lda, g.lda, gt.rows};
    GroupOperand b{static_cast<const char*>(g.B) + (int64_t)gt.group * g.b_group + (TB ? (int64_t)n0 * 2 : (int64_t)n0 * g.ldb), g.ldb, cols};
    const uint8_t* sa = MX4 ? g.SA + (int64_t)gt.row0 * g.ld_scale : nullptr;
    const uint8_t* sb = MX4 ? g.SB + (int64_t)gt.group * g.sb_group + (int64_t)n0 * g.ld_scale : nullptr;
    f32x16 acc[C::TM][C::TN];
    group_clear<C>(acc);
    int stages = (g.K + (MX4 ? 255 : 63)) / (MX4 ? 256 : 64), k_valid = g.K;
    float* c = g.C;
    bool first = true;
    if constexpr (C::BM <= 128 && C::NW == 4) {
        if (g.k_parts > 1) {                          // this workgroup's part of the contraction
            const int per = (stages + g.k_parts - 1) / g.k_parts, from = blockIdx.y * per;
            stages = stages - from < per ? stages - from : per;
            k_valid = k_valid - from * 64 < per * 64 ? k_valid - from * 64 : per * 64;
            a.p += (int64_t)from * 128;
            b.p += TB ? (int64_t)from * 64 * g.ldb : (int64_t)from * 128;
            sa += from * 8;
            sb += from * 8;
            c = g.partial + (int64_t)blockIdx.y * g.t * g.N;
            first = from == 0;
        }
    }
    group_mainloop<C>(a, b, sa, sb, g.ld_scale, stages, k_valid, (lds_i8*)lds_raw, group_ring(lds_raw), wave, lane, acc);
    const int m0 = (wave / C::WGN) * C::WM, nw = (wave % C::WGN) * C::WN;
    if constexpr (MX4) if (g.r && first) group_low_rank<C>(g, gt, acc, m0, nw, n0, cols, (lds_i8*)lds_raw, lane);
    const int64_t at = (int64_t)gt.row0 * g.ldc + n0;
    group_store<C>(g, acc, c ? c + at : nullptr, g.C16 ? g.C16 + at : nullptr, gt.rows, cols, m0, nw, lane);
}

template <int BM, int BN, int WGM, int WGN, int NS, bool MX4, bool TB>
__global__ void __launch_bounds__(WGM * WGN * 64) group_rows_kernel(GroupArgs g) {
    using C = GroupCfg<BM, BN, WGM, WGN, NS, MX4, false, TB>;
    constexpr bool QUARTERS = BM == 256 && BN == 256;
    using Q = GroupCfg<BM / (QUARTERS ? 2 : 1), BN / (QUARTERS ? 2 : 1), WGM, WGN, NS, MX4, false, TB>;
    __shared__ __attribute__((aligned(1024))) int8_t lds_raw[C::LDS_BYTES];
    GroupTile gt;
    if (!find_group_tile<8, QUARTERS>(g.offsets, g.n_groups, g.t, BM, (g.N + BN - 1) / BN, gt)) return;
    int n0 = gt.tn * BN;
    if constexpr (QUARTERS) {
        if (gt.quarter >= 0) {
            const int down = (gt.quarter >> 1) * (BM / 2);
            n0 += (gt.quarter & 1) * (BN / 2);
            gt.row0 += down;
            gt.rows -= down;
            if (gt.rows <= 0 || n0 >= g.N) return;
            if (gt.rows > BM / 2) gt.rows = BM / 2;
            group_rows_tile<Q>(g, gt, n0, lds_raw);
            return;
        }
    }
    group_rows_tile<C>(g, gt, n0, lds_raw);
}

// SPLIT: the rows of a group in slabs of g.slab rows; a group of one slab is written to the result, the slabs of others to g.partial, where
// group_reduce_kernel sums them in order.  Otherwise every tile takes all rows of its group.
template <int BM, int BN, int WGM, int WGN, int NS, bool SPLIT>
__global__ void __launch_bounds__(WGM * WGN * 64) group_ragged_kernel(GroupArgs g) {
    using C = GroupCfg<BM, BN, WGM, WGN, NS, false, true, true>;
    __shared__ __attribute__((aligned(1024))) int8_t lds_raw[C::LDS_BYTES];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int tiles_n = (g.N + BN - 1) / BN, tiles = (g.M + BM - 1) / BM * tiles_n;
    int begin, len, tile;
    float* c;
    if constexpr (SPLIT) {
        GroupTile gt;
        if (!find_group_tile<1>(g.offsets, g.n_groups, g.t, g.slab, tiles, gt)) return;
        begin = gt.row0;
        len = gt.rows;
        tile = gt.tn;
        c = gt.len <= g.slab ? g.C + (int64_t)gt.group * g.c_group : g.partial + (int64_t)gt.tm * g.c_group;
    } else {
        // (one after the other to all XCDs: an eighth of the tiles each, as in find_group_tile, leaves the XCD with the busiest groups
        // alone at the end - 2048 x 5632, 16 uneven groups of 512 rows on average: 435 us, so 308)
        const int group = (int)(blockIdx.x / (uint32_t)tiles);
        tile = (int)(blockIdx.x - (uint32_t)group * (uint32_t)tiles);
        begin = group_bound(g.offsets, group, g.t);
        const int end = group_bound(g.offsets, group + 1, g.t);
        len = __builtin_amdgcn_readfirstlane(end > begin ? end - begin : 0);
        begin = __builtin_amdgcn_readfirstlane(begin);
        c = g.C + (int64_t)group * g.c_group;
    }
    const int m0 = tile / tiles_n * BM, n0 = tile % tiles_n * BN;
    const int rows = g.M - m0 < BM ? g.M - m0 : BM, cols = g.N - n0 < BN ? g.N - n0 : BN;
    GroupOperand a{static_cast<const char*>(g.A) + (int64_t)begin * g.lda + (int64_t)m0 * 2, g.lda, rows};
    GroupOperand b{static_cast<const char*>(g.B) + (int64_t)begin * g.ldb + (int64_t)n0 * 2, g.ldb, cols};
    f32x16 acc[C::TM][C::TN];
    group_clear<C>(acc);
    group_mainloop<C>(a, b, nullptr, nullptr, 0, (len + 63) / 64, len, (lds_i8*)lds_raw, group_ring(lds_raw), wave, lane, acc);
    group_store<C>(g, acc, c + (int64_t)m0 * g.ldc + n0, nullptr, rows, cols, (wave / WGN) * C::WM, (wave % WGN) * C::WN, lane);
}

// ---- host side -----------------------------------------------------------------------------------------------------
// most row tiles that t rows in n_groups groups can have
inline int64_t group_row_tiles(const GroupArgs& g, int bm) {
    if (!g.offsets) return (g.t + bm - 1) / bm;
    return g.t / bm + (g.n_groups < g.t ? g.n_groups : g.t);
}

template <int BM, int BN, int WGM, int WGN, int NS, bool MX4, bool TB>
static hipError_t launch_group_rows_shape(const GroupArgs& g, hipStream_t stream) {
    const int64_t tiles = group_row_tiles(g, BM) * ((g.N + BN - 1) / BN);
    if (tiles + 1024 > 0x7fffffff) return hipErrorInvalidValue;
    // (the tiles beyond whole rounds may be four workgroups each)
    const int64_t groups = (tiles + 7) / 8 * 8 + (BM == 256 && BN == 256 ? 3 * kUnits / 4 + 8 : 0);
    group_rows_kernel<BM, BN, WGM, WGN, NS, MX4, TB><<<dim3((unsigned)groups, g.k_parts > 1 ? g.k_parts : 1), dim3(WGM * WGN * 64), 0, stream>>>(g);
    return hipGetLastError();
}

// the tile that group_rows_plan has chosen, and the join of a shared contraction
template <bool MX4, bool TB>
static hipError_t launch_group_rows(const GroupArgs& g, int prof_kind, hipStream_t stream) {
    GroupArgs p = g;
    if (g.k_parts > 1) {
        if (g.tile > 128) return hipErrorInvalidValue;
        p.C = nullptr;
        p.C16 = nullptr;
        p.ldc = g.N;
        p.scale = 1.0f;
        p.accumulate = 0;
    }
    hipError_t e;
    {
        ProfScope prof(prof_kind, stream);
        if (g.tile == 256) e = launch_group_rows_shape<256, 256, 2, 4, 2, MX4, TB>(p, stream);
        else if (g.tile == 128) e = launch_group_rows_shape<128, 128, 2, 2, 2, MX4, TB>(p, stream);
        else e = launch_group_rows_shape<64, 64, 2, 2, 2, MX4, TB>(p, stream);
    }
    if (e != hipSuccess || g.k_parts <= 1) return e;
    ProfScope prof(prof_kind, stream);
    return launch_group_join(g, stream);
}

template <int BM, int BN, int WGM, int WGN, int NS>
static hipError_t launch_group_ragged(const GroupArgs& g, hipStream_t stream) {
    const int64_t tiles = (int64_t)((g.M + BM - 1) / BM) * ((g.N + BN - 1) / BN);
    const int64_t all = tiles * (g.slab ? group_row_tiles(g, g.slab) : g.n_groups);
    if (all + 7 > 0x7fffffff) return hipErrorInvalidValue;
    const dim3 grid((unsigned)(g.slab ? (all + 7) / 8 * 8 : all)), block(WGM * WGN * 64);
    if (g.slab) {
        if constexpr (BM < 256) group_ragged_kernel<BM, BN, WGM, WGN, NS, true><<<grid, block, 0, stream>>>(g);
        else return hipErrorInvalidValue;              // (group_ragged_tile: slabs and the large tile exclude each other)
    } else group_ragged_kernel<BM, BN, WGM, WGN, NS, false><<<grid, block, 0, stream>>>(g);
    return hipGetLastError();
}

}  // namespace quaff
