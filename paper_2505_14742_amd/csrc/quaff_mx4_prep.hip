// What a 4-bit layer with an adapter needs of its input before the product, in one pass over X: its 4-bit codes and scales
// (quaff_mx4.hip has the arithmetic) and the adapter's down-projection T = scale X L (L [k x r], or [r x k] read transposed).
//
// HBM-bound in X: 2 k bytes per row read, 17 k / 32 + 4 r written.  A lane holds 32 consecutive values of a row - one block, whose
// scale it finds without another lane - as four fragments of v_mfma_f32_16x16x32_bf16 (row = lane & 15, contraction values
// 32 (lane >> 4) + 8 j ... of a step of 128; the factor's fragments take the same order).  A workgroup takes 16 rows of one
// group and a part of the contraction, its four wavefronts every fourth step of it; the sums of the wavefronts are joined in LDS, those
// of the parts by the product's epilogue, both in a fixed order.
#include "quaff_group_gemm.h"
#include "quaff_mx4_body.h"

namespace quaff {

// The factor of a step goes through LDS, every wavefront on its own.  L_KR: L is [k x r], gathered with transposing reads.  Otherwise
// [r x k]: 256 bytes of r rows, 16-byte chunk c of row p in slot c ^ (p & 15) (read from global memory as fragments, 64-byte pieces of rows: 4096 x
// 11008 at rank 64 74 us, so 53).
template <int R16, bool L_KR>
__global__ void __launch_bounds__(256) mx4_prep_kernel(Mx4PrepArgs g) {
    constexpr int r = R16 * 16, QBYTES = 32 * r * 2, QSTRIDE = QBYTES + 128;       // 32 contraction rows of L; padded to spread the banks
    constexpr int STAGE = L_KR ? 4 * QSTRIDE : r * 256, RED = 16 * r * 4;
    constexpr int LDS = 4 * STAGE > 4 * RED ? 4 * STAGE : 4 * RED;
    __shared__ __attribute__((aligned(1024))) int8_t lds_raw[LDS];
    GroupTile gt;
    if (!find_group_tile<1>(g.offsets, g.n_groups, g.t, 16, g.parts, gt)) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, q = lane >> 4;
    const uint16_t* L = g.L + (int64_t)gt.group * g.k * r;
    const int steps = g.kp / 128, first = gt.tn * g.steps_per_part;
    const int last = first + g.steps_per_part < steps ? first + g.steps_per_part : steps;
    const bool valid = n < gt.rows;
    const int64_t row = gt.row0 + (valid ? n : gt.rows - 1);
    lds_i8* const stage = (lds_i8*)lds_raw + wave * STAGE;
    i32x4 x[4];
    auto load = [&](int s) {
        const int kk = s * 128 + q * 32;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[j] = (i32x4){0, 0, 0, 0};
            if (kk + j * 8 < g.k) x[j] = *reinterpret_cast<const i32x4*>(g.X + row * g.ldx + kk + j * 8);
        }
#pragma unroll
        for (int i = 0; i < 4 * R16; ++i) {
            if constexpr (L_KR) {
                const int at = i * 1024 + lane * 16, left = (g.k - s * 128) * r * 2;      // bytes of L from here on (k may end before the step does)
                const char* src = reinterpret_cast<const char*>(L) + (int64_t)s * 128 * r * 2 + at;
                dma_load_16<false>(at < left ? src : reinterpret_cast<const char*>(kZeroChunk), stage + (i / R16) * QSTRIDE + (i % R16) * 1024);
            } else {
                const int p = i * 4 + (lane >> 4), kc = s * 128 + ((lane & 15) ^ (p & 15)) * 8;
                const void* src = kc < g.k ? static_cast<const void*>(L + (int64_t)p * g.k + kc) : static_cast<const void*>(kZeroChunk);
                dma_load_16<false>(src, stage + i * 1024);
            }
        }
    };
    f32x4 acc[R16];
#pragma unroll
    for (int c = 0; c < R16; ++c) acc[c] = (f32x4){0.f, 0.f, 0.f, 0.f};
    int s = first + wave;
    if (s < last) load(s);
    for (; s < last; s += 4) {
        i32x4 xc[4], lc[R16][4];
        QUAFF_WAIT_VMCNT(0);
#pragma unroll
        for (int c = 0; c < R16; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (L_KR) {
                    const lds_i8* p = stage + q * QSTRIDE + (j * 8 + (n >> 2)) * (r * 2) + c * 32 + (n & 3) * 8;
                    union { i16x4 h[2]; i32x4 v; } u;
                    u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)p);
                    u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(p + 4 * r * 2));
                    lc[c][j] = u.v;
                } else {
                    lc[c][j] = *(const lds_i32x4*)(stage + (c * 16 + n) * 256 + ((q * 4 + j) ^ n) * 16);
                }
            }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");            // read before the next step's rows arrive
#pragma unroll
        for (int j = 0; j < 4; ++j) xc[j] = x[j];
        if (s + 4 < last) load(s + 4);
        const int kk = s * 128 + q * 32;
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) m = mx4_max_bits(m, xc[j]);
        const uint32_t byte = mx4_scale_byte(m >> 7);
        const float sv = mx4_scale_value(byte);
        i32x4 codes;
#pragma unroll
        for (int j = 0; j < 4; ++j) codes[j] = (int)mx4_code8_bf16(xc[j], sv);
        if (valid) {
            *reinterpret_cast<i32x4*>(g.codes + row * (g.kp / 2) + kk / 2) = codes;
            g.scales[row * (g.kp / 32) + kk / 32] = (uint8_t)byte;
        }
#pragma unroll
        for (int c = 0; c < R16; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, xc[j]), __builtin_bit_cast(bf16x8, lc[c][j]), acc[c], 0, 0, 0);
    }
    // accumulator register i of a 16 x 16 block: row 4 q + i, column n
    __syncthreads();
    lds_f32* const red = (lds_f32*)lds_raw;
#pragma unroll
    for (int c = 0; c < R16; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) red[wave * (16 * r) + (4 * q + i) * r + c * 16 + n] = acc[c][i];
    __syncthreads();
    float* const T = g.T + ((int64_t)gt.tn * g.t + gt.row0) * r;
    for (int i = tid; i < gt.rows * r; i += 256) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) v += red[w * (16 * r) + i];
        T[i] = v * g.scale;
    }
}

// The same for groups of many rows: 64 rows of a group to a workgroup, 16 to a wavefront, whose X and factor stream through a ring of
// three steps of 128 contraction values.  X is read in whole 256-byte pieces of rows (the lanes' own blocks straight from global memory are
// 64-byte pieces in four loads: 16384 x 13824 at rank 16 163 us, so 138), the factor once for 64 rows.  One barrier a step; rows past the end
// of a group repeat its last one, with the same values to the same place, so that every wavefront has the same number of
// requests in flight.
template <int R16, bool L_KR>
__global__ void __launch_bounds__(256) mx4_prep_tile_kernel(Mx4PrepArgs g) {
    constexpr int r = R16 * 16, QSTRIDE = 32 * r * 2 + 128, NS = 3;
    constexpr int XBYTES = 64 * 256, LBYTES = L_KR ? 4 * QSTRIDE : r * 256, STEP = XBYTES + LBYTES;
    constexpr int LOADS = 4 + R16;                                              // of a wavefront per step
    __shared__ __attribute__((aligned(1024))) int8_t lds_raw[NS * STEP];
    GroupTile gt;
    if (!find_group_tile<1>(g.offsets, g.n_groups, g.t, 64, g.parts, gt)) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, q = lane >> 4;
    const char* const L = reinterpret_cast<const char*>(g.L + (int64_t)gt.group * g.k * r);
    const int steps = g.kp / 128, first = gt.tn * g.steps_per_part;
    const int last = first + g.steps_per_part < steps ? first + g.steps_per_part : steps;
    lds_i8* const lds = (lds_i8*)lds_raw;
    auto tile_row = [&](int i) { return (int64_t)gt.row0 + (i < gt.rows ? i : gt.rows - 1); };
    // rows of this wavefront's X loads: load i takes rows 4 i + lane / 16, 16-byte chunk c of row p in slot c ^ p
    const char* xrow[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) xrow[i] = reinterpret_cast<const char*>(g.X + tile_row(wave * 16 + i * 4 + (lane >> 4)) * g.ldx);
    auto issue = [&](int s, int buf) {
        if (s >= last) s = last - 1;                                            // (a harmless repeat)
        lds_i8* const st = lds + buf * STEP;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int k = s * 128 + ((lane & 15) ^ (i * 4 + (lane >> 4))) * 8;
            dma_load_16<true>(k < g.k ? xrow[i] + (int64_t)k * 2 : reinterpret_cast<const char*>(kZeroChunk), st + wave * 4096 + i * 1024);
        }
#pragma unroll
        for (int j = 0; j < R16; ++j) {
            const int i = j * 4 + wave;                                         // of 4 R16 loads
            if constexpr (L_KR) {
                const int at = i * 1024 + lane * 16, left = (g.k - s * 128) * r * 2;
                dma_load_16<true>(at < left ? L + (int64_t)s * 128 * r * 2 + at : reinterpret_cast<const char*>(kZeroChunk),
                                   st + XBYTES + (i / R16) * QSTRIDE + (i % R16) * 1024);
            } else {
                const int p = i * 4 + (lane >> 4), k = s * 128 + ((lane & 15) ^ (p & 15)) * 8;
                dma_load_16<true>(k < g.k ? L + ((int64_t)p * g.k + k) * 2 : reinterpret_cast<const char*>(kZeroChunk), st + XBYTES + i * 1024);
            }
        }
    };
    const int64_t row = tile_row(wave * 16 + n);
    uint8_t* const codes = g.codes + row * (g.kp / 2);
    uint8_t* const scales = g.scales + row * (g.kp / 32);
    f32x4 acc[R16];
#pragma unroll
    for (int c = 0; c < R16; ++c) acc[c] = (f32x4){0.f, 0.f, 0.f, 0.f};
    auto step = [&](int s, int buf, auto stores_in_flight) {
        // behind this step's loads: those of the next step, and the two stores of each of the last two steps
        QUAFF_WAIT_VMCNT(LOADS + decltype(stores_in_flight)::value);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        issue(s + 2, buf + 2 >= NS ? buf + 2 - NS : buf + 2);
        const lds_i8* const st = lds + buf * STEP;
        i32x4 x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = *(const lds_i32x4*)(st + wave * 4096 + n * 256 + ((q * 4 + j) ^ n) * 16);
        i32x4 lc[R16][4];
#pragma unroll
        for (int c = 0; c < R16; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (L_KR) {
                    const lds_i8* p = st + XBYTES + q * QSTRIDE + (j * 8 + (n >> 2)) * (r * 2) + c * 32 + (n & 3) * 8;
                    union { i16x4 h[2]; i32x4 v; } u;
                    u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)p);
                    u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(p + 4 * r * 2));
                    lc[c][j] = u.v;
                } else {
                    lc[c][j] = *(const lds_i32x4*)(st + XBYTES + (c * 16 + n) * 256 + ((q * 4 + j) ^ n) * 16);
                }
            }
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) m = mx4_max_bits(m, x[j]);
        const uint32_t byte = mx4_scale_byte(m >> 7);
        const float sv = mx4_scale_value(byte);
        i32x4 out;
#pragma unroll
        for (int j = 0; j < 4; ++j) out[j] = (int)mx4_code8_bf16(x[j], sv);
        *reinterpret_cast<i32x4*>(codes + s * 64 + q * 16) = out;
        scales[s * 4 + q] = (uint8_t)byte;
#pragma unroll
        for (int c = 0; c < R16; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x[j]), __builtin_bit_cast(bf16x8, lc[c][j]), acc[c], 0, 0, 0);
    };
    if (first < last) {
        issue(first, 0);
        issue(first + 1, 1);
        int buf = 0;
        auto next = [&] { buf = buf + 1 == NS ? 0 : buf + 1; };
        int s = first;
        step(s++, buf, std::integral_constant<int, 0>{});
        next();
        if (s < last) {
            step(s++, buf, std::integral_constant<int, 2>{});
            next();
        }
        for (; s < last; ++s) {
            step(s, buf, std::integral_constant<int, 4>{});
            next();
        }
        QUAFF_WAIT_VMCNT(0);
    }
    float* const T = g.T + ((int64_t)gt.tn * g.t + gt.row0) * r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int rr = wave * 16 + 4 * q + i;
        if (rr < gt.rows)
#pragma unroll
            for (int c = 0; c < R16; ++c) T[rr * r + c * 16 + n] = acc[c][i] * g.scale;
    }
}

// rows per group from which on 64 of them share a workgroup
static bool mx4_prep_tiles(int64_t t, int32_t n_groups) { return t / (n_groups > 0 ? n_groups : 1) >= 48; }

// Parts of the contraction: up to two workgroups of 16 rows a compute unit, 1.25 of 64 rows, and eight parts; before the steps are shared out evenly
// that is at least eight steps a part (two to a wavefront), four with 64 rows (whose wavefronts take all of them).  The last part may have
// fewer, none is empty: its zeros would be written, and read by every tile of the product.
int mx4_prep_parts(int64_t t, int64_t k, int32_t n_groups) {
    const int64_t partial = n_groups > 0 ? (n_groups < t ? n_groups : t) : 1;
    const bool large = mx4_prep_tiles(t, n_groups);
    const int64_t tiles = t / (large ? 64 : 16) + partial, most = mx4_padded(k) / 128 / (large ? 4 : 8);
    int64_t parts = (large ? 320 : 512) / (tiles > 0 ? tiles : 1);
    if (parts > most) parts = most;
    if (parts > kMx4MaxParts) parts = kMx4MaxParts;
    if (parts < 1) return 1;
    const int64_t steps = mx4_padded(k) / 128, per = (steps + parts - 1) / parts;
    return (int)((steps + per - 1) / per);
}

hipError_t launch_mx4_prep(Mx4PrepArgs g, int32_t r, bool l_kr, hipStream_t stream) {
    if (g.t == 0) return hipSuccess;
    ProfScope prof(K_MX4_QUANT, stream);
    const int steps = g.kp / 128;
    g.steps_per_part = (steps + g.parts - 1) / g.parts;
    const int64_t partial = g.offsets ? (g.n_groups < g.t ? g.n_groups : g.t) : 1;
    const bool large = mx4_prep_tiles(g.t, g.offsets ? g.n_groups : 0);
    const int64_t tiles = (g.t / (large ? 64 : 16) + partial) * g.parts;
    const dim3 grid((unsigned)((tiles + 7) / 8 * 8)), block(256);
#define QUAFF_PREP(R)                                                                             \
    if (r == 16 * R) {                                                                            \
        if (large && l_kr) mx4_prep_tile_kernel<R, true><<<grid, block, 0, stream>>>(g);          \
        else if (large) mx4_prep_tile_kernel<R, false><<<grid, block, 0, stream>>>(g);            \
        else if (l_kr) mx4_prep_kernel<R, true><<<grid, block, 0, stream>>>(g);                   \
        else mx4_prep_kernel<R, false><<<grid, block, 0, stream>>>(g);                            \
        return hipGetLastError();                                                                 \
    }
    QUAFF_PREP(1)
    QUAFF_PREP(2)
    QUAFF_PREP(3)
    QUAFF_PREP(4)
#undef QUAFF_PREP
    return hipErrorInvalidValue;
}

}  // namespace quaff
