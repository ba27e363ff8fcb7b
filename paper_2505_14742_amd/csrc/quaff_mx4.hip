// 4-bit microscaled floating point: blocks of 32 values along the contraction axis share a power-of-two scale.
//     E    = clamp(floor(log2 max|x|) - 2, -127, 127)          stored as the byte E + 127 (E8M0)
//     code = sign and nearest of {0, .5, 1, 1.5, 2, 3, 4, 6} to |x| 2^-E, ties to the even code, beyond 6 to 6 (E2M1)
// Dividing by a power of two is exact, so the codes are a function of the inputs alone: no order of operations enters.
// The exponent is taken from the bits of the largest magnitude, the codes from v_cvt_scalef32_pk_fp4 (which rounds as above
// for every input, scale and tie).  A block that holds an infinity or a NaN gets the scale byte 255 (NaN).
// Stored rows are padded to a multiple of 256 values: 128 bytes of codes (even values in the low four bits) and 8 scales,
// whole cache lines that a stage of the product takes without a case for the end of a row.  The padding holds zeros.
// HBM-bound: inputs are read once, 17 bytes per 32 values are written.
#include "quaff_mx4_body.h"

namespace quaff {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
    uint32_t o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xf, 0xf, true);      // lanes 1 0 3 2
    v = v > o ? v : o;
    o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xf, 0xf, true);               // lanes 2 3 0 1
    return v > o ? v : o;
}

// bf16 rows: four lanes to a block, eight values each
__global__ void __launch_bounds__(256) mx4_quantize_kernel(const uint16_t* __restrict__ X, int64_t rows, int k, int kp, int64_t ldx,
                                                           uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
    const int per_row = kp / 8;
    const int64_t n = rows * per_row;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / per_row;
        const int col = (int)(i - row * per_row) * 8;
        u32x4 x = {0u, 0u, 0u, 0u};
        if (col < k) x = *reinterpret_cast<const u32x4*>(X + row * ldx + col);
        const uint32_t m = quad_max(mx4_max_bits(0u, x));
        const uint32_t byte = mx4_scale_byte(m >> 7);
        const float s = mx4_scale_value(byte);
        const uint32_t c = mx4_code8_bf16(x, s);
        *reinterpret_cast<uint32_t*>(codes + row * (kp / 2) + col / 2) = c;
        if ((threadIdx.x & 3) == 0) scales[row * (kp / 32) + col / 32] = (uint8_t)byte;
    }
}

hipError_t launch_mx4_quantize(const uint16_t* X, int64_t rows, int64_t k, int64_t ldx, uint8_t* codes, uint8_t* scales, hipStream_t stream) {
    if (rows == 0) return hipSuccess;
    ProfScope prof(K_MX4_QUANT, stream);
    const int64_t kp = mx4_padded(k), blocks = (rows * (kp / 8) + 255) / 256;
    mx4_quantize_kernel<<<dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, stream>>>(X, rows, (int)k, (int)kp, ldx, codes, scales);
    return hipGetLastError();
}

// Codes back to the values they stand for, exact in bf16 (two significant bits; 2^-128 .. 6 x 2^127 past the largest finite
// value becomes an infinity as any conversion would make it)
__device__ __forceinline__ float mx4_value(uint32_t code, uint32_t byte) {
    if (byte == 255) return __uint_as_float(0x7fc00000u);
    // 2 |code| of codes 0 .. 7: 0 1 2 3 4 6 8 12
    const uint32_t twice = (0xC8643210u >> (4 * (code & 7))) & 15u;
    const float v = ldexpf((float)twice, (int)byte - 128);
    return (code & 8) ? -v : v;
}

__global__ void __launch_bounds__(256) mx4_dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t rows,
                                                             int k, int kp, uint16_t* __restrict__ out, int64_t ldo) {
    const int per_row = k / 8;
    const int64_t n = rows * per_row;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / per_row;
        const int col = (int)(i - row * per_row) * 8;
        const uint32_t c = *reinterpret_cast<const uint32_t*>(codes + row * (kp / 2) + col / 2);
        const uint32_t byte = scales[row * (kp / 32) + col / 32];
        u32x4 o;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            bf16x2 v;
            v[0] = (__bf16)mx4_value((c >> (8 * j)) & 15, byte);
            v[1] = (__bf16)mx4_value((c >> (8 * j + 4)) & 15, byte);
            o[j] = __builtin_bit_cast(uint32_t, v);
        }
        *reinterpret_cast<u32x4*>(out + row * ldo + col) = o;
    }
}

hipError_t launch_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t k, uint16_t* out, int64_t ldo,
                                 hipStream_t stream) {
    if (rows == 0) return hipSuccess;
    ProfScope prof(K_MX4_QUANT, stream);
    const int64_t blocks = (rows * (k / 8) + 255) / 256;
    mx4_dequantize_kernel<<<dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, stream>>>(codes, scales, rows, (int)k,
                                                                                                        (int)mx4_padded(k), out, ldo);
    return hipGetLastError();
}

// Both 4-bit copies of a frozen fp32 weight W [c_in x c_out] in one pass over it: tiles of 128 x 128 go through LDS; blocks along the output
// channels (input gradient) lie in rows of the tile, blocks along the input channels (forward) in columns.  Four lanes write 64
// bytes of a stored row (tiles of 256 x 32, whose rows gave 16 bytes: 4096 x 11008 76 us, so 65).
constexpr int kPrepTile = 128;

__device__ __forceinline__ uint32_t mx4_code8(const float* v, float s) {
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], s, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], s, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], s, 3);
    return c;
}

// `stride`: LDS floats between the values of the block; codes and scale go to `codes`, `scale`
__device__ __forceinline__ void mx4_block(const float* p, int stride, uint8_t* codes, uint8_t* scale) {
    float v[32];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        v[i] = p[i * stride];
        const uint32_t b = __float_as_uint(v[i]) & 0x7fffffffu;
        m = m > b ? m : b;
    }
    const uint32_t byte = mx4_scale_byte(m >> 23);
    const float s = mx4_scale_value(byte);
    u32x4 c;
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = mx4_code8(v + 8 * i, s);
    *reinterpret_cast<u32x4*>(codes) = c;
    *scale = (uint8_t)byte;
}

__global__ void __launch_bounds__(256) mx4_prepare_kernel(const float* __restrict__ W, int c_in, int c_out, int64_t ldw, int kp_in, int kp_out,
                                                          uint8_t* __restrict__ codes_f, uint8_t* __restrict__ scales_f,
                                                          uint8_t* __restrict__ codes_b, uint8_t* __restrict__ scales_b) {
    constexpr int LD = kPrepTile + 1;
    __shared__ float tile[kPrepTile * LD];
    const int tid = threadIdx.x, j0 = blockIdx.x * kPrepTile, k0 = blockIdx.y * kPrepTile;
    const int64_t e = blockIdx.z;
    W += e * c_in * ldw;
    f32x4 x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int r = i * 8 + (tid >> 5), c = (tid & 31) * 4;
        x[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
        if (k0 + r < c_in && j0 + c < c_out) x[i] = *reinterpret_cast<const f32x4*>(W + (int64_t)(k0 + r) * ldw + j0 + c);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) tile[(i * 8 + (tid >> 5)) * LD + (tid & 31) * 4 + q] = x[i][q];
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int line = h * 64 + (tid >> 2), b = tid & 3;
        if (codes_b && k0 + line < c_in) {
            const int64_t row = e * c_in + k0 + line;
            mx4_block(tile + line * LD + b * 32, 1, codes_b + row * (kp_out / 2) + j0 / 2 + b * 16, scales_b + row * (kp_out / 32) + j0 / 32 + b);
        }
        if (codes_f && j0 + line < c_out) {
            const int64_t row = e * c_out + j0 + line;
            mx4_block(tile + b * 32 * LD + line, LD, codes_f + row * (kp_in / 2) + k0 / 2 + b * 16, scales_f + row * (kp_in / 32) + k0 / 32 + b);
        }
    }
}

hipError_t launch_mx4_prepare(const float* W, int32_t n_groups, int64_t c_in, int64_t c_out, int64_t ldw, uint8_t* codes_f, uint8_t* scales_f,
                              uint8_t* codes_b, uint8_t* scales_b, hipStream_t stream) {
    ProfScope prof(K_PREPARE, stream);
    // the tiles cover the padding of both copies (values out of range are zeros)
    const int64_t kp_in = mx4_padded(c_in), kp_out = mx4_padded(c_out);
    const dim3 grid((unsigned)(kp_out / kPrepTile), (unsigned)(kp_in / kPrepTile), (unsigned)n_groups);
    mx4_prepare_kernel<<<grid, dim3(256), 0, stream>>>(W, (int)c_in, (int)c_out, ldw, (int)kp_in, (int)kp_out, codes_f, scales_f, codes_b, scales_b);
    return hipGetLastError();
}

}  // namespace quaff
