// Rows in 8-bit floating point with one power-of-two scale for each block of 128 along the row.
//
// For a block with largest finite size s:  e = the least whole number with s <= 448 * 2^e (at least -126; 0 for a block of zeros),
// code = e4m3(x * 2^-e), nearest even.  A power of two keeps every mantissa bit and is what the matrix instructions take as a scale, so that
// the product needs no arithmetic for it.  Both kernels read each element once and write a code and 1/128 of an exponent byte: they are bound by memory.
#include "class_ops.h"

namespace wpsgd {

constexpr int kBlockCols = 128;

// The least e with s <= 448 * 2^e: 448 = 1.75 * 2^8, so it is s's own exponent less 8, and one more where s's mantissa is over 1.75.
__device__ inline int block_exponent(float s)
{
    const uint32_t bits = __float_as_uint(s);
    const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return s == 0.0f ? 0 : (e < -126 ? -126 : e);        // (a subnormal s has exponent field 0, far below -126 either way)
}
__device__ inline float finite_size(float x)
{
    const float s = fabsf(x);
    return s < __builtin_inff() ? s : 0.0f;
}
// four values to codes, the first in the lowest byte; what is not finite becomes NaN
__device__ inline uint32_t four_codes(const float *x, float scale)
{
    float v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = fabsf(x[j]) < __builtin_inff() ? x[j] * scale : __builtin_nanf("");
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], w, true);
}

struct QuantizeArgs {
    const void *x;
    const int64_t *rows;       // which rows, or nullptr: all in order
    int64_t m, d, ld, n;       // the data set's rows, columns and stride; how many rows are taken
    uint8_t *codes, *exps;
    int64_t ld_codes, ld_exps;
    int64_t blocks;
};

template <typename T>
__device__ inline void load8(const T *p, int64_t left, float (&x)[8])
{
    if (left >= 8) {
        Bytes16 q[8 / Elem<T>::kPer16];
#pragma unroll
        for (int i = 0; i < 8 / Elem<T>::kPer16; ++i) q[i] = load16(p + i * Elem<T>::kPer16);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = Elem<T>::get(q[j / Elem<T>::kPer16].w, j % Elem<T>::kPer16);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = j < left ? Elem<T>::load(p + j) : 0.0f;
    }
}

// Sixteen lanes to a block of 128, eight elements to a lane.
template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(QuantizeArgs a)
{
    const int64_t first = (int64_t)blockIdx.x * 16;
    const int64_t row0 = first / a.blocks;
    const int64_t at = (first - row0 * a.blocks) + (threadIdx.x >> 4);     // (blocks < 2^25: the sum fits 32 bits)
    const uint32_t down = (uint32_t)at / (uint32_t)a.blocks;
    const int64_t row = row0 + down;
    if (row >= a.n) return;                                                 // (sixteen lanes at a time)
    const int64_t b = at - (int64_t)down * a.blocks;
    const int64_t from = a.rows ? a.rows[row] : row;
    const int64_t col = b * kBlockCols + (threadIdx.x & 15) * 8;
    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (from >= 0 && from < a.m && col < a.d) load8(static_cast<const T *>(a.x) + from * a.ld + col, a.d - col, x);
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fmaxf(s, finite_size(x[j]));
    s = fmaxf(s, dpp_move<0xB1, 0xF>(s));
    s = fmaxf(s, dpp_move<0x4E, 0xF>(s));
    s = fmaxf(s, dpp_move<0x141, 0xF>(s));
    s = fmaxf(s, dpp_move<0x140, 0xF>(s));
    const int e = block_exponent(s);
    const float scale = __uint_as_float((uint32_t)(127 - e) << 23);
    const uint2 q = make_uint2(four_codes(x, scale), four_codes(x + 4, scale));
    *reinterpret_cast<uint2 *>(a.codes + row * a.ld_codes + col) = q;
    if ((threadIdx.x & 15) == 0) a.exps[row * a.ld_exps + b] = (uint8_t)(e + 127);
}

// Transposed: the result's rows are the columns of x.  A workgroup takes 128 rows (one block) of 64 columns through LDS; a thread then
// owns 32 rows of one column.
template <typename T>
__global__ __launch_bounds__(256) void quantize_columns_kernel(QuantizeArgs a)
{
    constexpr int kCols = 64;
    __shared__ float tile[kBlockCols][kCols];
    __shared__ float size[4][kCols];
    const int64_t tiles = (a.d + kCols - 1) / kCols;
    const int64_t b = (int64_t)blockIdx.x / tiles, col0 = ((int64_t)blockIdx.x - b * tiles) * kCols;
    const int t = threadIdx.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = i * 32 + (t >> 3), c = (t & 7) * 8;
        const int64_t row = b * kBlockCols + r;
        float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (row < a.n && col0 + c < a.d) {
            const int64_t from = a.rows ? a.rows[row] : row;
            if (from >= 0 && from < a.m) load8(static_cast<const T *>(a.x) + from * a.ld + col0 + c, a.d - col0 - c, x);
        }
        *reinterpret_cast<float4 *>(&tile[r][c]) = make_float4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<float4 *>(&tile[r][c + 4]) = make_float4(x[4], x[5], x[6], x[7]);
    }
    __syncthreads();
    const int c = t & 63, part = t >> 6;
    float x[32];
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        x[j] = tile[part * 32 + j][c];
        s = fmaxf(s, finite_size(x[j]));
    }
    size[part][c] = s;
    __syncthreads();
    s = fmaxf(fmaxf(size[0][c], size[1][c]), fmaxf(size[2][c], size[3][c]));
    const int64_t col = col0 + c;
    if (col >= a.d) return;
    const int e = block_exponent(s);
    const float scale = __uint_as_float((uint32_t)(127 - e) << 23);
    uint8_t *out = a.codes + col * a.ld_codes + b * kBlockCols + part * 32;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const float *p = x + h * 16;
        reinterpret_cast<uint4 *>(out)[h] = make_uint4(four_codes(p, scale), four_codes(p + 4, scale), four_codes(p + 8, scale), four_codes(p + 12, scale));
    }
    if (part == 0) a.exps[col * a.ld_exps + b] = (uint8_t)(e + 127);
}

int check_blocks(const wpsgd_blocks *q)
{
    if (!q || q->rows < 0 || q->cols < 0 || q->cols > (1LL << 31)) return WPSGD_INVALID_ARG;
    if (q->rows == 0 || q->cols == 0) return WPSGD_OK;
    const int64_t blocks = (q->cols + kBlockCols - 1) / kBlockCols;
    if (!q->codes || !q->exps) return WPSGD_INVALID_ARG;
    if (q->ld < blocks * kBlockCols || q->ld % 16 != 0 || (uintptr_t)q->codes % 16 != 0) return WPSGD_INVALID_ARG;
    if (q->ld_exps < blocks || q->ld_exps % 4 != 0 || (uintptr_t)q->exps % 4 != 0) return WPSGD_INVALID_ARG;
    return WPSGD_OK;
}

}  // namespace wpsgd

using namespace wpsgd;

extern "C" int wpsgd_quantize(const wpsgd_matrix *X, const int64_t *rows, int64_t n, int transpose, const wpsgd_blocks *out, void *stream)
{
    int rc = check_matrix(X);
    if (rc != WPSGD_OK) return rc;
    if (!X->dense) return WPSGD_UNSUPPORTED;
    if ((uintptr_t)X->dense % (X->dtype == WPSGD_BF16 ? 2 : 4) != 0) return WPSGD_INVALID_ARG;
    if (n < 0 || (!rows && n > X->m) || n > (1LL << 31) || X->d > (1LL << 31)) return WPSGD_INVALID_ARG;
    rc = check_blocks(out);
    if (rc != WPSGD_OK) return rc;
    if (out->rows != (transpose ? X->d : n) || out->cols != (transpose ? n : X->d)) return WPSGD_INVALID_ARG;
    if (n == 0) return WPSGD_OK;
    const QuantizeArgs a{X->dense, rows, X->m, X->d, X->ld, n, static_cast<uint8_t *>(out->codes), static_cast<uint8_t *>(out->exps), out->ld, out->ld_exps,
                         (out->cols + kBlockCols - 1) / kBlockCols};
    const int64_t groups = transpose ? a.blocks * ((X->d + 63) / 64) : (n * a.blocks + 15) / 16;
    if (groups > 0x7FFFFFFFLL) return WPSGD_UNSUPPORTED;
    const dim3 grid((unsigned)groups), block(256);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool half = X->dtype == WPSGD_BF16;
    if (transpose) {
        if (half) hipLaunchKernelGGL(quantize_columns_kernel<uint16_t>, grid, block, 0, s, a);
        else hipLaunchKernelGGL(quantize_columns_kernel<float>, grid, block, 0, s, a);
    } else {
        if (half) hipLaunchKernelGGL(quantize_rows_kernel<uint16_t>, grid, block, 0, s, a);
        else hipLaunchKernelGGL(quantize_rows_kernel<float>, grid, block, 0, s, a);
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? WPSGD_OK : hip_fail(e);
}
