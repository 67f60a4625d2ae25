// Rows in 8-bit floating point with one power-of-two scale for each block of 128 along the row.
//
// For a block with largest finite size s:  e = the least whole number with s <= 448 * 2^e (at least -126; 0 for a block of zeros),
// code = e4m3(x * 2^-e), nearest even.  A power of two keeps every mantissa bit and is what the matrix instructions take as a scale, so that
// the product needs no arithmetic for it.  Both kernels read each element once and write a code and 1/128 of an exponent byte: they are bound by memory
// (8192 rows of 4096 bfloat16 picked: 30 us, 3.4 TB/s; 8192 x 16384 bfloat16 transposed: 94 us, 4.3 TB/s), and small ones by the launch (one row: 2.6 us).
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
    int64_t first;             // workgroup of the call at which the launch begins
};

// Sixteen lanes to a block of 128, eight elements to a lane.
template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(QuantizeArgs a)
{
    const int64_t first = (a.first + blockIdx.x) * 16;
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

// Transposed: the result's rows are the columns of x.  A workgroup takes 128 rows (one block) of 64 columns through LDS, as they are stored; a thread then owns
// sixteen rows of two columns, and its codes go back through LDS so that whole lines of 128 bytes leave (32 bytes of a line at a time: 131 us for 8192 x
// 16384 bfloat16, which reads and writes 403 MB).
template <typename T> struct ColumnPair;
template <> struct ColumnPair<uint16_t> {
    uint32_t w;
    __device__ float first() const { return bf16_lo(w); }
    __device__ float second() const { return bf16_hi(w); }
};
template <> struct ColumnPair<float> {
    float x, y;
    __device__ float first() const { return x; }
    __device__ float second() const { return y; }
};

template <typename T>
__global__ __launch_bounds__(256) void quantize_columns_kernel(QuantizeArgs a)
{
    constexpr int kCols = 64, E = Elem<T>::kPer16, kVectors = kCols / E;       // vectors of a tile's row
    __shared__ __attribute__((aligned(16))) T tile[kBlockCols][kCols];          // later the codes, 128 bytes to a column
    __shared__ float2 size[8][kCols / 2];
    const int64_t tiles = (a.d + kCols - 1) / kCols;
    const int64_t group = a.first + blockIdx.x, b = group / tiles, col0 = (group - b * tiles) * kCols;
    const int t = threadIdx.x;
#pragma unroll
    for (int i = 0; i < kBlockCols * kVectors / 256; ++i) {
        const int r = (i * 256 + t) / kVectors, c = (t % kVectors) * E;
        const int64_t row = b * kBlockCols + r;
        Bytes16 q{{0, 0, 0, 0}};
        if (row < a.n && col0 + c < a.d) {
            const int64_t from = a.rows ? a.rows[row] : row;
            if (from >= 0 && from < a.m) {
                const T *p = static_cast<const T *>(a.x) + from * a.ld + col0 + c;
                const int64_t left = a.d - col0 - c;
                if (left >= E) {
                    q = load16(p);
                } else {
#pragma unroll
                    for (int j = 0; j < E - 1; ++j)
                        if (j < left) {
                            const uint32_t bits = __float_as_uint(Elem<T>::load(p + j));
                            if constexpr (E == 8) q.w[j >> 1] |= (j & 1) ? bits & 0xFFFF0000u : bits >> 16;
                            else q.w[j] = bits;
                        }
                }
            }
        }
        *reinterpret_cast<uint4 *>(&tile[r][c]) = make_uint4(q.w[0], q.w[1], q.w[2], q.w[3]);
    }
    __syncthreads();
    const int pair = t & 31, part = t >> 5;
    float x[2][16];
    float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        const ColumnPair<T> v = reinterpret_cast<const ColumnPair<T> *>(&tile[part * 16 + j][0])[pair];
        x[0][j] = v.first();
        x[1][j] = v.second();
        s.x = fmaxf(s.x, finite_size(x[0][j]));
        s.y = fmaxf(s.y, finite_size(x[1][j]));
    }
    size[part][pair] = s;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float2 o = size[k][pair];
        s.x = fmaxf(s.x, o.x);
        s.y = fmaxf(s.y, o.y);
    }
    uint8_t *codes = reinterpret_cast<uint8_t *>(tile);
    const float most[2] = {s.x, s.y};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int col = pair * 2 + k, e = block_exponent(most[k]);
        const float scale = __uint_as_float((uint32_t)(127 - e) << 23);
        const float *p = x[k];
        // (sixteen bytes q of a column at place q ^ (its pair mod 8): neighbouring pairs meet different banks)
        *reinterpret_cast<uint4 *>(codes + col * 128 + ((part ^ (pair & 7)) * 16)) =
            make_uint4(four_codes(p, scale), four_codes(p + 4, scale), four_codes(p + 8, scale), four_codes(p + 12, scale));
        if (part == 0 && col0 + col < a.d) a.exps[(col0 + col) * a.ld_exps + b] = (uint8_t)(e + 127);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int col = (i * 256 + t) >> 3, piece = t & 7;
        if (col0 + col < a.d)
            *reinterpret_cast<uint4 *>(a.codes + (col0 + col) * a.ld_codes + b * kBlockCols + piece * 16) =
                *reinterpret_cast<const uint4 *>(codes + col * 128 + ((piece ^ ((col >> 1) & 7)) * 16));
    }
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
    QuantizeArgs a{X->dense, rows, X->m, X->d, X->ld, n, static_cast<uint8_t *>(out->codes), static_cast<uint8_t *>(out->exps), out->ld, out->ld_exps,
                         (out->cols + kBlockCols - 1) / kBlockCols, 0};
    const int64_t groups = transpose ? a.blocks * ((X->d + 63) / 64) : (n * a.blocks + 15) / 16;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool half = X->dtype == WPSGD_BF16;
    const auto kernel = transpose ? (half ? quantize_columns_kernel<uint16_t> : quantize_columns_kernel<float>)
                                  : (half ? quantize_rows_kernel<uint16_t> : quantize_rows_kernel<float>);
    const hipError_t e = in_launches(groups, 256, [&](int64_t first, unsigned count) {
        a.first = first;
        hipLaunchKernelGGL(kernel, dim3(count), dim3(256), 0, s, a);
    });
    return e == hipSuccess ? WPSGD_OK : hip_fail(e);
}
