// Scores: out[i,j] = sum over blocks b of 2^(ea[i,b] + eb[j,b]) * sum_k A[i,b,k] B[j,b,k], rounded once to the output's type.
//
// Sums of fp32 accuracy: codes become bfloat16 in registers, their block's power of two in the same instruction (four significant bits
// and the exponent both fit), and go to the bfloat16 matrix instruction, which adds in fp32.  The 8-bit matrix instructions are twice as fast, but
// inside a group of products they keep only what lies within 2^14 of the largest: 1.5e-5 (normal values) to 7e-5 (values over several
// powers of ten) of the result's norm, where fp32 sums are off by 1e-7.
#include "class_ops.h"

namespace wpsgd {

typedef float f32x4 __attribute__((ext_vector_type(4)));

struct MatmulArgs {
    const uint8_t *a, *b, *ea, *eb;
    int64_t lda, ldb, lde_a, lde_b;
    int64_t M, N;
    int blocks;
    void *out;
    int64_t ldo;
};

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

__device__ inline float power_of(int byte) { return __uint_as_float((uint32_t)byte << 23); }

// eight codes, two words, times a power of two
__device__ inline bf16x8 widen8(uint32_t lo, uint32_t hi, float scale)
{
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return bf16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

// 64 x 64 results to a workgroup, 32 x 32 to a wave, operands straight from memory.
template <typename TO>
__global__ __launch_bounds__(256) void matmul_simple_kernel(MatmulArgs g)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t tiles = (g.N + 63) / 64;
    const int64_t tm = (int64_t)blockIdx.x / tiles, tn = (int64_t)blockIdx.x - tm * tiles;
    const int64_t i0 = tm * 64 + (wave >> 1) * 32, j0 = tn * 64 + (wave & 1) * 32;
    const int r = lane & 15, k = (lane >> 4) * 32;
    const uint8_t *pa[2], *pb[2], *sa[2], *sb[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int64_t i = i0 + t * 16 + r < g.M ? i0 + t * 16 + r : g.M - 1, j = j0 + t * 16 + r < g.N ? j0 + t * 16 + r : g.N - 1;
        pa[t] = g.a + i * g.lda + k;
        pb[t] = g.b + j * g.ldb + k;
        sa[t] = g.ea + i * g.lde_a;
        sb[t] = g.eb + j * g.lde_b;
    }
    f32x4 acc[2][2];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int u = 0; u < 2; ++u) acc[t][u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int b = 0; b < g.blocks; ++b) {
        uint4 fa[2][2], fb[2][2];
        float ca[2], cb[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                fa[t][h] = *reinterpret_cast<const uint4 *>(pa[t] + (int64_t)b * 128 + h * 16);
                fb[t][h] = *reinterpret_cast<const uint4 *>(pb[t] + (int64_t)b * 128 + h * 16);
            }
            ca[t] = power_of(sa[t][b]);
            cb[t] = power_of(sb[t][b]);
        }
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            bf16x8 wa[2], wb[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                wa[t] = (h & 1) ? widen8(fa[t][h / 2].z, fa[t][h / 2].w, ca[t]) : widen8(fa[t][h / 2].x, fa[t][h / 2].y, ca[t]);
                wb[t] = (h & 1) ? widen8(fb[t][h / 2].z, fb[t][h / 2].w, cb[t]) : widen8(fb[t][h / 2].x, fb[t][h / 2].y, cb[t]);
            }
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int u = 0; u < 2; ++u) acc[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wa[t], wb[u], acc[t][u], 0, 0, 0);
        }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int64_t i = i0 + t * 16 + (lane >> 4) * 4 + q, j = j0 + u * 16 + r;
                if (i < g.M && j < g.N) Elem<TO>::put(static_cast<TO *>(g.out) + i * g.ldo + j, acc[t][u][q]);
            }
}

}  // namespace wpsgd

using namespace wpsgd;

extern "C" {

size_t wpsgd_block_matmul_workspace(int64_t rows_a, int64_t rows_b, int64_t cols)
{
    (void)rows_a; (void)rows_b; (void)cols;
    return 0;
}

int wpsgd_block_matmul(const wpsgd_blocks *A, const wpsgd_blocks *B, void *out, int64_t ld_out, wpsgd_dtype dtype, void *workspace, size_t workspace_bytes,
                       void *stream)
{
    int rc = check_blocks(A);
    if (rc == WPSGD_OK) rc = check_blocks(B);
    if (rc != WPSGD_OK) return rc;
    if (A->cols != B->cols || (dtype != WPSGD_F32 && dtype != WPSGD_BF16)) return WPSGD_INVALID_ARG;
    if (A->rows == 0 || B->rows == 0) return WPSGD_OK;
    if (!out || ld_out < B->rows || (uintptr_t)out % (dtype == WPSGD_F32 ? 4 : 2) != 0) return WPSGD_INVALID_ARG;
    const size_t need = wpsgd_block_matmul_workspace(A->rows, B->rows, A->cols);
    if (need && (!workspace || (uintptr_t)workspace % 256 != 0)) return WPSGD_INVALID_ARG;
    if (workspace_bytes < need) return WPSGD_WORKSPACE_TOO_SMALL;
    const MatmulArgs g{static_cast<const uint8_t *>(A->codes), static_cast<const uint8_t *>(B->codes), static_cast<const uint8_t *>(A->exps),
                       static_cast<const uint8_t *>(B->exps), A->ld, B->ld, A->ld_exps, B->ld_exps, A->rows, B->rows, (int)((A->cols + 127) / 128), out, ld_out};
    const int64_t groups = ((A->rows + 63) / 64) * ((B->rows + 63) / 64);
    if (groups > 0x7FFFFFFFLL) return WPSGD_UNSUPPORTED;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (dtype == WPSGD_F32) hipLaunchKernelGGL(matmul_simple_kernel<float>, dim3((unsigned)groups), dim3(256), 0, s, g);
    else hipLaunchKernelGGL(matmul_simple_kernel<uint16_t>, dim3((unsigned)groups), dim3(256), 0, s, g);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? WPSGD_OK : hip_fail(e);
}

}  // extern "C"
