// Elements dropped by a counter-based generator, the others scaled so that means stay: Philox4x32-10 with the key `seed` and the counter
// (column / 8, row, chain, 2^30 + step mod 2^30) gives four words, sixteen bits for each of the eight columns; element c of row i is dropped where its bits, c mod 8 of them
// in, are under t = floor(2^16 p + 1/2), and is else x 2^16 / (2^16 - t): the probability is t / 2^16, and the scale is that of it.  The mask is made where it is needed, and
// again for the gradient.  Bound by memory: 32768 x 8192 bfloat16 reads and writes 512 MiB each in 190 to 200 us, 5.5 TB/s; 64 picked rows of 4096 take 2.9, a launch.  Sixteen bits an element make one call of the
// generator, forty multiplications, do for sixteen bytes of bfloat16; with 32 bits it would be two, and the vector units' time as long as the memory's.
#include "class_ops.h"

namespace wpsgd {

struct DropoutArgs {
    const void *x;
    const int64_t *rows;       // which rows, or nullptr: all in order
    int64_t m, d, ld, n;
    void *out;
    int64_t ld_out;
    int64_t blocks;            // of eight columns, in a row
    uint32_t seed_lo, seed_hi, chain;
    int64_t step;
    const int64_t *more_steps;
    uint32_t drop;             // t
    float factor;
    int64_t first;             // workgroup of the call at which the launch begins
};

template <typename T>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a)
{
    constexpr int E = Elem<T>::kPer16;
    const int64_t first = (a.first + blockIdx.x) * 256;
    const int64_t row0 = first / a.blocks;
    const uint32_t at = (uint32_t)(first - row0 * a.blocks) + threadIdx.x;        // (blocks < 2^31)
    const uint32_t down = at / (uint32_t)a.blocks;
    const int64_t row = row0 + down;
    if (row >= a.n) return;
    const uint32_t b = at - down * (uint32_t)a.blocks;
    const int64_t from = a.rows ? a.rows[row] : row, col = (int64_t)b * 8, left = a.d - col;
    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (from >= 0 && from < a.m) load8(static_cast<const T *>(a.x) + from * a.ld + col, left, x);
    const uint64_t step = (uint64_t)a.step + (a.more_steps ? (uint64_t)*a.more_steps : 0);
    uint32_t w[4] = {b, (uint32_t)row, a.chain, 0x40000000u | (uint32_t)(step & 0x3FFFFFFFu)}, k0 = a.seed_lo, k1 = a.seed_hi;
    philox4x32_rounds(w[0], w[1], w[2], w[3], k0, k1, 10);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t bits = (j & 1) ? w[j >> 1] >> 16 : w[j >> 1] & 0xFFFFu;
        x[j] = bits < a.drop ? 0.0f : x[j] * a.factor;
    }
    T *o = static_cast<T *>(a.out) + row * a.ld_out + col;
    if (left >= 8) {
#pragma unroll
        for (int i = 0; i < 8 / E; ++i) {
            Bytes16 q;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (E == 8) q.w[j] = bf16_pack(x[2 * j], x[2 * j + 1]);
                else q.w[j] = __float_as_uint(x[4 * i + j]);
            }
            store16(o + i * E, q);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (j < left) Elem<T>::put(o + j, x[j]);
    }
}

}  // namespace wpsgd

using namespace wpsgd;

extern "C" int wpsgd_dropout(const wpsgd_matrix *X, const int64_t *rows, int64_t n, double p, uint64_t seed, int chain, int64_t step, const int64_t *more_steps,
                             void *out, int64_t ld_out, void *stream)
{
    const int rc = check_matrix(X);
    if (rc != WPSGD_OK) return rc;
    if (!X->dense) return WPSGD_UNSUPPORTED;
    const size_t elem = X->dtype == WPSGD_F32 ? 4 : 2;
    if ((uintptr_t)X->dense % elem != 0 || !(p >= 0.0 && p <= 1.0) || chain < 0 || step < 0) return WPSGD_INVALID_ARG;
    if (n < 0 || (!rows && n > X->m) || n > 0xFFFFFFFFLL || X->d > 0x7FFFFFFFLL) return WPSGD_INVALID_ARG;
    if (n == 0) return WPSGD_OK;
    if (!out || (uintptr_t)out % elem != 0 || ld_out < X->d) return WPSGD_INVALID_ARG;
    if (out == X->dense && (rows || ld_out != X->ld)) return WPSGD_INVALID_ARG;
    const uint32_t drop = (uint32_t)(p * 65536.0 + 0.5);
    const int64_t blocks = (X->d + 7) / 8;
    DropoutArgs a{X->dense, rows, X->m, X->d, X->ld, n, out, ld_out, blocks, (uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)chain, step, more_steps, drop,
                  drop < 65536 ? (float)(65536.0 / (65536.0 - drop)) : 0.0f, 0};
    hipStream_t s = static_cast<hipStream_t>(stream);
    const auto kernel = X->dtype == WPSGD_F32 ? dropout_kernel<float> : dropout_kernel<uint16_t>;
    const hipError_t e = in_launches((n * blocks + 255) / 256, 256, [&](int64_t first, unsigned count) {
        a.first = first;
        hipLaunchKernelGGL(kernel, dim3(count), dim3(256), 0, s, a);
    });
    return e == hipSuccess ? WPSGD_OK : hip_fail(e);
}
