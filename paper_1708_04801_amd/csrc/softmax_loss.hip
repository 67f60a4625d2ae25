// Softmax cross-entropy of a batch of scores, with its gradient:
//   loss_i = r_i (log sum_c exp(z_ic) - z_it),   grad_ic = scale r_i (exp(z_ic - m_i) / s_i - [c = t]),   m_i the row's maximum, s_i = sum_c exp(z_ic - m_i).
// One workgroup owns a row; the maximum and the sum are carried together in fp32 (a thread's running sum is rescaled when its maximum grows).
#include "class_ops.h"

namespace wpsgd {

struct LossArgs {
    const void *z;
    int64_t n, c, ld;
    const int64_t *labels;
    const float *row_weights;
    float scale;
    float *loss;
    void *grad;
    int64_t ld_grad;
};

constexpr float kLog2e = 1.44269504088896340736f;
__device__ inline float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }   // x <= 0

// (m, s) of two parts of a row; a part without a finite maximum has s = 0 or NaN
__device__ inline void join(float &m, float &s, float m2, float s2)
{
    const float top = fmaxf(m, m2);
    const float a = m == top ? s : s * exp_of(m - top), b = m2 == top ? s2 : s2 * exp_of(m2 - top);
    m = top;
    s = a + b;
}

template <typename T, int NT>
__global__ __launch_bounds__(NT) void softmax_row_kernel(LossArgs a)
{
    constexpr int E = Elem<T>::kPer16;
    __shared__ float part[2][NT / 64];
    const int64_t row = blockIdx.x;
    const int t = threadIdx.x;
    const T *z = static_cast<const T *>(a.z) + row * a.ld;
    T *g = a.grad ? static_cast<T *>(a.grad) + row * a.ld_grad : nullptr;
    const int64_t label = a.labels[row];
    const float r = a.row_weights ? a.row_weights[row] : 1.0f;
    const int64_t vectors = a.c / E, tail = a.c - vectors * E;
    const bool counts = label >= 0 && r != 0.0f;
    if (counts) {
        float m = -__builtin_inff(), s = 0.0f;
        for (int64_t v = t; v < vectors; v += NT) {
            const Bytes16 q = load16(z + v * E);
            float top = m;
#pragma unroll
            for (int j = 0; j < E; ++j) top = fmaxf(top, Elem<T>::get(q.w, j));
            const float base = top == -__builtin_inff() ? 0.0f : top;
            s = s * exp_of(m - base);
#pragma unroll
            for (int j = 0; j < E; ++j) s += exp_of(Elem<T>::get(q.w, j) - base);
            m = top;
        }
        if (t < tail) {
            const float x = Elem<T>::load(z + vectors * E + t);
            join(m, s, fmaxf(x, -__builtin_inff()), x == -__builtin_inff() ? 0.0f : x - x + 1.0f);
        }
        for (int d = 1; d < 64; d *= 2) {
            const float m2 = __shfl_xor(m, d), s2 = __shfl_xor(s, d);
            join(m, s, m2, s2);
        }
        if ((t & 63) == 0) { part[0][t >> 6] = m; part[1][t >> 6] = s; }
        __syncthreads();
        m = part[0][0];
        s = part[1][0];
#pragma unroll
        for (int w = 1; w < NT / 64; ++w) join(m, s, part[0][w], part[1][w]);
        const bool empty = m == -__builtin_inff() && s == 0.0f;
        const float bad = label >= a.c ? __builtin_nanf("") : 0.0f;              // no such class: loss and gradient say so
        if (t == 0) a.loss[row] = label >= a.c ? bad : empty ? __builtin_inff() : (m - Elem<T>::load(z + label) + logf(s)) * r;
        if (!g) return;
        __syncthreads();                                                          // (the label's score is read before it may be overwritten)
        const float f = a.scale * r, over = (empty ? 0.0f : f / s) + bad, base = empty ? 0.0f : m;
        for (int64_t v = t; v < vectors; v += NT) {
            const Bytes16 q = load16(z + v * E);
            float p[E];
#pragma unroll
            for (int j = 0; j < E; ++j) p[j] = exp_of(Elem<T>::get(q.w, j) - base) * over;
            if (label >= v * E && label < (v + 1) * E && !empty) {
#pragma unroll
                for (int j = 0; j < E; ++j) p[j] = j == (int)(label - v * E) ? p[j] - f : p[j];
            }
            Bytes16 o;
            if constexpr (E == 8) {
#pragma unroll
                for (int j = 0; j < 4; ++j) o.w[j] = bf16_pack(p[2 * j], p[2 * j + 1]);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) o.w[j] = __float_as_uint(p[j]);
            }
            store16(g + v * E, o);
        }
        if (t < tail) {
            const int64_t at = vectors * E + t;
            const float p = exp_of(Elem<T>::load(z + at) - base) * over;
            Elem<T>::put(g + at, at == label && !empty ? p - f : p);
        }
        return;
    }
    if (t == 0) a.loss[row] = 0.0f;
    if (!g) return;
    for (int64_t v = t; v < vectors; v += NT) store16(g + v * E, Bytes16{{0, 0, 0, 0}});
    if (t < tail) Elem<T>::put(g + vectors * E + t, 0.0f);
}

}  // namespace wpsgd

using namespace wpsgd;

extern "C" {

size_t wpsgd_softmax_loss_workspace(int64_t n, int64_t classes, wpsgd_dtype dtype)
{
    (void)n; (void)classes; (void)dtype;
    return 0;
}

int wpsgd_softmax_loss(const void *Z, int64_t n, int64_t classes, int64_t ld, wpsgd_dtype dtype, const int64_t *labels, const float *row_weights, double scale,
                       float *loss, void *grad, int64_t ld_grad, void *workspace, size_t workspace_bytes, void *stream)
{
    if (n < 0 || n > 0x7FFFFFFFLL || classes < 1 || classes > 0x7FFFFFFFLL || (dtype != WPSGD_F32 && dtype != WPSGD_BF16)) return WPSGD_INVALID_ARG;
    if (n == 0) return WPSGD_OK;
    const size_t elem = dtype == WPSGD_F32 ? 4 : 2;
    if (!Z || !labels || !loss || ld < classes || (uintptr_t)Z % elem != 0) return WPSGD_INVALID_ARG;
    if (grad && (ld_grad < classes || (uintptr_t)grad % elem != 0)) return WPSGD_INVALID_ARG;
    if (grad == Z && ld_grad != ld) return WPSGD_INVALID_ARG;
    if (!(scale - scale == 0.0)) return WPSGD_INVALID_ARG;
    const size_t need = wpsgd_softmax_loss_workspace(n, classes, dtype);
    if (need && (!workspace || (uintptr_t)workspace % 256 != 0)) return WPSGD_INVALID_ARG;
    if (workspace_bytes < need) return WPSGD_WORKSPACE_TOO_SMALL;
    const LossArgs a{Z, n, classes, ld, labels, row_weights, (float)scale, loss, grad, ld_grad};
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (dtype == WPSGD_F32) hipLaunchKernelGGL((softmax_row_kernel<float, 256>), dim3((unsigned)n), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((softmax_row_kernel<uint16_t, 256>), dim3((unsigned)n), dim3(256), 0, s, a);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? WPSGD_OK : hip_fail(e);
}

}  // extern "C"
