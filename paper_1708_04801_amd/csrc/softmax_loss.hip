// Softmax cross-entropy of a batch of scores, with its gradient:
//   loss_i = r_i (log sum_c exp(z_ic) - z_it),   grad_ic = scale r_i (exp(z_ic - m_i) / s_i - [c = t]),   m_i the row's maximum, s_i = sum_c exp(z_ic - m_i).
// Statistics are fp32.
#include <type_traits>

#include "class_ops.h"

namespace wpsgd {

struct LossArgs {
    const void *z;
    int64_t n, c, ld;
    const int64_t *labels;
    const float *row_weights;
    double scale;
    float *loss;
    void *grad;
    int64_t ld_grad;
    int64_t first;             // workgroup of the call at which the launch begins
};

constexpr float kLog2e = 1.44269504088896340736f, kLog2eRest = 1.92596299e-8f;      // log2 e, and what its fp32 value leaves
// e^x for x <= 0.  For fp32 rows to a last place or two, subnormal results too, since their gradient keeps it: with x log2 e rounded once the gradient of a class 100 under the largest is
// off by 7e-6 of itself.  x log2 e = n + f with f exact but for its own rounding; n is held at -300, so that -inf comes out as 2^-inf and a NaN as itself.  The row's sum and its
// gradient share the exponential: 4096 x 65536 fp32 with the gradient 414 us, 408 with the short form (loss alone 220 | 187; up to 32000 classes no difference).
// bfloat16 gradients round to 2^-8, and the short form is off by |x| 2^-23, least in the terms that make up the row's sum (and 0 under 2^-126).
template <typename T> __device__ inline float exp_of(float x)
{
    if constexpr (Elem<T>::kPer16 == 4) {
        const float n = fmaxf(__builtin_rintf(x * kLog2e), -300.0f);
        const float f = fmaf(x, kLog2eRest, fmaf(x, kLog2e, -n));
        return __builtin_amdgcn_ldexpf(__builtin_amdgcn_exp2f(f), (int)n);
    } else {
        return __builtin_amdgcn_exp2f(x * kLog2e);
    }
}

// The row waits in registers between its statistics and its gradient, V vectors of sixteen bytes to a thread, so that it is read once; NT threads to a row, 256 / NT
// rows to a workgroup where that is more than one.  LONG: what a row has beyond 16 NT V bytes is read again for the gradient.  Bound by memory: 8192 x 65536
// bfloat16 reads and writes 1 GiB each in 385 us, 5.6 TB/s; 1023 x 32001 takes 24 us, 5.4 TB/s; 64 x 1000 fp32 3.6 us, a launch.
template <typename T, int NT, int V, bool LONG>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void softmax_row_kernel(LossArgs a)
{
    constexpr int E = Elem<T>::kPer16, kRows = NT < 256 ? 256 / NT : 1, kWaves = NT / 64;
    constexpr float kInf = __builtin_inff();
    constexpr bool kKept = E == 4;         // exponentials take the scores' place in the registers: one for both, and none is rounded
    __shared__ float part[2][kWaves];
    const int64_t row = (a.first + blockIdx.x) * kRows + threadIdx.x / NT;
    if (kRows > 1 && row >= a.n) return;                                          // (whole waves)
    const int t = threadIdx.x % NT;
    const T *z = static_cast<const T *>(a.z) + row * a.ld;
    T *g = a.grad ? static_cast<T *>(a.grad) + row * a.ld_grad : nullptr;
    const int64_t label = a.labels[row];
    const float r = a.row_weights ? a.row_weights[row] : 1.0f;
    const int c = (int)a.c, vectors = c / E, tail = c - vectors * E;
    if (label < 0 || r == 0.0f) {
        if (t == 0) a.loss[row] = 0.0f;
        if (!g) return;
        for (int v = t; v < vectors; v += NT) store16(g + (int64_t)v * E, Bytes16{{0, 0, 0, 0}});
        if (t < tail) Elem<T>::put(g + (int64_t)vectors * E + t, 0.0f);
        return;
    }
    Bytes16 q[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int at = v * NT + t;
        q[v] = at < vectors ? load16(z + (int64_t)at * E) : E == 8 ? Bytes16{{0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u}}
                                                                   : Bytes16{{0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u}};      // -inf
    }
    const float last = t < tail ? Elem<T>::load(z + (int64_t)vectors * E + t) : -kInf;
    const float z_label = t == 0 && label < a.c ? Elem<T>::load(z + label) : 0.0f;
    // the packed words are what waits: without this the compiler keeps what it has unpacked beside them, twice the registers
    auto pack = [&]() {
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int j = 0; j < 4; ++j) asm volatile("" : "+v"(q[v].w[j]));
    };
    float m = last;                                                               // (fmaxf passes over a NaN, which then shows in the sum)
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int j = 0; j < E; ++j) m = fmaxf(m, Elem<T>::get(q[v].w, j));
    m = fmaxf(m, -kInf);
    float s = 0.0f;
    if constexpr (LONG) {
        for (int v = V * NT + t; v < vectors; v += NT) {
            const Bytes16 more = load16(z + (int64_t)v * E);
            float top = m;
#pragma unroll
            for (int j = 0; j < E; ++j) top = fmaxf(top, Elem<T>::get(more.w, j));
            const float base = top == -kInf ? 0.0f : top;
            s = s * exp_of<T>(m - base);
#pragma unroll
            for (int j = 0; j < E; ++j) s += exp_of<T>(Elem<T>::get(more.w, j) - base);
            m = top;
        }
    }
    pack();
    const float own = m;                                                          // what s is relative to
    m = wave_max(m);
    if constexpr (kWaves > 1) {
        if ((t & 63) == 0) part[0][t >> 6] = m;
        __syncthreads();
        m = part[0][0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) m = fmaxf(m, part[0][w]);
    }
    const bool none = m == -kInf;                                                 // every score is -inf or NaN
    const float base = none ? 0.0f : m;
    if constexpr (LONG) s = own == -kInf ? s : s * exp_of<T>(own - base);
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const float e = exp_of<T>(Elem<T>::get(q[v].w, j) - base);
            s += e;
            if constexpr (kKept) q[v].w[j] = __float_as_uint(e);
        }
    const float e_last = exp_of<T>(last - base);
    s += e_last;
    pack();
    s = wave_sum(s);
    if constexpr (kWaves > 1) {
        if ((t & 63) == 0) part[1][t >> 6] = s;
        __syncthreads();
        s = part[1][0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) s += part[1][w];
    }
    const bool empty = none && s == 0.0f;
    const float bad = label >= a.c ? __builtin_nanf("") : 0.0f;                   // no such class: loss and gradient say so
    if (t == 0) a.loss[row] = label >= a.c ? bad : empty ? kInf : (m - z_label + logf(s)) * r;
    if (!g) return;
    const float f = (float)(a.scale * (double)r), over = (empty ? 0.0f : f / s) + bad;
    const int at_label = empty || label >= a.c ? -1 : (int)label;
    auto gradient = [&](int v, const Bytes16 &x, auto kept) {
        float p[E];
#pragma unroll
        for (int j = 0; j < E; ++j) p[j] = (decltype(kept)::value ? Elem<T>::get(x.w, j) : exp_of<T>(Elem<T>::get(x.w, j) - base)) * over;
        if (at_label / E == v && at_label >= 0) {
#pragma unroll
            for (int j = 0; j < E; ++j) p[j] = at_label % E == j ? p[j] - f : p[j];
        }
        Bytes16 o;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (E == 8) o.w[j] = bf16_pack(p[2 * j], p[2 * j + 1]);
            else o.w[j] = __float_as_uint(p[j]);
        }
        store16(g + (int64_t)v * E, o);
    };
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (v * NT + t < vectors) gradient(v * NT + t, q[v], std::integral_constant<bool, kKept>{});
    if constexpr (LONG) {
        for (int v = V * NT + t; v < vectors; v += NT) gradient(v, load16(z + (int64_t)v * E), std::false_type{});
    }
    if (t < tail) {
        const float p = e_last * over;
        Elem<T>::put(g + (int64_t)vectors * E + t, at_label == vectors * E + t ? p - f : p);
    }
}

template <typename T>
static hipError_t launch_loss(LossArgs a, hipStream_t s)
{
    const int64_t vectors = a.c / Elem<T>::kPer16;
    const auto run = [&](auto kernel, int64_t groups, int threads) {
        return in_launches(groups, threads, [&](int64_t first, unsigned count) {
            a.first = first;
            hipLaunchKernelGGL(kernel, dim3(count), dim3(threads), 0, s, a);
        });
    };
    // the fewest threads whose registers hold a row; rows that half the registers of a compute unit cannot hold are its only one
    if (vectors <= 64 * 4) return run(softmax_row_kernel<T, 64, 4, false>, (a.n + 3) / 4, 256);
    if (vectors <= 256 * 4) return run(softmax_row_kernel<T, 256, 4, false>, a.n, 256);
    if (vectors <= 256 * 8) return run(softmax_row_kernel<T, 256, 8, false>, a.n, 256);
    if (vectors <= 256 * 16) return run(softmax_row_kernel<T, 256, 16, false>, a.n, 256);
    if (vectors <= 512 * 16) return run(softmax_row_kernel<T, 512, 16, false>, a.n, 512);
    if (vectors <= 1024 * 16) return run(softmax_row_kernel<T, 1024, 16, false>, a.n, 1024);
    return run(softmax_row_kernel<T, 1024, 16, true>, a.n, 1024);
}

}  // namespace wpsgd

using namespace wpsgd;

extern "C" {

int wpsgd_softmax_loss(const void *Z, int64_t n, int64_t classes, int64_t ld, wpsgd_dtype dtype, const int64_t *labels, const float *row_weights, double scale,
                       float *loss, void *grad, int64_t ld_grad, void *stream)
{
    if (n < 0 || n > 0x7FFFFFFFLL || classes < 1 || classes > 0x7FFFFFFFLL || (dtype != WPSGD_F32 && dtype != WPSGD_BF16)) return WPSGD_INVALID_ARG;
    if (n == 0) return WPSGD_OK;
    const size_t elem = dtype == WPSGD_F32 ? 4 : 2;
    if (!Z || !labels || !loss || ld < classes || (uintptr_t)Z % elem != 0) return WPSGD_INVALID_ARG;
    if (grad && (ld_grad < classes || (uintptr_t)grad % elem != 0)) return WPSGD_INVALID_ARG;
    if (grad == Z && ld_grad != ld) return WPSGD_INVALID_ARG;
    if (!(scale - scale == 0.0)) return WPSGD_INVALID_ARG;
    const LossArgs a{Z, n, classes, ld, labels, row_weights, scale, loss, grad, ld_grad, 0};
    hipStream_t s = static_cast<hipStream_t>(stream);
    const hipError_t e = dtype == WPSGD_F32 ? launch_loss<float>(a, s) : launch_loss<uint16_t>(a, s);
    return e == hipSuccess ? WPSGD_OK : hip_fail(e);
}

}  // extern "C"
