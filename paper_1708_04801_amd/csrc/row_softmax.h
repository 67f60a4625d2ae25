// A row of scores read once: its softmax's statistics, and from them what an operator makes of the row and the gradient that goes with it,
//   grad_ic = f_i (exp(z_ic - m_i) / s_i - [c = t]),   m_i the row's maximum, s_i = sum_c exp(z_ic - m_i), t the row's class, f_i the operator's.
// Exponentials are fp32.  An operator is a class with
//   kWideSum                           whether exponentials are summed in fp64, eight (bfloat16) or four at a time: a sum over many rows' logs shows what fp32 sums leave out, and a bias of each
//   kOneWave                           whether make() is so long that one wave makes it for its row; else every thread does, and gives `writes` for the first
//   counts(row, class, weight)         whether the row counts; the gradient of one that does not is 0
//   absent(row)                        what it writes for a row that does not count (one thread's work)
//   make(row, weight, RowState, writes)    what it writes for one that does, where `writes`; returns f_i
#pragma once

#include <type_traits>

#include "class_ops.h"

namespace wpsgd {

struct RowArgs {
    const void *z;
    int64_t n, c, ld;
    const int64_t *labels;     // a row's class
    const float *row_weights;  // or nullptr: 1
    void *grad;
    int64_t ld_grad;
    int64_t first;             // workgroup of the call at which the launch begins
};

struct RowState {
    float m, s, z_label;       // maximum, sum of exponentials relative to it, the class's score
    double sum;                // s, in fp64 where the operator sums so
    bool empty;                // every score is -inf
    bool unknown;              // no such class
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

// The same for sums in fp64: with the rest of log2 e (without it every exponential is off by 1.3e-8 of its exponent, always to the same side).
template <typename T, bool WIDE> __device__ inline float exp_for(float x)
{
    if constexpr (WIDE && Elem<T>::kPer16 == 8) return __builtin_amdgcn_exp2f(fmaf(x, kLog2e, x * kLog2eRest));
    else return exp_of<T>(x);
}

// The row waits in registers between its statistics and its gradient, V vectors of sixteen bytes to a thread, so that it is read once; NT threads to a row, 256 / NT
// rows to a workgroup where that is more than one.  LONG: what a row has beyond 16 NT V bytes is read again for the gradient.  Bound by memory: 8192 x 65536
// bfloat16 reads and writes 1 GiB each in 385 us, 5.6 TB/s; 1023 x 32001 takes 24 us, 5.4 TB/s; 64 x 1000 fp32 3.6 us, a launch.
template <typename T, int NT, int V, bool LONG, typename Op>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void softmax_row_kernel(RowArgs a, Op op)
{
    constexpr int E = Elem<T>::kPer16, kRows = NT < 256 ? 256 / NT : 1, kWaves = NT / 64;
    constexpr float kInf = __builtin_inff();
    constexpr bool kKept = E == 4;         // exponentials take the scores' place in the registers: one for both, and none is rounded
    using Sum = std::conditional_t<Op::kWideSum, double, float>;
    __shared__ float part[kWaves];
    __shared__ Sum sums[kWaves];
    const int64_t row = (a.first + blockIdx.x) * kRows + threadIdx.x / NT;
    if (kRows > 1 && row >= a.n) return;                                          // (whole waves)
    const int t = threadIdx.x % NT;
    const T *z = static_cast<const T *>(a.z) + row * a.ld;
    T *g = a.grad ? static_cast<T *>(a.grad) + row * a.ld_grad : nullptr;
    const int64_t label = a.labels[row];
    const float r = a.row_weights ? a.row_weights[row] : 1.0f;
    const int c = (int)a.c, vectors = c / E, tail = c - vectors * E;
    if (!op.counts(row, label, r)) {
        if (t == 0) op.absent(row);
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
    const float z_label = (t == 0 || (Op::kOneWave && t < 64)) && label < a.c ? Elem<T>::load(z + label) : 0.0f;
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
    Sum s = 0;
    if constexpr (LONG) {
        for (int v = V * NT + t; v < vectors; v += NT) {
            const Bytes16 more = load16(z + (int64_t)v * E);
            float top = m;
#pragma unroll
            for (int j = 0; j < E; ++j) top = fmaxf(top, Elem<T>::get(more.w, j));
            const float base = top == -kInf ? 0.0f : top;
            s = s * exp_for<T, Op::kWideSum>(m - base);
            float eight = 0.0f;
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const float e = exp_for<T, Op::kWideSum>(Elem<T>::get(more.w, j) - base);
                if constexpr (Op::kWideSum) eight += e;
                else s += e;
            }
            if constexpr (Op::kWideSum) s += eight;
            m = top;
        }
    }
    pack();
    const float own = m;                                                          // what s is relative to
    m = wave_max(m);
    if constexpr (kWaves > 1) {
        if ((t & 63) == 0) part[t >> 6] = m;
        __syncthreads();
        m = part[0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) m = fmaxf(m, part[w]);
    }
    const bool none = m == -kInf;                                                 // every score is -inf or NaN
    const float base = none ? 0.0f : m;
    if constexpr (LONG) s = own == -kInf ? s : s * exp_for<T, Op::kWideSum>(own - base);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        float eight = 0.0f;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const float e = exp_for<T, Op::kWideSum>(Elem<T>::get(q[v].w, j) - base);
            if constexpr (Op::kWideSum) eight += e;
            else s += e;
            if constexpr (kKept) q[v].w[j] = __float_as_uint(e);
        }
        if constexpr (Op::kWideSum) s += eight;
    }
    const float e_last = exp_for<T, Op::kWideSum>(last - base);
    s += e_last;
    pack();
    s = wave_sum(s);
    if constexpr (kWaves > 1) {
        if ((t & 63) == 0) sums[t >> 6] = s;
        __syncthreads();
        s = sums[0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) s += sums[w];
    }
    const bool empty = none && s == 0;
    const float bad = label >= a.c ? __builtin_nanf("") : 0.0f;                   // no such class: the gradient says so
    const RowState state{m, (float)s, z_label, (double)s, empty, label >= a.c};
    float f = 0.0f;
    if constexpr (Op::kOneWave) {
        if (t < 64) f = op.make(row, r, state, t == 0);
        if (!g) return;
        if constexpr (kWaves > 1) {
            if (t == 0) part[0] = f;
            __syncthreads();
            f = part[0];
        }
    } else {
        f = op.make(row, r, state, t == 0);
        if (!g) return;
    }
    const float over = (empty ? 0.0f : f / (float)s) + bad;
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

template <typename T, typename Op>
inline hipError_t launch_rows_softmax(RowArgs a, const Op &op, hipStream_t s)
{
    const int64_t vectors = a.c / Elem<T>::kPer16;
    const auto run = [&](auto kernel, int64_t groups, int threads) {
        return in_launches(groups, threads, [&](int64_t first, unsigned count) {
            a.first = first;
            hipLaunchKernelGGL(kernel, dim3(count), dim3(threads), 0, s, a, op);
        });
    };
    // the fewest threads whose registers hold a row; rows that half the registers of a compute unit cannot hold are its only one
    if (vectors <= 64 * 4) return run(softmax_row_kernel<T, 64, 4, false, Op>, (a.n + 3) / 4, 256);
    if (vectors <= 256 * 4) return run(softmax_row_kernel<T, 256, 4, false, Op>, a.n, 256);
    if (vectors <= 256 * 8) return run(softmax_row_kernel<T, 256, 8, false, Op>, a.n, 256);
    if (vectors <= 256 * 16) return run(softmax_row_kernel<T, 256, 16, false, Op>, a.n, 256);
    if (vectors <= 512 * 16) return run(softmax_row_kernel<T, 512, 16, false, Op>, a.n, 512);
    if (vectors <= 1024 * 16) return run(softmax_row_kernel<T, 1024, 16, false, Op>, a.n, 1024);
    return run(softmax_row_kernel<T, 1024, 16, true, Op>, a.n, 1024);
}

// What the entry points with scores and their gradient refuse alike.
inline int check_scores(const void *Z, int64_t n, int64_t classes, int64_t ld, wpsgd_dtype dtype, const void *grad, int64_t ld_grad)
{
    if (n < 0 || n > 0x7FFFFFFFLL || classes < 1 || classes > 0x7FFFFFFFLL || (dtype != WPSGD_F32 && dtype != WPSGD_BF16)) return WPSGD_INVALID_ARG;
    if (n == 0) return WPSGD_OK;
    const size_t elem = dtype == WPSGD_F32 ? 4 : 2;
    if (!Z || ld < classes || (uintptr_t)Z % elem != 0) return WPSGD_INVALID_ARG;
    if (grad && (ld_grad < classes || (uintptr_t)grad % elem != 0)) return WPSGD_INVALID_ARG;
    return grad == Z && ld_grad != ld ? WPSGD_INVALID_ARG : WPSGD_OK;
}

}  // namespace wpsgd
