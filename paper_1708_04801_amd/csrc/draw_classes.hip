// A class drawn for each row from its scores, with temperature, top-k, min-p and top-p, by a given random number.
//
// Classes stand in order of score, the lower index first among equals; -inf and NaN cannot be drawn.  What may be drawn is a run from the front of that
// order: the first top_k, of those the ones whose weight is at least min_p of the largest, and of those the shortest run that holds top_p of their weight.
// Weights are whole numbers, q = floor(2^((x - max) log2e / T) 2^31 + 1/2), and their sums 64-bit integers: no sum depends on the order it is taken
// in, so neither does a draw, and a weight is off by 2^-32 of the largest at most.  The run's end is found digit by digit on the
// scores' bits (four digits of eight bits, the counts or weights of each in LDS), and the draw walks the kept classes by index.
#include <cmath>

#include "class_ops.h"

namespace wpsgd {

struct DrawArgs {
    const void *z;
    int64_t n, c, ld;
    const float *u;
    wpsgd_draw_rule rule;
    int64_t *classes;
    float *probs;
};

constexpr float kOne = 2147483648.0f;           // the largest score's weight
constexpr float kLog2eDraw = 1.44269504088896340736f;

// a score that compares as a whole number; NaN counts as -inf, -0 as 0
__device__ inline float clean(float x) { return x == x ? x + 0.0f : -__builtin_inff(); }
__device__ inline uint32_t key_of(float x)
{
    const uint32_t b = __float_as_uint(x);
    return b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ inline float of_key(uint32_t k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xFFFFFFFFu)); }

struct Weigh {
    float top, slope, low;
    __device__ uint32_t operator()(float x) const
    {
        if (x == -__builtin_inff()) return 0;
        const float e = x == top ? 1.0f : __builtin_amdgcn_exp2f((x - top) * slope);
        return e >= low ? (uint32_t)(e * kOne + 0.5f) : 0u;
    }
};

template <int NT>
__device__ inline uint64_t group_scan(uint64_t v, uint64_t *part, uint64_t &total)
{
    // sums of the threads in front of this one, and of all
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint64_t in = v;
    for (int d = 1; d < 64; d *= 2) {
        const uint64_t o = __shfl_up(in, d);
        if (lane >= d) in += o;
    }
    __syncthreads();
    if (lane == 63) part[wave] = in;
    __syncthreads();
    uint64_t before = 0, all = 0;
    for (int w = 0; w < NT / 64; ++w) {
        const uint64_t p = part[w];
        if (w < wave) before += p;
        all += p;
    }
    total = all;
    return before + in - v;
}

template <typename T>
__global__ __launch_bounds__(256) void draw_simple_kernel(DrawArgs a)
{
    constexpr int NT = 256;
    __shared__ uint64_t part[4];
    __shared__ uint64_t hist[256];
    __shared__ uint64_t found[3];
    __shared__ float top_part[4];
    const int64_t row = blockIdx.x;
    const int t = threadIdx.x;
    const T *z = static_cast<const T *>(a.z) + row * a.ld;
    const int c = (int)a.c;
    const float temperature = a.rule.row_temperature ? a.rule.row_temperature[row] : a.rule.temperature;
    const int64_t top_k = a.rule.row_top_k ? a.rule.row_top_k[row] : a.rule.top_k;
    const float top_p = a.rule.row_top_p ? a.rule.row_top_p[row] : a.rule.top_p;
    const float u = a.u[row];
    Weigh weigh;
    weigh.low = fminf(a.rule.row_min_p ? a.rule.row_min_p[row] : a.rule.min_p, 1.0f);     // (the largest always stays)

    float m = -__builtin_inff();
    for (int i = t; i < c; i += NT) m = fmaxf(m, clean(Elem<T>::load(z + i)));
    m = wave_max(m);
    if ((t & 63) == 0) top_part[t >> 6] = m;
    __syncthreads();
    m = fmaxf(fmaxf(top_part[0], top_part[1]), fmaxf(top_part[2], top_part[3]));
    if (m == -__builtin_inff()) {
        if (t == 0) {
            a.classes[row] = -1;
            if (a.probs) a.probs[row] = 0.0f;
        }
        return;
    }
    const bool greedy = !(temperature > 0.0f);
    weigh.top = m + 0.0f;
    weigh.slope = kLog2eDraw / (greedy ? 1.0f : temperature);

    // Walks the order by digits of the key to where `counts` classes (or a weight of that much) have been seen.  floor: no key below it counts.
    auto select = [&](bool weights, uint64_t goal, uint32_t floor, uint32_t &at, uint64_t &before) {
        uint32_t prefix = 0;
        before = 0;
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = t; i < 256; i += NT) hist[i] = 0;
            __syncthreads();
            for (int i = t; i < c; i += NT) {
                const float x = clean(Elem<T>::load(z + i));
                const uint32_t k = key_of(x);
                if (k < floor || (shift < 24 && (k >> (shift + 8)) != (prefix >> (shift + 8)))) continue;
                const uint64_t v = weights ? weigh(x) : 1u;
                if (v) atomicAdd(reinterpret_cast<unsigned long long *>(&hist[(k >> shift) & 255]), (unsigned long long)v);
            }
            __syncthreads();
            if (t == 0) {
                uint64_t seen = before;
                int d = 255;
                for (; d > 0 && seen + hist[d] < goal; --d) seen += hist[d];
                found[0] = (uint64_t)d;
                found[1] = seen;
            }
            __syncthreads();
            prefix |= (uint32_t)found[0] << shift;
            before = found[1];
            __syncthreads();
        }
        at = prefix;
    };

    // the first top_k
    uint32_t floor = 0;
    uint64_t ties = ~0ull;                    // how many of the classes with key `floor` belong
    const int64_t k = greedy ? 1 : top_k;
    if (k > 0 && k < c) {
        uint64_t before;
        select(false, (uint64_t)k, 0, floor, before);
        ties = (uint64_t)k - before;
    }
    // the weight of those, and the shortest run that holds top_p of it
    uint64_t sum = 0, total;
    for (int i = t; i < c; i += NT) {
        const float x = clean(Elem<T>::load(z + i));
        const uint32_t key = key_of(x);
        if (key > floor || (key == floor && ties == ~0ull)) sum += weigh(x);
    }
    group_scan<NT>(sum, part, total);
    if (ties != ~0ull) total += ties * weigh(of_key(floor));
    if (top_p < 1.0f) {
        const double wanted = ceil((double)top_p * (double)total);
        uint64_t need = wanted > 1.0 ? (uint64_t)wanted : 1;
        need = need < total ? need : total;
        uint32_t at;
        uint64_t before;
        select(true, need, floor, at, before);
        const uint64_t q = weigh(of_key(at));
        const uint64_t mine = (need - before + q - 1) / q;       // (the run ends at a class with weight)
        if (at != floor || ties == ~0ull) ties = mine;
        else ties = mine < ties ? mine : ties;
        floor = at;
        total = before + ties * q;
    }
    uint64_t target = u > 0.0f ? (uint64_t)((double)u * (double)total) : 0;
    target = target < total ? target : total - 1;
    // by index
    uint64_t seen = 0, tied = 0;
    for (int base = 0; base < c; base += NT * 8) {
        float x[8];
        uint64_t mine = 0;
        int equal = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = base + t * 8 + j;
            x[j] = i < c ? clean(Elem<T>::load(z + i)) : -__builtin_inff();
            equal += i < c && key_of(x[j]) == floor;
        }
        uint64_t all_equal, all;
        uint64_t rank = tied + group_scan<NT>((uint64_t)equal, part, all_equal);
        uint32_t q[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t key = key_of(x[j]);
            const int i = base + t * 8 + j;
            q[j] = i < c && (key > floor || (key == floor && rank < ties)) ? weigh(x[j]) : 0u;
            rank += i < c && key == floor;
            mine += q[j];
        }
        uint64_t front = seen + group_scan<NT>(mine, part, all);
        if (target >= front && target < front + mine) {
            for (int j = 0; j < 8; ++j) {
                if (target < front + q[j]) {
                    a.classes[row] = base + t * 8 + j;
                    if (a.probs) a.probs[row] = (float)((double)q[j] / (double)total);
                    break;
                }
                front += q[j];
            }
        }
        seen += all;
        tied += all_equal;
        if (seen > target) break;
    }
}

}  // namespace wpsgd

using namespace wpsgd;

extern "C" {

size_t wpsgd_draw_classes_workspace(int64_t n, int64_t classes, wpsgd_dtype dtype)
{
    (void)n; (void)classes; (void)dtype;
    return 0;
}

int wpsgd_draw_classes(const void *Z, int64_t n, int64_t classes, int64_t ld, wpsgd_dtype dtype, const float *u, const wpsgd_draw_rule *rule, int64_t *drawn,
                       float *probs, void *workspace, size_t workspace_bytes, void *stream)
{
    if (n < 0 || n > 0x7FFFFFFFLL || classes < 1 || classes > (1LL << 24) || (dtype != WPSGD_F32 && dtype != WPSGD_BF16) || !rule) return WPSGD_INVALID_ARG;
    if (!rule->row_temperature && !(rule->temperature >= 0.0f)) return WPSGD_INVALID_ARG;
    if ((!rule->row_top_p && std::isnan(rule->top_p)) || (!rule->row_min_p && !(rule->min_p <= 1.0f))) return WPSGD_INVALID_ARG;
    if (n == 0) return WPSGD_OK;
    const size_t elem = dtype == WPSGD_F32 ? 4 : 2;
    if (!Z || !u || !drawn || ld < classes || (uintptr_t)Z % elem != 0) return WPSGD_INVALID_ARG;
    const size_t need = wpsgd_draw_classes_workspace(n, classes, dtype);
    if (need && (!workspace || (uintptr_t)workspace % 256 != 0)) return WPSGD_INVALID_ARG;
    if (workspace_bytes < need) return WPSGD_WORKSPACE_TOO_SMALL;
    const DrawArgs a{Z, n, classes, ld, u, *rule, drawn, probs};
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (dtype == WPSGD_F32) hipLaunchKernelGGL(draw_simple_kernel<float>, dim3((unsigned)n), dim3(256), 0, s, a);
    else hipLaunchKernelGGL(draw_simple_kernel<uint16_t>, dim3((unsigned)n), dim3(256), 0, s, a);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? WPSGD_OK : hip_fail(e);
}

}  // extern "C"
