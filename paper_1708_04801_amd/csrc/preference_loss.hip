// Loss of paired log ratios, with its gradient.  With l_i the log probability of row i's class and g_i = r_i (l_i - ref_i), a pair p of sequences of rows, the first of them
// preferred, has the margin
//   h_p = beta (sum of g_i over its first sequence - sum of g_i over its second),
//   loss_p = w_p ((1 - eps) L(h_p) + eps L(-h_p)),   L(h) = max(0, 1 - h) or log(1 + exp(-h)),
//   grad_ic = f_i (softmax(z_i)_c - [c = label_i]),  f_i = -+ scale beta r_i w_p ((1 - eps) L'(h_p) - eps L'(-h_p)).
// A row's gradient waits for its whole pair, so the scores are read twice: row_softmax.h's pass leaves each row's statistics and g_i, a workgroup a pair adds those up (in fp64,
// in an order that depends on the lengths alone) and leaves each row's f_i, and the last pass forms the gradient.  16 pairs of some 512 rows of 65536 bfloat16 scores: 197 us, 5.1 and 393, all
// of it memory, 5.4 TB/s of the three passes' 3.2 GB (reading alone reaches 6.4 TB/s on this card, writing alone 6.8 to 7.5, one beside the other the last pass's 5.4).  A pair at a time, whose
// 64 MB the Infinity Cache still holds for the second reading, the last passes take 365 us together, the first ones 420 instead of 197: too short to fill the card.
#include "row_softmax.h"

namespace wpsgd {

struct RowResult {             // of the first pass, in the workspace
    float2 *state;             // m_i and s_i
    float *factor;             // 0, and f_i from the second pass on
    double *gain;              // g_i
};

// g_i: 0 where the class has no probability under either model
__device__ inline double gain_of(const RowState &x, float r, double ref)
{
    constexpr double kInf = __builtin_inf();
    const double l = x.unknown ? __builtin_nan("") : x.empty ? -kInf : ((double)x.z_label - (double)x.m) - log(x.sum);
    return l == -kInf && ref == -kInf ? 0.0 : (double)r * (l - ref);
}

struct GainOfRow {
    static constexpr bool kOneWave = true, kWideSum = true;
    RowResult to;
    const float *ref_log;
    // (rows that no sequence holds too: no pair adds them up, and their factors stay 0.  The first and the last offset could tell them apart only if all offsets were right.)
    __device__ bool counts(int64_t, int64_t label, float r) const { return !(label < 0 || r == 0.0f); }
    __device__ void absent(int64_t row) const
    {
        to.factor[row] = 0.0f;
        to.gain[row] = 0.0;
    }
    __device__ float make(int64_t row, float r, const RowState &x, bool writes) const
    {
        const double ref = ref_log ? (double)ref_log[row] : 0.0;
        if (writes) {
            to.state[row] = make_float2(x.m, x.s);
            to.factor[row] = 0.0f;
            to.gain[row] = gain_of(x, r, ref);
        }
        return 0.0f;
    }
};

struct PairArgs {
    const int64_t *labels, *offsets;
    int64_t n, pairs;
    const float *row_weights, *pair_weights;
    int hinge;
    double beta, smoothing, scale;
    RowResult rows;
    float *loss, *margin;
    int64_t first;
};

// L(h) and L'(h)
__device__ inline double pair_loss(double h, bool hinge, double &slope)
{
    if (hinge) {
        slope = h < 1.0 ? -1.0 : h == h ? 0.0 : h;
        return h < 1.0 ? 1.0 - h : h == h ? 0.0 : h;
    }
    const double e = exp(-fabs(h));
    slope = -(h >= 0.0 ? e : 1.0) / (1.0 + e);
    return (h < 0.0 ? -h : 0.0) + log1p(e);
}

// what a pair with a margin of h comes to, written by `writes`; its rows' factors are this times -+ their weights
__device__ inline double pair_result(const PairArgs &a, int64_t p, double h, double w, bool writes)
{
    double slope, back;
    double loss = pair_loss(h, a.hinge != 0, slope);
    if (a.smoothing != 0.0) {
        loss = (a.smoothing != 1.0 ? (1.0 - a.smoothing) * loss : 0.0) + a.smoothing * pair_loss(-h, a.hinge != 0, back);   // (loss may be infinite)
        slope = (1.0 - a.smoothing) * slope - a.smoothing * back;
    }
    if (writes) {
        a.loss[p] = w == 0.0 ? 0.0f : (float)(w * loss);
        a.margin[p] = (float)h;
    }
    return -a.scale * a.beta * w * slope;
}

// A workgroup a pair, four rows to a thread at a time, all asked for before the first is added (one pair of 131072 rows, with the passes over 1024 bfloat16 scores a row: 430 us with 256
// threads that ask for one at a time, 213 so; 1024 pairs of 8 rows, of 4099 scores: 43 with 256 threads to a pair, 49 with 1024).
constexpr int kPairRows = 4;
template <int kPairThreads>
__global__ __launch_bounds__(kPairThreads) void pair_kernel(PairArgs a)
{
    __shared__ double part[kPairThreads / 64];
    const int64_t p = a.first + blockIdx.x;
    const int t = threadIdx.x;
    const int64_t from = a.offsets[2 * p], middle = a.offsets[2 * p + 1], to = a.offsets[2 * p + 2];
    const double w = a.pair_weights ? (double)a.pair_weights[p] : 1.0;
    if (from < 0 || middle < from || to < middle || to > a.n) {                   // no such rows
        if (t == 0) a.loss[p] = a.margin[p] = __builtin_nanf("");
        return;
    }
    double sum = 0.0;
    for (int64_t i = from + t; i < to; i += kPairThreads * kPairRows) {
        double gain[kPairRows];
#pragma unroll
        for (int y = 0; y < kPairRows; ++y) gain[y] = i + y * kPairThreads < to ? a.rows.gain[i + y * kPairThreads] : 0.0;
#pragma unroll
        for (int y = 0; y < kPairRows; ++y) sum += i + y * kPairThreads < middle ? gain[y] : -gain[y];
    }
    sum = wave_sum(sum);
    if ((t & 63) == 0) part[t >> 6] = sum;
    __syncthreads();
    sum = part[0];
#pragma unroll
    for (int o = 1; o < kPairThreads / 64; ++o) sum += part[o];
    const double f = pair_result(a, p, a.beta * sum, w, t == 0);
    if (w == 0.0) return;
    for (int64_t i = from + t; i < to; i += kPairThreads * kPairRows) {
        int64_t label[kPairRows];
        float r[kPairRows];
#pragma unroll
        for (int y = 0; y < kPairRows; ++y) {
            const int64_t row = i + y * kPairThreads;
            label[y] = row < to ? a.labels[row] : -1;
            r[y] = row < to && a.row_weights ? a.row_weights[row] : 1.0f;
        }
#pragma unroll
        for (int y = 0; y < kPairRows; ++y) {
            const int64_t row = i + y * kPairThreads;
            if (label[y] >= 0 && r[y] != 0.0f) a.rows.factor[row] = (float)(row < middle ? f * (double)r[y] : -f * (double)r[y]);
        }
    }
}

// The gradient, one row to NT threads, from the last row on: what the first pass read last may still be in the caches.
template <typename T, int NT>
__global__ __launch_bounds__(256) void pair_gradient_kernel(RowArgs a, RowResult rows)
{
    constexpr int E = Elem<T>::kPer16, kRows = 256 / NT;
    const int64_t place = (a.first + blockIdx.x) * kRows + threadIdx.x / NT;
    if (place >= a.n) return;
    const int64_t row = a.n - 1 - place;
    const int t = threadIdx.x % NT;
    const T *z = static_cast<const T *>(a.z) + row * a.ld;
    T *g = static_cast<T *>(a.grad) + row * a.ld_grad;
    const int c = (int)a.c, vectors = c / E, tail = c - vectors * E;
    const float f = rows.factor[row];
    const float2 x = f != 0.0f ? rows.state[row] : make_float2(0.0f, 0.0f);
    if (f == 0.0f || x.y == 0.0f) {                                               // does not count, or has no class left
        for (int v = t; v < vectors; v += NT) store16(g + (int64_t)v * E, Bytes16{{0, 0, 0, 0}});
        if (t < tail) Elem<T>::put(g + (int64_t)vectors * E + t, 0.0f);
        return;
    }
    const int64_t label = a.labels[row];
    const int at_label = label < a.c ? (int)label : -1;
    const float base = x.x, over = f / x.y;
    for (int v = t; v < vectors; v += NT) {
        const Bytes16 q = load16(z + (int64_t)v * E);
        float p[E];
#pragma unroll
        for (int j = 0; j < E; ++j) p[j] = exp_of<T>(Elem<T>::get(q.w, j) - base) * over;
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
    }
    if (t < tail) {
        const int at = vectors * E + t;
        const float p = exp_of<T>(Elem<T>::load(z + at) - base) * over;
        Elem<T>::put(g + at, at_label == at ? p - f : p);
    }
}

// Short rows and few of them: a workgroup forms a whole pair, its waves a row each in turn, statistics first (and for all its rows at once what a lane makes of each) and, when the pair's
// margin is known, the gradient, of the last row out of the registers, of the others once more from the caches.  One launch instead of three: 6 pairs of 18 rows of 1001 fp32 scores, 11.3 us
// a call of which the host takes most.  The workgroups behind the pairs' zero the gradient of rows that no sequence holds.
constexpr int kPairWaves = 16, kPairVectors = 4, kMostPairs = 32 * kPairWaves;      // (a thread looks at one step between two offsets)
template <typename T> constexpr int64_t most_pair_classes() { return 64 * kPairVectors * Elem<T>::kPer16; }
static bool pair_in_one(int64_t n, int64_t classes, int64_t pairs, wpsgd_dtype dtype)
{
    // us a call, so | by three kernels (these in a graph 10): 32 rows of one pair 12.3 | 18.4 (1001 fp32), 14.0 | 18.5 (2000 bfloat16); 64 of one 20 | 18.4; 200 of three 21 | 18.4.
    // All rows may belong to one pair: 256 take some 70.  Pairs of a row or none (200 rows of 300 fp32, in a graph): 300 pairs 8.5, 513 of them 10.6 | 10.0, 1000 15.4 | 10.7, 4000 48 | 15.
    return classes <= (dtype == WPSGD_F32 ? most_pair_classes<float>() : most_pair_classes<uint16_t>()) && n <= 256 && n <= 32 * pairs && pairs <= kMostPairs;
}

template <typename T>
__global__ __launch_bounds__(64 * kPairWaves) void whole_pair_kernel(PairArgs a, RowArgs z, const float *ref_log)
{
    constexpr int E = Elem<T>::kPer16, V = kPairVectors;
    constexpr float kInf = __builtin_inff();
    __shared__ double part[kPairWaves];
    __shared__ bool falls[kPairWaves];
    const int64_t p = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = (int)z.c, vectors = c / E, tail = c - vectors * E;
    auto zero = [&](int64_t row) {
        T *g = static_cast<T *>(z.grad) + row * z.ld_grad;
        for (int v = lane; v < vectors; v += 64) store16(g + (int64_t)v * E, Bytes16{{0, 0, 0, 0}});
        if (lane < tail) Elem<T>::put(g + (int64_t)vectors * E + lane, 0.0f);
    };
    // A gradient that takes the scores' place: where an offset is under the one before it, a row may belong to two pairs, or to one and to none, and would be written before all have
    // read it.  No gradient is written then.
    const bool in_place = z.grad == z.z;
    const bool down = in_place && threadIdx.x < 2 * a.pairs && a.offsets[threadIdx.x] > a.offsets[threadIdx.x + 1];
    if (p >= a.pairs) {
        if (!z.grad || (in_place && __syncthreads_or(down))) return;
        const int64_t first = a.offsets[0], last = a.offsets[2 * a.pairs], others = gridDim.x - a.pairs;
        for (int64_t row = (p - a.pairs) * kPairWaves + wave; row < a.n; row += others * kPairWaves)
            if (row < first || row >= last) zero(row);
        return;
    }
    const int64_t from = a.offsets[2 * p], middle = a.offsets[2 * p + 1], to = a.offsets[2 * p + 2];
    const double w = a.pair_weights ? (double)a.pair_weights[p] : 1.0;
    if (from < 0 || middle < from || to < middle || to > a.n) {                   // no such rows
        if (threadIdx.x == 0) a.loss[p] = a.margin[p] = __builtin_nanf("");
        return;
    }
    // Row wave + 16 i of the pair is the wave's i-th, and lane i keeps what is known of it.
    const int count = to - from > wave ? (int)((to - from - wave + kPairWaves - 1) / kPairWaves) : 0;
    const int64_t row0 = from + wave, mine = row0 + (int64_t)lane * kPairWaves;
    Bytes16 raw[V];
    float last;
    auto ask = [&](int i) {
        const T *q = static_cast<const T *>(z.z) + (row0 + (int64_t)i * kPairWaves) * z.ld;
#pragma unroll
        for (int v = 0; v < V; ++v) raw[v] = v * 64 + lane < vectors ? load16(q + (int64_t)(v * 64 + lane) * E) : Bytes16{{0, 0, 0, 0}};
        last = lane < tail ? Elem<T>::load(q + (int64_t)vectors * E + lane) : -kInf;
    };
    if (count) ask(0);                                                            // (before it is known whether it counts)
    const int64_t label = lane < count ? z.labels[mine] : -1;
    const float r = lane < count && z.row_weights ? z.row_weights[mine] : 1.0f;
    const double ref = lane < count && ref_log ? (double)ref_log[mine] : 0.0;
    const bool counts = label >= 0 && r != 0.0f;
    const uint64_t all = __ballot(counts), none = __ballot(lane < count && !counts);
    const float z_label = counts && label < z.c ? Elem<T>::load(static_cast<const T *>(z.z) + mine * z.ld + label) : 0.0f;
    // the scores asked for become exponentials relative to the row's maximum m
    float x[V * E], x_last = 0.0f, m = -kInf, my_m = -kInf;
    double my_s = 0.0;
    auto take = [&]() {
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int j = 0; j < E; ++j) x[v * E + j] = v * 64 + lane < vectors ? Elem<T>::get(raw[v].w, j) : -kInf;
        x_last = last;
    };
    auto exponentials = [&]() {
        const float base = m == -kInf ? 0.0f : m;
        x_last = exp_for<T, true>(x_last - base);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (v * 64 >= vectors) break;
#pragma unroll
            for (int j = v * E; j < v * E + E; ++j) x[j] = exp_for<T, true>(x[j] - base);
        }
    };
    int held = -1;                                                                // the row whose exponentials the registers hold
    for (uint64_t left = all; left; left &= left - 1) {
        const int i = __builtin_ctzll(left), next = (left & (left - 1)) ? __builtin_ctzll(left & (left - 1)) : i;
        if (held < 0 && i != 0) ask(i);
        take();
        ask(next);
        m = x_last;
#pragma unroll
        for (int j = 0; j < V * E; ++j) m = fmaxf(m, x[j]);
        m = wave_max(fmaxf(m, -kInf));
        exponentials();
        double s = x_last;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (v * 64 >= vectors) break;
            float eight = 0.0f;
#pragma unroll
            for (int j = v * E; j < v * E + E; ++j) eight += x[j];
            s += eight;
        }
        s = wave_sum(s);
        my_m = lane == i ? m : my_m;
        my_s = lane == i ? s : my_s;
        held = i;
    }
    const bool empty = my_m == -kInf && my_s == 0.0;                              // no class left
    double sum = counts ? gain_of(RowState{my_m, (float)my_s, z_label, my_s, empty, label >= z.c}, r, ref) : 0.0;
    sum = wave_sum(mine < middle ? sum : -sum);
    const bool wave_falls = __ballot(down) != 0;
    if (lane == 0) {
        part[wave] = sum;
        falls[wave] = wave_falls;
    }
    __syncthreads();                                                              // (every row's scores have been read: the gradient may take their place)
    sum = part[0];
#pragma unroll
    for (int o = 1; o < kPairWaves; ++o) sum += part[o];
    const double f0 = pair_result(a, p, a.beta * sum, w, threadIdx.x == 0);
    if (!z.grad) return;
    if (in_place) {
        bool any = false;
#pragma unroll
        for (int o = 0; o < kPairWaves; ++o) any |= falls[o];
        if (any) return;
    }
    const float f = (float)(mine < middle ? f0 * (double)r : -f0 * (double)r), over = f / (float)my_s;
    const int at_label = label < z.c ? (int)label : -1;
    const uint64_t nothing = none | __ballot(counts && (w == 0.0 || f == 0.0f || empty));
    for (uint64_t left = nothing; left; left &= left - 1) zero(row0 + (int64_t)__builtin_ctzll(left) * kPairWaves);
    // from the last row on, which is there
    uint64_t left = all & ~nothing;
    int next = left ? 63 - __builtin_clzll(left) : 0;
    if (left && next != held) ask(next);
    while (left) {
        const int i = next;
        left &= ~(1ull << i);
        next = left ? 63 - __builtin_clzll(left) : i;
        if (i != held) take();
        if (left) ask(next);
        if (i != held) {
            m = __shfl(my_m, i);
            exponentials();
        }
        const float f_i = __shfl(f, i), over_i = __shfl(over, i);
        const int at_i = __shfl(at_label, i);
        T *g = static_cast<T *>(z.grad) + (row0 + (int64_t)i * kPairWaves) * z.ld_grad;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (v * 64 + lane >= vectors) continue;
            Bytes16 o;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int at = (v * 64 + lane) * E + j * E / 4;
                if constexpr (E == 8) o.w[j] = bf16_pack(x[v * E + 2 * j] * over_i - (at == at_i ? f_i : 0.0f), x[v * E + 2 * j + 1] * over_i - (at + 1 == at_i ? f_i : 0.0f));
                else o.w[j] = __float_as_uint(x[v * E + j] * over_i - (at == at_i ? f_i : 0.0f));
            }
            store16(g + (int64_t)(v * 64 + lane) * E, o);
        }
        if (lane < tail) {
            const int at = vectors * E + lane;
            Elem<T>::put(g + at, x_last * over_i - (at == at_i ? f_i : 0.0f));
        }
    }
}

template <typename T>
static hipError_t launch_preference(RowArgs a, const GainOfRow &op, PairArgs p, void *grad, bool in_one, hipStream_t s)
{
    if (in_one) {
        a.grad = grad;
        const int64_t others = grad ? (p.n + kPairWaves - 1) / kPairWaves : 0;
        if (p.pairs + others == 0) return hipSuccess;
        hipLaunchKernelGGL(whole_pair_kernel<T>, dim3((unsigned)(p.pairs + others)), dim3(64 * kPairWaves), 0, s, p, a, op.ref_log);
        return hipGetLastError();
    }
    hipError_t e = launch_rows_softmax<T>(a, op, s);
    if (e == hipSuccess)
        e = in_launches(p.pairs, 1024, [&](int64_t first, unsigned count) {
            p.first = first;
            if (p.n <= 256 * p.pairs) hipLaunchKernelGGL(pair_kernel<256>, dim3(count), dim3(256), 0, s, p);
            else hipLaunchKernelGGL(pair_kernel<1024>, dim3(count), dim3(1024), 0, s, p);
        });
    if (e != hipSuccess || !grad) return e;
    a.grad = grad;
    const bool small = a.c <= 64 * 4 * Elem<T>::kPer16;
    return in_launches(small ? (a.n + 3) / 4 : a.n, 256, [&](int64_t first, unsigned count) {
        a.first = first;
        if (small) hipLaunchKernelGGL((pair_gradient_kernel<T, 64>), dim3(count), dim3(256), 0, s, a, op.to);
        else hipLaunchKernelGGL((pair_gradient_kernel<T, 256>), dim3(count), dim3(256), 0, s, a, op.to);
    });
}

}  // namespace wpsgd

using namespace wpsgd;

extern "C" {

size_t wpsgd_preference_loss_workspace(int64_t n, int64_t classes, int64_t pairs, wpsgd_dtype dtype)
{
    if (n <= 0 || n > 0x7FFFFFFFLL || pair_in_one(n, classes, pairs, dtype)) return 0;
    return ((size_t)n * 20 + 255) / 256 * 256;
}

int wpsgd_preference_loss(const void *Z, int64_t n, int64_t classes, int64_t ld, wpsgd_dtype dtype, const int64_t *labels, const int64_t *offsets, int64_t pairs,
                          const float *ref_log, const float *row_weights, const float *pair_weights, wpsgd_loss kind, double beta, double smoothing, double scale,
                          float *loss, float *margin, void *grad, int64_t ld_grad, void *workspace, size_t workspace_bytes, void *stream)
{
    if ((kind != WPSGD_HINGE && kind != WPSGD_LOGISTIC) || pairs < 0 || pairs > 0x3FFFFFFFLL) return WPSGD_INVALID_ARG;
    if (!(beta - beta == 0.0) || !(scale - scale == 0.0) || !(smoothing >= 0.0 && smoothing <= 1.0)) return WPSGD_INVALID_ARG;
    const int rc = check_scores(Z, n, classes, ld, dtype, grad, ld_grad);
    if (rc != WPSGD_OK) return rc;
    if (!offsets || (n > 0 && !labels) || (pairs > 0 && (!loss || !margin))) return WPSGD_INVALID_ARG;
    const size_t need = wpsgd_preference_loss_workspace(n, classes, pairs, dtype);
    if (need && (!workspace || (uintptr_t)workspace % 256 != 0)) return WPSGD_INVALID_ARG;
    if (workspace_bytes < need) return WPSGD_WORKSPACE_TOO_SMALL;
    const RowResult to{reinterpret_cast<float2 *>(static_cast<double *>(workspace) + n), reinterpret_cast<float *>(static_cast<double *>(workspace) + 2 * n),
                       static_cast<double *>(workspace)};
    const RowArgs a{Z, n, classes, ld, labels, row_weights, nullptr, ld_grad, 0};
    const GainOfRow op{to, ref_log};
    const PairArgs p{labels, offsets, n, pairs, row_weights, pair_weights, kind == WPSGD_HINGE, beta, smoothing, scale, to, loss, margin, 0};
    const bool in_one = pair_in_one(n, classes, pairs, dtype);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const hipError_t e = dtype == WPSGD_F32 ? launch_preference<float>(a, op, p, grad, in_one, s) : launch_preference<uint16_t>(a, op, p, grad, in_one, s);
    return e == hipSuccess ? WPSGD_OK : hip_fail(e);
}

}  // extern "C"
