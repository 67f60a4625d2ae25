// The global norm of a gradient that lies in many tensors, clipping, and the regularised SGD step on all of them.
//
//   norm = sqrt(sum over all tensors of g^2)      (fp64: squares of fp32 values neither overflow nor round there)
//   c    = min(1, max_norm / norm)
//   w   <- (1 - eta lambda) w - eta c g           a norm that is not finite changes nothing
//
// A list's table, made once, cuts the tensors into chunks of some thousand elements, so that the kernels see one flat sequence of equal pieces
// whatever the tensors' number and sizes.
#include <cmath>
#include <vector>

#include "class_ops.h"

namespace wpsgd {

// Elements of a chunk.  A small model in small chunks, so that it spreads over the chip; a large one in large ones, of which a workgroup asks for several vectors at a
// time (a small chunk of bfloat16 has one for each thread).  So an element of bfloat16 counts as four.  us for the norm and for the whole step, 2048 | 16384 to a chunk, out of the caches:
// fp32 1M 8.1, 7.8 | 8.3, 12.1; 3M 7.5, 13.6 | 8.5, 17.9; 8M 11.4, 28.8 | 13.1, 28.4; 12M 14.1, 39.7 | 14.8, 39.3; 128M 90.6, 391 | 86.9, 386;
// bfloat16 1M 7.3, 7.8 | 7.4, 8.7; 2M 7.2, 10.0 | 7.4, 9.5; 3M 7.5, 12.0 | 7.5, 10.5; 8M 9.9, 27.2 | 7.2, 22.7; 128M 87.1, 331 | 45.4, 286.
constexpr int kLargeChunk = 16384, kSmallChunk = 2048;
constexpr int64_t kSmallModel = 8 << 20;
constexpr int kNormGroups = 1024;        // partial sums at most, one per workgroup

struct Chunk {
    void *g;
    float *w;
    int32_t n;
    int32_t dtype;
    int64_t unused;
};
static_assert(sizeof(Chunk) == 32, "four to a line of 128 bytes");

constexpr int kAtOnce = 4;               // vectors on their way

template <typename T>
__device__ inline double sum_squares(const T *g, int n)
{
    constexpr int E = Elem<T>::kPer16;
    const int vectors = n / E;
    double s = 0.0;
    for (int v0 = threadIdx.x; v0 < vectors; v0 += 256 * kAtOnce) {
        Bytes16 q[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) q[u] = v0 + u * 256 < vectors ? load16(g + (v0 + u * 256) * E) : Bytes16{{0, 0, 0, 0}};
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const double x = (double)Elem<T>::get(q[u].w, j);
                s = fma(x, x, s);
            }
    }
    const int at = vectors * E + threadIdx.x;
    if (at < n) {
        const double x = (double)Elem<T>::load(g + at);
        s = fma(x, x, s);
    }
    return s;
}

__device__ inline double group_sum(double s, double *part)
{
    s = wave_sum(s);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    s = (part[0] + part[1]) + (part[2] + part[3]);
    __syncthreads();
    return s;
}

__global__ __launch_bounds__(256) void square_sums_kernel(const Chunk *chunks, int64_t count, double *partials)
{
    __shared__ double part[4];
    double s = 0.0;
    for (int64_t i = blockIdx.x; i < count; i += gridDim.x) {
        const Chunk c = chunks[i];
        s += c.dtype == WPSGD_BF16 ? sum_squares(static_cast<const uint16_t *>(c.g), c.n) : sum_squares(static_cast<const float *>(c.g), c.n);
    }
    s = group_sum(s, part);
    if (threadIdx.x == 0) partials[blockIdx.x] = s;
}

__device__ inline double total_of(const double *partials, int count, double *part)
{
    double s = 0.0;
    for (int i = threadIdx.x; i < count; i += 256) s += partials[i];
    return group_sum(s, part);
}

__global__ __launch_bounds__(256) void norm_kernel(const double *partials, int count, float *norm)
{
    __shared__ double part[4];
    const double s = total_of(partials, count, part);
    if (threadIdx.x == 0) *norm = (float)sqrt(s);
}

struct StepArgs {
    const Chunk *chunks;
    int64_t count;
    const double *partials;
    int groups;
    float *norm;
    double eta, shrink, max_norm;
};

// In fp64, rounded once: a factor that fp32 cannot hold (a huge norm) is no special case, and memory still bounds the kernel.
__device__ inline float stepped(float w, float g, double shrink, double factor) { return (float)fma((double)w, shrink, -factor * (double)g); }

template <typename T>
__device__ inline void step_chunk(const Chunk &c, double shrink, double factor)
{
    constexpr int E = Elem<T>::kPer16, U = 16 / E;
    const T *g = static_cast<const T *>(c.g);
    const int vectors = c.n / E;
    for (int v0 = threadIdx.x; v0 < vectors; v0 += 256 * U) {
        Bytes16 q[U], w[U][E / 4];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int v = v0 + u * 256 < vectors ? v0 + u * 256 : v0;
            q[u] = load16(g + v * E);
#pragma unroll
            for (int h = 0; h < E / 4; ++h) w[u][h] = load16(c.w + v * E + h * 4);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int v = v0 + u * 256;
            if (v >= vectors) break;
#pragma unroll
            for (int h = 0; h < E / 4; ++h) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    w[u][h].w[j] = __float_as_uint(stepped(__uint_as_float(w[u][h].w[j]), Elem<T>::get(q[u].w, h * 4 + j), shrink, factor));
                store16(c.w + v * E + h * 4, w[u][h]);
            }
        }
    }
    const int at = vectors * E + threadIdx.x;
    if (at < c.n) Elem<float>::put(c.w + at, stepped(Elem<float>::load(c.w + at), Elem<T>::load(g + at), shrink, factor));
}

// (Asking for the first chunk's vectors in front of the norm gains nothing: 9.2 us instead of 8.1 for 3M elements, 635 instead of 625 for 268M.)
__global__ __launch_bounds__(256) void clipped_step_kernel(StepArgs a)
{
    __shared__ double part[4];
    const double norm = sqrt(total_of(a.partials, a.groups, part));
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.norm = (float)norm;
    if (!(norm < __builtin_inf())) return;
    const double factor = norm > a.max_norm ? a.eta * (a.max_norm / norm) : a.eta;
    // from the end: what the norm has read last may still be in the caches
    for (int64_t i = a.count - 1 - blockIdx.x; i >= 0; i -= gridDim.x) {
        const Chunk c = a.chunks[i];
        if (c.dtype == WPSGD_BF16) step_chunk<uint16_t>(c, a.shrink, factor);
        else step_chunk<float>(c, a.shrink, factor);
    }
}

template <typename T>
__device__ inline void scale_chunk(const Chunk &c, double factor)
{
    constexpr int E = Elem<T>::kPer16;
    T *g = static_cast<T *>(c.g);
    const int vectors = c.n / E;
    for (int v = threadIdx.x; v < vectors; v += 256) {
        Bytes16 q = load16(g + v * E);
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            if constexpr (E == 8) q.w[h] = bf16_pack((float)(factor * Elem<T>::get(q.w, 2 * h)), (float)(factor * Elem<T>::get(q.w, 2 * h + 1)));
            else q.w[h] = __float_as_uint((float)(factor * Elem<T>::get(q.w, h)));
        }
        store16(g + v * E, q);
    }
    const int at = vectors * E + threadIdx.x;
    if (at < c.n) Elem<T>::put(g + at, (float)(factor * Elem<T>::load(g + at)));
}

__global__ __launch_bounds__(256) void clip_kernel(StepArgs a)
{
    __shared__ double part[4];
    const double norm = sqrt(total_of(a.partials, a.groups, part));
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.norm = (float)norm;
    if (!(norm < __builtin_inf()) || norm <= a.max_norm) return;             // nothing to scale: nothing is written
    const double factor = a.max_norm / norm;
    for (int64_t i = a.count - 1 - blockIdx.x; i >= 0; i -= gridDim.x) {
        const Chunk c = a.chunks[i];
        if (c.dtype == WPSGD_BF16) scale_chunk<uint16_t>(c, factor);
        else scale_chunk<float>(c, factor);
    }
}

static int norm_groups(int64_t chunks) { return (int)(chunks < kNormGroups ? chunks : kNormGroups); }

static int check_list(const wpsgd_tensor_list *l, float *norm, void *workspace, size_t bytes)
{
    if (!l || l->chunks < 0 || (l->chunks > 0 && !l->table) || !norm || (uintptr_t)norm % 4 != 0) return WPSGD_INVALID_ARG;
    if (!workspace || (uintptr_t)workspace % 256 != 0) return WPSGD_INVALID_ARG;
    return bytes < wpsgd_grad_norm_workspace(l) ? WPSGD_WORKSPACE_TOO_SMALL : WPSGD_OK;
}

static hipError_t launch_square_sums(const wpsgd_tensor_list *l, double *partials, hipStream_t s)
{
    if (l->chunks == 0) return hipSuccess;
    hipLaunchKernelGGL(square_sums_kernel, dim3(norm_groups(l->chunks)), dim3(256), 0, s, static_cast<const Chunk *>(l->table), l->chunks, partials);
    return hipGetLastError();
}

static int64_t chunk_of(int64_t counted) { return counted <= kSmallModel ? kSmallChunk : kLargeChunk; }
static int64_t counted_of(const wpsgd_tensor &t) { return t.dtype == WPSGD_BF16 ? 4 * t.n : t.n; }
// -1 for descriptions that cannot be
static int64_t count_chunks(const wpsgd_tensor *tensors, int64_t count)
{
    if (count < 0 || (count > 0 && !tensors)) return -1;
    int64_t elements = 0, counted = 0, chunks = 0;
    for (int64_t i = 0; i < count; ++i) {
        if (tensors[i].n < 0 || tensors[i].n > (1LL << 44) || elements > (1LL << 44)) return -1;
        elements += tensors[i].n;
        counted += counted_of(tensors[i]);
    }
    for (int64_t i = 0; i < count; ++i) chunks += (tensors[i].n + chunk_of(counted) - 1) / chunk_of(counted);
    return chunks;
}

static unsigned step_groups(int64_t chunks) { return (unsigned)(chunks < 1 ? 1 : chunks < 4096 ? chunks : 4096); }

}  // namespace wpsgd

using namespace wpsgd;

extern "C" {

size_t wpsgd_tensor_list_bytes(const wpsgd_tensor *tensors, int64_t count)
{
    const int64_t chunks = count_chunks(tensors, count);
    return chunks < 0 ? 0 : ((size_t)(chunks < 1 ? 1 : chunks) * sizeof(Chunk) + 255) & ~(size_t)255;
}

int wpsgd_tensor_list_make(const wpsgd_tensor *tensors, int64_t count, void *table, size_t table_bytes, wpsgd_tensor_list *list, void *stream)
{
    const int64_t chunks = count_chunks(tensors, count);
    if (chunks < 0 || !list || !table || (uintptr_t)table % 256 != 0) return WPSGD_INVALID_ARG;
    if (table_bytes < wpsgd_tensor_list_bytes(tensors, count)) return WPSGD_WORKSPACE_TOO_SMALL;
    bool weights = true;
    int64_t elements = 0, counted = 0;
    for (int64_t i = 0; i < count; ++i) {
        const wpsgd_tensor &t = tensors[i];
        if (t.dtype != WPSGD_F32 && t.dtype != WPSGD_BF16) return WPSGD_INVALID_ARG;
        if (t.n == 0) continue;
        if (!t.grad || (uintptr_t)t.grad % (t.dtype == WPSGD_F32 ? 4 : 2) != 0 || (uintptr_t)t.weight % 4 != 0) return WPSGD_INVALID_ARG;
        weights = weights && t.weight;
        elements += t.n;
        counted += counted_of(t);
    }
    try {
        const int64_t each = chunk_of(counted);
        std::vector<Chunk> host;
        host.reserve((size_t)chunks);
        for (int64_t i = 0; i < count; ++i) {
            const wpsgd_tensor &t = tensors[i];
            for (int64_t at = 0; at < t.n; at += each)
                host.push_back(Chunk{static_cast<char *>(t.grad) + at * (t.dtype == WPSGD_F32 ? 4 : 2), t.weight ? t.weight + at : nullptr,
                                     (int32_t)(t.n - at < each ? t.n - at : each), (int32_t)t.dtype, 0});
        }
        if (chunks > 0) {
            const int rc = upload(table, host.data(), host.size() * sizeof(Chunk), static_cast<hipStream_t>(stream));
            if (rc != WPSGD_OK) return rc;
        }
    } catch (...) {                          // no memory on the host
        return WPSGD_INVALID_ARG;
    }
    *list = wpsgd_tensor_list{table, chunks, elements, weights ? 1 : 0};
    return WPSGD_OK;
}

size_t wpsgd_grad_norm_workspace(const wpsgd_tensor_list *list)
{
    (void)list;
    return kNormGroups * sizeof(double);
}

int wpsgd_grad_norm(const wpsgd_tensor_list *list, float *norm, void *workspace, size_t workspace_bytes, void *stream)
{
    const int rc = check_list(list, norm, workspace, workspace_bytes);
    if (rc != WPSGD_OK) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    double *partials = static_cast<double *>(workspace);
    hipError_t e = launch_square_sums(list, partials, s);
    if (e != hipSuccess) return hip_fail(e);
    hipLaunchKernelGGL(norm_kernel, dim3(1), dim3(256), 0, s, partials, norm_groups(list->chunks), norm);
    e = hipGetLastError();
    return e == hipSuccess ? WPSGD_OK : hip_fail(e);
}

int wpsgd_clip_grads(const wpsgd_tensor_list *list, double max_norm, float *norm, void *workspace, size_t workspace_bytes, void *stream)
{
    const int rc = check_list(list, norm, workspace, workspace_bytes);
    if (rc != WPSGD_OK) return rc;
    if (!(max_norm > 0.0)) return WPSGD_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    double *partials = static_cast<double *>(workspace);
    hipError_t e = launch_square_sums(list, partials, s);
    if (e != hipSuccess) return hip_fail(e);
    const StepArgs a{static_cast<const Chunk *>(list->table), list->chunks, partials, norm_groups(list->chunks), norm, 0.0, 1.0, max_norm};
    hipLaunchKernelGGL(clip_kernel, dim3(step_groups(list->chunks)), dim3(256), 0, s, a);
    e = hipGetLastError();
    return e == hipSuccess ? WPSGD_OK : hip_fail(e);
}

int wpsgd_clipped_step(const wpsgd_tensor_list *list, double eta, double lambda, double max_norm, float *norm, void *workspace, size_t workspace_bytes,
                       void *stream)
{
    const int rc = check_list(list, norm, workspace, workspace_bytes);
    if (rc != WPSGD_OK) return rc;
    if (!list->has_weights || !(eta > 0.0) || !(lambda >= 0.0) || !(eta * lambda < 1.0) || !std::isfinite(eta) || !(max_norm > 0.0)) return WPSGD_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    double *partials = static_cast<double *>(workspace);
    hipError_t e = launch_square_sums(list, partials, s);
    if (e != hipSuccess) return hip_fail(e);
    const StepArgs a{static_cast<const Chunk *>(list->table), list->chunks, partials, norm_groups(list->chunks), norm, eta, 1.0 - eta * lambda, max_norm};
    hipLaunchKernelGGL(clipped_step_kernel, dim3(step_groups(list->chunks)), dim3(256), 0, s, a);
    e = hipGetLastError();
    return e == hipSuccess ? WPSGD_OK : hip_fail(e);
}

}  // extern "C"
