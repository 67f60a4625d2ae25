// Shared by the operators of the many-class linear model: loads of whatever alignment and reductions over a workgroup.
#pragma once

#include "device_utils.h"
#include "internal.h"

namespace wpsgd {

// Sixteen bytes at any address that an element may have: one load or store, which touches nine lines instead of eight per wave where
// rows are not aligned.  Said to be global memory, since some addresses come out of memory and flat accesses cost more.
struct Bytes16 {
    uint32_t w[4];
};
typedef uint32_t words4 __attribute__((ext_vector_type(4)));
typedef words4 any_words4 __attribute__((aligned(2)));
template <typename T> using global_ptr = __attribute__((address_space(1))) T *;

__device__ inline Bytes16 load16(const void *p)
{
    const words4 v = *(global_ptr<const any_words4>)p;
    return Bytes16{{v.x, v.y, v.z, v.w}};
}
__device__ inline void store16(void *p, const Bytes16 &q) { *(global_ptr<any_words4>)p = words4{q.w[0], q.w[1], q.w[2], q.w[3]}; }

template <typename T> struct Elem;
template <> struct Elem<float> {
    static constexpr int kPer16 = 4;
    __device__ static float load(const float *p) { return *(global_ptr<const float>)p; }
    __device__ static float get(const uint32_t (&w)[4], int j) { return __uint_as_float(w[j]); }
    __device__ static void put(float *p, float v) { *(global_ptr<float>)p = v; }
};
template <> struct Elem<uint16_t> {                      // bfloat16
    static constexpr int kPer16 = 8;
    __device__ static float load(const uint16_t *p) { return bf16_one(*(global_ptr<const uint16_t>)p); }
    __device__ static float get(const uint32_t (&w)[4], int j) { return (j & 1) ? bf16_hi(w[j >> 1]) : bf16_lo(w[j >> 1]); }
    __device__ static void put(uint16_t *p, float v);
};

// two fp32 values to bfloat16, nearest even, the first in the lower half
__device__ inline uint32_t bf16_pack(float a, float b)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 r = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, r);
}
__device__ inline void Elem<uint16_t>::put(uint16_t *p, float v) { *(global_ptr<uint16_t>)p = (uint16_t)bf16_pack(v, v); }

// Eight elements, of which the first `left` (1 or more) are there; 0 for the others.  (Those that are not there ask for the last that is: all loads on their way at once, where a branch
// around each would wait for one after the other.)
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
        for (int j = 0; j < 8; ++j) x[j] = Elem<T>::load(p + (j < left ? j : left - 1));
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = j < left ? x[j] : 0.0f;
    }
}

__device__ inline float wave_max(float v)
{
    // (fmaxf drops a NaN; the callers that want it kept look for it in the sums)
    v = fmaxf(v, dpp_move<0xB1, 0xF>(v));
    v = fmaxf(v, dpp_move<0x4E, 0xF>(v));
    v = fmaxf(v, dpp_move<0x141, 0xF>(v));
    v = fmaxf(v, dpp_move<0x140, 0xF>(v));
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}

// A launch has fewer than 2^32 threads along x.
constexpr int64_t most_groups(int threads) { return 0xFFFFFFFFLL / threads; }
// Any number of workgroups, in as many launches as that takes: run(first, count) queues one.
template <typename F>
inline hipError_t in_launches(int64_t groups, int threads, F &&run)
{
    const int64_t most = most_groups(threads);
    for (int64_t first = 0; first < groups; first += most) {
        run(first, (unsigned)(groups - first < most ? groups - first : most));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace wpsgd
