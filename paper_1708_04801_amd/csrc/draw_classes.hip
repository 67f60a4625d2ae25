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

// scores in whole numbers of the same order (x + 0, so that -0 is 0)
__device__ inline uint32_t key_of(float x)
{
    const uint32_t b = __float_as_uint(x);
    return b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ inline float of_key(uint32_t k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xFFFFFFFFu)); }

// classes as keys of 24 bits whose order is the other way round, and back
__device__ inline uint32_t index_key(uint32_t i) { return (0xFFFFFFu - i) << 8; }
__device__ inline uint32_t key_index(uint32_t k) { return 0xFFFFFFu - (k >> 8); }

struct Weigh {
    float top, slope, low;
    // how many powers of two a weight is under the largest, negative or 0; -inf for no weight, and for every other score where the largest is +inf
    __device__ float powers(float x) const { return x == top ? 0.0f : (x - top) * slope; }
    __device__ uint32_t of_powers(float z) const
    {
        const float e = __builtin_amdgcn_exp2f(z);
        return e >= low ? (uint32_t)fmaf(e, kOne, 0.5f) : 0u;           // (NaN: none)
    }
    __device__ uint32_t operator()(float x) const { return of_powers(powers(x)); }
};

// ---- a row in a workgroup ----
// Vector v of thread t holds classes (v NT + t) E and on, sixteen bytes: a wave's vectors are a run of 64 E classes, a "segment".  The row is read again for each
// step, from the caches: kept in registers, its every element would stand in the code of every step.
//   1. the largest score;
//   2. few classes kept (top_k <= NT): the top_k-th largest of the threads' own largest scores is a score that at least top_k classes reach; the classes that do
//      go to a list in LDS (a few times top_k), and everything else is done there;
//   3. else the end of the run: weights (or counts) in bins of 1/16 power of two below the largest, then the bin in which it lies as a list;
//   4. the draw: the kept weight of every segment, the segment, the class.
// Where a list has no room (scores that are nearly all alike) the digits are looked for among all classes of the row.
constexpr int kBins = 1024, kCopies = 4;
constexpr int kMostClasses = 1 << 18;

template <typename T, int NT, int CAP>
struct Row {
    static constexpr int E = Elem<T>::kPer16, kWaves = NT / 64;
    static constexpr int kSegments = kMostClasses / (64 * E);
    static constexpr int kAtATime = 16 / E;        // vectors
    struct Shared {
        union {
            uint64_t hist[256];
            unsigned long long bins[kCopies][kBins];
        };
        uint64_t list[CAP];                        // key << 32 | class
        union {
            uint64_t segment[kSegments];
            float tops[kWaves];
        };
        uint32_t ties[kSegments];
        uint64_t found[2];
        uint64_t sums[kWaves];
        uint32_t count;
        uint32_t cut;
    };
    Shared *sh;
    const T *z;
    int c, t, vectors;                             // vectors: of a thread
    Weigh weigh;

    __device__ __forceinline__ Bytes16 fetch(int v) const
    {
        const int64_t at = ((int64_t)v * NT + t) * E;
        if (at + E <= c) return load16(z + at);
        Bytes16 q;
#pragma unroll
        for (int j = 0; j < 4; ++j) q.w[j] = E == 8 ? 0xFF80FF80u : 0xFF800000u;       // -inf
        if (at < c) {
#pragma unroll
            for (int j = 0; j < E - 1; ++j)
                if (at + j < c) {
                    const uint32_t bits = __float_as_uint(Elem<T>::load(z + at + j));
                    if constexpr (E == 8) q.w[j >> 1] = (j & 1) ? (q.w[j >> 1] & 0xFFFFu) | (bits & 0xFFFF0000u) : (q.w[j >> 1] & 0xFFFF0000u) | (bits >> 16);
                    else q.w[j] = bits;
                }
        }
        return q;
    }
    template <typename F>
    __device__ __forceinline__ void each_vector(F &&f)
    {
        for (int v = 0; v < vectors; v += kAtATime) {
            Bytes16 q[kAtATime];
#pragma unroll
            for (int j = 0; j < kAtATime; ++j) q[j] = fetch(v + j);          // (-inf behind the last class)
#pragma unroll
            for (int j = 0; j < kAtATime; ++j) f(v + j, q[j]);
        }
    }
    // f(score, class) for this thread's classes; a NaN never passes a comparison and has no weight
    template <typename F>
    __device__ __forceinline__ void each(F &&f)
    {
        each_vector([&](int v, const Bytes16 &q) {
#pragma unroll
            for (int j = 0; j < E; ++j) f(Elem<T>::get(q.w, j), (v * NT + t) * E + j);
        });
    }
    __device__ void barrier() const
    {
        __syncthreads();
    }
    __device__ __forceinline__ uint64_t group_sum(uint64_t v)
    {
        for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
        barrier();
        if ((t & 63) == 0) sh->sums[t >> 6] = v;
        barrier();
        uint64_t s = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) s += sh->sums[w];
        return s;
    }
    // Where in descending order of a 32-bit key the sum of the values reaches goal: the key, and the sum in front of it.  walk(f) calls f(key, value) for
    // the classes of this thread that take part.  BITS: how many of the key's upper bits differ.
    template <int BITS, typename W>
    __device__ __forceinline__ uint32_t select(W &&walk, uint64_t goal, uint64_t &before)
    {
        uint32_t prefix = 0;
        before = 0;
#pragma unroll 1
        for (int shift = 24; shift >= 32 - BITS; shift -= 8) {
            barrier();
            for (int i = t; i < 256; i += NT) sh->hist[i] = 0;
            barrier();
            const uint32_t want = shift < 24 ? prefix >> (shift + 8) : 0;
            walk([&](uint32_t key, uint64_t v) {
                if ((shift == 24 || key >> (shift + 8) == want) && v) atomicAdd(reinterpret_cast<unsigned long long *>(&sh->hist[(key >> shift) & 255]), v);
            });
            barrier();
            if (t < 64) {                          // four digits to a lane, the largest first
                uint64_t h[4], mine = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    h[j] = sh->hist[255 - 4 * t - j];
                    mine += h[j];
                }
                uint64_t in = mine;
                for (int d = 1; d < 64; d *= 2) {
                    const uint64_t o = __shfl_up(in, d);
                    if (t >= d) in += o;
                }
                uint64_t front = before + in - mine;
                if (front < goal && goal <= before + in) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (front < goal && goal <= front + h[j]) {
                            sh->found[0] = (uint64_t)(255 - 4 * t - j);
                            sh->found[1] = front;
                        }
                        front += h[j];
                    }
                }
            }
            barrier();
            prefix |= (uint32_t)sh->found[0] << shift;
            before = sh->found[1];
        }
        if (BITS == 16 && !(prefix >> 31)) prefix |= 0xFFFFu;         // (a negative bfloat16's key ends in ones)
        return prefix;
    }
    static constexpr int kKeyBits = E == 8 ? 16 : 32;
    __device__ __forceinline__ void add_to_list(float x, int i)
    {
        const uint32_t at = atomicAdd(&sh->count, 1u);
        if (at < CAP) sh->list[at] = (uint64_t)key_of(x + 0.0f) << 32 | (uint32_t)i;
    }
    template <typename F>
    __device__ __forceinline__ void each_listed(F &&f)
    {
        for (uint32_t i = t; i < sh->count; i += NT) f((uint32_t)(sh->list[i] >> 32), (uint32_t)sh->list[i]);
    }
    // the bin of a score: how far it lies below the largest, in sixteenths of a power of two
    __device__ static int bin_of_powers(float z)
    {
        const float d = z * -16.0f;
        return d < (float)(kBins - 1) ? (int)d : kBins - 1;
    }
    __device__ int bin_of(float x) const { return bin_of_powers(weigh.powers(x)); }
    __device__ __forceinline__ void clear_bins()
    {
        barrier();
        for (int i = t; i < kCopies * kBins; i += NT) sh->bins[i / kBins][i % kBins] = 0;
        if (t == 0) sh->count = 0;
        barrier();
    }
    // the first bin at which the sum reaches goal and the sum in front of it, if all bins reach it; total: of all bins
    __device__ __forceinline__ int find_bin(uint64_t goal, uint64_t &before)
    {
        constexpr int kEach = kBins / 64;
        barrier();
        if (t < 64) {
            uint64_t mine = 0;
#pragma unroll
            for (int j = 0; j < kEach; ++j) mine += sh->bins[0][t * kEach + j];
            uint64_t in = mine;
            for (int d = 1; d < 64; d *= 2) {
                const uint64_t o = __shfl_up(in, d);
                if (t >= d) in += o;
            }
            uint64_t front = in - mine;
            if (front < goal && goal <= in) {
                for (int j = 0; j < kEach; ++j) {
                    const uint64_t h = sh->bins[0][t * kEach + j];
                    if (front < goal && goal <= front + h) {
                        sh->found[0] = (uint64_t)(t * kEach + j);
                        sh->found[1] = front;
                    }
                    front += h;
                }
            }
        }
        barrier();
        before = sh->found[1];
        return (int)sh->found[0];
    }
    // sums of the bins' copies, into the first; returns the sum of all
    __device__ __forceinline__ uint64_t merge_bins()
    {
        barrier();
        uint64_t mine = 0;
        for (int i = t; i < kBins; i += NT) {
            uint64_t s = sh->bins[0][i];
#pragma unroll
            for (int k = 1; k < kCopies; ++k) s += sh->bins[k][i];
            sh->bins[0][i] = s;
            mine += s;
        }
        return group_sum(mine);
    }
};

template <typename T, int NT, int CAP>
__global__ __launch_bounds__(NT) void draw_row_kernel(DrawArgs a)
{
    using R = Row<T, NT, CAP>;
    constexpr int E = R::E;
    __shared__ typename R::Shared sh;
    R row;
    const int64_t at_row = blockIdx.x;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    row.sh = &sh;
    row.z = static_cast<const T *>(a.z) + at_row * a.ld;
    row.c = (int)a.c;
    row.t = t;
    row.vectors = (int)((a.c + (int64_t)NT * E - 1) / ((int64_t)NT * E));
    const float temperature = a.rule.row_temperature ? a.rule.row_temperature[at_row] : a.rule.temperature;
    const int64_t top_k = a.rule.row_top_k ? a.rule.row_top_k[at_row] : a.rule.top_k;
    const float top_p = a.rule.row_top_p ? a.rule.row_top_p[at_row] : a.rule.top_p;
    const float u = a.u[at_row];

    // the largest score, and each thread's own
    float own = -__builtin_inff();
    row.each([&](float x, int) { own = fmaxf(own, x); });
    {
        const float m = wave_max(own);
        if (lane == 0) sh.tops[wave] = m;
    }
    __syncthreads();
    float top = sh.tops[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) top = fmaxf(top, sh.tops[w]);
    __syncthreads();
    top += 0.0f;
    const bool greedy = !(temperature > 0.0f);
    float slope = kLog2eDraw / (greedy ? 1.0f : temperature);
    auto answer = [&](int64_t which, float p) {
        a.classes[at_row] = which;
        if (a.probs) a.probs[at_row] = p;
    };
    if (top == -__builtin_inff()) {
        if (t == 0) answer(-1, 0.0f);
        return;
    }
    if (greedy) {                                  // the lowest index of the largest score
        if (t == 0) sh.count = 0xFFFFFFFFu;
        __syncthreads();
        if (own == top) {
            uint32_t first = 0xFFFFFFFFu;
            row.each([&](float x, int i) { first = x == top && (uint32_t)i < first ? (uint32_t)i : first; });
            atomicMin(&sh.count, first);
        }
        __syncthreads();
        if (t == 0) answer((int64_t)sh.count, 1.0f);
        return;
    }
    row.weigh.top = top;
    row.weigh.slope = slope;
    row.weigh.low = fminf(a.rule.row_min_p ? a.rule.row_min_p[at_row] : a.rule.min_p, 1.0f);     // (the largest always stays)
    const Weigh weigh = row.weigh;

    float floor = -__builtin_inff();               // what is kept: scores over it, and the first `ties` equal to it by index
    uint64_t ties = 0, total = 0;
    bool listed = false;                           // every kept class is in the list
    auto walk_list = [&](auto &&value) { return [&, value](auto &&f) { row.each_listed([&](uint32_t key, uint32_t) { f(key, value(key)); }); }; };
    auto walk_row = [&](auto &&value) { return [&, value](auto &&f) { row.each([&](float x, int) { if (x == x) f(key_of(x + 0.0f), value(x)); }); }; };
    const bool cut_k = top_k > 0 && top_k < row.c;
    if (cut_k && top_k <= NT) {
        // a score that top_k of the threads' largest reach
        row.clear_bins();
        if (own > -__builtin_inff()) atomicAdd(&sh.bins[0][row.bin_of(own)], 1ull);
        uint64_t front;
        const uint64_t with = row.group_sum(own > -__builtin_inff() ? 1 : 0);
        float reach = own;
        if (with >= (uint64_t)top_k) {
            const int bin = row.find_bin((uint64_t)top_k, front);
            reach = own > -__builtin_inff() && row.bin_of(own) <= bin ? own : __builtin_inff();
        }
        reach = -wave_max(-reach);
        __syncthreads();
        if (lane == 0) sh.tops[wave] = reach;
        __syncthreads();
        reach = sh.tops[0];
#pragma unroll
        for (int w = 1; w < NT / 64; ++w) reach = fminf(reach, sh.tops[w]);
        if (own >= reach) {
            row.each_vector([&](int v, const Bytes16 &q) {
                float most = Elem<T>::get(q.w, 0);
#pragma unroll
                for (int j = 1; j < E; ++j) most = fmaxf(most, Elem<T>::get(q.w, j));
                if (most >= reach && most > -__builtin_inff()) {
#pragma unroll
                    for (int j = 0; j < E; ++j) {
                        const float x = Elem<T>::get(q.w, j);
                        if (x >= reach && x > -__builtin_inff()) row.add_to_list(x, (v * NT + t) * E + j);
                    }
                }
            });
        }
        __syncthreads();
        listed = sh.count <= CAP;
    }
    if (cut_k) {
        uint64_t before = 0;
        const auto one = [](auto) -> uint64_t { return 1; };
        const uint64_t k = (uint64_t)top_k;
        if (listed) {
            if (sh.count > k) {
                floor = of_key(row.template select<R::kKeyBits>(walk_list(one), k, before));
                ties = k - before;
            }
        } else {
            uint64_t some = 0;                     // classes that have a score at all
            row.each([&](float x, int) { some += x > -__builtin_inff(); });
            some = row.group_sum(some);
            if (some > k) {
                row.clear_bins();
                row.each([&](float x, int) { if (x > -__builtin_inff()) atomicAdd(&sh.bins[lane % kCopies][row.bin_of(x)], 1ull); });
                row.merge_bins();
                const int bin = row.find_bin(k, before);
                row.each([&](float x, int i) { if (x > -__builtin_inff() && row.bin_of(x) == bin) row.add_to_list(x, i); });
                __syncthreads();
                uint64_t in = 0;
                if (sh.count <= CAP) {
                    floor = of_key(row.template select<R::kKeyBits>(walk_list(one), k - before, in));
                } else {
                    before = 0;
                    floor = of_key(row.template select<R::kKeyBits>(walk_row(one), k, in));
                }
                ties = k - before - in;
            }
        }
    }
    const uint64_t q_floor = floor > -__builtin_inff() ? weigh(floor) : 0;
    if (listed) {
        uint64_t mine = 0;
        row.each_listed([&](uint32_t key, uint32_t) { mine += of_key(key) > floor ? weigh(of_key(key)) : 0; });
        total = row.group_sum(mine) + ties * q_floor;
    }
    if (top_p < 1.0f) {
        const float over = floor;
        auto need_of = [&](uint64_t all) {
            const double wanted = ceil((double)top_p * (double)all);
            const uint64_t need = wanted > 1.0 ? (uint64_t)wanted : 1;
            return need < all ? need : all;
        };
        uint64_t before = 0, need = 0;
        float end = floor;
        bool inside = true;                        // the run ends over the floor that top_k has set
        if (listed) {
            need = need_of(total);
            inside = need <= total - ties * q_floor;
            before = total - ties * q_floor;
            if (inside)
                end = of_key(row.template select<R::kKeyBits>(walk_list([&](uint32_t key) -> uint64_t { return of_key(key) > over ? weigh(of_key(key)) : 0; }), need, before));
        } else {
            row.clear_bins();
            row.each([&](float x, int) {
                const float z = weigh.powers(x);
                const uint32_t q = weigh.of_powers(z);
                if (x > over && q) atomicAdd(&sh.bins[lane % kCopies][row.bin_of_powers(z)], (unsigned long long)q);
            });
            const uint64_t sum = row.merge_bins();
            need = need_of(sum + ties * q_floor);
            inside = need <= sum;
            before = sum;
            if (inside) {
                const int bin = row.find_bin(need, before);
                row.each([&](float x, int i) { if (x > over && row.bin_of(x) == bin) row.add_to_list(x, i); });
                __syncthreads();
                uint64_t in = 0;
                if (sh.count <= CAP) {
                    end = of_key(row.template select<R::kKeyBits>(walk_list([&](uint32_t key) -> uint64_t { return weigh(of_key(key)); }), need - before, in));
                } else {
                    before = 0;
                    end = of_key(row.template select<R::kKeyBits>(walk_row([&](float x) -> uint64_t { return x > over ? weigh(x) : 0; }), need, in));
                }
                before += in;
            }
        }
        const uint64_t q = weigh(end);         // (the run ends at a class with weight)
        ties = (need - before + q - 1) / q;
        floor = end;
        total = before + ties * q;
    }
    const uint64_t q_end = floor > -__builtin_inff() ? weigh(floor) : 0;
    auto target_of = [&](uint64_t all) {
        const uint64_t at = u > 0.0f ? (uint64_t)((double)u * (double)all) : 0;
        return at < all ? at : all - 1;
    };
    if (listed) {
        // by index: the ties that stay, then the class
        const uint64_t target = target_of(total);
        uint32_t last = 0xFFFFFFFFu;               // the highest index among the ties that stay
        const uint32_t floor_key = key_of(floor + 0.0f);
        uint64_t before;
        uint64_t equal = 0;
        row.each_listed([&](uint32_t key, uint32_t) { equal += key == floor_key; });
        equal = row.group_sum(equal);
        if (ties > 0 && equal > ties)
            last = key_index(row.template select<24>([&](auto &&f) { row.each_listed([&](uint32_t key, uint32_t i) { f(index_key(i), key == floor_key ? 1ull : 0ull); }); }, ties, before));
        const uint32_t which = key_index(row.template select<24>(
            [&](auto &&f) {
                row.each_listed([&](uint32_t key, uint32_t i) {
                    const float x = of_key(key);
                    f(index_key(i), x > floor || (key == floor_key && ties > 0 && i <= last) ? (uint64_t)weigh(x) : 0ull);
                });
            },
            target + 1, before));
        row.each_listed([&](uint32_t key, uint32_t i) {
            if (i == which) answer((int64_t)i, (float)((double)weigh(of_key(key)) / (double)total));
        });
        return;
    }
    // the kept weight of each segment, and its ties
    const bool tied = ties > 0;
    __syncthreads();
    row.each_vector([&](int v, const Bytes16 &q) {
        uint64_t mine = 0;
        uint32_t equal = 0;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const float x = Elem<T>::get(q.w, j);
            const uint32_t w = weigh(x);
            mine += x > floor ? w : 0u;
            equal += tied && x == floor;
        }
        for (int d = 1; d < 64; d *= 2) mine += __shfl_xor(mine, d);
        if (tied) {
            for (int d = 1; d < 64; d *= 2) equal += __shfl_xor(equal, d);
        }
        if (lane == 0) {
            sh.segment[v * (NT / 64) + wave] = mine;
            sh.ties[v * (NT / 64) + wave] = equal;
        }
    });
    __syncthreads();
    // the first wave walks them: where the sum passes the target, with the ties that stay
    const int segments = row.vectors * (NT / 64);
    if (wave == 0) {
        if (!(top_p < 1.0f)) {
            uint64_t mine = 0;
            for (int i = lane; i < segments; i += 64) mine += sh.segment[i];
            for (int d = 1; d < 64; d *= 2) mine += __shfl_xor(mine, d);
            total = mine + ties * q_end;
        }
        const uint64_t target = target_of(total);
        uint64_t seen = 0, used = 0;               // in front of these 64 segments
        for (int base = 0; base < segments; base += 64) {
            const int i = base + lane;
            uint64_t w = i < segments ? sh.segment[i] : 0, n = i < segments && tied ? sh.ties[i] : 0;
            uint64_t n_in = n;
            for (int d = 1; d < 64; d *= 2) {
                const uint64_t o = __shfl_up(n_in, d);
                if (lane >= d) n_in += o;
            }
            const uint64_t n_front = used + n_in - n;
            const uint64_t stay = n_front < ties ? (ties - n_front < n ? ties - n_front : n) : 0;
            w += stay * q_end;
            uint64_t w_in = w;
            for (int d = 1; d < 64; d *= 2) {
                const uint64_t o = __shfl_up(w_in, d);
                if (lane >= d) w_in += o;
            }
            const uint64_t front = seen + w_in - w;
            if (front <= target && target < front + w) {
                sh.found[0] = target - front;
                sh.found[1] = n_front;
                sh.count = (uint32_t)i;
                sh.sums[0] = total;
            }
            seen = __shfl(seen + w_in, 63);
            used = __shfl(used + n_in, 63);
            if (seen > target) break;
        }
    }
    __syncthreads();
    const int segment = (int)sh.count;
    if (segment % (NT / 64) != wave) return;
    total = sh.sums[0];
    const uint64_t inside = sh.found[0], front_ties = sh.found[1];
    const Bytes16 q = row.fetch(segment / (NT / 64));
    uint32_t w[E], equal = 0;
    uint64_t mine = 0;
#pragma unroll
    for (int j = 0; j < E; ++j) equal += tied && Elem<T>::get(q.w, j) == floor;
    uint32_t n_in = equal;
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t o = __shfl_up(n_in, d);
        if (lane >= d) n_in += o;
    }
    uint64_t rank = front_ties + n_in - equal;
#pragma unroll
    for (int j = 0; j < E; ++j) {
        const float x = Elem<T>::get(q.w, j);
        const bool tie = tied && x == floor;
        w[j] = x > floor || (tie && rank < ties) ? weigh(x) : 0u;
        rank += tie;
        mine += w[j];
    }
    uint64_t in = mine;
    for (int d = 1; d < 64; d *= 2) {
        const uint64_t o = __shfl_up(in, d);
        if (lane >= d) in += o;
    }
    uint64_t front = in - mine;
    if (front <= inside && inside < in) {
#pragma unroll
        for (int j = 0; j < E; ++j) {
            if (front <= inside && inside < front + w[j])
                answer(((int64_t)(segment / (NT / 64)) * NT + t) * E + j, (float)((double)w[j] / (double)total));
            front += w[j];
        }
    }
}

template <typename T>
static hipError_t launch_draw(const DrawArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)a.n);
    // short rows: four waves, several workgroups to a compute unit
    if (a.c <= 4096) hipLaunchKernelGGL((draw_row_kernel<T, 256, 2048>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((draw_row_kernel<T, 1024, 8192>), grid, dim3(1024), 0, s, a);
    return hipGetLastError();
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
    if (n < 0 || n > 0x7FFFFFFFLL || classes < 1 || (dtype != WPSGD_F32 && dtype != WPSGD_BF16) || !rule) return WPSGD_INVALID_ARG;
    if (!rule->row_temperature && !(rule->temperature >= 0.0f)) return WPSGD_INVALID_ARG;
    if ((!rule->row_top_p && std::isnan(rule->top_p)) || (!rule->row_min_p && !(rule->min_p <= 1.0f))) return WPSGD_INVALID_ARG;
    if (classes > kMostClasses) return WPSGD_UNSUPPORTED;
    if (n == 0) return WPSGD_OK;
    const size_t elem = dtype == WPSGD_F32 ? 4 : 2;
    if (!Z || !u || !drawn || ld < classes || (uintptr_t)Z % elem != 0) return WPSGD_INVALID_ARG;
    const size_t need = wpsgd_draw_classes_workspace(n, classes, dtype);
    if (need && (!workspace || (uintptr_t)workspace % 256 != 0)) return WPSGD_INVALID_ARG;
    if (workspace_bytes < need) return WPSGD_WORKSPACE_TOO_SMALL;
    const DrawArgs a{Z, n, classes, ld, u, *rule, drawn, probs};
    hipStream_t s = static_cast<hipStream_t>(stream);
    const hipError_t e = dtype == WPSGD_F32 ? launch_draw<float>(a, s) : launch_draw<uint16_t>(a, s);
    return e == hipSuccess ? WPSGD_OK : hip_fail(e);
}

}  // extern "C"
