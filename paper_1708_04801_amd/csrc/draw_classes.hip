// A class drawn for each row from its scores, with temperature, top-k, min-p and top-p, by a given random number.
//
// Classes stand in order of score, the lower index first among equals; -inf and NaN cannot be drawn.  What may be drawn is a run from the front of that
// order: the first top_k, of those the ones whose weight is at least min_p of the largest, and of those the shortest run that holds top_p of their weight.
// Weights are whole numbers, q = floor(2^((x - max) log2e / T) 2^31 + 1/2), the power of two in fp32 (off by up to 5e-6 of itself), and their sums 64-bit integers: no sum
// depends on the order it is taken in, so neither does a draw.  Few kept classes go to a list in LDS, where everything else is done; else the run's end is guessed from a sample, looked
// for in a list of what lies near it, and digit by digit among all scores only where that fails; the draw walks the kept classes by index.
#include <cmath>
#include <type_traits>

#include "class_ops.h"

namespace wpsgd {

struct DrawArgs {
    const void *z;
    int64_t n, c, ld;
    const float *u;
    wpsgd_draw_rule rule;
    int64_t *classes;
    float *probs;
    int64_t first;             // row at which the launch begins
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
    float top, slope;
    // powers of two that a weight is under the largest, negative or 0; top and slope are finite.  -inf and NaN have no weight.
    __device__ float powers(float x) const { return (x - top) * slope; }
    __device__ static uint32_t of_powers(float z) { return (uint32_t)fmaf(__builtin_amdgcn_exp2f(z), kOne, 0.5f); }
    __device__ uint32_t operator()(float x) const { return of_powers(powers(x)); }
};

// Sums over a wave and over the lanes up to each one, in whole numbers, on the DPP network.
template <int CTRL, int ROW_MASK, typename U>
__device__ inline U dpp_whole(U v)
{
    if constexpr (sizeof(U) == 4) return (U)dpp_move_bits<CTRL, ROW_MASK>((int)v);
    else return (U)(uint32_t)dpp_move_bits<CTRL, ROW_MASK>((int)(uint32_t)(v >> 32)) << 32 | (uint32_t)dpp_move_bits<CTRL, ROW_MASK>((int)(uint32_t)v);
}
template <typename U>
__device__ inline U up_to_lane_of_row(U v)         // with this lane's own; rows of sixteen lanes
{
    v += dpp_whole<0x111, 0xF>(v);                 // row_shr 1, 2, 4, 8
    v += dpp_whole<0x112, 0xF>(v);
    v += dpp_whole<0x114, 0xF>(v);
    v += dpp_whole<0x118, 0xF>(v);
    return v;
}
template <typename U>
__device__ inline U up_to_lane(U v)
{
    v = up_to_lane_of_row(v);
    v += dpp_whole<0x142, 0xA>(v);                 // lane 15 of a row to the next row: rows 1 and 3
    v += dpp_whole<0x143, 0xC>(v);                 // lane 31 to rows 2 and 3
    return v;
}
__device__ inline uint32_t of_lane(uint32_t v, int j) { return (uint32_t)__builtin_amdgcn_readlane((int)v, j); }
__device__ inline uint64_t of_lane(uint64_t v, int j) { return (uint64_t)of_lane((uint32_t)(v >> 32), j) << 32 | of_lane((uint32_t)v, j); }
template <typename U>
__device__ inline U wave_total(U v) { return of_lane(up_to_lane(v), kWave - 1); }
__device__ inline uint32_t wave_or(uint32_t v)
{
    v |= dpp_whole<0xB1, 0xF>(v);                  // lanes that differ in bits 0, 1, 2, 3: all of a row
    v |= dpp_whole<0x4E, 0xF>(v);
    v |= dpp_whole<0x141, 0xF>(v);
    v |= dpp_whole<0x140, 0xF>(v);
    return of_lane(v, 0) | of_lane(v, 16) | of_lane(v, 32) | of_lane(v, 48);
}
__device__ inline float row_max(float v)           // of sixteen lanes
{
    v = fmaxf(v, dpp_move<0xB1, 0xF>(v));
    v = fmaxf(v, dpp_move<0x4E, 0xF>(v));
    v = fmaxf(v, dpp_move<0x141, 0xF>(v));
    return fmaxf(v, dpp_move<0x140, 0xF>(v));
}

// ---- a row in a workgroup ----
// A wave owns a run of classes, in vectors of sixteen bytes to a lane; kRun vectors of a wave are a "segment".  The row is read again for each step, from the caches:
// kept in registers, its every element would stand in the code of every step.
//
//   1. the largest score, which is what reads the row from memory;
//   2. few classes kept (top_k <= NT): the top_k-th largest of the threads' own largest scores is a score that at least top_k classes reach, and so is the least of them, all but surely, where
//      not so many threads have any; the classes that do go to a list in LDS (a few times top_k), and everything else is done there;
//   3. top_p: weights of a sample (each thread's largest, two vectors of each for the others) in bins of powers of two say between which bins the run ends, give
//      or take kMargin top_p (1 - top_p) of the weight (a part's share of a whole is that much surer the nearer it is to none or all).  One pass over the row then adds up what lies above them by segments, lists what lies between, and has the weight of all: the
//      run's end is looked for in the list, and its classes are added to their segments.  Where it is not in the list, or the list has no room, what has been added up
//      corrects the sample for another try; after four the end is looked for among all classes digit by digit, and a pass adds up the segments;
//   4. the draw: the segment in which the target lies, then the class.
//
// (us a call, 256 rows of 131072 bfloat16: all kept 36, top 50 33, top_p 0.9 61; 512 threads with registers to spare 34, 36 and 58, but one row of 32000 with
// top 50 and top_p 0.95 took a fifth longer, and half as large a sample misses the run's end more often.)
// 256 rows of 131072 bfloat16 scores, a row to a compute unit: 10 us for the first step, which is bound by memory, 15 for a pass that forms weights
// (17 instructions an element, four of them the power of two), 22 for one that also lists; the sample 9, the run's end in a list of thousands 10.
constexpr int kBins = 1024, kCopies = 2;
constexpr int kMostClasses = 1 << 18;

constexpr double kMargin = 0.16;

template <typename T, int NT, int CAP>
struct Row {
    static constexpr int E = Elem<T>::kPer16, kWaves = NT / 64;
    static constexpr int kRun = 4;
    static constexpr int kShort = NT / 2 < 256 ? NT / 2 : 256;     // classes of a list in which each is compared with each
    static constexpr int kSegments = kMostClasses / (64 * E * kRun) + kWaves;
    static constexpr int kAtATime = 16 / E;        // vectors
    struct Shared {
        union {
            uint64_t hist[256];
            unsigned long long bins[kCopies][kBins];
        };
        uint64_t list[CAP];                        // key << 32 | class
        unsigned long long front[kShort];          // of the classes of a short list
        uint32_t weight[kShort], place[kShort];
        unsigned long long segment[kSegments];
        float tops[2 * kWaves];
        uint32_t ties[kSegments];
        uint64_t found[3];
        uint64_t sums[3][16];                      // of the waves, as many as there are
        uint32_t bits[16];
        uint32_t count;
    };
    Shared *sh;
    const T *z;
    int c, t, vectors;                             // vectors: of a lane
    float scale;                                   // bins to a power of two
    Weigh weigh;

    __device__ __forceinline__ int class_of(int v) const { return (((t >> 6) * vectors + v) * 64 + (t & 63)) * E; }
    // which segment a class is in
    __device__ __forceinline__ int segment_of(int i) const
    {
        const int vector = i / (64 * E), wave = vector / vectors;
        return wave * runs() + (vector - wave * vectors) / kRun;
    }
    __device__ __forceinline__ int runs() const { return (vectors + kRun - 1) / kRun; }
    __device__ __forceinline__ Bytes16 fetch(int v) const
    {
        const int at = class_of(v);
        if (v < vectors && at + E <= c) return load16(z + at);
        Bytes16 q;
#pragma unroll
        for (int j = 0; j < 4; ++j) q.w[j] = E == 8 ? 0xFF80FF80u : 0xFF800000u;       // -inf
        if (v < vectors && at < c) {
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
    template <int N = kAtATime, typename F>
    __device__ __forceinline__ void each_vector(F &&f)
    {
        for (int v = 0; v < vectors; v += N) {
            Bytes16 q[N];
#pragma unroll
            for (int j = 0; j < N; ++j) q[j] = fetch(v + j);          // (-inf behind the last class)
#pragma unroll
            for (int j = 0; j < N; ++j) f(v + j, q[j]);
        }
    }
    // f(score, class) for this thread's classes; a NaN never passes a comparison and has no weight
    template <typename F>
    __device__ __forceinline__ void each(F &&f)
    {
        each_vector([&](int v, const Bytes16 &q) {
#pragma unroll
            for (int j = 0; j < E; ++j) f(Elem<T>::get(q.w, j), class_of(v) + j);
        });
    }
    __device__ void barrier() const
    {
        __syncthreads();
    }
    // What the waves have left, a lane of each row of sixteen to a wave: a read for all of them, where a read each is sixteen to every wave.
    __device__ __forceinline__ uint64_t waves_total(int which) const
    {
        const int w = t & 15;
        return of_lane(up_to_lane_of_row(w < kWaves ? sh->sums[which][w] : (uint64_t)0), 15);
    }
    __device__ __forceinline__ uint64_t group_sum(uint64_t v)
    {
        v = wave_total(v);
        barrier();
        if ((t & 63) == 0) sh->sums[0][t >> 6] = v;
        barrier();
        return waves_total(0);
    }
    // three sums and the bits of a fourth value at once
    __device__ __forceinline__ void group_sums(uint64_t &a, uint64_t &b, uint64_t &c, uint32_t &bits)
    {
        a = wave_total(a);
        b = wave_total(b);
        c = wave_total(c);
        bits = wave_or(bits);
        barrier();
        if ((t & 63) == 0) {
            sh->sums[0][t >> 6] = a;
            sh->sums[1][t >> 6] = b;
            sh->sums[2][t >> 6] = c;
            sh->bits[t >> 6] = bits;
        }
        barrier();
        a = waves_total(0);
        b = waves_total(1);
        c = waves_total(2);
        bits = wave_or((t & 15) < kWaves ? sh->bits[t & 15] : 0);
    }
    // Where in descending order of a 32-bit key the sum of the values reaches goal: the key, and the sum in front of it.  walk(f) calls f(key, value) for
    // the classes of this thread that take part, whose keys lie between lo and hi; digits that these share are not looked at.  BITS: how many of the key's upper bits may differ.
    template <int BITS, typename W>
    __device__ __forceinline__ uint32_t select(W &&walk, uint64_t goal, uint64_t &before, uint32_t lo = 0, uint32_t hi = 0xFFFFFFFFu)
    {
        const int differ = lo == hi ? 0 : 32 - __clz(lo ^ hi);           // lower bits that may differ
        uint32_t prefix = differ >= 32 ? 0 : hi >> differ << differ;
        before = 0;
#pragma unroll 1
        for (int top = differ; top > 32 - BITS; top -= 8) {              // bits under `top` are not known yet
            const int shift = top > 8 ? top - 8 : 0;
            barrier();
            for (int i = t; i < 256; i += NT) sh->hist[i] = 0;
            barrier();
            walk([&](uint32_t key, uint64_t v) {
                if ((top == 32 || (key ^ prefix) >> top == 0) && v) atomicAdd(reinterpret_cast<unsigned long long *>(&sh->hist[(key >> shift) & (255u >> (8 - (top - shift)))]), v);
            });
            barrier();
            if (t < 64) {                          // four digits to a lane, the largest first
                uint64_t h[4], mine = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    h[j] = sh->hist[255 - 4 * t - j];
                    mine += h[j];
                }
                const uint64_t in = up_to_lane(mine);
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
        if (BITS == 16) prefix = prefix >> 31 ? prefix & 0xFFFF0000u : prefix | 0xFFFFu;         // (a negative bfloat16's key ends in ones)
        return prefix;
    }
    static constexpr int kKeyBits = E == 8 ? 16 : 32;
    template <typename F>
    __device__ __forceinline__ void each_listed(F &&f)
    {
        for (uint32_t i = t; i < sh->count; i += NT) f((uint32_t)(sh->list[i] >> 32), (uint32_t)sh->list[i]);
    }
    // two keys that differ where any in the list do (one at least)
    __device__ __forceinline__ void list_range(uint32_t &lo, uint32_t &hi)
    {
        barrier();
        lo = (uint32_t)(sh->list[0] >> 32);
        uint32_t differ = 0;
        each_listed([&](uint32_t key, uint32_t) { differ |= key ^ lo; });
        differ = wave_or(differ);
        if ((t & 63) == 0) sh->bits[t >> 6] = differ;
        barrier();
        hi = lo ^ wave_or((t & 15) < kWaves ? sh->bits[t & 15] : 0);
    }
    // the bin of a score: how far it lies below the largest, in powers of two times scale
    __device__ __forceinline__ int bin_of_powers(float z) const
    {
        const float d = z * -scale;
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
    // Adds up the copies of the bins and all bins in front of this thread's; returns the sum of all.
    static constexpr int kMine = kBins / NT;       // bins of a thread
    __device__ __forceinline__ uint64_t scan_bins(uint64_t (&front)[kMine + 1])
    {
        barrier();
        uint64_t h[kMine], mine = 0;
#pragma unroll
        for (int j = 0; j < kMine; ++j) {
            h[j] = 0;
#pragma unroll
            for (int k = 0; k < kCopies; ++k) h[j] += sh->bins[k][t * kMine + j];
            mine += h[j];
        }
        const uint64_t in = up_to_lane(mine);
        if ((t & 63) == 63) sh->sums[0][t >> 6] = in;
        barrier();
        const int w = t & 15, wave = __builtin_amdgcn_readfirstlane(t >> 6);
        const uint64_t waves = up_to_lane_of_row(w < kWaves ? sh->sums[0][w] : (uint64_t)0), all = of_lane(waves, 15);
        front[0] = in - mine + (wave > 0 ? of_lane(waves, wave - 1) : 0);
#pragma unroll
        for (int j = 0; j < kMine; ++j) front[j + 1] = front[j] + h[j];
        return all;
    }
    // the first bin at which the sum reaches goal (more than 0, at most the sum of all), and the sum in front of it; the same of a second goal, if that is more than 0
    __device__ __forceinline__ int find_bin(const uint64_t (&front)[kMine + 1], uint64_t goal, uint64_t &before, uint64_t goal2 = 0, int *bin2 = nullptr)
    {
        barrier();
#pragma unroll
        for (int j = 0; j < kMine; ++j) {
            if (front[j] < goal && goal <= front[j + 1]) {
                sh->found[0] = (uint64_t)(t * kMine + j);
                sh->found[1] = front[j];
            }
            if (front[j] < goal2 && goal2 <= front[j + 1]) sh->found[2] = (uint64_t)(t * kMine + j);
        }
        barrier();
        before = sh->found[1];
        if (bin2) *bin2 = (int)sh->found[2];
        return (int)sh->found[0];
    }
    // Appends a lane's classes to the list: bit j of which for class i(j).  One addition to its length for the wave.  KEYS: with the scores' keys, four looked up at
    // a time, which pays where thousands are listed a segment at a time: afterwards they would be one more way through the row (8 us for 4500 of 131072).
    template <bool KEYS = false, typename I>
    __device__ __forceinline__ void append(uint32_t which, I &&i)
    {
        const uint32_t n = (uint32_t)__popc(which), n_in = up_to_lane(n), all = of_lane(n_in, kWave - 1);
        if (all == 0) return;
        uint32_t at = 0;
        if ((t & 63) == 0) at = atomicAdd(&sh->count, all);
        at = of_lane(at, 0) + n_in - n;
        while (which) {
            constexpr int kMany = KEYS ? 4 : 1;
            int c[kMany];
            uint64_t o[kMany];
            const int n = __popc(which);
#pragma unroll
            for (int j = 0; j < kMany; ++j) {
                c[j] = which ? i(__ffs(which) - 1) : c[0];
                which &= which - 1;
            }
#pragma unroll
            for (int j = 0; j < kMany; ++j) o[j] = KEYS ? entry_of((uint32_t)c[j]) : (uint64_t)(uint32_t)c[j];
#pragma unroll
            for (int j = 0; j < kMany; ++j)
                if (j < n && at + j < CAP) sh->list[at + j] = o[j];
            at += kMany;
        }
    }
    __device__ __forceinline__ uint64_t entry_of(uint32_t i) const { return (uint64_t)key_of(Elem<T>::load(z + i) + 0.0f) << 32 | i; }
    // The keys beside the classes of a list that has room, behind a barrier after the last append: four of a thread's on their way at once, and a thread's own are those
    // that it walks in each_listed.  (For what is listed a vector at a time: looked up as they are
    // appended, a wave waits for each.  16 rows of 131072 fp32, top 1000: 39 us instead of 49.)
    __device__ __forceinline__ void fill_keys()
    {
        constexpr int kMany = 4;
        const uint32_t n = sh->count;
        for (uint32_t i0 = t; i0 < n; i0 += NT * kMany) {
            uint64_t o[kMany];
#pragma unroll
            for (int j = 0; j < kMany; ++j) o[j] = entry_of((uint32_t)sh->list[i0 + j * NT < n ? i0 + j * NT : i0]);
#pragma unroll
            for (int j = 0; j < kMany; ++j)
                if (i0 + j * NT < n) sh->list[i0 + j * NT] = o[j];
        }
    }
};

// The end of the run among all classes over `last`, by weight or by number.  Out of line: where it is needed thousands of scores are all but equal.
template <typename T, int NT, int CAP>
__device__ __attribute__((noinline)) uint32_t find_in_row(Row<T, NT, CAP> row, bool weights, float last, uint64_t goal, uint64_t &before)
{
    uint64_t b;
    const uint32_t key = row.template select<Row<T, NT, CAP>::kKeyBits>(
        [&](auto &&f) { row.each([&](float x, int) { if (x > last || (!weights && x == last)) f(key_of(x + 0.0f), weights ? (uint64_t)row.weigh(x) : 1ull); }); }, goal, b);
    before = b;
    return key;
}

template <typename T, int NT, int CAP>
__global__ __launch_bounds__(NT) void draw_row_kernel(DrawArgs a)
{
    using R = Row<T, NT, CAP>;
    constexpr int E = R::E;
    constexpr float kInf = __builtin_inff();
    __shared__ typename R::Shared sh;
    R row;
    const int64_t at_row = a.first + blockIdx.x;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    row.sh = &sh;
    row.z = static_cast<const T *>(a.z) + at_row * a.ld;
    row.c = (int)a.c;
    row.t = t;
    row.vectors = (int)((a.c + NT * E - 1) / (NT * E));
    const float temperature = a.rule.row_temperature ? a.rule.row_temperature[at_row] : a.rule.temperature;
    const int64_t top_k = a.rule.row_top_k ? a.rule.row_top_k[at_row] : a.rule.top_k;
    const float top_p = a.rule.row_top_p ? a.rule.row_top_p[at_row] : a.rule.top_p;
    const float low = fminf(a.rule.row_min_p ? a.rule.row_min_p[at_row] : a.rule.min_p, 1.0f);   // (the largest always stays)
    const float u = a.u[at_row];

    // the largest score, each thread's own, and the least of those
    float own = -kInf;
    row.template each_vector<8>([&](int, const Bytes16 &q) {             // (from memory: many on their way)
#pragma unroll
        for (int j = 0; j < E; ++j) own = fmaxf(own, Elem<T>::get(q.w, j));
    });
    {
        const float m = wave_max(own), n = wave_max(own > -kInf ? -own : -kInf);
        if (lane == 0) {
            sh.tops[wave] = m;
            sh.tops[R::kWaves + wave] = n;
        }
    }
    __syncthreads();
    float top = row_max(sh.tops[t % R::kWaves]);
    const float least = -row_max(sh.tops[R::kWaves + t % R::kWaves]);
    __syncthreads();
    top += 0.0f;
    auto answer = [&](int64_t which, float p) {
        a.classes[at_row] = which;
        if (a.probs) a.probs[at_row] = p;
    };
    if (top == -kInf) {
        if (t == 0) answer(-1, 0.0f);
        return;
    }
    const bool greedy = !(temperature > 0.0f);
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
    const float slope = kLog2eDraw / temperature;
    row.weigh.top = top;
    row.weigh.slope = slope;
    // A score can be worth a weight down to 32 powers of two below the largest; the threads' own span a part of the scores that matter: bins as fine as that allows.
    const float span = (top - least) * slope;
    row.scale = span < 8.0f ? fminf((float)kBins / (8.0f * span), 1e30f) : 16.0f;
    const Weigh weigh = row.weigh;
    auto target_of = [&](uint64_t all) {
        const uint64_t at = u > 0.0f ? (uint64_t)((double)u * (double)all) : 0;
        return at < all ? at : all - 1;
    };
    auto need_of = [&](uint64_t all) {
        const double wanted = ceil((double)top_p * (double)all);
        const uint64_t need = wanted > 1.0 ? (uint64_t)wanted : 1;
        return need < all ? need : all;
    };
    const auto one = [](auto) -> uint64_t { return 1; };
    auto walk_list = [&](auto &&value) { return [&, value](auto &&f) { row.each_listed([&](uint32_t key, uint32_t) { f(key, value(key)); }); }; };

    float floor = -kInf;                           // what is kept: scores over it, and the first `ties` equal to it by index
    uint64_t ties = 0, total = 0;
    bool listed = false;                           // every kept class is in the list
    const bool cut_k = top_k > 0 && top_k < row.c;
    // +inf, or a temperature so small that the slope is: the largest scores share everything
    const bool sharp = !(top < kInf) || !(slope < kInf);
    if (sharp) {
        uint64_t equal = 0;
        row.each([&](float x, int) { equal += x == top; });
        ties = row.group_sum(equal);
        if (cut_k && (uint64_t)top_k < ties) ties = (uint64_t)top_k;
        if (top_p < 1.0f) ties = (need_of(ties << 31) + (1ull << 31) - 1) >> 31;
        floor = top;
        total = ties << 31;
    } else {
        if (cut_k && top_k <= NT) {
            // a score that top_k of the threads' largest reach
            row.clear_bins();
            const bool some = own > -kInf;
            if (some) atomicAdd(&sh.bins[0][row.bin_of(own)], 1ull);
            uint64_t fronts[R::kMine + 1];
            const uint64_t with = row.scan_bins(fronts);
            // (fewer threads with a score than that: all classes, or where they have no room, those that reach the least of them)
            float reach = row.c <= CAP ? -kInf : least;
            const bool sure = with >= (uint64_t)top_k || row.c <= CAP;
            if (with >= (uint64_t)top_k) {
                uint64_t front;
                const int bin = row.find_bin(fronts, (uint64_t)top_k, front);
                reach = some && row.bin_of(own) <= bin ? own : kInf;
            }
            reach = wave_max(-reach);
            __syncthreads();
            if (lane == 0) sh.tops[wave] = reach;
            __syncthreads();
            reach = -row_max(sh.tops[t % R::kWaves]);
            row.each_vector([&](int v, const Bytes16 &q) {
                float most = Elem<T>::get(q.w, 0);
#pragma unroll
                for (int j = 1; j < E; ++j) most = fmaxf(most, Elem<T>::get(q.w, j));
                if (__ballot(most >= reach && most > -kInf)) {
                    uint32_t which = 0;
#pragma unroll
                    for (int j = 0; j < E; ++j) {
                        const float x = Elem<T>::get(q.w, j);
                        which |= x >= reach && x > -kInf ? 1u << j : 0u;
                    }
                    row.append(which, [&](int j) { return row.class_of(v) + j; });
                }
            });
            __syncthreads();
            listed = sh.count <= CAP && (sure || sh.count >= (uint64_t)top_k);
            if (listed && sh.count > R::kShort) row.fill_keys();
        }
        if (listed && sh.count <= R::kShort) {
            // A short list: each class is compared with each, as many threads to a class as there are, whole waves, and four at a time, so that they come from LDS
            // together (one row of 1000 with top 50: 6 us less than one at a time).  At least two threads to a class:
            // 256 threads take 23 us a call for a list of 200 bfloat16 scores, and 10 by digits.  Its place in order and the weight in front of it say whether it is
            // kept, the kept weight in front of it by index whether it is drawn.
            const int n = (int)sh.count, shift = n <= 64 ? 6 : n <= 128 ? 7 : 8, parts = NT >> shift, mine = t & ((1 << shift) - 1), part = t >> shift;
            const uint64_t me = mine < n ? row.entry_of((uint32_t)sh.list[mine]) : 0;
            __syncthreads();
            if (t < n) sh.list[t] = me;
            else if (t < n + 4) sh.list[t] = 0xFFFFFFFFull;              // in front of nothing, in either order
            const uint64_t order = me ^ 0xFFFFFFFFull;                   // larger: in front
            if (t < R::kShort) {
                const uint32_t q = t < n ? weigh(of_key((uint32_t)(me >> 32))) : 0u;
                sh.weight[t] = q;
                sh.place[t] = 0;
                sh.front[t] = 0;
            }
            __syncthreads();
            const uint32_t q = sh.weight[mine];
            auto sum_in_front = [&](auto &&in_front) {                   // of the weights of those; how many
                uint64_t w = 0;
                uint32_t places = 0;
                for (int j0 = part * 4; j0 < n; j0 += parts * 4) {
                    uint64_t o[4];
                    uint32_t of[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        o[j] = sh.list[j0 + j];
                        of[j] = sh.weight[j0 + j];
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const bool yes = in_front(o[j]);
                        w += yes ? of[j] : 0u;
                        places += yes;
                    }
                }
                if (mine < n) {
                    atomicAdd(&sh.front[mine], (unsigned long long)w);
                    atomicAdd(&sh.place[mine], places);
                }
                __syncthreads();
            };
            sum_in_front([&](uint64_t o) { return (o ^ 0xFFFFFFFFull) > order; });
            // the first top_k, those whose weight reaches min_p (a run from the front, too)
            bool kept = mine < n && sh.place[mine] < (uint32_t)top_k && __builtin_amdgcn_exp2f(weigh.powers(of_key((uint32_t)(me >> 32)))) >= low;
            const uint64_t all = row.group_sum(kept && part == 0 ? (uint64_t)q : 0);
            const uint64_t front = sh.front[mine];
            if (top_p < 1.0f) kept = kept && front < need_of(all);
            total = top_p < 1.0f ? row.group_sum(kept && part == 0 ? (uint64_t)q : 0) : all;
            __syncthreads();
            if (t < R::kShort) {
                sh.weight[t] = kept ? q : 0u;
                sh.front[t] = 0;
            }
            __syncthreads();
            sum_in_front([&](uint64_t o) { return (uint32_t)o < (uint32_t)me; });
            const uint64_t target = target_of(total), before = sh.front[mine];
            if (part == 0 && kept && before <= target && target < before + q) answer((int64_t)(uint32_t)me, (float)((double)q / (double)total));
            return;
        }
        if (cut_k) {
            uint64_t before = 0;
            const uint64_t k = (uint64_t)top_k;
            uint32_t lo, hi;
            if (listed) {
                if (sh.count > k) {
                    row.list_range(lo, hi);
                    floor = of_key(row.template select<R::kKeyBits>(walk_list(one), k, before, lo, hi));
                    ties = k - before;
                }
            } else {
                uint64_t some = 0;                 // classes that have a score at all
                row.each([&](float x, int) { some += x > -kInf; });
                some = row.group_sum(some);
                if (some > k) {
                    row.clear_bins();
                    row.each([&](float x, int) { if (x > -kInf) atomicAdd(&sh.bins[lane % kCopies][row.bin_of(x)], 1ull); });
                    uint64_t fronts[R::kMine + 1];
                    row.scan_bins(fronts);
                    const int bin = row.find_bin(fronts, k, before);
                    row.each_vector([&](int v, const Bytes16 &q) {
                        uint32_t which = 0;
#pragma unroll
                        for (int j = 0; j < E; ++j) {
                            const float x = Elem<T>::get(q.w, j);
                            which |= x > -kInf && row.bin_of(x) == bin ? 1u << j : 0u;
                        }
                        row.template append<true>(which, [&](int j) { return row.class_of(v) + j; });
                    });
                    __syncthreads();
                    uint64_t in = 0;
                    if (sh.count <= CAP) {
                        row.list_range(lo, hi);
                        floor = of_key(row.template select<R::kKeyBits>(walk_list(one), k - before, in, lo, hi));
                    } else {
                        before = 0;
                        floor = of_key(find_in_row(row, false, -kInf, k, in));
                    }
                    ties = k - before - in;
                }
            }
        }
        if (low > 0.0f) {
            // min_p: the least score whose weight reaches it, sixty-four tries at a time
            uint32_t from = key_of(-kInf), to = key_of(top);             // reaches: not `from`, `to`
            while (to - from > 1) {
                const uint32_t step = (to - from + 63) / 64, at = from + step * (uint32_t)(lane + 1);
                const bool reaches = at >= to || at < from || __builtin_amdgcn_exp2f(weigh.powers(of_key(at))) >= low;
                const int first = __ffsll((unsigned long long)__ballot(reaches)) - 1;
                const uint32_t hit = from + step * (uint32_t)(first + 1);
                from = from + step * (uint32_t)first;
                to = hit < to && hit > from ? hit : to;
            }
            // (<=: where top_k ends at the very score that falls short, its ties go, too)
            if (key_of(floor) <= from) {
                floor = of_key(from);
                ties = 0;
            }
        }
        const uint64_t q_floor = ties > 0 ? weigh(floor) : 0;
        if (listed) {
            uint64_t mine = 0;
            row.each_listed([&](uint32_t key, uint32_t) { mine += of_key(key) > floor ? weigh(of_key(key)) : 0; });
            const uint64_t over = row.group_sum(mine);
            total = over + ties * q_floor;
            if (top_p < 1.0f) {
                const uint64_t need = need_of(total);
                uint64_t before = over;
                const float last = floor;
                if (need <= over) {
                    uint32_t lo, hi;
                    row.list_range(lo, hi);
                    floor = of_key(row.template select<R::kKeyBits>(walk_list([&](uint32_t key) -> uint64_t { return of_key(key) > last ? weigh(of_key(key)) : 0; }), need, before, lo, hi));
                }
                const uint64_t q = weigh(floor);   // (the run ends at a class with weight)
                ties = (need - before + q - 1) / q;
                total = before + ties * q;
            }
            // by index: the ties that stay, then the class
            const uint64_t target = target_of(total);
            uint32_t last = 0xFFFFFFFFu;           // the highest index among the ties that stay
            const uint32_t floor_key = key_of(floor + 0.0f);
            uint64_t before, equal = 0;
            row.each_listed([&](uint32_t key, uint32_t) { equal += key == floor_key; });
            equal = row.group_sum(equal);
            if (ties > 0 && equal > ties)
                last = key_index(row.template select<24>([&](auto &&f) { row.each_listed([&](uint32_t key, uint32_t i) { f(index_key(i), key == floor_key ? 1ull : 0ull); }); }, ties, before, index_key((uint32_t)row.c - 1), index_key(0)));
            const uint32_t which = key_index(row.template select<24>(
                [&](auto &&f) {
                    row.each_listed([&](uint32_t key, uint32_t i) {
                        const float x = of_key(key);
                        f(index_key(i), x > floor || (key == floor_key && ties > 0 && i <= last) ? (uint64_t)weigh(x) : 0ull);
                    });
                },
                target + 1, before, index_key((uint32_t)row.c - 1), index_key(0)));
            row.each_listed([&](uint32_t key, uint32_t i) {
                if (i == which) answer((int64_t)i, (float)((double)weigh(of_key(key)) / (double)total));
            });
            return;
        }
    }

    // The kept weight of each segment, and its ties.  BETWEEN: scores over the floor count where they are less than `sure` powers of two below the largest; down
    // to `maybe` they go to the list, and each thread's weight of what counts is added to `counted`, that of all others returned.
    auto add_segments = [&](auto between, float sure, float maybe, uint64_t &counted) -> uint64_t {
        constexpr bool BETWEEN = decltype(between)::value;
        const bool tied = !BETWEEN && ties > 0;
        uint64_t rest = 0;
        for (int g = 0; g < row.runs(); ++g) {
            uint64_t mine = 0;
            uint32_t equal = 0, listed_ones = 0;   // (bit v E + j)
#pragma unroll 1
            for (int h = 0; h < R::kRun; h += R::kAtATime) {
                Bytes16 q[R::kAtATime];
#pragma unroll
                for (int v = 0; v < R::kAtATime; ++v) q[v] = row.fetch(g * R::kRun + h + v);
#pragma unroll
                for (int v = 0; v < R::kAtATime; ++v)
#pragma unroll
                    for (int j = 0; j < E; ++j) {
                        const float x = Elem<T>::get(q[v].w, j);
                        const float z = weigh.powers(x);
                        const uint32_t w = x > floor ? weigh.of_powers(z) : 0u;
                        if constexpr (BETWEEN) {
                            const bool in = z > sure;
                            mine += in ? w : 0u;
                            rest += w;
                            listed_ones |= z > maybe && !in && x > floor ? 1u << (v * E + j) << (h * E) : 0u;
                        } else {
                            mine += w;
                            equal += tied && x == floor;
                        }
                    }
            }
            if constexpr (BETWEEN) {
                rest -= mine;
                counted += mine;
                row.template append<true>(listed_ones, [&](int j) { return row.class_of(g * R::kRun + j / E) + j % E; });
            }
            mine = wave_total(mine);
            if (tied) equal = wave_total(equal);
            if (lane == 0) {
                sh.segment[wave * row.runs() + g] = mine;
                sh.ties[wave * row.runs() + g] = equal;
            }
        }
        return rest;
    };
    const int segments = R::kWaves * row.runs();
    bool added = false;
    if (top_p < 1.0f && !sharp) {
        row.clear_bins();
        // each thread's largest as it is, and two vectors of each for all of its others
        auto put = [&](float x, uint32_t times) {
            const float z = weigh.powers(x);
            const uint32_t w = x > floor ? weigh.of_powers(z) : 0u;
            if (w) atomicAdd(&sh.bins[lane % kCopies][row.bin_of_powers(z)], (unsigned long long)w * times);
        };
        put(own, 2);
        const int picks = row.vectors > 1 ? 2 : 1;
        for (int i = 0; i < picks; ++i) {
            const Bytes16 q = row.fetch((lane * 5 + wave + i * ((row.vectors + 1) / 2)) % row.vectors);
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (Elem<T>::get(q.w, j) < own) put(Elem<T>::get(q.w, j), (uint32_t)(2 * row.vectors / picks));
        }
        uint64_t fronts[R::kMine + 1];
        const uint64_t sample = row.scan_bins(fronts), q_floor = ties > 0 ? weigh(floor) : 0;
        double goal = (double)top_p * (double)sample, margin = kMargin * fmax((double)top_p * (1.0 - (double)top_p), 0.006) * (double)sample;     // in the sample's weight
        uint64_t need = 0, over = 0, rest = 0, before = 0;
        float end = floor;
        // min_p or top_k may say that few classes are kept at all (half the sample's weight is about the row's): a sample says little of their order then, and all of them
        // have room in the list
        double most = low > 0.0f ? 0.5 * (double)sample / ((double)low * (double)kOne) : (double)kMostClasses;
        if (cut_k && (double)top_k < most) most = (double)top_k;
        bool whole = most < 0.7 * CAP;
        bool found = false;
        uint32_t first = 0, differ = 0;            // a key of the list, and the bits in which any differ from it
        for (int tries = 0; tries < 4 && !found && sample > 0; ++tries) {
            uint64_t sampled = 0;                  // the sample's weight over `sure`
            float sure = 1.0f, maybe = -kInf;      // (even the largest may be the last)
            const uint64_t from = !whole && goal - margin > 1.0 ? (uint64_t)(goal - margin < (double)sample ? goal - margin : (double)sample) : 0;
            const uint64_t to = !whole && goal + margin < (double)sample ? (uint64_t)(goal + margin > 1.0 ? goal + margin : 1.0) : 0;
            int last = kBins - 1;
            const int bin = row.find_bin(fronts, from, sampled, to, &last);
            if (from > 0) sure = (float)bin / -row.scale;
            else sampled = 0;
            if (to > 0 && last < kBins - 1) maybe = (float)(last + 1) / -row.scale;
            if (t == 0) sh.count = 0;
            __syncthreads();
            over = 0;
            rest = add_segments(std::true_type{}, sure, maybe, over);
            __syncthreads();
            const bool room = sh.count <= CAP;
            uint64_t list = 0;
            differ = 0;
            first = 0;
            if (room && sh.count > 0) {
                first = (uint32_t)(sh.list[0] >> 32);
                row.each_listed([&](uint32_t key, uint32_t) {
                    list += weigh(of_key(key));
                    differ |= key ^ first;
                });
            }
            row.group_sums(rest, over, list, differ);
            need = need_of(over + rest + ties * q_floor);
            if (need > over + rest) break;         // among the ties that top_k has left
            found = room && need > over && need <= over + list;
            // what has been added up says what the sample's weights are worth on this side of `sure`
            if (need > over) goal = (double)sampled + (double)(need - over) * ((double)(sample - sampled) / (double)rest);
            else goal = (double)sampled * ((double)need / (double)over);
            if (!whole) margin *= room ? 0.5 : 0.2;
            whole = false;
        }
        if (found) {
            end = of_key(row.template select<R::kKeyBits>(walk_list([&](uint32_t key) -> uint64_t { return weigh(of_key(key)); }), need - over, before, first, first ^ differ));
            before += over;
            const uint32_t end_key = key_of(end + 0.0f);
            row.each_listed([&](uint32_t key, uint32_t i) {
                if (key > end_key) atomicAdd(&sh.segment[row.segment_of((int)i)], (unsigned long long)weigh(of_key(key)));
                else if (key == end_key) atomicAdd(&sh.ties[row.segment_of((int)i)], 1u);
            });
            added = true;
        } else if (sample == 0 || need <= over + rest) {
            const float last = floor;
            if (sample == 0) {                     // nothing of the sample lies over the floor
                uint64_t mine = 0;
                row.each([&](float x, int) { mine += x > last ? weigh(x) : 0u; });
                rest = row.group_sum(mine);
                need = need_of(rest + ties * q_floor);
            }
            before = rest;
            if (need <= over + rest) end = of_key(find_in_row(row, true, last, need, before));
        } else {
            before = over + rest;
        }
        const uint64_t q = weigh(end);             // (the run ends at a class with weight)
        ties = (need - before + q - 1) / q;
        floor = end;
        total = before + ties * q;
    }
    if (!added) {
        __syncthreads();
        uint64_t unused = 0;
        add_segments(std::false_type{}, 0.0f, 0.0f, unused);
    }
    __syncthreads();
    const bool tied = ties > 0;
    const uint64_t q_end = sharp ? 1ull << 31 : tied ? weigh(floor) : 0;
    // the first wave walks the segments: where the sum passes the target, with the ties that stay
    if (wave == 0) {
        if (!(top_p < 1.0f)) {
            uint64_t mine = 0;
            for (int i = lane; i < segments; i += 64) mine += sh.segment[i];
            total = wave_total(mine) + ties * q_end;
        }
        const uint64_t target = target_of(total);
        uint64_t seen = 0, used = 0;               // in front of these 64 segments
        for (int base = 0; base < segments; base += 64) {
            const int i = base + lane;
            uint64_t w = i < segments ? sh.segment[i] : 0, n = i < segments && tied ? sh.ties[i] : 0;
            const uint64_t n_in = up_to_lane(n);
            const uint64_t n_front = used + n_in - n;
            const uint64_t stay = n_front < ties ? (ties - n_front < n ? ties - n_front : n) : 0;
            w += stay * q_end;
            const uint64_t w_in = up_to_lane(w);
            const uint64_t front = seen + w_in - w;
            if (front <= target && target < front + w) {
                sh.found[0] = target - front;
                sh.found[1] = n_front;
                sh.count = (uint32_t)i;
                sh.sums[0][0] = total;
            }
            seen += of_lane(w_in, 63);
            used += of_lane(n_in, 63);
            if (seen > target) break;
        }
    }
    __syncthreads();
    const int segment = (int)sh.count;
    if (segment / row.runs() != wave) return;
    total = sh.sums[0][0];
    uint64_t inside = sh.found[0], rank0 = sh.found[1];
    for (int v = (segment % row.runs()) * R::kRun; v < (segment % row.runs() + 1) * R::kRun; ++v) {
        const Bytes16 q = row.fetch(v);
        uint32_t w[E], equal = 0;
        uint64_t mine = 0;
#pragma unroll
        for (int j = 0; j < E; ++j) equal += tied && Elem<T>::get(q.w, j) == floor;
        const uint32_t n_in = up_to_lane(equal);
        uint64_t rank = rank0 + n_in - equal;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const float x = Elem<T>::get(q.w, j);
            const bool tie = tied && x == floor;
            w[j] = tie ? (rank < ties ? (uint32_t)q_end : 0u) : x > floor ? weigh(x) : 0u;
            rank += tie;
            mine += w[j];
        }
        const uint64_t in = up_to_lane(mine);
        uint64_t front = in - mine;
        if (front <= inside && inside < in) {
#pragma unroll
            for (int j = 0; j < E; ++j) {
                if (front <= inside && inside < front + w[j]) answer((int64_t)row.class_of(v) + j, (float)((double)w[j] / (double)total));
                front += w[j];
            }
        }
        const uint64_t all = of_lane(in, 63);
        if (inside < all) return;
        inside -= all;
        rank0 += of_lane(n_in, 63);
    }
}

template <typename T>
static hipError_t launch_draw(DrawArgs a, hipStream_t s)
{
    // Short rows: four waves, whose barriers are shorter, and several workgroups to a compute unit.  us a call, four waves | sixteen, bfloat16 and fp32:
    //   8192 classes, 200 rows   top_p 0.9 16.1 | 18.8, 16.7 | 17.8    top 50 10.4 | 8.9, 12.1 | 8.8     1000 rows  top_p 0.9 31 | 68, 33 | 67    top 50 19 | 31, 21 | 32
    //   16384 classes, 200 rows  top_p 0.9 19.8 | 21.1, 29.0 | 19.9    top_p 0.5, whose list has no room in the smaller LDS, 54 | 21, 83 | 19
    const bool few = a.c <= 8192;
    return in_launches(a.n, few ? 256 : 1024, [&](int64_t first, unsigned count) {
        a.first = first;
        if (few) hipLaunchKernelGGL((draw_row_kernel<T, 256, 2048>), dim3(count), dim3(256), 0, s, a);
        else hipLaunchKernelGGL((draw_row_kernel<T, 1024, 14336>), dim3(count), dim3(1024), 0, s, a);
    });
}

}  // namespace wpsgd

using namespace wpsgd;

extern "C" {

int wpsgd_draw_classes(const void *Z, int64_t n, int64_t classes, int64_t ld, wpsgd_dtype dtype, const float *u, const wpsgd_draw_rule *rule, int64_t *drawn,
                       float *probs, void *stream)
{
    if (n < 0 || n > 0x7FFFFFFFLL || classes < 1 || (dtype != WPSGD_F32 && dtype != WPSGD_BF16) || !rule) return WPSGD_INVALID_ARG;
    if (!rule->row_temperature && !(rule->temperature >= 0.0f)) return WPSGD_INVALID_ARG;
    if ((!rule->row_top_p && std::isnan(rule->top_p)) || (!rule->row_min_p && !(rule->min_p <= 1.0f))) return WPSGD_INVALID_ARG;
    if (classes > kMostClasses) return WPSGD_UNSUPPORTED;
    if (n == 0) return WPSGD_OK;
    const size_t elem = dtype == WPSGD_F32 ? 4 : 2;
    if (!Z || !u || !drawn || ld < classes || (uintptr_t)Z % elem != 0) return WPSGD_INVALID_ARG;
    const DrawArgs a{Z, n, classes, ld, u, *rule, drawn, probs, 0};
    hipStream_t s = static_cast<hipStream_t>(stream);
    const hipError_t e = dtype == WPSGD_F32 ? launch_draw<float>(a, s) : launch_draw<uint16_t>(a, s);
    return e == hipSuccess ? WPSGD_OK : hip_fail(e);
}

}  // extern "C"
