// Class vectors of four bits and products of a few rows with them.
//
// A code has a sign and three bits for one of 0, 1/2, 1, 3/2, 2, 3, 4, 6; a group of 32, 64 or 128 elements of a row shares a bfloat16 scale s: the least value, 2^-126 or
// more, with 6 s >= the group's largest size (1 for a group of zeros, NaN where an element is not finite).  A code is the nearest value of x / s, half to the even code; the
// borders between codes times s are fp32 numbers, so that no quotient is rounded.
//
// A block of 128 elements of a row fills 64 bytes, element 32 j + 8 k + i of it (j, k < 4, i < 8) in byte 16 k + 4 j + i / 2, the even one in the lower half: the sixteen
// bytes that lane group k of a matrix instruction's operand loads hold its eight elements of each of the four 32s, and each 32 lies in one group.
#include "class_ops.h"

namespace wpsgd {

constexpr int kNibbleBlock = 128;

// The codes of eight elements, the first in the lowest bits.  The quotient x / s is formed to the last place (a product with about 1 / s and one correction).  bfloat16 elements: one that lies on
// no border between codes is 2^-11 of itself away from it, and one that does comes out as the border, a number of few bits; the conversion instruction, which rounds half to even,
// gives the code.  fp32 elements: the quotient is cut towards zero and its last bit set where it is not exact; such a number lies on the same side of every border as x / s, on it only if
// x / s does.  Five and thirteen instructions an element, where comparing with the seven borders takes some twenty.  Residuals under s 2^-33 have to be numbers: groups with scales under
// 2^-110 are compared.
template <bool HALF>
__device__ inline uint32_t codes_of(const float (&x)[8], float s)
{
    uint32_t w = 0;
    if (s >= 0x1p-110f) {
        const float r = __builtin_amdgcn_rcpf(s);
        float q[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float y = x[j] * r;
            y = fmaf(fmaf(-y, s, x[j]), r, y);
            if constexpr (!HALF) {
                const uint32_t left = __float_as_uint(fmaf(-y, s, x[j]));
                const uint32_t odd = min(left & 0x7FFFFFFFu, 1u), over = (left ^ __float_as_uint(x[j])) >> 31 & odd;      // not exact; rounded away from zero
                y = __uint_as_float((__float_as_uint(y) - over) | odd);
            }
            q[j] = copysignf(y, x[j]);                                                  // (a residual of 0 takes a zero's sign)
        }
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, q[0], q[1], 1.0f, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, q[2], q[3], 1.0f, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, q[4], q[5], 1.0f, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, q[6], q[7], 1.0f, 3);
    } else {
        const float border[7] = {0.25f * s, 0.75f * s, 1.25f * s, 1.75f * s, 2.5f * s, 3.5f * s, 5.0f * s};
#pragma unroll
        for (int j = 7; j >= 0; --j) {
            const float size = fabsf(x[j]);
            uint32_t c = __float_as_uint(x[j]) >> 28 & 8u;
#pragma unroll
            for (int i = 0; i < 7; ++i) c += (i & 1) ? size >= border[i] : size > border[i];      // (a border itself goes to the even code)
            w = w << 4 | c;
        }
    }
    return w;
}

// The bits of the least bfloat16 s >= 2^-126 with 6 s >= top; 1 for 0.  What the upper half of the product with about 1/6 stands for is the answer or one place under it: where the product is
// a little too large for its upper half, top / 6 lies right under that, and that is the answer.
__device__ inline uint32_t scale_bits(float top)
{
    if (top == 0.0f) return 0x3F800000u;
    const float s = __uint_as_float(__float_as_uint(fmaxf(top * 0.16666667f, 1.17549435e-38f)) & 0xFFFF0000u);
    return __float_as_uint(s) + (6.0f * s < top ? 0x10000u : 0u);
}

struct Quantize4Args {
    const void *x;
    const int64_t *rows;       // which rows, or nullptr: all in order
    int64_t m, d, ld, n;
    uint8_t *codes;
    uint16_t *scales;
    int64_t ld_codes, ld_scales;
    int64_t blocks;
    int64_t first;             // workgroup of the call at which the launch begins
};

// Sixteen lanes to a block of 128, eight elements to a lane; G groups to a block.  Bound by memory: 65536 x 4096 fp32 219 us, 5.5 TB/s; bfloat16, whose elements are twice as many, 147
// (groups of 32: 135, 5.1 TB/s; 188 with thirteen instructions an element and divisions for the scale).  Four blocks to sixteen lanes were slower (225 fp32, 5003 x 3001 17 instead of 14).
template <typename T, int G>
__global__ __launch_bounds__(256) void quantize4_kernel(Quantize4Args a)
{
    const int64_t first = (a.first + blockIdx.x) * 16;
    const int64_t row0 = first >> 32 ? first / a.blocks : (int64_t)((uint32_t)first / (uint32_t)a.blocks);
    const uint32_t at = (uint32_t)(first - row0 * a.blocks) + (threadIdx.x >> 4), blocks = (uint32_t)a.blocks;      // (blocks < 2^25)
    const uint32_t down = blocks >= 16 ? (at >= blocks ? 1u : 0u) : at / blocks;
    const int64_t row = row0 + down;
    if (row >= a.n) return;                                                            // (sixteen lanes at a time)
    const uint32_t b = at - down * blocks;
    const int64_t from = a.rows ? a.rows[row] : row;
    const int lane = threadIdx.x & 15;
    const int64_t col = (int64_t)b * kNibbleBlock + lane * 8;
    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (from >= 0 && from < a.m && col < a.d) load8(static_cast<const T *>(a.x) + from * a.ld + col, a.d - col, x);
    float top = 0.0f, sum = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        sum = fmaf(x[j], 0.0f, sum);                                                   // NaN where one is not finite
        top = fmaxf(top, fabsf(x[j]));
    }
    top = sum == 0.0f ? top : __builtin_inff();                                        // (no maximum drops that)
    top = fmaxf(top, dpp_move<0xB1, 0xF>(top));
    top = fmaxf(top, dpp_move<0x4E, 0xF>(top));
    if constexpr (G <= 2) top = fmaxf(top, dpp_move<0x141, 0xF>(top));
    if constexpr (G == 1) top = fmaxf(top, dpp_move<0x140, 0xF>(top));
    const bool whole = top < __builtin_inff();
    const uint32_t bits = whole ? scale_bits(top) : 0x7FC00000u;
    const uint32_t w = whole ? codes_of<sizeof(T) == 2>(x, __uint_as_float(bits)) : 0u;
    *reinterpret_cast<uint32_t *>(a.codes + row * a.ld_codes + (int64_t)b * 64 + (lane & 3) * 16 + (lane >> 2) * 4) = w;
    constexpr int kLanes = 16 / G;
    if (lane % kLanes == 0) a.scales[row * a.ld_scales + (int64_t)b * G + lane / kLanes] = col < a.d ? (uint16_t)(bits >> 16) : (uint16_t)0;
}

typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8v __attribute__((ext_vector_type(8)));
typedef float f32x4v __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));

// The eight values of a word's codes, times 2^-10: a group's sum, which meets its scale only when it is whole, is under 2^128 then whatever the rows (6 * 128 < 2^10), and results that fp32
// holds come out.  Results are multiplied by 2^10 where they are stored; both are exact, but for what that puts under 2^-126: less than 2^-116 of a group's sum or of a result.
constexpr float kCodeScale = 0x1p-10f, kResultScale = 0x1p10f;
__device__ inline bf16x8v widen_codes(uint32_t w)
{
    const bf16x2v a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, kCodeScale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, kCodeScale, 1),
                  c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, kCodeScale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, kCodeScale, 3);
    return bf16x8v{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

// Values as bfloat16 (PARTS 1: they are), or as sums of three bfloat16 values, eight significant bits each: what a value's upper half stands for, the same of the rest, and the rest of that.
// What is not finite stays in the first; a NaN becomes the quiet one, since the bits that tell another from an infinity may all lie in the lower half.
template <int PARTS>
__device__ inline void split8(const float (&x)[8], bf16x8v *part)
{
    const auto halves = [](const float (&v)[8]) {
        u32x4v w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = __builtin_amdgcn_perm(__float_as_uint(v[2 * j + 1]), __float_as_uint(v[2 * j]), 0x07060302);
        return __builtin_bit_cast(bf16x8v, w);
    };
    part[0] = halves(x);
    if constexpr (PARTS == 3) {
        float rest[8], last[8], most = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            rest[j] = x[j] - __uint_as_float(__float_as_uint(x[j]) & 0xFFFF0000u);
            last[j] = rest[j] - __uint_as_float(__float_as_uint(rest[j]) & 0xFFFF0000u);
            most += fabsf(rest[j]);                                                     // NaN where one is not finite
        }
        if (most != most) {
            float whole[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                whole[j] = x[j] == x[j] ? x[j] : __builtin_nanf("");
                last[j] = rest[j] == rest[j] ? last[j] : 0.0f;
                rest[j] = rest[j] == rest[j] ? rest[j] : 0.0f;
            }
            part[0] = halves(whole);
        }
        part[1] = halves(rest);
        part[2] = halves(last);
    }
}

// Eight elements of a row of d from column col (a multiple of eight) on, in two steps, so that many loads can be on their way without a branch between them: ask() reads what lies in
// the row there or before, give() is the elements if the row holds all eight, else zeros.  What a row ends with, where d is no multiple of eight, is put in by itself.
template <typename T> struct Eight {
    static constexpr int E = Elem<T>::kPer16;
    Bytes16 q[8 / E];
    // eight that are there for certain, and their parts
    __device__ void ask(const T *p)
    {
#pragma unroll
        for (int i = 0; i < 8 / E; ++i) q[i] = load16(p + i * E);
    }
    __device__ void parts(bf16x8v *part) const
    {
        if constexpr (E == 8) {
            part[0] = __builtin_bit_cast(bf16x8v, q[0]);
        } else {
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = Elem<T>::get(q[j / E].w, j % E);
            split8<3>(x, part);
        }
    }
    __device__ void ask(const T *row, int64_t col, int64_t d)
    {
        const T *p = row + (col + 8 <= d ? col : d >= 8 ? d - 8 : 0);
#pragma unroll
        for (int i = 0; i < 8 / E; ++i) q[i] = d >= 8 ? load16(p + i * E) : Bytes16{{0, 0, 0, 0}};
    }
    __device__ void give(int64_t col, int64_t d, bool there, float (&x)[8]) const
    {
        const bool whole = there && col + 8 <= d;
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = whole ? Elem<T>::get(q[j / E].w, j % E) : 0.0f;
    }
};

struct Matmul4Args {
    const void *x;
    const int64_t *rows;
    int64_t m, d, ld, n;
    const uint8_t *codes;
    const uint16_t *scales;
    int64_t ld_codes, ld_scales, classes;
    int blocks;
    bool half, wide;           // results are bfloat16; the rows are fp32
    void *out;
    int64_t ld_out;
    int64_t first, first_row;  // workgroup and row at which the launch begins
};

// Every other call.  The classes' codes go from memory straight into the matrix instructions, two blocks (a line of 128 bytes) of NT sixteens of classes at a time to a wave.  Row i of a
// tile of sixteen rows is row 4 (i mod 4) + i / 4 of the instruction, so that up to four rows need one result register of a lane, up to eight two (R).  A group's products are summed by
// themselves and times its scale added in fp32.  Of WAVES waves in a workgroup `along` share the sum, pairs of blocks in turn, and add up through LDS in their order; the others take the next
// classes.  HELD: the rows lie in LDS as fragments, up to 128 KiB of the sum at a time, fp32 ones as three parts; else each wave asks for its own part of them.
// 8 x 65536 x 4096 fp32 (LDS) 42 us, 3.2 TB/s of codes out of memory (38 where the caches still hold them); 1 x 4096 x 4096 (each wave) 7.1, a launch and three trips to memory one behind the other (row number, row, sum);
// 64 x 65536 x 4096 68, 500 TFLOP/s (74 with 64 KiB of rows at a time): fragments from LDS and codes widened for four tiles of rows at a time.
template <int MT, int R, int PARTS> constexpr int held_blocks4()
{
    int n = 64;
    while (n > 2 && n * MT * R * PARTS > 128) n /= 2;
    return n;
}

// pairs of blocks on their way while one is worked on
template <int MT, int R, int NT, int PARTS> constexpr int ahead4()
{
    const int pairs = held_blocks4<MT, R, PARTS>() / 2, most = NT == 1 ? 4 : 2;
    return pairs < most ? pairs : most;
}
// a barrier for what lies in LDS: loads from memory stay on their way
__device__ inline void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <typename T, int MT, int R, int NT, int G, int WAVES, bool HELD>
__global__ __launch_bounds__(64 * WAVES) void matmul4_kernel(Matmul4Args g, int along)
{
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1, kHeld = held_blocks4<MT, R, PARTS>(), kLanes = 16 * R, kThreads = 64 * WAVES;
    constexpr int kAhead = ahead4<MT, R, NT, PARTS>();
    constexpr int kSums = MT * NT * R;
    __shared__ union {
        bf16x8v held[HELD ? kHeld * MT * 4 * PARTS : 1][kLanes];
        float sums[WAVES][kSums][64];
    } lds;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), rho = lane & 15, k = lane >> 4;
    const int across = WAVES / along, mine = wave % along;
    const int64_t c0 = ((g.first + blockIdx.x) * across + wave / along) * (16 * NT), h0 = g.first_row + (int64_t)blockIdx.y * (16 * MT);
    const bool active = (rho & 3) < R;
    float acc[MT][NT][R];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int u = 0; u < NT; ++u)
#pragma unroll
            for (int r = 0; r < R; ++r) acc[t][u][r] = 0.0f;
    const uint8_t *codes[NT];
    const uint16_t *scales[NT];
#pragma unroll
    for (int u = 0; u < NT; ++u) {
        const int64_t cls = c0 + u * 16 + rho < g.classes ? c0 + u * 16 + rho : g.classes - 1;
        codes[u] = g.codes + cls * g.ld_codes + k * 16;
        scales[u] = g.scales + cls * g.ld_scales;
    }
    struct Pair {
        uint4 q[NT][2];
        uint32_t s[NT][G];                                                              // 2 G scales
    };
    auto fetch = [&](Pair &p, int pair) {
        const int last = g.blocks - 1, b = 2 * pair < last ? 2 * pair : last & ~1, next = b < last ? b + 1 : b;
#pragma unroll
        for (int u = 0; u < NT; ++u) {
            p.q[u][0] = *reinterpret_cast<const uint4 *>(codes[u] + (int64_t)b * 64);
            p.q[u][1] = *reinterpret_cast<const uint4 *>(codes[u] + (int64_t)next * 64);
            const uint16_t *s = scales[u] + (int64_t)b * G;
            if constexpr (G == 1) {
                p.s[u][0] = *reinterpret_cast<const uint32_t *>(s);
            } else if constexpr (G == 2) {
                const uint2 v = *reinterpret_cast<const uint2 *>(s);
                p.s[u][0] = v.x, p.s[u][1] = v.y;
            } else {
                const uint4 v = *reinterpret_cast<const uint4 *>(s);
                p.s[u][0] = v.x, p.s[u][1] = v.y, p.s[u][2] = v.z, p.s[u][3] = v.w;
            }
        }
    };
    // block `half` of a pair, with get(t, y, parts) the parts of tile t's fragment of the y-th 32 columns; before(t) comes before a tile of rows, there or not
    auto multiply = [&](const Pair &p, int half, auto before, auto get) {
        bf16x8v f[NT][4];
#pragma unroll
        for (int u = 0; u < NT; ++u) {
            const uint4 q = p.q[u][half];
            f[u][0] = widen_codes(q.x), f[u][1] = widen_codes(q.y), f[u][2] = widen_codes(q.z), f[u][3] = widen_codes(q.w);
        }
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            before(t);
            if (MT > 1 && h0 + t * 16 >= g.n) continue;                                 // (no such rows)
            f32x4v sum[NT];
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                if (y % (4 / G) == 0) {
#pragma unroll
                    for (int u = 0; u < NT; ++u) sum[u] = f32x4v{0.0f, 0.0f, 0.0f, 0.0f};
                }
                bf16x8v h[PARTS];
                get(t, y, h);
#pragma unroll
                for (int e = 0; e < PARTS; ++e)
#pragma unroll
                    for (int u = 0; u < NT; ++u) sum[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(h[e], f[u][y], sum[u], 0, 0, 0);
                if ((y + 1) % (4 / G) == 0) {
#pragma unroll
                    for (int u = 0; u < NT; ++u) {
                        const int at = half * G + y / (4 / G);
                        const float s = (at & 1) ? bf16_hi(p.s[u][at >> 1]) : bf16_lo(p.s[u][at >> 1]);
#pragma unroll
                        for (int r = 0; r < R; ++r) acc[t][u][r] = fmaf(sum[u][r], s, acc[t][u][r]);
                    }
                }
            }
        }
    };
    const int pairs = (g.blocks + 1) / 2;
    if constexpr (HELD) {
        // A thread's pieces of a filling: eight elements of one row each, the same row in every piece (or in every other one), and a wave's pieces of four rows that follow each other.
        // Loads come back in the order they are asked for: the rows' go out behind the first pair of the classes', the other pairs behind them.
        constexpr int kPieces = kHeld * MT * 4 * kLanes, kEach = (kPieces + kThreads - 1) / kThreads, kRowsOf = kThreads / 16 >= MT * 4 * R ? 1 : MT * 4 * R / (kThreads / 16);
        Pair p[kAhead];
        fetch(p[0], mine);
        const T *from[kRowsOf];
        bool there[kRowsOf];
#pragma unroll
        for (int y = 0; y < kRowsOf; ++y) {
            const int four = __builtin_amdgcn_readfirstlane((threadIdx.x + kThreads * y) >> 6) * 4, i = four % (4 * R), t = four / (4 * R) % MT;
            const int64_t h = h0 + t * 16 + i;
            int64_t row = -1;
#pragma unroll
            for (int o = 0; o < 4; ++o) {                                               // (by scalar loads, which wait for themselves)
                const int64_t one = h + o < g.n ? (g.rows ? g.rows[h + o] : h + o) : -1;
                row = (lane >> 4) == o ? one : row;
            }
            there[y] = row >= 0 && row < g.m;
            from[y] = static_cast<const T *>(g.x) + (there[y] ? row * g.ld : 0);
        }
        const int place = k * (4 * R) + (rho >> 2) * R + (rho & 3);
        const int per = kHeld / 2 / along, steps = (pairs + along - 1) / along;            // of a wave between two fillings, and in all: the same for every wave
        // a filling from block b0 on: between(), once the loads are on their way; whole: it ends within the rows
        auto fill = [&](int b0, auto between) {
            Eight<T> got[kEach];
            constexpr int kNext = kThreads / (16 * 4 * R * MT) * kNibbleBlock;           // columns from a piece to the thread's next one (of the same row)
            const int v0 = (threadIdx.x >> 4) / (4 * R) / MT, in_block = (threadIdx.x >> 2 & 3) * 32 + (threadIdx.x & 3) * 8;
            const int64_t col0 = (int64_t)(b0 + v0) * kNibbleBlock + in_block;
            const bool whole = kRowsOf == 1 && kPieces % kThreads == 0 && (int64_t)(b0 + kHeld) * kNibbleBlock <= g.d;
            auto col_of = [&](int y) { return kRowsOf == 1 ? col0 + y * kNext : (int64_t)(b0 + ((threadIdx.x + kThreads * y) >> 4) / (4 * R) / MT) * kNibbleBlock + in_block; };
            if (whole) {
#pragma unroll
                for (int y = 0; y < kEach; ++y)
#pragma unroll
                    for (int i = 0; i < 8 / Eight<T>::E; ++i) got[y].q[i] = load16(from[0] + col0 + y * kNext + i * Eight<T>::E);
            } else {
#pragma unroll
                for (int y = 0; y < kEach; ++y) got[y].ask(from[y % kRowsOf], col_of(y), g.d);
            }
            between();
#pragma unroll
            for (int y = 0; y < kEach; ++y) {
                const int piece = threadIdx.x + kThreads * y;
                const int pk = piece & 3, pj = piece >> 2 & 3, i = (piece >> 4) % (4 * R), v = (piece >> 4) / (4 * R), t = v % MT, in = v / MT;
                if (kPieces % kThreads != 0 && in >= kHeld) break;
                bf16x8v part[3];
                if (whole) {
#pragma unroll
                    for (int e = 0; e < PARTS; ++e) part[e] = bf16x8v{};
                    if (there[0]) got[y].parts(part);
                } else {
                    float x[8];
                    got[y].give(col_of(y), g.d, there[y % kRowsOf], x);
                    split8<PARTS>(x, part);
                }
                const int to = pk * (4 * R) + (i & 3) * R + (i >> 2);
#pragma unroll
                for (int e = 0; e < PARTS; ++e) lds.held[((in * MT + t) * 4 + pj) * PARTS + e][to] = part[e];
            }
            const int end = (int)(g.d >> 7) - b0;                                       // the block in which the rows end
            if ((g.d & 7) != 0 && end >= 0 && end < kHeld) {
                lds_barrier();
                if (threadIdx.x < MT * 4 * R) {
                    const int i = threadIdx.x % (4 * R), t = threadIdx.x / (4 * R), c = (int)(g.d & 127) >> 3, to = (c & 3) * (4 * R) + (i & 3) * R + (i >> 2);
                    const int64_t h = h0 + t * 16 + i, row = h < g.n ? (g.rows ? g.rows[h] : h) : -1;
                    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                    if (row >= 0 && row < g.m) load8(static_cast<const T *>(g.x) + row * g.ld + (g.d & ~7LL), g.d & 7, x);
                    bf16x8v part[3];
                    split8<PARTS>(x, part);
#pragma unroll
                    for (int e = 0; e < PARTS; ++e) lds.held[((end * MT + t) * 4 + (c >> 2)) * PARTS + e][to] = part[e];
                }
            }
            lds_barrier();
        };
        // (no branch around a load of the classes': the compiler counts what is on its way.  What is asked for behind the last pair is the last pair, out of the caches.)
        auto work = [&](int step0, int end) {
            for (int step1 = step0; step1 < end; step1 += kAhead) {
#pragma unroll
                for (int j = 0; j < kAhead; ++j) {
                    const int pair = (step1 + j) * along + mine;
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint32_t b = 2 * pair + half, at = b % kHeld;
                        if ((int)b < g.blocks)
                            multiply(p[j], half, [](int) {}, [&](int t, int y, bf16x8v *h) {
#pragma unroll
                                for (int e = 0; e < PARTS; ++e) {
                                    h[e] = bf16x8v{};
                                    if (R == 4 || active) h[e] = lds.held[((at * MT + t) * 4 + y) * PARTS + e][place];
                                }
                            });
                    }
                    fetch(p[j], pair + kAhead * along);
                }
            }
        };
        fill(0, [&] {
#pragma unroll
            for (int j = 1; j < kAhead; ++j) fetch(p[j], j * along + mine);
        });
        work(0, steps < per ? steps : per);
        for (int step0 = per; step0 < steps; step0 += per) {
            fill(step0 / per * kHeld, [] { lds_barrier(); });
            work(step0, steps - step0 < per ? steps : step0 + per);
        }
    } else {
        const T *from[MT];
        bool there[MT];
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            const int64_t h = h0 + t * 16 + 4 * (rho & 3) + (rho >> 2), row = active && h < g.n ? (g.rows ? g.rows[h] : h) : -1;
            there[t] = row >= 0 && row < g.m;
            from[t] = static_cast<const T *>(g.x) + (there[t] ? row * g.ld : 0);
        }
        auto ask = [&](Eight<T> (&got)[4], int t, int b) {                              // (what is not there is not asked for)
            if (!there[t] || b >= g.blocks) return;
            if ((int64_t)(b + 1) * kNibbleBlock <= g.d) {
                const T *p = from[t] + b * kNibbleBlock + k * 8;
#pragma unroll
                for (int y = 0; y < 4; ++y) got[y].ask(p + y * 32);
            } else {
#pragma unroll
                for (int y = 0; y < 4; ++y) got[y].ask(from[t], (int64_t)b * kNibbleBlock + y * 32 + k * 8, g.d);
            }
        };
        Pair p, after;
        fetch(p, mine);
        constexpr bool kEarly = PARTS * WAVES < 48;                                     // (sixteen waves' registers do not hold two fp32 tiles)
        Eight<T> got[kEarly ? 2 : 1][4];                                                // of a tile of rows and the next, of this block or the one behind it
        if (kEarly) ask(got[0], 0, 2 * mine);
        for (int pair = mine; pair < pairs; pair += along) {
            fetch(after, pair + along);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int b = 2 * pair + half;
                if (b < g.blocks) {
                    const auto col = [&](int y) { return (int64_t)b * kNibbleBlock + y * 32 + k * 8; };
                    const auto before = [&](int t) {
                        if constexpr (kEarly) {
                            if (t + 1 < MT) ask(got[(half * MT + t + 1) % 2], t + 1, b);
                            else ask(got[(half * MT + t + 1) % 2], 0, half == 0 ? b + 1 : 2 * (pair + along));
                            asm volatile("" ::: "memory");                              // (no tile earlier than that: they would not fit the registers)
                        } else {
                            ask(got[0], t, b);
                        }
                    };
                    multiply(p, half, before, [&](int t, int y, bf16x8v *h) {
                        const Eight<T> &mine_now = got[kEarly ? (half * MT + t) % 2 : 0][y];
                        if ((int64_t)(b + 1) * kNibbleBlock <= g.d) {
#pragma unroll
                            for (int e = 0; e < PARTS; ++e) h[e] = bf16x8v{};
                            if (there[t]) mine_now.parts(h);
                            return;
                        }
                        float x[8];
                        mine_now.give(col(y), g.d, there[t], x);
                        if ((g.d & 7) != 0 && there[t] && col(y) == (g.d & ~7LL)) load8(from[t] + col(y), g.d & 7, x);
                        split8<PARTS>(x, h);
                    });
                }
            }
            p = after;
        }
    }
    // the waves' sums, in their order, by all threads: value v of a lane at sums[wave][v][lane]
    if (HELD) __syncthreads();
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int u = 0; u < NT; ++u)
#pragma unroll
            for (int r = 0; r < R; ++r) lds.sums[wave][(t * NT + u) * R + r][lane] = acc[t][u][r];
    __syncthreads();
    for (int at = threadIdx.x; at < across * kSums * 64; at += kThreads) {
        const int l = at & 63, v = (at >> 6) % kSums, w = (at >> 6) / kSums;
        const int r = v % R, u = v / R % NT, t = v / R / NT;
        const int64_t c = ((g.first + blockIdx.x) * across + w) * (16 * NT) + u * 16 + (l & 15), h = h0 + t * 16 + 4 * r + (l >> 4);
        if (c >= g.classes || h >= g.n) continue;
        float sum = lds.sums[w * along][v][l];
        for (int o = 1; o < along; ++o) sum += lds.sums[w * along + o][v][l];
        sum *= kResultScale;
        if (g.half) Elem<uint16_t>::put(static_cast<uint16_t *>(g.out) + h * g.ld_out + c, sum);
        else Elem<float>::put(static_cast<float *>(g.out) + h * g.ld_out + c, sum);
    }
}

// Up to sixteen rows of up to 4096 columns against many classes.  The waves of a workgroup hold the rows in registers, `along` waves a pair of blocks each; kStreamWaves / along of
// them stand beside each other for other classes.  The classes' codes stream past, sixteen classes at a time, kBatch of those on their way, and every kBatch the waves' sums meet in
// LDS, in their order.  fp32 rows are three rows of bfloat16 parts each, which the last addition puts together.
// 16 x 65536 x 4096, groups of 32: 36 us, 4.3 TB/s; of 128: 33, 4.2; 1 x 65536 x 4096 28, 4.9 (several class matrices in turn, so that codes come out of memory; the same one again
// and again: 30, 28.5 and 25.6).  Reading the codes alone takes 22, at the 6.1 to 6.4 TB/s that reading alone reaches.  The rest: codes and rows come in cold for some 8 us
// before the first results (each kernel also reads its own instructions, one line behind the other: the way through the start is kept short), and the waves wait for each other at the
// end.  Batches of four tiles: 35 us for the first of these, but 1 x 65536 x 4096 29.4 and 4 x 16384 x 4096 12.7 instead of 11.5: twice the instructions.
constexpr int kStreamWaves = 16, kBatch = 2;

template <int R, int G>
__global__ __launch_bounds__(64 * kStreamWaves) void matmul4_stream_kernel(Matmul4Args g, int along)
{
    constexpr int kThreads = 64 * kStreamWaves;
    __shared__ float sums[2][kStreamWaves][kBatch][R][64];
    __shared__ uint4 scales[2][kThreads];              // of a batch's classes, a row's beside each other: eight to a thread
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), rho = lane & 15, k = lane >> 4;
    const int across = kStreamWaves / along, mine = wave % along;
    // a run of sixteens of classes for each workgroup, `across` of them at a time
    const int tiles = (int)((g.classes + 15) / 16), sets = (tiles + across - 1) / across;
    const int set0 = (int)((int64_t)blockIdx.x * sets / gridDim.x), count = (int)((int64_t)(blockIdx.x + 1) * sets / gridDim.x) - set0;
    const int tile0 = set0 * across + wave / along;
    const int each = G * along >= 4 ? G * along / 4 : 1, each_log = 31 - __builtin_clz(each);      // eights of scales in a row (a power of two)
    auto scales_of = [&](int it0) {
        const int eight = threadIdx.x & (each - 1), row = threadIdx.x >> each_log, it = it0 + (row >> 4) / across, w = (row >> 4) & (across - 1);
        const int64_t cls = ((int64_t)(set0 + (it < count ? it : count - 1)) * across + w) * 16 + (row & 15);
        const int64_t at = (cls < g.classes ? cls : g.classes - 1) * g.ld_scales + (eight * 8 < G * g.blocks ? eight * 8 : 0);
        return *reinterpret_cast<const uint4 *>(g.scales + at);
    };
    const int last = g.blocks - 1, b0 = 2 * mine < last ? 2 * mine : last & ~1, b1 = b0 < last ? b0 + 1 : b0;
    struct Codes {
        uint4 q[2];
    };
    auto fetch = [&](Codes &c, int it) {
        const int tile = tile0 + (it < count ? it : count - 1) * across;
        const int64_t cls = (int64_t)tile * 16 + rho < g.classes ? (int64_t)tile * 16 + rho : g.classes - 1;
        const uint8_t *codes = g.codes + cls * g.ld_codes + k * 16;
        c.q[0] = *reinterpret_cast<const uint4 *>(codes + (int64_t)b0 * 64);
        c.q[1] = *reinterpret_cast<const uint4 *>(codes + (int64_t)b1 * 64);
    };
    // Loads come back in the order they are asked for: the first batch's scales, the first codes, the rows, then the other codes.
    uint4 held = scales_of(0);
    Codes c[kBatch];
    fetch(c[0], 0);
    // the wave's columns
    bf16x8v x[8];
    {
        const int v = 4 * (rho & 3) + (rho >> 2), part = g.wide ? v % 3 : 0;
        const int64_t h = g.wide ? v / 3 : v, row = (rho & 3) < R && h < g.n ? (g.rows ? g.rows[h] : h) : -1;
#pragma unroll
        for (int y = 0; y < 8; ++y) x[y] = bf16x8v{};
        auto take = [&](auto *base) {
            using T = std::remove_const_t<std::remove_pointer_t<decltype(base)>>;
            constexpr int kParts = sizeof(T) == 4 ? 3 : 1, kAtATime = 16 / sizeof(T);
            const T *from = base + row * g.ld;
            const int64_t col0 = (int64_t)mine * (2 * kNibbleBlock) + k * 8;
            auto hold = [&](int y, const bf16x8v (&parts)[kParts]) {
                if constexpr (kParts == 1) {
                    x[y] = parts[0];
                } else {
                    const u32x4v a = __builtin_bit_cast(u32x4v, parts[0]), b = __builtin_bit_cast(u32x4v, parts[1]), c = __builtin_bit_cast(u32x4v, parts[2]);
                    u32x4v one;
#pragma unroll
                    for (int j = 0; j < 4; ++j) one[j] = part == 0 ? a[j] : part == 1 ? b[j] : c[j];
                    x[y] = __builtin_bit_cast(bf16x8v, one);
                }
            };
            bf16x8v parts[kParts];
            if ((int64_t)(mine + 1) * (2 * kNibbleBlock) <= g.d) {                          // all of the wave's columns are there
#pragma unroll
                for (int y0 = 0; y0 < 8; y0 += kAtATime) {
                    Eight<T> got[kAtATime];
#pragma unroll
                    for (int o = 0; o < kAtATime; ++o) got[o].ask(from + col0 + (y0 + o) * 32);
#pragma unroll
                    for (int o = 0; o < kAtATime; ++o) {
                        got[o].parts(parts);
                        hold(y0 + o, parts);
                    }
                }
                return;
            }
            float e[8];
#pragma unroll
            for (int y0 = 0; y0 < 8; y0 += kAtATime) {
                Eight<T> got[kAtATime];
#pragma unroll
                for (int o = 0; o < kAtATime; ++o) got[o].ask(from, col0 + (y0 + o) * 32, g.d);
#pragma unroll
                for (int o = 0; o < kAtATime; ++o) {
                    got[o].give(col0 + (y0 + o) * 32, g.d, true, e);
                    split8<kParts>(e, parts);
                    hold(y0 + o, parts);
                }
            }
            const int end = (int)(g.d >> 7);                                            // the block in which the rows end
            if ((g.d & 7) != 0 && end / 2 == mine) {
                load8(from + (g.d & ~7LL), g.d & 7, e);
                split8<kParts>(e, parts);
#pragma unroll
                for (int y = 0; y < 8; ++y)
                    if (((g.d & 255) >> 5) == y && ((g.d & 31) >> 3) == k) hold(y, parts);
            }
        };
        if (row >= 0 && row < g.m) {                                                    // (what is not there is not asked for)
            if (g.wide) take(static_cast<const float *>(g.x));
            else take(static_cast<const uint16_t *>(g.x));
        }
    }
#pragma unroll
    for (int j = 1; j < kBatch; ++j) fetch(c[j], j);
    scales[0][threadIdx.x] = held;
    lds_barrier();
    const int parts = g.wide ? 3 : 1;
    for (int it0 = 0; it0 < count; it0 += kBatch) {
        const int turn = it0 / kBatch & 1;
        float(*to)[kBatch][R][64] = sums[turn];
        held = scales_of(it0 + kBatch);
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            if (it0 + j < count) {
                // this tile's row of scales, from the wave's first block on
                const uint32_t *s0 = reinterpret_cast<const uint32_t *>(&scales[turn][((j * across + wave / along) * 16 + rho) * each]) + mine * G;
                float acc[R];
#pragma unroll
                for (int r = 0; r < R; ++r) acc[r] = 0.0f;
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    if (2 * mine + half >= g.blocks) continue;
                    const uint4 q = c[j].q[half];
                    const bf16x8v f[4] = {widen_codes(q.x), widen_codes(q.y), widen_codes(q.z), widen_codes(q.w)};
#pragma unroll
                    for (int y = 0; y < 4; y += 4 / G) {
                        const int at = half * G + y / (4 / G);
                        const uint32_t two = s0[at >> 1];
                        const float s = (at & 1) ? bf16_hi(two) : bf16_lo(two);
                        f32x4v sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                        for (int o = 0; o < 4 / G; ++o) sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[half * 4 + y + o], f[y + o], sum, 0, 0, 0);
#pragma unroll
                        for (int r = 0; r < R; ++r) acc[r] = fmaf(sum[r], s, acc[r]);
                    }
                }
#pragma unroll
                for (int r = 0; r < R; ++r) to[wave][j][r][lane] = acc[r];
            }
            // (no branch around a load of the classes': the compiler counts what is on its way.  What is asked for behind the last tile is the last tile, out of the caches.)
            fetch(c[j], it0 + j + kBatch);
        }
        scales[turn ^ 1][threadIdx.x] = held;
        lds_barrier();
        // results of the batch, sixteen classes to sixteen threads: row, tile of the batch, tile of the waves beside each other
        for (int at = threadIdx.x; at < across * kBatch * 4 * R * 16; at += kThreads) {
            const int l = at & 15, h = (at >> 4) % (4 * R), j = (at >> 4) / (4 * R) % kBatch, w = (at >> 4) / (4 * R) / kBatch;
            const int64_t cls = ((int64_t)(set0 + it0 + j) * across + w) * 16 + l;
            if (h >= g.n || it0 + j >= count || cls >= g.classes) continue;
            float sum = 0.0f;
            for (int part = 0; part < parts; ++part) {
                const int v = h * parts + part, from = (v & 3) * 16 + l;
                float one[kStreamWaves];
#pragma unroll
                for (int a = 0; a < kStreamWaves; ++a) one[a] = to[w * along + (a & (along - 1))][j][v >> 2][from];
#pragma unroll
                for (int a = 0; a < kStreamWaves; ++a) sum += a < along ? one[a] : 0.0f;
            }
            sum *= kResultScale;
            if (g.half) Elem<uint16_t>::put(static_cast<uint16_t *>(g.out) + h * g.ld_out + cls, sum);
            else Elem<float>::put(static_cast<float *>(g.out) + h * g.ld_out + cls, sum);
        }
    }
}

template <typename T, int MT, int R, int NT, int G, int WAVES, bool HELD>
static hipError_t launch_rows(Matmul4Args g, hipStream_t s)
{
    constexpr int kHeld = held_blocks4<MT, R, sizeof(T) == 4 ? 3 : 1>(), kAhead = ahead4<MT, R, NT, sizeof(T) == 4 ? 3 : 1>();
    const int64_t groups = (g.classes + 16 * NT - 1) / (16 * NT), panels = (g.n + 16 * MT - 1) / (16 * MT), pairs = (g.blocks + 1) / 2;
    int along = 1;
    while (along < WAVES && (!HELD || along * 2 * kAhead <= kHeld / 2) && along < pairs && groups * panels * along < 256 * WAVES) along *= 2;
    const int64_t grid = (groups * along + WAVES - 1) / WAVES;
    for (int64_t panel = 0; panel < panels; panel += 65535) {
        g.first_row = panel * (16 * MT);
        const hipError_t e = in_launches(grid, 64 * WAVES, [&](int64_t first, unsigned count) {
            g.first = first;
            hipLaunchKernelGGL((matmul4_kernel<T, MT, R, NT, G, WAVES, HELD>), dim3(count, (unsigned)(panels - panel < 65535 ? panels - panel : 65535)), dim3(64 * WAVES),
                               0, s, g, along);
        });
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <int R, int G>
static hipError_t launch_stream(const Matmul4Args &g, int along, hipStream_t s)
{
    const int64_t sets = ((g.classes + 15) / 16 + kStreamWaves / along - 1) / (kStreamWaves / along);
    hipLaunchKernelGGL((matmul4_stream_kernel<R, G>), dim3((unsigned)(sets < 256 ? sets : 256)), dim3(64 * kStreamWaves), 0, s, g, along);
    return hipGetLastError();
}

template <typename T, int G>
static hipError_t launch_matmul4(const Matmul4Args &g, hipStream_t s)
{
    const int pairs = (g.blocks + 1) / 2;
    const int64_t rows = g.wide ? 3 * g.n : g.n, tiles = (g.classes + 15) / 16;
    int along = 1;
    while (along < 16 && along < pairs) along *= 2;
    // More classes than a workgroup on every compute unit takes at a time, and rows that the waves' registers hold: the stream (bfloat16, us, stream | rows in LDS | rows asked for by each
    // wave: 1 x 65536 x 4096 28.3 | 34.0 | 45.5, 16 x 65536 x 4096 33.5 | 35.8 | 85.6, 4 x 16384 x 4096 11.5 | 15.6 | 14.9; 1 x 4096 x 4096, one tile a workgroup, 11.1 | 14.1 | 7.1).
    if (rows <= 16 && pairs <= 16 && tiles * along > 256 * 16) return rows <= 4 ? launch_stream<1, G>(g, along, s) : launch_stream<4, G>(g, along, s);
    // Rows in LDS where many classes share them, else asked for by each wave (us, in LDS | by each wave: 64 x 65536 x 4096 68 | 169 bfloat16, 143 | 286 fp32; 256 x 16384 x 4096 61 | 167;
    // 64 x 16384 x 4096 44 | 46, 133 | 75 fp32; 37 x 5003 x 3001 fp32 92 | 18; 20 x 20000 x 1000 fp32 22.7 | 24.6; 8 x 65536 x 4096 fp32 43 | 92).  The few percent lost
    // at 64 x 16384 x 4096 bfloat16 and 20 x 20000 x 1000 fp32 are the price of one number for both types.
    if (g.n <= 16 ? tiles > 1024 : tiles * ((g.n + 63) / 64) >= 2048) {
        if (g.n <= 8) return launch_rows<T, 1, 2, 1, G, 16, true>(g, s);
        if (g.n <= 16) return launch_rows<T, 1, 4, 1, G, 16, true>(g, s);
        if (g.n <= 32) return launch_rows<T, 2, 4, 2, G, 8, true>(g, s);
        return launch_rows<T, 4, 4, 2, G, 8, true>(g, s);
    }
    if (g.n <= 4) return launch_rows<T, 1, 1, 1, G, 16, false>(g, s);
    if (g.n <= 16) return launch_rows<T, 1, 4, 1, G, 16, false>(g, s);
    constexpr int kTiles = sizeof(T) == 4 && G == 4 ? 1 : 2;                            // (two would not fit the registers)
    return launch_rows<T, 2, 4, kTiles, G, 8, false>(g, s);
}
template <typename T>
static hipError_t launch_matmul4(const Matmul4Args &g, int group, hipStream_t s)
{
    return group == 32 ? launch_matmul4<T, 4>(g, s) : group == 64 ? launch_matmul4<T, 2>(g, s) : launch_matmul4<T, 1>(g, s);
}

static int check_nibbles(const wpsgd_nibbles *q)
{
    if (!q || q->rows < 0 || q->rows > 0x7FFFFFFFLL || q->cols < 0 || q->cols > (1LL << 31) || (q->group != 32 && q->group != 64 && q->group != 128)) return WPSGD_INVALID_ARG;
    if (q->rows == 0 || q->cols == 0) return WPSGD_OK;
    const int64_t blocks = (q->cols + kNibbleBlock - 1) / kNibbleBlock;
    if (!q->codes || !q->scales) return WPSGD_INVALID_ARG;
    if (q->ld < blocks * 64 || q->ld % 16 != 0 || (uintptr_t)q->codes % 16 != 0) return WPSGD_INVALID_ARG;
    if (q->ld_scales < blocks * (kNibbleBlock / q->group) || q->ld_scales % 8 != 0 || (uintptr_t)q->scales % 16 != 0) return WPSGD_INVALID_ARG;
    return WPSGD_OK;
}

}  // namespace wpsgd

using namespace wpsgd;

extern "C" {

int wpsgd_quantize_nibbles(const wpsgd_matrix *X, const int64_t *rows, int64_t n, const wpsgd_nibbles *out, void *stream)
{
    int rc = check_matrix(X);
    if (rc != WPSGD_OK) return rc;
    if (!X->dense) return WPSGD_UNSUPPORTED;
    if ((uintptr_t)X->dense % (X->dtype == WPSGD_BF16 ? 2 : 4) != 0 || n < 0 || (!rows && n > X->m)) return WPSGD_INVALID_ARG;
    rc = check_nibbles(out);
    if (rc != WPSGD_OK) return rc;
    if (out->rows != n || out->cols != X->d) return WPSGD_INVALID_ARG;
    if (n == 0) return WPSGD_OK;
    Quantize4Args a{X->dense, rows, X->m, X->d, X->ld, n, static_cast<uint8_t *>(out->codes), static_cast<uint16_t *>(out->scales), out->ld, out->ld_scales,
                    (out->cols + kNibbleBlock - 1) / kNibbleBlock, 0};
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool half = X->dtype == WPSGD_BF16;
    const auto kernel = out->group == 32   ? (half ? quantize4_kernel<uint16_t, 4> : quantize4_kernel<float, 4>)
                        : out->group == 64 ? (half ? quantize4_kernel<uint16_t, 2> : quantize4_kernel<float, 2>)
                                           : (half ? quantize4_kernel<uint16_t, 1> : quantize4_kernel<float, 1>);
    const hipError_t e = in_launches((n * a.blocks + 15) / 16, 256, [&](int64_t first, unsigned count) {
        a.first = first;
        hipLaunchKernelGGL(kernel, dim3(count), dim3(256), 0, s, a);
    });
    return e == hipSuccess ? WPSGD_OK : hip_fail(e);
}

int wpsgd_nibble_matmul(const wpsgd_matrix *X, const int64_t *rows, int64_t n, const wpsgd_nibbles *W, void *out, int64_t ld_out, wpsgd_dtype dtype, void *stream)
{
    int rc = check_matrix(X);
    if (rc != WPSGD_OK) return rc;
    if (!X->dense) return WPSGD_UNSUPPORTED;
    if ((uintptr_t)X->dense % (X->dtype == WPSGD_BF16 ? 2 : 4) != 0 || n < 0 || n > 0x7FFFFFFFLL || (!rows && n > X->m)) return WPSGD_INVALID_ARG;
    rc = check_nibbles(W);
    if (rc != WPSGD_OK) return rc;
    if (W->cols != X->d || (dtype != WPSGD_F32 && dtype != WPSGD_BF16)) return WPSGD_INVALID_ARG;
    if (n == 0 || W->rows == 0) return WPSGD_OK;
    if (!out || ld_out < W->rows || (uintptr_t)out % (dtype == WPSGD_F32 ? 4 : 2) != 0) return WPSGD_INVALID_ARG;
    const Matmul4Args g{X->dense, rows, X->m, X->d, X->ld, n, static_cast<const uint8_t *>(W->codes), static_cast<const uint16_t *>(W->scales), W->ld, W->ld_scales,
                        W->rows, (int)((W->cols + kNibbleBlock - 1) / kNibbleBlock), dtype == WPSGD_BF16, X->dtype == WPSGD_F32, out, ld_out, 0, 0};
    hipStream_t s = static_cast<hipStream_t>(stream);
    const hipError_t e = X->dtype == WPSGD_F32 ? launch_matmul4<float>(g, W->group, s) : launch_matmul4<uint16_t>(g, W->group, s);
    return e == hipSuccess ? WPSGD_OK : hip_fail(e);
}

}  // extern "C"
