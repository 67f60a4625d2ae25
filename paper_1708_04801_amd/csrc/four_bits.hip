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

// 1/4, 3/4 ... : where one code ends and the next begins, a border itself going to the even code
__device__ inline uint32_t code_of(float x, float s)
{
    const float size = fabsf(x);
    uint32_t c = size > 0.25f * s ? 1 : 0;
    c += size >= 0.75f * s ? 1 : 0;
    c += size > 1.25f * s ? 1 : 0;
    c += size >= 1.75f * s ? 1 : 0;
    c += size > 2.5f * s ? 1 : 0;
    c += size >= 3.5f * s ? 1 : 0;
    c += size > 5.0f * s ? 1 : 0;
    return c | (__float_as_uint(x) >> 28 & 8u);
}

// The bits of the least bfloat16 s >= 2^-126 with 6 s >= top; 1 for 0.  The quotient is off by half a place of fp32, so that what its upper half stands for is at most the
// answer and at most one place under it.
__device__ inline uint32_t scale_bits(float top)
{
    if (top == 0.0f) return 0x3F800000u;
    const float s = __uint_as_float(__float_as_uint(fmaxf(top / 6.0f, 1.17549435e-38f)) & 0xFFFF0000u);
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

// Sixteen lanes to a block of 128, eight elements to a lane; G groups to a block.
template <typename T, int G>
__global__ __launch_bounds__(256) void quantize4_kernel(Quantize4Args a)
{
    const int64_t first = (a.first + blockIdx.x) * 16;
    const int64_t row0 = first / a.blocks;
    const uint32_t at = (uint32_t)(first - row0 * a.blocks) + (threadIdx.x >> 4);      // (blocks < 2^25)
    const uint32_t down = at / (uint32_t)a.blocks;
    const int64_t row = row0 + down;
    if (row >= a.n) return;                                                            // (sixteen lanes at a time)
    const int64_t b = at - down * (uint32_t)a.blocks;
    const int64_t from = a.rows ? a.rows[row] : row;
    const int lane = threadIdx.x & 15;
    const int64_t col = b * kNibbleBlock + lane * 8;
    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (from >= 0 && from < a.m && col < a.d) load8(static_cast<const T *>(a.x) + from * a.ld + col, a.d - col, x);
    float top = 0.0f;
    bool fine = true;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        fine = fine && fabsf(x[j]) < __builtin_inff();
        top = fmaxf(top, fabsf(x[j]));
    }
    top = fine ? top : __builtin_inff();                                               // (no maximum drops that)
    top = fmaxf(top, dpp_move<0xB1, 0xF>(top));
    top = fmaxf(top, dpp_move<0x4E, 0xF>(top));
    if constexpr (G <= 2) top = fmaxf(top, dpp_move<0x141, 0xF>(top));
    if constexpr (G == 1) top = fmaxf(top, dpp_move<0x140, 0xF>(top));
    const bool whole = top < __builtin_inff();
    const uint32_t bits = whole ? scale_bits(top) : 0x7FC00000u;
    const float s = __uint_as_float(bits);
    uint32_t w = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) w |= (whole ? code_of(x[j], s) : 0u) << (4 * j);
    *reinterpret_cast<uint32_t *>(a.codes + row * a.ld_codes + b * 64 + (lane & 3) * 16 + (lane >> 2) * 4) = w;
    constexpr int kLanes = 16 / G;
    if (lane % kLanes == 0) a.scales[row * a.ld_scales + b * G + lane / kLanes] = col < a.d ? (uint16_t)(bits >> 16) : (uint16_t)0;
}

typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8v __attribute__((ext_vector_type(8)));
typedef float f32x4v __attribute__((ext_vector_type(4)));

// the eight values of a word's codes, as they are
__device__ inline bf16x8v widen_codes(uint32_t w)
{
    const bf16x2v a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 1),
                  c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 3);
    return bf16x8v{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

// fp32 values as sums of three bfloat16 values, eight significant bits each; what is not finite stays in the first
__device__ inline void split8(const float (&x)[8], bf16x8v (&part)[3])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t bits = __float_as_uint(x[j]);
        const bool finite = fabsf(x[j]) < __builtin_inff();
        const float hi = finite ? __uint_as_float(bits & 0xFFFF0000u) : x[j];
        const float rest = finite ? x[j] - hi : 0.0f;
        const float mid = __uint_as_float(__float_as_uint(rest) & 0xFFFF0000u);
        part[0][j] = (__bf16)hi;
        part[1][j] = (__bf16)mid;
        part[2][j] = (__bf16)(rest - mid);
    }
}

struct Matmul4Args {
    const void *x;
    const int64_t *rows;
    int64_t m, d, ld, n;
    const uint8_t *codes;
    const uint16_t *scales;
    int64_t ld_codes, ld_scales, classes;
    int blocks;
    int half;                  // results are bfloat16
    void *out;
    int64_t ld_out;
    int64_t first, first_row;  // workgroup and row at which the launch begins
};

// The classes' codes go from memory straight into the matrix instructions, sixteen classes to a wave; the few rows lie in LDS as fragments, up to 64 KiB of the sum at a time, fp32
// ones as three parts.  Row i of a tile is row 4 (i mod 4) + i / 4 of the instruction, so that up to four rows need one result register of a lane, up to eight two (R).  kWaves4 waves
// to a workgroup: `along` of them share the blocks of the sum in turn and add up through LDS in their order, the others take the next classes.  A group's products are
// summed by themselves and times its scale added in fp32.
constexpr int kWaves4 = 8;
template <int MT, int R, int PARTS> constexpr int held_blocks4()
{
    int n = 64;
    while (n > 1 && n * MT * R * PARTS > 64) n /= 2;
    return n;
}

template <typename T, int MT, int R, int G>
__global__ __launch_bounds__(64 * kWaves4) void matmul4_kernel(Matmul4Args g, int along)
{
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1, kHeld = held_blocks4<MT, R, PARTS>(), kLanes = 16 * R;
    constexpr int kAhead = 4;
    __shared__ union {
        bf16x8v held[kHeld * MT * 4 * PARTS][kLanes];
        f32x4v sums[kWaves4][MT][64];
    } lds;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, rho = lane & 15, k = lane >> 4;
    const int across = kWaves4 / along, mine = wave % along;
    const int64_t c0 = ((g.first + blockIdx.x) * across + wave / along) * 16, h0 = g.first_row + (int64_t)blockIdx.y * (16 * MT);
    const bool idle = c0 >= g.classes, active = (rho & 3) < R;
    const int place = k * (4 * R) + (rho >> 2) * R + (rho & 3);
    f32x4v acc[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[t] = f32x4v{0.0f, 0.0f, 0.0f, 0.0f};
    const int64_t cls = c0 + rho < g.classes ? c0 + rho : g.classes - 1;
    const uint8_t *codes = g.codes + cls * g.ld_codes + k * 16;
    const uint16_t *scales = g.scales + cls * g.ld_scales;
    uint4 q[kAhead];
    uint2 sc[kAhead];
    auto fetch = [&](int step, int j) {
        const int b = step * along + mine, at = b < g.blocks ? b : g.blocks - 1;
        q[j] = *reinterpret_cast<const uint4 *>(codes + (int64_t)at * 64);
        if constexpr (G == 1) sc[j].x = scales[at];
        else if constexpr (G == 2) sc[j].x = *reinterpret_cast<const uint32_t *>(scales + (int64_t)at * 2);
        else sc[j] = *reinterpret_cast<const uint2 *>(scales + (int64_t)at * 4);
    };
    // a thread's pieces of a filling: eight elements of one row each, the same row in every piece (MT 4: in every other one)
    constexpr int kPieces = kHeld * MT * 4 * kLanes, kEach = (kPieces + 511) / 512, kRowsOf = MT == 4 ? 2 : 1;
    const T *from[kRowsOf];
#pragma unroll
    for (int y = 0; y < kRowsOf; ++y) {
        const int piece = threadIdx.x + 512 * y, i = (piece >> 4) % (4 * R), t = (piece >> 4) / (4 * R) % MT;
        const int64_t h = h0 + t * 16 + i, row = h < g.n ? (g.rows ? g.rows[h] : h) : -1;
        from[y] = row >= 0 && row < g.m ? static_cast<const T *>(g.x) + row * g.ld : nullptr;
    }
    const int per = kHeld / along, steps = (g.blocks + kHeld - 1) / kHeld * per;        // of a wave between two fillings; the same for every wave
#pragma unroll
    for (int j = 0; j < kAhead; ++j) fetch(j, j);
    for (int step0 = 0; step0 < steps; step0 += kAhead) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int step = step0 + j;
            if (step >= steps) break;
            if (step % per == 0) {
                const int b0 = step / per * kHeld;
                if (step > 0) __syncthreads();
#pragma unroll
                for (int y = 0; y < kEach; ++y) {
                    const int piece = threadIdx.x + 512 * y;
                    if (kPieces % 512 != 0 && piece >= kPieces) break;
                    const int pk = piece & 3, pj = piece >> 2 & 3, i = (piece >> 4) % (4 * R), u = (piece >> 4) / (4 * R), t = u % MT, in = u / MT;
                    const int64_t col = (int64_t)(b0 + in) * kNibbleBlock + pj * 32 + pk * 8;
                    const T *p = from[kRowsOf == 2 ? y & 1 : 0];
                    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                    if (p && col < g.d) load8(p + col, g.d - col, x);
                    bf16x8v part[3];
                    if constexpr (PARTS == 3) {
                        split8(x, part);
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) part[0][e] = (__bf16)x[e];
                    }
                    const int to = pk * (4 * R) + (i & 3) * R + (i >> 2);
#pragma unroll
                    for (int e = 0; e < PARTS; ++e) lds.held[((in * MT + t) * 4 + pj) * PARTS + e][to] = part[e];
                }
                __syncthreads();
            }
            const int b = step * along + mine;
            if (b < g.blocks && !idle) {
                const uint32_t w[4] = {q[j].x, q[j].y, q[j].z, q[j].w};
                bf16x8v f[4];
#pragma unroll
                for (int y = 0; y < 4; ++y) f[y] = widen_codes(w[y]);
                const float s[4] = {bf16_lo(sc[j].x), G > 1 ? bf16_hi(sc[j].x) : 0.0f, G > 2 ? bf16_lo(sc[j].y) : 0.0f, G > 2 ? bf16_hi(sc[j].y) : 0.0f};
                const int at = b % kHeld;
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    f32x4v sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
#pragma unroll
                        for (int e = 0; e < PARTS; ++e) {
                            bf16x8v h = {};
                            if (R == 4 || active) h = lds.held[((at * MT + t) * 4 + y) * PARTS + e][place];
                            sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(h, f[y], sum, 0, 0, 0);
                        }
                        if ((y + 1) % (4 / G) == 0) {
#pragma unroll
                            for (int r = 0; r < R; ++r) acc[t][r] = fmaf(sum[r], s[y / (4 / G)], acc[t][r]);
                            sum = f32x4v{0.0f, 0.0f, 0.0f, 0.0f};
                        }
                    }
                }
            }
            fetch(step + kAhead, j);
        }
    }
    if (along > 1) {
        __syncthreads();
#pragma unroll
        for (int t = 0; t < MT; ++t) lds.sums[wave][t][lane] = acc[t];
        __syncthreads();
        if (mine != 0) return;
#pragma unroll
        for (int t = 0; t < MT; ++t)
            for (int w = 1; w < along; ++w) acc[t] += lds.sums[wave + w][t][lane];
    }
    if (c0 + rho >= g.classes) return;
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t h = h0 + t * 16 + 4 * r + k;
            if (h >= g.n) continue;
            if (g.half) Elem<uint16_t>::put(static_cast<uint16_t *>(g.out) + h * g.ld_out + c0 + rho, acc[t][r]);
            else Elem<float>::put(static_cast<float *>(g.out) + h * g.ld_out + c0 + rho, acc[t][r]);
        }
}

template <typename T, int MT, int R, int G>
static hipError_t launch_matmul4(Matmul4Args g, hipStream_t s)
{
    constexpr int kHeld = held_blocks4<MT, R, sizeof(T) == 4 ? 3 : 1>();
    const int64_t groups = (g.classes + 15) / 16, panels = (g.n + 16 * MT - 1) / (16 * MT);
    int along = 1;
    while (along < kWaves4 && along < kHeld && groups * panels * along < 2048 && g.blocks >= 2 * along) along *= 2;
    const int64_t grid = (groups * along + kWaves4 - 1) / kWaves4;
    for (int64_t panel = 0; panel < panels; panel += 65535) {
        g.first_row = panel * (16 * MT);
        const hipError_t e = in_launches(grid, 64 * kWaves4, [&](int64_t first, unsigned count) {
            g.first = first;
            hipLaunchKernelGGL((matmul4_kernel<T, MT, R, G>), dim3(count, (unsigned)(panels - panel < 65535 ? panels - panel : 65535)), dim3(64 * kWaves4), 0, s, g, along);
        });
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
template <typename T, int G>
static hipError_t launch_matmul4(const Matmul4Args &g, hipStream_t s)
{
    if (g.n <= 4) return launch_matmul4<T, 1, 1, G>(g, s);
    if (g.n <= 8) return launch_matmul4<T, 1, 2, G>(g, s);
    if (g.n <= 16) return launch_matmul4<T, 1, 4, G>(g, s);
    if (g.n <= 32) return launch_matmul4<T, 2, 4, G>(g, s);
    return launch_matmul4<T, 4, 4, G>(g, s);
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
                        W->rows, (int)((W->cols + kNibbleBlock - 1) / kNibbleBlock), dtype == WPSGD_BF16, out, ld_out, 0, 0};
    hipStream_t s = static_cast<hipStream_t>(stream);
    const hipError_t e = X->dtype == WPSGD_F32 ? launch_matmul4<float>(g, W->group, s) : launch_matmul4<uint16_t>(g, W->group, s);
    return e == hipSuccess ? WPSGD_OK : hip_fail(e);
}

}  // extern "C"
