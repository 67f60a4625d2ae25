// Scores: out[i,j] = sum over blocks b of 2^(ea[i,b] + eb[j,b]) * sum_k A[i,b,k] B[j,b,k], rounded once to the output's type.
//
// Sums of fp32 accuracy: codes become bfloat16 in registers, their block's power of two in the same instruction, and go to the bfloat16 matrix instruction, which
// adds in fp32.  Four significant bits fit, and the exponents of all fp32 values do with half the power: 1.94 * 2^127 and more has code 256 at 2^120, and 2^128
// would be infinite.  Results are taken times four at the end.  Exact for exponent bytes 4 to 247; with 1 to 3, bfloat16's subnormal spacing rounds values to multiples of 2^-132.
// The 8-bit matrix instructions are twice as fast, but inside a group of products they keep only what lies within 2^14 of the largest: 1.5e-5 (normal
// values) to 7e-5 (values over several powers of ten) of the result's norm, where fp32 sums are off by 1e-7.  So they are for bfloat16 results only, and a call may ask for
// fp32 sums of those, too (8192 x 65536 x 4096 3070 us instead of 1860).
#include <type_traits>

#include "block_plan.h"
#include "class_ops.h"

namespace wpsgd {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

struct MatmulArgs {
    const uint8_t *a, *b, *ea, *eb;
    int64_t lda, ldb, lde_a, lde_b;
    int64_t M, N;
    int blocks;
    void *out;
    int64_t ldo;
    int each;                  // blocks to a part of the sum (all, where it is not split)
    int64_t first;             // workgroup of the call at which the launch begins (few rows against many)
};

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// half a block's power of two (the instruction takes the exponent field 0, for byte 1, as 2^-127)
__device__ inline float half_power_of(int byte) { return __uint_as_float(((uint32_t)byte << 23) - (1u << 23)); }
constexpr float kHalves = 4.0f;        // what products of two halves are short of

// eight codes, two words, times a power of two
__device__ inline bf16x8 widen8(uint32_t lo, uint32_t hi, float scale)
{
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return bf16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

// four results side by side
__device__ inline void store4(float *p, const f32x4 &v) { store16(p, Bytes16{{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])}}); }
__device__ inline void store4(uint16_t *p, const f32x4 &v)
{
    typedef uint32_t words2 __attribute__((ext_vector_type(2)));
    typedef words2 any_words2 __attribute__((aligned(2)));
    *(global_ptr<any_words2>)p = words2{bf16_pack(v[0], v[1]), bf16_pack(v[2], v[3])};
}

// Few rows against many.  The one operand's rows (the class vectors of a serving call) are read once, straight from memory into the matrix instructions, sixteen
// rows times NT to a wave; the other's 16 MT rows lie in LDS as bfloat16 fragments, a few blocks of the sum at a time (asked for by each wave
// they are a trip to the L2 a block: 16 x 65536 x 4096 79 us, 64 x 65536 x 4096 138).  kRowWaves waves to a workgroup: `along` of them share the blocks of the
// sum in turn and add up through LDS, in their order, the others take the next rows.  Bound by memory: 16 x 65536 x 4096 reads 270 MB out of the caches in 66 us, 4.1 TB/s; 1 x 4096 x
// 4096, 17 MB in 8.6 us, is a start and a few trips.
// `turned`: the many rows are A's (results of a lane lie below each other), else B's (beside each other).
constexpr int kRowWaves = 8;
constexpr int kHeldBlocks = 16;                                       // of sixteen rows: 64 KiB
template <int MT, int NT, typename TO>
__global__ __launch_bounds__(64 * kRowWaves) void matmul_rows_kernel(MatmulArgs g, int along, bool turned)
{
    constexpr int kHeld = kHeldBlocks / MT;
    constexpr int kAhead = 2;                                         // blocks of the many rows on their way at a time (four: 64 us instead of 57)
    __shared__ union {
        bf16x8 held[kHeldBlocks * 4][64];                             // block, rows, quarter: a fragment for each lane
        f32x4 sums[kRowWaves][MT * NT][64];
    } lds;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint8_t *many = turned ? g.a : g.b, *few = turned ? g.b : g.a, *many_e = turned ? g.ea : g.eb, *few_e = turned ? g.eb : g.ea;
    const int64_t ld_many = turned ? g.lda : g.ldb, ld_few = turned ? g.ldb : g.lda, lde_many = turned ? g.lde_a : g.lde_b, lde_few = turned ? g.lde_b : g.lde_a;
    const int64_t rows_many = turned ? g.M : g.N, rows_few = turned ? g.N : g.M;
    const int across = kRowWaves / along, mine = wave % along;
    const int64_t s0 = ((g.first + blockIdx.x) * across + wave / along) * (16 * NT), h0 = (int64_t)blockIdx.y * (16 * MT);
    const int r = lane & 15, group = lane >> 4;
    const bool idle = s0 >= rows_many;
    f32x4 acc[MT][NT];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int u = 0; u < NT; ++u) acc[t][u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const uint8_t *ps[NT], *es[NT];
#pragma unroll
    for (int u = 0; u < NT; ++u) {
        const int64_t i = s0 + u * 16 + r < rows_many ? s0 + u * 16 + r : rows_many - 1;
        ps[u] = many + i * ld_many + group * 16;                      // (an instruction takes 64 bytes of a row)
        es[u] = many_e + i * lde_many;
    }
    uint4 qs[kAhead][NT][2];
    uint8_t cs[kAhead][NT];
    auto fetch = [&](int step, int j) {
        const int b = step * along + mine, at = b < g.blocks ? b : g.blocks - 1;
#pragma unroll
        for (int u = 0; u < NT; ++u) {
            const uint4 *p = reinterpret_cast<const uint4 *>(ps[u] + (int64_t)at * 128);
            qs[j][u][0] = p[0];
            qs[j][u][1] = p[4];
            cs[j][u] = es[u][at];
        }
    };
    const int per = kHeld / along;                                    // steps of a wave between two fillings
    const int steps = (g.blocks + kHeld - 1) / kHeld * per;           // the same for every wave
    if (steps > 0) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) fetch(j, j);
    }
    for (int step0 = 0; step0 < steps; step0 += kAhead) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int step = step0 + j;
            if (step >= steps) break;
            if (step % per == 0) {
                const int b0 = step / per * kHeld, n = g.blocks - b0 < kHeld ? g.blocks - b0 : kHeld;
                if (step > 0) __syncthreads();
                // items of block, rows and half, all of a wave's on their way at once
                constexpr int kItems = kHeldBlocks * 2 / kRowWaves;
                uint4 q[kItems];
                uint8_t c[kItems];
#pragma unroll
                for (int x = 0; x < kItems; ++x) {
                    const int item = wave + x * kRowWaves, t = (item >> 1) % MT, in = (item >> 1) / MT, at = b0 + (in < n ? in : n - 1);
                    const int64_t i = h0 + t * 16 + r < rows_few ? h0 + t * 16 + r : rows_few - 1;
                    q[x] = *reinterpret_cast<const uint4 *>(few + i * ld_few + (int64_t)at * 128 + (item & 1) * 64 + group * 16);
                    c[x] = few_e[i * lde_few + at];
                }
#pragma unroll
                for (int x = 0; x < kItems; ++x) {
                    const int item = wave + x * kRowWaves;
                    lds.held[(item >> 1) * 4 + (item & 1) * 2][lane] = widen8(q[x].x, q[x].y, half_power_of(c[x]));
                    lds.held[(item >> 1) * 4 + (item & 1) * 2 + 1][lane] = widen8(q[x].z, q[x].w, half_power_of(c[x]));
                }
                __syncthreads();
            }
            const int b = step * along + mine;
            if (b < g.blocks && !idle) {
                bf16x8 fs[NT][4];
#pragma unroll
                for (int u = 0; u < NT; ++u) {
                    const float c = half_power_of(cs[j][u]);
                    fs[u][0] = widen8(qs[j][u][0].x, qs[j][u][0].y, c);
                    fs[u][1] = widen8(qs[j][u][0].z, qs[j][u][0].w, c);
                    fs[u][2] = widen8(qs[j][u][1].x, qs[j][u][1].y, c);
                    fs[u][3] = widen8(qs[j][u][1].z, qs[j][u][1].w, c);
                }
                const int at = b % kHeld;
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const bf16x8 fh = lds.held[(at * MT + t) * 4 + k][lane];
#pragma unroll
                        for (int u = 0; u < NT; ++u) acc[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fs[u][k], fh, acc[t][u], 0, 0, 0);
                    }
            }
            fetch(step + kAhead, j);
        }
    }
    if (along > 1) {
        __syncthreads();
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int u = 0; u < NT; ++u) lds.sums[wave][t * NT + u][lane] = acc[t][u];
        __syncthreads();
        if (mine != 0) return;
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int u = 0; u < NT; ++u)
                for (int w = 1; w < along; ++w) acc[t][u] += lds.sums[wave + w][t * NT + u][lane];
    }
    if (idle) return;
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int u = 0; u < NT; ++u) acc[t][u] *= kHalves;
    TO *out = static_cast<TO *>(g.out);
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int u = 0; u < NT; ++u) {
            const int64_t h = h0 + t * 16 + r, s = s0 + u * 16 + group * 4;
            if (h >= rows_few || s >= rows_many) continue;
            if (!turned && s + 4 <= rows_many) {
                store4(out + h * g.ldo + s, acc[t][u]);
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (s + q < rows_many) Elem<TO>::put(out + (turned ? (s + q) * g.ldo + h : h * g.ldo + s + q), acc[t][u][q]);
            }
        }
}

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

// Sixteen bytes a lane from memory to LDS at `to` + 16 lane.  An assembly statement, since the compiler would wait for it before any LDS access
// behind it; whoever reads the bytes waits for the counter first.
__device__ inline void fetch_to_lds(const i32x4 &from, uint32_t to, int at, int along)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" : : "s"(to), "v"(at), "s"(from), "s"(along) : "memory", "m0");
}

// Which tile a workgroup computes.  Workgroups go to the eight XCDs in turn: each XCD gets a run of its own of the tiles, which walk down kTall tiles
// of A before the next of B, so that the tiles an XCD's 32 compute units hold at a time share a few rows of both in its L2.
constexpr int kTall = 8;
__device__ inline void tile_of(uint32_t id, uint32_t count, uint32_t tiles_m, uint32_t tiles_n, uint32_t &tm, uint32_t &tn)
{
    const uint32_t xcd = id & 7, each = count >> 3, more = count & 7;
    const uint32_t at = xcd * each + (xcd < more ? xcd : more) + (id >> 3);
    const uint32_t band = at / (kTall * tiles_n), first = band * kTall;
    const uint32_t tall = tiles_m - first < kTall ? tiles_m - first : kTall;
    const uint32_t in = at - band * kTall * tiles_n;
    tm = first + in % tall;
    tn = in / tall;
}

// Large products.  A workgroup of four waves, two by two, has 64 TM x 64 TN results, a wave 32 TM x 32 TN; blocks of 128 along the sum.
//
// Rows land in LDS by themselves, eight rows of 128 bytes to an instruction.  Sixteen bytes q of row r lie at place q ^ (r / 2 mod 8) of the row, so that any sixteen lanes
// that read the same piece of rows which differ modulo 16 meet all banks once (with r mod 8 half of the LDS cycles were conflicts); the loads fetch in that order.  Rows behind the last repeat it.  Each
// row's exponent bytes come four blocks at a time, a word a row, into two buffers in turn.
template <int TM, int TN>
struct Tile {
    static constexpr int BM = 64 * TM, BN = 64 * TN, LA = 2 * TM, LB = 2 * TN;      // LA, LB: a wave's loads for a block
    static constexpr int kExps = (BM + BN) * 4;
    i32x4 ra, rb, rea, reb;
    int from_a[LA], from_b[LB], from_e[2];
    int lane, wave, left_m, left_n;
    int64_t i0, j0;

    __device__ static i32x4 resource(const uint8_t *p)
    {
        const uint64_t at = (uint64_t)p;
        return i32x4{(int)(uint32_t)at, (int)(uint32_t)(at >> 32), 0x7FFFFFFF, 0x00020000};
    }
    // ROWS: how many of A's rows of each wave row are fetched at a time; first: block at which the workgroup's sum begins, a multiple of four
    template <int ROWS>
    __device__ void init(const MatmulArgs &g, int first)
    {
        lane = threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        uint32_t tm, tn;
        tile_of(blockIdx.x, gridDim.x, (uint32_t)((g.M + BM - 1) / BM), (uint32_t)((g.N + BN - 1) / BN), tm, tn);
        i0 = (int64_t)tm * BM;
        j0 = (int64_t)tn * BN;
        left_m = (int)(g.M - i0 < BM ? g.M - i0 : BM);
        left_n = (int)(g.N - j0 < BN ? g.N - j0 : BN);
        ra = resource(g.a + i0 * g.lda + (int64_t)first * 128);
        rb = resource(g.b + j0 * g.ldb + (int64_t)first * 128);
        const auto piece = [&](int row) { return ((lane & 7) ^ ((row >> 1) & 7)) * 16; };     // of a row of LDS
        constexpr int kUnit = 2 * ROWS, kUnits = BM / kUnit, kEach = LA / kUnits;      // rows of a unit, units, a wave's loads for one
#pragma unroll
        for (int t = 0; t < LA; ++t) {
            const int in = (wave * kEach + t % kEach) * 8 + (lane >> 3);            // row of the unit
            const int r = (in / ROWS) * (BM / 2) + (t / kEach) * ROWS + in % ROWS;
            from_a[t] = (r < left_m ? r : left_m - 1) * (int)g.lda + piece(in);
            asm volatile("" : "+v"(from_a[t]));            // (one register: the compiler's product has two)
        }
#pragma unroll
        for (int t = 0; t < LB; ++t) {
            const int r = (wave * LB + t) * 8 + (lane >> 3);
            from_b[t] = (r < left_n ? r : left_n - 1) * (int)g.ldb + piece(r);
            asm volatile("" : "+v"(from_b[t]));
        }
        // words of exponents: A's rows, then B's, 64 to an instruction, a wave's share in one or two
        rea = resource(g.ea + i0 * g.lde_a + first);
        reb = resource(g.eb + j0 * g.lde_b + first);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int c = exponent_chunk(t), r = (c < TM ? c : c - TM) * 64 + lane;
            const int left = c < TM ? left_m : left_n;
            from_e[t] = (r < left ? r : left - 1) * (int)(c < TM ? g.lde_a : g.lde_b);
            asm volatile("" : "+v"(from_e[t]));
        }
    }
    __device__ int exponent_chunk(int t) const { return (wave * 2 + t) % (TM + TN); }
    // every block asks for one of the two chunks of the next four blocks' words
    __device__ void fetch_exponents(uint32_t to, int t, int group) const
    {
        const int c = exponent_chunk(t);
        const i32x4 from = c < TM ? rea : reb;
        const int at = t ? from_e[1] : from_e[0];
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds" : : "s"(to + c * 256), "v"(at), "s"(from), "s"(group * 4)
                     : "memory", "m0");
    }
    // A wave's results, 32 rows at a time, through LDS of its own (32 rows of 32 TN results), so that whole rows of 128 bytes and more go out: with what
    // a lane holds (four results side by side) 32 bytes of a row at a time, bfloat16 results cost 0.8 ms per GiB on top of the products.
    template <typename TO>
    __device__ void store(const MatmulArgs &g, f32x16 (&acc)[TM][TN], float times, uint8_t *room) const
    {
        constexpr int kRow = 32 * TN * (int)sizeof(TO), kPieces = kRow / 16, E = Elem<TO>::kPer16;
        static_assert(kPieces >= 8, "pieces of a row are permuted within eight");
        const int m = lane & 31, half = lane >> 5;
        const int wm = (wave >> 1) * 32 * TM, wn = (wave & 1) * 32 * TN;
        TO *out = static_cast<TO *>(g.out);
#pragma unroll
        for (int t = 0; t < TM; ++t) {
#pragma unroll
            for (int u = 0; u < TN; ++u)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float x0 = acc[t][u][q * 4] * times, x1 = acc[t][u][q * 4 + 1] * times, x2 = acc[t][u][q * 4 + 2] * times, x3 = acc[t][u][q * 4 + 3] * times;
                    if constexpr (E == 8) {
                        const int piece = u * 4 + q;
                        *reinterpret_cast<uint2 *>(room + m * kRow + ((piece ^ (m & 7)) * 16) + half * 8) = make_uint2(bf16_pack(x0, x1), bf16_pack(x2, x3));
                    } else {
                        const int piece = u * 8 + q * 2 + half;
                        *reinterpret_cast<float4 *>(room + m * kRow + ((piece ^ (m & 7)) * 16)) = make_float4(x0, x1, x2, x3);
                    }
                }
            // (the wave's own LDS accesses are in order)
#pragma unroll
            for (int n = 0; n < kPieces / 2; ++n) {
                const int at = n * 64 + lane, row = at / kPieces, piece = at % kPieces;
                const uint4 v = *reinterpret_cast<const uint4 *>(room + row * kRow + ((piece ^ (row & 7)) * 16));
                const int i = wm + t * 32 + row, j = wn + piece * E;
                if (i < left_m && j < left_n) {
                    TO *p = out + (i0 + i) * g.ldo + j0 + j;
                    const Bytes16 q{{v.x, v.y, v.z, v.w}};
                    if (j + E <= left_n) {
                        store16(p, q);
                    } else {
#pragma unroll
                        for (int e = 0; e < E; ++e)
                            if (j + e < left_n) Elem<TO>::put(p + e, Elem<TO>::get(q.w, e));
                    }
                }
            }
        }
    }
};

__device__ inline uint32_t lds_address(const void *p) { return (uint32_t)(size_t)(__attribute__((address_space(3))) const uint8_t *)p; }

#define WPSGD_IN_ORDER __builtin_amdgcn_sched_barrier(0)

// Sums of fp32 accuracy (see the top).  A block is taken in four parts of 32: a wave holds B's part as bfloat16 and takes A's 32 rows in turn, a row
// being TN x 2 instructions; the next row's codes are on their way and the one before them is widened meanwhile.  B's next part is widened as the last row's products release
// its registers.  The barrier stands in front of the second to last row of a block: everything of it has been read, the next block is there, and the loads
// of the one behind that leave, a few to a row.  Bound by the matrix instructions, busy for 74 % of the cycles, and the card's power: 16384 x 4096 x 8192 750 to 790 us,
// 1.4 PFLOP/s, where the library's bfloat16 product, which need not widen anything, takes 809.
template <int TM, int TN, typename TO>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(TM * TN > 8 ? 1 : 2, TM * TN > 8 ? 1 : 2))) void matmul_tile_kernel(MatmulArgs g)
{
    using G = Tile<TM, TN>;
    constexpr int kStage = (G::BM + G::BN) * 128, kLoads = G::LA + G::LB;
    constexpr int kLds = 2 * kStage + 2 * G::kExps;
    static_assert(4 * 32 * 32 * TN * sizeof(TO) <= 2 * kStage, "room for the results");
    constexpr int kPer = TN < 3 ? TN : 3;                     // loads to a row
    static_assert(TM % 2 == 0 && kPer * (4 * TM - 2) >= kLoads, "rows enough for the loads");
    __shared__ __attribute__((aligned(1024))) uint8_t lds[kLds];
    G tile;
    // a part of the sum for each blockIdx.y, its results behind each other
    const int first = blockIdx.y * g.each;
    g.out = static_cast<TO *>(g.out) + (int64_t)blockIdx.y * g.M * g.N;
    tile.template init<G::BM / 2>(g, first);
    const uint32_t lds0 = lds_address(lds);
    const int lane = tile.lane, wave = tile.wave;
    const int r = lane & 31, half = lane >> 5;
    const int row_a = (wave >> 1) * 32 * TM + r, row_b = G::BM + (wave & 1) * 32 * TN + r;
    const int blocks = g.blocks - first < g.each ? g.blocks - first : g.each, end = blocks - 1, groups_end = end >> 2;

    f32x16 acc[TM][TN];
#pragma unroll
    for (int t = 0; t < TM; ++t)
#pragma unroll
        for (int u = 0; u < TN; ++u)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[t][u][q] = 0.0f;

    auto fetch = [&](int buffer, int b, int n) {              // the n-th of a wave's loads
        const uint32_t to = lds0 + (buffer & 1) * kStage;
        if (n < G::LA) fetch_to_lds(tile.ra, to + (wave * G::LA + n) * 1024, tile.from_a[n], b * 128);
        else fetch_to_lds(tile.rb, to + G::BM * 128 + (wave * G::LB + n - G::LA) * 1024, tile.from_b[n - G::LA], b * 128);
    };
    auto read = [&](int row, int b, int part) -> uint4 {
        return *reinterpret_cast<const uint4 *>(lds + (b & 1) * kStage + row * 128 + (((part * 2 + half) ^ ((r >> 1) & 7)) * 16));
    };
    auto scale = [&](int row, int b) -> float {
        return half_power_of(lds[2 * kStage + ((b >> 2) & 1) * G::kExps + row * 4 + (b & 3)]);
    };
    bf16x8 fa[2][2], fb[TN][2];
    uint4 qa[2], qb[TN];
    float ca[TM], cb[TN];
    auto widen = [](const uint4 &q, float c, bf16x8 (&to)[2]) {
        to[0] = widen8(q.x, q.y, c);
        to[1] = widen8(q.z, q.w, c);
    };
    tile.fetch_exponents(lds0 + 2 * kStage, 0, 0);
    tile.fetch_exponents(lds0 + 2 * kStage, 1, 0);
#pragma unroll
    for (int n = 0; n < kLoads; ++n) fetch(0, 0, n);
    asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" : : : "memory");
#pragma unroll
    for (int n = 0; n < 2 * kPer; ++n) fetch(1, end < 1 ? end : 1, n);
    tile.fetch_exponents(lds0 + 2 * kStage + G::kExps, 0, groups_end < 1 ? groups_end : 1);
    tile.fetch_exponents(lds0 + 2 * kStage + G::kExps, 1, groups_end < 1 ? groups_end : 1);
    qa[0] = read(row_a, 0, 0);
    qa[1] = read(row_a + 32, 0, 0);
#pragma unroll
    for (int u = 0; u < TN; ++u) qb[u] = read(row_b + u * 32, 0, 0);
#pragma unroll
    for (int t = 0; t < TM; ++t) ca[t] = scale(row_a + t * 32, 0);
#pragma unroll
    for (int u = 0; u < TN; ++u) {
        cb[u] = scale(row_b + u * 32, 0);
        widen(qb[u], cb[u], fb[u]);
    }
    widen(qa[0], ca[0], fa[0]);
    for (int b = 0; b < blocks; ++b) {
        const int ahead = b + 2 < blocks ? b + 2 : end, next = b + 1 < blocks ? b + 1 : end;
        const int later = b + 1 < blocks ? b + 1 : end;                  // the block that the previous barrier let in (behind the last one: once more)
#pragma unroll
        for (int part = 0; part < 4; ++part)
#pragma unroll
            for (int t = 0; t < TM; ++t) {
                const int i = part * TM + t;                              // row of the block; the barrier in front of row 4 TM - 2
                if (i == 4 * TM - 2) {
                    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" : : : "memory");
                }
                WPSGD_IN_ORDER;
                // codes two rows ahead (the loop's last ones are of the next block)
                const int j = i + 2;
                const bool over = j >= 4 * TM;
                qa[i & 1] = read(row_a + (j % TM) * 32, over ? next : b, (j / TM) & 3);
                if (t == TM - 2) {
#pragma unroll
                    for (int u = 0; u < TN; ++u) qb[u] = read(row_b + u * 32, part == 3 ? next : b, (part + 1) & 3);
                    if (part == 3) {
#pragma unroll
                        for (int u = 0; u < TN; ++u) cb[u] = scale(row_b + u * 32, next);
                    }
                }
                if (i == 4 * TM - 1) {
#pragma unroll
                    for (int u = 1; u < TM; ++u) ca[u] = scale(row_a + u * 32, next);
                }
                if (i == 4 * TM - 2) ca[0] = scale(row_a, next);
                WPSGD_IN_ORDER;
#pragma unroll
                for (int u = 0; u < TN; ++u) {
                    acc[t][u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[u][0], fa[i & 1][0], acc[t][u], 0, 0, 0);
                    // loads from the barrier on
                    const int slot = ((i + 2) % (4 * TM)) * kPer + u;
                    if (u < kPer && slot < kLoads) fetch(i >= 4 * TM - 2 ? b : b + 1, i >= 4 * TM - 2 ? ahead : later, slot);
                    if (u == 0 && i == 4 * TM / 2) tile.fetch_exponents(lds0 + 2 * kStage + (((b >> 2) + 1) & 1) * G::kExps, b & 1, (b >> 2) < groups_end ? (b >> 2) + 1 : groups_end);
                    WPSGD_IN_ORDER;
                    acc[t][u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[u][1], fa[i & 1][1], acc[t][u], 0, 0, 0);
                    if (t == TM - 1) widen(qb[u], cb[u], fb[u]);
                    if (u == TN - 2) widen(qa[(i + 1) & 1], ca[(t + 1) % TM], fa[(i + 1) & 1]);
                    WPSGD_IN_ORDER;
                }
            }
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" : : : "memory");
    tile.template store<TO>(g, acc, kHalves, lds + wave * (32 * 32 * TN * (int)sizeof(TO)));
}

// Products in the 8-bit matrix instruction, which takes the exponent bytes with it: twice the rate, sums as said at the top, so for bfloat16 results only.
// A wave holds the whole block of B and takes A's 32 rows in turn, a row being TN x 2 instructions; the next row is on its way, and B's next block is read as the last
// row's products release its registers.  LDS holds two blocks of B and five half blocks of A (rows 0 and 1, or 2 and 3, of both wave rows): B's room is free
// once every wave has it in registers, in front of row 1, so that loads have two blocks (A) or one and a half (B) to arrive: with two whole blocks in LDS,
// 2.0 instead of 2.6 PFLOP/s (a product whose loads are left out: 2.6).
// Bound by the card's power: matrix instructions are busy for 67 to 77 % of the cycles and the clock falls to 1.7 GHz (8192 x 65536 x 4096 1.7 to 1.8 ms, 2.4 to 2.6 PFLOP/s, by the card).
// Barriers stand in front of rows 1 and 3; loads complete in order, so a count of those that may still be on their way says which have come.
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1))) void matmul_fast_kernel(MatmulArgs g)
{
    constexpr int TM = 4, TN = 4;
    using G = Tile<TM, TN>;
    constexpr int kUnit = 128 * 128, kUnits = 5, kB = G::BN * 128;
    constexpr int kAtB = kUnits * kUnit, kAtE = kAtB + 2 * kB;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[kAtE + 2 * G::kExps];
    G tile;
    tile.template init<64>(g, 0);
    const uint32_t lds0 = lds_address(lds);
    const int lane = tile.lane, wave = tile.wave;
    const int r = lane & 31, half = lane >> 5;
    const int row_a = (wave >> 1) * 64 + r, row_b = (wave & 1) * 32 * TN + r;
    const int blocks = g.blocks, end = blocks - 1, groups_end = end >> 2;

    f32x16 acc[TM][TN];
#pragma unroll
    for (int t = 0; t < TM; ++t)
#pragma unroll
        for (int u = 0; u < TN; ++u)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[t][u][q] = 0.0f;

    auto clamp = [&](int b) { return b < end ? b : end; };
    auto fetch_a = [&](uint32_t slot, int b, int unit, int n) {       // n of 4
        fetch_to_lds(tile.ra, lds0 + slot * kUnit + (wave * 4 + n) * 1024, tile.from_a[unit * 4 + n], clamp(b) * 128);
    };
    auto fetch_b = [&](int b, int n) {                                // n of 8
        fetch_to_lds(tile.rb, lds0 + kAtB + (b & 1) * kB + (wave * G::LB + n) * 1024, tile.from_b[n], clamp(b) * 128);
    };
    auto fetch_e = [&](int group, int t) {
        tile.fetch_exponents(lds0 + kAtE + (group & 1) * G::kExps, t, group < groups_end ? group : groups_end);
    };
    auto read = [&](const uint8_t *p, int k) {
        i32x8 v;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint4 q = *reinterpret_cast<const uint4 *>(p + (((k * 4 + h * 2 + half) ^ ((r >> 1) & 7)) * 16));
            v[h * 4] = (int)q.x; v[h * 4 + 1] = (int)q.y; v[h * 4 + 2] = (int)q.z; v[h * 4 + 3] = (int)q.w;
        }
        return v;
    };
    auto read_a = [&](uint32_t slot, int t, int k) { return read(lds + slot * kUnit + (row_a + (t & 1) * 32) * 128, k); };
    auto read_b = [&](int b, int u, int k) { return read(lds + kAtB + (b & 1) * kB + (row_b + u * 32) * 128, k); };
    auto exponent_a = [&](int t, int b) { return (int)lds[kAtE + ((b >> 2) & 1) * G::kExps + ((wave >> 1) * 32 * TM + t * 32 + r) * 4 + (b & 3)]; };
    auto exponent_b = [&](int u, int b) { return (int)lds[kAtE + ((b >> 2) & 1) * G::kExps + (G::BM + row_b + u * 32) * 4 + (b & 3)]; };

    // in the order in which the loop would have issued them
    fetch_e(0, 0);
    fetch_e(0, 1);
#pragma unroll
    for (int n = 0; n < 8; ++n) fetch_a(n / 4, 0, n / 4, n & 3);
#pragma unroll
    for (int n = 0; n < 8; ++n) fetch_b(0, n);
#pragma unroll
    for (int n = 0; n < 4; ++n) fetch_a(2, 1, 0, n);
    fetch_e(1, 1);
#pragma unroll
    for (int n = 0; n < 4; ++n) fetch_a(3, 1, 1, n);
#pragma unroll
    for (int n = 0; n < 8; ++n) fetch_b(1, n);
#pragma unroll
    for (int n = 0; n < 4; ++n) fetch_a(4, 2, 0, n);
    fetch_e(1, 0);
    asm volatile("s_waitcnt vmcnt(22)\n\ts_barrier" : : : "memory");
    i32x8 fa[2][2], fb[TN][2];
    int ea[TM], eb[TN];
#pragma unroll
    for (int k = 0; k < 2; ++k) fa[0][k] = read_a(0, 0, k);
#pragma unroll
    for (int u = 0; u < TN; ++u) {
#pragma unroll
        for (int k = 0; k < 2; ++k) fb[u][k] = read_b(0, u, k);
        eb[u] = exponent_b(u, 0);
    }
#pragma unroll
    for (int t = 0; t < TM; ++t) ea[t] = exponent_a(t, 0);

    uint32_t slot = 0;                                                // of this block's rows 0 and 1
    auto behind = [](uint32_t s, uint32_t n) { return s + n >= kUnits ? s + n - kUnits : s + n; };
    for (int b = 0; b < blocks; ++b) {
        const int next = clamp(b + 1);
        const uint32_t slot1 = behind(slot, 1), slot2 = behind(slot, 2);
#pragma unroll
        for (int t = 0; t < TM; ++t) {
            if (t == 1) asm volatile("s_waitcnt vmcnt(30) lgkmcnt(0)\n\ts_barrier" : : : "memory");
            if (t == 3) asm volatile("s_waitcnt vmcnt(17) lgkmcnt(0)\n\ts_barrier" : : : "memory");
            WPSGD_IN_ORDER;
            if (t == 0) ea[3] = exponent_a(3, b);
#pragma unroll
            for (int u = 0; u < TN; ++u)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int i = u * 2 + k;
                    acc[t][u] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[u][k], fa[t & 1][k], acc[t][u], 0, 0, 0, eb[u], 0, ea[t]);
                    if (i == 1 || i == 2) fa[(t + 1) & 1][i - 1] = t == 3 ? read_a(slot2, 0, i - 1) : read_a(t == 0 ? slot : slot1, t + 1, i - 1);
                    if (t == 0 && i == 4) fetch_e((b >> 2) + 1, b & 1);
                    if (t == 1 && i < 6) {                            // four of A's rows 2 and 3, two blocks on (this block's rows 0 and 1 are read), then B
                        if (i < 4) fetch_a(slot, b + 2, 1, i);
                        else fetch_b(b + 2, i - 4);
                    }
                    if (t == 2 && i < 6) fetch_b(b + 2, i + 2);
                    if (t == 3) {
                        if (i >= 4) fetch_a(slot1, b + 3, 0, i - 4);
                        fb[u][k] = read_b(next, u, k);
                        if (k == 1) {
                            eb[u] = exponent_b(u, next);
                            if (u < 3) ea[u] = exponent_a(u, next);
                        }
                    }
                    WPSGD_IN_ORDER;
                }
        }
        slot = slot2;
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" : : : "memory");
    tile.template store<uint16_t>(g, acc, 1.0f, lds + wave * (32 * 32 * TN * 2));
}

// The parts of a split sum, added in their order and rounded once.
template <typename TO>
__global__ __launch_bounds__(256) void join_parts_kernel(const float *parts, int count, int64_t M, int64_t N, TO *out, int64_t ldo)
{
    const int64_t all = M * N;
    for (int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; at < all; at += (int64_t)gridDim.x * 1024) {
        float s[4] = {0, 0, 0, 0};
        const int n = (int)(all - at < 4 ? all - at : 4);
        for (int p = 0; p < count; ++p) {
            const float *from = parts + (int64_t)p * all + at;
            if (n == 4) {
                const Bytes16 q = load16(from);
#pragma unroll
                for (int j = 0; j < 4; ++j) s[j] += __uint_as_float(q.w[j]);
            } else {
                for (int j = 0; j < n; ++j) s[j] += from[j];
            }
        }
        const int64_t i = at / N, j = at - i * N;
        if (n == 4 && j + 4 <= N) {
            store4(out + i * ldo + j, f32x4{s[0], s[1], s[2], s[3]});
        } else {
            for (int q = 0; q < n; ++q) {
                const int64_t ii = (at + q) / N, jj = at + q - ii * N;
                Elem<TO>::put(out + ii * ldo + jj, s[q]);
            }
        }
    }
}

static size_t parts_bytes(const MatmulPlan &p, int64_t M, int64_t N) { return p.parts > 1 ? ((size_t)p.parts * M * N * sizeof(float) + 255) & ~(size_t)255 : 0; }

template <int MT, int NT, typename TO>
static hipError_t launch_rows_of(MatmulArgs g, bool turned, hipStream_t s)
{
    const int64_t many = turned ? g.M : g.N, few = turned ? g.N : g.M;
    const int64_t groups = (many + 16 * NT - 1) / (16 * NT), panels = (few + 16 * MT - 1) / (16 * MT);
    int along = 1;
    while (along < kRowWaves && along < kHeldBlocks / MT && groups * panels * along < 2048 && g.blocks >= 2 * along) along *= 2;
    const int64_t grid = (groups * along + kRowWaves - 1) / kRowWaves;
    if (many >= 1LL << 31 || panels > 65535) return hipErrorInvalidConfiguration;
    return in_launches(grid, 64 * kRowWaves, [&](int64_t first, unsigned count) {
        g.first = first;
        hipLaunchKernelGGL((matmul_rows_kernel<MT, NT, TO>), dim3(count, (unsigned)panels), dim3(64 * kRowWaves), 0, s, g, along, turned);
    });
}
template <typename TO>
static hipError_t launch_rows(const MatmulArgs &g, hipStream_t s)
{
    const RowsShape r = rows_shape(g.M, g.N);
    if (r.mt == 1) return launch_rows_of<1, 1, TO>(g, r.turned, s);
    if (r.mt == 2) return r.nt == 2 ? launch_rows_of<2, 2, TO>(g, r.turned, s) : launch_rows_of<2, 1, TO>(g, r.turned, s);
    return r.nt == 2 ? launch_rows_of<4, 2, TO>(g, r.turned, s) : launch_rows_of<4, 1, TO>(g, r.turned, s);
}

}  // namespace wpsgd

using namespace wpsgd;

extern "C" {

size_t wpsgd_block_matmul_workspace(int64_t rows_a, int64_t rows_b, int64_t cols)
{
    if (rows_a <= 0 || rows_b <= 0 || cols <= 0) return 0;
    // (whatever the results' type and sums)
    const int64_t blocks = (cols + 127) / 128;
    size_t most = 0;
    for (int f32 = 0; f32 < 2; ++f32)
        for (int sums = 0; sums < 2; ++sums) {
            const size_t one = parts_bytes(plan_matmul(rows_a, rows_b, blocks, f32 != 0, false, sums != 0), rows_a, rows_b);
            most = one > most ? one : most;
        }
    return most;
}

int wpsgd_block_matmul(const wpsgd_blocks *A, const wpsgd_blocks *B, void *out, int64_t ld_out, int dtype_and_sums, void *workspace, size_t workspace_bytes,
                       void *stream)
{
    int rc = check_blocks(A);
    if (rc == WPSGD_OK) rc = check_blocks(B);
    if (rc != WPSGD_OK) return rc;
    const int dtype = dtype_and_sums & ~WPSGD_FP32_SUMS;
    const bool sums = (dtype_and_sums & WPSGD_FP32_SUMS) != 0;
    if (A->cols != B->cols || (dtype != WPSGD_F32 && dtype != WPSGD_BF16)) return WPSGD_INVALID_ARG;
    if (A->rows == 0 || B->rows == 0) return WPSGD_OK;
    if (!out || ld_out < B->rows || (uintptr_t)out % (dtype == WPSGD_F32 ? 4 : 2) != 0) return WPSGD_INVALID_ARG;
    const size_t need = wpsgd_block_matmul_workspace(A->rows, B->rows, A->cols);
    if (need && (!workspace || (uintptr_t)workspace % 256 != 0)) return WPSGD_INVALID_ARG;
    if (workspace_bytes < need) return WPSGD_WORKSPACE_TOO_SMALL;
    MatmulArgs g{static_cast<const uint8_t *>(A->codes), static_cast<const uint8_t *>(B->codes), static_cast<const uint8_t *>(A->exps),
                 static_cast<const uint8_t *>(B->exps), A->ld, B->ld, A->ld_exps, B->ld_exps, A->rows, B->rows, (int)((A->cols + 127) / 128), out, ld_out, 0, 0};
    const bool f32 = dtype == WPSGD_F32;
    const MatmulPlan p = plan_matmul(g.M, g.N, g.blocks, f32, wide(g.lda, g.lde_a) || wide(g.ldb, g.lde_b), sums);
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e = hipSuccess;
    if (p.kind == MatmulPlan::Rows) {
        e = f32 ? launch_rows<float>(g, s) : launch_rows<uint16_t>(g, s);
        if (e == hipErrorInvalidConfiguration) return WPSGD_UNSUPPORTED;     // more rows than the header takes
    } else {
        const int64_t side = p.kind == MatmulPlan::Tile128 ? 128 : 256;
        const int64_t tiles = ((g.M + side - 1) / side) * ((g.N + side - 1) / side);
        if (tiles > most_groups(256)) return WPSGD_UNSUPPORTED;
        g.each = p.each;
        const dim3 grid((unsigned)tiles), block(256);
        if (p.kind == MatmulPlan::Fast256) {
            hipLaunchKernelGGL(matmul_fast_kernel, grid, block, 0, s, g);
        } else if (p.kind == MatmulPlan::Tile256) {
            if (f32) hipLaunchKernelGGL((matmul_tile_kernel<4, 4, float>), grid, block, 0, s, g);
            else hipLaunchKernelGGL((matmul_tile_kernel<4, 4, uint16_t>), grid, block, 0, s, g);
        } else if (p.parts == 1) {
            if (f32) hipLaunchKernelGGL((matmul_tile_kernel<2, 2, float>), grid, block, 0, s, g);
            else hipLaunchKernelGGL((matmul_tile_kernel<2, 2, uint16_t>), grid, block, 0, s, g);
        } else {
            if (p.parts > 1) {
                MatmulArgs part = g;
                part.out = workspace;
                part.ldo = g.N;
                hipLaunchKernelGGL((matmul_tile_kernel<2, 2, float>), dim3((unsigned)tiles, (unsigned)p.parts), block, 0, s, part);
                e = hipGetLastError();
                if (e != hipSuccess) return hip_fail(e);
            }
            const int64_t quads = (g.M * g.N + 3) / 4, groups = (quads + 255) / 256;
            const dim3 join((unsigned)(groups < 2048 ? groups : 2048));
            if (f32) hipLaunchKernelGGL(join_parts_kernel<float>, join, block, 0, s, static_cast<const float *>(workspace), p.parts, g.M, g.N, static_cast<float *>(out), ld_out);
            else hipLaunchKernelGGL(join_parts_kernel<uint16_t>, join, block, 0, s, static_cast<const float *>(workspace), p.parts, g.M, g.N, static_cast<uint16_t *>(out), ld_out);
        }
        e = hipGetLastError();
    }
    return e == hipSuccess ? WPSGD_OK : hip_fail(e);
}

}  // extern "C"
