// Which kernel a product of 8-bit blocks takes, by sizes and the results' type alone.  No device code.
#pragma once

#include <stdint.h>

namespace wpsgd {

// Which kernel, by sizes and the results' type alone.  Few rows: the one that reads the others once.  Else the one that should take the least time (us, measured for 1024 x 1024
// to 16384 x 4096 results and 4 to 64 blocks of the sum): a round of tiles on all compute units takes 0.98 a block for 128 x 128 (two workgroups to a unit, so that
// one's products hide the other's loads and results), 2.2 for 256 x 256 with fp32 sums and 1.09 in the 8-bit instruction (one to a unit, results not
// hidden).  4096 x 4096, 8 blocks: fp32 41 | 38 (128 | 256), bfloat16 43 | 26; 5003 x 3001, 8 blocks, fp32: 38 | 42; 2048 x 2048, 64 blocks: 64 | 80 (8-bit).
struct MatmulPlan {
    enum { Rows, Tile128, Tile256, Fast256 } kind;
    int parts, each;           // Tile128: parts of the sum and blocks to each
};
// f32: results in fp32, whose sums are, too; f32_sums: the sums of bfloat16 results as well
inline MatmulPlan plan_matmul(int64_t M, int64_t N, int64_t blocks, bool f32, bool wide_rows, bool f32_sums = false)
{
    f32_sums = f32_sums || f32;
    const int64_t few = M < N ? M : N;
    if (few <= 64 || wide_rows) return {MatmulPlan::Rows, 1, 0};
    if (blocks == 0) return {MatmulPlan::Tile128, 0, 0};                      // a sum over nothing
    const int64_t t256 = ((M + 255) / 256) * ((N + 255) / 256), t128 = ((M + 127) / 128) * ((N + 127) / 128);
    int parts = 1;
    while (t128 * parts < 256 && blocks >= parts * 16) parts *= 2;           // eight blocks to a part at least
    const int each = parts == 1 ? (int)blocks : (int)(((blocks + parts - 1) / parts + 3) / 4 * 4);
    parts = (int)((blocks + each - 1) / each);
    const double out = (double)M * (double)N * (f32 ? 4.0 : 2.0) / 4.6e6;    // to write the results
    const auto rounds = [](int64_t tiles) { return tiles < 256 ? 1.0 : (double)tiles / 256.0; };
    const double by128 = 5.0 + 0.98 * each * rounds(t128 * parts) + 0.5 * out + (parts > 1 ? 4.0 : 0.0);
    const double by256 = (f32_sums ? 13.0 + 2.2 * (double)blocks * rounds(t256) : 10.0 + 1.09 * (double)blocks * rounds(t256)) + out;
    if (by256 < by128) return {f32_sums ? MatmulPlan::Tile256 : MatmulPlan::Fast256, 1, (int)blocks};
    return {MatmulPlan::Tile128, parts, each};
}

// Few rows against many: the few in sixteens beside each other (mt), the sixteens of the many to a wave (nt); turned: the many rows are A's.
struct RowsShape {
    int mt, nt;
    bool turned;
};
inline RowsShape rows_shape(int64_t M, int64_t N)
{
    const bool turned = M > N;
    const int64_t many = turned ? M : N, few = turned ? N : M;
    // too few rows for the compute units: the few rows in sixteens beside each other, too (64 x 1000 x 4096: 28 us without that)
    const int mt = few <= 16 || many <= 2048 ? 1 : few <= 32 ? 2 : 4;
    // Two sixteens of the many share what is read of the few from LDS, and leave half the waves. us, one | two, sums of 4096, the many out of the caches:
    //   16 x 65536 66 | 71, x 131072 124 | 130, x 262144 243 | 251      32 x 65536 73 | 77, x 98304 108 | 123, x 131072 142 | 140, x 262144 273 | 261
    //   64 x 49152 84 | 88, x 65536 90 | 85, x 98304 134 | 140, x 131072 174 | 154, x 262144 333 | 291
    return {mt, mt > 1 && many * mt >= 1 << 18 ? 2 : 1, turned};
}

// rows of a tile are addressed with 32 bits
inline bool wide(int64_t ld, int64_t ld_exps) { return ld > (1LL << 22) || ld_exps > (1LL << 22); }

}  // namespace wpsgd
