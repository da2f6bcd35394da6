// Rows of a few tokens times packed 4-bit matrices, the rows as they are.
//
//   y[r, n] = sum_k x[row, k] W_e[n, k]
//
// What bounds it is the reading of W: 17/32 of a byte an element.  A lane takes one block of a row of W, 16 bytes and a scale, and the conversion makes
// 32 bf16 numbers of it, which have room for the sign, the two bits and the scale: no rounding.  x is written as a sum of bf16 numbers
// (one for bf16, two for f16's 11 bits, three for f32's 24), each a row of its own for the matrix instruction, whose 16 rows
// would stand empty otherwise; so all products are exact and a single row of f32 costs no more instructions than one of bf16.
//
// The rows of the instruction that x leaves empty take other columns: with SHARES of them to a row of x, each multiplies its own share of the columns, and 16 / SHARES rows of W take
// the instruction's 16 columns, so 16 lanes read 64 bytes of each of four rows (SHARES 4) and not 16 bytes of each of 16: the lines that a load
// touches bounded the kernel before, 65536 x 4096 35 us and 25 so.
//
// Measured in graphs of 32 calls: one row x 4096 x 4096 bf16 4.8 us, of which a launch is 2.3 and the bytes 1.4; 8192 x 8192 11.3 us, 65536 x 4096 25 us = 5.7 TB/s; 12 tokens x 4 of
// 64 experts of 1411 x 2049 f32 15.5 us for 45 MB: a workgroup finds its rows by three trips to memory, then waits for 140 KB of W, and a CU has two.
//
// A wave owns 16 rows of W and takes units of 256 or 512 columns; the waves of a workgroup share the units among them, and their sums are added
// in order.  The rows of x go to LDS once, split; long rows of many tokens in pieces, a workgroup each.
#include "qesgd_experts.h"
#include "qesgd_groups.h"
#include "qesgd_launch.h"
#include "qesgd_mx4_codes.h"

namespace qesgd {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float acc4 __attribute__((ext_vector_type(4)));

struct VParams {
    const void* x;
    uint64_t ld;
    uint32_t T;
    const int32_t* order;
    uint32_t per, per_factor, per_shift;
    const unsigned char* w;
    uint64_t w_stride, scales_off;
    const int32_t* offsets;
    uint32_t E, R, N, K;
    uint32_t row_codes, row_scales;
    void* y;
    uint64_t ldy;
    bool wide;                        // y is fp32, whatever x is
    uint32_t splits;                  // waves that share a row's columns: 1 .. kVWaves
    uint32_t room;                    // bytes of LDS for rows of x
    uint32_t pieces;                  // of the columns, a workgroup each; with more than one the sums go to partial [pieces, R, N]
    float* partial;
};

constexpr uint32_t kVLoads = 4;           // loads that a wave has on their way at a time, twice

// bf16 numbers that hold an element.
constexpr uint32_t parts_of(uint32_t dtype) { return dtype == QESGD_F32 ? 3 : dtype == QESGD_F16 ? 2 : 1; }

// The upper 16 bits of v: a bf16 number no larger than v, so that nothing overflows.
__device__ __forceinline__ uint32_t upper(float v) { return __float_as_uint(v) & 0xFFFF0000u; }

// An element as PARTS bf16 numbers, each in the upper half of a word, the largest part first.  Infinities and NaN are whole in the first one.
template <uint32_t DT, uint32_t PARTS>
__device__ __forceinline__ void split_one(float x, uint32_t (&part)[PARTS]) {
    if constexpr (PARTS == 1) {
        part[0] = __float_as_uint(x);                          // is one already
    } else {
        const bool fine = (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u;
        float v = x;
#pragma unroll
        for (uint32_t q = 0; q < PARTS; ++q) {
            part[q] = upper(v);
            v = fine ? v - __uint_as_float(part[q]) : 0.0f;
        }
        part[0] = x != x ? 0x7FC00000u : part[0];
    }
}

// Eight elements as PARTS times eight bf16 numbers.
template <uint32_t DT, uint32_t PARTS>
__device__ __forceinline__ void split(const Eight<DT>& x, uvec4 (&out)[PARTS]) {
    if constexpr (DT == QESGD_BF16) {
        out[0] = x.v;
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            uint32_t low[PARTS], high[PARTS];
            split_one<DT, PARTS>(x.at(2 * i), low);
            split_one<DT, PARTS>(x.at(2 * i + 1), high);
#pragma unroll
            for (uint32_t q = 0; q < PARTS; ++q) out[q][i] = low[q] >> 16 | high[q];
        }
    }
}

// The 32 bf16 numbers of a block as four operands of eight.
__device__ __forceinline__ void block_values(const uvec4& codes, uint32_t byte, bf16x8 (&out)[4]) {
    const float scale = __uint_as_float(byte << 23);              // the conversion reads the exponent field; 255 gives NaN
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t c = codes[i];
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1);
        const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2), e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3);
        out[i] = bf16x8{a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
    }
}

// TILES of 16 rows of the instruction, SHARES of which are one number of each element of a row of x: ROWS at a time.
// Four waves on a SIMD: two workgroups of 8 waves on a CU, which the compiler would not have registers for otherwise.
template <uint32_t DT, uint32_t TILES, uint32_t SHARES, uint32_t kVWaves>
__global__ void __launch_bounds__(kVWaves * 64, 4) k_mx4_vector_product(const VParams p) {
    constexpr uint32_t PARTS = parts_of(DT), KEPT = TILES * 16 / SHARES, ROWS = KEPT / PARTS, GROUP = 16 / SHARES;
    // a unit: 16 rows of W x 256 or 512 columns, in LOADS loads; BATCH units on their way
    constexpr uint32_t LOADS = SHARES < 2 ? 2 : SHARES, BATCH = kVLoads / LOADS, UNIT = LOADS * 128;
    extern __shared__ __attribute__((aligned(16))) unsigned char rows_lds[];            // rows of part_columns bf16 and 16 bytes
    __shared__ float sums[kVWaves][KEPT][16];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t l = lane & 15u, block = lane >> 4, piece = blockIdx.z;
    const uint32_t share = wave % p.splits, n0 = (blockIdx.x * (kVWaves / p.splits) + wave / p.splits) * 16u;
    // the wave's first row of W, and the scales (sixteen bytes of codes each) before the lane's row in load i of a unit
    const uint32_t row0 = min(n0, p.N - 1u);
    uint32_t before[SHARES];
#pragma unroll
    for (uint32_t i = 0; i < SHARES; ++i) before[i] = min(i * GROUP + l / SHARES, p.N - 1u - row0) * p.row_scales;
    const uint32_t own = block * SHARES + l % SHARES, blocks = p.row_scales;
    const uint32_t units = (blocks * 32u + UNIT - 1u) / UNIT, begin = piece * units / p.pieces * UNIT, end = (piece + 1u) * units / p.pieces * UNIT;
    for (uint32_t tile = blockIdx.y;; tile += gridDim.y) {
        Group g{0, 0, p.R, 0};
        if (p.offsets ? !group_of_tile(p.offsets, p.E, p.R, Times<ROWS>{}, 1, tile, g) : tile * ROWS >= p.R) break;        // uniform
        const uint32_t r0 = g.lo + (tile - g.first) * ROWS, rows = min(ROWS, g.hi - r0);
        // as many columns of x at a time as there is room for, in whole units, and 16 bytes behind each row
        const uint32_t part_columns = min((p.room / (rows * PARTS) - 16u) / (2u * UNIT) * UNIT, end - begin), pitch = part_columns * 2u + 16u;
        const unsigned char* w = p.w + g.e * p.w_stride;
        const unsigned char *codes = w + (uint64_t)row0 * p.row_codes, *scales = w + p.scales_off + (uint64_t)row0 * p.row_scales;
        // blocks of units j, j + 1 .. of the wave's in a part of n units from unit `from` on; behind the row's end its last one, for which x has zeros
        const auto fetch = [&](uvec4 (&c)[kVLoads], uint32_t (&byte)[kVLoads], uint32_t from, uint32_t j, uint32_t n) {
#pragma unroll
            for (uint32_t q = 0; q < BATCH; ++q) {
                if (share + (j + q) * p.splits >= n) break;                // uniform
#pragma unroll
                for (uint32_t i = 0; i < LOADS; ++i) {
                    const uint32_t at = min((from + share + (j + q) * p.splits) * (UNIT / 32u) + (SHARES < 2 ? i * 4u : 0u) + own, blocks - 1u) + before[SHARES < 2 ? 0 : i];
                    c[q * LOADS + i] = *(const uvec4*)(codes + at * 16u);
                    byte[q * LOADS + i] = scales[at];
                }
            }
        };
        acc4 acc[TILES][SHARES];
#pragma unroll
        for (uint32_t m = 0; m < TILES; ++m)
#pragma unroll
            for (uint32_t i = 0; i < SHARES; ++i) acc[m][i] = acc4{0.0f, 0.0f, 0.0f, 0.0f};
        for (uint32_t c0 = begin; c0 < end; c0 += part_columns) {
            const uint32_t here = min(part_columns, end - c0), n = here / UNIT;
            // the wave's first blocks are on their way while the rows are brought in
            uvec4 c[kVLoads], next_c[kVLoads];
            uint32_t byte[kVLoads], next_byte[kVLoads];
            fetch(c, byte, c0 / UNIT, 0u, n);
            __syncthreads();
            // whole pieces of eight, some of a thread's on their way at a time, and by the last threads what is left of the rows and zeros behind them
            const uint32_t filled = p.K > c0 ? min(here, p.K - c0) : 0u, whole = filled / 8u;
            const auto source = [&](uint32_t r) {
                const int32_t pair = p.order ? p.order[r0 + r] : (int32_t)(r0 + r);
                return pair < 0 ? p.T : p.per == 1u ? (uint32_t)pair : __umulhi((uint32_t)pair, p.per_factor) >> p.per_shift;
            };
            const uint32_t behind = here / 8u - whole;
            for (uint32_t i = kVWaves * 64u - 1u - threadIdx.x; i < rows * behind; i += kVWaves * 64u) {
                const uint32_t r = i / behind, col = (whole + i - r * behind) * 8u, s = source(r), there = s < p.T && col < filled ? filled - col : 0u;
                Eight<DT> v;
                uvec4 parts[PARTS];
                v.load(p.x, there ? s * p.ld + c0 + col : 0u, there);
                split<DT, PARTS>(v, parts);
#pragma unroll
                for (uint32_t h = 0; h < PARTS; ++h) *(uvec4*)(rows_lds + (r * PARTS + h) * pitch + col * 2u) = parts[h];
            }
            constexpr uint32_t kPieces = kVWaves == 8 ? 1 : DT == QESGD_BF16 ? 4 : 2;
            for (uint32_t i0 = threadIdx.x; i0 < rows * whole; i0 += kPieces * kVWaves * 64u) {
                Eight<DT> v[kPieces];
                uint32_t to[kPieces];
#pragma unroll
                for (uint32_t q = 0; q < kPieces; ++q) {
                    const uint32_t i = i0 + q * (kVWaves * 64u);
                    if (i >= rows * whole) break;
                    const uint32_t r = i / whole, col = (i - r * whole) * 8u, s = source(r);
                    v[q].load_whole(p.x, s < p.T ? s * p.ld + c0 + col : 0u, s < p.T);
                    to[q] = r * PARTS * pitch + col * 2u;
                }
#pragma unroll
                for (uint32_t q = 0; q < kPieces; ++q) {
                    if (i0 + q * (kVWaves * 64u) >= rows * whole) break;
                    uvec4 parts[PARTS];
                    split<DT, PARTS>(v[q], parts);
#pragma unroll
                    for (uint32_t h = 0; h < PARTS; ++h) *(uvec4*)(rows_lds + to[q] + h * pitch) = parts[h];
                }
            }
            __syncthreads();
            // rows of the instruction beyond those there are read the last one: what comes of them is not stored
            const unsigned char* x[TILES];
#pragma unroll
            for (uint32_t m = 0; m < TILES; ++m) x[m] = rows_lds + min(m * GROUP + l / SHARES, rows * PARTS - 1u) * pitch + own * 64u;
            for (uint32_t j = 0; share + j * p.splits < n; j += BATCH) {
                fetch(next_c, next_byte, c0 / UNIT, j + BATCH, n);
#pragma unroll
                for (uint32_t q = 0; q < BATCH; ++q) {
                    const uint32_t unit = share + (j + q) * p.splits;
                    if (unit >= n) break;                              // uniform
#pragma unroll
                    for (uint32_t h = 0; h < (SHARES < 2 ? LOADS : 1u); ++h) {
                        bf16x8 a[TILES][4];
#pragma unroll
                        for (uint32_t m = 0; m < TILES; ++m)
#pragma unroll
                            for (int i = 0; i < 4; ++i) a[m][i] = *(const bf16x8*)(x[m] + unit * (UNIT * 2u) + h * 256u + i * 16u);
#pragma unroll
                        for (uint32_t s = 0; s < SHARES; ++s) {
                            bf16x8 b[4];
                            block_values(c[q * LOADS + (SHARES < 2 ? h : s)], byte[q * LOADS + (SHARES < 2 ? h : s)], b);
#pragma unroll
                            for (int i = 0; i < 4; ++i)
#pragma unroll
                                for (uint32_t m = 0; m < TILES; ++m) acc[m][s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[m][i], b[i], acc[m][s], 0, 0, 0);
                        }
                    }
                }
#pragma unroll
                for (uint32_t q = 0; q < kVLoads; ++q) {
                    c[q] = next_c[q];
                    byte[q] = next_byte[q];
                }
            }
        }
        // A lane holds column l and rows 4 block + i of a result, and counts where both have the same share of the columns.
#pragma unroll
        for (uint32_t m = 0; m < TILES; ++m)
#pragma unroll
            for (uint32_t s = 0; s < SHARES; ++s)
#pragma unroll
                for (uint32_t i = 0; i < 4; i += SHARES) {
                    float v = acc[m][s][i];
#pragma unroll
                    for (uint32_t k = 1; k < SHARES; ++k) v = l % SHARES == k ? acc[m][s][i + k] : v;
                    if (SHARES >= 2) v += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0xB1, 0xF, 0xF, false));
                    if (SHARES >= 4) v += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x4E, 0xF, 0xF, false));
                    if (l % SHARES == 0) sums[wave][m * GROUP + (4u * block + i) / SHARES][s * GROUP + l / SHARES] = v;
                }
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < (kVWaves / p.splits) * 16u * rows; i += kVWaves * 64u) {
            const uint32_t col = i & 15u, r = (i >> 4) % rows, set = (i >> 4) / rows;
            const uint32_t n = (blockIdx.x * (kVWaves / p.splits) + set) * 16u + col;
            if (n >= p.N) continue;
            float v = 0.0f;
#pragma unroll
            for (int q = PARTS - 1; q >= 0; --q) {
                const float* from = &sums[set * p.splits][r * PARTS + q][col];
                float part[kVWaves];
#pragma unroll
                for (uint32_t s = 0; s < kVWaves; ++s) part[s] = s < p.splits ? from[s * (KEPT * 16u)] : 0.0f;
#pragma unroll
                for (uint32_t s = 0; s < kVWaves; ++s) v += part[s];
            }
            if (p.pieces > 1) p.partial[((uint64_t)piece * p.R + r0 + r) * p.N + n] = v;
            else if (DT != QESGD_F32 && p.wide) ((float*)p.y)[(uint64_t)(r0 + r) * p.ldy + n] = v;
            else put<DT>(p.y, (uint64_t)(r0 + r) * p.ldy + n, v);
        }
    }
}

struct Plan {
    uint32_t waves, splits, tiles, lds_rows, room, pieces, blocks, row_tiles, shares;
};

constexpr uint64_t kVFits = 131072, kVPiece = 98304;      // bytes of split rows: as many as fit LDS, and a piece's

Plan plan_of(const VectorProduct& a, uint32_t dtype) {
    Plan p{};
    const uint32_t steps = (uint32_t)((a.K + 127) / 128), parts = parts_of(dtype), across_rows = (uint32_t)((a.N + 15) / 16);
    // experts that may be taken to have rows, and tiles of `at` rows that they may be taken to make
    const double groups = a.E > 1 ? (double)a.E * -__builtin_expm1(-(double)a.R / (double)a.E) : 1.0;
    const auto tiles_of = [&](uint32_t at) {
        if (a.E == 1) return (uint32_t)((a.R + at - 1) / at);
        const double even = ((double)a.R + 0.5 * (at - 1) * groups) / at, n = (groups > even ? groups : even) + 0.5;
        return n < 1.0 ? 1u : (uint32_t)n;
    };
    // Four rows of the instruction to a row of x, unless tiles of so few rows make more workgroups than the CUs have places, or reading W once for each is most of the work;
    // then two, while the rows of an expert fit into one tile so, or else one.  Us with 4 / 2 / 1, graph of 16 calls: one row x 4096 x 4096 bf16 5.0 / 5.4 / 5.7, 16 rows
    // 7.4 / 8.5 / 8.9, 4 rows f32 7.1 / 8.3 / 8.3; 8 tokens x 8 of 128 experts 512 x 2048 bf16 8.2 / 10.5 / 12.1; 4 x 2 of 8, 4096 x 4096 f32 12.7 / 16.9 / 19; but 12 x 4 of 64,
    // 1411 x 2049 f32 19.0 / 15.3 / 16.9, 16 rows x 8192 x 8192 f32 48 / 50 / 25 and bf16 20.7 / - / 18.4, 64 x 4 of 64, 1411 x 2049 bf16 36 / 32 / 39.
    constexpr uint64_t kVPlaces = 4096, kVWork = 128 << 10;               // waves, and units of 16 rows of W x 128 columns
    p.tiles = 1;
    p.shares = 4;
    const uint64_t few = (uint64_t)across_rows * tiles_of(parts > 2 ? 1 : 4 / parts);
    if (few > kVPlaces || few * ((steps + 3) / 4 * 4) >= kVWork) p.shares = (double)a.R * parts <= 8.5 * groups ? 2 : 1;
    // rows that an expert has at a time, of which two in three are in its share twice over
    const uint32_t rows = (uint32_t)(a.E == 1 ? a.R : (2 * a.R + a.E - 1) / a.E);
    while (p.shares == 1 && p.tiles < parts && p.tiles * 16 / parts < rows) ++p.tiles;
    const uint32_t at_a_time = p.tiles * (16 / p.shares) / parts, kept = (rows < at_a_time ? rows : at_a_time) * parts;
    const uint64_t all_bytes = (uint64_t)kept * steps * 256u;
    p.lds_rows = parts * (a.R < at_a_time ? (uint32_t)a.R : at_a_time);
    // at most
    const uint32_t hit = a.E < a.R ? a.E : (uint32_t)a.R, busy = tiles_of(at_a_time);
    p.row_tiles = (uint32_t)((a.R + (at_a_time - 1) * (uint64_t)hit) / at_a_time);
    // Workgroups of 8 waves, two or three on a CU, where there is little to bring into LDS, else of 16, which bring it in faster.  8 / 16 waves, us, graph of 32 calls: one row
    // x 4096 x 4096 bf16 5.5 / 5.8, f32 6.2 / 8.7, 8 tokens x 2 of 64 experts 1024 x 2048 bf16 20.6 / 25.3; 8 rows x 4096 x 4096 bf16 8.4 / 7.0, 4 rows f32 8.6 / 8.3.
    // And as many waves to a row of W as make kVWavesFew or kVWavesMany of them, beyond which each has more steps instead: 4 tokens x 2 of 8 experts 4096 x 4096 bf16 19.5
    // with one, 12.4 with two; 12 x 4 of 64, 1411 x 2049 f32 17.5 with one, 19.2 with two.
    constexpr uint32_t kVWavesFew = 1536, kVWavesMany = 4096;
    p.waves = all_bytes < 65536u ? 8 : 16;
    p.splits = 1;
    while (p.splits < p.waves && p.splits * (p.shares == 4 ? 8 : 4) <= steps + 1 && (uint64_t)across_rows * busy * p.splits < (p.waves == 8 ? kVWavesFew : kVWavesMany)) p.splits *= 2;
    // Rows that do not fit LDS at once, split by every workgroup, are most of the work.  Where waves share the columns anyway, workgroups share them instead, about 96 KB of
    // split rows to each, and a second launch adds their sums.  One piece / as chosen, us, graph of 32 calls: 16 rows x 4096 x 4096 f32 17.6 / 13.5 (4 pieces), 16 x 8192 x 8192
    // f32 40 / 28 and bf16 21 / 18 (4), 16 x 1000 x 8192 f32 30 / 18 (8), 4 x 4096 x 25088 bf16 21 / 19 (8).  Rows that fit gain nothing: 16 x 4096 x 4096 bf16 8.9 / 9.8 (2).
    p.pieces = 1;
    while (all_bytes > kVFits && all_bytes > kVPiece * p.pieces && p.splits >= 4) {
        p.pieces *= 2;
        p.splits /= 2;
    }
    const uint32_t across = 16u * (p.waves / p.splits);
    p.blocks = ((uint32_t)a.N + across - 1) / across;
    // the rows whole, where a CU has one workgroup anyway, or else as much of them as leaves room for two
    const bool alone = (uint64_t)p.blocks * busy * p.pieces <= 256;
    const uint32_t room = (alone ? 140u : 60u) * 1024u * p.waves / 16u - (alone ? p.tiles * 1024u / p.shares * p.waves : 0u);
    const uint32_t unit = p.shares == 4 ? 4 : 2, units = (steps + unit - 1) / unit;
    const uint64_t whole = (uint64_t)p.lds_rows * ((units + p.pieces - 1) / p.pieces * unit * 256u + 16u);
    p.room = whole < room ? (uint32_t)whole : room;
    const uint64_t most_tiles = (1u << 20) / ((uint64_t)p.blocks * p.pieces);        // a workgroup takes several where there are more
    if (p.row_tiles > most_tiles) p.row_tiles = (uint32_t)most_tiles;
    if (p.row_tiles > 65535) p.row_tiles = 65535;
    return p;
}

}  // namespace

// As much as the type that needs most: the type is not known where it is asked for.
size_t vector_product_workspace(const VectorProduct& a) {
    if ((a.R < 16 ? a.R : 16) * 3 * ((a.K + 127) / 128) * 256 <= kVFits) return 0;          // no type has more to bring in
    uint32_t pieces = 1;
    for (uint32_t t : {QESGD_F32, QESGD_BF16, QESGD_F16}) {
        const uint32_t n = plan_of(a, t).pieces;
        if (n > pieces) pieces = n;
    }
    return pieces > 1 ? pieces * a.R * a.N * sizeof(float) : 0;
}

int launch_vector_product(const VectorProduct& a) {
    qesgd_mx4_layout W;
    if (const int rc = make_mx4_layout(a.N, a.K, &W); rc != QESGD_OK) return rc;
    const Plan plan = plan_of(a, a.dtype);
    VParams p{};
    p.x = a.x;
    p.ld = a.ld;
    p.T = (uint32_t)a.T;
    p.order = a.order;
    p.per = a.per;
    divide_by(a.per, p.per_factor, p.per_shift);
    p.w = a.w;
    p.w_stride = a.w_stride;
    p.scales_off = W.scales_off;
    p.offsets = a.offsets;
    p.E = a.E;
    p.R = (uint32_t)a.R;
    p.N = (uint32_t)a.N;
    p.K = (uint32_t)a.K;
    p.row_codes = (uint32_t)W.row_codes;
    p.row_scales = (uint32_t)W.row_scales;
    p.y = a.y;
    p.ldy = a.ldy;
    p.wide = a.rows_dtype == QESGD_F32;
    p.splits = plan.splits;
    p.room = plan.room;
    p.pieces = plan.pieces;
    p.partial = a.workspace;
    const uint32_t bytes = plan.room, tiles = plan.tiles;
    const dim3 grid(plan.blocks, plan.row_tiles, plan.pieces);
    by_type(a.dtype, [&](auto t) {
        using std::integral_constant;
        constexpr uint32_t DT = t.value;
        const auto go = [&](auto m, auto s) {
            if (plan.waves == 16) k_mx4_vector_product<DT, m.value, s.value, 16><<<grid, 16 * 64, bytes, a.stream>>>(p);
            else k_mx4_vector_product<DT, m.value, s.value, 8><<<grid, 8 * 64, bytes, a.stream>>>(p);
        };
        const integral_constant<uint32_t, 1> one{};
        const integral_constant<uint32_t, 2> two{};
        const integral_constant<uint32_t, 4> four{};
        if (plan.shares == 4) go(one, four);
        else if (plan.shares == 2) go(one, two);
        else if (tiles == 1) go(one, one);
        else if (tiles == 2) go(integral_constant<uint32_t, parts_of(DT) >= 2 ? 2 : 1>{}, one);
        else go(integral_constant<uint32_t, parts_of(DT) >= 3 ? 3 : 1>{}, one);
    });
    const int rc = launched();
    if (rc != QESGD_OK || plan.pieces == 1) return rc;
    return launch_piece_sum(PieceSum{a.workspace, plan.pieces, a.R * a.N, a.offsets, a.E, p.R, p.N, a.y, a.ldy}, a.rows_dtype, a.stream);
}

}  // namespace qesgd
