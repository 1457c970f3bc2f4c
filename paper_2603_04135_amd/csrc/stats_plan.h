// Which kernels and tiles the token statistics, their gradient and the 8-bit product take. Plain C++: the choice needs no device.
#pragma once
#include <cstddef>
#include <cstdint>

namespace dppo {

constexpr int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Groups of rows of a tile of the vocabulary GEMM (see StatsPart).
constexpr int STATS_GROUPS = 2;
// Tile of the vocabulary GEMM, rows (vocabulary) x columns (tokens); FEW: the kernel for few tokens. All but the largest read the tokens' rows
// of H through a map.
enum LogitsTile { TILE_FEW = 0, TILE_128x96 = 1, TILE_128x128 = 2, TILE_256x192 = 3, TILE_256x256 = 4 };
constexpr int32_t FEW_TILE_TOKENS = 16, FEW_TILE_ROWS = 32, FEW_ROW_BYTES_BF16 = 8192, FEW_ROW_BYTES_I8 = 6144;
inline int32_t tile_rows(int tile) { return tile == TILE_FEW ? FEW_TILE_ROWS : tile <= TILE_128x128 ? 128 : 256; }
// Rows of a group of a tile (see StatsPart).
inline int32_t group_rows(int tile) { return tile == TILE_FEW ? FEW_TILE_ROWS : tile_rows(tile) / STATS_GROUPS; }
// Groups of all tiles (the last may lie behind the vocabulary).
inline int32_t groups_of_tiles(int tile, int32_t V) { return (int32_t)div_up(V, tile_rows(tile)) * (tile == TILE_FEW ? 1 : STATS_GROUPS); }
// For n tokens with operand rows of 2 k2 bytes. Up to 16 tokens: rows of up to 8 KB (8-bit operands 6 KB) are what the registers of the
// kernel for few tokens hold. Up to 128 tokens as for the log-probabilities alone (see CfgFew; by 128 columns where every tile has a compute
// unit to itself). Beyond, the tile whose rounds of the chip
// take the least time, 256 x 256 : 256 x 192 : two of 128 x 128 as 20 : 18 : 15, the last while large tiles fill no more than two rounds.
// Statistics, 256 x 256 / 256 x 192 / 128 x 128, with the rounds of each: D = 1024, V = 32000: 224 tokens (1/1/1) 30 / 29 / 22 us, 384
// (1/1/2) 34 / 29 / 34, 512 (1/2/2) 35 / 44 / 37, 576 (2/2/3) 54 / 44 / 48, 768 (2/2/3) 55 / 48 / 52, 1024 (2/3/4) 61 / 72 / 72, 1152
// (3/3/5) 82 / 70 / 80; D = 4096, V = 60000: 224 (1/2/2) 144 / 163 / 157, 576 (3/3/5) 255 / 233 / 294, 1152 (5/6/9) 430 / 435 / 523;
// D = 2560, V = 151936: 192 (3/3/10) 216 / 201 / 244, 384 (5/5/14) 297 / 287 / 335, 640 (7/10/-) 423 / 496 / 530.
constexpr int64_t SMALL_TILES_MOST = 512;
inline int logits_tile(int32_t n, int32_t V, int32_t k2, bool i8) {
    if (n <= FEW_TILE_TOKENS && 2 * k2 <= (i8 ? FEW_ROW_BYTES_I8 : FEW_ROW_BYTES_BF16)) return TILE_FEW;
    constexpr int64_t CHIP = 256;                 // compute units
    if (n <= 96 && div_up(V, 128) > CHIP) return TILE_128x96;
    if (n <= 128) return TILE_128x128;
    const int64_t rows = div_up(V, 256), large = rows * div_up(n, 256);
    const int64_t t256 = 20 * div_up(large, CHIP), t192 = 18 * div_up(rows * div_up(n, 192), CHIP);
    const int64_t t128 = 15 * div_up(div_up(V, 128) * div_up(n, 128), 2 * CHIP);
    if (large <= SMALL_TILES_MOST && t128 < t256 && t128 < t192) return TILE_128x128;
    return t192 < t256 ? TILE_256x192 : TILE_256x256;
}
// Most pairs of (tile, token) that 128 x 128 tiles beyond 128 tokens make.
constexpr size_t SMALL_TILE_PAIRS = 2 * SMALL_TILES_MOST * 256;
// Tiles of 128 x 128 by eight wavefronts instead of four where no more than one workgroup runs on a compute unit (the reads of four from LDS show),
// or few slices leave prologue and statistics most of the time. D = 512, statistics, four / eight: V = 5000, 128 tokens (40 tiles) 8.3 / 6.7 us
// (8-bit product), V = 32000 (250) 12.4 / 10.8, 256 tokens (500) 15.1 / 14.4; D = 2560, V = 151936, 128 tokens 188 / 208; 8-bit product D = 4096,
// V = 32000: 128 tokens (250) 28.1 / 26.3, 256 (500) 37 / 42.
inline bool eight_wavefronts(int32_t n, int32_t V, int32_t k2) {
    const int64_t tiles = div_up(V, 128) * div_up(n, 128);
    return tiles <= 256 || (k2 <= 512 && tiles < (int64_t)1 << 23);       // (2^23 tiles of 512 threads are more than a launch has)
}

// Tokens that a workgroup joins: the more, the more of them read the maxima side by side; the fewer, the more workgroups. us with 4 / 8 / 16, 20
// alternatives: V = 151936, 400 tokens 21.3 / 22.1 / 26.5, 512 22.7 / 22.3 / 26.4, 1000 27.2 / 23.6 / 27.4, 2048 57 / 30.1 / 28.8, 2500 72 / 53 / 34,
// 8000 208 / 122 / 86; V = 32000, 512 15.5 / 15.9 / 18.3, 700 16.2 / 16.3 / 18.4, 1000 17.2 / 16.5 / 18.3, 2048 33 / 19.2 / 19.0; none: V = 151936, 400
// 6.7 / 6.4 / 7.2, 1000 12.5 / 8.0 / 8.2.
constexpr int JOIN_ALONE = 256;                   // (a token's groups lie side by side up to here, see StatsPart)
inline int join_tokens(int32_t n) { return n <= JOIN_ALONE ? 1 : n <= 512 ? 4 : n <= 2048 ? 8 : 16; }

// Whether the gradient goes by tiles of 128 x 128 (see SmallGrad): problems that large ones leave much of the chip idle in. One chunk, no more than a
// chip of large tiles of entries, and of dW few (or next to no sum to each). Large tiles / these: D = 512,
// V = 5000: 60 tokens 44 / 30 us, 1000 80 / 58; D = 2560, V = 3000: 60 68 / 52, 2500 193 / 149; D = 256, V = 20000: 300 68 / 52; D = 1024, V =
// 12000 (188 large tiles of dW): 600 99 / 84, 750 104 / 107; V = 32000 (500): 60 77 / 74, 500 135 / 150.
inline bool small_grad(int64_t N, int32_t D, int32_t V) {
    return div_up(V, 256) * div_up(N, 256) <= 256 && (N <= 64 || div_up(V, 256) * div_up(D, 256) <= 192);
}
// Parts along K of a GEMM of few tiles of 128 x 128: least estimated time of a slice's 0.45 us, 0.033 a partial tile (64 KB written and
// read) and 4 for the launch that sums them. Two workgroups a compute unit, 4 slices or more each.
constexpr int SMALL_PARTS_MOST = 2 * 256;         // partial tiles: 32 MB
inline int small_tiles_parts(int cus, int tiles, int slices) {
    const int slots = 2 * cus < SMALL_PARTS_MOST ? 2 * cus : SMALL_PARTS_MOST;
    int best = 1;
    double best_t = 0.45 * slices * (double)((tiles + slots - 1) / slots);
    for (int p = 2; p <= slices / 4 && tiles * p <= slots; ++p) {
        const double t = 0.45 * ((slices + p - 1) / p) + 4.0 + 0.033 * tiles * p;
        if (t < best_t) { best_t = t; best = p; }
    }
    return best;
}

}  // namespace dppo
