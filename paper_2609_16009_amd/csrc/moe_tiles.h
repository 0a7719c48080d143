// How the experts' products cut an expert's rows into tiles: plain arithmetic, which a test runs on the CPU.
#pragma once

#include <cstdint>

namespace nmm {
namespace rows {

// The bytes from the first of `count` rows of x to the last one's chunk that k ends in; loads address a tile's rows by 32-bit
// offsets, of which those from 2^31 on mean nothing is there.
constexpr int64_t tile_bytes(int64_t count, int64_t ld, int64_t K) { return ((count - 1) * ld + (K + 7) / 8 * 8) * 2; }
constexpr bool in_reach(int64_t count, int64_t ld, int64_t K) { return tile_bytes(count, ld, K) < int64_t(1) << 31; }

// Rows of x a tile of a product with local matrices of N rows of K: 4, 8, 16 (rows_kernel), 64, 128 or 256 (wide_kernel).
// A token chooses an expert once, so few tokens say how many rows an expert has at most.  With more, tiles hold about twice
// the rows that experts have on average, so that nearly all read their weights once: 16 experts of 7168 and 2048, 16 rows
// each 249 us in tiles of 64 (257 of 128), 64 rows 293 in tiles of 128 (310 of 64), 128 rows 360 of 256 (393 of 128);
// 64 experts of 8 rows 916 in tiles of 16 (930 of 64).
// Small experts have shorter walks, whose starts and ends count: up to 1024 x 512 tiles of 64 whatever the rows (16 experts of 128 rows 35
// us, 47 in 256s, of 512 rows 81 and 92), and many of them up to 2048 x 1024 from 16 tokens on rather than tiles of 16 (64 experts of 1024 x 512,
// 8 rows 49 us and 68, 2 rows 45 and 59; of 2048 x 1024, 8 rows 158 and 169, 2 rows 138 both; 16 experts of 512 x 256, 16 rows 18.4 and
// 15.3; 8 tokens on 64 of them 24 and 19).
constexpr int tile_rows_of(int64_t K, int64_t N, int64_t tokens, int64_t pairs, int64_t experts, int64_t local) {
    const int64_t expert = K * N;
    const bool many_small = tokens >= 16 && expert <= int64_t(1) << 21 && expert >= (int64_t(1) << 23) / local;
    if (tokens <= 4) return 4;
    if (tokens <= 8) return 8;
    if (!many_small && (tokens <= 16 || pairs <= 10 * experts)) return 16;
    if (expert <= int64_t(1) << 19 || pairs <= 40 * experts) return 64;
    return pairs <= 96 * experts ? 128 : 256;
}

// The same where a tile's rows lie `ld` apart and are addressed from its first one: as many of them as are in reach.  (A matrix of the first
// product stays below 2^31 bytes, so ld is 2^26 at most and 8 rows always are.)
constexpr int tile_rows_in_reach(int64_t K, int64_t N, int64_t tokens, int64_t pairs, int64_t experts, int64_t local, int64_t ld) {
    int rows = tile_rows_of(K, N, tokens, pairs, experts, local);
    while (rows > 4 && !in_reach(pairs < rows ? pairs : rows, ld, K)) rows = rows == 64 ? 16 : rows / 2;
    return rows;
}

// The walk over the items of a launch: an item is a tile of an expert's rows and a block of columns.  offsets are not trusted: they
// are cut to [0, pairs], a count below zero is none, and tiles in all are cut to those that pairs in some order can fill.
constexpr int cut_offset(int offset, int pairs) {
    const int o = offset > 0 ? offset : 0;
    return o < pairs ? o : pairs;
}
constexpr int tiles_of(int first, int end, int tile) { return end > first ? int(unsigned(end - first + tile - 1) / unsigned(tile)) : 0; }
constexpr int most_tiles(int pairs, int tile, int local) { return pairs / tile + local; }

// The expert whose tile is the u-th: starts[e] <= u < starts[e + 1], u < starts[local].
constexpr int expert_of(const int* starts, int local, int u) {
    int lo = 0, hi = local;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (starts[mid] <= u) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Blocks of columns that an XCD takes: every eighth, or where K is cut into 2, 4 or 8 slices every fourth, second or all of them
// in one slice (xcd % ks).
constexpr int64_t blocks_of_xcd(int n_blocks, int ks) {
    const int share = 8 / ks;
    return (int64_t(n_blocks) + share - 1) / share;
}

// Item `rem` of an XCD's items of an expert that has `tiles` tiles: the row tiles over the same weight rows follow each other, so
// the second one of wide_kernel finds them in the XCD's L2 (16 experts of 512 rows, 7168 x 2048: 840 MB read where
// walks do not start apart, 738 of them W and, by each L2, h).  rows_kernel marks the weight's loads
// non-temporal, and a second tile reads four fifths of it or more from memory again (64 experts, two to four of them with 17 to 19 rows).
struct Place {
    int nb, m0;
};
constexpr Place place_of(int64_t rem, int tiles, int tile, int ks, int xcd) {
    const int nbi = static_cast<int>(rem / tiles);
    return {8 / ks * nbi + xcd / ks, static_cast<int>(rem - int64_t(nbi) * tiles) * tile};
}

}  // namespace rows
}  // namespace nmm
