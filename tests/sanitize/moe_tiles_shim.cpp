// The experts' tiles (csrc/moe_tiles.h) as plain C calls, for tests/test_moe_tiles.py (built by g++, no device code).
#include <algorithm>
#include <vector>

#include "moe_tiles.h"

using namespace nmm::rows;

extern "C" {

int tile_rows(int64_t K, int64_t N, int64_t tokens, int64_t pairs, int64_t experts, int64_t local) {
    return tile_rows_of(K, N, tokens, pairs, experts, local);
}

int tile_rows_near(int64_t K, int64_t N, int64_t tokens, int64_t pairs, int64_t experts, int64_t local, int64_t ld) {
    return tile_rows_in_reach(K, N, tokens, pairs, experts, local, ld);
}

int64_t bytes_of_tile(int64_t count, int64_t ld, int64_t K) { return tile_bytes(count, ld, K); }

// The walk of a launch of `grid` workgroups over `pairs` pairs of `local` experts in tiles of `tile` rows and n_blocks blocks of columns:
// seen[place of a pair * n_blocks + block] counts how often a workgroup takes it.  Returns the tiles walked; -1: a row outside
// the pairs, -2: a tile without rows or with too many, -3: an item of no expert.
int64_t walk(const int* offsets, int local, int pairs, int tile, int n_blocks, int grid, int* seen) {
    std::vector<int> starts(local + 1, 0);
    const int most = most_tiles(pairs, tile, local);
    for (int e = 0; e < local; ++e)
        starts[e + 1] = std::min(starts[e] + tiles_of(cut_offset(offsets[e], pairs), cut_offset(offsets[e + 1], pairs), tile), most);
    const int64_t blocks = blocks_of_xcd(n_blocks, 1), total = starts[local] * blocks;
    for (int b = 0; b < grid; ++b)
        for (int64_t idx = b >> 3; idx < total; idx += grid >> 3) {
            const int u = int(idx / blocks), e = expert_of(starts.data(), local, u);
            if (e < 0 || e >= local || starts[e] > u || u >= starts[e + 1]) return -3;
            const Place at = place_of(idx - starts[e] * blocks, starts[e + 1] - starts[e], tile, 1, b & 7);
            if (at.nb >= n_blocks) continue;
            const int first = cut_offset(offsets[e], pairs), rows = std::min(tile, cut_offset(offsets[e + 1], pairs) - first - at.m0);
            if (at.nb < 0 || rows < 1 || rows > tile) return -2;
            if (first + at.m0 < 0 || first + at.m0 + rows > pairs) return -1;
            for (int r = 0; r < rows; ++r) ++seen[int64_t(first + at.m0 + r) * n_blocks + at.nb];
        }
    return starts[local];
}

// A dense product's: seen[(row * n_blocks + block) * ks + slice of K].
int walk_dense(int rows, int tile, int n_blocks, int ks, int grid, int* seen) {
    const int tiles = (rows + tile - 1) / tile;
    const int64_t total = tiles * blocks_of_xcd(n_blocks, ks);
    for (int b = 0; b < grid; ++b)
        for (int64_t idx = b >> 3; idx < total; idx += grid >> 3) {
            const Place at = place_of(idx, tiles, tile, ks, b & 7);
            if (at.nb >= n_blocks) continue;
            if (at.nb < 0 || at.m0 < 0 || at.m0 >= rows) return -1;
            for (int r = at.m0; r < std::min(rows, at.m0 + tile); ++r) ++seen[(int64_t(r) * n_blocks + at.nb) * ks + (b & 7) % ks];
        }
    return 0;
}

}  // extern "C"
