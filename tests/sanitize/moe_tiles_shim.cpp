// The experts' tiles (csrc/moe_tiles.h) as plain C calls, for tests/test_moe_tiles.py (built by g++, no device code).
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

}  // extern "C"
