// How attention to latent caches divides its work, behind C names, for tests/test_latent_division.py: the functions that the kernels call.
#include "kv_launch_rules.hpp"

extern "C" int32_t latent_run(int32_t units, int32_t pairs, int32_t groups) { return kvs::latent_run(units, pairs, groups); }
extern "C" int32_t latent_groups(int64_t pairs, int64_t tokens) { return kvs::latent_groups(pairs, tokens); }
extern "C" int32_t latent_places(int32_t units) { return kvs::latent_places(units); }
extern "C" void latent_piece(int32_t at, int32_t run_end, int32_t s_end, int32_t units, int32_t row_tiles, int32_t* piece) {
    const kvs::LatentPiece p = kvs::latent_piece(at, run_end, s_end, units, row_tiles);
    piece[0] = p.row_tile;
    piece[1] = p.begin;
    piece[2] = p.end;
    piece[3] = p.places;
}
extern "C" int64_t latent_slot(int32_t workgroup, int32_t s, int32_t row_tile, int32_t most_row_tiles) {
    return kvs::latent_slot(workgroup, s, row_tile, most_row_tiles);
}
extern "C" void latent_shares(int32_t s_end, int32_t units, int32_t row_tile, int32_t row_tiles, int32_t run, int32_t* shares) {
    const kvs::LatentShares x = kvs::latent_shares(s_end, units, row_tile, row_tiles, run);
    shares[0] = x.first;
    shares[1] = x.count;
}
