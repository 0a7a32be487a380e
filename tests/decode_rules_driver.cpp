// The launch rules of decoding behind C names, for tests/test_host_decode.py.
#include "kv_launch_rules.hpp"

extern "C" int64_t attend_groups(int64_t pairs, int64_t tokens, int head_dim) { return kvs::attend_groups(pairs, tokens, head_dim); }

extern "C" int64_t evict_blocks(int64_t pairs, int64_t list, int64_t rows) { return kvs::evict_blocks(pairs, list, rows); }

extern "C" int64_t append_pieces(int64_t n_rows, int pieces) { return kvs::append_pieces_per_lane(n_rows, pieces); }
