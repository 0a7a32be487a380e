// How attention over pages divides its work, behind a C name, for tests/division_cases.py: the sums that the kernel takes over the
// sequences, and the rule on them.
#include "kv_launch_rules.hpp"

extern "C" int32_t attend_round(int32_t n_seqs, const int32_t* len, const int32_t* rows, int32_t n_kv_heads, int32_t per, int32_t max_rows,
                                int32_t n_tokens, int32_t head_dim, int32_t* run) {
    const int64_t row_tiles = (per * max_rows + 15) / 16;
    const int32_t step = kvs::attend_step(head_dim);
    const int32_t groups = static_cast<int32_t>(kvs::attend_groups(n_seqs * n_kv_heads * row_tiles, n_tokens, head_dim));
    int32_t one = 0, two = 0, line = 0;
    for (int32_t s = 0; s < n_seqs; ++s) {
        const int32_t units = (len[s] + 31) / 32, pairs = n_kv_heads * ((std::min(rows[s], max_rows) * per + 15) / 16);
        one += pairs * kvs::attend_places(units, step, 0);
        two += pairs * kvs::attend_places(units, 2 * step, 0);
        line += pairs * kvs::attend_places(units, 1, kvs::kPieceCost);
    }
    const kvs::AttendDivision d = kvs::attend_division(one, two, line, groups, step);
    *run = d.run;
    return d.round;
}
