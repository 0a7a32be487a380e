// Latent caches: append, read, and attention in the absorbed and the expanded form.  Argument checks on the host, then launches on the
// caller's stream; nothing here synchronises or allocates.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "kv_decode_checks.hpp"
#include "kv_launch_rules.hpp"
#include "kv_latent_pages.hpp"
#include "kv_latent_attend_kernels.hpp"
#include "kv_latent_prompt_kernels.hpp"

using namespace kvs;

namespace {

int check_latent_pages(const kv_latent_shape_t* shape, const kv_pages_t* pages, int32_t layer) {
    if (int rc = check_latent_shape(shape)) return rc;
    if (int rc = check_page_table(pages, shape->n_tokens / shape->chunk_tokens)) return rc;
    return layer < 0 || layer >= shape->n_layers ? fail(KV_EINVAL, "layer %d outside [0,%d)", layer, shape->n_layers) : KV_OK;
}

LatentView latent_view(const kv_latent_shape_t& s, const kv_pages_t& p, int32_t layer) {
    LatentView v = {};
    v.p.pool = static_cast<uint8_t*>(p.pool);
    v.p.off = p.off;
    v.p.bits = p.bits;
    v.p.len = p.len;
    v.p.n_seqs = p.n_seqs;
    v.p.stride = p.stride;
    v.p.N = s.n_tokens;
    v.p.T = s.chunk_tokens;
    v.p.slabs = s.n_layers;
    v.p.groups = s.latent_dim / s.group;
    v.p.half_params = s.format == KV_FMT_F16_GROUPS_H ? 1 : 0;
    const uint32_t d = static_cast<uint32_t>(s.chunk_tokens) / 16;
    v.p.page_of_tile = d == 1 ? 0u : static_cast<uint32_t>(((1ull << 32) + d - 1) / d);
    v.p.pool_bytes = p.pool_bytes;
    v.p.bit_bytes = static_cast<uint64_t>(s.n_layers) * s.chunk_tokens * s.latent_dim / 8;
    v.p.param_bytes = latent_param_bytes(s);
    v.rope_bytes = static_cast<uint64_t>(s.n_layers) * s.chunk_tokens * s.rope_dim * 2;
    v.Dr = s.rope_dim;
    v.layer = layer;
    return v;
}

uint64_t up256(uint64_t x) { return (x + 255) & ~255ull; }

// The rows that append reads and read writes.
int check_moved_rows(const kv_latent_shape_t* shape, const kv_pages_t* pages, int32_t n_rows, const int32_t* row_start, const void* c,
                     int64_t c_stride, const void* r, int64_t r_stride) {
    if (int rc = check_rows(pages, n_rows, row_start, c_stride, shape->latent_dim)) return rc;
    if (int rc = check_rows(pages, n_rows, row_start, r_stride, shape->rope_dim)) return rc;
    if (n_rows == 0) return KV_OK;
    if (!c || !r) return fail(KV_EINVAL, "NULL device pointer");
    if (!aligned(c, 16) || !aligned(r, 16)) return fail(KV_EINVAL, "c and r must be 16-byte aligned");
    return KV_OK;
}

double latent_scale(const kv_latent_shape_t& s) { return 1.4426950408889634 / std::sqrt(static_cast<double>(s.key_dim + s.rope_dim)); }

// Query rows of a tile: the fewest that hold a sequence's, since the products and the probabilities of rows that are not there take their time: 64
// rows of 8 contexts 25.9 us, in tiles of 128 38.7; 40 rows of one 8.7 and 10.7; 32 rows of 24 contexts 38.8, in tiles of 64 41.1.  Of more
// rows than 128, three tiles of 64 take as long as two of 128 less a tenth (a tile of 64 six tenths of one of 128): 160 rows of 16 contexts 27.3 us
// and 31.5, 128 rows of 16 long ones 266 in tiles of 64 and 222 in one of 128.
int32_t tile_rows_log2(int64_t rows) {
    if (rows <= 64) return rows <= 16 ? 4 : rows <= 32 ? 5 : 6;
    return 3 * ((rows + 63) / 64) < 5 * ((rows + 127) / 128) ? 6 : 7;
}

LatentGeom latent_geom(const kv_latent_shape_t& s, int32_t n_seqs, int32_t max_rows) {
    LatentGeom g = {};
    const int64_t rows = static_cast<int64_t>(s.n_heads) * max_rows;
    g.max_rows = max_rows;
    g.H = s.n_heads;
    g.Dk = s.key_dim;
    g.Dv = s.value_dim;
    g.tile_log2 = tile_rows_log2(rows);
    g.row_tiles = static_cast<int32_t>((rows + (1 << g.tile_log2) - 1) >> g.tile_log2);
    g.groups = latent_groups(static_cast<int64_t>(n_seqs) * g.row_tiles, s.n_tokens);
    g.scale_log2e = static_cast<float>(latent_scale(s));
    return g;
}

struct LatentSpace {
    uint64_t qa, joined, part_o, part_ml, line, zeros, all;      // byte offsets and the size of the workspace
};
LatentSpace latent_space(const kv_latent_shape_t& s, int32_t n_seqs, const LatentGeom& g) {
    const uint64_t rows = (g.groups + static_cast<uint64_t>(n_seqs) * g.row_tiles) << g.tile_log2;
    LatentSpace w;
    w.qa = 0;
    const uint64_t latents = static_cast<uint64_t>(n_seqs) * g.max_rows * s.n_heads * s.latent_dim * 2;
    w.joined = w.qa + up256(latents);
    w.part_o = w.joined + up256(2 * latents);
    w.part_ml = w.part_o + up256(rows * s.latent_dim * 4);
    w.line = w.part_ml + up256(rows * 8);
    w.zeros = w.line + up256((4 + static_cast<uint64_t>(n_seqs)) * 4);
    w.all = w.zeros + kZeroBytes;
    return w;
}
// What a caller provides for steps of up to max_rows rows.  A step's own space grows with its rows but for one place: with three tiles of 64 (129 to
// 192 query rows) shares are half as high as in the tile of 128 that 65 to 128 rows take, so that their space may be the smaller one.  There the need
// is that of the most rows that one tile holds, and a workspace for the longest of a program's steps serves all of them.
uint64_t latent_need(const kv_latent_shape_t& s, int32_t n_seqs, int32_t max_rows) {
    const uint64_t need = latent_space(s, n_seqs, latent_geom(s, n_seqs, max_rows)).all;
    const int32_t in_one_tile = 128 / s.n_heads;
    if (in_one_tile == 0 || max_rows <= in_one_tile || tile_rows_log2(static_cast<int64_t>(s.n_heads) * max_rows) == 7) return need;
    return std::max(need, latent_space(s, n_seqs, latent_geom(s, n_seqs, in_one_tile)).all);
}

// The places of the line are counted in 31 bits; rows have workgroups of their own in the launches around the attention.
int check_latent_attend(const kv_latent_shape_t* shape, int32_t n_seqs, int32_t max_rows) {
    if (max_rows < 1 || max_rows > 16) return fail(KV_EINVAL, "max_rows %d outside [1,16]", max_rows);
    const int64_t rows = static_cast<int64_t>(shape->n_heads) * max_rows, tile = 1 << tile_rows_log2(rows);
    const int64_t pairs = n_seqs * ((rows + tile - 1) / tile), units = (shape->n_tokens + kLatentTile - 1) / kLatentTile;
    if (pairs * (units + kLatentCost + 1) > 0x7fffffffLL / 2 ||
        static_cast<int64_t>(n_seqs) * max_rows * (shape->n_heads * (shape->latent_dim / 128) + 1) > most_groups(256))
        return fail(KV_ESHAPE, "n_seqs * n_heads * n_tokens too large for one call");
    return KV_OK;
}

struct PromptSpace {
    uint64_t kv, latents, ropes, there, table, all;
};
int64_t prompt_tiles(int32_t n_seqs, int64_t n_tokens) { return n_tokens / kLatentTile + std::min<int64_t>(n_seqs, n_tokens); }
PromptSpace prompt_space(const kv_latent_shape_t& s, int32_t n_seqs, int64_t n_tokens) {
    const uint64_t rows = (static_cast<uint64_t>(prompt_tiles(n_seqs, n_tokens)) + 1) * kLatentTile;      // (a turn may reach a tile past the last)
    PromptSpace w;
    w.kv = 0;
    w.latents = w.kv + up256(rows * s.n_heads * (s.key_dim + s.value_dim) * 2);
    w.ropes = w.latents + up256(rows * s.latent_dim * 2);
    w.there = w.ropes + up256(rows * s.rope_dim * 2);
    w.table = w.there + up256(rows / 8);
    w.all = w.table + up256(static_cast<uint64_t>(n_seqs) * 8);
    return w;
}
int check_prompts(const kv_latent_shape_t* shape, int32_t n_seqs, int64_t n_tokens) {
    if (n_tokens < 1) return fail(KV_EINVAL, "n_tokens %lld is less than 1", static_cast<long long>(n_tokens));
    if (n_tokens > (1 << 26)) return fail(KV_ESHAPE, "n_tokens %lld exceeds 67108864", static_cast<long long>(n_tokens));
    const int64_t rows = prompt_tiles(n_seqs, n_tokens) * kLatentTile, cols = static_cast<int64_t>(shape->n_heads) * (shape->key_dim + shape->value_dim);
    if (((rows + 127) / 128) * ((cols + 255) / 256 + 7) > most_groups(256)) return fail(KV_ESHAPE, "n_tokens * n_heads too large for one call");
    return KV_OK;
}

}  // namespace

extern "C" {

int32_t kv_latent_append_tokens(const kv_latent_shape_t* shape, const kv_pages_t* pages, int32_t layer, const void* c, int64_t c_stride,
                                const void* r, int64_t r_stride, int32_t n_rows, const int32_t* row_start, void* stream) {
    if (int rc = check_latent_pages(shape, pages, layer)) return rc;
    if (int rc = check_moved_rows(shape, pages, n_rows, row_start, c, c_stride, r, r_stride)) return rc;
    if (n_rows == 0) return KV_OK;
    const LatentView view = latent_view(*shape, *pages, layer);
    const int lpg = log2_of(shape->group / 8);
    // Rows of a wavefront: one look at the tables for four rows against four wavefronts at once.  32768 rows of four sequences in pages of every width,
    // inputs and pages from memory, 16.8 us with four, 20.7 with one; 16384 rows 11.0 and 12.5; 8192 rows 8.2 and 7.7; 64 rows of as many sequences
    // 6.8 and 3.6.
    const int units = n_rows >= 16384 ? 4 : 1, rows = units * (shape->latent_dim == 512 ? 1 : 2) * 4;
    const int64_t groups = (static_cast<int64_t>(n_rows) + rows - 1) / rows;
    if (groups > most_groups(256)) return fail(KV_ESHAPE, "n_rows %d too many for one call", n_rows);
    const dim3 grid(static_cast<uint32_t>(groups));
    hipStream_t st = static_cast<hipStream_t>(stream);
#define KV_LAUNCH(D, UNITS)                                                                                                        \
    hipLaunchKernelGGL((latent_append_kernel<D, UNITS>), grid, dim3(256), 0, st, view, static_cast<const _Float16*>(c), c_stride, \
                       static_cast<const _Float16*>(r), r_stride, n_rows, lpg, row_start)
    if (shape->latent_dim == 512) {
        if (units == 4) KV_LAUNCH(512, 4);
        else KV_LAUNCH(512, 1);
    } else {
        if (units == 4) KV_LAUNCH(256, 4);
        else KV_LAUNCH(256, 1);
    }
#undef KV_LAUNCH
    return launch_status("latent_append_kernel launch");
}

int32_t kv_latent_read_tokens(const kv_latent_shape_t* shape, const kv_pages_t* pages, int32_t layer, void* c, int64_t c_stride, void* r,
                              int64_t r_stride, int32_t n_rows, const int32_t* row_start, void* stream) {
    if (int rc = check_latent_pages(shape, pages, layer)) return rc;
    if (int rc = check_moved_rows(shape, pages, n_rows, row_start, c, c_stride, r, r_stride)) return rc;
    if (n_rows == 0) return KV_OK;
    const LatentView view = latent_view(*shape, *pages, layer);
    const int lpg = log2_of(shape->group / 8);
    // As in appending; a row's loads and its results stand in registers, so two (24 ragged contexts of up to 16384 tokens: 112 us with two, 118 with four,
    // 126 with one; 8192 rows 7.4 with two, 8.2 with one; 2048 rows 5.2 and 4.6).
    const int units = n_rows >= 8192 ? 2 : 1, rows = units * (shape->latent_dim == 512 ? 1 : 2) * 4;
    const int64_t groups = (static_cast<int64_t>(n_rows) + rows - 1) / rows;
    if (groups > most_groups(256)) return fail(KV_ESHAPE, "n_rows %d too many for one call", n_rows);
    const dim3 grid(static_cast<uint32_t>(groups));
    hipStream_t st = static_cast<hipStream_t>(stream);
#define KV_LAUNCH(D, UNITS)                                                                                                \
    hipLaunchKernelGGL((latent_read_kernel<D, UNITS>), grid, dim3(256), 0, st, view, static_cast<_Float16*>(c), c_stride, \
                       static_cast<_Float16*>(r), r_stride, n_rows, lpg, row_start)
    if (shape->latent_dim == 512) {
        if (units == 2) KV_LAUNCH(512, 2);
        else KV_LAUNCH(512, 1);
    } else {
        if (units == 2) KV_LAUNCH(256, 2);
        else KV_LAUNCH(256, 1);
    }
#undef KV_LAUNCH
    return launch_status("latent_read_kernel launch");
}

uint64_t kv_latent_attend_workspace_bytes(const kv_latent_shape_t* shape, int32_t n_seqs, int32_t max_rows) {
    if (check_latent_shape(shape) || check_seqs(n_seqs) || check_latent_attend(shape, n_seqs, max_rows)) return 0;
    return latent_need(*shape, n_seqs, max_rows);
}

int32_t kv_latent_attend_tokens(const kv_latent_shape_t* shape, const kv_pages_t* pages, int32_t layer, const void* q, int64_t q_stride,
                                int32_t n_rows, const int32_t* row_start, int32_t max_rows, const void* w, void* workspace,
                                uint64_t workspace_bytes, void* out, void* stream) {
    if (int rc = check_latent_pages(shape, pages, layer)) return rc;
    if (int rc = check_latent_attend(shape, pages->n_seqs, max_rows)) return rc;
    if (int rc = check_rows(pages, n_rows, row_start, q_stride, static_cast<int64_t>(shape->n_heads) * (shape->key_dim + shape->rope_dim))) return rc;
    if (n_rows == 0) return KV_OK;
    if (!q || !w || !out || !workspace) return fail(KV_EINVAL, "NULL device pointer");
    if (!aligned(q, 16) || !aligned(w, 16) || !aligned(out, 16) || !aligned(workspace, 256))
        return fail(KV_EINVAL, "q, w and out must be 16-byte aligned, workspace 256-byte aligned");
    const int32_t n_seqs = pages->n_seqs;
    LatentGeom g = latent_geom(*shape, n_seqs, max_rows);
    g.n_rows = n_rows;
    g.q_stride = q_stride;
    const LatentSpace sp = latent_space(*shape, n_seqs, g);
    const uint64_t need = latent_need(*shape, n_seqs, max_rows);
    if (workspace_bytes < need)
        return fail(KV_ENOMEM, "workspace of %llu bytes, %llu needed", static_cast<unsigned long long>(workspace_bytes),
                    static_cast<unsigned long long>(need));
    const LatentView view = latent_view(*shape, *pages, layer);
    const int lpg = log2_of(shape->group / 8);
    uint8_t* space = static_cast<uint8_t*>(workspace);
    _Float16* qa = reinterpret_cast<_Float16*>(space + sp.qa);
    float* part_o = reinterpret_cast<float*>(space + sp.part_o);
    float* part_ml = reinterpret_cast<float*>(space + sp.part_ml);
    int32_t* line = reinterpret_cast<int32_t*>(space + sp.line);
    uint8_t* zeros = space + sp.zeros;
    const _Float16 *q16 = static_cast<const _Float16*>(q), *w16 = static_cast<const _Float16*>(w);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int32_t all_rows = n_seqs * max_rows, dc = shape->latent_dim;
    const int blocks = all_rows > 16 ? 4 : 1;                // of 16 rows
    const dim3 absorb(static_cast<uint32_t>(1 + shape->n_heads * (dc / 128)), static_cast<uint32_t>((all_rows + 16 * blocks - 1) / (16 * blocks)));
#define KV_LAUNCH(D, ROWS) \
    hipLaunchKernelGGL((latent_absorb_kernel<D, ROWS>), absorb, dim3(256), 0, st, view, g, q16, w16, row_start, qa, line, reinterpret_cast<uint32_t*>(zeros))
    if (dc == 512) {
        if (blocks == 4) KV_LAUNCH(512, 4);
        else KV_LAUNCH(512, 1);
    } else {
        if (blocks == 4) KV_LAUNCH(256, 4);
        else KV_LAUNCH(256, 1);
    }
#undef KV_LAUNCH
    if (int rc = launch_status("latent_absorb_kernel launch")) return rc;
    const dim3 attend(static_cast<uint32_t>(g.groups));
    const LatentAttendArgs args = {view, g, qa, q16, row_start, line, zeros, part_o, part_ml, lpg};
#define KV_LAUNCH(D, R, M) hipLaunchKernelGGL((latent_attend_kernel<D, R, M>), attend, dim3(64 * kLatentWaves), 0, st, args)
#define KV_BY_ROWS(D, R)                        \
    do {                                        \
        if (g.tile_log2 == 4) KV_LAUNCH(D, R, 16);      \
        else if (g.tile_log2 == 5) KV_LAUNCH(D, R, 32); \
        else if (g.tile_log2 == 6) KV_LAUNCH(D, R, 64); \
        else KV_LAUNCH(D, R, 128);              \
    } while (0)
    if (dc == 512) {
        if (shape->rope_dim == 64) KV_BY_ROWS(512, 64);
        else KV_BY_ROWS(512, 32);
    } else {
        if (shape->rope_dim == 64) KV_BY_ROWS(256, 64);
        else KV_BY_ROWS(256, 32);
    }
#undef KV_BY_ROWS
#undef KV_LAUNCH
    if (int rc = launch_status("latent_attend_kernel launch")) return rc;
    const int64_t heads_rows = static_cast<int64_t>(all_rows) * shape->n_heads;
    _Float16 *hi = reinterpret_cast<_Float16*>(space + sp.joined), *lo = hi + heads_rows * dc;
    const uint32_t lds = static_cast<uint32_t>(g.groups) * 4;
#define KV_LAUNCH(D)                                                                                                                    \
    hipLaunchKernelGGL((latent_join_kernel<D>), dim3(static_cast<uint32_t>(heads_rows)), dim3(256), lds, st, view, g, row_start, line, part_o, \
                       part_ml, hi, lo)
    if (dc == 512) KV_LAUNCH(512);
    else KV_LAUNCH(256);
#undef KV_LAUNCH
    if (int rc = launch_status("latent_join_kernel launch")) return rc;
    const dim3 values(static_cast<uint32_t>(shape->n_heads * (shape->value_dim / 64)), static_cast<uint32_t>((all_rows + 15) / 16));
#define KV_LAUNCH(D, V) \
    hipLaunchKernelGGL((latent_values_kernel<D, V>), values, dim3(256), 0, st, view, g, w16, row_start, hi, lo, static_cast<_Float16*>(out))
    if (dc == 512) {
        if (shape->value_dim == 128) KV_LAUNCH(512, 128);
        else KV_LAUNCH(512, 64);
    } else {
        if (shape->value_dim == 128) KV_LAUNCH(256, 128);
        else KV_LAUNCH(256, 64);
    }
#undef KV_LAUNCH
    return launch_status("latent_values_kernel launch");
}

uint64_t kv_latent_prompts_workspace_bytes(const kv_latent_shape_t* shape, int32_t n_seqs, int64_t n_tokens) {
    if (check_latent_shape(shape) || check_seqs(n_seqs) || check_prompts(shape, n_seqs, n_tokens)) return 0;
    return prompt_space(*shape, n_seqs, n_tokens).all;
}

int32_t kv_latent_attend_prompts(const kv_latent_shape_t* shape, const kv_pages_t* pages, int32_t layer, const void* q, int64_t q_stride,
                                 int32_t n_rows, const int32_t* row_start, int64_t n_tokens, const void* w, void* workspace,
                                 uint64_t workspace_bytes, void* out, void* stream) {
    if (int rc = check_latent_pages(shape, pages, layer)) return rc;
    if (int rc = check_prompts(shape, pages->n_seqs, n_tokens)) return rc;
    if (int rc = check_rows(pages, n_rows, row_start, q_stride, static_cast<int64_t>(shape->n_heads) * (shape->key_dim + shape->rope_dim))) return rc;
    if (n_rows == 0) return KV_OK;
    if (!q || !w || !out || !workspace) return fail(KV_EINVAL, "NULL device pointer");
    if (!aligned(q, 16) || !aligned(w, 16) || !aligned(out, 16) || !aligned(workspace, 256))
        return fail(KV_EINVAL, "q, w and out must be 16-byte aligned, workspace 256-byte aligned");
    const int32_t n_seqs = pages->n_seqs;
    const PromptSpace sp = prompt_space(*shape, n_seqs, n_tokens);
    if (workspace_bytes < sp.all)
        return fail(KV_ENOMEM, "workspace of %llu bytes, %llu needed", static_cast<unsigned long long>(workspace_bytes),
                    static_cast<unsigned long long>(sp.all));
    PromptGeom g = {};
    g.n_rows = n_rows;
    g.H = shape->n_heads;
    g.cap_tiles = static_cast<int32_t>(prompt_tiles(n_seqs, n_tokens));
    g.row_tiles = n_rows / kPromptRows + std::min(n_seqs, n_rows);
    g.q_stride = q_stride;
    g.scale_log2e = static_cast<float>(latent_scale(*shape));
    const int64_t groups = static_cast<int64_t>(g.row_tiles) * g.H;
    const int32_t cols = g.H * (shape->key_dim + shape->value_dim), token_tiles = (g.cap_tiles + kProjectTiles - 1) / kProjectTiles;
    const int32_t col_tiles = (cols + kProjectCols - 1) / kProjectCols;
    const int64_t project_groups = (col_tiles + 7) / 8 * 8 * static_cast<int64_t>(token_tiles);
    if (groups > most_groups(256)) return fail(KV_ESHAPE, "n_rows * n_heads too large for one call");
    const LatentView view = latent_view(*shape, *pages, layer);
    const int lpg = log2_of(shape->group / 8);
    uint8_t* space = static_cast<uint8_t*>(workspace);
    _Float16* kv = reinterpret_cast<_Float16*>(space + sp.kv);
    _Float16* latents = reinterpret_cast<_Float16*>(space + sp.latents);
    _Float16* ropes = reinterpret_cast<_Float16*>(space + sp.ropes);
    uint32_t* there = reinterpret_cast<uint32_t*>(space + sp.there);
    PromptTable table;
    table.tile_end = reinterpret_cast<int32_t*>(space + sp.table);
    table.row_end = table.tile_end + n_seqs;
    hipStream_t st = static_cast<hipStream_t>(stream);
    hipLaunchKernelGGL(latent_table_kernel, dim3(1), dim3(64), 0, st, view, g, row_start, table);
    if (int rc = launch_status("latent_table_kernel launch")) return rc;
    const dim3 tiles(static_cast<uint32_t>(g.cap_tiles));
#define KV_LAUNCH(D, R) hipLaunchKernelGGL((latent_gather_kernel<D, R>), tiles, dim3(256), 0, st, view, g, table, lpg, latents, ropes, there)
    if (shape->latent_dim == 512) {
        if (shape->rope_dim == 64) KV_LAUNCH(512, 64);
        else KV_LAUNCH(512, 32);
    } else {
        if (shape->rope_dim == 64) KV_LAUNCH(256, 64);
        else KV_LAUNCH(256, 32);
    }
#undef KV_LAUNCH
    if (int rc = launch_status("latent_gather_kernel launch")) return rc;
    const dim3 project(static_cast<uint32_t>(project_groups));
#define KV_LAUNCH(D)                                                                                                                         \
    hipLaunchKernelGGL((latent_project_kernel<D>), project, dim3(256), 0, st, table, n_seqs, cols, col_tiles, token_tiles, latents,          \
                       static_cast<const _Float16*>(w), kv)
    if (shape->latent_dim == 512) KV_LAUNCH(512);
    else KV_LAUNCH(256);
#undef KV_LAUNCH
    if (int rc = launch_status("latent_project_kernel launch")) return rc;
    const dim3 attend(static_cast<uint32_t>(groups));
#define KV_LAUNCH(K, R, V)                                                                                                                        \
    hipLaunchKernelGGL((latent_prompt_kernel<K, R, V>), attend, dim3(256), 0, st, view, g, table, row_start, static_cast<const _Float16*>(q), kv, \
                       ropes, there, static_cast<_Float16*>(out))
#define KV_BY_VALUE(K, R)                                \
    do {                                                 \
        if (shape->value_dim == 128) KV_LAUNCH(K, R, 128); \
        else KV_LAUNCH(K, R, 64);                        \
    } while (0)
    if (shape->key_dim == 128) {
        if (shape->rope_dim == 64) KV_BY_VALUE(128, 64);
        else KV_BY_VALUE(128, 32);
    } else {
        if (shape->rope_dim == 64) KV_BY_VALUE(64, 64);
        else KV_BY_VALUE(64, 32);
    }
#undef KV_BY_VALUE
#undef KV_LAUNCH
    return launch_status("latent_prompt_kernel launch");
}

}  // extern "C"
