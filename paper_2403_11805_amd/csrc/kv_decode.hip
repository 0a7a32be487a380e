// Decoding on the packed records: append, attention and eviction over the pages of running sequences.  Argument checks on the
// host, then launches on the caller's stream; nothing here synchronises or allocates.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "kv_internal.h"
#include "kv_launch_rules.hpp"
#include "kv_append_kernels.hpp"
#include "kv_attend_kernels.hpp"
#include "kv_evict_kernels.hpp"

using namespace kvs;

namespace {

int hip_fail(hipError_t e, const char* what) { return fail(KV_EHIP, "%s: %s", what, hipGetErrorString(e)); }

int launch_status(const char* what) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? KV_OK : hip_fail(e, what);
}

// Workgroups that one launch may have: a grid has less than 2^32 threads.
constexpr int64_t most_groups(int threads) { return 0xffffffffLL / threads; }

int check_paged_shape(const kv_shape_t* shape) {
    if (int rc = check_shape(shape)) return rc;
    if (!is_f16(*shape)) return fail(KV_ESHAPE, "paged sequences need an fp16 cache format");
    if (shape->head_dim != 64 && shape->head_dim != 128 && shape->head_dim != 256)
        return fail(KV_ESHAPE, "paged sequences need head_dim in {64,128,256}, got %d", shape->head_dim);
    if (shape->chunk_tokens % 16)
        return fail(KV_ESHAPE, "paged sequences need chunk_tokens %% 16 == 0, got %d", shape->chunk_tokens);
    return KV_OK;
}

int check_seqs(int32_t n_seqs) {
    return n_seqs < 1 || n_seqs > 65535 ? fail(KV_EINVAL, "n_seqs %d outside [1, 65535]", n_seqs) : KV_OK;
}

int check_pages(const kv_shape_t* shape, const kv_pages_t* pages) {
    if (int rc = check_paged_shape(shape)) return rc;
    if (!pages) return fail(KV_EINVAL, "pages is NULL");
    if (int rc = check_seqs(pages->n_seqs)) return rc;
    if (!pages->pool || !pages->off || !pages->bits || !pages->len) return fail(KV_EINVAL, "NULL device pointer in pages");
    if (!aligned(pages->pool, 16) || !aligned(pages->off, 8) || !aligned(pages->len, 4))
        return fail(KV_EINVAL, "pages: pool must be 16-byte aligned, off 8-byte, len 4-byte aligned");
    if (pages->stride < shape->n_tokens / shape->chunk_tokens)
        return fail(KV_EINVAL, "pages: stride %d is less than the %d pages of a sequence", pages->stride,
                    shape->n_tokens / shape->chunk_tokens);
    return KV_OK;
}

int check_layer(const kv_shape_t* shape, int32_t layer) {
    return layer < 0 || layer >= shape->n_layers ? fail(KV_EINVAL, "layer %d outside [0,%d)", layer, shape->n_layers) : KV_OK;
}

// The rows of a step: their number, their list, and the elements from one to the next.
int check_rows(const kv_pages_t* pages, int32_t n_rows, const int32_t* row_start, int64_t stride, int64_t least) {
    if (n_rows < 0) return fail(KV_EINVAL, "n_rows %d is negative", n_rows);
    if (!row_start && n_rows != pages->n_seqs)
        return fail(KV_EINVAL, "without row_start n_rows (%d) must be n_seqs (%d)", n_rows, pages->n_seqs);
    if (!aligned(row_start, 4)) return fail(KV_EINVAL, "row_start must be 4-byte aligned");
    if (stride < least || stride % 8) return fail(KV_EINVAL, "row stride %lld is less than %lld or no multiple of 8",
                                                  static_cast<long long>(stride), static_cast<long long>(least));
    return KV_OK;
}

PagesView pages_view(const kv_shape_t& s, const kv_pages_t& p) {
    PagesView v;
    v.pool = static_cast<uint8_t*>(p.pool);
    v.off = p.off;
    v.bits = p.bits;
    v.len = p.len;
    v.n_seqs = p.n_seqs;
    v.stride = p.stride;
    v.N = s.n_tokens;
    v.T = s.chunk_tokens;
    v.Hkv = s.n_kv_heads;
    v.Hq = s.n_q_heads;
    v.slabs = static_cast<int32_t>(slabs_of(s));
    v.groups = s.head_dim / s.group;
    v.half_params = s.format == KV_FMT_F16_GROUPS_H ? 1 : 0;
    const uint32_t d = static_cast<uint32_t>(s.chunk_tokens) / 16;
    v.page_of_tile = d == 1 ? 0u : static_cast<uint32_t>(((1ull << 32) + d - 1) / d);
    v.pool_bytes = p.pool_bytes;
    v.bit_bytes = record_bytes(s, 16) / 16;
    v.param_bytes = record_bytes(s, 2) - 2 * v.bit_bytes;
    return v;
}

int log2_of(int v) {
    int l = 0;
    while ((1 << l) < v) ++l;
    return l;
}

// Launches K<head_dim, ...>.
#define KV_BY_HEAD_DIM(d, LAUNCH) \
    do {                          \
        if ((d) == 64) LAUNCH(64); \
        else if ((d) == 128) LAUNCH(128); \
        else LAUNCH(256);         \
    } while (0)

AttendGeom attend_geom(const kv_shape_t& s, int32_t n_seqs, int32_t max_rows) {
    AttendGeom g = {};
    g.max_rows = max_rows;
    g.per = s.n_q_heads / s.n_kv_heads;
    g.rows = g.per * max_rows;
    g.row_tiles = (g.rows + 15) / 16;
    g.tile_rows = std::min(16, g.rows);
    g.step = attend_step(s.head_dim);
    g.groups = static_cast<int32_t>(attend_groups(static_cast<int64_t>(n_seqs) * s.n_kv_heads * g.row_tiles, s.n_tokens, s.head_dim));
    g.scale_log2e = static_cast<float>(1.4426950408889634 / std::sqrt(static_cast<double>(s.head_dim)));
    return g;
}

struct AttendSpace {
    uint64_t part_o, part_ml, note, logits, all;      // byte offsets and the size of the workspace
};
AttendSpace attend_space(const kv_shape_t& s, int32_t n_seqs, const AttendGeom& g, bool with_mass) {
    auto up = [](uint64_t x) { return (x + 255) & ~255ull; };
    const uint64_t rows = (g.groups + static_cast<uint64_t>(n_seqs) * s.n_kv_heads * g.row_tiles) * g.tile_rows;
    AttendSpace w;
    w.part_o = 0;
    w.part_ml = w.part_o + up(rows * s.head_dim * 4);
    w.note = w.part_ml + up(rows * 8);
    w.logits = w.note + up((4 + static_cast<uint64_t>(n_seqs)) * 4);
    w.all = w.logits + (with_mass ? up(static_cast<uint64_t>(n_seqs) * s.n_kv_heads * g.rows * s.n_tokens * 4) : 0);
    return w;
}

// The rows of a step and the work they make: units of 32 tokens of every (sequence, kv head, row tile) are counted in 31 bits, and
// every row and every 1024 weights of a (sequence, kv head) has a workgroup of the second launch.
int check_attend(const kv_shape_t* shape, int32_t n_seqs, int32_t max_rows) {
    if (max_rows < 1 || max_rows > 16) return fail(KV_EINVAL, "max_rows %d outside [1,16]", max_rows);
    const int64_t rows = static_cast<int64_t>(shape->n_q_heads / shape->n_kv_heads) * max_rows;
    if (rows > kMaxPairRows) return fail(KV_ESHAPE, "more than %d query rows per kv head", kMaxPairRows);
    const int64_t pairs = static_cast<int64_t>(n_seqs) * shape->n_kv_heads;
    if (pairs * ((rows + 15) / 16) > 0x7fffffffLL / ((shape->n_tokens + 2047) / 32) ||
        pairs * (rows + (shape->n_tokens + 1023) / 1024) > most_groups(256))
        return fail(KV_ESHAPE, "n_seqs * n_kv_heads * n_tokens too large for one call");
    return KV_OK;
}

uint64_t evict_space(const kv_shape_t& s, int64_t pairs, int32_t keep, int32_t* list) {
    *list = std::max(0, std::min(keep, s.n_tokens - keep));
    return ((static_cast<uint64_t>(pairs) * 4 + 255) & ~255ull) + static_cast<uint64_t>(pairs) * 2 * (*list) * 4 + 256;
}

}  // namespace

extern "C" {

int32_t kv_append_tokens(const kv_shape_t* shape, const kv_pages_t* pages, int32_t layer, const void* k, const void* v,
                         int64_t row_stride, int32_t n_rows, const int32_t* row_start, const int32_t* seen, float* mass,
                         int32_t* pos, void* stream) {
    if (int rc = check_pages(shape, pages)) return rc;
    if (int rc = check_layer(shape, layer)) return rc;
    if (int rc = check_rows(pages, n_rows, row_start, row_stride, static_cast<int64_t>(shape->n_kv_heads) * shape->head_dim)) return rc;
    if (n_rows == 0) return KV_OK;
    if (!k || !v) return fail(KV_EINVAL, "NULL device pointer");
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(seen, 4) || !aligned(mass, 4) || !aligned(pos, 4))
        return fail(KV_EINVAL, "k and v must be 16-byte aligned, seen, mass and pos 4-byte aligned");
    const int pieces = 2 * shape->n_kv_heads * shape->head_dim / 8;
    const int ppl = append_pieces_per_lane(n_rows, pieces);
    const int32_t tasks_per_row = (pieces + 64 * ppl - 1) / (64 * ppl);
    const int64_t tasks = static_cast<int64_t>(n_rows) * tasks_per_row, groups = (tasks + 3) / 4;
    if (groups > most_groups(256)) return fail(KV_ESHAPE, "n_rows * n_kv_heads * head_dim too large for one call");
    const PagesView view = pages_view(*shape, *pages);
    const int lpg = log2_of(shape->group / 8);
    hipStream_t st = static_cast<hipStream_t>(stream);
#define KV_LAUNCH_PPL(D, PPL)                                                                                                   \
    hipLaunchKernelGGL((append_kernel<D, PPL>), dim3(static_cast<uint32_t>(groups)), dim3(256), 0, st, view, layer,             \
                       static_cast<const u4_t*>(k), static_cast<const u4_t*>(v), row_stride / 8, n_rows, tasks_per_row, tasks, \
                       lpg, row_start, seen, mass, pos)
#define KV_LAUNCH(D)                        \
    do {                                    \
        if (ppl == 4) KV_LAUNCH_PPL(D, 4);  \
        else KV_LAUNCH_PPL(D, 1);           \
    } while (0)
    KV_BY_HEAD_DIM(shape->head_dim, KV_LAUNCH);
#undef KV_LAUNCH
#undef KV_LAUNCH_PPL
    return launch_status("append_kernel launch");
}

uint64_t kv_attend_workspace_bytes(const kv_shape_t* shape, int32_t n_seqs, int32_t max_rows, int32_t with_mass) {
    if (check_paged_shape(shape) || check_seqs(n_seqs) || check_attend(shape, n_seqs, max_rows)) return 0;
    return attend_space(*shape, n_seqs, attend_geom(*shape, n_seqs, max_rows), with_mass != 0).all;
}

int32_t kv_attend_tokens(const kv_shape_t* shape, const kv_pages_t* pages, int32_t layer, const void* q, int64_t q_stride,
                         int32_t n_rows, const int32_t* row_start, int32_t max_rows, const float* mass_in, float* mass,
                         void* workspace, uint64_t workspace_bytes, void* out, void* stream) {
    if (int rc = check_pages(shape, pages)) return rc;
    if (int rc = check_layer(shape, layer)) return rc;
    if (int rc = check_attend(shape, pages->n_seqs, max_rows)) return rc;
    if (int rc = check_rows(pages, n_rows, row_start, q_stride, static_cast<int64_t>(shape->n_q_heads) * shape->head_dim)) return rc;
    if (mass_in && !mass) return fail(KV_EINVAL, "mass_in without mass");
    if (n_rows == 0) return KV_OK;
    if (!q || !out || !workspace) return fail(KV_EINVAL, "NULL device pointer");
    if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 256) || !aligned(mass, 4) || !aligned(mass_in, 4))
        return fail(KV_EINVAL, "q and out must be 16-byte aligned, workspace 256-byte, mass 4-byte aligned");
    AttendGeom g = attend_geom(*shape, pages->n_seqs, max_rows);
    g.layer = layer;
    g.n_rows = n_rows;
    g.q_stride = q_stride;
    const AttendSpace w = attend_space(*shape, pages->n_seqs, g, mass != nullptr);
    if (workspace_bytes < w.all)
        return fail(KV_ENOMEM, "workspace of %llu bytes, %llu needed", static_cast<unsigned long long>(workspace_bytes),
                    static_cast<unsigned long long>(w.all));
    const int64_t pairs = static_cast<int64_t>(pages->n_seqs) * shape->n_kv_heads;
    const int32_t blocks = (shape->n_tokens + 1023) / 1024;
    const PagesView view = pages_view(*shape, *pages);
    uint8_t* space = static_cast<uint8_t*>(workspace);
    float* part_o = reinterpret_cast<float*>(space + w.part_o);
    float* part_ml = reinterpret_cast<float*>(space + w.part_ml);
    int32_t* note = reinterpret_cast<int32_t*>(space + w.note);
    float* logits = mass ? reinterpret_cast<float*>(space + w.logits) : nullptr;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const _Float16* q16 = static_cast<const _Float16*>(q);
    _Float16* o16 = static_cast<_Float16*>(out);
    const dim3 grid(static_cast<uint32_t>(g.groups)), block(64 * kAttendWaves);
    const uint32_t lds = static_cast<uint32_t>(kAttendWaves * g.tile_rows * shape->head_dim) * 4;   // at most 64 KB
#define KV_LAUNCH(D, G)                                                                                                                       \
    do {                                                                                                                                      \
        if (view.half_params)                                                                                                                 \
            hipLaunchKernelGGL((attend_kernel<D, G, true>), grid, block, lds, st, view, g, q16, row_start, o16, part_o, part_ml, logits, note); \
        else                                                                                                                                  \
            hipLaunchKernelGGL((attend_kernel<D, G, false>), grid, block, lds, st, view, g, q16, row_start, o16, part_o, part_ml, logits, note); \
    } while (0)
    switch (shape->head_dim * 1024 + shape->group) {
        case 64 * 1024 + 64: KV_LAUNCH(64, 64); break;
        case 128 * 1024 + 64: KV_LAUNCH(128, 64); break;
        case 128 * 1024 + 128: KV_LAUNCH(128, 128); break;
        case 256 * 1024 + 64: KV_LAUNCH(256, 64); break;
        case 256 * 1024 + 128: KV_LAUNCH(256, 128); break;
        default: KV_LAUNCH(256, 256); break;
    }
#undef KV_LAUNCH
    if (int rc = launch_status("attend_kernel launch")) return rc;
    const int32_t joins = static_cast<int32_t>(pairs * g.rows);
    const dim3 finish(static_cast<uint32_t>(joins + (mass ? pairs * blocks : 0)));
    const uint32_t weights = static_cast<uint32_t>(g.groups) * 4;
#define KV_LAUNCH(D)                                                                                                                  \
    hipLaunchKernelGGL((attend_finish_kernel<D>), finish, dim3(256), weights, st, view, g, joins, blocks, row_start, part_o, part_ml, \
                       logits, mass_in, mass, o16, note)
    KV_BY_HEAD_DIM(shape->head_dim, KV_LAUNCH);
#undef KV_LAUNCH
    return launch_status("attend_finish_kernel launch");
}

uint64_t kv_evict_workspace_bytes(const kv_shape_t* shape, int32_t n_seqs, int32_t n_layers, int32_t keep) {
    if (check_paged_shape(shape) || check_seqs(n_seqs)) return 0;
    if (n_layers < 1 || n_layers > shape->n_layers || keep < 1) {
        fail(KV_EINVAL, "n_layers %d outside [1,%d] or keep %d less than 1", n_layers, shape->n_layers, keep);
        return 0;
    }
    int32_t list = 0;
    return evict_space(*shape, static_cast<int64_t>(n_layers) * n_seqs * shape->n_kv_heads, keep, &list);
}

int32_t kv_evict_tokens(const kv_shape_t* shape, const kv_pages_t* pages, int32_t layer_begin, int32_t layer_end,
                        const float* mass_in, const int32_t* pos_in, const int32_t* seen, int32_t keep, int32_t sink, int32_t recent,
                        void* workspace, uint64_t workspace_bytes, float* mass, int32_t* pos, void* stream) {
    if (int rc = check_pages(shape, pages)) return rc;
    if (layer_begin < 0 || layer_end < layer_begin || layer_end > shape->n_layers)
        return fail(KV_EINVAL, "layers [%d,%d) outside [0,%d]", layer_begin, layer_end, shape->n_layers);
    if (keep < 1 || sink < 0 || recent < 0 || static_cast<int64_t>(sink) + recent > keep)
        return fail(KV_EINVAL, "keep %d, sink %d, recent %d: keep >= 1, sink + recent <= keep", keep, sink, recent);
    if (layer_begin == layer_end) return KV_OK;
    if (!mass_in || !pos_in || !mass || !pos || !workspace) return fail(KV_EINVAL, "NULL device pointer");
    if (!aligned(mass_in, 4) || !aligned(pos_in, 4) || !aligned(seen, 4) || !aligned(mass, 4) || !aligned(pos, 4) || !aligned(workspace, 256))
        return fail(KV_EINVAL, "mass, pos and seen must be 4-byte aligned, workspace 256-byte aligned");
    EvictGeom g = {};
    g.layer0 = layer_begin;
    g.n_layers = layer_end - layer_begin;
    g.keep = keep;
    g.sink = sink;
    g.recent = recent;
    const int64_t pairs = static_cast<int64_t>(g.n_layers) * pages->n_seqs * shape->n_kv_heads;
    const uint64_t need = evict_space(*shape, pairs, keep, &g.list);
    if (workspace_bytes < need)
        return fail(KV_ENOMEM, "workspace of %llu bytes, %llu needed", static_cast<unsigned long long>(workspace_bytes),
                    static_cast<unsigned long long>(need));
    const int32_t rows_per_group = 256 / (shape->head_dim / 8);
    const int32_t blocks = static_cast<int32_t>(evict_blocks(pairs, g.list, rows_per_group * kAtOnce));
    if (pairs > most_groups(kSelectThreads) || pairs * blocks > most_groups(256))
        return fail(KV_ESHAPE, "layers * n_seqs * n_kv_heads too large for one call");
    const PagesView view = pages_view(*shape, *pages);
    int32_t* n_moves = static_cast<int32_t*>(workspace);
    int32_t* moves = reinterpret_cast<int32_t*>(static_cast<uint8_t*>(workspace) + ((static_cast<uint64_t>(pairs) * 4 + 255) & ~255ull));
    hipStream_t st = static_cast<hipStream_t>(stream);
#define KV_LAUNCH(KEYS)                                                                                                                 \
    hipLaunchKernelGGL((evict_select_kernel<KEYS>), dim3(static_cast<uint32_t>(pairs)), dim3(kSelectThreads), 0, st, view, g, mass_in, \
                       pos_in, seen, moves, n_moves, mass, pos)
    // Keys of a lane in registers, as few as the longest sequence may have: 2049 slots take 9.4 us with 4, 16.1 with 32 (every pass is
    // written out key by key) and 12.7 read again by every pass; 6144 12.4 with 8, 17.6 with 32; 16384 19.5 with 16, 23.5 with 32;
    // 32768 32 with 32, 79 read again.
    if (shape->n_tokens <= 4 * kSelectThreads) KV_LAUNCH(4);
    else if (shape->n_tokens <= 8 * kSelectThreads) KV_LAUNCH(8);
    else if (shape->n_tokens <= 16 * kSelectThreads) KV_LAUNCH(16);
    else if (shape->n_tokens <= 32 * kSelectThreads) KV_LAUNCH(32);
    else KV_LAUNCH(0);
#undef KV_LAUNCH
    if (int rc = launch_status("evict_select_kernel launch")) return rc;
    if (g.list == 0) return KV_OK;                          // no sequence can have more than `keep` tokens
    const dim3 grid(static_cast<uint32_t>(pairs * blocks));
    const int lpg = log2_of(shape->group / 8);
#define KV_LAUNCH(D)                                                                                                              \
    hipLaunchKernelGGL((evict_move_kernel<D>), grid, dim3(256), 0, st, view, g, blocks, lpg, moves, n_moves, mass_in, pos_in, mass, pos)
    KV_BY_HEAD_DIM(shape->head_dim, KV_LAUNCH);
#undef KV_LAUNCH
    return launch_status("evict_move_kernel launch");
}

}  // extern "C"
