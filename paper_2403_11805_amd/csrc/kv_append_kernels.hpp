// Append: K and V rows of new tokens into the pages of their sequences (one layer), quantised where the page is packed.
#pragma once

#include "kv_pages_kernels.hpp"

namespace kvs {

// Bytes bound it in fp16 pages: a row is read once and written once, 16 bytes a lane, past the caches.  Six prompts of 300 to 4096
// tokens, 32 kv heads of 128 (458 MB): 88 to 91 us, 5.0 to 5.2 TB/s.  Packed pages take as long for fewer bytes: 88 us at 8 bits (355
// MB), 83 at 4 (298), 92 at 2 (270, two groups per row).  The memory gets as many write requests as in fp16 (4.4 million against 4.1
// at 8 bits, half of them not whole; 3.3 at 2 bits, seven eighths), and vector instructions take 50 us of it.  One token for each
// of 64 sequences takes 3.1 us, 3.5 to 3.7 packed, which is a launch and three dependent loads.
// Work unit: up to PPL * 64 pieces (8 elements, 16 bytes) of one row's K and V heads, K's first, per wavefront.  The row's
// sequence, its page and the page's width are wave-uniform, so the width is one branch for the whole wavefront, and the rows'
// loads are issued before the three dependent list loads that lead to the page.
template <int D, int PPL>
__global__ __launch_bounds__(256) void append_kernel(PagesView v, int32_t layer, const u4_t* __restrict__ k,
                                                     const u4_t* __restrict__ vv, int64_t row_pieces, int32_t n_rows,
                                                     int32_t tasks_per_row, int64_t n_tasks, int32_t lpg_log2,
                                                     const int32_t* __restrict__ row_start, const int32_t* __restrict__ seen,
                                                     float* __restrict__ mass, int32_t* __restrict__ pos) {
    constexpr int kRow = D / 8;                                   // pieces of one head's row
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    const int64_t task = static_cast<int64_t>(blockIdx.x) * 4 + wave;
    if (task >= n_tasks) return;
    const int r = static_cast<int>(task / tasks_per_row), part = static_cast<int>(task - static_cast<int64_t>(r) * tasks_per_row);
    const int k_pieces = v.Hkv * kRow, all = 2 * k_pieces;
    u4_t raw[PPL];
#pragma unroll
    for (int u = 0; u < PPL; ++u) {
        const int p = min((part * PPL + u) * 64 + lane, all - 1);
        raw[u] = p < k_pieces ? k[r * row_pieces + p] : vv[r * row_pieces + p - k_pieces];
    }
    const int s = __builtin_amdgcn_readfirstlane(seq_of_row(row_start, v.n_seqs, r, lane));
    if (s < 0) return;
    const SeqRows rows = seq_rows(row_start, s, n_rows);
    const int n = seq_len(v, s), back = rows.count - (r - rows.first);       // token n - back
    const int token = n - back;
    if (token < 0 || back < 1) return;
    const int page = token / v.T, in_page = token - page * v.T;
    if (part == 0) {
        const int position = (seen ? seen[s] : n) - back;
        for (int h = lane; h < v.Hkv; h += 64) {
            const int64_t at = (static_cast<int64_t>(s) * v.Hkv + h) * v.N + token;
            if (mass) mass[at] = 0.0f;
            if (pos) pos[at] = position;
        }
    }
    const int64_t entry = static_cast<int64_t>(s) * v.stride + page;
    const uint64_t off = v.off[entry];
    const int b = __builtin_amdgcn_readfirstlane(static_cast<int>(v.bits[entry]));
    if (!page_present(v, off, b)) return;
    uint8_t* record = v.pool + off;
    const uint64_t code_bytes = static_cast<uint64_t>(v.T) * kRow * b;       // per slab
    const uint64_t params = static_cast<uint64_t>(v.T) * v.groups;
    const uint32_t each = v.half_params ? 2 : 4;
#pragma unroll
    for (int u = 0; u < PPL; ++u) {
        const int p = (part * PPL + u) * 64 + lane;
        if (p >= all) continue;                                   // (whole heads: a group's lanes stay together)
        const int slab = layer * 2 * v.Hkv + p / kRow;
        uint8_t* codes = record + slab * code_bytes;
        const int piece = in_page * kRow + p % kRow;
        if (b == 16) {
            stream_store<true>(raw[u], reinterpret_cast<u4_t*>(codes) + piece);
            continue;
        }
        uint8_t* scale = record + v.slabs * code_bytes + slab * params * each;
        uint8_t* mn = scale + v.slabs * params * each;
        if (v.half_params) {
            if (b == 8) compress_piece<8, true>(raw[u], codes, scale, mn, piece, lpg_log2, lane);
            else if (b == 4) compress_piece<4, true>(raw[u], codes, scale, mn, piece, lpg_log2, lane);
            else compress_piece<2, true>(raw[u], codes, scale, mn, piece, lpg_log2, lane);
        } else {
            if (b == 8) compress_piece<8, false>(raw[u], codes, scale, mn, piece, lpg_log2, lane);
            else if (b == 4) compress_piece<4, false>(raw[u], codes, scale, mn, piece, lpg_log2, lane);
            else compress_piece<2, false>(raw[u], codes, scale, mn, piece, lpg_log2, lane);
        }
    }
}

}  // namespace kvs
