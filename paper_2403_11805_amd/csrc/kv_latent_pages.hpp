// Latent caches: the rows of one layer of a record, and the kernels that write and read them.
//
// A token has one row per layer, a latent of DC numbers and a position part of Dr, shared by all heads.  A record of width b holds, one
// layer after the other in each section: codes [T][DC * b / 8] (b = 16: the latents), scales and minima [T][DC / G] (b < 16), position
// parts [T][Dr] in fp16.  That is one slab per layer of the record format of the per-head caches, with the position parts behind it.
#pragma once

#include <type_traits>

#include "kv_pages_kernels.hpp"

namespace kvs {

struct LatentView {
    PagesView p;                  // slabs: the layers; bit_bytes, param_bytes: of all layers
    uint64_t rope_bytes;          // of a record's position parts
    int32_t Dr, layer;
};

// Whether a page of width b at `off` is there (page_present with the position parts).
__device__ __forceinline__ bool latent_present(const LatentView& v, uint64_t off, uint32_t b) {
    const uint64_t bytes = v.p.bit_bytes * b + (b == 16 ? 0u : v.p.param_bytes) + v.rope_bytes;
    const bool known = (__builtin_popcount(b) == 1) & ((b & 30u) != 0);
    return known & ((off & 15) == 0) & (off <= v.p.pool_bytes) & (v.p.pool_bytes - off >= bytes);
}

// Byte offset of the layer's position parts from a record's start.
__device__ __forceinline__ uint64_t rope_at(const LatentView& v, uint32_t b) {
    return v.p.bit_bytes * b + (b == 16 ? 0u : v.p.param_bytes) + static_cast<uint64_t>(v.layer) * (v.p.T * v.Dr * 2);
}

// Where the row of a token lies: its page's record and width (0: nowhere), its place in the page.
struct RowPlace {
    uint64_t off;
    int b, in_page;
};
// Row r of a step (wave-uniform); `s` the sequence of the row in front of it (-1: not known), which is tried first.
__device__ __forceinline__ RowPlace row_place(const LatentView& v, const int32_t* __restrict__ row_start, int n_rows, int r, int& s, int lane) {
    SeqRows rows = {0, 0};
    if (s >= 0) rows = seq_rows(row_start, s, n_rows);
    if (s < 0 || r >= rows.first + rows.count) {
        s = __builtin_amdgcn_readfirstlane(seq_of_row(row_start, v.p.n_seqs, r, lane));
        if (s < 0) return {0, 0, 0};
        rows = seq_rows(row_start, s, n_rows);
    }
    const int token = seq_len(v.p, s) - rows.count + (r - rows.first);
    if (token < 0 || r < rows.first || r >= rows.first + rows.count) return {0, 0, 0};
    const int page = token / v.p.T;
    const int64_t entry = static_cast<int64_t>(s) * v.p.stride + page;
    const uint64_t off = v.p.off[entry];
    const int b = v.p.bits[entry];
    return {off, latent_present(v, off, b) ? b : 0, token - page * v.p.T};
}

// Whether rows r .. last lie in one page, r's (whose place is `at` and whose sequence s).
__device__ __forceinline__ bool rows_in_page(const LatentView& v, const int32_t* __restrict__ row_start, int n_rows, int last, int r, int s,
                                             const RowPlace& at) {
    if (at.b == 0) return false;
    const SeqRows rows = seq_rows(row_start, s, n_rows);
    return last < rows.first + rows.count && at.in_page + (last - r) < v.p.T;
}

// A wavefront has kSide rows side by side (two where a row is half a wavefront wide), UNITS times.
template <int DC> struct LatentLanes {
    static constexpr int kPieces = DC / 8, kSide = 64 / kPieces;
};

// Append: rows of new tokens into their pages.  Each row is read once and written once, 16 bytes a lane.  Bound by HBM where there are many and
// their pages are fp16 (105000 rows of 1152 bytes 47.5 us, 5.1 TB/s, where a large copy reaches 4.9; 37 us while the rows still lie in the chip's last
// cache), by the chain from row to sequence to length to page where there are few (64 rows 3.0 us).  Into pages of 8, 4 and 2 bits 69000 rows take 34 us;
// with four rows a wavefront the kernel is 91 to 97 KB of code, three widths, two types of parameters, four rows and two ways each, more than the
// instruction cache of 64 KB, and what that costs beside the arithmetic is not measured.
template <int DC, int UNITS>
__global__ __launch_bounds__(256) void latent_append_kernel(LatentView v, const _Float16* __restrict__ c, int64_t c_stride,
                                                            const _Float16* __restrict__ r, int64_t r_stride, int32_t n_rows,
                                                            int32_t lpg_log2, const int32_t* __restrict__ row_start) {
    using L = LatentLanes<DC>;
    const int lane = threadIdx.x & 63, piece = lane % L::kPieces, side = lane / L::kPieces;
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    const int64_t first = (static_cast<int64_t>(blockIdx.x) * 4 + wave) * (UNITS * L::kSide);
    if (first >= n_rows) return;
    const int r0 = static_cast<int>(first);
    const bool has_rope = piece < v.Dr / 8;
    u4_t raw[UNITS], rope[UNITS];
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        const int row = min(r0 + u * L::kSide + side, n_rows - 1);
        raw[u] = *reinterpret_cast<const u4_t*>(c + row * c_stride + piece * 8);
        if (has_rope) rope[u] = *reinterpret_cast<const u4_t*>(r + row * r_stride + piece * 8);
    }
    auto store = [&](int u, const RowPlace& at) __attribute__((always_inline)) {
        uint8_t* record = v.p.pool + at.off;
        const SlabAt slab = slab_at<DC>(v.p, at.b, v.layer);
        const int p = at.in_page * L::kPieces + piece;
        if (at.b == 16) stream_store<true>(raw[u], reinterpret_cast<u4_t*>(record + slab.codes) + p);
        else if (v.p.half_params) {
            if (at.b == 8) compress_piece<8, true>(raw[u], record + slab.codes, record + slab.scale, record + slab.mn, p, lpg_log2, lane);
            else if (at.b == 4) compress_piece<4, true>(raw[u], record + slab.codes, record + slab.scale, record + slab.mn, p, lpg_log2, lane);
            else compress_piece<2, true>(raw[u], record + slab.codes, record + slab.scale, record + slab.mn, p, lpg_log2, lane);
        } else {
            if (at.b == 8) compress_piece<8, false>(raw[u], record + slab.codes, record + slab.scale, record + slab.mn, p, lpg_log2, lane);
            else if (at.b == 4) compress_piece<4, false>(raw[u], record + slab.codes, record + slab.scale, record + slab.mn, p, lpg_log2, lane);
            else compress_piece<2, false>(raw[u], record + slab.codes, record + slab.scale, record + slab.mn, p, lpg_log2, lane);
        }
        if (has_rope) stream_store<true>(rope[u], reinterpret_cast<u4_t*>(record + rope_at(v, at.b)) + at.in_page * (v.Dr / 8) + piece);
    };
    int s = -1;
    if constexpr (UNITS > 1) {
        const RowPlace at = row_place(v, row_start, n_rows, r0, s, lane);
        const int last = min(r0 + UNITS * L::kSide, n_rows) - 1;
        if (rows_in_page(v, row_start, n_rows, last, r0, s, at)) {          // (most: one look at the tables)
#pragma unroll
            for (int u = 0; u < UNITS; ++u)
                if (r0 + u * L::kSide + side <= last) store(u, {at.off, at.b, at.in_page + u * L::kSide + side});
            return;
        }
    }
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        RowPlace at = {0, 0, 0};
#pragma unroll
        for (int i = 0; i < L::kSide; ++i) {
            const int row = r0 + u * L::kSide + i;
            if (row >= n_rows) break;
            const RowPlace one = row_place(v, row_start, n_rows, row, s, lane);
            if (side == i) at = one;
        }
        if (at.b != 0) store(u, at);
    }
}

// Parameter i of a section in binary16 or binary32.
__device__ __forceinline__ float latent_param(const uint8_t* section, int64_t i, bool half) {
    return half ? static_cast<float>(reinterpret_cast<const _Float16*>(section)[i]) : reinterpret_cast<const float*>(section)[i];
}

// Piece p (eight latents) of a record's layer as fp16, as a Load gives it.
template <int DC>
__device__ __forceinline__ u4_t read_piece(const LatentView& v, const uint8_t* record, const SlabAt& slab, int b, int p, int lpg_log2) {
    if (b == 16) return stream_load<true>(reinterpret_cast<const u4_t*>(record + slab.codes) + p);
    const float sc = latent_param(record + slab.scale, p >> lpg_log2, v.p.half_params);
    const float mn = latent_param(record + slab.mn, p >> lpg_log2, v.p.half_params);
    if (b == 8) return dequantise_piece<8>(load_codes<8>(record + slab.codes, p), sc, mn);
    if (b == 4) return dequantise_piece<4>(load_codes<4>(record + slab.codes, p), sc, mn);
    return dequantise_piece<2>(load_codes<2>(record + slab.codes, p), sc, mn);
}

// Read: the rows of a step from their pages, as fp16; rows that have no place, or one in an absent page, are left as they are.  24 contexts of up to
// 16384 tokens in pages of every width, parameters in binary16, 112 us, 3.2 TB/s.  Bound by trips to memory that wait for each other: a parameter's
// type is looked at where it is read, and a binary16 one is waited for there (latent_param), so that two rows of packed latents take four such trips
// besides those of the tables, each with whatever else the wavefront has asked for.
template <int DC, int UNITS>
__global__ __launch_bounds__(256) void latent_read_kernel(LatentView v, _Float16* __restrict__ c, int64_t c_stride, _Float16* __restrict__ r,
                                                          int64_t r_stride, int32_t n_rows, int32_t lpg_log2,
                                                          const int32_t* __restrict__ row_start) {
    using L = LatentLanes<DC>;
    const int lane = threadIdx.x & 63, piece = lane % L::kPieces, side = lane / L::kPieces;
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    const int64_t first = (static_cast<int64_t>(blockIdx.x) * 4 + wave) * (UNITS * L::kSide);
    if (first >= n_rows) return;
    const int r0 = static_cast<int>(first);
    const bool has_rope = piece < v.Dr / 8;
    int s = -1;
    if constexpr (UNITS > 1) {
        const RowPlace at = row_place(v, row_start, n_rows, r0, s, lane);
        const int last = min(r0 + UNITS * L::kSide, n_rows) - 1;
        if (rows_in_page(v, row_start, n_rows, last, r0, s, at)) {          // (most: one look at the tables; rows of fp16 are asked for all at once)
            const uint8_t* record = v.p.pool + at.off;
            const SlabAt slab = slab_at<DC>(v.p, at.b, v.layer);
            auto move = [&](auto WIDTH) __attribute__((always_inline)) {
                u4_t rope[UNITS], x[UNITS];
#pragma unroll
                for (int u = 0; u < UNITS; ++u) {
                    const int in_page = at.in_page + min(u * L::kSide + side, last - r0);
                    if (has_rope) rope[u] = stream_load<true>(reinterpret_cast<const u4_t*>(record + rope_at(v, at.b)) + in_page * (v.Dr / 8) + piece);
                    x[u] = read_piece<DC>(v, record, slab, decltype(WIDTH)::value, in_page * L::kPieces + piece, lpg_log2);
                }
#pragma unroll
                for (int u = 0; u < UNITS; ++u) {
                    const int row = r0 + u * L::kSide + side;
                    if (row > last) break;
                    *reinterpret_cast<u4_t*>(c + row * c_stride + piece * 8) = x[u];
                    if (has_rope) *reinterpret_cast<u4_t*>(r + row * r_stride + piece * 8) = rope[u];
                }
            };
            if (at.b == 16) move(std::integral_constant<int, 16>{});
            else if (at.b == 8) move(std::integral_constant<int, 8>{});
            else if (at.b == 4) move(std::integral_constant<int, 4>{});
            else move(std::integral_constant<int, 2>{});
            return;
        }
    }
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        RowPlace at = {0, 0, 0};
#pragma unroll
        for (int i = 0; i < L::kSide; ++i) {
            const int row = r0 + u * L::kSide + i;
            if (row >= n_rows) break;
            const RowPlace one = row_place(v, row_start, n_rows, row, s, lane);
            if (side == i) at = one;
        }
        if (at.b != 0) {
            const int row = r0 + u * L::kSide + side;
            const uint8_t* record = v.p.pool + at.off;
            const SlabAt slab = slab_at<DC>(v.p, at.b, v.layer);
            u4_t rope;
            if (has_rope) rope = stream_load<true>(reinterpret_cast<const u4_t*>(record + rope_at(v, at.b)) + at.in_page * (v.Dr / 8) + piece);
            const u4_t x = read_piece<DC>(v, record, slab, at.b, at.in_page * L::kPieces + piece, lpg_log2);
            *reinterpret_cast<u4_t*>(c + row * c_stride + piece * 8) = x;
            if (has_rope) *reinterpret_cast<u4_t*>(r + row * r_stride + piece * 8) = rope;
        }
    }
}

}  // namespace kvs
