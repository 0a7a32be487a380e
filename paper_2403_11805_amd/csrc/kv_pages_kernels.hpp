// What the kernels that work on paged sequences share: the page table, the record sections of one layer, the rows of a step.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kv_quant_kernels.hpp"

namespace kvs {

struct PagesView {
    uint8_t* pool;
    const uint64_t* off;
    const uint8_t* bits;
    const int32_t* len;
    int32_t n_seqs, stride;
    int32_t N, T;                 // most tokens of a sequence, tokens per page
    int32_t Hkv, Hq;
    int32_t slabs;                // layers * 2 * kv_heads: fixes the record layout
    int32_t groups;               // D / G
    int32_t half_params;          // scale and mn in binary16 (format 3)
    uint32_t page_of_tile;        // ceil(2^32 / (T / 16)), 0 for T = 16: tile -> page by a multiplication
    uint64_t pool_bytes;
    uint64_t bit_bytes;           // of a record, per bit of its width
    uint64_t param_bytes;         // of a record's scales and minima (none at width 16)
};

// Whether a page of width b at `off` is there: the width is one the format has, its record lies in the pool.  Arithmetic
// only, no table and no branch: a wavefront looks up the pages of 64 tiles at once.
__device__ __forceinline__ bool page_present(const PagesView& v, uint64_t off, uint32_t b) {
    const uint64_t bytes = v.bit_bytes * b + (b == 16 ? 0u : v.param_bytes);
    const bool known = (__builtin_popcount(b) == 1) & ((b & 30u) != 0);
    return known & ((off & 15) == 0) & (off <= v.pool_bytes) & (v.pool_bytes - off >= bytes);
}

__device__ __forceinline__ int seq_len(const PagesView& v, int s) { return min(max(v.len[s], 0), v.N); }

// Codes, scales and minima of one slab of a record (for width 16 `codes` are the values).
struct SlabAt {
    uint64_t codes, scale, mn;    // byte offsets from the record's start
};
template <int D>
__device__ __forceinline__ SlabAt slab_at(const PagesView& v, int b, int slab) {
    const uint64_t code_bytes = static_cast<uint64_t>(v.T) * (D / 8) * static_cast<uint32_t>(b);
    const uint64_t param_bytes = static_cast<uint64_t>(v.T) * static_cast<uint32_t>(v.groups) * (v.half_params ? 2u : 4u);
    SlabAt a;
    a.codes = slab * code_bytes;
    a.scale = v.slabs * code_bytes + slab * param_bytes;
    a.mn = a.scale + v.slabs * param_bytes;
    return a;
}

// The new rows of a sequence: [first, first + count) of the step's n_rows, the list's bounds kept to whatever it says.
struct SeqRows {
    int first, count;
};
__device__ __forceinline__ SeqRows seq_rows(const int32_t* __restrict__ row_start, int s, int n_rows) {
    if (!row_start) return {s, s < n_rows ? 1 : 0};
    const int a = min(max(row_start[s], 0), n_rows), b = min(max(row_start[s + 1], a), n_rows);
    return {a, b - a};
}

// The sequence that row r belongs to (wave-uniform), -1 if none: the last s with row_start[s] <= r, found by all lanes
// together, 64 probes a step, so that up to 64 sequences take one load and 4096 two.
__device__ __forceinline__ int seq_of_row(const int32_t* __restrict__ row_start, int n_seqs, int r, int lane) {
    if (!row_start) return r < n_seqs ? r : -1;
    int lo = 0, n = n_seqs + 1;                       // entries [lo, lo + n) of the list are in question
    while (true) {
        const int step = (n + 63) >> 6, at = lo + lane * step;
        const bool in = lane * step < n;
        const bool le = in && row_start[in ? at : lo] <= r;
        const int cnt = __builtin_popcountll(__ballot(le));
        if (cnt == 0) return -1;                      // (an ascending list: in front of the first sequence)
        lo += (cnt - 1) * step;
        n = min(step, n - (cnt - 1) * step);
        if (step == 1) break;
    }
    return lo < n_seqs ? lo : -1;
}

}  // namespace kvs
