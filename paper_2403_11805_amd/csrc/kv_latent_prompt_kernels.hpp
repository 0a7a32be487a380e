// Latent attention in the expanded form, for many new rows at once: keys and values of every head are made from the latents,
//     k[h] = (c w_k[h], r),   v[h] = c w_v[h],
// by one product over all tokens (latent_project_kernel), and the new rows attend to them, 2 H (Dk + Dr + Dv) operations a (row, token).
//
// Room for the tokens: each sequence that has new rows gets whole tiles of 32 tokens, one sequence after the other, as far as the room
// reaches; a sequence that does not fit in gets none, and its rows are not computed.
#pragma once

#include "kv_latent_attend_kernels.hpp"

namespace kvs {

typedef float lf16_t __attribute__((ext_vector_type(16)));

constexpr int kPromptRows = 128;          // query rows of a workgroup

struct PromptGeom {
    int32_t n_rows, H;
    int32_t cap_tiles;                    // tiles of 32 tokens that there is room for
    int32_t row_tiles;                    // row tiles of the grid
    int64_t q_stride;
    float scale_log2e;
};

// What the first kernel leaves: where each sequence's token tiles and row tiles end.
struct PromptTable {
    int32_t* tile_end;                    // [n_seqs]
    int32_t* row_end;                     // [n_seqs]
};

__global__ __launch_bounds__(64) void latent_table_kernel(LatentView v, PromptGeom g, const int32_t* __restrict__ row_start, PromptTable t) {
    const int lane = threadIdx.x;
    int tiles = 0, row_tiles = 0;
    for (int s0 = 0; s0 < v.p.n_seqs; s0 += 64) {
        const int s = s0 + lane;
        SeqRows rows = {0, 0};
        int units = 0;
        if (s < v.p.n_seqs) {
            rows = seq_rows(row_start, s, g.n_rows);
            units = rows.count ? (seq_len(v.p, s) + kLatentTile - 1) / kLatentTile : 0;
        }
        // (in order: what does not fit in leaves its room to nobody)
        const int end = tiles + latent_prefix_sum(units);
        const bool fits = end <= g.cap_tiles;
        const int row_to = row_tiles + latent_prefix_sum(fits ? (rows.count + kPromptRows - 1) / kPromptRows : 0);
        if (s < v.p.n_seqs) {
            t.tile_end[s] = min(end, g.cap_tiles);
            t.row_end[s] = row_to;
        }
        tiles = min(__builtin_amdgcn_readlane(end, 63), g.cap_tiles + 1);
        row_tiles = min(__builtin_amdgcn_readlane(row_to, 63), 1 << 29);      // (more than any grid: lists that do not ascend must not overflow)
    }
}

// The first s with end[s] > x (ascending), -1 if there is none (wave-uniform).
__device__ __forceinline__ int first_behind(const int32_t* __restrict__ end, int n_seqs, int x, int lane) {
    int lo = 0, n = n_seqs;
    while (n > 64) {
        const int step = (n + 63) >> 6, i = min(lane * step + step - 1, n - 1);
        const int cnt = __builtin_popcountll(__ballot(lane * step < n && end[lo + i] <= x));
        lo += min(cnt * step, n);
        n = min(step, n - min(cnt * step, n));
    }
    if (n <= 0) return -1;
    const uint64_t any = __ballot(lane < n && end[lo + min(lane, n - 1)] > x);
    return any ? lo + __builtin_ctzll(any) : -1;
}

// A tile of 32 tokens from their pages: latents in the product's fragment order, position parts row-major, which halves' pages are there
// (bits 0 and 1); tokens that are not there are zeros.  40000 tokens of 8, 4 and 2 bits 27 us,
// 66 MB, 2.5 TB/s: not bound by HBM but by a lane's pieces, each of which waits for its own loads (the branches on width and parameter type in
// read_piece stand inside the loop) before the next is asked for.
template <int DC, int DR>
__global__ __launch_bounds__(256) void latent_gather_kernel(LatentView v, PromptGeom g, PromptTable t, int32_t lpg_log2, _Float16* __restrict__ latents,
                                                            _Float16* __restrict__ ropes, uint32_t* __restrict__ there) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    const int tile = static_cast<int>(blockIdx.x);
    const int s = __builtin_amdgcn_readfirstlane(first_behind(t.tile_end, v.p.n_seqs, tile, lane));
    if (s < 0) return;
    const int base = s ? t.tile_end[s - 1] : 0, n = seq_len(v.p, s);
    const int token0 = (tile - base) * kLatentTile + (wave >> 1) * 16;      // of this wavefront's half
    const int page = min(token0, v.p.N - 1) / v.p.T;
    const int64_t entry = static_cast<int64_t>(s) * v.p.stride + page;
    const uint64_t off = v.p.off[entry];
    const int b = v.p.bits[entry];
    const bool have = token0 < n && latent_present(v, off, b);
    __shared__ uint32_t halves[2];
    if (threadIdx.x % 128 == 0) halves[wave >> 1] = have ? 1u << (wave >> 1) : 0u;
    __syncthreads();
    if (threadIdx.x == 0) there[tile] = halves[0] | halves[1];
    // a lane has one token and every eighth piece, so that sixteen tokens' pieces are written side by side
    const int tk = (wave >> 1) * 16 + (lane & 15), token = token0 + (lane & 15);
    const bool ok = have && token < n;
    const uint8_t* record = v.p.pool + (have ? off : 0);
    const int in_page = token - page * v.p.T;
    const SlabAt slab = slab_at<DC>(v.p, b, v.layer);
    u4_t* to = reinterpret_cast<u4_t*>(latents) + static_cast<int64_t>(tile) * (kLatentTile * DC / 8);
    const int first = (wave & 1) * 4 + (lane >> 4);
#pragma unroll 4
    for (int p = first; p < DC / 8; p += 8) {
        u4_t x = {0u, 0u, 0u, 0u};
        if (ok) x = read_piece<DC>(v, record, slab, b, in_page * (DC / 8) + p, lpg_log2);
        to[p * kLatentTile + tk] = x;
    }
    if (first < DR / 8) {
        u4_t x = {0u, 0u, 0u, 0u};
        if (ok) x = reinterpret_cast<const u4_t*>(record + rope_at(v, b))[in_page * (DR / 8) + first];
        reinterpret_cast<u4_t*>(ropes)[(static_cast<int64_t>(tile) * kLatentTile + tk) * (DR / 8) + first] = x;
    }
}

// permutations of the 16-byte pieces of a row of values in LDS (see latent_swizzle; a read has four pieces of each of four rows)
__device__ __forceinline__ int value_swizzle(int token, int pieces) { return pieces >= 16 ? (token & 3) << 2 : (token & 2) << 1; }

// The operand of 16 rows x 32 columns from row-major LDS, eight rows in each half of the wavefront: rows 0..7 and 8..15, or (HALVES = 4: the order
// in which a product S^T leaves its probabilities) 0..3 and 8..11, 4..7 and 12..15.  A lane hands in four columns of one of its group's four rows
// and receives its column of all four.  columns_at(): the lane's place in the first four rows of its half.
template <int ROW_BYTES, int HALVES> __device__ __forceinline__ uint32_t columns_at(int lane) {
    const int row = HALVES * (lane >> 5) + ((lane & 15) >> 2), piece = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    return row * ROW_BYTES + ((piece ^ value_swizzle(row, ROW_BYTES / 16)) << 4) + (lane & 1) * 8;
}
template <int ROW_BYTES, int HALVES> __device__ __forceinline__ h8_t read_columns(const uint8_t* from) {
    const ls4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) ls4_t*)(from));
    const ls4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) ls4_t*)(from + (12 - HALVES) * ROW_BYTES));
    const lh4_t a = __builtin_bit_cast(lh4_t, lo), c = __builtin_bit_cast(lh4_t, hi);
    return h8_t{a[0], a[1], a[2], a[3], c[0], c[1], c[2], c[3]};
}

// Keys and values of all heads from the latents: a workgroup makes 128 tokens (four gathered tiles) x 256 columns, a wavefront 64 columns of them.
// 32 of the latents' dimensions a stage, both operands straight to LDS, two stages ahead: the tokens as they were gathered are an operand as it
// lies, rows of weights are transposed by the reads.  Two workgroups to a CU, so that one's results are written while the other multiplies: with 256
// tokens in 512 threads, one to a CU, 40000 tokens x 8192 columns took 1.26 times as long.  4096 tokens x 32768 columns 148 to 155 us, 0.9 PFLOP/s;
// 292 with results written from registers in pieces of 32 bytes and each column tile taken through all tokens.  Whole column tiles go to an XCD, so
// that few heads leave some without work: 256 columns (one head of 128 + 128) are made by one XCD of eight, 1024 by four, 2304 by five that have
// two tiles each but one; the measurements are of 32768 columns, where all have the same.
constexpr int kProjectTiles = 4, kProjectCols = 256;
template <int DC>
__global__ __launch_bounds__(256, 2) void latent_project_kernel(PromptTable t, int32_t n_seqs, int32_t N, int32_t col_tiles, int32_t token_tiles,
                                                             const _Float16* __restrict__ latents, const _Float16* __restrict__ w,
                                                             _Float16* __restrict__ kv) {
    constexpr int kStages = 3, kSteps = DC / 32, kTokens = kProjectTiles * 2048, kWeights = 32 * kProjectCols * 2, kStageBytes = kTokens + kWeights;
    __shared__ __attribute__((aligned(16))) uint8_t lds[kStages * kStageBytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    // Workgroups are dealt to the eight XCDs in turn: one of them has an eighth of the columns, which it takes through eight token tiles at a time.
    const int per_xcd = (col_tiles + 7) / 8, id = static_cast<int>(blockIdx.x) >> 3;
    const int eight = id / (per_xcd * 8) * 8, in_eight = id - eight * per_xcd, wide = min(8, token_tiles - eight);
    const int ct = (static_cast<int>(blockIdx.x) & 7) * per_xcd + in_eight / wide, tile0 = (eight + in_eight % wide) * kProjectTiles;
    const int tiles = t.tile_end[n_seqs - 1];
    if (ct >= col_tiles || tile0 >= tiles) return;
    const int n0 = ct * kProjectCols;
    const uint8_t* token_from = reinterpret_cast<const uint8_t*>(latents) + static_cast<int64_t>(min(tile0 + wave, tiles - 1)) * (kLatentTile * DC * 2);
    const uint8_t* weight_from = reinterpret_cast<const uint8_t*>(w) + n0 * 2;
    uint32_t weight_at[4];                                                  // (columns past the last repeat it)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = wave * 8 + 2 * i + (lane >> 5), piece = min((lane & 31) ^ value_swizzle(row, kProjectCols / 8), (N - n0) / 8 - 1);
        weight_at[i] = static_cast<uint32_t>(row) * static_cast<uint32_t>(N) * 2u + piece * 16;
    }
    auto fetch = [&](int step) __attribute__((always_inline)) {
        uint8_t* to = lds + step % kStages * kStageBytes;
        const uint32_t tokens = lds_place(to + wave * 2048), weights = lds_place(to + kTokens + wave * 4096);
        const uint8_t* from = token_from + step * 2048;
        to_lds(tokens, from, lane * 16);
        to_lds<1024>(tokens, from, lane * 16);
        const uint8_t* rows = weight_from + static_cast<int64_t>(step) * 32 * N * 2;
        to_lds(weights, rows, weight_at[0]);
        to_lds<1024>(weights, rows - 1024, weight_at[1]);                   // (the lanes' offsets are not negative: a row may be shorter than 512 bytes)
        to_lds<2048>(weights, rows - 2048, weight_at[2]);
        to_lds<3 * 1024>(weights, rows - 3 * 1024, weight_at[3]);
    };
    lf16_t acc[2][4];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[b][m][e] = 0.0f;
    const uint32_t cols_at = columns_at<kProjectCols * 2, 8>(lane);
    static_assert(kSteps >= kStages, "stages ahead");
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) fetch(i);
#pragma unroll
    for (int step = 0; step < kSteps; ++step) {
        // a wavefront's own six loads of this stage are done, and then everybody's; the stage that is fetched was used a step ago
        if (step + 1 < kSteps) asm volatile("s_waitcnt vmcnt(6) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (step + kStages - 1 < kSteps) fetch(step + kStages - 1);
        const uint8_t* at = lds + step % kStages * kStageBytes;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            h8_t wf[2], cf[4];
#pragma unroll
            for (int b = 0; b < 2; ++b)
                wf[b] = read_columns<kProjectCols * 2, 8>(at + kTokens + (cols_at ^ ((2 * wave + b) << 6)) + k * (16 * kProjectCols * 2));
#pragma unroll
            for (int m = 0; m < 4; ++m) cf[m] = *reinterpret_cast<const h8_t*>(at + m * 2048 + k * 1024 + lane * 16);
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int b = 0; b < 2; ++b) acc[b][m] = __builtin_amdgcn_mfma_f32_32x32x16_f16(wf[b], cf[m], acc[b][m], 0, 0, 0);
        }
    }
    // acc[b][m][e]: column 32 b + 8 (e / 4) + 4 half + e % 4 of token lane % 32.  Through LDS, so that whole rows are written (pieces of 16 bytes
    // change places by the token: a wavefront writes one piece of 32 tokens).
    const int half = lane >> 5, l32 = lane & 31;
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                lh4_t x;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = static_cast<_Float16>(acc[b][m][4 * j + e]);
                const int piece = wave * 8 + 4 * b + j;
                *reinterpret_cast<lh4_t*>(lds + (32 * m + l32) * (kProjectCols * 2) + ((piece ^ l32) << 4) + half * 8) = x;
            }
    __syncthreads();
#pragma unroll 4
    for (int i = 0; i < 16; ++i) {
        const int token = 8 * i + 2 * wave + half;
        if (tile0 + token / kLatentTile < tiles && n0 + l32 * 8 < N) {
            const u4_t x = *reinterpret_cast<const u4_t*>(lds + token * (kProjectCols * 2) + ((l32 ^ (token & 31)) << 4));
            *reinterpret_cast<u4_t*>(kv + (static_cast<int64_t>(tile0) * kLatentTile + token) * N + n0 + l32 * 8) = x;
        }
    }
}

// Causal attention of the new rows to the expanded keys and values: a workgroup has 128 rows of one head, a wavefront 32 of them, and takes
// 64 tokens a turn, two independent products S^T = K Q^T of 32 tokens each.  Keys and values go straight to LDS, the next turn's while this one's
// are used; a turn makes the next one's logits beside its own probabilities.  Probabilities are rounded to fp16, and their sum is that of the
// rounded ones, so that it has no part in the result's error.  (The last turn of a sequence may reach 32 tokens past its room; nobody sees them.)
// Two workgroups to a CU, 242 of 256 registers.  One prompt of 4096 tokens and 128 heads, 0.69 TFLOP, takes 1.36 to 1.43 M cycles, in 47 to 49 % of
// which the matrix pipe is busy, and 780 to 880 us at 1.56 to 1.76 GHz, the clock that the chip's power leaves (744 at best, when it is cool).  LDS gives a
// wavefront 56 KB a turn, a quarter of its rate.  Not all of the idle cycles are explained: the compiler waits for the query rows where they are first
// used, which is inside the walk, so that the first of every two turns waits between its products (vmcnt 11 to 0) for the keys and values that it has
// just asked for; what that costs is not measured.
// Tokens are not divided: H * (row tiles) workgroups walk a context each from its beginning, and few rows of few heads behind a long one leave most
// CUs idle.
constexpr int kPromptTile = 64, kPromptHeads = 4;
template <int DK, int DR, int DV>
__global__ __launch_bounds__(256, 2) void latent_prompt_kernel(LatentView v, PromptGeom g, PromptTable t, const int32_t* __restrict__ row_start,
                                                               const _Float16* __restrict__ q, const _Float16* __restrict__ kv,
                                                               const _Float16* __restrict__ ropes, const uint32_t* __restrict__ there,
                                                               _Float16* __restrict__ out) {
    constexpr int kRopeAt = kPromptTile * DK * 2, kValueAt = kRopeAt + kPromptTile * DR * 2, kTileBytes = kValueAt + kPromptTile * DV * 2;
    constexpr int KS = DK / 16, KR = DR / 16, VB = DV / 32;
    __shared__ __attribute__((aligned(16))) uint8_t lds[2 * kTileBytes];
    const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    // Workgroups are dealt to the eight XCDs in turn: those of a head go to one of them, whose L2 then holds its keys and values.  Four heads at a
    // time, the longest rows first: with the heads one after the other the last one's longest rows would run when all else is done.
    const int n_xcd = g.H % 8 == 0 ? 8 : 1, per_xcd = g.H / n_xcd;
    const int id = static_cast<int>(blockIdx.x) / n_xcd, four = id / (g.row_tiles * kPromptHeads) * kPromptHeads;
    const int heads = min(kPromptHeads, per_xcd - four), in_four = id - four * g.row_tiles;
    const int h = (four + in_four % heads) * n_xcd + static_cast<int>(blockIdx.x) % n_xcd, rt = g.row_tiles - 1 - in_four / heads;
    const int s = __builtin_amdgcn_readfirstlane(first_behind(t.row_end, v.p.n_seqs, rt, lane));
    if (s < 0) return;
    const int rt_in = rt - (s ? t.row_end[s - 1] : 0), base = s ? t.tile_end[s - 1] : 0;
    const int n = seq_len(v.p, s);
    const SeqRows rows = seq_rows(row_start, s, g.n_rows);
    const int row0 = rt_in * kPromptRows, m = row0 + wave * 32 + l32;
    const bool ok = m < rows.count;
    const int behind = n - rows.count;                                     // the token of row 0
    const int pos = ok ? behind + m : -1;
    const bool idle = row0 + wave * 32 >= rows.count;                       // (a wavefront without rows)
    const int min_pos = idle ? -1 : behind + row0 + wave * 32, max_pos = idle ? -1 : behind + min(row0 + wave * 32 + 31, rows.count - 1);
    const int end_pos = behind + min(row0 + kPromptRows, rows.count) - 1;  // of the workgroup's last row
    const int n_tiles = end_pos < 0 ? 0 : end_pos / kPromptTile + 1;
    h8_t qf[KS + KR];
    {
        const _Float16* from = q + (rows.first + (ok ? m : 0)) * g.q_stride + h * (DK + DR) + 8 * half;
#pragma unroll
        for (int k = 0; k < KS + KR; ++k) qf[k] = *reinterpret_cast<const h8_t*>(from + 16 * k);
    }
    const uint32_t kv_row = static_cast<uint32_t>(g.H) * (DK + DV) * 2;
    const uint8_t* keys = reinterpret_cast<const uint8_t*>(kv) + static_cast<int64_t>(base) * kLatentTile * kv_row + h * ((DK + DV) * 2);
    const uint8_t* rope = reinterpret_cast<const uint8_t*>(ropes) + static_cast<int64_t>(base) * kLatentTile * (DR * 2);
    // permutation of the pieces of a row of keys (a read has one piece of 32 tokens)
    auto key_swz = [](int token, int pieces) __attribute__((always_inline)) {
        return pieces == 16 ? token & 15 : pieces == 8 ? (token >> 1) & 7 : (token >> 2) & 3;
    };
    // Where a lane's piece lies in memory, for the loads of a wavefront's quarter of the tile, one after the other in LDS (1 KB each, which the
    // load's own offset adds on both sides).
    constexpr int kk = DK / 8, kv_ = DV / 8, kr = DR / 8, kRopeLoads = DR / 32;
    uint32_t key_at_[DK / 32], rope_at_[kRopeLoads], value_at_[DV / 32];
#pragma unroll
    for (int i = 0; i < DK / 32; ++i) {
        const int p = (wave * (DK / 32) + i) * 64 + lane, tk = p / kk;
        key_at_[i] = tk * kv_row + ((p % kk ^ key_swz(tk, kk)) << 4) - i * 1024;
    }
#pragma unroll
    for (int i = 0; i < kRopeLoads; ++i) {
        const int p = (wave * kRopeLoads + i) * 64 + lane, tk = p / kr;
        rope_at_[i] = static_cast<uint32_t>(tk * (DR * 2) + ((p % kr ^ key_swz(tk, kr)) << 4) - i * 1024);
    }
#pragma unroll
    for (int i = 0; i < DV / 32; ++i) {
        const int p = (wave * (DV / 32) + i) * 64 + lane, tk = p / kv_;
        value_at_[i] = tk * kv_row + DK * 2 + ((p % kv_ ^ value_swizzle(tk, kv_)) << 4) - i * 1024;
    }
    auto fetch_keys = [&](int tile) __attribute__((always_inline)) {
        uint8_t* to = lds + (tile & 1) * kTileBytes;
        const uint8_t* from = keys + static_cast<int64_t>(tile) * (kPromptTile * static_cast<int64_t>(kv_row));
        const uint8_t* rope_at = rope + static_cast<int64_t>(tile) * (kPromptTile * DR * 2);
        const uint32_t place = lds_place(to + wave * (DK * 32));
        to_lds(place, from, key_at_[0]);
        to_lds<1024>(place, from, key_at_[1]);
        if constexpr (DK == 128) {
            to_lds<2048>(place, from, key_at_[2]);
            to_lds<3 * 1024>(place, from, key_at_[3]);
        }
        const uint32_t place1 = lds_place(to + kRopeAt + wave * (DR * 32));
        to_lds(place1, rope_at, rope_at_[0]);
        if constexpr (DR == 64) to_lds<1024>(place1, rope_at, rope_at_[1]);
    };
    auto fetch_values = [&](int tile) __attribute__((always_inline)) {
        const uint8_t* from = keys + static_cast<int64_t>(tile) * (kPromptTile * static_cast<int64_t>(kv_row));
        const uint32_t place2 = lds_place(lds + (tile & 1) * kTileBytes + kValueAt + wave * (DV * 32));
        to_lds(place2, from, value_at_[0]);
        to_lds<1024>(place2, from, value_at_[1]);
        if constexpr (DV == 128) {
            to_lds<2048>(place2, from, value_at_[2]);
            to_lds<3 * 1024>(place2, from, value_at_[3]);
        }
    };
    lf16_t o[VB];
#pragma unroll
    for (int b = 0; b < VB; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[b][e] = 0.0f;
    float ref = -INFINITY, sum = 0.0f;
    // sc[i][e]: token 32 i + 8 (e / 4) + 4 half + e % 4 against this lane's row
    auto key_read = [&](const uint8_t* at, int ln, int k, int i) __attribute__((always_inline)) {
        const int tk = ln & 31, hf = ln >> 5;
        const uint32_t key_at = tk * (DK * 2) + ((hf ^ key_swz(tk, kk)) << 4), rope_key_at = tk * (DR * 2) + ((hf ^ key_swz(tk, kr)) << 4);
        const uint8_t* p = k < KS ? at + (key_at ^ (k << 5)) + i * (32 * DK * 2) : at + kRopeAt + (rope_key_at ^ ((k - KS) << 5)) + i * (32 * DR * 2);
        return *reinterpret_cast<const h8_t*>(p);
    };
    auto value_read = [&](const uint8_t* at, int ln, int st, int b) __attribute__((always_inline)) {
        return read_columns<DV * 2, 4>(at + kValueAt + (columns_at<DV * 2, 4>(ln) ^ (b << 6)) + st * (16 * DV * 2));
    };
    auto zero = [&](lf16_t (&sc)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) sc[i][e] = 0.0f;
    };
    auto logits = [&](int tile, lf16_t (&sc)[2]) __attribute__((always_inline)) {
        const uint8_t* at = lds + (tile & 1) * kTileBytes;
        int ln = lane;
        asm volatile("" : "+v"(ln));
        zero(sc);
#pragma unroll
        for (int k = 0; k < KS + KR; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i) sc[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(key_read(at, ln, k, i), qf[k], sc[i], 0, 0, 0);
    };
    const uint32_t* have_at = there + base;
    auto have_of = [&](int tile) __attribute__((always_inline)) { return tile < n_tiles ? have_at[2 * tile] | have_at[2 * tile + 1] << 2 : 0u; };
    uint32_t have_next = have_of(0);
    lf16_t sc0[2], sc1[2];
    if (n_tiles > 0) {
        fetch_keys(0);
        fetch_values(0);
        if (n_tiles > 1) fetch_keys(1);
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        logits(0, sc0);
    }
    // A turn: the next tile's logits, this one's probabilities and values.  EDGE, if some of its tokens may be behind some of the wavefront's rows.
    auto turn = [&](int tile, auto EDGE, lf16_t (&sc)[2], lf16_t (&next)[2]) __attribute__((always_inline)) {
        constexpr bool edge = decltype(EDGE)::value;
        const uint32_t have = have_next;                                    // of the four times 16 tokens
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (tile + 1 < n_tiles) {
            if (tile + 2 < n_tiles) fetch_keys(tile + 2);
            fetch_values(tile + 1);
        }
        have_next = have_of(tile + 1);
        const uint8_t* at = lds + (tile & 1) * kTileBytes;
        const int token0 = tile * kPromptTile;
        if (edge && token0 > max_pos) return;                              // (uniform; behind all of this wavefront's rows)
        int ln = lane;
        asm volatile("" : "+v"(ln));
        const int hf = ln >> 5;
        uint64_t bad = 0u;
        if constexpr (edge) {
            // Values that are not finite must not reach rows that do not see their token, whose probability of 0 does not hold them off: they
            // are left out below, and rows that see them are NaN.
            bool found = false;
#pragma unroll 1
            for (int p = 0; p < DV / 8; ++p) {
                const u4_t y = *reinterpret_cast<const u4_t*>(at + kValueAt + ln * (DV * 2) + (p << 4));
#pragma unroll
                for (int e = 0; e < 4; ++e) found |= (y[e] & 0x7c00u) == 0x7c00u || (y[e] & 0x7c000000u) == 0x7c000000u;
            }
            bad = __ballot(found);
        }
        if (edge || have != 15u) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int tk = 32 * i + 8 * (e / 4) + 4 * hf + e % 4;
                    if (bad >> tk & 1) sc[i][e] = NAN;
                    if (!(have >> (2 * i + e / 8) & 1) || token0 + tk > pos) sc[i][e] = -INFINITY;
                }
        }
        // (the instruction itself: fmaxf() takes two, and one for each operand besides)
        float top = sc[0][0];
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
            const float x = sc[e / 16][e % 16], y = sc[e / 16][e % 16 + 1];
            asm("v_max3_f32 %0, %0, %1, %2" : "+v"(top) : "v"(x), "v"(y));
        }
        top *= g.scale_log2e;
        if (__any(top > ref + kLatentSlack)) {                              // (rare: the reference has room)
            const float hi = xhalf_max(top);
            const float to = hi > ref + kLatentSlack ? hi - kLatentTop : ref;
            const float alpha = to == ref ? 1.0f : __builtin_amdgcn_exp2f(ref - to);
            ref = to;
            sum *= alpha;
#pragma unroll
            for (int b = 0; b < VB; ++b) o[b] *= alpha;
        }
        const float r = ref == -INFINITY ? 0.0f : ref;
        h8_t p[4];
        auto weigh = [&](int pair) __attribute__((always_inline)) {
            typedef float f2_t __attribute__((ext_vector_type(2)));
            typedef _Float16 h2_t __attribute__((ext_vector_type(2)));
            const int i = pair / 8, e = pair % 8 * 2;
            const f2_t x = {__builtin_amdgcn_exp2f(__builtin_fmaf(sc[i][e], g.scale_log2e, -r)),
                            __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i][e + 1], g.scale_log2e, -r))};
            const h2_t y = __builtin_convertvector(x, h2_t), ones = {static_cast<_Float16>(1.0f), static_cast<_Float16>(1.0f)};
            sum = __builtin_amdgcn_fdot2(y, ones, sum, false);              // (of the rounded ones, which the values are weighted with)
            p[2 * i + e / 8][e % 8] = y[0];
            p[2 * i + e / 8][e % 8 + 1] = y[1];
        };
        constexpr int kSteps = KS + KR, kFrags = 4 * VB, kAheadKeys = 2, kAheadValues = 4;
        if constexpr (!edge) {
            // In this order: reads of LDS ahead of the products that they are for, probabilities between the products.
            const uint8_t* next_at = lds + (tile + 1 & 1) * kTileBytes;
            h8_t kf[kSteps][2], vf[kFrags];
            auto read_keys = [&](int k) __attribute__((always_inline)) {
                kf[k][0] = key_read(next_at, ln, k, 0);
                kf[k][1] = key_read(next_at, ln, k, 1);
            };
            zero(next);
#pragma unroll
            for (int k = 0; k < kAheadKeys; ++k) read_keys(k);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
                if (k + kAheadKeys < kSteps)
                    read_keys(k + kAheadKeys);
                else
#pragma unroll
                    for (int f = 0; f < kAheadValues / kAheadKeys; ++f) {
                        const int at_f = (k + kAheadKeys - kSteps) * (kAheadValues / kAheadKeys) + f;
                        vf[at_f] = value_read(at, ln, at_f / VB, at_f % VB);
                    }
                next[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[k][0], qf[k], next[0], 0, 0, 0);
                next[1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[k][1], qf[k], next[1], 0, 0, 0);
#pragma unroll
                for (int pair = k * 16 / kSteps; pair < (k + 1) * 16 / kSteps; ++pair) weigh(pair);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int f = 0; f < kFrags; ++f) {
                if (f + kAheadValues < kFrags) vf[f + kAheadValues] = value_read(at, ln, (f + kAheadValues) / VB, (f + kAheadValues) % VB);
                o[f % VB] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[f], p[f / VB], o[f % VB], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            if (token0 + kPromptTile <= max_pos) logits(tile + 1, next);
#pragma unroll
            for (int pair = 0; pair < 16; ++pair) weigh(pair);
#pragma unroll
            for (int f = 0; f < kFrags; ++f) {
                u4_t y = __builtin_bit_cast(u4_t, value_read(at, ln, f / VB, f % VB));
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if ((y[e] & 0x7c00u) == 0x7c00u) y[e] &= 0xffff0000u;
                    if ((y[e] & 0x7c000000u) == 0x7c000000u) y[e] &= 0xffffu;
                }
                o[f % VB] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8_t, y), p[f / VB], o[f % VB], 0, 0, 0);
            }
        }
    };
    const int clear = min(n_tiles, (min_pos + 1) / kPromptTile);             // turns whose tokens all of the rows see
    int tile = 0;
    for (; tile + 1 < clear; tile += 2) {
        turn(tile, std::false_type{}, sc0, sc1);
        turn(tile + 1, std::false_type{}, sc1, sc0);
    }
    for (; tile < n_tiles; ++tile) {
        turn(tile, std::true_type{}, sc0, sc1);
        sc0[0] = sc1[0];
        sc0[1] = sc1[1];
    }
    if (ok) {
        const float all = xhalf_sum(sum), inv = all > 0.0f ? 1.0f / all : all;     // a row that sees nothing: zeros; NaN stays
        _Float16* to = out + (static_cast<int64_t>(rows.first + m) * g.H + h) * DV;
#pragma unroll
        for (int b = 0; b < VB; ++b)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                lh4_t x;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = static_cast<_Float16>(o[b][4 * j + e] * inv);
                *reinterpret_cast<lh4_t*>(to + 32 * b + 8 * j + 4 * half) = x;
            }
    }
}

}  // namespace kvs
