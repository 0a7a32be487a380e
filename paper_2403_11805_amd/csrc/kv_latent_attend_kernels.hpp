// Latent attention in the absorbed form: queries are taken to the latents' space, where one row a token is key and value of all heads,
//     q'[h] = w_k[h] q[h],   s = (q'[h] c + q_r[h] r) / sqrt(Dk + Dr),   out[h] = w_v[h]^T (softmax(s) c),
// so that a token's row is read once for all heads and the wide products are those with the cache, 2 H (2 DC + Dr) operations a (query
// row, token), instead of the 2 DC H (Dk + Dv) a token that making its keys and values takes.  Three launches: latent_absorb_kernel (q' of
// the new rows, and how the work is divided), latent_attend_kernel (shares of the attention), latent_project_kernel (the shares joined,
// the values made).
#pragma once

#include "kv_lane_ops.hpp"
#include "kv_latent_pages.hpp"
#include "kv_launch_rules.hpp"

namespace kvs {

typedef float lf4_t __attribute__((ext_vector_type(4)));
typedef _Float16 lh4_t __attribute__((ext_vector_type(4)));
typedef short ls4_t __attribute__((ext_vector_type(4)));

constexpr int kLatentTile = 32;            // tokens of a tile
constexpr float kLatentTop = 7.0f;         // a row's reference is set 2^7 below its largest logit so far ...
constexpr float kLatentSlack = 15.0f;      // ... and moves when a logit passes 2^15 above it: probabilities stay in fp16's range
constexpr int kZeroBytes = 2048;           // of zeros, which stand for rows that are not there

struct LatentGeom {
    int32_t n_rows, max_rows;
    int32_t H, Dk, Dv;
    int32_t tile_log2;                     // query rows of a tile
    int32_t row_tiles;                     // most tiles of a sequence
    int32_t groups;                        // workgroups that share the attention
    int64_t q_stride;
    float scale_log2e;                     // log2(e) / sqrt(Dk + Dr)
};

// Where the work lies in a line of places, tile by tile, row tile by row tile, sequence by sequence: the places in front of a row tile
// and of a workgroup's run, then where each sequence's work ends.
struct LatentLine {
    int32_t round, cost, run, unused;
};
struct LatentSeq {
    int n, first, count, rows, row_tiles, units;     // tokens; new rows; query rows, tiles of them; tiles of tokens
};
__device__ __forceinline__ LatentSeq latent_seq(const LatentView& v, const LatentGeom& g, const int32_t* __restrict__ row_start, int s) {
    LatentSeq w = {0, 0, 0, 0, 0, 0};
    if (s < v.p.n_seqs) {
        w.n = seq_len(v.p, s);
        const SeqRows rows = seq_rows(row_start, s, g.n_rows);
        w.first = rows.first;
        w.count = rows.count;
        w.rows = min(w.count, g.max_rows) * g.H;
        w.row_tiles = (w.rows + (1 << g.tile_log2) - 1) >> g.tile_log2;
        w.units = (w.n + kLatentTile - 1) / kLatentTile;
    }
    return w;
}

__device__ __forceinline__ int latent_prefix_sum(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    return x;
}

// One wavefront makes the line.
__device__ __forceinline__ void latent_make_line(const LatentView& v, const LatentGeom& g, const int32_t* __restrict__ row_start,
                                                 int32_t* __restrict__ line, int lane) {
    int t1 = 0, t2 = 0, tl = 0;
    for (int s0 = 0; s0 < v.p.n_seqs; s0 += 64) {
        const LatentSeq w = latent_seq(v, g, row_start, s0 + lane);
        t1 += __builtin_amdgcn_readlane(latent_prefix_sum(attend_places(w.units, 1, 0) * w.row_tiles), 63);
        t2 += __builtin_amdgcn_readlane(latent_prefix_sum(attend_places(w.units, 2, 0) * w.row_tiles), 63);
        tl += __builtin_amdgcn_readlane(latent_prefix_sum(attend_places(w.units, 1, kPieceCost) * w.row_tiles), 63);
    }
    const AttendDivision d = attend_division(t1, t2, tl, g.groups, 1);
    if (lane == 0) *reinterpret_cast<LatentLine*>(line) = LatentLine{d.round, d.cost, d.run, 0};
    int before = 0;
    for (int s0 = 0; s0 < v.p.n_seqs; s0 += 64) {
        const LatentSeq w = latent_seq(v, g, row_start, s0 + lane);
        const int end = before + latent_prefix_sum(attend_places(w.units, d.round, d.cost) * w.row_tiles);
        if (s0 + lane < v.p.n_seqs) line[4 + s0 + lane] = end;
        before = __builtin_amdgcn_readlane(end, 63);
    }
}

// q' of the new rows, fp16 [n_seqs * max_rows][H][DC] (row nth of sequence s at s * max_rows + nth): a product per head of w's columns
// [h][0, Dk) with the rows, whose contraction runs along both operands' memory, so that neither passes through LDS.  (Rounding q' to fp16
// changes a logit by 2^-12 of the products it sums at random, as rounding a query does.)
// Bound by reading w, half of it.  A wavefront has 32 latents and ROWS * 16 rows of one head.
// Grid (1 + H * DC / 128, row blocks), 256 threads: the first column makes the line and the zeros.
template <int DC, int ROWS>
__global__ __launch_bounds__(256) void latent_absorb_kernel(LatentView v, LatentGeom g, const _Float16* __restrict__ q, const _Float16* __restrict__ w,
                                                            const int32_t* __restrict__ row_start, _Float16* __restrict__ qa,
                                                            int32_t* __restrict__ line, uint32_t* __restrict__ zeros) {
    const int lane = threadIdx.x & 63, l16 = lane & 15, g4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    if (blockIdx.x == 0) {
        if (blockIdx.y == 0) {
            if (wave == 0) latent_make_line(v, g, row_start, line, lane);
            else
                for (int i = threadIdx.x - 64; i < kZeroBytes / 4; i += 192) zeros[i] = 0u;
        }
        return;
    }
    constexpr int kParts = DC / 128;
    const int part = static_cast<int>(blockIdx.x - 1), h = part / kParts, c0 = (part % kParts) * 128 + wave * 32;
    const int64_t w_row = static_cast<int64_t>(g.H) * (g.Dk + g.Dv);
    const int all = v.p.n_seqs * g.max_rows;
    int64_t from[ROWS];
    bool there[ROWS];
#pragma unroll
    for (int b = 0; b < ROWS; ++b) {
        const int i = (static_cast<int>(blockIdx.y) * ROWS + b) * 16 + l16, s = i / g.max_rows, nth = i - s * g.max_rows;
        there[b] = false;
        from[b] = 0;
        if (i < all) {
            const SeqRows rows = seq_rows(row_start, s, g.n_rows);
            there[b] = nth < rows.count;
            from[b] = (rows.first + nth) * g.q_stride;
        }
    }
    lf4_t acc[2][ROWS];
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int b = 0; b < ROWS; ++b) acc[a][b] = lf4_t{0.0f, 0.0f, 0.0f, 0.0f};
    const _Float16* w_at = w + (c0 + l16) * w_row + h * (g.Dk + g.Dv) + 8 * g4;
    const _Float16* q_at = q + static_cast<int64_t>(h) * (g.Dk + v.Dr) + 8 * g4;
    for (int k = 0; k < g.Dk; k += 32) {
        h8_t a[2], x[ROWS];
#pragma unroll
        for (int i = 0; i < 2; ++i) a[i] = *reinterpret_cast<const h8_t*>(w_at + 16 * i * w_row + k);
#pragma unroll
        for (int b = 0; b < ROWS; ++b) {
            x[b] = h8_t{0, 0, 0, 0, 0, 0, 0, 0};
            if (there[b]) x[b] = *reinterpret_cast<const h8_t*>(q_at + from[b] + k);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int b = 0; b < ROWS; ++b) acc[i][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[i], x[b], acc[i][b], 0, 0, 0);
    }
    // acc[i][b][e]: latent c0 + 16 i + 4 g4 + e of row l16
#pragma unroll
    for (int b = 0; b < ROWS; ++b) {
        const int64_t i = (static_cast<int>(blockIdx.y) * ROWS + b) * 16 + l16;
        if (there[b])
#pragma unroll
            for (int a = 0; a < 2; ++a) {
                lh4_t x;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = static_cast<_Float16>(acc[a][b][e]);
                *reinterpret_cast<lh4_t*>(qa + (i * g.H + h) * DC + c0 + 16 * a + 4 * g4) = x;
            }
    }
}

// Where piece p (16 bytes) of token t of a tile stands in LDS: the latents' rows first, then the position parts'.  Pieces are permuted by
// the token, so that neither reading eight tokens' piece at once (keys) nor two pieces of four tokens (values, transposed) meets a bank twice.
__device__ __forceinline__ int latent_swizzle(int t) { return ((t & 3) << 1) | ((t >> 2) & 1) | (t & 8); }
template <int DC> __device__ __forceinline__ int tile_latent(int t, int p) { return t * (DC * 2) + ((p ^ latent_swizzle(t)) << 4); }
template <int DC, int DR> __device__ __forceinline__ int tile_rope(int t, int p) {
    const int s = DR == 64 ? latent_swizzle(t) & 7 : (t >> 1) & 3;
    return kLatentTile * DC * 2 + t * (DR * 2) + ((p ^ s) << 4);
}

// Waits until at most N of a wavefront's loads are in flight, then for the other wavefronts; memory is not touched across it.
template <int N> __device__ __forceinline__ void arrive() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// 16 bytes a lane from memory to LDS, lane i's at 16 i behind `to` (the same for all lanes), without registers in between: from a base for all
// lanes and an offset of the lane, or from an address of the lane.  The compiler would wait for all such loads in front of every read of LDS
// that they might write to, and a tile ahead would never be one; so they are written out, and arrive() waits for them.
__device__ __forceinline__ void to_lds(const uint8_t* base, uint32_t at, uint8_t* to) {
    const uint32_t lds_at = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t*)to)));
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds_at), "v"(at), "s"(base) : "memory");
}
__device__ __forceinline__ void to_lds(const uint8_t* from, uint8_t* to) {
    const uint32_t lds_at = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t*)to)));
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds_at), "v"(from) : "memory");
}

// What a wavefront brings of a tile: eight tokens, half of one page's sixteen; wave-uniform.
struct TileHalf {
    const uint8_t *codes, *scale, *rope;   // of its first token; from scale to mn: mn_step
    int width, valid;                      // 0: absent; how many of the eight tokens there are
};

// Packed latents of the eight tokens: their codes come to LDS as they are, into the place that the wavefront's eight rows will have there;
// lane i keeps the parameters of token i / groups, group i % groups (at most 8 * 8 pairs).
struct HalfParams {
    uint32_t sc, mn;                       // as they lie in memory
};
__device__ __forceinline__ uint32_t raw_param(const uint8_t* section, uint32_t i, bool half) {
    return half ? reinterpret_cast<const uint16_t*>(section)[i] : reinterpret_cast<const uint32_t*>(section)[i];
}
__device__ __forceinline__ float raw_value(uint32_t raw, bool half) {
    return half ? static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(raw))) : __builtin_bit_cast(float, raw);
}
template <int DC, int W>
__device__ __forceinline__ void packed_fetch(HalfParams& x, const TileHalf& t, uint8_t* rows, uint64_t mn_step, int groups, bool half, uint32_t lane) {
    constexpr int kBytes = 8 * DC * W / 8;
#pragma unroll
    for (int i = 0; i < (kBytes + 1023) / 1024; ++i)
        if (kBytes >= 1024 || lane * 16 < kBytes) to_lds(t.codes, i * 1024 + lane * 16, rows + i * 1024);
    const uint32_t at = min(lane, static_cast<uint32_t>(8 * groups - 1));
    x.sc = raw_param(t.scale, at, half);
    x.mn = raw_param(t.scale + mn_step, at, half);
}

// Dequantises them in their place (missing tokens: zeros).  All codes are read before the first row is written.
template <int DC, int W>
__device__ __forceinline__ void packed_unpack(const HalfParams& x, uint8_t* tile, int token0, int valid, int groups, int lpg_log2, bool half, int lane) {
    constexpr int kRow = DC * W / 128, kN = (8 * kRow + 63) / 64, kOut = 16 / W;       // pieces of a token's codes, of a lane, and what one makes
    const uint8_t* rows = tile + token0 * (DC * 2);
    u4_t code[kN];
#pragma unroll
    for (int i = 0; i < kN; ++i) code[i] = *reinterpret_cast<const u4_t*>(rows + i * 1024 + (8 * kRow < 64 ? lane % (8 * kRow) : lane) * 16);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int i = 0; i < kN; ++i) {
        const int p = (i * 64 + lane) % (8 * kRow), token = p / kRow, in = p % kRow;
        const int of = token * groups + ((in * kOut) >> lpg_log2);
        const float sc = raw_value(__shfl(x.sc, of), half), mn = raw_value(__shfl(x.mn, of), half);
        const bool there = token < valid;
        if (8 * kRow < 64 && lane >= 8 * kRow) continue;
#pragma unroll
        for (int o = 0; o < kOut; ++o) {
            u2_t w;
            if constexpr (W == 8) w = u2_t{code[i][2 * o], code[i][2 * o + 1]};
            else if constexpr (W == 4) w = u2_t{code[i][o], 0u};
            else w = u2_t{code[i][o / 2] >> (16 * (o % 2)), 0u};
            u4_t y = dequantise_piece<W>(w, sc, mn);
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = there ? y[e] : 0u;
            *reinterpret_cast<u4_t*>(tile + tile_latent<DC>(token0 + token, in * kOut + o)) = y;
        }
    }
}

// Attention of a tile of M query rows to a run of tiles of tokens, the four wavefronts of a workgroup together.  A tile of 32 tokens comes
// to LDS once, as fp16; each of the first M / 16 (at most four) wavefronts has the logits S^T = K Q^T and the softmax of its own rows, leaves
// their probabilities in LDS, and each wavefront has a quarter of the dimensions of O^T += V^T P^T for all rows: keys are read from LDS
// by M / 16 wavefronts, values by one.
template <int DC, int DR, int M>
__global__ __launch_bounds__(256, 2) void latent_attend_kernel(LatentView v, LatentGeom g, const _Float16* __restrict__ qa,
                                                                              const _Float16* __restrict__ q, const int32_t* __restrict__ row_start,
                                                                              const int32_t* __restrict__ line, const uint8_t* __restrict__ zeros,
                                                                              int32_t lpg_log2, float* __restrict__ part_o, float* __restrict__ part_ml) {
    constexpr int kTileBytes = kLatentTile * (DC + DR) * 2, kBufs = 2;
    constexpr int kWaves = M >= 64 ? 4 : M / 16, RB = M / 16 / kWaves;         // wavefronts with rows, blocks of 16 rows of each
    constexpr int KS = DC / 32, KR = DR / 32, DB = DC / 64, MB = M / 16;
    __shared__ __attribute__((aligned(16))) uint8_t lds[kBufs * kTileBytes];
    __shared__ __attribute__((aligned(16))) uint8_t probs[M * 64];             // [MB][64 lanes][16 bytes]
    __shared__ float alphas[M];                                                // what the rows' outputs are rescaled by,
    __shared__ int32_t moved[4];                                               // if any of the wavefront's rows are
    __shared__ uint32_t bad_tokens;                                            // tokens of a tile that are not finite
    const int lane0 = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    const LatentLine ll = *reinterpret_cast<const LatentLine*>(line);
    int at = static_cast<int>(blockIdx.x) * ll.run;
    const int run_end = at + ll.run;
    if (threadIdx.x == 0) bad_tokens = 0u;
    if (threadIdx.x < 4) moved[threadIdx.x] = 0;
    int s = -1, s_end = 0;
    while (at < run_end) {
        // the sequence in whose work place `at` lies: the first that ends behind it
        if (at >= s_end) {
            int lo = s + 1, n = v.p.n_seqs - lo;
            while (n > 64) {
                const int step = (n + 63) >> 6, i = min(lane0 * step + step - 1, n - 1);
                const int cnt = __builtin_popcountll(__ballot(line[4 + lo + i] <= at && lane0 * step < n));
                lo += min(cnt * step, n);
                n = min(step, n - min(cnt * step, n));
            }
            if (n <= 0) return;
            const bool behind = lane0 < n && line[4 + lo + min(lane0, n - 1)] > at;
            const uint64_t any = __ballot(behind);
            if (!any) return;                                   // the end of the line
            s = __builtin_amdgcn_readfirstlane(lo + __builtin_ctzll(any));
            s_end = __builtin_amdgcn_readfirstlane(line[4 + s]);
        }
        const LatentSeq sw = latent_seq(v, g, row_start, s);
        const int each = attend_places(sw.units, ll.round, ll.cost), local = at - (s_end - each * sw.row_tiles);
        const int rt = local / each, place = local - rt * each, places = min(each - place, run_end - at);
        const int u_begin = max(place - ll.cost, 0), u_end = min(place + places - ll.cost, sw.units);
        at += places;
        if (u_end <= u_begin) continue;

        // this wavefront's rows: queries, what they see
        const int count = min(sw.count, g.max_rows), H = g.H;
        h8_t qf[RB][KS + KR];
        int last[RB];
        float ref[RB], sum[RB];
        if (wave < kWaves) {
            int lane = lane0;
            asm volatile("" : "+v"(lane));
            const int l16 = lane & 15, g4 = lane >> 4;
#pragma unroll
            for (int b = 0; b < RB; ++b) {
                const int j = rt * M + (wave * RB + b) * 16 + l16, nth = j / H, h = j - nth * H;
                const bool ok = j < sw.rows;
                last[b] = ok ? sw.n - sw.count + nth : -1;
                ref[b] = -INFINITY;
                sum[b] = 0.0f;
                const _Float16* lat = qa + (static_cast<int64_t>(s) * g.max_rows * H + (ok ? j : 0)) * DC + 8 * g4;
                const _Float16* pos = q + (sw.first + (ok ? nth : 0)) * g.q_stride + (ok ? h : 0) * (g.Dk + DR) + g.Dk + 8 * g4;
#pragma unroll
                for (int k = 0; k < KS; ++k) qf[b][k] = *reinterpret_cast<const h8_t*>(lat + 32 * k);
#pragma unroll
                for (int k = 0; k < KR; ++k) qf[b][KS + k] = *reinterpret_cast<const h8_t*>(pos + 32 * k);
            }
        }
        const int all_see = sw.n - sw.count + rt * M / H;       // tokens up to this one are seen by every row
        const int none_sees = sw.n - sw.count + min(count, (rt * M + M - 1) / H + 1);
        lf4_t o[MB][DB];
#pragma unroll
        for (int b = 0; b < MB; ++b)
#pragma unroll
            for (int d = 0; d < DB; ++d) o[b][d] = lf4_t{0.0f, 0.0f, 0.0f, 0.0f};

        // the pages of 64 halves of tiles (16 tokens each), one per lane
        const uint64_t* offs = v.p.off + static_cast<int64_t>(s) * v.p.stride;
        const uint8_t* bits = v.p.bits + static_cast<int64_t>(s) * v.p.stride;
        uint64_t half_off = 0;
        uint32_t half_row = 0, half_width = 0;                  // (row: of the first token, of the record's rows of a section)
        int batch0 = -1;                                        // first tile of the batch
        auto look_up = [&](int u) __attribute__((always_inline)) {
            batch0 = u;
            int lane = lane0;
            asm volatile("" : "+v"(lane));
            const int half = 2 * u + lane;
            const bool in = (half * 16 < min(sw.n, none_sees)) & (half < 2 * u_end);
            const int half_page = v.p.page_of_tile ? static_cast<int>(__umulhi(static_cast<uint32_t>(half), v.p.page_of_tile)) : half;
            const int page = in ? half_page : 0;
            const uint64_t off = offs[page];
            const uint32_t b = bits[page];
            half_width = (in & latent_present(v, off, b)) ? b : 0u;
            half_off = off;
            half_row = static_cast<uint32_t>(v.layer * v.p.T + half * 16 - page * v.p.T);
        };
        auto lane_u64 = [&](uint64_t x, int l) __attribute__((always_inline)) {
            const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(x), l), hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(x >> 32), l);
            return static_cast<uint64_t>(hi) << 32 | lo;
        };
        const uint64_t mn_step = static_cast<uint64_t>(v.p.slabs) * v.p.T * static_cast<uint32_t>(v.p.groups * (v.p.half_params ? 2 : 4));
        const int my_half = wave >> 1, my_token = wave * 8;    // the eight tokens of a tile that this wavefront brings
        auto half_of = [&](int u) __attribute__((always_inline)) {
            TileHalf t;
            const int l = 2 * (u - batch0) + my_half;
            const int first = (wave & 1) * 8;
            t.width = static_cast<int>(__builtin_amdgcn_readlane(half_width, l));
            const uint8_t* record = v.p.pool + lane_u64(half_off, l);
            const uint32_t row = __builtin_amdgcn_readlane(half_row, l) + first, b = t.width;
            t.codes = record + static_cast<uint64_t>(row) * (DC / 8 * b);
            record += v.p.bit_bytes * b;
            t.scale = record + static_cast<uint64_t>(row) * static_cast<uint32_t>(v.p.groups * (v.p.half_params ? 2 : 4));
            t.rope = record + (b == 16 ? 0u : v.p.param_bytes) + static_cast<uint64_t>(row) * (DR * 2);
            t.valid = t.width ? max(0, min(8, sw.n - (u * kLatentTile + my_token))) : 0;
            return t;
        };
        HalfParams packed = {0u, 0u};
        int packed_width = 0, packed_valid = 0;
        // Issues the loads of tile u into buffer `buf`.  fp16 rows and position parts go straight to LDS, rows that are not there come from the
        // zeros; packed ones are unpacked behind this tile's values.
        auto fetch = [&](int u, int buf) __attribute__((always_inline)) {
            const TileHalf t = half_of(u);
            uint8_t *tile = lds + buf * kTileBytes, *rows = tile + my_token * (DC * 2);
            constexpr int kRopeRow = DR / 8, kRow = DC / 8, kSide = 64 / kRow;
            uint32_t lane_at = lane0;                           // (offsets of lanes are made here, not kept)
            asm volatile("" : "+v"(lane_at));
            if (lane_at < 8 * kRopeRow) {
                const uint32_t tk = lane_at / kRopeRow, slot = lane_at % kRopeRow;
                const uint32_t sw_t = DR == 64 ? latent_swizzle(my_token + tk) & 7 : ((my_token + tk) >> 1) & 3;
                const uint8_t* from = static_cast<int>(tk) < t.valid ? t.rope + (tk * (DR * 2) + ((slot ^ sw_t) << 4)) : zeros + slot * 16;
                to_lds(from, tile + kLatentTile * DC * 2 + my_token * (DR * 2));
            }
            packed_width = t.valid ? t.width : 16;
            packed_valid = t.valid;
            if (packed_width == 16) {
#pragma unroll
                for (int i = 0; i < 8 / kSide; ++i) {
                    uint8_t* to = rows + i * kSide * (DC * 2);
                    if constexpr (kSide == 1) {
                        const uint8_t* from = i < t.valid ? t.codes + i * (DC * 2) : zeros;       // (as many zeros as a row has)
                        to_lds(from, (lane_at ^ static_cast<uint32_t>(latent_swizzle(my_token + i))) << 4, to);
                    } else {
                        const uint32_t tk = i * kSide + lane_at / kRow, slot = lane_at % kRow;
                        const uint32_t in = (slot ^ static_cast<uint32_t>(latent_swizzle(my_token + tk))) << 4;
                        const uint8_t* from = static_cast<int>(tk) < t.valid ? t.codes + (tk * (DC * 2) + in) : zeros + in;
                        to_lds(from, to);
                    }
                }
            } else if (packed_width == 8) packed_fetch<DC, 8>(packed, t, rows, mn_step, v.p.groups, v.p.half_params, lane_at);
            else if (packed_width == 4) packed_fetch<DC, 4>(packed, t, rows, mn_step, v.p.groups, v.p.half_params, lane_at);
            else packed_fetch<DC, 2>(packed, t, rows, mn_step, v.p.groups, v.p.half_params, lane_at);
        };
        auto unpack = [&](int buf) __attribute__((always_inline)) {
            uint8_t* tile = lds + buf * kTileBytes;
            int lane_at = lane0;
            asm volatile("" : "+v"(lane_at));
            if (packed_width != 16) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // the codes are there
            if (packed_width == 8) packed_unpack<DC, 8>(packed, tile, my_token, packed_valid, v.p.groups, lpg_log2, v.p.half_params, lane_at);
            else if (packed_width == 4) packed_unpack<DC, 4>(packed, tile, my_token, packed_valid, v.p.groups, lpg_log2, v.p.half_params, lane_at);
            else if (packed_width == 2) packed_unpack<DC, 2>(packed, tile, my_token, packed_valid, v.p.groups, lpg_log2, v.p.half_params, lane_at);
        };

        look_up(u_begin);
        __syncthreads();                                        // (the piece before is done with LDS)
        fetch(u_begin, 0);
        int buf = 0;
        for (int u = u_begin; u < u_end; ++u) {
            // which of the tile's halves are there
            const int l = 2 * (u - batch0);
            const bool have0 = __builtin_amdgcn_readlane(half_width, l) != 0, have1 = __builtin_amdgcn_readlane(half_width, l + 1) != 0;
            const int token0 = u * kLatentTile;
            const bool masked = token0 + kLatentTile - 1 > all_see || !have0 || !have1;
            uint8_t* tile = lds + buf * kTileBytes;
            unpack(buf);
            arrive<0>();                                        // the tile is there; values of the one before have been used
            buf = buf + 1 == kBufs ? 0 : buf + 1;
            if (u + 1 < u_end) {
                if (u + 1 - batch0 >= 32) look_up(u + 1);
                fetch(u + 1, buf);
            }
            // (what depends on the lane is worked out here again: kept over the loop it would not fit the registers)
            int lane = lane0;
            asm volatile("" : "+v"(lane));
            const int l16 = lane & 15, g4 = lane >> 4, thread_at = wave * 64 + lane;
            // A latent that is not finite must not reach rows that do not see its token, whose probability of 0 does not hold it off: where
            // some row does not see all tokens it is replaced, and rows that see it are NaN.
            uint32_t bad = 0u;
            if (token0 + kLatentTile - 1 > all_see) {
                const int t = thread_at >> 3;
                bool found = false;
#pragma unroll 1
                for (int p = thread_at & 7; p < DC / 8; p += 8) {
                    u4_t* x = reinterpret_cast<u4_t*>(tile + tile_latent<DC>(t, p));
                    u4_t y = *x;
                    bool any = false;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if ((y[e] & 0x7c00u) == 0x7c00u) { y[e] &= 0xffff0000u; any = true; }
                        if ((y[e] & 0x7c000000u) == 0x7c000000u) { y[e] &= 0xffffu; any = true; }
                    }
                    if (any) *x = y;
                    found |= any;
                }
                if (found) atomicOr(&bad_tokens, 1u << t);
                __syncthreads();
                bad = bad_tokens;
            }
            if (wave < kWaves) {
                lf4_t sc[RB][2];
#pragma unroll
                for (int b = 0; b < RB; ++b)
#pragma unroll
                    for (int i = 0; i < 2; ++i) sc[b][i] = lf4_t{0.0f, 0.0f, 0.0f, 0.0f};
                // (of a row's pieces four steps have the same low bits, which are all that the swizzle, the same for both halves, changes)
                uint32_t key_at = tile_latent<DC>(l16, g4), rope_key_at = tile_rope<DC, DR>(l16, g4);
                asm volatile("" : "+v"(key_at), "+v"(rope_key_at));
                // Keys of the next two steps are on their way while these are multiplied; the fences keep the compiler from fetching them all
                // first, for which there are no registers.
                h8_t kf[2][4];
                auto key = [&](int k, int i) __attribute__((always_inline)) {
                    const uint32_t in = k < KS ? (key_at ^ ((k & 3) << 6)) + (k >> 2) * 256 + i * (16 * DC * 2)
                                               : (rope_key_at ^ ((k - KS) << 6)) + i * (16 * DR * 2);
                    return *reinterpret_cast<const h8_t*>(tile + in);
                };
#pragma unroll
                for (int f = 0; f < 4; ++f) kf[0][f] = key(f / 2, f % 2);
#pragma unroll
                for (int k = 0; k < KS + KR; k += 2) {
                    __builtin_amdgcn_sched_barrier(0);
                    const int set = (k / 2) & 1;
#pragma unroll
                    for (int f = 0; f < 4; ++f)
                        if (k + 2 + f / 2 < KS + KR) kf[set ^ 1][f] = key(k + 2 + f / 2, f % 2);
#pragma unroll
                    for (int f = 0; f < 4; ++f)
                        if (k + f / 2 < KS + KR) {
#pragma unroll
                            for (int b = 0; b < RB; ++b)
                                sc[b][f % 2] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[set][f], qf[b][k + f / 2], sc[b][f % 2], 0, 0, 0);
                        }
                }
                __builtin_amdgcn_sched_barrier(0);
                // sc[b][i][e]: token 16 i + 4 g4 + e against row l16 of block b
                if (masked) {
#pragma unroll
                    for (int b = 0; b < RB; ++b)
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const int t = 16 * i + 4 * g4 + e;
                                if (bad >> t & 1) sc[b][i][e] = NAN;
                                if (!(i ? have1 : have0) || token0 + t > last[b]) sc[b][i][e] = -INFINITY;
                            }
                }
                float top[RB];
                bool move = false;
#pragma unroll
                for (int b = 0; b < RB; ++b) {
                    float m = fmaxf(fmaxf(sc[b][0][0], sc[b][0][1]), fmaxf(sc[b][0][2], sc[b][0][3]));
                    m = fmaxf(m, fmaxf(fmaxf(sc[b][1][0], sc[b][1][1]), fmaxf(sc[b][1][2], sc[b][1][3])));
                    top[b] = m * g.scale_log2e;
                    move |= top[b] > ref[b] + kLatentSlack;
                }
                if (__any(move)) {                              // (rare: the reference has room)
#pragma unroll
                    for (int b = 0; b < RB; ++b) {
                        float m = fmaxf(top[b], __shfl_xor(top[b], 16));
                        m = fmaxf(m, __shfl_xor(m, 32));
                        const float to = m > ref[b] + kLatentSlack ? m - kLatentTop : ref[b];
                        const float alpha = to == ref[b] ? 1.0f : __builtin_amdgcn_exp2f(ref[b] - to);
                        ref[b] = to;
                        sum[b] *= alpha;
                        if (g4 == 0) alphas[(wave * RB + b) * 16 + l16] = alpha;
                    }
                    if (lane == 0) moved[wave] = 1;
                } else if (lane == 0) moved[wave] = 0;
#pragma unroll
                for (int b = 0; b < RB; ++b) {
                    const float r = ref[b] == -INFINITY ? 0.0f : ref[b];
                    h8_t p;
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[b][i][e], g.scale_log2e, -r));
                            sum[b] += x;
                            p[4 * i + e] = static_cast<_Float16>(x);
                        }
                    *reinterpret_cast<h8_t*>(probs + (wave * RB + b) * 1024 + lane * 16) = p;
                }
            }
            __syncthreads();
            if (bad && thread_at == 0) bad_tokens = 0u;
#pragma unroll
            for (int w = 0; w < kWaves; ++w)
                if (moved[w]) {
#pragma unroll
                    for (int b = 0; b < RB; ++b) {
                        const float a = alphas[(w * RB + b) * 16 + l16];
#pragma unroll
                        for (int d = 0; d < DB; ++d) o[w * RB + b][d] *= a;
                    }
                }
            h8_t pf[MB];
#pragma unroll
            for (int b = 0; b < MB; ++b) pf[b] = *reinterpret_cast<const h8_t*>(probs + b * 1024 + lane * 16);
            // a lane hands in four dimensions of one of its group's four tokens and receives its dimension of all four
            uint32_t value_at = tile_latent<DC>(4 * g4 + (l16 >> 2), wave * DB * 2 + ((lane & 3) >> 1)) + (lane & 1) * 8;
            asm volatile("" : "+v"(value_at));
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                if (M == 128) __builtin_amdgcn_sched_barrier(0);
                const uint8_t* from = tile + (value_at ^ (d << 5));
                const ls4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) ls4_t*)(from));
                const ls4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) ls4_t*)(from + 16 * DC * 2));
                const lh4_t a = __builtin_bit_cast(lh4_t, lo), c = __builtin_bit_cast(lh4_t, hi);
                const h8_t vf = {a[0], a[1], a[2], a[3], c[0], c[1], c[2], c[3]};
#pragma unroll
                for (int b = 0; b < MB; ++b) o[b][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pf[b], o[b][d], 0, 0, 0);
            }
        }
        int lane = lane0;
        asm volatile("" : "+v"(lane));
        const int l16 = lane & 15, g4 = lane >> 4;
        // the share: o[b][d][e] is latent (wave * DB + d) * 16 + 4 g4 + e of row b * 16 + l16
        const int64_t slot = (blockIdx.x + static_cast<int64_t>(s) * g.row_tiles + rt) * M;
        const int here = min(M, sw.rows - rt * M);
#pragma unroll
        for (int b = 0; b < MB; ++b)
            if (b * 16 + l16 < here) {
#pragma unroll
                for (int d = 0; d < DB; ++d)
                    *reinterpret_cast<lf4_t*>(part_o + (slot + b * 16 + l16) * DC + (wave * DB + d) * 16 + 4 * g4) = o[b][d];
            }
        if (wave < kWaves) {
#pragma unroll
            for (int b = 0; b < RB; ++b) {
                float l = sum[b] + __shfl_xor(sum[b], 16);
                l += __shfl_xor(l, 32);
                const int row = (wave * RB + b) * 16 + l16;
                if (g4 == 0 && row < here) *reinterpret_cast<float2*>(part_ml + (slot + row) * 2) = float2{ref[b], l};
            }
        }
    }
}

// The shares of a row joined and its values made: out[h] = w_v[h]^T (sum of shares / sum of their weights), for ROWS rows of one head in a
// workgroup.  The joined latents enter the product as the sum of two halves, 22 bits, which costs nothing next to reading shares and w.
// Grid (H, row blocks), 256 threads.
template <int DC, int DV, int ROWS>
__global__ __launch_bounds__(256) void latent_project_kernel(LatentView v, LatentGeom g, const _Float16* __restrict__ w,
                                                             const int32_t* __restrict__ row_start, const int32_t* __restrict__ line,
                                                             const float* __restrict__ part_o, const float* __restrict__ part_ml,
                                                             _Float16* __restrict__ out) {
    constexpr int kPitch = DC + 8, kSplit = 256 / DV;               // wavefronts that share a column's contraction
    extern __shared__ float weights[];                              // [4][groups]
    __shared__ __attribute__((aligned(16))) _Float16 joined[2][ROWS][kPitch];
    __shared__ lf4_t sums[4][16][16];
    __shared__ int32_t to[ROWS];
    const int lane = threadIdx.x & 63, l16 = lane & 15, g4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    const int h = static_cast<int>(blockIdx.x);
    const LatentLine ll = *reinterpret_cast<const LatentLine*>(line);
    float* weight = weights + wave * g.groups;
    for (int i = wave; i < ROWS; i += 4) {
        const int64_t nr = static_cast<int64_t>(blockIdx.y) * ROWS + i;
        const int s = static_cast<int>(nr / g.max_rows), nth = static_cast<int>(nr - static_cast<int64_t>(s) * g.max_rows);
        const LatentSeq sw = latent_seq(v, g, row_start, s);
        const bool ok = nth < min(sw.count, g.max_rows);
        if (lane == 0) to[i] = ok ? sw.first + nth : -1;
        lf4_t x[DC / 256];
#pragma unroll
        for (int k = 0; k < DC / 256; ++k) x[k] = lf4_t{0.0f, 0.0f, 0.0f, 0.0f};
        float total = 0.0f;
        if (ok && sw.units > 0) {
            const int M = 1 << g.tile_log2, j = nth * g.H + h, rt = j >> g.tile_log2, each = attend_places(sw.units, ll.round, ll.cost);
            const int begin = line[4 + s] - each * (sw.row_tiles - rt) + ll.cost, wg = begin / ll.run;
            const int used = (begin + sw.units - 1) / ll.run - wg + 1;
            const int64_t first = (wg + static_cast<int64_t>(s) * g.row_tiles + rt) * M + (j & (M - 1));
            float ref = -INFINITY;
            for (int k = lane; k < used; k += 64) ref = fmaxf(ref, part_ml[(first + static_cast<int64_t>(k) * M) * 2]);
#pragma unroll
            for (int d = 32; d; d >>= 1) ref = fmaxf(ref, __shfl_xor(ref, d));
            for (int k = lane; k < used; k += 64) {
                const float2 ml = *reinterpret_cast<const float2*>(part_ml + (first + static_cast<int64_t>(k) * M) * 2);
                const float f = ml.x == -INFINITY ? 0.0f : ml.x == ref ? 1.0f : __builtin_amdgcn_exp2f(ml.x - ref);
                weight[k] = f;
                total += f * ml.y;
            }
#pragma unroll
            for (int d = 32; d; d >>= 1) total += __shfl_xor(total, d);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            const float* src = part_o + first * DC + lane * 4;
#pragma unroll 4
            for (int k = 0; k < used; ++k) {
                const float f = weight[k];
#pragma unroll
                for (int c = 0; c < DC / 256; ++c) x[c] += *reinterpret_cast<const lf4_t*>(src + static_cast<int64_t>(k) * M * DC + c * 256) * f;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
        const float inv = total > 0.0f ? 1.0f / total : total;       // a row that sees nothing: zeros; NaN stays
#pragma unroll
        for (int c = 0; c < DC / 256; ++c) {
            lh4_t hi, lo;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float y = x[c][e] * inv;
                hi[e] = static_cast<_Float16>(y);
                lo[e] = static_cast<_Float16>(y - static_cast<float>(hi[e]));
            }
            *reinterpret_cast<lh4_t*>(&joined[0][i][lane * 4 + c * 256]) = hi;
            *reinterpret_cast<lh4_t*>(&joined[1][i][lane * 4 + c * 256]) = lo;
        }
    }
    __syncthreads();
    // 64 columns and a share of the contraction per wavefront: a lane loads four adjacent columns of eight latents, column 4 l16 + n is
    // row l16 of the n-th product's operand
    const int col0 = DV == 128 ? (wave & 1) * 64 : 0, split = DV == 128 ? wave >> 1 : wave;
    const int64_t w_row = static_cast<int64_t>(g.H) * (g.Dk + DV);
    const _Float16* w_at = w + static_cast<int64_t>(h) * (g.Dk + DV) + g.Dk + col0 + 4 * l16;
    lf4_t acc[4];
#pragma unroll
    for (int n = 0; n < 4; ++n) acc[n] = lf4_t{0.0f, 0.0f, 0.0f, 0.0f};
    constexpr int kLen = DC / kSplit;
    for (int k = split * kLen; k < (split + 1) * kLen; k += 32) {
        const int c0 = k + 8 * g4;
        u2_t x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = *reinterpret_cast<const u2_t*>(w_at + (c0 + e) * w_row);
        const h8_t hi = *reinterpret_cast<const h8_t*>(&joined[0][l16 % ROWS][c0]), lo = *reinterpret_cast<const h8_t*>(&joined[1][l16 % ROWS][c0]);
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            u4_t f;
#pragma unroll
            for (int p = 0; p < 4; ++p) f[p] = __builtin_amdgcn_perm(x[2 * p + 1][n / 2], x[2 * p][n / 2], n % 2 ? 0x07060302u : 0x05040100u);
            acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8_t, f), lo, acc[n], 0, 0, 0);
            acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8_t, f), hi, acc[n], 0, 0, 0);
        }
    }
    // acc[n][e]: column col0 + 4 (4 g4 + e) + n of row l16
#pragma unroll
    for (int e = 0; e < 4; ++e) sums[wave][4 * g4 + e][l16] = lf4_t{acc[0][e], acc[1][e], acc[2][e], acc[3][e]};
    __syncthreads();
    for (int i = threadIdx.x; i < ROWS * (DV / 4); i += 256) {
        const int row = i / (DV / 4), quad = i % (DV / 4), wv = DV == 128 ? quad / 16 : 0;
        if (to[row] < 0) continue;
        lf4_t x = sums[wv][quad % 16][row];
#pragma unroll
        for (int k = 1; k < kSplit; ++k) x += sums[wv + k * (4 / kSplit)][quad % 16][row];
        lh4_t y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = static_cast<_Float16>(x[e]);
        *reinterpret_cast<lh4_t*>(out + (static_cast<int64_t>(to[row]) * g.H + h) * DV + 4 * quad) = y;
    }
}

}  // namespace kvs
