// Latent attention in the absorbed form: queries are taken to the latents' space, where one row a token is key and value of all heads,
//     q'[h] = w_k[h] q[h],   s = (q'[h] c + q_r[h] r) / sqrt(Dk + Dr),   out[h] = w_v[h]^T (softmax(s) c),
// so that a token's row is read once for all heads and the wide products are those with the cache, 2 H (2 DC + Dr) operations a (query
// row, token), instead of the 2 DC H (Dk + Dv) a token that making its keys and values takes.  Four launches: latent_absorb_kernel (q' of
// the new rows, and how the work is divided), latent_attend_kernel (shares of the attention), latent_join_kernel (the shares joined) and
// latent_values_kernel.
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
constexpr int kLatentWaves = 8;             // wavefronts of an attention workgroup
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

// How the work is divided.  The token tiles of all sequences and row tiles stand in one line, row tile by row tile, sequence by sequence, with
// kLatentCost places in front of each row tile's for what beginning and ending takes, and every workgroup takes a run of it (latent_run).
// line: the run's length, then, from line[4] on, where each sequence's places end.
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
    int units = 0, pairs = 0;
    for (int s0 = 0; s0 < v.p.n_seqs; s0 += 64) {
        const LatentSeq w = latent_seq(v, g, row_start, s0 + lane);
        units += __builtin_amdgcn_readlane(latent_prefix_sum(w.units * w.row_tiles), 63);
        pairs += __builtin_amdgcn_readlane(latent_prefix_sum(w.units ? w.row_tiles : 0), 63);
    }
    if (lane == 0) line[0] = latent_run(units, pairs, g.groups);
    int before = 0;
    for (int s0 = 0; s0 < v.p.n_seqs; s0 += 64) {
        const LatentSeq w = latent_seq(v, g, row_start, s0 + lane);
        const int end = before + latent_prefix_sum(latent_places(w.units) * w.row_tiles);
        if (s0 + lane < v.p.n_seqs) line[4 + s0 + lane] = end;
        before = __builtin_amdgcn_readlane(end, 63);
    }
}

// q' of the new rows, fp16 [n_seqs * max_rows][H][DC] (row nth of sequence s at s * max_rows + nth): a product per head of w's columns
// [h][0, Dk) with the rows, whose contraction runs along both operands' memory, so that neither passes through LDS.  (Rounding q' to fp16
// changes a logit by 2^-12 of the products it sums at random, as rounding a query does.)
// 3.1 to 7.4 us: reading half of w, and the loop over Dk, whose 32 dimensions a turn wait for their own loads.  A wavefront has 32 latents and
// ROWS * 16 rows of one head.
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

// Where piece p (16 bytes) of token t of a tile stands in LDS, in rows of latents and of position parts: pieces are permuted by the token.  A read
// of 16 bytes a lane takes four turns, of lanes 0-3, 12-15, 20-27, then 4-11, 16-19, 28-31, and the same of the upper half; one of 8 bytes
// two, of half the lanes each.  The permutations put the pieces of a turn on different banks, both for keys (the same piece of 16 tokens, then the
// one beside it) and for values (two pieces of eight tokens).  Measured with a permutation that does not, 43 % of the turns twice.
__device__ __forceinline__ int latent_swizzle(int t) { return (t & 7) << 1; }
template <int DR> __device__ __forceinline__ int rope_swizzle(int t) {
    if (DR == 64) return (t >> 1) & 7;                                      // two tokens of eight pieces stand side by side,
    const int q = t >> 2;                                                   // four of four pieces
    return ((q ^ (q >> 1)) & 1) << 1 | ((q >> 1) & 1);
}
template <int DC> __device__ __forceinline__ int tile_latent(int t, int p) { return t * (DC * 2) + ((p ^ latent_swizzle(t)) << 4); }
template <int DR> __device__ __forceinline__ int tile_rope(int t, int p) { return t * (DR * 2) + ((p ^ rope_swizzle<DR>(t)) << 4); }

// Waits until at most n (3, 4, 5, else none) of the wavefront's loads are in flight.
__device__ __forceinline__ void wait_loads(int n) {
    if (n == 5) asm volatile("s_waitcnt vmcnt(5)" ::: "memory");
    else if (n == 4) asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
    else if (n == 3) asm volatile("s_waitcnt vmcnt(3)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}
// Waits for the other wavefronts; LDS is not touched across it.
__device__ __forceinline__ void arrive() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Loads from memory to LDS, without registers in between: lane i's 16 bytes (to_lds_dwords: 4) to 16 i (4 i) behind a place plus OFFSET, from a
// base for all lanes, an offset of the lane, and OFFSET again; or (to_lds_from) from an address of the lane.  The compiler would wait for all such
// loads in front of every read of LDS that they might write to, and a tile ahead would never be one; so they are written out, and wait_loads()
// waits for them.  The place is in m0 (a register that the compiler knows as the instruction's operand); it must be there one state before.
__device__ __forceinline__ uint32_t lds_place(uint8_t* to) {
    return __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t*)to)));
}
template <int OFFSET = 0> __device__ __forceinline__ void to_lds(uint32_t place, const uint8_t* base, uint32_t at) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 offset:%2" ::"v"(at), "s"(base), "n"(OFFSET), "{m0}"(place) : "memory");
}
template <int OFFSET = 0> __device__ __forceinline__ void to_lds_dwords(uint32_t place, const uint8_t* base, uint32_t at) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dword %0, %1 offset:%2" ::"v"(at), "s"(base - OFFSET), "n"(OFFSET), "{m0}"(place) : "memory");
}
template <int OFFSET = 0> __device__ __forceinline__ void to_lds_from(uint32_t place, const uint8_t* from) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off offset:%1" ::"v"(from - OFFSET), "n"(OFFSET), "{m0}"(place) : "memory");
}

// Packed latents of a wavefront's TW tokens: codes and parameters come to LDS as they are, into the place that its rows will have there (codes in
// front, scales and minima in the last quarter).  -> the loads issued.
template <int DC, int W, int TW>
__device__ __forceinline__ int packed_fetch(const uint8_t* codes, const uint8_t* scales, uint8_t* rows, uint32_t mn_step, uint32_t param_bytes,
                                            uint32_t lane) {
    constexpr int kBytes = TW * DC * W / 8, kParams = TW * DC * 2 * 3 / 4;
    static_assert(kBytes <= kParams, "codes and parameters do not overlap");
    const uint32_t place = lds_place(rows);
    if (kBytes >= 1024 || lane * 16 < kBytes) to_lds(place, codes, lane * 16);
    if constexpr (kBytes > 1024) to_lds<1024>(place, codes, lane * 16);
    static_assert(kBytes <= 2048, "two loads of codes");
    if (lane * 4 < param_bytes) {
        to_lds_dwords<kParams>(place, scales, lane * 4);
        to_lds_dwords<kParams + TW * DC / 4>(place, scales + mn_step, lane * 4);
    }
    return (kBytes + 1023) / 1024 + 2;
}

// Eight latents from their codes, as a Load gives them: product and sum rounded to binary32 one after the other, then to fp16.  HP: a code of 8 bits
// times a scale of 11 is exact, so that one multiply-add rounds as the two steps do.
template <int W, bool HP>
__device__ __forceinline__ u4_t latent_dequantise(u2_t w, float sc, float mn) {
    typedef float f2_t __attribute__((ext_vector_type(2)));
    typedef _Float16 h2_t __attribute__((ext_vector_type(2)));
    float x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const uint32_t c = W == 8 ? ((k < 4 ? w.x : w.y) >> ((k & 3) * 8)) & 0xffu : (w.x >> (k * W)) & ((1u << W) - 1u);
        const float code = static_cast<float>(c);
        x[k] = HP ? __builtin_fmaf(code, sc, mn) : code * sc + mn;
    }
    u4_t y;
#pragma unroll
    for (int k = 0; k < 4; ++k) y[k] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f2_t{x[2 * k], x[2 * k + 1]}, h2_t));
    return y;
}

// Dequantises them in their place, a lane eight latents at a time, side by side with its neighbours' (missing tokens: zeros).  All codes are
// read before the first row is written; the parameters lie where the last one will be.  TIGHT: one step after the other, parameters a step ahead:
// side by side they take registers that are not there.
template <int DC, int W, int TW, bool HP, bool TIGHT>
__device__ __forceinline__ void packed_unpack(uint8_t* tile, int token0, int valid, int groups, int lpg_log2, int lane) {
    constexpr int kRow = DC / 8, kN = TW * kRow / 64, kParams = TW * DC * 2 * 3 / 4;   // pieces of a row, of a lane
    static_assert((kN - 1) * 1024 <= kParams, "only the last step writes where the parameters lie");
    uint8_t* rows = tile + token0 * (DC * 2);
    const int param0 = lane / kRow * groups + ((lane % kRow) >> lpg_log2);
    auto param = [&](int i, int section) __attribute__((always_inline)) {
        return latent_param(rows + kParams + section * (TW * DC / 4), param0 + i * (64 / kRow) * groups, HP);
    };
    u2_t code[kN];
#pragma unroll
    for (int i = 0; i < kN; ++i) {
        const uint8_t* from = rows + (i * 64 + lane) * W;
        if constexpr (W == 8) code[i] = *reinterpret_cast<const u2_t*>(from);
        else if constexpr (W == 4) code[i].x = *reinterpret_cast<const uint32_t*>(from);
        else code[i].x = *reinterpret_cast<const uint16_t*>(from);
    }
    float sc[kN], mn[kN];
#pragma unroll
    for (int i = 0; i < (TIGHT ? 1 : kN); ++i) {
        sc[i] = param(i, 0);
        mn[i] = param(i, 1);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int i = 0; i < kN; ++i) {
        const int token = (i * 64 + lane) / kRow, in = lane % kRow;
        u4_t y = latent_dequantise<W, HP>(code[i], sc[i], mn[i]);
        if (TIGHT && i + 1 < kN) {
            sc[(i + 1) % kN] = param(i + 1, 0);
            mn[(i + 1) % kN] = param(i + 1, 1);
        }
        if (valid < TW) {
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = token < valid ? y[e] : 0u;
        }
        *reinterpret_cast<u4_t*>(tile + tile_latent<DC>(token0 + token, in)) = y;
        if (TIGHT && i + 1 < kN) asm volatile("" : "+v"(code[(i + 1) % kN].x), "+v"(code[(i + 1) % kN].y)::"memory");
    }
}

struct LatentAttendArgs {
    LatentView v;
    LatentGeom g;
    const _Float16 *qa, *q;
    const int32_t *row_start, *line;
    const uint8_t* zeros;
    float *part_o, *part_ml;
    int32_t lpg_log2;
};

// Attention of a tile of M query rows to a run of tiles of tokens, the eight wavefronts of a workgroup together.  A tile of 32 tokens comes to
// LDS once, as fp16; each of the first M / 16 wavefronts has the logits S^T = K Q^T and the softmax of its own 16 rows and leaves their
// probabilities in LDS, and each wavefront has an eighth of the dimensions of O^T += V^T P^T for all rows: keys are read from LDS by M / 16
// wavefronts, values by one.  A turn of the loop, with one barrier, asks for tile t + 3, has the logits and the softmax of tile t + 1 and the
// values of tile t, and brings tile t + 2 into its form.  (With half of the wavefronts in another order, values before logits, 128 rows took 5 % longer.)
//
// The weights of O are halves (11 bits; a turn's matrix instructions would be half as many again with the 22 bits of two), their sum is of the
// unrounded ones, so that each weight is off by half a step on its own.
//
// 128 rows: 16 sequences of 32768 tokens in fp16, 604 MB read once, 187 us when the chip is cool, 199 to 218 after a few milliseconds of it: 3.2 to 2.8
// TB/s, 0.78 to 0.67 PFLOP/s.  The same loop with the loads alone takes 132 us, with the products alone 141 to 165 (LDS gives 64 rows of keys 16
// times, of values 8 times), with neither 31.  16 to 64 rows: 24 packed contexts of up to 8000 tokens and 32 rows 39 us in 12 turns.
// A turn's time is a chain, logits to weights to values with a barrier, and at present a trip to memory besides: the compiler waits for the query rows
// where they are first used, between the products of the logits in every turn (vmcnt 17 to 0 at 512 + 64), and so for the tile that this wavefront
// has just asked for.  Only wavefronts without rows are three tiles ahead.  How much of a turn that is has not been measured.
template <int DC, int DR, int M>
__global__ __launch_bounds__(512, 2) void latent_attend_kernel(LatentAttendArgs args) {
    // (arguments are fetched where they are used, in the loop only by what is rare: kept in registers all the time they do not fit, and what
    // does not fit is fetched from vector registers, one by one)
    auto here = [&]() __attribute__((always_inline)) {
        auto at = (const __attribute__((address_space(4))) LatentAttendArgs*)__builtin_amdgcn_kernarg_segment_ptr();
        asm volatile("" : "+s"(at));
        return (const LatentAttendArgs*)at;
    };
    const int32_t* line = args.line;
    const uint8_t* zeros = args.zeros;
    uint8_t* const pool = args.v.p.pool;
    const float scale_log2e = args.g.scale_log2e;
    constexpr int kTileBytes = kLatentTile * DC * 2, kRopeBytes = kLatentTile * DR * 2;
    constexpr int NW = kLatentWaves, kWaves = M / 16;                          // wavefronts, those with rows (16 each)
    constexpr int KS = DC / 32, KR = DR / 32, DB = DC / 16 / NW, MB = M / 16;  // steps over the dimensions; a wavefront's blocks of 16 of them
    constexpr int TW = kLatentTile / NW;                                       // tokens that a wavefront brings
    __shared__ __attribute__((aligned(16))) uint8_t lds[4 * kTileBytes], rope_lds[3 * kRopeBytes];      // of the tiles in turn
    // of the tiles in turn: probabilities [MB][64 lanes][16 bytes], what the rows' outputs are rescaled by, blocks of rows that are, tokens that
    // are not finite
    __shared__ __attribute__((aligned(16))) uint8_t probs_lds[2][M * 64];
    __shared__ float alphas_lds[2][M];
    __shared__ uint32_t moved_lds[3];
    __shared__ uint32_t bad_lds[2];
    const int lane0 = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    const int run = line[0];
    int at = static_cast<int>(blockIdx.x) * run;
    const int run_end = at + run;
    const int n_seqs = args.v.p.n_seqs;
    int s = -1, s_end = 0;
    LatentSeq sw;
    if (n_seqs <= 64) {
        // the first piece's sequence: all there is to know of up to 64 comes together, a sequence per lane, in one trip to memory
        const LatentSeq of_lane = latent_seq(args.v, args.g, args.row_start, lane0);
        const int end_of_lane = line[4 + min(lane0, n_seqs - 1)];
        const uint64_t any = __ballot(lane0 < n_seqs && end_of_lane > at);
        if (!any) return;                                       // behind the end of the line
        s = __builtin_ctzll(any);
        s_end = __builtin_amdgcn_readlane(end_of_lane, s);
        sw = {__builtin_amdgcn_readlane(of_lane.n, s),    __builtin_amdgcn_readlane(of_lane.first, s),     __builtin_amdgcn_readlane(of_lane.count, s),
              __builtin_amdgcn_readlane(of_lane.rows, s), __builtin_amdgcn_readlane(of_lane.row_tiles, s), __builtin_amdgcn_readlane(of_lane.units, s)};
    }
    while (at < run_end) {
        const LatentAttendArgs* a0 = here();
        // the sequence in whose work place `at` lies: the first that ends behind it
        if (at >= s_end) {
            int lo = s + 1, n = n_seqs - lo;
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
            sw = latent_seq(a0->v, a0->g, a0->row_start, s);
        }
        const LatentPiece piece = latent_piece(at, run_end, s_end, sw.units, sw.row_tiles);
        const int rt = piece.row_tile, u_begin = piece.begin, u_end = piece.end;
        at += piece.places;
        if (u_end <= u_begin) continue;

        const int count = min(sw.count, a0->g.max_rows), H = a0->g.H;
        const int all_see = sw.n - sw.count + rt * M / H;       // tokens up to this one are seen by every row
        const int none_sees = sw.n - sw.count + min(count, (rt * M + M - 1) / H + 1);
        lf4_t o[MB][DB];
#pragma unroll
        for (int b = 0; b < MB; ++b)
#pragma unroll
            for (int d = 0; d < DB; ++d) o[b][d] = lf4_t{0.0f, 0.0f, 0.0f, 0.0f};

        // What this wavefront brings of 64 tiles, a tile per lane: the record of its tokens' page and where their rows lie in it, and of which tiles
        // either half (16 tokens, one page) is there.
        const int my_token = wave * TW, my_half = my_token / 16, seq_n = sw.n;
        uint64_t tile_off = 0, have_low = 0, have_high = 0;
        uint32_t tile_row = 0, tile_width = 0;
        int batch0 = -1;                                        // first tile of the batch
        const uint32_t rope16 = static_cast<uint32_t>(a0->v.p.bit_bytes) * 16;      // where position parts begin in fp16 records
        auto look_up = [&](int u) __attribute__((always_inline)) {
            batch0 = u;
            int lane = lane0;
            asm volatile("" : "+v"(lane));
            const LatentAttendArgs* a = here();
            const LatentView v = a->v;
            const uint64_t* offs = v.p.off + static_cast<int64_t>(s) * v.p.stride;
            const uint8_t* bits = v.p.bits + static_cast<int64_t>(s) * v.p.stride;
            int page[2];
            bool in[2];
            uint64_t off[2];
            uint32_t b[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int half = 2 * (u + lane) + i;
                in[i] = (half * 16 < min(seq_n, none_sees)) & (u + lane < u_end);
                const int half_page = v.p.page_of_tile ? static_cast<int>(__umulhi(static_cast<uint32_t>(half), v.p.page_of_tile)) : half;
                page[i] = in[i] ? half_page : 0;
                off[i] = offs[page[i]];
                b[i] = bits[page[i]];
            }
            uint32_t width[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) width[i] = (in[i] & latent_present(v, off[i], b[i])) ? b[i] : 0u;
            have_low = __ballot(width[0] != 0);
            have_high = __ballot(width[1] != 0);
            const bool second = my_half == 1;
            tile_off = second ? off[1] : off[0];
            tile_width = second ? width[1] : width[0];
            tile_row = static_cast<uint32_t>(v.layer * v.p.T + (2 * (u + lane) + my_half) * 16 + my_token % 16 - (second ? page[1] : page[0]) * v.p.T);
        };
        // Asks for tile u.  Whole rows and position parts come as they stay, those of tokens that are not there from the zeros.
        int loads = 0, width1 = 16, valid1 = 0;                 // of the tile that was asked for last: the loads, what this wavefront has of it,
        int have1 = 0, have2 = 0;                               // which halves are there; the same of the tile before
        auto fetch = [&](int u, uint8_t* rope) __attribute__((always_inline)) {
            constexpr int kRopeRow = DR / 8, kRow = DC / 8, kSide = 64 / kRow;
            const int l = u - batch0;
            have1 = static_cast<int>((have_low >> l & 1) | (have_high >> l & 1) << 1);
            width1 = static_cast<int>(__builtin_amdgcn_readlane(tile_width, l));
            valid1 = width1 ? max(0, min(TW, seq_n - (u * kLatentTile + my_token))) : 0;
            const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(tile_off), l);
            const uint32_t hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(tile_off >> 32), l);
            const uint8_t* record = pool + (static_cast<uint64_t>(hi) << 32 | lo);
            const uint32_t row = __builtin_amdgcn_readlane(tile_row, l);       // (offsets in a record fit in 32 bits)
            uint8_t* rows = lds + (u & 3) * kTileBytes + my_token * (DC * 2);
            rope += my_token * (DR * 2);
            uint32_t lane_at = lane0;                           // (offsets of lanes are made here, not kept)
            asm volatile("" : "+v"(lane_at));
            const uint32_t rope_tk = lane_at / kRopeRow, rope_in = ((lane_at % kRopeRow) ^ rope_swizzle<DR>(my_token + rope_tk)) << 4;
            // piece `lane` of the wavefront's rows, `i` loads on: its place from the load's first row on, as it comes from memory
            auto in_rows = [&](int i) __attribute__((always_inline)) {
                const uint32_t tk = lane_at / kRow;
                return tk * (DC * 2) + (((lane_at % kRow) ^ static_cast<uint32_t>(latent_swizzle(my_token + i * kSide + tk))) << 4);
            };
            static_assert(TW / kSide == 4 || TW / kSide == 2, "four loads of whole rows, or two");
            constexpr bool kFour = TW / kSide == 4;
            const uint32_t rope_place = lds_place(rope), place = lds_place(rows);
            if (valid1 == TW && width1 == 16) {
                if (lane_at < TW * kRopeRow) to_lds(rope_place, record + (rope16 + row * (DR * 2)), rope_tk * (DR * 2) + rope_in);
                const uint8_t* codes = record + row * (DC * 2);
                to_lds(place, codes, in_rows(0));
                to_lds<1024>(place, codes, in_rows(1));
                if constexpr (kFour) {
                    to_lds<2048>(place, codes, in_rows(2));
                    to_lds<3 * 1024>(place, codes, in_rows(3));
                }
                loads = TW / kSide + 1;
                return;
            }
            const LatentAttendArgs* a = here();
            const uint32_t behind_codes = static_cast<uint32_t>(a->v.p.bit_bytes) * width1;
            const uint8_t* codes = record + row * (DC / 8 * width1);
            const uint8_t* ropes = record + (behind_codes + (width1 == 16 ? 0u : static_cast<uint32_t>(a->v.p.param_bytes)) + row * (DR * 2));
            if (lane_at < TW * kRopeRow)
                to_lds_from(rope_place, static_cast<int>(rope_tk) < valid1 ? ropes + (rope_tk * (DR * 2) + rope_in) : zeros + rope_in);
            if (valid1 == 0) width1 = 16;
            if (width1 == 16) {
                auto from = [&](int i) __attribute__((always_inline)) {
                    return static_cast<int>(i * kSide + lane_at / kRow) < valid1 ? codes + i * 1024 + in_rows(i) : zeros + in_rows(i);
                };
                to_lds_from(place, from(0));
                to_lds_from<1024>(place, from(1));
                if constexpr (kFour) {
                    to_lds_from<2048>(place, from(2));
                    to_lds_from<3 * 1024>(place, from(3));
                }
                loads = TW / kSide + 1;
            } else {
                const uint32_t param_row = a->v.p.groups * (a->v.p.half_params ? 2 : 4), mn_step = a->v.p.slabs * a->v.p.T * param_row;
                const uint8_t* scales = record + (behind_codes + row * param_row);
                if (width1 == 8) loads = 1 + packed_fetch<DC, 8, TW>(codes, scales, rows, mn_step, TW * param_row, lane_at);
                else if (width1 == 4) loads = 1 + packed_fetch<DC, 4, TW>(codes, scales, rows, mn_step, TW * param_row, lane_at);
                else loads = 1 + packed_fetch<DC, 2, TW>(codes, scales, rows, mn_step, TW * param_row, lane_at);
            }
        };
        auto unpack = [&](int u, int width, int valid) __attribute__((always_inline)) {
            uint8_t* tile = lds + (u & 3) * kTileBytes;
            int lane_at = lane0;
            asm volatile("" : "+v"(lane_at));
            const LatentAttendArgs* a = here();
            const int groups = a->v.p.groups, lpg_log2 = a->lpg_log2;
            const bool half_params = a->v.p.half_params;
#define KV_UNPACK(W)                                                                                                       \
    do {                                                                                                                   \
        if (half_params) packed_unpack<DC, W, TW, true, (M * DC > 64 * 512)>(tile, my_token, valid, groups, lpg_log2, lane_at);         \
        else packed_unpack<DC, W, TW, false, (M * DC > 64 * 512)>(tile, my_token, valid, groups, lpg_log2, lane_at);                        \
    } while (0)
            if (width == 8) KV_UNPACK(8);
            else if (width == 4) KV_UNPACK(4);
            else if (width == 2) KV_UNPACK(2);
#undef KV_UNPACK
        };

        look_up(u_begin);
        // this wavefront's rows: queries, what they see
        h8_t qf[KS + KR];
        int last = -1;
        float ref = -INFINITY, sum = 0.0f;
        if (wave < kWaves) {
            int lane = lane0;
            asm volatile("" : "+v"(lane));
            const int l16 = lane & 15, g4 = lane >> 4;
            const int j = rt * M + wave * 16 + l16, nth = j / H, h = j - nth * H;
            const bool ok = j < sw.rows;
            last = ok ? sw.n - sw.count + nth : -1;
            const _Float16* lat = a0->qa + (static_cast<int64_t>(s) * a0->g.max_rows * H + (ok ? j : 0)) * DC + 8 * g4;
            const _Float16* pos = a0->q + (sw.first + (ok ? nth : 0)) * a0->g.q_stride + (ok ? h : 0) * (a0->g.Dk + DR) + a0->g.Dk + 8 * g4;
#pragma unroll
                for (int k = 0; k < KS; ++k) qf[k] = *reinterpret_cast<const h8_t*>(lat + 32 * k);
#pragma unroll
                for (int k = 0; k < KR; ++k) qf[KS + k] = *reinterpret_cast<const h8_t*>(pos + 32 * k);
        }
        __syncthreads();                                        // (the piece before is done with LDS)
        if (threadIdx.x < 2) bad_lds[threadIdx.x] = 0u;
        if (threadIdx.x < 3) moved_lds[threadIdx.x] = 0u;
        int third = 0;                                          // u % 3, counted from the first turn
        bool was_edge = false, was_moved = false;               // of the turn before
        for (int u = u_begin - 3; u < u_end; ++u) {             // (the first three turns bring tiles, the third has logits)
            const int token0 = (u + 1) * kLatentTile;           // of the tile whose logits are made
            const int have = have2;                             // which of its halves are there
            const bool edge = token0 + kLatentTile - 1 > all_see, masked = edge || have != 3;
            const int next_third = third == 2 ? 0 : third + 1;
            arrive();                                           // tile u + 1 and the probabilities of tile u are there, tile u - 1 has been used
            const int width2 = width1, valid2 = valid1;         // of tile u + 2
            have2 = have1;
            loads = 0;
            auto ask = [&]() __attribute__((always_inline)) {
                if (u + 3 < u_end) {
                    if (u + 3 - batch0 >= 64) look_up(u + 3);
                    fetch(u + 3, rope_lds + third * kRopeBytes);        // (where tile u was)
                }
            };
            const uint32_t moved_word = moved_lds[third];       // (read early: it is needed behind the first loads)
            const int odd = u & 1;                              // (of tile u; tile u + 1 has the other)
            // (what depends on the lane is worked out here again: kept over the loop it would not fit the registers)
            int lane = lane0;
            asm volatile("" : "+v"(lane));
            const int l16 = lane & 15, g4 = lane >> 4;
            // A latent that is not finite must not reach rows that do not see its token, whose probability of 0 does not hold it off: where
            // some row does not see all tokens it is replaced, and rows that see it are NaN.  -> such tokens of tile u + 1.
            auto scan = [&]() __attribute__((always_inline)) {
                if (!edge) return 0u;
                uint8_t* tile = lds + ((u + 1) & 3) * kTileBytes;
                constexpr int kPer = 64 * NW / kLatentTile;     // threads per token
                const int thread_at = wave * 64 + lane, t = thread_at / kPer;
                bool found = false;
#pragma unroll 1
                for (int p = thread_at % kPer; p < DC / 8; p += kPer) {
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
                if (found) atomicOr(&bad_lds[odd ^ 1], 1u << t);
                __syncthreads();
                return bad_lds[odd ^ 1];
            };
            auto logits = [&](uint32_t bad) __attribute__((always_inline)) {
                const uint8_t* tile = lds + ((u + 1) & 3) * kTileBytes;
                const uint8_t* rope = rope_lds + next_third * kRopeBytes;
                uint8_t* probs = probs_lds[odd ^ 1];
                if (wave < kWaves) {
                    lf4_t sc[2] = {lf4_t{0.0f, 0.0f, 0.0f, 0.0f}, lf4_t{0.0f, 0.0f, 0.0f, 0.0f}};
                    // (of a row's pieces four steps have the same low bits, which are all that the swizzle, the same for both halves, changes)
                    uint32_t key_at = tile_latent<DC>(l16, g4), rope_key_at = tile_rope<DR>(l16, g4);
                    asm volatile("" : "+v"(key_at), "+v"(rope_key_at));
                    // Keys of the next steps are on their way while a step's are multiplied; the fences keep the compiler from fetching them all
                    // first, for which there are no registers.
                    constexpr int kAhead = M * (DC + DR) > 128 * 544 ? 1 : 2;
                    h8_t kf[kAhead + 1][2];
                    auto key = [&](int k, int i) __attribute__((always_inline)) {
                        return *reinterpret_cast<const h8_t*>(k < KS ? tile + (key_at ^ ((k & 3) << 6)) + (k >> 2) * 256 + i * (16 * DC * 2)
                                                                     : rope + (rope_key_at ^ ((k - KS) << 6)) + i * (16 * DR * 2));
                    };
#pragma unroll
                    for (int f = 0; f < 2 * kAhead; ++f) kf[f / 2][f % 2] = key(f / 2, f % 2);
#pragma unroll
                    for (int k = 0; k < KS + KR; ++k) {
                        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                        for (int i = 0; i < 2; ++i)
                            if (k + kAhead < KS + KR) kf[(k + kAhead) % (kAhead + 1)][i] = key(k + kAhead, i);
#pragma unroll
                        for (int i = 0; i < 2; ++i) sc[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[k % (kAhead + 1)][i], qf[k], sc[i], 0, 0, 0);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                    // sc[i][e]: token 16 i + 4 g4 + e against row l16
                    if (masked) {
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const int t = 16 * i + 4 * g4 + e;
                                if (bad >> t & 1) sc[i][e] = NAN;
                                if (!(have >> i & 1) || token0 + t > last) sc[i][e] = -INFINITY;
                            }
                    }
                    float top = fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[0][2], sc[0][3]));
                    top = fmaxf(top, fmaxf(fmaxf(sc[1][0], sc[1][1]), fmaxf(sc[1][2], sc[1][3]))) * scale_log2e;
                    const bool move = __any(top > ref + kLatentSlack);
                    if (move) {                                     // (rare: the reference has room)
                        float m = fmaxf(top, __shfl_xor(top, 16));
                        m = fmaxf(m, __shfl_xor(m, 32));
                        const float to = m > ref + kLatentSlack ? m - kLatentTop : ref;
                        const float alpha = to == ref ? 1.0f : __builtin_amdgcn_exp2f(ref - to);
                        ref = to;
                        sum *= alpha;
                        if (g4 == 0) alphas_lds[odd ^ 1][wave * 16 + l16] = alpha;
                        if (lane == 0) atomicOr(&moved_lds[next_third], 1u << wave);
                    }
                    const float r = ref == -INFINITY ? 0.0f : ref;
                    h8_t p;
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i][e], scale_log2e, -r));
                            sum += x;
                            p[4 * i + e] = static_cast<_Float16>(x);
                        }
                    *reinterpret_cast<h8_t*>(probs + wave * 1024 + lane * 16) = p;
                }
            };
            auto rescale = [&]() __attribute__((always_inline)) {
                const uint32_t moved = __builtin_amdgcn_readfirstlane(moved_word);
                if (moved == 0) return;
#pragma unroll
                for (int b = 0; b < MB; ++b)
                    if (moved >> b & 1) {
                        const float a = alphas_lds[odd][b * 16 + l16];
#pragma unroll
                        for (int d = 0; d < DB; ++d) o[b][d] *= a;
                    }
            };
            auto values = [&]() __attribute__((always_inline)) {
                const uint8_t *tile = lds + (u & 3) * kTileBytes, *probs = probs_lds[odd];
                // a lane hands in four dimensions of one of its group's four tokens and receives its dimension of all four
                uint32_t value_at = tile_latent<DC>(4 * g4 + (l16 >> 2), wave * DB * 2 + ((lane & 3) >> 1)) + (lane & 1) * 8;
                asm volatile("" : "+v"(value_at));
                auto value = [&](int d) __attribute__((always_inline)) {
                    const uint8_t* from = tile + (value_at ^ (d << 5));
                    const ls4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) ls4_t*)(from));
                    const ls4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) ls4_t*)(from + 16 * DC * 2));
                    const lh4_t a = __builtin_bit_cast(lh4_t, lo), c = __builtin_bit_cast(lh4_t, hi);
                    return h8_t{a[0], a[1], a[2], a[3], c[0], c[1], c[2], c[3]};
            };
            auto weights = [&](int b) __attribute__((always_inline)) { return *reinterpret_cast<const h8_t*>(probs + b * 1024 + lane * 16); };
            // (the fewer operands are kept)
            if constexpr (MB > DB) {
                h8_t vf[DB];
#pragma unroll
                for (int d = 0; d < DB; ++d) vf[d] = value(d);
#pragma unroll
                for (int b = 0; b < MB; ++b) {
                    const h8_t pf = weights(b);
#pragma unroll
                    for (int d = 0; d < DB; ++d) o[b][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf[d], pf, o[b][d], 0, 0, 0);
                }
            } else {
                h8_t pf[MB];
#pragma unroll
                for (int b = 0; b < MB; ++b) pf[b] = weights(b);
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    const h8_t vf = value(d);
#pragma unroll
                    for (int b = 0; b < MB; ++b) o[b][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pf[b], o[b][d], 0, 0, 0);
                }
            }
            };
            const bool has = u >= u_begin - 1 && u + 1 < u_end;
            ask();
            if (u >= u_begin) rescale();
            if (has) logits(scan());
            if (u >= u_begin) values();
            // (what was read a turn ago is used again in the next)
            if (was_edge && threadIdx.x == 0) bad_lds[odd] = 0u;
            if (was_moved && threadIdx.x == 0) moved_lds[third == 0 ? 2 : third - 1] = 0u;
            was_edge = has && edge;
            was_moved = u >= u_begin && __builtin_amdgcn_readfirstlane(moved_word) != 0u;
            // tile u + 2 is there, tile u + 3 may be on its way
            if (loads == TW * DC / 512 + 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(TW * DC / 512 + 1) : "memory");
            else wait_loads(loads);
            if (width2 != 16 && u + 2 < u_end && u + 2 >= u_begin) unpack(u + 2, width2, valid2);
            third = next_third;
        }
        int lane = lane0;
        asm volatile("" : "+v"(lane));
        const int l16 = lane & 15, g4 = lane >> 4;
        // the share: o[b][d][e] is latent (wave * DB + d) * 16 + 4 g4 + e of row b * 16 + l16
        const LatentAttendArgs* a1 = here();
        float *part_o = a1->part_o, *part_ml = a1->part_ml;
        const int64_t slot = latent_slot(static_cast<int32_t>(blockIdx.x), s, rt, a1->g.row_tiles) * M;
        const int here = min(M, sw.rows - rt * M);
#pragma unroll
        for (int b = 0; b < MB; ++b)
            if (b * 16 + l16 < here) {
#pragma unroll
                for (int d = 0; d < DB; ++d)
                    *reinterpret_cast<lf4_t*>(part_o + (slot + b * 16 + l16) * DC + (wave * DB + d) * 16 + 4 * g4) = o[b][d];
            }
        if (wave < kWaves) {
            float l = sum + __shfl_xor(sum, 16);
            l += __shfl_xor(l, 32);
            const int row = wave * 16 + l16;
            if (g4 == 0 && row < here) *reinterpret_cast<float2*>(part_ml + (slot + row) * 2) = float2{ref, l};
        }
    }
}

// The shares of a query row joined: their sum over the sum of their weights, as the sum of two halves (22 bits, so that the product behind it
// is not the result's largest error), hi and lo [n_seqs * max_rows][H][DC] each.  Latency bounds it, row, line, references, weights and shares being
// loads that wait for each other (the shares' addresses are known before the weights are, and they are asked for after), and reading the shares.  A
// workgroup's four wavefronts share a row (768 rows of 24 sequences 6.5 us, with a wavefront to a row 7.7; 512 rows of 8 longer ones 8.9 and 12.5; 2048
// rows of 32768 tokens 15.4 and 16.7; 2560 rows of up to 3001 tokens 9.6 and 9.3).
template <int DC>
__global__ __launch_bounds__(256) void latent_join_kernel(LatentView v, LatentGeom g, const int32_t* __restrict__ row_start,
                                                          const int32_t* __restrict__ line, const float* __restrict__ part_o,
                                                          const float* __restrict__ part_ml, _Float16* __restrict__ hi, _Float16* __restrict__ lo) {
    constexpr int PER = 4;
    extern __shared__ float weight[];                               // [groups]
    __shared__ lf4_t parts[PER][DC / 4];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    const int64_t at = static_cast<int64_t>(blockIdx.x);
    const int row = static_cast<int>(at / g.H), h = static_cast<int>(at - static_cast<int64_t>(row) * g.H);
    const int s = row / g.max_rows, nth = row - s * g.max_rows;
    const int run = line[0];
    const LatentSeq sw = latent_seq(v, g, row_start, s);
    const bool ok = nth < min(sw.count, g.max_rows);
    if (!ok) return;                                                // (uniform)
    lf4_t x[DC / 256];
#pragma unroll
    for (int k = 0; k < DC / 256; ++k) x[k] = lf4_t{0.0f, 0.0f, 0.0f, 0.0f};
    float total = 0.0f;
    if (sw.units > 0) {
        const int M = 1 << g.tile_log2, j = nth * g.H + h, rt = j >> g.tile_log2;
        const LatentShares shares = latent_shares(line[4 + s], sw.units, rt, sw.row_tiles, run);
        const int used = shares.count;
        const int64_t first = latent_slot(shares.first, s, rt, g.row_tiles) * M + (j & (M - 1));
        // (the wavefronts all work the weights out, each writes and reads the same)
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
        for (int k0 = wave; k0 < used; k0 += 8 * PER) {
            lf4_t y[8][DC / 256];
#pragma unroll
            for (int k = 0; k < 8; ++k)                              // (behind the last share it is read again, for nothing)
#pragma unroll
                for (int c = 0; c < DC / 256; ++c)
                    y[k][c] = *reinterpret_cast<const lf4_t*>(src + static_cast<int64_t>(min(k0 + k * PER, used - 1)) * M * DC + c * 256);
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k0 + k * PER < used) {
                    const float f = weight[k0 + k * PER];
#pragma unroll
                    for (int c = 0; c < DC / 256; ++c) x[c] += y[k][c] * f;
                }
        }
    }
#pragma unroll
    for (int c = 0; c < DC / 256; ++c) parts[wave][lane + c * 64] = x[c];
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int k = 1; k < PER; ++k)
#pragma unroll
        for (int c = 0; c < DC / 256; ++c) x[c] += parts[k][lane + c * 64];
    const float inv = total > 0.0f ? 1.0f / total : total;           // a row that sees nothing: zeros; NaN stays
#pragma unroll
    for (int c = 0; c < DC / 256; ++c) {
        lh4_t a, b;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float y = x[c][e] * inv;
            a[e] = static_cast<_Float16>(y);
            b[e] = static_cast<_Float16>(y - static_cast<float>(a[e]));
        }
        *reinterpret_cast<lh4_t*>(hi + at * DC + lane * 4 + c * 256) = a;
        *reinterpret_cast<lh4_t*>(lo + at * DC + lane * 4 + c * 256) = b;
    }
}

// Values from joined latents: out[h] = w_v[h]^T (hi + lo) for 16 rows of one head and 64 of its columns in a workgroup, whose wavefronts have a
// quarter of the contraction each.  Bound by reading w: a lane loads four adjacent columns of eight latents, column 4 l16 + n is row l16 of the
// n-th product's operand.  Grid (H * DV / 64, row blocks), 256 threads.
template <int DC, int DV>
__global__ __launch_bounds__(256) void latent_values_kernel(LatentView v, LatentGeom g, const _Float16* __restrict__ w,
                                                            const int32_t* __restrict__ row_start, const _Float16* __restrict__ hi,
                                                            const _Float16* __restrict__ lo, _Float16* __restrict__ out) {
    constexpr int kSteps = DC / 32 / 4;
    __shared__ lf4_t sums[4][16][17];
    const int lane = threadIdx.x & 63, l16 = lane & 15, g4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    const int h = static_cast<int>(blockIdx.x) / (DV / 64), col0 = static_cast<int>(blockIdx.x) % (DV / 64) * 64;
    const int row0 = static_cast<int>(blockIdx.y) * 16, all = v.p.n_seqs * g.max_rows;
    const int64_t w_row = static_cast<int64_t>(g.H) * (g.Dk + DV);
    const int c0 = wave * (DC / 4) + 8 * g4;
    const _Float16* w_at = w + static_cast<int64_t>(h) * (g.Dk + DV) + g.Dk + col0 + 4 * l16 + c0 * w_row;
    const int64_t from = (static_cast<int64_t>(min(row0 + l16, all - 1)) * g.H + h) * DC + c0;
    u2_t wx[kSteps][8];
    h8_t a[kSteps], b[kSteps];
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
#pragma unroll
        for (int e = 0; e < 8; ++e) wx[k][e] = *reinterpret_cast<const u2_t*>(w_at + (k * 32 + e) * w_row);
        a[k] = *reinterpret_cast<const h8_t*>(hi + from + k * 32);
        b[k] = *reinterpret_cast<const h8_t*>(lo + from + k * 32);
    }
    lf4_t acc[4];
#pragma unroll
    for (int n = 0; n < 4; ++n) acc[n] = lf4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < kSteps; ++k)
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            u4_t f;
#pragma unroll
            for (int p = 0; p < 4; ++p)
                f[p] = __builtin_amdgcn_perm(wx[k][2 * p + 1][n / 2], wx[k][2 * p][n / 2], n % 2 ? 0x07060302u : 0x05040100u);
            acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8_t, f), b[k], acc[n], 0, 0, 0);
            acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8_t, f), a[k], acc[n], 0, 0, 0);
        }
    // acc[n][e]: column col0 + 4 (4 g4 + e) + n of row l16
#pragma unroll
    for (int e = 0; e < 4; ++e) sums[wave][4 * g4 + e][l16] = lf4_t{acc[0][e], acc[1][e], acc[2][e], acc[3][e]};
    __syncthreads();
    const int r = static_cast<int>(threadIdx.x) / 16, quad = static_cast<int>(threadIdx.x) % 16, row = row0 + r;
    if (row >= all) return;
    const int s = row / g.max_rows, nth = row - s * g.max_rows;
    const SeqRows rows = seq_rows(row_start, s, g.n_rows);
    if (nth >= min(rows.count, g.max_rows)) return;
    const lf4_t x = (sums[0][quad][r] + sums[1][quad][r]) + (sums[2][quad][r] + sums[3][quad][r]);
    lh4_t y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = static_cast<_Float16>(x[e]);
    *reinterpret_cast<lh4_t*>(out + (static_cast<int64_t>(rows.first + nth) * g.H + h) * DV + col0 + 4 * quad) = y;
}

}  // namespace kvs
