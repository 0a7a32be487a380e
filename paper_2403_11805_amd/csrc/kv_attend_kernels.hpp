// Attention of the newest tokens to one layer of their sequences' pages, as the pages are packed.
//
// A wavefront walks units of 32 tokens, two tiles of 16; a tile lies in one page (chunk_tokens is a multiple of 16), so its
// width and addresses are wave-uniform.  Both products run on 16x16x32 MFMAs in the transposed form,
//     S^T[token][row] = K Q^T,      O^T[dim][row] = V^T P^T,
// in which a lane keeps one query row (lane % 16) throughout: reference, sum and rescaling of a row need no exchange
// between lanes, and the four S^T values of a lane (tokens 4 * (lane / 16) + 0..3 of each tile) ARE the operand P^T of the second
// product, without a move.  The k index of an MFMA is free as long as both operands agree on it:
//   K: a lane reads one contiguous piece of its token per group of dimensions; within eight dimensions Q is held in the pairs (0,4) (1,5)
//      (2,6) (3,7), which is how codes of 8, 4 and 2 bits fall out of their words (fp16 is put into that order);
//   V: k runs over the unit's tokens, four per quarter wavefront and tile; a lane reads the rows of its tokens at its own D/16
//      contiguous dimensions, and one v_perm per register pairs two tokens.
// A code of b bits in the mantissa of a half, the other bits 0, is the subnormal number code * 2^-24 (times the power of two of where
// it stands) exactly, so a shift and a mask make an operand of two codes.  K is not dequantised: the MFMAs sum q * code per group, and
// scale and minimum enter once per (token, group),
//     S = sum_g (s_g / 2^-24) acc_g + mn_g qsum_g.
// An MFMA lines its products up by the exponents without shifting a subnormal's leading zeros out first, and keeps so many bits less of
// them: K's codes therefore stand at the mantissa's top (weights of 2-bit pages are off by 8e-7 so, by 7e-5 with
// the codes at its low end; of 8-bit pages by 4e-7, and by up to 1.7e-6 at its low end, a shift less per pair).
// V is dequantised by one v_fma_mix per element, fp16(code * s + mn), the power of two taken into s: off by 2^-11 of itself at most, as the
// result is when it is rounded.  (A Load rounds the product to binary32 first, so that its half can be the neighbour of this one.)  More
// bits would take a second MFMA and half as many operands again; as it is, results over packed pages are off by 2.3e-4 of their norm
// against 64 bits, and by 2.0e-4 if V is not rounded.  P enters as the sum of two halves (22 bits): the second MFMA costs nothing next to the
// loads, and 11 bits would be the largest error of a result.
//
// What bounds it.  fp16 pages: HBM, 16 contexts of 32768 tokens, 32 query heads on 8 kv heads of 128 (2.15 GB) 364 to 375 us, 5.7 to 5.9 TB/s;
// one of 32768 30 us, of which some 6 are the chain below.  Packed pages: vector instructions, of which a unit of 32 tokens at head_dim 128
// takes 346 (8 bits) to 380 (2 bits) beside 24 MFMAs with one group per row and parameters in binary16, 406 to 441 with two in
// binary32, 196 in fp16 (at head_dim 256 a unit is 16 tokens: 320 to 342, 40 MFMAs); 24 contexts of 4096 take 47 us at 8 bits, 36 at
// 4, 34 at 2, 76 in fp16.  Short contexts: the chain of loads from the lengths to the keys and of the arithmetic behind them, 5 to 9.5
// us for one context of up to 1000 tokens (head_dim 64 to 256).
#pragma once

#include "kv_launch_rules.hpp"
#include "kv_pages_kernels.hpp"

namespace kvs {

typedef float f4_t __attribute__((ext_vector_type(4)));
typedef _Float16 h2_t __attribute__((ext_vector_type(2)));
typedef _Float16 h4_t __attribute__((ext_vector_type(4)));

constexpr int kAttendWaves = 4;
constexpr float kTop = 7.0f;         // a row's reference is set 2^7 below its largest logit so far ...
constexpr float kSlack = 15.0f;      // ... and moves when a logit passes 2^15 above it: probabilities stay in fp16's range, and those
                                     // 2^-31 below the largest still count
constexpr int kNowhere = -1;         // first token of a tile that is not there

struct AttendGeom {
    int32_t layer, n_rows, max_rows;
    int32_t per;                     // query heads per kv head
    int32_t rows;                    // per * max_rows: query rows of a (sequence, kv head) pair
    int32_t row_tiles;               // ceil(rows / 16)
    int32_t tile_rows;               // min(16, rows)
    int32_t groups;                  // workgroups that the work of all sequences is divided among
    int32_t step;                    // units that a workgroup's wavefronts take at once
    int64_t q_stride;
    float scale_log2e;               // log2(e) / sqrt(D)
};

// How the work is divided.  The units of all sequences, kv heads and row tiles stand in one line (sequence by sequence, head by head),
// and every workgroup takes an equal run of it, whatever the lengths are: all run at once and end together.  The lengths are on the
// device, so a workgroup finds its run itself, a lane per sequence, 64 sequences a step.
//   Little work: a run is `step` units, one of its wavefronts' steps, or two such, and the units of every (kv head, row tile) pair are
//     rounded up to whole runs, so that a workgroup has part of one pair only.
//   More than that: a run goes on through the next pair where one ends.  In front of a pair's units the line has kPieceCost places for
//     what beginning and ending a piece takes, so that runs through many short ones are shorter.
// One context, 32 kv heads of 128, whole steps against the line: 64 tokens 6.8 against 11.2 us, 512 8.3 and 12.5, 2048 10.6 and 12.8, 4096
// 14.1 and 16.1.  24 ragged contexts: 49 us with 8 places, 50 with 16, 71 with none; 8 of 32 kv heads 43, 45 and 43.
struct SeqWork {
    int n, first, count;             // tokens; its new rows
    __device__ __forceinline__ int units() const { return (n + 31) >> 5; }                 // of 32 tokens
    __device__ __forceinline__ int row_tiles(const AttendGeom& g) const { return (min(count, g.max_rows) * g.per + 15) >> 4; }
};
__device__ __forceinline__ SeqWork work_of(const PagesView& v, const AttendGeom& g, const int32_t* __restrict__ row_start, int s) {
    SeqWork w = {0, 0, 0};
    if (s < v.n_seqs) {
        w.n = seq_len(v, s);
        const SeqRows rows = seq_rows(row_start, s, g.n_rows);
        w.first = rows.first;
        w.count = rows.count;
    }
    return w;
}
__device__ __forceinline__ SeqWork of_lane(const SeqWork& w, int l) {
    return {__builtin_amdgcn_readlane(w.n, l), __builtin_amdgcn_readlane(w.first, l), __builtin_amdgcn_readlane(w.count, l)};
}

// Sum over the lanes up to this one (all active): within rows of 16, then the rows' last lanes.
__device__ __forceinline__ int prefix_sum(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);      // row_shr 1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);      // lane 15 to row 1, 47 to row 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);      // lane 31 to rows 2 and 3
    return x;
}

// Where the lanes' sequences lie in the line.
struct Line {
    SeqWork mine;                    // of sequence s0 + lane
    int s0, end;                     // end: of the lane's sequence
    int round, cost;                 // of a pair's places
    int run;                         // places of a workgroup's run

    __device__ __forceinline__ int each(const SeqWork& w) const { return attend_places(w.units(), round, cost); }
    __device__ __forceinline__ void start(const PagesView& v, const AttendGeom& g, const int32_t* __restrict__ row_start, int lane) {
        s0 = 0;
        mine = work_of(v, g, row_start, lane);
        const int units = mine.units(), pairs = v.Hkv * mine.row_tiles(g);
        const int one = prefix_sum(attend_places(units, g.step, 0) * pairs), two = prefix_sum(attend_places(units, 2 * g.step, 0) * pairs);
        const int long_ = prefix_sum(attend_places(units, 1, kPieceCost) * pairs);
        int t1 = __builtin_amdgcn_readlane(one, 63), t2 = __builtin_amdgcn_readlane(two, 63), tl = __builtin_amdgcn_readlane(long_, 63);
        for (int s = 64; s < v.n_seqs; s += 64) {
            const SeqWork w = work_of(v, g, row_start, s + lane);
            const int u = w.units(), p = v.Hkv * w.row_tiles(g);
            t1 += __builtin_amdgcn_readlane(prefix_sum(attend_places(u, g.step, 0) * p), 63);
            t2 += __builtin_amdgcn_readlane(prefix_sum(attend_places(u, 2 * g.step, 0) * p), 63);
            tl += __builtin_amdgcn_readlane(prefix_sum(attend_places(u, 1, kPieceCost) * p), 63);
        }
        const AttendDivision d = attend_division(t1, t2, tl, g.groups, g.step);
        round = d.round;
        cost = d.cost;
        run = d.run;
        end = round == g.step ? one : round == 1 ? long_ : two;
    }
    __device__ __forceinline__ void next(const PagesView& v, const AttendGeom& g, const int32_t* __restrict__ row_start, int lane) {
        const int before = __builtin_amdgcn_readlane(end, 63);
        s0 += 64;
        mine = work_of(v, g, row_start, s0 + lane);
        end = before + prefix_sum(each(mine) * v.Hkv * mine.row_tiles(g));
    }
};

// Partial results: a workgroup leaves those of pair p (numbered over all sequences) at slot workgroup + p, which no other has: from one
// piece of the line to the next the workgroup, the pair or both go up.
__device__ __forceinline__ int64_t pair_number(const PagesView& v, const AttendGeom& g, int s, int pair) {
    return static_cast<int64_t>(s) * v.Hkv * g.row_tiles + pair;
}

// What attend_kernel leaves of the line for the launch behind it, so that that one need not go through all sequences again: the places of a
// pair and of a run, then where each sequence ends (only of those that have places).
struct LineNote {
    int round, cost, run, unused;
};
__device__ __forceinline__ void leave_line(int32_t* __restrict__ note, const PagesView& v, const Line& line, int lane) {
    if (line.s0 + lane < v.n_seqs) note[4 + line.s0 + lane] = line.end;
}

// The shares of row j of (sequence s, kv head h): `used` slots from `first` on.
struct RowShares {
    SeqWork w;
    int used;
    int64_t first;
};
__device__ __forceinline__ RowShares row_shares(const PagesView& v, const AttendGeom& g, const int32_t* __restrict__ row_start,
                                                const int32_t* __restrict__ note, int s, int h, int j) {
    RowShares x;
    x.w = work_of(v, g, row_start, s);
    x.used = 0;
    x.first = 0;
    const int units = x.w.units(), row_tiles = x.w.row_tiles(g);
    if (units == 0 || row_tiles == 0) return x;
    const LineNote l = *reinterpret_cast<const LineNote*>(note);
    const int pair = h * row_tiles + j / 16;
    const int begin = note[4 + s] - attend_places(units, l.round, l.cost) * (v.Hkv * row_tiles - pair) + l.cost, wg = begin / l.run;
    x.used = (begin + units - 1) / l.run - wg + 1;
    x.first = wg + pair_number(v, g, s, pair);
    return x;
}

__device__ __forceinline__ uint32_t perm(uint32_t hi, uint32_t lo, uint32_t sel) { return __builtin_amdgcn_perm(hi, lo, sel); }

// Eight halves in the order (0,4) (1,5) (2,6) (3,7).
__device__ __forceinline__ u4_t paired(const uint32_t* w) {
    return u4_t{perm(w[2], w[0], 0x05040100u), perm(w[2], w[0], 0x07060302u), perm(w[3], w[1], 0x05040100u), perm(w[3], w[1], 0x07060302u)};
}

constexpr float kCode = 16777216.0f;       // 2^24: what a code in the low bits of a half has to be multiplied by

// Eight dimensions of K from their 8 * W bits, in the order of paired(); codes come out as code / k_code<W>().  (W = 2: the
// bits of dimensions 0-3 in the upper byte of the low half, those of 4-7 in that of the high one.)
template <int W> __device__ __forceinline__ constexpr float k_code() { return kCode / (W == 8 ? 4 : W == 4 ? 64 : W == 2 ? 256 : 1); }
template <int W> __device__ __forceinline__ u4_t k_operand(const uint32_t* w) {
    if constexpr (W == 16) return paired(w);
    else if constexpr (W == 8)
        return u4_t{perm(w[1], w[0], 0x0c040c00u) << 2, perm(w[1], w[0], 0x0c050c01u) << 2, perm(w[1], w[0], 0x0c060c02u) << 2,
                    perm(w[1], w[0], 0x0c070c03u) << 2};
    else if constexpr (W == 4)
        return u4_t{(w[0] << 6) & 0x03c003c0u, (w[0] << 2) & 0x03c003c0u, (w[0] >> 2) & 0x03c003c0u, (w[0] >> 6) & 0x03c003c0u};
    else return u4_t{w[0] & 0x03000300u, (w[0] >> 2) & 0x03000300u, (w[0] >> 4) & 0x03000300u, (w[0] >> 6) & 0x03000300u};
}

__device__ __forceinline__ h8_t as_h8(u4_t v) { return __builtin_bit_cast(h8_t, v); }

// Codes of two tokens for dimension d of the words a and b that hold them, as a pair of subnormal halves; those of odd dimensions of
// widths 4 and 2 are left 2^W times as large (their scale makes up for it).
template <int W, int d> __device__ __forceinline__ uint32_t v_codes(uint32_t a, uint32_t b) {
    if constexpr (W == 8) return perm(b, a, 0x0c040c00u + 0x00010001u * d);
    else if constexpr (W == 4) {
        const uint32_t x = perm(b, a, d < 4 ? 0x05040100u : 0x07060302u);
        return (x >> (4 * (d & 2))) & (d & 1 ? 0x00f000f0u : 0x000f000fu);
    } else {
        const uint32_t x = perm(b, a, d < 8 ? 0x05040100u : 0x07060302u);
        return (x >> (2 * (d & 6))) & (d & 1 ? 0x000c000cu : 0x00030003u);
    }
}

// BYTES contiguous bytes as 32-bit words (less than four: the low end of one).
template <int BYTES> __device__ __forceinline__ void load_words(const uint8_t* p, uint32_t* w) {
    if constexpr (BYTES >= 16) {
#pragma unroll
        for (int i = 0; i < BYTES / 16; ++i) {
            const u4_t x = reinterpret_cast<const u4_t*>(p)[i];
            w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w;
        }
    } else if constexpr (BYTES == 8) {
        const u2_t x = *reinterpret_cast<const u2_t*>(p);
        w[0] = x.x; w[1] = x.y;
    } else if constexpr (BYTES == 4) w[0] = *reinterpret_cast<const uint32_t*>(p);
    else if constexpr (BYTES == 2) w[0] = *reinterpret_cast<const uint16_t*>(p);
    else w[0] = *p;
}

// The state of a wavefront's walk over a pair's tokens, for one tile of 16 query rows.
template <int D> struct RowState {
    f4_t o[D / 16];                  // o[i][r]: dimension (D/16) * (4 * (lane / 16) + r) + i of row lane % 16
    float ref, sum;                  // the row's reference (same in its four lanes), the lane's own share of the sum
};

// What is loaded of a tile, as it lies in memory: K at the lane's token with the parameters of the lane's four tokens 4q .. 4q+3 in
// every group; V of these four tokens at the lane's dimensions, with the parameters of the group of these (side by side where there
// is one group, else each in a word of its own).  HP: parameters in binary16.
template <int D, int G, int W, bool HP> struct KRegs {
    static constexpr int kWords = D * W / 128, kParams = W == 16 ? 1 : 4 * (D / G) / (HP ? 2 : 1);
    uint32_t k[kWords], s[kParams], m[kParams];
};
template <int D, int G, int W, bool HP> struct VRegs {
    static constexpr int kWords = D / 16 * W / 32 > 0 ? D / 16 * W / 32 : 1, kParams = W == 16 ? 1 : (D == G && HP ? 2 : 4);
    uint32_t v[4][kWords], s[kParams], m[kParams];
    __device__ __forceinline__ static float param(const uint32_t* w, int r) {
        if constexpr (!HP) return __builtin_bit_cast(float, w[r]);
        else if constexpr (D == G) return static_cast<float>(__builtin_bit_cast(h2_t, w[r / 2])[r % 2]);
        else return static_cast<float>(__builtin_bit_cast(h2_t, w[r])[0]);
    }
};

// Parameter i of those loaded.
template <bool HP> __device__ __forceinline__ float param(const uint32_t* w, int i) {
    if constexpr (HP) return static_cast<float>(__builtin_bit_cast(h2_t, w[i / 2])[i % 2]);
    else return __builtin_bit_cast(float, w[i]);
}

// Where a tile lies (all wave-uniform): its K codes and the K scales of its first token, its first token, and how many of its 16 tokens
// there are.
struct Tile {
    const uint8_t *codes, *scales;
    int first, valid;
};
// From there to the minima (any width), and to the same of V.
struct SlabSteps {
    uint64_t mn, v_codes, v_scales;
};

// A lane's byte offsets from a tile's K codes, V codes, parameters, and parameters of the group of its V dimensions: the same for every
// tile of a width, so that an address is a wave-uniform base and one of these.
template <int D, int G, int W, bool HP> struct LaneAt {
    static constexpr int kRowBytes = D * W / 8, kPiece = G / 4 * W / 8;       // bytes of a token's row, of a lane's piece of K per group
    static constexpr int kMine = D / 16 * W / 8, kParam = HP ? 2 : 4, kParams = 4 * (D / G) * kParam;
    uint32_t k, v, p, vp;
    __device__ __forceinline__ explicit LaneAt(int lane)
        : k(static_cast<uint32_t>((lane & 15) * kRowBytes + (lane >> 4) * kPiece)),
          v(static_cast<uint32_t>((lane >> 4) * 4 * kRowBytes + (lane & 15) * kMine)), p(static_cast<uint32_t>((lane >> 4) * kParams)),
          vp(static_cast<uint32_t>((lane >> 4) * kParams + (lane & 15) * (D / 16) / G * kParam)) {}
    // Where loads are issued the offsets have to be 32-bit numbers made there (not 64-bit ones made in front of the loop) for the loads to
    // take base and offset as they are: an instruction less per load.
    __device__ __forceinline__ void here() { asm volatile("" : "+v"(k), "+v"(v), "+v"(p), "+v"(vp)); }
};

// Issues the loads of a tile.  (WHOLE: all of its 16 tokens are there.)
template <int D, int G, int W, bool HP>
__device__ __forceinline__ void load_k(KRegs<D, G, W, HP>& t, const Tile& tile, const SlabSteps& step, const LaneAt<D, G, W, HP>& at) {
    using A = LaneAt<D, G, W, HP>;
#pragma unroll
    for (int gi = 0; gi < D / G; ++gi) load_words<A::kPiece>(tile.codes + at.k + gi * (G * W / 8), &t.k[gi * A::kPiece / 4]);
    if constexpr (W != 16) {
        load_words<A::kParams>(tile.scales + at.p, t.s);
        load_words<A::kParams>(tile.scales + step.mn + at.p, t.m);
    }
}
// (What lies behind a sequence's tokens may be anything: V rows of missing tokens are replaced by the last one there is, and their
// parameters are not used.)
template <bool WHOLE, int D, int G, int W, bool HP>
__device__ __forceinline__ void load_v(VRegs<D, G, W, HP>& t, const Tile& tile, const SlabSteps& step, const LaneAt<D, G, W, HP>& at, int lane) {
    using A = LaneAt<D, G, W, HP>;
    const uint8_t* vb = tile.codes + step.v_codes;
    if constexpr (WHOLE) {
#pragma unroll
        for (int r = 0; r < 4; ++r) load_words<A::kMine>(vb + at.v + r * A::kRowBytes, t.v[r]);
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            load_words<A::kMine>(vb + static_cast<uint32_t>(min((lane >> 4) * 4 + r, tile.valid - 1) * A::kRowBytes + (lane & 15) * A::kMine), t.v[r]);
    }
    if constexpr (W != 16) {
        const uint8_t *sb = tile.scales + step.v_scales, *mb = sb + step.mn;
        if constexpr (D == G) {
            load_words<A::kParams>(sb + at.vp, t.s);
            load_words<A::kParams>(mb + at.vp, t.m);
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                load_words<A::kParam>(sb + at.vp + r * (D / G) * A::kParam, t.s + r);
                load_words<A::kParam>(mb + at.vp + r * (D / G) * A::kParam, t.m + r);
            }
        }
    }
}

// q K^T of a tile; for codes that divided by k_code (qsum is, too).
template <int D, int G, int W, bool HP>
__device__ __forceinline__ f4_t tile_logits(const KRegs<D, G, W, HP>& t, const u4_t* q, const float* qsum) {
    constexpr int NG = D / G, kPer = G / 32;
    f4_t s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int gi = 0; gi < NG; ++gi) {
        f4_t acc = W == 16 ? s : f4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int j = gi * kPer + i;
            u4_t a;
            if constexpr (W == 2) {
                const uint32_t one = perm(0u, t.k[j / 2], (j & 1) ? 0x030c020cu : 0x010c000cu);
                a = k_operand<2>(&one);
            } else a = k_operand<W>(&t.k[j * (W / 4)]);
            acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_h8(a), as_h8(q[j]), acc, 0, 0, 0);
        }
        if constexpr (W == 16) s = acc;
        else {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float m = param<HP>(t.m, r * NG + gi);
                s[r] = __builtin_fmaf(param<HP>(t.s, r * NG + gi), acc[r], gi ? __builtin_fmaf(m, qsum[gi], s[r]) : m * qsum[gi]);
            }
        }
    }
    return s;
}

// Scales and minima of a lane's four tokens in the group of its dimensions; `odd` for codes that v_codes leaves larger.
template <int W> struct VScale {
    float s[4], odd[4], m[4];
};
template <int D, int G, int W, bool HP> __device__ __forceinline__ VScale<W> v_scale(const VRegs<D, G, W, HP>& t) {
    VScale<W> x;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        x.s[r] = __builtin_fmaf(t.param(t.s, r), kCode, 0.0f);
        x.m[r] = t.param(t.m, r);
        x.odd[r] = x.s[r] * (W == 4 ? 1.0f / 16 : 1.0f / 4);            // (unused at width 8)
    }
    return x;
}

// V^T of one dimension for tokens (4q + 2j, 4q + 2j + 1) of a tile, as a pair of halves.
template <int D, int G, int W, bool HP, int i>
__device__ __forceinline__ uint32_t v_pair(const VRegs<D, G, W, HP>& t, const VScale<W>& x, int j) {
    if constexpr (W == 16) return perm(t.v[2 * j + 1][i / 2], t.v[2 * j][i / 2], (i & 1) ? 0x07060302u : 0x05040100u);
    else {
        constexpr int kIn = 32 / W;                                     // dimensions of a word
        constexpr bool odd = W != 8 && (i & 1);
        const h2_t h = __builtin_bit_cast(h2_t, v_codes<W, i % kIn>(t.v[2 * j][i / kIn], t.v[2 * j + 1][i / kIn]));
        h2_t y;
        y[0] = static_cast<_Float16>(__builtin_fmaf(static_cast<float>(h[0]), odd ? x.odd[2 * j] : x.s[2 * j], x.m[2 * j]));
        y[1] = static_cast<_Float16>(__builtin_fmaf(static_cast<float>(h[1]), odd ? x.odd[2 * j + 1] : x.s[2 * j + 1], x.m[2 * j + 1]));
        return __builtin_bit_cast(uint32_t, y);
    }
}

// O^T += V^T P^T of a unit of NT tiles, two dimensions at a time (an MFMA that adds to the sum of the one right before it would wait for
// it); P as the sum of two halves.
template <int NT> struct Halves;
template <> struct Halves<1> { typedef h4_t type; };
template <> struct Halves<2> { typedef h8_t type; };
__device__ __forceinline__ f4_t mfma(h8_t a, h8_t b, f4_t c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f4_t mfma(h4_t a, h4_t b, f4_t c) { return __builtin_amdgcn_mfma_f32_16x16x16f16(a, b, c, 0, 0, 0); }
template <int D, int G, int W, bool HP, int NT, int i>
__device__ __forceinline__ typename Halves<NT>::type v_operand(const VRegs<D, G, W, HP>* t, const VScale<W>* x) {
    const u2_t a = {v_pair<D, G, W, HP, i>(t[0], x[0], 0), v_pair<D, G, W, HP, i>(t[0], x[0], 1)};
    if constexpr (NT == 1) return __builtin_bit_cast(h4_t, a);
    else return as_h8(u4_t{a.x, a.y, v_pair<D, G, W, HP, i>(t[1], x[1], 0), v_pair<D, G, W, HP, i>(t[1], x[1], 1)});
}
template <int D, int G, int W, bool HP, int NT, int i = 0>
__device__ __forceinline__ void unit_values(const VRegs<D, G, W, HP>* t, const VScale<W>* x, const typename Halves<NT>::type& hi,
                                            const typename Halves<NT>::type& lo, RowState<D>& st) {
    const auto a = v_operand<D, G, W, HP, NT, i>(t, x), b = v_operand<D, G, W, HP, NT, i + 1>(t, x);
    st.o[i] = mfma(a, lo, st.o[i]);
    st.o[i + 1] = mfma(b, lo, st.o[i + 1]);
    st.o[i] = mfma(a, hi, st.o[i]);
    st.o[i + 1] = mfma(b, hi, st.o[i + 1]);
    if constexpr (i + 2 < D / 16) unit_values<D, G, W, HP, NT, i + 2>(t, x, hi, lo, st);
}

// What a wavefront knows of its rows.
template <int D, int G> struct RowsOfWave {
    u4_t q[D / 32];                            // the lane's pieces, in the order of paired()
    float qsum[D / G];                         // of every group, the row's sum of q
    int last;                                  // the last token the lane's row sees (-1: none)
    int all_see;                               // tokens up to this one are seen by every row
    float* logits;                             // where the row's logits go (NULL: nowhere)
    float scale;
};

// A workgroup's batch of up to 64 tiles, one per lane of each of its wavefronts: what a Tile says.
struct TileBatch {
    uint64_t codes, scales;
    int tile0;                                 // lane l has tile tile0 + l
};

__device__ __forceinline__ uint64_t lane_value(uint64_t v, int lane) {
    const uint32_t lo = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v), lane));
    const uint32_t hi = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v >> 32), lane));
    return static_cast<uint64_t>(hi) << 32 | lo;
}

// The next NT of the batch's `tiles` (a bit each); a last one without a partner comes twice, the second time nowhere.
template <int NT> __device__ __forceinline__ void next_tiles(uint64_t& tiles, const TileBatch& tb, int n, uint8_t* pool, Tile* tile) {
    int at = __builtin_ctzll(tiles);
#pragma unroll
    for (int k = 0; k < NT; ++k) {
        if (k) at = tiles ? __builtin_ctzll(tiles) : at;
        tile[k].codes = pool + lane_value(tb.codes, at);
        tile[k].scales = pool + lane_value(tb.scales, at);
        const int first = 16 * (tb.tile0 + at);
        tile[k].valid = min(16, n - first);
        tile[k].first = k && !tiles ? kNowhere : first;
        tiles &= tiles - 1;                                              // (0 stays 0)
    }
}

// The wavefront's share of a batch's tiles of one width: tiles are put together within their width, whatever the order of the pages
// (the order of tokens does not matter to attention), and the units of NT, counted over all widths, go to the wavefronts in turn.
// (Without a branch: copies that the compiler made of registers where a branch of some lanes ended were made for these lanes only, when the
// kernel had more to hold than its registers; tests/test_kernel_resources.py keeps it below that.)
template <int NT> __device__ __forceinline__ uint64_t own_tiles(uint64_t all, int wave, int& units) {
    const int rank = __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(all >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(all), 0));
    const int turn = (units + rank / NT) & (kAttendWaves - 1);
    units += (__builtin_popcountll(all) + NT - 1) / NT;
    return all & __ballot(turn == wave);
}

// What a walk over tiles of one width needs beside them.
template <int D, int G, int W, bool HP> struct WidthWalk {
    SlabSteps step;
    float qsum[D / G], scale;                  // of what tile_logits takes and gives (scale: logits in units of log2)
    __device__ __forceinline__ WidthWalk(const PagesView& v, const RowsOfWave<D, G>& rw) {
        const uint64_t rows = static_cast<uint64_t>(v.T) * static_cast<uint32_t>(v.Hkv), params = static_cast<uint32_t>(v.groups * (HP ? 2 : 4));
        step = {static_cast<uint64_t>(v.slabs) * v.T * params, rows * (D * W / 8), rows * params};
#pragma unroll
        for (int i = 0; i < D / G; ++i) qsum[i] = rw.qsum[i] * (1.0f / k_code<W>());
        scale = W == 16 ? rw.scale : rw.scale * k_code<W>();
    }
};

// The probabilities of a unit's logits s (in units of 1 / scale) against the rows' references, which move if they have to; the
// sums take them in.
template <int D, int NT>
__device__ __forceinline__ void probabilities(const f4_t* s, float scale, RowState<D>& st, typename Halves<NT>::type& hi, typename Halves<NT>::type& lo) {
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < NT; ++k) top = fmaxf(fmaxf(fmaxf(s[k][0], s[k][1]), fmaxf(s[k][2], s[k][3])), top);
    top *= scale;
    if (__ballot(top > st.ref + kSlack)) {                               // (uniform)
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const bool moves = top > st.ref + kSlack;
        const float to = moves ? top - kTop : st.ref, f = moves ? __builtin_amdgcn_exp2f(st.ref - to) : 1.0f;
        st.ref = to;
        st.sum *= f;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) st.o[i] *= f;
    }
    const float ref = st.ref == -INFINITY ? 0.0f : st.ref;               // (a row that has seen nothing: every logit is -inf)
    // P = hi + lo: hi has the leading 11 bits of e, so that both conversions are exact (but for what lies below 2^-24)
#pragma unroll
    for (int k = 0; k < NT; ++k)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[k][r], scale, -ref));
            const float lead = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, e) & 0xffffe000u);
            st.sum += e;
            hi[4 * k + r] = static_cast<_Float16>(lead);
            lo[4 * k + r] = static_cast<_Float16>(e - lead);
        }
}

// A wavefront's tiles of width W that every row sees whole, NT at a time.  K of the next unit is loaded once K of this one has been used,
// and V likewise: the loads are in flight during the other half of the arithmetic, without a second set of registers.
template <int D, int G, int W, bool HP, int NT>
__device__ __forceinline__ void walk(uint64_t tiles, const TileBatch& tb, int n, const PagesView& v, const RowsOfWave<D, G>& rw,
                                     RowState<D>& st, int lane) {
    if (!tiles) return;
    // What depends on the lane is worked out here, width by width: the compiler would keep it in registers for all four.
    asm volatile("" : "+v"(lane));
    const int q4 = lane >> 4;
    const WidthWalk<D, G, W, HP> ww(v, rw);
    KRegs<D, G, W, HP> kr[NT];
    VRegs<D, G, W, HP> vr[NT];
    Tile tile[NT], next[NT];
    LaneAt<D, G, W, HP> at(lane);
    next_tiles<NT>(tiles, tb, n, v.pool, next);
#pragma unroll
    for (int k = 0; k < NT; ++k) load_k<D, G, W, HP>(kr[k], next[k], ww.step, at);
#pragma unroll
    for (int k = 0; k < NT; ++k) load_v<true, D, G, W, HP>(vr[k], next[k], ww.step, at, lane);
    bool more = true;
    while (more) {
        f4_t s[NT];
#pragma unroll
        for (int k = 0; k < NT; ++k) {
            tile[k] = next[k];
            s[k] = tile_logits<D, G, W, HP>(kr[k], rw.q, ww.qsum);
            // (Worked out before the next K is loaded: put off behind that, what they are made of would not fit the registers beside it.)
            if constexpr (D == 256 && W != 16) asm volatile("" : "+v"(s[k]));
        }
        more = tiles != 0;
        if (more) {
            next_tiles<NT>(tiles, tb, n, v.pool, next);
            at.here();
#pragma unroll
            for (int k = 0; k < NT; ++k) load_k<D, G, W, HP>(kr[k], next[k], ww.step, at);
        }
#pragma unroll
        for (int k = 0; k < NT; ++k) {
            if (k && tile[k].first == kNowhere) s[k] = f4_t{-INFINITY, -INFINITY, -INFINITY, -INFINITY};             // (uniform)
            else if (rw.logits) *reinterpret_cast<f4_t*>(rw.logits + tile[k].first + 4 * q4) = s[k] * ww.scale;
        }
        typename Halves<NT>::type hi, lo;
        probabilities<D, NT>(s, ww.scale, st, hi, lo);
        VScale<W> x[NT];
        if constexpr (W != 16) {
#pragma unroll
            for (int k = 0; k < NT; ++k) x[k] = v_scale<D, G, W, HP>(vr[k]);
        }
        unit_values<D, G, W, HP, NT>(vr, x, hi, lo, st);
        if (more) {
            at.here();
#pragma unroll
            for (int k = 0; k < NT; ++k) load_v<true, D, G, W, HP>(vr[k], next[k], ww.step, at, lane);
        }
    }
}

// V^T of a tile, every dimension of the lane's, as operands.
template <int D, int G, int W, bool HP, int i = 0>
__device__ __forceinline__ void tile_values(const VRegs<D, G, W, HP>& t, const VScale<W>& x, u2_t* y) {
    y[i] = u2_t{v_pair<D, G, W, HP, i>(t, x, 0), v_pair<D, G, W, HP, i>(t, x, 1)};
    if constexpr (i + 1 < D / 16) tile_values<D, G, W, HP, i + 1>(t, x, y);
}

// A wavefront's tiles of width W of which some row does not see some token: a sequence's last one or two, by themselves, so that nothing of
// this takes registers or instructions from the walk above.  Logits behind a row's token are left out.  0 * V is 0 only if
// V is finite: where a token that some row does not see has a value that is not (as it enters the product, a half: code * scale + mn can
// pass a half's range with finite parameters), the token counts as 0 for all rows, and makes those that do see it NaN.
template <int D, int G, int W, bool HP>
__device__ __forceinline__ void walk_partly(uint64_t tiles, const TileBatch& tb, int n, const PagesView& v, const RowsOfWave<D, G>& rw,
                                            RowState<D>& st, int lane) {
    if (!tiles) return;
    asm volatile("" : "+v"(lane));
    const int q4 = lane >> 4;
    const WidthWalk<D, G, W, HP> ww(v, rw);
    const LaneAt<D, G, W, HP> at(lane);
    do {
        KRegs<D, G, W, HP> kr;
        VRegs<D, G, W, HP> vr;
        Tile tile;
        next_tiles<1>(tiles, tb, n, v.pool, &tile);
        load_k<D, G, W, HP>(kr, tile, ww.step, at);
        load_v<false, D, G, W, HP>(vr, tile, ww.step, at, lane);
        f4_t s = tile_logits<D, G, W, HP>(kr, rw.q, ww.qsum);
#pragma unroll
        for (int r = 0; r < 4; ++r) s[r] = tile.first + 4 * q4 + r <= rw.last ? s[r] : -INFINITY;
        if (rw.logits) *reinterpret_cast<f4_t*>(rw.logits + tile.first + 4 * q4) = s * ww.scale;
        h4_t hi, lo;
        probabilities<D, 1>(&s, ww.scale, st, hi, lo);
        VScale<W> x;
        if constexpr (W != 16) {
            x = v_scale<D, G, W, HP>(vr);
#pragma unroll
            for (int r = 0; r < 4; ++r) {                                // missing tokens: 0
                const bool there = 4 * q4 + r < tile.valid;
                x.s[r] = there ? x.s[r] : 0.0f;
                x.odd[r] = there ? x.odd[r] : 0.0f;
                x.m[r] = there ? x.m[r] : 0.0f;
            }
        }
        u2_t y[D / 16];
        tile_values<D, G, W, HP>(vr, x, y);
        typedef uint16_t us2_t __attribute__((ext_vector_type(2)));
        us2_t most[2] = {{0, 0}, {0, 0}};                                // of the magnitudes' bits, token by token
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) most[j] = __builtin_elementwise_max(most[j], __builtin_bit_cast(us2_t, y[i][j] & 0x7fff7fffu));
        uint64_t lanes[4], any = 0;
#pragma unroll
        for (int r = 0; r < 4; ++r) any |= lanes[r] = __ballot((tile.first + 4 * q4 + r > rw.all_see) & (most[r / 2][r % 2] >= 0x7c00));
        if (any) {                                                       // (uniform)
            uint32_t keep[2] = {0, 0};
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const bool bad = (lanes[r] >> (16 * q4) & 0xffffull) != 0;                 // in any of the token's lanes
                keep[r / 2] |= bad ? 0u : 0xffffu << (16 * (r % 2));
                hi[r] = (bad & (tile.first + 4 * q4 + r <= rw.last)) ? static_cast<_Float16>(NAN) : hi[r];
            }
#pragma unroll
            for (int i = 0; i < D / 16; ++i) y[i] = u2_t{y[i].x & keep[0], y[i].y & keep[1]};
        }
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            st.o[i] = mfma(__builtin_bit_cast(h4_t, y[i]), lo, st.o[i]);
            st.o[i] = mfma(__builtin_bit_cast(h4_t, y[i]), hi, st.o[i]);
        }
    } while (tiles);
}

// Where dimensions d .. d + 3 of a state's row stand in LDS: the rows' quads are exchanged by the row's number, or else the 16 rows that a
// wavefront writes at once would lie in the same banks (a row is a multiple of them).
template <int D> __device__ __forceinline__ int o_at(int state_row, int row, int d) { return state_row * D + (d ^ (row * 4)); }

// Grid: g.groups workgroups, each a run of the line.  The wavefronts of a workgroup take the pairs of tiles of a piece of the run (the part
// that lies in one sequence, kv head and row tile) in turn, each with a state of its own; the four states meet in LDS.
template <int D, int G, bool HP>
__global__ __launch_bounds__(64 * kAttendWaves, 2) void attend_kernel(PagesView v, AttendGeom g, const _Float16* __restrict__ q,
                                                                   const int32_t* __restrict__ row_start, _Float16* __restrict__ out,
                                                                   float* __restrict__ part_o, float* __restrict__ part_ml,
                                                                   float* __restrict__ logits, int32_t* __restrict__ note) {
    constexpr int DL = D / 16, NG = D / G, NT = D == 256 ? 1 : 2;      // (256: two tiles spill 42 to 119 registers)
    extern __shared__ float o_lds[];                 // [kAttendWaves][tile_rows][D]
    __shared__ float ml_lds[kAttendWaves][2][16];
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    Line line;
    int lane = threadIdx.x & 63;
    line.start(v, g, row_start, lane);
    int at = static_cast<int>(blockIdx.x) * line.run;
    const int run_begin = at, run_end = at + line.run;
    if (blockIdx.x == 0 && wave == 0) {
        if (lane == 0) *reinterpret_cast<LineNote*>(note) = LineNote{line.round, line.cost, line.run, 0};
        leave_line(note, v, line, lane);
    }
    while (at < run_end) {
        // the piece that begins at `at`: its sequence, pair and units
        uint64_t behind = __ballot(line.end > at);
        while (!behind && line.s0 + 64 < v.n_seqs) {
            const int before = __builtin_amdgcn_readlane(line.end, 63);
            line.next(v, g, row_start, lane);
            behind = __ballot(line.end > at);
            // 64 sequences are noted by the workgroup whose run they begin in (where they have no places, by one or none)
            if (wave == 0 && before >= run_begin && before < run_end) leave_line(note, v, line, lane);
        }
        if (!behind) return;                         // (the end of the line; uniform in the workgroup)
        const int l = __builtin_ctzll(behind), s = line.s0 + l;
        const SeqWork sw = of_lane(line.mine, l);
        const int row_tiles = sw.row_tiles(g), units = sw.units();
        const int each = line.each(sw), n = sw.n, local = at - (__builtin_amdgcn_readlane(line.end, l) - each * v.Hkv * row_tiles);
        const int pair = local / each, place = local - pair * each, places = min(each - place, run_end - at);
        const int u_begin = max(place - line.cost, 0), u_end = min(place + places - line.cost, units);
        const int h = pair / row_tiles, rt = pair - h * row_tiles;
        const int count = min(sw.count, g.max_rows);
        at += places;
        if (u_end <= u_begin) continue;              // the run ends in front of the pair's first unit

        // What depends on the lane is worked out piece by piece, and again where the piece ends: kept over the walk it would not fit the
        // registers at head_dim 256.
        asm volatile("" : "+v"(lane));
        // this lane's query row
        const int l16 = lane & 15, q4 = lane >> 4;
        const int j = rt * 16 + l16, nth = j / g.per, head = h * g.per + j % g.per;
        const bool ok = j < count * g.per;
        RowsOfWave<D, G> rw;
        rw.scale = g.scale_log2e;
        rw.last = ok ? n - sw.count + nth : -1;
        rw.all_see = n - sw.count + rt * 16 / g.per;
        const int none_sees = n - sw.count + min(count, (rt * 16 + 15) / g.per + 1);       // tokens from this one on are seen by no row
        rw.logits = logits && ok ? logits + ((static_cast<int64_t>(s) * v.Hkv + h) * g.rows + j) * v.N : nullptr;
        const _Float16* qp = q + static_cast<int64_t>(sw.first + (ok ? nth : 0)) * g.q_stride + (ok ? head : 0) * D;     // (count >= 1)
#pragma unroll
        for (int gi = 0; gi < NG; ++gi) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < G / 32; ++i) {
                u4_t w = *reinterpret_cast<const u4_t*>(qp + gi * G + q4 * (G / 4) + i * 8);
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = ok ? w[e] : 0u;
                const h8_t x = as_h8(w);
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += static_cast<float>(x[e]);
                const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
                rw.q[gi * (G / 32) + i] = paired(ws);
            }
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            rw.qsum[gi] = sum;
        }
        RowState<D> st;
#pragma unroll
        for (int i = 0; i < DL; ++i) st.o[i] = f4_t{0.0f, 0.0f, 0.0f, 0.0f};
        st.ref = -INFINITY;
        st.sum = 0.0f;

        const int k_slab = (g.layer * 2) * v.Hkv + h;
        const uint64_t* offs = v.off + static_cast<int64_t>(s) * v.stride;
        const uint8_t* bits = v.bits + static_cast<int64_t>(s) * v.stride;
        for (int u = u_begin; u < u_end; u += 32) {
            // the pages of the next 32 units, a tile per lane
            TileBatch tb;
            tb.tile0 = 2 * u;
            const int tile = 2 * u + lane;
            const bool in = (tile < 2 * u_end) & (tile * 16 < n);
            const int tile_page = v.page_of_tile ? static_cast<int>(__umulhi(static_cast<uint32_t>(tile), v.page_of_tile)) : tile;
            const int page = in ? tile_page : 0;
            const uint64_t off = offs[page];
            const uint32_t b = bits[page];
            // (what no row sees is left out like an absent page)
            const uint32_t width = (in & page_present(v, off, b) & (tile * 16 < none_sees)) ? b : 0u;
            const bool whole = tile * 16 + 15 <= rw.all_see;
            const uint32_t row = static_cast<uint32_t>(k_slab * v.T + tile * 16 - page * v.T);     // of the record's rows
            tb.codes = off + static_cast<uint64_t>(row) * (D / 8 * b);
            tb.scales = off + v.bit_bytes * b + static_cast<uint64_t>(row) * static_cast<uint32_t>(v.groups * (HP ? 2 : 4));
            const uint64_t of16 = __ballot(width == 16), of8 = __ballot(width == 8), of4 = __ballot(width == 4), of2 = __ballot(width == 2);
            const uint64_t seen_whole = __ballot(whole), none = __ballot(in && width == 0);
            int dealt = 0;
            const uint64_t tiles16 = own_tiles<NT>(of16 & seen_whole, wave, dealt), tiles8 = own_tiles<NT>(of8 & seen_whole, wave, dealt);
            const uint64_t tiles4 = own_tiles<NT>(of4 & seen_whole, wave, dealt), tiles2 = own_tiles<NT>(of2 & seen_whole, wave, dealt);
            const uint64_t partly = own_tiles<1>((of16 | of8 | of4 | of2) & ~seen_whole, wave, dealt);
            walk<D, G, 16, HP, NT>(tiles16, tb, n, v, rw, st, lane);
            walk<D, G, 8, HP, NT>(tiles8, tb, n, v, rw, st, lane);
            walk<D, G, 4, HP, NT>(tiles4, tb, n, v, rw, st, lane);
            walk<D, G, 2, HP, NT>(tiles2, tb, n, v, rw, st, lane);
            if (partly) {
                walk_partly<D, G, 16, HP>(partly & of16, tb, n, v, rw, st, lane);
                walk_partly<D, G, 8, HP>(partly & of8, tb, n, v, rw, st, lane);
                walk_partly<D, G, 4, HP>(partly & of4, tb, n, v, rw, st, lane);
                walk_partly<D, G, 2, HP>(partly & of2, tb, n, v, rw, st, lane);
            }
            if (logits && wave == 0) {               // what the tokens of absent tiles would have had
                for (uint64_t left = none; left; left &= left - 1) {
                    const int t = 16 * (2 * u + __builtin_ctzll(left));
                    if (rw.logits) *reinterpret_cast<f4_t*>(rw.logits + t + 4 * q4) = f4_t{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                }
            }
        }
        // the four states against one reference per row
        st.sum += __shfl_xor(st.sum, 16);
        st.sum += __shfl_xor(st.sum, 32);
        const int here = min(16, count * g.per - rt * 16);               // rows of this tile
        asm volatile("" : "+v"(lane));
        const int end_row = lane & 15, end_q4 = lane >> 4;
        if (end_q4 == 0) {
            ml_lds[wave][0][end_row] = st.ref;
            ml_lds[wave][1][end_row] = st.sum;
        }
        if (end_row < here) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int i = 0; i < DL; i += 4)
                    *reinterpret_cast<f4_t*>(o_lds + o_at<D>(wave * g.tile_rows + end_row, end_row, DL * (4 * end_q4 + r) + i)) =
                        f4_t{st.o[i][r], st.o[i + 1][r], st.o[i + 2][r], st.o[i + 3][r]};
        }
        __syncthreads();
        const bool whole = u_begin == 0 && u_end == units;
        const int64_t slot0 = (blockIdx.x + pair_number(v, g, s, pair)) * g.tile_rows;
        for (int i = wave * 64 + lane; i < here * (D / 4); i += 64 * kAttendWaves) {
            const int row = i / (D / 4), d = i % (D / 4) * 4;
            float ref = -INFINITY, sum = 0.0f;
#pragma unroll
            for (int k = 0; k < kAttendWaves; ++k) ref = fmaxf(ref, ml_lds[k][0][row]);
            f4_t o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < kAttendWaves; ++k) {
                const float m = ml_lds[k][0][row], f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - ref);
                sum += f * ml_lds[k][1][row];
                o += *reinterpret_cast<const f4_t*>(o_lds + o_at<D>(k * g.tile_rows + row, row, d)) * f;
            }
            const int64_t slot = slot0 + row;
            if (d == 0) *reinterpret_cast<float2*>(part_ml + slot * 2) = float2{ref, sum};
            if (whole) {
                const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;        // a row that sees nothing: zeros
                const int jr = rt * 16 + row;
                h4_t x;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = static_cast<_Float16>(o[e] * inv);
                *reinterpret_cast<h4_t*>(out + (static_cast<int64_t>(sw.first + jr / g.per) * v.Hq + h * g.per + jr % g.per) * D + d) = x;
            } else {
                *reinterpret_cast<f4_t*>(part_o + slot * D + d) = o;
            }
        }
        if (at < run_end) __syncthreads();           // the next piece writes to LDS again
    }
}

// Reference and sum of a row over its shares (rows first, first + step, ..), by all lanes of a wavefront together, 64 shares a step;
// weight[k] the factor of share k against the reference.
__device__ __forceinline__ void row_total(const float* __restrict__ part_ml, int64_t first, int step, int used, int lane, float* weight,
                                          float& ref, float& sum) {
    ref = -INFINITY;
    for (int k = lane; k < used; k += 64) ref = fmaxf(ref, part_ml[(first + static_cast<int64_t>(k) * step) * 2]);
#pragma unroll
    for (int d = 32; d; d >>= 1) ref = fmaxf(ref, __shfl_xor(ref, d));
    sum = 0.0f;
    for (int k = lane; k < used; k += 64) {
        const float2 ml = *reinterpret_cast<const float2*>(part_ml + (first + static_cast<int64_t>(k) * step) * 2);
        const float f = ml.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ml.x - ref);
        if (weight) weight[k] = f;
        sum += f * ml.y;
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
}

// What is left when every workgroup has done its run.  The first `joins` workgroups, one per row of a (sequence, kv head), join the
// shares of rows that several workgroups have had a part of (and write the zeros of an empty sequence): a thread four channels and
// every (1024 / D)-th share.  The others, `blocks` of them per (sequence, kv head), make the weights of 1024 keys each from the logits
// that the rows have left: mass = mass_in + sum over rows of 2^(logit - reference) / sum.
// `weight` holds as many floats as the attention has workgroups.
// Latency bounds it: a launch, the row's place in the line, the shares' sums, the shares: 4 to 5 us (2.4 where no row is divided).  Weights
// of 24 contexts of up to 8000 tokens (13 MB of logits read, 6 MB of weights read and written) 10.6 us in all.  Nearly all workgroups of many
// sequences find nothing divided: 1024 contexts, 32 query heads, 41 us, 4096 contexts 149.
constexpr int kMaxPairRows = 1024;
constexpr int kEarly = 4;
template <int D>
__global__ __launch_bounds__(256) void attend_finish_kernel(PagesView v, AttendGeom g, int32_t joins, int32_t blocks,
                                                            const int32_t* __restrict__ row_start, const float* __restrict__ part_o,
                                                            const float* __restrict__ part_ml, const float* __restrict__ logits,
                                                            const float* mass_in, float* mass, _Float16* __restrict__ out,
                                                            const int32_t* __restrict__ note) {
    constexpr int kQuads = D / 4, kParts = 256 / kQuads;
    extern __shared__ float weight[];
    __shared__ float total;
    __shared__ f4_t o_lds[kParts][kQuads];
    __shared__ float refs[kMaxPairRows], invs[kMaxPairRows];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    const int id = static_cast<int>(blockIdx.x);
    if (id < joins) {
        const int pair = id / g.rows, j = id - pair * g.rows, s = pair / v.Hkv, h = pair - s * v.Hkv;
        const RowShares sh = row_shares(v, g, row_start, note, s, h, j);
        if (sh.used == 1 || j >= min(sh.w.count, g.max_rows) * g.per) return;
        const int64_t first = sh.first * g.tile_rows + j % 16;
        const int quad = threadIdx.x % kQuads, part = threadIdx.x / kQuads;
        if (wave == 0) {
            float ref, sum;
            row_total(part_ml, first, g.tile_rows, sh.used, lane, weight, ref, sum);
            if (lane == 0) total = sum;
        }
        __syncthreads();
        f4_t o = {0.0f, 0.0f, 0.0f, 0.0f};
        const f4_t* src = reinterpret_cast<const f4_t*>(part_o + first * D) + quad;
        const int64_t step = static_cast<int64_t>(g.tile_rows) * kQuads;
#pragma unroll 4
        for (int k = part; k < sh.used; k += kParts) o += src[k * step] * weight[k];
        o_lds[part][quad] = o;
        __syncthreads();
        if (part) return;
#pragma unroll
        for (int k = 1; k < kParts; ++k) o += o_lds[k][quad];
        const float inv = total > 0.0f ? 1.0f / total : 0.0f;
        h4_t x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = static_cast<_Float16>(o[e] * inv);
        reinterpret_cast<h4_t*>(out + (static_cast<int64_t>(sh.w.first + j / g.per) * v.Hq + h * g.per + j % g.per) * D)[quad] = x;
        return;
    }
    const int64_t pair = (id - joins) / blocks;
    const int s = static_cast<int>(pair / v.Hkv), h = static_cast<int>(pair % v.Hkv), t0 = (id - joins) % blocks * 1024;
    const RowShares sh = row_shares(v, g, row_start, note, s, h, 0);
    const int n = sh.w.n, count = min(sh.w.count, g.max_rows) * g.per;
    if (t0 >= n || count == 0) return;
    const int t = t0 + static_cast<int>(threadIdx.x) * 4;
    const int64_t at = pair * v.N + t;
    const float* x_at = logits + pair * g.rows * v.N + min(t, n - 1) / 4 * 4;
    // The weights so far and the first rows' logits are on their way while references and sums are worked out (8 contexts of up to 4096
    // tokens, 32 heads: 6.5 us, 7.4 without).  Past the last row it is read again; N and the logits' rows are multiples of 16.
    f4_t early[kEarly];
    float w[4];
#pragma unroll
    for (int e = 0; e < kEarly; ++e) early[e] = *reinterpret_cast<const f4_t*>(x_at + static_cast<int64_t>(min(e, count - 1)) * v.N);
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = mass_in && t + e < n ? mass_in[at + e] : 0.0f;
    for (int j = wave; j < count; j += 4) {
        const RowShares of = j < 16 ? sh : row_shares(v, g, row_start, note, s, h, j);
        float ref, sum;
        row_total(part_ml, of.first * g.tile_rows + j % 16, g.tile_rows, of.used, lane, nullptr, ref, sum);
        if (lane == 0) {
            refs[j] = sum > 0.0f ? ref : 0.0f;                   // (a row that sees nothing weighs nothing: its logits are -inf)
            invs[j] = sum > 0.0f ? 1.0f / sum : sum;             // (0 then; NaN if a logit is NaN or +inf)
        }
    }
    __syncthreads();
    if (t >= n) return;
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    auto add = [&](const f4_t& x, int j) {
        const float ref = refs[j], inv = invs[j];
        if (inv != inv) {                                        // a row that is NaN: so are its weights, of the tokens it sees
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] = x[e] == -INFINITY ? sum[e] : inv;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] = __builtin_fmaf(__builtin_amdgcn_exp2f(x[e] - ref), inv, sum[e]);
        }
    };
#pragma unroll
    for (int j = 0; j < kEarly; ++j)
        if (j < count) add(early[j], j);
#pragma unroll 4
    for (int j = kEarly; j < count; ++j) add(*reinterpret_cast<const f4_t*>(x_at + static_cast<int64_t>(j) * v.N), j);
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (t + e < n) mass[at + e] = w[e] + sum[e];
}

}  // namespace kvs
