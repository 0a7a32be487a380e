// Attention of the newest tokens to one layer of their sequences' pages, as the pages are packed.
//
// A wavefront walks units of 32 tokens, two tiles of 16; a tile lies in one page (chunk_tokens is a multiple of 16), so its
// width and addresses are wave-uniform.  Both products run on 16x16x32 MFMAs in the transposed form,
//     S^T[token][row] = K Q^T,      O^T[dim][row] = V^T P^T,
// in which a lane keeps one query row (lane % 16) throughout: reference, sum and rescaling of a row need no exchange
// between lanes, and the four S^T values of a lane (tokens 4 * (lane / 16) + 0..3 of each tile) ARE the operand P^T of the second
// product, without a move.  The k index of an MFMA is free as long as both operands agree on it:
//   K: k runs over head dimensions in the order 64*.. + 16 * (lane / 16) + ..: a lane reads one contiguous piece per group, and
//      within eight dimensions the pairs (0,4) (1,5) (2,6) (3,7), which is how codes of 4 and 2 bits fall out of a word;
//   V: k runs over the unit's tokens, four per quarter wavefront and tile; a lane reads the rows of its tokens at its own D/16
//      contiguous dimensions, and one v_perm per register pairs two tokens.
// Codes are not dequantised for K: a half with the code in the top bits of its mantissa is 2^b + code exactly (1024 + code at 8
// bits, from a byte), the MFMA sums q * that per group, and scale and minimum enter once per (token, group):
//     S = sum_g s_g (acc_g - 2^b qsum_g) + mn_g qsum_g.
// V is dequantised by one v_fma_mix per element, fp16(code * s + mn).
#pragma once

#include "kv_pages_kernels.hpp"

namespace kvs {

typedef float f4_t __attribute__((ext_vector_type(4)));
typedef _Float16 h2_t __attribute__((ext_vector_type(2)));
typedef _Float16 h4_t __attribute__((ext_vector_type(4)));

constexpr int kAttendWaves = 4;
constexpr float kTop = 7.0f;         // a row's reference is set 2^7 below its largest logit so far ...
constexpr float kSlack = 15.0f;      // ... and moves when a logit passes 2^15 above it: probabilities stay in fp16's range, and those
                                     // 2^-31 below the largest still count

struct AttendGeom {
    int32_t layer, n_rows, max_rows;
    int32_t per;                     // query heads per kv head
    int32_t rows;                    // per * max_rows: query rows of a (sequence, kv head) pair
    int32_t row_tiles;               // ceil(rows / 16)
    int32_t splits;                  // shares a pair's tokens are divided among at most
    int32_t min_units;               // units of a share at least
    int64_t q_stride;
    float scale_log2e;               // log2(e) / sqrt(D)
};

// Shares of a sequence of n tokens: `units` units each, `used` of them.
struct Shares {
    int units, used;
};
__device__ __forceinline__ Shares shares_of(const AttendGeom& g, int n) {
    const int all = (n + 31) >> 5;
    Shares s;
    s.units = max((all + g.splits - 1) / g.splits, g.min_units);
    s.used = (all + s.units - 1) / s.units;
    return s;
}

__device__ __forceinline__ uint32_t perm(uint32_t hi, uint32_t lo, uint32_t sel) { return __builtin_amdgcn_perm(hi, lo, sel); }

// What a code of width W becomes by the bits below: kOffset + code.
template <int W> struct CodeOffset { static constexpr float value = W == 8 ? 1024.0f : (W == 4 ? 16.0f : 4.0f); };

// Shift by a signed constant.
template <int S> __device__ __forceinline__ uint32_t shift(uint32_t x) {
    if constexpr (S >= 0) return x << S;
    else return x >> -S;
}

// Eight dimensions of K, in the order (0,4) (1,5) (2,6) (3,7), from their 8 * W bits.
template <int W> __device__ __forceinline__ u4_t k_operand(const uint32_t* w) {
    u4_t r;
    if constexpr (W == 16) {
        r.x = perm(w[2], w[0], 0x05040100u);
        r.y = perm(w[2], w[0], 0x07060302u);
        r.z = perm(w[3], w[1], 0x05040100u);
        r.w = perm(w[3], w[1], 0x07060302u);
    } else if constexpr (W == 8) {
        r.x = perm(w[1], w[0], 0x0c040c00u) | 0x64006400u;
        r.y = perm(w[1], w[0], 0x0c050c01u) | 0x64006400u;
        r.z = perm(w[1], w[0], 0x0c060c02u) | 0x64006400u;
        r.w = perm(w[1], w[0], 0x0c070c03u) | 0x64006400u;
    } else if constexpr (W == 4) {
        r.x = (shift<6>(w[0]) & 0x03c003c0u) | 0x4c004c00u;
        r.y = (shift<2>(w[0]) & 0x03c003c0u) | 0x4c004c00u;
        r.z = (shift<-2>(w[0]) & 0x03c003c0u) | 0x4c004c00u;
        r.w = (shift<-6>(w[0]) & 0x03c003c0u) | 0x4c004c00u;
    } else {                                                // the bytes of dimensions 0-3 and 4-7, one in each half
        r.x = (shift<8>(w[0]) & 0x03000300u) | 0x44004400u;
        r.y = (shift<6>(w[0]) & 0x03000300u) | 0x44004400u;
        r.z = (shift<4>(w[0]) & 0x03000300u) | 0x44004400u;
        r.w = (shift<2>(w[0]) & 0x03000300u) | 0x44004400u;
    }
    return r;
}

__device__ __forceinline__ h8_t as_h8(u4_t v) { return __builtin_bit_cast(h8_t, v); }

// Codes of two tokens for one dimension, as halves 2^b + code, from the words that hold them (dimension d of the word).
template <int W, int d> __device__ __forceinline__ uint32_t v_codes(uint32_t a, uint32_t b) {
    if constexpr (W == 8) return perm(b, a, 0x0c040c00u + 0x00010001u * d) | 0x64006400u;
    else if constexpr (W == 4) {
        const uint32_t x = perm(b, a, d < 4 ? 0x05040100u : 0x07060302u);
        return (shift<6 - 4 * (d & 3)>(x) & 0x03c003c0u) | 0x4c004c00u;
    } else {
        const uint32_t x = perm(b, a, d < 8 ? 0x05040100u : 0x07060302u);
        return (shift<8 - 2 * (d & 7)>(x) & 0x03000300u) | 0x44004400u;
    }
}

// Loads n contiguous 32-bit words (n a power of two; less than one: BYTES bytes into the low end of one).
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

// A tile whose loads are issued: raw words of K and V, parameters of K for the lane's four tokens and every group, of V for its four
// tokens and the group of its dimensions.
template <int D, int G, int W> struct TileRegs {
    static constexpr int NG = D / G, DL = D / 16;
    static constexpr int kK = D * W / 128;                              // words of a lane's share of a K tile
    static constexpr int kV = DL * W / 32 > 0 ? DL * W / 32 : 1;        // words of one token's row at the lane's dimensions
    uint32_t k[kK];
    uint32_t v[4][kV];
    float ks[W == 16 ? 1 : 4 * NG], km[W == 16 ? 1 : 4 * NG];
    float vs[W == 16 ? 1 : 4], vm[W == 16 ? 1 : 4];
};

// Parameters of the tokens 4q .. 4q+3 of the tile: 4 * NG values that lie side by side.
template <int N> __device__ __forceinline__ void load_params(const uint8_t* p, int half_params, int first, float* out) {
    if (half_params) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const h4_t x = reinterpret_cast<const h4_t*>(reinterpret_cast<const _Float16*>(p) + first)[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) out[4 * i + j] = static_cast<float>(x[j]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const f4_t x = reinterpret_cast<const f4_t*>(reinterpret_cast<const float*>(p) + first)[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) out[4 * i + j] = x[j];
        }
    }
}

// Issues the loads of a tile: `record` its page's record, `in_page` its first token's row, `valid` how many of its 16 tokens there
// are (what lies behind them may be anything: V rows of missing tokens are replaced by the last one there is, their parameters by 0).
template <int D, int G, int W>
__device__ __forceinline__ void tile_load(TileRegs<D, G, W>& t, const uint8_t* __restrict__ record, const PagesView& v, int k_slab,
                                          int in_page, int valid, int lane) {
    constexpr int NG = D / G, DL = D / 16, kRowBytes = D * W / 8;
    const int l16 = lane & 15, q4 = lane >> 4;
    const SlabAt ka = slab_at<D>(v, W, k_slab), va = slab_at<D>(v, W, k_slab + v.Hkv);
    const uint8_t* kb = record + ka.codes + static_cast<uint32_t>(in_page) * kRowBytes;
    const uint8_t* vb = record + va.codes + static_cast<uint32_t>(in_page) * kRowBytes;
    constexpr int kPiece = G / 4 * W / 8;                               // bytes of a lane's piece per group
#pragma unroll
    for (int gi = 0; gi < NG; ++gi)
        load_words<kPiece>(kb + static_cast<uint32_t>(l16 * kRowBytes + gi * (G * W / 8) + q4 * kPiece), &t.k[gi * kPiece / 4]);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int row = min(4 * q4 + r, valid - 1);
        load_words<DL * W / 8>(vb + static_cast<uint32_t>(row * kRowBytes + l16 * (DL * W / 8)), t.v[r]);
    }
    if constexpr (W != 16) {
        const int first = (in_page + 4 * q4) * NG;
        load_params<4 * NG>(record + ka.scale, v.half_params, first, t.ks);
        load_params<4 * NG>(record + ka.mn, v.half_params, first, t.km);
        float s[4 * NG], m[4 * NG];
        load_params<4 * NG>(record + va.scale, v.half_params, first, s);
        load_params<4 * NG>(record + va.mn, v.half_params, first, m);
        const int mine = l16 * DL / G;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float a = s[r * NG], b = m[r * NG];
#pragma unroll
            for (int gi = 1; gi < NG; ++gi) {
                a = mine == gi ? s[r * NG + gi] : a;
                b = mine == gi ? m[r * NG + gi] : b;
            }
            if (valid < 16) {                                           // (uniform)
                const bool there = 4 * q4 + r < valid;
                a = there ? a : 0.0f;
                b = there ? b : 0.0f;
            }
            t.vs[r] = a;
            t.vm[r] = b - a * CodeOffset<W>::value;
        }
    }
}

// S^T of a tile, scaled to logits in units of log2.
template <int D, int G, int W>
__device__ __forceinline__ f4_t tile_logits(const TileRegs<D, G, W>& t, const u4_t* q, const float* qsum, float scale) {
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
                const uint32_t both = t.k[j / 2];
                const uint32_t one = perm(0u, both, (j & 1) ? 0x0c030c02u : 0x0c010c00u);
                a = k_operand<2>(&one);
            } else a = k_operand<W>(&t.k[j * (W / 4)]);
            acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_h8(a), as_h8(q[j]), acc, 0, 0, 0);
        }
        if constexpr (W == 16) s = acc;
        else {
            const float off = CodeOffset<W>::value * qsum[gi];
#pragma unroll
            for (int r = 0; r < 4; ++r)
                s[r] += __builtin_fmaf(t.ks[r * NG + gi], acc[r] - off, t.km[r * NG + gi] * qsum[gi]);
        }
    }
    return s * scale;
}

// V^T of one dimension for tokens (4q + 2j, 4q + 2j + 1) of a tile, as a pair of halves.
template <int D, int G, int W, int i>
__device__ __forceinline__ uint32_t v_pair(const TileRegs<D, G, W>& t, int j) {
    if constexpr (W == 16) return perm(t.v[2 * j + 1][i / 2], t.v[2 * j][i / 2], (i & 1) ? 0x07060302u : 0x05040100u);
    else {
        constexpr int kIn = 32 / W;                                     // dimensions of a word
        const uint32_t c = v_codes<W, i % kIn>(t.v[2 * j][i / kIn], t.v[2 * j + 1][i / kIn]);
        const h2_t h = __builtin_bit_cast(h2_t, c);
        h2_t x;
        x[0] = static_cast<_Float16>(__builtin_fmaf(static_cast<float>(h[0]), t.vs[2 * j], t.vm[2 * j]));
        x[1] = static_cast<_Float16>(__builtin_fmaf(static_cast<float>(h[1]), t.vs[2 * j + 1], t.vm[2 * j + 1]));
        return __builtin_bit_cast(uint32_t, x);
    }
}

template <int D, int G, int W, int NT, int i = 0>
__device__ __forceinline__ void tile_values(const TileRegs<D, G, W>* t, u4_t p, RowState<D>& st) {
    u4_t a;
    a.x = v_pair<D, G, W, i>(t[0], 0);
    a.y = v_pair<D, G, W, i>(t[0], 1);
    a.z = NT == 2 ? v_pair<D, G, W, i>(t[NT - 1], 0) : 0u;
    a.w = NT == 2 ? v_pair<D, G, W, i>(t[NT - 1], 1) : 0u;
    st.o[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_h8(a), as_h8(p), st.o[i], 0, 0, 0);
    if constexpr (i + 1 < D / 16) tile_values<D, G, W, NT, i + 1>(t, p, st);
}

// What a wavefront knows of its rows.
template <int D> struct RowsOfWave {
    u4_t q[D / 32];
    float qsum[D / 64 > 0 ? D / 64 : 1];       // of every group, the row's sum of q (as many groups as there are at most)
    int last;                                  // the last token the lane's row sees (-1: none)
    int all_see;                               // tokens up to this one are seen by every row
    float* logits;                             // where the row's logits go (NULL: nowhere)
};

// One or two tiles of one width.  first[]: the tiles' first tokens.
template <int D, int G, int W, int NT>
__device__ __forceinline__ void unit(const uint8_t* const* record, const int* in_page, const int* first, int n, const PagesView& v, int k_slab,
                                     float scale, const RowsOfWave<D>& rw, RowState<D>& st, int lane) {
    const int q4 = lane >> 4;
    TileRegs<D, G, W> t[NT];
#pragma unroll
    for (int k = 0; k < NT; ++k) tile_load<D, G, W>(t[k], record[k], v, k_slab, in_page[k], min(16, n - first[k]), lane);
    f4_t s[NT];
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < NT; ++k) {
        s[k] = tile_logits<D, G, W>(t[k], rw.q, rw.qsum, scale);
        if (first[k] + 15 > rw.all_see) {                                // (uniform)
#pragma unroll
            for (int r = 0; r < 4; ++r) s[k][r] = first[k] + 4 * q4 + r <= rw.last ? s[k][r] : -INFINITY;
        }
        if (rw.logits) *reinterpret_cast<f4_t*>(rw.logits + first[k] + 4 * q4) = s[k];
        top = fmaxf(fmaxf(fmaxf(s[k][0], s[k][1]), fmaxf(s[k][2], s[k][3])), top);
    }
    if (__ballot(top > st.ref + kSlack)) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        if (top > st.ref + kSlack) {
            const float to = top - kTop, f = __builtin_amdgcn_exp2f(st.ref - to);
            st.ref = to;
            st.sum *= f;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) st.o[i] *= f;
        }
    }
    const float ref = st.ref == -INFINITY ? 0.0f : st.ref;               // (a row that has seen nothing: every logit is -inf)
    h8_t p = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < NT; ++k)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float e = __builtin_amdgcn_exp2f(s[k][r] - ref);
            st.sum += e;
            p[4 * k + r] = static_cast<_Float16>(e);
        }
    tile_values<D, G, W, NT>(t, __builtin_bit_cast(u4_t, p), st);
}

template <int D, int G, int NT>
__device__ __forceinline__ void unit_of_width(int b, const uint8_t* const* record, const int* in_page, const int* first, int n, const PagesView& v,
                                              int k_slab, float scale, const RowsOfWave<D>& rw, RowState<D>& st, int lane) {
    if (b == 16) unit<D, G, 16, NT>(record, in_page, first, n, v, k_slab, scale, rw, st, lane);
    else if (b == 8) unit<D, G, 8, NT>(record, in_page, first, n, v, k_slab, scale, rw, st, lane);
    else if (b == 4) unit<D, G, 4, NT>(record, in_page, first, n, v, k_slab, scale, rw, st, lane);
    else unit<D, G, 2, NT>(record, in_page, first, n, v, k_slab, scale, rw, st, lane);
}

// One share of a (sequence, kv head, row tile): grid splits * row_tiles * kv heads * sequences, the shares of a pair side by side.
// The wavefronts of a workgroup take the share's units in turn, each with a state of its own; the four states meet in LDS.
template <int D, int G>
__global__ __launch_bounds__(64 * kAttendWaves, 2) void attend_kernel(PagesView v, AttendGeom g, const _Float16* __restrict__ q,
                                                                   const int32_t* __restrict__ row_start, _Float16* __restrict__ out,
                                                                   float* __restrict__ part_o, float* __restrict__ part_ml,
                                                                   float* __restrict__ logits) {
    constexpr int DL = D / 16, NG = D / G;
    __shared__ float o_lds[kAttendWaves][16][D];
    __shared__ float ml_lds[kAttendWaves][2][16];
    const int lane = threadIdx.x & 63, l16 = lane & 15, q4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    uint32_t id = blockIdx.x;
    const int share = static_cast<int>(id % g.splits);
    id /= g.splits;
    const int rt = static_cast<int>(id % g.row_tiles);
    id /= g.row_tiles;
    const int h = static_cast<int>(id % v.Hkv), s = static_cast<int>(id / v.Hkv);
    const SeqRows rows = seq_rows(row_start, s, g.n_rows);
    const int n = seq_len(v, s), count = min(rows.count, g.max_rows);
    const Shares sh = shares_of(g, n);
    if (share >= max(sh.used, 1) || rt * 16 >= count * g.per) return;    // (an empty sequence: its first share writes zeros)

    // this lane's query row
    const int j = rt * 16 + l16, nth = j / g.per, head = h * g.per + j % g.per;
    const bool ok = j < count * g.per;
    RowsOfWave<D> rw;
    rw.last = ok ? n - rows.count + nth : -1;
    rw.all_see = n - rows.count + rt * 16 / g.per;
    const int64_t pair = static_cast<int64_t>(s) * v.Hkv + h;
    rw.logits = logits && ok ? logits + (pair * g.rows + j) * v.N : nullptr;
    {
        const _Float16* qp = q + static_cast<int64_t>(rows.first + (ok ? nth : 0)) * g.q_stride + head * (ok ? 1 : 0) * D;
#pragma unroll
        for (int gi = 0; gi < NG; ++gi) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < G / 32; ++i) {
                u4_t w = {0u, 0u, 0u, 0u};
                if (ok) w = *reinterpret_cast<const u4_t*>(qp + gi * G + q4 * (G / 4) + i * 8);
                const h8_t x = as_h8(w);
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += static_cast<float>(x[e]);
                const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
                rw.q[gi * (G / 32) + i] = k_operand<16>(ws);
            }
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            rw.qsum[gi] = sum;
        }
    }
    RowState<D> st;
#pragma unroll
    for (int i = 0; i < DL; ++i) st.o[i] = f4_t{0.0f, 0.0f, 0.0f, 0.0f};
    st.ref = -INFINITY;
    st.sum = 0.0f;

    const int k_slab = (g.layer * 2) * v.Hkv + h;
    const int u_end = min((n + 31) >> 5, (share + 1) * sh.units);          // (none for an empty sequence)
    const uint64_t* offs = v.off + static_cast<int64_t>(s) * v.stride;
    const uint8_t* bits = v.bits + static_cast<int64_t>(s) * v.stride;
    const int tiles_per_page = v.T >> 4;
    // the pages of the wavefront's next 32 units, a tile per lane: offset, and width (0: absent or behind the end)
    uint32_t off_lo = 0, off_hi = 0, width = 0;
    auto look_up = [&](int u) {
        const int tile = min(2 * (u + kAttendWaves * (lane >> 1)) + (lane & 1), (n - 1) >> 4);
        const int page = v.page_of_tile ? static_cast<int>(__umulhi(static_cast<uint32_t>(tile), v.page_of_tile)) : tile;
        const uint64_t off = offs[page];
        const uint32_t b = bits[page];
        off_lo = static_cast<uint32_t>(off);
        off_hi = static_cast<uint32_t>(off >> 32);
        width = page_present(v, off, b) ? b : 0u;
    };
    int ahead = 0;                                    // units looked up and not yet walked
    for (int u = share * sh.units + wave; u < u_end; u += kAttendWaves) {
        if (ahead == 0) {
            look_up(u);
            ahead = 32;
        }
        const uint8_t* record[2];
        int in_page[2], first[2], b[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int at = 2 * (32 - ahead) + k, tile = 2 * u + k;
            const uint64_t off = static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(off_hi), at))) << 32 |
                                 static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(off_lo), at));
            const int page = v.page_of_tile ? static_cast<int>(__umulhi(static_cast<uint32_t>(tile), v.page_of_tile)) : tile;
            first[k] = tile * 16;
            b[k] = first[k] < n ? __builtin_amdgcn_readlane(static_cast<int>(width), at) : 0;
            record[k] = v.pool + off;
            in_page[k] = (tile - page * tiles_per_page) * 16;
        }
        --ahead;
        if (b[0] == b[1]) {
            if (b[0]) unit_of_width<D, G, 2>(b[0], record, in_page, first, n, v, k_slab, g.scale_log2e, rw, st, lane);
        } else {
            if (b[0]) unit_of_width<D, G, 1>(b[0], record, in_page, first, n, v, k_slab, g.scale_log2e, rw, st, lane);
            if (b[1]) unit_of_width<D, G, 1>(b[1], record + 1, in_page + 1, first + 1, n, v, k_slab, g.scale_log2e, rw, st, lane);
        }
        if (rw.logits) {                             // what an absent tile would have had
#pragma unroll
            for (int k = 0; k < 2; ++k)
                if (!b[k] && first[k] < n) *reinterpret_cast<f4_t*>(rw.logits + first[k] + 4 * q4) = f4_t{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        }
    }
    // the four states against one reference per row
    st.sum += __shfl_xor(st.sum, 16);
    st.sum += __shfl_xor(st.sum, 32);
    if (q4 == 0) {
        ml_lds[wave][0][l16] = st.ref;
        ml_lds[wave][1][l16] = st.sum;
    }
    if (ok) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < DL; i += 4)
                *reinterpret_cast<f4_t*>(&o_lds[wave][l16][DL * (4 * q4 + r) + i]) = f4_t{st.o[i][r], st.o[i + 1][r], st.o[i + 2][r], st.o[i + 3][r]};
    }
    __syncthreads();
    const int here = min(16, count * g.per - rt * 16);                   // rows of this tile
    for (int i = threadIdx.x; i < here * (D / 4); i += 64 * kAttendWaves) {
        const int row = i / (D / 4), d = i % (D / 4) * 4;
        float ref = -INFINITY, sum = 0.0f;
#pragma unroll
        for (int k = 0; k < kAttendWaves; ++k) ref = fmaxf(ref, ml_lds[k][0][row]);
        f4_t o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < kAttendWaves; ++k) {
            const float m = ml_lds[k][0][row], f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - ref);
            sum += f * ml_lds[k][1][row];
            o += *reinterpret_cast<const f4_t*>(&o_lds[k][row][d]) * f;
        }
        const int jr = rt * 16 + row;
        if (part_ml && d == 0) {
            float* ml = part_ml + ((pair * g.splits + share) * g.rows + jr) * 2;
            ml[0] = ref;
            ml[1] = sum;
        }
        if (sh.used <= 1) {
            const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;            // a row that sees nothing: zeros
            h4_t x;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = static_cast<_Float16>(o[e] * inv);
            const int64_t at = (static_cast<int64_t>(rows.first + jr / g.per) * v.Hq + h * g.per + jr % g.per) * D + d;
            *reinterpret_cast<h4_t*>(out + at) = x;
        } else {
            *reinterpret_cast<f4_t*>(part_o + ((pair * g.splits + share) * g.rows + jr) * D + d) = o;
        }
    }
}

// Reference and sum of a row over its shares, taken in ascending order.
__device__ __forceinline__ void row_total(const float* __restrict__ part_ml, int64_t first, int used, int rows, float& ref, float& sum) {
    ref = -INFINITY;
    sum = 0.0f;
    for (int k = 0; k < used; ++k) ref = fmaxf(ref, part_ml[(first + static_cast<int64_t>(k) * rows) * 2]);
    for (int k = 0; k < used; ++k) {
        const float2 ml = *reinterpret_cast<const float2*>(part_ml + (first + static_cast<int64_t>(k) * rows) * 2);
        sum += ml.x == -INFINITY ? 0.0f : ml.y * __builtin_amdgcn_exp2f(ml.x - ref);
    }
}

// Joins the shares of the pairs whose tokens were divided: one thread per four channels of a row.
template <int D>
__global__ __launch_bounds__(256) void attend_join_kernel(PagesView v, AttendGeom g, const int32_t* __restrict__ row_start,
                                                          const float* __restrict__ part_o, const float* __restrict__ part_ml,
                                                          _Float16* __restrict__ out) {
    constexpr int kQuads = D / 4;
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int d = static_cast<int>(i % kQuads) * 4;
    const int64_t row = i / kQuads;
    const int64_t pair = row / g.rows;
    const int j = static_cast<int>(row - pair * g.rows);
    const int s = static_cast<int>(pair / v.Hkv), h = static_cast<int>(pair - static_cast<int64_t>(s) * v.Hkv);
    if (s >= v.n_seqs) return;
    const SeqRows rows = seq_rows(row_start, s, g.n_rows);
    const int n = seq_len(v, s), count = min(rows.count, g.max_rows);
    const Shares sh = shares_of(g, n);
    if (sh.used <= 1 || j >= count * g.per) return;
    const int64_t first = pair * g.splits * g.rows + j;
    float ref, sum;
    row_total(part_ml, first, sh.used, g.rows, ref, sum);
    f4_t o = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int k = 0; k < sh.used; ++k) {
        const int64_t at = first + static_cast<int64_t>(k) * g.rows;
        const float m = part_ml[at * 2], f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - ref);
        o += *reinterpret_cast<const f4_t*>(part_o + at * D + d) * f;
    }
    const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
    h4_t x;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = static_cast<_Float16>(o[e] * inv);
    *reinterpret_cast<h4_t*>(out + (static_cast<int64_t>(rows.first + j / g.per) * v.Hq + h * g.per + j % g.per) * D + d) = x;
}

// The weights of a pair's keys, from the logits its rows left: mass = mass_in + sum over rows of 2^(logit - reference) / sum.
// One workgroup per pair and 1024 tokens (`blocks` of them per pair).
constexpr int kMaxPairRows = 1024;
__global__ __launch_bounds__(256) void attend_mass_kernel(PagesView v, AttendGeom g, int32_t blocks, const int32_t* __restrict__ row_start,
                                                          const float* __restrict__ part_ml, const float* __restrict__ logits,
                                                          const float* mass_in, float* mass) {
    __shared__ float refs[kMaxPairRows], invs[kMaxPairRows];
    const int64_t pair = blockIdx.x / blocks;
    const int s = static_cast<int>(pair / v.Hkv), t0 = static_cast<int>(blockIdx.x % blocks) * 1024;
    const int n = seq_len(v, s);
    if (t0 >= n) return;
    const SeqRows rows = seq_rows(row_start, s, g.n_rows);
    const int count = min(rows.count, g.max_rows) * g.per;
    if (count == 0) return;
    const Shares sh = shares_of(g, n);
    for (int j = threadIdx.x; j < count; j += 256) {
        float ref, sum;
        row_total(part_ml, pair * g.splits * g.rows + j, sh.used, g.rows, ref, sum);
        refs[j] = sum > 0.0f ? ref : 0.0f;                       // (a row that sees nothing weighs nothing: its logits are -inf)
        invs[j] = sum > 0.0f ? 1.0f / sum : 0.0f;
    }
    __syncthreads();
    const int t = t0 + static_cast<int>(threadIdx.x) * 4;
    if (t >= n) return;
    f4_t w = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int j = 0; j < count; ++j) {
        const f4_t x = *reinterpret_cast<const f4_t*>(logits + (pair * g.rows + j) * v.N + t);
        const float ref = refs[j], inv = invs[j];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = __builtin_fmaf(__builtin_amdgcn_exp2f(x[e] - ref), inv, w[e]);
    }
    const int64_t at = pair * v.N + t;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (t + e < n) mass[at + e] = (mass_in ? mass_in[at + e] : 0.0f) + w[e];
}

}  // namespace kvs
