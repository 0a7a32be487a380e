// Eviction by accumulated attention weight: which tokens a kv head keeps, and the rows that have to move for it.
#pragma once

#include "kv_pages_kernels.hpp"

namespace kvs {

struct EvictGeom {
    int32_t layer0, n_layers;
    int32_t keep, sink, recent;
    int32_t list;                    // entries of a pair's move list: min(keep, n_tokens - keep)
};

// What tokens are ranked by, as an unsigned number: the order of binary32 values (-0 equal to +0), NaN below everything,
// protected tokens above it.
__device__ __forceinline__ uint32_t evict_key(float mass, int pos, int sink, int from) {
    if (pos < sink || pos >= from) return 0xffffffffu;
    if (mass != mass) return 0u;
    const uint32_t u = __builtin_bit_cast(uint32_t, plus_zero(mass));
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

constexpr int kSelectThreads = 1024;
constexpr int kSelectWaves = kSelectThreads / 64;

// One workgroup per pair = (layer, sequence, kv head).  A wavefront owns a contiguous range of slots and a lane every 64th of them; up to
// KEYS keys of a lane are read once and kept in registers (KEYS = 0: the range is longer, and every pass reads it again).  The key of
// the keep-th token is found digit by digit (11, 11 and 10 bits) from histograms in LDS; of the tokens that have exactly that key the
// lowest slots are kept, as many as there is room for.  Kept tokens above `keep` and evicted ones below come out in ascending order
// without a sort: ballots count within 64 slots, and one pass counts for the wavefronts behind.
// Latency bounds it: a workgroup reads a few hundred KB at most.
template <int KEYS>
__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(PagesView v, EvictGeom g, const float* mass_in, const int32_t* pos_in,
                                                                      const int32_t* __restrict__ seen, int32_t* __restrict__ moves,
                                                                      int32_t* __restrict__ n_moves, float* mass, int32_t* pos) {
    constexpr int kKeys = KEYS ? KEYS : 1;
    __shared__ uint32_t hist[2048];
    __shared__ uint32_t found[2];                                 // digit, tokens still wanted within it
    __shared__ uint32_t wave_total[kSelectWaves];
    __shared__ int32_t wave_eq[kSelectWaves], wave_hole[kSelectWaves], wave_mover[kSelectWaves];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t pair = blockIdx.x;
    const int s = static_cast<int>(pair / v.Hkv % v.n_seqs);
    const int n = seq_len(v, s), keep = g.keep;
    mass_in += pair * v.N;
    pos_in += pair * v.N;
    mass += pair * v.N;
    pos += pair * v.N;
    if (n <= keep) {                                              // everything stays
        if (tid == 0) n_moves[pair] = 0;
        for (int i = tid; i < n; i += kSelectThreads) {
            if (mass != mass_in) mass[i] = mass_in[i];
            if (pos != pos_in) pos[i] = pos_in[i];
        }
        return;
    }
    const int from = (seen ? seen[s] : n) - g.recent;
    const int steps = (n + kSelectThreads - 1) / kSelectThreads;                 // of 64 slots, of a wavefront's range
    const int begin = wave * steps * 64 + lane;                                  // the lane's first slot
    auto key_at = [&](int i) { return i < n ? evict_key(mass_in[i], pos_in[i], g.sink, from) : 0u; };
    // (a lane's slots behind n have the lowest key, and `here` keeps them out of every count)
    uint32_t keys[kKeys];
    if constexpr (KEYS > 0) {
        float m[kKeys];
        int p[kKeys];
#pragma unroll
        for (int i = 0; i < KEYS; ++i) {
            const int at = min(begin + i * 64, n - 1);
            m[i] = mass_in[at];
            p[i] = pos_in[at];
        }
#pragma unroll
        for (int i = 0; i < KEYS; ++i) keys[i] = evict_key(m[i], p[i], g.sink, from);
    }
    // visits the lane's slots: f(slot, key, whether there is one); every lane of the wavefront together
    auto each = [&](auto&& f) {
        if constexpr (KEYS > 0) {
#pragma unroll
            for (int i = 0; i < KEYS; ++i) {
                const int at = begin + i * 64;
                if (i < steps) f(at, keys[i], at < n);
            }
        } else {
            for (int i = 0; i < steps; ++i) {
                const int at = begin + i * 64;
                f(at, key_at(at), at < n);
            }
        }
    };
    uint32_t prefix = 0, want = static_cast<uint32_t>(keep);      // the want-th largest of the keys that begin with prefix
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        const int low = pass == 0 ? 21 : (pass == 1 ? 10 : 0), bins = pass == 2 ? 1024 : 2048;
        for (int i = tid; i < bins; i += kSelectThreads) hist[i] = 0;
        __syncthreads();
        each([&](int, uint32_t k, bool here) {
            if (here && (pass == 0 || (k >> (low + (pass == 2 ? 10 : 11))) == prefix)) atomicAdd(&hist[(k >> low) & (bins - 1)], 1u);
        });
        __syncthreads();
        // from the highest bin down: thread t has the bins below bins - t * per
        const int per = bins / kSelectThreads;
        uint32_t mine = 0;
        for (int e = 0; e < per; ++e) mine += hist[bins - 1 - (tid * per + e)];
        uint32_t upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t x = __shfl_up(upto, d);
            upto += lane >= d ? x : 0;
        }
        if (lane == 63) wave_total[wave] = upto;
        __syncthreads();
        for (int k = 0; k < wave; ++k) upto += wave_total[k];
        const uint32_t before = upto - mine;
        if (before < want && want <= upto) {                      // exactly one thread: some n > keep tokens are counted
            uint32_t left = want - before;
            for (int e = 0; e < per; ++e) {
                const int bin = bins - 1 - (tid * per + e);
                if (left <= hist[bin]) {
                    found[0] = static_cast<uint32_t>(bin);
                    found[1] = left;
                    break;
                }
                left -= hist[bin];
            }
        }
        __syncthreads();
        prefix = (prefix << (pass == 2 ? 10 : 11)) | found[0];
        want = found[1];
        __syncthreads();
    }
    // kept: keys above `prefix`, and the first `want` slots whose key it is.  A wavefront needs the number of such ties in front of it,
    // then of holes (evicted, below keep) and movers (kept, at or above it).
    int eq = 0;
    each([&](int, uint32_t k, bool here) { eq += __builtin_popcountll(__ballot(here && k == prefix)); });
    if (lane == 0) wave_eq[wave] = eq;
    __syncthreads();
    int eq_before = 0;
    for (int k = 0; k < wave; ++k) eq_before += wave_eq[k];
    const uint64_t below_lane = (1ull << lane) - 1;
    auto walk = [&](auto&& visit) {                                // visit(slot, whether there is one, kept)
        int seen_eq = eq_before;
        each([&](int i, uint32_t k, bool here) {
            const uint64_t ties = __ballot(here && k == prefix);
            const bool kept = here && (k > prefix || (k == prefix && seen_eq + __builtin_popcountll(ties & below_lane) < static_cast<int>(want)));
            seen_eq += __builtin_popcountll(ties);
            visit(i, here, kept);
        });
    };
    int holes = 0, movers = 0;
    walk([&](int i, bool here, bool kept) {
        holes += __builtin_popcountll(__ballot(here && !kept && i < keep));
        movers += __builtin_popcountll(__ballot(kept && i >= keep));
    });
    if (lane == 0) {
        wave_hole[wave] = holes;
        wave_mover[wave] = movers;
    }
    __syncthreads();
    int hole_at = 0, mover_at = 0, all = 0;
    for (int k = 0; k < kSelectWaves; ++k) {
        hole_at += k < wave ? wave_hole[k] : 0;
        mover_at += k < wave ? wave_mover[k] : 0;
        all += wave_hole[k];
    }
    if (tid == 0) n_moves[pair] = all;
    int32_t* to = moves + pair * 2 * g.list;
    int32_t* from_slot = to + g.list;
    walk([&](int i, bool here, bool kept) {
        const bool hole = here && !kept && i < keep, mover = kept && i >= keep;
        const uint64_t hb = __ballot(hole), mb = __ballot(mover);
        if (hole) to[hole_at + __builtin_popcountll(hb & below_lane)] = i;
        if (mover) from_slot[mover_at + __builtin_popcountll(mb & below_lane)] = i;
        hole_at += __builtin_popcountll(hb);
        mover_at += __builtin_popcountll(mb);
        if (kept && i < keep) {
            if (mass != mass_in) mass[i] = mass_in[i];
            if (pos != pos_in) pos[i] = pos_in[i];
        }
    });
}

// Eight elements of a row as they lie in a page: codes and the parameters of their group.
struct Piece {
    u4_t values;                     // fp16, or up to eight bytes of codes
    float scale, mn;
};

__device__ __forceinline__ float param_at(const uint8_t* p, int half_params, uint64_t i) {
    return half_params ? static_cast<float>(reinterpret_cast<const _Float16*>(p)[i]) : reinterpret_cast<const float*>(p)[i];
}

template <int D>
__device__ __forceinline__ Piece piece_load(const PagesView& v, const uint8_t* record, int b, int slab, int piece, int lpg_log2) {
    const SlabAt a = slab_at<D>(v, b, slab);
    const uint8_t* codes = record + a.codes;
    Piece x;
    x.values = u4_t{0u, 0u, 0u, 0u};
    x.scale = x.mn = 0.0f;
    if (b == 16) {
        x.values = reinterpret_cast<const u4_t*>(codes)[piece];
        return x;
    }
    if (b == 8) {
        const u2_t w = reinterpret_cast<const u2_t*>(codes)[piece];
        x.values.x = w.x;
        x.values.y = w.y;
    } else if (b == 4) x.values.x = reinterpret_cast<const uint32_t*>(codes)[piece];
    else x.values.x = reinterpret_cast<const uint16_t*>(codes)[piece];
    x.scale = param_at(record + a.scale, v.half_params, piece >> lpg_log2);
    x.mn = param_at(record + a.mn, v.half_params, piece >> lpg_log2);
    return x;
}

template <int D>
__device__ __forceinline__ void piece_store(const PagesView& v, uint8_t* record, int b, int from_b, int slab, int piece, int lpg_log2, int lane,
                                            const Piece& x) {
    const SlabAt a = slab_at<D>(v, b, slab);
    uint8_t* codes = record + a.codes;
    u4_t values = x.values;
    if (b == from_b) {                                            // the bytes as they are
        if (b == 16) reinterpret_cast<u4_t*>(codes)[piece] = values;
        else {
            if (b == 8) reinterpret_cast<u2_t*>(codes)[piece] = u2_t{values.x, values.y};
            else if (b == 4) reinterpret_cast<uint32_t*>(codes)[piece] = values.x;
            else reinterpret_cast<uint16_t*>(codes)[piece] = static_cast<uint16_t>(values.x);
            if ((piece & ((1 << lpg_log2) - 1)) == 0) {
                const int i = piece >> lpg_log2;
                if (v.half_params) {
                    reinterpret_cast<_Float16*>(record + a.scale)[i] = static_cast<_Float16>(x.scale);
                    reinterpret_cast<_Float16*>(record + a.mn)[i] = static_cast<_Float16>(x.mn);
                } else {
                    reinterpret_cast<float*>(record + a.scale)[i] = x.scale;
                    reinterpret_cast<float*>(record + a.mn)[i] = x.mn;
                }
            }
        }
        return;
    }
    if (from_b != 16) {
        const u2_t w = {values.x, values.y};
        if (from_b == 8) values = dequantise_piece<8>(w, x.scale, x.mn);
        else if (from_b == 4) values = dequantise_piece<4>(w, x.scale, x.mn);
        else values = dequantise_piece<2>(w, x.scale, x.mn);
    }
    if (b == 16) {
        reinterpret_cast<u4_t*>(codes)[piece] = values;
        return;
    }
    if (v.half_params) {
        if (b == 8) compress_piece<8, true>(values, codes, record + a.scale, record + a.mn, piece, lpg_log2, lane);
        else if (b == 4) compress_piece<4, true>(values, codes, record + a.scale, record + a.mn, piece, lpg_log2, lane);
        else compress_piece<2, true>(values, codes, record + a.scale, record + a.mn, piece, lpg_log2, lane);
    } else {
        if (b == 8) compress_piece<8, false>(values, codes, record + a.scale, record + a.mn, piece, lpg_log2, lane);
        else if (b == 4) compress_piece<4, false>(values, codes, record + a.scale, record + a.mn, piece, lpg_log2, lane);
        else compress_piece<2, false>(values, codes, record + a.scale, record + a.mn, piece, lpg_log2, lane);
    }
}

// The moves of a pair's list, `blocks` workgroups per pair: D/8 neighbouring lanes carry kAtOnce rows, their K and their V, with their
// weight and position.  Rows come from slots at or above `keep` and go to slots below it, so no move reads what another has written.
// A row's way is list entry - page entry - row - store: the four steps of the kAtOnce rows are taken together.
constexpr int kAtOnce = 4;
template <int D>
__global__ __launch_bounds__(256) void evict_move_kernel(PagesView v, EvictGeom g, int32_t blocks, int32_t lpg_log2,
                                                         const int32_t* __restrict__ moves, const int32_t* __restrict__ n_moves,
                                                         const float* mass_in, const int32_t* pos_in, float* mass, int32_t* pos) {
    constexpr int kRow = D / 8, kRows = 256 / kRow;
    const int lane = threadIdx.x & 63;
    const int64_t pair = blockIdx.x / blocks;
    const int block = static_cast<int>(blockIdx.x % blocks);
    const int layer = g.layer0 + static_cast<int>(pair / v.Hkv / v.n_seqs), s = static_cast<int>(pair / v.Hkv % v.n_seqs);
    const int h = static_cast<int>(pair % v.Hkv);
    const int count = n_moves[pair], in_row = threadIdx.x % kRow, row = threadIdx.x / kRow;
    const int32_t* to_list = moves + pair * 2 * g.list;
    const int32_t* from_list = to_list + g.list;
    const uint64_t* offs = v.off + static_cast<int64_t>(s) * v.stride;
    const uint8_t* bits = v.bits + static_cast<int64_t>(s) * v.stride;
    const int k_slab = layer * 2 * v.Hkv + h;
    for (int i0 = block * kRows * kAtOnce; i0 < count; i0 += blocks * kRows * kAtOnce) {
        int to[kAtOnce], from[kAtOnce], to_b[kAtOnce], from_b[kAtOnce];
        uint64_t to_off[kAtOnce], from_off[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {                       // (behind the list: the last move again, not stored)
            const int i = min(i0 + k * kRows + row, count - 1);
            to[k] = to_list[i];
            from[k] = from_list[i];
        }
        float m[kAtOnce];
        int p[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int a = to[k] / v.T, b = from[k] / v.T;
            to_off[k] = offs[a];
            from_off[k] = offs[b];
            to_b[k] = bits[a];
            from_b[k] = bits[b];
            m[k] = mass_in[pair * v.N + from[k]];
            p[k] = pos_in[pair * v.N + from[k]];
        }
        bool fp16 = true;                                         // every row between fp16 pages: the common case, without branches
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
            fp16 = fp16 && to_b[k] == 16 && from_b[k] == 16 && page_present(v, to_off[k], 16) && page_present(v, from_off[k], 16);
        if (__all(fp16)) {
            u4_t x[kAtOnce], y[kAtOnce];
            const int64_t slab = static_cast<int64_t>(k_slab) * v.T * kRow, v_step = static_cast<int64_t>(v.Hkv) * v.T * kRow;
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const u4_t* src = reinterpret_cast<const u4_t*>(v.pool + from_off[k]) + slab + from[k] % v.T * kRow + in_row;
                x[k] = stream_load<true>(src);
                y[k] = stream_load<true>(src + v_step);
            }
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                u4_t* dst = reinterpret_cast<u4_t*>(v.pool + to_off[k]) + slab + to[k] % v.T * kRow + in_row;
                if (i0 + k * kRows + row < count) {
                    stream_store<true>(x[k], dst);
                    stream_store<true>(y[k], dst + v_step);
                }
            }
        } else {
#pragma unroll 1
            for (int i = i0 + row; i < min(i0 + kRows * kAtOnce, count); i += kRows) {
                const int a = to_list[i], b = from_list[i];
                const uint64_t a_off = offs[a / v.T], b_off = offs[b / v.T];
                const int a_bits = bits[a / v.T], b_bits = bits[b / v.T];
                if (!page_present(v, a_off, a_bits) || !page_present(v, b_off, b_bits)) continue;
                const int a_piece = a % v.T * kRow + in_row, b_piece = b % v.T * kRow + in_row;
#pragma unroll 1
                for (int slab = k_slab; slab <= k_slab + v.Hkv; slab += v.Hkv)                 // K, then V
                    piece_store<D>(v, v.pool + a_off, a_bits, b_bits, slab, a_piece, lpg_log2, lane,
                                   piece_load<D>(v, v.pool + b_off, b_bits, slab, b_piece, lpg_log2));
            }
        }
        if (in_row == 0) {
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k)
                if (i0 + k * kRows + row < count) {
                    mass[pair * v.N + to[k]] = m[k];
                    pos[pair * v.N + to[k]] = p[k];
                }
        }
    }
}

}  // namespace kvs
