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
constexpr int kCopies = 4;

// The sum of x over the lanes 0 .. count - 1 (of at most kSelectWaves), in every lane.
__device__ __forceinline__ int sum_of_first(int x, int count, int lane) {
    x = lane < count ? x : 0;
#pragma unroll
    for (int d = 1; d < kSelectWaves; d <<= 1) x += __shfl_xor(x, d);
    return __builtin_amdgcn_readfirstlane(x);
}

// One workgroup per pair = (layer, sequence, kv head).  A wavefront owns a contiguous range of slots and a lane every 64th of them; up to
// KEYS keys of a lane are read once and kept in registers (KEYS = 0: the range is longer, and every pass reads it again).  The key of
// the keep-th token is found digit by digit (11, 11 and 10 bits) from histograms in LDS; of the tokens that have exactly that key the
// lowest slots are kept, as many as there is room for.  Kept tokens above `keep` and evicted ones below come out in ascending order
// without a sort: ballots count within 64 slots, and one pass counts for the wavefronts behind.
// Instructions bound it, of 16 wavefronts on one CU for a pair: 4 sequences of 2049 slots, 8 kv heads, 4 layers 9.4 us; 2 of 4096, 32 kv
// heads, 8 layers (512 pairs, two rounds of workgroups) 16.8; 12 pairs of up to 32768 slots 32.  (The histograms' atomics are not what
// it waits for: 32 copies of the first digit's took as long, and so did fewer vector and more scalar instructions.)
template <int KEYS>
__global__ __launch_bounds__(kSelectThreads, KEYS >= 16 ? 4 : 8) void evict_select_kernel(PagesView v, EvictGeom g, const float* mass_in, const int32_t* pos_in,
                                                                      const int32_t* __restrict__ seen, int32_t* __restrict__ moves,
                                                                      int32_t* __restrict__ n_moves, float* mass, int32_t* pos) {
    constexpr int kKeys = KEYS ? KEYS : 1;
    // one histogram per digit, cleared together; the first digit, where most keys meet in few bins (sign, exponent and two bits),
    // has kCopies, so that fewer lanes of an LDS atomic hit one address
    __shared__ uint32_t hist[2048 * kCopies + 2048 + 1024];
    __shared__ uint32_t found[3][2];                              // digit, tokens still wanted within it
    __shared__ uint32_t wave_total[3][kSelectWaves];
    __shared__ int32_t wave_count[4][kSelectWaves];
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
    for (int i = tid; i < 2048 * kCopies + 2048 + 1024; i += kSelectThreads) hist[i] = 0;
    __syncthreads();
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        const int low = pass == 0 ? 21 : (pass == 1 ? 10 : 0), bins = pass == 2 ? 1024 : 2048, copies = pass == 0 ? kCopies : 1;
        uint32_t* h = hist + (pass == 0 ? 0 : 2048 * kCopies + (pass == 1 ? 0 : 2048));
        each([&](int, uint32_t k, bool here) {
            if (here && (pass == 0 || (k >> (low + (pass == 2 ? 10 : 11))) == prefix))
                atomicAdd(&h[((k >> low) & (bins - 1)) * copies + (lane & (copies - 1))], 1u);
        });
        __syncthreads();
        // from the highest bin down: thread t has the bins below bins - t * per
        constexpr int kMostPer = 2048 / kSelectThreads;
        const int per = bins / kSelectThreads;
        uint32_t own[kMostPer], mine = 0;
#pragma unroll
        for (int e = 0; e < kMostPer; ++e) {
            own[e] = 0;
            if (e < per)
                for (int c = 0; c < copies; ++c) own[e] += h[(bins - 1 - (tid * per + e)) * copies + c];
            mine += own[e];
        }
        uint32_t upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t x = __shfl_up(upto, d);
            upto += lane >= d ? x : 0;
        }
        if (lane == 63) wave_total[pass][wave] = upto;
        __syncthreads();
        upto += sum_of_first(wave_total[pass][lane & (kSelectWaves - 1)], wave, lane);
        const uint32_t before = upto - mine;
        if (before < want && want <= upto) {                      // exactly one thread: some n > keep tokens are counted
            uint32_t left = want - before, bin = bins - 1 - tid * per;
#pragma unroll
            for (int e = 0; e + 1 < kMostPer; ++e) {
                if (e + 1 < per && left > own[e]) {
                    left -= own[e];
                    --bin;
                }
            }
            found[pass][0] = bin;
            found[pass][1] = left;
        }
        __syncthreads();
        prefix = (prefix << (pass == 2 ? 10 : 11)) | found[pass][0];
        want = found[pass][1];
    }
    // Kept: keys above `prefix`, and the first `want` slots whose key it is.  A wavefront needs the number of such ties in front of it, and
    // of holes (evicted, below keep) and movers (kept, at or above it): all follow from four counts of every wavefront.
    int above[2] = {0, 0}, ties[2] = {0, 0};                       // [slots below keep, others]
    each([&](int i, uint32_t k, bool here) {
        const uint64_t gt = __ballot(here && k > prefix), eq = __ballot(here && k == prefix), low = __ballot(i < keep);
        above[0] += __builtin_popcountll(gt & low);
        above[1] += __builtin_popcountll(gt & ~low);
        ties[0] += __builtin_popcountll(eq & low);
        ties[1] += __builtin_popcountll(eq & ~low);
    });
    if (lane == 0) {
        wave_count[0][wave] = above[0];
        wave_count[1][wave] = above[1];
        wave_count[2][wave] = ties[0];
        wave_count[3][wave] = ties[1];
    }
    __syncthreads();
    int eq_before, hole_at, mover_at, all;
    {                                                              // lane k: the counts of wavefront k
        const int k = lane & (kSelectWaves - 1);
        const int eq_low = wave_count[2][k], eq_high = wave_count[3][k];
        int eq = eq_low + eq_high;                                 // up to wavefront k
#pragma unroll
        for (int d = 1; d < kSelectWaves; d <<= 1) {
            const int x = __shfl_up(eq, d);
            eq += k >= d ? x : 0;
        }
        const int left = max(static_cast<int>(want) - (eq - eq_low - eq_high), 0);
        const int first = min(k * steps * 64, n), slots_low = max(0, min(min(first + steps * 64, n), keep) - first);
        const int holes = slots_low - wave_count[0][k] - min(left, eq_low);
        const int movers = wave_count[1][k] + min(max(left - eq_low, 0), eq_high);
        eq_before = sum_of_first(eq_low + eq_high, wave, lane);
        hole_at = sum_of_first(holes, wave, lane);
        mover_at = sum_of_first(movers, wave, lane);
        all = sum_of_first(holes, kSelectWaves, lane);
    }
    const uint64_t below_lane = (1ull << lane) - 1;
    auto walk = [&](auto&& visit) {                                // visit(slot, whether there is one, kept)
        int seen_eq = eq_before;
        each([&](int i, uint32_t k, bool here) {
            const uint64_t eq = __ballot(here && k == prefix);
            const bool kept = here && (k > prefix || (k == prefix && seen_eq + __builtin_popcountll(eq & below_lane) < static_cast<int>(want)));
            seen_eq += __builtin_popcountll(eq);
            visit(i, here, kept);
        });
    };
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
// HBM bounds it in fp16 pages: 512 pairs of 1170 moves of 512 bytes, 32 kv heads of 128 (613 MB) take 130 us, 4.7 TB/s; rows of one
// head lie 256 bytes apart, K from V megabytes.  One move per pair takes 4 us: three dependent loads behind a launch.
// Rows of packed pages are moved one at a time, and the chain of their loads bounds it (wavefronts wait for three quarters of their time): the
// same moves take 275 us at 8 bits, 252 at 4, 237 at 2 (345, 192, 115 MB), 302 where pages of all three change a row's width.
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
