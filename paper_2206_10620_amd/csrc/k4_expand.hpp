// The adapters' part of a block product in binary16 (include/pp_adapter.h): c_s B_s u added to the accumulators of a wavefront
// before the product's own sum, so that it meets the sum, the bias and the activation in fp32.
//
// u is in fp32 and far smaller than x.  A lane of the matrix instruction's second operand holds eight consecutive ranks of one token,
// which is how u lies in memory: no staging.  They enter as two binary16 parts, hi and lo, after a power of two that brings the
// token's largest |u| of 16 ranks to [2^14, 2^15) is taken out: 20 bits, whatever the size of u, where y keeps 11.  B lies in operand
// order, 1 KB per 32 rows and 16 ranks.
// What it costs is reading u, once for every 64 rows of y: 4096 x 1024 at 0.17 on 2048 tokens takes 18 us without adapters, 4, 7, 13 and
// 24 more with rank 16, 32, 64 and 128 (two shares of u, 8 bytes a token and rank, are four times a row of x).
//
// The tokens of a wavefront are taken slot by slot.  A matrix instruction computes all its columns with the one slot's B;
// only the columns of that slot's tokens are taken over, so nothing a slot holds can reach another slot's tokens.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "adapter_rules.hpp"

namespace ppc {

// What a token has: the projection leaves it for whoever reads u, which saves them a load that waits for another.
struct KxToken {
    int32_t slot;               // -1: no adapter
    int32_t rank;               // 0 for none
    float factor;
    int32_t unused;
};

struct K4Expand {
    const KxToken* tokens;      // [n]
    const float* u;             // [splits][kx_share], kx_at
    const void* operands;       // [slot][64-row tile][rank_pad / 16][2][64 lanes][8] binary16
    int64_t slot_bytes, split_elems;
    int32_t splits, rank_pad;
};

typedef _Float16 kx_h8 __attribute__((ext_vector_type(8)));
typedef float kx_f4 __attribute__((ext_vector_type(4)));
typedef float kx_f16 __attribute__((ext_vector_type(16)));

// v = hi + lo up to 2^-22 of v (or 2^-25 absolute); an infinity or a NaN is hi alone
__device__ __forceinline__ void kx_parts(float v, _Float16& hi, _Float16& lo) {
    hi = (_Float16)v;
    const float rest = v - (float)hi;
    lo = __builtin_fabsf(v) <= 65504.0f ? (_Float16)rest : (_Float16)0.0f;
}

// The power of two that brings the largest finite magnitude (its bits) of a token's u to [2^14, 2^15); 2^126 at most, so that
// its inverse is a normal number.
__device__ __forceinline__ int kx_shift(uint32_t top_bits) {
    const int s = 127 + 14 - (int)(top_bits >> 23);
    return s > 126 ? 126 : s;
}
__device__ __forceinline__ float kx_pow2(int e) { return __builtin_bit_cast(float, (uint32_t)(127 + e) << 23); }

typedef __fp16 kx_p2 __attribute__((ext_vector_type(2)));
typedef _Float16 kx_h2 __attribute__((ext_vector_type(2)));

// Eight fp32 values as two binary16 parts, v * 2^shift = hi + lo up to 2^-20 of it (or 2^-38 of the token's largest), and the
// factor that undoes the shift.  Both parts are cut, not rounded: what hi leaves, lo takes.  A lane holds half of its token's values,
// lane ^ 32 the other.  An infinity or a NaN is hi alone, and the shift that of the token's other values.
template <int G> __device__ __forceinline__ void kx_split(const float (&v)[G][8], kx_h8 (&hi)[G], kx_h8 (&lo)[G], float& down) {
    float top = 0.0f;
#pragma unroll
    for (int c = 0; c < G; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) top = __builtin_fmaxf(top, __builtin_fabsf(v[c][i]));
    top = __builtin_fmaxf(top, __shfl_xor(top, 32));
    const bool odd = __builtin_amdgcn_ballot_w64(top > 3.4028235e38f) != 0;   // an infinity somewhere: rare
    if (odd) {
        top = 0.0f;
#pragma unroll
        for (int c = 0; c < G; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float m = __builtin_fabsf(v[c][i]);
                top = m <= 3.4028235e38f && m > top ? m : top;
            }
        top = __builtin_fmaxf(top, __shfl_xor(top, 32));
    }
    const int shift = kx_shift(__builtin_bit_cast(uint32_t, top));
    const float up = kx_pow2(shift);
    down = kx_pow2(-shift);
#pragma unroll
    for (int c = 0; c < G; ++c)
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const float a = v[c][i] * up, b = v[c][i + 1] * up;
            const kx_h2 h = __builtin_bit_cast(kx_h2, __builtin_amdgcn_cvt_pkrtz(a, b));
            const kx_h2 l = __builtin_bit_cast(kx_h2, __builtin_amdgcn_cvt_pkrtz(a - (float)h.x, b - (float)h.y));
            hi[c][i] = h.x, hi[c][i + 1] = h.y;
            lo[c][i] = l.x, lo[c][i + 1] = l.y;
        }
    if (odd) {                                                                // an infinity leaves itself less itself, no number
#pragma unroll
        for (int c = 0; c < G; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) lo[c][i] = __builtin_fabsf(v[c][i]) <= 3.4028235e38f ? lo[c][i] : (_Float16)0.0f;
    }
}

// The next slot: that of the first token left (sl < 0: none, or taken already), which it takes with all others of the slot;
// sel: whose they are.  -1 and nobody's if no token is left.
template <int N> __device__ __forceinline__ int kx_take(int (&sl)[N], bool (&sel)[N]) {
    int s = -1;
#pragma unroll
    for (int i = N - 1; i >= 0; --i) {
        const uint64_t left = __builtin_amdgcn_ballot_w64(sl[i] >= 0);
        const int first = __builtin_amdgcn_readlane(sl[i], left ? (int)__builtin_ctzll(left) : 0);
        s = left ? first : s;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        sel[i] = s >= 0 && sl[i] == s;
        sl[i] = sel[i] ? -1 : sl[i];
    }
    return s;
}

__device__ __forceinline__ KxToken kx_token(const int32_t* slot_of, const int32_t* rank, const float* scale, int slots, int token, int n) {
    KxToken k = {-1, 0, 0.0f, 0};
    const int s = token < n ? slot_of[token] : -1;
    if ((uint32_t)s < (uint32_t)slots) k.rank = rank[s], k.factor = scale[s];
    k.slot = k.rank > 0 ? s : -1;
    return k;
}

// The first lane of every slot among lanes 0 .. 31 (slot < 0: none), as a mask.
__device__ __forceinline__ uint32_t kx_leaders(int slot) {
    const uint32_t valid = (uint32_t)__builtin_amdgcn_ballot_w64(slot >= 0);
    if (valid == 0) return 0;
    const int s0 = __builtin_amdgcn_readlane(slot, __builtin_ctz(valid));
    if ((uint32_t)__builtin_amdgcn_ballot_w64(slot == s0) == valid) return valid & (0u - valid);
    uint32_t later = 0;
#pragma unroll
    for (int i = 0; i < 31; ++i) later |= (uint32_t)__builtin_amdgcn_ballot_w64(slot == __builtin_amdgcn_readlane(slot, i)) & (~1u << i);
    return valid & ~later;
}

// The adapters' part of a wavefront's product, 16 ranks at a time: u of all its tokens, whatever their slots, is loaded at once, without
// a branch between the loads that would make each wait for the last, then tile by tile of 32 columns the slots are gone through.
// Of `parts` wavefronts with the same columns this one takes every by_chunk-th 16 ranks and every by_slot-th slot from my_slot on.
template <int NT, int D> struct KxItems {
    static constexpr int kShares = NT == 1 ? kAdapterMaxShares : 2;      // of u at once; there are seldom more
    static constexpr int kAtOnce = NT == 4 ? 2 : NT;            // tiles; four would not fit the registers beside their accumulators
    struct Operand {
        kx_h8 v[2];
        int slot;               // whose it is, -1 for nobody's
    };
    const K4Expand& e;
    int my_slot, by_slot;
    const float* u0;
    const unsigned char* ops0;

    // ranks from 16 c on; unwritten memory where a token has no adapter or a lower rank.  tile: 0 .. NT - 1, one that there is
    __device__ __forceinline__ const float* at(int share, int tile, int c) const {
        return u0 + share * e.split_elems + (tile * (e.rank_pad / 16) + c) * 512;
    }
    __device__ __forceinline__ void load(int tile, int c, kx_f4 (&w)[kShares][2]) const {
#pragma unroll
        for (int b = 0; b < kShares; ++b) {
            const kx_f4* p = reinterpret_cast<const kx_f4*>(at(b < e.splits ? b : 0, tile, c));
            w[b][0] = p[0], w[b][1] = p[64];
        }
    }
    __device__ __forceinline__ void sum(int tile, int c, const kx_f4 (&w)[kShares][2], float (&v)[1][8]) const {
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            v[0][q] = w[0][q >> 2][q & 3];
#pragma unroll
            for (int b = 1; b < kShares; ++b) v[0][q] += b < e.splits ? w[b][q >> 2][q & 3] : 0.0f;
        }
        if constexpr (kShares < kAdapterMaxShares) {
            for (int s = kShares; s < e.splits; ++s) {
                const kx_f4* p = reinterpret_cast<const kx_f4*>(at(s, tile, c));
                const kx_f4 x = p[0], y = p[64];
#pragma unroll
                for (int q = 0; q < 4; ++q) v[0][q] += x[q], v[0][4 + q] += y[q];
            }
        }
    }

    __device__ __forceinline__ void fetch(int s, int c, Operand& to) const {
        if (to.slot == s) return;
        const unsigned char* ops = ops0 + s * e.slot_bytes + c * 2048;
        to.v[0] = *reinterpret_cast<const kx_h8*>(ops), to.v[1] = *reinterpret_cast<const kx_h8*>(ops + 1024);
        to.slot = s;
    }

    // The slots (those of the leaders) with ranks from 16 c on that are this wavefront's, as a mask of their first lanes
    __device__ __forceinline__ uint32_t slots_of(const KxToken& tok, uint32_t leaders, int c) const {
        uint32_t left = leaders & (uint32_t)__builtin_amdgcn_ballot_w64(tok.rank > c * 16);
        for (int i = 0; i < my_slot; ++i) left &= left - 1;
        return left;
    }

    // Tile NTI: D slots have their B on the way at once.  b may hold one's, of the tile before.
    template <int NTI>
    __device__ __forceinline__ void multiply(int c, const KxToken& tok, uint32_t left, float (&v)[1][8], Operand (&b)[D], kx_f16 (&acc)[2][NT]) const {
        bool have[D];
        auto next = [&](int d) {
            have[d] = left != 0;
            if (have[d]) {
                const int s = __builtin_amdgcn_readlane(tok.slot, __builtin_ctz(left));
                for (int i = 0; i < by_slot; ++i) left &= left - 1;
                fetch(s, c, b[d]);
            }
        };
#pragma unroll
        for (int d = 0; d < D; ++d) next(d);
        kx_h8 hi[1], lo[1];
        float down;
#pragma unroll
        for (int q = 0; q < 8; ++q) v[0][q] = tok.rank > c * 16 ? v[0][q] : 0.0f;             // (not written there)
        kx_split<1>(v, hi, lo, down);
        // the factor of the token's sums: its slot's and what undoes the shift, kept finite so that a sum of 0 stays one
        const float f = __builtin_fminf(__builtin_fmaxf(down * tok.factor, -3.4028235e38f), 3.4028235e38f);
#pragma unroll 1
        while (have[0]) {
#pragma unroll
            for (int d = 0; d < D; ++d) {
                if (!have[d]) continue;
                const bool sel = tok.slot == b[d].slot;
#pragma unroll
                for (int mt = 0; mt < 2; ++mt) {
                    kx_f16 t = kx_f16(0.0f);
                    t = __builtin_amdgcn_mfma_f32_32x32x16_f16(b[d].v[mt], hi[0], t, 0, 0, 0);
                    t = __builtin_amdgcn_mfma_f32_32x32x16_f16(b[d].v[mt], lo[0], t, 0, 0, 0);
#pragma unroll
                    for (int q = 0; q < 16; ++q) acc[mt][NTI][q] = sel ? __builtin_fmaf(t[q], f, acc[mt][NTI][q]) : acc[mt][NTI][q];
                    __builtin_amdgcn_sched_barrier(0);           // one tile's sums at a time: with all of them in registers the rest would spill
                }
            }
#pragma unroll
            for (int d = 0; d < D; ++d) next(d);
        }
    }
    template <int NTI>
    __device__ __forceinline__ void tiles(int c, const KxToken (&tok)[NT], const uint32_t (&leaders)[NT], const int (&tile)[NT], kx_f4 (&w)[kAtOnce][kShares][2],
                                          Operand (&b)[D], kx_f16 (&acc)[2][NT]) const {
        if constexpr (NTI % kAtOnce == 0) {
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) load(tile[NTI + i], c, w[i]);
        }
        const uint32_t left = slots_of(tok[NTI], leaders[NTI], c);
        if (left) {
            float v[1][8];
            sum(tile[NTI], c, w[NTI % kAtOnce], v);
            multiply<NTI>(c, tok[NTI], left, v, b, acc);
        }
        if constexpr (NTI + 1 < NT) tiles<NTI + 1>(c, tok, leaders, tile, w, b, acc);
    }
};

// Adds to acc (two 32-row tiles of row tile rt by NT tiles of 32 columns from col0) the adapters' part, or, of `parts` wavefronts
// with the same columns, the part of wavefront `part`: they deal the ranks out among them first, 16 at a time, then the slots.
template <int NT>
__device__ __forceinline__ void k4_expand(const K4Expand& e, kx_f16 (&acc)[2][NT], int col0, int n, int rt, int lane, int part, int parts) {
    constexpr int D = NT == 1 ? 8 : (NT == 2 ? 4 : 1);
    if (col0 >= n) return;
    int by_chunk = 1;
    while (by_chunk < parts && 2 * by_chunk * 16 <= e.rank_pad) by_chunk *= 2;
    const int c0 = part % by_chunk;
    const KxItems<NT, D> items = {e, part / by_chunk, parts / by_chunk, e.u + kx_at(col0, 0, e.rank_pad) + lane * 4,
                                  static_cast<const unsigned char*>(e.operands) + (int64_t)rt * (e.rank_pad / 16) * 2048 + lane * 16};
    KxToken tok[NT];
    int tile[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int t = col0 + nt * 32 + (lane & 31);
        tok[nt] = e.tokens[t < n ? t : n - 1];
        tile[nt] = col0 + nt * 32 < n ? nt : 0;
    }
    kx_f4 w[KxItems<NT, D>::kAtOnce][KxItems<NT, D>::kShares][2];
    int top = 0;
    uint32_t leaders[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        if (col0 + nt * 32 + (lane & 31) >= n) tok[nt].slot = -1, tok[nt].rank = 0;
        top = tok[nt].rank > top ? tok[nt].rank : top;
        leaders[nt] = kx_leaders(tok[nt].slot);
    }
#pragma unroll 1
    for (int c = c0; __builtin_amdgcn_ballot_w64(top > c * 16); c += by_chunk) {
        typename KxItems<NT, D>::Operand b[D];
#pragma unroll
        for (int d = 0; d < D; ++d) b[d].slot = -1;
        items.template tiles<0>(c, tok, leaders, tile, w, b, acc);
    }
}

}  // namespace ppc
