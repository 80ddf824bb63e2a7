// The adapters' part of a block product in binary16 (include/pp_adapter.h): c_s B_s u added to the accumulators of a wavefront
// before the product's own sum, so that it meets the sum, the bias and the activation in fp32.
//
// u [split][token][rank] is in fp32 and far smaller than x.  A lane of the matrix instruction's second operand holds eight
// consecutive ranks of one token, which is how u lies in memory: no staging.  They enter as two binary16 parts, hi and lo, after
// a power of two that brings the token's largest |u| to [2^14, 2^15) is taken out: 22 bits, whatever the size of u.  B lies in
// operand order, 1 KB per 32 rows and 16 ranks.
//
// The tokens of a wavefront are taken slot by slot.  A matrix instruction computes all its columns with the one slot's B;
// only the columns of that slot's tokens are taken over, so nothing a slot holds can reach another slot's tokens.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace ppc {

struct K4Expand {
    const float* u;             // [splits][n][rank_pad]
    const int32_t* slot_of;     // [n]
    const int32_t* rank;        // [slots]
    const float* scale;         // [slots]
    const void* operands;       // [slot][64-row tile][rank_pad / 16][2][64 lanes][8] binary16
    int64_t slot_bytes, split_elems;
    int32_t slots, splits, rank_pad;
};

typedef _Float16 kx_h8 __attribute__((ext_vector_type(8)));
typedef float kx_f4 __attribute__((ext_vector_type(4)));
typedef float kx_f16 __attribute__((ext_vector_type(16)));

// The power of two that brings the largest finite magnitude (its bits) of a token's u to [2^14, 2^15); 2^126 at most, so that
// its inverse is a normal number.
__device__ __forceinline__ int kx_shift(uint32_t top_bits) {
    const int s = 127 + 14 - (int)(top_bits >> 23);
    return s > 126 ? 126 : s;
}
__device__ __forceinline__ float kx_pow2(int e) { return __builtin_bit_cast(float, (uint32_t)(127 + e) << 23); }

// v = hi + lo up to 2^-22 of v (or 2^-25 absolute); an infinity or a NaN is hi alone
__device__ __forceinline__ void kx_parts(float v, _Float16& hi, _Float16& lo) {
    hi = (_Float16)v;
    const float rest = v - (float)hi;
    lo = __builtin_fabsf(v) <= 65504.0f ? (_Float16)rest : (_Float16)0.0f;
}

// The slot that a token's entry stands for: -1 for none.
__device__ __forceinline__ int kx_slot(const int32_t* slot_of, const int32_t* rank, int slots, int token, int n) {
    if (token >= n) return -1;
    const int s = slot_of[token];
    return (uint32_t)s < (uint32_t)slots && rank[s] > 0 ? s : -1;
}

// The slot of the first token that is left (sl < 0: none, or taken already); -1 if none is.
template <int N> __device__ __forceinline__ int kx_next(const int (&sl)[N]) {
    int s = -1;
#pragma unroll
    for (int i = N - 1; i >= 0; --i) {
        const uint64_t left = __builtin_amdgcn_ballot_w64(sl[i] >= 0);
        const int first = __builtin_amdgcn_readlane(sl[i], left ? (int)__builtin_ctzll(left) : 0);
        s = left ? first : s;
    }
    return s;
}

// Adds to acc (two 32-row tiles of row tile rt by NT tiles of 32 columns from col0) the adapters' part of every `parts`-th
// slot from `part` on.
template <int NT>
__device__ __forceinline__ void k4_expand(const K4Expand& e, kx_f16 (&acc)[2][NT], int col0, int n, int rt, int lane, int part, int parts) {
    int sl[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) sl[nt] = kx_slot(e.slot_of, e.rank, e.slots, col0 + nt * 32 + (lane & 31), n);
    int index = 0;
    for (;;) {
        const int s = kx_next(sl);
        if (s < 0) break;
        const bool mine = parts == 1 || index % parts == part;
        ++index;
        const int chunks = mine ? (__builtin_amdgcn_readfirstlane(e.rank[s]) + 15) / 16 : 0;
        const float factor = e.scale[s];
        const unsigned char* ops = static_cast<const unsigned char*>(e.operands) + s * e.slot_bytes + (int64_t)rt * (e.rank_pad / 16) * 2048 + lane * 16;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const bool sel = sl[nt] == s;
            if (sel) sl[nt] = -1;
            if (chunks == 0 || __builtin_amdgcn_ballot_w64(sel) == 0) continue;
            const float* up = e.u + (int64_t)(col0 + nt * 32 + (lane & 31)) * e.rank_pad + 8 * (lane >> 5);
            auto fetch = [&](int c, float (&v)[8]) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = 0.0f;
                if (sel)
                    for (int sp = 0; sp < e.splits; ++sp) {
                        const kx_f4* p = reinterpret_cast<const kx_f4*>(up + sp * e.split_elems + c * 16);
                        const kx_f4 a = p[0], b = p[1];
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[i] += a[i], v[4 + i] += b[i];
                    }
            };
            float v[8];
            uint32_t top = 0;
            for (int c = chunks - 1; c >= 0; --c) {                 // ends on chunk 0, which stays in v
                fetch(c, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t b = __builtin_bit_cast(uint32_t, v[i]) & 0x7fffffffu;
                    if (b < 0x7f800000u && b > top) top = b;
                }
            }
            const uint32_t other = (uint32_t)__shfl_xor((int)top, 32);
            top = top > other ? top : other;
            const int shift = kx_shift(top);
            const float up2 = kx_pow2(shift), down2 = kx_pow2(-shift);
            kx_f16 t[2] = {kx_f16(0.0f), kx_f16(0.0f)};
            for (int c = 0; c < chunks; ++c) {
                if (c) fetch(c, v);
                kx_h8 hi, lo;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    _Float16 h, l;
                    kx_parts(v[i] * up2, h, l);
                    hi[i] = h, lo[i] = l;
                }
#pragma unroll
                for (int mt = 0; mt < 2; ++mt) {
                    const kx_h8 b = *reinterpret_cast<const kx_h8*>(ops + c * 2048 + mt * 1024);
                    t[mt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(b, hi, t[mt], 0, 0, 0);
                    t[mt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(b, lo, t[mt], 0, 0, 0);
                }
            }
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[mt][nt][i] = sel ? __builtin_fmaf(t[mt][i] * down2, factor, acc[mt][nt][i]) : acc[mt][nt][i];
        }
    }
}

}  // namespace ppc
