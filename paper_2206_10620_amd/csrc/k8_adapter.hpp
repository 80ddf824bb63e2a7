// Kernels of the low-rank adapters (include/pp_adapter.h), gfx950: the loading of a slot, the projections u = A x and v = B^T g, the
// expansion in binary32 and the gradients of A and B.  The expansion in binary16 is part of the block product (k4_expand.hpp).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "k4_expand.hpp"
#include "pieces.hpp"

namespace ppc {

typedef float k8_f4 __attribute__((ext_vector_type(4)));
typedef _Float16 k8_h8 __attribute__((ext_vector_type(8)));

// Eight values of a matrix operand, as a lane of the 16-row instructions holds them: one 16 x 16 x 32 step in binary16, eight
// 16 x 16 x 4 steps in binary32.  Lane l is row (column) l % 16 and reduction index 8 (l / 16) + i; the result's register i is row
// 4 (l / 16) + i, column l % 16.
template <typename T> struct K8Vec;
template <> struct K8Vec<_Float16> { typedef k8_h8 type; };
template <> struct K8Vec<float> { typedef float type __attribute__((ext_vector_type(8))); };
template <typename T> using k8_v8 = typename K8Vec<T>::type;

__device__ __forceinline__ k8_f4 k8_mfma(const k8_v8<_Float16>& a, const k8_v8<_Float16>& b, k8_f4 acc) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, acc, 0, 0, 0);
}
__device__ __forceinline__ k8_f4 k8_mfma(const k8_v8<float>& a, const k8_v8<float>& b, k8_f4 acc) {
#pragma unroll
    for (int i = 0; i < 8; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], acc, 0, 0, 0);
    return acc;
}

// ---- loading ----
// Copies A [rank][k] and B [m][rank] into operand order for both directions, zeros behind the rank and the sizes, one lane to
// eight values.  Only the ranks' tiles of 16 that the rank reaches are written: no kernel reads the others.
struct K8Load {
    const void* a;
    const void* b;
    void *a_project, *b_project;     // A and B^T, rows = ranks
    void *a_expand, *b_expand;       // A^T and B, rows = k and m
    int32_t* rank;
    float* scale;
    float factor;
    int32_t m, k, r, rank_pad, slot;
    int64_t items[4];                // eights of a_project, b_project, a_expand, b_expand
};
template <typename T> __global__ __launch_bounds__(256) void k8_load_slot(const K8Load p) {
    if (blockIdx.x == 0 && threadIdx.x == 0) p.rank[p.slot] = p.r, p.scale[p.slot] = p.factor;
    const T* a = static_cast<const T*>(p.a);
    const T* b = static_cast<const T*>(p.b);
    constexpr bool half = sizeof(T) == 2;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;; at += (int64_t)gridDim.x * 256) {
        int64_t i = at;
        int what = 0;
        while (what < 4 && i >= p.items[what]) i -= p.items[what++];
        if (what == 4) break;
        const bool of_a = (what & 1) == 0;
        const int width = of_a ? p.k : p.m;
        k8_v8<T> v;
        T* dst;
        if (what < 2) {                                          // [rank tile][width / 32][64][8]
            const int lane = (int)(i & 63), steps = (width + 31) / 32;
            const int64_t group = i >> 6;
            const int row = (int)(group / steps) * 16 + (lane & 15), c0 = (int)(group % steps) * 32 + (lane >> 4) * 8;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                T x = (T)0.0f;
                if (row < p.r && c0 + e < width) x = of_a ? a[(int64_t)row * p.k + c0 + e] : b[(int64_t)(c0 + e) * p.r + row];
                v[e] = x;
            }
            dst = static_cast<T*>(of_a ? p.a_project : p.b_project) + i * 8;
        } else {
            const int tiles = (p.r + 15) / 16;                   // of the rank: the ones written
            int row, j0;
            if (half) {                                          // [width / 64][rank_pad / 16][2][64][8]
                const int lane = (int)(i & 63), side = (int)(i >> 6) & 1;
                const int64_t group = i >> 7;
                const int64_t tile = group / tiles;
                const int chunk = (int)(group - tile * tiles);
                row = (int)tile * 64 + side * 32 + (lane & 31), j0 = chunk * 16 + (lane >> 5) * 8;
                dst = static_cast<T*>(of_a ? p.a_expand : p.b_expand) + (((tile * (p.rank_pad / 16) + chunk) * 2 + side) * 64 + lane) * 8;
            } else {                                             // [width][rank_pad]
                const int64_t eighth = i / (2 * tiles);
                row = (int)eighth, j0 = (int)(i - eighth * (2 * tiles)) * 8;
                dst = static_cast<T*>(of_a ? p.a_expand : p.b_expand) + (int64_t)row * p.rank_pad + j0;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                T x = (T)0.0f;
                if (row < width && j0 + e < p.r) x = of_a ? a[(int64_t)(j0 + e) * p.k + row] : b[(int64_t)row * p.r + j0 + e];
                v[e] = x;
            }
        }
        *reinterpret_cast<k8_v8<T>*>(dst) = v;
    }
}

// ---- projection ----
// u[split][t][j] = sum over a share of x's rows of A_s[j][row] x[row][t], s the slot of token t.
//
// x has its tokens next to each other, the matrix instruction wants eight consecutive rows of one token in a lane: a lane loads
// FT tokens of eight rows and takes the eight values of each from those registers, so that token c FT + f of a tile is column c of
// instruction f, with neither LDS nor a transposing read.  The wavefronts of a workgroup take shares of the rows and are added up
// through LDS in order.  A workgroup takes its tokens slot by slot; an instruction's columns do not touch each other, and only the
// columns of the slot's own tokens are stored.
// GATED: x is dy, taken as 0 where the layer's output, held in 8 bits, is not above 0; the result is also written to g.
struct K8Project {
    const void* x;              // [rows][n]
    const int8_t* gate;         // [rows][gate_pitch]
    void* g;                    // [rows][n]
    float* u;                   // [splits][n][rank_pad]
    const int32_t* slot_of;
    const int32_t* rank;
    const void* operands;       // [slot][rank tile][steps][64 lanes][8]
    int64_t slot_elems, gate_pitch;
    int32_t rows, n, steps, slots, rank_pad, splits;
};
constexpr int k8_project_lds(int ft, int waves) { return waves * ft * 64 * 16; }

template <typename T, int FT, int RG, int W, bool GATED>
__global__ __launch_bounds__(64 * W) void k8_project(const K8Project a) {
    __shared__ k8_f4 red[W * FT * 64];
    const int lane = (int)(threadIdx.x & 63u), wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int c = lane & 15, g = lane >> 4;
    const int tile = (int)blockIdx.x / a.splits, split = (int)blockIdx.x - tile * a.splits;
    const int t0 = tile * 16 * FT, mine0 = t0 + c * FT;
    const int s0 = (int)((int64_t)a.steps * split / a.splits), s1 = (int)((int64_t)a.steps * (split + 1) / a.splits);
    const int w0 = s0 + (int)((int64_t)(s1 - s0) * wave / W), w1 = s0 + (int)((int64_t)(s1 - s0) * (wave + 1) / W);
    const int left = a.n - mine0;
    const T* x = static_cast<const T*>(a.x);
    float* u = a.u + (int64_t)split * a.n * a.rank_pad;

    // One slot's tokens (slot -1: only the gate), ranks from tile rt0 on.
    auto pass = [&](int slot, int rt0, int tiles, bool write_g) {
        k8_f4 acc[RG][FT];
#pragma unroll
        for (int r = 0; r < RG; ++r)
#pragma unroll
            for (int f = 0; f < FT; ++f) acc[r][f] = k8_f4(0.0f);
        const T* ops = static_cast<const T*>(a.operands) + (slot < 0 ? 0 : slot * a.slot_elems) + (int64_t)rt0 * a.steps * 512 + lane * 8;
        auto load = [&](int st, T (&v)[8][FT]) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int row = st * 32 + g * 8 + i;
                k8_load<T, FT>(x + (int64_t)row * a.n + mine0, row < a.rows ? left : 0, v[i]);
            }
            if constexpr (GATED) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int row = st * 32 + g * 8 + i;
                    if (row < a.rows && left > 0) {
                        int8_t q[FT];
                        k8_load<int8_t, FT>(a.gate + (int64_t)row * a.gate_pitch + mine0, FT, q);
#pragma unroll
                        for (int f = 0; f < FT; ++f) v[i][f] = q[f] > 0 ? v[i][f] : (T)0.0f;
                        if (write_g) k8_store<T, FT>(static_cast<T*>(a.g) + (int64_t)row * a.n + mine0, left, v[i]);
                    }
                }
            }
        };
#pragma unroll 2
        for (int st = w0; st < w1; ++st) {
            T v[8][FT];
            load(st, v);
#pragma unroll
            for (int r = 0; r < RG; ++r)
                if (r < tiles) {
                    const k8_v8<T> op = *reinterpret_cast<const k8_v8<T>*>(ops + ((int64_t)r * a.steps + st) * 512);
#pragma unroll
                    for (int f = 0; f < FT; ++f) {
                        k8_v8<T> b;
#pragma unroll
                        for (int i = 0; i < 8; ++i) b[i] = v[i][f];
                        acc[r][f] = k8_mfma(op, b, acc[r][f]);
                    }
                }
        }
        if (slot < 0) return;
        const int rank = a.rank[slot];
#pragma unroll
        for (int r = 0; r < RG; ++r) {
            if (r < tiles) {
                __syncthreads();                                 // what was there has been read
#pragma unroll
                for (int f = 0; f < FT; ++f) red[(wave * FT + f) * 64 + lane] = acc[r][f];
                __syncthreads();
                for (int i = (int)threadIdx.x; i < FT * 64; i += 64 * W) {
                    const int f = i >> 6, ln = i & 63, t = t0 + (ln & 15) * FT + f, j = (rt0 + r) * 16 + (ln >> 4) * 4;
                    k8_f4 v = red[i];
#pragma unroll
                    for (int w = 1; w < W; ++w) v += red[w * FT * 64 + i];
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = j + e < rank ? v[e] : 0.0f;
                    if (t < a.n && a.slot_of[t] == slot) *reinterpret_cast<k8_f4*>(u + (int64_t)t * a.rank_pad + j) = v;
                }
            }
        }
    };

    int sl[FT];
#pragma unroll
    for (int f = 0; f < FT; ++f) sl[f] = kx_slot(a.slot_of, a.rank, a.slots, mine0 + f, a.n);
    bool write_g = GATED && blockIdx.y == 0;
    for (int index = 0;; ++index) {
        const int s = kx_next(sl);
        if (s < 0) break;
#pragma unroll
        for (int f = 0; f < FT; ++f) sl[f] = sl[f] == s ? -1 : sl[f];
        if (index % (int)gridDim.y != (int)blockIdx.y) continue;
        const int tiles = (__builtin_amdgcn_readfirstlane(a.rank[s]) + 15) / 16;
        for (int rt0 = 0; rt0 < tiles; rt0 += RG) {
            pass(s, rt0, tiles - rt0, write_g);
            write_g = false;
        }
    }
    if (write_g) pass(-1, 0, 0, true);
}

// ---- expansion in binary32 ----
// y = act(y + c_s B_s u), in place, behind the product: the sum is in binary32 either way, and y is read and written once more.
// A wavefront takes 16 rows of y and 64 tokens, four to a lane.
struct K8Expand {
    float* y;                   // [m][n]
    const float* u;             // [splits][n][rank_pad]
    const int32_t* slot_of;
    const int32_t* rank;
    const float* scale;
    const float* operands;      // [slot][m][rank_pad]
    int64_t slot_elems, split_elems;
    int32_t m, n, slots, splits, rank_pad, relu;
};
__global__ __launch_bounds__(256) void k8_expand_f32(const K8Expand a) {
    const int lane = (int)(threadIdx.x & 63u), wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int c = lane & 15, g = lane >> 4;
    const int row0 = ((int)blockIdx.x * 4 + wave) * 16, t0 = (int)blockIdx.y * 64 + c * 4, left = a.n - t0;
    if (row0 >= a.m) return;
    int sl[4];
    bool any = false;
#pragma unroll
    for (int f = 0; f < 4; ++f) {
        sl[f] = kx_slot(a.slot_of, a.rank, a.slots, t0 + f, a.n);
        any = any || sl[f] >= 0;
    }
    if (!a.relu && __builtin_amdgcn_ballot_w64(any) == 0) return;
    float y[4][4];                                               // [row][token]
#pragma unroll
    for (int i = 0; i < 4; ++i) k8_load<float, 4>(a.y + (int64_t)(row0 + 4 * g + i) * a.n + t0, row0 + 4 * g + i < a.m ? left : 0, y[i]);
    for (;;) {
        const int s = kx_next(sl);
        if (s < 0) break;
        const int tiles = (__builtin_amdgcn_readfirstlane(a.rank[s]) + 15) / 16;
        const float factor = a.scale[s];
        const float* ops = a.operands + s * a.slot_elems + (int64_t)(row0 + c) * a.rank_pad + 4 * g;
        const float* up = a.u + (int64_t)t0 * a.rank_pad + 4 * g;
        bool sel[4];
        k8_f4 acc[4];
#pragma unroll
        for (int f = 0; f < 4; ++f) {
            sel[f] = sl[f] == s;
            if (sel[f]) sl[f] = -1;
            acc[f] = k8_f4(0.0f);
        }
        for (int r = 0; r < tiles; ++r) {
            k8_f4 op = k8_f4(0.0f);
            if (row0 + c < a.m) op = *reinterpret_cast<const k8_f4*>(ops + r * 16);
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                k8_f4 w = k8_f4(0.0f);
                if (sel[f])
                    for (int sp = 0; sp < a.splits; ++sp) w += *reinterpret_cast<const k8_f4*>(up + sp * a.split_elems + (int64_t)f * a.rank_pad + r * 16);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[f] = __builtin_amdgcn_mfma_f32_16x16x4f32(op[i], w[i], acc[f], 0, 0, 0);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int f = 0; f < 4; ++f) y[i][f] = sel[f] ? __builtin_fmaf(acc[f][i], factor, y[i][f]) : y[i][f];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int f = 0; f < 4; ++f)
            if (a.relu) y[i][f] = y[i][f] > 0.0f ? y[i][f] : 0.0f;
        k8_store<float, 4>(a.y + (int64_t)(row0 + 4 * g + i) * a.n + t0, row0 + 4 * g + i < a.m ? left : 0, y[i]);
    }
}

// ---- gradients of A and B ----
// G[p][j] = c_s sum over the tokens t of slot s of z[p][t] w[t][j], with z = x and w = v for A, z = g and w = u for B.
//
// Both operands have the tokens, the reduction, next to each other in memory or can be had so: z's 16 bytes of a row come straight
// from memory, w's 128 tokens are turned through LDS once for the workgroup's 64 RW rows.  In binary16 they are two parts, hi and lo,
// after a power of two taken out for each rank and block; x in 8 bits is exact in binary16, its power of two for each row and block
// joins the other when a block's sum is added to the whole.  Tokens of other slots in a block are taken as zeros on both sides; blocks
// without one of the slot's are passed over.
// A workgroup takes a share of the blocks; with several shares the sums are joined in order by k8_grad_join.
struct K8Grad {
    const void* x;              // [k][n], or int8 [k][x_pitch]
    const uint8_t* x_scale;     // [block][x_scale_pitch]
    const void* g;              // [m][n]
    const float* v;             // [v_splits][n][rank_pad]
    const float* u;             // [u_splits][n][rank_pad]
    const int32_t* slot_of;
    const int32_t* which;
    const int32_t* rank;
    const float* scale;
    float *da, *db, *work;
    int64_t x_pitch, x_scale_pitch;
    int32_t m, k, n, slots, rank_pad, max_rank, tiles_k, count, splits, u_splits, v_splits;
};

// The workgroup's LDS: 128 tokens of RG rank tiles of w, [32 tokens][rank tile][part][64 lanes][8], and a factor for each rank.
template <typename T, int RG> struct K8GradLds {
    static constexpr int parts = sizeof(T) == 2 ? 2 : 1;
    k8_v8<T> w[4][RG][parts][64];
    float down[RG][16];
};

// Eight values of z for a lane: row p, tokens t ..  Zeros from `left` on; `byte`: which of the eight tokens are the slot's.
template <typename T> __device__ __forceinline__ k8_v8<T> k8_z(const T* row, int left, bool row_ok) {
    T v[8];
    k8_load<T, 8>(row, row_ok ? left : 0, v);
    k8_v8<T> z;
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = v[i];
    return z;
}
template <typename T> __device__ __forceinline__ k8_v8<T> k8_z8(const int8_t* row, bool row_ok) {
    k8_v8<T> z;
    uint2 q = {0u, 0u};
    if (row_ok) q = *reinterpret_cast<const uint2*>(row);
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = (T)(float)(int8_t)((i < 4 ? q.x : q.y) >> (8 * (i & 3)));
    return z;
}

template <typename T, int RG, int RW, bool HELD8>
__global__ __launch_bounds__(256) void k8_grad(const K8Grad a) {
    __shared__ K8GradLds<T, RG> lds;
    constexpr bool half = sizeof(T) == 2;
    constexpr int PARTS = K8GradLds<T, RG>::parts;
    const int lane = (int)(threadIdx.x & 63u), wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int c = lane & 15, g = lane >> 4;
    const bool of_a = (int)blockIdx.x < a.tiles_k;
    const int rows = of_a ? a.k : a.m;
    const int row0 = ((int)blockIdx.x - (of_a ? 0 : a.tiles_k)) * 64 * RW + wave * 16 * RW;
    const int at = (int)blockIdx.y, split = (int)blockIdx.z;
    const int wanted = a.which[at];
    const int slot = (uint32_t)wanted < (uint32_t)a.slots ? wanted : -1;
    const int rank = slot < 0 ? 0 : __builtin_amdgcn_readfirstlane(a.rank[slot]);
    const int blocks = (a.n + 127) / 128;
    const int b0 = (int)((int64_t)blocks * split / a.splits), b1 = (int)((int64_t)blocks * (split + 1) / a.splits);
    const float* w = of_a ? a.v : a.u;
    const int w_splits = of_a ? a.v_splits : a.u_splits;
    const int64_t w_split = (int64_t)a.n * a.rank_pad;
    const int tiles_all = a.rank_pad / 16;

    for (int rt0 = 0; rt0 < tiles_all; rt0 += RG) {
        const int tiles = min((rank + 15) / 16 - rt0, RG);       // of this slot, here (none: zeros are stored)
        k8_f4 acc[RW][RG];
#pragma unroll
        for (int i = 0; i < RW; ++i)
#pragma unroll
            for (int r = 0; r < RG; ++r) acc[i][r] = k8_f4(0.0f);
        for (int b = b0; b < (tiles > 0 ? b1 : b0); ++b) {
            const int tb = b * 128;
            const bool in0 = tb + lane < a.n && a.slot_of[tb + lane] == slot, in1 = tb + 64 + lane < a.n && a.slot_of[tb + 64 + lane] == slot;
            const uint64_t m0 = __builtin_amdgcn_ballot_w64(in0), m1 = __builtin_amdgcn_ballot_w64(in1);
            if ((m0 | m1) == 0) continue;
            __syncthreads();                                     // the last block's operands have been read
            {
                // a wavefront turns four ranks of each tile: lane 4 q + j has tokens 8 q .. of rank j
                const int j4 = lane & 3, q = lane >> 2;
                const uint32_t byte = (uint32_t)((q < 8 ? m0 : m1) >> (8 * (q & 7))) & 0xffu;
#pragma unroll
                for (int r = 0; r < RG; ++r)
                    if (r < tiles) {
                        const int j = wave * 4 + j4;
                        const float* p = w + (int64_t)(tb + 8 * q) * a.rank_pad + (rt0 + r) * 16 + j;
                        float v[8];
                        uint32_t top = 0;
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            v[i] = 0.0f;
                            if ((byte >> i) & 1u)
                                for (int sp = 0; sp < w_splits; ++sp) v[i] += p[sp * w_split + (int64_t)i * a.rank_pad];
                            const uint32_t bits = __builtin_bit_cast(uint32_t, v[i]) & 0x7fffffffu;
                            if (bits < 0x7f800000u && bits > top) top = bits;
                        }
                        const int dst = (q & 3) * 16 + j;
                        if constexpr (half) {
#pragma unroll
                            for (int x = 4; x < 64; x *= 2) {
                                const uint32_t o = (uint32_t)__shfl_xor((int)top, x);
                                top = o > top ? o : top;
                            }
                            const int shift = kx_shift(top);
                            const float up = kx_pow2(shift);
                            k8_v8<T> hi, lo;
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                _Float16 h, l;
                                kx_parts(v[i] * up, h, l);
                                hi[i] = (T)h, lo[i] = (T)l;
                            }
                            lds.w[q >> 2][r][0][dst] = hi;
                            lds.w[q >> 2][r][PARTS - 1][dst] = lo;
                            if (q == 0) lds.down[r][j] = kx_pow2(-shift);
                        } else {
                            k8_v8<T> o;
#pragma unroll
                            for (int i = 0; i < 8; ++i) o[i] = (T)v[i];
                            lds.w[q >> 2][r][0][dst] = o;
                            if (q == 0) lds.down[r][j] = 1.0f;
                        }
                    }
            }
            __syncthreads();
            const bool whole = (m0 & m1) == ~0ull;
#pragma unroll
            for (int i = 0; i < RW; ++i) {
                const int row = row0 + i * 16 + c;
                const bool row_ok = row < rows;
                k8_v8<T> z[4];
#pragma unroll
                for (int st = 0; st < 4; ++st) {
                    const int t = tb + st * 32 + g * 8;
                    if (HELD8 && of_a) z[st] = k8_z8<T>(static_cast<const int8_t*>(a.x) + (int64_t)row * a.x_pitch + t, row_ok);
                    else z[st] = k8_z<T>(static_cast<const T*>(of_a ? a.x : a.g) + (int64_t)row * a.n + t, a.n - t, row_ok);
                    if (!whole) {
                        const uint32_t byte = (uint32_t)((st < 2 ? m0 : m1) >> (32 * (st & 1) + 8 * g)) & 0xffu;
#pragma unroll
                        for (int e = 0; e < 8; ++e) z[st][e] = (byte >> e) & 1u ? z[st][e] : (T)0.0f;
                    }
                }
                float zs[4] = {1.0f, 1.0f, 1.0f, 1.0f};          // of the rows of this lane's results
                if (HELD8 && of_a) {
                    const int r4 = row0 + i * 16 + 4 * g;
                    uint32_t s4 = 0;
                    if (r4 < a.x_scale_pitch) s4 = *reinterpret_cast<const uint32_t*>(a.x_scale + (int64_t)b * a.x_scale_pitch + r4);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t s = (s4 >> (8 * e)) & 0xffu;
                        zs[e] = __builtin_bit_cast(float, s == 255u ? 0x7fc00000u : s << 23);
                    }
                }
#pragma unroll
                for (int r = 0; r < RG; ++r)
                    if (r < tiles) {
                        k8_f4 sum = k8_f4(0.0f);
#pragma unroll
                        for (int st = 0; st < 4; ++st)
#pragma unroll
                            for (int part = 0; part < PARTS; ++part) sum = k8_mfma(z[st], lds.w[st][r][part][lane], sum);
                        const float down = lds.down[r][c];
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][r][e] = __builtin_fmaf(sum[e] * down, zs[e], acc[i][r][e]);
                    }
            }
        }
        // lane's results: rows 4 g + e, rank c
        const float factor = slot < 0 ? 0.0f : a.scale[slot];
#pragma unroll
        for (int i = 0; i < RW; ++i)
#pragma unroll
            for (int r = 0; r < RG; ++r) {
                if (rt0 + r >= tiles_all) continue;
                const int j = (rt0 + r) * 16 + c, p = row0 + i * 16 + 4 * g;
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = j < rank ? acc[i][r][e] : 0.0f;
                if (a.splits > 1) {
                    float* part = a.work + ((int64_t)split * a.count + at) * ((int64_t)a.k + a.m) * a.rank_pad;
                    if (of_a) k8_store<float, 4>(part + (int64_t)j * a.k + p, rows - p, v);
                    else
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (p + e < rows) part[(int64_t)a.rank_pad * a.k + (int64_t)(p + e) * a.rank_pad + j] = v[e];
                } else if (j < a.max_rank) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = j < rank ? v[e] * factor : 0.0f;
                    if (of_a) k8_store<float, 4>(a.da + ((int64_t)at * a.max_rank + j) * a.k + p, rows - p, v);
                    else
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (p + e < rows) a.db[((int64_t)at * a.m + p + e) * a.max_rank + j] = v[e];
                }
            }
    }
}

// Adds the shares up, in order, and takes the slot's factor in.
struct K8Join {
    const float* work;
    const int32_t* which;
    const int32_t* rank;
    const float* scale;
    float *da, *db;
    int32_t m, k, slots, rank_pad, max_rank, count, splits;
};
__global__ __launch_bounds__(256) void k8_grad_join(const K8Join a) {
    const int64_t per = ((int64_t)a.k + a.m) * a.max_rank, stride = (int64_t)a.count * ((int64_t)a.k + a.m) * a.rank_pad;
    const int at = (int)blockIdx.y, wanted = a.which[at];
    const int slot = (uint32_t)wanted < (uint32_t)a.slots ? wanted : -1;
    const int rank = slot < 0 ? 0 : a.rank[slot];
    const float factor = slot < 0 ? 0.0f : a.scale[slot];
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < per; i += (int64_t)gridDim.x * 256) {
        const bool of_a = i < (int64_t)a.k * a.max_rank;
        const int64_t o = of_a ? i : i - (int64_t)a.k * a.max_rank;
        const int j = of_a ? (int)(o / a.k) : (int)(o % a.max_rank);
        float v = 0.0f;
        if (j < rank) {
            const int64_t src = of_a ? o : (int64_t)a.rank_pad * a.k + o / a.max_rank * a.rank_pad + j;
            const float* p = a.work + (int64_t)at * ((int64_t)a.k + a.m) * a.rank_pad + src;
            for (int sp = 0; sp < a.splits; ++sp) v += p[sp * stride];
            v *= factor;
        }
        if (of_a) a.da[(int64_t)at * a.k * a.max_rank + o] = v;
        else a.db[(int64_t)at * a.m * a.max_rank + o] = v;
    }
}

}  // namespace ppc
