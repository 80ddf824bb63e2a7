// Kernels of the low-rank adapters (include/pp_adapter.h), gfx950: the loading of a slot, the projections u = A x and v = B^T g, the
// expansion in binary32 and the gradients of A and B.  The expansion in binary16 is part of the block product (k4_expand.hpp).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "adapter_rules.hpp"
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
// Copies A [rank][k] and B [m][rank] of up to N slots into operand order for both directions, zeros behind the rank and the sizes, one lane
// to eight values.  Only the ranks' tiles of 16 that the rank reaches are written: no kernel reads the others.  The slots are arguments of
// the kernel, 32 bytes each: no table has to reach the device first.  What a single load costs is its launch: 64 slots of rank 16 take 4.3 us
// in a launch and 174 in one each with 300 x 300, 24 and 187 with 4096 x 4096.  N = 1 is there because 2 KB of arguments cost the host
// 0.5 us: a call of one slot takes 6.8 us, 7.3 with room for 64.
struct K8LoadSlot {
    const void* a;
    const void* b;
    float factor;
    int32_t r, slot, unused;
};
template <int N> struct K8Load {
    void *a_project, *b_project;     // A and B^T, rows = ranks: slot 0's
    void *a_expand, *b_expand;       // A^T and B, rows = k and m
    int64_t a_project_slot, b_project_slot, a_expand_slot, b_expand_slot;     // elements of one slot
    int32_t* rank;
    float* scale;
    int32_t m, k, rank_pad;
    K8LoadSlot of[N];
};
template <typename T, int N> __global__ __launch_bounds__(256) void k8_load_slots(const K8Load<N> p) {
    const K8LoadSlot s = p.of[N == 1 ? 0 : blockIdx.y];
    if (blockIdx.x == 0 && threadIdx.x == 0) p.rank[s.slot] = s.r, p.scale[s.slot] = s.factor;
    const T* a = static_cast<const T*>(s.a);
    const T* b = static_cast<const T*>(s.b);
    constexpr bool half = sizeof(T) == 2;
    const int tiles = (s.r + 15) / 16;                           // of the rank: the ones written
    const int64_t items[4] = {adapter_project_elems(p.k, tiles * 16) / 8, adapter_project_elems(p.m, tiles * 16) / 8,
                              adapter_expand_elems(p.k, tiles * 16, half) / 8, adapter_expand_elems(p.m, tiles * 16, half) / 8};
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;; at += (int64_t)gridDim.x * 256) {
        int64_t i = at;
        int what = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (what == q && i >= items[q]) i -= items[q], ++what;
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
                if (row < s.r && c0 + e < width) x = of_a ? a[(int64_t)row * p.k + c0 + e] : b[(int64_t)(c0 + e) * s.r + row];
                v[e] = x;
            }
            dst = static_cast<T*>(of_a ? p.a_project : p.b_project) + s.slot * (of_a ? p.a_project_slot : p.b_project_slot) + i * 8;
        } else {
            int row, j0;
            dst = static_cast<T*>(of_a ? p.a_expand : p.b_expand) + s.slot * (of_a ? p.a_expand_slot : p.b_expand_slot);
            if (half) {                                          // [width / 64][rank_pad / 16][2][64][8]
                const int lane = (int)(i & 63), side = (int)(i >> 6) & 1;
                const int64_t group = i >> 7;
                const int64_t tile = group / tiles;
                const int chunk = (int)(group - tile * tiles);
                row = (int)tile * 64 + side * 32 + (lane & 31), j0 = chunk * 16 + (lane >> 5) * 8;
                dst += (((tile * (p.rank_pad / 16) + chunk) * 2 + side) * 64 + lane) * 8;
            } else {                                             // [width][rank_pad]
                const int64_t eighth = i / (2 * tiles);
                row = (int)eighth, j0 = (int)(i - eighth * (2 * tiles)) * 8;
                dst += (int64_t)row * p.rank_pad + j0;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                T x = (T)0.0f;
                if (row < width && j0 + e < s.r) x = of_a ? a[(int64_t)(j0 + e) * p.k + row] : b[(int64_t)row * s.r + j0 + e];
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
// Ranks above 64 (32 in binary32 with four tokens to a lane: registers) are gone through in parts, each of which reads x: 4096 rows, 4096
// tokens, ranks 16 / 64 / 65 / 128 9.7 / 14.3 / 21.1 / 24.1 us, binary32 14.9 / 32.6 / 42.4 / 58.5.
// GATED: x is dy, taken as 0 where the layer's output, held in 8 bits, is not above 0; the result is also written to g.
struct K8Project {
    const void* x;              // [rows][n]
    const int8_t* gate;         // [rows][gate_pitch]
    void* g;                    // [rows][n]
    KxToken* tokens;            // [n]
    float* u;                   // [splits][kx_share], kx_at
    const int32_t* slot_of;
    const int32_t* rank;
    const float* scale;
    const void* operands;       // [slot][rank tile][steps][64 lanes][8]
    int64_t slot_elems, gate_pitch;
    int32_t rows, n, steps, slots, rank_pad, splits;
};
template <typename T, int FT, int RG, bool GATED>
__global__ __launch_bounds__(64 * kProjectWaves) void k8_project(const K8Project a) {
    constexpr int W = kProjectWaves;
    __shared__ k8_f4 red[W * FT * 64];
    const int lane = (int)(threadIdx.x & 63u), wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int c = lane & 15, g = lane >> 4;
    const int tile = (int)blockIdx.x / a.splits, split = (int)blockIdx.x - tile * a.splits;
    // The last tile is moved back to end with the last token, or, of one token to a lane, its last lanes repeat that: every load is whole
    const int own0 = tile * 16 * FT, t0 = project_first_token(tile, a.n, FT);
    const int mine0 = FT == 1 ? min(own0 + c, a.n - 1) : t0 + c * FT;
    const int s0 = (int)((int64_t)a.steps * split / a.splits), s1 = (int)((int64_t)a.steps * (split + 1) / a.splits);
    const int w0 = s0 + (int)((int64_t)(s1 - s0) * wave / W), w1 = s0 + (int)((int64_t)(s1 - s0) * (wave + 1) / W);
    const T* x = static_cast<const T*>(a.x);
    float* u = a.u + split * kx_share(a.n, a.rank_pad);

    typedef k8_any<T, FT> Piece;
    typedef k8_any<int8_t, FT> Gate;
    struct Rows {
        Piece v[8];
        Gate q[GATED ? 8 : 1];
        k8_v8<T> op[RG];
    };
    // Steps on their way at a time, as registers allow: one step's loads are back in about 1 us, and few wavefronts have more than eight
    constexpr int kStage = (FT * (int)sizeof(T) < 4 ? 8 : FT * (int)sizeof(T) * 2) + (GATED ? 8 : 0) + RG * (int)sizeof(T) * 2;
    constexpr int kAhead = kStage <= (GATED ? 24 : 40) ? 4 : 2;
    // Where row i of a lane's eight of a step is: what is the same for all lanes, and 32 bits.  WHOLE: all rows are there; otherwise the
    // last one is read in place of those behind it, and 0 taken: no branch between the loads, which would make the wait for one a wait for all.
    auto spot = [&](auto whole, const auto* p, int64_t pitch, int st, int i) {
        constexpr bool WHOLE = decltype(whole)::value;
        const int row = WHOLE ? g * 8 : min(g * 8 + i, a.rows - 1 - st * 32);
        const char* all = reinterpret_cast<const char*>(p + (int64_t)(st * 32 + (WHOLE ? i : 0)) * pitch);
        return all + (uint32_t)(row * (int)pitch + mine0) * (uint32_t)sizeof(*p);
    };
    auto load = [&](auto whole, int st, Rows& r) {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.v[i] = *reinterpret_cast<const Piece*>(spot(whole, x, a.n, st, i));
        if constexpr (GATED) {
#pragma unroll
            for (int i = 0; i < 8; ++i) r.q[i] = *reinterpret_cast<const Gate*>(spot(whole, a.gate, a.gate_pitch, st, i));
        }
    };
    // What was loaded, behind the gate
    auto take = [&](auto whole, auto write_g, int st, Rows& r) {
        constexpr bool WHOLE = decltype(whole)::value;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bool there = WHOLE || st * 32 + g * 8 + i < a.rows;
#pragma unroll
            for (int f = 0; f < FT; ++f) {
                bool through = there;
                if constexpr (GATED) through = through && k8_at<Gate, int8_t>(r.q[i], f) > 0;
                if (!through) k8_put(r.v[i], f, (T)0.0f);
            }
            if constexpr (decltype(write_g)::value) {
                if (there) *reinterpret_cast<Piece*>(const_cast<char*>(spot(whole, static_cast<const T*>(a.g), a.n, st, i))) = r.v[i];
            }
        }
    };

    // One slot's tokens (slot -1: only the gate), ranks from tile rt0 on.
    auto pass = [&](int slot, int rt0, int tiles, bool is_first) {
        k8_f4 acc[RG][FT];
#pragma unroll
        for (int r = 0; r < RG; ++r)
#pragma unroll
            for (int f = 0; f < FT; ++f) acc[r][f] = k8_f4(0.0f);
        const T* ops = static_cast<const T*>(a.operands) + (slot < 0 ? 0 : slot * a.slot_elems) + (int64_t)rt0 * a.steps * 512 + lane * 8;
        // The operands come with the rows: loads are waited for in their order
        auto steps = [&](auto whole, auto write_g, int from, int to) {
            asm("" : "+s"(from));                                // addresses are not kept from one pass for the next: registers
            auto fetch = [&](int st, Rows& r) {
#pragma unroll
                for (int i = 0; i < RG; ++i) r.op[i] = *reinterpret_cast<const k8_v8<T>*>(ops + ((int64_t)(i < tiles ? i : 0) * a.steps + st) * 512);
                load(whole, st, r);
                __builtin_amdgcn_sched_barrier(0);
            };
            auto multiply = [&](int st, Rows& r) {
                take(whole, write_g, st, r);
#pragma unroll
                for (int f = 0; f < FT; ++f) {
                    k8_v8<T> b;
#pragma unroll
                    for (int i = 0; i < 8; ++i) b[i] = k8_at<Piece, T>(r.v[i], f);
#pragma unroll
                    for (int i = 0; i < RG; ++i)
                        if (i < tiles) acc[i][f] = k8_mfma(r.op[i], b, acc[i][f]);
                }
                __builtin_amdgcn_sched_barrier(0);
            };
            constexpr int P = kAhead;
            Rows r[P];
#pragma unroll
            for (int j = 0; j < P; ++j) fetch(min(from + j, to - 1), r[j]);
            int st = from;
            for (; st + 2 * P <= to; st += P) {
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    multiply(st + j, r[j]);
                    fetch(st + P + j, r[j]);
                }
            }
#pragma unroll
            for (int j = 0; j < P; ++j)
                if (st + j < to) {
                    multiply(st + j, r[j]);
                    if (st + P + j < to) fetch(st + P + j, r[j]);
                }
#pragma unroll
            for (int j = 0; j + 1 < P; ++j)
                if (st + P + j < to) multiply(st + P + j, r[j]);
        };
        auto all = [&](auto write_g) {
            if (w1 * 32 <= a.rows) steps(std::true_type{}, write_g, w0, w1);
            else steps(std::false_type{}, write_g, w0, w1);
        };
        if (w0 < w1) {
            if (GATED && is_first && blockIdx.y == 0) all(std::integral_constant<bool, GATED>{});
            else all(std::false_type{});
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
#pragma unroll 4
                    for (int w = 1; w < W; ++w) v += red[w * FT * 64 + i];
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = j + e < rank ? v[e] : 0.0f;
                    if (t >= own0 && t < a.n && a.slot_of[t] == slot) *reinterpret_cast<k8_f4*>(u + kx_at(t, j, a.rank_pad)) = v;
                }
            }
        }
    };

    int sl[FT];
    bool sel[FT];
#pragma unroll
    for (int f = 0; f < FT; ++f) {
        const KxToken tok = kx_token(a.slot_of, a.rank, a.scale, a.slots, mine0 + f, a.n);
        sl[f] = tok.slot;
        if (split == 0 && blockIdx.y == 0 && threadIdx.x < 16) a.tokens[mine0 + f] = tok;
    }
    bool is_first = true;
    uint32_t leaders = 0;                                        // one token to a lane: the slots' first ones, from this workgroup's first on
    if constexpr (FT == 1) {
        leaders = kx_leaders(sl[0]);
        for (int i = 0; i < (int)blockIdx.y; ++i) leaders &= leaders - 1;
    }
    for (int index = 0;; ++index) {
        int s;
        if constexpr (FT == 1) {
            s = leaders ? __builtin_amdgcn_readlane(sl[0], __builtin_ctz(leaders ? leaders : 1u)) : -1;
            for (int i = 0; i < (int)gridDim.y; ++i) leaders &= leaders - 1;
        } else {
            s = kx_take(sl, sel);
        }
        if (s < 0 && !(GATED && is_first && blockIdx.y == 0)) break;
        if (FT > 1 && s >= 0 && index % (int)gridDim.y != (int)blockIdx.y) continue;
        const int tiles = s < 0 ? 1 : (__builtin_amdgcn_readfirstlane(a.rank[s]) + 15) / 16;
        for (int rt0 = 0; rt0 < tiles; rt0 += RG) {
            pass(s, rt0, s < 0 ? 0 : tiles - rt0, is_first);
            is_first = false;
        }
        if (s < 0) break;
    }
}

// ---- expansion in binary32 ----
// y = act(y + c_s B_s u), in place, behind the product: the sum is in binary32 either way, and y is read and written once more.
// A wavefront takes 16 rows of y and 64 tokens, four to a lane.
struct K8Expand {
    float* y;                   // [m][n]
    const KxToken* tokens;      // [n]
    const float* u;             // [splits][kx_share], kx_at
    const float* operands;      // [slot][m][rank_pad]
    int64_t slot_elems, split_elems;
    int32_t m, n, splits, rank_pad, relu;
};
__device__ __forceinline__ void k8_expand_tile(const K8Expand& a, int token_tile) {
    const int lane = (int)(threadIdx.x & 63u), wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int c = lane & 15, g = lane >> 4;
    const int row0 = ((int)blockIdx.x * 4 + wave) * 16, t0 = token_tile * 64 + c * 4, left = a.n - t0;
    if (row0 >= a.m) return;
    KxToken tok[4];
    bool any = false;
#pragma unroll
    for (int f = 0; f < 4; ++f) {
        tok[f] = KxToken{-1, 0, 0.0f, 0};
        if (f < left) tok[f] = a.tokens[t0 + f];
        any = any || tok[f].slot >= 0;
    }
    k8_any<float, 4> y[4];                                       // [row][token]
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = k8_load<float, 4>(a.y + (int64_t)(row0 + 4 * g + i) * a.n + t0, row0 + 4 * g + i < a.m ? left : 0);
    if (!a.relu && __builtin_amdgcn_ballot_w64(any) == 0) return;
    const float* ops0 = a.operands + (int64_t)(row0 + c) * a.rank_pad + 4 * g;
    for (int r0 = 0; r0 < a.rank_pad; r0 += 16) {
        // every lane its own tokens' u, whatever their slots; then slot by slot
        k8_f4 w[4], v[kAdapterMaxShares][4];
#pragma unroll
        for (int b = 0; b < kAdapterMaxShares; ++b)
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                v[b][f] = k8_f4(0.0f);
                if (b < a.splits && f < left) v[b][f] = *reinterpret_cast<const k8_f4*>(a.u + b * a.split_elems + kx_at(t0 + f, r0 + 4 * g, a.rank_pad));
            }
#pragma unroll
        for (int f = 0; f < 4; ++f) w[f] = v[0][f] + v[1][f] + v[2][f] + v[3][f];
        int sl[4];
        bool sel[4];
#pragma unroll
        for (int f = 0; f < 4; ++f) sl[f] = tok[f].rank > r0 ? tok[f].slot : -1;
        for (;;) {
            const int s = kx_take(sl, sel);
            if (s < 0) break;
            k8_f4 op = k8_f4(0.0f);
            if (row0 + c < a.m) op = *reinterpret_cast<const k8_f4*>(ops0 + s * a.slot_elems + r0);
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                k8_f4 acc = k8_f4(0.0f);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(op[i], w[f][i], acc, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) y[i][f] = sel[f] ? __builtin_fmaf(acc[i], tok[f].factor, y[i][f]) : y[i][f];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int f = 0; f < 4; ++f)
            if (a.relu) y[i][f] = y[i][f] > 0.0f ? y[i][f] : 0.0f;
        k8_store<float, 4>(a.y + (int64_t)(row0 + 4 * g + i) * a.n + t0, row0 + 4 * g + i < a.m ? left : 0, y[i]);
    }
}
// The same for 16 tokens, one to a lane, which name 16 slots at most: a workgroup takes 16 rows, and its wavefronts deal the ranks out among
// them, 16 at a time, then the slots; what each adds up is joined through LDS in order.  B of kExpandAhead slots is on its way at a time: slot by
// slot, each waiting for its B, 64 tokens of 64 slots of rank 128 took 350 us, 12 here.
constexpr int kExpandAhead = 8;
__device__ __forceinline__ void k8_expand_few_tile(const K8Expand& a, int token_tile, k8_f4* red) {
    const int lane = (int)(threadIdx.x & 63u), wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int c = lane & 15, g = lane >> 4;
    const int row0 = (int)blockIdx.x * 16, t = token_tile * 16 + c;
    KxToken tok = {-1, 0, 0.0f, 0};
    if (t < a.n) tok = a.tokens[t];
    float* y = a.y + (int64_t)(row0 + 4 * g) * a.n + t;
    float old[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        old[i] = 0.0f;
        if (wave == 0 && t < a.n && row0 + 4 * g + i < a.m) old[i] = y[(int64_t)i * a.n];
    }
    const uint32_t leaders = kx_leaders(tok.slot);
    if (!a.relu && leaders == 0) return;
    const int tiles = a.rank_pad / 16, row = min(row0 + c, a.m - 1);
    int by_chunk = 1;
    while (by_chunk < kExpandWaves && 2 * by_chunk <= tiles) by_chunk *= 2;
    const int my_slot = wave / by_chunk, by_slot = kExpandWaves / by_chunk;
    const float* ops0 = a.operands + (int64_t)row * a.rank_pad + 4 * g;
    const int tu = min(t, a.n - 1);
    k8_f4 sum = k8_f4(0.0f);
    for (int chunk = wave % by_chunk; chunk < tiles; chunk += by_chunk) {
        uint32_t left = leaders & (uint32_t)__builtin_amdgcn_ballot_w64(tok.rank > chunk * 16);
        for (int i = 0; i < my_slot; ++i) left &= left - 1;
        if (left == 0) continue;
        k8_f4 v[kAdapterMaxShares], op[kExpandAhead];
#pragma unroll
        for (int b = 0; b < kAdapterMaxShares; ++b)
            v[b] = *reinterpret_cast<const k8_f4*>(a.u + (b < a.splits ? b : 0) * a.split_elems + kx_at(tu, chunk * 16 + 4 * g, a.rank_pad));
        k8_f4 w = v[0];
        bool first = true;
        while (left) {
            int slot[kExpandAhead];
#pragma unroll
            for (int d = 0; d < kExpandAhead; ++d) {
                slot[d] = left ? __builtin_amdgcn_readlane(tok.slot, __builtin_ctz(left)) : -1;
                for (int i = 0; i < by_slot; ++i) left &= left - 1;
                op[d] = *reinterpret_cast<const k8_f4*>(ops0 + (slot[d] < 0 ? slot[0] : slot[d]) * a.slot_elems + chunk * 16);
            }
            if (first) {
#pragma unroll
                for (int b = 1; b < kAdapterMaxShares; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] += b < a.splits ? v[b][i] : 0.0f;
                first = false;
            }
#pragma unroll
            for (int d = 0; d < kExpandAhead; ++d) {
                if (slot[d] < 0) break;
                k8_f4 acc = k8_f4(0.0f);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(op[d][i], w[i], acc, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[i] = tok.slot == slot[d] ? __builtin_fmaf(acc[i], tok.factor, sum[i]) : sum[i];
            }
        }
    }
    __syncthreads();                                             // what was there has been read
    red[wave * 64 + lane] = sum;
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int w = 1; w < kExpandWaves; ++w) sum += red[w * 64 + lane];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float v = old[i] + sum[i];
        if (a.relu) v = v > 0.0f ? v : 0.0f;
        if (t < a.n && row0 + 4 * g + i < a.m) y[(int64_t)i * a.n] = v;
    }
}
__global__ __launch_bounds__(64 * kExpandWaves) void k8_expand_few(const K8Expand a) {
    __shared__ k8_f4 red[kExpandWaves * 64];
    for (int tile = (int)blockIdx.y; tile * 16 < a.n; tile += (int)gridDim.y) k8_expand_few_tile(a, tile, red);
}
__global__ __launch_bounds__(256) void k8_expand_f32(const K8Expand a) {
    for (int tile = (int)blockIdx.y; tile * 64 < a.n; tile += (int)gridDim.y) k8_expand_tile(a, tile);
}

// ---- gradients of A and B ----
// G[p][j] = c_s sum over the tokens t of slot s of z[p][t] w[t][j], with z = x and w = v for A, z = g and w = u for B.
//
// Both operands have the tokens, the reduction, next to each other: 16 bytes of a row of z come straight from memory in the order the
// matrix instruction wants.  w is small and wanted by every 16 rows of z: k8_turn brings it into operand order once, slot by slot and block
// of 128 tokens by block, with zeros for the tokens of other slots; blocks without one of the slot's are passed over.  In binary16 it is in
// two parts, hi and lo, after a power of two taken out for each rank and block; x in 8 bits is exact in binary16, and its power of
// two for each row and block joins the other when a block's sum is added to the whole.

// What k8_turn leaves, for each slot listed and side (v, u) and block.  Rank and factor are those that the projection found, which its tokens'
// records name: of other ranks nothing stands in v and u, whatever has been loaded into the slot since.
struct K8Mask {
    uint64_t half[2];           // which of a block's 128 tokens are the slot's
    int32_t rank;               // 0: none is
    float factor;
    int32_t unused[2];
};
// and what k8_grad leaves for k8_grad_join
struct K8Slot {
    int32_t rank;               // 0: nothing was found
    float factor;
    int32_t unused[2];
};
struct K8Turned {
    K8Slot* slots;              // [count][2: v, u]
    K8Mask* masks;              // [count][2][blocks]
    void* w;                    // [count][2: v, u][blocks][rank tile][4][parts][64 lanes][8]
    float* down;                // [count][2][blocks][rank_pad]: undoes the power of two
};
template <typename T> constexpr int kK8Parts = sizeof(T) == 2 ? 2 : 1;

struct K8Turn {
    K8Turned out;
    const KxToken* tokens[2];   // v's, u's: [n]
    const float* w[2];          // v, u: [splits][kx_share], kx_at
    const int32_t* slot_of;
    const int32_t* which;
    int32_t n, blocks, rank_pad, splits[2];
    int32_t x_is_act8;          // v's tokens in the order in which lanes take 32 bytes of x: see k8_grad
};

// A workgroup turns a block of a rank tile of v or u for one slot, a wavefront four of its ranks: lane 4 q + j has tokens 8 q .. of rank j.
template <typename T> __global__ __launch_bounds__(256) void k8_turn(const K8Turn a) {
    constexpr bool half = sizeof(T) == 2;
    constexpr int PARTS = kK8Parts<T>;
    const int lane = (int)(threadIdx.x & 63u), wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int tiles_all = a.rank_pad / 16;
    const int b = (int)blockIdx.x, at = (int)blockIdx.y, side = (int)blockIdx.z / tiles_all, r = (int)blockIdx.z - side * tiles_all, t0 = b * 128;
    // u of the tokens, whatever their slots: one latency for all loads.  What no token of the slot's wrote is taken out below
    const int j4 = lane & 3, q = lane >> 2;
    const int t8 = min(t0 + 8 * q, (a.n - 1) & ~7);
    const float* p = a.w[side] + kx_at(t8, r * 16 + wave * 4, a.rank_pad) + j4;      // tokens of a group of eight follow each other
    const int64_t share = kx_share(a.n, a.rank_pad);
    float v[8];
    for (int sp = 0; sp < a.splits[side]; ++sp)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float x = p[sp * share + i * 4];
            v[i] = sp ? v[i] + x : x;
        }
    const int wanted = a.which[at];
    KxToken tok[2];
    uint64_t m[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int t = t0 + h * 64 + lane;
        tok[h] = KxToken{-1, 0, 0.0f, 0};
        int32_t named = -1;
        if (t < a.n) tok[h] = a.tokens[side][t], named = a.slot_of[t];
        m[h] = __builtin_amdgcn_ballot_w64(wanted >= 0 && named == wanted && tok[h].slot == wanted);
    }
    const uint64_t m0 = m[0], m1 = m[1];
    const int first = (int)__builtin_ctzll(m0 ? m0 : (m1 ? m1 : 1));
    const bool any = (m0 | m1) != 0;
    const int rank = any ? __builtin_amdgcn_readlane(m0 ? tok[0].rank : tok[1].rank, first) : 0;
    if (r == 0 && threadIdx.x == (unsigned)first)
        a.out.masks[((int64_t)at * 2 + side) * a.blocks + b] = K8Mask{{m0, m1}, rank, any ? (m0 ? tok[0].factor : tok[1].factor) : 0.0f, {0, 0}};
    if (r * 16 >= rank) return;
    const uint32_t byte = (uint32_t)((q < 8 ? m0 : m1) >> (8 * (q & 7))) & 0xffu;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (byte >> i) & 1u ? v[i] : 0.0f;
    const int64_t part_of = ((int64_t)at * 2 + side) * a.blocks + b;
    const bool swapped = side == 0 && a.x_is_act8;
    const int step = swapped ? q & 3 : q >> 2, quarter = swapped ? q >> 2 : q & 3;       // of the 16 x 16 x 32 products; lanes of one
    k8_v8<T>* dst = static_cast<k8_v8<T>*>(a.out.w) + ((part_of * tiles_all + r) * 4 + step) * PARTS * 64 + quarter * 16 + wave * 4 + j4;
    if constexpr (half) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t bits = __builtin_bit_cast(uint32_t, v[i]) & 0x7fffffffu;
            top = bits < 0x7f800000u && bits > top ? bits : top;
        }
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
        dst[0] = hi, dst[64] = lo;
        if (q == 0) a.out.down[part_of * a.rank_pad + r * 16 + wave * 4 + j4] = kx_pow2(-shift);
    } else {
        k8_v8<T> o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = (T)v[i];
        dst[0] = o;
    }
}

struct K8Grad {
    K8Turned in;
    const void* x;              // [k][n], or int8 [k][x_pitch]
    const uint8_t* x_scale;     // [block][x_scale_pitch]
    const void* g;              // [m][n]
    float *da, *db, *work;
    int64_t x_pitch, x_scale_pitch;
    int32_t m, k, n, blocks, rank_pad, max_rank, tiles_k, count, splits;
};

// A wavefront takes 16 RW rows, the workgroup's four 64 RW, and of the blocks with a token of the slot's a share; no wavefront waits for
// another.  z of the next block is on its way while a block is multiplied.  Several shares are joined in order by k8_grad_join.
// Ranks above 64 are gone through 64 at a time, each of which reads z: 4096 + 4096 rows of one slot, 4096 tokens, rank 48 / 64 / 128 in all three
// launches 31.9 / 35.8 / 59.2 us, x in 8 bits 33.7 / 38.8 / 66.9, binary32 53.8 / 65.2 / 115.
template <typename T, int RG, int RW, bool HELD8>
__global__ __launch_bounds__(256) void k8_grad(const K8Grad a) {
    constexpr bool half = sizeof(T) == 2;
    constexpr int PARTS = kK8Parts<T>;
    const int lane = (int)(threadIdx.x & 63u), wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int c = lane & 15, g = lane >> 4;
    const bool of_a = (int)blockIdx.x < a.tiles_k;
    const int rows = of_a ? a.k : a.m;
    const int row0 = ((int)blockIdx.x - (of_a ? 0 : a.tiles_k)) * 64 * RW + wave * 16 * RW;
    if (row0 >= rows) return;
    const int at = (int)blockIdx.y, split = (int)blockIdx.z;
    const int tiles_all = a.rank_pad / 16;
    // No branch stands between z's loads.  Rows that are not there are the last one's; tokens that are not there whatever follows, up to
    // the matrix's end, and are masked.  Rows of which an eighth of a block has tokens both before and behind that end read the last block twice.
    const T* const z_all = static_cast<const T*>(of_a ? a.x : a.g);
    const int64_t z_size = (int64_t)rows * a.n;
    const T* const z_from = z_size < 8 ? static_cast<const T*>(a.in.w) : z_all;             // (too few to read eight: any memory)
    const int64_t z_room = z_size < 8 ? 8 : z_size;
    const bool z_again = !(HELD8 && of_a) && grad_reads_again(row0, 16 * RW, rows, a.n);
    const K8Mask* masks = a.in.masks + ((int64_t)at * 2 + (of_a ? 0 : 1)) * a.blocks;

    // 64 blocks at a time, one to a lane; rank and factor are in every block found: the first one's
    int rank = 0;
    float factor = 0.0f;
    auto found = [&](int group) {
        const int b = group * 64 + lane;
        K8Mask mask = {{0, 0}, 0, 0.0f, {0, 0}};
        if (b < a.blocks) mask = masks[b];
        const uint64_t some = __builtin_amdgcn_ballot_w64(mask.rank > 0);
        if (rank == 0 && some) {
            const int first = (int)__builtin_ctzll(some);
            const float f = mask.factor;
            rank = __builtin_amdgcn_readlane(mask.rank, first);
            factor = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f), first));
        }
        return some;
    };
    const int groups = (a.blocks + 63) / 64;
    const uint64_t found0 = found(0);
    int mine = 0, skip = 0;                                      // this workgroup's share of the blocks found
    int count = __builtin_popcountll(found0);
    for (int i = 1; i < groups; ++i) count += __builtin_popcountll(found(i));
    skip = (int)((int64_t)count * split / a.splits);
    mine = (int)((int64_t)count * (split + 1) / a.splits) - skip;
    if (a.splits > 1 && split == 0 && row0 == 0 && lane == 0) a.in.slots[at * 2 + (of_a ? 0 : 1)] = K8Slot{rank, factor, {0, 0}};

    for (int rt0 = 0; rt0 < tiles_all; rt0 += RG) {
        const int tiles = min((rank + 15) / 16 - rt0, RG);       // of this slot, here (none: zeros are stored)
        const int todo = tiles > 0 ? mine : 0;
        k8_f4 acc[RW][RG];
#pragma unroll
        for (int i = 0; i < RW; ++i)
#pragma unroll
            for (int r = 0; r < RG; ++r) acc[i][r] = k8_f4(0.0f);

        int group = 0;
        uint64_t left = 0;
        if (todo > 0) {
            int over = skip;
            left = found0;
            while (__builtin_popcountll(left) <= over && group + 1 < groups) over -= __builtin_popcountll(left), left = found(++group);
            for (; over > 0; --over) left &= left - 1;
        }
        // called `todo` times only; it ends, in a block that there is, also where another call writes to the scratch memory meanwhile
        auto next_block = [&]() {
            while (left == 0 && group + 1 < groups) left = found(++group);
            const int b = group * 64 + (left ? __builtin_ctzll(left) : 0);
            left &= left - 1;
            return b;
        };

        k8_any<T, 8> z[RW][4];                                   // on its way: the next block's
        uint4 z8[RW][2];
        uint32_t zs[RW];
        auto load_z = [&](int b) {
            const int tb = b * 128;
#pragma unroll
            for (int i = 0; i < RW; ++i) {
                const int row = min(row0 + i * 16 + c, rows - 1);
                if (HELD8 && of_a) {
                    // 32 bytes of a row to a lane: product st takes tokens 32 g + 8 st .., not 32 st + 8 g .. as otherwise
                    const uint4* src = reinterpret_cast<const uint4*>(static_cast<const int8_t*>(a.x) + (int64_t)row * a.x_pitch + tb + g * 32);
                    z8[i][0] = src[0], z8[i][1] = src[1];
                    const int64_t r4 = min((int64_t)(row0 + i * 16 + 4 * g), a.x_scale_pitch - 4);
                    zs[i] = *reinterpret_cast<const uint32_t*>(a.x_scale + (int64_t)b * a.x_scale_pitch + r4);
                } else {
                    const int64_t from = (int64_t)row * a.n + tb + g * 8;
#pragma unroll
                    for (int st = 0; st < 4; ++st) z[i][st] = *reinterpret_cast<const k8_any<T, 8>*>(z_from + grad_load_from(from + st * 32, z_room));
                }
            }
        };
        auto load_z_again = [&](int b) {
#pragma unroll
            for (int i = 0; i < RW; ++i) {
                const int row = min(row0 + i * 16 + c, rows - 1), t = b * 128 + g * 8;
#pragma unroll
                for (int st = 0; st < 4; ++st) z[i][st] = k8_load<T, 8>(z_all + (int64_t)row * a.n + t + st * 32, a.n - t - st * 32);
            }
        };

        int b = 0;
        if (todo > 0) b = next_block(), load_z(b);
        // (the last block has no next one: were that a condition, the wait for w would be one for the next z too)
        auto block = [&](auto last) {
            const int64_t part_of = ((int64_t)at * 2 + (of_a ? 0 : 1)) * a.blocks + b;
            const k8_v8<T>* ops = static_cast<const k8_v8<T>*>(a.in.w) + (part_of * tiles_all + rt0) * 4 * PARTS * 64 + lane;
            const float* downs = a.in.down + part_of * a.rank_pad + rt0 * 16 + c;
            // w of all rank tiles at once, or, beside two row tiles for which the registers do not suffice, of one and of the next
            constexpr int OPS = RW == 1 ? RG : 2;
            k8_v8<T> op[OPS][4][PARTS];
            float down[OPS];
#pragma unroll
            for (int r = 0; r < OPS; ++r) down[r] = 1.0f;
            auto load_op = [&](int r) {
#pragma unroll
                for (int st = 0; st < 4; ++st)
#pragma unroll
                    for (int part = 0; part < PARTS; ++part) op[r % OPS][st][part] = ops[((r * 4 + st) * PARTS + part) * 64];
                if (half) down[r % OPS] = downs[r * 16];
            };
            load_op(0);
            const uint64_t m0 = masks[b].half[0], m1 = masks[b].half[1];
#pragma unroll
            for (int r = 1; r < RG; ++r)
                if (OPS == RG && r < tiles) load_op(r);
            const bool whole = (m0 & m1) == ~0ull;
            if constexpr (decltype(last)::value) {
                if (z_again && b == a.blocks - 1) load_z_again(b);
            }
            k8_v8<T> cur[RW][4];
            float scales[RW][4];
#pragma unroll
            for (int i = 0; i < RW; ++i) {
#pragma unroll
                for (int st = 0; st < 4; ++st) {
                    if (HELD8 && of_a) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const uint4 w = z8[i][st >> 1];
                            cur[i][st][e] = (T)(float)(int8_t)((st & 1 ? (e < 4 ? w.z : w.w) : (e < 4 ? w.x : w.y)) >> (8 * (e & 3)));
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) cur[i][st][e] = z[i][st][e];
                    }
                    if (!whole) {                                // tokens of other slots: whatever z holds there, not a number even
                        const int of = HELD8 && of_a ? g * 4 + st : st * 4 + g;           // eighth of the block, of sixteen
                        const uint32_t byte = (uint32_t)((of < 8 ? m0 : m1) >> (8 * (of & 7))) & 0xffu;
#pragma unroll
                        for (int e = 0; e < 8; ++e) cur[i][st][e] = (byte >> e) & 1u ? cur[i][st][e] : (T)0.0f;
                    }
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t s = (zs[i] >> (8 * e)) & 0xffu;
                    scales[i][e] = HELD8 && of_a ? __builtin_bit_cast(float, s == 255u ? 0x7fc00000u : s << 23) : 1.0f;
                }
            }
            if constexpr (!decltype(last)::value) b = next_block(), load_z(b);
#pragma unroll
            for (int r = 0; r < RG; ++r)
                if (r < tiles) {
                    if (OPS < RG && r + 1 < tiles) load_op(r + 1);
                    k8_f4 sum[RW];
#pragma unroll
                    for (int i = 0; i < RW; ++i) sum[i] = k8_f4(0.0f);
#pragma unroll
                    for (int st = 0; st < 4; ++st)
#pragma unroll
                        for (int part = 0; part < PARTS; ++part)
#pragma unroll
                            for (int i = 0; i < RW; ++i) sum[i] = k8_mfma(cur[i][st], op[r % OPS][st][part], sum[i]);
#pragma unroll
                    for (int i = 0; i < RW; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][r][e] = __builtin_fmaf(sum[i][e] * down[r % OPS], scales[i][e], acc[i][r][e]);
                }
        };
        for (int done = 0; done + 1 < todo; ++done) block(std::false_type{});
        if (todo > 0) block(std::true_type{});
        // lane's results: rows 4 g + e, rank c
#pragma unroll
        for (int i = 0; i < RW; ++i)
#pragma unroll
            for (int r = 0; r < RG; ++r) {
                // k8_grad_join reads the ranks that the slot has, of all shares
                if (rt0 + r >= tiles_all || (a.splits > 1 && r >= tiles)) continue;
                const int j = (rt0 + r) * 16 + c, p = row0 + i * 16 + 4 * g;
                k8_any<float, 4> v;
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
    const K8Slot* slots;        // [count][2]
    const float* work;
    float *da, *db;
    int64_t wgs_a;              // workgroups of 256 values of A's gradient; B's follow
    int32_t m, k, rank_pad, max_rank, count, splits;
};
__global__ __launch_bounds__(256) void k8_grad_join(const K8Join a) {
    const int at = (int)blockIdx.y;
    const bool of_a = (int64_t)blockIdx.x < a.wgs_a;
    const int64_t first = ((int64_t)blockIdx.x - (of_a ? 0 : a.wgs_a)) * 256, o = first + threadIdx.x;
    if (o >= (int64_t)(of_a ? a.k : a.m) * a.max_rank) return;
    const int64_t per = ((int64_t)a.k + a.m) * a.rank_pad, stride = a.count * per;
    // in a share: A's [rank_pad][k], B's [m][rank_pad]
    int64_t src = o;
    int j = 0;
    if (!of_a) {
        const int64_t row = first / a.max_rank;                  // the workgroup's first row, once for all lanes
        const uint32_t off = (uint32_t)(first - row * a.max_rank) + threadIdx.x;
        j = (int)(off % (uint32_t)a.max_rank);
        src = (int64_t)a.rank_pad * a.k + (row + off / (uint32_t)a.max_rank) * a.rank_pad + j;
    }
    const float* p = a.work + at * per + src;
    const K8Slot slot = a.slots[at * 2 + (of_a ? 0 : 1)];
    const bool some = of_a ? o < (int64_t)slot.rank * a.k : j < slot.rank;
    float v[8], sum = 0.0f;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
        v[s] = 0.0f;
        if (some && s < a.splits) v[s] = p[s * stride];
    }
#pragma unroll
    for (int s = 0; s < 8; ++s) sum += v[s];
    (of_a ? a.da + (int64_t)at * a.k * a.max_rank : a.db + (int64_t)at * a.m * a.max_rank)[o] = some ? sum * slot.factor : 0.0f;
}

}  // namespace ppc
