// Sizes and launch shapes of the low-rank adapters (include/pp_adapter.h) and the layout of activations in 8 bits
// (include/pp_act8.h): plain arithmetic, shared by the library and the host tests.
#pragma once

#include <cstdint>

namespace ppc {

constexpr int kAct8Block = 128;                 // columns that share a scale
constexpr int kAdapterMaxRank = 128;
constexpr int kAdapterMaxSlots = 65536;
constexpr int kAdapterMaxTokens = 1 << 22;      // keeps every grid below 2^32 threads

inline int64_t act8_pitch(int64_t n) { return (n + kAct8Block - 1) / kAct8Block * kAct8Block; }
inline int64_t act8_scale_pitch(int64_t rows) { return (rows + 15) / 16 * 16; }
inline int64_t act8_bytes(int64_t rows, int64_t n) { return rows * act8_pitch(n) + act8_pitch(n) / kAct8Block * act8_scale_pitch(rows); }

inline int adapter_rank_pad(int max_rank) { return (max_rank + 15) / 16 * 16; }

// Elements of one slot's matrix (a rank x width one, or its transpose) in the two orders kept of it:
// for projections [rank / 16][width / 32][64 lanes][8], for expansions (binary16) [width / 64][rank / 16][2][64 lanes][8] or
// (binary32) [width][rank].
inline int64_t adapter_project_elems(int width, int rank_pad) { return (int64_t)(rank_pad / 16) * ((width + 31) / 32) * 512; }
inline int64_t adapter_expand_elems(int width, int rank_pad, bool half) {
    return half ? (int64_t)((width + 63) / 64) * (rank_pad / 16) * 1024 : (int64_t)width * rank_pad;
}

// A projection (u = A x): a workgroup takes 16 ft tokens, one of `splits` shares of the rows of x, whose sums are kept apart and
// added by whoever reads u, and every `subsets`-th of the slots that its tokens name.  Splits follow from the sizes alone, since they are
// part of u's layout.
struct ProjectShape {
    int ft, waves, tiles, splits;
};
inline ProjectShape project_shape(int rows, int n) {
    ProjectShape s;
    s.waves = 8;
    s.ft = n <= 256 ? 1 : (n <= 1024 ? 2 : 4);
    s.tiles = (n + 16 * s.ft - 1) / (16 * s.ft);
    const int steps = (rows + 31) / 32, most = (steps + 2 * s.waves - 1) / (2 * s.waves);
    const int want = 256 / s.tiles;
    s.splits = want < 1 ? 1 : want;
    if (s.splits > most) s.splits = most;
    if (s.splits > 16) s.splits = 16;
    return s;
}
inline int project_subsets(const ProjectShape& s, int slots) {
    int z = 512 / (s.tiles * s.splits);
    const int most = slots < 16 * s.ft ? slots : 16 * s.ft;
    if (z > most) z = most;
    return z < 1 ? 1 : z;
}
inline int64_t adapter_state_bytes(int rows, int n, int rank_pad) { return (int64_t)project_shape(rows, n).splits * n * rank_pad * 4; }

// The gradients of A (k rows of x) and B (m rows of g): a workgroup takes 64 rw rows of one of them and one of `splits` shares of the
// blocks of 128 tokens.
struct GradShape {
    int rw, tiles_k, tiles_m, splits;
};
inline GradShape grad_shape(int m, int k, int n, int count, int rank_pad) {
    GradShape s;
    s.rw = rank_pad <= 16 ? 4 : 2;
    s.tiles_k = (k + 64 * s.rw - 1) / (64 * s.rw);
    s.tiles_m = (m + 64 * s.rw - 1) / (64 * s.rw);
    const int64_t blocks = (n + kAct8Block - 1) / kAct8Block, wgs = (int64_t)(s.tiles_k + s.tiles_m) * count;
    int64_t w = 512 / wgs;
    if (w > blocks) w = blocks;
    if (w > 16) w = 16;
    s.splits = w < 1 ? 1 : (int)w;
    return s;
}
inline int64_t adapter_work_bytes(int m, int k, int n, int count, int rank_pad) {
    const GradShape s = grad_shape(m, k, n, count, rank_pad);
    return s.splits == 1 ? 16 : (int64_t)s.splits * count * ((int64_t)m + k) * rank_pad * 4;
}

}  // namespace ppc
