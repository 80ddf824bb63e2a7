// Sizes and launch shapes of the low-rank adapters (include/pp_adapter.h) and the layout of activations in 8 bits
// (include/pp_act8.h): plain arithmetic, shared by the library and the host tests.
#pragma once

#include <cstdint>

#if defined(__HIP__)
#define PP_HOST_DEVICE __host__ __device__
#else
#define PP_HOST_DEVICE
#endif

namespace ppc {

constexpr int kAct8Block = 128;                 // columns that share a scale
constexpr int kAdapterMaxRank = 128;
constexpr int kAdapterMaxSlots = 65536;
constexpr int kAdapterMaxTokens = 1 << 22;      // these two keep every grid below 2^32 threads
constexpr int kAdapterMaxRows = 1 << 22;

inline int64_t act8_pitch(int64_t n) { return (n + kAct8Block - 1) / kAct8Block * kAct8Block; }
inline int64_t act8_scale_pitch(int64_t rows) { return (rows + 15) / 16 * 16; }
inline int64_t act8_bytes(int64_t rows, int64_t n) { return rows * act8_pitch(n) + act8_pitch(n) / kAct8Block * act8_scale_pitch(rows); }

// How the rows are gone through: sixteen lanes take `ahead` blocks of a row at a time, a unit; a workgroup sixteen units.  n may be 2^31 - 1:
// rounded up it passes 31 bits.
struct Act8Shape {
    int blocks, runs;           // of a row: blocks, and units
    int64_t units;
    unsigned wgs;
};
inline Act8Shape act8_shape(int32_t rows, int32_t n, int ahead) {
    Act8Shape s;
    s.blocks = (int)(act8_pitch(n) / kAct8Block);
    s.runs = (s.blocks + ahead - 1) / ahead;
    s.units = (int64_t)rows * s.runs;
    const int64_t wgs = (s.units + 15) / 16;
    s.wgs = (unsigned)(wgs < (1 << 20) ? wgs : (1 << 20));
    return s;
}

inline int adapter_rank_pad(int max_rank) { return (max_rank + 15) / 16 * 16; }

constexpr int kAdapterLoads = 64;               // slots that one launch loads at most

// Elements of one slot's matrix (a rank x width one, or its transpose) in the two orders kept of it:
// for projections [rank / 16][width / 32][64 lanes][8], for expansions (binary16) [width / 64][rank / 16][2][64 lanes][8] or
// (binary32) [width][rank].
PP_HOST_DEVICE inline int64_t adapter_project_elems(int width, int rank_pad) { return (int64_t)(rank_pad / 16) * ((width + 31) / 32) * 512; }
PP_HOST_DEVICE inline int64_t adapter_expand_elems(int width, int rank_pad, bool half) {
    return half ? (int64_t)((width + 63) / 64) * (rank_pad / 16) * 1024 : (int64_t)width * rank_pad;
}

// A projection (u = A x, or v = B^T g): a workgroup takes 16 ft tokens and one of `splits` shares of the rows, whose sums are kept apart and
// added by whoever reads them, and every `subsets`-th of the slots that its tokens name.  Splits follow from the sizes alone, since they
// are part of the layout of what is left.
//   ft: with one token of binary16 to a lane a row gives 32 bytes, and many tokens ask the cache for every line four times; few tokens make
//   few workgroups.  4096 rows, rank 16, 4 / 2 / 1 tokens to a lane: 4096 tokens 9.4 / 13.9 / - us, 2048 8.3 / 8.0 / 13.5, 1024
//   8.2 / 5.4 / 7.5, 512 8.2 / 5.3 / 4.8.  A value of binary32 is twice as wide: 2048 rows, rank 32, 4096 tokens 18.7 / 11.1 / -, 1024
//   18.3 / 10.1 / 7.5.  More than one to a lane only where there are more tokens than a tile has: k8_project relies on that.
//   splits: more shares fill the GPU, but the product that reads u does so once for every 64 rows of its own.  4096 x 4096, projection and
//   product less the product without adapters, 2 / 4 / 8 shares: 512 tokens of eight slots of rank 32 12.7 / 10.8 / 15.0 us, 1024 of 64
//   slots of rank 16 15.6 / 18.1 / 24.9.  v's projection may also read the gate and write g; a backward pass's whole first half: 1024
//   tokens of rank 16 49.9 / 46.2 / 48.2, 4096 85.2 / 85.2 / 92.3, of rank 64 101.6 / 116.5 / 136.2.
constexpr int kProjectWaves = 8;
constexpr int kAdapterMaxShares = 4;
struct ProjectShape {
    int ft, tiles, splits;
};
inline ProjectShape project_shape(int rows, int n, bool half, bool of_v) {
    ProjectShape s;
    const int unit = half ? 512 : 1024;
    s.ft = n <= unit ? 1 : (n <= 4 * unit ? 2 : 4);
    s.tiles = (n + 16 * s.ft - 1) / (16 * s.ft);
    s.splits = 512 / s.tiles;
    const int steps = (rows + 31) / 32, most = (steps + 2 * kProjectWaves - 1) / (2 * kProjectWaves), limit = n <= (of_v ? 1024 : 512) ? kAdapterMaxShares : 2;
    if (s.splits > most) s.splits = most;
    if (s.splits > limit) s.splits = limit;
    if (s.splits < 1) s.splits = 1;
    return s;
}
// 64 tokens with a slot of rank 16 each: 26.1 us with one subset, 9.3 with 4, 5.9 with 16.
inline int project_subsets(const ProjectShape& s, int slots) {
    int z = 512 / (s.tiles * s.splits);
    const int most = slots < 16 * s.ft ? slots : 16 * s.ft;
    if (z > most) z = most;
    return z < 1 ? 1 : z;
}
// The first token that tile `tile` loads: the last tile is moved back to end with the last token, unless a lane has one token only (its last
// lanes repeat the last one then).
PP_HOST_DEVICE inline int project_first_token(int tile, int n, int ft) {
    const int own = tile * 16 * ft;
    return ft == 1 || own < n - 16 * ft ? own : n - 16 * ft;
}

// u of 32 tokens and 16 ranks stands as the matrix instruction's lanes take it, in two planes of 16 bytes a lane: every load and store of
// it is a run of 512 bytes or more.  Laid out [token][rank] a lane's load met a line of its own: 4096 x 4096 on 4096 tokens of
// ranks up to 32 took 2 us more.  The plain offset of (token, rank), of a multiple of four ranks:
PP_HOST_DEVICE inline int64_t kx_at(int64_t token, int rank, int rank_pad) {
    return ((token >> 5) * (rank_pad >> 4) + (rank >> 4)) * 512 + ((rank >> 2) & 1) * 256 + (((rank >> 3) & 1) * 32 + (int)(token & 31)) * 4;
}
PP_HOST_DEVICE inline int64_t kx_share(int64_t n, int rank_pad) { return (n + 31) / 32 * 32 * rank_pad; }      // elements of a share
// What a projection leaves: 16 bytes for each token, then the sums, of whole groups of 32 tokens.
inline int64_t adapter_state_bytes(int rows, int n, int rank_pad, bool half, bool of_v) {
    return (int64_t)n * 16 + project_shape(rows, n, half, of_v).splits * kx_share(n, rank_pad) * 4;
}

// The expansion in binary32: 64 tokens and 16 rows to a wavefront, which goes through the tokens' slots one by one, or 16 tokens and 16 rows to
// a workgroup, whose four wavefronts share slots and ranks.  The first reads B once for four times as many tokens, the second is done
// soon where tokens name many slots, and fills the GPU where there is little to do.  The expansion alone, m x n, rank 8 / 128, first and second:
//   one slot    1024 x 1 3.4 / 12.0, 3.3 / 3.9 us   1024 x 256 3.6 / 12.7, 3.4 / 9.7   4096 x 128 4.4 / 14.5, 6.7 / 19.1   1024 x 1024 5.4 / 16, 12 / 37
//   64 slots    1024 x 64 39 / 353, 3.9 / 12.2      4096 x 128 30 / 198, 11 / 29       1024 x 1024 9.6 / 46, 14 / 36       4096 x 1024 24 / 107, 48 / 130
// and with 64 slots in no order 1024 x 1024 27 / 185, 19 / 64, 4096 x 1024 69 / 541, 63 / 244.
constexpr int kExpandWaves = 4;
inline bool expand_few(int m, int n, int slots) {
    return (int64_t)((m + 15) / 16) * ((n + 15) / 16) <= (slots > 16 ? 4096 : 1024);
}

// The gradients of A (k rows of x) and B (m rows of g): a workgroup takes 64 rw rows of one of them and one of `splits` shares of the
// blocks of 128 tokens.  Shares fill the GPU but cost a launch that joins them, 4 us.  4096 + 4096 rows of one slot, 1 / 2 / 4 / 8 shares:
// 4096 tokens 38.4 / 26.5 / 22.7 / 24.0 us, 512 10.2 / 11.2 / 11.5 / 14.2.  1024 + 4096 rows, 2000 tokens of six slots of rank 64: 29.8 /
// 35.0 / 35.4 / 44.6.  Ranks above 32 are read from the cache once for every 16 rw rows, so long sums take rw 2 where its half as many
// workgroups still fill the GPU: more of them for binary32 and for x from 8 bits, of which two row tiles leave room for one wavefront to a
// SIMD.  Rank 64, rw 1 / 2, the workgroups that rw 1 has in front (ranks 48 and 128 turn at the same places):
//                                   binary16 x    binary16, 8 bits   binary32 x    binary32, 8 bits
//   128: 4096 + 4096 rows,  4096 t  38.6 / 35.8   38.8 / 40.9        65.2 / 69.1   65.2 / 68.4 us
//        the same,         16384 t  155 / 111     115 / 106          216 / 210     212 / 221
//    80: 1024 + 4096 rows, 16384 t  84.2 / 81.6   79.7 / 101         153 / 206     143 / 192
//    32: 1024 + 1024 rows, 16384 t  42.9 / 59.1   43.0 / 60.1        63.2 / 109    63.9 / 111
//   512: 4096 + 4096, four slots    155 / 118     117 / 116          215 / 220     213 / 230
//   320: 1024 + 4096, four slots    113 / 71.4    107 / 85.3         208 / 163     197 / 152
struct GradShape {
    int rw, tiles_k, tiles_m, splits;
};
inline GradShape grad_shape(int m, int k, int n, int count, int rank_pad, bool half, bool x_is_act8) {
    GradShape s;
    const int64_t blocks = (n + kAct8Block - 1) / kAct8Block, each = (blocks + count - 1) / count;      // a slot's, if they are alike
    const int64_t small = (int64_t)((k + 63) / 64 + (m + 63) / 64) * count;
    s.rw = rank_pad > 32 && each >= 16 && small >= (half && !x_is_act8 ? 128 : 256) ? 2 : 1;
    s.tiles_k = (k + 64 * s.rw - 1) / (64 * s.rw);
    s.tiles_m = (m + 64 * s.rw - 1) / (64 * s.rw);
    const int64_t wgs = (int64_t)(s.tiles_k + s.tiles_m) * count;
    int64_t w = each <= (half ? 4 : 1) ? 1 : 512 / wgs;
    if (w > each) w = each;
    if (w > 8) w = 8;
    s.splits = w < 1 ? 1 : (int)w;
    return s;
}
// A lane loads eight values of a row of z, from `from` on, without a look at the row's end: what follows is another row's, and masked.  Only
// the matrix's end holds loads back (size: its values, eight or more).  Where that moves a load of which some tokens are there, the block
// is read again, with a look: always the last block of the tile's last rows.
PP_HOST_DEVICE inline int64_t grad_load_from(int64_t from, int64_t size) { return from < size - 8 ? from : size - 8; }
PP_HOST_DEVICE inline bool grad_reads_again(int row0, int tile_rows, int rows, int n) {
    const int last = row0 + tile_rows - 1 < rows - 1 ? row0 + tile_rows - 1 : rows - 1;
    return (int64_t)last * n + (n + 7) / 8 * 8 > (int64_t)rows * n;
}

// Scratch memory of the gradients, x as it is or in 8 bits: offsets in bytes, multiples of 16.  Every listed slot has room for all tokens in
// it, so long lists are gone through `batch` slots at a time: as many as 256 MB hold, what the last-level cache does, and one at least.
constexpr int64_t kGradWork = (int64_t)1 << 28;
struct GradWork {
    int batch;
    int64_t masks, w, down, sums, bytes;
};
inline GradWork grad_work(int m, int k, int n, int count, int rank_pad, bool half) {
    const int64_t blocks = (n + kAct8Block - 1) / kAct8Block;
    const int as_it_is = grad_shape(m, k, n, count, rank_pad, half, false).splits, held = grad_shape(m, k, n, count, rank_pad, half, true).splits;
    const int splits = as_it_is > held ? as_it_is : held;
    // of a slot: K8Slot and K8Mask for v and for u, their operands (two binary16 parts or one binary32), powers of two, shares of the sums
    const int64_t slots = 2 * 16, masks = 2 * blocks * 32, w = 2 * blocks * rank_pad * kAct8Block * 4, down = half ? 2 * blocks * rank_pad * 4 : 0,
                  sums = splits > 1 ? splits * ((int64_t)m + k) * rank_pad * 4 : 0;
    const int64_t fit = kGradWork / (slots + masks + w + down + sums);
    GradWork o;
    o.batch = fit < 1 ? 1 : (fit < count ? (int)fit : count);
    o.masks = o.batch * slots;
    o.w = o.masks + o.batch * masks;
    o.down = o.w + o.batch * w;
    o.sums = o.down + o.batch * down;
    o.bytes = o.sums + o.batch * sums;
    return o;
}

}  // namespace ppc
