// The adapters' and the 8-bit activations' sizes and launch shapes on the CPU: what keeps their kernels inside their buffers.
#include <cstdint>
#include <cstdio>
#include <vector>

#include "adapter_rules.hpp"

using namespace ppc;

static int fail(const char* what, long a, long b, long c) {
    std::printf("FAIL %s %ld %ld %ld\n", what, a, b, c);
    return 1;
}

// Blocks, runs and units of a matrix in 8 bits cover it and no more, up to the largest sizes.
static int act8_one(int32_t rows, int32_t n) {
    constexpr int kAhead = 4;
    const Act8Shape s = act8_shape(rows, n, kAhead);
    if (s.blocks < 1 || (int64_t)s.blocks * kAct8Block < n || ((int64_t)s.blocks - 1) * kAct8Block >= n) return fail("8 bits: blocks", rows, n, s.blocks);
    if ((int64_t)s.runs * kAhead < s.blocks || ((int64_t)s.runs - 1) * kAhead >= s.blocks) return fail("8 bits: runs", rows, n, s.runs);
    if (s.units != (int64_t)rows * s.runs) return fail("8 bits: units", rows, n, (long)s.units);
    if (s.wgs < 1 || s.wgs > (1u << 20) || ((int64_t)s.wgs * 16 < s.units && s.wgs != (1u << 20))) return fail("8 bits: workgroups", rows, n, s.wgs);
    const int64_t q = (int64_t)rows * act8_pitch(n), scales = (int64_t)s.blocks * act8_scale_pitch(rows);
    if (act8_pitch(n) != (int64_t)s.blocks * kAct8Block || act8_scale_pitch(rows) < rows || act8_scale_pitch(rows) % 16) return fail("8 bits: pitches", rows, n, 0);
    if (act8_bytes(rows, n) != q + scales || q % 16) return fail("8 bits: bytes", rows, n, 0);
    return 0;
}
static int act8_sizes() {
    constexpr int32_t kMost = 2147483647;
    for (int32_t rows = 1; rows <= 40; ++rows)
        for (int32_t n = 1; n <= 1300; ++n)
            if (act8_one(rows, n)) return 1;
    for (int32_t less = 0; less < 300; ++less)
        for (int32_t rows = 1; rows <= 3; ++rows)
            if (act8_one(rows, kMost / rows - less) || act8_one(kMost / rows - less, rows)) return 1;
    return 0;
}

// Scratch memory of the gradients: regions one behind the other, on multiples of 16, and no more than the bound or one slot's.
static int grad_works() {
    const int widths[] = {1, 2, 63, 64, 65, 130, 4096, 1 << 22}, tokens[] = {1, 127, 128, 129, 4096, 20000, 1 << 22}, counts[] = {1, 2, 3, 61, 64, 500, 65535};
    for (int m : widths)
        for (int k : widths)
            for (int n : tokens)
                for (int count : counts)
                    for (int rank_pad = 16; rank_pad <= 128; rank_pad += 16)
                        for (int half = 0; half < 2; ++half) {
                            if ((int64_t)m * k >= ((int64_t)1 << 31) || (int64_t)m * n >= ((int64_t)1 << 31) || (int64_t)k * n >= ((int64_t)1 << 31)) continue;
                            for (int held = 0; held < 2; ++held) {
                                const GradShape s = grad_shape(m, k, n, count, rank_pad, half != 0, held != 0);
                                const GradWork w = grad_work(m, k, n, count, rank_pad, half != 0);
                                const int64_t blocks = (n + 127) / 128;
                                if (s.splits < 1 || s.splits > 8 || s.splits > blocks) return fail("gradients: shares", m, n, s.splits);
                                if (s.rw < 1 || s.rw > 2 || (int64_t)s.tiles_k * 64 * s.rw < k || (int64_t)s.tiles_m * 64 * s.rw < m) return fail("gradients: tiles", m, k, s.rw);
                                if (w.batch < 1 || w.batch > count) return fail("gradients: slots at a time", m, count, w.batch);
                                if (w.masks % 16 || w.w % 16 || w.down % 16 || w.sums % 16) return fail("gradients: alignment", m, n, count);
                                if (w.masks < (int64_t)w.batch * 2 * 16 || w.w - w.masks < w.batch * 2 * blocks * 32) return fail("gradients: masks", m, n, count);
                                if (w.down - w.w < w.batch * 2 * blocks * rank_pad * 512) return fail("gradients: operands", m, n, count);
                                if (w.sums - w.down < (half ? w.batch * 2 * blocks * rank_pad * 4 : 0)) return fail("gradients: powers of two", m, n, count);
                                if (w.bytes - w.sums < (s.splits > 1 ? (int64_t)s.splits * w.batch * ((int64_t)m + k) * rank_pad * 4 : 0)) return fail("gradients: sums", m, n, count);
                                if (w.batch > 1 && w.bytes > kGradWork) return fail("gradients: more than the bound", m, n, w.batch);
                                if (w.batch < count && w.bytes / w.batch * (w.batch + 1) + 1024 < kGradWork) return fail("gradients: less than would fit", m, n, w.batch);
                            }
                        }
    return 0;
}

// Projections: every token is some tile's and loaded by it, no tile loads one that is not there, the shares of the rows are nobody's twice,
// and u holds a place of its own for every token and rank.
static int projections() {
    for (int half = 0; half < 2; ++half)
        for (int of_v = 0; of_v < 2; ++of_v)
            for (int rows : {1, 31, 32, 33, 511, 512, 513, 1024, 4096, 1 << 22})
                for (int n = 1; n < 1 << 22; n = n < 4500 ? n + 1 : n * 9 / 8 + 1) {
                    if ((int64_t)rows * n >= ((int64_t)1 << 31)) break;
                    const ProjectShape s = project_shape(rows, n, half != 0, of_v != 0);
                    if (s.ft != 1 && s.ft != 2 && s.ft != 4) return fail("projection: tokens to a lane", rows, n, s.ft);
                    if (s.splits < 1 || s.splits > kAdapterMaxShares) return fail("projection: shares", rows, n, s.splits);
                    if ((int64_t)s.tiles * 16 * s.ft < n || ((int64_t)s.tiles - 1) * 16 * s.ft >= n) return fail("projection: tiles", rows, n, s.tiles);
                    if (s.ft > 1 && n < 16 * s.ft) return fail("projection: a tile of more tokens than there are", rows, n, s.ft);
                    for (int tile : {0, 1, s.tiles / 2, s.tiles - 2, s.tiles - 1}) {
                        if (tile < 0 || tile >= s.tiles) continue;
                        const int first = project_first_token(tile, n, s.ft), own = tile * 16 * s.ft;
                        if (first < 0 || first > own || (s.ft > 1 && first + 16 * s.ft > n)) return fail("projection: a tile loads past the tokens", rows, n, tile);
                        if (s.ft > 1 && first != own && tile != s.tiles - 1) return fail("projection: a tile moved that is not the last", rows, n, tile);
                        const int end = own + 16 * s.ft < n ? own + 16 * s.ft : n;
                        if (s.ft > 1 && first + 16 * s.ft < end) return fail("projection: a tile's own tokens are not loaded", rows, n, tile);
                    }
                    for (int slots : {1, 3, 64, 65536}) {
                        const int z = project_subsets(s, slots);
                        if (z < 1 || z > 16 * s.ft || z > slots) return fail("projection: slots dealt out", n, slots, z);
                    }
                    for (int rank_pad : {16, 48, 128}) {
                        const int64_t share = kx_share(n, rank_pad);
                        if (adapter_state_bytes(rows, n, rank_pad, half != 0, of_v != 0) != (int64_t)n * 16 + s.splits * share * 4) return fail("projection: bytes", rows, n, rank_pad);
                        // whole groups of eight tokens are read
                        if (kx_at(((int64_t)n - 1) | 7, rank_pad - 4, rank_pad) + 4 > share) return fail("projection: u ends early", rows, n, rank_pad);
                    }
                }
    std::vector<char> taken;
    for (int n : {1, 31, 32, 33, 100})
        for (int rank_pad = 16; rank_pad <= 128; rank_pad += 16) {
            taken.assign((size_t)kx_share(n, rank_pad), 0);
            for (int t = 0; t < n; ++t)
                for (int r = 0; r < rank_pad; r += 4)
                    for (int e = 0; e < 4; ++e)
                        if (taken[(size_t)kx_at(t, r, rank_pad) + e]++) return fail("projection: a place twice", t, r, rank_pad);
        }
    return 0;
}

// Gradients: every load of eight values ends inside the matrix, and where one is held back that has tokens, the block is read again.
static int grad_loads() {
    for (int rw = 1; rw <= 2; ++rw)
        for (int rows = 1; rows <= 70; ++rows)
            for (int n = 1; n <= 300; ++n) {
                const int64_t size = (int64_t)rows * n, room = size < 8 ? 8 : size;
                const int blocks = (n + 127) / 128;
                for (int row0 = 0; row0 < rows; row0 += 16 * rw) {
                    const bool again = grad_reads_again(row0, 16 * rw, rows, n);
                    for (int i = 0; i < 16 * rw; ++i) {
                        const int row = row0 + i < rows ? row0 + i : rows - 1;
                        for (int t = 0; t < blocks * 128; t += 8) {
                            const int64_t from = (int64_t)row * n + t, at = grad_load_from(from, room);
                            if (at < 0 || at + 8 > room) return fail("gradients: a load past the matrix", rows, n, t);
                            if (at != from && t < n && !again) return fail("gradients: tokens that are not loaded", rows, n, t);
                            if (at != from && t < n && t / 128 != blocks - 1) return fail("gradients: a block before the last", rows, n, t);
                            if (size < 8 && t < n && !again) return fail("gradients: a matrix too small to load is not read again", rows, n, t);
                        }
                    }
                }
            }
    return 0;
}

int main() {
    if (act8_sizes() || grad_works() || projections() || grad_loads()) return 1;
    std::printf("ok\n");
    return 0;
}
