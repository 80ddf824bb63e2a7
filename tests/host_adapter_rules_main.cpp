// The adapters' and the 8-bit activations' sizes and launch shapes on the CPU: what keeps their kernels inside their buffers.
#include <cstdint>
#include <cstdio>

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
                            const GradShape s = grad_shape(m, k, n, count, rank_pad, half != 0);
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
    return 0;
}

int main() {
    if (act8_sizes() || grad_works()) return 1;
    std::printf("ok\n");
    return 0;
}
