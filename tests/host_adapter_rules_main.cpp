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

int main() {
    if (act8_sizes()) return 1;
    std::printf("ok\n");
    return 0;
}
