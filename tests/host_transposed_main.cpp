// Plans of transposed weights under AddressSanitizer and UndefinedBehaviorSanitizer: sizes that no block divides, blocks larger than the
// matrix, masks that are there, one alone or not at all.  Every row tile unpacks to the transpose of the pruned weights.
#include <cstdint>
#include <cstdio>
#include <vector>

#include "block_plan.hpp"

int main() {
    using namespace ppc;
    const int sizes[] = {1, 2, 7, 16, 31, 33, 64, 65, 100}, blocks[] = {1, 3, 16, 40, 130};
    uint32_t seed = 1;
    auto next = [&] { return seed = seed * 1664525u + 1013904223u, seed >> 16; };
    int cases = 0;
    for (int m : sizes)
        for (int k : sizes)
            for (int bm : blocks)
                for (int bk : blocks)
                    for (int masks = 0; masks < 4; ++masks) {
                        const int rows = (m + bm - 1) / bm, cols = (k + bk - 1) / bk;
                        std::vector<uint8_t> rk((size_t)rows * cols * bm), ck((size_t)rows * cols * bk);
                        for (auto& v : rk) v = next() % 3 != 0;
                        for (auto& v : ck) v = next() % 3 != 0;
                        std::vector<float> w((size_t)m * k), bias((size_t)m, 1.0f);
                        for (auto& v : w) v = (float)(1 + next() % 1000);        // exact in binary16
                        pp_block_gemm_desc_t d{};
                        d.m = m, d.k = k, d.block_m = bm, d.block_k = bk;
                        d.row_keep = masks & 1 ? rk.data() : nullptr, d.col_keep = masks & 2 ? ck.data() : nullptr;
                        d.weights = w.data(), d.bias = bias.data(), d.flags = PP_FLAG_RELU | PP_FLAG_HOST_ONLY;
                        d.dtype = cases % 2 ? PP_F16 : PP_F32;
                        BlockHostPlan p;
                        if (build_block_plan_transposed(d, p) != PP_OK || !p.transposed || p.m != k || p.k != m || (p.flags & PP_FLAG_RELU)) return std::printf("FAIL plan %d\n", cases), 1;
                        for (float b : p.bias)
                            if (b != 0.0f) return std::printf("FAIL bias %d\n", cases), 1;
                        std::vector<float> tile((size_t)64 * m);
                        for (int t = 0; t < p.row_tiles; ++t) {
                            if (unpack_block_tile(p, t, tile.data()) != PP_OK) return std::printf("FAIL unpack %d\n", cases), 1;
                            for (int r = 0; r < 64; ++r)
                                for (int c = 0; c < m; ++c) {
                                    const int at = t * 64 + r;                   // row of the transpose: a column of the weights
                                    bool kept = at < k;
                                    if (kept && (masks & 1)) kept = rk[((size_t)(c / bm) * cols + at / bk) * bm + c % bm] != 0;
                                    if (kept && (masks & 2)) kept = ck[((size_t)(c / bm) * cols + at / bk) * bk + at % bk] != 0;
                                    if (tile[(size_t)r * m + c] != (kept ? w[(size_t)c * k + at] : 0.0f)) return std::printf("FAIL value %d\n", cases), 1;
                                }
                        }
                        ++cases;
                    }
    std::printf("ok %d\n", cases);
    return 0;
}
