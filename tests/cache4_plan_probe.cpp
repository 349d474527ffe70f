// Prints how the attention over the 4-bit cache divides the calls that stand on its standard input, one a line, for test_cache4_plan.py.
#include <cstdio>

#include "../paper_2603_08343_b200/csrc/cache4_plan.h"

int main() {
    long long n[10];  // width T B max_q_len Hq Hkv D page dtype weigh
    for (;;) {
        for (long long& v : n)
            if (std::scanf("%lld", &v) != 1) return 0;
        const auto i = [&](int k) { return static_cast<int32_t>(n[k]); };
        const wht_plan::Attend4Plan f = wht_plan::plan_attend4(i(0), n[1], i(2), i(3), i(4), i(5), i(6), i(7), i(8), n[9] != 0, 148);
        std::printf("umma=%d row_tiles=%d warps=%d grain=%d least=%d part_rows=%d ml_bytes=%zu o_bytes=%zu lse_bytes=%zu scores_bytes=%zu bytes=%zu\n", f.umma, f.row_tiles,
                    f.warps, f.grain, f.least, f.part_rows, f.ml_bytes, f.o_bytes, f.lse_bytes, f.scores_bytes, f.bytes);
    }
}
