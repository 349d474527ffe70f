// Prints how the serving attention divides the calls that stand on its standard input, one a line, for test_attention_plan.py.
#include <cstdio>
#include <cstring>

#include "../paper_2603_08343_b200/csrc/attn_plan.h"

int main() {
    char kind[16];
    long long n[11];
    while (std::scanf("%15s", kind) == 1) {
        for (long long& v : n)
            if (std::scanf("%lld", &v) != 1) return 2;
        const auto i = [&](int k) { return static_cast<int32_t>(n[k]); };
        if (!std::strcmp(kind, "prefix")) {  // prefix_len width T B max_q_len Hq Hkv D page dtype tcgen05
            const wht_plan::PrefixPlan f = wht_plan::plan_prefix(n[0], i(1), n[2], i(3), i(4), i(5), i(6), i(7), i(8), i(9), n[10] != 0, 148);
            std::printf("joint=%d umma=%d umma_splits=%d prefix_wpu=%d prefix_splits=%d own_wpu=%d own_splits=%d parts=%d bytes=%zu\n", f.joint, f.umma,
                        f.umma_splits, f.prefix_wpu, f.prefix_splits, f.own_wpu, f.own_splits, f.parts, f.bytes);
        } else {  // width select T B max_q_len Hq Hkv D page dtype -
            const wht_plan::SelectPlan f = wht_plan::plan_select(i(0), i(1), n[2], i(3), i(4), i(5), i(6), i(7), i(8), i(9), 148);
            std::printf("wpu=%d splits=%d one_kernel=%d scores_bytes=%zu bytes=%zu\n", f.wpu, f.splits, f.one_kernel, f.scores_bytes, f.bytes);
        }
        std::fflush(stdout);
    }
}
