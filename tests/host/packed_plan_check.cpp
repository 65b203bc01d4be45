// Goes over sizes of packed forward launches: splits only few rows' keys, and every bf16 form that is chosen is one of the kernels that are built (lss_fwd_bf16.hip), and all of those
// are chosen somewhere.
#include "lss_packed_plan.h"

#include <cstdio>
#include <set>
#include <utility>

int main()
{
    const std::set<std::pair<int, int>> built[2] = {{{4, 1}, {2, 1}, {2, 2}, {4, 2}, {2, 4}, {1, 4}}, {{4, 1}, {8, 1}, {4, 2}, {2, 2}}};
    std::set<std::pair<int, int>> seen[2];
    const int64_t heads[][2] = {{1, 1}, {8, 8}, {8, 1}, {16, 4}, {32, 8}, {64, 64}, {65535, 1}};
    for (int64_t B = 1; B <= (int64_t)1 << 24; B = B * 3 + 1)
        for (int64_t rows = 1; rows <= (int64_t)1 << 30; rows = rows * 5 / 3 + 1)
            for (int64_t keys = 0; keys <= (int64_t)1 << 30; keys = keys * 7 / 3 + 1)
                for (const auto &h : heads)
                    for (int64_t d = 64; d <= 128; d += 64) {
                        const lss::PackedPlan f = lss::pick_packed_plan(rows, keys, B, h[0], h[1], d, 2);
                        const std::pair<int, int> form{f.row_blocks, f.groups};
                        if (!built[d / 128].count(form)) {
                            std::printf("no kernel of %d x %d for d = %d\n", f.row_blocks, f.groups, (int)d);
                            return 1;
                        }
                        seen[d / 128].insert(form);
                        const lss::PackedPlan g = lss::pick_packed_plan(rows, keys, B, h[0], h[1], d, 4);
                        for (const int splits : {f.splits, g.splits})       // (a lane each in the joining launch; none where rows alone fill the chip)
                            if (splits < 1 || splits > 16 || (splits > 1 && rows * (h[0] / h[1]) * h[1] > 800 * 128)) {
                                std::printf("%d splits of %lld rows\n", splits, (long long)rows);
                                return 1;
                            }
                    }
    if (seen[0] != built[0] || seen[1] != built[1]) {
        std::printf("a form is never chosen\n");
        return 1;
    }
    std::printf("clean\n");
    return 0;
}
