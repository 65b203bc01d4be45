// Goes over sizes of packed forward launches: every form that is chosen is one of the kernels that are built (lss_fwd_bf16.hip), and all of those
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
                        const lss::PackedForm f = lss::pick_packed_form(rows, keys, B, h[0], h[1], d);
                        const std::pair<int, int> form{f.row_blocks, f.groups};
                        if (!built[d / 128].count(form)) {
                            std::printf("no kernel of %d x %d for d = %d\n", f.row_blocks, f.groups, (int)d);
                            return 1;
                        }
                        seen[d / 128].insert(form);
                    }
    if (seen[0] != built[0] || seen[1] != built[1]) {
        std::printf("a form is never chosen\n");
        return 1;
    }
    std::printf("clean\n");
    return 0;
}
