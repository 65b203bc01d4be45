// The rows of csrc/lss_starts.h on the host, for starts at the ends of 32 bits and on either side of a tensor's.
#include "lss_starts.h"

#include <climits>
#include <cstdio>
#include <initializer_list>

int main()
{
    const int starts[] = {INT_MIN, INT_MIN + 1, -5, -1, 0, 1, 7, 23, 24, 25, 60, 1 << 24, 1 << 30, INT_MAX - 1, INT_MAX};
    for (const int rows : {1, 24, 1 << 24, 1 << 30})
        for (const int start : starts)
            for (const int next : starts) {
                // rows t of the tensor with start <= t < next
                const long long from = start > 0 ? start : 0, to = next < rows ? next : rows, want = to > from ? to - from : 0;
                if (lss::rows_between(start, next, rows) != want) {
                    std::printf("%d of %d rows between %d and %d\n", lss::rows_between(start, next, rows), rows, start, next);
                    return 1;
                }
                if (lss::start_within(start, rows) < 0 || lss::start_within(start, rows) > rows) return 1;
            }
    std::printf("clean\n");
    return 0;
}
