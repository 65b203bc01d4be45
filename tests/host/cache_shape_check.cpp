// The sizes of csrc/lss_cache_shape.h on the host, on either side of their bounds and at the ends of 64 bits.
#include "lss_cache_shape.h"

#include <cstdio>
#include <initializer_list>

int main()
{
    for (int64_t page = 16; page <= 65536; page *= 2) {
        const int64_t most = ((int64_t)1 << 30) / page;
        const struct { int64_t pages; bool ok; } tables[] = {{1, true}, {most, true}, {most + 1, false}, {0, false}, {-1, false}, {(int64_t)1 << 30, page == 1},
                                                             {(int64_t)1 << 60, false}, {((int64_t)1 << 62) / page * 4, false}, {INT64_MAX, false}, {INT64_MIN, false}};
        for (const auto &t : tables)
            if (!lss::cache_page_ok(page) || lss::cache_table_ok(t.pages, page) != t.ok) {
                std::printf("%lld pages of %lld\n", (long long)t.pages, (long long)page);
                return 1;
            }
    }
    for (const int64_t page : {(int64_t)0, (int64_t)-16, (int64_t)1, (int64_t)8, (int64_t)17, (int64_t)48, (int64_t)131072, INT64_MAX, INT64_MIN})
        if (lss::cache_page_ok(page)) {
            std::printf("a page of %lld\n", (long long)page);
            return 1;
        }
    std::printf("clean\n");
    return 0;
}
