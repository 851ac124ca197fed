// Host check of the paged cache's index arithmetic (the same inline functions
// the kernels use): prints one line per case for the test to compare with
// exact arithmetic.
#include <cstdio>
#include <cstdint>
#include <vector>

#include "rr_paged.hpp"

static uint64_t next(uint64_t &s)
{
    s ^= s << 13;
    s ^= s >> 7;
    s ^= s << 17;
    return s;
}

int main()
{
    uint64_t s = 0x9E3779B97F4A7C15ull;
    const int32_t top = 0x7fffffff;
    std::vector<int32_t> pages = {1, 2, 3, 5, 7, 16, 48, 64, 100, 255, 256, 257, 65535, 65536, 65537, 1 << 30, (1 << 30) + 1, top};
    for (int i = 0; i < 200; ++i) pages.push_back((int32_t)(next(s) >> (33 + next(s) % 30)) + 1);
    for (int32_t p : pages) {
        const rr::PageDiv d = rr::page_div(p);
        std::vector<int32_t> ns = {0, 1, p - 1, p, top, top - 1};
        if (p < top) ns.push_back(p + 1);
        const int32_t m = top / p * p;  // the last multiple
        ns.push_back(m);
        ns.push_back(m - 1);
        for (int i = 0; i < 40; ++i) ns.push_back((int32_t)(next(s) >> (33 + next(s) % 31)));
        for (int32_t n : ns) std::printf("div %d %d %d\n", n, p, d.div(n));
    }
    const int32_t ids[] = {-2147483647 - 1, -1, 0, 1, 9, 10, 11, top};
    for (int32_t id : ids) std::printf("page %d 10 %d\n", id, rr::pool_page(id, 10));
    for (int i = 0; i < 200; ++i) {
        const int32_t phys = (int32_t)(next(s) % 100000), kv = 1 + (int32_t)(next(s) % 128), g = (int32_t)(next(s) % kv);
        const int32_t page = 1 + (int32_t)(next(s) % 4096), place = (int32_t)(next(s) % page), d = 8 * (1 + (int32_t)(next(s) % 128));
        std::printf("row %d %d %d %d %d %d %lld\n", phys, kv, g, page, place, d,
                    (long long)rr::pool_row(phys, kv, g, page, place, d));
    }
    const int32_t lens[] = {-2147483647 - 1, -1, 0, 1, 63, 64, 65, top};
    for (int32_t n : lens) std::printf("held %d 64 %d\n", n, rr::held_tokens(n, 64));
    // token -> sequence, empty sequences among them; then starts that do not ascend: any answer within bounds
    for (int r = 0; r < 300; ++r) {
        const int32_t B = 1 + (int32_t)(next(s) % 9);
        std::vector<int32_t> st(B + 1, 0);
        for (int b = 0; b < B; ++b) st[b + 1] = st[b] + (int32_t)(next(s) % 4);
        for (int32_t i = 0; i < st[B] + 2; ++i) {
            std::printf("seq %d", i);
            std::printf(" %d |", rr::sequence_of(st.data(), B, i));
            for (int32_t v : st) std::printf(" %d", v);
            std::printf("\n");
        }
        for (int32_t &v : st) v = (int32_t)(next(s) % 20) - 5;
        for (int32_t i = 0; i < 20; ++i) {
            const int32_t b = rr::sequence_of(st.data(), B, i);
            if (b < -1 || b >= B) {
                std::printf("out of bounds\n");
                return 1;
            }
        }
    }
    std::printf("paged driver ok\n");
    return 0;
}
