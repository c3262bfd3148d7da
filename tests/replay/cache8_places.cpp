// Reads "seqs tokens cap pages page table_cols" and the lists from standard input, and prints the place of every
// token as the kernels find it: page and offset.  Lists are kept at the end of their own allocations, and
// every read is checked, so a number that leads out of them ends the program.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "cache8.h"

struct Checked {
    std::vector<int32_t> v;
    int32_t operator[](int64_t i) const {
        if (i < 0 || i >= int64_t(v.size())) {
            std::printf("read %lld of %zu\n", (long long)i, v.size());
            std::exit(3);
        }
        return v[size_t(i)];
    }
};

int main() {
    long long seqs, tokens, pages, page, cols;
    if (std::scanf("%lld %lld %lld %lld %lld", &seqs, &tokens, &pages, &page, &cols) != 5) return 2;
    Checked starts{std::vector<int32_t>(size_t(seqs + 1))};
    std::vector<int32_t> lengths(static_cast<size_t>(seqs)), table(static_cast<size_t>(seqs * cols));
    for (auto *l : {&starts.v, &lengths, &table})
        for (auto &x : *l) {
            long long in;
            if (std::scanf("%lld", &in) != 1) return 2;
            x = int32_t(in);
        }
    ds_cache8 cache{};
    cache.pages = pages;
    cache.page = int32_t(page);
    const ds::CacheView c = ds::cache_view(&cache);
    ds_chunk chunk{starts.v.data(), lengths.data(), table.data(), seqs, cols, cols};
    const ds::ChunkView n = ds::chunk_view(&chunk, &cache, tokens);
    for (int t = 0; t < tokens; ++t) {
        const ds::Place p = ds::place_of(c, n, starts, t);
        if (p.page >= pages || p.off < 0 || p.off >= page) return 4;
        std::printf("%d %d\n", p.page, p.off);
    }
    return 0;
}
