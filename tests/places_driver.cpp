// Compares share_memory() of csrc/places.h with the sets of bytes themselves, over random small operands: prints "pairs sharing".
#include <cstdio>
#include <cstdlib>
#include <random>
#include <set>

#include "../paper_2009_05766_amd/csrc/places.h"

using netmax::Place;

struct Lattice { int64_t p, size, batch, rows, cols, ld, step; };

static std::set<int64_t> bytes_of(const Lattice &l)
{
    std::set<int64_t> s;
    for (int64_t b = 0; b < l.batch; ++b)
        for (int64_t r = 0; r < l.rows; ++r)
            for (int64_t c = 0; c < l.cols * l.size; ++c) s.insert(l.p + (b * l.step + r * l.ld) * l.size + c);
    return s;
}

int main()
{
    std::mt19937 g(1);
    const auto any = [&](int64_t lo, int64_t hi) { return lo + (int64_t)(g() % (uint64_t)(hi - lo + 1)); };
    int64_t sharing = 0, pairs = 0;
    for (; pairs < 200000; ++pairs) {
        Lattice l[2];
        const int64_t ld = any(1, 12), step = any(0, 40), size = any(0, 1) ? 4 : 2;
        for (Lattice &o : l) {
            o.size = size;
            o.batch = any(0, 4); o.rows = any(0, 5); o.cols = any(0, 6);
            o.ld = any(0, 2) ? ld : any(1, 12);
            o.step = any(0, 2) ? step : any(0, 40);
            if (any(0, 5) == 0) o.ld = o.cols;                      // dense rows
            if (any(0, 5) == 0) o.step = o.rows * o.ld;             // dense matrices
            if (o.ld < o.cols) o.ld = o.cols;                       // what the checks before admit
            o.p = 4096 + any(0, 60) * size;
        }
        const std::set<int64_t> a = bytes_of(l[0]), b = bytes_of(l[1]);
        bool want = false;
        for (int64_t at : a) want = want || b.count(at);
        const auto place = [](const Lattice &o) { return Place((const void *)(uintptr_t)o.p, o.size, o.batch, o.rows, o.cols, o.ld, o.step); };
        const Place p = place(l[0]), q = place(l[1]);
        if (netmax::share_memory(p, q) != want || netmax::share_memory(q, p) != want) {
            for (const Lattice &o : l)
                fprintf(stderr, "p %lld size %lld batch %lld rows %lld cols %lld ld %lld step %lld\n", (long long)o.p, (long long)o.size, (long long)o.batch, (long long)o.rows,
                        (long long)o.cols, (long long)o.ld, (long long)o.step);
            return 1;
        }
        sharing += want;
    }
    printf("%lld %lld\n", (long long)pairs, (long long)sharing);
    return 0;
}
