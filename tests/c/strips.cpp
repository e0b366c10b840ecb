// Host-only test of the loops over strips (strips.h): every number once and in order, up to the largest int, in
// a build where an int that overflows ends the program. Exit status 0 on success.
#include <climits>
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

#include "strips.h"

static long failures = 0;

template <int L>
static void check(int first, int end) {
    long long next = first;
    int strips = 0;
    trivance::for_strips<L>(first, end, [&](int at, int here) {
        if (++strips > 100) std::exit(2);  // it would go on for ever
        const bool last = end - at <= L;
        if (at != next || here < 1 || (last ? here != end - at : here != L)) ++failures;
        next = (long long)at + here;
    });
    if (next != (end > first ? end : first)) ++failures;
}

template <int L>
static void all() {
    for (int end : {0, 1, L - 1, L, L + 1, 3 * L - 1, INT_MAX, INT_MAX - 1, INT_MAX - L + 1, INT_MAX - L, INT_MAX - L - 1})
        for (int before : {0, 1, 2, L - 1, L, L + 1, 5 * L, 5 * L + 3})
            if (before <= end) check<L>(end - before, end);
    check<L>(INT_MAX, 5);
}

int main() {
    all<1>(), all<2>(), all<4>(), all<8>(), all<16>(), all<32>(), all<64>();
    if (failures == 0) std::printf("strips ok\n");
    return failures == 0 ? 0 : 1;
}
