// Prints, for matrices "batch rows cols" in lines of the input, which kernels a call takes and whether
// what it launches fits the indexes and the padding that the kernels assume.
#include <cstdio>

#include "orthogonalize_plan.h"

using namespace trivance;

static void print(const char* what, const ProductForm& f) {
    printf(" %s-%d%s%s", what, f.tile, f.few ? "few" : "", f.workers ? "-shared" : "");
}

int main() {
    long long b, r, c;
    while (scanf("%lld %lld %lld", &b, &r, &c) == 3) {
        const int64_t m = r < c ? r : c, n = r < c ? c : r;
        printf("%lld %lld %lld", b, r, c);
        if (m <= kSmallSide && n <= kSmallLong) {
            printf(" small\n");
            continue;
        }
        if (m <= kSmallSide && n <= kSmallLong * kMostStrips) {
            printf(" strips\n");
            continue;
        }
        const Tiles t = tiles_of(b, m, n);
        const int64_t pm = padded(m, t.pad()), pn = padded(n, t.pad());
        const ProductForm gram = form_of(b, pm, pm, pn, t.symmetric, true),
                          square = form_of(b, pm, pm, pm, t.symmetric, true),
                          update = form_of(b, pm, pn, pm, t.update, false);
        print("gram", gram);
        print("polynomial", square);
        print("update", update);
        const ProductForm forms[3] = {gram, square, update};
        for (int i = 0; i < 3; ++i) {
            const ProductForm& f = forms[i];
            const int64_t depth = i == 0 ? pn : pm;
            if (f.workers && (f.workers > f.tiles * (depth / 64) || f.workers > kMostWorkers)) printf(" WORKERS");
            if (f.workers && f.tiles * (depth / 64) > INT32_MAX / 2) printf(" STAGES");
            if (f.tiles > UINT32_MAX / 512) printf(" GRID");  // 512 threads at most
        }
        printf("\n");
    }
}
