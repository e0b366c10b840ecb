// Loops over whole numbers in strips, without HIP, so that they can be looked over without a GPU.
#pragma once

namespace trivance {

// run(at, here) for every strip of up to L of the numbers [first, end), 0 <= first, end <= 2^31 - 1. `at` goes on by what a strip
// holds: a whole strip behind the last may not fit an int.
template <int L, typename F>
__attribute__((always_inline)) constexpr void for_strips(int first, int end, F run) {
    for (int at = first; at < end;) {
        const int here = end - at < L ? end - at : L;
        run(at, here);
        at += here;
    }
}

}  // namespace trivance
