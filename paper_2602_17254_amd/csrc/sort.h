// Stable sorts of each rank's numbers (experts of slots, vocabulary entries of tokens) by counting (sort.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "plan.h"

namespace trivance {

constexpr int kMaxBins = 4096;  // of one pass: a wave's counters of them lie in local memory

// Memory that the launches of a sort fill with zeros on the way: their workgroups leave most of the GPU and of its memory's rate unused. A
// rank's values are cut into blocks, of which a launch fills `blocks`, from the `first` on.
struct Zeros {
    float* at;
    int64_t values, rank_stride;
    int64_t first, blocks;
};

constexpr int64_t kZerosBlock = 1024;  // values: a store of each lane, as blocks of 16 took 50 us in place of 40 for 266 MB

// One pass puts each rank's keys in the order of their digit (key >> shift) & digits, those of equal digits in the order
// that they came in. Keys are a caller's numbers, of which those outside [0, bound) and those of masked tokens are
// left out, or what an earlier pass wrote.
struct SortPass {
    const void* ids;  // [ranks][slots], int32 or, where wide, int64; NULL: keys
    const uint8_t* mask;  // [ranks][tokens] or NULL: slot i is of token i / top_k
    int wide;
    FastDiv32 by_top_k;
    int64_t tokens;
    const int *keys, *order;  // [ranks][slots]: keys and the slots they came from; the first counts[r * count_stride] count
    const int* counts;
    int64_t count_stride;
    int64_t ranks, slots;
    int64_t bound;
    int shift, digits;
    int bins;  // one more than the largest digit, at most kMaxBins
    // what is written, each unless NULL
    int* places;    // [ranks][slots]: where each slot went, -1 for those left out
    int* offsets;   // [ranks][bins + 1]: the first place of each digit, then the number of keys
    int *to_keys, *to_order;  // [ranks][slots]: keys and slots in their new order; of to_order, -1 behind the last
    int* hist;      // [ranks][chunks][bins] of workspace; unused where one workgroup sorts a rank's keys
    Zeros zeros;
};

// How a pass shares out a rank's slots: to `chunks` workgroups of `waves` waves, `per` consecutive slots each.
struct SortShape {
    int waves;
    int64_t chunks, per;
};

SortShape sort_shape(int64_t ranks, int64_t slots, int bins);
int64_t sort_hist_values(int64_t ranks, int64_t slots, int bins);
int sort_launches(int64_t ranks, int64_t slots, int bins);
// Of `zeros` (first and blocks are not looked at) the launches of this pass fill the parts from `launch` on of `launches`.
int run_sort_pass(SortPass a, hipStream_t stream, int launch = 0, int launches = 0);

}  // namespace trivance
