// Launches of the parameter gradients' sums over tokens, by sizes.  (Plain C++: sizes in, answers out.)
#pragma once

namespace mdn {

constexpr int kMaxSlabs = 128;

// Slabs of tokens that workgroups of their own sum, whose sums another launch of one workgroup adds up; 1: one workgroup, one launch.
// About as many slabs as a slab has tokens, so that either launch's workgroups have as much to do (4 096 heads, 4 tokens: 11.9 us, as 128
// slabs whatever the tokens 90).  Front end's backward of heads of 64 in us, one workgroup / slabs, 4 096 rows 12.0 / 15.0 and then
//   16 heads      16 384 12.1 / 15.1    24 576 14.1 / 15.0    32 768 16.8 / 15.2    65 536 29.4 / 22.2   131 072 49.3 / 31.0
//   4             16 384 13.8 / 16.6    24 576 16.2 / 17.7    32 768 18.8 / 18.7    65 536 31.7 / 25.9   131 072 51.5 / 35.2
//   512           16 384 12.2 / 15.3    24 576 13.1 / 15.1    32 768 16.0 / 15.2    65 536 28.4 / 21.6   131 072 48.3 / 31.1
// With one head or two, whose few threads add up the others' sums in either launch, later: 1 head 32 768 27.7 / 37.5, 65 536 40.2 / 44.0, 131 072
// 60.3 / 53.7; 2 heads 32 768 21.7 / 24.9, 65 536 34.3 / 31.7.  (4 096 heads: 32 768 16.3 / 19.1, 65 536 28.2 / 26.8.)
constexpr int kept_slabs(unsigned rows, int heads) {
    if (rows <= 24576 + 65536 / (unsigned)heads) return 1;
    const unsigned tokens = rows / (unsigned)heads;
    unsigned n = 1;
    while (n < kMaxSlabs && 4 * n * n <= tokens) n *= 2;
    return (int)n;
}

} // namespace mdn
