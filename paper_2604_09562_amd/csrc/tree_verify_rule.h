// Which form the verification of trees takes (tree_verify.hip): all rows at once, or those on the paths in rounds.  Plain host code, with a test of its own.
#pragma once

#include <stdint.h>

namespace ss {

constexpr int64_t kVerifyGroups = 1 << 23;   // workgroups of a launch, of 256 threads each

inline int64_t verify_fours(int vocab) { return ((int64_t)vocab + 4 * 2048 - 1) / (4 * 2048); }   // of blocks of a row, a workgroup's each

// Times in us.  All rows at once: three launches, every row.  Rounds: a launch for each, those behind the fifth mostly of ended requests.
inline double verify_all_time(int /*batch*/, int64_t rows, int vocab) { return 11.0 + (double)rows * vocab / 1.1e6; }
inline double verify_rounds_time(int /*batch*/, int /*vocab*/, int max_depth) { return 8.0 + 10.0 * (max_depth < 4 ? max_depth + 1 : 5) + 3.0 * (max_depth < 4 ? 0 : max_depth - 4); }

// Whether all rows at once are the faster form.
inline bool verify_all_rows(int batch, int64_t rows, int vocab, int max_depth)
{
    if (rows * verify_fours(vocab) >= kVerifyGroups) return false;   // (more than a launch takes)
    return verify_all_time(batch, rows, vocab) <= verify_rounds_time(batch, vocab, max_depth);
}

// The most rows that calls of this size take at once, whatever their max_depth (deepest: the largest there is, with which it is most).
inline int64_t verify_most_rows(int batch, int vocab, int deepest)
{
    int64_t lo = -1, hi = kVerifyGroups;   // the times grow with the rows: between one that is taken and one that is not
    while (hi - lo > 1) {
        const int64_t mid = (lo + hi) / 2;
        if (verify_all_rows(batch, mid, vocab, deepest)) lo = mid; else hi = mid;
    }
    return lo < 0 ? 0 : lo;
}

}  // namespace ss
