// Which form the verification of trees takes (tree_verify.hip): all rows at once, or those on the paths in rounds.  Plain host code, with a test of its own.
//
// Both forms' times, in us, from the sizes that the host knows.  All rows at once: three launches; 6.2 ns a row for its two workgroups and more, its entries at 3 TB/s of bf16, and every
// workgroup's search through the requests for its own.  Rounds: a launch for each, 7.5 us while requests walk (taken to be four rounds) and 2.7 behind that, with a row of every
// request's at a time.  Measured, all at once | rounds (the formulas in brackets), bf16 logits, a child of three of four nodes carrying the drawn token:
//     requests x nodes, entries, max_depth
//     1 x 12, 32000, 4                 14 | 21 (14 | 38)        64 x 12, 32000, 8           33 | 41 (35 | 51)
//     16 x 48, 128256, 4               86 | 41 (84 | 40)        64 x 3, 128256, 4           29 | 37 (31 | 47)
//     256 x 48, 1000, 4                90 | 47 (100 | 41)       1000 x 48, 1000, 8         319 | 70 (375 | 62)
//     4000 x 3, 1000, 1               134 | 70 (128 | 74)       20000 x 3, 1000, 4        1594 | 376 (1226 | 308)
// Of 243 such calls (1 .. 20000 requests of 3 .. 48 nodes, 100 .. 128256 entries, depths 1, 4, 8) the rule takes the faster form, or one within 15 %, in 236, and 1.4 % more time
// than it in the mean (profiles/tree_verify_forms.txt has them all).
#pragma once

#include <stdint.h>

namespace ss {

constexpr int64_t kVerifyGroups = 1 << 23;   // workgroups of a launch, of 256 threads each

inline int64_t verify_fours(int vocab) { return ((int64_t)vocab + 4 * 2048 - 1) / (4 * 2048); }   // of blocks of a row, a workgroup's each

inline double verify_all_time(int batch, int64_t rows, int vocab) { return 13.5 + (double)rows * (0.0062 + vocab / 1.5e6 + batch / 1.5e6); }
inline double verify_rounds_time(int batch, int vocab, int max_depth)
{
    return 5.0 + 7.5 * (max_depth < 3 ? max_depth + 1 : 4) + 2.7 * (max_depth < 3 ? 0 : max_depth - 3) + batch * (vocab / 1.0e6 + 0.0125);
}

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
