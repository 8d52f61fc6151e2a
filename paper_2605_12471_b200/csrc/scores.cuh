// What the kernels of scored steps share: the rows a token sees, and the cap on a score (kvf_scores).
#pragma once
#include <limits.h>

#include "kvfold_internal.h"

namespace kvf {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

struct RowRange {
    int64_t begin, end;              // begin >= end: nothing
};
// Rows that token `tok` of a chunk sees of the L rows there are (P of them before the chunk); `at` is its place in the arrays.  Entries
// out of range mean the nearest row there is.
__device__ __forceinline__ RowRange seen_rows(const ScoreMods &m, int64_t at, int tok, int64_t P, int64_t L, int self_rows) {
    RowRange r;
    r.begin = m.first ? (int64_t)max(m.first[at], 0) : 0;
    r.end = m.end ? min((int64_t)max(m.end[at], 0), L) : P + (int64_t)(tok + 1) * self_rows;
    return r;
}

}  // namespace
}  // namespace kvf
