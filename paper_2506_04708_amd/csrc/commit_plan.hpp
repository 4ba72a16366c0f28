// commit_plan.hpp -- how stand_cache_commit's positions are shared out, the same on the host, in the kernel and in tests.
#pragma once
#include "attn_plan.hpp"

namespace stand {

constexpr int kCommitThreads = 256;

// Positions that a workgroup copies at a time: as many rows of row_words 16-byte words as make four words a thread.
STAND_BOTH int commit_per_group(int row_words) { return (1024 + row_words - 1) / row_words; }
// Workgroups of a trajectory in a layer: one for each such piece of the width, as far as a launch's dimension has threads for them
// (2^32 - 1); past that they go on by `groups` pieces at a time.  (Positions past 2^31 fit 32 bits without a sign.)
STAND_BOTH long long commit_groups(int width, int per_group)
{
    const long long pieces = (width + (long long)per_group - 1) / per_group, most = 0xFFFFFFFFll / kCommitThreads;
    return pieces < most ? pieces : most;
}
// Positions that a trajectory has, whatever its count is.
STAND_BOTH int commit_positions(int count, int width) { return count < 0 ? 0 : (count < width ? count : width); }
// Words of the piece at position j0, of n positions.  (A piece has less than 1024 words more than a row; what is left of the n is
// bounded before it is multiplied: a product with how far j0 is behind n would pass 32 bits in wide tables.)
STAND_BOTH int commit_words(int n, unsigned j0, int per_group, int row_words)
{
    if ((unsigned)n <= j0) return 0;
    const unsigned left = (unsigned)n - j0;
    return (int)(left < (unsigned)per_group ? left : (unsigned)per_group) * row_words;
}

}  // namespace stand
