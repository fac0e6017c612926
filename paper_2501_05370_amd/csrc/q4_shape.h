// Sizes of a 4-bit matrix and of the launches on it: host arithmetic in plain C++.
#pragma once
#include <cstdint>

namespace q4 {

// Scales of an output of K inputs, one per `group` of them.  (K + group - 1 does not fit 32 bits for every group that is accepted.)
constexpr int groups_of(int K, int group) { return K / group + (K % group != 0); }

// A launch's grid times its workgroup has to stay below 2^32 threads in each dimension.
constexpr int64_t kMaxThreads = (int64_t{1} << 32) - 1;

// many_kernel: workgroups of 256 threads for one group of rows (eight XCDs take the tiles of 128 columns in turn), and how many
// groups of rows one launch holds: 2047 at least, with N = 2^20.
constexpr int many_columns(int ntiles) { return ((ntiles + 7) / 8 + 7) / 8 * 8; }
constexpr int many_groups(int ntiles) { return static_cast<int>(kMaxThreads / 256 / many_columns(ntiles)); }

// pack_kernel: workgroups of 256 threads that walk the `blocks` blocks of 64 threads' work each.
constexpr unsigned pack_grid(int64_t blocks) { return static_cast<unsigned>(blocks < (int64_t{1} << 22) ? (blocks + 3) / 4 : int64_t{1} << 20); }

}  // namespace q4
