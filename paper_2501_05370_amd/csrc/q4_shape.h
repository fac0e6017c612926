// Sizes of a 4-bit matrix and of the launches on it: host arithmetic in plain C++.
#pragma once

namespace q4 {

// Scales of an output of K inputs, one per `group` of them.  (K + group - 1 does not fit 32 bits for every group that is accepted.)
constexpr int groups_of(int K, int group) { return K / group + (K % group != 0); }

}  // namespace q4
