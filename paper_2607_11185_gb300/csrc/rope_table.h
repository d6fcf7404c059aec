// rope_table.h - size and layout of the table of angles that a block of rope_rows (rope.cu) keeps in shared memory.
// Plain C++, so that it can be checked without a GPU.
#pragma once

#include <cstddef>

namespace vcs {

constexpr int kRopeWarps = 4;
constexpr int kRopeCopies = 8;       // copies of rows whose angles a warp holds at most
constexpr int kRopeEntryBytes = 16;  // an entry: two pairs' cosines and sines

// Pairs a lane computes the angles of: the kernels are built for 1, 2 and 4, and the table's size is that of the one
// launched (96 pairs run in the kernel for 4).
constexpr int rope_lane_pairs(int pairs) { return pairs <= 32 ? 1 : pairs <= 64 ? 2 : 4; }

// First entry of a warp's copy.
template <int NP>
constexpr int rope_copy_at(int warp, int copies, int copy) {
  return (warp * copies + copy) * (NP * 16);
}
// Entry of an item's k-th two pairs within its copy; a row has `turned` items.
constexpr int rope_entry(int k, int turned, int item) { return k * turned + item; }

template <int NP>
constexpr size_t rope_table_bytes(int copies) {
  return (size_t)rope_copy_at<NP>(kRopeWarps, copies, 0) * kRopeEntryBytes;
}

}  // namespace vcs
