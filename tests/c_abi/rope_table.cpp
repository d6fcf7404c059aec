// What the rotation's launch asks for and what its kernel reaches, of every rotated size: a line
// "rot interleaved copies bytes reached", in bytes of shared memory.
#include <cstdio>

#include "rope_table.h"

template <int NP>
void line(int rot, bool inter, int copies) {
  const int turned = inter ? rot / 8 : rot / 16, two_pairs = inter ? 2 : 4;  // items of a row, entries of an item
  int last = 0;
  for (int warp = 0; warp < vcs::kRopeWarps; ++warp)
    for (int copy = 0; copy < copies; ++copy)
      for (int k = 0; k < two_pairs; ++k)
        for (int item = 0; item < turned; ++item) {
          const int at = vcs::rope_copy_at<NP>(warp, copies, copy) + vcs::rope_entry(k, turned, item);
          last = at > last ? at : last;
        }
  std::printf("%d %d %d %zu %d\n", rot, inter, copies, vcs::rope_table_bytes<NP>(copies),
              (last + 1) * vcs::kRopeEntryBytes);
}

int main() {
  for (int rot = 16; rot <= 256; rot += 16)
    for (int inter = 0; inter < 2; ++inter)
      for (int copies = 1; copies <= vcs::kRopeCopies; ++copies) {
        const int np = vcs::rope_lane_pairs(rot / 2);
        if (np == 1) line<1>(rot, inter, copies);
        else if (np == 2) line<2>(rot, inter, copies);
        else if (np == 4) line<4>(rot, inter, copies);
        else return 1;
        if (np * 32 < rot / 2) return 2;  // pairs that no lane computes
      }
}
