// What is found of what was kept, by device and share: exits with the number of the first check that fails.
#include "cluster_counts.h"

int main() {
  static vcs::ClusterCounts c;
  if (c.find(0, 0) != 0 || c.find(0, 65552) != 0 || c.find(7, 16) != 0) return 1;
  c.keep(0, 65552, 57);
  c.keep(1, 65552, 54);               // another device
  c.keep(0, 64000, 60);               // another vocabulary
  if (c.find(0, 65552) != 57 || c.find(1, 65552) != 54 || c.find(0, 64000) != 60) return 2;
  if (c.find(2, 65552) != 0 || c.find(0, 65568) != 0) return 3;
  c.keep(0, 65552, 56);
  if (c.find(0, 65552) != 56 || c.find(1, 65552) != 54) return 4;
  for (int device = 0; device < 64; ++device)
    for (uint32_t share = 16; share <= 213008; share += 16) {
      const int count = (int)(share / 16 % 456) + 1;
      c.keep(device, share, count);
      if (c.find(device, share) != count) return 5;
      c.keep(device ^ 1, share, 999);
      if (c.find(device, share) == 999) return 6;
      if (c.find(device, share + 16 * vcs::ClusterCounts::kPlaces) == 999) return 7;
    }
  static vcs::ClusterCounts none;
  none.keep(0, 16, 0);
  none.keep(3, 48, 1 << 16);          // does not fit: not kept
  return none.find(0, 16) != 0 || none.find(3, 48) != 0 ? 8 : 0;
}
