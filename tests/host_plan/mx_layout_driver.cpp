// Prints what the 4-bit cache's layout comes to: bytes of a head's part of a page, and of a page.
//   mx_layout_driver page_size D Hkv
#include "mx_layout.h"

int main(int argc, char** argv) {
  if (argc != 4) return 2;
  const int ps = std::atoi(argv[1]), D = std::atoi(argv[2]), Hkv = std::atoi(argv[3]);
  std::printf("%zu %zu\n", hspec::mx_head_bytes(ps, D), hspec::mx_page_bytes(ps, D, Hkv));
}
