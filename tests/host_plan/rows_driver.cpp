// Rows of requests with bad divisions, wave by wave: every row that is in some request's range is left to one request alone,
// the first of those, whatever pieces of at most 64 rows the requests' rows are looked at in.
//   rows_driver seed
#include "target_rows.h"

int main(int, char** argv) {
  std::mt19937 rng(std::atoi(argv[1]));
  auto pick = [&](int lo, int hi) { return (int)(lo + rng() % (unsigned)(hi - lo + 1)); };
  long shared = 0;
  for (int round = 0; round < 20; ++round) {
    const int B = pick(1, 150), T = pick(1, 200), max_n = pick(1, 90), kind = pick(0, 2);
    std::vector<int32_t> cu(B + 1);
    for (int i = 0; i <= B; ++i) cu[i] = kind == 0 ? pick(-5, T + 5) : std::max(0, i * T / B + pick(-3, 3) * (kind == 2));
    std::vector<int> owner(T, -1), first(T, -1);
    for (int b = 0; b < B; ++b) {
      const hspec::ChunkRows r = hspec::chunk_rows(cu.data(), b, T, max_n);
      if (r.n < 0 || r.row0 < 0 || r.row0 + r.n > T) emu::die("a range past the rows");
      for (int i = 0; i < r.n; ++i)
        if (first[r.row0 + i] < 0) first[r.row0 + i] = b;
        else ++shared;
      const int part = pick(1, 64);
      for (int j0 = 0; j0 < r.n; j0 += part) {
        const int n = std::min(part, r.n - j0);
        unsigned long long taken[64];
        emu::run(64, rng(), [&] { taken[threadIdx.x] = hspec::rows_taken(cu.data(), b, T, max_n, r.row0 + j0, n); });
        bool any = false;
        for (int i = 0; i < b; ++i) {
          const hspec::RowsBefore x = hspec::rows_before(cu.data(), i, b, T, max_n, r.row0 + j0, n);
          any |= x.from < x.to;
        }
        if (any != (taken[0] != 0)) emu::die("whether rows are shared");
        for (int l = 0; l < 64; ++l)
          if (taken[l] != taken[0]) emu::die("lanes that differ");
        if (n < 64 && taken[0] >> n) emu::die("rows past the piece");
        for (int i = 0; i < n; ++i)
          if (!(taken[0] >> i & 1)) {
            int& o = owner[r.row0 + j0 + i];
            if (o >= 0) emu::die("a row of two requests");
            o = b;
          }
      }
    }
    if (owner != first) emu::die("a row that is not its first request's");
  }
  std::printf("%ld rows of several ranges\n", shared);
  return shared ? 0 : 1;
}
