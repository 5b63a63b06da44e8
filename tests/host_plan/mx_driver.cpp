// The chunk attention's plan over the 4-bit cache: driver.cpp's checks with that cache's tiles and bounds, with new tokens
// in the cache, beside it, and in a block beside it; and of the plans in columns: every unit in one column, all columns
// of the same number of steps but the last that has any.
//   mx_driver valid | malformed | longest
#include <vector>

#include "chunk_plan.h"

namespace {

int g_form = 0;
std::vector<int> g_first;
long g_columns = 0;

void bounds_of_form(hspec::ChunkAttnArgs& a) {
  if (g_form) a.held = a.cap;
  a.block = g_form == 2;
  if (a.block) a.window = 0;
  hspec::mx_bounds(a);
  g_first.assign((size_t)a.columns + 1 + 64, -77);
  a.first = g_first.data();
}

void check_columns(const hspec::ChunkAttnArgs& a) {
  if (!a.columns) return;
  for (size_t i = a.columns + 1; i < g_first.size(); ++i)
    if (g_first[i] != -77) emu::die("columns past the workspace");
  if (a.first[0] != 0 || a.first[a.columns] != a.status[1]) emu::die("ends of the columns");
  long long most = 0;
  bool last = false;
  for (int w = 0; w < a.columns; ++w) {
    if (a.first[w + 1] < a.first[w]) emu::die("order of the columns");
    long long steps = 0;
    for (int i = a.first[w]; i < a.first[w + 1]; ++i)
      steps += std::max(((long long)a.units[i].k1 - a.units[i].k0 + a.key_tile - 1) / a.key_tile, 1LL);
    if (w == 0) most = steps;
    if (steps > most || (last && steps)) emu::die("steps of a column");
    last |= steps < most;
  }
  ++g_columns;
}

}  // namespace

namespace hspec {
inline void plan_and_columns(const ChunkAttnArgs& a) {
  chunk_plan(a);
  __syncthreads();
  if (threadIdx.x == 0) check_columns(a);
}
}  // namespace hspec

#define chunk_bounds bounds_of_form
#define chunk_plan plan_and_columns
#define main plans
#include "driver.cpp"
#undef main

int main(int argc, char** argv) {
  for (g_form = 0; g_form < 3; ++g_form)
    if (int rc = plans(argc, argv)) return rc;
  std::printf("%ld plans in columns\n", g_columns);
  return g_columns ? 0 : 1;
}
