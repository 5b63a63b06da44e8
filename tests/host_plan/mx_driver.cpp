// The chunk attention's plan over the 4-bit cache: driver.cpp's checks with that cache's tiles and bounds, with new tokens
// in the cache, beside it, and in a block beside it; and of the plans in columns: every unit in one column, all columns
// of the same number of steps but the last that has any.  Up to 64 requests, what a wave finds of the plan for itself is the
// same, with a slot for every unit.
//   mx_driver valid | malformed | longest
#include <vector>

#include "chunk_columns.h"
#include "chunk_plan.h"

namespace {

int g_form = 0;
bool g_few = false;   // few rows a request, whatever is asked for (where the rows are badly divided all the same)
std::vector<int> g_first;
long g_columns = 0, g_lanes = 0;

void bounds_of_form(hspec::ChunkAttnArgs& a) {
  if (g_form) a.held = a.cap;
  a.block = g_form == 2;
  if (a.block) a.window = 0;
  if (g_few) {
    a.f32 = 0;
    a.max_new = std::max(1, std::min(a.max_new, 128 / (a.Hq / a.Hkv) >> g_form));
  }
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

// By the lanes of a wave.
void check_lanes(const hspec::ChunkAttnArgs& a) {
  static hspec::ChunkUnit units[hspec::CO_REQUESTS];
  const hspec::LanePlan p = hspec::lane_plan(a);
  const bool one = (threadIdx.x & 63) == 0;
  if (p.bits != a.status[0]) emu::die("bits of the lanes");
  for (int w = 0; w < a.columns; ++w) {
    const int n = hspec::column_units(a, p, w, units), first = a.first[w];
    if (n != a.first[w + 1] - first) emu::die("units of a column of the lanes");
    __ballot(true);   // every lane's entries are written
    if (one)
      for (int i = 0; i < n; ++i) {
        const hspec::ChunkUnit &x = units[i], &y = a.units[first + i];
        if (x.b != y.b || x.tile != y.tile || x.k0 != y.k0 || x.k1 != y.k1 || x.row0 != y.row0 || x.n != y.n || x.L != y.L ||
            x.slot != (y.slot < 0 ? -1 : first + i) || x.slot >= a.max_slots)
          emu::die("a unit of the lanes");
      }
    __ballot(true);
  }
  if ((threadIdx.x & 63) < (unsigned)a.B && p.pieces > 1 && (p.unit < 0 || p.unit + p.pieces > a.max_slots)) emu::die("slots of the lanes");
  if (one) ++g_lanes;
}

}  // namespace

namespace hspec {
inline void plan_and_columns(const ChunkAttnArgs& a) {
  chunk_plan(a);
  __syncthreads();
  if (threadIdx.x == 0) check_columns(a);
  if (threadIdx.x < 64 && a.columns && a.B <= CO_REQUESTS) check_lanes(a);
}
}  // namespace hspec

#define chunk_bounds bounds_of_form
#define chunk_plan plan_and_columns
#define main plans
#include "driver.cpp"
#undef main

int main(int argc, char** argv) {
  g_few = argc > 1 && argv[1][0] == 'm';
  for (g_form = 0; g_form < 3; ++g_form)
    if (int rc = plans(argc, argv)) return rc;
  std::printf("%ld plans in columns, %ld of lanes\n", g_columns, g_lanes);
  return g_columns ? 0 : 1;
}
