// Runs the chunk attention's plan kernel on the host over random batches, divided well and badly, and checks what it
// leaves: units and split tiles inside the workspace that the host reserves, every entry written, rows of no two
// requests the same, every key of every tile of rows in exactly one unit.
//   driver valid | malformed | longest
#include <hip/hip_runtime.h>

#include <map>
#include <set>
#include <string>

#include "chunk_plan.h"

using namespace hspec;

namespace {

// n entries between two guards, all of it filled with a byte that is no valid entry.
template <class T>
struct Guarded {
  std::vector<unsigned char> mem;
  size_t n;
  static constexpr size_t kGuard = 1 << 14;
  explicit Guarded(size_t count) : mem(2 * kGuard + count * sizeof(T), 0xa5), n(count) {}
  T* data() { return reinterpret_cast<T*>(mem.data() + kGuard); }
  void check(const char* what) {
    for (size_t i = 0; i < kGuard; ++i)
      if (mem[i] != 0xa5 || mem[mem.size() - 1 - i] != 0xa5) emu::die(what);
  }
};

struct Batch {
  std::vector<int32_t> cu, lens;
};

// Checks one plan; `valid`: cu divides the rows.
void check(ChunkAttnArgs a, const Batch& x, bool valid, unsigned seed) {
  chunk_bounds(a);
  Guarded<int> status(64), queue(kChunkClasses * kChunkQueueStride);
  Guarded<ChunkUnit> units(a.max_units);
  Guarded<ChunkSplit> splits(a.max_splits);
  a.status = status.data();
  a.queue = queue.data();
  a.units = units.data();
  a.splits = splits.data();
  a.cu = x.cu.data();
  a.ctx_lens = x.lens.data();
  emu::run(PL_THREADS, seed, [&] { chunk_plan(a); });
  status.check("status");
  queue.check("queue");
  units.check("units past the workspace");
  splits.check("splits past the workspace");

  const int g = a.Hq / a.Hkv;
  if (valid == ((a.status[0] & ST_BAD_ROWS) != 0)) emu::die("the flag of bad rows");
  if (a.status[1] < 0 || a.status[1] > a.max_units || a.status[2] < 0 || a.status[2] > a.max_splits) emu::die("counts");
  std::map<std::pair<int, int>, std::vector<ChunkUnit>> tiles;
  std::map<int, ChunkUnit> requests;
  std::set<int> slots;
  for (int i = 0; i < a.status[1]; ++i) {
    const ChunkUnit& u = a.units[i];
    if (u.b < 0 || u.b >= a.B || u.row0 < 0 || u.n < 1 || u.n > a.max_new || u.row0 > a.T - u.n || u.L < 0 || u.L >= a.cap)
      emu::die("rows of a unit");
    if (u.tile < 0 || (long long)u.tile * a.tile_rows >= (long long)u.n * g) emu::die("tile of a unit");
    if (u.slot >= 0 && (u.slot >= a.max_slots || !slots.insert(u.slot).second)) emu::die("slot of a unit");
    tiles[{u.b, u.tile}].push_back(u);
    if (auto [at, fresh] = requests.insert({u.b, u}); !fresh && (at->second.row0 != u.row0 || at->second.n != u.n))
      emu::die("a request in two places");
  }
  int last = 0;
  long long want = 0;
  for (auto& [b, u] : requests) {   // in the order of b
    if (u.row0 < last) emu::die("a row of two requests");
    last = u.row0 + u.n;
    want += ((long long)u.n * g + a.tile_rows - 1) / a.tile_rows;
    if (valid && (u.row0 != x.cu[b] || u.n != x.cu[b + 1] - x.cu[b])) emu::die("rows of a request");
  }
  if ((long long)tiles.size() != want) emu::die("tiles left out");
  if (valid && last != x.cu[a.B]) emu::die("rows left out");
  std::map<std::pair<int, int>, ChunkSplit> cut;
  for (int e = 0; e < a.status[2]; ++e) {
    const ChunkSplit& s = a.splits[e];
    if (s.pieces < 2 || !cut.insert({{s.b, s.tile}, s}).second) emu::die("a split tile that nothing wrote");
  }
  for (auto& [at, us] : tiles) {
    std::sort(us.begin(), us.end(), [](const ChunkUnit& p, const ChunkUnit& q) { return p.k0 < q.k0; });
    const TileKeys k = tile_keys(a, g, at.second, us[0].n, us[0].L);
    if (us[0].k0 != k.k0 || us.back().k1 != max(k.k0, k.k1)) emu::die("keys of a tile");
    const auto c = cut.find(at);
    if ((c != cut.end()) != (us.size() > 1)) emu::die("pieces without a merge");
    for (size_t i = 0; i < us.size(); ++i) {
      if (i && us[i].k0 != us[i - 1].k1) emu::die("keys between pieces");
      if (us.size() == 1 ? us[i].slot >= 0 : us[i].slot != c->second.slot + (int)i) emu::die("slots of pieces");
    }
    if (us.size() > 1) {
      const ChunkSplit& s = c->second;
      if (s.pieces != (int)us.size() || s.row0 != us[0].row0 || s.n != us[0].n || s.L != us[0].L) emu::die("a split tile");
      cut.erase(c);
    }
  }
  if (!cut.empty()) emu::die("a merge without pieces");
}

int pick(std::mt19937& r, int lo, int hi) { return (int)(lo + r() % (unsigned)(hi - lo + 1)); }

ChunkAttnArgs heads(std::mt19937& r) {
  ChunkAttnArgs a;
  a.Hkv = 1 << pick(r, 0, 4);
  a.Hq = a.Hkv * pick(r, 1, 16);
  a.D = pick(r, 0, 1) ? 128 : 64;
  a.f32 = pick(r, 0, 1);
  a.ps = 16;
  return a;
}

}  // namespace

int main(int argc, char** argv) {
  const std::string mode = argc > 1 ? argv[1] : "";
  std::mt19937 r(11);
  int n = 0;
  if (mode == "valid") {
    for (; n < 150; ++n) {
      ChunkAttnArgs a = heads(r);
      a.B = pick(r, 1, n % 10 ? 60 : 700);
      const int top = 1 << pick(r, 0, 8), longest = 1 << pick(r, 0, 15);
      Batch x{{0}, {}};
      a.max_new = 1;
      for (int b = 0; b < a.B; ++b) {
        const int m = pick(r, 0, 3) ? pick(r, 0, top) : 0, L = pick(r, 0, 4) ? pick(r, 0, longest) : longest;
        x.cu.push_back(x.cu.back() + m);
        x.lens.push_back(L);
        a.max_new = max(a.max_new, m);
        a.cap = max(a.cap, L + max(m, 1));
      }
      a.T = max(x.cu.back() + pick(r, 0, 3), 1);
      a.window = pick(r, 0, 2) ? 0 : pick(r, 1, longest);
      check(a, x, true, n);
    }
  } else if (mode == "malformed") {
    for (; n < 150; ++n) {
      ChunkAttnArgs a = heads(r);
      if (n % 2) a.Hkv = 1, a.Hq = 8;   // few heads: the most slots a tile
      a.B = pick(r, 2, n % 10 ? 60 : 300);
      a.T = pick(r, 100, 600);
      a.max_new = pick(r, 0, 1) ? a.T : pick(r, 1, a.T);
      a.cap = pick(r, 100, 700);
      Batch x;
      const int kind = n % 3;   // up and down, any numbers, good but for one entry
      for (int b = 0; b <= a.B; ++b)
        x.cu.push_back(kind == 0 ? (b % 2 ? a.T : 0) : kind == 1 ? pick(r, -50, a.T + 50) : (int)((long long)a.T * b / a.B));
      if (kind == 1 && pick(r, 0, 1)) x.cu[a.B / 2] = pick(r, 0, 1) ? INT_MAX : INT_MIN;
      if (kind == 2) x.cu[pick(r, 0, a.B)] = a.T + 1;
      for (int b = 0; b < a.B; ++b) x.lens.push_back(pick(r, 0, 9) ? pick(r, 0, a.cap) : (int)r());
      check(a, x, false, n);
    }
  } else if (mode == "longest") {   // more keys in all than S can count in 32 bits
    for (int hkv : {1, 4}) {
      ChunkAttnArgs a;
      a.Hkv = hkv, a.Hq = 4 * hkv, a.D = 64, a.ps = 1 << 20, a.B = 3000, a.T = 3000, a.max_new = 1, a.cap = INT_MAX - 65536;
      Batch x{{0}, {}};
      for (int b = 0; b < a.B; ++b) x.cu.push_back(b + 1), x.lens.push_back(a.cap - 1);
      check(a, x, true, n++);
    }
  } else {
    return 2;
  }
  std::printf("%d plans\n", n);
  return 0;
}
