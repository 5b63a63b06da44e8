// Launchers of the target's side of a step: append of new tokens to the paged cache, attention of a
// ragged chunk over it, verification of drafted tokens.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>
#include <climits>

namespace hspec {

// ------------------------------------------------------------------------------ append
struct ChunkAppendArgs {
  const void* qkv = nullptr;          // [T, (Hq + 2 Hkv) D], fp32 or bf16
  void* q = nullptr;                  // [T, Hq, D] storage type
  void *k_cache = nullptr, *v_cache = nullptr;
  const float *qw = nullptr, *kw = nullptr;   // [D] gains, or null: no norm
  const int32_t *cu = nullptr, *ctx_lens = nullptr, *page_table = nullptr;
  int B = 0, T = 0, max_new = 0, Hq = 0, Hkv = 0, D = 0, ps = 0, max_pages = 0, num_pages = 0;
  int cap = 0;                        // positions a request can have: max_pages ps, at most 2^31 - 1
  float eps = 0.f;
  double rope_theta = 0.;
  int* status = nullptr;
  int in_f32 = 1, out_f32 = 0;
};
hipError_t launch_chunk_append(const ChunkAppendArgs& a, hipStream_t s);
// 4-bit caches: append; rows of the cache out to k, v [T, Hkv, D] (of `a`: the batch, the caches, out_f32)
hipError_t launch_chunk_append_mx(const ChunkAppendArgs& a, hipStream_t s);
hipError_t launch_chunk_read_mx(const ChunkAppendArgs& a, void* k, void* v, hipStream_t s);

// --------------------------------------------------------------------------- attention
// One piece of work of every KV head: `row0`, `n`, `L` are the request's checked first row, number of new
// tokens and cached length; rows [32 NW tile, ..) of its n g (token, head) rows over keys [k0, k1).
// slot < 0: the piece holds every key of its rows and writes the output.
struct ChunkUnit {
  int b, tile, k0, k1;
  int slot, row0, n, L;
};
// Rows whose keys were split over `pieces` units, whose partial results begin at `slot`.
struct ChunkSplit {
  int b, tile, slot, pieces;
  int row0, n, L, pad;
};
constexpr int kChunkClasses = 8;      // work queues: one per accelerator die (XCD)
constexpr int kChunkQueueStride = 16; // ints between two queue counters (one 64-byte line each)
struct ChunkAttnArgs {
  const void *q = nullptr, *k_cache = nullptr, *v_cache = nullptr;
  void* o = nullptr;                  // [T, Hq, D] storage type
  const int32_t *cu = nullptr, *ctx_lens = nullptr, *page_table = nullptr;
  int B = 0, T = 0, max_new = 0, Hq = 0, Hkv = 0, D = 0, ps = 0, max_pages = 0, num_pages = 0;
  int window = 0, f32 = 0;
  int cap = 0;                        // positions a request can have: min(max_len, max_pages ps)
  float scale_log2 = 0.f;
  // 4-bit caches: K and V of the new tokens [T, Hkv, D] beside the cache, or null; `block`: every new token of a
  // request sees every other; `held`: positions the cache has room for
  const void *k_new = nullptr, *v_new = nullptr;
  int block = 0, held = INT_MAX;
  int* status = nullptr;              // [0] status, [1] units, [2] split tiles, [3] items to do again
  int* queue = nullptr;               // [kChunkClasses * kChunkQueueStride]
  ChunkUnit* units = nullptr;
  ChunkSplit* splits = nullptr;
  int* first = nullptr;               // [columns + 1] the first unit of each column; null: each finds its own
  int* flags = nullptr;               // [columns][Hkv][waves] what a column's waves found; null: no columns
  int* redo = nullptr;                // items to do again, status[3] of them; null: rows of a request see the same keys
  float* part_o = nullptr;            // [slots][Hkv][tile rows][D]
  float* part_ml = nullptr;           // [slots][Hkv][tile rows][2]
  // chunk_bounds
  int tile_rows = 0, key_tile = 0, once = 0, slots = 0, target = 0, min_split = 0;
  int columns = 0;                    // 0: units go by a queue
  int max_units = 0, max_slots = 0, max_splits = 0, max_redo = 0, max_flags = 0;
};
// Keys per tile, and waves per SIMD the registers are sized for, of a workgroup of `waves` waves.
constexpr int chunk_key_tile(int waves, bool f32) { return f32 || waves == 1 ? 32 : 64; }
constexpr int chunk_waves_per_simd(bool f32, int D) { return f32 && D == 128 ? 1 : 2; }
constexpr int kChunkMinSplit = 64;   // keys a piece of a split tile has at least
constexpr int kMaxPositions = INT_MAX - 65536;   // of a request: places past the end of a tile stay inside 31 bits

// Keys a unit takes at most, in whole key tiles, for `keys` keys of `tiles` tiles of rows: where the tiles leave most of
// the chip free, what makes one round of units (so every piece starts at once: 1 request of 32768 tokens 43 us, 54 in
// two short rounds; 8 of 4000 tokens 39 and 45), else 13/8 rounds, which the queue evens out.  At least keys Hkv / target, which the workspace
// counts on (the factor covers the float roundings).
__host__ __device__ inline int chunk_unit_keys(const ChunkAttnArgs& a, unsigned long long keys, int tiles) {
  const float spare = (float)a.slots - (float)tiles * (float)a.Hkv;
  const float units = spare * 4.f >= (float)a.slots * 3.f ? spare : (float)a.target;
  const float per = (float)keys * (float)a.Hkv / units * 1.0001f;
  // (at the most no tile is split, so that the bound on the pieces holds for any number of keys)
  const float least = (float)a.min_split, most = (float)kMaxPositions;
  return ((int)(per < least ? least : per > most ? most : per) + a.key_tile) / a.key_tile * a.key_tile;
}
// Even pieces of a tile of len keys, each a whole number of key tiles but the last: their number, and their length in q.
__host__ __device__ inline int chunk_pieces(int len, int S, int key_tile, int& q) {
  q = len > 1 ? len : 1;
  if (len <= S) return 1;
  const unsigned p = ((unsigned)len + S - 1) / (unsigned)S;
  q = (int)((((unsigned)len + p - 1) / p + key_tile - 1) / key_tile * key_tile);
  return (int)(((unsigned)len + q - 1) / (unsigned)q);
}

// What the plan's bounds come to for a tile, its workgroups of `waves` and the target (chunk_bounds and mx_bounds).
inline void plan_bounds(ChunkAttnArgs& a, int waves) {
  const long long g = a.Hq / a.Hkv, R = a.max_new * g;
  a.once = R <= a.tile_rows;
  a.min_split = kChunkMinSplit;
  const long long per_req = (R + a.tile_rows - 1) / a.tile_rows;
  const long long tiles = std::min(a.T * g / a.tile_rows + a.B, per_req * a.B);
  // pieces of a tile, and of all tiles: see chunk_plan
  const long long len = (long long)a.cap + a.key_tile;
  const long long cuts = (len + a.min_split - 1) / a.min_split;
  const long long extra = (a.target + a.Hkv - 1) / a.Hkv;
  a.max_units = (int)std::min(tiles * cuts, tiles + extra);
  a.max_slots = cuts > 1 ? (int)std::min(tiles * cuts, 2 * extra) : 0;
  a.max_splits = (int)std::min(tiles, (long long)a.max_slots / 2);
  a.max_redo = a.max_units * a.Hkv * waves;   // an entry for every wave
}
// Tile of the units, and the most units, partial slots and split tiles the plan can make of any lengths.  32 rows per
// wave; past four waves a request has several tiles (once = 0).  fp32 takes one, two or four waves by the rows a request
// can have (n g): its key tile and LDS are the same for all, so waves without rows only keep others out (64 requests of
// 512..8192 cached, 16 and 4 heads of 128: 1 token 484 us, 888 with four; 3 tokens 489 and 895).  bf16 takes four, whose
// idle waves still load (32 and 8 heads of 128: 1 request of 1 token and 16000 cached 32 us, 36 with one; 200 of at most
// 3000 cached 218 and 224), but one for up to 32 rows over many long caches, where small workgroups keep more of them
// reading (64 requests of 1 token and 512..8192 cached 212 us, 223 with four).
inline void chunk_bounds(ChunkAttnArgs& a) {
  const long long g = a.Hq / a.Hkv, R = a.max_new * g;
  const bool many_long = a.cap >= 4096 && (long long)a.B * a.Hkv >= 32;
  const int waves = R <= 32 && (a.f32 || many_long) ? 1 : R <= 64 && a.f32 ? 2 : 4;
  a.tile_rows = 32 * waves;
  a.key_tile = chunk_key_tile(waves, a.f32);
  // workgroups that run at once on 256 compute units: LDS (two stages of K and V) goes in 128 pieces of 1280 bytes
  const int lds = (4 * a.key_tile * a.D * (a.f32 ? 4 : 2) + 8 + 1279) / 1280;
  a.slots = std::min(128 / lds, 4 * chunk_waves_per_simd(a.f32, a.D) / waves) * 256;
  a.target = a.slots * 13 / 8;
  plan_bounds(a, waves);
}

// Over the 4-bit cache, up to 128 rows of a request take the tiles of chunk_few.h: bf16 rows up to 32 are a wave's, more
// are divided over the waves of a workgroup; fp32 rows are 16 a wave.
struct MxTile {
  int rows, rw, kw;   // of a wave, waves that divide the rows and a step's keys; rows = 0: the tiles of chunk_bounds
};
inline MxTile mx_tile(const ChunkAttnArgs& a) {
  const long long R = (long long)a.max_new * (a.Hq / a.Hkv);
  if (R > 128) return MxTile{0, 0, 0};
  if (R <= 16) return MxTile{16, 1, 1};
  if (a.f32) return MxTile{16, R <= 32 ? 2 : R <= 64 ? 4 : 8, 1};
  return R <= 32 ? MxTile{32, 1, 1} : R <= 64 ? MxTile{32, 2, 2} : MxTile{32, 4, 1};
}
inline void mx_bounds(ChunkAttnArgs& a) {
  const MxTile t = mx_tile(a);
  if (!t.rows) return chunk_bounds(a);
  a.tile_rows = t.rows * t.rw;
  a.key_tile = 64;
  // as many columns as workgroups run at once, and no more than there can be steps
  const long long most = std::min<long long>(a.T, a.B) * ((a.cap + 63LL) / 64 + 1);
  const int waves = t.rw * t.kw;
  a.slots = (t.rows == 16 && !a.f32 ? 12 : 8) / waves * 256;
  a.columns = (int)std::max(1LL, std::min<long long>(a.slots / a.Hkv, most));
  a.target = a.columns * a.Hkv;
  plan_bounds(a, waves);
  a.max_flags = a.columns * a.Hkv * waves;
  if (a.B <= 64) {   // no plan: a slot for every unit, an entry for every request
    a.max_slots = a.max_units = a.B + a.columns;
    a.max_splits = a.B;
  }
}
hipError_t launch_chunk_attn(const ChunkAttnArgs& a, hipStream_t s);
hipError_t launch_chunk_attn_mx(const ChunkAttnArgs& a, hipStream_t s);

// ------------------------------------------------------------------------ verification
// A row's largest logit, and log2 of the sum of 2^((l - m) c).
struct RowSum {
  float m, log_s;
};
// What a finished row leaves for the choice: the sums of the target's and the draft's row, status bits, greedy's argmax.
struct VerifyRow {
  RowSum p, q;
  int flags, top;
};
constexpr int kVerifyLine = 32;   // ints between counters: a 128-byte line each, so that they are not one line's traffic
// 64-bit words of a request's pieces of the choice, two each, in whole lines.
__host__ __device__ constexpr int verify_key_stride(int pieces_r) {
  return (2 * pieces_r + kVerifyLine / 2 - 1) / (kVerifyLine / 2) * (kVerifyLine / 2);
}
struct VerifyArgs {
  const void* target = nullptr;       // [rows, V]
  const float* draft = nullptr;       // [B, k, Vd] or null
  const int32_t *draft_tokens = nullptr, *cu = nullptr, *d2t = nullptr, *t2d = nullptr;
  const float *u = nullptr, *gumbel = nullptr;   // null: greedy
  int32_t *tokens = nullptr, *accepted = nullptr;
  int B = 0, k = 0, rows = 0, V = 0, Vd = 0, f32 = 0;
  float c_t = 1.f, c_d = 1.f;             // log2(e) / temperature, of the target and of the drafts
  double c64_t = 1., c64_d = 1.;
  int* status = nullptr;
  unsigned long long* stat_t = nullptr;   // [rows][pieces_t]
  unsigned long long* stat_d = nullptr;   // [B*k][pieces_d]
  VerifyRow* row = nullptr;               // [B][k + 1]
  int* count = nullptr;                   // [B][k + 1][kVerifyLine] pieces of a row that are done
  int* n = nullptr;                       // [B][kVerifyLine] first draft found not to stand
  int2* req = nullptr;                    // [B] first row, drafts
  int* done = nullptr;                    // [B][kVerifyLine] workgroups of the choice that are done
  unsigned long long* keys = nullptr;     // [B][verify_key_stride] of each piece of the choice: best (score, token), bounds
  int pieces_t = 0, pieces_d = 0, pieces_r = 0;
};
constexpr int kVerifyPiece = 32768;   // bytes of a row that a workgroup takes at a time, all its loads under way together
inline void verify_bounds(VerifyArgs& a) {
  auto pieces = [](long long bytes) { return (int)((bytes + kVerifyPiece - 1) / kVerifyPiece); };   // at most 64 (host check)
  a.pieces_t = pieces((long long)a.V * (a.f32 ? 4 : 2));
  a.pieces_d = pieces((long long)a.Vd * 4);
  // the choice reads one row a request: enough workgroups for the chip, of at least 4096 logits
  a.pieces_r = (int)std::max(1LL, std::min({1024LL / a.B, a.V / 4096LL, 64LL}));
}
hipError_t launch_verify(const VerifyArgs& a, hipStream_t s);

// -------------------------------------------------------------------------- adjustment
struct AdjustArgs {
  const void* logits = nullptr;       // [rows, V]
  void* out = nullptr;
  const int32_t *cu = nullptr, *draft_tokens = nullptr, *d2t = nullptr;
  const int32_t *history = nullptr, *hist_lens = nullptr, *prompt_lens = nullptr;   // [B, max_hist], [B]
  const float *repetition = nullptr, *frequency = nullptr, *presence = nullptr;     // [B] or null
  const int32_t* bias_ids = nullptr;  // [B, n_bias]
  const float* bias = nullptr;
  const uint32_t* mask = nullptr;     // [masks, words of V bits]
  const int32_t* mask_rows = nullptr; // [rows] or null: row r's is r
  int B = 0, k = 0, rows = 0, V = 0, Vd = 0, max_hist = 0, n_bias = 0, masks = 0;
  int in_f32 = 0, out_f32 = 0;
  int* status = nullptr;
};
hipError_t launch_adjust(const AdjustArgs& a, hipStream_t s);

}  // namespace hspec
