// Launchers of the target's side of a step: append of new tokens to the paged cache, attention of a
// ragged chunk over it, verification of drafted tokens.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace hspec {

// Status bit of a ragged row array (cu_new, cu_rows) that is no increasing division of the rows.
enum : int { ST_BAD_ROWS = 16 };

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
  int* status = nullptr;              // [0] status, [1] units, [2] split tiles, [3] items to do again
  int* queue = nullptr;               // [kChunkClasses * kChunkQueueStride]
  ChunkUnit* units = nullptr;
  ChunkSplit* splits = nullptr;
  int* redo = nullptr;                // items to do again, status[3] of them; null: rows of a request see the same keys
  float* part_o = nullptr;            // [slots][Hkv][tile rows][D]
  float* part_ml = nullptr;           // [slots][Hkv][tile rows][2]
  // filled from chunk_shape / chunk_bounds
  int tile_rows = 0, key_tile = 0, min_split = 0, slots = 0, target = 0, max_units = 0, max_slots = 0, max_splits = 0, max_redo = 0;
};
// The tile the launch uses for these arguments, and the most units, partial slots and split tiles it can need.
void chunk_bounds(ChunkAttnArgs& a);
hipError_t launch_chunk_attn(const ChunkAttnArgs& a, hipStream_t s);

// ------------------------------------------------------------------------ verification
// What a finished row leaves for the choice: log2 of its sums of 2^x, status bits, greedy's argmax.
struct VerifyRow {
  float lse_p, lse_q;
  int flags, top;
};
constexpr int kVerifyLine = 32;   // ints between counters: a 128-byte line each, so that they are not one line's traffic
struct VerifyArgs {
  const void* target = nullptr;       // [rows, V]
  const float* draft = nullptr;       // [B, k, Vd] or null
  const int32_t *draft_tokens = nullptr, *cu = nullptr, *d2t = nullptr, *t2d = nullptr;
  const float *u = nullptr, *gumbel = nullptr;   // null: greedy
  int32_t *tokens = nullptr, *accepted = nullptr;
  int B = 0, k = 0, rows = 0, V = 0, Vd = 0, f32 = 0;
  float c_t = 1.f, c_d = 1.f;             // log2(e) / temperature, of the target and of the drafts
  int* status = nullptr;
  unsigned long long* stat_t = nullptr;   // [rows][pieces_t]
  unsigned long long* stat_d = nullptr;   // [B*k][pieces_d]
  VerifyRow* row = nullptr;               // [B][k + 1]
  int* count = nullptr;                   // [B][k + 1][kVerifyLine] pieces of a row that are done
  int* n = nullptr;                       // [B][kVerifyLine] first draft found not to stand
  int2* req = nullptr;                    // [B] first row, drafts
  int* done = nullptr;                    // [B][kVerifyLine] workgroups of the choice that are done
  unsigned long long* keys = nullptr;     // [B][kVerifyLine / 2] best (score, token)
  int pieces_t = 0, pieces_d = 0, pieces_r = 0;
};
void verify_bounds(VerifyArgs& a);
hipError_t launch_verify(const VerifyArgs& a, hipStream_t s);

}  // namespace hspec
