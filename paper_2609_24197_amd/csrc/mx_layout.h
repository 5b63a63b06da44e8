// Layout of the 4-bit cache.  For each page and KV head: page_size rows of D / 2 bytes (channel 2i in the low half of byte
// i), then page_size rows of D / 32 scale bytes s, 2^(s - 127), 255 for a block that is NaN.  A head's part of a page is
// one run of memory, so that a unit of attention, which takes one head, reads whole lines.  Nothing here is particular to
// this chip's instructions, so that a test can run it on the host.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>

namespace hspec {
namespace {

constexpr int MX_BLOCK = 32;

__host__ __device__ inline size_t mx_head_bytes(int ps, int D) { return (size_t)ps * (D / 2 + D / MX_BLOCK); }
// All heads of a page: past 32 bits where a request's whole cache is a page (64 heads of 128 and 2^20 positions, 4.6 GB).
__host__ __device__ inline size_t mx_page_bytes(int ps, int D, int Hkv) { return mx_head_bytes(ps, D) * (size_t)Hkv; }

}  // namespace
}  // namespace hspec
