// Bits of the device status word, the first int32 of every workspace.
#pragma once

namespace hspec {

enum : int {
  ST_BAD_PAGE = 1,      // a page id outside [0, num_pages)
  ST_BAD_CTX_LEN = 2,   // ctx_len < 0 or beyond the table / max_ctx_len
  ST_BAD_ROWS = 16,     // a ragged row array (cu_new, cu_rows) that is no increasing division of the rows
};

}  // namespace hspec
