// Workspace sizes of the operators in flop_rows.cu, for the size query in flop_lib.cu.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace flop {
size_t embedding_rows_ws_bytes(int64_t T, int64_t d);
size_t layer_norm_ws_bytes(int64_t T, int64_t d, int dt);
}  // namespace flop
