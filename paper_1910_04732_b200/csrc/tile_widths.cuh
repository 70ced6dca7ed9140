// Which N widths a tensor-core tile can have (plain C++, no CUDA).
#pragma once

namespace flop {
namespace tc {

// 64, 128, 192 and 256 columns: one CTA or a pair (whose CTAs hold half of B each; an MN-major half comes in 64-wide boxes).
// 208: bf16 pairs with K-major B only.  kind::i8 takes a pair's N in steps of 32, and its epilogue stores whole 64-column groups.
constexpr bool tile_width_ok(int bn, bool pair, bool b_mn_major, bool bytes) {
  if (bn == 208) return pair && !b_mn_major && !bytes;
  if (bn < 64 || bn > 256 || bn % 64 != 0) return false;
  return !(pair && b_mn_major && (bn / 2) % 64 != 0);
}

}  // namespace tc
}  // namespace flop
