// The driver of the calls on pages and on beginnings in common once more, with every piece of the shared attention's workspace: also the lowest positions,
// the sources' sizes and the blocks' sums, which launches of their own fill where there are many sources.
#define launch_cache_shared launch_cache_shared_pieces
#include "share_driver.hip"
#undef launch_cache_shared

namespace ap {
hipError_t launch_cache_shared(const Shape& s, const SharedArgs& a, bool decode, hipStream_t st) {
  // Sources: the instances, and groups of two members at least; in blocks of 256, which have a sum each.  Two numbers of 64 bits a source, and a block.
  const size_t n = s.n_inst, blocks = (n + n / 2 + 255) / 256, q_rows = n * (decode ? 1 : a.q_cap) * s.g, pieces = shared_pieces(s, a.q_cap);
  check_pieces({{a.begun, n * 4}, {a.behind, n * 4}, {a.row, 2 * q_rows * 8}, {a.low, n * 4}, {a.sizes, blocks * 256 * 16}, {a.totals, blocks * 16},
                {a.ml, pieces * 8}, {a.o, pieces * s.d * 4}});
  return launch_cache_shared_pieces(s, a, decode, st);
}
}  // namespace ap
