// Attention of chunks of new tokens over a paged cache in 8 bits (attn_tiles.hpp).
#include "attn_tiles.hpp"

namespace pair {

int tiles::launch_mx8(const TileArgs& s, const Plan& p, const rows::RowArgs* w,
                      const rows::Plan* wp, hipStream_t stream) {
  return launch_of<8>(s, p, w, wp, stream);
}

}  // namespace pair
