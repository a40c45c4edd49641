// Attention of chunks of new tokens over a paged cache in 4 bits (attn_tiles.hpp).
#include "attn_tiles.hpp"

namespace pair {

int tiles::launch_mx4(const TileArgs& s, const Plan& p, const rows::RowArgs* w,
                      const rows::Plan* wp, hipStream_t stream) {
  return launch_of<4>(s, p, w, wp, stream);
}

}  // namespace pair
