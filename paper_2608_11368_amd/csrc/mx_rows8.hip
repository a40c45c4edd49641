// Attention of a few new tokens per request over a paged cache in 8 bits
// (attn_rows.hpp).
#include "attn_rows.hpp"

namespace pair {

int rows::launch_mx8(const RowArgs& s, const Plan& p, hipStream_t stream) {
  return launch_of<8>(s, p, stream);
}

}  // namespace pair
