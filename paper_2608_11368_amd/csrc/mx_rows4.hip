// Attention of a few new tokens per request over a paged cache in 4 bits
// (attn_rows.hpp).
#include "attn_rows.hpp"

namespace pair {

int rows::launch_mx4(const RowArgs& s, const Plan& p, hipStream_t stream) {
  return launch_of<4>(s, p, stream);
}

}  // namespace pair
