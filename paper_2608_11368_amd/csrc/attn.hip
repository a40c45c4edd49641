// Causal attention over a paged cache: which kernels a call takes.
#include "attn.hpp"

namespace pair {

namespace {

int64_t most_rows(int32_t q_heads, int32_t kv_heads, int32_t max_q) {
  return (int64_t)max_q * (q_heads / kv_heads);
}

size_t rounded(size_t bytes) { return (bytes + 255) / 256 * 256; }

// A call of chunks may hold requests of a few rows beside them, which the tile
// kernel would serve without splitting their keys.  If every request has the
// bound's tokens, or there is only one, none does.
bool has_few(int64_t n, int64_t tokens, int32_t max_q) { return n > 1 && tokens < n * max_q; }

}  // namespace

size_t attention_workspace_bytes(int64_t n, int64_t tokens, int32_t q_heads, int32_t kv_heads,
                                 int32_t dim, int32_t max_q, int32_t max_len) {
  const size_t rows = rounded(attention_rows_workspace(n, q_heads, kv_heads, dim, max_q, max_len));
  if (most_rows(q_heads, kv_heads, max_q) <= kRowsMost) return rows;
  return (has_few(n, tokens, max_q) ? rows : 0) +
         rounded(attention_tiles_workspace(n, tokens, q_heads, kv_heads, dim, max_len));
}

int launch_attention(const AttnCall& a, void* workspace, hipStream_t stream) {
  if (most_rows(a.q_heads, a.kv_heads, a.max_q) <= kRowsMost)
    return launch_attention_rows(a, workspace, stream);
  if (!has_few(a.n, a.tokens, a.max_q)) return launch_attention_tiles(a, 0, workspace, stream);
  const int rc = launch_attention_rows(a, workspace, stream);
  if (rc != PAIR_OK) return rc;
  const size_t rows = rounded(
      attention_rows_workspace(a.n, a.q_heads, a.kv_heads, a.dim, a.max_q, a.max_len));
  return launch_attention_tiles(a, kRowsMost + 1, static_cast<unsigned char*>(workspace) + rows,
                                stream);
}

}  // namespace pair
