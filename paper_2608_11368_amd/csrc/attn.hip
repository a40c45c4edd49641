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
// bound's tokens, or there is only one, none does.  The host knows no more: in a
// call of uneven chunks without short requests the two launches for those find
// nothing to do, 5 us each (of the 150 us of eight prompts, say).
bool has_few(int64_t n, int64_t tokens, int32_t max_q) { return n > 1 && tokens < n * max_q; }

// One launch serves both kinds side by side where most requests must be short
// against the longest (two chunks of 1024 tokens beside 130 single ones over 4000
// keys, 8 heads of 128: 409 us, two launches 479), or the tiles do not fill the
// card (one of 90 beside 15 over 3000: 57 and 76; three prompts of 300 to 512, 4
// heads of 64, none short: 12.7 and 15).  It holds the registers of both, for which
// chunks pay where they are all there is (8 prompts of 301 to 4096, 4 heads of 64:
// 162 and 152 us; three chunks over 4000 to 8000 keys, 8 of 128: 655 both).
bool together(const AttnCall& a) {
  const int64_t group = a.q_heads / a.kv_heads;
  const int64_t tiles = a.tokens * group / 128 + (a.n < a.tokens ? a.n : a.tokens);
  return a.tokens < a.n * a.max_q / 4 || tiles * a.kv_heads <= 2 * (int64_t)device_cu_count();
}

}  // namespace

int64_t attention_groups(int64_t n, int64_t tokens, int32_t q_heads, int32_t kv_heads,
                         int32_t dim, int32_t max_q, int32_t max_len) {
  const int64_t rows = attention_rows_groups(n, q_heads, kv_heads, dim, max_q, max_len);
  if (most_rows(q_heads, kv_heads, max_q) <= kRowsMost) return rows;
  return (has_few(n, tokens, max_q) ? rows : 0) +
         attention_tiles_groups(n, tokens, q_heads, kv_heads, dim, max_len);
}

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
  if (!has_few(a.n, a.tokens, a.max_q))
    return launch_attention_tiles(a, 0, nullptr, workspace, stream);
  void* few = workspace;
  void* tiles = static_cast<unsigned char*>(workspace) +
                rounded(attention_rows_workspace(a.n, a.q_heads, a.kv_heads, a.dim, a.max_q,
                                                 a.max_len));
  if (together(a))
    return launch_attention_tiles(a, kRowsMost + 1, few, tiles, stream);
  const int rc = launch_attention_rows(a, few, stream);
  if (rc != PAIR_OK) return rc;
  return launch_attention_tiles(a, kRowsMost + 1, nullptr, tiles, stream);
}

}  // namespace pair
