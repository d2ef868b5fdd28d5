// The division of chunk attention calls (paper_2608_07009_amd/csrc/chunk_plan.h) over random batches, on
// the host: whatever the device finds from starts and lengths has to fit the host's grid and workspace.
// Prints "ok <calls> <checksum of all part lengths>".
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "chunk_plan.h"

using namespace hisparse;

static std::mt19937_64 rng(1);
static int64_t upto(int64_t most) {  // 1 .. most, spread over the logarithm
  std::uniform_real_distribution<double> u(0.0, std::log((double)most + 1.0));
  return std::max<int64_t>(1, std::min<int64_t>(most, (int64_t)std::exp(u(rng))));
}
static bool chance(double p) { return std::uniform_real_distribution<double>(0, 1)(rng) < p; }

static void fail(const char* what, const ChunkShape& a, const ChunkPlan& p, int64_t got, int64_t most) {
  std::printf("%s: %lld, at most %lld (requests %d heads %d x %d total %d chunk %d tokens %d window %d "
              "splits %d target %d tiles %lld)\n",
              what, (long long)got, (long long)most, a.requests, a.kv_heads, a.g, a.total, a.max_chunk,
              a.max_tokens, a.window, a.num_splits, a.target, (long long)p.tiles);
  std::exit(1);
}

// Starts in any order: no row tile that is done has partial results outside the workspace. Requests 64 at
// a time, as a wave takes them.
static void check_disorder(const ChunkShape& a, const ChunkPlan& p, bool latent, int part) {
  int64_t rows = 0;
  for (int base = 0; base < a.requests; base += 64) {
    uint32_t in_wave = 0;
    for (int r = base; r < std::min(base + 64, a.requests); ++r) {
      const Request q = request_of(a, r);
      if (q.begin < 0 || q.n < 0 || (int64_t)q.begin + q.n > a.total) fail("rows", a, p, q.begin, q.n);
      int groups;
      const int tiles = tiles_of(a, latent, q, groups), splits = splits_of(a, q, part);
      const uint32_t items = items_of(tiles, splits);
      for (uint32_t tile : {0u, items / splits / 2, items / splits - 1}) {
        if (splits == 1 || tile >= items / splits) continue;
        const int64_t first = (rows + in_wave + (int64_t)tile * splits * groups) * 32;
        const int64_t end = first + (int64_t)splits * groups * 32;
        if (partial_rows_fit(a, first, splits, groups) && (first < 0 || end > a.head_part_rows))
          fail("partial results", a, p, end, a.head_part_rows);
      }
      if (splits > 1 && __builtin_add_overflow(in_wave, items * (uint32_t)groups, &in_wave))
        fail("sum over a wave", a, p, items, 0);
    }
    rows += in_wave;
  }
}

int main() {
  uint64_t sum = 0;
  int calls = 0;
  for (int round = 0; round < 30000; ++round) {
    hisparse_kv_desc_t kv{};
    hisparse_chunk_desc_t c{};
    const bool latent = chance(0.5);
    kv.layout = latent ? HISPARSE_KV_LATENT : HISPARSE_KV_GROUPED;
    kv.tokens_per_record = 1 << (rng() % 7);
    c.kv_heads = (int)(latent ? 1 : upto(chance(0.1) ? 600 : 16));
    c.q_heads = (int)upto(256);
    c.num_requests = (int)upto(chance(0.1) ? 5000 : 300);
    c.max_chunk = (int)upto(3000);
    c.max_records = (int)std::max<int64_t>(1, upto(chance(0.1) ? 1 << 22 : 50000) / kv.tokens_per_record);
    c.window = chance(0.3) ? (int)upto(20000) : 0;
    c.num_splits = chance(0.2) ? (int)upto(64) : 0;
    // chunks and lengths: few or many rows of what the descriptor allows for
    std::vector<int32_t> start(c.num_requests + 1), len(c.num_requests);
    const int most_new = (int)upto(c.max_chunk), kind = rng() % 3;
    const int64_t tokens = (int64_t)c.max_records * kv.tokens_per_record;
    const int64_t most_len = upto(tokens);
    for (int r = 0; r < c.num_requests; ++r) {
      const int64_t n = chance(0.1) ? 0 : kind == 0 ? 1 : kind == 1 ? upto(most_new) : most_new;
      start[r + 1] = (int32_t)std::min<int64_t>(start[r] + n, 1 << 22);
      len[r] = (int32_t)(chance(0.05) ? tokens : chance(0.5) ? upto(most_len) : most_len);
    }
    c.total_tokens = start[c.num_requests] + (chance(0.3) ? (int)upto(5000) : 0);
    const bool disorder = chance(0.2);
    if (disorder) {
      if (chance(0.3)) c.total_tokens = (int)std::min<int64_t>(INT32_MAX / (c.kv_heads * c.q_heads), 1 << 30);
      if (chance(0.3)) c.max_chunk = (int)upto(INT32_MAX);
      for (int32_t& x : start) x = (int32_t)(rng() % 3 == 0 ? rng() : rng() % (c.total_tokens + 1u));
    }
    if (c.total_tokens == 0 || (int64_t)c.total_tokens * c.kv_heads * c.q_heads > INT32_MAX) continue;
    const ChunkPlan p = plan_chunk(kv, c);
    const ChunkShape a = chunk_shape(kv, c, p, start.data(), len.data());
    uint64_t blocks = 0;
    int64_t tiles = 0;
    int groups;
    for (int r = 0; r < a.requests; ++r) {
      const Request q = request_of(a, r);
      const int t = tiles_of(a, latent, q, groups);
      tiles += t;
      blocks += blocks_of(a, q, t);
    }
    const int part = !a.target || a.num_splits ? 0 :
        choose_part(blocks, (int)tiles, a.kv_heads, latent, [&](int x) {
          int64_t n = 0;
          for (int r = 0; r < a.requests; ++r) {
            const Request q = request_of(a, r);
            n += tiles_of(a, latent, q, groups) * splits_of(a, q, x);
          }
          return n;
        });
    if (disorder) {
      check_disorder(a, p, latent, part);
      continue;
    }
    int64_t items = 0, rows = 0, split = 0;
    for (int r = 0; r < a.requests; ++r) {
      const Request q = request_of(a, r);
      const int t = tiles_of(a, latent, q, groups), s = splits_of(a, q, part);
      items += t * s;
      if (s == 1 || t == 0) continue;
      rows += (int64_t)t * s * groups * 32;
      split += t;
      if (groups > p.groups) fail("groups of a split tile", a, p, groups, p.groups);
      if (s > p.max_splits) fail("splits", a, p, s, p.max_splits);
    }
    if (items > p.items) fail("items", a, p, items, p.items);
    if (tiles > p.tiles) fail("row tiles", a, p, tiles, p.tiles);
    if (split > p.tiles) fail("row tiles to merge", a, p, split, p.tiles);
    if (rows > a.head_part_rows) fail("rows of partial results", a, p, rows, a.head_part_rows);
    if (p.workspace_bytes > p.serves_bytes) fail("workspace", a, p, p.workspace_bytes, p.serves_bytes);
    // chunks without starts and lengths
    if ((int64_t)a.requests * c.max_chunk <= a.total) {
      const int64_t all = (int64_t)a.requests * p.uni_tiles;
      const int64_t bm = 32 * row_groups(a.max_chunk * a.g, latent, a.split);
      if (all * p.uni_splits > p.items) fail("alike items", a, p, all * p.uni_splits, p.items);
      if (all > p.tiles) fail("alike row tiles", a, p, all, p.tiles);
      if (p.uni_splits > 1 && all * p.uni_splits * bm > a.head_part_rows)
        fail("alike rows", a, p, all * p.uni_splits * bm, a.head_part_rows);
    }
    sum = (sum ^ (uint64_t)part) * 0x9E3779B97F4A7C15ull;
    ++calls;
  }
  for (int i = 0; i < 1000000; ++i) {  // parts long enough, and not longer by more than a part in 2^22
    const uint64_t blocks = upto(((int64_t)1 << 32) - 1);
    const uint32_t parts = 128 + rng() % 385;
    const uint64_t x = part_length(blocks, share_of(parts), false);
    if (x * parts < 64 * blocks && x < 1 << 30) { std::printf("part too short\n"); return 1; }
    if (x > 256 && x < 1 << 30 && (x - 1) * parts > 64 * blocks + (blocks >> 15)) {
      std::printf("part too long\n");
      return 1;
    }
    sum = (sum ^ x) * 0x9E3779B97F4A7C15ull;
  }
  std::printf("ok %d %llx\n", calls, (unsigned long long)sum);
  return 0;
}
