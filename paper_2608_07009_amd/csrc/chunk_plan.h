// How a chunk attention call is divided into workgroups: the host's bounds (plan_chunk) and, from chunk
// starts and lengths that only the device knows, each request's row tiles and splits. The attention and
// the merge, two kernels compiled apart, work it out each for itself and have to agree to the last
// token: all of it is whole numbers.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "hisparse.h"

#ifdef __HIPCC__
#define HISPARSE_BOTH __host__ __device__ __forceinline__
#else
#define HISPARSE_BOTH inline
#endif

namespace hisparse {

template <class T>
HISPARSE_BOTH constexpr T least_of(T a, T b) { return a < b ? a : b; }
template <class T>
HISPARSE_BOTH constexpr T most_of(T a, T b) { return a < b ? b : a; }

constexpr int kMaxSplits = 128;  // parts of one request's cached tokens
// The least tokens of a split: a workgroup's two rounds of two tiles (latent records), its eight
// tiles (grouped-query ones).
HISPARSE_BOTH constexpr int min_split(bool latent) { return latent ? 128 : 256; }
// Workgroups that splitting aims at: one per CU, which is what LDS holds. (512: 24% more time for 8
// requests of 8 kv heads x 4 over 4096 8-bit tokens, 30% for one over 32768 16-bit ones.)
constexpr int kTargetWorkgroups = 256;

// Rows (new token, query head of the kv head) of one workgroup, in groups of 32; what waves are left
// over take other tokens. Grouped-query records: as many groups as the request's rows fill, up to
// eight (four at most: a 2048-token chunk of 16384 1140 us instead of 1043). Latent ones: four, or two
// where tiles of 64 rows are fewer than the CUs (`split`): a split's partial results are 2 KB a row,
// written and read again, and a workgroup of half the rows covers twice the tokens (32 requests of 128
// heads over 2048 8-bit tokens: 59 us with four, 51 with two; 3 requests' 2 tokens of 100, 64 heads: 25
// and 18.5).
HISPARSE_BOTH int row_groups(int rows, bool latent, bool split) {
  if (latent) return rows <= 64 || split ? 2 : 4;
  return rows <= 32 ? 1 : rows <= 64 ? 2 : rows <= 128 ? 4 : 8;
}

// What a call's division follows from.
struct ChunkShape {
  const int32_t *start, *kv_len;
  int32_t requests, kv_heads, g, total, max_chunk, max_tokens, window;
  int32_t split;                // row tiles are split as a rule, not only those of long requests
  int32_t target;               // workgroups that splitting aims at (0: none)
  int32_t num_splits;           // asked for (0: chosen)
  int32_t uni_tiles, uni_splits;  // of every request, where they are alike (start and kv_len null)
  int64_t head_part_rows;       // rows of partial results of a kv head
};

struct Request {
  int begin, n, len;
};
HISPARSE_BOTH Request request_of(const ChunkShape& a, int r) {
  Request q;
  if (a.start) {
    q.begin = least_of(most_of(a.start[r], 0), a.total);
    q.n = least_of(least_of(most_of(a.start[r + 1], q.begin), a.total) - q.begin, a.max_chunk);
  } else {
    q.begin = r * a.max_chunk;
    q.n = a.max_chunk;
  }
  q.len = a.kv_len ? least_of(most_of(a.kv_len[r], 0), a.max_tokens) : a.max_tokens;
  return q;
}
// Row tiles of a request, of `groups` groups of 32 rows.
HISPARSE_BOTH int tiles_of(const ChunkShape& a, bool latent, const Request& q, int& groups) {
  const int rows = q.n * a.g;
  groups = row_groups(rows, latent, a.split);
  return (int)(((uint32_t)rows + 32 * groups - 1) / (32 * groups));
}
HISPARSE_BOTH int span_of(const ChunkShape& a, const Request& q) {
  return a.window ? least_of(q.len, a.window + q.n - 1) : q.len;
}
HISPARSE_BOTH int splits_of(const ChunkShape& a, const Request& q, int part) {
  const int span = span_of(a, q);
  if (a.num_splits) return least_of(a.num_splits, most_of(1, (span + 63) >> 6));
  return a.target ? least_of(most_of((span + part - 1) / part, 1), kMaxSplits) : 1;
}
// 64-token blocks that a request's row tiles read.
HISPARSE_BOTH uint64_t blocks_of(const ChunkShape& a, const Request& q, int tiles) {
  return (uint64_t)(uint32_t)tiles * (uint32_t)((span_of(a, q) + 63) >> 6);
}

// A request's (row tile, split)s. A call has fewer than 2^23, but starts that descend give requests more
// rows between them than there are, so that each is held to it: sums over 64 requests then stay in 32
// bits, in groups of 32 rows too, and what does not fit the workspace is seen in partial_rows_fit.
HISPARSE_BOTH uint32_t items_of(int tiles, int splits) {
  constexpr uint32_t most = (1u << 23) - 1;
  return least_of(least_of((uint32_t)tiles, most) * (uint32_t)splits, most);
}
// Whether the partial results of a row tile, from row `first` on, lie in the workspace. Always, if
// starts ascend; else such a tile is left out by the attention and the merge.
HISPARSE_BOTH bool partial_rows_fit(const ChunkShape& a, int64_t first, int splits, int groups) {
  return splits == 1 || first + splits * groups * 32 <= a.head_part_rows;
}

// Tokens of a part, of which `blocks` blocks make at most n (128 .. 512) and a started one per row tile;
// share = share_of(n), apart because it is a division where n is not a constant.
HISPARSE_BOTH constexpr uint32_t share_of(uint32_t n) { return (0x80000000u + n - 1) / n; }
HISPARSE_BOTH int part_length(uint64_t blocks, uint32_t share, bool latent) {
  if (blocks >> 32) return 1 << 30;  // (2^38 tokens: longer than any request, or twice as long)
  const uint32_t p = (uint32_t)(blocks * share >> 25) + 1;
  return (int)least_of<uint32_t>(most_of<uint32_t>(p, min_split(latent)), 1 << 30);
}
// Splits follow from the requests' lengths alone. With fewer row tiles than kTargetWorkgroups, cached
// tokens lie in parts of W / target, W the tokens of all row tiles, if those are at most `target` parts
// (a tile's last may be short), so that all start at once; else of 4/3 of that, or of W / (target - row
// tiles) if that is less: with those they always are. (16 requests of 4096 8-bit tokens, 8 kv heads x 4,
// 128 row tiles: 40 us in two parts each, 52 in one.) With more row tiles, in parts of W / (2 target),
// which only the tiles of long requests are split into, so that the last of them ends not long after
// the others.
// `blocks`, `tiles`: of one kv head, all requests; items(p): its (row tile, split)s with parts of p.
template <class Items>
HISPARSE_BOTH int choose_part(uint64_t blocks, int tiles, int kv_heads, bool latent, Items&& items) {
  constexpr int target = kTargetWorkgroups;
  blocks *= (uint32_t)kv_heads;
  const int64_t all = (int64_t)tiles * kv_heads;
  if (all >= target) return part_length(blocks, share_of(2 * target), latent);
  const int sure = most_of(target - (int)all, target / 2);
  for (int parts = target; parts > sure; parts -= target / 4) {
    const int p = part_length(
        blocks, parts == target ? share_of(target) : share_of(target - target / 4), latent);
    if ((int64_t)items(p) * kv_heads <= target) return p;
  }
  return part_length(blocks, share_of(sure), latent);
}

struct ChunkPlan {
  int64_t tiles, items;  // at most so many row tiles, (tile, split)s of a kv head
  int64_t part_rows;     // rows of partial results, all kv heads
  int32_t d_v, target, uni_tiles, uni_splits, max_splits;
  int32_t groups;        // of 32 rows of the largest row tile
  bool split;            // row tiles are split as a rule, not only those of long requests
  size_t workspace_bytes;  // of this call
  size_t serves_bytes;     // of this call and every smaller batch's
};

inline ChunkPlan plan_chunk(const hisparse_kv_desc_t& kv, const hisparse_chunk_desc_t& c) {
  ChunkPlan p{};
  p.d_v = kv.layout == HISPARSE_KV_GROUPED ? 128 : 512;
  const bool latent = kv.layout == HISPARSE_KV_LATENT;
  const int64_t chunk = least_of<int64_t>(c.max_chunk, most_of(c.total_tokens, 1));
  const int64_t max_rows = chunk * c.q_heads;
  const int64_t tokens = (int64_t)c.max_records * kv.tokens_per_record;
  const int64_t span =
      c.window ? least_of<int64_t>(tokens, c.window + chunk - 1) : tokens;
  const int64_t blocks = (span + 63) / 64 + 1;  // a first token inside a block adds one
  int64_t bm = 0;     // rows of a tile
  int64_t parts = 0;  // items of a kv head with partial results
  auto count_tiles = [&](bool split) {
    bm = 32 * row_groups((int)least_of<int64_t>(max_rows, 1 << 20), latent, split);
    p.uni_tiles = (int32_t)((max_rows + bm - 1) / bm);
    // every request has a last row tile that may not be full; the others are of the most rows
    const int64_t most = latent ? bm : 256;
    p.tiles = least_of<int64_t>((int64_t)c.total_tokens * c.q_heads / most + c.num_requests,
                                (int64_t)c.num_requests * p.uni_tiles);
  };
  auto bytes_of = [&](int64_t part_rows) {
    return part_rows == 0 ? 0 : (size_t)part_rows * (p.d_v * sizeof(float) + 2 * sizeof(float)) +
                                    sizeof(int32_t);
  };
  // Splits of fewer row tiles than CUs: the most of one tile, and of `tiles` of them together (what
  // choose_part allows for).
  const int64_t least = (span + min_split(latent) - 1) / min_split(latent);
  const int64_t few_splits = least_of<int64_t>(least, kMaxSplits);
  auto few_items = [&](int64_t tiles) {
    const int64_t t = kTargetWorkgroups;
    return least_of(tiles * few_splits,
                    most_of<int64_t>(t / c.kv_heads, tiles + t / 2 / c.kv_heads) + 2);
  };
  size_t smaller = 0;  // what the largest batch of fewer row tiles than CUs needs
  p.max_splits = 1;
  p.uni_splits = 1;
  count_tiles(true);
  if (c.num_splits > 0) {
    p.max_splits = (int32_t)least_of<int64_t>(c.num_splits, blocks);
    p.uni_splits = p.max_splits;
    p.split = p.max_splits > 1;
    count_tiles(p.split);
    p.items = p.tiles * p.max_splits;
    parts = p.items;
  } else if (p.tiles * c.kv_heads < kTargetWorkgroups) {
    // (latent: tiles of 64 rows; as soon as those would be more than the CUs, tiles of 128 rows: 190
    // requests of 128 heads over 2048 16-bit tokens 150 us, 202 with 64; 240 8-bit ones 190, 208)
    p.split = true;
    p.items = p.tiles;
    if (least > 1) {
      p.target = kTargetWorkgroups;
      p.max_splits = (int32_t)few_splits;
      // requests alike (p.tiles is then exact): as many splits as all start at once
      p.uni_splits = (int32_t)least_of<int64_t>(
          p.max_splits, most_of<int64_t>(1, p.target / (p.tiles * c.kv_heads)));
      p.items = few_items(p.tiles);
      parts = p.items;
    }
  } else {
    const int64_t fewer = (kTargetWorkgroups - 1) / c.kv_heads;
    if (least > 1 && fewer > 0) smaller = bytes_of(few_items(fewer) * bm * c.kv_heads);
    // Parts of W / (2 target): at most 2 target more items than row tiles, and a tile that is split
    // is longer than one, so that it has at most twice as many as it is long. One request of 65536
    // 8-bit tokens among 63 of 1000, 8 kv heads x 4: 578 us without, 84 with; latent, 16 heads, among
    // 299: 2480 and 146. 64 requests of 4096 tokens, which are not split: 109 and 113 for working
    // that out. Where no request can have four parts of the least length that is not tried (64 of
    // 512: 25 us, 33).
    count_tiles(false);
    p.items = p.tiles;
    const int64_t more = 2 * kTargetWorkgroups / c.kv_heads;
    if (least >= 4 && more > 0) {
      p.target = kTargetWorkgroups;
      p.max_splits = (int32_t)few_splits;
      p.items = least_of(p.tiles * p.max_splits, p.tiles + more);
      parts = least_of(p.items, 2 * more + 1);
    }
  }
  if (p.max_splits > 1) {
    p.groups = (int32_t)(bm / 32);
    p.part_rows = parts * bm * c.kv_heads;
  }
  p.workspace_bytes = bytes_of(p.part_rows);
  p.serves_bytes = most_of(p.workspace_bytes, smaller);
  return p;
}

inline ChunkShape chunk_shape(const hisparse_kv_desc_t& kv, const hisparse_chunk_desc_t& c,
                              const ChunkPlan& p, const int32_t* start, const int32_t* kv_len) {
  ChunkShape a{};
  a.start = start;
  a.kv_len = kv_len;
  a.requests = c.num_requests;
  a.kv_heads = c.kv_heads;
  a.g = c.q_heads;
  a.total = c.total_tokens;
  a.max_chunk = least_of(c.max_chunk, c.total_tokens);
  a.max_tokens = c.max_records * kv.tokens_per_record;
  a.window = c.window < a.max_tokens ? c.window : 0;  // (its sums stay in 32 bits)
  a.split = p.split;
  a.target = p.target;
  a.num_splits = c.num_splits;
  a.uni_tiles = p.uni_tiles;
  a.uni_splits = p.uni_splits;
  a.head_part_rows = p.part_rows / c.kv_heads;
  return a;
}

}  // namespace hisparse
