// Units of work of the packed attention, laid out on the host from the sequences'
// lengths, which a program knows there.  Everything about a sequence's split follows
// from its own lengths and the group size, never from the batch around it, so it gives
// the same bits alone and packed among others.
#include <algorithm>

#include "packed.hpp"

namespace losa {

namespace {

// Keys of a part of a few-row sequence (a multiple of the 32-key sub-tile): one
// workgroup of four waves (bf16) or eight (fp32), two sub-tiles each at least, so that a
// part's partial rows stay small beside its K and V; 256 parts at most, so that the
// join stays short.
int part_keys(bool bf16, int k_len) {
  const int least = bf16 ? 256 : 512;
  const int64_t even = ((int64_t)k_len + kMostParts - 1) / kMostParts;
  const int64_t keys = (even + 63) / 64 * 64;
  return (int)(keys < least ? least : keys);
}

// Keys of a part of a sequence's tiles.  Above 16 tiles: all of them, so a call of few heads
// lasts as long as its longest tile (one head, 3,264 tokens causal, d = 128: 52 us, 3.3 MB).
// Up to 16 tiles: all of them, but where they are many (a chunk of a prompt, drafted tokens,
// over a long cache), a walk that would leave most CUs idle.  A part costs its rows' partial
// results once more, written and read: the more rows, the more keys it takes.  us, whole /
// split, one sequence and eight (fp32 four), causal, d = 128:
//   bf16, 32 / 4 heads, 7 tokens over 4,096 keys 65 / 17, 66 / 22; 32,768 470 / 27, 479 / 121
//   32 / 8 heads, 256 tokens over 4,096 keys 68 / 49, 124 / 158; 32,768 488 / 161, 977 / 1,026
//   512 tokens over 32,768 keys 490 / 281, 1,920 / 1,998
//   fp32, 12 / 4 heads, 64 tokens over 2,048 keys 45 / 24, 50 / 53; 32,768 570 / 142, 658 / 464
// and with 512 keys a part at least 256 tokens over 2,048 keys took 31 and 120 (whole 38
// and 68).  The rule does not see the batch, so that a sequence gives the same bits in any:
// eight chunks that fill the chip by themselves are up to 27 % slower for being split.
constexpr int kSplitTiles = 16;
int tile_part_keys(bool bf16, int64_t rows, int k_len) {
  const int block = kPackedTile[bf16];
  const int64_t tiles = (rows + block - 1) / block;
  if (tiles > kSplitTiles) return k_len;
  const bool many = tiles > kSplitTiles / 2;
  const int least = !bf16 ? (many ? 1024 : 512) : rows <= block / 2 ? 512 : many ? 8192 : 2048;
  const int parts = std::min(k_len / least, (bf16 ? 32 : 64) / (int)tiles);
  if (parts < 2) return k_len;
  const int step = bf16 ? 64 : 256;  // whole rounds of a workgroup's sub-tiles
  return ((k_len + parts - 1) / parts + step - 1) / step * step;
}

// fp32: binary logarithm of the waves that share a row set: no more than there are 32-key
// sub-tiles, so that none idles and few states are merged.  us, all eight / these, dense,
// d = 64: 8,192 x 12 heads over 32 keys 85 / 24, over 64 88 / 36, over 128 93 / 65; but 300
// x 4, where few workgroups are left, 6.3 / 8.3, 6.5 / 8.2, 6.9 / 8.0.  More sub-tiles a wave
// gain in large calls and lose in small ones, which this rule does not tell apart: one / two
// / four, 128 keys 65 / 49 / 45 and 8.0 / 10.3 / 14.7, 256 keys 121 / 91 / 78 and 8.3 / 10.1 /
// 14.5; causal 256 tokens, 64 / 8 heads, eight sequences 143 / 99 / 76, two of 8 heads 8.7 /
// 10.3 / 14.8.  Kept is what the small calls want.
constexpr int kAllWaves = 3;
static_assert(1 << kAllWaves == kPackedWaves[0], "a workgroup's waves");
int key_waves(int k_len) {
  int by = 0;
  while (by < kAllWaves && k_len > (32 << by)) ++by;
  return by;
}
// Rows of a unit of a sequence's tiles, `rows` those of a tile or row set.
int unit_rows(bool bf16, int rows, int k_len) {
  return bf16 ? rows : rows * kPackedWaves[0] >> key_waves(k_len);
}

// fp32 units of 32 rows below which a call takes 16.  us in tiles of 16 / of 32, dense:
// 128 units (1,024 x 4 heads, d = 128) 25.6 / 39.7; 256 47.2 / 40.2 and causal 31.7 / 40.2;
// 555 410 / 427, at d = 64 200 / 232; 768 255 / 211, at d = 64 119 / 116.
constexpr int64_t kWideUnits = 640;

struct Counts {
  int64_t tiles, few, joins, wide, part_rows;
};

// Rows of a call's tiles.  fp32: 16 where tiles of 32 would make few rounds of the
// machine's 256 CUs; a row's arithmetic is the same in either.
int tile_rows(const PackedSeqs& s) {
  if (s.bf16) return kPackedTile[1];
  int64_t wide = 0;
  for (int i = 0; i < s.n; ++i) {
    const int64_t rows = (int64_t)s.q_len[i] * s.G;
    if (rows <= kPackedFew[0]) continue;
    const int keys = std::max(1, tile_part_keys(false, rows, s.k_len[i]));
    const int unit = unit_rows(false, kPackedTile[0], s.k_len[i]);
    wide += (rows + unit - 1) / unit * std::max(1, (s.k_len[i] + keys - 1) / keys);
  }
  return wide * s.H_kv < kWideUnits ? kPackedNarrow : kPackedTile[0];
}

// Calls tile(item), few(item), join(row) for every unit, in order; returns their number.
template <typename Tile, typename Few, typename Join>
Counts walk(const PackedSeqs& s, int tile_rows, Tile&& tile, Few&& few, Join&& join) {
  Counts c = {};
  int64_t q0 = 0, k0 = 0;
  for (int i = 0; i < s.n; ++i) {
    const int64_t q_start = s.q_start ? s.q_start[i] : q0, k_start = s.k_start ? s.k_start[i] : k0;
    const int q_len = s.q_len[i], k_len = s.k_len[i];
    q0 += q_len;
    k0 += k_len;
    const int shift = k_len - q_len;  // causal: token t sees keys up to t + shift
    const int64_t rows = (int64_t)q_len * s.G;
    if (rows == 0) continue;
    const bool tiled = rows > kPackedFew[s.bf16];
    PackedItem it = {};
    it.part = -1;
    it.split = s.bf16 ? 0 : tiled ? key_waves(k_len) : kAllWaves;
    const int block = unit_rows(s.bf16, tile_rows, k_len);
    const int keys = tiled ? tile_part_keys(s.bf16, rows, k_len) : part_keys(s.bf16, k_len);
    const int parts = std::max(1, (int)(((int64_t)k_len + keys - 1) / std::max(1, keys)));
    if (tiled) {
      for (int64_t r = 0; r < rows; r += block) {
        const int tok = (int)(r / s.G);
        const int last = (int)std::min<int64_t>(q_len - 1, (r + block - 1) / s.G);
        it.q_row = q_start + tok;
        it.head0 = (int)(r - (int64_t)tok * s.G);
        it.rows = (int)(rows - r);
        const int seen = s.causal ? std::max(0, std::min(k_len, last + shift + 1)) : k_len;
        for (int p = 0; p < parts; ++p) {
          const int first = p * keys;
          it.keys = std::max(0, std::min(seen - first, keys));
          it.k_row = it.keys > 0 ? k_start + first : 0;
          it.seen = s.causal ? tok + shift + 1 - first : kAllSeen;
          if (parts > 1) it.part = (int)(c.part_rows + p * rows + r);
          tile(it);
          ++c.tiles;
        }
      }
    } else {
      it.q_row = q_start;
      it.rows = (int)rows;
      for (int p = 0; p < parts; ++p) {
        const int first = p * keys;
        it.keys = std::min(k_len - first, keys);
        it.k_row = it.keys > 0 ? k_start + first : 0;
        it.seen = s.causal ? shift + 1 - first : kAllSeen;
        if (parts > 1) it.part = (int)(c.part_rows + p * rows);
        few(it);
        ++c.few;
      }
    }
    if (parts > 1) {
      for (int64_t r = 0; r < rows; ++r) {
        join(PackedJoin{q_start + r / s.G, (int)(r % s.G), (int)(c.part_rows + r), (int)rows, parts});
        ++c.joins;
        c.wide += parts > kFewParts;
      }
      c.part_rows += parts * rows;
    }
    if (std::max(c.tiles + c.few, c.part_rows) >= ((int64_t)1 << 31)) break;  // too many
  }
  return c;
}

}  // namespace

bool packed_counts(const PackedSeqs& s, PackedCounts* out) {
  out->tile_rows = tile_rows(s);
  const Counts c = walk(s, out->tile_rows, [](const PackedItem&) {}, [](const PackedItem&) {},
                        [](const PackedJoin&) {});
  // (tiles and few-row units may share a launch)
  const int64_t units = (c.tiles + c.few) * s.H_kv;
  const int64_t joins = c.wide * s.H_kv + ((c.joins - c.wide) * s.H_kv + kJoinWaves - 1) / kJoinWaves;
  if (units > most_workgroups(kPackedWaves[s.bf16]) || joins > most_workgroups(kJoinWaves) ||
      c.part_rows >= ((int64_t)1 << 31))
    return false;
  out->tiles = (int)c.tiles;
  out->few = (int)c.few;
  out->joins = (int)c.joins;
  out->wide = (int)c.wide;
  out->part_rows = c.part_rows;
  return true;
}

void packed_fill(const PackedSeqs& s, const PackedCounts& n, void* plan) {
  PackedItem* const tiles = static_cast<PackedItem*>(plan);
  PackedItem* const few = tiles + n.tiles;
  PackedJoin* const joins = reinterpret_cast<PackedJoin*>(few + n.few);
  int64_t t = 0, f = 0, j[2] = {n.wide, 0};
  walk(s, n.tile_rows, [&](const PackedItem& x) { tiles[t++] = x; }, [&](const PackedItem& x) { few[f++] = x; },
       [&](const PackedJoin& x) { joins[j[x.n > kFewParts]++] = x; });
  // longest first, so that the launch's tail is made of short units; order changes only
  // the schedule.  (std::sort: no allocation)
  auto longer = [](const PackedItem& a, const PackedItem& b) {
    if (a.keys != b.keys) return a.keys > b.keys;
    if (a.q_row != b.q_row) return a.q_row < b.q_row;
    return a.head0 != b.head0 ? a.head0 < b.head0 : a.k_row < b.k_row;
  };
  std::sort(tiles, tiles + n.tiles, longer);
  std::sort(few, few + n.few, longer);
}

}  // namespace losa
