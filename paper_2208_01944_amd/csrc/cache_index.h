// Index arithmetic of the cache's kernels in plain constant functions, so that
// the host can check it for every page and head size that is taken.
#pragma once

namespace palq {

constexpr int kPages[] = {16, 32, 64, 128};   // tokens of a page
constexpr int kDims[] = {64, 96, 128, 256};   // channels of a head

// cache_append_kernel: a block goes by items of 4 tokens x 8 channels, one for a
// thread at a time, and a thread holds all of its items at once (1, 2 or 4).
constexpr int kAppendThreads = 256;
constexpr int append_items(int page, int dim) { return page / 4 * (dim / 8); }
constexpr int append_rounds(int page, int dim) {
  const int n = (append_items(page, dim) + kAppendThreads - 1) / kAppendThreads;
  return n <= 2 ? n : 4;
}
// Values turned in LDS: page / 4 words a channel, and one that keeps banks apart.
constexpr int turned_stride(int page) { return page / 4 + 1; }
constexpr int turned_words(int rounds) { return rounds * kAppendThreads * 8 + 256; }

constexpr bool append_holds_every_block() {
  for (const int page : kPages)
    for (const int dim : kDims) {
      const int n = append_rounds(page, dim);
      if (n > 4 || append_items(page, dim) > n * kAppendThreads || dim * turned_stride(page) > turned_words(n)) return false;
    }
  return true;
}
static_assert(append_holds_every_block(), "a block that the append's threads or LDS do not hold");

// attend_tile_kernel: a tile of 64 tokens comes as 4 dim pieces of 16 bytes of keys (16
// channels of a token) and as many of values (16 tokens of a channel); thread t of 256
// takes pieces t, t + 256, ..  Past the last piece it loads the last one again, so that
// loads stand under no condition, and stores nothing.
constexpr int kTileThreads = 256;
struct TilePiece {
  int tok, s, kr;  // keys: token, 16 channels, row of the matrix operand
  int d, vt;       // values: channel, first token
};
constexpr bool tile_piece_past(int n, int dim) { return 4 * dim % kTileThreads && n >= 4 * dim; }
constexpr TilePiece tile_piece(int n, int dim) {
  const int p = tile_piece_past(n, dim) ? 4 * dim - 1 : n, ks = dim / 16;
  const int j = p & 7, s = p / 8 % ks, gu = p / (8 * ks), g = gu & 3, u = gu >> 2;
  return TilePiece{u * 32 + (j >> 2) * 16 + g * 4 + (j & 3), s, u * 32 + g * 8 + j, (p >> 6) * 16 + (p & 15), (p >> 4 & 3) * 16};
}
// Bytes from the start of a block; tile: the tile's first token within a page of more
// than 64 tokens, mask: page - 1 or 63, the smaller.
constexpr unsigned tile_key_at(const TilePiece &p, int tile, int mask, int dim) { return (tile + (p.tok & mask)) * dim + p.s * 16; }
constexpr unsigned tile_value_at(const TilePiece &p, int tile, int mask, int shift) { return (p.d << shift) + tile + (p.vt & mask); }

constexpr bool tile_stays_inside(int dim) {
  for (int shift = 4; shift <= 7; ++shift)
    for (int n = 0; n < (4 * dim + kTileThreads - 1) / kTileThreads * kTileThreads; ++n) {
      const int page = 1 << shift, mask = (page < 64 ? page : 64) - 1, tile = page > 64 ? page - 64 : 0;
      const TilePiece p = tile_piece(n, dim);
      if (tile_key_at(p, tile, mask, dim) + 16 > unsigned(page * dim) || tile_value_at(p, tile, mask, shift) + 16 > unsigned(page * dim)) return false;
    }
  return true;
}
static_assert(tile_stays_inside(64) && tile_stays_inside(96) && tile_stays_inside(128) && tile_stays_inside(256),
              "a piece of a tile outside its block");

// The tiles of 64 tokens of rows that see [lo, hi) and, before lo, the first `sinks` tokens:
// `count` of them from number 0 on, the first tokens' before the others, so that what lies
// between is never read.  Numbers past the last are asked for ahead (up to 8 more): their places
// stay below 2^31 where hi is at most 2^31 - 1024, also where lo, a row's wish, lies far past hi.
struct TileOrder {
  int count, sink, gap;
  constexpr int at(int i) const { return i < sink ? i : i + gap; }
};
// Of an empty range (hi <= lo) only the tiles before lo's: tiles_seen is for those.
constexpr TileOrder tile_order(int lo, int hi, int sinks) {
  if (hi <= 0) return {0, 0, 0};
  const int seen = sinks < hi ? sinks : hi, tiles = seen / 64 + (seen % 64 > 0), tile0 = lo >> 6;
  const int sink = tiles < tile0 ? tiles : tile0;
  if (hi <= lo) return {sink, sink, 0};
  return {sink + (hi + 63) / 64 - tile0, sink, tile0 - sink};
}
// The same for any rows: where the range is empty (a window that begins behind the last token that is there) nothing
// of it brings the tile of lo, so the first tokens are the range.
constexpr TileOrder tiles_seen(int lo, int hi, int sinks) {
  const int seen = sinks < hi ? sinks : hi;
  return hi <= lo && seen > 0 ? tile_order(0, seen, 0) : tile_order(lo, hi, sinks);
}

}  // namespace palq
