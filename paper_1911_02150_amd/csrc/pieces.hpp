// How the work of the paged attentions is cut into pieces: arithmetic on lengths that the kernels and, on the host, its test share.  No rule makes more pieces of all groups than there are
// groups and kShares, which the grid and the workspace have places for.
#pragma once

namespace mqa {

constexpr int kComputeUnits = 256, kShares = 768, kSharesOfMany = 512, kLeast = 16, kLongest = 64, kLongestScaled = 256;

// Tiles of a piece, at most: a whole number for each of the workgroup's four waves.
__host__ __device__ inline int whole_waves(int tiles) { return ((tiles < 1 ? 1 : tiles) + 3) / 4 * 4; }
__host__ __device__ inline int pieces_of(int tiles, int per) {
  const int n = (int)((unsigned)(tiles + per - 1) / (unsigned)per);
  return n < 1 ? 1 : n;
}
// Many groups: are they left whole?  blocks: of a group's query rows; total: tiles of all groups
__host__ __device__ inline bool left_whole(int blocks, int longest, int total) { return longest <= kLongest && longest * (kComputeUnits / blocks) <= total; }
__host__ __device__ inline int share_of(int blocks, int total) {
  const int shares = blocks > 1 ? kSharesOfMany : kShares, share = (total + shares - 1) / shares;
  return share < kLeast ? kLeast : share;
}
// Tiles of a piece where the pieces are listed.
__host__ __device__ inline int listed_share(int blocks, int longest, int total) { return whole_waves(left_whole(blocks, longest, total) ? longest : share_of(blocks, total)); }

// pieces_of by a reciprocal (less than 2^20 tiles: the quotient is off by one at most).
struct PiecesOf {
  int per;
  float inverse;
  __host__ __device__ static PiecesOf cut(int tiles) {     // into pieces of at most so many
    const int per = whole_waves(tiles);
    return PiecesOf{per, 1.f / (float)per};
  }
  __host__ __device__ int operator()(int tiles) const {
    const int a = tiles + per - 1;
    int n = (int)((float)a * inverse);
    const int rest = a - n * per;
    n += (rest >= per) - (rest < 0);
    return n < 1 ? 1 : n;
  }
};

// Caches of 8 bits, up to 1024 sequences.  cut(tiles) cuts them into pieces of so many tiles and returns how many one head of all sequences has; the last cut stands.  longest: needed where
// there are scaled_many.
// Whole groups where there is one for every compute unit and none is longer than the units' mean, up to 256 tiles (512 sequences of up to 4000, 32 heads: 73.5 us, as in look_for 83.5; 64
// heads 121 and 129.5; 300 of up to 6000, 64 heads 100.7 and 113.9; 300 of 2500, 32 heads, 62.5 and 73; 200 of up to 3000, 64 heads 69.7 and 67.8).  Else as many pieces as leave every
// compute unit one workgroup at most, or two, two from the start where a unit's share is more than 16 tiles (48 sequences of 2048, 32 heads: one 21.3 us, two 22.7; 256 of up to 2000 41.2 and
// 35.0; 64 of 8192 40.1 and 39.5), and up to half over an even share each (256 of up to 2000, 32 heads: 35.0, a quarter over it 44.9; 300 of up to 1500 35.6 and 45.2).  Else shares.
__host__ __device__ inline bool scaled_many(int b, int heads, int blocks) { return b * heads * blocks >= kComputeUnits; }
template <typename Cut>
__host__ __device__ inline void scaled_cut(int b, int heads, int blocks, int longest, int total, Cut&& cut) {
  bool fits = false;
  if (scaled_many(b, heads, blocks)) {
    fits = longest <= kLongestScaled && longest * (kComputeUnits / blocks) <= total;
    if (fits) cut(longest);
  }
  for (int most = (long long)total * blocks > 16 * kComputeUnits ? 2 * kComputeUnits : kComputeUnits; most <= 2 * kComputeUnits; most *= 2) {
    const int units = most / blocks;
    if (!fits && b * heads <= units)
      for (int x = 8; x <= 12 && !fits; ++x) fits = cut((int)(((long long)total * x + 8 * units - 1) / (8 * units))) * heads <= units;
  }
  if (!fits) cut(share_of(blocks, total));
}

// The long pieces come first, by quarters of the longest that there may be, so that short ones fill the end (512 sequences of up to 4096, 64 heads: 133.6 us in the sequences' order, so
// 128.8).  A quarter's counts of pieces are 16 bits of a sum.
__host__ __device__ inline int quarter_of(int tiles, int pieces, int per) {
  return 3 - ((4 * tiles >= pieces * per) + (4 * tiles >= 2 * pieces * per) + (4 * tiles >= 3 * pieces * per));
}
__host__ __device__ inline unsigned long long quarters_before(unsigned long long whole) { return (whole << 16) + (whole << 32) + (whole << 48); }

}  // namespace mqa
