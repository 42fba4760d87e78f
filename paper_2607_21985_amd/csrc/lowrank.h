// Kernel arguments of the low-rank adapters' launches (adapt.hip).
#pragma once

#include <cstdint>

namespace spdp_low {

constexpr int kMaxBanks = 8;
constexpr int kMaxRank = 128;
constexpr int kMaxAdapters = 2048;  // of a bank: the sort's counters are in LDS
constexpr int kSmall = 64;          // up to so many tokens a wave sorts the ids in its lanes

// A group of tokens that share an adapter.
struct Tile {
  int adapter;  // -1: none
  int start;    // of the tokens in `perm`
  int count;    // 0: no tile
  int pad;
};

// Where a workgroup's tokens come from: ids NULL: adapter 0, tokens in
// sequence. Tiles NULL: `n_tokens` <= kSmall ids, sorted by every wave for
// itself. Else the sort's tiles.
struct Tokens {
  const int* ids;
  const int* perm;
  const Tile* tiles;
  int n_tokens;
  int count;  // adapters
};

// in [tokens, width] times factor [adapter][rank][width]^T -> part
// [split][token][rank]
struct Shrink {
  const uint16_t* in;
  const uint16_t* factor;
  float* part;
  int width;
  int per;  // steps of 64 columns per split
};
struct ShrinkArgs {
  Shrink m[kMaxBanks];
  Tokens t;
  int rank;
};

// out [tokens, width] = base + scale * part's sum times factor
// [adapter][rank][width]; the sum to `keep` [token][rank] unless NULL; the
// largest magnitude of each token's sum and of its `other` [token][rank] to
// `most` [2][token] unless NULL
struct Expand {
  const float* part;
  const uint16_t* factor;
  const float* scale;
  const uint16_t* base;
  uint16_t* out;
  float* keep;
  float* most;
  const float* other;
  const uint16_t* in;            // the fused form's: part is computed from it
  const uint16_t* first_factor;  // and from this, as by Shrink
  int width;
  int splits;
  int in_width;
};
struct ExpandArgs {
  Expand m[kMaxBanks];
  Tokens t;
  int rank;
  int blocks;  // 256-column blocks per workgroup
  int subs;    // parts of a tile, each a workgroup's
};

// out [adapter][rank][width] = scale * the sum over an adapter's tokens of
// rank activation times input
struct Outer {
  const float* act;      // [token][rank]
  const uint16_t* in;    // [token][width]
  float* out;            // [adapter][rank][width], or [split][adapter][rank][width]
  const float* most;     // [token]: the largest magnitude of act
  unsigned char* packed; // the activations as operands
  float* down;           // [adapter][split]: what their scale has to be undone with
  int width;
  int stream;            // the input is larger than the caches
};
struct OuterArgs {
  Outer m[2];
  const float* scale;
  const int* perm;  // tokens by adapter, or NULL: in sequence
  const int* first; // [adapters + 1] in perm, or NULL: one adapter of n_tokens
  int n_tokens;
  int count;
  int rank;
  int splits;
  int waves;        // of a workgroup of outer_kernel: 4 or 8
  int wide;         // 128 columns instead of 64
  int packed;       // the activations are
};

}  // namespace spdp_low
