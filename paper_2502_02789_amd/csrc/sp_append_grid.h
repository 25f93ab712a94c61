// How sp_cache_append cuts a call into workgroups.  Plain C++: the call and a test without a GPU go through the same function.
#pragma once

#include <stdint.h>

#include <algorithm>

#include "specprefill.h"

namespace sp {

constexpr int kTokens = 4;  // most tokens of a workgroup (8192 tokens into 8 bits: 8 takes 2 % longer, 16 18 %; 100K of d = 64: 3 and 8 %)

constexpr int64_t kMostTokens = INT64_C(1) << 25;  // of a call
constexpr int64_t kMostBlocks = (INT64_C(1) << 24) - 1;  // of 256 threads: a launch has fewer than 2^32

struct AppendGrid { int tokens; uint32_t blocks, parts; };  // tokens of a workgroup; parts: workgroups to the same tokens

// rows: heads of queries, keys and values of a token, 0 < T <= kMostTokens
inline AppendGrid append_grid(int64_t T, int rows, int d, int dtype) {
  // few tokens: one to a workgroup, and several workgroups to a token, until the device has some hundred
  // (into 4 bits fewer, three chunks to a lane: with their reading back, 6592 tokens of 64 heads, one to a workgroup instead of four, 62.6 us instead of 69.0;
  // 8192 of 8 heads, four instead of one, 16.2 instead of 20.9; 8192 of 32 heads and 100K of d = 64, two and four, the same within 2 %)
  const int per_token = rows * (d / 16), most = dtype == SP_K_MXFP4 ? std::max(1, std::min(kTokens, 768 / per_token)) : kTokens;
  AppendGrid g;
  g.tokens = (int)std::min<int64_t>(most, std::max<int64_t>(1, T / 512));
  g.tokens = (int)std::max<int64_t>(g.tokens, (T + kMostBlocks - 1) / kMostBlocks);  // (what a launch can hold: three at most)
  const int64_t blocks = (T + g.tokens - 1) / g.tokens;
  const int chunks = (g.tokens * per_token + 255) / 256;
  g.blocks = (uint32_t)blocks;
  g.parts = blocks >= 512 ? 1u : (uint32_t)std::max(1, (int)std::min<int64_t>(chunks, 512 / blocks));
  return g;
}

}  // namespace sp
