// How the heads of a rows call are dealt to waves, and its tokens to launches: the host's side, and where a wave finds itself.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace tl {

constexpr int kMostHeads = 1 << 16;
constexpr int kWaveHeads = 8;            // heads that a wave takes at once: 8 lanes with 16 values each to a head
constexpr int kMostTokensLog2 = 3;       // tokens that a wave has

enum { kQ = 0, kK = 1, kV = 2 };

// A quotient by a number that the host knows: n / d = n * magic >> 32 for n d < 2^32.
struct Div {
  uint32_t d, magic;
};
inline Div div_of(uint32_t d) { return {d, d == 1 ? 0u : (uint32_t)(((uint64_t)1 << 32) / d) + 1u}; }
__host__ __device__ __forceinline__ uint32_t div_by(uint32_t n, Div x) { return x.d == 1 ? n : (uint32_t)((uint64_t)n * x.magic >> 32); }

// How the heads of one kind are dealt to waves.  A wave takes 8 heads: of one token or, where there are at most 4 (2, 1), of 2 (4, 8) tokens.
struct Deal {
  int32_t heads, tokens_log2, waves;     // waves: that the tokens of a group have for this kind
  Div per_tokens;                        // waves of 1 << tokens_log2 tokens
};

struct Dealing {
  Deal kind[3];
  int32_t group_log2;                    // tokens that waves are counted for
  Div group_waves;
};

// Kinds of few heads are packed, up to 8 tokens to a wave, unless a group of that many tokens has more than kMostGroupWaves waves of the
// kind with many: 2^32 / waves / waves - 1 groups to a launch (most_groups) are 3 or more up to there and none from 46341 waves on.  One token to
// a group is at most 3 x 8192 waves, so the loop ends.
constexpr uint32_t kMostGroupWaves = 1 << 15;

inline Dealing deal_heads(const int32_t (&heads)[3]) {
  Dealing a;
  uint32_t waves = 0;
  for (int most_log2 = kMostTokensLog2; most_log2 >= 0; --most_log2) {
    a.group_log2 = 0;
    for (int i = 0; i < 3; ++i) {
      Deal& d = a.kind[i];
      d.heads = heads[i];
      d.tokens_log2 = 0;
      while (heads[i] && d.tokens_log2 < most_log2 && heads[i] << (d.tokens_log2 + 1) <= kWaveHeads) ++d.tokens_log2;
      if (d.tokens_log2 > a.group_log2) a.group_log2 = d.tokens_log2;
    }
    waves = 0;
    for (int i = 0; i < 3; ++i) {
      Deal& d = a.kind[i];
      const int32_t at_once = kWaveHeads >> d.tokens_log2;
      const uint32_t per = heads[i] ? (uint32_t)(heads[i] + at_once - 1) / at_once : 1;
      d.per_tokens = div_of(per);
      d.waves = heads[i] ? (int32_t)(per << (a.group_log2 - d.tokens_log2)) : 0;
      waves += d.waves;
    }
    if (waves <= kMostGroupWaves) break;
  }
  a.group_waves = div_of(waves);
  return a;
}

// Groups of tokens that one launch takes: wave numbers stay below 2^25, and below 2^32 / waves for their quotient.
inline int64_t most_groups(const Dealing& a) {
  const uint32_t waves = a.group_waves.d;
  const int64_t most = (1 << 25) / waves, exact = ((int64_t)1 << 32) / waves / waves - 1;
  return most < exact ? most : exact;
}

// What wave number `wave` of a launch has: heads from `head` on of one kind, of up to 1 << tokens_log2 tokens from the launch's number `token` on.
struct Place {
  int kind;
  Deal deal;                             // the kind's
  int64_t token;
  int head;
};
__host__ __device__ __forceinline__ Place place_of(const Deal (&deal)[3], int32_t group_log2, const Div& group_waves, uint32_t wave) {
  const uint32_t group = div_by(wave, group_waves);
  uint32_t part = wave - group * group_waves.d;
  int kind = kQ;
  if (part >= (uint32_t)deal[kQ].waves) {
    part -= deal[kQ].waves;
    kind = kK;
    if (part >= (uint32_t)deal[kK].waves) {
      part -= deal[kK].waves;
      kind = kV;
    }
  }
  const Deal d = deal[kind];
  const uint32_t tg = div_by(part, d.per_tokens);
  return {kind, d, ((int64_t)group << group_log2) + ((int64_t)tg << d.tokens_log2), (int)(part - tg * d.per_tokens.d) * (kWaveHeads >> d.tokens_log2)};
}

}  // namespace tl
