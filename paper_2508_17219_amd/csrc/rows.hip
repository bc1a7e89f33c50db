// Rows on their way between a layer's projection and the attention: norms of queries and keys for each head, position rotation,
// writes to the pool's slots, and rows of the pool that move to other positions.
//
// Mathematics.  One head's 128 values x of one token:
//   norm      y = x w / sqrt(mean(x^2) + eps)
//   rotation  pair (a, b) of frequency f at position p: a' = m (a cos pf - b sin pf), b' = m (a sin pf + b cos pf)
// rounded once, to bf16, at the end.  The angle is never a float: f / 2 pi is a 64-bit fraction of a turn, and p times it modulo
// 2^64 is the phase of every 32-bit position of either sign to 2^-32 of a turn, without a table.
//
// What bounds it: every value is read once and written once, about ten operations each, so HBM, and at a few tokens the launch.
// A wave is 8 heads of one token (8192 tokens of 32/8 heads with norms, 201 MB: 34.2 us, 5.9 TB/s; a copy of as many bytes by a
// library 38; the 58.5 us of waves that computed all cosines in every lane were the vector unit's).  Waves that take two or four
// times as many heads share a cosine with more of them and wait longer: 0 to 3 % slower from 20 MB on, 0.3 us at a token;
// a workgroup that shares them across its waves 5 to 20 % slower, for its barrier.
#include <cmath>
#include <type_traits>

#include "attn_common.h"
#include "rows_deal.h"

namespace tl {

constexpr int kRowThreads = 256;
// What a call moves decides whether the 256 MB of cache in front of HBM are to keep it.  From 104 MiB on what is read makes room for
// what is written; from 256 MiB on neither would be there when the attention reads it.  us with neither / loads / both passing by the cache
// (rotations of 32/8 heads with norms, 15 blocks of each in turn, which differ by 1 to 4 %), alone and with a copy of other rows to the call's
// inputs in front of it and one of its outputs behind it, both timed with it:
//    67 MB  13.6 / 14.6 / 14.3    39.6 / 38.1 / 39.9        201 MB  37.2 / 34.8 / 34.7    111 / 105 / 107
//    90 MB  17.2 / 17.6 / 17.7    50.8 / 50.1 / 53.7        230 MB  42.6 / 40.8 / 39.1    130 / 119 / 124
//   110 MB  21.2 / 20.4 / 20.7    61.1 / 58.7 / 63.2        258 MB  47.3 / 45.7 / 43.4    150 / 134 / 136
//   134 MB  26.1 / 24.6 / 24.1    73.2 / 69.9 / 74.9        302 MB  54.6 / 53.2 / 50.2    180 / 158 / 158
//   165 MB  31.4 / 28.8 / 29.2    91.1 / 86.0 / 89.2        470 MB  82.1 / 81.5 / 76.5    261 / 268 / 248
// Loads alone are first between the copies from 67 to 258 MB and from 110 MB on do not lose to neither by themselves; both are
// 4 to 6 % ahead by themselves from 230 MB on and first between the copies behind 302.
constexpr int64_t kStreamIn = (int64_t)104 << 20, kStreamAll = (int64_t)256 << 20;

enum { kDense = 0, kToPool = 1, kMove = 2 };      // where rows come from and go to

struct RowsArgs {
  const char* in[3];                     // queries, keys, values (kMove: the pool's keys and values)
  int64_t row[3], head[3];               // strides in bytes
  uint16_t* out[3];                      // dense, or null
  uint16_t* pool[3];                     // kToPool, kMove: where the rows named by dst go
  const float* weight[3];                // null: no norm
  Deal deal[3];
  const int32_t *src, *dst;              // rows of the pool; src: kMove
  const int32_t* pos;                    // positions (kMove: by how many they move)
  const uint64_t* steps;
  float eps, factor;
  int32_t n_pool_rows;
  int32_t rot_lanes;                     // rot_dim / 16: lanes of a head whose values turn; 0: no rotation
  int32_t group_log2;                    // tokens that waves are counted for
  Div group_waves;
  uint32_t n_waves, block_waves;
  int64_t first, end;                    // tokens of this launch
};

// 16 bytes from or to any address
typedef unsigned any_u32x4 __attribute__((ext_vector_type(4), aligned(2)));
template <bool STREAM>
__device__ __forceinline__ uint4 get16(const char* p) {
  return __builtin_bit_cast(uint4, STREAM ? __builtin_nontemporal_load((const any_u32x4*)p) : *(const any_u32x4*)p);
}
template <bool STREAM>
__device__ __forceinline__ void put16(uint16_t* p, uint4 x) {
  if (STREAM)
    __builtin_nontemporal_store(__builtin_bit_cast(any_u32x4, x), (any_u32x4*)p);
  else
    *(any_u32x4*)p = __builtin_bit_cast(any_u32x4, x);
}

__device__ __forceinline__ void widen(uint4 u, float* x) {
  const unsigned w[4] = {u.x, u.y, u.z, u.w};
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __builtin_bit_cast(float, w[i] << 16);
    x[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ float add_square_pair(float acc, unsigned pair) {       // acc + both squares of a packed pair of bf16
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  const bf16x2_t x = __builtin_bit_cast(bf16x2_t, pair);
  return __builtin_amdgcn_fdot2_f32_bf16(x, x, acc, false);
}
__device__ __forceinline__ uint4 narrow(const float* x) {
  return __builtin_bit_cast(uint4, pack_bf16x8(x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]));
}

// cos and sin of a phase (2^64 = one turn), rounded to 2^-32 of a turn: with the step's own 2^-65 times a position, what is turned by is off by at most
// 2^-33 + 2^-34 of a turn.  Quarter turns are taken off the integer; what is left, at most an eighth of a turn, is exact to 3 x 2^-24 of itself
// (the number, the constant and their product in 24 bits), and the power series up to x^9 and x^8 are off by 2e-9 and 2.5e-8 there.
__device__ __forceinline__ void cos_sin(uint64_t phase, float& c, float& s) {
  const uint32_t t = (uint32_t)(phase >> 32) + ((uint32_t)phase >> 31);
  const uint32_t quarter = (t + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(t - (quarter << 30)) * 1.46291807926715968e-9f;      // 2 pi / 2^32
  const float z = x * x;
  const float sx = x + x * z * (-1.f / 6 + z * (1.f / 120 + z * (-1.f / 5040 + z * (1.f / 362880))));
  const float cx = 1.f + z * (-0.5f + z * (1.f / 24 + z * (-1.f / 720 + z * (1.f / 40320))));
  const float u = quarter & 1 ? sx : cx, w = quarter & 1 ? cx : sx;
  c = (quarter + 1) & 2 ? -u : u;
  s = quarter & 2 ? -w : w;
}

// Sum over the 8 lanes of a head.
template <int CTRL>
__device__ __forceinline__ float dpp_add(float x) {
  return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float sum8(float x) {
  return dpp_add<0x141>(dpp_add<0x4e>(dpp_add<0xb1>(x)));   // lanes 1 apart, 2 apart, and the other four by a mirrored half row
}

// A lane holds two runs of 8 values of its head, in memory those that begin at 8 l and 64 + 8 l: each of the wave's loads and stores
// covers whole lines (runs next to each other in a lane touch every line twice: 8192 tokens of 32/8 heads 41 to 44 us for 37,
// fp32 73 for 51).  That has both values of a pair in one lane where they are neighbours or i turns with i + 64.  Where i turns
// with i + rot_dim / 2 nearer by, the runs change lanes through LDS, there and back, and the first rot_lanes lanes
// have one of each half, the others what does not turn (37.5 us, fp32 51 to 53, as with all dimensions; loaded and stored like
// that 40 to 44, 55 to 69).
__device__ __forceinline__ int2 paired_runs(int l, int rot_lanes) {
  return l < rot_lanes ? make_int2(8 * l, 8 * (rot_lanes + l)) : make_int2(8 * (rot_lanes + l), 64 + 8 * l);
}

// Where the lane that turns it finds the cosine and sine of a pair: (j, l) of [4][8] entries of two pairs, the lane's own in entries j = 0..3.
template <bool INTER>
__device__ __forceinline__ int2 entry_of(int pair) {
  return INTER ? make_int2((pair >> 5) * 2 + ((pair >> 1) & 1), (pair & 31) >> 2) : make_int2((pair >> 1) & 3, pair >> 3);
}

// What lanes of a wave have written to LDS is there for its other lanes (they run in step, and LDS serves a wave in order).
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A lane's 16 values as they are in memory, two runs of 8.
template <bool BF16>
struct Lane16 {
  uint4 u[BF16 ? 2 : 4];
  template <bool STREAM>
  __device__ __forceinline__ void load(const char* p, int2 at) {
    const char *x = p + (BF16 ? 2 : 4) * at.x, *y = p + (BF16 ? 2 : 4) * at.y;
    if (BF16) {
      u[0] = get16<STREAM>(x);
      u[1] = get16<STREAM>(y);
    } else {
      u[0] = get16<STREAM>(x);
      u[1] = get16<STREAM>(x + 16);
      u[2] = get16<STREAM>(y);
      u[3] = get16<STREAM>(y + 16);
    }
  }
  // through 128 values of LDS from the runs that the lane has to others
  __device__ __forceinline__ void exchange(char* lds, int2 from, int2 to) {
    constexpr int size = BF16 ? 2 : 4, n = BF16 ? 1 : 2;
    wave_fence();
#pragma unroll
    for (int i = 0; i < n; ++i) {
      *(uint4*)(lds + from.x * size + 16 * i) = u[i];
      *(uint4*)(lds + from.y * size + 16 * i) = u[n + i];
    }
    wave_fence();
#pragma unroll
    for (int i = 0; i < n; ++i) {
      u[i] = *(const uint4*)(lds + to.x * size + 16 * i);
      u[n + i] = *(const uint4*)(lds + to.y * size + 16 * i);
    }
  }
  __device__ __forceinline__ void values(float* x) const {
    if (BF16) {
      widen(u[0], x);
      widen(u[1], x + 8);
    } else {
      __builtin_memcpy(x, u, 64);
    }
  }
};

// Sum of the squares of a head, to each of its 8 lanes.
template <bool BF16>
__device__ __forceinline__ float squares(const Lane16<BF16>& raw, const float* x) {
  float ss = 0;
  if (BF16) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      ss = add_square_pair(add_square_pair(add_square_pair(add_square_pair(ss, raw.u[i].x), raw.u[i].y), raw.u[i].z), raw.u[i].w);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) ss += x[i] * x[i];
  }
  return sum8(ss);
}

// The lane's 16 values over the root of the mean of the head's squares plus eps, times the lane's weights.
template <bool BF16>
__device__ __forceinline__ void norm16(const Lane16<BF16>& raw, float* x, float eps, const float* w) {
  float mean = squares(raw, x) * (1.f / kHeadDim) + eps;
  // Beyond 32 bits (rows that large mean that something is wrong upstream, but their norm is an ordinary number) it is taken again of
  // the values times 2^-70 and eps times 2^-140.
  if (__builtin_expect(mean > 3.4e38f, 0)) {
    float ss = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      x[i] *= 0x1p-70f;
      ss += x[i] * x[i];
    }
    mean = sum8(ss) * (1.f / kHeadDim) + eps * 0x1p-70f * 0x1p-70f;
  }
  const float r = __builtin_amdgcn_rsqf(mean);
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] *= r * w[i];
}

__device__ __forceinline__ void turn2(float& a, float& b, float c, float s) {
  const float u = a * c - b * s;
  b = a * s + b * c;
  a = u;
}

// The lane's pairs turned, cosine and sine of two in each of cs[0..4).
template <bool INTER>
__device__ __forceinline__ void turn16(float* x, const float4* cs, bool first_run, bool second_run) {
  if (!INTER) {                  // both or none
    if (first_run) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        turn2(x[2 * j], x[8 + 2 * j], cs[j].x, cs[j].y);
        turn2(x[2 * j + 1], x[9 + 2 * j], cs[j].z, cs[j].w);
      }
    }
  } else {
    if (first_run) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        turn2(x[4 * j], x[4 * j + 1], cs[j].x, cs[j].y);
        turn2(x[4 * j + 2], x[4 * j + 3], cs[j].z, cs[j].w);
      }
    }
    if (second_run) {
#pragma unroll
      for (int j = 2; j < 4; ++j) {
        turn2(x[4 * j], x[4 * j + 1], cs[j].x, cs[j].y);
        turn2(x[4 * j + 2], x[4 * j + 3], cs[j].z, cs[j].w);
      }
    }
  }
}

// One wave: 8 heads of one kind.  Its lanes compute the cosines and sines of the tokens' positions, a pair each, and hand them over
// through LDS.  The loads go out first, what is small and wanted first in front.
template <int MODE, bool BF16, bool INTER, int STREAM>
__global__ __launch_bounds__(kRowThreads) void rows_kernel(const RowsArgs a) {
  constexpr bool kStreamLoads = STREAM >= 1, kStreamStores = STREAM >= 2;
  extern __shared__ float4 lds_cs[][4][8];              // [wave and token] and what entry_of says; behind that the heads whose runs change lanes
  const uint32_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * a.block_waves + threadIdx.x / 64);
  if (wave >= a.n_waves) return;
  const Place place = place_of(a.deal, a.group_log2, a.group_waves, wave);
  const Deal deal = place.deal;
  const int kind = place.kind, h0 = place.head;
  const int at_once = kWaveHeads >> deal.tokens_log2;
  const int64_t token0 = a.first + place.token;
  if (token0 >= a.end) return;
  const int tokens = (int)min((int64_t)1 << deal.tokens_log2, a.end - token0);

  const int lane = threadIdx.x & 63, l = lane & 7;
  const int sub = (lane >> 3) >> (3 - deal.tokens_log2), g = (lane >> 3) & (at_once - 1);      // token and head of the lane
  const bool there = sub < tokens && h0 + g < deal.heads;
  const int2 at = make_int2(8 * l, 64 + 8 * l);
  const float* weight = MODE == kMove ? nullptr : a.weight[kind];
  const bool any_turn = a.rot_lanes && kind != kV;
  const bool turns = any_turn && (INTER ? l < 2 * a.rot_lanes : l < a.rot_lanes), turns_too = INTER ? any_turn && l + 8 < 2 * a.rot_lanes : turns;
  const bool swap = !INTER && any_turn && a.rot_lanes < 8;
  const int2 runs = swap ? paired_runs(l, a.rot_lanes) : at;

  uint64_t step = 0;
  if (any_turn && lane < 8 * a.rot_lanes) step = a.steps[lane];
  int32_t row_in = 0, row_out = -1;
  if (MODE != kDense && deal.tokens_log2 == 0) {             // (by scalar loads)
    if (MODE == kMove) row_in = a.src[token0];
    if (kind != kQ) row_out = a.dst[token0];
  } else if (MODE != kDense && there) {
    if (MODE == kMove) row_in = a.src[token0 + sub];
    if (kind != kQ) row_out = a.dst[token0 + sub];
  }
  float w[16];
  if (weight) {
    __builtin_memcpy(w, weight + runs.x, 32);
    __builtin_memcpy(w + 8, weight + runs.y, 32);
  }
  if (MODE == kMove && (uint32_t)row_in >= (uint32_t)a.n_pool_rows) row_in = 0, row_out = -1;
  Lane16<BF16> raw;
  if (there) {
    const char* in = a.in[kind] + h0 * a.head[kind] + g * a.head[kind];
    raw.template load<kStreamLoads>(in + (MODE == kMove ? row_in * a.row[kind] : token0 * a.row[kind] + sub * a.row[kind]), at);
  }

  auto* const mine = lds_cs + ((threadIdx.x / 64) << a.group_log2);
  if (any_turn) {
    const int2 e = entry_of<INTER>(lane);
    for (int i = 0; i < tokens; ++i) {
      float c, s;
      cos_sin((uint64_t)(int64_t)a.pos[token0 + i] * step, c, s);
      ((float2*)&mine[i][e.x][e.y])[lane & 1] = make_float2(c * a.factor, s * a.factor);
    }
    wave_fence();
  }
  if (!there) return;
  uint4 lo, hi;
  char* const head = (char*)(lds_cs + (a.block_waves << a.group_log2)) + threadIdx.x / 8 * (kHeadDim * (BF16 ? 2 : 4));
  if (swap) raw.exchange(head, at, runs);
  if (BF16 && !weight && !any_turn) {       // values keep their bits
    lo = raw.u[0];
    hi = raw.u[1];
  } else {
    float x[16];
    raw.values(x);
    if (weight) norm16(raw, x, a.eps, w);
    if (turns) {
      float4 cs[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) cs[j] = mine[sub][j][l];
      turn16<INTER>(x, cs, turns, turns_too);
      lo = narrow(x);
      hi = narrow(x + 8);
    } else {
      lo = narrow(x);
      hi = narrow(x + 8);
    }
    if (swap) {
      Lane16<true> y = {{lo, hi}};
      y.exchange(head, runs, at);
      lo = y.u[0];
      hi = y.u[1];
    }
  }
  if (MODE != kMove && a.out[kind]) {
    uint16_t* p = a.out[kind] + ((token0 + sub) * deal.heads + h0 + g) * kHeadDim;
    put16<kStreamStores>(p + at.x, lo);
    put16<kStreamStores>(p + at.y, hi);
  }
  if (MODE != kDense && (uint32_t)row_out < (uint32_t)a.n_pool_rows) {
    uint16_t* p = a.pool[kind] + ((int64_t)row_out * deal.heads + h0 + g) * kHeadDim;
    put16<kStreamStores>(p + at.x, lo);
    put16<kStreamStores>(p + at.y, hi);
  }
}

// Deals the heads of queries, keys and values and launches; `bytes`: what the call reads and writes.
template <int MODE>
static tl_status launch(RowsArgs& a, const int32_t (&heads)[3], int32_t n, bool bf16, bool interleaved, int64_t bytes, hipStream_t stream) {
  const Dealing dealing = deal_heads(heads);
  for (int i = 0; i < 3; ++i) a.deal[i] = dealing.kind[i];
  a.group_log2 = dealing.group_log2;
  a.group_waves = dealing.group_waves;
  const auto pick = [&](auto is_bf16, auto stream_mode) {
    return interleaved ? rows_kernel<MODE, is_bf16.value, true, stream_mode.value> : rows_kernel<MODE, is_bf16.value, false, stream_mode.value>;
  };
  const auto pick_stream = [&](auto is_bf16) {
    return bytes >= kStreamAll ? pick(is_bf16, std::integral_constant<int, 2>())
                               : bytes >= kStreamIn ? pick(is_bf16, std::integral_constant<int, 1>()) : pick(is_bf16, std::integral_constant<int, 0>());
  };
  const auto kernel = bf16 || MODE == kMove ? pick_stream(std::true_type()) : pick_stream(std::bool_constant<MODE == kMove>());
  // (workgroups of one wave for moves of more than the cache: 131072 rows of 8 heads 179 us, in ones of four 200; 65536 90 and 95; 33000, the first
  // behind the line, 46.3 and 46.8.  Below it 24000 rows 35.2 and 36.4, 16000 24.2 and 25.7, 8000 and fewer the same within 3 %: fours there too, for
  // one line with the stores' way.  Rotations and writes of 1 to 8000 tokens and of 100 to 470 MB are the same within 4 % but for 16 tokens, 2.9 and
  // 3.1, and writes of 200 MB, 31.8 and 33.9: fours.)
  a.block_waves = MODE == kMove && bytes >= kStreamAll ? 1 : kRowThreads / 64;
  const size_t lds = a.block_waves * ((512 << a.group_log2) + (!interleaved && a.rot_lanes % 8 ? kWaveHeads * kHeadDim * (bf16 ? 2 : 4) : 0));
  const int64_t most = most_groups(dealing), groups = ((int64_t)n + (1 << a.group_log2) - 1) >> a.group_log2;
  for (int64_t done = 0; done < groups; done += most) {
    const int64_t m = groups - done < most ? groups - done : most;
    a.first = done << a.group_log2;
    a.end = (done + m) << a.group_log2 < n ? (done + m) << a.group_log2 : n;
    a.n_waves = (uint32_t)(m * a.group_waves.d);
    hipLaunchKernelGGL(kernel, dim3((a.n_waves + a.block_waves - 1) / a.block_waves), dim3(a.block_waves * 64), lds, stream, a);
  }
  TL_HIP(hipGetLastError());
  return TL_OK;
}

static tl_status check_rope(const char* who, const tl_rope* rope) {
  if (!rope) return TL_OK;
  if (rope->rot_dim < 16 || rope->rot_dim > kHeadDim || rope->rot_dim % 16)
    TL_FAIL(TL_EINVAL, "%s: rot_dim must be a multiple of 16 from 16 to %d, is %d", who, kHeadDim, rope->rot_dim);
  if (!rope->steps_dev) TL_FAIL(TL_EINVAL, "%s: null steps", who);
  if (!std::isfinite(rope->factor)) TL_FAIL(TL_EINVAL, "%s: the rotation's factor is not finite", who);
  return TL_OK;
}

namespace {
struct Span {                  // bytes [lo, hi) that a tensor lies in
  __int128 lo, hi;
};
}  // namespace

static Span dense_span(const void* p, int64_t n, int64_t heads) {
  const __int128 lo = (__int128)(uintptr_t)p;
  return {lo, lo + (__int128)n * heads * kHeadDim * 2};
}
static bool meet(const Span& x, const Span& y) { return x.lo < y.hi && y.lo < x.hi; }

// One input with its dense output (either may be absent), its strides in elements.
struct Rows {
  const char* name;
  const void* in;
  int64_t row, head;
  int32_t heads;
  void* out;
};

static tl_status check_rows(const char* who, const tl_qkv* d, int64_t n, const tl_pool* pool, Rows (&t)[3]) {
  if (!d) TL_FAIL(TL_EINVAL, "%s: null rows", who);
  t[0] = {"q", d->q, d->q_row_stride, d->q_head_stride, d->q_heads, d->q_out};
  t[1] = {"k", d->k, d->k_row_stride, d->k_head_stride, d->kv_heads, d->k_out};
  t[2] = {"v", d->v, d->v_row_stride, d->v_head_stride, d->kv_heads, d->v_out};
  if (!d->q && !d->k && !d->v) TL_FAIL(TL_EINVAL, "%s: no rows", who);
  const int64_t size = d->is_bf16 ? 2 : 4;
  Span in[3];
  for (int i = 0; i < 3; ++i) {
    Rows& x = t[i];
    if (!x.in) {
      if (x.out) TL_FAIL(TL_EINVAL, "%s: an output for %s without %s", who, x.name, x.name);
      continue;
    }
    if (x.heads <= 0 || x.heads > kMostHeads) TL_FAIL(TL_EINVAL, "%s: %d heads of %s", who, x.heads, x.name);
    if (!x.out && !(pool && i > 0)) TL_FAIL(TL_EINVAL, "%s: %s without an output", who, x.name);
    if (x.row > INT64_MAX / 8 || x.row < INT64_MIN / 8 || x.head > INT64_MAX / 8 || x.head < INT64_MIN / 8)
      TL_FAIL(TL_EINVAL, "%s: strides of %s", who, x.name);
    if (x.heads == 1) x.head = kHeadDim;                       // strides of a single head or token are never taken
    if (n == 1) x.row = (int64_t)x.heads * kHeadDim;
    const __int128 rows = (__int128)(n - 1) * x.row * size, heads = (__int128)(x.heads - 1) * x.head * size;
    const __int128 base = (__int128)(uintptr_t)x.in;
    in[i] = {base + (rows < 0 ? rows : 0) + (heads < 0 ? heads : 0), base + (rows > 0 ? rows : 0) + (heads > 0 ? heads : 0) + kHeadDim * size};
    if (in[i].lo < 0 || in[i].hi > (__int128)1 << 57) TL_FAIL(TL_EINVAL, "%s: strides of %s lead out of the address space", who, x.name);
  }
  for (int i = 0; i < 3; ++i) {
    if (!t[i].out) continue;
    const Span out = dense_span(t[i].out, n, t[i].heads);
    for (int j = 0; j < 3; ++j) {
      if (j < i && t[j].out && meet(out, dense_span(t[j].out, n, t[j].heads)))
        TL_FAIL(TL_EINVAL, "%s: the outputs of %s and %s overlap", who, t[j].name, t[i].name);
      // in place: every value is read by the lane that writes it
      const bool same = i == j && d->is_bf16 && t[i].in == t[i].out && t[i].row == (int64_t)t[i].heads * kHeadDim && t[i].head == kHeadDim;
      if (t[j].in && !same && meet(out, in[j])) TL_FAIL(TL_EINVAL, "%s: the output of %s overlaps %s", who, t[i].name, t[j].name);
    }
  }
  if (pool) {
    const int64_t rows = (int64_t)pool->n_slots * pool->seg_len;
    const Span slots[2] = {dense_span(pool->k_dev, rows, pool->kv_heads), dense_span(pool->v_dev, rows, pool->kv_heads)};
    for (int i = 0; i < 3; ++i)
      for (int j = 0; j < 2; ++j)
        if ((t[i].in && meet(in[i], slots[j])) || (t[i].out && meet(dense_span(t[i].out, n, t[i].heads), slots[j])))
          TL_FAIL(TL_EINVAL, "%s: %s lies in the pool's slots", who, t[i].name);
  }
  if ((d->q_weight && d->q) || (d->k_weight && d->k)) {
    if (!(d->eps >= 0x1p-126f) || !std::isfinite(d->eps)) TL_FAIL(TL_EINVAL, "%s: eps must be a positive normal number", who);
  }
  return TL_OK;
}

static tl_status launch_rows(const char* who, const tl_rope* rope, const tl_qkv* d, const int32_t* pos_dev, const tl_pool* pool,
                             const int32_t* pool_rows_dev, int32_t n, void* stream) {
  Rows t[3];
  tl_status st = check_rope(who, rope);
  if (st == TL_OK) st = check_rows(who, d, n, pool, t);
  if (st != TL_OK) return st;
  if (rope && !pos_dev && (d->q || d->k)) TL_FAIL(TL_EINVAL, "%s: null positions", who);
  const int64_t size = d->is_bf16 ? 2 : 4;
  RowsArgs a{};
  int32_t heads[3];
  for (int i = 0; i < 3; ++i) {
    a.in[i] = (const char*)t[i].in;
    a.row[i] = t[i].row * size;
    a.head[i] = t[i].head * size;
    a.out[i] = (uint16_t*)t[i].out;
    heads[i] = t[i].in ? t[i].heads : 0;
  }
  a.weight[kQ] = d->q ? d->q_weight : nullptr;
  a.weight[kK] = d->k ? d->k_weight : nullptr;
  a.eps = d->eps;
  a.pos = pos_dev;
  if (rope) {
    a.steps = rope->steps_dev;
    a.factor = rope->factor;
    a.rot_lanes = rope->rot_dim / 16;
  }
  const bool interleaved = rope && rope->interleaved;
  int64_t head_bytes = 0;
  for (int i = 0; i < 3; ++i) head_bytes += heads[i] * (size + (t[i].out ? 2 : 0) + (pool && i != kQ ? 2 : 0)) * kHeadDim;
  const int64_t bytes = head_bytes * n;
  if (!pool) return launch<kDense>(a, heads, n, d->is_bf16 != 0, interleaved, bytes, (hipStream_t)stream);
  a.pool[kK] = (uint16_t*)pool->k_dev, a.pool[kV] = (uint16_t*)pool->v_dev;
  a.dst = pool_rows_dev;
  a.n_pool_rows = pool->n_slots * pool->seg_len;
  return launch<kToPool>(a, heads, n, d->is_bf16 != 0, interleaved, bytes, (hipStream_t)stream);
}

// 1 / 2 pi, from its first bit behind the point on.
static const uint64_t kTurns[19] = {
    0x28be60db9391054aull, 0x7f09d5f47d4d3770ull, 0x36d8a5664f10e410ull, 0x7f9458eaf7aef158ull, 0x6dc91b8e909374b8ull,
    0x01924bba82746487ull, 0x3f877ac72c4a69cfull, 0xba208d7d4baed121ull, 0x3a671c09ad17df90ull, 0x4e64758e60d4ce7dull,
    0x272117e2ef7e4a0eull, 0xc7fe25fff7816603ull, 0xfbcbc462d6829b47ull, 0xdb4d9fb3c9f2c26dull, 0xd3d18fd9a797fa8bull,
    0x5d49eeb1faf97c5eull, 0xcf41ce7de294a4baull, 0x9afed7ec47e35742ull, 0x1580cc11bf1edaeaull};

// 64 of its bits, those of weight 2^-(at + 1) and below.
static uint64_t turns_bits(int at) {
  if (at <= -64 || at >= 19 * 64) return 0;
  if (at < 0) return kTurns[0] >> -at;
  const int i = at / 64, r = at % 64;
  return r == 0 ? kTurns[i] : kTurns[i] << r | (i + 1 < 19 ? kTurns[i + 1] >> (64 - r) : 0);
}

// Radians as a fraction of a turn times 2^64, modulo 2^64, to the nearest: |radians| = m 2^e with a whole m below 2^53, times those bits of
// 2^(64 + e) / 2 pi that count: 64 in front of the point (m times the others is a multiple of 2^64) and 128 behind it (the others
// are below 2^-75 together).  Payne and Hanek's reduction (Radian reduction for trigonometric functions, 1983), to turns in place of quarters.
static uint64_t step_of(double radians) {
  int e;
  const uint64_t m = (uint64_t)ldexp(frexp(fabs(radians), &e), 53);
  const int at = 64 + e - 53 - 64;
  typedef unsigned __int128 u128;
  const u128 low = (u128)m * turns_bits(at + 64) + (uint64_t)((u128)m * turns_bits(at + 128) >> 64);
  const uint64_t step = m * turns_bits(at) + (uint64_t)(low >> 64) + ((uint64_t)low >> 63);
  return radians < 0 ? 0 - step : step;
}

}  // namespace tl

using namespace tl;

extern "C" {

tl_status tl_rope_steps(const double* inv_freq, int32_t n, uint64_t* steps_out) {
  if (n < 0 || (n > 0 && (!inv_freq || !steps_out))) TL_FAIL(TL_EINVAL, "tl_rope_steps: bad argument");
  for (int32_t i = 0; i < n; ++i)
    if (!std::isfinite(inv_freq[i])) TL_FAIL(TL_EINVAL, "tl_rope_steps: frequency %d is not finite", i);
  for (int32_t i = 0; i < n; ++i) steps_out[i] = step_of(inv_freq[i]);
  return TL_OK;
}

tl_status tl_rotate_rows(const tl_rope* rope, const tl_qkv* rows, const int32_t* pos_dev, int32_t n_tokens, void* stream) {
  if (n_tokens == 0) return TL_OK;
  if (n_tokens < 0) TL_FAIL(TL_EINVAL, "tl_rotate_rows: negative number of tokens");
  return launch_rows("tl_rotate_rows", rope, rows, pos_dev, nullptr, nullptr, n_tokens, stream);
}

tl_status tl_pool_write_rows(tl_pool* pool, const tl_rope* rope, const tl_qkv* rows, const int32_t* pos_dev, const int32_t* pool_rows_dev,
                             int32_t n_tokens, void* stream) {
  if (n_tokens == 0) return TL_OK;
  if (!pool) TL_FAIL(TL_EINVAL, "tl_pool_write_rows: null pool");
  if (n_tokens < 0) TL_FAIL(TL_EINVAL, "tl_pool_write_rows: negative number of tokens");
  if (!rows || !rows->k || !rows->v) TL_FAIL(TL_EINVAL, "tl_pool_write_rows: null keys or values");
  if (rows->kv_heads != pool->kv_heads)
    TL_FAIL(TL_EINVAL, "tl_pool_write_rows: rows of %d heads, the pool has %d", rows->kv_heads, pool->kv_heads);
  if (!pool_rows_dev) TL_FAIL(TL_EINVAL, "tl_pool_write_rows: null pool rows");
  return launch_rows("tl_pool_write_rows", rope, rows, pos_dev, pool, pool_rows_dev, n_tokens, stream);
}

tl_status tl_pool_move_rows(tl_pool* pool, const tl_rope* rope, const int32_t* src_rows_dev, const int32_t* dst_rows_dev,
                            const int32_t* shift_dev, int32_t n_rows, void* stream) {
  if (n_rows == 0) return TL_OK;
  if (!pool) TL_FAIL(TL_EINVAL, "tl_pool_move_rows: null pool");
  if (pool->kv_heads > kMostHeads) TL_FAIL(TL_EINVAL, "tl_pool_move_rows: %d heads", pool->kv_heads);
  if (n_rows < 0) TL_FAIL(TL_EINVAL, "tl_pool_move_rows: negative number of rows");
  const tl_status st = check_rope("tl_pool_move_rows", rope);
  if (st != TL_OK) return st;
  if (!src_rows_dev || !dst_rows_dev || (rope && !shift_dev)) TL_FAIL(TL_EINVAL, "tl_pool_move_rows: null rows or shifts");
  RowsArgs a{};
  const int32_t heads[3] = {0, pool->kv_heads, pool->kv_heads};
  a.in[kK] = (const char*)pool->k_dev, a.in[kV] = (const char*)pool->v_dev;
  a.pool[kK] = (uint16_t*)pool->k_dev, a.pool[kV] = (uint16_t*)pool->v_dev;
  for (int i = kK; i <= kV; ++i) a.head[i] = kHeadDim * 2, a.row[i] = pool->kv_heads * a.head[i];
  a.src = src_rows_dev, a.dst = dst_rows_dev, a.pos = shift_dev;
  if (rope) {
    a.steps = rope->steps_dev;
    a.factor = 1.f;
    a.rot_lanes = rope->rot_dim / 16;
  }
  a.n_pool_rows = pool->n_slots * pool->seg_len;
  return launch<kMove>(a, heads, n_rows, true, rope && rope->interleaved, (int64_t)n_rows * pool->kv_heads * (8 * kHeadDim), (hipStream_t)stream);
}

}  // extern "C"
