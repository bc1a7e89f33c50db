// Rows on their way between a layer's projection and the attention: norms of queries and keys for each head, position rotation,
// writes to the pool's slots, and rows of the pool that move to other positions.
//
// Mathematics.  One head's 128 values x of one token:
//   norm      y = x w / sqrt(mean(x^2) + eps)
//   rotation  pair (a, b) of frequency f at position p: a' = m (a cos pf - b sin pf), b' = m (a sin pf + b cos pf)
// rounded once, to bf16, at the end.  The angle is never a float: f / 2 pi is a 64-bit fraction of a turn, and p times it modulo
// 2^64 is the phase of every 32-bit position of either sign to 2^-33 of a turn, without a table.
//
// What bounds it: every value is read once and written once, about ten operations each, so HBM, and at a few tokens the launch.
#include <cmath>

#include "attn_common.h"

namespace tl {

constexpr int kRowThreads = 256;
constexpr int kMostHeads = 1 << 16;
constexpr int kWaveHeads = 8;            // heads that a wave takes at once: 8 lanes with 16 values each to a head

struct RowsArgs {
  const char *q, *k, *v;                 // null: not there
  int64_t q_row, q_head, k_row, k_head, v_row, v_head;   // strides in bytes
  uint16_t *q_out, *k_out, *v_out;       // dense, or null
  uint16_t *pool_k, *pool_v;
  const int32_t* pool_rows;
  const float *q_weight, *k_weight;      // null: no norm
  const int32_t* pos;
  const uint64_t* steps;                 // null: no rotation
  float eps, factor;
  int32_t n_pool_rows;
  int32_t q_heads, k_heads, heads;       // heads = all that a token has, in the order q, k, v
  int32_t rot_lanes, interleaved;        // rot_lanes = rot_dim / 16: lanes of a head whose values turn
  uint32_t first, n_waves, wave_blocks;  // wave_blocks = waves that a token has
};

struct MoveArgs {
  uint16_t *pool_k, *pool_v;
  const int32_t *src, *dst, *shift;
  const uint64_t* steps;
  int32_t n_pool_rows, kv_heads, rot_lanes, interleaved;
  uint32_t first, n_waves, wave_blocks;
};

// 16 bytes from or to any address
__device__ __forceinline__ uint4 get16(const char* p) {
  uint4 x;
  __builtin_memcpy(&x, p, sizeof(x));
  return x;
}
__device__ __forceinline__ void put16(uint16_t* p, uint4 x) { __builtin_memcpy(p, &x, sizeof(x)); }

__device__ __forceinline__ void widen(uint4 u, float* x) {
  const unsigned w[4] = {u.x, u.y, u.z, u.w};
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __builtin_bit_cast(float, w[i] << 16);
    x[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ uint4 narrow(const float* x) {
  return __builtin_bit_cast(uint4, pack_bf16x8(x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]));
}

// cos and sin of a phase (2^64 = one turn).  Quarter turns are taken off the integer; what is left, at most an eighth of a
// turn, is exact to 2^-25 of itself, and the power series up to x^9 and x^8 are off by 2e-9 and 2.5e-8 there.
__device__ __forceinline__ void cos_sin(uint64_t phase, float& c, float& s) {
  const uint32_t t = (uint32_t)(phase >> 32);
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

// x[16] of the lane, normed.  A sum of squares beyond 32 bits (rows that large mean something is wrong upstream, but their norm
// is an ordinary number) is taken again of the values times 2^-70.
__device__ __forceinline__ void norm16(float* x, float eps, const float* w0, const float* w1) {
  float ss = 0;
  for (int i = 0; i < 16; ++i) ss += x[i] * x[i];
  ss = sum8(ss);
  if (__builtin_expect(ss > 3.4e38f, 0)) {
    ss = 0;
    for (int i = 0; i < 16; ++i) {
      x[i] *= 0x1p-70f;
      ss += x[i] * x[i];
    }
    ss = sum8(ss);
    eps = 0;
  }
  const float r = __builtin_amdgcn_rsqf(ss * (1.f / kHeadDim) + eps);
  for (int i = 0; i < 8; ++i) {
    x[i] = x[i] * r * w0[i];
    x[8 + i] = x[8 + i] * r * w1[i];
  }
}

// x[16] of the lane, turned: pairs 8 l .. 8 l + 7 of the head, c and s theirs.
__device__ __forceinline__ void turn16(float* x, bool interleaved, const float* c, const float* s) {
  if (interleaved) {
    for (int i = 0; i < 8; ++i) {
      const float a = x[2 * i], b = x[2 * i + 1];
      x[2 * i] = a * c[i] - b * s[i];
      x[2 * i + 1] = a * s[i] + b * c[i];
    }
  } else {
    for (int i = 0; i < 8; ++i) {
      const float a = x[i], b = x[8 + i];
      x[i] = a * c[i] - b * s[i];
      x[8 + i] = a * s[i] + b * c[i];
    }
  }
}

// Where the two runs of 8 values of lane l of a head begin.  Lanes whose values turn against each other from afar (i with
// i + rot_dim / 2) hold one run of each half of the turning dimensions, so that both of a pair are in one lane; others 16 in a row.
__device__ __forceinline__ int2 runs_of(int l, int rot_lanes, int interleaved) {
  return !interleaved && l < rot_lanes ? make_int2(8 * l, 8 * (rot_lanes + l)) : make_int2(16 * l, 16 * l + 8);
}

__device__ __forceinline__ void cos_sin8(const uint64_t* steps, int l, int64_t p, float factor, float* c, float* s) {
  for (int i = 0; i < 8; ++i) {
    cos_sin((uint64_t)p * steps[8 * l + i], c[i], s[i]);
    c[i] *= factor;
    s[i] *= factor;
  }
}

// One wave: 8 heads of one token.
template <bool BF16, bool TO_POOL>
__global__ __launch_bounds__(kRowThreads) void rotate_rows_kernel(const RowsArgs a) {
  const uint32_t wave = blockIdx.x * (kRowThreads / 64) + threadIdx.x / 64;
  if (wave >= a.n_waves) return;
  const uint32_t in_launch = wave / a.wave_blocks;
  const int64_t token = (int64_t)a.first + in_launch;
  const int lane = threadIdx.x & 63, l = lane & 7;
  int h = (int)(wave - in_launch * a.wave_blocks) * kWaveHeads + lane / 8;
  if (h >= a.heads) return;
  const bool is_q = h < a.q_heads, is_v = h >= a.q_heads + a.k_heads;
  const char* src;
  uint16_t *out, *slots = nullptr;
  const float* weight = nullptr;
  int64_t out_row;
  if (is_q) {
    src = a.q + token * a.q_row + h * a.q_head;
    out = a.q_out;
    out_row = a.q_heads;
    weight = a.q_weight;
  } else {
    h -= a.q_heads;
    out_row = a.k_heads ? a.k_heads : a.heads - a.q_heads;
    if (!is_v) {
      src = a.k + token * a.k_row + h * a.k_head;
      out = a.k_out;
      slots = a.pool_k;
      weight = a.k_weight;
    } else {
      h -= a.k_heads;
      src = a.v + token * a.v_row + h * a.v_head;
      out = a.v_out;
      slots = a.pool_v;
    }
  }
  const int2 at = runs_of(l, a.steps ? a.rot_lanes : 0, a.interleaved);
  uint4 lo, hi;
  if (is_v && BF16) {                       // values keep their bits
    lo = get16(src + 2 * at.x);
    hi = get16(src + 2 * at.y);
  } else {
    float x[16];
    if (BF16) {
      widen(get16(src + 2 * at.x), x);
      widen(get16(src + 2 * at.y), x + 8);
    } else {
      for (int i = 0; i < 2; ++i) {
        __builtin_memcpy(x + 4 * i, src + 4 * at.x + 16 * i, 16);
        __builtin_memcpy(x + 8 + 4 * i, src + 4 * at.y + 16 * i, 16);
      }
    }
    if (weight) {
      float w0[8], w1[8];
      for (int i = 0; i < 8; ++i) w0[i] = weight[at.x + i], w1[i] = weight[at.y + i];
      norm16(x, a.eps, w0, w1);
    }
    if (!is_v && a.steps && l < a.rot_lanes) {
      float c[8], s[8];
      cos_sin8(a.steps, l, a.pos[token], a.factor, c, s);
      turn16(x, a.interleaved, c, s);
    }
    lo = narrow(x);
    hi = narrow(x + 8);
  }
  if (out) {
    uint16_t* p = out + (token * out_row + h) * kHeadDim;
    put16(p + at.x, lo);
    put16(p + at.y, hi);
  }
  if (TO_POOL && slots) {
    const int32_t row = a.pool_rows[token];
    if ((uint32_t)row < (uint32_t)a.n_pool_rows) {
      uint16_t* p = slots + ((int64_t)row * out_row + h) * kHeadDim;
      put16(p + at.x, lo);
      put16(p + at.y, hi);
    }
  }
}

// One wave: 8 of a pool row's 2 kv_heads heads, keys first.
__global__ __launch_bounds__(kRowThreads) void move_rows_kernel(const MoveArgs a) {
  const uint32_t wave = blockIdx.x * (kRowThreads / 64) + threadIdx.x / 64;
  if (wave >= a.n_waves) return;
  const uint32_t in_launch = wave / a.wave_blocks;
  const int64_t entry = (int64_t)a.first + in_launch;
  const int lane = threadIdx.x & 63, l = lane & 7;
  int h = (int)(wave - in_launch * a.wave_blocks) * kWaveHeads + lane / 8;
  if (h >= 2 * a.kv_heads) return;
  const bool is_v = h >= a.kv_heads;
  if (is_v) h -= a.kv_heads;
  const int32_t src = a.src[entry], dst = a.dst[entry];
  if ((uint32_t)src >= (uint32_t)a.n_pool_rows || (uint32_t)dst >= (uint32_t)a.n_pool_rows) return;
  uint16_t* pool = is_v ? a.pool_v : a.pool_k;
  const uint16_t* from = pool + ((int64_t)src * a.kv_heads + h) * kHeadDim;
  uint16_t* to = pool + ((int64_t)dst * a.kv_heads + h) * kHeadDim;
  const int2 at = runs_of(l, a.steps ? a.rot_lanes : 0, a.interleaved);
  uint4 lo = get16((const char*)(from + at.x)), hi = get16((const char*)(from + at.y));
  if (!is_v && a.steps && l < a.rot_lanes) {
    float x[16], c[8], s[8];
    widen(lo, x);
    widen(hi, x + 8);
    cos_sin8(a.steps, l, a.shift[entry], 1.f, c, s);
    turn16(x, a.interleaved, c, s);
    lo = narrow(x);
    hi = narrow(x + 8);
  }
  put16(to + at.x, lo);
  put16(to + at.y, hi);
}

// Tokens of one launch: the grid stays below 2^31 threads and wave numbers below 2^26.
static uint32_t launch_tokens(uint32_t wave_blocks) {
  const uint32_t n = (1u << 25) / wave_blocks;
  return n ? n : 1;
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

// One input with its dense output (either may be absent), its strides in bytes; `span` its bytes.
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
  a.q = (const char*)d->q, a.k = (const char*)d->k, a.v = (const char*)d->v;
  a.q_row = t[0].row * size, a.q_head = t[0].head * size;
  a.k_row = t[1].row * size, a.k_head = t[1].head * size;
  a.v_row = t[2].row * size, a.v_head = t[2].head * size;
  a.q_out = (uint16_t*)d->q_out, a.k_out = (uint16_t*)d->k_out, a.v_out = (uint16_t*)d->v_out;
  a.q_weight = d->q_weight, a.k_weight = d->k_weight;
  a.eps = d->eps;
  a.pos = pos_dev;
  if (rope) {
    a.steps = rope->steps_dev;
    a.factor = rope->factor;
    a.rot_lanes = rope->rot_dim / 16;
    a.interleaved = rope->interleaved != 0;
  }
  a.q_heads = d->q ? d->q_heads : 0;
  a.k_heads = d->k ? d->kv_heads : 0;
  a.heads = a.q_heads + a.k_heads + (d->v ? d->kv_heads : 0);
  if (pool) {
    a.pool_k = (uint16_t*)pool->k_dev, a.pool_v = (uint16_t*)pool->v_dev;
    a.pool_rows = pool_rows_dev;
    a.n_pool_rows = pool->n_slots * pool->seg_len;
  }
  a.wave_blocks = (uint32_t)(a.heads + kWaveHeads - 1) / kWaveHeads;
  const uint32_t most = launch_tokens(a.wave_blocks);
  for (uint32_t first = 0; first < (uint32_t)n; first += most) {
    const uint32_t m = (uint32_t)n - first < most ? (uint32_t)n - first : most;
    a.first = first;
    a.n_waves = m * a.wave_blocks;
    const dim3 grid((a.n_waves + kRowThreads / 64 - 1) / (kRowThreads / 64)), block(kRowThreads);
    const auto kernel = d->is_bf16 ? (pool ? rotate_rows_kernel<true, true> : rotate_rows_kernel<true, false>)
                                   : (pool ? rotate_rows_kernel<false, true> : rotate_rows_kernel<false, false>);
    hipLaunchKernelGGL(kernel, grid, block, 0, (hipStream_t)stream, a);
  }
  TL_HIP(hipGetLastError());
  return TL_OK;
}

}  // namespace tl

using namespace tl;

extern "C" {

tl_status tl_rope_steps(const double* inv_freq, int32_t n, uint64_t* steps_out) {
  if (n < 0 || (n > 0 && (!inv_freq || !steps_out))) TL_FAIL(TL_EINVAL, "tl_rope_steps: bad argument");
  for (int32_t i = 0; i < n; ++i)
    if (!std::isfinite(inv_freq[i])) TL_FAIL(TL_EINVAL, "tl_rope_steps: frequency %d is not finite", i);
  // (the host's long double has 64 bits of mantissa: the step is off by less than 2^-63 of itself)
  const long double two_pi = 6.283185307179586476925286766559005768L;
  for (int32_t i = 0; i < n; ++i) {
    const long double turns = (long double)inv_freq[i] / two_pi, part = turns - floorl(turns);
    const long double scaled = rintl(ldexpl(part, 64));
    steps_out[i] = scaled >= 0x1p64L ? 0 : (uint64_t)scaled;
  }
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
  MoveArgs a{};
  a.pool_k = (uint16_t*)pool->k_dev, a.pool_v = (uint16_t*)pool->v_dev;
  a.src = src_rows_dev, a.dst = dst_rows_dev, a.shift = shift_dev;
  if (rope) {
    a.steps = rope->steps_dev;
    a.rot_lanes = rope->rot_dim / 16;
    a.interleaved = rope->interleaved != 0;
  }
  a.n_pool_rows = pool->n_slots * pool->seg_len;
  a.kv_heads = pool->kv_heads;
  a.wave_blocks = (uint32_t)(2 * a.kv_heads + kWaveHeads - 1) / kWaveHeads;
  const uint32_t most = launch_tokens(a.wave_blocks);
  for (uint32_t first = 0; first < (uint32_t)n_rows; first += most) {
    const uint32_t m = (uint32_t)n_rows - first < most ? (uint32_t)n_rows - first : most;
    a.first = first;
    a.n_waves = m * a.wave_blocks;
    hipLaunchKernelGGL(move_rows_kernel, dim3((a.n_waves + kRowThreads / 64 - 1) / (kRowThreads / 64)), dim3(kRowThreads), 0,
                       (hipStream_t)stream, a);
  }
  TL_HIP(hipGetLastError());
  return TL_OK;
}

}  // extern "C"
