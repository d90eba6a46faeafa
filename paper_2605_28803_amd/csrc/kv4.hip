// Key/value cache in 4 bits: append, gather and attention over its pages.
//
// A cached row (one token and kv head, head_dim = d channels) is quantized as
// a token is (eq:scale, eq:quant): Delta = max|x| / 7, q = clamp(rne(7 x /
// max|x|), -7, 7), the value it stands for q Delta.  Keys may be rotated by
// H_d / sqrt(d) first (eq:blockdiag with one block per head): the query is
// rotated alike, so q . k is unchanged, and the outlier channels that keys have
// no longer set the step.  A rotation of the values folds into the value and
// output projections offline, as U and P do.
//
// Layout, per page and head (page_tokens tokens, a multiple of 32):
//   k_codes [token][d / 2]: byte b holds channels 2 b (low nibble), 2 b + 1;
//   v_codes [token / 16][d / 2][16]: byte (b, t) holds channels 2 b and 2 b + 1
//     of token t of the 16, so a token's write is whole bytes (no neighbour
//     shares one) and the second product's operand, 8 tokens of a channel, is
//     two words;
//   k_scale, v_scale fp32 [token].
#include <cmath>

#include "common.h"
#include "rq_device.h"

namespace oq {
namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));

using rqd::lane_xor_far;

struct Cache {
  uint8_t* kc;
  uint8_t* vc;
  float* ks;
  float* vs;
  int64_t n_slots;  // n_pages * page_tokens
  int page, hk;
};

__device__ __forceinline__ float load16(const uint16_t* p, bool bf) {
  const uint32_t b = *p;
  return bf ? __uint_as_float(b << 16) : rqd::h2f(b);
}
__device__ __forceinline__ void load8(const uint16_t* p, bool bf, float (&v)[8]) {
  const uint4 r = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = bf ? __uint_as_float(w[i] << 16) : rqd::h2f(w[i] & 0xFFFFu);
    v[2 * i + 1] = bf ? __uint_as_float(w[i] & 0xFFFF0000u) : rqd::h2f(w[i] >> 16);
  }
}
__device__ __forceinline__ uint32_t pack2(float a, float b, bool bf) {
  if (bf) {
    const __bf16 x = static_cast<__bf16>(a), y = static_cast<__bf16>(b);
    return __builtin_bit_cast(uint16_t, x) | static_cast<uint32_t>(__builtin_bit_cast(uint16_t, y)) << 16;
  }
  return rqd::f2h(a) | static_cast<uint32_t>(rqd::f2h(b)) << 16;
}

// x[0..7] of the lanes of a row (D / 8 lanes, lane j holds channels 8 j ..):
// unnormalized Sylvester butterflies over the row's channels.
template <int D, typename T>
__device__ __forceinline__ void fwht_row(T (&x)[8], int j) {
#pragma unroll
  for (int s = 1; s < 8; s *= 2)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (!(i & s)) {
        const T a = x[i], b = x[i + s];
        x[i] = a + b;
        x[i + s] = a - b;
      }
#pragma unroll
  for (int s = 1; s < D / 8; s *= 2)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const T o = __shfl_xor(x[i], s);
      x[i] = (j & s) ? o - x[i] : x[i] + o;
    }
}

// Code of one element: the integer nearest to 7 u / top, ties to even, |u| <=
// top.  7 u, q top and their difference are exact (u and top are inputs of at
// most 11 bits, or sums of up to 256 of them in fp64), so a quotient next to
// a half integer is decided exactly: the estimate is at most one off, and only
// beside a boundary.
template <typename T>
__device__ __forceinline__ int code_of(T u, T top, T inv) {
  T q = rint(u * inv);
  const T e = fma(-q, top, T(7) * u), d = T(2) * fabs(e) - top;
  const int n = static_cast<int>(q);
  const int up = e > T(0) ? 1 : -1;
  return d > T(0) || (d == T(0) && (n & 1)) ? n + up : n;
}

// ---------------------------------------------------------------------------
// Append.  D / 8 lanes take one row of K or V.  HBM bound: 4 d bytes read and
// d + 8 written per token and head.
// ---------------------------------------------------------------------------
template <int D, bool ROT>
__global__ __launch_bounds__(256) void kv4_append_kernel(Cache c, const uint16_t* K, const uint16_t* V, int64_t n,
                                                         int64_t ldk, int64_t ldv, bool bf, const int64_t* slots) {
  constexpr int LR = D / 8, RW = 256 / LR;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * RW + threadIdx.x / LR;
  const int j = threadIdx.x % LR;
  const bool is_v = blockIdx.y == 1;
  const int64_t rr = row < n * c.hk ? row : 0;  // (lanes past the end keep the exchanges whole)
  const int64_t tok = rr / c.hk;
  const int h = static_cast<int>(rr % c.hk);
  float x[8];
  load8((is_v ? V + tok * ldv : K + tok * ldk) + h * D + 8 * j, bf, x);
  int q[8];
  float scale;
  if (ROT && !is_v) {
    double u[8], top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = x[i];
    fwht_row<D>(u, j);
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmax(top, fabs(u[i]));
#pragma unroll
    for (int s = 1; s < LR; s *= 2) top = fmax(top, __shfl_xor(top, s));
    const double inv = 7.0 / top;
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = top > 0 ? code_of<double>(u[i], top, inv) : 0;
    scale = static_cast<float>(top / (7.0 * sqrt(static_cast<double>(D))));
  } else {
    float top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(x[i]));
#pragma unroll
    for (int s = 1; s < LR; s *= 2) top = fmaxf(top, __shfl_xor(top, s));
    // (Scaled by a power of two to [1, 2), so that nothing overflows.)
    const int e = top > 0 ? -ilogbf(top) : 0;
    const float t = ldexpf(top, e), inv = 7.0f / t;
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = top > 0 ? code_of<float>(ldexpf(x[i], e), t, inv) : 0;
    scale = top / 7.0f;
  }
  const int64_t slot = row < n * c.hk ? slots[tok] : -1;
  if (slot < 0 || slot >= c.n_slots) return;
  const int64_t page = slot / c.page;
  const int t = static_cast<int>(slot % c.page);
  const int64_t base = (page * c.hk + h) * c.page;  // rows of D / 2 bytes before this page's head
  uint32_t b[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) b[i] = (q[2 * i] & 15) | (q[2 * i + 1] & 15) << 4;
  if (!is_v) {
    *reinterpret_cast<uint32_t*>(c.kc + (base + t) * (D / 2) + 4 * j) = b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24;
    if (j == 0) c.ks[base + t] = scale;
  } else {
    uint8_t* o = c.vc + (base + (t & ~15)) * (D / 2) + (t & 15) + 64 * j;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[16 * i] = static_cast<uint8_t>(b[i]);
    if (j == 0) c.vs[base + t] = scale;
  }
}

// ---------------------------------------------------------------------------
// Gather: the values of cached rows (slots out of range give zeros), keys
// rotated back.
// ---------------------------------------------------------------------------
template <int D, bool ROT>
__global__ __launch_bounds__(256) void kv4_gather_kernel(Cache c, const int64_t* slots, int64_t n, void* K, void* V,
                                                         int64_t ldk, int64_t ldv, int dtype) {
  constexpr int LR = D / 8, RW = 256 / LR;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * RW + threadIdx.x / LR;
  const int j = threadIdx.x % LR;
  const bool is_v = blockIdx.y == 1;
  const bool in = row < n * c.hk;
  const int64_t tok = in ? row / c.hk : 0;
  const int h = in ? static_cast<int>(row % c.hk) : 0;
  int64_t slot = slots[tok];
  const bool ok = slot >= 0 && slot < c.n_slots;
  slot = ok ? slot : 0;
  const int64_t page = slot / c.page;
  const int t = static_cast<int>(slot % c.page);
  const int64_t base = (page * c.hk + h) * c.page;
  uint32_t w;
  if (!is_v) {
    w = *reinterpret_cast<const uint32_t*>(c.kc + (base + t) * (D / 2) + 4 * j);
  } else {
    const uint8_t* p = c.vc + (base + (t & ~15)) * (D / 2) + (t & 15) + 64 * j;
    w = p[0] | p[16] << 8 | p[32] << 16 | static_cast<uint32_t>(p[48]) << 24;
  }
  float scale = (is_v ? c.vs : c.ks)[base + t];
  scale = ok ? scale : 0.0f;
  w = ok ? w : 0;
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = static_cast<float>(static_cast<int32_t>(w << (28 - 4 * i)) >> 28);
  if (ROT && !is_v) {
    fwht_row<D>(x, j);  // sums of up to 256 codes, exact
    scale *= 1.0f / sqrtf(static_cast<float>(D));
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] *= scale;
  if (!in) return;
  const int64_t off = tok * (is_v ? ldv : ldk) + h * D + 8 * j;
  if (dtype == OQ_OUT_F32) {
    float4* o = reinterpret_cast<float4*>(static_cast<float*>(is_v ? V : K) + off);
    o[0] = make_float4(x[0], x[1], x[2], x[3]);
    o[1] = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    const bool bf = dtype == OQ_OUT_BF16;
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(is_v ? V : K) + off) =
        make_uint4(pack2(x[0], x[1], bf), pack2(x[2], x[3], bf), pack2(x[4], x[5], bf), pack2(x[6], x[7], bf));
  }
}

// ---------------------------------------------------------------------------
// Attention over the pages.
//
// The rows of a sequence and kv head (its query tokens times the R heads of
// the group, row = token R + head) are columns of 16-wide matrix products; the
// cache is read once per 16 QT rows.  Both products are transposed: S^T = K
// Q^T (tokens x rows), O^T = V^T P^T (channels x rows), on
// v_mfma_f32_16x16x32_f16.
//
// A wave takes 128 tokens at a time; lane group g (lane / 16) owns tokens
// 32 g .. 32 g + 31 of them.  The order of tokens in the first product's tiles
// is free: tile i has token 32 g + 4 i + e in row 4 g + e, so the group's lanes
// end with the probabilities of exactly its own 32 tokens, in the order in
// which the second product's operand takes them (k step j: tiles 2 j, 2 j + 1)
// and nothing crosses lanes.
//
// Codes become fp16 by placing a nibble in the mantissa of 64 (or 1024):
// 64 + n, n = c + 8 the biased code; the bias goes with one exclusive or.  For
// keys the 72 is taken out by the accumulator's start, -72 sum(q) (an error
// of 2^-24 of that sum); for values by a packed subtraction, exact.
// The step of a key scales its row of S in fp32.  The step of a value is
// folded into the exponent: P' = 2^(s + log2(step) - m'), with a running
// maximum m' of its own, so that P' is at most 1 and its fp16 rounding is
// relative to the largest contribution whatever the steps' range; the sum l of
// the softmax is formed from 2^(s - m) in fp32.
// Queries are scaled by a power of two to at most 1 and rounded to fp16 (exact
// for unrotated fp16 and bf16 rows but for values below 2^-24 of the row's
// largest); rotated ones are split in two fp16 parts (22 bits).
// ---------------------------------------------------------------------------
struct AttnKv4 {
  Cache c;
  const uint16_t* q;
  uint16_t* o;
  const int32_t* cu_q;
  const int32_t* table;
  const int32_t* lens;
  float* part;     // [tokens * hq][splits][D + 2], null with one split
  int64_t tokens, ldq, ldo, table_ld, n_pages;
  int n_seqs, hq, R, max_q, max_len, splits;
  float scale_log2e;
  bool bf, causal;
};

constexpr int kTile = 128;  // tokens of one step of a wave
constexpr int kWaves = 4;

__device__ __forceinline__ uint32_t and_xor(uint32_t a, uint32_t m, uint32_t x) { return (a & m) ^ x; }

template <int D, int QT, bool ROT>
__global__ __launch_bounds__(64 * kWaves) void attn_kv4_kernel(AttnKv4 a) {
  constexpr int ROWS = 16 * QT, KW = D / 32, PT = D / 32, NQ = ROT ? 2 : 1;
  __shared__ float so[kWaves][ROWS][D + 4];
  __shared__ float sm[kWaves][ROWS][3];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, g = lane >> 4;
  const int b = blockIdx.y / a.c.hk, h = blockIdx.y % a.c.hk;
  const int split = blockIdx.z;
  int64_t q0 = b;
  int nq = 1;
  if (a.cu_q) {
    q0 = a.cu_q[b];
    nq = a.cu_q[b + 1] - static_cast<int>(q0);
    q0 = q0 < 0 ? 0 : q0 > a.tokens ? a.tokens : q0;
    nq = max(0, min(static_cast<int64_t>(min(nq, a.max_q)), a.tokens - q0));
  }
  q0 = __builtin_amdgcn_readfirstlane(static_cast<int>(q0));
  nq = __builtin_amdgcn_readfirstlane(nq);
  const int L = __builtin_amdgcn_readfirstlane(max(0, min(a.lens[b], a.max_len)));
  const int rows = nq * a.R, r0 = blockIdx.x * ROWS;
  if (r0 >= rows) return;

  // Keys that a row sees: the first `seen` tokens.
  int seen[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int r = min(r0 + 16 * t + col, rows - 1);
    seen[t] = a.causal ? max(0, L - nq + 1 + r / a.R) : L;
  }
  const int last_seen = a.causal ? max(0, L - nq + 1 + min(r0 + ROWS - 1, rows - 1) / a.R) : L;
  const int tiles = (L + kTile - 1) / kTile, per = (tiles + a.splits - 1) / a.splits;
  const int t_end = min(min(tiles, (split + 1) * per), (last_seen + kTile - 1) / kTile);

  // Queries.
  v8h qf[QT][NQ][KW];
  float corr[QT], qscale[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int r = min(r0 + 16 * t + col, rows - 1);
    const uint16_t* qp = a.q + (q0 + r / a.R) * a.ldq + (h * a.R + r % a.R) * D;
    float x[KW][8];
#pragma unroll
    for (int s = 0; s < KW; ++s)
      load8(qp + (s / 4) * 128 + (D == 64 ? 16 : 32) * g + 8 * (s % 4), a.bf, x[s]);
    float norm = 1.0f;
    if (ROT) {
      // Channel bits: 0-2 in a word, then the words of a lane, the lane group, (d = 256) the half.
#pragma unroll
      for (int st = 1; st < 8; st *= 2)
#pragma unroll
        for (int s = 0; s < KW; ++s)
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (!(i & st)) {
              const float u = x[s][i], v = x[s][i + st];
              x[s][i] = u + v;
              x[s][i + st] = u - v;
            }
#pragma unroll
      for (int st = 1; st < KW; st *= 2)
#pragma unroll
        for (int s = 0; s < KW; ++s)
          if (!(s & st))
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float u = x[s][i], v = x[s + st][i];
              x[s][i] = u + v;
              x[s + st][i] = u - v;
            }
#pragma unroll
      for (int s = 0; s < KW; ++s)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float v = lane_xor_far<16>(x[s][i]);
          x[s][i] = (g & 1) ? v - x[s][i] : x[s][i] + v;
          const float w = lane_xor_far<32>(x[s][i]);
          x[s][i] = (g & 2) ? w - x[s][i] : x[s][i] + w;
        }
      norm = 1.0f / sqrtf(static_cast<float>(D));
    }
    float top = 0.0f;
#pragma unroll
    for (int s = 0; s < KW; ++s)
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(x[s][i]));
    top = fmaxf(top, lane_xor_far<16>(top));
    top = fmaxf(top, lane_xor_far<32>(top));
    const int e = top > 0.0f && top < INFINITY ? ilogbf(top) + 1 : 0;
    float sum = 0.0f;
    constexpr int kOrder[8] = {0, 4, 1, 5, 2, 6, 3, 7};  // channels of a word in the order the codes come out
#pragma unroll
    for (int s = 0; s < KW; ++s)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float v = ldexpf(x[s][kOrder[i]], -e);
        const _Float16 hi = static_cast<_Float16>(v);
        qf[t][0][s][i] = hi;
        sum += static_cast<float>(hi);
        if constexpr (ROT) {
          const _Float16 lo = static_cast<_Float16>(v - static_cast<float>(hi));
          qf[t][NQ - 1][s][i] = lo;
          sum += static_cast<float>(lo);
        }
      }
    sum += lane_xor_far<16>(sum);
    sum += lane_xor_far<32>(sum);
    corr[t] = -72.0f * sum;
    qscale[t] = ldexpf(a.scale_log2e * norm, e);
  }

  v4f acc[QT][PT][2];
  float m[QT], mv[QT], l[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    m[t] = mv[t] = -INFINITY;
    l[t] = 0.0f;
#pragma unroll
    for (int p = 0; p < PT; ++p) acc[t][p][0] = acc[t][p][1] = v4f{0, 0, 0, 0};
  }
  const int32_t* table = a.table + b * a.table_ld;
  for (int tile = split * per + wave; tile < t_end; tile += kWaves) {
    const int tok0 = tile * kTile;
    // The page of this lane group's 32 tokens, and of the 4 groups of K rows this lane reads.
    auto block_base = [&](int grp, bool& ok) -> int64_t {
      const int tok = tok0 + 32 * grp;
      const int pi = tok / a.c.page;
      const int64_t pg = tok < L ? table[pi] : -1;
      ok = pg >= 0 && pg < a.n_pages;
      return ((ok ? pg : 0) * a.c.hk + h) * a.c.page + tok % a.c.page;
    };
    bool own_ok, k_ok;
    const int64_t own = block_base(g, own_ok);
    const int64_t kb = block_base(col >> 2, k_ok) + (col & 3);
    // First product.
    v4f s[QT][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint8_t* kp = a.c.kc + (kb + 4 * i) * (D / 2);
      uint32_t w[KW];
      if constexpr (D == 64) {
        const uint2 r = *reinterpret_cast<const uint2*>(kp + 8 * g);
        w[0] = r.x;
        w[1] = r.y;
      } else {
#pragma unroll
        for (int c = 0; c < KW / 4; ++c) {
          const uint4 r = *reinterpret_cast<const uint4*>(kp + 64 * c + 16 * g);
          w[4 * c] = r.x;
          w[4 * c + 1] = r.y;
          w[4 * c + 2] = r.z;
          w[4 * c + 3] = r.w;
        }
      }
#pragma unroll
      for (int t = 0; t < QT; ++t) s[t][i] = v4f{corr[t], corr[t], corr[t], corr[t]};
#pragma unroll
      for (int k = 0; k < KW; ++k) {
        uint4 u;
        u.x = and_xor(w[k] << 4, 0x00F000F0u, 0x54805480u);
        u.y = and_xor(w[k], 0x00F000F0u, 0x54805480u);
        u.z = and_xor(w[k] >> 4, 0x00F000F0u, 0x54805480u);
        u.w = and_xor(w[k] >> 8, 0x00F000F0u, 0x54805480u);
        const v8h ka = __builtin_bit_cast(v8h, u);
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
          for (int p = 0; p < NQ; ++p) s[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ka, qf[t][p][k], s[t][i], 0, 0, 0);
      }
    }
    // Softmax of this lane's row over its 32 tokens; log2 of the values' steps.
    const float* ksp = a.c.ks + own;
    const float* vsp = a.c.vs + own;
    float lv[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float4 k4 = *reinterpret_cast<const float4*>(ksp + 4 * i);
      const float4 v4 = *reinterpret_cast<const float4*>(vsp + 4 * i);
      const float ke[4] = {k4.x, k4.y, k4.z, k4.w}, ve[4] = {v4.x, v4.y, v4.z, v4.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        lv[i][e] = __builtin_amdgcn_logf(ve[e]);
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          const float v = s[t][i][e] * ke[e] * qscale[t];
          s[t][i][e] = own_ok && tok0 + 32 * g + 4 * i + e < seen[t] ? v : -INFINITY;
        }
      }
    }
    v8h pf[QT][4];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      float mn = m[t], mvn = mv[t];
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          mn = fmaxf(mn, s[t][i][e]);
          mvn = fmaxf(mvn, s[t][i][e] == -INFINITY ? -INFINITY : s[t][i][e] + lv[i][e]);
        }
      mn = fmaxf(mn, lane_xor_far<16>(mn));
      mn = fmaxf(mn, lane_xor_far<32>(mn));
      mvn = fmaxf(mvn, lane_xor_far<16>(mvn));
      mvn = fmaxf(mvn, lane_xor_far<32>(mvn));
      const float mr = mn == -INFINITY ? 0.0f : mn, mvr = mvn == -INFINITY ? 0.0f : mvn;
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float sv = s[t][i][e];
          sum += __builtin_amdgcn_exp2f(sv - mr);
          const float p = sv == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(sv + lv[i][e] - mvr);
          // Tokens of a word come out as 0, 2, 1, 3.
          constexpr int kPos[4] = {0, 2, 1, 3};
          pf[t][i / 2][4 * (i & 1) + kPos[e]] = static_cast<_Float16>(p);
        }
      l[t] = l[t] * __builtin_amdgcn_exp2f(m[t] - mr) + sum;
      const float al = __builtin_amdgcn_exp2f(mv[t] - mvr);
      m[t] = mn;
      mv[t] = mvn;
#pragma unroll
      for (int p = 0; p < PT; ++p)
#pragma unroll
        for (int x = 0; x < 2; ++x) acc[t][p][x] *= al;
    }
    // Second product.
    const uint8_t* vp = a.c.vc + own * (D / 2) + 16 * col;
#pragma unroll
    for (int p = 0; p < PT; ++p) {
      uint32_t w[8];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const uint4 r = *reinterpret_cast<const uint4*>(vp + x * 16 * (D / 2) + 256 * p);
        w[4 * x] = r.x;
        w[4 * x + 1] = r.y;
        w[4 * x + 2] = r.z;
        w[4 * x + 3] = r.w;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v8h lo, hi;
        const v2h c72 = {72, 72}, c1032 = {1032, 1032};
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const uint32_t y = w[2 * j + x], z = y >> 8;
          const v2h l0 = __builtin_bit_cast(v2h, and_xor(y, 0x000F000Fu, 0x64086408u)) - c1032;
          const v2h l1 = __builtin_bit_cast(v2h, and_xor(z, 0x000F000Fu, 0x64086408u)) - c1032;
          const v2h h0 = __builtin_bit_cast(v2h, and_xor(y, 0x00F000F0u, 0x54805480u)) - c72;
          const v2h h1 = __builtin_bit_cast(v2h, and_xor(z, 0x00F000F0u, 0x54805480u)) - c72;
          lo[4 * x] = l0[0]; lo[4 * x + 1] = l0[1]; lo[4 * x + 2] = l1[0]; lo[4 * x + 3] = l1[1];
          hi[4 * x] = h0[0]; hi[4 * x + 1] = h0[1]; hi[4 * x + 2] = h1[0]; hi[4 * x + 3] = h1[1];
        }
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          acc[t][p][0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo, pf[t][j], acc[t][p][0], 0, 0, 0);
          acc[t][p][1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi, pf[t][j], acc[t][p][1], 0, 0, 0);
        }
      }
    }
  }

  // Join the waves.
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    float s = l[t];
    s += lane_xor_far<16>(s);
    s += lane_xor_far<32>(s);
#pragma unroll
    for (int p = 0; p < PT; ++p)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int x = 0; x < 2; ++x) so[wave][16 * t + col][32 * p + 8 * g + 2 * e + x] = acc[t][p][x][e];
    if (g == 0) {
      sm[wave][16 * t + col][0] = m[t];
      sm[wave][16 * t + col][1] = mv[t];
      sm[wave][16 * t + col][2] = s;
    }
  }
  __syncthreads();
  constexpr int TPR = D / 8;
  for (int i = threadIdx.x; i < ROWS * TPR; i += 64 * kWaves) {
    const int r = i / TPR, c = (i % TPR) * 8;
    if (r0 + r >= rows) continue;
    float M = -INFINITY, MV = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      M = fmaxf(M, sm[w][r][0]);
      MV = fmaxf(MV, sm[w][r][1]);
    }
    const float mr = M == -INFINITY ? 0.0f : M, mvr = MV == -INFINITY ? 0.0f : MV;
    float L_ = 0.0f, y[8] = {};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      L_ += sm[w][r][2] * __builtin_amdgcn_exp2f(sm[w][r][0] - mr);
      const float f = __builtin_amdgcn_exp2f(sm[w][r][1] - mvr);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] += so[w][r][c + e] * f;
    }
    const float f = L_ > 0.0f ? __builtin_amdgcn_exp2f(mvr - mr) / L_ : 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] *= f;
    const int64_t tok = q0 + (r0 + r) / a.R;
    const int head = h * a.R + (r0 + r) % a.R;
    if (a.splits == 1) {
      *reinterpret_cast<uint4*>(a.o + tok * a.ldo + head * D + c) =
          make_uint4(pack2(y[0], y[1], a.bf), pack2(y[2], y[3], a.bf), pack2(y[4], y[5], a.bf), pack2(y[6], y[7], a.bf));
    } else {
      float* o = a.part + ((tok * a.hq + head) * a.splits + split) * (D + 4);
      *reinterpret_cast<float4*>(o + c) = make_float4(y[0], y[1], y[2], y[3]);
      *reinterpret_cast<float4*>(o + c + 4) = make_float4(y[4], y[5], y[6], y[7]);
      if (c == 0) {
        o[D] = M;
        o[D + 1] = L_;
      }
    }
  }
}

// o = sum_s w_s o_s / sum_s w_s with w_s = l_s 2^(m_s - m), 8 channels a thread.
template <int D>
__global__ __launch_bounds__(256) void attn_kv4_join_kernel(AttnKv4 a) {
  constexpr int TPR = D / 8;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * (256 / TPR) + threadIdx.x / TPR;
  const int c = (threadIdx.x % TPR) * 8;
  if (row >= a.tokens * a.hq) return;
  const int64_t tok = row / a.hq;
  // Tokens that no sequence has (or that are past max_q in theirs) are left as they were.
  if (a.cu_q) {
    int lo = 0, hi = a.n_seqs;  // the last sequence that starts at or before tok
    while (lo + 1 < hi) {
      const int mid = (lo + hi) / 2;
      if (a.cu_q[mid] <= tok) lo = mid;
      else hi = mid;
    }
    const int s0 = a.cu_q[lo];
    if (tok < s0 || tok >= a.cu_q[lo + 1] || tok - s0 >= a.max_q) return;
  } else if (tok >= a.n_seqs) {
    return;
  }
  const float* p = a.part + row * a.splits * (D + 4);
  float M = -INFINITY;
  for (int s = 0; s < a.splits; ++s) M = fmaxf(M, p[s * (D + 4) + D]);
  const float mr = M == -INFINITY ? 0.0f : M;
  float L = 0.0f, y[8] = {};
  for (int s = 0; s < a.splits; ++s) {
    const float* ps = p + s * (D + 4);
    const float w = ps[D + 1] * __builtin_amdgcn_exp2f(ps[D] - mr);
    L += w;
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] += w * ps[c + e];
  }
  const float f = L > 0.0f ? 1.0f / L : 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] *= f;
  *reinterpret_cast<uint4*>(a.o + tok * a.ldo + (row % a.hq) * D + c) =
      make_uint4(pack2(y[0], y[1], a.bf), pack2(y[2], y[3], a.bf), pack2(y[4], y[5], a.bf), pack2(y[6], y[7], a.bf));
}

int cache_validate(const oq_kv4_cache* c) {
  if (!c || !c->k_codes || !c->v_codes || !c->k_scale || !c->v_scale) return OQ_ERR_NULL;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return OQ_ERR_SHAPE;
  if (c->n_pages < 1 || c->n_pages > INT32_MAX || c->n_kv_heads < 1 || c->page_tokens < 32 || c->page_tokens % 32 != 0 ||
      c->page_tokens > 65536 || c->n_kv_heads > 65535)
    return OQ_ERR_SHAPE;
  if (!aligned(c->k_codes, 16) || !aligned(c->v_codes, 16) || !aligned(c->k_scale, 16) || !aligned(c->v_scale, 16))
    return OQ_ERR_ALIGN;
  if (c->rotate_k != 0 && c->rotate_k != 1) return OQ_ERR_ARG;
  return OQ_OK;
}

Cache device_cache(const oq_kv4_cache* c) {
  return Cache{c->k_codes, c->v_codes, c->k_scale, c->v_scale, c->n_pages * c->page_tokens, c->page_tokens, c->n_kv_heads};
}

// Splits of the cache's length.  (Rule of the first version: enough workgroups for two per CU.)
int kv4_splits(int64_t n_seqs, int hk, int64_t row_blocks, int64_t max_len) {
  const int64_t wgs = n_seqs * hk * row_blocks;
  const int64_t tiles = (max_len + kTile - 1) / kTile;
  int64_t s = (512 + wgs - 1) / wgs;
  s = s > (tiles + kWaves - 1) / kWaves ? (tiles + kWaves - 1) / kWaves : s;
  return static_cast<int>(s < 1 ? 1 : s > 64 ? 64 : s);
}

struct Kv4Plan {
  int qt, splits;
  int64_t row_blocks;
};
Kv4Plan kv4_plan(int n_seqs, int hk, int R, int max_q, int64_t max_len) {
  const int64_t rows = static_cast<int64_t>(max_q) * R;
  Kv4Plan p;
  p.qt = rows <= 16 ? 1 : 2;
  p.row_blocks = (rows + 16 * p.qt - 1) / (16 * p.qt);
  p.splits = kv4_splits(n_seqs, hk, p.row_blocks, max_len);
  return p;
}

template <int D, int QT>
void launch_attn(const AttnKv4& a, dim3 grid, bool rot, hipStream_t st) {
  if (rot) hipLaunchKernelGGL((attn_kv4_kernel<D, QT, true>), grid, dim3(64 * kWaves), 0, st, a);
  else hipLaunchKernelGGL((attn_kv4_kernel<D, QT, false>), grid, dim3(64 * kWaves), 0, st, a);
}

}  // namespace
}  // namespace oq

extern "C" int oq_kv4_append(const oq_kv4_cache* cache, const void* K, const void* V, int64_t n, int64_t ldk, int64_t ldv,
                             int32_t dtype, const int64_t* slots, void* stream) {
  int st = oq::cache_validate(cache);
  if (st != OQ_OK) return st;
  const int64_t w = static_cast<int64_t>(cache->n_kv_heads) * cache->head_dim;
  if (n < 0 || n > INT32_MAX || ldk < w || ldv < w) return OQ_ERR_SHAPE;
  if (dtype != OQ_OUT_F16 && dtype != OQ_OUT_BF16) return OQ_ERR_ARG;
  if (ldk % 8 != 0 || ldv % 8 != 0) return OQ_ERR_ALIGN;
  if (n == 0) return OQ_OK;
  if (!K || !V || !slots) return OQ_ERR_NULL;
  if (!oq::aligned(K, 16) || !oq::aligned(V, 16) || !oq::aligned(slots, 8)) return OQ_ERR_ALIGN;
  if ((st = oq::device_check()) != OQ_OK) return st;
  const oq::Cache c = oq::device_cache(cache);
  const int64_t per = 2048 / cache->head_dim, blocks = (n * c.hk + per - 1) / per;
  if (blocks > INT32_MAX) return OQ_ERR_SHAPE;
  const dim3 grid(static_cast<unsigned>(blocks), 2);
  const bool bf = dtype == OQ_OUT_BF16;
  hipStream_t s = static_cast<hipStream_t>(stream);
#define OQ_APPEND(D, R)                                                                                               \
  if (cache->head_dim == D && cache->rotate_k == R)                                                                   \
  hipLaunchKernelGGL((oq::kv4_append_kernel<D, R>), grid, dim3(256), 0, s, c, static_cast<const uint16_t*>(K),        \
                     static_cast<const uint16_t*>(V), n, ldk, ldv, bf, slots)
  OQ_APPEND(64, 0);
  OQ_APPEND(64, 1);
  OQ_APPEND(128, 0);
  OQ_APPEND(128, 1);
  OQ_APPEND(256, 0);
  OQ_APPEND(256, 1);
#undef OQ_APPEND
  return oq::launch_status();
}

extern "C" int oq_kv4_gather(const oq_kv4_cache* cache, const int64_t* slots, int64_t n, void* K, void* V, int64_t ldk,
                             int64_t ldv, int32_t dtype, void* stream) {
  int st = oq::cache_validate(cache);
  if (st != OQ_OK) return st;
  const int64_t w = static_cast<int64_t>(cache->n_kv_heads) * cache->head_dim;
  if (n < 0 || n > INT32_MAX || ldk < w || ldv < w) return OQ_ERR_SHAPE;
  if (dtype != OQ_OUT_F16 && dtype != OQ_OUT_BF16 && dtype != OQ_OUT_F32) return OQ_ERR_ARG;
  if (ldk % 8 != 0 || ldv % 8 != 0) return OQ_ERR_ALIGN;
  if (n == 0) return OQ_OK;
  if (!K || !V || !slots) return OQ_ERR_NULL;
  if (!oq::aligned(K, 16) || !oq::aligned(V, 16) || !oq::aligned(slots, 8)) return OQ_ERR_ALIGN;
  if ((st = oq::device_check()) != OQ_OK) return st;
  const oq::Cache c = oq::device_cache(cache);
  const int64_t per = 2048 / cache->head_dim, blocks = (n * c.hk + per - 1) / per;
  if (blocks > INT32_MAX) return OQ_ERR_SHAPE;
  const dim3 grid(static_cast<unsigned>(blocks), 2);
  hipStream_t s = static_cast<hipStream_t>(stream);
#define OQ_GATHER(D, R)                             \
  if (cache->head_dim == D && cache->rotate_k == R) \
  hipLaunchKernelGGL((oq::kv4_gather_kernel<D, R>), grid, dim3(256), 0, s, c, slots, n, K, V, ldk, ldv, dtype)
  OQ_GATHER(64, 0);
  OQ_GATHER(64, 1);
  OQ_GATHER(128, 0);
  OQ_GATHER(128, 1);
  OQ_GATHER(256, 0);
  OQ_GATHER(256, 1);
#undef OQ_GATHER
  return oq::launch_status();
}

static int attn_kv4_shape(const oq_kv4_cache* cache, int64_t tokens, int32_t n_heads, int32_t n_seqs, int32_t max_q,
                          int32_t max_len) {
  if (tokens < 0 || tokens > INT32_MAX || n_seqs < 0 || max_q < 1 || max_len < 0 || n_heads < 1) return OQ_ERR_SHAPE;
  if (n_heads % cache->n_kv_heads != 0) return OQ_ERR_SHAPE;
  if (static_cast<int64_t>(n_seqs) * cache->n_kv_heads > 65535) return OQ_ERR_SHAPE;
  if (static_cast<int64_t>(max_q) * (n_heads / cache->n_kv_heads) > INT32_MAX / 2) return OQ_ERR_SHAPE;
  return OQ_OK;
}

extern "C" size_t oq_attention_kv4_workspace_bytes(const oq_kv4_cache* cache, int64_t tokens, int32_t n_heads,
                                                   int32_t n_seqs, int32_t max_q, int32_t max_len) {
  if (!cache || cache->n_kv_heads < 1 || attn_kv4_shape(cache, tokens, n_heads, n_seqs, max_q, max_len) != OQ_OK || n_seqs == 0)
    return 0;
  const oq::Kv4Plan p = oq::kv4_plan(n_seqs, cache->n_kv_heads, n_heads / cache->n_kv_heads, max_q, max_len);
  return p.splits == 1 ? 0 : static_cast<size_t>(tokens) * n_heads * p.splits * (cache->head_dim + 4) * 4;
}

extern "C" int oq_attention_kv4(const oq_kv4_cache* cache, const void* Q, int64_t tokens, int64_t ldq, int32_t n_heads,
                                int32_t dtype, const int32_t* cu_q, int32_t max_q, const int32_t* block_table,
                                int64_t table_ld, const int32_t* seq_lens, int32_t n_seqs, int32_t max_len,
                                int32_t causal, float scale, void* O, int64_t ldo, void* work, size_t work_bytes,
                                void* stream) {
  int st = oq::cache_validate(cache);
  if (st != OQ_OK) return st;
  if ((st = attn_kv4_shape(cache, tokens, n_heads, n_seqs, max_q, max_len)) != OQ_OK) return st;
  const int64_t w = static_cast<int64_t>(n_heads) * cache->head_dim;
  if (ldq < w || ldo < w) return OQ_ERR_SHAPE;
  if (!cu_q && (max_q != 1 || tokens != n_seqs)) return OQ_ERR_SHAPE;
  if (table_ld < 0 || (static_cast<int64_t>(max_len) + cache->page_tokens - 1) / cache->page_tokens > table_ld) return OQ_ERR_SHAPE;
  if (dtype != OQ_OUT_F16 && dtype != OQ_OUT_BF16) return OQ_ERR_ARG;
  if (causal != 0 && causal != 1) return OQ_ERR_ARG;
  if (!(scale > 0.0f) || !std::isfinite(scale)) return OQ_ERR_ARG;
  if (ldq % 8 != 0 || ldo % 8 != 0) return OQ_ERR_ALIGN;
  if (tokens == 0 || n_seqs == 0) return OQ_OK;
  if (!Q || !O || !seq_lens || (!block_table && max_len > 0)) return OQ_ERR_NULL;
  if (!oq::aligned(Q, 16) || !oq::aligned(O, 16) || !oq::aligned(seq_lens, 4) || !oq::aligned(block_table, 4) ||
      !oq::aligned(cu_q, 4) || !oq::aligned(work, 16))
    return OQ_ERR_ALIGN;
  const int R = n_heads / cache->n_kv_heads;
  const oq::Kv4Plan p = oq::kv4_plan(n_seqs, cache->n_kv_heads, R, max_q, max_len);
  if (p.splits > 1 && (!work || work_bytes < oq_attention_kv4_workspace_bytes(cache, tokens, n_heads, n_seqs, max_q, max_len)))
    return OQ_ERR_WORKSPACE;
  if ((st = oq::device_check()) != OQ_OK) return st;
  oq::AttnKv4 a{};
  a.c = oq::device_cache(cache);
  a.q = static_cast<const uint16_t*>(Q);
  a.o = static_cast<uint16_t*>(O);
  a.cu_q = cu_q;
  a.table = block_table;
  a.lens = seq_lens;
  a.part = static_cast<float*>(work);
  a.tokens = tokens;
  a.ldq = ldq;
  a.ldo = ldo;
  a.table_ld = table_ld;
  a.n_pages = cache->n_pages;
  a.n_seqs = n_seqs;
  a.hq = n_heads;
  a.R = R;
  a.max_q = max_q;
  a.max_len = max_len;
  a.splits = p.splits;
  a.scale_log2e = scale * 1.4426950408889634f;
  a.bf = dtype == OQ_OUT_BF16;
  a.causal = causal == 1;
  const dim3 grid(static_cast<unsigned>(p.row_blocks), static_cast<unsigned>(n_seqs * cache->n_kv_heads),
                  static_cast<unsigned>(p.splits));
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool rot = cache->rotate_k == 1;
#define OQ_ATTN(D)                                              \
  if (cache->head_dim == D) {                                   \
    if (p.qt == 1) oq::launch_attn<D, 1>(a, grid, rot, s);      \
    else oq::launch_attn<D, 2>(a, grid, rot, s);                \
  }
  OQ_ATTN(64) OQ_ATTN(128) OQ_ATTN(256)
#undef OQ_ATTN
  if ((st = oq::launch_status()) != OQ_OK || p.splits == 1) return st;
  const int64_t rows = tokens * n_heads, per = 2048 / cache->head_dim;
  const dim3 jg(static_cast<unsigned>((rows + per - 1) / per));
  if (cache->head_dim == 64) hipLaunchKernelGGL((oq::attn_kv4_join_kernel<64>), jg, dim3(256), 0, s, a);
  else if (cache->head_dim == 128) hipLaunchKernelGGL((oq::attn_kv4_join_kernel<128>), jg, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((oq::attn_kv4_join_kernel<256>), jg, dim3(256), 0, s, a);
  return oq::launch_status();
}
