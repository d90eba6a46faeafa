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
// Layout, per page and head (page_tokens tokens, a multiple of 16):
//   k_codes [token][d / 2]: byte b holds channels 2 b (low nibble), 2 b + 1;
//   v_codes [token / 16][d / 2][16]: byte (b, t) holds channels 2 b and 2 b + 1
//     of token t of the 16, so a token's write is whole bytes (no neighbour
//     shares one) and the second product's operand, 8 tokens of a channel, is
//     two words;
//   k_scale, v_scale fp32 [token].
#include <algorithm>
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
  int hk;
  uint32_t p16, p16_inv;  // 16-token blocks of a page, and floor(2^32 / p16) (p16 = 1: 2^32 - 1)
};

template <bool BF>
__device__ __forceinline__ void load8(const uint16_t* p, float (&v)[8]) {
  const uint4 r = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = BF ? __uint_as_float(w[i] << 16) : rqd::h2f(w[i] & 0xFFFFu);
    v[2 * i + 1] = BF ? __uint_as_float(w[i] & 0xFFFF0000u) : rqd::h2f(w[i] >> 16);
  }
}
template <bool BF>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  if constexpr (BF) {
    const __bf16 x = static_cast<__bf16>(a), y = static_cast<__bf16>(b);
    return __builtin_bit_cast(uint16_t, x) | static_cast<uint32_t>(__builtin_bit_cast(uint16_t, y)) << 16;
  }
  return rqd::f2h(a) | static_cast<uint32_t>(rqd::f2h(b)) << 16;
}
// 8 outputs as one 16-byte store of fp16 or bf16.
template <bool BF>
__device__ __forceinline__ void store8(uint16_t* p, const float (&y)[8]) {
  *reinterpret_cast<uint4*>(p) = make_uint4(pack2<BF>(y[0], y[1]), pack2<BF>(y[2], y[3]), pack2<BF>(y[4], y[5]), pack2<BF>(y[6], y[7]));
}

// Value of lane ^ H (H < 32) on the vector unit.
template <int H>
__device__ __forceinline__ float lane_swap(float v) {
  if constexpr (H <= 2) return rqd::lane_xor<H>(v);
  else if constexpr (H <= 8) return rqd::lane_xor_dpp<H>(v);
  else return lane_xor_far<H>(v);
}
template <int H>
__device__ __forceinline__ double lane_swap(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const float lo = lane_swap<H>(__uint_as_float(static_cast<uint32_t>(b)));
  const float hi = lane_swap<H>(__uint_as_float(static_cast<uint32_t>(b >> 32)));
  return __builtin_bit_cast(double, static_cast<uint64_t>(__float_as_uint(hi)) << 32 | __float_as_uint(lo));
}
// f(H) for the lane bits H = 1, 2 .. LR / 2 of a row of LR lanes.
template <int LR, int H = 1, typename F>
__device__ __forceinline__ void over_lanes(F&& f) {
  if constexpr (H < LR) {
    f(std::integral_constant<int, H>{});
    over_lanes<LR, 2 * H>(f);
  }
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
  over_lanes<D / 8>([&](auto H) {
    constexpr int h = decltype(H)::value;
    const T sgn = (j & h) ? T(-1) : T(1);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = fma(sgn, x[i], lane_swap<h>(x[i]));
  });
}
// Largest |x| of a row.
template <int D, typename T>
__device__ __forceinline__ T top_row(const T (&x)[8]) {
  T top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = fmax(top, fabs(x[i]));
  over_lanes<D / 8>([&](auto H) { top = fmax(top, lane_swap<decltype(H)::value>(top)); });
  return top;
}

// Code of one element: the integer nearest to 7 u / top, ties to even, |u| <=
// top.  7 u, q top and their difference are exact (u and top are inputs of at
// most 11 bits, or sums of up to 256 of them in fp64: fp16's need 51 bits, bf16's
// as many as their exponents span and 19), so a quotient next to
// a half integer is decided exactly: the estimate is at most one off, and only
// beside a boundary.  In rotated bf16 rows whose nonzero elements span more than 2^34 the sums round
// (by up to 2^-46 of the largest: eight stages, and the sum of magnitudes at most 16 times the norm), and a
// quotient within 2^-42 of a half integer may go either way.
template <typename T>
__device__ __forceinline__ float exact_code(T u, T top) {
  const T q = rint(u * (T(7) / top));
  const T e = fma(-q, top, T(7) * u), d = T(2) * fabs(e) - top;
  const int n = static_cast<int>(q);
  const int up = e > T(0) ? 1 : -1;
  return static_cast<float>(d > T(0) || (d == T(0) && (n & 1)) ? n + up : n);
}
// The codes of a lane's 8 channels as one word.  The fp32 quotient is within
// 2^-19 of the exact one (7 times four roundings), so only a quotient within
// 2^-16 of a half integer has to be decided exactly: ties mostly, which half the
// waves of bf16 rows have, but in one or two of their 8 channels.
template <typename T>
__device__ __forceinline__ uint32_t codes8(const T (&u)[8], T top) {
  const float inv = 7.0f * __builtin_amdgcn_rcpf(static_cast<float>(top));
  const bool range = inv > 1e-30f && inv < 1e30f;
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float r = static_cast<float>(u[i]) * inv;
    float q = rintf(r);
    if (__builtin_amdgcn_ballot_w64(!(range && fabsf(r - q) < 0.5f - 0x1p-16f)) != 0) {
      // (Scaled by a power of two to [1, 2), so that nothing overflows.)
      const int e = top > 0 ? -ilogb(top) : 0;
      q = top > 0 ? exact_code(ldexp(u[i], e), ldexp(top, e)) : 0;
    }
    w |= static_cast<uint32_t>(static_cast<int>(q) & 15) << (4 * i);
  }
  return w;
}

// ---------------------------------------------------------------------------
// Append.  HBM bound: 4 d bytes read and d + 8 written per token and head.
//
// A workgroup takes the keys and the values of 2048 / d tokens and one head, d / 8
// lanes a row, both loads in flight from the start.  Rotated keys are summed in
// fp64, where sums of inputs are exact (exact_code); that is 8 us of the 30 that 16000 tokens
// of 8 heads of 128 take (83 MB, 2.8 TB/s; unrotated 22 us, 3.8 TB/s), the rest of
// it the vector work of max and codes beside the loads.  Codes of values go through LDS, so that a wave stores 16
// tokens of a channel pair as neighbouring bytes: tokens of a prompt fill their
// blocks with whole 16-byte runs whatever place they start at.
// ---------------------------------------------------------------------------
template <int D>
struct Rows {
  static constexpr int LR = D / 8, N = 256 / LR;  // lanes of a row, tokens of a workgroup
};

// blk / p16, and the remainder in `in`: inv = floor(2^32 / p16) (p16 = 1: 2^32 - 1)
// gives the quotient or one less.
__device__ __forceinline__ uint32_t div_blocks(uint32_t blk, uint32_t p16, uint32_t inv, uint32_t& in) {
  uint32_t q = __umulhi(blk, inv);
  in = blk - q * p16;
  const bool over = in >= p16;
  in -= over ? p16 : 0;
  return q + (over ? 1 : 0);
}
// First token of the 16-token block that a slot's token lies in, in the
// cache's order [page][head][token]; t: the token's place in the block.
__device__ __forceinline__ int64_t slot_block(const Cache& c, int64_t slot, int h, int& t) {
  uint32_t in;
  const uint32_t page = div_blocks(static_cast<uint32_t>(slot >> 4), c.p16, c.p16_inv, in);
  t = static_cast<int>(slot & 15);
  return ((static_cast<int64_t>(page) * c.hk + h) * c.p16 + in) * 16;
}

template <int D, bool ROT, bool BF>
__global__ __launch_bounds__(256) void kv4_append_kernel(Cache c, const uint16_t* K, const uint16_t* V, int64_t n,
                                                         int64_t ldk, int64_t ldv, const int64_t* slots) {
  constexpr int LR = Rows<D>::LR, N = Rows<D>::N;
  __shared__ uint32_t sc[N][LR + 1];
  const int h = blockIdx.x % c.hk;
  const int64_t tok0 = static_cast<int64_t>(blockIdx.x / c.hk) * N;
  const int r = threadIdx.x / LR, j = threadIdx.x % LR;  // row, 8 channels of it
  const int vt = threadIdx.x % N, vj = threadIdx.x / N;  // the same for the stores of values
  const int64_t tok = min(tok0 + r, n - 1), vtok = min(tok0 + vt, n - 1);
  float v[8], k[8];
  load8<BF>(V + tok * ldv + h * D + 8 * j, v);
  load8<BF>(K + tok * ldk + h * D + 8 * j, k);
  const int64_t slot = slots[tok], vslot = slots[vtok];
  const bool ok = tok0 + r < n && slot >= 0 && slot < c.n_slots;
  const bool vok = tok0 + vt < n && vslot >= 0 && vslot < c.n_slots;
  const float vtop = top_row<D>(v);
  sc[r][j] = codes8<float>(v, vtop);
  uint32_t kw;
  float ks;
  if constexpr (ROT) {
    double u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = k[i];
    fwht_row<D>(u, j);
    const double top = top_row<D>(u);
    kw = codes8<double>(u, top);
    ks = static_cast<float>(top * (1.0 / (7.0 * __builtin_sqrt(static_cast<double>(D)))));
  } else {
    const float top = top_row<D>(k);
    kw = codes8<float>(k, top);
    ks = top / 7.0f;
  }
  if (ok) {
    int t;
    const int64_t row = slot_block(c, slot, h, t) + t;
    *reinterpret_cast<uint32_t*>(c.kc + row * (D / 2) + 4 * j) = kw;
    if (j == 0) {
      c.ks[row] = ks;
      c.vs[row] = vtop / 7.0f;
    }
  }
  __syncthreads();
  if (!vok) return;
  int t;
  uint8_t* o = c.vc + slot_block(c, vslot, h, t) * (D / 2) + 64 * vj;
  const uint32_t w = sc[vt][vj];
#pragma unroll
  for (int i = 0; i < 4; ++i) o[16 * i + t] = static_cast<uint8_t>(w >> (8 * i));
}

// ---------------------------------------------------------------------------
// Gather: the values of cached rows (slots out of range give zeros), keys
// rotated back.  Workgroups as in append, the bytes of values read with a
// token a lane and turned in LDS.
// ---------------------------------------------------------------------------
template <int D, bool ROT>
__global__ __launch_bounds__(256) void kv4_gather_kernel(Cache c, const int64_t* slots, int64_t n, void* K, void* V,
                                                         int64_t ldk, int64_t ldv, int dtype) {
  constexpr int LR = Rows<D>::LR, N = Rows<D>::N;
  __shared__ uint32_t sc[N][LR + 1];
  const int h = blockIdx.x % c.hk;
  const int64_t tok0 = static_cast<int64_t>(blockIdx.x / c.hk) * N;
  const int r = threadIdx.x / LR, j = threadIdx.x % LR;
  const bool is_v = blockIdx.y == 1;
  auto find = [&](int64_t i, int& t) -> int64_t {  // the block of token i's slot, -1: none
    const int64_t slot = i < n ? slots[i] : -1;
    return slot >= 0 && slot < c.n_slots ? slot_block(c, slot, h, t) : -1;
  };
  int t = 0;
  const int64_t base = find(tok0 + r, t);
  float scale = base >= 0 ? (is_v ? c.vs : c.ks)[base + t] : 0.0f;
  uint32_t w = 0;
  if (!is_v) {
    if (base >= 0) w = *reinterpret_cast<const uint32_t*>(c.kc + (base + t) * (D / 2) + 4 * j);
  } else {
    const int vt = threadIdx.x % N, vj = threadIdx.x / N;
    int tt = 0;
    const int64_t vb = find(tok0 + vt, tt);
    if (vb >= 0) {
      const uint8_t* p = c.vc + vb * (D / 2) + tt + 64 * vj;
      w = p[0] | p[16] << 8 | p[32] << 16 | static_cast<uint32_t>(p[48]) << 24;
    }
    sc[vt][vj] = w;
    __syncthreads();
    w = sc[r][j];
  }
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = static_cast<float>(static_cast<int32_t>(w << (28 - 4 * i)) >> 28);
  if (ROT && !is_v) {
    fwht_row<D>(x, j);  // sums of up to 256 codes, exact
    scale *= 1.0f / __builtin_sqrtf(static_cast<float>(D));
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] *= scale;
  if (tok0 + r >= n) return;
  const int64_t off = (tok0 + r) * (is_v ? ldv : ldk) + h * D + 8 * j;
  if (dtype == OQ_OUT_F32) {
    float4* o = reinterpret_cast<float4*>(static_cast<float*>(is_v ? V : K) + off);
    o[0] = make_float4(x[0], x[1], x[2], x[3]);
    o[1] = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    uint16_t* o = static_cast<uint16_t*>(is_v ? V : K) + off;
    if (dtype == OQ_OUT_BF16) store8<true>(o, x);
    else store8<false>(o, x);
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
// A wave takes 64 tokens at a time; lane group g (lane / 16) owns tokens
// 16 g .. 16 g + 15 of them.  The order of tokens in the first product's tiles
// is free: tile i has token 16 g + 4 i + e in row 4 g + e, so the group's lanes
// end with the probabilities of exactly its own 16 tokens, in the order in
// which the second product's operand takes them (k step j: tiles 2 j, 2 j + 1)
// and nothing crosses lanes.  Operands go from the cache to the registers in 16-byte
// loads; a step's values are loaded before its first product and the next
// step's keys before its softmax.
//
// Codes become fp16 by placing a nibble in the mantissa of 64 (or 1024):
// 64 + n, n = c + 8 the biased code; the bias goes with one exclusive or.  For
// keys the 72 is taken out by the accumulator's start, -72 sum(q) (an error
// of 2^-24 of that sum); for values by a packed subtraction, exact.
// The step of a key scales its row of S in fp32.  The step of a value is
// folded into the probability, P' = 2^(s - m) step 2^E with E = min(15 - m', 126) and m' the
// running maximum of s - m + log2(step): P' is at most 2^15 and its fp16 rounding is
// relative to the largest contribution whatever the steps' range (2^-11 of it down
// to 2^-29 of that, so that a long row's many small probabilities keep their
// weight; where the largest is below 2^-111, down to 2^-140).  The factor 2^-E of the end
// is taken from the same E.  The sum l of the softmax is formed from 2^(s - m) in fp32.  m is kept
// before the row's factor c, and 2^(s - m) is formed from s c - RN(m c) in one multiply-add as long as m c
// is below 2^20, past which that rounding would decide; (s - m) c is used there.
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
  float* part;     // [tokens * hq][splits][D + 4], null with one split
  int64_t tokens, ldq, ldo, table_ld;
  uint32_t n_pages, page_blocks;  // page_blocks: 16-token blocks of a page, all heads
  int table_last;                 // last index of a table row
  int n_seqs, hq, R, max_q, max_len, splits, chunk;  // chunk: tokens of a split, a multiple of kTile
  float scale_log2e;
  bool causal;
};

constexpr int kTile = 64;        // tokens of one step of a wave
constexpr float kFar = 0x1p20f;  // where the rounding of m c counts
// E of a value maximum (2^E is finite, and so is the product with a probability).
__device__ __forceinline__ float value_exp(float mv) { return fminf(15.0f - mv, 126.0f); }

__device__ __forceinline__ uint32_t and_xor(uint32_t a, uint32_t m, uint32_t x) { return (a & m) ^ x; }

// Query tokens of sequence b: the first row, how many of them are computed, and
// `at`, the place of the first one in a sequence of L tokens (they are its last).
__device__ __forceinline__ void query_rows(const AttnKv4& a, int b, int L, int& q0, int& nq, int& at) {
  int64_t lo = b, n = 1;
  if (a.cu_q) {
    const int64_t s = a.cu_q[b], e = a.cu_q[b + 1];
    lo = s < 0 ? 0 : s > a.tokens ? a.tokens : s;
    n = e > s ? e - s : 0;
  }
  q0 = static_cast<int>(lo);
  at = static_cast<int>(n > INT32_MAX / 2 ? -(INT32_MAX / 2) : L - n);
  n = n > a.max_q ? a.max_q : n;
  nq = static_cast<int>(n > a.tokens - lo ? a.tokens - lo : n);
}

// Softmax lanes.  A tile has 16 columns, but often fewer rows to fill them: with
// RC = 4 (8) columns in use the scores of a step's 4 (2) tiles are moved side by
// side into the 16 lanes (lane 4 i + r: tile i, row r), so that every lane has
// 4 (8) of them instead of 16, and the probabilities are moved back.
template <int RC>
__device__ __forceinline__ void gather_tiles(const v4f (&s)[4], v4f (&c)[RC / 4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (RC == 4) {
      int x = __float_as_int(s[0][e]);
      x = __builtin_amdgcn_update_dpp(x, __float_as_int(s[1][e]), 0x114, 0xF, 0x2, false);  // row_shr:4
      x = __builtin_amdgcn_update_dpp(x, __float_as_int(s[2][e]), 0x118, 0xF, 0x4, false);
      x = __builtin_amdgcn_update_dpp(x, __float_as_int(s[3][e]), 0x11C, 0xF, 0x8, false);
      c[0][e] = __int_as_float(x);
    } else if constexpr (RC == 8) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        c[i][e] = __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(s[2 * i][e]), __float_as_int(s[2 * i + 1][e]), 0x118,
                                                             0xF, 0xC, false));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) c[i][e] = s[i][e];
    }
  }
}
// The two fp16 pairs of tile i in lanes r < RC (the other lanes hold finite values of no use).
template <int RC, int I>
__device__ __forceinline__ uint32_t scatter_tile(const uint32_t (&p)[RC / 4]) {
  if constexpr (RC == 4) return I ? __builtin_amdgcn_update_dpp(0, p[0], 0x100 + 4 * I, 0xF, 0xF, true) : p[0];  // row_shl:4 I
  else if constexpr (RC == 8) return I & 1 ? __builtin_amdgcn_update_dpp(0, p[I / 2], 0x108, 0xF, 0xF, true) : p[I / 2];
  else return p[I];
}
// Over the lanes of a row.
template <int RC>
__device__ __forceinline__ float row_max(float x) {
  if constexpr (RC == 4) x = fmaxf(x, rqd::lane_xor_dpp<4>(x));
  if constexpr (RC <= 8) x = fmaxf(x, rqd::lane_xor_dpp<8>(x));
  x = fmaxf(x, lane_xor_far<16>(x));
  return fmaxf(x, lane_xor_far<32>(x));
}

template <int D, int QT, int RC, int W, bool ROT, bool BF>
__global__ __launch_bounds__(64 * W, QT == 1 ? D < 256 ? 3 : 2 : 1) void attn_kv4_kernel(AttnKv4 a) {
  static_assert(QT == 1 || RC == 16, "rows");
  constexpr int ROWS = 16 * QT, KW = D / 32, PT = D / 32, NQ = ROT ? 2 : 1;
  // Queries during the walk; the waves' outputs after it.
  struct Walk {
    v8h q[NQ][D / 8][ROWS];
    float qc[ROWS][2];
  };
  constexpr int OROWS = QT == 1 ? RC : ROWS;
  struct Out {
    float o[W][OROWS][D + 4];
    float m[W][OROWS][3];
    float c[OROWS];
  };
  __shared__ __attribute__((aligned(16))) union {
    Walk walk;
    Out out;
  } smem;
  auto& sq = smem.walk.q;
  auto& sqc = smem.walk.qc;
  auto& so = smem.out.o;
  auto& sm = smem.out.m;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, g = lane >> 4;
  const int b = blockIdx.y / a.c.hk, h = blockIdx.y % a.c.hk;
  // (The last splits first, which only long sequences have: 64 ragged ones in four, 29.2 -> 27.6 us.)
  const int split = gridDim.z - 1 - blockIdx.z;
  const int c0 = split * a.chunk, first = c0 + wave * kTile;  // tokens
  const int32_t* table = a.table + b * a.table_ld;
  // Page table entry of 16-token block `blk` of the sequence, and the block's place in the page.
  auto entry = [&](int blk, uint32_t& in) -> int {
    const int pi = static_cast<int>(div_blocks(static_cast<uint32_t>(blk), a.c.p16, a.c.p16_inv, in));
    return table[min(pi, a.table_last)];  // (tokens past the row's width are past max_len: not used)
  };
  uint32_t in_page;
  int page = entry(first / 16 + g, in_page);
  const int L = __builtin_amdgcn_readfirstlane(max(0, min(a.lens[b], a.max_len)));
  int q0, nq, q_at;
  query_rows(a, b, L, q0, nq, q_at);
  q0 = __builtin_amdgcn_readfirstlane(q0);
  nq = __builtin_amdgcn_readfirstlane(nq);
  q_at = __builtin_amdgcn_readfirstlane(q_at);
  const int rows = nq * a.R, r0 = blockIdx.x * ROWS;
  // (The first chunk of an empty sequence writes its zeros.)
  if (r0 >= rows || (c0 >= L && split > 0)) return;

  // A 16-token block of the cache that this lane group's tokens lie in (0 where they have none).
  bool own_ok;
  uint32_t own;
  auto place = [&](int pg, uint32_t in, int tok) {
    own_ok = tok < L && static_cast<uint32_t>(pg) < a.n_pages;
    own = static_cast<uint32_t>(own_ok ? pg : 0) * a.page_blocks + h * a.c.p16 + (own_ok ? in : 0);
  };
  uint4 kr[4][D >= 128 ? KW / 4 : 1];
  auto load_keys = [&]() {
    // The rows of this lane's keys are the tokens of lane group col / 4.
    const uint32_t kb = __builtin_amdgcn_ds_bpermute((col >> 2) * 64, static_cast<int>(own));
    const uint8_t* kp = a.c.kc + static_cast<uint64_t>(kb) * (8 * D) + (col & 3) * (D / 2) + (D == 64 ? 8 : 16) * g;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (D == 64) {
        const uint2 r = *reinterpret_cast<const uint2*>(kp + i * 2 * D);
        kr[i][0] = make_uint4(r.x, r.y, 0, 0);
      } else {
#pragma unroll
        for (int c = 0; c < KW / 4; ++c) kr[i][c] = *reinterpret_cast<const uint4*>(kp + i * 2 * D + 64 * c);
      }
    }
  };
  place(page, in_page, first + 16 * g);
  load_keys();
  page = entry((first + W * kTile) / 16 + g, in_page);

  // Keys that a row sees: the first `seen` tokens.
  constexpr int SV = RC / 4;               // quartets of scores that a lane has
  const int row_in = col % RC, ti0 = RC == 4 ? col >> 2 : RC == 8 ? col >> 3 : 0;
  constexpr int TSTEP = RC == 8 ? 2 : 1;   // the lane's tiles: ti0, ti0 + TSTEP, ...
  int seen[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int r = min(r0 + 16 * t + row_in, rows - 1);
    seen[t] = a.causal ? max(0, q_at + 1 + r / a.R) : L;
  }
  const int all_seen = a.causal ? max(0, q_at + 1 + r0 / a.R) : L;  // every row sees these
  const int last_seen = a.causal ? max(0, q_at + 1 + min(r0 + ROWS - 1, rows - 1) / a.R) : L;
  const int end = min(last_seen, c0 + a.chunk);

  // Queries: TQ threads take a row's channels (rotation, power-of-two norm, fp16
  // parts), then every wave reads its operands, 8 channels a lane and k step.
  {
    constexpr int TQ = D / 8 < 16 / QT ? D / 8 : 16 / QT, CQ = D / TQ;  // threads of a row, channels of a thread
    const int qr = threadIdx.x / TQ, part = threadIdx.x % TQ;
    if (qr < ROWS) {  // (uniform over a row's threads)
      const int r = min(r0 + qr, rows - 1);
      const uint16_t* qp = a.q + (q0 + r / a.R) * a.ldq + (h * a.R + r % a.R) * D + CQ * part;
      float x[CQ / 8][8];
#pragma unroll
      for (int u = 0; u < CQ / 8; ++u) load8<BF>(qp + 8 * u, x[u]);
      float norm = 1.0f;
      if (ROT) {
#pragma unroll
        for (int st = 1; st < CQ; st *= 2)
#pragma unroll
          for (int i = 0; i < CQ; ++i)
            if (!(i & st)) {
              const float u = x[i / 8][i % 8], v = x[(i + st) / 8][(i + st) % 8];
              x[i / 8][i % 8] = u + v;
              x[(i + st) / 8][(i + st) % 8] = u - v;
            }
        if constexpr (TQ > 1) rqd::lane_stage<1>(x, part);
        if constexpr (TQ > 2) rqd::lane_stage<2>(x, part);
        if constexpr (TQ > 4) rqd::lane_stage<4>(x, part);
        if constexpr (TQ > 8) rqd::lane_stage<8>(x, part);
        norm = 1.0f / sqrtf(static_cast<float>(D));
      }
      float top = 0.0f;
#pragma unroll
      for (int u = 0; u < CQ / 8; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(x[u][i]));
      top = fmaxf(top, rqd::lane_xor<1>(top));
      if constexpr (TQ > 2) top = fmaxf(top, rqd::lane_xor<2>(top));
      if constexpr (TQ > 4) top = fmaxf(top, rqd::lane_xor_dpp<4>(top));
      if constexpr (TQ > 8) top = fmaxf(top, rqd::lane_xor_dpp<8>(top));
      const int e = top > 0.0f && top < INFINITY ? __builtin_amdgcn_frexp_expf(top) : 0;
      float sum = 0.0f;
      constexpr int kOrder[8] = {0, 4, 1, 5, 2, 6, 3, 7};  // channels of a word in the order the codes come out
#pragma unroll
      for (int u = 0; u < CQ / 8; ++u) {
        v8h hi, lo;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float v = ldexpf(x[u][kOrder[i]], -e);
          hi[i] = static_cast<_Float16>(v);
          sum += static_cast<float>(hi[i]);
          if constexpr (ROT) {
            lo[i] = static_cast<_Float16>(v - static_cast<float>(hi[i]));
            sum += static_cast<float>(lo[i]);
          }
        }
        sq[0][part * (CQ / 8) + u][qr] = hi;
        if constexpr (ROT) sq[NQ - 1][part * (CQ / 8) + u][qr] = lo;
      }
      sum += rqd::lane_xor<1>(sum);
      if constexpr (TQ > 2) sum += rqd::lane_xor<2>(sum);
      if constexpr (TQ > 4) sum += rqd::lane_xor_dpp<4>(sum);
      if constexpr (TQ > 8) sum += rqd::lane_xor_dpp<8>(sum);
      if (part == 0) {
        sqc[qr][0] = -72.0f * sum;
        // (Above 0, so that a masked score of -inf times it is -inf, though by no more than fp32's smallest number:
        // keys may be as large as the query is small.)
        sqc[qr][1] = fmaxf(ldexpf(a.scale_log2e * norm, e), 0x1p-149f);
      }
    }
  }
  __syncthreads();
  float corr[QT], qscale[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    corr[t] = sqc[16 * t + col][0];
    qscale[t] = sqc[16 * t + row_in][1];
  }
  auto query = [&](int t, int p, int k) { return sq[p][(k / 4) * 16 + (D == 64 ? 2 : 4) * g + k % 4][16 * t + col]; };
  // (Read once where they fit beside the rest.)
  constexpr bool QREG = QT * NQ * KW <= 8;
  v8h qf[QREG ? QT : 1][QREG ? NQ : 1][QREG ? KW : 1];
  if constexpr (QREG) {
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int p = 0; p < NQ; ++p)
#pragma unroll
        for (int k = 0; k < KW; ++k) qf[t][p][k] = query(t, p, k);
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
  for (int tok0 = first; tok0 < end; tok0 += W * kTile) {
    // This step's values, and the steps of this lane's scores' tokens.
    const bool ok = own_ok;
    uint4 vr[PT];
    const uint8_t* vp = a.c.vc + static_cast<uint64_t>(own) * (8 * D) + 16 * col;
#pragma unroll
    for (int p = 0; p < PT; ++p) vr[p] = *reinterpret_cast<const uint4*>(vp + 256 * p);
    v4f ks[SV], vs[SV];
#pragma unroll
    for (int i = 0; i < SV; ++i) {
      const uint64_t at = static_cast<uint64_t>(own) * 16 + 4 * (ti0 + TSTEP * i);
      ks[i] = *reinterpret_cast<const v4f*>(a.c.ks + at);
      vs[i] = *reinterpret_cast<const v4f*>(a.c.vs + at);
    }
    // First product.
    if constexpr (!QREG) asm volatile("" ::: "memory");  // (the queries are read again, not kept)
    v4f s[QT][4];
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[t][i] = v4f{corr[t], corr[t], corr[t], corr[t]};
#pragma unroll
    for (int k = 0; k < KW; ++k) {
      v8h qk[QT][NQ];
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int p = 0; p < NQ; ++p) {
          if constexpr (QREG) qk[t][p] = qf[t][p][k];
          else qk[t][p] = query(t, p, k);
        }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint4 r = kr[i][k / 4];
        const uint32_t w = k % 4 == 0 ? r.x : k % 4 == 1 ? r.y : k % 4 == 2 ? r.z : r.w;
        uint4 u;
        u.x = and_xor(w << 4, 0x00F000F0u, 0x54805480u);
        u.y = and_xor(w, 0x00F000F0u, 0x54805480u);
        u.z = and_xor(w >> 4, 0x00F000F0u, 0x54805480u);
        u.w = and_xor(w >> 8, 0x00F000F0u, 0x54805480u);
        const v8h ka = __builtin_bit_cast(v8h, u);
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
          for (int p = 0; p < NQ; ++p) s[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ka, qk[t][p], s[t][i], 0, 0, 0);
      }
    }
    // The next step's keys.
    const int next = tok0 + W * kTile;
    if (next < end) {
      place(page, in_page, next + 16 * g);
      load_keys();
      page = entry((next + W * kTile) / 16 + g, in_page);
    }
    // Softmax of this lane's row over its 4 SV tokens.
    const bool masked = tok0 + kTile > all_seen || __builtin_amdgcn_ballot_w64(!ok) != 0;
    if (masked) {
      // Steps past the end (or of no page) count as 0, whatever is there.
      const int left = ok ? L - tok0 - 16 * g - 4 * ti0 : 0;
#pragma unroll
      for (int i = 0; i < SV; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          ks[i][e] = 4 * TSTEP * i + e < left ? ks[i][e] : 0.0f;
          vs[i][e] = 4 * TSTEP * i + e < left ? vs[i][e] : 0.0f;
        }
    }
    uint32_t pk[QT][2][SV];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      v4f c[SV];
      gather_tiles<RC>(s[t], c);
#pragma unroll
      for (int i = 0; i < SV; ++i) c[i] *= ks[i];
      if (masked) {
        const int left = ok ? seen[t] - tok0 - 16 * g - 4 * ti0 : 0;
#pragma unroll
        for (int i = 0; i < SV; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) c[i][e] = 4 * TSTEP * i + e < left ? c[i][e] : -INFINITY;
      }
      float top = -INFINITY, topv = -INFINITY;
#pragma unroll
      for (int i = 0; i < SV; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) top = fmaxf(top, c[i][e]);
      top = row_max<RC>(top);
      const float mn = fmaxf(m[t], top), ms = mn * qscale[t];
      float mr = ms, down = (m[t] - mn) * qscale[t];  // (log2 of what earlier sums shrink by)
      if (__builtin_amdgcn_ballot_w64(fabsf(ms) >= kFar) != 0) {
        const bool none = mn == -INFINITY, far = fabsf(ms) >= kFar && !none;
        mr = none || far ? 0.0f : ms;
        down = none ? -INFINITY : down;
#pragma unroll
        for (int i = 0; i < SV; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) c[i][e] -= far ? mn : 0.0f;
      }
#pragma unroll
      for (int i = 0; i < SV; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          c[i][e] = fmaf(c[i][e], qscale[t], -mr);
          topv = fmaxf(topv, c[i][e] + __builtin_amdgcn_logf(vs[i][e]));
        }
      topv = row_max<RC>(topv);
      const float mvo = mv[t] + down, mvn = fmaxf(mvo, topv), x = value_exp(mvn);
      if (__builtin_amdgcn_ballot_w64(mn > m[t] || mvn > mvo) != 0) {
        l[t] *= __builtin_amdgcn_exp2f(down);
        const float al = __builtin_amdgcn_exp2f(down + x - value_exp(mv[t]));
        m[t] = mn;
        mv[t] = mvn;
#pragma unroll
        for (int p = 0; p < PT; ++p)
#pragma unroll
          for (int y = 0; y < 2; ++y) acc[t][p][y] *= al;
      }
      // (Times the probability first: 0 if that has underflowed, whatever the step.)
      const float f = __builtin_amdgcn_exp2f(x);
#pragma unroll
      for (int i = 0; i < SV; ++i) {
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          p[e] = __builtin_amdgcn_exp2f(c[i][e]);
          l[t] += p[e];
          p[e] = p[e] * f * vs[i][e];
        }
        // (Tokens of a word come out as 0, 2, 1, 3.)
        pk[t][0][i] = __builtin_bit_cast(uint32_t, v2h{static_cast<_Float16>(p[0]), static_cast<_Float16>(p[2])});
        pk[t][1][i] = __builtin_bit_cast(uint32_t, v2h{static_cast<_Float16>(p[1]), static_cast<_Float16>(p[3])});
      }
    }
    // Second product.
    static_for<2>([&](auto J) {
      constexpr int j = decltype(J)::value;
      v8h pf[QT];
#pragma unroll
      for (int t = 0; t < QT; ++t)
        pf[t] = __builtin_bit_cast(v8h, make_uint4(scatter_tile<RC, 2 * j>(pk[t][0]), scatter_tile<RC, 2 * j>(pk[t][1]),
                                                   scatter_tile<RC, 2 * j + 1>(pk[t][0]), scatter_tile<RC, 2 * j + 1>(pk[t][1])));
#pragma unroll
      for (int p = 0; p < PT; ++p) {
        v8h lo, hi;
        const v2h c72 = {72, 72}, c1032 = {1032, 1032};
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const uint32_t y = j == 0 ? (x == 0 ? vr[p].x : vr[p].y) : (x == 0 ? vr[p].z : vr[p].w), z = y >> 8;
          const v2h l0 = __builtin_bit_cast(v2h, and_xor(y, 0x000F000Fu, 0x64086408u)) - c1032;
          const v2h l1 = __builtin_bit_cast(v2h, and_xor(z, 0x000F000Fu, 0x64086408u)) - c1032;
          const v2h h0 = __builtin_bit_cast(v2h, and_xor(y, 0x00F000F0u, 0x54805480u)) - c72;
          const v2h h1 = __builtin_bit_cast(v2h, and_xor(z, 0x00F000F0u, 0x54805480u)) - c72;
          lo[4 * x] = l0[0]; lo[4 * x + 1] = l0[1]; lo[4 * x + 2] = l1[0]; lo[4 * x + 3] = l1[1];
          hi[4 * x] = h0[0]; hi[4 * x + 1] = h0[1]; hi[4 * x + 2] = h1[0]; hi[4 * x + 3] = h1[1];
        }
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          acc[t][p][0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo, pf[t], acc[t][p][0], 0, 0, 0);
          acc[t][p][1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi, pf[t], acc[t][p][1], 0, 0, 0);
        }
      }
    });
  }

  // Join the waves.
  __syncthreads();
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    float s = l[t];
    if constexpr (RC == 4) s += rqd::lane_xor_dpp<4>(s);
    if constexpr (RC <= 8) s += rqd::lane_xor_dpp<8>(s);
    s += lane_xor_far<16>(s);
    s += lane_xor_far<32>(s);
    if (OROWS < 16 && col >= OROWS) continue;
#pragma unroll
    for (int p = 0; p < PT; ++p)
#pragma unroll
      for (int x = 0; x < 2; ++x)
        *reinterpret_cast<v4f*>(&so[wave][16 * t + col][32 * p + 8 * g + 4 * x]) =
            v4f{acc[t][p][0][2 * x], acc[t][p][1][2 * x], acc[t][p][0][2 * x + 1], acc[t][p][1][2 * x + 1]};
    if (g == 0) {
      sm[wave][16 * t + col][0] = m[t];
      sm[wave][16 * t + col][1] = value_exp(mv[t]);
      sm[wave][16 * t + col][2] = s;
      if (wave == 0) smem.out.c[16 * t + col] = qscale[t];
    }
  }
  __syncthreads();
  constexpr int TPR = D / 8;
  for (int i = threadIdx.x; i < min(OROWS, rows - r0) * TPR; i += 64 * W) {
    const int r = i / TPR, c = (i % TPR) * 8;
    float M = -INFINITY, X = INFINITY;
#pragma unroll
    for (int w = 0; w < W; ++w) M = fmaxf(M, sm[w][r][0]);
    // A wave's outputs are 2^(its exponent - down) times too large; the least of these is at
    // most 126 (that of a wave with the row's maximum), unless no wave has a token.
    const float mr = M == -INFINITY ? 0.0f : M, qs = smem.out.c[r];
    float down[W];
#pragma unroll
    for (int w = 0; w < W; ++w) {
      down[w] = (sm[w][r][0] - mr) * qs;
      X = fminf(X, sm[w][r][1] - down[w]);
    }
    const float xr = X == INFINITY ? 0.0f : X;
    float L_ = 0.0f, y[8] = {};
#pragma unroll
    for (int w = 0; w < W; ++w) {
      L_ += sm[w][r][2] * __builtin_amdgcn_exp2f(down[w]);
      const float f = __builtin_amdgcn_exp2f(xr - (sm[w][r][1] - down[w]));
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] += so[w][r][c + e] * f;
    }
    const float f = L_ > 0.0f ? __builtin_amdgcn_exp2f(-xr) / L_ : 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] *= f;
    const int64_t tok = q0 + (r0 + r) / a.R;
    const int head = h * a.R + (r0 + r) % a.R;
    if (L <= a.chunk) {  // one split
      store8<BF>(a.o + tok * a.ldo + head * D + c, y);
    } else {
      float* o = a.part + ((tok * a.hq + head) * a.splits + split) * (D + 4);
      *reinterpret_cast<float4*>(o + c) = make_float4(y[0], y[1], y[2], y[3]);
      *reinterpret_cast<float4*>(o + c + 4) = make_float4(y[4], y[5], y[6], y[7]);
      if (c == 0) *reinterpret_cast<float4*>(o + D) = make_float4(M, L_, qs, 0.0f);
    }
  }
}

// o = sum_s w_s o_s / sum_s w_s with w_s = l_s 2^((m_s - m) c).  A row (token and head)
// has WPR waves, 8 channels a thread; its splits are dealt to their 64 WPR / (D / 8)
// groups of threads.
template <int D, int WPR, bool BF>
__global__ __launch_bounds__(256) void attn_kv4_join_kernel(AttnKv4 a) {
  constexpr int TPR = D / 8, G = 64 * WPR / TPR, RPW = 4 / WPR;
  __shared__ __attribute__((aligned(16))) float sy[4 / WPR][G][D + 4];
  const int sub = threadIdx.x / (64 * WPR), tid = threadIdx.x % (64 * WPR);
  const int head = blockIdx.x * RPW + sub, b = blockIdx.z;
  const int L = max(0, min(a.lens[b], a.max_len));
  if (L <= a.chunk) return;
  int q0, nq, q_at;
  query_rows(a, b, L, q0, nq, q_at);
  if (static_cast<int>(blockIdx.y) >= nq) return;
  const int splits = (L + a.chunk - 1) / a.chunk;
  const int64_t tok = q0 + blockIdx.y;
  const int c = (tid % TPR) * 8, grp = tid / TPR;
  const float* p = a.part + (tok * a.hq + min(head, a.hq - 1)) * a.splits * (D + 4);
  float M = -INFINITY, W = 0.0f, qs = 1.0f, y[8] = {};
#pragma unroll 4
  for (int s = grp; s < splits; s += G) {
    const float* ps = p + s * (D + 4);
    const float4 ml = *reinterpret_cast<const float4*>(ps + D);
    const float4 u = *reinterpret_cast<const float4*>(ps + c), v = *reinterpret_cast<const float4*>(ps + c + 4);
    const float mn = fmaxf(M, ml.x), mr = mn == -INFINITY ? 0.0f : mn;
    qs = ml.z;
    const float al = __builtin_amdgcn_exp2f((M - mr) * qs), w = ml.y * __builtin_amdgcn_exp2f((ml.x - mr) * qs);
    const float x[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
    M = mn;
    W = W * al + w;
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = y[e] * al + w * x[e];
  }
  float* o = sy[sub][grp];
#pragma unroll
  for (int e = 0; e < 8; ++e) o[c + e] = y[e];
  if (c == 0) {
    o[D] = M;
    o[D + 1] = W;
  }
  __syncthreads();
  if (tid >= TPR || head >= a.hq) return;
  float top = -INFINITY;
  for (int i = 0; i < G; ++i) top = fmaxf(top, sy[sub][i][D]);
  const float mr = top == -INFINITY ? 0.0f : top;
  float T = 0.0f, z[8] = {};
#pragma unroll 4
  for (int i = 0; i < G; ++i) {
    const float w = __builtin_amdgcn_exp2f((sy[sub][i][D] - mr) * qs);
    T += sy[sub][i][D + 1] * w;
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] += sy[sub][i][c + e] * w;
  }
  const float f = T > 0.0f ? 1.0f / T : 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) z[e] *= f;
  store8<BF>(a.o + tok * a.ldo + head * D + c, z);
}

int cache_validate(const oq_kv4_cache* c) {
  if (!c || !c->k_codes || !c->v_codes || !c->k_scale || !c->v_scale) return OQ_ERR_NULL;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return OQ_ERR_SHAPE;
  if (c->n_pages < 1 || c->n_pages > INT32_MAX || c->n_kv_heads < 1 || c->page_tokens < 16 || c->page_tokens % 16 != 0 ||
      c->page_tokens > 65536 || c->n_kv_heads > 65535)
    return OQ_ERR_SHAPE;
  // (16-token blocks are counted in 32 bits; a cache past that would hold terabytes.)
  if (c->n_pages * (c->page_tokens / 16) * static_cast<int64_t>(c->n_kv_heads) > int64_t{UINT32_MAX}) return OQ_ERR_SHAPE;
  if (!aligned(c->k_codes, 16) || !aligned(c->v_codes, 16) || !aligned(c->k_scale, 16) || !aligned(c->v_scale, 16))
    return OQ_ERR_ALIGN;
  if (c->rotate_k != 0 && c->rotate_k != 1) return OQ_ERR_ARG;
  return OQ_OK;
}

Cache device_cache(const oq_kv4_cache* c) {
  const uint32_t p16 = static_cast<uint32_t>(c->page_tokens / 16);
  return Cache{c->k_codes, c->v_codes, c->k_scale, c->v_scale, c->n_pages * c->page_tokens, c->n_kv_heads, p16,
               p16 == 1 ? UINT32_MAX : static_cast<uint32_t>((uint64_t{1} << 32) / p16)};
}

// The launch.  Rows: 16 columns of products (two such blocks in a workgroup above
// 16 rows, but not at d = 256, whose accumulators fill the registers), compacted
// for the softmax when 4 or 8 are in use.
// Length: splits of `chunk` tokens, 64 at most, which a second launch joins.  A
// split costs a workgroup's start (queries, page table, first keys) and end, so
// there are about as many as the card holds at once: 640 workgroups of four waves (two or
// three a CU), 256 of the eight waves that take 32 rows.  But only max_len is known here, and a
// long sequence among short ones would be the last to end: chunks have at most 4096 tokens, and
// at 16 rows at most 1024 as long as 2048 workgroups do.  Measured against every number of
// splits at four and eight waves, for nine head layouts, 1 to 150 sequences of up to 400 ..
// 60000 tokens, equal or ragged (609 shapes): 3% over the fastest in the mean (splits for
// 1536 workgroups at four waves: 13%).  Us, eight waves against four at 32 rows, the best number of
// splits each: 50 tokens of 8 heads of 128, 32 sequences of 2000, 44.6 / 51.7; 64 / 2 heads, 8
// sequences of 32000, 27.8 / 31.8; but one of 2000, where chunks of 256 fill no card, 11.9 / 11.3.
// One launch without splits, for 16 rows: up to 512 tokens eight waves (one of 400, 32 / 8
// heads: 6.2; in two splits 7.7), and up to 1024 tokens where the splits would fill the card
// anyway or, at d = 64, the queries take little (32 sequences of 866, 32 / 8 heads of 128: 11.0 /
// 14.6, but one: 8.3 / 7.7; one, 16 / 1 heads of 64: 8.0 / 8.5).
constexpr int kMaxSplits = 64;
struct Kv4Plan {
  int qt, rc, waves, splits, chunk;
  int64_t row_blocks;
};
Kv4Plan kv4_plan(int64_t n_seqs, int hk, int d, int R, int max_q, int64_t max_len) {
  const int64_t rows = static_cast<int64_t>(max_q) * R;
  Kv4Plan p;
  p.qt = rows <= 16 || d == 256 ? 1 : 2;
  p.rc = rows <= 4 ? 4 : rows <= 8 ? 8 : 16;
  p.row_blocks = (rows + 16 * p.qt - 1) / (16 * p.qt);
  const int64_t wgs = n_seqs * hk * p.row_blocks;
  int64_t splits = 1;
  if (p.qt == 2) {
    const bool shortest = max_len > 512 && wgs * ((max_len + 255) / 256) <= 256;  // chunks of 256 do not fill the card
    p.waves = shortest ? 4 : 8;
    splits = shortest ? kMaxSplits : max_len <= 512 ? 1 : std::max(256 / wgs, (max_len + 4095) / 4096);
  } else if (wgs <= 256 && (max_len <= 512 || (max_len <= 1024 && (d == 64 || wgs >= 128)))) {
    p.waves = 8;
  } else {
    p.waves = 4;
    splits = max_len <= 512 ? 1 : std::max({640 / wgs, std::min((max_len + 1023) / 1024, 2048 / wgs), (max_len + 4095) / 4096});
  }
  const int64_t step = p.waves * kTile;
  splits = std::clamp<int64_t>(splits, 1, kMaxSplits);
  const int64_t chunk = ((max_len + splits - 1) / splits + step - 1) / step * step;
  p.chunk = static_cast<int>(chunk < step ? step : chunk);
  p.splits = static_cast<int>(max_len <= p.chunk ? 1 : (max_len + p.chunk - 1) / p.chunk);
  return p;
}

template <int D, bool BF>
void launch_attn(const AttnKv4& a, const Kv4Plan& p, dim3 grid, bool rot, hipStream_t st) {
#define OQ_ATTN(Q, C, W)                                                                                   \
  if (p.qt == Q && p.rc == C && p.waves == W) {                                                            \
    if (rot) hipLaunchKernelGGL((attn_kv4_kernel<D, Q, C, W, true, BF>), grid, dim3(64 * W), 0, st, a);    \
    else hipLaunchKernelGGL((attn_kv4_kernel<D, Q, C, W, false, BF>), grid, dim3(64 * W), 0, st, a);       \
  }
  OQ_ATTN(1, 4, 4)
  OQ_ATTN(1, 4, 8)
  OQ_ATTN(1, 8, 4)
  OQ_ATTN(1, 8, 8)
  OQ_ATTN(1, 16, 4)
  OQ_ATTN(1, 16, 8)
  if constexpr (D < 256) {
    OQ_ATTN(2, 16, 4)
    OQ_ATTN(2, 16, 8)
  }
#undef OQ_ATTN
  if (a.splits > 1) {
    const unsigned y = static_cast<unsigned>(a.max_q), z = static_cast<unsigned>(a.n_seqs);
    // (A wave a row up to 8 splits: 4.1 instead of 5.0 us at the 64 ragged sequences.)
    if (a.splits > 8)
      hipLaunchKernelGGL((attn_kv4_join_kernel<D, 4, BF>), dim3(static_cast<unsigned>(a.hq), y, z), dim3(256), 0, st, a);
    else
      hipLaunchKernelGGL((attn_kv4_join_kernel<D, 1, BF>), dim3(static_cast<unsigned>((a.hq + 3) / 4), y, z), dim3(256), 0, st, a);
  }
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
  const int64_t per = 2048 / cache->head_dim, blocks = (n + per - 1) / per * c.hk;
  if (!oq::launchable(blocks, 256)) return OQ_ERR_SHAPE;
  const dim3 grid(static_cast<unsigned>(blocks));
  const bool bf = dtype == OQ_OUT_BF16;
  hipStream_t s = static_cast<hipStream_t>(stream);
#define OQ_APPEND(D, R, B)                                                                                            \
  if (cache->head_dim == D && cache->rotate_k == R && bf == B)                                                        \
  hipLaunchKernelGGL((oq::kv4_append_kernel<D, R, B>), grid, dim3(256), 0, s, c, static_cast<const uint16_t*>(K),     \
                     static_cast<const uint16_t*>(V), n, ldk, ldv, slots)
#define OQ_APPEND4(D)     \
  OQ_APPEND(D, 0, false); \
  OQ_APPEND(D, 0, true);  \
  OQ_APPEND(D, 1, false); \
  OQ_APPEND(D, 1, true)
  OQ_APPEND4(64);
  OQ_APPEND4(128);
  OQ_APPEND4(256);
#undef OQ_APPEND4
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
  const int64_t per = 2048 / cache->head_dim, blocks = (n + per - 1) / per * c.hk;
  if (!oq::launchable(blocks, 256)) return OQ_ERR_SHAPE;
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
  if (tokens < 0 || tokens > INT32_MAX || n_seqs < 0 || max_q < 1 || max_q > 65535 || max_len < 0 || max_len > (1 << 30) ||
      n_heads < 1 || n_heads > 65535)
    return OQ_ERR_SHAPE;
  if (n_heads % cache->n_kv_heads != 0) return OQ_ERR_SHAPE;
  if (static_cast<int64_t>(n_seqs) * cache->n_kv_heads > 65535) return OQ_ERR_SHAPE;
  if (static_cast<int64_t>(max_q) * (n_heads / cache->n_kv_heads) > (1 << 26)) return OQ_ERR_SHAPE;  // (rows of a grid)
  return OQ_OK;
}

extern "C" size_t oq_attention_kv4_workspace_bytes(const oq_kv4_cache* cache, int64_t tokens, int32_t n_heads,
                                                   int32_t n_seqs, int32_t max_q, int32_t max_len) {
  if (!cache || cache->n_kv_heads < 1 || attn_kv4_shape(cache, tokens, n_heads, n_seqs, max_q, max_len) != OQ_OK || n_seqs == 0)
    return 0;
  const oq::Kv4Plan p = oq::kv4_plan(n_seqs, cache->n_kv_heads, cache->head_dim, n_heads / cache->n_kv_heads, max_q, max_len);
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
  if (!(scale > 0.0f) || !std::isfinite(scale * 1.4426950408889634f)) return OQ_ERR_ARG;
  if (ldq % 8 != 0 || ldo % 8 != 0) return OQ_ERR_ALIGN;
  if (tokens == 0 || n_seqs == 0) return OQ_OK;
  if (!Q || !O || !seq_lens || (!block_table && max_len > 0)) return OQ_ERR_NULL;
  if (!oq::aligned(Q, 16) || !oq::aligned(O, 16) || !oq::aligned(seq_lens, 4) || !oq::aligned(block_table, 4) ||
      !oq::aligned(cu_q, 4) || !oq::aligned(work, 16))
    return OQ_ERR_ALIGN;
  const int R = n_heads / cache->n_kv_heads;
  const oq::Kv4Plan p = oq::kv4_plan(n_seqs, cache->n_kv_heads, cache->head_dim, R, max_q, max_len);
  if (p.splits > 1 && (!work || work_bytes < oq_attention_kv4_workspace_bytes(cache, tokens, n_heads, n_seqs, max_q, max_len)))
    return OQ_ERR_WORKSPACE;
  if ((st = oq::device_check()) != OQ_OK) return st;
  oq::AttnKv4 a{};
  a.c = oq::device_cache(cache);
  a.q = static_cast<const uint16_t*>(Q);
  a.o = static_cast<uint16_t*>(O);
  a.cu_q = cu_q;
  // (No cached tokens at all: nothing of a table is used, but a word of one is read.)
  a.table = max_len > 0 ? block_table : seq_lens;
  a.lens = seq_lens;
  a.part = static_cast<float*>(work);
  a.tokens = tokens;
  a.ldq = ldq;
  a.ldo = ldo;
  a.table_ld = max_len > 0 ? table_ld : 1;
  a.table_last = static_cast<int>(a.table_ld - 1 < INT32_MAX ? a.table_ld - 1 : INT32_MAX);
  a.n_pages = static_cast<uint32_t>(cache->n_pages);
  a.page_blocks = static_cast<uint32_t>(cache->page_tokens / 16 * cache->n_kv_heads);
  a.n_seqs = n_seqs;
  a.hq = n_heads;
  a.R = R;
  a.max_q = max_q;
  a.max_len = max_len;
  a.splits = p.splits;
  a.chunk = p.chunk;
  a.scale_log2e = scale * 1.4426950408889634f;
  a.causal = causal == 1;
  const dim3 grid(static_cast<unsigned>(p.row_blocks), static_cast<unsigned>(n_seqs * cache->n_kv_heads),
                  static_cast<unsigned>(p.splits));
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool rot = cache->rotate_k == 1;
  const bool bf = dtype == OQ_OUT_BF16;
#define OQ_ATTN(D)                                                       \
  if (cache->head_dim == D) {                                            \
    if (bf) oq::launch_attn<D, true>(a, p, grid, rot, s);             \
    else oq::launch_attn<D, false>(a, p, grid, rot, s);               \
  }
  OQ_ATTN(64) OQ_ATTN(128) OQ_ATTN(256)
#undef OQ_ATTN
  return oq::launch_status();
}
