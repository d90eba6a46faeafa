// Softmax self-attention within packed sequences (prompts), grouped heads,
// causal or full.
//
// A workgroup takes 32 query tokens a row wave (2 or 4 of them) of one sequence and head
// and walks the sequence's keys in steps of BN with a running maximum m and sum l
// per row (one pass over K and V; nothing of the pair matrix leaves the
// registers).  Both products are transposed, on v_mfma_f32_32x32x16: S^T = K Q^T
// (keys x rows) leaves each lane half of one row's probabilities, already in the
// operand layout of O^T = V^T P^T (channels x rows) once the keys of a 16-key
// step are taken in the order 4 h .. 4 h + 3, 8 + 4 h .. 8 + 4 h + 3 (h = lane /
// 32), the same in both operands; V is read from LDS with the transposing 16-bit
// read, four keys of a channel a lane.  K and V tiles go from global memory into
// two LDS buffers with 16-byte direct loads, the next tile's while this one is
// multiplied, one barrier per step.
//
// What bounds it: at d = 128 a step of 64 keys and 32 rows costs a wave 1024
// cycles of matrix instructions, about 700 of the vector unit (32 exponentials at a
// quarter of its rate, as many multiply-adds, half as many maxima, packed roundings and dot
// products that add the rounded probabilities) and 32 KB of LDS reads; two waves a SIMD
// overlap them.  One causal sequence of 8192, 32 / 8 heads of 128: 537 to 598 us on several cards, 1024 to 920
// TFLOP/s, about 85% of what the library's 8192-cubed bf16 product reaches; 64 rows
// a wave (half the LDS reads, one wave a SIMD) 857 against 561 us; 32-key steps 604.
//
// Probabilities are rounded to the inputs' type for the second product and
// summed as rounded, so that the weights add up to one.  fp16 ones are taken times
// 2^15 (the division by l removes it): those above 2^-29 of a row's largest are
// normal numbers, and many small ones keep their weight together.
//
// The exponent is s c - RN(m c) in one multiply-add (c = scale log2(e)) where m c is
// below 2^20: RN(m c) is then within 2^-5 of m c, and a probability at most 2^(15 + 1/16).  Past that
// the rounding could make it any number, inf and 0 among them, so there m is taken from the
// scores first, (s - m) c.
//
// LDS rows are not padded; 16-byte pieces of a row are stored at piece ^ a
// function of the row.  K: 16 rows of one piece cover all banks.  V: 4 rows of 4
// pieces do.
//
// Keys past the sequence's end are read as its last row, so that what lies
// behind it (other sequences, unused rows) never enters a product.
#include <cmath>

#include "common.h"
#include "rq_device.h"

namespace oq {
namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));
typedef __bf16 v2b __attribute__((ext_vector_type(2)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));

struct PromptArgs {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* o;
  const int32_t* cu;
  int64_t ldq, ldk, ldv, ldo;
  int tokens, n_seqs, hq, rep, tiles;  // tiles: of one head, at most
  float scale_log2e;
  bool causal;
};

// Lane l's 16 bytes at base + voff to LDS byte lds + 16 l.
__device__ __forceinline__ void dma16(uint32_t lds, uint32_t voff, const void* base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(voff), "s"(base)
               : "memory", "m0");
}

// The types' operations; probabilities are scaled by 2^kShift.
template <bool BF>
struct Half;
template <>
struct Half<false> {
  typedef v8h v8;
  static constexpr float kShift = 15.0f;
  static __device__ __forceinline__ v16f mfma(v8 a, v8 b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    return rqd::f2h(a) | static_cast<uint32_t>(rqd::f2h(b)) << 16;
  }
  static __device__ __forceinline__ float add2(uint32_t p, float l) {
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(v2h, p), v2h{1, 1}, l, false);
  }
};
template <>
struct Half<true> {
  typedef v8b v8;
  static constexpr float kShift = 0.0f;
  static __device__ __forceinline__ v16f mfma(v8 a, v8 b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    const v2b p = {static_cast<__bf16>(a), static_cast<__bf16>(b)};
    return __builtin_bit_cast(uint32_t, p);
  }
  static __device__ __forceinline__ float add2(uint32_t p, float l) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2b, p), v2b{static_cast<__bf16>(1.0f), static_cast<__bf16>(1.0f)}, l,
                                           false);
  }
};

constexpr float kFar = 0x1p20f;  // where the rounding of m c counts (m: a row's largest score)
// RN(m c), whatever it is used in (in a fused multiply-add it would not cancel with itself).
__device__ __forceinline__ float scaled(float m, float c) {
#pragma clang fp contract(off)
  return m * c;
}
// Exponent that turns sums relative to the maximum a into those relative to b >= a.
__device__ __forceinline__ float from_to(float a, float b, float c) {
  const float bs = scaled(b, c);
  return fabsf(bs) >= kFar ? (a - b) * c : scaled(a, c) - bs;
}

template <bool BF, int D, int BN, int RW, int KG>
__global__ __launch_bounds__(64 * RW * KG, 2) void prompt_attn_kernel(PromptArgs a) {
  typedef Half<BF> H;
  typedef typename H::v8 v8;
  constexpr int BM = 32 * RW, PCS = D / 8, ROWB = 2 * D;
  constexpr int KB = BN * ROWB, STAGE = 2 * KB;
  constexpr int LK = KB / 1024 / RW;  // 1 KB loads of K (and of V) per wave and tile
  constexpr int SUB = BN / 32, CT = D / 32, KS = D / 16;
  constexpr int JOINB = KG > 1 ? (KG - 1) * RW * 64 * (16 * CT + 2) * 4 : 0;
  __shared__ __attribute__((aligned(16))) uint8_t smem[2 * STAGE * KG > JOINB ? 2 * STAGE * KG : JOINB];

  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wave = wv % RW, grp = wv / RW;
  const int col = lane & 31, h = lane >> 5;
  // Consecutive ids go to different XCDs (id % 8).  With a multiple of 8 heads an
  // XCD takes whole heads, so that those which share K and V share its L2; else
  // the heads go round.  Tiles come in falling order (the later a causal tile, the
  // more keys it has), but where a CU holds several workgroups the second of each
  // of an XCD's 32 CUs in rising order, so that long and short ones meet (one
  // causal sequence of 4096, 32 / 8 heads of 128: 180 -> 151 us).
  const int id = blockIdx.x;
  int head, tile;
  {
    const bool whole = a.hq % 8 == 0;
    const int heads = whole ? a.hq / 8 : a.hq, cus = whole ? 32 : 256, n = heads * a.tiles;
    int k = whole ? id >> 3 : id;
    if ((KG == 1 || D == 64) && k >= cus && k < 2 * cus) k = min(2 * cus, n) - 1 - (k - cus);
    tile = k / heads;
    head = (whole ? (id & 7) * heads : 0) + k % heads;
  }
  // The tile's sequence: a running count of the sequences' tiles, 64 at a time.
  int lo = 0, hi = 0, found = 0;
  for (int s0 = 0; s0 < a.n_seqs; s0 += 64) {
    const int s = s0 + lane;
    int b = 0, e = 0;
    if (s < a.n_seqs) {
      b = min(max(a.cu[s], 0), a.tokens);
      e = min(max(a.cu[s + 1], b), a.tokens);
    }
    const int nt = (e - b + BM - 1) / BM;
    int sum = nt;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int u = __shfl_up(sum, d);
      sum += lane >= d ? u : 0;
    }
    const int all = __builtin_amdgcn_readlane(sum, 63);
    if (tile < all) {
      const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(sum > tile));
      lo = __builtin_amdgcn_readlane(b, at);
      hi = __builtin_amdgcn_readlane(e, at);
      // The tiles with the most keys first.
      tile = __builtin_amdgcn_readlane(sum, at) - 1 - tile;
      found = 1;
      break;
    }
    tile -= all;
  }
  if (!found) return;
  const int r0 = lo + tile * BM;
  const int kend = a.causal ? min(hi, r0 + BM) : hi;
  const int wrow = r0 + wave * 32;  // the wave's first row

  const uint16_t* kbase = a.k + (head / a.rep) * D + static_cast<int64_t>(lo) * a.ldk;
  const uint16_t* vbase = a.v + (head / a.rep) * D + static_cast<int64_t>(lo) * a.ldv;
  const uint32_t ring = grp * 2 * STAGE;  // the key group's two buffers
  const uint32_t lds0 = ring + static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t*)smem));
  const uint32_t ldk2 = static_cast<uint32_t>(2 * a.ldk), ldv2 = static_cast<uint32_t>(2 * a.ldv);
  auto swzk = [](int row) { return PCS == 8 ? (row >> 1) & 7 : row & 15; };
  auto swzv = [](int row) { return PCS == 8 ? ((row >> 1) & 1) << 2 : (row & 3) << 2; };
  auto issue = [&](int k0, int buf) {
    const uint16_t* kb = kbase + (k0 - lo) * a.ldk;
    const uint16_t* vb = vbase + (k0 - lo) * a.ldv;
    const int lim = hi - 1 - k0;
#pragma unroll
    for (int i = 0; i < LK; ++i) {
      const int l = wave * LK + i;
      const int row = l * (64 / PCS) + lane / PCS, slot = lane % PCS;
      const uint32_t rr = static_cast<uint32_t>(min(row, lim));
      dma16(lds0 + buf * STAGE + l * 1024, rr * ldk2 + 16 * (slot ^ swzk(row)), kb);
      dma16(lds0 + buf * STAGE + KB + l * 1024, rr * ldv2 + 16 * (slot ^ swzv(row)), vb);
    }
  };
  const int k_first = lo + grp * BN;
  if (k_first < kend) issue(k_first, 0);

  v8 qf[KS];
  {
    const int r = min(wrow + col, hi - 1);
    const uint16_t* qp = a.q + static_cast<int64_t>(r) * a.ldq + head * D + 8 * h;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const v8*>(qp + 16 * ks);
  }
  v16f acc[CT];
  // The maximum, what a score has to pass to change it, and what the exponents are taken from.
  float m = -INFINITY, seen = -INFINITY, mr = -H::kShift, l = 0.0f;
#pragma unroll
  for (int c = 0; c < CT; ++c)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[c][e] = 0.0f;
  // LDS byte offsets of this lane's reads within a buffer; the rest of an address is constant.
  // K: row 32 u + col, piece 2 ks + h at slot piece ^ swzk(col): 2 ks differs from
  // (2 ks) % (2 KO) by whole runs of 2 KO pieces, which the exclusive or leaves.
  constexpr int KO = KS < 8 ? KS : 8;
  uint32_t koff[KO];
#pragma unroll
  for (int i = 0; i < KO; ++i) koff[i] = ring + col * ROWB + (((2 * i) ^ h ^ swzk(col)) << 4);
  // V: row 32 u + 16 j + 8 y + 4 h + vi / 4, channels 32 ct + 16 vg + 4 (vi % 4).
  constexpr int VO = CT < 4 ? CT : 4;
  const int vi = lane & 15, vg = (lane >> 4) & 1, vrow = 4 * h + (vi >> 2);
  uint32_t voff[VO];
#pragma unroll
  for (int i = 0; i < VO; ++i)
    voff[i] = ring + KB + vrow * ROWB + (((4 * i + 2 * vg + ((vi & 3) >> 1)) ^ swzv(vrow)) << 4) + 8 * (vi & 1);
  const float c = a.scale_log2e;
  uint32_t buf = 0;
  // Where the loop begins counts by up to 5%: 28 bytes past a 64-byte line is among the best of the 16 places
  // (one causal sequence of 8192, 32 / 8 heads of 128, bf16: 565 us, at even ones 584; 2000 of d = 256 77.6, 81.5).
  asm volatile(".p2align 6\n\t.rept 7\n\ts_nop 0\n\t.endr");
  // (Every wave passes every barrier: the groups take the same number of steps.)
  for (int k0 = k_first, kb0 = lo; kb0 < kend; k0 += KG * BN, kb0 += KG * BN, buf ^= 1) {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (k0 + KG * BN < kend) issue(k0 + KG * BN, buf ^ 1);
    const int wlast = min(wrow + 32, hi) - 1;
    if (k0 >= kend || (a.causal && k0 > wlast)) continue;  // (this wave's rows see none of the tile)
    const uint8_t* sb = smem + buf * STAGE;
    v16f s[SUB];
#pragma unroll
    for (int u = 0; u < SUB; ++u)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[u][e] = 0.0f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int u = 0; u < SUB; ++u) {
        const v8 kf = *reinterpret_cast<const v8*>(sb + koff[ks % KO] + (ks / KO) * (32 * KO) + 32 * u * ROWB);
        s[u] = H::mfma(kf, qf[ks], s[u]);
      }
    // Masked tiles: past the end, or on the diagonal.
    if (k0 + BN > hi || (a.causal && k0 + BN - 1 > wrow)) {
      const int r = min(wrow + col, hi - 1);
      const int left = (a.causal ? r + 1 : hi) - k0 - 4 * h;
#pragma unroll
      for (int u = 0; u < SUB; ++u)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (32 * u + 8 * (e / 4) + e % 4 >= left) s[u][e] = -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int u = 0; u < SUB; ++u)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, s[u][e]);
    top = fmaxf(top, rqd::lane_xor_far<32>(top));
    if (__builtin_amdgcn_ballot_w64(top > seen) != 0) {
      const float mn = fmaxf(m, top), ms = scaled(mn, c);
      float al = __builtin_amdgcn_exp2f(scaled(m, c) - ms);
      seen = mn;
      mr = ms - H::kShift;
      if (__builtin_amdgcn_ballot_w64(fabsf(ms) >= kFar) != 0) {
        const bool none = KG > 1 && mn == -INFINITY;  // (with key groups a row may have seen nothing yet)
        const bool far = fabsf(ms) >= kFar && !none;
        al = none ? 1.0f : far ? __builtin_amdgcn_exp2f((m - mn) * c) : al;
        seen = far ? -INFINITY : mn;  // (a far row comes here in every step)
        mr = (none || far ? 0.0f : ms) - H::kShift;
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
          for (int e = 0; e < 16; ++e) s[u][e] -= far ? mn : 0.0f;
      }
      l *= al;
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[ct][e] *= al;
      m = mn;
    }
    v8 pf[SUB][2];
#pragma unroll
    for (int u = 0; u < SUB; ++u)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        uint4 pk;
        uint32_t* w = &pk.x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p0 = __builtin_amdgcn_exp2f(fmaf(s[u][8 * j + 2 * i], c, -mr));
          const float p1 = __builtin_amdgcn_exp2f(fmaf(s[u][8 * j + 2 * i + 1], c, -mr));
          w[i] = H::pack(p0, p1);
          l = H::add2(w[i], l);
        }
        pf[u][j] = __builtin_bit_cast(v8, pk);
      }
    // The second product goes before another wave's softmax (1 x 4096, 16 full heads of 128: 144 -> 139 us;
    // of 256 270 -> 268; 32 / 8 causal ones of 128 150 -> 144; at d = 64, and at 128 with key groups, in step at their
    // barrier, up to 1% slower).
    if constexpr (D == 256 || (KG == 1 && D == 128)) __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int u = 0; u < SUB; ++u)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          union {
            v4s q[2];
            v8 o;
          } vf;
#pragma unroll
          for (int y = 0; y < 2; ++y)
            vf.q[y] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) v4s*)(reinterpret_cast<v4s*>(const_cast<uint8_t*>(
                    sb + voff[ct % VO] + (ct / VO) * (64 * VO) + (32 * u + 16 * j + 8 * y) * ROWB))));
          acc[ct] = H::mfma(vf.o, pf[u][j], acc[ct]);
        }
    if constexpr (D == 256 || (KG == 1 && D == 128)) __builtin_amdgcn_s_setprio(0);
  }
  l += rqd::lane_xor_far<32>(l);
  if constexpr (KG > 1) {
    // The groups' outputs, through LDS in the accumulators' own order.
    __syncthreads();
    float* part = reinterpret_cast<float*>(smem);
    constexpr int REGS = 16 * CT + 2;
    if (grp > 0) {
      float* o = part + ((grp - 1) * RW + wave) * 64 * REGS + lane;
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[64 * (16 * ct + e)] = acc[ct][e];
      o[64 * 16 * CT] = m;
      o[64 * (16 * CT + 1)] = l;
    }
    __syncthreads();
    if (grp > 0) return;
#pragma unroll
    for (int g = 1; g < KG; ++g) {
      const float* o = part + ((g - 1) * RW + wave) * 64 * REGS + lane;
      const float m2 = o[64 * 16 * CT], l2 = o[64 * (16 * CT + 1)];
      const float mn = fmaxf(m, m2);  // (group 0 has the sequence's first key, which every row of a full or causal mask sees)
      const float f1 = __builtin_amdgcn_exp2f(from_to(m, mn, c)), f2 = __builtin_amdgcn_exp2f(from_to(m2, mn, c));
      m = mn;
      l = l * f1 + l2 * f2;
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[ct][e] = acc[ct][e] * f1 + o[64 * (16 * ct + e)] * f2;
    }
  }
  const int r = wrow + col;
  if (r >= hi) return;
  const float inv = 1.0f / l;
  uint16_t* op = a.o + static_cast<int64_t>(r) * a.ldo + head * D + 4 * h;
#pragma unroll
  for (int ct = 0; ct < CT; ++ct)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<uint2*>(op + 32 * ct + 8 * q) = make_uint2(H::pack(acc[ct][4 * q] * inv, acc[ct][4 * q + 1] * inv),
                                                                   H::pack(acc[ct][4 * q + 2] * inv, acc[ct][4 * q + 3] * inv));
}

template <bool BF, int D, int BN, int RW, int KG>
int launch_prompt(PromptArgs a, hipStream_t st) {
  constexpr int BM = 32 * RW;
  const int64_t tiles = (static_cast<int64_t>(a.tokens) + BM - 1) / BM + a.n_seqs;
  const int64_t total = tiles * a.hq;
  if (!launchable(total, 64 * RW * KG)) return OQ_ERR_SHAPE;
  a.tiles = static_cast<int>(tiles);
  hipLaunchKernelGGL((prompt_attn_kernel<BF, D, BN, RW, KG>), dim3(static_cast<unsigned>(total)), dim3(64 * RW * KG), 0, st, a);
  return launch_status();
}
// Shape of a workgroup: row waves of 32 queries, key groups.  Key groups take the
// key tiles in turn and are joined at the end; they pay where there are fewer
// workgroups than the card holds (two a CU for d >= 128) and sequences are long
// enough for each to have several steps, since a row's walk over its keys
// is then what takes the time; with half as many rows the few are spread over twice as many CUs.
// More of either costs loads and LDS reads of the same keys.  wgs: workgroups of 128 rows, len: mean
// length.  Us of (row waves, key groups) (4, 1) / (4, 2) / (2, 2), at d = 64 / (2, 4):
//   d = 128, full, 8 heads on 1: 1 x 200 (wgs 16) 11.2 / 11.4 / 9.6; 4 x 300 (104) 13.0 / 13.1 / 11.8; 1 x 2000 (128) 52 / 40 / 39;
//     1 x 4096 (264) 104 / 83 / 144; 16 heads, 1 x 4096 (528) 151 / 162 / 289;
//     causal, 16 heads: 4 x 300 (208) 12.1 / 12.2 / 16.2; 1 x 2000 (256) 52 / 41 / 46; 1 x 4096 (528) 108 / 90 / 154; 4 x 1000
//     (560) 34 / 44 / 57; 3 x 2500 (976) 116 / 116 / 190;
//   d = 256, causal: 8 heads, 1 x 200 (16) 16.4 / 17.2 / 15.1; 1 x 2000 (128) 104 / 77 / 80; 1 x 4096 (264) 205 / 145 / 173; 4 x
//     2000, ragged (344) 105 / 79 / 117; 16 heads, 4 x 1000 (560) 69 / 82 / 112;
//   d = 64 (a CU holds four, or two of two groups), causal: 1 x 200 (16) 7.7 / 7.4 / 6.5 / 7.0; 1 x 816 (56) 16.1 / 13.3 / 11.4 / 10.7;
//     1 x 2000 (256) 34 / 26 / 22 / 27; 1 x 4096 (528) 76 / 58 / 55 / 71; 16 heads, 4 x 1000 (560) 25 / 20 / 26 / 34; 32 heads, 1 x
//     4096 (1056) 92 / 92 / 106 / 136; full, 4 x 1000 (560) 31 / 28 / 33 / 48, 16 heads, 16 x 300 (848) 17.4 / 20.1 / 23.6 / 36.1.
// Over 272 shapes the rule is within 1% of the fastest in the mean.
template <bool BF>
int launch_prompt_any(const PromptArgs& a, int d, hipStream_t st) {
  const int64_t wgs = (static_cast<int64_t>(a.tokens) / 128 + a.n_seqs) * a.hq, len = a.tokens / a.n_seqs;
  if (d == 64) {
    if (wgs <= 144 && len >= 384) return launch_prompt<BF, 64, 64, 2, 4>(a, st);
    if ((wgs <= 144 && len >= 128) || (wgs <= (a.causal ? 448 : 300) && len >= 384)) return launch_prompt<BF, 64, 64, 2, 2>(a, st);
    const bool two = wgs <= (a.causal ? 720 : 576) && len >= 512;
    return two ? launch_prompt<BF, 64, 64, 4, 2>(a, st) : launch_prompt<BF, 64, 64, 4, 1>(a, st);
  }
  const bool few = wgs <= 128 && len >= 160;
  const bool two = (wgs <= 300 && len >= 256) || (a.causal && wgs <= 544 && len >= 1200);
  if (d == 128)
    return few   ? launch_prompt<BF, 128, 64, 2, 2>(a, st)
           : two ? launch_prompt<BF, 128, 64, 4, 2>(a, st)
                 : launch_prompt<BF, 128, 64, 4, 1>(a, st);
  return few   ? launch_prompt<BF, 256, 32, 2, 2>(a, st)
         : two ? launch_prompt<BF, 256, 32, 4, 2>(a, st)
               : launch_prompt<BF, 256, 32, 4, 1>(a, st);
}

}  // namespace
}  // namespace oq

extern "C" int oq_attention_prompt(const void* Q, const void* K, const void* V, int64_t tokens, int64_t ldq, int64_t ldk,
                                   int64_t ldv, int32_t dtype, const int32_t* cu_seqlens, int32_t n_seqs, int32_t n_heads,
                                   int32_t n_kv_heads, int32_t head_dim, int32_t causal, float scale, void* O, int64_t ldo,
                                   void* stream) {
  if (head_dim != 64 && head_dim != 128 && head_dim != 256) return OQ_ERR_SHAPE;
  if (tokens < 0 || tokens > (1 << 30) || n_seqs < 0 || n_seqs > (1 << 24) || n_heads < 1 || n_heads > 65535 ||
      n_kv_heads < 1 || n_heads % n_kv_heads != 0)
    return OQ_ERR_SHAPE;
  const int64_t wq = static_cast<int64_t>(n_heads) * head_dim, wk = static_cast<int64_t>(n_kv_heads) * head_dim;
  // (A tile's row offsets are 32-bit.)
  if (ldq < wq || ldo < wq || ldk < wk || ldv < wk || ldk > (1 << 24) || ldv > (1 << 24)) return OQ_ERR_SHAPE;
  if (dtype != OQ_OUT_F16 && dtype != OQ_OUT_BF16) return OQ_ERR_ARG;
  if (causal != 0 && causal != 1) return OQ_ERR_ARG;
  if (!(scale > 0.0f) || !std::isfinite(scale * 1.4426950408889634f)) return OQ_ERR_ARG;
  if (ldq % 8 != 0 || ldk % 8 != 0 || ldv % 8 != 0 || ldo % 8 != 0) return OQ_ERR_ALIGN;
  if (tokens == 0 || n_seqs == 0) return OQ_OK;
  if (!Q || !K || !V || !O || !cu_seqlens) return OQ_ERR_NULL;
  if (!oq::aligned(Q, 16) || !oq::aligned(K, 16) || !oq::aligned(V, 16) || !oq::aligned(O, 16) || !oq::aligned(cu_seqlens, 4))
    return OQ_ERR_ALIGN;
  int st = oq::device_check();
  if (st != OQ_OK) return st;
  oq::PromptArgs a{static_cast<const uint16_t*>(Q), static_cast<const uint16_t*>(K), static_cast<const uint16_t*>(V),
                   static_cast<uint16_t*>(O), cu_seqlens, ldq, ldk, ldv, ldo, static_cast<int>(tokens), n_seqs, n_heads,
                   n_heads / n_kv_heads, 0, scale * 1.4426950408889634f, causal == 1};
  hipStream_t s = static_cast<hipStream_t>(stream);
  return dtype == OQ_OUT_BF16 ? oq::launch_prompt_any<true>(a, head_dim, s) : oq::launch_prompt_any<false>(a, head_dim, s);
}
