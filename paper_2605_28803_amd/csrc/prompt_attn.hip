// Softmax self-attention within packed sequences (prompts), grouped heads,
// causal or full.
//
// A workgroup of 4 waves takes 128 QT query tokens of one sequence and head
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

template <bool BF>
struct Half;
template <>
struct Half<false> {
  typedef v8h v8;
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

template <bool BF, int D, int QT, int BN>
__global__ __launch_bounds__(256, QT == 1 ? 2 : 1) void prompt_attn_kernel(PromptArgs a) {
  typedef Half<BF> H;
  typedef typename H::v8 v8;
  constexpr int BM = 128 * QT, PCS = D / 8, ROWB = 2 * D;
  constexpr int KB = BN * ROWB, STAGE = 2 * KB;
  constexpr int LK = KB / 1024 / 4;  // 1 KB loads of K (and of V) per wave and tile
  constexpr int SUB = BN / 32, CT = D / 32, KS = D / 16;
  __shared__ __attribute__((aligned(16))) uint8_t smem[2 * STAGE];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, h = lane >> 5;
  // Consecutive ids go to different XCDs (id % 8): XCD x takes the x-th
  // contiguous part of (head, tile), so that heads which share K and V share its L2.
  const int total = a.hq * a.tiles;
  const int id = blockIdx.x, per = total >> 3, rem = total & 7, x = id & 7;
  const int lin = x * per + min(x, rem) + (id >> 3);
  const int head = lin / a.tiles;
  int tile = lin % a.tiles;
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
  const int wrow = r0 + wave * 32 * QT;  // the wave's first row

  const uint16_t* kbase = a.k + (head / a.rep) * D + static_cast<int64_t>(lo) * a.ldk;
  const uint16_t* vbase = a.v + (head / a.rep) * D + static_cast<int64_t>(lo) * a.ldv;
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t*)smem));
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
  issue(lo, 0);

  v8 qf[QT][KS];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int r = min(wrow + 32 * t + col, hi - 1);
    const uint16_t* qp = a.q + static_cast<int64_t>(r) * a.ldq + head * D + 8 * h;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[t][ks] = *reinterpret_cast<const v8*>(qp + 16 * ks);
  }
  v16f acc[QT][CT];
  float m[QT], l[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    m[t] = -INFINITY;
    l[t] = 0.0f;
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[t][c][e] = 0.0f;
  }
  // Addresses of this lane's reads.
  const int vi = lane & 15, vg = (lane >> 4) & 1;
  const float c = a.scale_log2e;
  int buf = 0;
  for (int k0 = lo; k0 < kend; k0 += BN, buf ^= 1) {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (k0 + BN < kend) issue(k0 + BN, buf ^ 1);
    const int wlast = min(wrow + 32 * QT, hi) - 1;
    if (a.causal && k0 > wlast) continue;  // (this wave's rows see none of the tile)
    const uint8_t* sk = smem + buf * STAGE;
    const uint8_t* sv = sk + KB;
    v16f s[QT][SUB];
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int u = 0; u < SUB; ++u)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[t][u][e] = 0.0f;
#pragma unroll
    for (int u = 0; u < SUB; ++u)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const int row = 32 * u + col;
        const v8 kf = *reinterpret_cast<const v8*>(sk + row * ROWB + (((2 * ks + h) ^ swzk(row)) * 16));
#pragma unroll
        for (int t = 0; t < QT; ++t) s[t][u] = H::mfma(kf, qf[t][ks], s[t][u]);
      }
    // Masked tiles: past the end, or on the diagonal.
    if (k0 + BN > hi || (a.causal && k0 + BN - 1 > wrow)) {
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        const int r = min(wrow + 32 * t + col, hi - 1);
        const int end = a.causal ? r + 1 : hi;
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (k0 + 32 * u + 8 * (e / 4) + 4 * h + e % 4 >= end) s[t][u][e] = -INFINITY;
      }
    }
    v8 pf[QT][SUB][2];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      float top = s[t][0][0];
#pragma unroll
      for (int u = 0; u < SUB; ++u)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, s[t][u][e]);
      top = fmaxf(top, rqd::lane_xor_far<32>(top));
      const float mn = fmaxf(m[t], top * c);
      if (__builtin_amdgcn_ballot_w64(mn > m[t]) != 0) {
        const float al = __builtin_amdgcn_exp2f(m[t] - mn);
        l[t] *= al;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[t][ct][e] *= al;
        m[t] = mn;
      }
#pragma unroll
      for (int u = 0; u < SUB; ++u)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          uint4 pk;
          uint32_t* w = &pk.x;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float p0 = __builtin_amdgcn_exp2f(fmaf(s[t][u][8 * j + 2 * i], c, -mn));
            const float p1 = __builtin_amdgcn_exp2f(fmaf(s[t][u][8 * j + 2 * i + 1], c, -mn));
            w[i] = H::pack(p0, p1);
            l[t] = H::add2(w[i], l[t]);
          }
          pf[t][u][j] = __builtin_bit_cast(v8, pk);
        }
    }
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
          for (int y = 0; y < 2; ++y) {
            const int row = 32 * u + 16 * j + 8 * y + 4 * h + (vi >> 2);
            const int piece = 4 * ct + 2 * vg + ((vi & 3) >> 1);
            const uint8_t* p = sv + row * ROWB + (piece ^ swzv(row)) * 16 + 8 * (vi & 1);
            vf.q[y] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) v4s*)(reinterpret_cast<v4s*>(const_cast<uint8_t*>(p))));
          }
#pragma unroll
          for (int t = 0; t < QT; ++t) acc[t][ct] = H::mfma(vf.o, pf[t][u][j], acc[t][ct]);
        }
  }
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int r = wrow + 32 * t + col;
    const float sum = l[t] + rqd::lane_xor_far<32>(l[t]);
    const float inv = 1.0f / sum;
    if (r >= hi) continue;
    uint16_t* op = a.o + static_cast<int64_t>(r) * a.ldo + head * D + 4 * h;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<uint2*>(op + 32 * ct + 8 * q) =
            make_uint2(H::pack(acc[t][ct][4 * q] * inv, acc[t][ct][4 * q + 1] * inv),
                       H::pack(acc[t][ct][4 * q + 2] * inv, acc[t][ct][4 * q + 3] * inv));
  }
}

template <bool BF, int D, int QT, int BN>
int launch_prompt(PromptArgs a, hipStream_t st) {
  constexpr int BM = 128 * QT;
  const int64_t tiles = (static_cast<int64_t>(a.tokens) + BM - 1) / BM + a.n_seqs;
  const int64_t total = tiles * a.hq;
  if (total > INT32_MAX) return OQ_ERR_SHAPE;
  a.tiles = static_cast<int>(tiles);
  hipLaunchKernelGGL((prompt_attn_kernel<BF, D, QT, BN>), dim3(static_cast<unsigned>(total)), dim3(256), 0, st, a);
  return launch_status();
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
  if (!(scale > 0.0f) || !std::isfinite(scale)) return OQ_ERR_ARG;
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
  const bool bf = dtype == OQ_OUT_BF16;
  switch (head_dim) {
    case 64: return bf ? oq::launch_prompt<true, 64, 1, 64>(a, s) : oq::launch_prompt<false, 64, 1, 64>(a, s);
    case 128: return bf ? oq::launch_prompt<true, 128, 1, 64>(a, s) : oq::launch_prompt<false, 128, 1, 64>(a, s);
    default: return bf ? oq::launch_prompt<true, 256, 1, 32>(a, s) : oq::launch_prompt<false, 256, 1, 32>(a, s);
  }
}
