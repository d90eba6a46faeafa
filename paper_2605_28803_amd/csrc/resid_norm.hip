// The residual stream between two blocks: the norm behind a block, its gate and
// residual scale, and the norm before the next block, in one pass over a row.
//
//   y' = post(y)                              (or y)
//   r' = alpha r + gate[g] y'
//   h  = pre(r') (1 + scale[g]) + shift[g]    (16 bits, or microscaled 4-bit codes)
//
// A row's values stay in registers between its sums, so r and y are read once
// and r' and h written once.  A thread holds P pieces of 8 channels of a row, W
// waves a row (W = 1: four rows a workgroup, and no barrier).  (A workgroup that
// takes row after row with the next one's loads under way holds more registers
// and was 2% to 12% slower up to 4096 channels, even beyond; pieces of an fp32 residual
// two fours apart, so that its accesses are of whole kilobytes, cost 4% to 17%.)
// Sums of a thread's values are float (double where codes are written), sums
// over threads double.  LayerNorm sums (x - mean)^2 with the mean known: a
// second exchange, but no cancellation.
// Where codes are written, everything is double: the codes are then those of the
// formula in 64 bits, not those of a nearby float.
// Bound by memory: 16384 x 4096 with both norms, fp32 residual into codes 705 MB in
// 144-163 us, 4.3-4.9 TB/s (a copy reaches 5.1); into 16 bits 805 MB in 140 us; bf16 residual
// into 16 bits 537 MB in 96-101 us, into codes, where the double operations show, 437 MB in 114-119 us.
#include <algorithm>

#include "mx4_device.h"

namespace oq {
namespace {

struct NormOf {
  const uint16_t* gain;
  const uint16_t* bias;
  int kind;
  float eps, offset;
};
struct NormArgs {
  const void* R;
  const uint16_t* Y;
  NormOf post, pre;
  const uint16_t *gate, *scale, *shift;
  const int32_t* mod_row;
  void* Ro;
  uint16_t* H;
  uint8_t *Hq, *steps;
  int64_t ldr, ldy, ldm, ldro, ldh, lds;
  int64_t M;
  int D, n_mod;
  float alpha;
  double inv_d;
};

template <int CTRL>
__device__ __forceinline__ double dpp64(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  return __builtin_bit_cast(double, static_cast<uint64_t>(dpp<CTRL>(static_cast<uint32_t>(b >> 32))) << 32 |
                                        dpp<CTRL>(static_cast<uint32_t>(b)));
}
__device__ __forceinline__ double wave_sum(double x) {
  x += dpp64<kQuadXor1>(x);
  x += dpp64<kQuadXor2>(x);
  x += dpp64<0x141>(x);  // row_half_mirror: the other quad of eight lanes
  x += dpp64<0x140>(x);  // row_mirror: the other eight of sixteen
  // (A swap of a value with itself leaves either half's sum in all lanes of both.)
  auto halves = [](double v, auto swap) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const auto lo = swap(static_cast<uint32_t>(b)), hi = swap(static_cast<uint32_t>(b >> 32));
    return __builtin_bit_cast(double, static_cast<uint64_t>(hi[0]) << 32 | lo[0]) +
           __builtin_bit_cast(double, static_cast<uint64_t>(hi[1]) << 32 | lo[1]);
  };
  x = halves(x, [](uint32_t u) { return __builtin_amdgcn_permlane16_swap(u, u, false, false); });
  return halves(x, [](uint32_t u) { return __builtin_amdgcn_permlane32_swap(u, u, false, false); });
}

// 1 / sqrt(x) for x > 0: the hardware's estimate (29 bits) and two steps of
// Newton's, within a few units of 2^-53.  (The library's root and division are a
// chain several times as long, twice a row.)
__device__ __forceinline__ double inverse_root(double x) {
  const double r0 = __builtin_amdgcn_rsq(x);
  double r = r0 * fma(-0.5 * x * r0, r0, 1.5);
  r = r * fma(-0.5 * x * r, r, 1.5);
  return x < __builtin_huge_val() ? r : r0;  // (infinite: 0; a NaN stays one)
}

// Sum over a row's threads.
template <int W>
__device__ __forceinline__ double row_sum(double x, double* red) {
  x = wave_sum(x);
  if constexpr (W > 1) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.0;
#pragma unroll
    for (int w = 0; w < W; ++w) x += red[w];
  }
  return x;
}

template <bool BF, bool RF32, bool MX4, int W, int P>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void residual_norm_kernel(NormArgs a) {
  using Acc = std::conditional_t<MX4, double, float>;
  constexpr int T = 64 * W;  // threads of a row
  __shared__ double red[4][W];  // (an exchange each)
  const int tid = W == 1 ? threadIdx.x & 63 : threadIdx.x;
  const bool all = a.D == 8 * T * P;
  // First channel of piece c, and whether the row has it.
  auto at = [&](int c) { return 8 * (T * c + tid); };
  auto on = [&](int c) { return all || at(c) < a.D; };
  // (Loads past the row's end read its first piece: with none of them conditional they leave together.)
  auto from = [&](int c) { return on(c) ? at(c) : 0; };
  auto get = [&](const uint16_t* p, int c) { return *reinterpret_cast<const uint4*>(p + from(c)); };

  const int64_t row = W == 1 ? static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6) : blockIdx.x;
  if (row >= a.M) return;
  int64_t g = 0;
  if (a.mod_row && (a.gate || a.scale || a.shift)) {
    const int k = a.mod_row[row];
    if (k < 0 || k >= a.n_mod) return;  // (the whole row is left)
    g = k * a.ldm;
  }
  Acc v[P][8];
  uint4 y[P], r[P][RF32 ? 2 : 1];
#pragma unroll
  for (int c = 0; c < P; ++c) {
    // (No choice between a row and a constant by reference: its loads would be flat ones.)
    y[c] = a.Y ? get(a.Y + row * a.ldy, c) : make_uint4(0, 0, 0, 0);
    if constexpr (RF32) {
      const uint4* s = reinterpret_cast<const uint4*>(static_cast<const float*>(a.R) + row * a.ldr + from(c));
#pragma unroll
      for (int h = 0; h < 2; ++h) r[c][h] = a.R ? uint4(s[h]) : make_uint4(0, 0, 0, 0);
    } else {
      r[c][0] = a.R ? get(static_cast<const uint16_t*>(a.R) + row * a.ldr, c) : make_uint4(0, 0, 0, 0);
    }
  }
  // (One piece a thread into 16 bits: the parameters come with the row, 1024 x 1536 with a modulation 9.5 us, so 8.9,
  // 16384 x 4096 143.6, so 139.4.  Beside doubles they hold too many registers: 151, so 159.)
  constexpr bool EARLY = P == 1 && !MX4;
  auto early = [&](const uint16_t* p) { return EARLY && p ? get(p, 0) : make_uint4(0, 0, 0, 0); };
  const uint4 post_gain = early(a.post.gain), post_bias = early(a.post.bias), gate = early(a.gate ? a.gate + g : nullptr);
  const uint4 pre_gain = early(a.pre.gain), pre_bias = early(a.pre.bias);
  const uint4 scale = early(a.scale ? a.scale + g : nullptr), shift = early(a.shift ? a.shift + g : nullptr);
#pragma unroll
  for (int c = 0; c < P; ++c)
#pragma unroll
    for (int e = 0; e < 8; ++e) v[c][e] = on(c) ? half8<BF>(y[c], e) : 0.0f;
  // Mean (LayerNorm) and 1 / sqrt(mean square + eps) of the row's v (0 past its end).
  auto statistics = [&](const NormOf& k, int slot, Acc* mean, Acc* rstd) {
    Acc s = 0;
    *mean = 0;
    if (k.kind == OQ_NORM_LAYER) {
#pragma unroll
      for (int c = 0; c < P; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) s += v[c][e];
      const Acc m = static_cast<Acc>(row_sum<W>(s, red[slot]) * a.inv_d);
      s = 0;
#pragma unroll
      for (int c = 0; c < P; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const Acc d = on(c) ? v[c][e] - m : static_cast<Acc>(0);
          s = fma(d, d, s);
        }
      *mean = m;
    } else {
#pragma unroll
      for (int c = 0; c < P; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fma(v[c][e], v[c][e], s);
    }
    *rstd = static_cast<Acc>(inverse_root(row_sum<W>(s, red[slot + 1]) * a.inv_d + static_cast<double>(k.eps)));
  };
  // x = piece c's values normed (past the row's end: anything).
  auto apply = [&](const NormOf& k, const uint4& gain, const uint4& bias, auto (&x)[8], int c, auto mean, auto rstd) {
    using F = decltype(rstd);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (k.kind == OQ_NORM_LAYER ? x[e] - mean : x[e]) * rstd;
    if (k.gain) {
      const uint4 q = EARLY ? uint4(gain) : get(k.gain, c);
      if (k.offset != 0.0f) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= static_cast<F>(k.offset) + static_cast<F>(half8<BF>(q, e));
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= static_cast<F>(half8<BF>(q, e));
      }
    }
    if (k.bias) {
      const uint4 q = EARLY ? uint4(bias) : get(k.bias, c);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] += static_cast<F>(half8<BF>(q, e));
    }
  };
  auto modulate = [&](auto (&x)[8], int c) {
    using F = std::remove_reference_t<decltype(x[0])>;
    if (a.scale) {
      const uint4 q = EARLY ? uint4(scale) : get(a.scale + g, c);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] *= static_cast<F>(1) + static_cast<F>(half8<BF>(q, e));
    }
    if (a.shift) {
      const uint4 q = EARLY ? uint4(shift) : get(a.shift + g, c);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] += static_cast<F>(half8<BF>(q, e));
    }
  };
  if (a.post.kind != OQ_NORM_NONE) {
    Acc mean, rstd;
    statistics(a.post, 0, &mean, &rstd);
#pragma unroll
    for (int c = 0; c < P; ++c) apply(a.post, post_gain, post_bias, v[c], c, mean, rstd);
  }
#pragma unroll
  for (int c = 0; c < P; ++c) {
    if (a.gate) {
      const uint4 q = EARLY ? uint4(gate) : get(a.gate + g, c);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[c][e] *= static_cast<Acc>(half8<BF>(q, e));
    }
    float o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      Acc x;
      if constexpr (RF32) {
        const uint4 w = r[c][e >> 2];
        x = __uint_as_float((e & 3) == 0 ? w.x : (e & 3) == 1 ? w.y : (e & 3) == 2 ? w.z : w.w);
      } else {
        x = half8<BF>(r[c][0], e);
      }
      v[c][e] = fma(static_cast<Acc>(a.alpha), x, v[c][e]);
      o[e] = static_cast<float>(v[c][e]);
    }
    if (!all) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[c][e] = on(c) ? v[c][e] : static_cast<Acc>(0);
    }
    if (a.Ro && on(c)) {
      if constexpr (RF32) {
        float4* d = reinterpret_cast<float4*>(static_cast<float*>(a.Ro) + row * a.ldro + at(c));
        d[0] = make_float4(o[0], o[1], o[2], o[3]);
        d[1] = make_float4(o[4], o[5], o[6], o[7]);
      } else {
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.Ro) + row * a.ldro + at(c)) = pack_half8<BF>(o);
      }
    }
  }
  if (a.pre.kind != OQ_NORM_NONE) {
    Acc mean, rstd;
    statistics(a.pre, 2, &mean, &rstd);
#pragma unroll
    for (int c = 0; c < P; ++c) {
      apply(a.pre, pre_gain, pre_bias, v[c], c, mean, rstd);
      modulate(v[c], c);
      if constexpr (MX4) {
        uint32_t byte;
        const uint32_t code = quad_codes(v[c], &byte);
        if (on(c)) {  // (whole quads)
          const int p = at(c) / 8;
          reinterpret_cast<uint32_t*>(a.Hq + row * (a.D / 2))[p] = code;
          if ((p & 3) == 0) a.steps[row * a.lds + (p >> 2)] = static_cast<uint8_t>(byte);
        }
      } else if (on(c)) {
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = v[c][e];
        *reinterpret_cast<uint4*>(a.H + row * a.ldh + at(c)) = pack_half8<BF>(o);
      }
    }
  }
}

template <bool BF, bool RF32, bool MX4, int W, int P>
int launch_norm(const NormArgs& a, hipStream_t stream) {
  constexpr int threads = W == 1 ? 256 : 64 * W;
  constexpr int64_t slab = int64_t{1} << 21;  // rows of a launch (2^31 threads at most)
  for (int64_t r0 = 0; r0 < a.M; r0 += slab) {
    NormArgs b = a;
    b.M = std::min(slab, a.M - r0);
    if (a.R) b.R = static_cast<const uint8_t*>(a.R) + r0 * a.ldr * (RF32 ? 4 : 2);
    if (a.Y) b.Y = a.Y + r0 * a.ldy;
    if (a.mod_row) b.mod_row = a.mod_row + r0;
    if (a.Ro) b.Ro = static_cast<uint8_t*>(a.Ro) + r0 * a.ldro * (RF32 ? 4 : 2);
    if (a.H) b.H = a.H + r0 * a.ldh;
    if (a.Hq) {
      b.Hq = a.Hq + r0 * (a.D / 2);
      b.steps = a.steps + r0 * a.lds;
    }
    const int64_t blocks = W == 1 ? (b.M + 3) / 4 : b.M;
    hipLaunchKernelGGL((residual_norm_kernel<BF, RF32, MX4, W, P>), dim3(static_cast<unsigned>(blocks)), dim3(threads), 0, stream, b);
    const int st = launch_status();
    if (st != OQ_OK) return st;
  }
  return OQ_OK;
}

// Waves of a row and pieces of a thread, us at 16384 rows (4096 of 8192 channels and more) in bf16 with both RMS norms: W, P
// of the one taken / of another.
//                      fp32 residual                         bf16 residual
//   codes     1024     2, 1 38.3 / 1, 2 42.6                 2, 1 32.1 / 1, 2 33.5
//             2048     4, 1 73.1 / 2, 2 82.0                 2, 2 58.4 / 4, 1 61.3
//             4096     8, 1 144 / 4, 2 155                   4, 2 114 / 8, 1 125
//             8192     8, 2 86.8 / 16, 1 87.4                8, 2 60.5 / 16, 1 69.7
//            16384     16, 2 184 / 8, 4 199                  8, 4 126 / 16, 2 142
//   16 bits   1024     2, 1 35.6 / 1, 2 37.2                 2, 1 24.9 / 1, 2 24.1
//             2048     4, 1 74.4 / 2, 2 77.5                 2, 2 45.6 / 4, 1 47.3
//             4096     8, 1 142 / 4, 2 143                   8, 1 95.9 / 4, 2 97.3
//             8192     8, 2 78.8 / 16, 1 78.1                8, 2 48.1 / 16, 1 50.2
//            16384     16, 2 152 / 8, 4 159                  16, 2 102 / 8, 4 103
// Few rows take one piece a thread: codes of 64 x 4096 8, 1 4.6 / 4, 2 5.5; of 1024 x 4096 12.2 / 12.7.
template <bool BF, bool RF32, bool MX4>
int launch_norm(const NormArgs& a, hipStream_t stream) {
  const int n = a.D / 8;
  const bool few = a.M <= 1024;
  if (n <= 64) return launch_norm<BF, RF32, MX4, 1, 1>(a, stream);
  if (n <= 128) return launch_norm<BF, RF32, MX4, 2, 1>(a, stream);
  if constexpr (!RF32) {
    if (!few && n <= 256) return launch_norm<BF, RF32, MX4, 2, 2>(a, stream);
  }
  if (n <= 256) return launch_norm<BF, RF32, MX4, 4, 1>(a, stream);
  if constexpr (MX4 && !RF32) {
    if (!few && n <= 512) return launch_norm<BF, RF32, MX4, 4, 2>(a, stream);
    if (!few && n > 1024) return launch_norm<BF, RF32, MX4, 8, 4>(a, stream);
  }
  if (n <= 512) return launch_norm<BF, RF32, MX4, 8, 1>(a, stream);
  if (n <= 1024) return few ? launch_norm<BF, RF32, MX4, 16, 1>(a, stream) : launch_norm<BF, RF32, MX4, 8, 2>(a, stream);
  return launch_norm<BF, RF32, MX4, 16, 2>(a, stream);
}

bool norm_of(const oq_norm* k, NormOf* out, int* st) {
  *out = NormOf{nullptr, nullptr, OQ_NORM_NONE, 0.0f, 0.0f};
  if (!k || k->kind == OQ_NORM_NONE) return true;
  if (k->kind != OQ_NORM_RMS && k->kind != OQ_NORM_LAYER) *st = OQ_ERR_ARG;
  else if (!(k->eps > 0.0f) || !(k->eps <= 1.0f)) *st = OQ_ERR_ARG;
  else if (!(k->gain_offset == k->gain_offset) || k->gain_offset - k->gain_offset != 0.0f) *st = OQ_ERR_ARG;
  else if (!aligned(k->gain, 16) || !aligned(k->bias, 16)) *st = OQ_ERR_ALIGN;
  else {
    *out = NormOf{static_cast<const uint16_t*>(k->gain), static_cast<const uint16_t*>(k->bias), k->kind, k->eps, k->gain_offset};
    return true;
  }
  return false;
}

}  // namespace
}  // namespace oq

extern "C" int oq_residual_norm(const void* R, int64_t ldr, int32_t r_dtype, const void* Y, int64_t ldy, int32_t dtype,
                                int64_t M, int64_t D, const oq_norm* post, const oq_norm* pre, float alpha,
                                const void* gate, const void* scale, const void* shift, int64_t ld_mod, int64_t n_mod,
                                const int32_t* mod_row, void* R_out, int64_t ldro, void* H, int64_t ldh, uint8_t* Hq,
                                uint8_t* steps, void* stream) {
  using namespace oq;
  const bool mx4 = Hq != nullptr || steps != nullptr;
  const bool mods = gate || scale || shift;
  if (M < 0 || D < 8 || D % 8 != 0 || D > OQ_NORM_MAX_D || (mx4 && D % 32 != 0)) return OQ_ERR_SHAPE;
  if (dtype != OQ_OUT_F16 && dtype != OQ_OUT_BF16) return OQ_ERR_ARG;
  if (r_dtype != dtype && r_dtype != OQ_OUT_F32) return OQ_ERR_ARG;
  if (!(alpha - alpha == 0.0f)) return OQ_ERR_ARG;
  NormArgs a{};
  int st = OQ_OK;
  if (!norm_of(post, &a.post, &st) || !norm_of(pre, &a.pre, &st)) return st;
  const bool out = a.pre.kind != OQ_NORM_NONE;
  if ((H && mx4) || (!out && (H || mx4 || scale || shift))) return OQ_ERR_ARG;
  if ((R && ldr < D) || (Y && ldy < D) || (R_out && ldro < D) || (H && ldh < D)) return OQ_ERR_SHAPE;
  if (mods && (ld_mod < D || n_mod < 1 || n_mod > INT32_MAX)) return OQ_ERR_SHAPE;
  if ((R && ldr % 8 != 0) || (Y && ldy % 8 != 0) || (R_out && ldro % 8 != 0) || (H && ldh % 8 != 0) || (mods && ld_mod % 8 != 0))
    return OQ_ERR_ALIGN;
  if (M == 0) return OQ_OK;
  if ((!R && !Y) || (mx4 && (!Hq || !steps)) || (out && !H && !mx4) || (!out && !R_out)) return OQ_ERR_NULL;
  for (const void* p : {R, Y, gate, scale, shift, static_cast<const void*>(R_out), static_cast<const void*>(H),
                        static_cast<const void*>(Hq), static_cast<const void*>(steps)})
    if (!aligned(p, 16)) return OQ_ERR_ALIGN;
  if (!aligned(mod_row, 4)) return OQ_ERR_ALIGN;
  if ((st = device_check()) != OQ_OK) return st;
  a.R = R;
  a.Y = static_cast<const uint16_t*>(Y);
  a.gate = static_cast<const uint16_t*>(gate);
  a.scale = static_cast<const uint16_t*>(scale);
  a.shift = static_cast<const uint16_t*>(shift);
  a.mod_row = mod_row;
  a.Ro = R_out;
  a.H = static_cast<uint16_t*>(H);
  a.Hq = Hq;
  a.steps = steps;
  a.ldr = ldr;
  a.ldy = ldy;
  a.ldm = ld_mod;
  a.ldro = ldro;
  a.ldh = ldh;
  a.lds = mx4_step_bytes(D);
  a.M = M;
  a.D = static_cast<int>(D);
  a.n_mod = static_cast<int>(n_mod);
  a.alpha = alpha;
  a.inv_d = 1.0 / static_cast<double>(D);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const bool f32 = r_dtype == OQ_OUT_F32;
  if (dtype == OQ_OUT_BF16) {
    if (f32) return mx4 ? launch_norm<true, true, true>(a, s) : launch_norm<true, true, false>(a, s);
    return mx4 ? launch_norm<true, false, true>(a, s) : launch_norm<true, false, false>(a, s);
  }
  if (f32) return mx4 ? launch_norm<false, true, true>(a, s) : launch_norm<false, true, false>(a, s);
  return mx4 ? launch_norm<false, false, true>(a, s) : launch_norm<false, false, false>(a, s);
}
