// The residual stream between two blocks: the norm behind a block, its gate and
// residual scale, and the norm before the next block, in one pass over a row.
//
//   y' = post(y)                              (or y)
//   r' = alpha r + gate[g] y'
//   h  = pre(r') (1 + scale[g]) + shift[g]    (16 bits, or microscaled 4-bit codes)
//
// A row's values stay in registers between its sums, so r and y are read once
// and r' and h written once.  A thread holds P pieces of 8 channels of a row, W
// waves a row (W = 1: a wave a row, four rows a workgroup, and no barrier).
// Sums of a thread's values are float (double where codes are written), sums
// over threads double.  LayerNorm sums (x - mean)^2 with the mean known: a
// second exchange, but no cancellation.
// Where codes are written, everything is double: the codes are then those of the
// formula in 64 bits, not those of a nearby float (a double operation costs what
// a float one does here; the registers bound P).
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
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// Sum over a row's threads; `slot` names an exchange of the row (0 .. 3).
template <int W>
__device__ __forceinline__ double row_sum(double x, double (*red)[W], int slot) {
  x = wave_sum(x);
  if constexpr (W > 1) {
    if ((threadIdx.x & 63) == 0) red[slot][threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.0;
#pragma unroll
    for (int w = 0; w < W; ++w) x += red[slot][w];
  }
  return x;
}

template <bool BF, bool RF32, bool MX4, int W, int P>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void residual_norm_kernel(NormArgs a) {
  using Acc = std::conditional_t<MX4, double, float>;
  __shared__ double red[4][W];
  const int tid = W == 1 ? threadIdx.x & 63 : threadIdx.x;
  const int64_t row = W == 1 ? static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6) : blockIdx.x;
  if (row >= a.M) return;
  const bool mods = a.gate || a.scale || a.shift;
  int64_t g = 0;
  if (mods && a.mod_row) {
    const int k = a.mod_row[row];
    if (k < 0 || k >= a.n_mod) return;  // (the whole row)
    g = k;
  }
  g *= a.ldm;
  const int n = a.D >> 3;

  Acc v[P][8];
  uint4 y[P], r[P][RF32 ? 2 : 1];
  bool on[P];
#pragma unroll
  for (int c = 0; c < P; ++c) {
    const int p = tid + c * 64 * W;
    on[c] = p < n;
    const int q = on[c] ? p : 0;
    y[c] = a.Y ? *reinterpret_cast<const uint4*>(a.Y + row * a.ldy + 8 * q) : make_uint4(0, 0, 0, 0);
    if constexpr (RF32) {
      const uint4* s = reinterpret_cast<const uint4*>(static_cast<const float*>(a.R) + row * a.ldr + 8 * q);
      r[c][0] = a.R ? s[0] : make_uint4(0, 0, 0, 0);
      r[c][1] = a.R ? s[1] : make_uint4(0, 0, 0, 0);
    } else {
      r[c][0] = a.R ? *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.R) + row * a.ldr + 8 * q)
                    : make_uint4(0, 0, 0, 0);
    }
  }
  // Mean (0 for RMS) and 1 / sqrt(mean square + eps) of the row's v.
  auto statistics = [&](const NormOf& k, int slot, Acc* mean, Acc* rstd) {
    Acc m = 0;
    if (k.kind == OQ_NORM_LAYER) {
      Acc s = 0;
#pragma unroll
      for (int c = 0; c < P; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) s += on[c] ? v[c][e] : static_cast<Acc>(0);
      m = static_cast<Acc>(row_sum<W>(s, red, slot) * a.inv_d);
    }
    Acc s = 0;
#pragma unroll
    for (int c = 0; c < P; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const Acc d = on[c] ? v[c][e] - m : static_cast<Acc>(0);
        s = fma(d, d, s);
      }
    *rstd = static_cast<Acc>(1.0 / sqrt(row_sum<W>(s, red, slot + 1) * a.inv_d + static_cast<double>(k.eps)));
    *mean = m;
  };
  // v = norm of v, of piece c.
  auto apply = [&](const NormOf& k, int c, int q, Acc mean, Acc rstd) {
    const uint4 gn = k.gain ? *reinterpret_cast<const uint4*>(k.gain + 8 * q) : make_uint4(0, 0, 0, 0);
    const uint4 bs = k.bias ? *reinterpret_cast<const uint4*>(k.bias + 8 * q) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const Acc gain = k.gain ? static_cast<Acc>(half8<BF>(gn, e)) + static_cast<Acc>(k.offset) : static_cast<Acc>(1);
      v[c][e] = (v[c][e] - mean) * rstd * gain + static_cast<Acc>(half8<BF>(bs, e));
    }
  };

#pragma unroll
  for (int c = 0; c < P; ++c)
#pragma unroll
    for (int e = 0; e < 8; ++e) v[c][e] = half8<BF>(y[c], e);
  if (a.post.kind != OQ_NORM_NONE) {
    Acc mean, rstd;
    statistics(a.post, 0, &mean, &rstd);
#pragma unroll
    for (int c = 0; c < P; ++c) apply(a.post, c, on[c] ? tid + c * 64 * W : 0, mean, rstd);
  }
#pragma unroll
  for (int c = 0; c < P; ++c) {
    const int q = on[c] ? tid + c * 64 * W : 0;
    const uint4 gt = a.gate ? *reinterpret_cast<const uint4*>(a.gate + g + 8 * q) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      Acc old;
      if constexpr (RF32) {
        const uint4 w = r[c][e >> 2];
        old = __uint_as_float((e & 3) == 0 ? w.x : (e & 3) == 1 ? w.y : (e & 3) == 2 ? w.z : w.w);
      } else {
        old = half8<BF>(r[c][0], e);
      }
      if (a.gate) v[c][e] *= static_cast<Acc>(half8<BF>(gt, e));
      v[c][e] = fma(static_cast<Acc>(a.alpha), old, v[c][e]);
    }
    if (a.Ro && on[c]) {
      float o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = static_cast<float>(v[c][e]);
      if constexpr (RF32) {
        float4* d = reinterpret_cast<float4*>(static_cast<float*>(a.Ro) + row * a.ldro + 8 * q);
        d[0] = make_float4(o[0], o[1], o[2], o[3]);
        d[1] = make_float4(o[4], o[5], o[6], o[7]);
      } else {
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.Ro) + row * a.ldro + 8 * q) = pack_half8<BF>(o);
      }
    }
  }
  if (a.pre.kind == OQ_NORM_NONE) return;
  Acc mean, rstd;
  statistics(a.pre, 2, &mean, &rstd);
#pragma unroll
  for (int c = 0; c < P; ++c) {
    const int p = tid + c * 64 * W, q = on[c] ? p : 0;
    apply(a.pre, c, q, mean, rstd);
    const uint4 sc = a.scale ? *reinterpret_cast<const uint4*>(a.scale + g + 8 * q) : make_uint4(0, 0, 0, 0);
    const uint4 sh = a.shift ? *reinterpret_cast<const uint4*>(a.shift + g + 8 * q) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      v[c][e] = v[c][e] * (static_cast<Acc>(1) + static_cast<Acc>(half8<BF>(sc, e))) + static_cast<Acc>(half8<BF>(sh, e));
    if constexpr (MX4) {
      uint32_t byte;
      const uint32_t code = quad_codes(v[c], &byte);
      if (on[c]) {  // (whole quads)
        reinterpret_cast<uint32_t*>(a.Hq + row * (a.D / 2))[p] = code;
        if ((p & 3) == 0) a.steps[row * a.lds + (p >> 2)] = static_cast<uint8_t>(byte);
      }
    } else if (on[c]) {
      float o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = v[c][e];
      *reinterpret_cast<uint4*>(a.H + row * a.ldh + 8 * p) = pack_half8<BF>(o);
    }
  }
}

template <bool BF, bool RF32, bool MX4, int W, int P>
int launch_norm(const NormArgs& a, hipStream_t stream) {
  const int64_t blocks = W == 1 ? (a.M + 3) / 4 : a.M;
  if (!launchable(blocks, W == 1 ? 256 : 64 * W)) return OQ_ERR_SHAPE;
  hipLaunchKernelGGL((residual_norm_kernel<BF, RF32, MX4, W, P>), dim3(static_cast<unsigned>(blocks)), dim3(W == 1 ? 256 : 64 * W),
                     0, stream, a);
  return launch_status();
}

template <bool BF, bool RF32, bool MX4>
int launch_norm(const NormArgs& a, hipStream_t stream) {
  const int n = a.D / 8;
  const bool few = a.M <= 512;
  if (n <= 64) return launch_norm<BF, RF32, MX4, 1, 1>(a, stream);
  if (few) {
    if (n <= 256) return launch_norm<BF, RF32, MX4, 4, 1>(a, stream);
    if (n <= 1024) return launch_norm<BF, RF32, MX4, 16, 1>(a, stream);
    return launch_norm<BF, RF32, MX4, 16, 2>(a, stream);
  }
  if (n <= 128) return launch_norm<BF, RF32, MX4, 1, 2>(a, stream);
  if (n <= 256) return launch_norm<BF, RF32, MX4, 4, 1>(a, stream);
  if (n <= 512) return launch_norm<BF, RF32, MX4, 4, 2>(a, stream);
  if (n <= 1024) return launch_norm<BF, RF32, MX4, 4, 4>(a, stream);
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
