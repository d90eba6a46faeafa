// Microscaled 4-bit codes: quantization of 16-bit rows (rotated if wanted),
// their values read back, and the gated activation that writes them.
#include <algorithm>

#include "mx4_device.h"

namespace oq {
namespace {

constexpr int kThreads = 256;

// n / d for n < 2^31 by a multiplication: q = (n * m) >> (31 + s).
struct Divisor {
  uint32_t d, m, s;
};
Divisor divisor(uint32_t d) {
  uint32_t s = 0;
  while ((uint64_t{1} << s) < d) ++s;
  // m = ceil(2^(31 + s) / d) < 2^32, exact for n < 2^31.
  return Divisor{d, static_cast<uint32_t>(((uint64_t{1} << (31 + s)) + d - 1) / d), s};
}
__device__ __forceinline__ uint32_t divide(uint32_t n, const Divisor& v) {
  return static_cast<uint32_t>((static_cast<uint64_t>(n) * v.m) >> (31 + v.s));
}

// ---- quantization -------------------------------------------------------------
struct QuantArgs {
  const uint16_t* X;
  int64_t ldx, lds;
  uint8_t* Xq;
  uint8_t* steps;
  uint32_t pieces;   // of this launch (rows * K / 8)
  Divisor row;       // pieces of a row
};

// Without rotation: the maximum is taken on the bits (their order is that of the
// magnitudes) and the conversion from 16 bits is exact before it rounds.
template <bool BF>
__global__ __launch_bounds__(kThreads) void mx4_quantize_kernel(QuantArgs a) {
  const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
  if (i >= a.pieces) return;  // (whole quads)
  const uint32_t r = divide(i, a.row), p = i - r * a.row.d;
  const uint4 q = *reinterpret_cast<const uint4*>(a.X + r * a.ldx + p * 8);
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t w = e == 0 ? q.x : e == 1 ? q.y : e == 2 ? q.z : q.w;
    top = max(top, max(w & 0x7FFFu, (w >> 16) & 0x7FFFu));
  }
  top = quad_max(top);
  const float f = BF ? __uint_as_float(top << 16) : static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(top)));
  const uint32_t field = __float_as_uint(f) >> 23;
  uint32_t byte = step_byte(field), c = 0;
  if (field == 255) {
    byte = 255;
  } else {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = half8<BF>(q, e);
    c = codes8(v, step_of(byte));
  }
  reinterpret_cast<uint32_t*>(a.Xq)[i] = c;
  if ((p & 3) == 0) a.steps[r * a.lds + (p >> 2)] = static_cast<uint8_t>(byte);
}

// Rotated in blocks of 2^LOG channels (5, 6, 7): a thread takes a block of 32,
// whose five stages are its own; the others exchange with the lanes 1 and 2 away.
//
// The stages run in float.  A sum of 2^LOG inputs is then off by at most LOG 2^-24
// sum|x|, and twice a rounding more follow, so codes that the two ends of that
// interval share are the exact ones'; a wave that holds another (about 1 in 50
// for blocks of 32, 1 in 15 for 128) repeats its blocks in double, where the sums of
// fp16 values are exact.  Double for all of them costs twice the operations
// (16384 x 4096 in blocks of 128: 57 us, so 43).
template <int LOG, typename F>
__device__ __forceinline__ void hadamard32(F (&v)[32]) {
#pragma unroll
  for (int h = 1; h < 32; h *= 2)
#pragma unroll
    for (int e = 0; e < 32; ++e)
      if (!(e & h)) {
        const F x = v[e], y = v[e + h];
        v[e] = x + y;
        v[e + h] = x - y;
      }
  auto exchange = [&](auto CTRL, bool upper) {
    constexpr int c = decltype(CTRL)::value;
    const F sign = upper ? static_cast<F>(-1) : static_cast<F>(1);
#pragma unroll
    for (int e = 0; e < 32; ++e) {
      if constexpr (sizeof(F) == 8) {
        const uint64_t b = __builtin_bit_cast(uint64_t, v[e]);
        const uint64_t o = static_cast<uint64_t>(dpp<c>(static_cast<uint32_t>(b >> 32))) << 32 | dpp<c>(static_cast<uint32_t>(b));
        v[e] = fma(sign, v[e], __builtin_bit_cast(F, o));
      } else {
        v[e] = fmaf(sign, v[e], __uint_as_float(dpp<c>(__float_as_uint(v[e]))));
      }
    }
  };
  if constexpr (LOG >= 6) exchange(std::integral_constant<int, kQuadXor1>{}, threadIdx.x & 1);
  if constexpr (LOG >= 7) exchange(std::integral_constant<int, kQuadXor2>{}, threadIdx.x & 2);
}

template <bool BF, int LOG>
__global__ __launch_bounds__(kThreads) void mx4_rotate_quantize_kernel(QuantArgs a) {
  const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
  if (i >= a.pieces) return;  // (pieces of 32 here; whole rotation blocks)
  const uint32_t r = divide(i, a.row), p = i - r * a.row.d;
  const uint4* src = reinterpret_cast<const uint4*>(a.X + r * a.ldx + p * 32);
  constexpr double norm = LOG == 5 ? 0.17677669529663688110 : LOG == 6 ? 0.125 : 0.08838834764831844055;
  uint32_t c[4], byte;
  bool open;
  {
    float v[32], sum = 0.0f;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const uint4 q = src[g];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[8 * g + e] = half8<BF>(q, e);
        sum += fabsf(v[8 * g + e]);
      }
    }
    if constexpr (LOG >= 6) sum += __uint_as_float(dpp<kQuadXor1>(__float_as_uint(sum)));
    if constexpr (LOG >= 7) sum += __uint_as_float(dpp<kQuadXor2>(__float_as_uint(sum)));
    hadamard32<LOG>(v);
    float top = 0.0f;
#pragma unroll
    for (int e = 0; e < 32; ++e) {
      v[e] *= static_cast<float>(norm);
      top = fmaxf(top, fabsf(v[e]));
    }
    const float off = sum * static_cast<float>(norm) * ((LOG + 4) * 0x1p-24f);  // (the sum's and the product's own roundings too)
    const uint32_t th = __float_as_uint(top + off), tl = __float_as_uint(top - off);
    byte = step_byte(th >> 23);
    const float step = step_of(byte);
    // Undecided: the step, a code, or a block outside the range in which floats are this near.  (A block of zeros is decided.)
    open = (th ^ tl) >> 23 != 0 || !(sum < 0x1p100f) || (sum < 0x1p-90f && sum != 0.0f);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float up[8], down[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        up[e] = v[8 * g + e] + off;
        down[e] = v[8 * g + e] - off;
      }
      c[g] = codes8(up, step);
      open |= c[g] != codes8(down, step);
    }
  }
  if (__any(open)) {
    double v[32];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const uint4 q = src[g];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[8 * g + e] = static_cast<double>(half8<BF>(q, e));
    }
    hadamard32<LOG>(v);
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 32; ++e) {
      v[e] *= norm;
      top = max(top, high_word(v[e]));
    }
    byte = step_byte64(top);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      double w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = v[8 * g + e];
      c[g] = codes8(w, byte);
    }
  }
  reinterpret_cast<uint4*>(a.Xq)[i] = make_uint4(c[0], c[1], c[2], c[3]);
  a.steps[r * a.lds + p] = static_cast<uint8_t>(byte);
}

// ---- values -------------------------------------------------------------------
struct ValueArgs {
  const uint8_t* Xq;
  const uint8_t* steps;
  int64_t lds, ldx;
  void* X;
  uint32_t pieces;
  Divisor row;
};

template <int OUT>
__global__ __launch_bounds__(kThreads) void mx4_dequantize_kernel(ValueArgs a) {
  const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
  if (i >= a.pieces) return;
  const uint32_t r = divide(i, a.row), p = i - r * a.row.d;
  const uint32_t c = reinterpret_cast<const uint32_t*>(a.Xq)[i];
  const uint32_t byte = a.steps[r * a.lds + (p >> 2)];
  const float step = byte == 255 ? __uint_as_float(0x7FC00000u) : step_of(byte);
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    // 0, 1/2, 1 .. 6: mantissa and exponent as they lie, the subnormal 1/2 apart.
    const uint32_t m = (c >> (4 * e)) & 7u;
    const float g = m < 2 ? 0.5f * static_cast<float>(m) : __uint_as_float((m << 22) + (126u << 23));
    v[e] = ((c >> (4 * e)) & 8u ? -g : g) * step;
  }
  if constexpr (OUT == OQ_OUT_F32) {
    float4* o = reinterpret_cast<float4*>(static_cast<float*>(a.X) + r * a.ldx + p * 8);
    o[0] = make_float4(v[0], v[1], v[2], v[3]);
    o[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.X) + r * a.ldx + p * 8) = pack_half8<OUT == OQ_OUT_BF16>(v);
  }
}

// ---- gated activation ---------------------------------------------------------
struct ActArgs {
  const uint16_t* GU;
  int64_t ld, ldh, lds, F;
  void* H;           // 16-bit rows, or codes
  uint8_t* steps;
  uint32_t pieces;
  Divisor row;
};

// The exponent t of act(g) = g / (1 + e^-t).
template <int ACT, typename F>
__device__ __forceinline__ F act_exponent(F g) {
  if constexpr (ACT == OQ_ACT_SILU) return g;
  else return static_cast<F>(1.5957691216057307117597842397375) * fma(static_cast<F>(0.044715) * g * g, g, g);  // 2 sqrt(2 / pi)
}

template <bool BF, int ACT, bool MX4>
__global__ __launch_bounds__(kThreads) void gated_activation_kernel(ActArgs a) {
  const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
  if (i >= a.pieces) return;  // (MX4: whole quads)
  const uint32_t r = divide(i, a.row), p = i - r * a.row.d;
  const uint16_t* src = a.GU + r * a.ld + p * 8;
  const uint4 qg = *reinterpret_cast<const uint4*>(src), qu = *reinterpret_cast<const uint4*>(src + a.F);
  float v[8], rel[8], x[8], most = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float g = half8<BF>(qg, e), u = half8<BF>(qu, e), t = act_exponent<ACT>(g);
    x[e] = t * -1.4426950408889634f;  // e^-t = 2^x
    most = fmaxf(most, x[e]);
    v[e] = u * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x[e])) * g;
    // Over what the roundings of t, of its product with log2 e and of their constants
    // (nine at most, 2^-24 each) and of the other steps (seven) can add up to, relative.
    rel[e] = 2.0f * (fabsf(t) * 0x1p-21f + 0x1p-20f);
  }
  // Past x = 126 the reciprocal leaves the normal floats, and u of bf16 can bring the
  // product back: there 1 + 2^x is 2^x, taken 2^-144 times, and the rest of the power
  // goes to u and to the result (from x = 270 on 0: act(g) u is below 2^-134 then, half the
  // smallest bf16).  A wave without such a gate, as nearly all are, does not compute it.
  if (__any(most > 120.0f)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float far = half8<BF>(qu, e) * 0x1p-72f * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(x[e] - 144.0f)) * half8<BF>(qg, e) * 0x1p-72f;
      v[e] = x[e] > 120.0f ? far : v[e];
    }
  }
  if constexpr (!MX4) {
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.H) + r * a.ldh + p * 8) = pack_half8<BF>(v);
  } else {
    float hi = 0.0f, lo = 0.0f;
    float up[8], down[8];
    bool live = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      up[e] = v[e] + v[e] * rel[e];
      down[e] = v[e] - v[e] * rel[e];
      hi = fmaxf(hi, fabsf(up[e]));
      lo = fmaxf(lo, fabsf(down[e]));
      live |= up[e] != up[e];  // (also 0 times a bound that is infinite)
    }
    const uint32_t th = quad_max(__float_as_uint(hi)), tl = quad_max(__float_as_uint(lo));
    uint32_t byte = step_byte(th >> 23), c = codes8(up, step_of(byte));
    // Undecided: a code or the step, a block past the range in which floats are
    // this near, or one with a value that is not a number.  (Blocks of zeros are decided.)
    bool open = live | (c != codes8(down, step_of(byte))) | ((th ^ tl) >> 23 != 0) | (th >= 0x7B000000u);
    if (th < 0x12000000u) {
#pragma unroll
      for (int e = 0; e < 8; ++e) open |= half8<BF>(qg, e) != 0.0f && half8<BF>(qu, e) != 0.0f;
    }
    if (__any(open)) {
      // (One rolled loop: the pieces shift down by a value a turn, the results follow.)
      double w[8] = {};
      uint4 g4 = qg, u4 = qu;
      auto shift = [](uint4& q) {
        q = make_uint4(q.x >> 16 | q.y << 16, q.y >> 16 | q.z << 16, q.z >> 16 | q.w << 16, q.w >> 16);
      };
#pragma unroll 1
      for (int e = 0; e < 8; ++e) {
        const double g = half8<BF>(g4, 0), u = half8<BF>(u4, 0);
#pragma unroll
        for (int k = 0; k < 7; ++k) w[k] = w[k + 1];
        w[7] = g / (1.0 + exp(-act_exponent<ACT>(g))) * u;
        shift(g4);
        shift(u4);
      }
      c = quad_codes(w, &byte);
    }
    reinterpret_cast<uint32_t*>(a.H)[i] = c;
    if ((p & 3) == 0) a.steps[r * a.lds + (p >> 2)] = static_cast<uint8_t>(byte);
  }
}

// Launches of at most 2^30 pieces: f(first row, rows).
template <typename F>
int in_slabs(int64_t M, int64_t per_row, F&& f) {
  const int64_t step = (int64_t{1} << 30) / per_row;
  for (int64_t r = 0; r < M; r += step) {
    const int st = f(r, std::min(step, M - r));
    if (st != OQ_OK) return st;
  }
  return OQ_OK;
}
dim3 grid_of(uint32_t pieces) { return dim3((pieces + kThreads - 1) / kThreads); }

int mx4_codes_validate(int64_t M, int64_t K, const void* Xq, const void* steps) {
  if (M < 0 || K < 32 || K % 32 != 0 || K > OQ_MX4_MAX_K) return OQ_ERR_SHAPE;
  if (M == 0) return OQ_OK;
  if (!Xq || !steps) return OQ_ERR_NULL;
  return aligned(Xq, 16) && aligned(steps, 16) ? OQ_OK : OQ_ERR_ALIGN;
}

template <int ACT>
int launch_activation(bool bf, bool mx4, const ActArgs& a, hipStream_t stream) {
  const dim3 g = grid_of(a.pieces), b(kThreads);
  if (mx4) {
    if (bf) hipLaunchKernelGGL((gated_activation_kernel<true, ACT, true>), g, b, 0, stream, a);
    else hipLaunchKernelGGL((gated_activation_kernel<false, ACT, true>), g, b, 0, stream, a);
  } else {
    if (bf) hipLaunchKernelGGL((gated_activation_kernel<true, ACT, false>), g, b, 0, stream, a);
    else hipLaunchKernelGGL((gated_activation_kernel<false, ACT, false>), g, b, 0, stream, a);
  }
  return launch_status();
}

}  // namespace
}  // namespace oq

extern "C" size_t oq_mx4_step_bytes(int64_t K) { return K < 1 ? 0 : static_cast<size_t>(oq::mx4_step_bytes(K)); }

extern "C" int oq_mx4_quantize(const void* X, int64_t M, int64_t K, int64_t ldx, int32_t dtype, int32_t had_block,
                               uint8_t* Xq, uint8_t* steps, void* stream) {
  using namespace oq;
  int st = mx4_codes_validate(M, K, Xq, steps);
  if (st != OQ_OK) return st;
  if (ldx < K) return OQ_ERR_SHAPE;
  if (dtype != OQ_OUT_F16 && dtype != OQ_OUT_BF16) return OQ_ERR_ARG;
  if (had_block != 1 && had_block != 32 && had_block != 64 && had_block != 128) return OQ_ERR_ARG;
  if (K % had_block != 0) return OQ_ERR_SHAPE;
  if (ldx % 8 != 0) return OQ_ERR_ALIGN;
  if (M == 0) return OQ_OK;
  if (!X) return OQ_ERR_NULL;
  if (!aligned(X, 16)) return OQ_ERR_ALIGN;
  if ((st = device_check()) != OQ_OK) return st;
  const bool bf = dtype == OQ_OUT_BF16;
  const int64_t lds = mx4_step_bytes(K), per_row = K / (had_block == 1 ? 8 : 32);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return in_slabs(M, per_row, [&](int64_t r, int64_t rows) {
    const QuantArgs a{static_cast<const uint16_t*>(X) + r * ldx, ldx, lds, Xq + r * (K / 2), steps + r * lds,
                      static_cast<uint32_t>(rows * per_row), divisor(static_cast<uint32_t>(per_row))};
    const dim3 g = grid_of(a.pieces), b(kThreads);
    switch (had_block + (bf ? 1 : 0)) {
      case 1: hipLaunchKernelGGL((mx4_quantize_kernel<false>), g, b, 0, s, a); break;
      case 2: hipLaunchKernelGGL((mx4_quantize_kernel<true>), g, b, 0, s, a); break;
      case 32: hipLaunchKernelGGL((mx4_rotate_quantize_kernel<false, 5>), g, b, 0, s, a); break;
      case 33: hipLaunchKernelGGL((mx4_rotate_quantize_kernel<true, 5>), g, b, 0, s, a); break;
      case 64: hipLaunchKernelGGL((mx4_rotate_quantize_kernel<false, 6>), g, b, 0, s, a); break;
      case 65: hipLaunchKernelGGL((mx4_rotate_quantize_kernel<true, 6>), g, b, 0, s, a); break;
      case 128: hipLaunchKernelGGL((mx4_rotate_quantize_kernel<false, 7>), g, b, 0, s, a); break;
      default: hipLaunchKernelGGL((mx4_rotate_quantize_kernel<true, 7>), g, b, 0, s, a); break;
    }
    return launch_status();
  });
}

extern "C" int oq_mx4_dequantize(const uint8_t* Xq, const uint8_t* steps, int64_t M, int64_t K, void* X, int64_t ldx,
                                 int32_t out_dtype, void* stream) {
  using namespace oq;
  int st = mx4_codes_validate(M, K, Xq, steps);
  if (st != OQ_OK) return st;
  if (ldx < K) return OQ_ERR_SHAPE;
  if (out_dtype != OQ_OUT_F16 && out_dtype != OQ_OUT_BF16 && out_dtype != OQ_OUT_F32) return OQ_ERR_ARG;
  if (ldx % 8 != 0) return OQ_ERR_ALIGN;
  if (M == 0) return OQ_OK;
  if (!X) return OQ_ERR_NULL;
  if (!aligned(X, 16)) return OQ_ERR_ALIGN;
  if ((st = device_check()) != OQ_OK) return st;
  const int64_t lds = mx4_step_bytes(K), per_row = K / 8, size = out_dtype == OQ_OUT_F32 ? 4 : 2;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return in_slabs(M, per_row, [&](int64_t r, int64_t rows) {
    const ValueArgs a{Xq + r * (K / 2), steps + r * lds, lds, ldx, static_cast<uint8_t*>(X) + r * ldx * size,
                      static_cast<uint32_t>(rows * per_row), divisor(static_cast<uint32_t>(per_row))};
    const dim3 g = grid_of(a.pieces), b(kThreads);
    if (out_dtype == OQ_OUT_F16) hipLaunchKernelGGL((mx4_dequantize_kernel<OQ_OUT_F16>), g, b, 0, s, a);
    else if (out_dtype == OQ_OUT_BF16) hipLaunchKernelGGL((mx4_dequantize_kernel<OQ_OUT_BF16>), g, b, 0, s, a);
    else hipLaunchKernelGGL((mx4_dequantize_kernel<OQ_OUT_F32>), g, b, 0, s, a);
    return launch_status();
  });
}

extern "C" int oq_gated_activation(const void* GU, int64_t M, int64_t F, int64_t ld, int32_t dtype, int32_t act, void* H,
                                   int64_t ldh, uint8_t* Hq, uint8_t* steps, void* stream) {
  using namespace oq;
  const bool mx4 = Hq != nullptr || steps != nullptr;
  if (M < 0 || F < 8 || F % 8 != 0 || F > OQ_MX4_MAX_K || ld < 2 * F) return OQ_ERR_SHAPE;
  if (dtype != OQ_OUT_F16 && dtype != OQ_OUT_BF16) return OQ_ERR_ARG;
  if (act != OQ_ACT_GELU_TANH && act != OQ_ACT_SILU) return OQ_ERR_ARG;
  if (H && mx4) return OQ_ERR_ARG;
  int st = OQ_OK;
  if (mx4 && (st = mx4_codes_validate(M, F, Hq, steps)) != OQ_OK) return st;
  // (Without rows the codes' pointers may be null too: only an H has a stride.)
  if (H && ldh < F) return OQ_ERR_SHAPE;
  if (ld % 8 != 0 || (H && ldh % 8 != 0)) return OQ_ERR_ALIGN;
  if (M == 0) return OQ_OK;
  if (!GU || (!mx4 && !H)) return OQ_ERR_NULL;
  if (!aligned(GU, 16) || (!mx4 && !aligned(H, 16))) return OQ_ERR_ALIGN;
  if ((st = device_check()) != OQ_OK) return st;
  const bool bf = dtype == OQ_OUT_BF16;
  const int64_t lds = mx4_step_bytes(F), per_row = F / 8;
  return in_slabs(M, per_row, [&](int64_t r, int64_t rows) {
    const ActArgs a{static_cast<const uint16_t*>(GU) + r * ld, ld, ldh, lds, F,
                    mx4 ? static_cast<void*>(Hq + r * (F / 2)) : static_cast<void*>(static_cast<uint16_t*>(H) + r * ldh),
                    mx4 ? steps + r * lds : nullptr, static_cast<uint32_t>(rows * per_row),
                    divisor(static_cast<uint32_t>(per_row))};
    return act == OQ_ACT_SILU ? launch_activation<OQ_ACT_SILU>(bf, mx4, a, static_cast<hipStream_t>(stream))
                              : launch_activation<OQ_ACT_GELU_TANH>(bf, mx4, a, static_cast<hipStream_t>(stream));
  });
}
