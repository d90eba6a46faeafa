// The residual stream between two blocks: the norm behind a block, its gate and
// residual scale, and the norm before the next block, in one pass over a row.
//
//   y' = post(y)                              (or y)
//   r' = alpha r + gate[g] y'
//   h  = pre(r') (1 + scale[g]) + shift[g]    (16 bits, or microscaled 4-bit codes)
//
// A row's values stay in registers between its sums, so r and y are read once
// and r' and h written once, and a workgroup takes row after row, the next one's
// loads under way.  A thread holds P pieces of 8 channels of a row, W waves a row
// (W = 1: a wave a row, four rows a workgroup, and no barrier).  With an fp32
// residual a piece is two fours apart, so that every 16-byte access of a wave is
// of one kilobyte (eight together, 32 bytes a lane: 16384 x 4096 into 16 bits 199
// us, so 180).
// Sums of a thread's values are float (double where codes are written), sums
// over threads double.  LayerNorm sums (x - mean)^2 with the mean known: a
// second exchange, but no cancellation.
// Where codes are written, everything is double: the codes are then those of the
// formula in 64 bits, not those of a nearby float.  (Only r' in double and h in
// float with a bound, undecided codes again in double, held more registers and
// was no faster.)
// Bound by memory with 16-bit outputs (16384 x 4096, bf16 residual: 537 MB in 114
// us, 4.7 TB/s; a copy reaches 5.1), by the double operations and the registers that
// they hold with codes (fp32 residual: 705 MB in 196 us).
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
  constexpr bool AHEAD = !(MX4 && P * W > 16);  // (there the registers do not reach)
  // (An exchange of a row of its own, rows in turn of two sets: a set is written again behind another row's
  // barriers.  A row that is left has none, and takes no set.)
  __shared__ double red[2][4][W];
  const int tid = W == 1 ? threadIdx.x & 63 : threadIdx.x;
  const bool all = a.D == 8 * T * P;
  const int64_t step = W == 1 ? 4 * static_cast<int64_t>(gridDim.x) : gridDim.x;
  // First channel of half h of piece c (fp32 residual: fours of a thread's own, T fours apart), and whether the row has it.
  auto at = [&](int c, int h) { return RF32 ? 8 * T * c + 4 * T * h + 4 * tid : 8 * T * c + 8 * tid + 4 * h; };
  auto on = [&](int c, int h) { return all || at(c, h) < a.D; };
  // Piece c of 16-bit rows (0 past their end).
  auto get = [&](const uint16_t* p, int c) {
    if constexpr (RF32) {
      const uint2 z = make_uint2(0, 0);
      const uint2 u = on(c, 0) ? *reinterpret_cast<const uint2*>(p + at(c, 0)) : z;
      const uint2 v = on(c, 1) ? *reinterpret_cast<const uint2*>(p + at(c, 1)) : z;
      return make_uint4(u.x, u.y, v.x, v.y);
    } else {
      return on(c, 0) ? *reinterpret_cast<const uint4*>(p + at(c, 0)) : make_uint4(0, 0, 0, 0);
    }
  };
  auto put = [&](uint16_t* p, int c, const uint4& q) {
    if constexpr (RF32) {
      if (on(c, 0)) *reinterpret_cast<uint2*>(p + at(c, 0)) = make_uint2(q.x, q.y);
      if (on(c, 1)) *reinterpret_cast<uint2*>(p + at(c, 1)) = make_uint2(q.z, q.w);
    } else {
      if (on(c, 0)) *reinterpret_cast<uint4*>(p + at(c, 0)) = q;
    }
  };

  const uint4 zero = make_uint4(0, 0, 0, 0);
  uint4 y[P], r[P][RF32 ? 2 : 1];
  auto load = [&](int64_t row) {
#pragma unroll
    for (int c = 0; c < P; ++c) {
      y[c] = a.Y ? get(a.Y + row * a.ldy, c) : zero;
      if constexpr (RF32) {
        const float* s = static_cast<const float*>(a.R) + row * a.ldr;
#pragma unroll
        for (int h = 0; h < 2; ++h) r[c][h] = a.R && on(c, h) ? *reinterpret_cast<const uint4*>(s + at(c, h)) : zero;
      } else {
        r[c][0] = a.R ? get(static_cast<const uint16_t*>(a.R) + row * a.ldr, c) : zero;
      }
    }
  };
  int64_t row = W == 1 ? static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6) : blockIdx.x;
  if (row >= a.M) return;
  load(row);
  for (int set = 0;;) {
    const int64_t next = row + step;
    int64_t g = 0;
    bool there = true;
    if (a.mod_row && (a.gate || a.scale || a.shift)) {
      const int k = a.mod_row[row];
      there = k >= 0 && k < a.n_mod;  // (else the whole row is left)
      g = there ? k * a.ldm : 0;
    }
    Acc v[P][8];
    uint4 old[P][RF32 ? 2 : 1];
#pragma unroll
    for (int c = 0; c < P; ++c) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[c][e] = half8<BF>(y[c], e);
#pragma unroll
      for (int h = 0; h < (RF32 ? 2 : 1); ++h) old[c][h] = r[c][h];
    }
    if (AHEAD && next < a.M) load(next);  // (under way while this row is worked on)
    // Mean (LayerNorm) and 1 / sqrt(mean square + eps) of the row's v (0 past its end).
    auto statistics = [&](const NormOf& k, int slot, Acc* mean, Acc* rstd) {
      Acc s = 0;
      *mean = 0;
      if (k.kind == OQ_NORM_LAYER) {
#pragma unroll
        for (int c = 0; c < P; ++c)
#pragma unroll
          for (int e = 0; e < 8; ++e) s += v[c][e];
        const Acc m = static_cast<Acc>(row_sum<W>(s, red[set][slot]) * a.inv_d);
        s = 0;
#pragma unroll
        for (int c = 0; c < P; ++c)
#pragma unroll
          for (int h = 0; h < 2; ++h)
            if (on(c, h)) {
#pragma unroll
              for (int e = 4 * h; e < 4 * h + 4; ++e) {
                const Acc d = v[c][e] - m;
                s = fma(d, d, s);
              }
            }
        *mean = m;
      } else {
#pragma unroll
        for (int c = 0; c < P; ++c)
#pragma unroll
          for (int e = 0; e < 8; ++e) s = fma(v[c][e], v[c][e], s);
      }
      *rstd = static_cast<Acc>(inverse_root(row_sum<W>(s, red[set][slot + 1]) * a.inv_d + static_cast<double>(k.eps)));
    };
    // x = piece c's values normed (past the row's end: anything).
    auto apply = [&](const NormOf& k, auto (&x)[8], int c, auto mean, auto rstd) {
      using F = decltype(rstd);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = (k.kind == OQ_NORM_LAYER ? x[e] - mean : x[e]) * rstd;
      if (k.gain) {
        const uint4 q = get(k.gain, c);
        if (k.offset != 0.0f) {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] *= static_cast<F>(k.offset) + static_cast<F>(half8<BF>(q, e));
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] *= static_cast<F>(half8<BF>(q, e));
        }
      }
      if (k.bias) {
        const uint4 q = get(k.bias, c);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] += static_cast<F>(half8<BF>(q, e));
      }
    };
    auto modulate = [&](auto (&x)[8], int c) {
      using F = std::remove_reference_t<decltype(x[0])>;
      if (a.scale) {
        const uint4 q = get(a.scale + g, c);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= static_cast<F>(1) + static_cast<F>(half8<BF>(q, e));
      }
      if (a.shift) {
        const uint4 q = get(a.shift + g, c);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] += static_cast<F>(half8<BF>(q, e));
      }
    };
    if (there) {
      if (a.post.kind != OQ_NORM_NONE) {
        Acc mean, rstd;
        statistics(a.post, 0, &mean, &rstd);
#pragma unroll
        for (int c = 0; c < P; ++c) apply(a.post, v[c], c, mean, rstd);
      }
#pragma unroll
      for (int c = 0; c < P; ++c) {
        if (a.gate) {
          const uint4 q = get(a.gate + g, c);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[c][e] *= static_cast<Acc>(half8<BF>(q, e));
        }
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          Acc x;
          if constexpr (RF32) {
            const uint4 w = old[c][e >> 2];
            x = __uint_as_float((e & 3) == 0 ? w.x : (e & 3) == 1 ? w.y : (e & 3) == 2 ? w.z : w.w);
          } else {
            x = half8<BF>(old[c][0], e);
          }
          v[c][e] = fma(static_cast<Acc>(a.alpha), x, v[c][e]);
          o[e] = static_cast<float>(v[c][e]);
        }
        if (!all) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (!on(c, e >> 2)) v[c][e] = 0;
        }
        if (a.Ro) {
          if constexpr (RF32) {
            float* d = static_cast<float*>(a.Ro) + row * a.ldro;
#pragma unroll
            for (int h = 0; h < 2; ++h)
              if (on(c, h)) *reinterpret_cast<float4*>(d + at(c, h)) = make_float4(o[4 * h], o[4 * h + 1], o[4 * h + 2], o[4 * h + 3]);
          } else {
            put(static_cast<uint16_t*>(a.Ro) + row * a.ldro, c, pack_half8<BF>(o));
          }
        }
      }
      if (a.pre.kind != OQ_NORM_NONE) {
        Acc mean, rstd;
        statistics(a.pre, 2, &mean, &rstd);
#pragma unroll
        for (int c = 0; c < P; ++c) {
          apply(a.pre, v[c], c, mean, rstd);
          modulate(v[c], c);
          if constexpr (MX4 && RF32) {
            // Blocks of eight lanes, one for each half.
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              uint32_t top = 0;
#pragma unroll
              for (int e = 4 * h; e < 4 * h + 4; ++e) top = max(top, high_word(v[c][e]));
              top = quad_max(top);
              const uint32_t byte = step_byte64(max(top, dpp<0x141>(top)));  // (row_half_mirror: the other quad)
              double w[8] = {};
#pragma unroll
              for (int e = 0; e < 4; ++e) w[e] = v[c][4 * h + e];
              const uint32_t code = codes8(w, byte);
              if (on(c, h)) {
                const int p = at(c, h) / 4;
                reinterpret_cast<uint16_t*>(a.Hq + row * (a.D / 2))[p] = static_cast<uint16_t>(code);
                if ((p & 7) == 0) a.steps[row * a.lds + (p >> 3)] = static_cast<uint8_t>(byte);
              }
            }
          } else if constexpr (MX4) {
            uint32_t byte;
            const uint32_t code = quad_codes(v[c], &byte);
            if (on(c, 0)) {  // (whole quads)
              const int p = at(c, 0) / 8;
              reinterpret_cast<uint32_t*>(a.Hq + row * (a.D / 2))[p] = code;
              if ((p & 3) == 0) a.steps[row * a.lds + (p >> 2)] = static_cast<uint8_t>(byte);
            }
          } else {
            float o[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = v[c][e];
            put(a.H + row * a.ldh, c, pack_half8<BF>(o));
          }
        }
      }
    }
    if (next >= a.M) return;
    row = next;
    if (there) set ^= 1;
    if (!AHEAD) load(next);
  }
}

template <bool BF, bool RF32, bool MX4, int W, int P>
int launch_norm(const NormArgs& a, hipStream_t stream) {
  // (At most what the chip holds at once: a workgroup then takes row after row.)
  const int threads = W == 1 ? 256 : 64 * W;
  const int64_t blocks = std::min<int64_t>(W == 1 ? (a.M + 3) / 4 : a.M, 256 * 2048 / threads);
  hipLaunchKernelGGL((residual_norm_kernel<BF, RF32, MX4, W, P>), dim3(static_cast<unsigned>(blocks)), dim3(threads), 0, stream, a);
  return launch_status();
}

// Waves of a row and pieces of a thread, us at 16384 rows (4096 of 8192 channels and more) in bf16 with both RMS norms: W, P
// of the one taken, and of another (timed when a row's roots took longer: up to 9% of these).
//                      fp32 residual                             bf16 residual
//   codes     1024     2, 1 53 / 1, 2 61                         1, 2 39 / 2, 1 45
//             2048     4, 1 100 / 1, 4 151                       4, 1 74 / 1, 4 84
//             4096     8, 1 196 / 4, 2 223                       4, 2 131 / 8, 1 157
//             8192     16, 1 103 / 4, 4 165                      16, 1 89 / 8, 2 97
//            16384     8, 4 223 / 16, 2 245                      16, 2 153 / 8, 4 178
//   16 bits   2048     2, 2 97 / 4, 1 98                         2, 2 60 / 4, 1 64
//             4096     4, 2 180 / 8, 1 188                       4, 2 114 / 8, 1 120
//             8192     16, 1 99 / 8, 2 110                       8, 2 61 / 16, 1 69
// Few rows take one piece a thread: 64 x 4096 8, 1 5.4 / 4, 2 6.4.
template <bool BF, bool RF32, bool MX4>
int launch_norm(const NormArgs& a, hipStream_t stream) {
  const int n = (a.D + 7) / 8;
  const bool few = a.M <= 512;
  if (n <= 64) return launch_norm<BF, RF32, MX4, 1, 1>(a, stream);
  if (n <= 128) return RF32 || few ? launch_norm<BF, RF32, MX4, 2, 1>(a, stream) : launch_norm<BF, RF32, MX4, 1, 2>(a, stream);
  if (n <= 256) return MX4 || few ? launch_norm<BF, RF32, MX4, 4, 1>(a, stream) : launch_norm<BF, RF32, MX4, 2, 2>(a, stream);
  if (n <= 512) return (MX4 && RF32) || few ? launch_norm<BF, RF32, MX4, 8, 1>(a, stream) : launch_norm<BF, RF32, MX4, 4, 2>(a, stream);
  if constexpr (MX4 || RF32) {
    if (n <= 1024) return launch_norm<BF, RF32, MX4, 16, 1>(a, stream);
  } else {
    if (n <= 1024) return launch_norm<BF, RF32, MX4, 8, 2>(a, stream);
  }
  if constexpr (RF32) return launch_norm<BF, RF32, MX4, 8, 4>(a, stream);
  else return launch_norm<BF, RF32, MX4, 16, 2>(a, stream);
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
