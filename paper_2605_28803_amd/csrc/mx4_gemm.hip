// The product of two operands in microscaled 4-bit codes, Y = X . W^T + bias.
//
// The matrix instruction takes both operands' codes and, per lane, the step of
// the 32 codes that the lane holds; products and sums are exact to fp32.
#include <algorithm>

#include "mx4_device.h"

namespace oq {
namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));

struct Mx4Args {
  const uint8_t* A;      // codes [M][K / 2]
  const uint8_t* sa;     // steps [M][lds]
  const uint8_t* B;      // [N][K / 2]
  const uint8_t* sb;
  const uint16_t* bias;  // fp16 [N] or null
  void* C;
  int64_t M, N, ldc, lds;
  int K;
};

template <int OUT>
__device__ __forceinline__ void mx4_store(const Mx4Args& a, int64_t off, float y) {
  if constexpr (OUT == OQ_OUT_F32) static_cast<float*>(a.C)[off] = y;
  else static_cast<uint16_t*>(a.C)[off] = to_half<OUT == OQ_OUT_BF16>(y);
}

__device__ __forceinline__ v8i fragment(const uint4& q) {
  return v8i{static_cast<int>(q.x), static_cast<int>(q.y), static_cast<int>(q.z), static_cast<int>(q.w), 0, 0, 0, 0};
}

// A workgroup of WAVES waves owns 16 MB rows and 16 NB columns; the waves take
// units of 512 codes in turn.  In a unit, lane l holds row l % 16 and the four
// blocks 4 (l / 16) .. + 3: 64 bytes of codes and a word of four steps, whose
// byte s goes with matrix instruction s.  Any order of the blocks serves as long
// as both operands have it.
template <int OUT, int NB, int WAVES, int MB>
__global__ __launch_bounds__(64 * WAVES) void mx4_small_kernel(Mx4Args a) {
  constexpr int ROWS = 16 * MB, COLS = 16 * NB, NOUT = ROWS * COLS, NT = 64 * WAVES;
  __shared__ float red[WAVES][NOUT];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t n0 = static_cast<int64_t>(blockIdx.x) * COLS, m0 = static_cast<int64_t>(blockIdx.y) * ROWS;
  const int64_t Kb = a.K / 2;
  const int blocks = a.K / 32, units = (a.K + 511) / 512;
  const int grp = lane >> 4;
  const uint8_t *ap[MB], *as[MB], *bp[NB], *bs[NB];
#pragma unroll
  for (int i = 0; i < MB; ++i) {
    const int64_t r = min<int64_t>(m0 + 16 * i + (lane & 15), a.M - 1);  // (rows past M: not stored)
    ap[i] = a.A + r * Kb;
    as[i] = a.sa + r * a.lds;
  }
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const int64_t r = min<int64_t>(n0 + 16 * j + (lane & 15), a.N - 1);
    bp[j] = a.B + r * Kb;
    bs[j] = a.sb + r * a.lds;
  }
  v4f acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = v4f{0, 0, 0, 0};
  for (int u = wave; u < units; u += WAVES) {
    uint4 qa[MB][4], qb[NB][4];
    uint32_t xa[MB], xb[NB];
    const int b0 = 16 * u + 4 * grp, have = min(max(blocks - b0, 0), 4);  // blocks of this lane
    const uint32_t keep = have == 4 ? 0xFFFFFFFFu : (1u << (8 * have)) - 1;
#pragma unroll
    for (int i = 0; i < MB; ++i) {
      xa[i] = *reinterpret_cast<const uint32_t*>(as[i] + b0) & keep;
#pragma unroll
      for (int c = 0; c < 4; ++c) qa[i][c] = *reinterpret_cast<const uint4*>(ap[i] + 16 * (c < have ? b0 + c : 0));
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      xb[j] = *reinterpret_cast<const uint32_t*>(bs[j] + b0) & keep;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        qb[j][c] = *reinterpret_cast<const uint4*>(bp[j] + 16 * (c < have ? b0 + c : 0));
        if (c >= have) qb[j][c] = make_uint4(0, 0, 0, 0);
      }
    }
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fragment(qa[i][0]), fragment(qb[j][0]), acc[i][j], 4, 4, 0, xa[i], 0, xb[j]);
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fragment(qa[i][1]), fragment(qb[j][1]), acc[i][j], 4, 4, 1, xa[i], 1, xb[j]);
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fragment(qa[i][2]), fragment(qb[j][2]), acc[i][j], 4, 4, 2, xa[i], 2, xb[j]);
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fragment(qa[i][3]), fragment(qb[j][3]), acc[i][j], 4, 4, 3, xa[i], 3, xb[j]);
      }
  }
  // Element e of lane l: row 4 (l / 16) + e, column l % 16.
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) red[wave][(16 * i + 4 * grp + e) * COLS + 16 * j + (lane & 15)] = acc[i][j][e];
  __syncthreads();
  for (int o = threadIdx.x; o < NOUT; o += NT) {
    const int64_t gr = m0 + o / COLS, gc = n0 + o % COLS;
    if (gr >= a.M || gc >= a.N) continue;
    float y = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) y += red[w][o];
    if (a.bias) y += static_cast<float>(__builtin_bit_cast(_Float16, a.bias[gc]));
    mx4_store<OUT>(a, gr * a.ldc + gc, y);
  }
}

template <int OUT>
int mx4_launch(const Mx4Args& a, hipStream_t stream) {
  constexpr int MB = 4, NB = 1, WAVES = 4;
  const int64_t nx = (a.N + 16 * NB - 1) / (16 * NB), rows = 16 * MB * int64_t{65535};
  if (!launchable(nx, 64 * WAVES)) return OQ_ERR_SHAPE;
  for (int64_t r = 0; r < a.M; r += rows) {
    Mx4Args p = a;
    p.A += r * (a.K / 2);
    p.sa += r * a.lds;
    p.C = static_cast<uint8_t*>(a.C) + r * a.ldc * (OUT == OQ_OUT_F32 ? 4 : 2);
    p.M = std::min(rows, a.M - r);
    hipLaunchKernelGGL((mx4_small_kernel<OUT, NB, WAVES, MB>),
                       dim3(static_cast<unsigned>(nx), static_cast<unsigned>((p.M + 16 * MB - 1) / (16 * MB))), dim3(64 * WAVES),
                       0, stream, p);
    const int st = launch_status();
    if (st != OQ_OK) return st;
  }
  return OQ_OK;
}

}  // namespace
}  // namespace oq

extern "C" int oq_mx4_linear(const uint8_t* Xq, const uint8_t* x_steps, int64_t M, const uint8_t* Wq, const uint8_t* w_steps,
                             const void* bias, int64_t N, int64_t K, void* Y, int64_t ldy, int32_t out_dtype, void* stream) {
  using namespace oq;
  if (M < 0 || N < 1 || K < 32 || K % 32 != 0 || K > OQ_MX4_MAX_K || ldy < N) return OQ_ERR_SHAPE;
  if (out_dtype != OQ_OUT_F16 && out_dtype != OQ_OUT_BF16 && out_dtype != OQ_OUT_F32) return OQ_ERR_ARG;
  if (ldy % 8 != 0) return OQ_ERR_ALIGN;
  if (M == 0) return OQ_OK;
  if (!Xq || !x_steps || !Wq || !w_steps || !Y) return OQ_ERR_NULL;
  for (const void* p : {static_cast<const void*>(Xq), static_cast<const void*>(x_steps), static_cast<const void*>(Wq),
                        static_cast<const void*>(w_steps), static_cast<const void*>(Y)})
    if (!aligned(p, 16)) return OQ_ERR_ALIGN;
  if (!aligned(bias, 2)) return OQ_ERR_ALIGN;
  const int st = device_check();
  if (st != OQ_OK) return st;
  const Mx4Args a{Xq, x_steps, Wq, w_steps, static_cast<const uint16_t*>(bias), Y, M, N, ldy, mx4_step_bytes(K),
                  static_cast<int>(K)};
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (out_dtype == OQ_OUT_F16) return mx4_launch<OQ_OUT_F16>(a, s);
  return out_dtype == OQ_OUT_BF16 ? mx4_launch<OQ_OUT_BF16>(a, s) : mx4_launch<OQ_OUT_F32>(a, s);
}
