// The product of two operands in microscaled 4-bit codes, Y = X . W^T + bias.
//
// The matrix instruction takes both operands' codes and, per lane, the step of
// the 32 codes that the lane holds; products and sums are exact to fp32.
#include <algorithm>

#include "gemm_ring.h"
#include "gemm_rules.h"
#include "mx4_device.h"

namespace oq {
namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

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

template <typename Q>
__device__ __forceinline__ v8i fragment(const Q& q) {
  return v8i{static_cast<int>(q.x), static_cast<int>(q.y), static_cast<int>(q.z), static_cast<int>(q.w), 0, 0, 0, 0};
}

// Few rows: the weight is streamed once, and every wave has its loads under way
// before it multiplies.
//
// A workgroup of WAVES waves owns 16 rows and 16 columns; the waves take units of
// 512 codes in turn, and their sums meet in LDS.  In a unit, lane l holds row l % 16
// and blocks l / 16, l / 16 + 4, .. + 12: a load takes 64 bytes of each row (with
// blocks 4 (l / 16) .. + 3, one word of steps as it lies, every lane's 16 bytes were a
// request of their own: 16 x 8192 x 8192 18.9 us, so 13.5; 1 x 8192 x 8192 10.9, so
// 10.1).  Two or four row blocks a workgroup, or two units at once, were slower for up
// to 16 rows and behind the ring for more.
template <int OUT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void mx4_small_kernel(Mx4Args a) {
  __shared__ float red[WAVES][256];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t n0 = static_cast<int64_t>(blockIdx.x) * 16, m0 = static_cast<int64_t>(blockIdx.y) * 16;
  const int Kb = a.K / 2, blocks = a.K / 32, units = (a.K + 511) / 512, grp = lane >> 4;
  // (Rows past M or N read the last one: not stored.)
  const int64_t ar = min<int64_t>(m0 + (lane & 15), a.M - 1), br = min<int64_t>(n0 + (lane & 15), a.N - 1);
  const uint8_t *ap = a.A + ar * Kb, *as = a.sa + ar * a.lds, *bp = a.B + br * Kb, *bs = a.sb + br * a.lds;
  const uint32_t pick = 0x0C0C0400u + 0x0101u * grp;
  auto gather = [&](const uint4& q) {  // byte grp of each word
    return __builtin_amdgcn_perm(q.y, q.x, pick) | __builtin_amdgcn_perm(q.w, q.z, pick) << 16;
  };
  v4f acc = v4f{0, 0, 0, 0};
  for (int u = wave; u < units; u += WAVES) {
    uint4 qa[4], qb[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {  // (blocks past K: the row's last; their steps are cleared)
      const int o = 16 * min(16 * u + 4 * c + grp, blocks - 1);
      qb[c] = *reinterpret_cast<const uint4*>(bp + o);
      qa[c] = *reinterpret_cast<const uint4*>(ap + o);
    }
    const uint4 xb = *reinterpret_cast<const uint4*>(bs + 16 * u), xa = *reinterpret_cast<const uint4*>(as + 16 * u);
    const int have = min(max((blocks - 16 * u - grp + 3) >> 2, 0), 4);  // this lane's blocks
    const uint32_t keep = have == 4 ? 0xFFFFFFFFu : (1u << (8 * have)) - 1;
    const uint32_t ea = gather(xa) & keep, eb = gather(xb) & keep;
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fragment(qa[0]), fragment(qb[0]), acc, 4, 4, 0, ea, 0, eb);
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fragment(qa[1]), fragment(qb[1]), acc, 4, 4, 1, ea, 1, eb);
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fragment(qa[2]), fragment(qb[2]), acc, 4, 4, 2, ea, 2, eb);
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fragment(qa[3]), fragment(qb[3]), acc, 4, 4, 3, ea, 3, eb);
  }
  // Element e of lane l: row 4 (l / 16) + e, column l % 16.
#pragma unroll
  for (int e = 0; e < 4; ++e) red[wave][(4 * grp + e) * 16 + (lane & 15)] = acc[e];
  __syncthreads();
  const int o = threadIdx.x;
  const int64_t gr = m0 + o / 16, gc = n0 + o % 16;
  if (o >= 256 || gr >= a.M || gc >= a.N) return;
  float y = 0.0f;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) y += red[w][o];
  if (a.bias) y += static_cast<float>(__builtin_bit_cast(_Float16, a.bias[gc]));
  mx4_store<OUT>(a, gr * a.ldc + gc, y);
}

template <int OUT, int WAVES>
int launch_mx4_small(const Mx4Args& a, hipStream_t stream) {  // (few rows: grid.y is small)
  const int64_t nx = (a.N + 15) / 16;
  if (!launchable(nx, 64 * WAVES)) return OQ_ERR_SHAPE;
  hipLaunchKernelGGL((mx4_small_kernel<OUT, WAVES>), dim3(static_cast<unsigned>(nx), static_cast<unsigned>((a.M + 15) / 16)),
                     dim3(64 * WAVES), 0, stream, a);
  return launch_status();
}

// ---------------------------------------------------------------------------
// Products with more rows: both operands streamed into an LDS ring.
//
// A workgroup of WM x WN waves owns (16 TM WM) rows of X and (16 TN WN) rows of
// W; a wave owns (16 TM) x (16 TN) in blocks of 16 x 16, W as the instruction's
// first operand, so that a lane ends up with four consecutive columns of Y.  K
// is walked in stages of 128 codes, one instruction a block; two stages are a
// buffer, 128 bytes a row (whole cache lines: with 64 the level-two cache gave
// half the bytes), and NB buffers are filled by direct-to-LDS loads.  Piece p of a
// row is at slot p ^ f(row / 2 % 8): any sixteen lanes that read at once, taken in
// order or in the fours that 16-byte reads are served in, meet all banks.  The
// steps of sixteen stages of a row are 64 bytes in a buffer of their own, swizzled
// alike (without it their reads took a third of the time); a lane gathers its
// byte of each of four stages into one register.
//
// A wave's fragments of the next stage take the place of this stage's: those of
// X each after its last use, those of W in a second set.  The one barrier of a
// buffer stands in its second stage behind the first instructions, when every
// wave holds all of its fragments: it publishes the next buffer and frees this
// one, which is refilled at once.  A stage is one basic block (only there does the
// order written here hold), so nothing in it is conditional.
__device__ __forceinline__ uint32_t here_and_now(uint32_t v) {
  asm volatile("" : "+v"(v));
  return v;
}
template <int X>
__device__ __forceinline__ uint32_t xor_add(uint32_t v, uint32_t add) {  // (v ^ X) + add, made here and now
  uint32_t r;
  asm volatile("v_xad_u32 %0, %1, %2, %3" : "=v"(r) : "v"(v), "n"(X), "s"(add));
  return r;
}
__device__ __forceinline__ int mx4_slot8(int row, int piece) {
  const int h = row >> 1;
  return piece ^ ((h & 1) | ((h >> 1) & 2) | (((h << 1) ^ h) & 4));
}
__device__ __forceinline__ int mx4_slot4(int row, int piece) {
  const int q = row >> 2;
  return piece ^ ((((q ^ (q >> 1)) & 1) << 1) | ((q >> 1) & 1));
}

// Instruction of a stage behind which its read r is issued: X's first IB
// fragments and W's, one an instruction from the barrier on, then X's each when
// it has been used.
template <int TM, int TN, int IB>
constexpr int mx4_read_at(int r) {
  int t = IB * TN;
  for (int k = 0;; ++k) {
    const int i = k - TN;  // (k >= IB + TN: X's fragment i)
    const int at = std::min(k >= IB + TN ? std::max(t, (i + 1) * TN - 1) : t, TM * TN - 1);
    if (k == r) return at;
    t = at + 1;
  }
}

// And of the last of four stages behind which fragment f's next steps are
// gathered (read three instructions before): W's first, to be taken over at the
// end, then X's, each when this stage's have been used.
template <int TM, int TN, int IB>
constexpr int mx4_take_at(int f) {
  const int order = f < TM ? TN + f : f - TM, at = IB * TN + 3 + order;
  return std::min(f < TM ? std::max(at, (f + 1) * TN - 1) : at, TM * TN - 1);
}

template <int OUT, int WM, int WN, int TM, int TN, int NB, int EU>
__global__ __launch_bounds__(64 * WM * WN, EU) void mx4_ring_kernel(Mx4Args a) {
  constexpr int NW = WM * WN;
  constexpr int BM = 16 * TM * WM, BN = 16 * TN * WN, ROWS = BM + BN;
  constexpr int BUF = ROWS * 128, STEPS = ROWS * 64;
  constexpr int LPW = BUF / 1024 / NW, SPW = STEPS / 1024 / NW;
  static_assert(STEPS % (1024 * NW) == 0, "loads per wave");
  constexpr int TP = BN + 8;  // halves per staged output row
  // NB buffers, then SB times 64 bytes of steps a row (after the K loop: the output
  // tile).  With four buffers under way the next sixteen stages' steps come with them.
  constexpr int SB = NB > 2 ? 2 : 1;
  __shared__ __attribute__((aligned(128))) uint8_t smem[std::max(NB * BUF + SB * STEPS, OUT == OQ_OUT_F32 ? 0 : BM * TP * 2)];
  static_assert(__alignof__(smem) % 128 == 0, "a buffer's second stage is found by flipping bit 6 of an address");

  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wv / WN, wn = wv % WN;
  const int tiles_m = static_cast<int>((a.M + BM - 1) / BM), tiles_n = static_cast<int>((a.N + BN - 1) / BN);
  const int Kb = a.K / 2, lds = static_cast<int>(a.lds), blocks = a.K / 32;
  const int nk = (blocks + 3) / 4;

  int tm, tn;
  ring_tile(static_cast<int>(blockIdx.x), tiles_m, tiles_n, &tm, &tn);
  const int64_t m0 = static_cast<int64_t>(tm) * BM, n0 = static_cast<int64_t>(tn) * BN;

  // Load l of a buffer is rows 8 l .. 8 l + 7 of the tile, X's first (of steps: 16 l ..).
  // Every load's address is held below the end of its operand's rows of the tile:
  // what would lie past it (rows past M or N, whose outputs are not stored; stages
  // past K) is the last piece there is, and what lies behind a row's K within (its
  // last stage's pieces, groups of steps past it) is of the rows behind it, and its
  // steps are cleared.
  const uint8_t *const Ab = a.A + m0 * Kb, *const Bb = a.B + n0 * Kb, *const As = a.sa + m0 * a.lds, *const Bs = a.sb + n0 * a.lds;
  const int Arows = __builtin_amdgcn_readfirstlane(static_cast<int>(min<int64_t>(a.M - m0, BM)));
  const int Brows = __builtin_amdgcn_readfirstlane(static_cast<int>(min<int64_t>(a.N - n0, BN)));
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t*)smem));
  static_assert(LPW % 2 == 0, "with 16 rows the swizzle repeats");
  uint32_t voff[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) voff[i] = static_cast<uint32_t>(lane / 8 * Kb) + mx4_slot8(8 * i + lane / 8, lane & 7) * 16;
  // The wave's load i of the two stages from s on (of those past the last one: one piece for all lanes) into buffer b.
  auto issue = [&](int s, int b, int i) __attribute__((always_inline)) {
    const int l = wv * LPW + i;
    const bool x = l * 8 < BM;
    const uint32_t k = (s < nk ? 64u * s : 0x40000000u) + static_cast<uint32_t>((l * 8 - (x ? 0 : BM)) * Kb);
    dma16(lds0 + b * BUF + l * 1024, min(voff[i & 1] + k, static_cast<uint32_t>((x ? Arows : Brows) * Kb) - 16), x ? Ab : Bb);
  };
  // (Opaque, so that what is made of it is not held in registers over the K loop.)
  auto lane_now = [&]() __attribute__((always_inline)) {
    int l = tid & 63;
    asm volatile("" : "+v"(l));
    return l;
  };
  // The steps of the sixteen stages from s on: four groups of 512 codes a row.
  auto issue_steps = [&](int s) __attribute__((always_inline)) {
    const int lane = lane_now();
#pragma unroll
    for (int i = 0; i < SPW; ++i) {
      const int l = wv * SPW + i;
      const bool x = l * 16 < BM;
      const uint32_t off = static_cast<uint32_t>((l * 16 - (x ? 0 : BM) + lane / 4) * lds) + mx4_slot4(lane / 4, lane & 3) * 16 + static_cast<uint32_t>(s) * 4u;
      dma16(__builtin_amdgcn_readfirstlane(lds0 + NB * BUF + (SB > 1 ? (s >> 4) & 1 : 0) * STEPS + l * 1024), min(off, static_cast<uint32_t>((x ? Arows : Brows) * lds) - 16), x ? As : Bs);
    }
  };

  v4f acc[TM][TN];
  const int frow = lane & 15, grp = lane >> 4;
  // Where this lane's fragments lie in a buffer's first stage (its second: ^ 64),
  // and its steps.  The address of a stage's reads is made when they begin: the
  // assembly keeps the compiler from holding one for each.
  const uint32_t fX = lds0 + (wm * 16 * TM + frow) * 128 + mx4_slot8(frow, grp) * 16;
  const uint32_t fW = lds0 + (BM + wn * 16 * TN + frow) * 128 + mx4_slot8(frow, grp) * 16;
  const uint32_t sX = lds0 + NB * BUF + (wm * 16 * TM + frow) * 64, sW = lds0 + NB * BUF + (BM + wn * 16 * TN + frow) * 64;
  uint32_t aX, aW;
  auto address = [&](auto T_) __attribute__((always_inline)) {
    constexpr int t = decltype(T_)::value;
    aX = xor_add<t % 2 * 64>(fX, t / 2 * BUF);
    aW = xor_add<t % 2 * 64>(fW, t / 2 * BUF);
  };
  auto lds16 = [](uint32_t at) __attribute__((always_inline)) {
    return *reinterpret_cast<__attribute__((address_space(3))) const v4u*>(at);
  };
  constexpr int NF = TM + TN, NM = TM * TN, U = 2 * NB, IB = TM >= 4 ? TM / 4 : 1;
  v4u qx[TM], qw[2][TN];
  uint32_t ex[NF], en[TN];  // a byte of each of four stages, X's first; W's of the next four
  v4u raw[NF];
  auto read_x = [&](auto I_) __attribute__((always_inline)) {
    constexpr int i = decltype(I_)::value;
    qx[i] = lds16(aX + i * 2048);
  };
  auto read_w = [&](auto T_, auto J_) __attribute__((always_inline)) {
    constexpr int t = decltype(T_)::value, j = decltype(J_)::value;
    qw[t & 1][j] = lds16(aW + j * 2048);
  };
  // Steps of fragment f's rows in the four stages from s on (s % 4 == 0), and
  // this lane's bytes of them; those past K are cleared.
  uint32_t bX, bW;
  auto steps_address = [&](int s) __attribute__((always_inline)) {
    const uint32_t at = mx4_slot4(frow, (s >> 2) & 3) * 16 + (SB > 1 ? ((s >> 4) & 1) * STEPS : 0);
    bX = here_and_now(sX + at);
    bW = here_and_now(sW + at);
  };
  auto read_steps = [&](auto F_) __attribute__((always_inline)) {
    constexpr int f = decltype(F_)::value;
    raw[f] = lds16(f < TM ? bX + f * 1024 : bW + (f - TM) * 1024);
  };
  const uint32_t pick = 0x0C0C0400u + 0x0101u * grp;  // byte grp of two words
  auto keep_of = [&](int s) {
    const int have = min(max((blocks - 4 * s - grp + 3) >> 2, 0), 4);  // stages with a block of this lane
    return have == 4 ? 0xFFFFFFFFu : (1u << (8 * have)) - 1;
  };
  auto take_steps = [&](auto F_, uint32_t keep) {
    constexpr int f = decltype(F_)::value;
    const uint32_t e = (__builtin_amdgcn_perm(raw[f].y, raw[f].x, pick) | __builtin_amdgcn_perm(raw[f].w, raw[f].z, pick) << 16) & keep;
    if constexpr (f < TM) ex[f] = e;
    else en[f - TM] = e;
  };

  issue_steps(0);
  if (SB > 1 && nk > 16) issue_steps(16);
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < LPW; ++i) issue(2 * b, b, i);
  wait_vm<(NB - 1) * LPW>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  steps_address(0);
  static_for<NF>([&](auto F_) { read_steps(F_); });
  address(std::integral_constant<int, 0>{});
  static_for<TM>([&](auto I_) { read_x(I_); });
  static_for<TN>([&](auto J_) { read_w(std::integral_constant<int, 0>{}, J_); });
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = v4f{0, 0, 0, 0};
  const uint32_t keep0 = keep_of(0);
  static_for<NF>([&](auto F_) { take_steps(F_, keep0); });
#pragma unroll
  for (int j = 0; j < TN; ++j) ex[TM + j] = en[j];
  // Stage s, s % U == t; false: it was the last one.
  auto stage = [&](int s, auto T_) __attribute__((always_inline)) {
    constexpr int t = decltype(T_)::value, jb = t & 3;
    constexpr auto next = std::integral_constant<int, (t + 1) % U>{};
    const uint32_t keep = jb == 3 ? keep_of(s + 1) : 0;
    static_for<NM>([&](auto M_) __attribute__((always_inline)) {
      constexpr int m = decltype(M_)::value, i = m / TN, j = m % TN;
      if constexpr (t % 2 == 1 && m == IB * TN) {
        // Every wave has this buffer's fragments, and the next buffer is there.
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        wait_vm<(NB - 2) * LPW>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
      }
      acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fragment(qw[t & 1][j]), fragment(qx[i]), acc[i][j], 4, 4, jb,
                                                                   ex[TM + j], jb, ex[i]);
      // Reads of the next stage's fragments.
      if constexpr (m == IB * TN) {
        address(next);
        if constexpr (jb == 3) steps_address(s + 1);
      }
      static_for<NF>([&](auto R_) {
        constexpr int r = decltype(R_)::value;
        if constexpr (mx4_read_at<TM, TN, IB>(r) == m) {
          if constexpr (r < IB) read_x(R_);
          else if constexpr (r < IB + TN) read_w(next, std::integral_constant<int, r - IB>{});
          else read_x(std::integral_constant<int, r - TN>{});
        }
        // And of the next four stages' steps.
        if constexpr (jb == 3) {
          constexpr int at = mx4_take_at<TM, TN, IB>(r);
          if constexpr (std::max(at - 3, IB * TN) == m) read_steps(R_);
          if constexpr (at == m) take_steps(R_, keep);
        }
      });
      if constexpr (t % 2 == 1 && m >= IB * TN) {
        constexpr int l0 = LPW * (m - IB * TN) / (NM - IB * TN), l1 = LPW * (m + 1 - IB * TN) / (NM - IB * TN);
#pragma unroll
        for (int l = l0; l < l1; ++l) issue(s - 1 + U, t / 2, l);
      }
      __builtin_amdgcn_sched_barrier(0);
    });
    if constexpr (jb == 3) {
#pragma unroll
      for (int j = 0; j < TN; ++j) ex[TM + j] = en[j];
    }
  };
  auto step = [&](int s, auto T_) __attribute__((always_inline)) {
    stage(s, T_);
    if (s + 1 >= nk) return false;
    // (Every wave has read the steps of these four stages, the last of sixteen.)
    if (decltype(T_)::value % 4 == 1 && (s & 12) == 12 && s + 3 + 16 * (SB - 1) < nk) issue_steps(s + 3 + 16 * (SB - 1));
    return true;
  };
  auto four = [&](int s, auto T_) __attribute__((always_inline)) {
    constexpr int t = decltype(T_)::value;
    return step(s, std::integral_constant<int, t>{}) && step(s + 1, std::integral_constant<int, t + 1>{}) &&
           step(s + 2, std::integral_constant<int, t + 2>{}) && step(s + 3, std::integral_constant<int, t + 3>{});
  };
  for (int s = 0; four(s, std::integral_constant<int, 0>{}) && (U == 4 || four(s + 4, std::integral_constant<int, U - 4>{})); s += U) {
  }

  // Element e of a lane: W's row 4 (lane / 16) + e, X's row lane % 16.
  wait_vm<0>();  // (no load into LDS outlives the loop)
  const int64_t gc0 = n0 + wn * 16 * TN;
  auto bias4 = [&](int64_t gc, float (&b)[4]) {
#pragma unroll
    for (int u = 0; u < 4; ++u) b[u] = static_cast<float>(__builtin_bit_cast(_Float16, a.bias[min<int64_t>(gc + u, a.N - 1)]));
  };
  if constexpr (OUT != OQ_OUT_F32) {
    // Through LDS, so that rows leave in whole pieces.
    __syncthreads();
    uint16_t* tile = reinterpret_cast<uint16_t*>(smem);
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int lc = wn * 16 * TN + j * 16 + 4 * grp;
      float bias[4] = {};
      if (a.bias) bias4(n0 + lc, bias);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        uint32_t w[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
          w[u] = to_half<OUT == OQ_OUT_BF16>(acc[i][j][2 * u] + bias[2 * u]) |
                 static_cast<uint32_t>(to_half<OUT == OQ_OUT_BF16>(acc[i][j][2 * u + 1] + bias[2 * u + 1])) << 16;
        *reinterpret_cast<uint2*>(tile + (wm * 16 * TM + i * 16 + frow) * TP + lc) = make_uint2(w[0], w[1]);
      }
    }
    __syncthreads();
    constexpr int PIECES = BM * BN / 8 / (64 * NW), STEP = 64 * NW / (BN / 8);
    static_assert(64 * NW % (BN / 8) == 0 && BM % STEP == 0, "output pieces per thread");
    const int lr = tid / (BN / 8), lc = tid % (BN / 8) * 8;
    const int64_t gc = n0 + lc;
    uint16_t* o = static_cast<uint16_t*>(a.C) + (m0 + lr) * a.ldc + gc;
    const uint16_t* t = tile + lr * TP + lc;
    if (gc + 8 <= a.N && m0 + BM <= a.M) {
#pragma unroll 4
      for (int c = 0; c < PIECES; ++c) {
        *reinterpret_cast<uint4*>(o) = *reinterpret_cast<const uint4*>(t);
        o += STEP * a.ldc;
        t += STEP * TP;
      }
    } else if (gc < a.N) {
      const int n = static_cast<int>(min<int64_t>(a.N - gc, 8));
#pragma unroll 1
      for (int64_t gr = m0 + lr; gr < min<int64_t>(a.M, m0 + BM); gr += STEP) {
        if (n == 8) {
          *reinterpret_cast<uint4*>(o) = *reinterpret_cast<const uint4*>(t);
        } else {
#pragma unroll 1
          for (int e = 0; e < n; ++e) o[e] = t[e];
        }
        o += STEP * a.ldc;
        t += STEP * TP;
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int64_t gc = gc0 + 16 * j + 4 * grp;
      float bias[4] = {};
      if (a.bias) bias4(gc, bias);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const int64_t gr = m0 + wm * 16 * TM + i * 16 + frow;
        if (gr >= a.M) continue;
        float* o = static_cast<float*>(a.C) + gr * a.ldc + gc;
        const float x[4] = {acc[i][j][0] + bias[0], acc[i][j][1] + bias[1], acc[i][j][2] + bias[2], acc[i][j][3] + bias[3]};
        if (gc + 4 <= a.N) {
          *reinterpret_cast<float4*>(o) = make_float4(x[0], x[1], x[2], x[3]);
        } else {
#pragma unroll
          for (int u = 0; u < 4; ++u)
            if (gc + u < a.N) o[u] = x[u];
        }
      }
    }
  }
}

template <int OUT, int WM, int WN, int TM, int TN, int NB, int EU>
int launch_mx4_ring(const Mx4Args& a, hipStream_t stream) {
  constexpr int BM = 16 * TM * WM, BN = 16 * TN * WN;
  const int64_t tiles = ((a.M + BM - 1) / BM) * ((a.N + BN - 1) / BN);
  if (!launchable(tiles, 64 * WM * WN)) return OQ_ERR_SHAPE;
  hipLaunchKernelGGL((mx4_ring_kernel<OUT, WM, WN, TM, TN, NB, EU>), dim3(static_cast<unsigned>(tiles)), dim3(64 * WM * WN), 0,
                     stream, a);
  return launch_status();
}

template <int OUT>
int mx4_launch(const Mx4Args& a, hipStream_t stream) {
  if (mx4_few_rows(a.M, a.N, a.K)) {
    switch (mx4_small_waves(a.K)) {
      case 4: return launch_mx4_small<OUT, 4>(a, stream);
      case 8: return launch_mx4_small<OUT, 8>(a, stream);
      default: return launch_mx4_small<OUT, 16>(a, stream);
    }
  }
  const W8Split sp = mx4_split(a.M, a.N, a.K);
  if (sp.at > 0) {
    constexpr int64_t size = OUT == OQ_OUT_F32 ? 4 : 2;
    Mx4Args x = a, y = a;
    if (sp.columns) {
      x.N = sp.at;
      y.N = a.N - sp.at;
      y.B = a.B + sp.at * (a.K / 2);
      y.sb = a.sb + sp.at * a.lds;
      y.bias = a.bias ? a.bias + sp.at : nullptr;
      y.C = static_cast<uint8_t*>(a.C) + sp.at * size;
    } else {
      x.M = sp.at;
      y.M = a.M - sp.at;
      y.A = a.A + sp.at * (a.K / 2);
      y.sa = a.sa + sp.at * a.lds;
      y.C = static_cast<uint8_t*>(a.C) + sp.at * a.ldc * size;
    }
    const int st = mx4_launch<OUT>(x, stream);
    return st != OQ_OK ? st : mx4_launch<OUT>(y, stream);
  }
  switch (mx4_tiling(a.M, a.N, a.K)) {
    case 0: return launch_mx4_ring<OUT, 2, 4, 8, 4, 2, 2>(a, stream);
    case 1: return launch_mx4_ring<OUT, 2, 4, 4, 2, 4, 2>(a, stream);
    case 2: return launch_mx4_ring<OUT, 2, 2, 4, 4, 2, 2>(a, stream);
    case 3: return launch_mx4_ring<OUT, 2, 2, 2, 2, 4, 2>(a, stream);
    default: return launch_mx4_ring<OUT, 2, 2, 4, 2, 4, 1>(a, stream);
  }
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
