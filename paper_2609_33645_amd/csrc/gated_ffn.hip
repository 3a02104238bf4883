// Gated feed-forward block and its gradients (gfx950).
//
//   a = x Wg^T, b = x Wu^T, h = act(a) b, y = h Wd^T          (act: silu, or gelu by the error function)
//   dh = dy Wd, da = dh b act'(a), db = dh act(a)
//   dx = da Wg + db Wu,  dWg = da^T x,  dWu = db^T x,  dWd = dy^T h
//
// Launches on the tile engines of gemm_bf16.h and gemm_f32.h (bf16 on the ping-pong schedule: 1 to 4% faster here):
//   ffn_pair      both projections, the activation and the product: a tile holds 128 rows of Wg and the same
//                 rows of Wu in blocks of 64, so that a wavefront ends with a and b of the same places
//                 in its registers; what is written is h (and a, b for a backward);
//   ffn_products  y;
//   ffn_back      dh, whose epilogue reads a and b and writes da, db and h (formed again);
//   ffn_products  dx and the three weight gradients, which need only what is there by then, in one launch.
// Every product is laid out with the output's contiguous dimension as the tile's rows, so that a lane's
// accumulators are runs of 4 output values.  h, da and db have the type of x, being operands of the next
// products; a and b are kept in float: rounded to bf16 they alone would make the gradients' error of two
// roundings (an operand's and the result's, 0.0023) one of four (0.0035; 14 us of 1,770 saved at M = 2,567,
// 4,096 x 10,240).
// Bound by the matrix products, 6 M D F operations forward and 12 M D F backward, for few rows by reading the
// weights.
#include <algorithm>

#include "gemm_f32.h"
#include "head_tiles.h"
#include "pctc_internal.h"

namespace pctc {

namespace {

using bf::LL;

constexpr int kFew = 512;  // most rows of x that the forward takes without tiles
constexpr int kLoRows = 8;  // most rows whose h is kept in two parts
constexpr int kT = 256;  // tile rows and columns
constexpr int kWc = 4;   // wavefronts across a tile's columns (two across its rows)

struct B16 {
  using T = uint16_t;
  using Op = bf::GOp;
  static constexpr bool kBf = true;
  template <LL LA, LL LB>
  using G = bf::Gemm<kT, kT, 32, LA, LB, 4, 2, 4, true>;
  using Pair = bf::Gemm<kT, kT, 32, LL::KC, LL::KC, 4, 2, 4, true, true, bf::PairCopy<kT, 32, 8>>;
};
struct F32 {
  using T = float;
  using Op = f3::GOp;
  static constexpr bool kBf = false;
  template <LL LA, LL LB>
  using G = f3::Gemm<LA, LB>;
  using Pair = f3::Gemm<LL::KC, LL::KC, true, f3::PairCopy>;
};
constexpr int kStage = 32768;
static_assert(B16::Pair::kStageBytes == kStage && F32::Pair::kStageBytes == kStage, "one set of stages");

#define PCTC_FFN_STAGES                                                \
  __shared__ __attribute__((aligned(1024))) char st0_[kStage];         \
  __shared__ __attribute__((aligned(1024))) char st1_[kStage];         \
  __shared__ __attribute__((aligned(1024))) char st2_[kStage];         \
  __shared__ __attribute__((aligned(1024))) char st3_[kStage];         \
  char* const st[4] = {st0_, st1_, st2_, st3_};

// ---- activations ---------------------------------------------------------------------------

constexpr int kSilu = 0, kGelu = 1;

// A factor c of act(a) = a c, and what the derivative needs besides (silu: nothing; gelu: exp(-a^2 / 2)).
// silu: c = 1 / (1 + exp(-a)).  gelu: c = (1 + erf(a / sqrt 2)) / 2, the error function by the rational
// approximation 7.1.26 of Abramowitz and Stegun, off by at most 1.5e-7 (with float roundings 3.1e-7 of
// c, 8e-8 of gelu root mean square over normal values): 15 instructions that share their exponential with the
// derivative, where the library's erff, expf and division take 80, which is as long as a float product
// 512 deep.
template <int ACT>
__device__ __forceinline__ float act_factor(float a, float& e) {
  if constexpr (ACT == kSilu) {
    e = 0.f;
    return __builtin_amdgcn_rcpf(1.f + fast_exp2(a * -kLog2e));
  } else {
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(a), 0.3275911f * 0.70710678118654752f, 1.f));
    float p = fmaf(t, 1.061405429f, -1.453152027f);
    p = fmaf(p, t, 1.421413741f);
    p = fmaf(p, t, -0.284496736f);
    p = fmaf(p, t, 0.254829592f);
    e = fast_exp2(a * a * (-0.5f * kLog2e));
    const float half = 0.5f * p * t * e;
    return a < 0.f ? half : 1.f - half;
  }
}
template <int ACT>
__device__ __forceinline__ float act(float a) {
  float e;
  return a * act_factor<ACT>(a, e);
}
// f = act(a), d = act'(a)
template <int ACT>
__device__ __forceinline__ void act_grad(float a, float& f, float& d) {
  float e;
  const float c = act_factor<ACT>(a, e);
  f = a * c;
  if constexpr (ACT == kSilu) d = fmaf(f, 1.f - c, c);
  else d = fmaf(a * 0.3989422804014327f, e, c);
}

// From dh, a and b: h, and da in a's place, db in b's.
template <int ACT>
__device__ __forceinline__ void back_values(const float (&dh)[8], float (&a)[8], float (&b)[8], float (&h)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float f, d;
    act_grad<ACT>(a[e], f, d);
    h[e] = f * b[e];
    a[e] = dh[e] * b[e] * d;
    b[e] = dh[e] * f;
  }
}

// ---- eight consecutive values (16-byte aligned) --------------------------------------------

template <class E>
__device__ __forceinline__ void store8(typename E::T* p, const float (&v)[8]) {
  if constexpr (E::kBf) {
    *reinterpret_cast<u32x4*>(p) = u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                                         pack_bf16x2(v[6], v[7])};
  } else {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
  }
}
template <class E>
__device__ __forceinline__ void store4(typename E::T* p, const float (&v)[4]) {
  if constexpr (E::kBf) *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  else *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
}
template <class E>
struct Raw;  // eight values as they lie in memory
template <>
struct Raw<B16> {
  struct __attribute__((aligned(16))) Eight {
    u32x4 w;
  };
  __device__ static __forceinline__ void values(const Eight& x, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = __uint_as_float(x.w[e] << 16);
      v[2 * e + 1] = __uint_as_float(x.w[e] & 0xffff0000u);
    }
  }
};
template <>
struct Raw<F32> {
  struct __attribute__((aligned(16))) Eight {
    float4 a, b;
  };
  __device__ static __forceinline__ void values(const Eight& x, float (&v)[8]) {
    v[0] = x.a.x;
    v[1] = x.a.y;
    v[2] = x.a.z;
    v[3] = x.a.w;
    v[4] = x.b.x;
    v[5] = x.b.y;
    v[6] = x.b.z;
    v[7] = x.b.w;
  }
};
template <class E>
__device__ __forceinline__ void load8(const typename E::T* p, float (&v)[8]) {
  Raw<E>::values(*reinterpret_cast<const typename Raw<E>::Eight*>(p), v);
}

// ---- few rows ------------------------------------------------------------------------------

// The projections (MATS 2: the same rows of w0 and w1, then h = act(a) b) or a plain product (MATS 1) for few
// rows of x.  A workgroup takes 16 RB rows of the weights and 16 NT of x, its wavefronts a share of k each, and
// adds the shares up in order through LDS.  Weights and rows go from memory to the matrix instructions' registers
// (16 x 16, 16 bytes a lane: 64 bytes of each of 16 rows an instruction) without LDS: every weight is used by
// one wavefront only, and what bounds the kernel is reading the weights (from 32 rows on, those and x from the caches).
// Rows past R or M repeat the last one; what they give is not written.  LO (bf16, at most 8 rows): h in two parts, the
// second what the rounding of the first leaves, which takes the columns of the matrix instruction that 8 rows leave
// free: y is off by its own rounding alone (0.0024 -> 0.0017 of its norm), for nothing (one row of 4,096 x 10,240; as
// rows and instructions of their own, 52 -> 56 us).
template <class E>
struct FewArgs {
  const typename E::T *x, *w0, *w1;
  typename E::T* out;
  float *a, *b;  // null: not kept
  int M, K, R;
  const typename E::T* xlo = nullptr;  // LO: what the rounding of x left
  typename E::T* lo = nullptr;         // LO: what the rounding of h leaves
};
typedef __attribute__((ext_vector_type(4))) float f32x4;

template <class E>
__device__ __forceinline__ void few_step(const u32x4& w, const u32x4& x, f32x4& acc) {
  if constexpr (E::kBf) {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x), acc, 0,
                                                  0, 0);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)  // k in another order, the same for both operands
      acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[e]), __uint_as_float(x[e]), acc, 0, 0, 0);
  }
}

template <class E, int MATS, int RB, int NT, int KS, int ACT, bool LO = false>
__global__ void __launch_bounds__(KS * 64) ffn_few(FewArgs<E> P) {
  using T = typename E::T;
  constexpr int kPer = E::kBf ? 8 : 4, kStep = 4 * kPer;  // values of a lane, k of a step
  constexpr int U = MATS * RB + NT >= 6 ? 2 : 4;          // steps read ahead
  constexpr int NA = MATS * RB * NT;                      // accumulators
  __shared__ f32x4 sum[KS][NA][64];
  const int lane = threadIdx.x & 63, ks = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r0 = blockIdx.x * 16 * RB, m0 = blockIdx.y * 16 * NT;
  const int ko = (lane >> 4) * kPer;
  const T* w[MATS][RB];
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const int64_t at = static_cast<int64_t>(min(r0 + 16 * b + (lane & 15), P.R - 1)) * P.K + ko;
    w[0][b] = P.w0 + at;
    if constexpr (MATS == 2) w[1][b] = P.w1 + at;
  }
  const T* x[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) x[n] = P.x + static_cast<int64_t>(min(m0 + 16 * n + (lane & 15), P.M - 1)) * P.K + ko;
  constexpr bool kLoX = LO && MATS == 1;
  if constexpr (kLoX)
    x[0] = ((lane & 8) ? P.xlo : P.x) + static_cast<int64_t>(min(lane & 7, P.M - 1)) * P.K + ko;
  f32x4 acc[MATS][RB][NT];
#pragma unroll
  for (int q = 0; q < MATS; ++q)
#pragma unroll
    for (int b = 0; b < RB; ++b)
#pragma unroll
      for (int n = 0; n < NT; ++n) acc[q][b][n] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int share = (P.K + KS * kStep - 1) / (KS * kStep) * kStep;
  const int kb = min(P.K, ks * share), ke = min(P.K, kb + share);
  auto piece = [](const T* p) { return *reinterpret_cast<const u32x4*>(p); };
  int k = kb;
  u32x4 wv[2][MATS][RB][U], xv[2][NT][U];
  auto read = [&](int s, int at) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int q = 0; q < MATS; ++q)
#pragma unroll
        for (int b = 0; b < RB; ++b) wv[s][q][b][u] = piece(w[q][b] + at + u * kStep);
#pragma unroll
      for (int n = 0; n < NT; ++n) xv[s][n][u] = piece(x[n] + at + u * kStep);
    }
  };
  auto use = [&](int s) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int q = 0; q < MATS; ++q)
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
          for (int n = 0; n < NT; ++n) few_step<E>(wv[s][q][b][u], xv[s][n][u], acc[q][b][n]);
  };
  constexpr int kBlock = U * kStep;
  const int blocks = (ke - kb) / kBlock;
  if (blocks > 0) {
    read(0, k);
    int i = 0;
    for (; i + 2 < blocks; i += 2) {
      read(1, k + kBlock);
      use(0);
      read(0, k + 2 * kBlock);
      use(1);
      k += 2 * kBlock;
    }
    if (i + 1 < blocks) {
      read(1, k + kBlock);
      use(0);
      use(1);
      k += 2 * kBlock;
    } else {
      use(0);
      k += kBlock;
    }
  }
  for (; k < ke; k += kStep) {  // the last steps; lanes past K have zeros
    const bool in = k + ko < P.K;
    const u32x4 zero = {0u, 0u, 0u, 0u};
    u32x4 xt[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) xt[n] = in ? piece(x[n] + k) : zero;
#pragma unroll
    for (int q = 0; q < MATS; ++q)
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        const u32x4 wt = in ? piece(w[q][b] + k) : zero;
#pragma unroll
        for (int n = 0; n < NT; ++n) few_step<E>(wt, xt[n], acc[q][b][n]);
      }
  }
#pragma unroll
  for (int q = 0; q < MATS; ++q)
#pragma unroll
    for (int b = 0; b < RB; ++b)
#pragma unroll
      for (int n = 0; n < NT; ++n) sum[ks][(q * RB + b) * NT + n][lane] = acc[q][b][n];
  __syncthreads();
  for (int i = threadIdx.x; i < RB * NT * 64; i += KS * 64) {
    const int l = i & 63, n = (i >> 6) % NT, b = (i >> 6) / NT;
    const int m = m0 + 16 * n + (l & 15), r = r0 + 16 * b + 4 * (l >> 4);
    if (m >= P.M || r >= P.R) continue;
    float v[MATS][4] = {};
#pragma unroll
    for (int g = 0; g < KS; ++g)
#pragma unroll
      for (int q = 0; q < MATS; ++q) {
        const f32x4 s = sum[g][(q * RB + b) * NT + n][l];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[q][e] += s[e];
        if constexpr (kLoX) {
          const f32x4 t = sum[g][(q * RB + b) * NT + n][l + 8];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[q][e] += t[e];
        }
      }
    const int64_t at = static_cast<int64_t>(m) * P.R + r;
    if constexpr (MATS == 2) {
      float h[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) h[e] = act<ACT>(v[0][e]) * v[1][e];
      store4<E>(P.out + at, h);
      if constexpr (LO) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float rest = h[e] - bf16_to_f32(f32_to_bf16(h[e]));
          h[e] = rest - rest == 0.f ? rest : 0.f;  // (an infinite h has none: it would undo the first part)
        }
        store4<E>(P.lo + at, h);
      }
      if (P.a) {
        store4<F32>(P.a + at, v[0]);
        store4<F32>(P.b + at, v[1]);
      }
    } else {
      store4<E>(P.out + at, v[0]);
    }
  }
}

// How a launch is cut: 16 RB rows of the weights and 16 NT rows of x a workgroup, KS shares of k.  Rows of x are
// read by every workgroup of other weights and weights by every one of other rows, from the caches; the least of
// that which leaves a workgroup for every compute unit is best from 32 rows on (the most workgroups where none
// does), and up to 16 rows, which memory bounds, 16 rows of weights.  The block of 1,024 x 4,096 in bf16, 128
// rows: 31 us by the most workgroups, 24 so.
template <class E, int MATS, int ACT>
void launch_few(const FewArgs<E>& P, hipStream_t stream) {
  static const int cuts[5][2] = {{1, 1}, {1, 2}, {2, 2}, {1, 4}, {2, 4}};
  int best = 0;
  int64_t least = -1;
  for (int c = 0; c < 5 && P.M > 16; ++c) {
    const int rb = cuts[c][0], nt = cuts[c][1];
    const int64_t nr = (P.R + 16 * rb - 1) / (16 * rb), nm = (P.M + 16 * nt - 1) / (16 * nt);
    if (c > 0 && (nr * nm < 256 || 16 * (nt / 2) >= P.M)) continue;
    const int64_t read = nr * P.M + nm * P.R * MATS;  // times K
    if (least < 0 || read < least) {
      least = read;
      best = c;
    }
  }
  if constexpr (E::kBf) {
    if (P.xlo || P.lo) {  // (at most kLoRows rows)
      hipLaunchKernelGGL((ffn_few<E, MATS, 1, 1, 8, ACT, true>), dim3((P.R + 15) / 16), dim3(512), 0, stream, P);
      return;
    }
  }
#define PCTC_FEW(C, RB, NT, KS)                                                                                     \
  case C:                                                                                                           \
    hipLaunchKernelGGL((ffn_few<E, MATS, RB, NT, KS, ACT>), dim3((P.R + 16 * RB - 1) / (16 * RB),                   \
                       (P.M + 16 * NT - 1) / (16 * NT)), dim3(KS * 64), 0, stream, P);                              \
    break
  switch (best) {
    PCTC_FEW(0, 1, 1, 8);
    PCTC_FEW(1, 1, 2, 8);
    PCTC_FEW(2, 2, 2, 8);
    PCTC_FEW(3, 1, 4, 8);
    PCTC_FEW(4, 2, 4, 4);
  }
#undef PCTC_FEW
}

// ---- forward -------------------------------------------------------------------------------

template <class E>
struct PairArgs {
  const typename E::T *x, *wg, *wu;
  typename E::T* h;
  float *a, *b;  // null: not kept
  int M, D, F;
};

template <class E, int ACT>
__global__ void __launch_bounds__(512, 1) ffn_pair(PairArgs<E> P) {
  using G = typename E::Pair;
  PCTC_FFN_STAGES
  int mt, ft;
  if (!grouped_tile(xcd_swz(blockIdx.x, gridDim.x), (P.M + kT - 1) / kT, (P.F + kT / 2 - 1) / (kT / 2), mt, ft)) return;
  const int m0 = mt * kT, f0 = ft * (kT / 2);
  typename E::Op A{P.wg, P.D, P.F, P.D, nullptr};
  A.base2 = P.wu;
  const typename E::Op B{P.x, P.D, P.M, P.D, nullptr};
  f32x16 acc[G::FR][G::FC];
  if constexpr (E::kBf) G::run_pp(A, B, f0, m0, 0, P.D, st, acc);
  else G::run(A, B, f0, m0, 0, P.D, st, acc);
  // 64 rows of Wg, then the same of Wu: lanes b and b + 8 of a column have a and b of the same places
  const int wave = threadIdx.x >> 6;
  const int fw = f0 + wave / kWc * 64, mw = m0 + wave % kWc * 64;
  by_columns<G>(acc, st, [&](int block, int col, const float (&v)[8]) {
    const int f = fw + (block & 7) * 8, m = mw + col;
    const bool in = f < P.F && m < P.M;
    const int64_t at = static_cast<int64_t>(m) * P.F + f;
    float h[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float o = __shfl_xor(v[e], 8, 64);
      h[e] = act<ACT>(block < 8 ? v[e] : o) * (block < 8 ? o : v[e]);
    }
    if (in && block < 8) store8<E>(P.h + at, h);
    if (in && P.a) store8<F32>((block < 8 ? P.a : P.b) + at, v);
  });
}

// ---- backward ------------------------------------------------------------------------------

template <class E>
struct BackArgs {
  const typename E::T *dy, *wd;
  const float *a, *b;
  typename E::T *da, *db, *h;
  int M, F, O;
};

template <class E, int ACT>
__global__ void __launch_bounds__(512, 1) ffn_back(BackArgs<E> P) {
  using G = typename E::template G<LL::MC, LL::KC>;
  PCTC_FFN_STAGES
  int mt, ft;
  if (!grouped_tile(xcd_swz(blockIdx.x, gridDim.x), (P.M + kT - 1) / kT, (P.F + kT - 1) / kT, mt, ft)) return;
  const typename E::Op A{P.wd, P.F, P.F, P.O, nullptr};  // rows f, k-lines of Wd
  const typename E::Op B{P.dy, P.O, P.M, P.O, nullptr};
  f32x16 acc[G::FR][G::FC];
  if constexpr (E::kBf) G::run_pp(A, B, ft * kT, mt * kT, 0, P.O, st, acc);
  else G::run(A, B, ft * kT, mt * kT, 0, P.O, st, acc);
  const int wave = threadIdx.x >> 6;
  const int fw = ft * kT + wave / kWc * 128, mw = mt * kT + wave % kWc * 64;
  struct AB {
    Raw<F32>::Eight a, b;
  };
  // (places outside read the tile's first: no branch between the reads)
  by_columns<G, AB>(
      acc, st,
      [&](int block, int col, const float (&dh)[8], const AB& x) {
        const int f = fw + block * 8, m = mw + col;
        if (f >= P.F || m >= P.M) return;
        const int64_t at = static_cast<int64_t>(m) * P.F + f;
        float a[8], b[8], h[8];
        Raw<F32>::values(x.a, a);
        Raw<F32>::values(x.b, b);
        back_values<ACT>(dh, a, b, h);
        store8<E>(P.da + at, a);
        store8<E>(P.db + at, b);
        store8<E>(P.h + at, h);
      },
      [&](int block, int col, AB& x) {
        const int f = fw + block * 8, m = mw + col;
        const int64_t at = f < P.F && m < P.M ? static_cast<int64_t>(m) * P.F + f : 0;
        x.a = *reinterpret_cast<const Raw<F32>::Eight*>(P.a + at);
        x.b = *reinterpret_cast<const Raw<F32>::Eight*>(P.b + at);
      });
}

// ---- products -------------------------------------------------------------------------------

// out[c][r] = sum over k of A[r][k] B[c][k] (+ A2[r][k] B2[c][k]), r < rows, c < cols, for up to four
// products in one launch, each cut along k into `slices` of `depth` (a multiple of 32; the second operands' k
// begins at kp, K rounded up to it).  A product of one slice is written as it is to be; of several, every
// slice's float sums are written and ffn_join adds them in order.  Without `out` the sums are always written,
// for join_pair or join_back, which make something else of them.
struct Product {
  const void *A, *B, *A2, *B2;  // A2 null: none
  void* out;
  float* part;  // [slices][cols][rows]
  int pa, pb;   // pitches
  int rows, cols, K, kp, slices, depth;
  int mc_b;     // B's columns are contiguous in memory (else its k)
  int first;    // workgroups of the products before
};
struct Products {
  Product p[4];
  int n;
};

// LA: the layout of every A; MCB, KCB: which layouts of B there are.
template <class E, LL LA, bool KCB, bool MCB>
__global__ void __launch_bounds__(512, 1) ffn_products(Products Q) {
  using T = typename E::T;
  using Op = typename E::Op;
  using GK = typename E::template G<LA, LL::KC>;
  using GM = typename E::template G<LA, LL::MC>;
  PCTC_FFN_STAGES
  int which = 0;
  while (which + 1 < Q.n && static_cast<int>(blockIdx.x) >= Q.p[which + 1].first) ++which;
  const Product& P = Q.p[which];
  const int nR = (P.rows + kT - 1) / kT, nC = (P.cols + kT - 1) / kT;
  const int w = xcd_swz(blockIdx.x - P.first, nR * nC * P.slices);
  const int slice = w / (nR * nC), rest = w % (nR * nC);
  // the shorter side fastest: the workgroups of an XCD share what they read
  const int rt = nR <= nC ? rest % nR : rest / nC, ct = nR <= nC ? rest / nR : rest % nC;
  const int r0 = rt * kT, c0 = ct * kT;
  const int kb = slice * P.depth, ke = kb + P.depth;
  f32x16 acc[GK::FR][GK::FC];
  const Op A{static_cast<const T*>(P.A), P.pa, P.rows, P.K, nullptr};
  const Op B{static_cast<const T*>(P.B), P.pb, P.cols, P.K, nullptr};
  if (MCB && (!KCB || P.mc_b)) {
    if constexpr (E::kBf) GM::run_pp(A, B, r0, c0, kb, min(ke, P.K), st, acc);
    else GM::run(A, B, r0, c0, kb, min(ke, P.K), st, acc);
  } else if constexpr (KCB) {
    if constexpr (E::kBf) {
      GK::run_pp(A, B, r0, c0, kb, min(ke, P.K), st, acc);  // (nothing where the slice begins past the first half)
      if (P.A2) {
        const Op A2{static_cast<const T*>(P.A2), P.pa, P.rows, P.K, nullptr};
        const Op B2{static_cast<const T*>(P.B2), P.pb, P.cols, P.K, nullptr};
        GK::template run_pp<false>(A2, B2, r0, c0, max(kb - P.kp, 0), min(ke - P.kp, P.K), st, acc);
      }
    } else {  // a slice of a float product lies in one half
      const bool second = P.A2 && kb >= P.kp;
      const Op A1{static_cast<const T*>(second ? P.A2 : P.A), P.pa, P.rows, P.K, nullptr};
      const Op B1{static_cast<const T*>(second ? P.B2 : P.B), P.pb, P.cols, P.K, nullptr};
      const int from = second ? kb - P.kp : kb;
      GK::run(A1, B1, r0, c0, from, min(from + P.depth, P.K), st, acc);
    }
  }
  const int wave = threadIdx.x >> 6;
  const int rw = r0 + wave / kWc * 128, cw = c0 + wave % kWc * 64;
  float* const part = P.slices > 1 || !P.out ? P.part + static_cast<int64_t>(slice) * P.rows * P.cols : nullptr;
  by_columns<GK>(acc, st, [&](int block, int col, const float (&v)[8]) {
    const int r = rw + block * 8, c = cw + col;
    if (r >= P.rows || c >= P.cols) return;
    const int64_t at = static_cast<int64_t>(c) * P.rows + r;
    if (part) store8<F32>(part + at, v);
    else store8<E>(static_cast<T*>(P.out) + at, v);
  });
}

// Eight of a product's values from its slices' sums.
__device__ __forceinline__ void joined(const Product& P, int64_t i, float (&s)[8]) {
  const int64_t n = static_cast<int64_t>(P.rows) * P.cols;
  load8<F32>(P.part + i, s);
#pragma unroll 4
  for (int k = 1; k < P.slices; ++k) {
    float v[8];
    load8<F32>(P.part + k * n + i, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] += v[e];
  }
}

// The sliced products' sums; blockIdx.y: product.
template <class E>
__global__ void __launch_bounds__(256) ffn_join(Products Q) {
  const Product& P = Q.p[blockIdx.y];
  const int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 8;
  if (P.slices < 2 || i >= static_cast<int64_t>(P.rows) * P.cols) return;
  float s[8];
  joined(P, i, s);
  store8<E>(static_cast<typename E::T*>(P.out) + i, s);
}

// Both projections' sums (products 0 and 1) to h, and a and b where they are kept.
template <class E, int ACT>
__global__ void __launch_bounds__(256) join_pair(Products Q, typename E::T* h, float* pa, float* pb) {
  const int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 8;
  if (i >= static_cast<int64_t>(Q.p[0].rows) * Q.p[0].cols) return;
  float a[8], b[8], v[8];
  joined(Q.p[0], i, a);
  joined(Q.p[1], i, b);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = act<ACT>(a[e]) * b[e];
  store8<E>(h + i, v);
  if (pa) {
    store8<F32>(pa + i, a);
    store8<F32>(pb + i, b);
  }
}

// dh's sums to da, db and h.
template <class E, int ACT>
__global__ void __launch_bounds__(256) join_back(Products Q, BackArgs<E> P) {
  const int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 8;
  if (i >= static_cast<int64_t>(P.M) * P.F) return;
  float dh[8], a[8], b[8], h[8];
  joined(Q.p[0], i, dh);
  load8<F32>(P.a + i, a);
  load8<F32>(P.b + i, b);
  back_values<ACT>(dh, a, b, h);
  store8<E>(P.da + i, a);
  store8<E>(P.db + i, b);
  store8<E>(P.h + i, h);
}

int tiles(int n, int t = kT) { return (n + t - 1) / t; }

// Slices.  A launch on 256 compute units takes at most whole rounds of its longest workgroup, and of workgroups
// of several lengths, longest first, about the work of one unit and half the shortest; a k-step (32 deep in
// bf16, 16 in float) takes 0.95 or 1.6 us, a workgroup 6 us more, sliced sums cost 5 us and their bytes at 3 TB/s
// (written beside products, read again from the caches), within kPartBytes.  Tried are the depths that cut the
// longest product into 1 to 16.
constexpr size_t kPartBytes = size_t{128} << 20;
double step_us(bool bf) { return bf ? 0.95 / 32 : 1.6 / 16; }  // per k
// Returns the time by this model.  always_joined: one slice is joined too.
double plan(Products& Q, bool bf, bool always_joined = false) {
  const double step = step_us(bf);
  int longest = 0;
  for (int i = 0; i < Q.n; ++i) longest = std::max(longest, Q.p[i].A2 ? 2 * Q.p[i].kp : Q.p[i].kp);
  double best = -1;
  int best_s[4] = {1, 1, 1, 1};
  for (int cut = 1; cut <= 16; ++cut) {
    const int depth = std::max((longest + cut - 1) / cut, 128);
    double work = 0, most = 0, least = 1e30, bytes = 0;
    int s[4], count = 0;
    for (int i = 0; i < Q.n; ++i) {
      const Product& P = Q.p[i];
      const int halves = P.A2 ? 2 : 1;
      s[i] = std::max((P.kp * halves + depth - 1) / depth, 1);
      if (P.A2 && !bf) s[i] = 2 * std::max((P.kp + depth - 1) / depth, 1);
      const double len = static_cast<double>(P.kp) * halves / s[i] * step + 6;
      work += len * s[i] * tiles(P.rows) * tiles(P.cols);
      most = std::max(most, len);
      least = std::min(least, len);
      count += s[i] * tiles(P.rows) * tiles(P.cols);
      if (s[i] > 1 || always_joined) bytes += 4.0 * s[i] * P.rows * P.cols;
    }
    // (a float product of two halves is sliced whatever its room: cut 1 stays)
    if (cut > 1 && bytes > kPartBytes) break;
    const double rounds = (count + 255) / 256 * most;
    const double launch = Q.n == 1 ? rounds : std::min(rounds, std::max(work / 256 + least / 2, most));
    const double t = launch + (bytes > 0 ? 5 + bytes / 3.0e6 : 0);
    if (best < 0 || t < best) {
      best = t;
      for (int i = 0; i < Q.n; ++i) best_s[i] = s[i];
    }
  }
  for (int i = 0; i < Q.n; ++i) {
    Product& P = Q.p[i];
    const int halves = P.A2 ? 2 : 1;
    if (P.A2 && !bf) {  // slices end where the first half does
      const int per = best_s[i] / 2;
      P.depth = ((P.kp + per - 1) / per + 31) / 32 * 32;
      P.slices = 2 * per;
      if (P.depth * per != P.kp) P.kp = P.depth * per;
    } else {
      P.depth = ((P.kp * halves + best_s[i] - 1) / best_s[i] + 31) / 32 * 32;
      P.slices = (P.kp * halves + P.depth - 1) / P.depth;
    }
  }
  return best;
}

// Bytes of the sliced sums, and their places from `part` on.
size_t place_parts(Products& Q, char* part, bool always_joined = false) {
  size_t at = 0;
  for (int i = 0; i < Q.n; ++i) {
    Product& P = Q.p[i];
    P.part = reinterpret_cast<float*>(part + at);
    if (P.slices > 1 || always_joined) at += align_up(static_cast<size_t>(P.slices) * P.rows * P.cols * 4, 256);
  }
  return at;
}

Product product(const void* A, int pa, const void* B, int pb, bool mc_b, int rows, int cols, int K, void* out) {
  Product P{};
  P.A = A;
  P.B = B;
  P.pa = pa;
  P.pb = pb;
  P.mc_b = mc_b;
  P.rows = rows;
  P.cols = cols;
  P.K = K;
  P.kp = (K + 31) / 32 * 32;
  P.out = out;
  return P;
}

template <class E, LL LA, bool KCB, bool MCB>
hipError_t run_products(Products& Q, const char* name, hipStream_t stream) {
  // longest first
  std::stable_sort(Q.p, Q.p + Q.n, [](const Product& x, const Product& y) { return x.depth > y.depth; });
  int total = 0;
  int64_t most = 0;  // values to join
  for (int i = 0; i < Q.n; ++i) {
    Q.p[i].first = total;
    total += tiles(Q.p[i].rows) * tiles(Q.p[i].cols) * Q.p[i].slices;
    if (Q.p[i].slices > 1 && Q.p[i].out) most = std::max(most, static_cast<int64_t>(Q.p[i].rows) * Q.p[i].cols);
  }
  {
    Prof pr(name, stream);
    hipLaunchKernelGGL((ffn_products<E, LA, KCB, MCB>), dim3(total), dim3(512), 0, stream, Q);
  }
  if (most > 0) {
    Prof pr("ffn_join", stream);
    hipLaunchKernelGGL(ffn_join<E>, dim3(static_cast<unsigned>((most / 8 + 255) / 256), Q.n), dim3(256), 0, stream, Q);
  }
  return hipGetLastError();
}

Products down_products(const FfnArgs& q, const void* h, bool bf) {
  Products Q{};
  Q.n = 1;
  Q.p[0] = product(q.wd, q.F, h, q.F, false, q.O, q.M, q.F, q.y);
  plan(Q, bf);
  return Q;
}

// How the projections are formed.  The times are those of plan()'s model, and for few rows what was measured:
// the weights at 5.3 TB/s and as much again for every 44 rows (36 in float; bf16, 4,096 x 10,240, the whole
// block: 1 row 52 us, 16 rows 68, 64 130, 128 210).
enum class Pair { kFew, kTiles, kSliced };
double few_us(const FfnArgs& q, bool bf, double weights) {
  return 6 + weights * (bf ? 2 : 4) / 5.3e6 * (1 + q.M / (bf ? 44.0 : 36.0));
}
double tiles_us(int count, int K, bool bf) { return (count + 255) / 256 * (K * step_us(bf) + (bf ? 10 : 25)); }
// The rows past the last whole tile go without tiles where that saves a round of the chip (M = 4,215, 512 x 2,048,
// float: 17 x 16 tiles are two rounds, 182 us, 16 x 16 one, 116 and 12 for the rest).
int rows_apart(const FfnArgs& q) {
  const int nF = tiles(q.F, kT / 2), rest = q.M % kT;
  if (rest == 0 || rest > kT / 2 || q.M <= kT) return 0;
  return (q.M / kT * nF + 255) / 256 < (tiles(q.M) * nF + 255) / 256 ? rest : 0;
}
Pair pair_plan(const FfnArgs& q, bool bf, Products& Q) {
  Q = Products{};
  Q.n = 2;
  Q.p[0] = product(q.wg, q.D, q.x, q.D, false, q.F, q.M, q.D, nullptr);
  Q.p[1] = product(q.wu, q.D, q.x, q.D, false, q.F, q.M, q.D, nullptr);
  const double weights = 2.0 * q.D * q.F, sliced = plan(Q, bf, true);
  FfnArgs last = q;
  last.M = rows_apart(q);
  double whole = tiles_us(tiles(q.M - last.M) * tiles(q.F, kT / 2), q.D, bf);
  if (last.M) whole += few_us(last, bf, weights);
  if (q.M <= kFew && few_us(q, bf, weights) <= std::min(sliced, whole)) return Pair::kFew;
  return sliced < whole ? Pair::kSliced : Pair::kTiles;
}
bool down_by_few(const FfnArgs& q, bool bf) {
  if (q.M > kFew) return false;
  Products Q{};
  Q.n = 1;
  Q.p[0] = product(nullptr, q.F, nullptr, q.F, false, q.O, q.M, q.F, nullptr);
  return few_us(q, bf, static_cast<double>(q.O) * q.F) <= plan(Q, bf);
}
// dh by slices (then Q is their plan), or whole tiles with the activation's part in their epilogue.
bool back_sliced(const FfnArgs& q, const void* dy, bool bf, Products& Q) {
  Q = Products{};
  Q.n = 1;
  Q.p[0] = product(q.wd, q.F, dy, q.O, false, q.F, q.M, q.O, nullptr);
  return plan(Q, bf, true) < tiles_us(tiles(q.M) * tiles(q.F), q.O, bf);
}

// The slices are those of all four, so that a gradient does not change with the others that are asked for.
Products grad_products(const FfnArgs& q, const FfnGrads& g, const void* da, const void* db, const void* h, bool bf) {
  Products Q{};
  Q.n = 4;
  Q.p[0] = product(q.wg, q.D, da, q.F, false, q.D, q.M, q.F, g.dx);
  Q.p[0].A2 = q.wu;
  Q.p[0].B2 = db;
  Q.p[1] = product(q.x, q.D, da, q.F, true, q.D, q.F, q.M, g.dwg);
  Q.p[2] = product(q.x, q.D, db, q.F, true, q.D, q.F, q.M, g.dwu);
  Q.p[3] = product(h, q.F, g.dy, q.O, true, q.F, q.O, q.M, g.dwd);
  plan(Q, bf);
  return Q;
}

// h in two parts: for the rows that the matrix instruction holds twice, if both products go without tiles.
bool two_parts(const FfnArgs& q, bool bf) {
  Products Q;
  return bf && q.M <= kLoRows && pair_plan(q, bf, Q) == Pair::kFew && down_by_few(q, bf);
}

template <class E>
hipError_t forward(const FfnArgs& q, void* h, char* part, hipStream_t stream) {
  using T = typename E::T;
  T* const hh = static_cast<T*>(h);
  float *const a = q.a, *const b = q.b;
  const T *const x = static_cast<const T*>(q.x);
  const T *const wg = static_cast<const T*>(q.wg), *const wu = static_cast<const T*>(q.wu);
  const bool silu = q.act == kSilu;
  T* const lo = two_parts(q, E::kBf) ? reinterpret_cast<T*>(part) : nullptr;
  auto few = [&](int m0, int rows) {
    Prof pr("ffn_few", stream);
    const int64_t at = static_cast<int64_t>(m0) * q.F;
    FewArgs<E> f{x + static_cast<int64_t>(m0) * q.D, wg, wu, hh + at, a ? a + at : nullptr, b ? b + at : nullptr,
                 rows, q.D, q.F};
    f.lo = lo;
    if (silu) launch_few<E, 2, kSilu>(f, stream);
    else launch_few<E, 2, kGelu>(f, stream);
  };
  Products Q;
  const Pair how = pair_plan(q, E::kBf, Q);
  if (how == Pair::kFew) {
    few(0, q.M);
  } else if (how == Pair::kSliced) {
    place_parts(Q, part, true);
    const hipError_t e = run_products<E, LL::KC, true, false>(Q, "ffn_pair", stream);
    if (e != hipSuccess) return e;
    Prof pr("ffn_join", stream);
    const dim3 grid(static_cast<unsigned>((static_cast<int64_t>(q.M) * q.F / 8 + 255) / 256));
    if (silu) hipLaunchKernelGGL((join_pair<E, kSilu>), grid, dim3(256), 0, stream, Q, hh, a, b);
    else hipLaunchKernelGGL((join_pair<E, kGelu>), grid, dim3(256), 0, stream, Q, hh, a, b);
  } else {
    const int rest = rows_apart(q), m = q.M - rest, nF = tiles(q.F, kT / 2);
    if (rest > 0) few(m, rest);
    const PairArgs<E> p{x, wg, wu, hh, a, b, m, q.D, q.F};
    Prof pr("ffn_pair", stream);
    const dim3 grid(grouped_grid(tiles(m), nF));
    if (silu) hipLaunchKernelGGL((ffn_pair<E, kSilu>), grid, dim3(512), 0, stream, p);
    else hipLaunchKernelGGL((ffn_pair<E, kGelu>), grid, dim3(512), 0, stream, p);
  }
  if (down_by_few(q, E::kBf)) {
    Prof pr("ffn_few", stream);
    FewArgs<E> d{hh, static_cast<const T*>(q.wd), nullptr, static_cast<T*>(q.y), nullptr, nullptr, q.M, q.F, q.O};
    d.xlo = lo;
    launch_few<E, 1, kSilu>(d, stream);
    return hipGetLastError();
  }
  Q = down_products(q, h, E::kBf);
  place_parts(Q, part);
  return run_products<E, LL::KC, true, false>(Q, "ffn_down", stream);
}

template <class E>
hipError_t backward(const FfnArgs& q, const FfnGrads& g, char* ws, hipStream_t stream) {
  using T = typename E::T;
  const size_t n = align_up(static_cast<size_t>(q.M) * q.F * sizeof(T), 256);
  T *da = reinterpret_cast<T*>(ws), *db = reinterpret_cast<T*>(ws + n), *h = reinterpret_cast<T*>(ws + 2 * n);
  const BackArgs<E> b{static_cast<const T*>(g.dy), static_cast<const T*>(q.wd), q.a, q.b, da, db, h, q.M, q.F, q.O};
  const bool silu = q.act == kSilu;
  Products B;
  if (back_sliced(q, g.dy, E::kBf, B)) {
    place_parts(B, ws + 3 * n, true);
    const hipError_t e = run_products<E, LL::MC, true, true>(B, "ffn_back", stream);
    if (e != hipSuccess) return e;
    Prof pr("ffn_join", stream);
    const dim3 grid(static_cast<unsigned>((static_cast<int64_t>(q.M) * q.F / 8 + 255) / 256));
    if (silu) hipLaunchKernelGGL((join_back<E, kSilu>), grid, dim3(256), 0, stream, B, b);
    else hipLaunchKernelGGL((join_back<E, kGelu>), grid, dim3(256), 0, stream, B, b);
  } else {
    Prof pr("ffn_back", stream);
    const dim3 grid(grouped_grid(tiles(q.M), tiles(q.F)));
    if (silu) hipLaunchKernelGGL((ffn_back<E, kSilu>), grid, dim3(512), 0, stream, b);
    else hipLaunchKernelGGL((ffn_back<E, kGelu>), grid, dim3(512), 0, stream, b);
  }
  Products Q = grad_products(q, g, da, db, h, E::kBf);
  place_parts(Q, ws + 3 * n);
  Q.n = static_cast<int>(std::remove_if(Q.p, Q.p + Q.n, [](const Product& P) { return !P.out; }) - Q.p);
  if (Q.n == 0) return hipGetLastError();
  return run_products<E, LL::MC, true, true>(Q, "ffn_grads", stream);
}

}  // namespace

static size_t ffn_values_bytes(int dtype, int M, int F) {
  return align_up(static_cast<size_t>(M > 0 ? M : 1) * F * (dtype == 1 ? 2 : 4), 256);
}

size_t ffn_workspace_bytes(int dtype, const FfnArgs& q, bool back) {
  const size_t n = ffn_values_bytes(dtype, q.M, q.F);
  if (q.M == 0) return n;
  const bool bf = dtype == 1;
  Products Q;
  size_t part = 0;  // of one step at a time
  if (!back) {
    if (two_parts(q, bf)) return 2 * n;
    if (pair_plan(q, bf, Q) == Pair::kSliced) part = place_parts(Q, nullptr, true);
    if (!down_by_few(q, bf)) {
      Q = down_products(q, nullptr, bf);
      part = std::max(part, place_parts(Q, nullptr));
    }
    return n + part;
  }
  if (back_sliced(q, nullptr, bf, Q)) part = place_parts(Q, nullptr, true);
  FfnArgs w = q;
  w.wu = &w;  // (that there is a second half)
  Q = grad_products(w, FfnGrads{}, nullptr, nullptr, nullptr, bf);
  return 3 * n + std::max(part, place_parts(Q, nullptr));
}

hipError_t launch_gated_ffn(int dtype, const FfnArgs& q, void* ws, hipStream_t stream) {
  char* const part = static_cast<char*>(ws) + ffn_values_bytes(dtype, q.M, q.F);
  return dtype == 1 ? forward<B16>(q, ws, part, stream) : forward<F32>(q, ws, part, stream);
}

hipError_t launch_gated_ffn_backward(int dtype, const FfnArgs& q, const FfnGrads& g, void* ws, hipStream_t stream) {
  if (q.M == 0) {
    const int64_t e = dtype == 1 ? 2 : 4, n = static_cast<int64_t>(q.F) * q.D * e;
    hipError_t r = hipSuccess;
    if (g.dwg && (r = launch_clear(g.dwg, n, stream)) != hipSuccess) return r;
    if (g.dwu && (r = launch_clear(g.dwu, n, stream)) != hipSuccess) return r;
    return g.dwd ? launch_clear(g.dwd, static_cast<int64_t>(q.F) * q.O * e, stream) : r;
  }
  char* const w = static_cast<char*>(ws);
  return dtype == 1 ? backward<B16>(q, g, w, stream) : backward<F32>(q, g, w, stream);
}

}  // namespace pctc
