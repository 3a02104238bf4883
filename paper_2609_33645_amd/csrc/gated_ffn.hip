// Gated feed-forward block and its gradients (gfx950).
//
//   a = x Wg^T, b = x Wu^T, h = act(a) b, y = h Wd^T          (act: silu, or gelu by the error function)
//   dh = dy Wd, da = dh b act'(a), db = dh act(a)
//   dx = da Wg + db Wu,  dWg = da^T x,  dWu = db^T x,  dWd = dy^T h
//
// Four launches on the tile engines of gemm_bf16.h and gemm_f32.h:
//   ffn_pair    both projections, the activation and the product: a tile holds 128 rows of Wg and the same
//               rows of Wu in blocks of 64, so that a wavefront ends with a and b of the same places
//               in its registers; what is written is h (and a, b for a backward);
//   ffn_down    y;
//   ffn_back    dh, whose epilogue reads a and b and writes da, db and h (formed again);
//   ffn_grads   dx and the three weight gradients, which need only what is there by then, in one launch.
// Every product is laid out with the output's contiguous dimension as the tile's rows, so that a lane's
// accumulators are runs of 4 output values.  a, b, h, da and db are kept in the type of x: they are
// operands of the next products.
// Bound by the matrix products, 6 M D F operations forward and 12 M D F backward, for few rows by reading the
// weights.
#include <algorithm>

#include "gemm_f32.h"
#include "head_tiles.h"
#include "pctc_internal.h"

namespace pctc {

namespace {

using bf::LL;

constexpr int kT = 256;  // tile rows and columns

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

template <int ACT>
__device__ __forceinline__ float act(float a) {
  if constexpr (ACT == kSilu) return a / (1.f + expf(-a));
  else return 0.5f * a * (1.f + erff(a * 0.70710678118654752f));
}
// f = act(a), d = act'(a)
template <int ACT>
__device__ __forceinline__ void act_grad(float a, float& f, float& d) {
  if constexpr (ACT == kSilu) {
    const float s = 1.f / (1.f + expf(-a));
    f = a * s;
    d = s * (1.f + a * (1.f - s));
  } else {
    const float c = 0.5f * (1.f + erff(a * 0.70710678118654752f));
    f = a * c;
    d = c + a * 0.3989422804014327f * expf(-0.5f * a * a);
  }
}

// ---- four consecutive values ---------------------------------------------------------------

template <class E>
__device__ __forceinline__ void store4(typename E::T* p, const float (&v)[4]) {
  if constexpr (E::kBf) *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  else *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
}
template <class E>
__device__ __forceinline__ void load4(const typename E::T* p, float (&v)[4]) {
  if constexpr (E::kBf) {
    const u32x2 w = *reinterpret_cast<const u32x2*>(p);
    v[0] = __uint_as_float(w[0] << 16);
    v[1] = __uint_as_float(w[0] & 0xffff0000u);
    v[2] = __uint_as_float(w[1] << 16);
    v[3] = __uint_as_float(w[1] & 0xffff0000u);
  } else {
    const float4 w = *reinterpret_cast<const float4*>(p);
    v[0] = w.x;
    v[1] = w.y;
    v[2] = w.z;
    v[3] = w.w;
  }
}

// fn(row, col, values) for each run of 4 rows of this lane's accumulators (blocks I0 .. I1 - 1) inside
// rows x cols; rows is a multiple of 4.
template <class G, int I0, int I1, class Fn>
__device__ __forceinline__ void for_runs(f32x16 (&acc)[G::FR][G::FC], int row0, int col0, int rows, int cols, Fn&& fn) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int j = 0; j < G::FC; ++j) {
    const int col = col0 + G::col_of(wave, lane, j);
    if (col >= cols) continue;
#pragma unroll
    for (int i = I0; i < I1; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int row = row0 + G::row_of(wave, lane, i, 4 * q);
        if (row >= rows) continue;
        fn(i, j, q, row, col);
      }
  }
}

// ---- forward -------------------------------------------------------------------------------

template <class E>
struct PairArgs {
  const typename E::T *x, *wg, *wu;
  typename E::T *h, *a, *b;  // a and b null: not kept
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
  G::run(A, B, f0, m0, 0, P.D, st, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int j = 0; j < G::FC; ++j) {
    const int m = m0 + G::col_of(wave, lane, j);
    if (m >= P.M) continue;
#pragma unroll
    for (int i = 0; i < 2; ++i)  // blocks i and i + 2: the same rows of Wg and Wu
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int r = G::row_of(wave, lane, i, 4 * q);  // tile rows 128 q + r hold rows 64 q + r
        const int f = f0 + (r >> 7) * 64 + (r & 63);
        if (f >= P.F) continue;
        float a[4], b[4], h[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          a[e] = acc[i][j][4 * q + e];
          b[e] = acc[i + 2][j][4 * q + e];
          h[e] = act<ACT>(a[e]) * b[e];
        }
        const int64_t at = static_cast<int64_t>(m) * P.F + f;
        store4<E>(P.h + at, h);
        if (P.a) {
          store4<E>(P.a + at, a);
          store4<E>(P.b + at, b);
        }
      }
  }
}

template <class E>
struct DownArgs {
  const typename E::T *h, *wd;
  typename E::T* y;
  int M, F, O;
};

template <class E>
__global__ void __launch_bounds__(512, 1) ffn_down(DownArgs<E> P) {
  using G = typename E::template G<LL::KC, LL::KC>;
  PCTC_FFN_STAGES
  int mt, ot;
  if (!grouped_tile(xcd_swz(blockIdx.x, gridDim.x), (P.M + kT - 1) / kT, (P.O + kT - 1) / kT, mt, ot)) return;
  const typename E::Op A{P.wd, P.F, P.O, P.F, nullptr};
  const typename E::Op B{P.h, P.F, P.M, P.F, nullptr};
  f32x16 acc[G::FR][G::FC];
  G::run(A, B, ot * kT, mt * kT, 0, P.F, st, acc);
  for_runs<G, 0, G::FR>(acc, ot * kT, mt * kT, P.O, P.M, [&](int i, int j, int q, int o, int m) {
    const float v[4] = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    store4<E>(P.y + static_cast<int64_t>(m) * P.O + o, v);
  });
}

// ---- backward ------------------------------------------------------------------------------

template <class E>
struct BackArgs {
  const typename E::T *dy, *wd, *a, *b;
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
  G::run(A, B, ft * kT, mt * kT, 0, P.O, st, acc);
  for_runs<G, 0, G::FR>(acc, ft * kT, mt * kT, P.F, P.M, [&](int i, int j, int q, int f, int m) {
    const int64_t at = static_cast<int64_t>(m) * P.F + f;
    float a[4], b[4], h[4];
    load4<E>(P.a + at, a);
    load4<E>(P.b + at, b);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float dh = acc[i][j][4 * q + e];
      float fa, ga;
      act_grad<ACT>(a[e], fa, ga);
      h[e] = fa * b[e];
      a[e] = dh * b[e] * ga;
      b[e] = dh * fa;
    }
    store4<E>(P.da + at, a);
    store4<E>(P.db + at, b);
    store4<E>(P.h + at, h);
  });
}

template <class E>
struct GradArgs {
  const typename E::T *x, *dy, *wg, *wu, *da, *db, *h;
  typename E::T *dx, *dwg, *dwu, *dwd;  // null: not wanted
  int M, D, F, O;
  int n_dx, n_w, n_d;  // tiles of dx, of dWg (and dWu), of dWd (0: not wanted)
};

// out[col][row ..] = the tile's sums
template <class E, class G>
__device__ __forceinline__ void put_tile(f32x16 (&acc)[G::FR][G::FC], int row0, int col0, int rows, int cols,
                                         typename E::T* out) {
  for_runs<G, 0, G::FR>(acc, row0, col0, rows, cols, [&](int i, int j, int q, int r, int c) {
    const float v[4] = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    store4<E>(out + static_cast<int64_t>(c) * rows + r, v);
  });
}

// dx's tiles first: they are the longest (2 F deep, the others M).
template <class E>
__global__ void __launch_bounds__(512, 1) ffn_grads(GradArgs<E> P) {
  PCTC_FFN_STAGES
  using Op = typename E::Op;
  const int nD = (P.D + kT - 1) / kT, nF = (P.F + kT - 1) / kT, nM = (P.M + kT - 1) / kT;
  int w = blockIdx.x;
  if (w < P.n_dx) {
    using G = typename E::template G<LL::MC, LL::KC>;
    w = xcd_swz(w, P.n_dx);
    const int d0 = w / nM * kT, m0 = w % nM * kT;
    f32x16 acc[G::FR][G::FC];
    const Op Ag{P.wg, P.D, P.D, P.F, nullptr}, Au{P.wu, P.D, P.D, P.F, nullptr};
    const Op Bg{P.da, P.F, P.M, P.F, nullptr}, Bu{P.db, P.F, P.M, P.F, nullptr};
    if constexpr (E::kBf) {
      G::run(Ag, Bg, d0, m0, 0, P.F, st, acc);
      G::template run<false>(Au, Bu, d0, m0, 0, P.F, st, acc);
      put_tile<E, G>(acc, d0, m0, P.D, P.M, P.dx);
    } else {
      G::run(Ag, Bg, d0, m0, 0, P.F, st, acc);
      put_tile<E, G>(acc, d0, m0, P.D, P.M, P.dx);
      G::run(Au, Bu, d0, m0, 0, P.F, st, acc);
      for_runs<G, 0, G::FR>(acc, d0, m0, P.D, P.M, [&](int i, int j, int q, int d, int m) {
        float* const o = P.dx + static_cast<int64_t>(m) * P.D + d;
        float v[4];
        load4<E>(o, v);  // (this lane's own of the first product)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += acc[i][j][4 * q + e];
        store4<E>(o, v);
      });
    }
    return;
  }
  w -= P.n_dx;
  using G = typename E::template G<LL::MC, LL::MC>;
  f32x16 acc[G::FR][G::FC];
  if (w < 2 * P.n_w) {  // rows d, columns f
    w = xcd_swz(w, 2 * P.n_w);
    const bool up = w >= P.n_w;
    w = up ? w - P.n_w : w;
    const int d0 = w % nD * kT, f0 = w / nD * kT;
    const Op A{P.x, P.D, P.D, P.M, nullptr}, B{up ? P.db : P.da, P.F, P.F, P.M, nullptr};
    G::run(A, B, d0, f0, 0, P.M, st, acc);
    put_tile<E, G>(acc, d0, f0, P.D, P.F, up ? P.dwu : P.dwg);
    return;
  }
  w = xcd_swz(w - 2 * P.n_w, P.n_d);  // rows f, columns o
  const int nO = (P.O + kT - 1) / kT;
  const int o0 = w % nO * kT, f0 = w / nO * kT;
  (void)nF;
  const Op A{P.h, P.F, P.F, P.M, nullptr}, B{P.dy, P.O, P.O, P.M, nullptr};
  G::run(A, B, f0, o0, 0, P.M, st, acc);
  put_tile<E, G>(acc, f0, o0, P.F, P.O, P.dwd);
}

int tiles(int n, int t = kT) { return (n + t - 1) / t; }

template <class E>
hipError_t forward(const FfnArgs& q, void* h, hipStream_t stream) {
  using T = typename E::T;
  PairArgs<E> p{static_cast<const T*>(q.x),  static_cast<const T*>(q.wg), static_cast<const T*>(q.wu),
                static_cast<T*>(h), static_cast<T*>(q.a), static_cast<T*>(q.b), q.M, q.D, q.F};
  {
    Prof pr("ffn_pair", stream);
    const dim3 grid(grouped_grid(tiles(q.M), tiles(q.F, kT / 2)));
    if (q.act == kSilu) hipLaunchKernelGGL((ffn_pair<E, kSilu>), grid, dim3(512), 0, stream, p);
    else hipLaunchKernelGGL((ffn_pair<E, kGelu>), grid, dim3(512), 0, stream, p);
  }
  DownArgs<E> d{static_cast<const T*>(h), static_cast<const T*>(q.wd), static_cast<T*>(q.y), q.M, q.F, q.O};
  Prof pr("ffn_down", stream);
  hipLaunchKernelGGL((ffn_down<E>), dim3(grouped_grid(tiles(q.M), tiles(q.O))), dim3(512), 0, stream, d);
  return hipGetLastError();
}

template <class E>
hipError_t backward(const FfnArgs& q, const FfnGrads& g, char* ws, hipStream_t stream) {
  using T = typename E::T;
  const size_t n = align_up(static_cast<size_t>(q.M) * q.F * sizeof(T), 256);
  T *da = reinterpret_cast<T*>(ws), *db = reinterpret_cast<T*>(ws + n), *h = reinterpret_cast<T*>(ws + 2 * n);
  BackArgs<E> b{static_cast<const T*>(g.dy), static_cast<const T*>(q.wd), static_cast<const T*>(q.a),
                static_cast<const T*>(q.b), da, db, h, q.M, q.F, q.O};
  {
    Prof pr("ffn_back", stream);
    const dim3 grid(grouped_grid(tiles(q.M), tiles(q.F)));
    if (q.act == kSilu) hipLaunchKernelGGL((ffn_back<E, kSilu>), grid, dim3(512), 0, stream, b);
    else hipLaunchKernelGGL((ffn_back<E, kGelu>), grid, dim3(512), 0, stream, b);
  }
  GradArgs<E> p{};
  p.x = static_cast<const T*>(q.x);
  p.dy = static_cast<const T*>(g.dy);
  p.wg = static_cast<const T*>(q.wg);
  p.wu = static_cast<const T*>(q.wu);
  p.da = da;
  p.db = db;
  p.h = h;
  p.dx = static_cast<T*>(g.dx);
  p.dwg = static_cast<T*>(g.dwg);
  p.dwu = static_cast<T*>(g.dwu);
  p.dwd = static_cast<T*>(g.dwd);
  p.M = q.M;
  p.D = q.D;
  p.F = q.F;
  p.O = q.O;
  p.n_dx = g.dx ? tiles(q.M) * tiles(q.D) : 0;
  p.n_w = g.dwg ? tiles(q.F) * tiles(q.D) : 0;
  p.n_d = g.dwd ? tiles(q.F) * tiles(q.O) : 0;
  const int total = p.n_dx + 2 * p.n_w + p.n_d;
  if (total > 0) {
    Prof pr("ffn_grads", stream);
    hipLaunchKernelGGL((ffn_grads<E>), dim3(total), dim3(512), 0, stream, p);
  }
  return hipGetLastError();
}

}  // namespace

size_t ffn_workspace_bytes(int dtype, int M, int F, bool back) {
  const size_t n = align_up(static_cast<size_t>(M > 0 ? M : 1) * F * (dtype == 1 ? 2 : 4), 256);
  return back ? 3 * n : n;
}

hipError_t launch_gated_ffn(int dtype, const FfnArgs& q, void* ws, hipStream_t stream) {
  return dtype == 1 ? forward<B16>(q, ws, stream) : forward<F32>(q, ws, stream);
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
