// Clipped policy loss with a KL term on the tokens of a vocabulary head (gfx950).
//
//   lp_m = z_m[token_m] - lambda_m (z = H W^T + b, lambda over the full vocabulary),  r = exp(lp - old)
//   loss_m = -min(r A, clip(r, 1 - lo, 1 + hi) A) + kl (exp(ref - lp) - (ref - lp) - 1)
//   g_m = w_m dloss_m / dlp_m,   dZ[m] = g_m (onehot(token_m) - p(m)),   dH = dZ W,  dW = dZ^T H
//
// The logits are not stored: the normaliser and the recomputed backward are those of the Pruned CTC
// loss, whose union columns here are one class per frame.  bf16 rows whose token is left out (prompts)
// are left out of the products too: the counted rows are gathered, and every launch ends at their
// number, which only the device knows.  Between the products: the tokens' normalisers, logits and losses (a
// wavefront a token), and in every chunk of the backward the tokens' own entries of dZ, the sum of the
// losses beside the first.  Bound by the matrix products, 8 M V D operations (the logits are formed twice).
#include "gemm_f32.h"
#include "head_tiles.h"
#include "pctc_internal.h"

namespace pctc {

namespace {

constexpr int kThreads = 256;
constexpr int kLossThreads = 512;

// Sum of products of this lane's pieces of two rows of D values (a multiple of 8), 16 bytes at a time.
template <bool BF>
__device__ __forceinline__ float dot_share(const void* a, const void* b, int D, int lane) {
  constexpr int kPer = BF ? 8 : 4;
  float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int d = lane * kPer; d < D; d += 64 * kPer) {
    u32x4 x, y;
    if constexpr (BF) {
      x = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a) + d);
      y = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(b) + d);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[e] = fmaf(__uint_as_float(x[e] << 16), __uint_as_float(y[e] << 16), s[e]);
        s[e] = fmaf(__uint_as_float(x[e] & 0xffff0000u), __uint_as_float(y[e] & 0xffff0000u), s[e]);
      }
    } else {
      x = *reinterpret_cast<const u32x4*>(static_cast<const float*>(a) + d);
      y = *reinterpret_cast<const u32x4*>(static_cast<const float*>(b) + d);
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] = fmaf(__uint_as_float(x[e]), __uint_as_float(y[e]), s[e]);
    }
  }
  return (s[0] + s[1]) + (s[2] + s[3]);
}

// counts[b]: counted tokens of the rows [kCountRows b, kCountRows (b + 1)).
constexpr int kCountRows = 8192;
__global__ void __launch_bounds__(kThreads)
policy_count(const int32_t* __restrict__ tokens, int M, int V, int32_t* __restrict__ counts) {
  const int b = blockIdx.x * kCountRows, e = min(M, b + kCountRows);
  int n = 0;
  for (int m = b + threadIdx.x; m < e; m += kThreads) n += static_cast<uint32_t>(tokens[m]) < static_cast<uint32_t>(V);
  __shared__ int sh[kThreads / 64];
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) n += __shfl_xor(n, o, 64);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = n;
  __syncthreads();
  if (threadIdx.x == 0) counts[blockIdx.x] = sh[0] + sh[1] + sh[2] + sh[3];
}

// The counted rows of H, one behind the other: Hc[j] = H[rows[j]], inv[m] = j (-1: left out), *count of
// them; what a left out row reports.  A workgroup takes kGatherRows rows and counts those before by
// itself (counts: in whole blocks, where there are many).  2,567 rows of 4,096: 16 us.
constexpr int kGatherRows = 8;
__global__ void __launch_bounds__(kThreads)
policy_gather(const uint16_t* __restrict__ H, int M, int D, int V, PolicyArgs a, const int32_t* __restrict__ counts,
              uint16_t* __restrict__ Hc, int32_t* __restrict__ rows, int32_t* __restrict__ inv,
              int32_t* __restrict__ count) {
  const int m0 = blockIdx.x * kGatherRows;
  auto counted = [&](int m) { return m < M && static_cast<uint32_t>(a.tokens[m]) < static_cast<uint32_t>(V); };
  int n = 0, from = 0;
  if (counts) {
    const int blocks = m0 / kCountRows;
    for (int b = threadIdx.x; b < blocks; b += kThreads) n += counts[b];
    from = blocks * kCountRows;
  }
#pragma unroll 8
  for (int m = from + threadIdx.x; m < m0; m += kThreads) n += counted(m);
  __shared__ int sh[kThreads / 64];
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) n += __shfl_xor(n, o, 64);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = n;
  __syncthreads();
  int j = sh[0] + sh[1] + sh[2] + sh[3];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  for (int r = 0; r < kGatherRows; ++r) {
    const int m = m0 + r;
    const bool in = counted(m);
    if (wave == r % (kThreads / 64) && m < M) {
      if (in) {
        const uint16_t* src = H + static_cast<int64_t>(m) * D;
        uint16_t* dst = Hc + static_cast<int64_t>(j) * D;
#pragma unroll 4
        for (int d = lane * 8; d < D; d += 512)
          *reinterpret_cast<u32x4*>(dst + d) = *reinterpret_cast<const u32x4*>(src + d);
      }
      if (lane == 0) {
        inv[m] = in ? j : -1;
        if (in) {
          rows[j] = m;
        } else {
          a.logp[m] = a.losses[m] = 0.f;
          a.status[m] = 1;
        }
      }
    }
    j += in;
  }
  if (m0 + kGatherRows >= M && threadIdx.x == 0) *count = j;
}

// Where the tokens kernel finds its rows and what it leaves for the backward, by place j in H.
struct PolicyRows {
  const int32_t* rows;   // [.]: the row of place j (null: j itself)
  const int32_t* count;  // how many places (null: M)
  const float2* partials;
  int P;          // the normaliser's partial pairs (max, sum) of each place, [P][places]
  float2* lam2;   // lambda log2(e) in two floats
  float* g;
  int32_t* token;
  float* logp;
};

// A logit as the normaliser's products give it, to the bit: the same matrix instructions over the same k, for 32
// rows of H and of W at once, of whose 32 x 32 products the diagonal is wanted.  h, w: this lane's rows (lane mod 32);
// start: the bias of the class (in bf16 the sums start from it, in float it is added).  Lanes whose half does not hold
// their column's return another.
template <bool BF>
__device__ __forceinline__ float tile_logit(const void* h, const void* w, float start, int D, int lane) {
  f32x16 acc;
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[r] = BF ? start : 0.f;
  const int ko = 8 * (lane >> 5);
  if constexpr (BF) {
    constexpr int U = 16;
    const uint16_t *a = static_cast<const uint16_t*>(w) + ko, *b = static_cast<const uint16_t*>(h) + ko;
    for (int k0 = 0; k0 < D; k0 += 16 * U) {
      u32x4 x[U], y[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool in = k0 + 16 * u + ko < D;
        x[u] = in ? *reinterpret_cast<const u32x4*>(a + k0 + 16 * u) : u32x4{0u, 0u, 0u, 0u};
        y[u] = in ? *reinterpret_cast<const u32x4*>(b + k0 + 16 * u) : u32x4{0u, 0u, 0u, 0u};
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x[u]), __builtin_bit_cast(bf16x8, y[u]),
                                                      acc, 0, 0, 0);
    }
  } else {
    constexpr int U = 4;
    const float *a = static_cast<const float*>(w) + ko, *b = static_cast<const float*>(h) + ko;
    f3::f32x4 x[2][U][2], y[2][U][2];
    auto read = [&](int s, int k0) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool in = k0 + 16 * u + ko < D;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          x[s][u][e] = in ? *reinterpret_cast<const f3::f32x4*>(a + k0 + 16 * u + 4 * e) : f3::f32x4{0.f, 0.f, 0.f, 0.f};
          y[s][u][e] = in ? *reinterpret_cast<const f3::f32x4*>(b + k0 + 16 * u + 4 * e) : f3::f32x4{0.f, 0.f, 0.f, 0.f};
        }
      }
    };
    auto use = [&](int s) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        f3::Tri p, q;
        f3::split4<0>(x[s][u][0], p);
        f3::split4<1>(x[s][u][1], p);
        f3::split4<0>(y[s][u][0], q);
        f3::split4<1>(y[s][u][1], q);
#pragma unroll
        for (int i = 2; i >= 0; --i)
#pragma unroll
          for (int e = i; e >= 0; --e) {
            bf16x8 f, g;
            __builtin_memcpy(&f, p.d[e], 16);
            __builtin_memcpy(&g, q.d[i - e], 16);
            acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, g, acc, 0, 0, 0);
          }
      }
    };
    read(0, 0);
    for (int k0 = 0; k0 < D; k0 += 32 * U) {  // (k past D: zeros, which change nothing)
      read(1, k0 + 16 * U);
      use(0);
      read(0, k0 + 32 * U);
      use(1);
    }
  }
  const int c = lane & 31, at = 4 * (c >> 3) + (c & 3);
  float z = 0.f;
#pragma unroll
  for (int r = 0; r < 16; ++r) z = r == at ? acc[r] : z;
  return BF ? z : z + start;
}

// A wavefront a place, eight of them a workgroup.  lambda in double from the pairs; the token's logit from two
// rows of D values, lanes' float sums joined in double; the loss in double.  The normaliser's products round that
// logit otherwise; lambda is corrected by what the difference makes of the token's own share of it (tile_logit), so
// that the log probability of a nearly certain token is right (losses 1.4e-6 -> 2e-7 off 64 bits, fp32 gradients
// 3e-6 -> 3e-7; the first wavefront's sums take 3 us of 331 rows at D = 512, 11 in float, 20 of 1,925 at D = 4,096).
// mask (null: none): a row without a gradient is cleared there, so that what is not finite in it reaches no product.
template <bool BF>
__global__ void __launch_bounds__(kLossThreads)
policy_tokens(const void* H, int M, int D, const void* __restrict__ W, const float* __restrict__ bias, int V,
              PolicyRows R, PolicyArgs a, uint16_t* mask) {
  const int n = R.count ? min(M, *R.count) : M;
  constexpr int kPlaces = kLossThreads / 64;
  const int j0 = blockIdx.x * kPlaces, j = j0 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (j0 >= n) return;
  constexpr int kBytes = BF ? 2 : 4;
  __shared__ float tile[kPlaces];
  if (threadIdx.x < 64) {
    const int c = lane & 31, q = min(j0 + (c & (kPlaces - 1)), n - 1);
    const int t0 = a.tokens[R.rows ? R.rows[q] : q], t = t0 >= 0 && t0 < V ? t0 : 0;
    const float z = tile_logit<BF>(static_cast<const char*>(H) + static_cast<int64_t>(q) * D * kBytes,
                                   static_cast<const char*>(W) + static_cast<int64_t>(t) * D * kBytes,
                                   bias ? bias[t] : 0.f, D, lane);
    if (c < kPlaces && (lane >> 5) == ((c >> 2) & 1)) tile[c] = z;
  }
  __syncthreads();
  if (j >= n) return;
  // lambda: the largest maximum is exact, each sum is scaled by the float exponential of an exact difference, and by
  // what the normaliser's rounding of max log2(e) put into each of its exponents (beside logits of 2,000 that is
  // 8.5e-5 of the sum, and so much of a certain token's log probability)
  constexpr int kPer = kMaxLseParts / 64;
  float2 q[kPer];
  float top = -INFINITY;
  bool nan = false;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int p = lane + 64 * i;
    q[i] = p < R.P ? R.partials[static_cast<int64_t>(p) * n + j] : make_float2(-INFINITY, 0.f);
    nan |= (q[i].x != q[i].x) || (q[i].y != q[i].y);
    top = fmaxf(top, q[i].x);
  }
  top = wave_max(top);
  double sum = 0.0;
  if (top != -INFINITY)
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (q[i].x != -INFINITY) {
        const double r = static_cast<double>(lse_rounding(q[i].x)) * kLn2D;  // exp(-r) to r^4 / 24
        sum += static_cast<double>(q[i].y) * (1.0 - r * (1.0 - r * (0.5 - r / 6.0))) *
               static_cast<double>(fast_exp2(static_cast<float>(static_cast<double>(q[i].x) - top) * kLog2e));
      }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) sum += __shfl_xor(sum, o, 64);
  double lam = top == -INFINITY ? -INFINITY : static_cast<double>(top) + log(sum);
  if (__ballot(nan) != 0) lam = __longlong_as_double(0x7ff8000000000000LL);
  const int m = R.rows ? R.rows[j] : j;
  const int tok = a.tokens[m];
  const bool counted = tok >= 0 && tok < V;
  const char* const row = static_cast<const char*>(H) + static_cast<int64_t>(j) * D * kBytes;
  double z = 0.0;
  if (counted) {
    z = dot_share<BF>(row, static_cast<const char*>(W) + static_cast<int64_t>(tok) * D * kBytes, D, lane);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) z += __shfl_xor(z, o, 64);
  }
  float lp32 = 0.f, loss32 = 0.f, g32 = 0.f;
  int status = 1;  // left out
  if (counted) {
    if (bias) z += static_cast<double>(bias[tok]);
    const double zt = tile[threadIdx.x >> 6], off = z - zt;
    if (fabs(off) < 1.0 && lam - lam == 0.0) lam += log1p(exp(zt - lam) * expm1(off));
    const double lp = z - lam;
    const double A = a.adv[m], w = a.weights ? static_cast<double>(a.weights[m]) : 1.0;
    double loss = 0.0, c = 0.0;
    if (A != 0.0) {  // (a NaN is not)
      const double r = a.old_logp ? exp(lp - static_cast<double>(a.old_logp[m])) : 1.0;
      const double lo = 1.0 - static_cast<double>(a.clip_lo), hi = 1.0 + static_cast<double>(a.clip_hi);
      const double cut = (A > 0.0 ? fmin(r, hi) : fmax(r, lo)) * A;  // the smaller of r A and clip(r) A
      const bool flat = A > 0.0 ? r > hi : r < lo;
      loss = -cut;
      c = flat ? 0.0 : -A * r;
    }
    if (a.ref_logp && a.kl != 0.f) {  // (0 times an infinite difference is not zero)
      const double d = static_cast<double>(a.ref_logp[m]) - lp, x = expm1(d);
      loss += static_cast<double>(a.kl) * (x - d);
      c -= static_cast<double>(a.kl) * x;
    }
    lp32 = static_cast<float>(lp);
    loss32 = static_cast<float>(loss);
    g32 = static_cast<float>(c * w);
    status = 0;
    // (x - x is zero for finite values alone; a weighted loss beyond float's range cannot be kept either)
    const float all = (lp32 - lp32) + (loss32 - loss32) + (g32 - g32) + static_cast<float>(w - w);
    if (!(all == 0.f)) {
      status = 2;
      loss32 = g32 = 0.f;
    }
  }
  if (mask && g32 == 0.f) {
    uint16_t* const out = mask + static_cast<int64_t>(j) * D;
    for (int d = lane * 8; d < D; d += 512) *reinterpret_cast<u32x4*>(out + d) = u32x4{0u, 0u, 0u, 0u};
  }
  if (lane != 0) return;
  const double l2 = lam * kLog2eD;
  const float hi2 = static_cast<float>(l2);
  R.lam2[j] = make_float2(hi2, static_cast<float>(l2 - static_cast<double>(hi2)));
  R.g[j] = g32;
  R.token[j] = tok;
  R.logp[j] = lp32;
  a.logp[m] = lp32;
  a.losses[m] = loss32;
  a.status[m] = status;
}

// The sum of w_n losses_n over the counted tokens, in double and a fixed order.
__device__ __forceinline__ void sum_losses(const DzTokens& t) {
  __shared__ double sh[kThreads / 64];
  double s = 0.0;
#pragma unroll 4
  for (int n = threadIdx.x; n < t.N; n += kThreads)
    if (t.status[n] == 0) s += static_cast<double>(t.losses[n]) * (t.weights ? static_cast<double>(t.weights[n]) : 1.0);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) *t.loss = ((sh[0] + sh[1]) + sh[2]) + sh[3];
}

// A token's own entry of dZ: g (1 - p), 1 - p = -expm1(lp).
__device__ __forceinline__ float own_entry(const DzTokens& t, int j) { return -expm1f(t.logp[j]) * t.g[j]; }

__device__ __forceinline__ float own_rest(const DzTokens& t, int j) {
  if (t.g[j] == 0.f) return 0.f;
  const float x = own_entry(t, j);
  return x - bf16_to_f32(f32_to_bf16(x));
}

// The tokens of 256 classes, a lane a class: the first kOwnMost of each in the order of their rows, with what the
// rounding took off their entries.  A wavefront stops after kOwnWave tokens of its 64 classes: where there
// are more the roundings average out, and a class may have them all.
constexpr int kOwnWave = 512;
__device__ __forceinline__ void list_tokens(const DzTokens& t, int M, int c0, int tile) {
  const int lane = threadIdx.x & 63;
  const int cls = tile * 256 + threadIdx.x, lo = c0 + cls - lane;  // of the chunk; this wavefront's first class
  OwnRest* const more = t.rest + static_cast<int64_t>(cls) * (kOwnMost - 1);
  OwnFirst first{0, 0, 0.f};
  int seen = 0;
  constexpr int kAhead = 8;
  for (int m0 = 0; m0 < M && seen < kOwnWave; m0 += 64 * kAhead) {
    int at[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) at[k] = m0 + 64 * k + lane < M ? t.token[m0 + 64 * k + lane] - lo : -1;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      uint64_t hits = __ballot(static_cast<unsigned>(at[k]) < 64u);
      for (; hits; hits &= hits - 1, ++seen) {
        const int b = __builtin_ctzll(hits);
        if (__builtin_amdgcn_readlane(at[k], b) == lane) {
          const int m = m0 + 64 * k + b;
          if (first.count == 0) first.row = m;
          else if (first.count < kOwnMost) more[first.count - 1].row = m;
          ++first.count;
        }
      }
    }
  }
  first.count = min(first.count, kOwnMost);
  if (first.count > 0) first.rest = own_rest(t, first.row);
  for (int e = 1; e < first.count; ++e) more[e - 1].rest = own_rest(t, more[e - 1].row);
  t.first[cls] = first;
}

// The tokens' own entries of a chunk.  Of a launch that sums the last workgroup does nothing else, and of one
// that lists them the ceil(cw / 256) before it.
template <bool BF>
__global__ void __launch_bounds__(kThreads)
dz_tokens(void* __restrict__ dZ, int pitch, int M, int c0, int cw, DzTokens t, float scale) {
  if (t.loss && blockIdx.x + 1 == gridDim.x) {
    sum_losses(t);
    return;
  }
  const int rows = (M + kThreads - 1) / kThreads;
  if (t.Mdev) M = min(M, *t.Mdev);
  if (static_cast<int>(blockIdx.x) >= rows) {
    if constexpr (BF) list_tokens(t, M, c0, blockIdx.x - rows);
    return;
  }
  const int m = blockIdx.x * kThreads + threadIdx.x;
  if (m >= M) return;
  if constexpr (BF)  // the columns that dH's 16-byte pieces hold past the last class (exp(-lambda) may be infinite)
    for (int v = cw; v < (cw + 7) / 8 * 8; ++v) static_cast<uint16_t*>(dZ)[static_cast<int64_t>(m) * pitch + v] = 0;
  const int v = t.token[m] - c0;
  const float g = t.g[m];
  if (v < 0 || v >= cw || g == 0.f) return;
  const float x = own_entry(t, m) * scale;
  const int64_t at = static_cast<int64_t>(m) * pitch + v;
  if constexpr (BF) static_cast<uint16_t*>(dZ)[at] = f32_to_bf16(x);
  else static_cast<float*>(dZ)[at] = x;
}

// db of a bf16 chunk: column sums of dZ, with what the rounding took off the own entries, over slices of the
// frames, then over the slices.  32 lanes of 8 columns and 8 frames at a time.
__global__ void __launch_bounds__(kThreads)
db_slices(const uint16_t* __restrict__ dZ, int M, int pitch, int mper, float* __restrict__ part, int c0, DzTokens t) {
  M = min(M, *t.Mdev);
  __shared__ float x[8][kThreads];
  const int col = (threadIdx.x & 31) * 8, row = threadIdx.x >> 5;
  const int v = blockIdx.x * 256 + col;  // the pitch is a multiple of 256
  const int mb = blockIdx.y * mper, me = min(M, mb + mper);
  float s[8] = {};
#pragma unroll 4
  for (int m = mb + row; m < me; m += 8) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(dZ + static_cast<int64_t>(m) * pitch + v);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s[2 * e] += __uint_as_float(w[e] << 16);
      s[2 * e + 1] += __uint_as_float(w[e] & 0xffff0000u);
    }
    const int own = t.token[m] - c0 - v;
    if (static_cast<unsigned>(own) < 8u) {
      const float r = own_rest(t, m);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] += e == own ? r : 0.f;
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) x[row][col + e] = s[e];
  __syncthreads();
  float total = 0.f;
#pragma unroll
  for (int r = 0; r < 8; ++r) total += x[r][threadIdx.x];
  part[static_cast<int64_t>(blockIdx.y) * pitch + blockIdx.x * 256 + threadIdx.x] = total;
}
__global__ void __launch_bounds__(kThreads)
db_join(const float* __restrict__ part, int slices, int pitch, int cw, uint16_t* __restrict__ db) {
  const int v = blockIdx.x * kThreads + threadIdx.x;
  if (v >= cw) return;
  float s = 0.f;
  for (int z = 0; z < slices; ++z) s += part[static_cast<int64_t>(z) * pitch + v];
  db[v] = f32_to_bf16(s);
}

// dH[m] = the split-K slices' sum of place inv[m], and what the rounding to bf16 took off the token's own entry
// times its row of W, rounded to bf16 (zeros for a row that is left out or has no gradient: 0 times a value of W that is
// not finite is none).  The own entry is the largest of
// its row of dZ by far: with its rounding in, the row's error is that of two roundings (0.0025 of dH's norm),
// without it of one (0.0017).  n values, a multiple of 4; the slices lie *t.Mdev D values apart.
__global__ void __launch_bounds__(kThreads)
dh_reduce_b16(const float* __restrict__ part, int splits, int64_t n, int D, const int32_t* __restrict__ inv, DzTokens t,
              const uint16_t* __restrict__ W, uint16_t* __restrict__ dH) {
  const int64_t i = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) * 4;
  if (i >= n) return;
  const int m = static_cast<int>(i / D), j = inv[m];
  if (j < 0 || t.g[j] == 0.f) {
    *reinterpret_cast<u32x2*>(dH + i) = u32x2{0u, 0u};
    return;
  }
  const int64_t step = static_cast<int64_t>(*t.Mdev) * D;
  const int64_t d = i - static_cast<int64_t>(m) * D;
  const float* at = part + static_cast<int64_t>(j) * D + d;
  float4 s = *reinterpret_cast<const float4*>(at);
#pragma unroll 4
  for (int k = 1; k < splits; ++k) {
    const float4 p = *reinterpret_cast<const float4*>(at + k * step);
    s.x += p.x;
    s.y += p.y;
    s.z += p.z;
    s.w += p.w;
  }
  const float x = own_entry(t, j), rest = x - bf16_to_f32(f32_to_bf16(x));
  const u32x2 w = *reinterpret_cast<const u32x2*>(W + static_cast<int64_t>(t.token[j]) * D + d);
  s.x = fmaf(rest, __uint_as_float(w[0] << 16), s.x);
  s.y = fmaf(rest, __uint_as_float(w[0] & 0xffff0000u), s.y);
  s.z = fmaf(rest, __uint_as_float(w[1] << 16), s.z);
  s.w = fmaf(rest, __uint_as_float(w[1] & 0xffff0000u), s.w);
  *reinterpret_cast<u32x2*>(dH + i) = u32x2{pack_bf16x2(s.x, s.y), pack_bf16x2(s.z, s.w)};
}

#define PCTC_POLICY_STAGES(G)                                            \
  __shared__ __attribute__((aligned(1024))) char st0[G::kStageBytes];    \
  __shared__ __attribute__((aligned(1024))) char st1[G::kStageBytes];    \
  __shared__ __attribute__((aligned(1024))) char st2[G::kStageBytes];    \
  __shared__ __attribute__((aligned(1024))) char st3[G::kStageBytes];    \
  char* const st[4] = {st0, st1, st2, st3};

// A chunk's share of dH by slices of `slice` of its columns: part[slice][frame][D], written by the first chunk (add
// false), added to by the others.  Tiles of 256 values of a row x 256 frames, which leave in lines: 331 frames, D =
// 512, 5,000 columns 18 us, where the fused call's kernel, whose tiles lie the other way and leave by single values,
// takes 31; large products are the same (1,925 frames, D = 4,096, 50,688 columns 636 and 641).
__global__ void __launch_bounds__(512, 1)
policy_dh(const uint16_t* __restrict__ dZ, int pitch, int M, const uint16_t* __restrict__ W, int D, int cw, int slice,
          bool add, float* __restrict__ part, const int32_t* __restrict__ Mdev) {
  using G = bf::Gemm<256, 256, 32, bf::LL::MC, bf::LL::KC, 4, 2, 4, true>;
  PCTC_POLICY_STAGES(G)
  M = min(M, *Mdev);
  const int nM = (M + 255) / 256, nD = (D + 255) / 256;
  const int works = nM * nD * gridDim.y;
  const int id = blockIdx.y * gridDim.x + blockIdx.x;
  if (id >= works) return;
  const int w = xcd_swz(id, works);
  const int s = w / (nM * nD), rest = w % (nM * nD);
  const int d0 = (nD <= nM ? rest % nD : rest / nM) * 256, m0 = (nD <= nM ? rest / nD : rest % nM) * 256;
  const int kb = s * slice, ke = min(cw, kb + slice);
  if (add && kb >= ke) return;
  const bf::GOp A{W, D, D, cw, nullptr}, B{dZ, pitch, M, cw, nullptr};
  f32x16 acc[G::FR][G::FC];
  G::run_pp(A, B, d0, m0, kb, ke, st, acc);
  const int wave = threadIdx.x >> 6;
  const int dw = d0 + wave / 4 * 128, mw = m0 + wave % 4 * 64;
  float* const out = part + static_cast<int64_t>(s) * M * D;
  struct __attribute__((aligned(16))) Eight {
    float4 a, b;
  };
  auto place = [&](int block, int col) {
    const int d = dw + block * 8, m = mw + col;
    return d < D && m < M ? static_cast<int64_t>(m) * D + d : int64_t{-1};
  };
  by_columns<G, Eight>(
      acc, st,
      [&](int block, int col, const float (&v)[8], const Eight& x) {
        const int64_t at = place(block, col);
        if (at < 0) return;
        float4* const o = reinterpret_cast<float4*>(out + at);
        o[0] = make_float4(v[0] + x.a.x, v[1] + x.a.y, v[2] + x.a.z, v[3] + x.a.w);
        o[1] = make_float4(v[4] + x.b.x, v[5] + x.b.y, v[6] + x.b.z, v[7] + x.b.w);
      },
      [&](int block, int col, Eight& x) {
        const int64_t at = place(block, col);
        x = Eight{make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
        if (add)  // (places outside read the first: no branch between the reads)
          x = *reinterpret_cast<const Eight*>(out + (at < 0 ? 0 : at));
      });
}

// dW of a bf16 chunk: tiles of 256 values of a row x 256 classes, so that the accumulators leave in lines, each
// class with what the rounding took off its tokens' own entries times their rows of H, before its one rounding
// to bf16 (0.0023 -> 0.0017 of dW's norm; of few rows one rounding may be most of the error: 40 rows of 100
// classes, up to 0.0034).
__global__ void __launch_bounds__(512, 1)
policy_dw(const uint16_t* __restrict__ dZ, int pitch, int M, const uint16_t* __restrict__ H, int D, int c0, int cw,
          uint16_t* __restrict__ dW, DzTokens t) {
  using G = bf::Gemm<256, 256, 32, bf::LL::MC, bf::LL::MC, 4, 2, 4, true>;
  PCTC_POLICY_STAGES(G)
  M = min(M, *t.Mdev);  // (with none, zeros are written)
  const int nDt = (D + 255) / 256;
  const int w = xcd_swz(blockIdx.x, gridDim.x);
  const int d0 = w % nDt * 256, v0 = w / nDt * 256;
  const bf::GOp A{H, D, D, M, nullptr}, B{dZ, pitch, cw, M, nullptr};
  f32x16 acc[G::FR][G::FC];
  G::run_pp(A, B, d0, v0, 0, M, st, acc);
  const int wave = threadIdx.x >> 6;
  const int dw = d0 + wave / 4 * 128, vw = v0 + wave % 4 * 64;
  by_columns<G, OwnFirst>(
      acc, st,
      [&](int block, int col, float (&s)[8], const OwnFirst& own) {
        const int d = dw + block * 8, v = vw + col;
        if (v >= cw || d >= D) return;
        auto add = [&](int row, float rest) {
          const u32x4 h = *reinterpret_cast<const u32x4*>(H + static_cast<int64_t>(row) * D + d);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s[2 * e] = fmaf(rest, __uint_as_float(h[e] << 16), s[2 * e]);
            s[2 * e + 1] = fmaf(rest, __uint_as_float(h[e] & 0xffff0000u), s[2 * e + 1]);
          }
        };
        if (own.count > 0) add(own.row, own.rest);
        const OwnRest* const more = t.rest + static_cast<int64_t>(v) * (kOwnMost - 1);
#pragma unroll 4
        for (int e = 1; e < own.count; ++e) add(more[e - 1].row, more[e - 1].rest);
        *reinterpret_cast<u32x4*>(dW + static_cast<int64_t>(c0 + v) * D + d) =
            u32x4{pack_bf16x2(s[0], s[1]), pack_bf16x2(s[2], s[3]), pack_bf16x2(s[4], s[5]), pack_bf16x2(s[6], s[7])};
      },
      [&](int, int col, OwnFirst& own) { own = t.first[vw + col]; });
}

constexpr int kDbSlices = 16;

}  // namespace

hipError_t launch_dz_tokens(int dtype, void* dZ, int pitch, int M, int c0, int cw, const DzTokens& tokens, float scale,
                            hipStream_t stream) {
  Prof pr("dz_tokens", stream);
  DzTokens t = tokens;
  if (c0 > 0) t.loss = nullptr;
  const dim3 grid((M + kThreads - 1) / kThreads + (t.first ? (cw + 255) / 256 : 0) + (t.loss ? 1 : 0));
  if (dtype == 1) hipLaunchKernelGGL(dz_tokens<true>, grid, dim3(kThreads), 0, stream, dZ, pitch, M, c0, cw, t, scale);
  else hipLaunchKernelGGL(dz_tokens<false>, grid, dim3(kThreads), 0, stream, dZ, pitch, M, c0, cw, t, scale);
  return hipGetLastError();
}

PolicyLayout policy_layout(int dtype, int M, int D, int V, bool bias, bool grads, int chunk) {
  PolicyLayout L{};
  const size_t m = M > 0 ? M : 1;
  L.bwd = plan_bwd(dtype, M, D, V, chunk);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += align_up(bytes, 256);
    return o;
  };
  L.o_lam2 = take(m * sizeof(float2));
  L.o_g = take(m * sizeof(float));
  L.o_tok = take(m * sizeof(int32_t));
  L.o_lp = take(m * sizeof(float));
  if (dtype == 1) {
    L.o_rows = take(m * sizeof(int32_t));
    L.o_inv = take(m * sizeof(int32_t));
    L.o_count = take((m / kCountRows + 2) * sizeof(int32_t));
    L.o_h = take(m * D * sizeof(uint16_t));
  }
  const size_t fwd = at;
  L.o_part = take(lse_partial_bytes(M, D));
  L.ht = dtype == 1 && (bias ? bias_reads_ht_bf16(M, D) : frames_from_ht_bf16(M, D, V));
  L.o_ht = take(L.ht ? lse_ht_bytes_bf16(M, D) : 0);
  if (grads) {
    // the backward's room is that of the normaliser, which is done
    const size_t end = at;
    at = fwd;
    // one slice of the dH product has no room of its own in the plan
    L.o_dh = take(dtype == 1 && L.bwd.part_bytes == 0 ? m * D * sizeof(float) : 0);
    L.o_own = take(dtype == 1 ? L.bwd.chunk * (sizeof(OwnFirst) + (kOwnMost - 1) * sizeof(OwnRest)) : 0);
    L.o_bwd = take(L.bwd.total);
    at = at > end ? at : end;
  }
  L.total = at;
  return L;
}

// Hc: the counted rows, those without a gradient cleared; tokens.Mdev of them.
static hipError_t policy_bwd_bf16(uint16_t* Hc, int M, int D, const uint16_t* W, const float* bias, int V,
                                  const float2* lam2, const DzTokens& tokens, const int32_t* inv, uint16_t* dH,
                                  uint16_t* dW, uint16_t* db, char* scratch, const BwdPlan& plan, float* one,
                                  hipStream_t stream) {
  uint16_t* dZ = reinterpret_cast<uint16_t*>(scratch);
  // the recompute reads the frames transposed where that pays for its launch (with a bias it never does)
  uint16_t* Hst = !bias && frames_from_ht_bf16(M, D, V) ? bwd_hst(scratch, plan) : nullptr;
  float* part = one ? one : reinterpret_cast<float*>(scratch + plan.dz_bytes + plan.ht_bytes);
  float* dbpart = reinterpret_cast<float*>(scratch + plan.dz_bytes + plan.ht_bytes + plan.part_bytes + plan.lam2_bytes);
  const int chunk = plan.chunk;
  hipError_t e;
  // (rows behind the last counted one hold anything; their columns of the transpose reach no result)
  if (Hst && (e = launch_ht_build_bf16(Hc, M, D, nullptr, nullptr, Hst, plan.Mp, stream)) != hipSuccess) return e;
  // slices of the dH product as in the Pruned CTC backward
  const int slice = (chunk / plan.splits + 63) / 64 * 64;
  const int nslices = ((chunk < V ? chunk : V) + slice - 1) / slice;
  for (int c0 = 0; c0 < V; c0 += chunk) {
    const int cw = V - c0 < chunk ? V - c0 : chunk;
    int sl = slice;
    if (c0 > 0) {
      sl = ((cw + nslices - 1) / nslices + 63) / 64 * 64;
      if (sl < 64) sl = 64;
    }
    e = launch_bwd_chunk_bf16(Hc, M, D, W, bias, c0, cw, lam2, nullptr, 0, tokens.g, nullptr, nullptr, 0, dZ, chunk, part,
                              sl, true, false, false, nullptr, nullptr, nullptr, stream, nullptr, nullptr, Hst, plan.Mp,
                              tokens.Mdev);
    if (e != hipSuccess) return e;
    if ((e = launch_dz_tokens(1, dZ, chunk, M, c0, cw, tokens, 1.f, stream)) != hipSuccess) return e;
    if (db) {
      Prof pr("db_colsum", stream);
      const int most = (M + 127) / 128 < kDbSlices ? (M + 127) / 128 : kDbSlices;  // (dbpart has a row per 128 frames)
      const int mper = ((M + most - 1) / most + 7) / 8 * 8, slices = (M + mper - 1) / mper, tiles = (cw + 255) / 256;
      hipLaunchKernelGGL(db_slices, dim3(tiles, slices), dim3(kThreads), 0, stream, dZ, M, chunk, mper, dbpart, c0,
                         tokens);
      hipLaunchKernelGGL(db_join, dim3(tiles), dim3(kThreads), 0, stream, dbpart, slices, chunk, cw, db + c0);
    }
    if (dH) {
      Prof pr("dh_gemm", stream);
      const dim3 grid((M + 255) / 256 * ((D + 255) / 256), (cw + sl - 1) / sl);
      hipLaunchKernelGGL(policy_dh, grid, dim3(512), 0, stream, dZ, chunk, M, W + static_cast<int64_t>(c0) * D, D, cw, sl,
                         c0 > 0, part, tokens.Mdev);
    }
    if (dW) {
      Prof pr("dw_gemm", stream);
      const dim3 grid((cw + 255) / 256 * ((D + 255) / 256));
      hipLaunchKernelGGL(policy_dw, grid, dim3(512), 0, stream, dZ, chunk, M, Hc, D, c0, cw, dW, tokens);
    }
  }
  if (dH) {
    const int64_t n = static_cast<int64_t>(M) * D;
    Prof pr("dh_reduce", stream);
    hipLaunchKernelGGL(dh_reduce_b16, dim3(static_cast<unsigned>((n / 4 + kThreads - 1) / kThreads)), dim3(kThreads), 0,
                       stream, part, one ? 1 : nslices, n, D, inv, tokens, W, dH);
  }
  return hipGetLastError();
}

hipError_t launch_policy_loss(int dtype, const void* H, int M, int D, const void* W, const float* bias, int V,
                              const PolicyArgs& a, void* dH, void* dW, void* db, char* ws, const PolicyLayout& L,
                              hipStream_t stream) {
  hipError_t e;
  const int64_t es = dtype == 1 ? 2 : 4;
  if (M == 0) {
    if ((e = launch_clear(a.loss, sizeof(double), stream)) != hipSuccess) return e;
    if (dW && (e = launch_clear(dW, es * V * D, stream)) != hipSuccess) return e;
    return db ? launch_clear(db, es * V, stream) : hipSuccess;
  }
  const bool grads = dH || dW || db;
  auto i32 = [&](size_t o) { return reinterpret_cast<int32_t*>(ws + o); };
  auto f32 = [&](size_t o) { return reinterpret_cast<float*>(ws + o); };
  float2* partials = reinterpret_cast<float2*>(ws + L.o_part);
  float2* lam2 = reinterpret_cast<float2*>(ws + L.o_lam2);
  PolicyRows R{nullptr, nullptr, partials, 0, lam2, f32(L.o_g), i32(L.o_tok), f32(L.o_lp)};
  const dim3 grid((M + kLossThreads / 64 - 1) / (kLossThreads / 64));
  DzTokens tokens{R.token, R.logp, R.g};
  tokens.losses = a.losses;
  tokens.weights = a.weights;
  tokens.status = a.status;
  tokens.N = M;
  tokens.loss = a.loss;
  if (dtype == 1) {
    uint16_t* Hc = reinterpret_cast<uint16_t*>(ws + L.o_h);
    const uint16_t* Wb = static_cast<const uint16_t*>(W);
    int32_t *const count = i32(L.o_count), *const counts = count + 1;
    const bool many = M > 4 * kCountRows;
    {
      Prof pr("policy_gather", stream);
      if (many)
        hipLaunchKernelGGL(policy_count, dim3((M + kCountRows - 1) / kCountRows), dim3(kThreads), 0, stream, a.tokens, M,
                           V, counts);
      hipLaunchKernelGGL(policy_gather, dim3((M + kGatherRows - 1) / kGatherRows), dim3(kThreads), 0, stream,
                         static_cast<const uint16_t*>(H), M, D, V, a, many ? counts : nullptr, Hc, i32(L.o_rows),
                         i32(L.o_inv), count);
    }
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (L.ht) {
      uint16_t* Ht = reinterpret_cast<uint16_t*>(ws + L.o_ht);
      const int Mp = (M + 63) / 64 * 64;
      if ((e = launch_ht_build_bf16(Hc, M, D, nullptr, nullptr, Ht, Mp, stream)) != hipSuccess) return e;
      e = launch_lse_partial_e_bf16(Hc, M, D, Wb, bias, V, partials, &R.P, nullptr, 0, 0, nullptr, stream, Ht, Mp, false,
                                    count);
    } else {
      e = launch_lse_partial_bf16(Hc, M, D, Wb, bias, V, partials, &R.P, stream, false, count);
    }
    if (e != hipSuccess) return e;
    R.rows = i32(L.o_rows);
    R.count = tokens.Mdev = count;
    {
      Prof pr("policy_tokens", stream);
      hipLaunchKernelGGL(policy_tokens<true>, grid, dim3(kLossThreads), 0, stream, Hc, M, D, W, bias, V, R, a,
                         grads ? Hc : nullptr);
    }
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (dW) {
      tokens.first = reinterpret_cast<OwnFirst*>(ws + L.o_own);
      tokens.rest = reinterpret_cast<OwnRest*>(tokens.first + L.bwd.chunk);
    }
    if (grads)
      return policy_bwd_bf16(Hc, M, D, Wb, bias, V, lam2, tokens, i32(L.o_inv), static_cast<uint16_t*>(dH),
                             static_cast<uint16_t*>(dW), static_cast<uint16_t*>(db), ws + L.o_bwd, L.bwd,
                             L.bwd.part_bytes == 0 ? f32(L.o_dh) : nullptr, stream);
  } else {
    if ((e = launch_lse_partials(0, H, M, D, W, bias, V, partials, &R.P, stream)) != hipSuccess) return e;
    {
      Prof pr("policy_tokens", stream);
      hipLaunchKernelGGL(policy_tokens<false>, grid, dim3(kLossThreads), 0, stream, H, M, D, W, bias, V, R, a, nullptr);
    }
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (grads)
      return head_bwd_f32(static_cast<const float*>(H), M, D, static_cast<const float*>(W), bias, V, lam2, nullptr, 0,
                          R.g, nullptr, static_cast<float*>(dH), static_cast<float*>(dW), static_cast<float*>(db),
                          ws + L.o_bwd, L.bwd, stream, &tokens);
  }
  // no chunk to sum beside
  return launch_dz_tokens(dtype, nullptr, 0, 0, 0, 0, tokens, 1.f, stream);
}

}  // namespace pctc
