// Clipped policy loss with a KL term on the tokens of a vocabulary head (gfx950).
//
//   lp_m = z_m[token_m] - lambda_m (z = H W^T + b, lambda over the full vocabulary),  r = exp(lp - old)
//   loss_m = -min(r A, clip(r, 1 - lo, 1 + hi) A) + kl (exp(ref - lp) - (ref - lp) - 1)
//   g_m = w_m dloss_m / dlp_m,   dZ[m] = g_m (onehot(token_m) - p(m)),   dH = dZ W,  dW = dZ^T H
//
// The logits are not stored: the normaliser and the recomputed backward are those of the Pruned CTC
// loss, whose union columns here are one class per frame.  Three small kernels come between: the tokens'
// logits and losses (a wavefront a token; two rows of D values each), the loss, and in every chunk of
// the backward the tokens' own entries of dZ.  Bound by the matrix products, 8 M V D operations
// (the logits are formed twice).
#include "pctc_internal.h"

namespace pctc {

namespace {

constexpr int kThreads = 256;
constexpr int kLossThreads = 1024;

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

// A wavefront a token: its logit (lanes' float sums joined in double), then the loss in double.
template <bool BF>
__global__ void __launch_bounds__(kThreads)
policy_tokens(const void* __restrict__ H, int M, int D, const void* __restrict__ W, const float* __restrict__ bias, int V,
              const double* __restrict__ lam, PolicyArgs a, float* __restrict__ g) {
  const int m = blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (m >= M) return;
  const int tok = a.tokens[m];
  const bool counted = tok >= 0 && tok < V;
  double z = 0.0;
  if (counted) {
    constexpr int kBytes = BF ? 2 : 4;
    z = dot_share<BF>(static_cast<const char*>(H) + static_cast<int64_t>(m) * D * kBytes,
                      static_cast<const char*>(W) + static_cast<int64_t>(tok) * D * kBytes, D, lane);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) z += __shfl_xor(z, o, 64);
  }
  if (lane != 0) return;
  float lp32 = 0.f, loss32 = 0.f, g32 = 0.f;
  int status = 1;  // left out
  if (counted) {
    if (bias) z += static_cast<double>(bias[tok]);
    const double lp = z - lam[m];
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
    if (a.ref_logp) {
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
  a.logp[m] = lp32;
  a.losses[m] = loss32;
  a.status[m] = status;
  g[m] = g32;
}

// loss = sum of w_m loss_m over the counted tokens, in double and a fixed order.
__global__ void __launch_bounds__(kLossThreads)
policy_sum(const float* __restrict__ losses, const float* __restrict__ weights, const int32_t* __restrict__ status,
           int M, double* __restrict__ loss) {
  __shared__ double sh[kLossThreads / 64];
  double s = 0.0;
#pragma unroll 4
  for (int m = threadIdx.x; m < M; m += kLossThreads)
    if (status[m] == 0) s += static_cast<double>(losses[m]) * (weights ? static_cast<double>(weights[m]) : 1.0);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    double t = 0.0;
    for (int w = 0; w < kLossThreads / 64; ++w) t += sh[w];
    *loss = t;
  }
}

// The tokens' own entries of a chunk: g (1 - p), 1 - p = -expm1(lp).
template <bool BF>
__global__ void __launch_bounds__(kThreads)
dz_tokens(void* __restrict__ dZ, int pitch, int M, int c0, int cw, DzTokens t, float scale) {
  const int m = blockIdx.x * kThreads + threadIdx.x;
  if (m >= M) return;
  const int v = t.token[m] - c0;
  const float g = t.g[m];
  if (v < 0 || v >= cw || g == 0.f) return;
  const float x = -expm1f(t.logp[m]) * g * scale;
  const int64_t at = static_cast<int64_t>(m) * pitch + v;
  if constexpr (BF) static_cast<uint16_t*>(dZ)[at] = f32_to_bf16(x);
  else static_cast<float*>(dZ)[at] = x;
}

// db of a bf16 chunk: column sums of dZ over slices of the frames, then over the slices.  32 lanes of 8
// columns and 8 frames at a time.
__global__ void __launch_bounds__(kThreads)
db_slices(const uint16_t* __restrict__ dZ, int M, int pitch, int mper, float* __restrict__ part) {
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
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) x[row][col + e] = s[e];
  __syncthreads();
  float t = 0.f;
#pragma unroll
  for (int r = 0; r < 8; ++r) t += x[r][threadIdx.x];
  part[static_cast<int64_t>(blockIdx.y) * pitch + blockIdx.x * 256 + threadIdx.x] = t;
}
__global__ void __launch_bounds__(kThreads)
db_join(const float* __restrict__ part, int slices, int pitch, int cw, uint16_t* __restrict__ db) {
  const int v = blockIdx.x * kThreads + threadIdx.x;
  if (v >= cw) return;
  float s = 0.f;
  for (int z = 0; z < slices; ++z) s += part[static_cast<int64_t>(z) * pitch + v];
  db[v] = f32_to_bf16(s);
}

// dH = the split-K slices' sum, rounded to bf16; n a multiple of 8.
__global__ void __launch_bounds__(kThreads)
dh_reduce_b16(const float* __restrict__ part, int splits, int64_t n, uint16_t* __restrict__ dH) {
  const int64_t i = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) * 4;
  if (i >= n) return;
  float4 s = *reinterpret_cast<const float4*>(part + i);
  for (int k = 1; k < splits; ++k) {
    const float4 p = *reinterpret_cast<const float4*>(part + k * n + i);
    s.x += p.x;
    s.y += p.y;
    s.z += p.z;
    s.w += p.w;
  }
  *reinterpret_cast<u32x2*>(dH + i) = u32x2{pack_bf16x2(s.x, s.y), pack_bf16x2(s.z, s.w)};
}

constexpr int kDbSlices = 16;

}  // namespace

hipError_t launch_dz_tokens(int dtype, void* dZ, int pitch, int M, int c0, int cw, const DzTokens& t, float scale,
                            hipStream_t stream) {
  Prof pr("dz_tokens", stream);
  const dim3 grid((M + kThreads - 1) / kThreads);
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
  L.o_lam = take(m * sizeof(double));
  L.o_lam2 = take(m * sizeof(float2));
  L.o_g = take(m * sizeof(float));
  const size_t fwd = at;
  L.o_part = take(lse_partial_bytes(M, D));
  const bool ht = dtype == 1 && (bias ? bias_reads_ht_bf16(M, D) : frames_from_ht_bf16(M, D, V));
  L.o_ht = take(ht ? lse_ht_bytes_bf16(M, D) : 0);
  if (!ht) L.o_ht = 0;
  if (grads) {
    // the backward's room is that of the normaliser, which is done
    const size_t end = at;
    at = fwd;
    // one slice of the dH product has no room of its own in the plan
    L.o_dh = take(dtype == 1 && L.bwd.part_bytes == 0 ? m * D * sizeof(float) : 0);
    L.o_bwd = take(L.bwd.total);
    at = at > end ? at : end;
  }
  L.total = at;
  return L;
}

static hipError_t policy_bwd_bf16(const uint16_t* H, int M, int D, const uint16_t* W, const float* bias, int V,
                                  const float2* lam2, const DzTokens& tokens, uint16_t* dH, uint16_t* dW, uint16_t* db,
                                  char* scratch, const BwdPlan& plan, float* one, hipStream_t stream) {
  uint16_t* dZ = reinterpret_cast<uint16_t*>(scratch);
  uint16_t* Hs = bwd_hs(scratch, plan);
  uint16_t* Hst = bwd_hst(scratch, plan);
  float* part = one ? one : reinterpret_cast<float*>(scratch + plan.dz_bytes + plan.ht_bytes);
  float* dbpart = reinterpret_cast<float*>(scratch + plan.dz_bytes + plan.ht_bytes + plan.part_bytes + plan.lam2_bytes);
  const int chunk = plan.chunk;
  hipError_t e = Hst ? launch_ht_build_bf16(H, M, D, tokens.g, Hs, Hst, plan.Mp, stream)
                     : launch_hs_build_bf16(H, M, D, tokens.g, Hs, stream);
  if (e != hipSuccess) return e;
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
    e = launch_bwd_chunk_bf16(Hs, M, D, W, bias, c0, cw, lam2, nullptr, 0, tokens.g, nullptr, nullptr, 0, dZ, chunk, part,
                              sl, true, false, false, nullptr, nullptr, nullptr, stream, nullptr, nullptr, Hst, plan.Mp);
    if (e != hipSuccess) return e;
    if ((e = launch_dz_tokens(1, dZ, chunk, M, c0, cw, tokens, 1.f, stream)) != hipSuccess) return e;
    if (db) {
      Prof pr("db_colsum", stream);
      const int most = (M + 127) / 128 < kDbSlices ? (M + 127) / 128 : kDbSlices;  // (dbpart has a row per 128 frames)
      const int mper = ((M + most - 1) / most + 7) / 8 * 8, slices = (M + mper - 1) / mper, tiles = (cw + 255) / 256;
      hipLaunchKernelGGL(db_slices, dim3(tiles, slices), dim3(kThreads), 0, stream, dZ, M, chunk, mper, dbpart);
      hipLaunchKernelGGL(db_join, dim3(tiles), dim3(kThreads), 0, stream, dbpart, slices, chunk, cw, db + c0);
    }
    e = launch_bwd_chunk_bf16(Hs, M, D, W, bias, c0, cw, lam2, nullptr, 0, tokens.g, nullptr, nullptr, 0, dZ, chunk, part,
                              sl, false, dH != nullptr, dW != nullptr, nullptr, nullptr, nullptr, stream, nullptr, nullptr,
                              Hst, plan.Mp, dW);
    if (e != hipSuccess) return e;
  }
  if (dH) {
    const int64_t n = static_cast<int64_t>(M) * D;
    Prof pr("dh_reduce", stream);
    hipLaunchKernelGGL(dh_reduce_b16, dim3(static_cast<unsigned>((n / 4 + kThreads - 1) / kThreads)), dim3(kThreads), 0,
                       stream, part, one ? 1 : nslices, n, dH);
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
  double* lam = reinterpret_cast<double*>(ws + L.o_lam);
  float2* lam2 = reinterpret_cast<float2*>(ws + L.o_lam2);
  float* g = reinterpret_cast<float*>(ws + L.o_g);
  e = launch_lse(dtype, H, M, D, W, bias, V, reinterpret_cast<float2*>(ws + L.o_part), lam, lam2, stream,
                 L.o_ht ? reinterpret_cast<uint16_t*>(ws + L.o_ht) : nullptr);
  if (e != hipSuccess) return e;
  {
    Prof pr("policy_tokens", stream);
    const dim3 grid((M + kThreads / 64 - 1) / (kThreads / 64));
    if (dtype == 1)
      hipLaunchKernelGGL(policy_tokens<true>, grid, dim3(kThreads), 0, stream, H, M, D, W, bias, V, lam, a, g);
    else hipLaunchKernelGGL(policy_tokens<false>, grid, dim3(kThreads), 0, stream, H, M, D, W, bias, V, lam, a, g);
    hipLaunchKernelGGL(policy_sum, dim3(1), dim3(kLossThreads), 0, stream, a.losses, a.weights, a.status, M, a.loss);
  }
  if ((e = hipGetLastError()) != hipSuccess || (!dH && !dW && !db)) return e;
  const DzTokens tokens{a.tokens, a.logp, g};
  if (dtype == 1)
    return policy_bwd_bf16(static_cast<const uint16_t*>(H), M, D, static_cast<const uint16_t*>(W), bias, V, lam2, tokens,
                           static_cast<uint16_t*>(dH), static_cast<uint16_t*>(dW), static_cast<uint16_t*>(db), ws + L.o_bwd,
                           L.bwd, L.bwd.part_bytes == 0 ? reinterpret_cast<float*>(ws + L.o_dh) : nullptr, stream);
  return head_bwd_f32(static_cast<const float*>(H), M, D, static_cast<const float*>(W), bias, V, lam2, nullptr, 0, g,
                      nullptr, static_cast<float*>(dH), static_cast<float*>(dW), static_cast<float*>(db), ws + L.o_bwd,
                      L.bwd, stream, &tokens);
}

}  // namespace pctc
