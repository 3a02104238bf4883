// Global gradient norm over a list of tensors, and clipping (gfx950).
//
//   n = sqrt(sum over all values g^2),  s = min(1, max_norm / (n + 1e-6)),  g <- s g
//
// Squares are taken and summed in double: no square of a finite value overflows, and the order of
// the sums, fixed by the sizes alone, moves the float result by at most its last bit.  Bound by
// memory: the values are read twice (the scale is known only after the last of them) and written
// once.  Two launches per group of tensors: the partial sums of a fixed grid, then the scaling,
// each workgroup of which first adds the partial sums up itself (at most 16 KB, read from L2) so
// that no third launch stands between the two.
#include <algorithm>
#include <type_traits>

#include "pctc_internal.h"

namespace pctc {

namespace {

constexpr int kThreads = 256;
constexpr int kVec = 8;                             // 16-byte pieces a thread has in flight
constexpr int kChunkBytes = kThreads * kVec * 16;   // one workgroup's step
constexpr int kGroup = 96;                          // tensors of a launch: their table is a kernel argument
constexpr int kMaxParts = 2048;                     // workgroups (8 a compute unit) that share the sums

struct ClipTable {
  const void* in[kGroup];
  void* out[kGroup];
  int64_t n[kGroup];         // values
  int32_t first[kGroup + 1]; // chunks of the tensors before
  uint32_t bf16[(kGroup + 31) / 32];
  int32_t tensors;
};
static_assert(sizeof(ClipTable) <= 3600, "kernel arguments");

// 16 bytes at any alignment of its own values (views into flat buffers start where the tensors
// before them end); unaligned vector accesses are ordinary ones on this target.
struct __attribute__((packed, aligned(2))) Piece {
  uint32_t w[4];
};

__device__ __forceinline__ int find_tensor(const ClipTable& t, int chunk) {
  int lo = 0, hi = t.tensors - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.first[mid] <= chunk) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ double block_sum(double x, double* sh) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor(x, o, 64);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) s += sh[w];
  return s;
}

template <bool BF>
__device__ __forceinline__ void add_squares(const Piece& p, double& a, double& b) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if constexpr (BF) {
      const double x = __uint_as_float(p.w[q] << 16), y = __uint_as_float(p.w[q] & 0xffff0000u);
      a = fma(x, x, a);
      b = fma(y, y, b);
    } else {
      const double x = __uint_as_float(p.w[q]);
      if (q & 1) b = fma(x, x, b);
      else a = fma(x, x, a);
    }
  }
}

// Sum of squares of this workgroup's chunk of a tensor.
template <bool BF>
__device__ __forceinline__ void chunk_squares(const void* base, int64_t n, int64_t first, double& a, double& b) {
  constexpr int kPer = BF ? 8 : 4;                       // values of a piece
  constexpr int kValues = kChunkBytes / (BF ? 2 : 4);
  using T = std::conditional_t<BF, uint16_t, float>;
  const T* p = static_cast<const T*>(base) + first;
  const int64_t left = n - first;
  if (left >= kValues) {
    Piece v[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = *reinterpret_cast<const Piece*>(p + (i * kThreads + threadIdx.x) * kPer);
#pragma unroll
    for (int i = 0; i < kVec; ++i) add_squares<BF>(v[i], a, b);
    return;
  }
  for (int64_t at = static_cast<int64_t>(threadIdx.x) * kPer; at < left; at += kThreads * kPer) {
    if (at + kPer <= left) {
      add_squares<BF>(*reinterpret_cast<const Piece*>(p + at), a, b);
    } else {
      for (int64_t e = at; e < left; ++e) {
        const double x = BF ? bf16_to_f32(static_cast<uint16_t>(p[e])) : static_cast<float>(p[e]);
        a = fma(x, x, a);
      }
    }
  }
}

// S float, or double for scales below float's normal range (norms of 1e38 times the bound).
template <bool BF, class S>
__device__ __forceinline__ void chunk_scale(const void* in, void* out, int64_t n, int64_t first, S s) {
  constexpr int kPer = BF ? 8 : 4;
  constexpr int kValues = kChunkBytes / (BF ? 2 : 4);
  using T = std::conditional_t<BF, uint16_t, float>;
  const T* p = static_cast<const T*>(in) + first;
  T* o = static_cast<T*>(out) + first;
  auto times = [&](float x) { return static_cast<float>(x * s); };
  auto scaled = [&](const Piece& v) {
    Piece r;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if constexpr (BF)
        r.w[q] = pack_bf16x2(times(__uint_as_float(v.w[q] << 16)), times(__uint_as_float(v.w[q] & 0xffff0000u)));
      else
        r.w[q] = __float_as_uint(times(__uint_as_float(v.w[q])));
    }
    return r;
  };
  const int64_t left = n - first;
  if (left >= kValues) {
    Piece v[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = *reinterpret_cast<const Piece*>(p + (i * kThreads + threadIdx.x) * kPer);
#pragma unroll
    for (int i = 0; i < kVec; ++i) *reinterpret_cast<Piece*>(o + (i * kThreads + threadIdx.x) * kPer) = scaled(v[i]);
    return;
  }
  for (int64_t at = static_cast<int64_t>(threadIdx.x) * kPer; at < left; at += kThreads * kPer) {
    if (at + kPer <= left) {
      *reinterpret_cast<Piece*>(o + at) = scaled(*reinterpret_cast<const Piece*>(p + at));
    } else {
      for (int64_t e = at; e < left; ++e) {
        if constexpr (BF) o[e] = f32_to_bf16(times(bf16_to_f32(p[e])));
        else o[e] = times(p[e]);
      }
    }
  }
}

__global__ void __launch_bounds__(kThreads) grad_squares(ClipTable t, double* __restrict__ parts) {
  __shared__ double sh[kThreads / 64];
  double a = 0.0, b = 0.0;
  const int chunks = t.first[t.tensors];
  for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
    const int k = find_tensor(t, c);
    const int64_t step = c - t.first[k];
    if ((t.bf16[k >> 5] >> (k & 31)) & 1) chunk_squares<true>(t.in[k], t.n[k], step * (kChunkBytes / 2), a, b);
    else chunk_squares<false>(t.in[k], t.n[k], step * (kChunkBytes / 4), a, b);
  }
  const double s = block_sum(a + b, sh);
  if (threadIdx.x == 0) parts[blockIdx.x] = s;
}

// The norm and the scale from the partial sums, then this workgroup's chunks of the tensors.  The
// first workgroup of the first launch (norm not null) writes both out.
__global__ void __launch_bounds__(kThreads)
grad_scale(ClipTable t, const double* __restrict__ parts, int nparts, float max_norm, bool in_place,
           float* __restrict__ norm, float* __restrict__ scale) {
  __shared__ double sh[kThreads / 64];
  double x = 0.0;
  for (int i = threadIdx.x; i < nparts; i += kThreads) x += parts[i];
  const double n = sqrt(block_sum(x, sh));
  // a norm that is not finite clips nothing: the caller sees it in the norm and drops the step
  double sd = 1.0;
  if (n <= 1.7976931348623157e308) sd = fmin(1.0, static_cast<double>(max_norm) / (n + 1e-6));
  const float s = static_cast<float>(sd);
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) {
    *norm = static_cast<float>(n);
    if (scale) *scale = s;
  }
  if (in_place && s == 1.f) return;
  const int chunks = t.first[t.tensors];
  for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
    const int k = find_tensor(t, c);
    const int64_t step = c - t.first[k];
    const bool bf = (t.bf16[k >> 5] >> (k & 31)) & 1, tiny = sd > 0.0 && s < 1.17549435e-38f;
    if (tiny && bf) chunk_scale<true>(t.in[k], t.out[k], t.n[k], step * (kChunkBytes / 2), sd);
    else if (tiny) chunk_scale<false>(t.in[k], t.out[k], t.n[k], step * (kChunkBytes / 4), sd);
    else if (bf) chunk_scale<true>(t.in[k], t.out[k], t.n[k], step * (kChunkBytes / 2), s);
    else chunk_scale<false>(t.in[k], t.out[k], t.n[k], step * (kChunkBytes / 4), s);
  }
}

int64_t chunks_of(int64_t n, int dtype) {
  const int64_t per = kChunkBytes / (dtype == 1 ? 2 : 4);
  return (n + per - 1) / per;
}

}  // namespace

int clip_groups(int tensors) { return std::max(1, (tensors + kGroup - 1) / kGroup); }
// Most values of a tensor: a group's chunks are counted in 32 bits.
int64_t clip_max_values() { return static_cast<int64_t>(1) << 36; }

// A partial sum for every workgroup: kMaxParts shared out among the launches, one at least each.
size_t clip_workspace_bytes(int tensors) {
  return align_up(static_cast<size_t>(kMaxParts + clip_groups(tensors)) * sizeof(double), 256);
}

hipError_t launch_clip_grad_norm(int tensors, const void* const* grads, void* const* out, const int64_t* n,
                                 const int32_t* dtypes, float max_norm, float* norm, float* scale, void* workspace,
                                 hipStream_t stream) {
  double* parts = static_cast<double*>(workspace);
  int64_t total = 0;
  for (int i = 0; i < tensors; ++i) total += chunks_of(n[i], dtypes[i]);
  ClipTable t;
  // fills the table with the tensors [g kGroup, ...) and returns its chunks (0: a launch without work)
  auto table = [&](int g) {
    t = ClipTable{};
    const int k0 = g * kGroup, k1 = std::min(tensors, k0 + kGroup);
    t.tensors = std::max(1, k1 - k0);
    int64_t c = 0;
    for (int k = k0; k < k1; ++k) {
      t.in[k - k0] = grads[k];
      t.out[k - k0] = out ? out[k] : const_cast<void*>(grads[k]);
      t.n[k - k0] = n[k];
      t.first[k - k0] = static_cast<int32_t>(c);
      if (dtypes[k] == 1) t.bf16[(k - k0) >> 5] |= 1u << ((k - k0) & 31);
      c += chunks_of(n[k], dtypes[k]);
    }
    t.first[t.tensors] = static_cast<int32_t>(c);
    return static_cast<int>(c);
  };
  // workgroups of a launch: its share of kMaxParts by chunks (rounded down, so that the sum over the
  // launches stays within kMaxParts + launches), no more than it has chunks
  auto grid_of = [&](int chunks) {
    const int64_t share = total > 0 ? static_cast<int64_t>(kMaxParts) * chunks / total : 0;
    return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(share, chunks)));
  };
  const int groups = clip_groups(tensors);
  int nparts = 0;
  for (int g = 0; g < groups; ++g) {
    const int chunks = table(g);
    const int grid = grid_of(chunks);
    Prof pr("grad_squares", stream);
    hipLaunchKernelGGL(grad_squares, dim3(grid), dim3(kThreads), 0, stream, t, parts + nparts);
    nparts += grid;
  }
  for (int g = 0; g < groups; ++g) {
    const int chunks = groups == 1 ? t.first[t.tensors] : table(g);
    Prof pr("grad_scale", stream);
    hipLaunchKernelGGL(grad_scale, dim3(grid_of(chunks)), dim3(kThreads), 0, stream, t, parts, nparts, max_norm,
                       out == nullptr, g == 0 ? norm : nullptr, g == 0 ? scale : nullptr);
  }
  return hipGetLastError();
}

}  // namespace pctc
