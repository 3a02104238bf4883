// Global gradient norm over a list of tensors, and clipping (gfx950).
//
//   n = sqrt(sum over all values g^2),  s = min(1, max_norm / (n + 1e-6)),  g <- s g
//
// Squares are taken and summed in double: no square of a finite value overflows (a norm beyond float's range
// is reported as infinite, and its double still clips), and the order of
// the sums, fixed by the sizes alone, moves the float result by at most its last bit.  Bound by
// memory: the values are read twice (the scale is known only after the last of them) and written once.
// Three kernels: partial sums on a fixed grid, one workgroup that adds them up, and the scaling; for
// short lists each workgroup of the scaling adds them up itself, and the second kernel is left out.
// 2.5 GB of fp32 out of place: 370 us for the sums, 6.8 TB/s, and 811 for the scaling, 6.2; 325 MB in 362
// tensors (four tables of both kernels) 62 + 124 us; 0.26 MB 4.1 + 4.6.
#include <algorithm>
#include <type_traits>

#include "pctc_internal.h"

namespace pctc {

namespace {

constexpr int kThreads = 256;
constexpr int kGroup = 96;       // tensors of a launch: their table is a kernel argument
constexpr int kMaxParts = 2048;  // workgroups (8 a compute unit) of a launch of the sums
constexpr int kPartsBudget = 16384;
// Bytes of a tensor that a workgroup takes at a time.  Scaling runs
// best in short workgroups: 2.5 GB fp32 out of place, 4 KB each 813 us, 16 KB 857; but 600,000 workgroups
// that find nothing to do take 134 us, so in place, where a scale of 1 is ordinary, each takes 32 KB (20 us
// then, and 898 where it clips; 4 KB 813).
constexpr int kSumBytes = kThreads * 8 * 16;
constexpr int kOutBytes = kThreads * 16;
constexpr int kInPlaceBytes = kThreads * 8 * 16;
constexpr int kNormThreads = 1024;
// Lists up to this size (one launch's tensors): two launches, 4.2 + 4.8 us at 0.26 MB (a kernel of its own for
// the norm is 4.4 more); at 32 MB 1,024 workgroups add up as many partial sums each.
constexpr int64_t kShortBytes = int64_t{32} << 20;
// Lists of this size are still cached (256 MB beside the memory) when they are read again, and are
// loaded as usual; longer ones past the caches: 2.5 GB summed in 370 us, as usual 415.
constexpr int64_t kCachedBytes = int64_t{192} << 20;

struct ClipTable {
  const void* in[kGroup];
  void* out[kGroup];
  int64_t n[kGroup];          // values
  int32_t first[kGroup + 1];  // chunks of the tensors before
  uint32_t bf16[(kGroup + 31) / 32];
  int32_t tensors;
};
static_assert(sizeof(ClipTable) <= 3600, "kernel arguments");

// 16 bytes at any alignment of its own values (views into flat buffers start where the tensors
// before them end); unaligned vector accesses are ordinary ones on this target.
typedef u32x4 __attribute__((aligned(2))) Piece;

template <bool NT>
__device__ __forceinline__ u32x4 load_piece(const void* p) {
  if constexpr (NT) return __builtin_nontemporal_load(static_cast<const Piece*>(p));
  else return *static_cast<const Piece*>(p);
}
__device__ __forceinline__ void store_piece(void* p, const u32x4& v) {
  __builtin_nontemporal_store(v, static_cast<Piece*>(p));
}

__device__ __forceinline__ int find_tensor(const ClipTable& t, int chunk) {
  int lo = 0, hi = t.tensors - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.first[mid] <= chunk) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// Sum over a workgroup of THREADS, in every thread (sh: one double a wavefront).
template <int THREADS>
__device__ __forceinline__ double block_sum(double x, double* sh) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor(x, o, 64);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) s += sh[w];
  return s;
}

template <bool BF>
__device__ __forceinline__ void add_squares(const u32x4& p, double& a, double& b) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if constexpr (BF) {
      const double x = __uint_as_float(p[q] << 16), y = __uint_as_float(p[q] & 0xffff0000u);
      a = fma(x, x, a);
      b = fma(y, y, b);
    } else {
      const double x = __uint_as_float(p[q]);
      if (q & 1) b = fma(x, x, b);
      else a = fma(x, x, a);
    }
  }
}

// S float, or double for scales below float's normal range (norms of 1e38 times the bound).
template <bool BF, class S>
__device__ __forceinline__ u32x4 scaled(const u32x4& v, S s) {
  u32x4 r;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if constexpr (BF)
      r[q] = pack_bf16x2(static_cast<float>(__uint_as_float(v[q] << 16) * s),
                         static_cast<float>(__uint_as_float(v[q] & 0xffff0000u) * s));
    else
      r[q] = __float_as_uint(static_cast<float>(__uint_as_float(v[q]) * s));
  }
  return r;
}

// A piece of which only `left` < 8 (4) values exist: the others zero, and not written.
template <bool BF>
__device__ __forceinline__ u32x4 load_part(const void* p, int left) {
  u32x4 v = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int e = 0; e < (BF ? 8 : 4); ++e) {
    if (e < left) {
      if constexpr (BF) v[e >> 1] |= static_cast<uint32_t>(static_cast<const uint16_t*>(p)[e]) << (16 * (e & 1));
      else v[e] = static_cast<const uint32_t*>(p)[e];
    }
  }
  return v;
}
template <bool BF>
__device__ __forceinline__ void store_part(void* p, const u32x4& v, int left) {
#pragma unroll
  for (int e = 0; e < (BF ? 8 : 4); ++e) {
    if (e < left) {
      if constexpr (BF) static_cast<uint16_t*>(p)[e] = static_cast<uint16_t>(v[e >> 1] >> (16 * (e & 1)));
      else static_cast<uint32_t*>(p)[e] = v[e];
    }
  }
}

// Sum of squares of a workgroup's chunk of a tensor, from value `first` on.
template <bool BF, bool NT>
__device__ __forceinline__ void chunk_squares(const void* base, int64_t n, int64_t first, double& a, double& b) {
  constexpr int kPer = BF ? 8 : 4, kSize = BF ? 2 : 4;
  constexpr int kVec = kSumBytes / (kThreads * 16);
  const char* p = static_cast<const char*>(base) + first * kSize + threadIdx.x * 16;
  const int64_t left = n - first;
  if (left >= kSumBytes / kSize) {
    u32x4 v[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = load_piece<NT>(p + i * kThreads * 16);
#pragma unroll
    for (int i = 0; i < kVec; ++i) add_squares<BF>(v[i], a, b);
    return;
  }
  for (int64_t at = threadIdx.x * kPer; at < left; at += kThreads * kPer, p += kThreads * 16) {
    if (at + kPer <= left) add_squares<BF>(load_piece<NT>(p), a, b);
    else add_squares<BF>(load_part<BF>(p, static_cast<int>(left - at)), a, b);
  }
}

template <bool BF, int BYTES, class S>
__device__ __forceinline__ void chunk_scale(const void* in, void* out, int64_t n, int64_t first, S s) {
  constexpr int kPer = BF ? 8 : 4, kSize = BF ? 2 : 4;
  constexpr int kVec = BYTES / (kThreads * 16) < 4 ? BYTES / (kThreads * 16) : 4;
  const char* p = static_cast<const char*>(in) + first * kSize + threadIdx.x * 16;
  char* o = static_cast<char*>(out) + first * kSize + threadIdx.x * 16;
  const int64_t left = n - first;
  if (left >= BYTES / kSize) {
#pragma unroll
    for (int h = 0; h < BYTES / (kThreads * 16 * kVec); ++h, p += kVec * kThreads * 16, o += kVec * kThreads * 16) {
      u32x4 v[kVec];
#pragma unroll
      for (int i = 0; i < kVec; ++i) v[i] = load_piece<true>(p + i * kThreads * 16);
#pragma unroll
      for (int i = 0; i < kVec; ++i) store_piece(o + i * kThreads * 16, scaled<BF>(v[i], s));
    }
    return;
  }
  for (int64_t at = threadIdx.x * kPer; at < left; at += kThreads * kPer, p += kThreads * 16, o += kThreads * 16) {
    const int here = static_cast<int>(left - at < kPer ? left - at : kPer);
    if (here == kPer) store_piece(o, scaled<BF>(load_piece<true>(p), s));
    else store_part<BF>(o, scaled<BF>(load_part<BF>(p, here), s), here);
  }
}

__device__ __forceinline__ bool is_bf16(const ClipTable& t, int k) { return (t.bf16[k >> 5] >> (k & 31)) & 1; }

template <bool NT>
__global__ void __launch_bounds__(kThreads) grad_squares(ClipTable t, double* __restrict__ parts) {
  __shared__ double sh[kThreads / 64];
  double a = 0.0, b = 0.0;
  const int chunks = t.first[t.tensors];
  for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
    const int k = find_tensor(t, c);
    const int64_t step = c - t.first[k];
    if (is_bf16(t, k)) chunk_squares<true, NT>(t.in[k], t.n[k], step * (kSumBytes / 2), a, b);
    else chunk_squares<false, NT>(t.in[k], t.n[k], step * (kSumBytes / 4), a, b);
  }
  const double s = block_sum<kThreads>(a + b, sh);
  if (threadIdx.x == 0) parts[blockIdx.x] = s;
}

// The scale of a sum of squares.  A norm that is not finite clips nothing: the caller sees it in the
// norm and drops the step.
__device__ __forceinline__ double scale_of(double sum, float max_norm, float* norm, float* scale) {
  const double n = sqrt(sum);
  double s = 1.0;
  if (n <= 1.7976931348623157e308) s = fmin(1.0, static_cast<double>(max_norm) / (n + 1e-6));
  if (norm && threadIdx.x == 0) {
    *norm = static_cast<float>(n);
    if (scale) *scale = static_cast<float>(s);
  }
  return s;
}
__global__ void __launch_bounds__(kNormThreads)
grad_norm(const double* __restrict__ parts, int nparts, float max_norm, float* __restrict__ norm,
          float* __restrict__ scale, double* __restrict__ factor) {
  __shared__ double sh[kNormThreads / 64];
  double x = 0.0;
  for (int i = threadIdx.x; i < nparts; i += kNormThreads) x += parts[i];
  const double s = scale_of(block_sum<kNormThreads>(x, sh), max_norm, norm, scale);
  if (threadIdx.x == 0) *factor = s;
}

// This workgroup's chunk of the list times sd.
template <int BYTES>
__device__ __forceinline__ void scale_list(const ClipTable& t, double sd) {
  const float s = static_cast<float>(sd);
  const int c = blockIdx.x, k = find_tensor(t, c);
  const int64_t step = c - t.first[k];
  const bool bf = is_bf16(t, k);
  const int64_t first = step * (bf ? BYTES / 2 : BYTES / 4);
  if (sd > 0.0 && s < 1.17549435e-38f) {
    if (bf) chunk_scale<true, BYTES>(t.in[k], t.out[k], t.n[k], first, sd);
    else chunk_scale<false, BYTES>(t.in[k], t.out[k], t.n[k], first, sd);
  } else {
    if (bf) chunk_scale<true, BYTES>(t.in[k], t.out[k], t.n[k], first, s);
    else chunk_scale<false, BYTES>(t.in[k], t.out[k], t.n[k], first, s);
  }
}

template <int BYTES>
__global__ void __launch_bounds__(kThreads) grad_scale(ClipTable t, const double* __restrict__ factor, bool in_place) {
  const double sd = *factor;
  if (in_place && static_cast<float>(sd) == 1.f) return;
  scale_list<BYTES>(t, sd);
}

// The same for short lists, the partial sums added up by every workgroup; the first one writes the norm.
__global__ void __launch_bounds__(kThreads)
grad_norm_scale(ClipTable t, const double* __restrict__ parts, int nparts, float max_norm, bool in_place,
                float* __restrict__ norm, float* __restrict__ scale) {
  __shared__ double sh[kThreads / 64];
  double x = 0.0;
  for (int i = threadIdx.x; i < nparts; i += kThreads) x += parts[i];
  const double sum = block_sum<kThreads>(x, sh);
  const double sd = scale_of(sum, max_norm, blockIdx.x == 0 ? norm : nullptr, scale);
  if (static_cast<int>(blockIdx.x) >= t.first[t.tensors] || (in_place && static_cast<float>(sd) == 1.f)) return;
  scale_list<kSumBytes>(t, sd);
}

int64_t chunks_of(int64_t n, int dtype, int bytes) {
  const int64_t per = bytes / (dtype == 1 ? 2 : 4);
  return (n + per - 1) / per;
}

int groups_of(int tensors) { return std::max(1, (tensors + kGroup - 1) / kGroup); }
// Workgroups of a launch of the sums: no more than kPartsBudget (or 64 each) over all launches.
int most_parts(int groups) { return std::max(64, std::min(kMaxParts, kPartsBudget / groups)); }

}  // namespace

// Most values of a tensor: a group's chunks are counted in 32 bits.
int64_t clip_max_values() { return static_cast<int64_t>(1) << 34; }

// The factor, then the partial sums.
size_t clip_workspace_bytes(int tensors) {
  const int groups = groups_of(tensors);
  return 256 + align_up(static_cast<size_t>(groups) * most_parts(groups) * sizeof(double), 256);
}

hipError_t launch_clip_grad_norm(int tensors, const void* const* grads, void* const* out, const int64_t* n,
                                 const int32_t* dtypes, float max_norm, float* norm, float* scale, void* workspace,
                                 hipStream_t stream) {
  double* factor = static_cast<double*>(workspace);
  double* parts = reinterpret_cast<double*>(static_cast<char*>(workspace) + 256);
  const int groups = groups_of(tensors);
  int64_t total = 0;
  for (int i = 0; i < tensors; ++i) total += n[i] * (dtypes[i] == 1 ? 2 : 4);
  ClipTable t;
  // fills the table with the tensors [g kGroup, ...) in chunks of `bytes` and returns their number
  auto table = [&](int g, int bytes) {
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
      c += chunks_of(n[k], dtypes[k], bytes);
    }
    t.first[t.tensors] = static_cast<int32_t>(c);
    return static_cast<int>(c);
  };
  int nparts = 0;
  for (int g = 0; g < groups; ++g) {
    const int grid = std::min(most_parts(groups), table(g, kSumBytes));
    if (grid == 0) continue;
    Prof pr("grad_squares", stream);
    if (total > kCachedBytes)
      hipLaunchKernelGGL(grad_squares<true>, dim3(grid), dim3(kThreads), 0, stream, t, parts + nparts);
    else
      hipLaunchKernelGGL(grad_squares<false>, dim3(grid), dim3(kThreads), 0, stream, t, parts + nparts);
    nparts += grid;
  }
  if (groups == 1 && total <= kShortBytes) {
    Prof pr("grad_norm_scale", stream);
    hipLaunchKernelGGL(grad_norm_scale, dim3(std::max(1, t.first[t.tensors])), dim3(kThreads), 0, stream, t, parts,
                       nparts, max_norm, out == nullptr, norm, scale);
    return hipGetLastError();
  }
  {
    Prof pr("grad_norm", stream);
    hipLaunchKernelGGL(grad_norm, dim3(1), dim3(kNormThreads), 0, stream, parts, nparts, max_norm, norm, scale, factor);
  }
  for (int g = 0; g < groups; ++g) {
    int chunks = out ? table(g, kOutBytes) : 0;
    const bool small = out && chunks <= kMaxGrid;
    if (!small) chunks = table(g, kInPlaceBytes);  // (of 96 tensors at most 0.27 TB)
    if (chunks == 0) continue;
    Prof pr("grad_scale", stream);
    if (small) hipLaunchKernelGGL(grad_scale<kOutBytes>, dim3(chunks), dim3(kThreads), 0, stream, t, factor, false);
    else hipLaunchKernelGGL(grad_scale<kInPlaceBytes>, dim3(chunks), dim3(kThreads), 0, stream, t, factor, !out);
  }
  return hipGetLastError();
}

}  // namespace pctc
