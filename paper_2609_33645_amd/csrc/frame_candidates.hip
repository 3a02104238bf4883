// Frame candidates (gfx950): the C most probable classes of every frame other than blank, with
// their log probabilities and blank's, over the full vocabulary.
//
//   z = H W^T + b,  lambda_m = log sum_v exp z_mv,  logp = float(z - lambda_m), z and lambda in the order
//   of falling z, the lowest class first among equal ones
//
// One vocabulary pass on the matrix cores gives the normaliser's partial pairs and the largest logit
// of every block of 8 classes.  A class among a frame's C best lies in one of the C + 1 blocks with the
// largest maxima (one more for blank, which is left out; and one for the block whose classes lie between
// the last one's, where maxima are equal), so a second kernel needs 8 (C + 2) logits a frame, and orders
// them.  Where the vocabulary is long beside the rows that those take, they are formed again from H and W
// and the frame x vocabulary logits are never stored; where it is short, the pass keeps them (keeps_logits).
// The scratch is held to 512 MB by passing over the vocabulary once per that many frames.
//
// The product is bound by the matrix cores from some 600 frames on (4,347 frames, D = 512, V = 180,000, bf16:
// 811 us, 0.99 PFLOP/s of 1.20 in a large library product) and by the reading of W below (64 frames: 34 us, 5.4
// TB/s).  The choice is bound by the rows of W that it reads again (8 (C + 2) a frame, 640 MB there: 104 us, 6
// TB/s).
#include <algorithm>

#include "pctc_internal.h"

namespace pctc {

namespace {

constexpr size_t kMaxPassBytes = static_cast<size_t>(512) << 20;
// Up to two workgroups a compute unit: 1024 threads each, whose loads cover one another (150 frames of 180,000
// classes, D = 512: 14.9 us, with 256 threads 26; 109 frames, D = 3512, C = 24: 39 and 56).  More frames fill the
// card as workgroups of 256 (2,155 frames of 6,700 classes: 18 us, with 1024 threads 50).
constexpr int kFewFrames = 512;
constexpr int kList = 256;  // blocks kept for ordering; more only where maxima are equal
constexpr int kMaxSel = kMaxCandidates + 2;

// Floats in the order of unsigned integers.
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// The largest key t (its low 12 bits zero) that at least `need` of 256 groups of threads reach (thread
// tid is of group tid mod 256; keys of NT threads); 0 when there are fewer.  For one wavefront: the
// others' issue slots are for other workgroups.
template <int NT>
__device__ __forceinline__ uint32_t reach(const uint32_t* keys, int need, int lane) {
  uint32_t k[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    k[i] = keys[64 * i + lane];
#pragma unroll
    for (int j = 256; j < NT; j += 256) k[i] = max(k[i], keys[j + 64 * i + lane]);
  }
  uint32_t t = 0;
  for (int bit = 31; bit >= 12; --bit) {
    const uint32_t c = t | (1u << bit);
    int n = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) n += __popcll(__ballot(k[i] >= c));
    if (n >= need) t = c;
  }
  return t;
}

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
__device__ __forceinline__ float dot16(const u32x4& w, const u32x4& h, float s, uint16_t) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const uint32_t a = w[q], b = h[q];
    s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, a), __builtin_bit_cast(bf16x2, b), s, false);
  }
  return s;
}
__device__ __forceinline__ float dot16(const u32x4& w, const u32x4& h, float s, float) {
#pragma unroll
  for (int q = 0; q < 4; ++q) s = fmaf(__uint_as_float(w[q]), __uint_as_float(h[q]), s);
  return s;
}

}  // namespace

// One workgroup of NT threads per frame.
template <class T, int NT, bool KEPT>
__global__ void __launch_bounds__(NT)
cand_select_kernel(const T* __restrict__ H, int m0, int D, const T* __restrict__ W, const float* __restrict__ bias,
                   int V, int blank, int C, const float* __restrict__ bmax, int nb,
                   const float2* __restrict__ partials, int M, int P, int vper, const float* __restrict__ Z, int ldz,
                   int32_t* __restrict__ ids, float* __restrict__ logp, float* __restrict__ blank_logp) {
  constexpr int kPer = 16 / sizeof(T);
  constexpr int kValues = kMaxSel * kCandRows;
  constexpr int kParts = kMaxLseParts / NT;
  __shared__ uint32_t keys[NT];
  __shared__ float list_v[kList];
  __shared__ int list_b[kList];
  __shared__ int count;
  __shared__ uint32_t bound;
  __shared__ float part_max[NT / 64];
  __shared__ double part_sum[NT / 64];
  __shared__ int part_nan[NT / 64];
  __shared__ double lam_s;
  __shared__ uint16_t scan_s[kMaxLseParts];
  __shared__ int scans;
  __shared__ int sel[kMaxSel];
  __shared__ float z[kValues];
  __shared__ float val_v[kValues];
  __shared__ int val_i[kValues];
  __shared__ float zblank;
  __shared__ unsigned long long moved;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int m = m0 + blockIdx.x;
  const float* const row = bmax + static_cast<int64_t>(blockIdx.x) * nb;
  const int nsel = min(C + 2, nb);

  // ---- the normaliser of each wavefront's partitions ----
  float2 q[kParts];  // the largest logit of partition tid + i NT, and its sum
  float mx = -INFINITY;
  {
    const float2* const q0 = partials + blockIdx.x;
    int nan = 0;
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
      const int p = tid + i * NT;
      q[i] = p < P ? q0[static_cast<int64_t>(p) * M] : make_float2(-INFINITY, 0.f);
      nan |= (q[i].x != q[i].x) | (q[i].y != q[i].y);
      mx = fmaxf(mx, q[i].x);
    }
    float top = mx;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < kParts; ++i)
      if (q[i].x > -INFINITY)
        sum += static_cast<double>(q[i].y) *
               static_cast<double>(fast_exp2(static_cast<float>(static_cast<double>(q[i].x) - top) * kLog2e));
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) sum += __shfl_xor(sum, o, 64);
    nan = __any(nan);
    if (lane == 0) {
      part_max[wave] = top;
      part_sum[wave] = sum;
      part_nan[wave] = nan;
    }
  }

  // ---- the nsel blocks with the largest maxima (equal ones: the lowest) ----
  // Where there are many partitions, those blocks lie in the ones whose largest logit is at least the nsel-th of
  // theirs, a few of them, and only these are read (4,347 frames, V = 180,000: 103 us, by the
  // threads' maxima 193; 2,669 frames, V = 151,936, D = 4096: 270 and 323); else the blocks of at least
  // the nsel-th of the threads' maxima, from two readings of all.
  const bool by_parts = P >= 2 * nsel;
  if (!by_parts) {
    mx = -INFINITY;
    for (int i = tid * 4; i < nb; i += NT * 4) {
      const float4 v = *reinterpret_cast<const float4*>(row + i);
      mx = fmaxf(mx, fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w)));
    }
  }
  keys[tid] = order_key(mx);
  if (tid == 0) {
    count = 0;
    scans = 0;
    moved = 0;
  }
  __syncthreads();
  if (wave == 0) {
    const uint32_t r = reach<NT>(keys, nsel, lane);
    if (lane == 0) bound = r;
  } else if (wave == 1) {  // lambda meanwhile
    float top = -INFINITY;
    int nan = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
      top = fmaxf(top, part_max[w]);
      nan |= part_nan[w];
    }
    double sum = 0.0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w)
      if (part_max[w] > -INFINITY)
        sum += part_sum[w] *
               static_cast<double>(fast_exp2(static_cast<float>(static_cast<double>(part_max[w]) - top) * kLog2e));
    const double l = top > -INFINITY ? static_cast<double>(top) + log(sum) : -INFINITY;
    if (lane == 0) lam_s = nan ? __longlong_as_double(0x7ff8000000000000LL) : l;
  }
  __syncthreads();
  uint32_t t = bound;
  auto take = [&](int i) {  // the blocks in places i .. i + 3 that are large enough
    const float4 v4 = *reinterpret_cast<const float4*>(row + i);
    const float v[4] = {v4.x, v4.y, v4.z, v4.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (v[e] > -INFINITY && order_key(v[e]) >= t) {
        const int at = atomicAdd(&count, 1);
        if (at < kList) {
          list_v[at] = v[e];
          list_b[at] = CandBlocks::at(i + e);
        }
      }
    }
  };
  if (by_parts) {
#pragma unroll
    for (int i = 0; i < kParts; ++i)
      if (q[i].x > -INFINITY && order_key(q[i].x) >= t)
        scan_s[atomicAdd(&scans, 1)] = static_cast<uint16_t>(tid + i * NT);
    __syncthreads();
    const int quads = vper / (4 * kCandRows), all = scans * quads;
    for (int x = tid; x < all; x += NT) {
      const int i = (scan_s[x / quads] * quads + x % quads) * 4;
      if (i < nb) take(i);
    }
  } else {  // (most threads have no block that large)
    for (int i = order_key(mx) >= t ? tid * 4 : nb; i < nb; i += NT * 4) take(i);
  }
  __syncthreads();
  int n = count;
  if (n <= kList) {
    // the list in the order of (maximum, block): a block's place is the number of those before it
    if (tid < n) {
      const float v = list_v[tid];
      const int b = list_b[tid];
      int rank = 0;
#pragma unroll 4
      for (int q = 0; q < n; ++q) rank += list_v[q] > v || (list_v[q] == v && list_b[q] < b);
      if (rank < nsel) sel[rank] = b;
    }
    n = min(n, nsel);
  } else {
    // many equal maxima: the key of the nsel-th block exactly, the blocks above it in any order, then
    // those at it from the lowest on
    t = 0;
    for (int bit = 31; bit >= 0; --bit) {
      const uint32_t c = t | (1u << bit);
      __syncthreads();
      if (tid == 0) count = 0;
      __syncthreads();
      int mine = 0;
      for (int i = tid; i < nb; i += NT) mine += row[i] > -INFINITY && order_key(row[i]) >= c;
      if (mine) atomicAdd(&count, mine);
      __syncthreads();
      if (count >= nsel) t = c;
    }
    __syncthreads();
    if (tid == 0) count = 0;
    __syncthreads();
    for (int i = tid; i < nb; i += NT)
      if (row[i] > -INFINITY && order_key(row[i]) > t) sel[atomicAdd(&count, 1)] = CandBlocks::at(i);
    __syncthreads();
    n = count;
    if (wave == 0) {
      for (int i0 = 0; i0 < nb && n < nsel; i0 += 64) {
        const float v = i0 + lane < nb ? row[CandBlocks::place(i0 + lane)] : -INFINITY;
        const bool at = v > -INFINITY && order_key(v) == t;
        const uint64_t who = __ballot(at);
        const int q = n + __popcll(who & ((uint64_t{1} << lane) - 1));
        if (at && q < nsel) sel[q] = i0 + lane;
        n += __popcll(who);
      }
      if (lane == 0) count = min(n, nsel);
    }
    __syncthreads();
    n = count;
  }
  __syncthreads();

  // ---- their logits ----
  const double lam0 = lam_s;
  const float was = !KEPT && tid < n ? row[CandBlocks::place(sel[tid])] : 0.f;
  if constexpr (KEPT) {
    const float* const zrow = Z + static_cast<int64_t>(blockIdx.x) * ldz;
    for (int i = tid; i < n * kCandRows; i += NT) {
      const int v = CandBlocks::class_of(sel[i / kCandRows], i % kCandRows);
      z[i] = v == blank ? -INFINITY : zrow[v];  // (-inf from V on)
    }
    if (tid == 0) zblank = zrow[blank];
  } else {
    // eight lanes a class, a block of a wavefront at a time
    static_assert(kCandRows == 8, "a wavefront's classes");
    const T* const h = H + static_cast<int64_t>(m) * D;
    const int part = lane & 7;
    for (int g = wave; g <= n; g += NT / 64) {  // (the last: blank)
      const int v = g < n ? CandBlocks::class_of(sel[g], lane >> 3) : blank;
      const T* const w = W + static_cast<int64_t>(min(v, V - 1)) * D;
      float x = 0.f;
#pragma unroll 4
      for (int k = part * kPer; k < D; k += 8 * kPer)
        x = dot16(*reinterpret_cast<const u32x4*>(w + k), *reinterpret_cast<const u32x4*>(h + k), x, T{});
#pragma unroll
      for (int o = 4; o >= 1; o >>= 1) x += __shfl_xor(x, o, 64);
      if (part != 0) continue;
      if (bias && v < V) x += bias[v];
      if (g == n) zblank = x;  // every class's first lane holds it
      else z[g * kCandRows + (lane >> 3)] = v >= V || v == blank ? -INFINITY : x;
    }
  }
  if (tid == 0) count = 0;
  __syncthreads();

  // The vocabulary pass rounded these logits in another order.  Where one class has nearly all of the
  // probability, the difference would be the whole of logp = z - lambda, so lambda takes the largest of each
  // block as they are here: lambda + log(1 + sum over the blocks (exp(z' - lambda) - exp(z - lambda))), the
  // sum in integers of 2^-56, which have the same sum in any order.
  if (!KEPT && tid < n) {
    float top = sel[tid] == CandBlocks::block_of(blank) ? zblank : -INFINITY;
#pragma unroll
    for (int k = 0; k < kCandRows; ++k) top = fmaxf(top, z[tid * kCandRows + k]);
    const float d = expf(static_cast<float>(was - lam0)) * expm1f(top - was);
    if (fabsf(d) < 0.5f)  // (not where a logit is infinite or NaN)
      atomicAdd(&moved, static_cast<unsigned long long>(llrint(static_cast<double>(d) * 0x1p56)));
  }

  // ---- the C best of them ----
  const int nz = n * kCandRows;
  mx = -INFINITY;
  for (int i = tid; i < nz; i += NT) mx = fmaxf(mx, z[i]);
  keys[tid] = order_key(mx);
  __syncthreads();
  if (wave == 0) {
    const uint32_t r = reach<NT>(keys, C, lane);
    if (lane == 0) bound = r;
  }
  __syncthreads();
  t = bound;
  for (int i = tid; i < nz; i += NT) {
    const float v = z[i];
    if (v > -INFINITY && order_key(v) >= t) {
      const int q = atomicAdd(&count, 1);
      val_v[q] = v;
      val_i[q] = CandBlocks::class_of(sel[i / kCandRows], i % kCandRows);
    }
  }
  __syncthreads();
  const int nv = count;
  const float by = static_cast<float>(static_cast<double>(static_cast<long long>(moved)) * 0x1p-56);
  const double l = lam0 + (fabsf(by) < 0.5f ? static_cast<double>(log1pf(by)) : 0.);
  for (int i = tid; i < nv; i += NT) {
    const float v = val_v[i];
    const int id = val_i[i];
    int rank = 0;
#pragma unroll 4
    for (int q = 0; q < nv; ++q) rank += val_v[q] > v || (val_v[q] == v && val_i[q] < id);
    if (rank < C) {
      ids[static_cast<int64_t>(m) * C + rank] = id;
      logp[static_cast<int64_t>(m) * C + rank] = static_cast<float>(v - l);
    }
  }
  for (int r = nv + tid; r < C; r += NT) {
    ids[static_cast<int64_t>(m) * C + r] = -1;
    logp[static_cast<int64_t>(m) * C + r] = -INFINITY;
  }
  if (tid == 0) blank_logp[m] = zblank == -INFINITY ? -INFINITY : static_cast<float>(zblank - l);
}

namespace {
// Whether the product writes its logits for the choice to read (4 V bytes a frame, and 32 (C + 2) of them
// back) instead of the choice forming them again from 8 (C + 2) rows of W, which come through the L2s at twice
// the rate.  Product and choice, kept and formed again: fp32, 1,600 frames, D = 512, V = 5,000, C = 16: 81 + 12
// us, 73 + 48; 753 frames, D = 2480, V = 17,052, C = 7: 373 + 10, 364 + 77; bf16, 138 frames, D = 448,
// V = 29,197, C = 29 (near the rule's edge): 23.6 + 13.7, 18.3 + 20.2; 205 frames, D = 3008, V = 157,375, C = 14
// (past it): 322 + 16, 279 + 40; 798 frames, D = 160, V = 11,099, C = 12 (past it): 24 + 11, 14 + 16.  At 32,768
// classes a pass's scratch holds 3,584 frames; fewer to a pass would read W more often than they save.
bool keeps_logits(int dtype, int D, int V, int C) {
  return V <= 32768 && V < static_cast<int64_t>(C + 2) * D * (dtype == 1 ? 2 : 4);
}
// Scratch of a pass: the normaliser's partial pairs, the block maxima, the logits where they are kept and, where
// the product reads it, H transposed.
struct CandLayout {
  int frames, blocks, ldz;
  size_t o_bmax, o_z, o_ht, total;
};
CandLayout cand_layout(int dtype, int M, int D, int V, int C) {
  CandLayout L;
  L.blocks = cand_blocks(V);
  L.ldz = keeps_logits(dtype, D, V, C) ? L.blocks * kCandRows : 0;
  const size_t per = static_cast<size_t>(L.blocks + L.ldz) * sizeof(float);
  const int most = static_cast<int>(std::min<size_t>(kMaxPassBytes / per / 256 * 256, 1 << 30));
  L.frames = std::max(1, std::min(M, std::max(most, 256)));
  L.o_bmax = lse_partial_bytes(L.frames, D);
  L.o_z = L.o_bmax + align_up(static_cast<size_t>(L.frames) * L.blocks * sizeof(float), 256);
  L.o_ht = L.o_z + align_up(static_cast<size_t>(L.frames) * L.ldz * sizeof(float), 256);
  L.total = L.o_ht + (dtype == 1 ? cand_ht_bytes(L.frames, D, V) : 0);
  return L;
}
// Bytes of H transposed for a pass over `here` frames (0: the product reads H itself).  A full pass's are too many
// to be addressed where D is large beside V; the layout then has no room for them, nor for a shorter last pass's.
size_t pass_ht_bytes(const CandLayout& L, int here, int D, int V) {
  return L.total > L.o_ht ? cand_ht_bytes(here, D, V) : 0;
}
}  // namespace

size_t cand_scratch_bytes(int dtype, int M, int D, int V, int C) { return cand_layout(dtype, M, D, V, C).total; }

size_t cand_pass_bytes(int dtype, int M, int D, int V, int C, int m0, int* frames) {
  const CandLayout L = cand_layout(dtype, M, D, V, C);
  *frames = std::min(L.frames, M - m0);
  return L.o_ht + (dtype == 1 ? pass_ht_bytes(L, *frames, D, V) : 0);
}

hipError_t launch_frame_candidates(int dtype, const void* H, int M, int D, const void* W, const float* bias, int V,
                                   int blank, int C, int32_t* ids, float* logp, float* blank_logp, void* scratch,
                                   hipStream_t stream) {
  const CandLayout L = cand_layout(dtype, M, D, V, C);
  const int F = L.frames, nb = L.blocks;
  char* s = static_cast<char*>(scratch);
  float2* partials = reinterpret_cast<float2*>(s);
  float* bmax = reinterpret_cast<float*>(s + L.o_bmax);
  float* Z = L.ldz ? reinterpret_cast<float*>(s + L.o_z) : nullptr;
  for (int m0 = 0; m0 < M; m0 += F) {
    const int here = std::min(F, M - m0);
    int P = 0, vper = 0;
    hipError_t e;
    if (dtype == 1) {
      const uint16_t* Hm = static_cast<const uint16_t*>(H) + static_cast<int64_t>(m0) * D;
      const int Mp = (here + 63) / 64 * 64;
      uint16_t* Ht = pass_ht_bytes(L, here, D, V) > 0 ? reinterpret_cast<uint16_t*>(s + L.o_ht) : nullptr;
      if (Ht && (e = launch_ht_build_bf16(Hm, here, D, nullptr, nullptr, Ht, Mp, stream)) != hipSuccess) return e;
      e = launch_cand_partial_bf16(Hm, here, D, static_cast<const uint16_t*>(W), bias, V, partials, &P, &vper, bmax, Z,
                                   L.ldz, stream, Ht, Mp);
    } else {
      e = launch_cand_partial_f32(static_cast<const float*>(H) + static_cast<int64_t>(m0) * D, here, D,
                                  static_cast<const float*>(W), bias, V, partials, &P, &vper, bmax, Z, L.ldz, stream);
    }
    if (e != hipSuccess) return e;
    Prof pr("cand_select", stream);
#define PCTC_SELECT(T, NT, KEPT)                                                                                      \
  hipLaunchKernelGGL((cand_select_kernel<T, NT, KEPT>), dim3(here), dim3(NT), 0, stream, static_cast<const T*>(H),    \
                     m0, D, static_cast<const T*>(W), bias, V, blank, C, bmax, nb, partials, here, P, vper, Z, L.ldz, \
                     ids, logp, blank_logp)
    const bool few = here <= kFewFrames;
    if (Z) {  // (H and W are not read)
      if (few) PCTC_SELECT(float, 1024, true);
      else PCTC_SELECT(float, 256, true);
    } else if (dtype == 1) {
      if (few) PCTC_SELECT(uint16_t, 1024, false);
      else PCTC_SELECT(uint16_t, 256, false);
    } else {
      if (few) PCTC_SELECT(float, 1024, false);
      else PCTC_SELECT(float, 256, false);
    }
#undef PCTC_SELECT
  }
  return hipGetLastError();
}

}  // namespace pctc
