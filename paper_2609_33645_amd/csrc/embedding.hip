// Token embedding and its gradient (gfx950).
//
//   y[m] = scale table[token_m]  (zeros for a token outside [0, V))
//   dW[v] (+)= scale sum over m with token_m = v of dy[m]
//
// Both are bound by memory: rows in, rows out.  The gradient sums the rows of a class in the order of
// their places, in float, so that it does not change from call to call: the tokens are sorted
// stably by class, ranges of sorted places are summed each by its own lanes, and the sums of a class that
// lies in several ranges are joined in order by a second kernel (a class may have most of the
// tokens).
//
// Sorting.  Up to kRankTokens tokens: a token's place is the number of tokens before it in the
// order, counted against all of them (N^2 compares, N / 64 workgroups).  More: a radix sort, at
// most two passes of up to 10 bits, with counts per wavefront and digit.
#include <algorithm>

#include "pctc_internal.h"

namespace pctc {

namespace {

constexpr int kThreads = 256;
constexpr int kRankTokens = 15360;  // their classes and the counts take 64 KB of LDS
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kMaxBits = 10, kMaxBins = 1 << kMaxBits;
constexpr int kMaxTiles = 128;  // workgroups of a radix pass
// Tokens that a wavefront of rank_tokens counts.
__host__ __device__ __forceinline__ int rank_share(int N) { return ((N + kSortWaves - 1) / kSortWaves + 63) / 64 * 64; }

typedef u32x4 __attribute__((aligned(2))) Piece;

template <bool BF>
struct Vals {  // values of a 16-byte piece
  static constexpr int kN = BF ? 8 : 4;
  float v[kN];
};

template <bool BF>
__device__ __forceinline__ void unpack(const u32x4& w, float* v) {
  if constexpr (BF) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = __uint_as_float(w[e] << 16);
      v[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(w[e]);
  }
}

// n values (at most N) from p, the rest zeros.
template <bool BF, int N>
__device__ __forceinline__ void load_vals(const void* p, int n, float (&v)[N]) {
  constexpr int kPer = BF ? 8 : 4;
  if (n >= N) {
#pragma unroll
    for (int h = 0; h < N / kPer; ++h)
      unpack<BF>(*reinterpret_cast<const Piece*>(static_cast<const char*>(p) + 16 * h), v + h * kPer);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      if constexpr (BF) v[e] = e < n ? bf16_to_f32(static_cast<const uint16_t*>(p)[e]) : 0.f;
      else v[e] = e < n ? static_cast<const float*>(p)[e] : 0.f;
    }
  }
}
template <bool BF, int N>
__device__ __forceinline__ void store_vals(void* p, int n, const float (&v)[N]) {
  constexpr int kPer = BF ? 8 : 4;
  if (n >= N) {
#pragma unroll
    for (int h = 0; h < N / kPer; ++h) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (BF) w[e] = pack_bf16x2(v[h * 8 + 2 * e], v[h * 8 + 2 * e + 1]);
        else w[e] = __float_as_uint(v[h * 4 + e]);
      }
      *reinterpret_cast<Piece*>(static_cast<char*>(p) + 16 * h) = w;
    }
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < n) {
        if constexpr (BF) static_cast<uint16_t*>(p)[e] = static_cast<uint16_t>(pack_bf16x2(v[e], 0.f));
        else static_cast<float*>(p)[e] = v[e];
      }
  }
}

// Class of token i; V for one outside [0, V).
template <bool I64>
__device__ __forceinline__ int class_of(const void* tokens, int64_t i, int V) {
  if constexpr (I64) {
    const int64_t t = static_cast<const int64_t*>(tokens)[i];
    return (t >= 0 && t < V) ? static_cast<int>(t) : V;
  } else {
    const int32_t t = static_cast<const int32_t*>(tokens)[i];
    return (t >= 0 && t < V) ? t : V;
  }
}

// ---- lookup --------------------------------------------------------------------------------

// `lanes` (a power of two) lanes a row, 256 / lanes rows a workgroup.  Few rows: the launch, 2.9 us for 128 of 512.
template <bool BF, bool I64>
__global__ void __launch_bounds__(kThreads)
embedding_kernel(const void* __restrict__ table, int V, int D, const void* __restrict__ tokens, int64_t N, float scale,
                 int lanes, void* __restrict__ y) {
  constexpr int kPer = BF ? 8 : 4, kBytes = BF ? 2 : 4;
  const int rows = kThreads / lanes, sub = threadIdx.x / lanes, at = threadIdx.x % lanes;
  for (int64_t m = static_cast<int64_t>(blockIdx.x) * rows + sub; m < N; m += static_cast<int64_t>(gridDim.x) * rows) {
    const int c = class_of<I64>(tokens, m, V);
    const char* src = static_cast<const char*>(table) + static_cast<int64_t>(c) * D * kBytes;
    char* dst = static_cast<char*>(y) + m * D * kBytes;
    for (int d = at * kPer; d < D; d += lanes * kPer) {
      float v[kPer];
      load_vals<BF>(src + static_cast<int64_t>(d) * kBytes, c < V ? D - d : 0, v);
#pragma unroll
      for (int e = 0; e < kPer; ++e) v[e] *= scale;
      store_vals<BF>(dst + static_cast<int64_t>(d) * kBytes, D - d, v);
    }
  }
}

// ---- sorting -------------------------------------------------------------------------------

// Short workgroups run best (1.2 GB: 16 bytes a thread 187 us, 128 bytes 210); very long clears take more of
// them in turn, so that a grid's threads stay below 2^32.
__device__ __forceinline__ void clear_share(void* p, int64_t bytes, int64_t block, int64_t blocks, int threads) {
  char* const q = static_cast<char*>(p);
  for (int64_t i = (block * threads + threadIdx.x) * 16; i < bytes; i += blocks * threads * 16) {
    if (bytes - i >= 16) __builtin_nontemporal_store(u32x4{0u, 0u, 0u, 0u}, reinterpret_cast<Piece*>(q + i));
    else
      for (int64_t b = i; b < bytes; b += 2) *reinterpret_cast<uint16_t*>(q + b) = 0;
  }
}

// keys[p], perm[p]: class and place of the p-th token in the order of (class, place).  64 tokens a
// workgroup, a lane each in every wavefront; wavefront w counts the tokens of its share (a whole number
// of 64, in LDS, the same in every lane) that come before.  Two instructions a compare: 11,458 tokens 10 us.
// The workgroups past the first `ranks` clear `bytes` at `zero` meanwhile (1.2 GB take 187 us).
template <bool I64>
__global__ void __launch_bounds__(kSortThreads)
rank_tokens(const void* __restrict__ tokens, int N, int V, int32_t* __restrict__ keys, int32_t* __restrict__ perm,
            int ranks, void* zero, int64_t bytes) {
  extern __shared__ __attribute__((aligned(16))) int32_t shares[];
  __shared__ int32_t count[kSortWaves][64];
  if (static_cast<int>(blockIdx.x) >= ranks) {
    clear_share(zero, bytes, blockIdx.x - ranks, gridDim.x - ranks, kSortThreads);
    return;
  }
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g0 = blockIdx.x * 64, i = g0 + lane;
  const int own = i < N ? class_of<I64>(tokens, i, V) : V;
  const int share = rank_share(N);
  const int jb = wave * share, je = jb + share;
  int32_t* const mine = shares + jb;
  for (int j = jb + lane; j < je; j += 64) mine[j - jb] = j < N ? class_of<I64>(tokens, j, V) : 0x7fffffff;
  __syncthreads();
  int before = 0;
  const int j1 = min(max(g0, jb), je), j2 = min(max(g0 + 64, jb), je);
  auto four = [&](int j) { return *reinterpret_cast<const int4*>(mine + (j - jb)); };
#pragma unroll 4
  for (int j = jb; j < j1; j += 4) {
    const int4 k = four(j);
    before += (k.x <= own) + (k.y <= own) + (k.z <= own) + (k.w <= own);
  }
  for (int j = j1; j < j2; ++j) {
    const int k = mine[j - jb];
    before += k < own || (k == own && j < i);
  }
#pragma unroll 4
  for (int j = j2; j < je; j += 4) {
    const int4 k = four(j);
    before += (k.x < own) + (k.y < own) + (k.z < own) + (k.w < own);
  }
  count[wave][lane] = before;
  __syncthreads();
  if (wave == 0 && i < N) {
    int p = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) p += count[w][lane];
    keys[p] = own;
    perm[p] = i;
  }
}

// A radix pass: digit (key >> shift) & (bins - 1).  Tile b is `tile` consecutive places, a whole number of
// 64 for each of its 16 wavefronts.  The first pass takes its keys from the tokens (perm null).
struct SortPass {
  const void* tokens;
  const int32_t *keys_in, *perm_in;  // null in the first pass
  int32_t *keys_out, *perm_out;
  int32_t* hist;  // [tiles][bins]
  int N, V, shift, bits, tile, tiles;
};

template <bool I64>
__device__ __forceinline__ int key_at(const SortPass& P, int p) {
  return P.keys_in ? P.keys_in[p] : class_of<I64>(P.tokens, p, P.V);
}

template <bool I64>
__global__ void __launch_bounds__(kSortThreads)
radix_count(SortPass P) {
  __shared__ int32_t h[kMaxBins];
  const int bins = 1 << P.bits;
  for (int d = threadIdx.x; d < bins; d += kSortThreads) h[d] = 0;
  __syncthreads();
  const int b = blockIdx.x * P.tile, e = min(P.N, b + P.tile);
  for (int p = b + threadIdx.x; p < e; p += kSortThreads)
    atomicAdd(&h[(key_at<I64>(P, p) >> P.shift) & (bins - 1)], 1);
  __syncthreads();
  for (int d = threadIdx.x; d < bins; d += kSortThreads) P.hist[blockIdx.x * bins + d] = h[d];
}

// A thread a digit: its tokens in all tiles and in those before, and a scan over the digits, give the first
// place of the tile's tokens of the digit (at most kMaxTiles rows of counts, read from the caches; a launch
// of its own for the scan took 5 us).  Each wavefront counts its own share of the tile by digit, the counts
// become first places (over the wavefronts before it), and it goes through its share again in order, 64
// tokens at a time: lanes of the same digit are found by a ballot per bit.
template <bool I64>
__global__ void __launch_bounds__(kSortThreads)
radix_place(SortPass P) {
  __shared__ int32_t at[kSortWaves][kMaxBins];
  __shared__ int32_t wave_sum[kSortWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int bins = 1 << P.bits;
  static_assert(kSortThreads >= kMaxBins, "a thread a digit");
  const int digit0 = threadIdx.x;
  int total = 0, earlier = 0;
  if (digit0 < bins) {
#pragma unroll 16
    for (int t = 0; t < P.tiles; ++t) {
      const int n = P.hist[t * bins + digit0];
      total += n;
      earlier += t < static_cast<int>(blockIdx.x) ? n : 0;
    }
  }
  int incl = total;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int x = __shfl_up(incl, o, 64);
    if (lane >= o) incl += x;
  }
  if (lane == 63) wave_sum[wave] = incl;
  for (int d = threadIdx.x; d < kSortWaves * bins; d += kSortThreads) at[d / bins][d % bins] = 0;
  __syncthreads();
  const int share = P.tile / kSortWaves;
  const int b = blockIdx.x * P.tile + wave * share, e = min(P.N, b + share);
  for (int p = b + lane; p < e; p += 64) atomicAdd(&at[wave][(key_at<I64>(P, p) >> P.shift) & (bins - 1)], 1);
  __syncthreads();
  if (digit0 < bins) {
    int first = incl - total + earlier;
    for (int w = 0; w < wave; ++w) first += wave_sum[w];
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      const int n = at[w][threadIdx.x];
      at[w][threadIdx.x] = first;
      first += n;
    }
  }
  __syncthreads();
  for (int p0 = b; p0 < e; p0 += 64) {
    const int p = p0 + lane;
    const bool live = p < e;
    const int key = live ? key_at<I64>(P, p) : 0;
    const int from = live ? (P.perm_in ? P.perm_in[p] : p) : 0;
    const int digit = (key >> P.shift) & (bins - 1);
    uint64_t same = __ballot(live);
    for (int q = 0; q < P.bits; ++q) {
      const bool bit = (digit >> q) & 1;
      const uint64_t m = __ballot(bit);
      same &= bit ? m : ~m;
    }
    if (live) {
      const int rank = __popcll(same & ((uint64_t{1} << lane) - 1));
      const int to = at[wave][digit] + rank;
      P.keys_out[to] = key;
      P.perm_out[to] = from;
      // the last lane of a digit moves its counter on, once every lane has read it
      wave_exchange();
      if ((same >> lane) == 1) at[wave][digit] = to + 1;
    }
    wave_exchange();  // before the next 64 read it
  }
}

// ---- sums ----------------------------------------------------------------------------------

constexpr int kVals = 8;  // columns a lane

struct SumArgs {
  const void* dy;
  const int32_t *keys, *perm;
  void* dW;
  float* part;  // [ranges][2][D]: the sum of a class that began before the range, and of one that goes on behind it
  int N, V, D, range, ranges, lanes;
  float scale;
  bool accumulate;
};

template <bool OBF>
__device__ __forceinline__ void put_row(const SumArgs& A, int c, int d, const float (&s)[kVals]) {
  char* o = static_cast<char*>(A.dW) + (static_cast<int64_t>(c) * A.D + d) * (OBF ? 2 : 4);
  float v[kVals];
#pragma unroll
  for (int e = 0; e < kVals; ++e) v[e] = s[e] * A.scale;
  if (A.accumulate) {
    float w[kVals];
    load_vals<OBF>(o, A.D - d, w);
#pragma unroll
    for (int e = 0; e < kVals; ++e) v[e] = fmaf(s[e], A.scale, w[e]);
  }
  store_vals<OBF>(o, A.D - d, v);
}

__device__ __forceinline__ void put_part(const SumArgs& A, int range, int slot, int d, const float (&s)[kVals]) {
  store_vals<false>(A.part + (static_cast<int64_t>(range) * 2 + slot) * A.D + d, A.D - d, s);
}

// A range of sorted places, `lanes` lanes of 8 columns each; blockIdx.y: columns.  Four rows are read ahead.  11,458
// rows of 4,096 in bf16 25 us; 65,536 of 1,024 added to float rows 84 (294 MB, 3.5 TB/s: one round of workgroups, each a
// chain of steps that stops at every class for a row of dW).
template <bool BF, bool OBF>
__global__ void __launch_bounds__(kThreads)
embedding_sum(SumArgs A) {
  const int r = blockIdx.x * (kThreads / A.lanes) + threadIdx.x / A.lanes;
  const int d = (blockIdx.y * A.lanes + threadIdx.x % A.lanes) * kVals;
  if (r >= A.ranges || d >= A.D) return;
  const int b = r * A.range, e = min(A.N, b + A.range);
  int c = A.keys[b];
  bool head = b > 0 && A.keys[b - 1] == c;  // the class began in an earlier range
  float s[kVals] = {};
  constexpr int kAhead = 4;
  for (int p0 = b; p0 < e; p0 += kAhead) {
    float x[kAhead][kVals];
    int key[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int p = p0 + k;
      key[k] = p < e ? A.keys[p] : -1;
      const int64_t row = p < e ? A.perm[p] : 0;
      load_vals<BF>(static_cast<const char*>(A.dy) + (row * A.D + d) * (BF ? 2 : 4),
                    (p < e && key[k] < A.V) ? A.D - d : 0, x[k]);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (key[k] < 0) break;
      if (key[k] != c) {
        if (c < A.V) {
          if (head) put_part(A, r, 0, d, s);
          else put_row<OBF>(A, c, d, s);
        }
        c = key[k];
        head = false;
#pragma unroll
        for (int q = 0; q < kVals; ++q) s[q] = 0.f;
      }
#pragma unroll
      for (int q = 0; q < kVals; ++q) s[q] += x[k][q];
    }
  }
  if (c >= A.V) return;
  const bool tail = e < A.N && A.keys[e] == c;  // it goes on in the next range
  if (head) put_part(A, r, 0, d, s);
  else if (tail) put_part(A, r, 1, d, s);
  else put_row<OBF>(A, c, d, s);
}

// The classes that lie in several ranges, by the range in which each begins (blockIdx.x).  32 lanes take
// 8 columns each, and the ranges in eight runs, whose sums are added in order: a class that has most of the
// tokens lies in hundreds of ranges (65,536 tokens of D = 1,024: 16 us for even classes, 48 for one).
template <bool OBF>
__global__ void __launch_bounds__(kThreads)
embedding_join(SumArgs A) {
  constexpr int kRuns = kThreads / 32;
  __shared__ float part[kRuns][32][kVals];
  const int lane = threadIdx.x & 31, run = threadIdx.x >> 5;
  const int d = (blockIdx.y * 32 + lane) * kVals;
  for (int r = blockIdx.x; r < A.ranges - 1; r += gridDim.x) {  // (the same for the whole workgroup)
    const int b = r * A.range, e = b + A.range;
    const int c = A.keys[e - 1];
    if (c >= A.V || A.keys[e] != c || (b > 0 && A.keys[b - 1] == c && A.keys[b] == c)) continue;
    // the last range with the class: the first place past it by bisection (keys rise)
    int lo = e, hi = A.N;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (A.keys[mid] <= c) lo = mid + 1;
      else hi = mid;
    }
    const int last = (lo - 1) / A.range;
    const int per = (last - r + 1 + kRuns - 1) / kRuns;
    float s[kVals] = {};
    if (d < A.D) {
      const int qb = r + run * per, qe = min(last + 1, qb + per);
#pragma unroll 4
      for (int q = qb; q < qe; ++q) {  // its first part is the second of range r, then the first of each
        float x[kVals];
        load_vals<false>(A.part + (static_cast<int64_t>(q) * 2 + (q == r)) * A.D + d, A.D - d, x);
#pragma unroll
        for (int k = 0; k < kVals; ++k) s[k] += x[k];
      }
    }
#pragma unroll
    for (int k = 0; k < kVals; ++k) part[run][lane][k] = s[k];
    __syncthreads();
    if (run == 0 && d < A.D) {
#pragma unroll
      for (int g = 1; g < kRuns; ++g)
#pragma unroll
        for (int k = 0; k < kVals; ++k) s[k] += part[g][lane][k];
      put_row<OBF>(A, c, d, s);
    }
    __syncthreads();  // before the next range's sums
  }
}

__global__ void __launch_bounds__(kThreads) fill_zero(void* p, int64_t bytes) {
  clear_share(p, bytes, blockIdx.x, gridDim.x, kThreads);
}

// Workgroups that clear.
unsigned clear_blocks(int64_t bytes, int threads) {
  const int64_t each = threads * 16;
  return static_cast<unsigned>(std::min<int64_t>((bytes + each - 1) / each, (int64_t{1} << 31) / threads));
}

int lanes_for(int pieces) {
  int l = 1;
  while (l < pieces && l < kThreads) l <<= 1;
  return l;
}

// Places of a range: as short as keeps its partial rows few beside the rows it reads; short where a row has
// few lanes, and ranges alone fill the chip.
int range_of(int N, int D) {
  if (lanes_for((D + kVals - 1) / kVals) < 32) return 8;
  return N >= 16384 ? 32 : N >= 1024 ? 16 : 8;
}

struct Layout {
  size_t o_keys, o_perm, o_keys2, o_perm2, o_hist, o_part, total;
};
Layout layout(int N, int D) {
  Layout L{};
  const size_t n = align_up(static_cast<size_t>(N > 0 ? N : 1) * 4, 256);
  L.o_keys = 0;
  L.o_perm = n;
  L.o_keys2 = 2 * n;
  L.o_perm2 = 3 * n;
  L.o_hist = N > kRankTokens ? 4 * n : 2 * n;
  L.o_part = L.o_hist + (N > kRankTokens ? static_cast<size_t>(kMaxTiles) * kMaxBins * 4 : 0);
  const int range = range_of(N, D);
  const size_t ranges = static_cast<size_t>((static_cast<int64_t>(N) + range - 1) / range);
  L.total = L.o_part + align_up((ranges > 1 ? ranges : 0) * 2 * D * sizeof(float), 256);
  return L;
}

}  // namespace

hipError_t launch_clear(void* p, int64_t bytes, hipStream_t stream) {
  Prof pr("clear", stream);
  if (bytes > 0)
    hipLaunchKernelGGL(fill_zero, dim3(clear_blocks(bytes, kThreads)), dim3(kThreads), 0, stream, p, bytes);
  return hipGetLastError();
}

hipError_t launch_embedding(int dtype, const void* table, int V, int D, const void* tokens, bool i64, int64_t N,
                            float scale, void* y, hipStream_t stream) {
  const int per = dtype == 1 ? 8 : 4;
  const int lanes = lanes_for((D + per - 1) / per), rows = kThreads / lanes;
  const dim3 grid(static_cast<unsigned>(std::min((N + rows - 1) / rows, kMaxGrid)));
  Prof pr("embedding", stream);
#define PCTC_EMBED(BF, I64)                                                                                      \
  hipLaunchKernelGGL((embedding_kernel<BF, I64>), grid, dim3(kThreads), 0, stream, table, V, D, tokens, N, scale, \
                     lanes, y)
  if (dtype == 1) {
    if (i64) PCTC_EMBED(true, true);
    else PCTC_EMBED(true, false);
  } else {
    if (i64) PCTC_EMBED(false, true);
    else PCTC_EMBED(false, false);
  }
#undef PCTC_EMBED
  return hipGetLastError();
}

size_t embedding_backward_bytes(int N, int D) { return layout(N, D).total; }

// Sorted keys and places at the start of the workspace; `bytes` at `zero` are cleared too (0: nothing).
static hipError_t sort_tokens(const void* tokens, bool i64, int N, int V, char* ws, const Layout& L, void* zero,
                              int64_t bytes, hipStream_t stream) {
  auto at = [&](size_t o) { return reinterpret_cast<int32_t*>(ws + o); };
  if (N <= kRankTokens) {
    Prof pr("embedding_rank", stream);
    const int ranks = (N + 63) / 64;
    const dim3 grid(ranks + clear_blocks(bytes, kSortThreads));
    const size_t lds = static_cast<size_t>(kSortWaves) * rank_share(N) * 4;
    if (i64)
      hipLaunchKernelGGL(rank_tokens<true>, grid, dim3(kSortThreads), lds, stream, tokens, N, V, at(L.o_keys),
                         at(L.o_perm), ranks, zero, bytes);
    else
      hipLaunchKernelGGL(rank_tokens<false>, grid, dim3(kSortThreads), lds, stream, tokens, N, V, at(L.o_keys),
                         at(L.o_perm), ranks, zero, bytes);
    return hipGetLastError();
  }
  if (bytes > 0) {
    const hipError_t e = launch_clear(zero, bytes, stream);
    if (e != hipSuccess) return e;
  }
  int bits = 1;
  while ((V >> bits) != 0) ++bits;  // keys reach V
  const int passes = (bits + kMaxBits - 1) / kMaxBits, per = (bits + passes - 1) / passes;
  SortPass P{};
  P.tokens = tokens;
  P.hist = at(L.o_hist);
  P.N = N;
  P.V = V;
  P.bits = per;
  const int unit = 64 * kSortWaves;
  P.tile = std::max(unit, static_cast<int>((static_cast<int64_t>(N) + kMaxTiles * unit - 1) / (kMaxTiles * unit)) * unit);
  P.tiles = (N + P.tile - 1) / P.tile;
  for (int q = 0; q < passes; ++q) {
    const bool last = q == passes - 1;
    // the last pass writes the places that the sums read
    P.keys_out = at(last ? L.o_keys : L.o_keys2);
    P.perm_out = at(last ? L.o_perm : L.o_perm2);
    P.shift = q * per;
    Prof pr("embedding_sort", stream);
    if (i64) hipLaunchKernelGGL(radix_count<true>, dim3(P.tiles), dim3(kSortThreads), 0, stream, P);
    else hipLaunchKernelGGL(radix_count<false>, dim3(P.tiles), dim3(kSortThreads), 0, stream, P);
    if (i64) hipLaunchKernelGGL(radix_place<true>, dim3(P.tiles), dim3(kSortThreads), 0, stream, P);
    else hipLaunchKernelGGL(radix_place<false>, dim3(P.tiles), dim3(kSortThreads), 0, stream, P);
    P.keys_in = P.keys_out;
    P.perm_in = P.perm_out;
  }
  return hipGetLastError();
}

hipError_t launch_embedding_backward(int dtype, const void* dy, const void* tokens, bool i64, int N, int V, int D,
                                     float scale, int out_dtype, void* dW, bool accumulate, void* workspace,
                                     hipStream_t stream) {
  const int64_t bytes = accumulate ? 0 : static_cast<int64_t>(V) * D * (out_dtype == 1 ? 2 : 4);
  if (N == 0) return bytes > 0 ? launch_clear(dW, bytes, stream) : hipSuccess;
  const Layout L = layout(N, D);
  char* ws = static_cast<char*>(workspace);
  hipError_t e = sort_tokens(tokens, i64, N, V, ws, L, dW, bytes, stream);
  if (e != hipSuccess) return e;
  SumArgs A{};
  A.dy = dy;
  A.keys = reinterpret_cast<const int32_t*>(ws + L.o_keys);
  A.perm = reinterpret_cast<const int32_t*>(ws + L.o_perm);
  A.dW = dW;
  A.part = reinterpret_cast<float*>(ws + L.o_part);
  A.N = N;
  A.V = V;
  A.D = D;
  A.range = range_of(N, D);
  A.ranges = (N + A.range - 1) / A.range;
  A.lanes = lanes_for((D + kVals - 1) / kVals);
  A.scale = scale;
  A.accumulate = accumulate;
  const int per = kThreads / A.lanes;
  const dim3 grid((A.ranges + per - 1) / per, (D + A.lanes * kVals - 1) / (A.lanes * kVals));
  {
    Prof pr("embedding_sum", stream);
#define PCTC_SUM(BF, OBF) hipLaunchKernelGGL((embedding_sum<BF, OBF>), grid, dim3(kThreads), 0, stream, A)
    if (dtype == 1) {
      if (out_dtype == 1) PCTC_SUM(true, true);
      else PCTC_SUM(true, false);
    } else {
      if (out_dtype == 1) PCTC_SUM(false, true);
      else PCTC_SUM(false, false);
    }
#undef PCTC_SUM
  }
  if (A.ranges > 1) {
    Prof pr("embedding_join", stream);
    const dim3 joins(std::min(A.ranges - 1, 1 << 18), (D + 32 * kVals - 1) / (32 * kVals));
    if (out_dtype == 1) hipLaunchKernelGGL(embedding_join<true>, joins, dim3(kThreads), 0, stream, A);
    else hipLaunchKernelGGL(embedding_join<false>, joins, dim3(kThreads), 0, stream, A);
  }
  return hipGetLastError();
}

}  // namespace pctc
