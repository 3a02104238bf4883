// CTC prefix beam search on candidate classes (gfx950): the selection over beams and classes, the
// label sequences of the beams, and the reordering of a caller's per-beam state.
//
// A beam is a label prefix y with the log masses pb and pn of its alignments that end in blank and
// in y's last label, relative to the best beam's total (an offset per utterance, in double, holds
// the rest); s = pb (+) pn, where (+) adds masses.  A frame offers blank (score b) and C classes
// (scores l, descending); w is added per label.  With l(c) = -inf for a class that is not offered:
//   stay    pb' = s + b,  pn' = (pn + l(last)) (+) (x_p + l(last) + w)   over the beam p, if any,
//           whose prefix is y without its last label; x_p = pb_p if p ends in that label too, else s_p
//   grow    by class c, unless that prefix is a beam already:  pn' = x + l(c) + w, x = pb if c = last
//           else s;  pb' = -inf
// The K largest totals are kept, ties in the order: staying beams, then grown ones by (beam, class).
//
// What bounds it: a chain of dependent frames, each a chain of K selections; memory and arithmetic
// are negligible.  One wavefront per utterance keeps everything in registers: lane i holds beam
// i mod KT; lanes [0, KT) offer the staying beams, lanes [KT, 2 KT) the best class by which their beam
// can still grow (the classes come sorted, so a beam's next best is the next bit of a mask of
// classes, and only 2 KT values take part in a selection whatever C is).  Prefixes are compared by
// 64-bit hashes of their labels and their lengths: two different ones meet with a probability of
// about K^2 / 2^65 per frame.
#include <algorithm>
#include <type_traits>

#include "pctc_internal.h"

namespace pctc {

namespace {

constexpr float kNegInf = -INFINITY;
constexpr int kCkStep = 32;  // labels between two nodes that remember the one before (result kernel)

__device__ __forceinline__ float log_add(float a, float b) {
  const float hi = fmaxf(a, b), lo = fminf(a, b);
  if (hi == kNegInf) return kNegInf;
  return hi + kLn2 * fast_log2(1.f + fast_exp2((lo - hi) * kLog2e));
}

__device__ __forceinline__ uint64_t grow_hash(uint64_t h, int label) {
  h = (h ^ static_cast<uint32_t>(label + 1)) * 0x9fb21c651e98df25ull;
  h ^= h >> 29;
  h = h * 0xd6e8feb86659fd93ull + 0x2545f4914f6cdd1dull;
  return h ^ (h >> 32);
}

__device__ __forceinline__ float lane_f(float x, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane));
}

// Maximum over lanes [0, W), W = 8, 16, 32 or 64, in every lane.
template <int W>
__device__ __forceinline__ float lanes_max(float x) {
  auto step = [&](auto ctrl) {
    const int v = __builtin_amdgcn_update_dpp(__float_as_int(x), __float_as_int(x), decltype(ctrl)::value, 0xf, 0xf,
                                              false);
    x = fmaxf(x, __int_as_float(v));
  };
  step(std::integral_constant<int, 0x111>{});  // from one, two, four, eight lanes below in the row of 16
  step(std::integral_constant<int, 0x112>{});
  step(std::integral_constant<int, 0x114>{});
  if constexpr (W >= 16) step(std::integral_constant<int, 0x118>{});
  if constexpr (W >= 32) step(std::integral_constant<int, 0x142>{});  // a row's last lane to the next row
  if constexpr (W >= 64) step(std::integral_constant<int, 0x143>{});  // lane 31 to the upper half
  return lane_f(x, W - 1);
}

// The beams of N utterances between frames.  node: the newest node of the prefix (-1: empty); ck: its
// newest node at a multiple of kCkStep labels.
struct BeamFields {
  float *pb, *pn, *s;  // s: their sum, kept as the selection had it
  uint64_t *hash, *phash;
  int32_t *last, *len, *node, *ck;
  double* offset;  // [N]
  int2* nodes;     // [N][cap] {node of the prefix before, label}
  int32_t* cks;    // [N][cap] of a node at a multiple of kCkStep labels: the one kCkStep labels before
  int64_t cap;
};

}  // namespace

size_t beam_state_layout(int N, int K, int max_frames, size_t (&at)[12]) {
  const size_t nk = static_cast<size_t>(N) * K, cap = static_cast<size_t>(max_frames) * K;
  const size_t sizes[12] = {nk * 4, nk * 4, nk * 4, nk * 8, nk * 8, nk * 4, nk * 4, nk * 4, nk * 4,
                            static_cast<size_t>(N) * 8, N * cap * sizeof(int2), N * cap * 4};
  size_t o = 0;
  for (int i = 0; i < 12; ++i) {
    at[i] = o;
    o += align_up(sizes[i] > 0 ? sizes[i] : 1, 256);
  }
  return o;
}

static BeamFields beam_fields(void* state, int N, int K, int max_frames) {
  size_t at[12];
  beam_state_layout(N, K, max_frames, at);
  char* s = static_cast<char*>(state);
  BeamFields f;
  f.pb = reinterpret_cast<float*>(s + at[0]);
  f.pn = reinterpret_cast<float*>(s + at[1]);
  f.s = reinterpret_cast<float*>(s + at[2]);
  f.hash = reinterpret_cast<uint64_t*>(s + at[3]);
  f.phash = reinterpret_cast<uint64_t*>(s + at[4]);
  f.last = reinterpret_cast<int32_t*>(s + at[5]);
  f.len = reinterpret_cast<int32_t*>(s + at[6]);
  f.node = reinterpret_cast<int32_t*>(s + at[7]);
  f.ck = reinterpret_cast<int32_t*>(s + at[8]);
  f.offset = reinterpret_cast<double*>(s + at[9]);
  f.nodes = reinterpret_cast<int2*>(s + at[10]);
  f.cks = reinterpret_cast<int32_t*>(s + at[11]);
  f.cap = static_cast<int64_t>(max_frames) * K;
  return f;
}

// Every utterance: the empty prefix with mass 1 in the first beam, the others empty-handed.
__global__ void __launch_bounds__(256) beam_reset_kernel(BeamFields f, int N, int K) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
  if (i < N) f.offset[i] = 0.0;
  if (i >= static_cast<int64_t>(N) * K) return;
  const bool root = i % K == 0;
  f.pb[i] = root ? 0.f : kNegInf;
  f.pn[i] = kNegInf;
  f.s[i] = root ? 0.f : kNegInf;
  f.hash[i] = 0;
  f.phash[i] = 0;
  f.last[i] = -2;
  f.len[i] = root ? 0 : -2;  // a beam without a prefix has length -2: it neither has nor is a prefix of another
  f.node[i] = -1;
  f.ck[i] = -1;
}

// KT: beams rounded up to 4, 8, 16 or 32.
template <int KT>
__global__ void __launch_bounds__(64)
beam_advance_kernel(FrameRows rows, int n0, int K, int C, const int32_t* __restrict__ ids,
                    const float* __restrict__ logp, const float* __restrict__ blank_logp, float bonus, BeamFields f,
                    int32_t* __restrict__ parents) {
  __shared__ float lp_s[64];
  __shared__ int32_t id_s[64];
  const int lane = threadIdx.x, i = lane & (KT - 1);
  const bool stays = lane < KT, grows = lane >= KT && lane < 2 * KT;
  const int n = n0 + blockIdx.x;
  const int t0 = rows.off[blockIdx.x], t1 = rows.off[blockIdx.x + 1];
  int frame = rows.done[blockIdx.x];  // frames before this one
  const int64_t at = static_cast<int64_t>(n) * K + i;
  float pb = kNegInf, pn = kNegInf, s = kNegInf;
  uint64_t hash = 0, phash = 0;
  int last = -2, len = -2, node = -1, ck = -1;
  if (i < K) {
    pb = f.pb[at];
    pn = f.pn[at];
    s = f.s[at];
    hash = f.hash[at];
    phash = f.phash[at];
    last = f.last[at];
    len = f.len[at];
    node = f.node[at];
    ck = f.ck[at];
  }
  int2* const nodes = f.nodes + n * f.cap;
  int32_t* const cks = f.cks + n * f.cap;
  double offset = f.offset[n];
  int origin = i;

  // a frame's classes, one a lane; a score that is no number counts as -inf
  auto fetch = [&](int m, int& id, float& l, float& b) {
    id = -1;
    l = b = kNegInf;
    if (m >= t1) return;
    if (lane < C) {
      id = ids[static_cast<int64_t>(m) * C + lane];
      l = logp[static_cast<int64_t>(m) * C + lane];
    }
    b = blank_logp[m];
    if (id < 0 || !(l > kNegInf)) {
      id = -1;
      l = kNegInf;
    }
    if (!(b > kNegInf)) b = kNegInf;
  };
  int id, nid;
  float l, b, nl, nb;
  fetch(t0, id, l, b);
  for (int m = t0; m < t1; ++m, ++frame) {
    fetch(m + 1, nid, nl, nb);
    lp_s[lane] = l;
    id_s[lane] = id;
    __builtin_amdgcn_wave_barrier();
    const uint64_t offered = __ballot(id >= 0);
    // where each beam's last label stands among the classes, which beam is its prefix without that
    // label, and the classes by which a beam would grow into another
    uint64_t skip = 0;
    int pos = -1, par = -1;
#pragma unroll 8
    for (int j = 0; j < KT; ++j) {
      const int lj = __builtin_amdgcn_readlane(last, j), nj = __builtin_amdgcn_readlane(len, j);
      const uint32_t hl = __builtin_amdgcn_readlane(static_cast<uint32_t>(phash), j);
      const uint32_t hh = __builtin_amdgcn_readlane(static_cast<uint32_t>(phash >> 32), j);
      const uint64_t pm = __ballot(id == lj);
      const bool into = len + 1 == nj && hash == ((static_cast<uint64_t>(hh) << 32) | hl) && i != j;
      const uint64_t im = __ballot(into) & ((uint64_t{1} << KT) - 1);
      if (into) skip |= pm;
      if (i == j) {
        pos = pm ? __builtin_ctzll(pm) : -1;
        par = im ? __builtin_ctzll(im) : -1;
      }
    }
    const float l_last = pos >= 0 ? lp_s[pos] : kNegInf;
    const int p = par >= 0 ? par : 0;
    const float pb_p = __shfl(pb, p, 64), s_p = __shfl(s, p, 64);
    const int last_p = __shfl(last, p, 64);
    const float join = par >= 0 ? (last_p == last ? pb_p : s_p) + (l_last + bonus) : kNegInf;
    const float sb = s + b, sn = log_add(pn + l_last, join);
    // this lane's offer: a staying beam's total, or the best class left to grow by
    const uint64_t own = pos >= 0 ? uint64_t{1} << pos : 0;
    uint64_t left = grows ? offered & ~skip & ~own : 0;
    float again = grows && (own & ~skip) ? pb + (l_last + bonus) : kNegInf;  // its last label once more
    int rank = 0;
    float val = kNegInf;
    auto offer = [&]() {
      const int r = left ? __builtin_ctzll(left) : 63;
      const float v = left ? s + (lp_s[r] + bonus) : kNegInf;
      const bool rep = again > v || (again == v && pos < r);
      rank = rep ? pos : r;
      val = rep ? again : v;
    };
    if (grows) offer();
    if (stays) val = log_add(sb, sn);
    float best = kNegInf, won = kNegInf;
    int src = -1, wrank = 0;
    for (int r = 0; r < K; ++r) {
      const float top = lanes_max<2 * KT>(val);
      const uint64_t who = __ballot(val == top) & (2 * KT == 64 ? ~uint64_t{0} : (uint64_t{1} << (2 * KT)) - 1);
      if (!(top > kNegInf) || who == 0) break;
      const int w = __builtin_ctzll(who);
      const int wr = __builtin_amdgcn_readlane(rank, w);
      if (r == 0) best = top;
      if (i == r) {
        src = w;
        won = top;
        wrank = wr;
      }
      if (lane == w) {
        if (stays) {
          val = kNegInf;
        } else {
          if (rank == pos) again = kNegInf;
          else left &= left - 1;
          offer();
        }
      }
    }
    // the new beam i descends from beam src mod KT
    const bool grown = src >= KT, live = src >= 0;
    const int from = live ? src & (KT - 1) : 0;
    const float f_sb = __shfl(sb, from, 64), f_sn = __shfl(sn, from, 64);
    const uint64_t f_hash = __shfl(hash, from, 64), f_phash = __shfl(phash, from, 64);
    const int f_last = __shfl(last, from, 64), f_len = __shfl(len, from, 64), f_node = __shfl(node, from, 64);
    const int f_ck = __shfl(ck, from, 64), f_origin = __shfl(origin, from, 64);
    if (!live) {
      pb = pn = s = kNegInf;
      len = last = -2;
      origin = -1;
    } else {
      const int label = id_s[wrank];
      const int fresh = frame * K + i;
      pb = grown ? kNegInf : f_sb - best;
      pn = (grown ? won : f_sn) - best;
      s = won - best;
      hash = grown ? grow_hash(f_hash, label) : f_hash;
      phash = grown ? f_hash : f_phash;
      last = grown ? label : f_last;
      len = grown ? f_len + 1 : f_len;
      node = grown ? fresh : f_node;
      ck = f_ck;
      origin = f_origin;
      if (grown) {
        if (lane < KT) nodes[fresh] = make_int2(f_node, label);
        if (len % kCkStep == 0) {
          if (lane < KT) cks[fresh] = f_ck;
          ck = fresh;
        }
      }
    }
    if (best > kNegInf) offset += best;
    id = nid;
    l = nl;
    b = nb;
  }
  if (lane < KT && i < K) {
    f.pb[at] = pb;
    f.pn[at] = pn;
    f.s[at] = s;
    f.hash[at] = hash;
    f.phash[at] = phash;
    f.last[at] = last;
    f.len[at] = len;
    f.node[at] = node;
    f.ck[at] = ck;
    if (parents) parents[at] = len >= 0 ? origin : -1;
  }
  if (lane == 0) f.offset[n] = offset;
}

// One wavefront per beam: the labels of its prefix, -1 past them.  The nodes hang together newest
// first, a load behind a load; the nodes at multiples of kCkStep labels are visited first, and from
// each a lane of its own walks the kCkStep labels before it.
__global__ void __launch_bounds__(64)
beam_result_kernel(BeamFields f, int K, int max_tokens, int32_t* __restrict__ tokens, int32_t* __restrict__ lengths,
                   float* __restrict__ scores) {
  __shared__ int32_t start[64];
  const int lane = threadIdx.x;
  const int64_t at = blockIdx.x;
  const int n = static_cast<int>(at / K);
  const int len = f.len[at];
  const int2* const nodes = f.nodes + n * f.cap;
  const int32_t* const cks = f.cks + n * f.cap;
  int32_t* const out = tokens + at * max_tokens;
  for (int t = max(len, 0) + lane; t < max_tokens; t += 64) out[t] = -1;
  if (lane == 0) {
    lengths[at] = len >= 0 ? len : -1;
    scores[at] = len >= 0 ? static_cast<float>(f.offset[n] + f.s[at]) : kNegInf;
  }
  if (len <= 0) return;
  const int whole = len / kCkStep;
  int next = f.ck[at];
  // lanes [0, 63) take the whole segments, newest first, lane 63 the labels past them
  for (int seg = whole, first = 1; seg > 0 || first; seg -= 63, first = 0) {
    const int here = min(seg, 63);
    if (lane == 0) {
      for (int q = 0; q < here; ++q) {
        start[q] = next;
        next = cks[next];
      }
    }
    __syncthreads();
    int node = -1, from = 0, to = 0;  // labels [to, from), the last of them in node
    if (lane < here) {
      node = start[lane];
      from = (seg - lane) * kCkStep;
      to = from - kCkStep;
    } else if (lane == 63 && first) {
      node = f.node[at];
      from = len;
      to = whole * kCkStep;
    }
    for (int t = from - 1; t >= to; --t) {
      const int2 v = nodes[node];
      if (t < max_tokens) out[t] = v.y;
      node = v.x;
    }
    __syncthreads();
  }
}

// ---- reordering of per-beam state ---------------------------------------------------------

namespace {

constexpr int kReorderGroup = 64;  // tensors of a launch (their table is a kernel argument)
struct ReorderTable {
  const char* in[kReorderGroup];
  char* out[kReorderGroup];
  int64_t bytes[kReorderGroup];   // of one beam's state
  int64_t first[kReorderGroup + 1];  // columns of 4 KB of the tensors before
  int32_t tensors;
};
static_assert(sizeof(ReorderTable) <= 3600, "kernel arguments");

// 16 bytes at any address; unaligned vector accesses are ordinary ones on this target.
__device__ __forceinline__ u32x4 load16(const char* p) {
  u32x4 v;
  __builtin_memcpy(&v, p, 16);
  return v;
}
__device__ __forceinline__ void store16(char* p, const u32x4& v) { __builtin_memcpy(p, &v, 16); }

constexpr int kColBytes = 256 * 16;

}  // namespace

// Workgroup: 4 KB of the state of each beam of one utterance and tensor.  Every beam's piece is read
// before any is written, so that input and output may be the same memory.
template <int KT>
__global__ void __launch_bounds__(256)
beam_reorder_kernel(ReorderTable t, const int32_t* __restrict__ parents, int n0, int K) {
  const int64_t col = static_cast<int64_t>(blockIdx.x);
  const int n = n0 + blockIdx.y;
  int lo = 0, hi = t.tensors - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.first[mid] <= col) lo = mid;
    else hi = mid - 1;
  }
  const int64_t bytes = t.bytes[lo];
  const int64_t off = (col - t.first[lo]) * kColBytes + static_cast<int64_t>(threadIdx.x) * 16;
  if (off >= bytes) return;
  const char* const in = t.in[lo] + static_cast<int64_t>(n) * K * bytes + off;
  char* const out = t.out[lo] + static_cast<int64_t>(n) * K * bytes + off;
  const bool same = t.in[lo] == t.out[lo];
  // a beam without a parent (or with one that is none) keeps its own state
  auto parent = [&](int k) {
    const int p = parents[static_cast<int64_t>(n) * K + k];
    return p >= 0 && p < K ? p : k;
  };
  if (off + 16 <= bytes) {
    u32x4 v[KT];
#pragma unroll
    for (int k = 0; k < KT; ++k) {
      v[k] = u32x4{0u, 0u, 0u, 0u};
      if (k < K) {
        const int p = parent(k);
        if (!same || p != k) v[k] = load16(in + p * bytes);
      }
    }
#pragma unroll
    for (int k = 0; k < KT; ++k)
      if (k < K && (!same || parent(k) != k)) store16(out + k * bytes, v[k]);
  } else {
    for (int64_t e = 0; off + e < bytes; ++e) {
      int v[KT];
#pragma unroll
      for (int k = 0; k < KT; ++k) v[k] = k < K ? in[parent(k) * bytes + e] : 0;
#pragma unroll
      for (int k = 0; k < KT; ++k)
        if (k < K) out[k * bytes + e] = static_cast<char>(v[k]);
    }
  }
}

// ---- launchers ------------------------------------------------------------------------------

hipError_t launch_beam_reset(void* state, int N, int K, int max_frames, hipStream_t stream) {
  if (N <= 0) return hipSuccess;
  Prof pr("beam_reset", stream);
  const int64_t nk = static_cast<int64_t>(N) * K;
  hipLaunchKernelGGL(beam_reset_kernel, dim3(static_cast<unsigned>((nk + 255) / 256)), dim3(256), 0, stream,
                     beam_fields(state, N, K, max_frames), N, K);
  return hipGetLastError();
}

hipError_t launch_beam_advance(const int32_t* ids, const float* logp, const float* blank_logp, int C,
                               const int32_t* frames, int N, int K, int max_frames, float bonus,
                               const int32_t* done, void* state, int32_t* parents, hipStream_t stream) {
  const BeamFields f = beam_fields(state, N, K, max_frames);
  int32_t row = 0;
  for (int n0 = 0; n0 < N; n0 += kBeamGroup) {
    const int here = std::min(kBeamGroup, N - n0);
    FrameRows rows{};
    for (int q = 0; q < here; ++q) {
      rows.off[q] = row;
      rows.done[q] = done ? done[n0 + q] : 0;
      row += frames[n0 + q];
    }
    rows.off[here] = row;
    Prof pr("beam_advance", stream);
#define PCTC_ADVANCE(KT)                                                                                        \
  hipLaunchKernelGGL(beam_advance_kernel<KT>, dim3(here), dim3(64), 0, stream, rows, n0, K, C, ids, logp,       \
                     blank_logp, bonus, f, parents)
    if (K <= 4) PCTC_ADVANCE(4);
    else if (K <= 8) PCTC_ADVANCE(8);
    else if (K <= 16) PCTC_ADVANCE(16);
    else PCTC_ADVANCE(32);
#undef PCTC_ADVANCE
  }
  return hipGetLastError();
}

hipError_t launch_beam_result(void* state, int N, int K, int max_frames, int max_tokens, int32_t* tokens,
                              int32_t* lengths, float* scores, hipStream_t stream) {
  if (N <= 0) return hipSuccess;
  Prof pr("beam_result", stream);
  hipLaunchKernelGGL(beam_result_kernel, dim3(static_cast<unsigned>(N * K)), dim3(64), 0, stream,
                     beam_fields(state, N, K, max_frames), K, max_tokens, tokens, lengths, scores);
  return hipGetLastError();
}

hipError_t launch_beam_reorder(int tensors, const void* const* in, void* const* out, const int64_t* beam_bytes,
                               const int32_t* parents, int N, int K, hipStream_t stream) {
  for (int k0 = 0; k0 < tensors; k0 += kReorderGroup) {
    ReorderTable t{};
    t.tensors = std::min(kReorderGroup, tensors - k0);
    int64_t c = 0;
    for (int k = 0; k < t.tensors; ++k) {
      t.in[k] = static_cast<const char*>(in[k0 + k]);
      t.out[k] = static_cast<char*>(out ? out[k0 + k] : const_cast<void*>(in[k0 + k]));
      t.bytes[k] = beam_bytes[k0 + k];
      t.first[k] = c;
      c += (beam_bytes[k0 + k] + kColBytes - 1) / kColBytes;
    }
    t.first[t.tensors] = c;
    if (c == 0) continue;
    Prof pr("beam_reorder", stream);
    for (int n0 = 0; n0 < N; n0 += 65535) {
      const dim3 grid(static_cast<unsigned>(c), static_cast<unsigned>(std::min(65535, N - n0)));
#define PCTC_REORDER(KT) \
  hipLaunchKernelGGL(beam_reorder_kernel<KT>, grid, dim3(256), 0, stream, t, parents, n0, K)
      if (K <= 4) PCTC_REORDER(4);
      else if (K <= 8) PCTC_REORDER(8);
      else if (K <= 16) PCTC_REORDER(16);
      else PCTC_REORDER(32);
#undef PCTC_REORDER
    }
  }
  return hipGetLastError();
}

}  // namespace pctc
