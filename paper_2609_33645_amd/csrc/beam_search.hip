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
// What bounds it: a chain of dependent frames; memory and arithmetic are negligible.  16 utterances of 150 to
// 348 frames, K = 8, C = 16: 186 us (the median of 60), 0.53 us a frame of the longest (4 beams and 8 classes
// 0.54, 16 beams and 40 classes 0.83; a frame of a live stream by itself, launch included, 3.5 us).  A frame is
// 172 instructions of a wavefront alone on its SIMD, 7.6 cycles each (plain additions take 4, comparisons
// whose masks are used, cross-lane reads and branches more), and fewer instructions are what makes it faster:
// with the exchanges through the LDS taken off the chain it was no faster.  Several
// wavefronts to an utterance would wait at a barrier for each exchange.  One wavefront per
// utterance holds the beams in registers (lane l: beam l mod KT, the copies share out the comparisons
// over classes and beams), and every exchange is a cross-lane move or a wavefront's own LDS.
// Of the K (C + 1) totals few have to be looked at.  Beams and classes come sorted: with beam i (from 0)
// and class c (from 0), all of i' <= i, c' <= c but a beam's own last label have totals no smaller, as
// prefixes of their own, so that (i, c) can only be kept where (i + 1) c <= K (28 pairs for K = 8, 66 for
// 16, 151 for 32); and where all K beams can stay, only pairs above the least of their totals.  These
// few are ordered by counting, each lane the totals above its own.  A frame that none of them enters and
// that leaves the order as it is (most frames, where a head is sure) moves nothing, and one that does not
// offer any beam's last label either leaves every beam as it is: blank's score goes to the utterance's
// total.  Where the beams' last labels stand among the classes is looked up for 64 / KT frames at once
// (at most eight), a lane for each beam and frame.  Frames come from memory eight at a time, eight frames
// and more ahead of their use.
// Prefixes are compared by 64-bit hashes of their labels and their lengths: two different ones meet
// with a probability of about K^2 / 2^65 per frame.
#include <algorithm>
#include <type_traits>

#include "pctc_internal.h"

namespace pctc {

namespace {

constexpr float kNegInf = -INFINITY;
constexpr int kBufWord3 = 0x00020000;  // word 3 of a raw buffer resource: 32-bit data, no swizzle
constexpr int kCkStep = 16;  // labels between two nodes that remember the one before (result kernel)

constexpr float kLow = -3.4028235e38f;  // float's lowest: a reference that stays finite where all masses are zero

// Sums of two and of three masses; -inf where all are zero.
__device__ __forceinline__ float log_add(float a, float b) {
  const float hi = fmaxf(fmaxf(a, b), kLow);
  return hi + kLn2 * fast_log2(fast_exp2((a - hi) * kLog2e) + fast_exp2((b - hi) * kLog2e));
}
__device__ __forceinline__ float log_add(float a, float b, float c) {
  const float hi = fmaxf(fmaxf(a, b), fmaxf(c, kLow));
  return hi + kLn2 * fast_log2(fast_exp2((a - hi) * kLog2e) + fast_exp2((b - hi) * kLog2e) +
                               fast_exp2((c - hi) * kLog2e));
}

// 1 where x > y, for y above -inf (from the sign of the difference: a comparison's mask takes an addition
// several times as long).
__device__ __forceinline__ uint32_t above(float x, float y) { return __float_as_uint(y - x) >> 31; }

// What a lane wrote to the LDS before is there for the others after: a wavefront's LDS operations run in program
// order, and the fence keeps the compiler from reordering them or from taking a lane's own value for what it reads.
__device__ __forceinline__ void exchange() {
  __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

__device__ __forceinline__ uint64_t lanes_where(bool x) { return __builtin_amdgcn_ballot_w64(x); }

// The hash of a prefix with one more label.
__device__ __forceinline__ uint64_t grow_hash(uint64_t hash, int label) {
  uint64_t h = static_cast<uint32_t>(label + 1) * 0x9fb21c651e98df25ull;
  h = (h ^ (h >> 29)) * 0xd6e8feb86659fd93ull;
  h = (hash + (h ^ (h >> 32))) * 0x2545f4914f6cdd1dull;
  return h ^ (h >> 32);
}

__device__ __forceinline__ float lane_f(float x, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane));
}
__device__ __forceinline__ uint64_t from_lane(uint64_t x, int lane) {
  const uint32_t lo = __shfl(static_cast<int>(x), lane, 64), hi = __shfl(static_cast<int>(x >> 32), lane, 64);
  return (static_cast<uint64_t>(hi) << 32) | lo;
}

// The value of the lane below in the row of 16 (the first lane of a row keeps its own).
__device__ __forceinline__ float lane_below(float x) {
  return __int_as_float(
      __builtin_amdgcn_update_dpp(__float_as_int(x), __float_as_int(x), 0x111, 0xf, 0xf, false));
}

// Minimum over lanes [0, W), W = 4, 8, 16 or 32.
template <int W>
__device__ __forceinline__ float lanes_min(float x) {
  auto step = [&](auto ctrl) {
    const int v = __builtin_amdgcn_update_dpp(__float_as_int(x), __float_as_int(x), decltype(ctrl)::value, 0xf, 0xf,
                                              false);
    x = fminf(x, __int_as_float(v));
  };
  step(std::integral_constant<int, 0x111>{});  // from one, two, four, eight lanes below in the row of 16
  step(std::integral_constant<int, 0x112>{});
  if constexpr (W >= 8) step(std::integral_constant<int, 0x114>{});
  if constexpr (W >= 16) step(std::integral_constant<int, 0x118>{});
  if constexpr (W >= 32) step(std::integral_constant<int, 0x142>{});  // a row's last lane to the next row
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
beam_advance_kernel(FrameRows rows, int n0, int K, int C, bool fresh_start, const int32_t* __restrict__ ids,
                    const float* __restrict__ logp, const float* __restrict__ blank_logp, float bonus, BeamFields f,
                    int32_t* __restrict__ parents) {
  constexpr int kCopies = 64 / KT;                        // lanes of a beam
  constexpr int kPairs = KT <= 8 ? 1 : KT <= 16 ? 2 : 3;  // (beam, class) pairs a lane looks at
  constexpr int kBatches = KT <= 8 ? 1 : KT <= 16 ? 2 : 3;  // of 64 totals to be ordered (36, 82, 183 at most)
  constexpr int kAhead = 8;                               // frames fetched at a time
  constexpr int kRing = 32;                               // frames held
  constexpr int kLook = kCopies < 8 ? kCopies : 8;        // frames looked up at a time
  constexpr uint64_t kBeamBits = (uint64_t{1} << KT) - 1;
  constexpr uint64_t kEvery = KT == 4 ? 0x1111111111111111ull : KT == 8 ? 0x0101010101010101ull
                              : KT == 16 ? 0x0001000100010001ull : 0x0000000100000001ull;  // a beam's lanes
  __shared__ float lp_s[kRing][64];  // the classes of frame t0 + f in row f mod kRing, and blank's score
  __shared__ __attribute__((aligned(16))) int32_t id_s[kRing][64];
  __shared__ float bl_s[kRing];
  __shared__ int first_s[KT + 1];     // pairs of the beams before
  __shared__ int merged_s[64 * kPairs];  // frame (from 1) in which a pair's prefix was last a beam
  // totals to be ordered: staying beams, pairs
  __shared__ __attribute__((aligned(16))) float val_s[64 * kBatches + 16];
  __shared__ int what_s[64 * kBatches];  // of a pair: beam + 256 class
  __shared__ int2 place_s[KT];        // of each place: what, with bit 30 for a pair, and the total
  const int lane = threadIdx.x, i = lane & (KT - 1), copy = lane / KT;
  const int n = n0 + blockIdx.x;
  const int t0 = rows.off[blockIdx.x], t1 = rows.off[blockIdx.x + 1];
  const int done = rows.done[blockIdx.x];  // frames before this call
  const int64_t at = static_cast<int64_t>(n) * K + i;
  const bool mine = i < K;
  float pb = kNegInf, pn = kNegInf, s = kNegInf;
  uint64_t hash = 0, phash = 0;
  int last = -2, len = -2, node = -1, ck = -1;
  double offset = 0.0;
  if (fresh_start) {  // as beam_reset_kernel leaves it
    if (i == 0) {
      pb = s = 0.f;
      len = 0;
    }
  } else if (mine) {
    offset = f.offset[n];
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
  int origin = i;

  // the pairs that can be kept: classes c <= K / (i + 1) of beam i, beam by beam
  int first = 0, pairs;  // pairs of the beams before, and of all
  {
    // (a quotient that is no whole number is at least 1/32 away from one)
    const int classes = static_cast<int>(static_cast<float>(K) / static_cast<float>(lane + 1) + 0.01f) + 1;
    const int here = lane < K ? min(C, classes) : 0;
    int sum = here;
#pragma unroll
    for (int o = 1; o < KT; o <<= 1) {
      const int v = __shfl_up(sum, o, 64);
      if (lane >= o) sum += v;
    }
    pairs = __builtin_amdgcn_readlane(sum, K - 1);
    first = sum - here;
    if (lane < K) first_s[lane] = first;
    if (lane == 0) first_s[K] = pairs;
  }
  int pi[kPairs], pc[kPairs];  // beam and class of this lane's pairs (beam -1: none)
#pragma unroll
  for (int q = 0; q < kPairs; ++q) {
    const int e = lane + 64 * q;
    merged_s[e] = 0;
    pi[q] = -1;
    pc[q] = 0;
    for (int k = 0; k < K; ++k) {
      const int a = __builtin_amdgcn_readlane(first, k);
      if (e >= a && e < pairs) {
        pi[q] = k;
        pc[q] = e - a;
      }
    }
  }

  // eight frames' classes, one a lane, and (lanes [0, 8)) blank scores, through buffer resources that
  // end with the utterance (what lies past reads as zeros and is not used)
  int fid[kAhead];
  float fl[kAhead], fb;
  const int T = t1 - t0;
  auto fetch = [&](int f) {  // frames t0 + f ..
#if defined(__HIP_DEVICE_COMPILE__)  // the buffer-resource type exists on the device side only
    const int left = f < T ? min(T - f, kAhead) : 0;
    const int64_t at_row = static_cast<int64_t>(t0 + f) * C;
    auto resource = [&](const void* p, int values) {
      return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), static_cast<short>(0), values * 4, kBufWord3);
    };
    const __amdgpu_buffer_rsrc_t ri = resource(ids + at_row, left * C), rl = resource(logp + at_row, left * C),
                                 rb = resource(blank_logp + t0 + f, left);
#pragma unroll
    for (int g = 0; g < kAhead; ++g) {
      const int at_class = (g * C + lane) * 4;  // (the whole offset takes part in the range check)
      fid[g] = __builtin_amdgcn_raw_buffer_load_b32(ri, at_class, 0, 0);
      fl[g] = __int_as_float(__builtin_amdgcn_raw_buffer_load_b32(rl, at_class, 0, 0));
    }
    fb = __int_as_float(__builtin_amdgcn_raw_buffer_load_b32(rb, lane * 4, 0, 0));
#endif
  };
  const int no_class = lane < C ? 0 : -1;
  const uint64_t places = ~uint64_t{0} >> (64 - C);
  auto stage = [&](int f) {  // the same frames (f a multiple of 8)
    const int r0 = f & (kRing - 1);
    exchange();  // (the rows' frames before have been read)
    float x[kAhead], least = INFINITY;
#pragma unroll
    for (int g = 0; g < kAhead; ++g) {
      const int id = fid[g] | no_class;
      // all ones, no number, where the class is none; the maximum takes -inf for no number
      x[g] = fmaxf(__int_as_float(__float_as_int(fl[g]) | (id >> 31)), kNegInf);
      least = fminf(least, x[g]);
      lp_s[r0 + g][lane] = x[g];
      id_s[r0 + g][lane] = id;
    }
    if (lane < kAhead) bl_s[r0 + lane] = fmaxf(fb, kNegInf);
    // the pairs looked at go by a class's place among the classes there are, so empty places move behind them
    if (__builtin_expect(lanes_where(least > kNegInf) != places, 0)) {
      exchange();
#pragma unroll
      for (int g = 0; g < kAhead; ++g) {
        const uint64_t full = lanes_where(x[g] > kNegInf);
        const int before = __popcll(full & ((uint64_t{1} << lane) - 1));
        const int at = x[g] > kNegInf ? before : __popcll(full) + lane - before;
        lp_s[r0 + g][at] = x[g];
        id_s[r0 + g][at] = fid[g] | no_class;
      }
    }
    exchange();
  };
  // the beam whose prefix is this beam's without its last label
  auto find_parent = [&]() {
    int found = -1;
#pragma unroll
    for (int q = 0; q < (KT + kCopies - 1) / kCopies; ++q) {
      const int o = q * kCopies + copy;
      const uint64_t h = from_lane(hash, o & (KT - 1));
      const int ln = __shfl(len, o & (KT - 1), 64);
      if (o < KT && ln + 1 == len && h == phash) found = o;
    }
    const uint64_t who = (lanes_where(found >= 0) >> i) & kEvery;
    return __shfl(found, (who ? __builtin_ctzll(who) & ~(KT - 1) : 0) + i, 64);
  };

  int staged = 0;  // frames in the ring
  auto more = [&]() {
    stage(staged);
    staged += kAhead;
    fetch(staged);
  };
  if (T > 0) {
    fetch(0);
    more();
  }
  int par = -1;
  bool par_known = false;  // par is formed when a frame asks for it
  float ps[kPairs], ppb[kPairs];  // s and pb of the pairs' beams
  float floor_s;                  // s of the last beam
  auto spread = [&]() {
#pragma unroll
    for (int q = 0; q < kPairs; ++q) {
      ps[q] = __shfl(s, pi[q] & 63, 64);
      ppb[q] = __shfl(pb, pi[q] & 63, 64);
    }
    floor_s = lane_f(s, K - 1);
  };
  spread();
  // whether beam lane mod KT's last label is among the classes of frame looked + lane / KT, from differences
  // and their minimum (a comparison's mask takes a select several times as long)
  int looked = -kLook;
  uint64_t stands = 0;
  auto look = [&](int fr) {
    looked = fr;
    uint32_t x = 0xffffffffu;
    const int32_t* const r = id_s[(fr + copy) & (kRing - 1)];
    for (int c = 0; c < C; c += 16) {
      int4 v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = *reinterpret_cast<const int4*>(r + c + 4 * k);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        x = min(min(static_cast<uint32_t>(v[k].x ^ last), static_cast<uint32_t>(v[k].y ^ last)), x);
        x = min(min(static_cast<uint32_t>(v[k].z ^ last), static_cast<uint32_t>(v[k].w ^ last)), x);
      }
    }
    stands = lanes_where(x == 0);
  };
  // the frame at hand: its pairs' scores and blank's
  float pl[kPairs], bl = bl_s[0];
#pragma unroll
  for (int q = 0; q < kPairs; ++q) pl[q] = lp_s[0][pc[q]] + bonus;
  for (int fr = 0; fr < T; ++fr) {
    const int row = fr & (kRing - 1), row1 = (fr + 1) & (kRing - 1);
    if (staged < fr + kLook + 1) more();
    const float b = bl;
    float plb[kPairs];
#pragma unroll
    for (int q = 0; q < kPairs; ++q) plb[q] = pl[q];
    bl = bl_s[row1];
#pragma unroll
    for (int q = 0; q < kPairs; ++q) pl[q] = lp_s[row1][pc[q]] + bonus;
    if (fr >= looked + kLook) look(fr);
    const uint64_t met = (stands >> ((fr - looked) * KT)) & kBeamBits;  // beams whose last label is offered
    const float sb = s + b;
    float total, sn, pv[kPairs];
    uint64_t enter[kPairs], any = 0;
    if (met == 0) {
      // every beam can only end in blank, and their order stands
      const float least = floor_s + b;
#pragma unroll
      for (int q = 0; q < kPairs; ++q) {
        pv[q] = ps[q] + plb[q];
        enter[q] = lanes_where(pi[q] >= 0 & pv[q] > least);
        any |= enter[q];
      }
      if (any == 0 && b > kNegInf) {
        pb = s;
        pn = kNegInf;
#pragma unroll
        for (int q = 0; q < kPairs; ++q) ppb[q] = ps[q];
        offset += b;
        continue;
      }
      total = sb;
      sn = kNegInf;
    } else {
      if (!par_known) par = find_parent();
      par_known = true;
      const int p = par >= 0 ? par : i;
      const float pb_p = __shfl(pb, p, 64), s_p = __shfl(s, p, 64);
      const int last_p = __shfl(last, p, 64);
      // where the beams' last labels stand, label by label
      int pos = -1;
      const int id_now = id_s[row][lane];
      for (uint64_t todo = met; todo != 0;) {
        const int label = __builtin_amdgcn_readlane(last, __builtin_ctzll(todo));
        const uint64_t at_class = lanes_where(id_now == label), has = lanes_where(last == label);
        pos = last == label ? __builtin_ctzll(at_class) : pos;
        todo &= ~has;
      }
      const float l_pos = lp_s[row][pos & 63];
      const float l_last = pos >= 0 ? l_pos : kNegInf;
      const float join = par >= 0 ? (last_p == last ? pb_p : s_p) + (l_last + bonus) : kNegInf;
      const float again = pn + l_last;
      total = log_add(sb, again, join);  // pb' (+) pn' of a staying beam
      sn = log_add(again, join);
      // a pair whose prefix is a beam already is no new one
      const bool joins = par >= 0 && pos >= 0 && copy == 0, joined = lanes_where(joins) != 0;
      exchange();  // (the frame before has been read)
      if (joins) {
        const int e = first_s[par] + pos;
        if (e < first_s[par + 1]) merged_s[e] = fr + 1;
      }
      exchange();
      const float least = lanes_min<KT>(mine ? total : INFINITY);
#pragma unroll
      for (int q = 0; q < kPairs; ++q) {
        const int own = __shfl(pos, pi[q] & 63, 64);
        pv[q] = (own == pc[q] ? ppb[q] : ps[q]) + plb[q];
        const bool is_beam = joined && merged_s[lane + 64 * q] == fr + 1;
        enter[q] = lanes_where(pi[q] >= 0 && pv[q] > least && !is_beam);
        any |= enter[q];
      }
      // no pair enters, no beam leaves, and their order stands
      const float before = KT <= 16 ? lane_below(total) : __shfl(total, lane > 0 ? lane - 1 : 0, 64);
      const bool moves = mine && ((i > 0 && total > before) || (len >= 0 && !(total > kNegInf)));
      const float lead = lane_f(total, 0);
      if (any == 0 && lead > kNegInf && lanes_where(moves) == 0) {
        pb = sb - lead;
        pn = sn - lead;
        s = total - lead;
        spread();
        offset += lead;
        continue;
      }
    }

    // the totals to be ordered, in the order of ties
    int count = K;
    exchange();  // (the frame before has been read)
    if (copy == 0 && mine) val_s[i] = total;
#pragma unroll
    for (int q = 0; q < kPairs; ++q) {
      if ((enter[q] >> lane) & 1) {
        const int e = count + __popcll(enter[q] & ((uint64_t{1} << lane) - 1));
        val_s[e] = pv[q];
        what_s[e] = pi[q] + 256 * pc[q];
      }
      count += __popcll(enter[q]);
    }
    if (lane < 16) val_s[count + lane] = kNegInf;
    exchange();
    // entry e = 64 q + lane in this lane's registers
    float v[kBatches];
    int what[kBatches], place[kBatches];
    int live = 0;  // entries above -inf
#pragma unroll
    for (int q = 0; q < kBatches; ++q) {
      const int e = 64 * q + lane;
      const float x = val_s[e];
      const int pair = what_s[e] | 1 << 30;
      v[q] = e < count ? x : kNegInf;
      what[q] = e < K ? e : pair;
      place[q] = 0;
      live += __popcll(lanes_where(v[q] > kNegInf));
    }
    for (int o = 0; o < count; o += 16) {
      float4 w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = *reinterpret_cast<const float4*>(&val_s[o + 4 * k]);
#pragma unroll
      for (int q = 0; q < kBatches; ++q) {
        if (q > 0 && count <= 64 * q) break;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          place[q] += above(w[k].x, v[q]) + above(w[k].y, v[q]) + above(w[k].z, v[q]) + above(w[k].w, v[q]);
      }
    }
    // equal totals have one place: who finds another there goes by the entries' order
    auto put = [&]() {
#pragma unroll
      for (int q = 0; q < kBatches; ++q)
        if (v[q] > kNegInf && place[q] < K) place_s[place[q]] = make_int2(what[q], __float_as_int(v[q]));
      exchange();
    };
    put();
    bool tied = false;
#pragma unroll
    for (int q = 0; q < kBatches; ++q)
      tied |= v[q] > kNegInf && place[q] < K && place_s[place[q] & (KT - 1)].x != what[q];
    if (__builtin_expect(lanes_where(tied) != 0, 0)) {
      exchange();
#pragma unroll
      for (int q = 0; q < kBatches; ++q)
        for (int o = 0; o < 64 * q + lane && o < count; ++o) place[q] += val_s[o] == v[q];
      put();
    }
    // the new beam i
    const bool lives = i < min(live, K);
    const int2 here = place_s[lives ? i : 0];
    const bool grown = lives && (here.x >> 30) != 0;
    const int src = lives ? here.x & 255 : 0, c = grown ? (here.x >> 8) & 63 : 0;
    const float won = __int_as_float(here.y);
    const float best = live > 0 ? lane_f(won, 0) : 0.f;
    const float f_sb = __shfl(sb, src, 64), f_sn = __shfl(sn, src, 64);
    const uint64_t f_hash = from_lane(hash, src), f_phash = from_lane(phash, src);
    const int f_last = __shfl(last, src, 64), f_len = __shfl(len, src, 64), f_node = __shfl(node, src, 64);
    const int f_ck = __shfl(ck, src, 64), f_origin = __shfl(origin, src, 64);
    if (!lives) {
      pb = pn = s = kNegInf;
      len = last = -2;
      origin = -1;
    } else {
      const int label = id_s[row][c];
      const int fresh = (done + fr) * K + i;
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
        if (copy == 0) nodes[fresh] = make_int2(f_node, label);
        if (len % kCkStep == 0) {
          if (copy == 0) cks[fresh] = f_ck;
          ck = fresh;
        }
      }
    }
    offset += best;
    par_known = false;
    looked = -kLook;
    spread();
  }
  if (copy == 0 && mine) {
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
// each a lane of its own walks the kCkStep labels before it.  Bound by those loads, len / kCkStep + kCkStep
// behind one another: prefixes of up to 190 labels 16.5 us, 60 labels 11.5 (with steps of 32 labels 20 and 17).
// Lengths and nodes are held to the state's bounds: an advance that was captured at one position and replayed at
// another writes over nodes in use, and a prefix's nodes may then end before its labels do.
__global__ void __launch_bounds__(64)
beam_result_kernel(BeamFields f, int K, int max_frames, int max_tokens, int32_t* __restrict__ tokens, int32_t* __restrict__ lengths,
                   float* __restrict__ scores) {
  __shared__ int32_t start[64];
  const int lane = threadIdx.x;
  const int64_t at = blockIdx.x;
  const int n = static_cast<int>(at / K);
  const int len = min(f.len[at], max_frames);
  const uint32_t last_node = static_cast<uint32_t>(f.cap) - 1;  // (there are some where a prefix has labels)
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
        next = cks[min(static_cast<uint32_t>(next), last_node)];
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
      const int2 v = nodes[min(static_cast<uint32_t>(node), last_node)];
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
// before any is written, so that input and output may be the same memory; up to 32 loads of 16 bytes are
// under way in a thread.  Bound by memory: 0.79 GB read and written in 238 us, 6.6 TB/s (with stores past the
// caches 389 us); 16 KB in 3.5 us.
template <int KT>
__global__ void __launch_bounds__(256)
beam_reorder_kernel(ReorderTable t, int64_t col0, const int32_t* __restrict__ parents, int n0, int K) {
  const int64_t col = col0 + blockIdx.x;
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
                               const int32_t* done, bool fresh_start, void* state, int32_t* parents,
                               hipStream_t stream) {
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
  hipLaunchKernelGGL(beam_advance_kernel<KT>, dim3(here), dim3(64), 0, stream, rows, n0, K, C, fresh_start, ids, logp, \
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
                     beam_fields(state, N, K, max_frames), K, max_frames, max_tokens, tokens, lengths, scores);
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
      for (int64_t col0 = 0; col0 < c; col0 += kMaxGrid) {
        const dim3 grid(static_cast<unsigned>(std::min<int64_t>(kMaxGrid, c - col0)),
                        static_cast<unsigned>(std::min(65535, N - n0)));
#define PCTC_REORDER(KT) \
  hipLaunchKernelGGL(beam_reorder_kernel<KT>, grid, dim3(256), 0, stream, t, col0, parents, n0, K)
        if (K <= 4) PCTC_REORDER(4);
        else if (K <= 8) PCTC_REORDER(8);
        else if (K <= 16) PCTC_REORDER(16);
        else PCTC_REORDER(32);
#undef PCTC_REORDER
      }
    }
  }
  return hipGetLastError();
}

}  // namespace pctc
