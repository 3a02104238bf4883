// Output-tile order and epilogue pieces shared by the bf16 and fp32 vocabulary-head products
// (head_gemm_bf16.hip, head_gemm_f32.hip).  G is a tile engine: a WR x WC grid of wavefronts,
// each with FR x FC accumulator blocks of 32 x 32 (row_of / col_of give an accumulator's place).
#pragma once

#include "pctc_device.h"

namespace pctc {

__device__ __forceinline__ int xcd_swz(int bid, int nblocks) {
  const int full = (nblocks / 8) * 8;
  if (bid >= full) return bid;
  return (bid % 8) * (full / 8) + bid / 8;
}

// Tile order for an nA x nB grid of output tiles, A = frame tiles (few), B = vocabulary
// tiles or partitions (many).  Consecutive work ids walk groups of ga x gb tiles (a
// fastest) with about 64 tiles per group (what one XCD runs at a time) and ga ~ 11 frame
// tiles; the groups walk the frame groups fastest, so the few groups that cover every frame
// tile of a run of vocabulary rows are consecutive: that XCD fetches the rows once and the
// frame tiles (the small operand) stay in its L2.  Grid = ceil(nA/ga) ga * ceil(nB/gb) gb;
// ids past the edge return false.
__host__ __device__ __forceinline__ void group_shape(int nA, int& ga, int& gb) {
  const int groups = (nA + 10) / 11;
  ga = (nA + groups - 1) / groups;
  gb = 64 / ga;
  if (gb < 1) gb = 1;
}
__host__ __device__ __forceinline__ int grouped_grid(int nA, int nB) {
  int ga, gb;
  group_shape(nA, ga, gb);
  return ((nA + ga - 1) / ga) * ga * ((nB + gb - 1) / gb) * gb;
}
__device__ __forceinline__ bool grouped_tile(int work, int nA, int nB, int& a, int& b) {
  int ga, gb;
  group_shape(nA, ga, gb);
  const int gA = (nA + ga - 1) / ga;
  const int blk = work / (ga * gb), in = work % (ga * gb);
  a = (blk % gA) * ga + in % ga;
  b = (blk / gA) * gb + in / ga;
  return a < nA && b < nB;
}

// Accumulators of a tile start at the bias of their row (bt: the tile's rows, in LDS).
template <int FR, int FC, class G>
__device__ __forceinline__ void bias_init(f32x16 (&acc)[FR][FC], const float* bt, int wave, int lane) {
#pragma unroll
  for (int i = 0; i < FR; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float4 b4 = *reinterpret_cast<const float4*>(bt + G::row_of(wave, lane, i, 4 * q));
#pragma unroll
      for (int j = 0; j < FC; ++j) {
        acc[i][j][4 * q + 0] = b4.x;
        acc[i][j][4 * q + 1] = b4.y;
        acc[i][j][4 * q + 2] = b4.z;
        acc[i][j][4 * q + 3] = b4.w;
      }
    }
}

// Adds the bias of each row to a tile (bt: the tile's rows, in LDS).
template <int FR, int FC, class G>
__device__ __forceinline__ void bias_add(f32x16 (&acc)[FR][FC], const float* bt, int wave, int lane) {
#pragma unroll
  for (int i = 0; i < FR; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float4 b4 = *reinterpret_cast<const float4*>(bt + G::row_of(wave, lane, i, 4 * q));
#pragma unroll
      for (int j = 0; j < FC; ++j) {
        acc[i][j][4 * q + 0] += b4.x;
        acc[i][j][4 * q + 1] += b4.y;
        acc[i][j][4 * q + 2] += b4.z;
        acc[i][j][4 * q + 3] += b4.w;
      }
    }
}

// Logits of rows at or past vend (a partition's ragged last tile, whose rows read as zeros)
// become -inf in place, so that the update below treats every tile alike.  Each row test is
// used at once for the FC columns it covers (a lane holds 4 consecutive rows per group):
// keeping one test per accumulator live across both passes of the update would take a mask
// register pair per element.
template <int FR, int FC, class G>
__device__ __forceinline__ void mask_rows_inf(f32x16 (&acc)[FR][FC], int v0, int vend, int wave, int lane) {
#pragma unroll
  for (int i = 0; i < FR; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int lim = vend - v0 - G::row_of(wave, lane, i, 4 * q);  // rows e < lim are in range
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool out = e >= lim;
#pragma unroll
        for (int j = 0; j < FC; ++j) acc[i][j][4 * q + e] = out ? -INFINITY : acc[i][j][4 * q + e];
      }
    }
}

// What the exponents of log2(e) z are taken relative to: the maximum's, but none below that of -1e9, so that a column
// whose rows are all masked yet adds nothing, by a bias of -inf, of -1e30 or of the type's lowest value; and by how much
// it is off log2(e) times that maximum, exactly.  (That rounding enters every exponent: 64 at 1e9, beyond every
// exponential's range from 3e9 on.)
constexpr float kLseFloor = -1e9f;
__device__ __forceinline__ float lse_reference(float max) { return fmaxf(max, kLseFloor) * kLog2e; }
__device__ __forceinline__ float lse_rounding(float max) {
  return fmaf(fmaxf(max, kLseFloor), kLog2e, -lse_reference(max));
}

// Online log-sum-exp update of the running (max, sum) of this lane's frames with one
// tile of logits (bias included; out-of-range rows already -inf).
template <int FR, int FC, class G>
__device__ __forceinline__ void lse_tile_update(const f32x16 (&acc)[FR][FC], float (&run_max)[FC],
                                                float (&run_sum)[FC]) {
#pragma unroll
  for (int j = 0; j < FC; ++j) {
    float tmax = -INFINITY;
#pragma unroll
    for (int i = 0; i < FR; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) tmax = fmaxf(tmax, acc[i][j][r]);
    tmax = fmaxf(tmax, swap_halves(tmax));
    const float nmax = fmaxf(run_max[j], tmax);
    const float ms = lse_reference(nmax);
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < FR; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) s += fast_exp2(fmaf(acc[i][j][r], kLog2e, -ms));
    s += swap_halves(s);
    const float scale = (run_max[j] == -INFINITY) ? 0.f : fast_exp2((run_max[j] - nmax) * kLog2e);
    run_sum[j] = fmaf(run_sum[j], scale, s);
    run_max[j] = nmax;
  }
}

// The same, and bm[j][..]: the largest logits of the lane's blocks of frame column j.  A block is ROWS
// of the 16 rows that a lane holds of 32: of rows 8 q + 4 h + e (h the lane's half, e < 4) those of ROWS / 4
// consecutive q.  Where one class has nearly all of a frame's probability, the classes beside it are each below
// the sum's last bit and would all be lost to it: a block's eight are added among themselves first, and run_lo
// holds what the running sum's roundings left.
template <int FR, int FC, class G, int ROWS>
__device__ __forceinline__ void lse_block_update(const f32x16 (&acc)[FR][FC], float (&run_max)[FC],
                                                 float (&run_sum)[FC], float (&run_lo)[FC],
                                                 float (&bm)[FC][FR * 16 / ROWS]) {
  constexpr int kSub = 16 / ROWS;
#pragma unroll
  for (int j = 0; j < FC; ++j) {
    float tmax = -INFINITY;
#pragma unroll
    for (int i = 0; i < FR; ++i)
#pragma unroll
      for (int u = 0; u < kSub; ++u) {
        float x = acc[i][j][u * ROWS];
#pragma unroll
        for (int r = 1; r < ROWS; ++r) x = fmaxf(x, acc[i][j][u * ROWS + r]);
        bm[j][i * kSub + u] = x;
        tmax = fmaxf(tmax, x);
      }
    tmax = fmaxf(tmax, swap_halves(tmax));
    const float nmax = fmaxf(run_max[j], tmax);
    const float ms = lse_reference(nmax);
    float s = 0.f;
    if (__builtin_expect(__any(fabsf(nmax) > 1e37f && nmax > -INFINITY), 0)) {
      // a column of masked classes only, the mask a type's lowest value: its products with log2(e)
      // overflow, the differences do not
#pragma unroll
      for (int i = 0; i < FR; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) s += fast_exp2((acc[i][j][r] - (nmax == -INFINITY ? 0.f : nmax)) * kLog2e);
    } else {
#pragma unroll
      for (int i = 0; i < FR; ++i)
#pragma unroll
        for (int u = 0; u < 16; u += 8) {
          float e[8];
#pragma unroll
          for (int r = 0; r < 8; ++r) e[r] = fast_exp2(fmaf(acc[i][j][u + r], kLog2e, -ms));
          s += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
        }
      // ms is nmax log2(e) rounded; its rounding, up to 1e-6 at a logit of 20, is taken off the sum again
      s *= fast_exp2(-lse_rounding(nmax));
    }
    s += swap_halves(s);
    const float scale = (run_max[j] == -INFINITY) ? 0.f : fast_exp2((run_max[j] - nmax) * kLog2e);
    const float was = run_sum[j] * scale, sum = was + s, of_s = sum - was;
    run_lo[j] = fmaf(run_lo[j], scale, (was - (sum - of_s)) + (s - of_s));
    run_sum[j] = sum;
    run_max[j] = nmax;
  }
}

// Writes the block maxima of a tile whose first class is v0; a frame's row has nb of them, a lane's
// side by side (CandBlocks in pctc_internal.h has the order).  kBlockStores stores in every wavefront, also where
// its frames lie past M (the resource ends there), so that waits for copies in flight can count on them.
constexpr int kRawBuffer = 0x00020000;  // word 3 of a raw buffer resource: 32-bit data, no swizzle
template <class G, int ROWS>
constexpr int kBlockStores = G::FC * G::FR * 4 / ROWS;
template <class G, int ROWS>
__device__ __forceinline__ void store_block_max(const float (&bm)[G::FC][G::FR * 16 / ROWS], int v0, int wave, int lane,
                                                int m0, int M, int nb, float* __restrict__ bmax) {
#if defined(__HIP_DEVICE_COMPILE__)  // the buffer-resource type exists on the device side only
  constexpr int kRun = G::FR * 16 / ROWS;
  static_assert(G::FR == 4 && kRun % 4 == 0, "wavefronts of 128 rows");
  const __amdgpu_buffer_rsrc_t rows =
      __builtin_amdgcn_make_buffer_rsrc(bmax + static_cast<int64_t>(m0) * nb, static_cast<short>(0),
                                        min(M - m0, G::kBC) * nb * 4, kRawBuffer);
  const int at = ((v0 + G::row_of(wave, 0, 0, 0)) >> 7) * 2 * kRun + (lane >> 5) * kRun;
#pragma unroll
  for (int j = 0; j < G::FC; ++j) {
    const int off = (G::col_of(wave, lane, j) * nb + at) * 4;
#pragma unroll
    for (int k = 0; k < kRun / 4; ++k) {
      const u32x4 v = {__float_as_uint(bm[j][4 * k]), __float_as_uint(bm[j][4 * k + 1]),
                       __float_as_uint(bm[j][4 * k + 2]), __float_as_uint(bm[j][4 * k + 3])};
      __builtin_amdgcn_raw_buffer_store_b128(v, rows, off + 16 * k, 0, 0);
    }
  }
#endif
}

// Writes the logits of a tile whose first class is v0, ld (a whole number of tiles) to a frame.
template <class G>
__device__ __forceinline__ void store_logits(const f32x16 (&acc)[G::FR][G::FC], int v0, int wave, int lane, int m0,
                                             int M, int ld, float* __restrict__ Z) {
#pragma unroll
  for (int j = 0; j < G::FC; ++j) {
    const int m = m0 + G::col_of(wave, lane, j);
    if (m >= M) continue;
    float* const out = Z + static_cast<int64_t>(m) * ld + v0 + G::row_of(wave, lane, 0, 0);
#pragma unroll
    for (int i = 0; i < G::FR; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4*>(out + 32 * i + 8 * q) =
            make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
  }
}

// The two wavefronts of each frame column (row halves) combine their running (max, sum)
// pairs through LDS (xch: any drained stage) and write the partition's pair of every frame.
template <class G>
__device__ __forceinline__ void lse_store_partials(const float (&run_max)[G::FC], const float (&run_sum)[G::FC],
                                                   char* xchb, int wave, int lane, int m0, int M,
                                                   float2* __restrict__ out) {
  constexpr int FC = G::FC;
  __syncthreads();
  constexpr int WC = G::NW / 2;  // column groups (the wave grid is 2 x WC)
  float2* xch = reinterpret_cast<float2*>(xchb);
  const int rowhalf = wave / WC, colq = wave % WC;
  if (rowhalf == 1 && lane < 32) {
#pragma unroll
    for (int j = 0; j < FC; ++j) xch[colq * (FC * 32) + j * 32 + lane] = make_float2(run_max[j], run_sum[j]);
  }
  __syncthreads();
  if (rowhalf == 0 && lane < 32) {
#pragma unroll
    for (int j = 0; j < FC; ++j) {
      const float2 o = xch[colq * (FC * 32) + j * 32 + lane];
      const float nmax = fmaxf(run_max[j], o.x);
      float s = 0.f;
      if (run_max[j] != -INFINITY) s += run_sum[j] * fast_exp2((run_max[j] - nmax) * kLog2e);
      if (o.x != -INFINITY) s += o.y * fast_exp2((o.x - nmax) * kLog2e);
      if (nmax != nmax) s = nmax;
      const int m = m0 + G::col_of(wave, lane, j);
      if (m < M) out[m] = make_float2(nmax, s);
    }
  }
}

__device__ __forceinline__ void amax_merge(float& bv, int& bi, float ov, int oi) {
  if (ov > bv || (ov == bv && oi < bi)) {
    bv = ov;
    bi = oi;
  }
}

// Framewise best (value, class) of this lane's rows with one tile of logits (out-of-range rows
// already -inf, which never replaces the best).
template <int FR, int FC, class G>
__device__ __forceinline__ void amax_tile_update(const f32x16 (&a)[FR][FC], int v0, int wave, int lane,
                                                 float (&bv)[FC], int (&bi)[FC]) {
  // the lane's rows increase with (i, r): the tile's best is its largest logit at the first
  // row holding it (found scanning backwards), and it replaces the running best only when
  // strictly larger, so ties keep the smallest id; NaN never compares equal or larger
  const int rbase = v0 + G::row_of(wave, lane, 0, 0);
#pragma unroll
  for (int j = 0; j < FC; ++j) {
    float tmax = -INFINITY;
#pragma unroll
    for (int i = 0; i < FR; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) tmax = fmaxf(tmax, a[i][j][r]);
    int off = 0;
#pragma unroll
    for (int i = FR - 1; i >= 0; --i)
#pragma unroll
      for (int r = 15; r >= 0; --r) off = (a[i][j][r] == tmax) ? 32 * i + 8 * (r >> 2) + (r & 3) : off;
    if (tmax > bv[j]) {
      bv[j] = tmax;
      bi[j] = rbase + off;
    }
  }
}

// The lane halves, then the two wavefronts of each frame column, combine their best pairs
// (xchb: any drained stage) and write the partition's pair of every frame.
template <class G>
__device__ __forceinline__ void amax_store_partials(float (&bv)[G::FC], int (&bi)[G::FC], char* xchb, int wave,
                                                    int lane, int m0, int M, float2* __restrict__ out) {
  constexpr int FC = G::FC;
  // lane halves hold the other half of each 32-row block, then the row halves of the tile
#pragma unroll
  for (int j = 0; j < FC; ++j) {
    const float ov = swap_halves(bv[j]);
    const int oi = __shfl_xor(bi[j], 32, 64);
    amax_merge(bv[j], bi[j], ov, oi);
  }
  __syncthreads();
  float2* xch = reinterpret_cast<float2*>(xchb);
  constexpr int WC = G::NW / 2;  // column groups (the wave grid is 2 x WC)
  const int rowhalf = wave / WC, colq = wave % WC;
  if (rowhalf == 1 && lane < 32) {
#pragma unroll
    for (int j = 0; j < FC; ++j)
      xch[colq * (FC * 32) + j * 32 + lane] = make_float2(bv[j], __int_as_float(bi[j]));
  }
  __syncthreads();
  if (rowhalf == 0 && lane < 32) {
#pragma unroll
    for (int j = 0; j < FC; ++j) {
      const float2 o = xch[colq * (FC * 32) + j * 32 + lane];
      amax_merge(bv[j], bi[j], o.x, __float_as_int(o.y));
      const int m = m0 + G::col_of(wave, lane, j);
      if (m < M) out[m] = make_float2(bv[j], __int_as_float(bi[j]));
    }
  }
}

// A wavefront's accumulators (128 tile rows x 64 columns) as rows of the output: 32 columns at a time go
// through its own 16 KB of the drained stages (16-byte slots XORed with the column, so that neither
// writes nor reads meet in a bank), and come back 8 consecutive tile rows a lane, 16 lanes a column, so that
// memory is read and written in lines.  Straight from the accumulators a store is 32 pieces of 16 bytes: the
// epilogue of ffn_back then took longer than its product (M = 2,567, 4,096 x 10,240: 419 us, now 255).
// fn(block, col, v, x): tile rows 8 block .. 8 block + 7 of the wavefront's 128, column col of its 64; x is what
// pre(block, col, x) read for these places, for 32 columns before any of them is used, so that many
// reads are in flight (there is one workgroup on a compute unit, whose products are over).
// The 16 KB are one wavefront's: its exchanges need no barrier of the workgroup.
struct Nothing {};
template <class G, class X = Nothing, class Fn, class Pre>
__device__ __forceinline__ void by_columns(f32x16 (&acc)[G::FR][G::FC], char* const (&st)[4], Fn&& fn, Pre&& pre) {
  static_assert(G::FR == 4 && G::FC == 2, "128 x 64");
  int lane = threadIdx.x & 63;
  // opaque: what is derived from it is not kept in registers through the product (it would spill there)
  asm volatile("" : "+v"(lane));
  const int wave = threadIdx.x >> 6;
  char* const base = (wave < 2 ? st[0] : wave < 4 ? st[1] : wave < 6 ? st[2] : st[3]) + (wave & 1) * 16384;
  constexpr int NB = sizeof(X) > 32 ? 4 : 8;  // places a lane reads ahead
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int c = lane & 31;
    wave_exchange();  // (the columns before have been read)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int slot = 8 * i + 2 * q + (lane >> 5);  // tile rows 4 slot ..
        *reinterpret_cast<float4*>(base + c * 512 + ((slot ^ (c & 31)) << 4)) =
            make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
      }
    wave_exchange();
    const int block = lane & 15;
#pragma unroll
    for (int t0 = 0; t0 < 8; t0 += NB) {
      X x[NB];
#pragma unroll
      for (int t = 0; t < NB; ++t) pre(block, 32 * j + 4 * (t0 + t) + (lane >> 4), x[t]);
#pragma unroll
      for (int t = 0; t < NB; ++t) {
        const int col = 4 * (t0 + t) + (lane >> 4);
        float v[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float4 y = *reinterpret_cast<const float4*>(base + col * 512 + (((2 * block + h) ^ (col & 31)) << 4));
          v[4 * h] = y.x;
          v[4 * h + 1] = y.y;
          v[4 * h + 2] = y.z;
          v[4 * h + 3] = y.w;
        }
        fn(block, 32 * j + col, v, x[t]);
      }
    }
  }
}
template <class G, class Fn>
__device__ __forceinline__ void by_columns(f32x16 (&acc)[G::FR][G::FC], char* const (&st)[4], Fn&& fn) {
  by_columns<G>(acc, st, [&](int block, int col, const float (&v)[8], const Nothing&) { fn(block, col, v); },
                [](int, int, Nothing&) {});
}

}  // namespace pctc
