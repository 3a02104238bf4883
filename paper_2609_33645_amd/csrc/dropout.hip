// Dropout whose mask comes from a counter-based generator and is never stored (gfx950).
//
//   y_i = x_i 65536 / t where h_i < t, else 0   (+ r_i),   t = round((1 - p) 65536)
//
// h_i is the 16-bit half i mod 8 (low half first, word by word) of the four words of Philox4x32-10
// (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011) with counter
// offset + i / 8 and key seed: the mask of a value depends on its index alone, so the gradient, the
// same call on dy, makes the same mask again, whatever the launch.  16 bits a value, because a
// word each would take twice the generator's integer products, which then bound the kernel; the share
// kept is t / 65536, and the scale is that share's inverse, so that E[y] = x for every p.
#include "pctc_internal.h"

namespace pctc {

namespace {

constexpr int kThreads = 256;
constexpr int kGroups = 2;  // groups of 8 values (one counter each) a thread

// 16 bytes at any alignment of its own values
typedef u32x4 __attribute__((aligned(2))) Piece;

// The four words of counter c under key k.
__device__ __forceinline__ u32x4 philox(uint64_t c, uint64_t key) {
  uint32_t c0 = static_cast<uint32_t>(c), c1 = static_cast<uint32_t>(c >> 32), c2 = 0u, c3 = 0u;
  uint32_t k0 = static_cast<uint32_t>(key), k1 = static_cast<uint32_t>(key >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = static_cast<uint64_t>(c0) * 0xD2511F53u, b = static_cast<uint64_t>(c2) * 0xCD9E8D57u;
    c0 = static_cast<uint32_t>(b >> 32) ^ c1 ^ k0;
    c1 = static_cast<uint32_t>(b);
    c2 = static_cast<uint32_t>(a >> 32) ^ c3 ^ k1;
    c3 = static_cast<uint32_t>(a);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return u32x4{c0, c1, c2, c3};
}

template <bool BF>
__device__ __forceinline__ void load8(const void* p, int64_t i, int left, float (&v)[8]) {
  if constexpr (BF) {
    const uint16_t* q = static_cast<const uint16_t*>(p) + i;
    if (left >= 8) {
      const u32x4 w = __builtin_nontemporal_load(reinterpret_cast<const Piece*>(q));
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[2 * e] = __uint_as_float(w[e] << 16);
        v[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = e < left ? bf16_to_f32(q[e]) : 0.f;
    }
  } else {
    const float* q = static_cast<const float*>(p) + i;
    if (left >= 8) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const u32x4 w = __builtin_nontemporal_load(reinterpret_cast<const Piece*>(q + 4 * h));
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * h + e] = __uint_as_float(w[e]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = e < left ? q[e] : 0.f;
    }
  }
}

template <bool BF>
__device__ __forceinline__ void store8(void* p, int64_t i, int left, const float (&v)[8]) {
  if constexpr (BF) {
    uint16_t* q = static_cast<uint16_t*>(p) + i;
    if (left >= 8) {
      const u32x4 w = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                       pack_bf16x2(v[6], v[7])};
      __builtin_nontemporal_store(w, reinterpret_cast<Piece*>(q));
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < left) q[e] = static_cast<uint16_t>(pack_bf16x2(v[e], 0.f));
    }
  } else {
    float* q = static_cast<float*>(p) + i;
    if (left >= 8) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        __builtin_nontemporal_store(u32x4{__float_as_uint(v[4 * h]), __float_as_uint(v[4 * h + 1]),
                                          __float_as_uint(v[4 * h + 2]), __float_as_uint(v[4 * h + 3])},
                                    reinterpret_cast<Piece*>(q + 4 * h));
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < left) q[e] = v[e];
    }
  }
}

// Two groups of 8 values a thread, all read before the generator runs, past the caches (nothing is read again).  Bound by
// memory: 11,458 x 4,096 in bf16 31 us, with a residual 46 (6.1 TB/s); 331 x 512 3.0.
// x, residual and y may be the same memory: a thread reads its values before it writes them.
template <bool BF, bool RES>
__global__ void __launch_bounds__(kThreads)
dropout_kernel(const void* x, const void* residual, void* y, int64_t n, uint32_t t, float scale, uint64_t seed,
               uint64_t offset, const uint64_t* offset_dev) {
  const uint64_t base = offset + (offset_dev ? *offset_dev : 0u);
  const int64_t g0 = static_cast<int64_t>(blockIdx.x) * (kThreads * kGroups) + threadIdx.x;
  float v[kGroups][8], r[kGroups][RES ? 8 : 1];
#pragma unroll
  for (int k = 0; k < kGroups; ++k) {
    const int64_t i = (g0 + k * kThreads) * 8;
    const int left = static_cast<int>(min(n - i, static_cast<int64_t>(8)));
    load8<BF>(x, i, left, v[k]);  // (nothing for left <= 0)
    if constexpr (RES) load8<BF>(residual, i, left, r[k]);
  }
#pragma unroll
  for (int k = 0; k < kGroups; ++k) {
    const int64_t g = g0 + k * kThreads, i = g * 8;
    const int left = static_cast<int>(min(n - i, static_cast<int64_t>(8)));
    const u32x4 w = philox(base + static_cast<uint64_t>(g), seed);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t h = (e & 1) ? w[e >> 1] >> 16 : w[e >> 1] & 0xffffu;
      float f = h < t ? v[k][e] * scale : 0.f;  // (a dropped infinity or NaN is zero)
      if constexpr (RES) f += r[k][e];
      v[k][e] = f;
    }
    store8<BF>(y, i, left, v[k]);
  }
}

}  // namespace

hipError_t launch_dropout(int dtype, const void* x, const void* residual, void* y, int64_t n, uint32_t t,
                          uint64_t seed, uint64_t offset, const uint64_t* offset_dev, hipStream_t stream) {
  const float scale = static_cast<float>(65536.0 / t);
  const dim3 grid(static_cast<unsigned>((n + kThreads * kGroups * 8 - 1) / (kThreads * kGroups * 8)));
  Prof pr("dropout", stream);
#define PCTC_DROPOUT(BF, RES)                                                                                       \
  hipLaunchKernelGGL((dropout_kernel<BF, RES>), grid, dim3(kThreads), 0, stream, x, residual, y, n, t, scale, seed, \
                     offset, offset_dev)
  if (dtype == 1) {
    if (residual) PCTC_DROPOUT(true, true);
    else PCTC_DROPOUT(true, false);
  } else {
    if (residual) PCTC_DROPOUT(false, true);
    else PCTC_DROPOUT(false, false);
  }
#undef PCTC_DROPOUT
  return hipGetLastError();
}

}  // namespace pctc
