// Keys and values of new tokens into a paged cache, quantised on the way, and back
// (lcvq_kv_write, lcvq_kv_read).
//
// Write, 8 bits: per token and head, amax over the D finite entries, the power of two of
// kv_exponent, and each entry x 2^-e (exact) rounded to the nearest e4m3 code, ties to
// even; a NaN or infinity becomes the NaN code, so that it stays visible.  Read: code 2^e,
// exact in bf16.
//
// Bound: HBM, the source once and the entries once.  D / 8 lanes take one head of one
// token, eight entries each (16 bytes of bf16), and share amax by lane moves.  A block takes
// 16 (D = 128) or 32 tokens of four heads of K or V: the tokens that follow one another in a page
// make whole lines of codes and runs of scale bytes, the four heads a run of 1 KiB (512
// bytes) of the dense side.  4999 tokens of 32 heads of 128, e4m3 (246 MB both ways): write 29 us,
// read 22, 4.2 and 5.7 TB/s; in bf16 (328 MB) 35 and 30; from fp32 and to fp32 (410 MB) 48 and
// 35.  100000 tokens of 8 heads read 119 us, 5.2 TB/s, a large copy's rate; 50000 in bf16 (410 MB) 81.
// One token: 3 us, its launch.
#include "lcvq_prep.hpp"
#include "lcvq_serve.hpp"

namespace lcvq {

constexpr int kKvHeads = 4;  // heads per block: one per trip

// Row of the slot's entry, or -1 for a slot outside the cache.
__device__ __forceinline__ int64_t kv_row(int64_t slot, int64_t pages, int page_shift, int H, int h) {
  if (slot < 0 || slot >= pages << page_shift) return -1;
  const int64_t page = slot >> page_shift;
  return ((page * H + h) << page_shift) + (slot - (page << page_shift));
}

constexpr uint32_t kKvTop = 0x7f600000u;  // 448 2^119: above it the scale's exponent has reached its end

// Largest of kL = 8 or 16 neighbouring lanes' values, in all of them (lane ^ 1, ^ 2, then the
// mirror images of 8 and 16).
template <int kL>
__device__ __forceinline__ uint32_t kv_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xb1, 0xf, 0xf, true));
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4e, 0xf, 0xf, true));
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xf, 0xf, true));
  if constexpr (kL == 16) v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x140, 0xf, 0xf, true));
  return v;
}

// Eight entries of the source as fp32 bits.
template <bool kBf16>
__device__ __forceinline__ void kv_load8(const void *src, int64_t at, uint32_t (&x)[8]) {
  if constexpr (kBf16) {
    const u32x4 w = *reinterpret_cast<const u32x4 *>(reinterpret_cast<const uint16_t *>(src) + at);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t v = w[i];
      x[2 * i] = v << 16;
      x[2 * i + 1] = v & 0xffff0000u;
    }
  } else {
    const uint32_t *p = reinterpret_cast<const uint32_t *>(src) + at;
    const u32x4 a = *reinterpret_cast<const u32x4 *>(p), b = *reinterpret_cast<const u32x4 *>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = a[i];
      x[4 + i] = b[i];
    }
  }
}

template <int D, bool kFp8, bool kSrcBf16>
__global__ __launch_bounds__(256) void k_kv_write(KvCache c, int64_t T, const void *__restrict__ K, const void *__restrict__ V,
                                                  int64_t k_token, int64_t k_head, int64_t v_token, int64_t v_head,
                                                  const int64_t *__restrict__ slots) {
  constexpr int kL = D / 8, kRows = 256 / kL, kN = kKvHeads;  // lanes per entry, entries per trip, trips
  const int h0 = (int)blockIdx.y * kKvHeads;
  const bool val = blockIdx.z != 0;
  const void *src = val ? V : K;
  const int64_t ts = val ? v_token : k_token, hs = val ? v_head : k_head;
  char *data = reinterpret_cast<char *>(val ? c.v : c.k);
  uint8_t *scale = val ? c.vs : c.ks;
  const int lane = threadIdx.x % kL, sub = threadIdx.x / kL;
  const int64_t t = (int64_t)blockIdx.x * kRows + sub;
  if (t >= T) return;  // (the lanes of an entry agree)
  int64_t row[kN];
  uint32_t x[kN][8];
#pragma unroll
  for (int i = 0; i < kN; ++i)  // all loads first
    if (h0 + i < c.H) kv_load8<kSrcBf16>(src, t * ts + (h0 + i) * hs + lane * 8, x[i]);
  const int64_t slot = slots[t];
#pragma unroll
  for (int i = 0; i < kN; ++i) row[i] = h0 + i < c.H ? kv_row(slot, c.pages, c.page_shift, c.H, h0 + i) : -1;
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    if (row[i] < 0) continue;
    if constexpr (kFp8) {
      uint32_t top = 0;  // largest |x| as bits; with a NaN or an infinity in it, or too large, the slow way
#pragma unroll
      for (int j = 0; j < 8; ++j) top = max(top, x[i][j] & 0x7fffffffu);
      top = kv_max<kL>(top);
      float y[8];
      int e;
      if (__ballot(top > kKvTop) == 0) {
        e = kv_exponent(top);
        const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = __uint_as_float(x[i][j]) * inv;
      } else {
        uint32_t amax = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint32_t u = x[i][j] & 0x7fffffffu;
          amax = max(amax, u < 0x7f800000u ? u : 0u);
        }
        e = kv_exponent(kv_max<kL>(amax));
        const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const bool finite = (x[i][j] & 0x7fffffffu) < 0x7f800000u;
          const float z = __builtin_amdgcn_fmed3f(__uint_as_float(x[i][j]) * inv, -kE4m3Max, kE4m3Max);
          y[j] = finite ? z : __uint_as_float(0x7fc00000u);
        }
      }
      int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
      lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
      int hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false);
      hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], hi, true);
      *reinterpret_cast<u32x2 *>(data + row[i] * D + lane * 8) = u32x2{(uint32_t)lo, (uint32_t)hi};
      if (lane == 0) scale[row[i]] = (uint8_t)(e + 127);
    } else {
      u32x4 w;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (kSrcBf16) {
          w[j] = (x[i][2 * j] >> 16) | x[i][2 * j + 1];  // bits as they are
        } else {
          w[j] = pack_bf16x2(__uint_as_float(x[i][2 * j]), __uint_as_float(x[i][2 * j + 1]));
        }
      }
      *reinterpret_cast<u32x4 *>(data + (row[i] * D + lane * 8) * 2) = w;
    }
  }
}

// Values of any slots, (T, H, D) dense; a slot outside the cache reads as zeros.
template <int D, bool kFp8, bool kOutBf16>
__global__ __launch_bounds__(256) void k_kv_read(KvCache c, int64_t T, const int64_t *__restrict__ slots, void *__restrict__ K,
                                                 void *__restrict__ V) {
  constexpr int kL = D / 8, kRows = 256 / kL, kN = kKvHeads;
  const int h0 = (int)blockIdx.y * kKvHeads;
  const bool val = blockIdx.z != 0;
  void *dst = val ? V : K;
  const char *data = reinterpret_cast<const char *>(val ? c.v : c.k);
  const uint8_t *scale = val ? c.vs : c.ks;
  const int lane = threadIdx.x % kL, sub = threadIdx.x / kL;
  const int64_t t = (int64_t)blockIdx.x * kRows + sub;
  if (t >= T) return;
  int64_t row[kN];
  u32x4 w[kN];
  uint32_t s[kN];
  const int64_t slot = slots[t];
#pragma unroll
  for (int i = 0; i < kN; ++i) row[i] = h0 + i < c.H ? kv_row(slot, c.pages, c.page_shift, c.H, h0 + i) : -1;
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    w[i] = u32x4{0, 0, 0, 0};
    s[i] = 127;
    if (row[i] < 0) continue;
    if constexpr (kFp8) {
      const u32x2 p = *reinterpret_cast<const u32x2 *>(data + row[i] * D + lane * 8);
      w[i][0] = p[0];
      w[i][1] = p[1];
      s[i] = scale[row[i]];
    } else {
      w[i] = *reinterpret_cast<const u32x4 *>(data + (row[i] * D + lane * 8) * 2);
    }
  }
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    if (h0 + i >= c.H) continue;
    u32x4 v = w[i];
    if constexpr (kFp8) v = __builtin_bit_cast(u32x4, e4m3_to_bf16x8(w[i][0], w[i][1], kv_scale(s[i])));
    const int64_t at = (t * c.H + h0 + i) * D + lane * 8;
    if constexpr (kOutBf16) {
      *reinterpret_cast<u32x4 *>(reinterpret_cast<uint16_t *>(dst) + at) = v;
    } else {
      float *p = reinterpret_cast<float *>(dst) + at;
      *reinterpret_cast<floatx4 *>(p) = floatx4{bf16_lo(v[0]), bf16_hi(v[0]), bf16_lo(v[1]), bf16_hi(v[1])};
      *reinterpret_cast<floatx4 *>(p + 4) = floatx4{bf16_lo(v[2]), bf16_hi(v[2]), bf16_lo(v[3]), bf16_hi(v[3])};
    }
  }
}

// ---------------------------------------------------------------- launch ---
static dim3 kv_grid(const KvCache &c, int64_t T) {
  return dim3((unsigned)ceil_div(T, 2048 / c.D), (unsigned)ceil_div(c.H, kKvHeads), 2);
}

template <int D, bool kFp8>
static hipError_t write(const KvCache &c, int64_t T, const void *K, const void *V, bool src_bf16, int64_t k_token, int64_t k_head,
                        int64_t v_token, int64_t v_head, const int64_t *slots, hipStream_t st) {
  auto k = src_bf16 ? k_kv_write<D, kFp8, true> : k_kv_write<D, kFp8, false>;
  k<<<kv_grid(c, T), 256, 0, st>>>(c, T, K, V, k_token, k_head, v_token, v_head, slots);
  return hipGetLastError();
}

hipError_t launch_kv_write(const KvCache &c, int64_t T, const void *K, const void *V, bool src_bf16, int64_t k_token,
                           int64_t k_head, int64_t v_token, int64_t v_head, const int64_t *slots, hipStream_t st) {
  auto go = c.D == 64 ? (c.fp8 ? write<64, true> : write<64, false>) : (c.fp8 ? write<128, true> : write<128, false>);
  return go(c, T, K, V, src_bf16, k_token, k_head, v_token, v_head, slots, st);
}

template <int D, bool kFp8>
static hipError_t read(const KvCache &c, int64_t T, const int64_t *slots, void *K, void *V, bool out_bf16, hipStream_t st) {
  auto k = out_bf16 ? k_kv_read<D, kFp8, true> : k_kv_read<D, kFp8, false>;
  k<<<kv_grid(c, T), 256, 0, st>>>(c, T, slots, K, V);
  return hipGetLastError();
}

hipError_t launch_kv_read(const KvCache &c, int64_t T, const int64_t *slots, void *K, void *V, bool out_bf16,
                          hipStream_t st) {
  auto go = c.D == 64 ? (c.fp8 ? read<64, true> : read<64, false>) : (c.fp8 ? read<128, true> : read<128, false>);
  return go(c, T, slots, K, V, out_bf16, st);
}

}  // namespace lcvq
