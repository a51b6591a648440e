// Device helpers of the attention kernels (gfx950): the sequences' bounds, the operands
// from the staged tiles and the rows' statistics.
#pragma once

#include "lcvq_mfma.hpp"
#include "lcvq_serve.hpp"

namespace lcvq {

// Running maximum of a row that has seen nothing: finite, so that the factor of a hidden
// score (-inf) is exp2(-inf) = 0 and never inf - inf, and no score lies below it.
constexpr float kAttnLow = -3.402823466e38f;
// A probability is exp2(c (x - m)), as one fma exp2(c x - [c m]).  The rounding of [c m] is then a
// factor of all of a row's probabilities under one maximum, up to 2^(|c m| 2^-24): beyond
// this |c m| the difference x - m is taken first, which is exact at the maximum and near it.
constexpr float kAttnFar = 4096.0f;
__device__ __forceinline__ bool attn_far(float m, float c) { return fabsf(m * c) > kAttnFar; }

template <int N>
__device__ __forceinline__ void attn_wait_vm() {
  LCVQ_WAIT_VM(N);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// A sequence: new tokens q0 .. q0 + nq - 1 of the call, `len` cached ones with the new
// ones among them.  What the caller's arrays hold is clamped to what the call was given.
struct AttnSeq {
  int q0, nq, len;
  // the first token that any row sees
  __device__ __forceinline__ int first(const AttnArgs &a) const {
    return a.window > 0 ? max(0, len - nq - a.window + 1) : 0;
  }
};
__device__ __forceinline__ AttnSeq attn_seq(const AttnArgs &a, int b) {
  AttnSeq s;
  s.q0 = max(0, min(a.T, a.q_starts[b]));
  s.nq = min(max(0, min(a.T, a.q_starts[b + 1]) - s.q0), a.max_q);
  s.len = (int)max((int64_t)0, min((int64_t)a.kv_lens[b], a.width << a.page_shift));
  return s;
}
// Values that are the same in every lane, into scalar registers.
__device__ __forceinline__ int attn_uni(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t attn_uni(int64_t x) {
  const uint32_t lo = (uint32_t)attn_uni((int)(uint32_t)x), hi = (uint32_t)attn_uni((int)(uint32_t)((uint64_t)x >> 32));
  return (int64_t)(((uint64_t)hi << 32) | lo);
}
__device__ __forceinline__ AttnSeq attn_uni(const AttnSeq &s) { return AttnSeq{attn_uni(s.q0), attn_uni(s.nq), attn_uni(s.len)}; }
// Sequence b's items (granules, tiles, ..) follow those of b - 1: where an item, or where a
// sequence, lies among all.  Every wave finds it by itself; lane l counts the sequences
// l * per .. + per - 1.
struct AttnPlace {
  int64_t total;  // items of all sequences
  int b;          // the sequence; -1: no such item
  int64_t at;     // items before it
};
template <class Count, class Target>
__device__ __forceinline__ AttnPlace attn_place(const AttnArgs &a, Count count, Target target, int want_b) {
  const int lane = threadIdx.x & 63, per = (a.B + 63) / 64;
  const int b0 = lane * per, b1 = min(a.B, b0 + per);
  int64_t sum = 0;
  for (int b = b0; b < b1; ++b) sum += count(attn_seq(a, b));
  int64_t incl = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t up = __shfl_up(incl, o, 64);
    if (lane >= o) incl += up;
  }
  AttnPlace r;
  r.total = attn_uni((int64_t)__shfl(incl, 63, 64));
  int64_t at = incl - sum;
  int b = b0;
  bool mine;
  if (want_b >= 0) {
    mine = want_b >= b0 && want_b < b1;
    if (mine)
      for (; b < want_b; ++b) at += count(attn_seq(a, b));
  } else {
    const int64_t item = target(r.total);
    mine = item >= at && item < incl;
    if (mine)
      for (;; ++b) {
        const int64_t n = count(attn_seq(a, b));
        if (item < at + n) break;
        at += n;
      }
  }
  const uint64_t who = __ballot(mine);
  if (who == 0) {
    r.b = -1;
    r.at = 0;
    return r;
  }
  const int src = __builtin_ctzll(who);
  r.b = attn_uni(__shfl(b, src, 64));
  r.at = attn_uni((int64_t)__shfl(at, src, 64));
  return r;
}

// Row i of the sequence sees the tokens lo .. hi - 1.
__device__ __forceinline__ void attn_range(const AttnArgs &a, const AttnSeq &s, int i, int &lo, int &hi) {
  const int at = s.len - s.nq + i;
  hi = a.causal ? min(s.len, at + 1) : s.len;
  lo = a.window > 0 ? max(0, at - a.window + 1) : 0;
}

// Chunk c (16 bytes) of entry r of a tile lies at chunk c ^ attn_swz(r) of its row, so that the
// same chunk of sixteen entries falls on sixteen different 16-byte columns of the banks (256
// bytes; one row, two or four of them).
template <int kChunks>
__device__ __forceinline__ int attn_swz(int r) {
  return kChunks == 16 ? r & 15 : kChunks == 8 ? (r >> 1) & 7 : (r >> 2) & 3;
}

// s += K Q^T for one 16-token block: entry `row` of the tile (this lane's token), K in the
// order of the Q operand (32 ks + 8 g + i for bf16, 64 (ks / 2) + 16 g + 8 (ks % 2) + i for
// e4m3, whose 16-byte read feeds two steps).
template <int D, bool kFp8, int NB>
__device__ __forceinline__ void attn_scores(const char *tile, int row, int g, const bf16x8 (&qf)[NB][D / 32],
                                            floatx4 (&s)[NB]) {
  constexpr int kRow = kFp8 ? D : 2 * D, kChunks = kRow / 16;
  const char *p = tile + row * kRow;
  const int swz = attn_swz<kChunks>(row);
  if constexpr (kFp8) {
#pragma unroll
    for (int k2 = 0; k2 < D / 64; ++k2) {
      const u32x4 w = *reinterpret_cast<const u32x4 *>(p + (((4 * k2 + g) ^ swz) << 4));
      const bf16x8 a0 = e4m3_to_bf16x8(w[0], w[1], 1.0f), a1 = e4m3_to_bf16x8(w[2], w[3], 1.0f);
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        s[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a0, qf[n][2 * k2], s[n], 0, 0, 0);
        s[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a1, qf[n][2 * k2 + 1], s[n], 0, 0, 0);
      }
    }
  } else {
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks) {
      const bf16x8 w = *reinterpret_cast<const bf16x8 *>(p + (((4 * ks + g) ^ swz) << 4));
#pragma unroll
      for (int n = 0; n < NB; ++n) s[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, qf[n][ks], s[n], 0, 0, 0);
    }
  }
}

// V^T operand of 32 tokens (in the order of the probabilities) and the entries' elements
// 16 db .. + 15, from the row-major tile by the transposing LDS reads.
template <int D, bool kFp8>
__device__ __forceinline__ bf16x8 attn_v_operand(const char *tile, int lane, int db) {
  constexpr int kRow = kFp8 ? D : 2 * D, kChunks = kRow / 16;
  const int g = lane >> 4;
  if constexpr (kFp8) {
    typedef int int2v __attribute__((ext_vector_type(2)));
    typedef __attribute__((address_space(3))) int2v lds_int2v;
    const int j16 = lane & 15, k = j16 >> 1, row = 4 * g + (k & 3) + 16 * (k >> 2);
    const int2v t = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
        (lds_int2v *)(tile + row * kRow + ((db ^ attn_swz<kChunks>(row)) << 4) + 8 * (j16 & 1)));
    return e4m3_to_bf16x8((uint32_t)t[0], (uint32_t)t[1], 1.0f);
  } else {
    const int e = (lane >> 2) & 3, q = lane & 3, r0 = 4 * g + e, r1 = r0 + 16, c = 2 * db + (q >> 1);
    const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
        (lds_bf16x4 *)(tile + r0 * kRow + ((c ^ attn_swz<kChunks>(r0)) << 4) + 8 * (q & 1)));
    const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
        (lds_bf16x4 *)(tile + r1 * kRow + ((c ^ attn_swz<kChunks>(r1)) << 4) + 8 * (q & 1)));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
}

// Over the four lanes L, L ^ 16, L ^ 32, L ^ 48 that hold one row's tokens.
__device__ __forceinline__ float attn_max4(float x) {
  const uint32_t u = __float_as_uint(x);
  const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(u, u, false, false));
  const uint32_t w = __float_as_uint(fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1])));
  const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(w, w, false, false));
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float attn_sum4(float x) {
  x += __shfl_xor(x, 16, 64);
  x += __shfl_xor(x, 32, 64);
  return x;
}

// Four elements d .. d + 3 of row r (new token r / G, query head h G + r % G): v / sum, and
// with d == 0 the row's lse = ln(sum) + scale times the maximum mx.  A row that saw nothing
// gives 0 and -inf.
__device__ __forceinline__ void attn_store(const AttnArgs &a, const AttnSeq &s, int h, int r, int d, int D, const floatx4 &v,
                                           float mx, float sum) {
  const int i = r / a.G, head = h * a.G + r - i * a.G;
  const int64_t row = (int64_t)(s.q0 + i) * a.Hq + head;
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  const u32x2 w = {pack_bf16x2(v[0] * inv, v[1] * inv), pack_bf16x2(v[2] * inv, v[3] * inv)};
  *reinterpret_cast<u32x2 *>(a.out + row * D + d) = w;
  if (d == 0 && a.lse != nullptr)
    a.lse[row] = sum == 0.0f ? -__builtin_inff() : fmaf(mx, a.c, __builtin_amdgcn_logf(sum)) * 0.69314718055994530942f;
}

// ---- values that are no numbers ------------------------------------------------
// A token that some rows of a block see and others do not must not reach the others, but 0
// times a NaN or an infinity is NaN.  Where a partly hidden tile of V holds such values they
// are replaced by zeros before the product, and what they add is put in behind the
// block's results (attn_put_odd).  An entry whose scale byte the format has not (its values may
// reach infinity) counts as one of NaNs.  Such a value in the entries' words, and the words without:
template <bool kFp8>
__device__ __forceinline__ bool attn_odd(const u32x4 &w) {
  uint32_t odd = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {  // all ones above the sign: a carry into the sign's place
    const uint32_t x = w[i];
    odd |= kFp8 ? ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u : ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
  }
  return odd != 0;
}
template <bool kFp8>
__device__ __forceinline__ u32x4 attn_without_odd(const u32x4 &w) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t x = w[i];
    uint32_t keep = 0;
    if constexpr (kFp8) {
#pragma unroll
      for (int j = 0; j < 32; j += 8) keep |= ((x >> j) & 0x7fu) == 0x7fu ? 0u : 0xffu << j;
    } else {
#pragma unroll
      for (int j = 0; j < 32; j += 16) keep |= ((x >> j) & 0x7f80u) == 0x7f80u ? 0u : 0xffffu << j;
    }
    r[i] = x & keep;
  }
  return r;
}
// Element d of token t: 0 a number (or no such page), else one in the place of its kind's count: a
// NaN, infinity, -infinity.  (Some page is there, or nothing had been left out.)
constexpr int kAttnNan = 1, kAttnInf = 1 << 10, kAttnNegInf = 1 << 20;
template <int D, bool kFp8>
__device__ __forceinline__ int attn_odd_kind(const AttnArgs &a, int b, int h, int d, int t) {
  const int id = a.table[(int64_t)b * a.width + (t >> a.page_shift)];
  const bool there = (uint32_t)id < (uint32_t)a.pages;
  const int64_t row = (((int64_t)(there ? id : 0) * a.Hkv + h) << a.page_shift) + (t & ((1 << a.page_shift) - 1));
  if constexpr (kFp8) {
    const uint32_t v = reinterpret_cast<const uint8_t *>(a.v)[row * D + d], scale = a.vs[row];
    return there && ((v & 0x7fu) == 0x7fu || scale > kKvByteTop) ? kAttnNan : 0;
  } else {
    const uint32_t v = reinterpret_cast<const uint16_t *>(a.v)[row * D + d];
    return !there || (v & 0x7f80u) != 0x7f80u ? 0 : (v & 0x7fu) != 0 ? kAttnNan : (v & 0x8000u) != 0 ? kAttnNegInf : kAttnInf;
  }
}
// For rows r0 .. r1 - 1: the sum of such values among the tokens from .. to - 1 that each sees, where
// there are any, through put(r, d, sum) (NaN or an infinity).  256 threads; a thread takes an
// element of some rows in order, whose first and last tokens never fall: each token comes in
// once and goes out once, four loads at a time.
template <int D, bool kFp8, class Put>
__device__ __forceinline__ void attn_put_odd_of(const AttnArgs &a, const AttnSeq &s, int b, int h, int r0, int r1, int from, int to,
                                                Put put) {
  constexpr int kParts = 256 / D;
  const int d = threadIdx.x % D, per = (r1 - r0 + kParts - 1) / kParts;
  const int ra = r0 + (int)threadIdx.x / D * per, rb = min(r1, ra + per);
  int first = from, last = from, kinds = 0;  // the counts of the tokens first .. last - 1
  auto move = [&](int &t, int end, int sign) __attribute__((always_inline)) {
#pragma unroll 1
    while (t < end) {
      int k[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) k[j] = attn_odd_kind<D, kFp8>(a, b, h, d, min(t + j, end - 1));
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (t + j < end) kinds += sign * k[j];
      t = min(t + 4, end);
    }
  };
#pragma unroll 1
  for (int r = ra; r < rb; ++r) {
    int lo, hi;
    attn_range(a, s, r / a.G, lo, hi);
    lo = max(from, min(lo, to));
    hi = max(lo, min(hi, to));
    move(last, hi, 1);
    move(first, lo, -1);
    if (kinds == 0) continue;
    const bool nan = (kinds & 1023) != 0, inf = (kinds >> 10 & 1023) != 0, neg = kinds >> 20 != 0;
    put(r, d, nan || (inf && neg) ? __builtin_nanf("") : neg ? -__builtin_inff() : __builtin_inff());
  }
}
// Of a block whose tiles of kTile tokens stand at from .. to - 1, and of whose tokens every row sees
// all_lo .. all_hi - 1: values are left out of tiles before and behind these alone (at most a tile
// and the rows' tokens each, or the window and the rows').
template <int D, bool kFp8, int kTile, class Put>
__device__ __forceinline__ void attn_put_odd(const AttnArgs &a, const AttnSeq &s, int b, int h, int r0, int r1, int from, int to,
                                             int all_lo, int all_hi, Put put) {
  int end = max(from, min(to, (all_lo + kTile - 1) & -kTile));
#pragma unroll 1
  for (int e = 0; e < 2; ++e) {
    attn_put_odd_of<D, kFp8>(a, s, b, h, r0, r1, from, end, put);
    from = min(to, max(end, all_hi & -kTile));
    end = to;
  }
}
// ... into a finished row (whose element may be no number by itself: it stays one).
template <int D>
__device__ __forceinline__ void attn_put_out(const AttnArgs &a, const AttnSeq &s, int h, int r, int d, float sum) {
  const int i = r / a.G;
  uint16_t *o = a.out + ((int64_t)(s.q0 + i) * a.Hq + h * a.G + r - i * a.G) * D + d;
  *o = (uint16_t)f32_to_bf16(bf16_to_f32(*o) + sum);
}

}  // namespace lcvq
