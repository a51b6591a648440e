// Internal launchers of the serving operators (host side) and what their kernels share:
// the paged cache of keys and values, the attention that reads it, 4-bit weights.
#pragma once

#include "lcvq_common.hpp"

namespace lcvq {

// ---- the 8-bit cache format ----------------------------------------------
// Each token's head is D e4m3 codes (OCP: 4 exponent bits, bias 7, largest 448, one NaN)
// and one scale byte E for the factor 2^(E - 127).  E - 127 is the smallest e with
// amax <= 448 2^e over the finite entries, kept in [-117, 119]: every value is then exact
// in bf16 (2^-9 2^-117 is its least normal number) and finite (448 2^119).  A power of two
// costs up to one bit of the codes' range against amax / 448, which e4m3's own exponents
// take up, and makes both directions exact but for the one rounding of a code.
constexpr int kKvExpLo = -117, kKvExpHi = 119;
constexpr uint32_t kKvByteTop = 127 + kKvExpHi;  // the largest scale byte
constexpr float kE4m3Max = 448.0f;

// e from the bits of |amax| (finite): 448 = 1.75 2^8.
__device__ __forceinline__ int kv_exponent(uint32_t amax_bits) {
  const int e = (int)(amax_bits >> 23) - 127 - 8 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return max(kKvExpLo, min(kKvExpHi, e));
}
// 2^(E - 127); a scale byte of 0 gives 0, 255 infinity.
__device__ __forceinline__ float kv_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight e4m3 codes (two dwords) times `scale` -> eight bf16 values (exact).
__device__ __forceinline__ bf16x8 e4m3_to_bf16x8(uint32_t lo, uint32_t hi, float scale) {
  const bf16x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  const bf16x2 p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  const bf16x2 p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  bf16x8 r;
  r[0] = p0[0]; r[1] = p0[1]; r[2] = p1[0]; r[3] = p1[1];
  r[4] = p2[0]; r[5] = p2[1]; r[6] = p3[0]; r[7] = p3[1];
  return r;
}

// ---- paged cache (lcvq_kv.hip) -------------------------------------------
// Entry (page, head, offset) is row (page * H + head) * page_size + offset of `data` (D
// codes or D bf16) and of `scale` (one byte; nullptr for bf16).  page_size = 2^page_shift.
struct KvCache {
  void *k, *v;
  uint8_t *ks, *vs;
  int64_t pages;
  int H, D, page_shift;
  bool fp8;
};
hipError_t launch_kv_write(const KvCache &c, int64_t T, const void *K, const void *V, bool src_bf16, int64_t k_token,
                           int64_t k_head, int64_t v_token, int64_t v_head, const int64_t *slots, hipStream_t st);
hipError_t launch_kv_read(const KvCache &c, int64_t T, const int64_t *slots, void *K, void *V, bool out_bf16,
                          hipStream_t st);

// ---- attention over the cache (lcvq_attn.hip) ------------------------------
struct AttnArgs {
  const uint16_t *q;
  int64_t q_token, q_head;  // strides, elements
  const char *k, *v;
  const uint8_t *ks, *vs;
  const int32_t *table, *kv_lens, *q_starts;
  int64_t width;            // pages a row of the table holds
  int pages, page_shift;
  int T, B, Hq, Hkv, G;     // G = Hq / Hkv rows per token and cached head
  int max_q, window, causal;
  float c;                  // softmax scale * log2(e)
  uint16_t *out;
  float *lse;               // or nullptr
  float *part, *part_wide;  // partial results of split units
  int32_t *units, *items;   // where they are: B * Hkv pairs, 2 * kAttnWideUnits pairs
  int few_rows;             // sequences with at most that many rows go to lcvq_attn.hip
};
// Sequences with at most 16 NB rows (new tokens times G), NB 1, 2 or 4
constexpr int kAttnFewBlocks = 512;
hipError_t launch_attn_few(const AttnArgs &a, int D, bool fp8, int NB, hipStream_t st);
int64_t attn_span(const AttnArgs &a, int64_t rows);  // the most tokens that `rows` rows in order see
bool attn_few_whole(const AttnArgs &a);      // no unit is split
int64_t attn_few_blocks(const AttnArgs &a);  // else: blocks that share the units' tokens,
hipError_t launch_attn_join(const AttnArgs &a, int D, int NB, hipStream_t st);  // and their pieces' join (NB 1, 2)
// Sequences with more than few_rows rows, kAttnWideRows at a time; with NB != 0 the others
// beside them
constexpr int kAttnWideRows = 128;
constexpr int kAttnWideUnits = 512;  // fewer units are split
hipError_t launch_attn_wide(const AttnArgs &a, int D, bool fp8, int NB, hipStream_t st);

// ---- 4-bit weights (lcvq_int4.hip) -----------------------------------------
struct Int4Args {
  const uint8_t *packed;
  const uint16_t *scales, *zeros;  // zeros: or nullptr
  int64_t m, n;
  int group;
  bool by_row;  // scales and zeros: m x n / group, else n / group x m
  bool y_bf16;
  float *part;  // int4_bytes of the tokens of a pass
};
struct Int4Plan {
  int KT, mr, spans, span;  // steps of 128 columns, 16-row blocks per block, spans of K, steps of a span
};
Int4Plan int4_plan(int64_t m, int64_t n, bool many, int most_mr);  // many: more than four tokens
int64_t int4_bytes(int64_t N, int64_t m, int64_t n);
// up to 16 tokens
hipError_t launch_int4(const Int4Args &a, const uint16_t *X, int Nc, char *Y, hipStream_t st);

}  // namespace lcvq
