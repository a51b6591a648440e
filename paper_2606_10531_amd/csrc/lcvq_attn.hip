// Attention of new tokens over a paged cache, few rows per sequence (decode, speculative
// tokens): each cached head's G query heads times the sequence's new tokens are the rows.
//
//   S = scale Q K^T over the visible tokens,  out = softmax(S) V,  lse = log sum exp S
//
// in one pass over the cache with a running maximum and sum per row (both fp32).
//
// Both products run on v_mfma_f32_16x16x32_bf16 with the rows on N: S^T = K Q^T leaves four
// tokens 4 (L / 16) + e of a row L % 16 in lane L, two 16-token blocks make eight, and those
// eight are the lane's K positions of the second product out^T = V^T P^T as they stand: the
// probabilities never leave their lane.  (Position 8 g + j of the 32 is token 4 g + j for
// j < 4 and 16 + 4 g + j - 4 above; V's operand is read in that order.)  V^T comes from the
// row-major tile in LDS by the transposing LDS reads.
//
// 8-bit entries: the codes go to the matrix core as bf16 without their scale (exact); K's
// scale multiplies the scores of its token, V's the probabilities, before they are
// rounded to bf16 (a power of two, so the rounding is the same as without it but for entries of
// scales near 2^-117, whose small probabilities go below the least normal number).
// Probabilities in bf16 cost up to 2^-8 relative each, as the output's own rounding does; their
// sum is taken from the unrounded values.
//
// Work: a unit is (sequence, cached head); its visible tokens are granules of 128, 32 per
// wave.  Where units are short or many, each has a block.  Else all units' granules in a row
// are dealt out in equal runs to the blocks, whatever the sequences' lengths; each block finds
// its first unit by a prefix sum over the sequences.  A unit inside one block is finished
// there; the pieces of a split one leave unnormalised sums, maximum and sum in the workspace
// for k_attn_join.
//
// Each wave stages its own 32-token tiles of K and V in LDS by direct loads, the next one
// in flight while the current one is multiplied: no barrier in the loop.
//
// Bound: HBM, the visible entries once, and for a few hundred tokens the latency of a chain of
// loads.  64 heads of 128 on 8: 64 sequences of up to 8000 in e4m3 (620 MB) 120 us, 5.2 TB/s, the rate
// of a large copy; one of 130001 53 us, 5 TB/s; 16 of 8000 in bf16 (524 MB) 95 us, 5.5 TB/s; one of
// 50000 in bf16 (205 MB) 40 us, 5.1 TB/s.  One of 333, 32 heads, bf16: 7 us.
#include <algorithm>

#include "lcvq_attn_few.hpp"

namespace lcvq {

// One LDS array: with others beside it the compiler waits for all direct loads before each read.
template <int D, bool kFp8, int NB, bool kWhole>
__global__ __launch_bounds__(256, NB == 4 && D == 128 ? 1 : 2) void k_attn_few(AttnArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[attn_few_lds<D, kFp8, NB>()];
  attn_few<D, kFp8, NB, kWhole>(a, lds, (int)blockIdx.x, (int)gridDim.x);
}

template <int D, int NB, int kShare>
__global__ __launch_bounds__(256) void k_attn_join(AttnArgs a) {
  __shared__ __attribute__((aligned(16))) char lds[attn_join_lds<D, kShare>()];
  attn_join_few<D, NB, kShare>(a, lds, (int)blockIdx.x);
}

// ---------------------------------------------------------------- launch ---
int64_t attn_span(const AttnArgs &a, int64_t rows) {
  const int64_t all = a.width << a.page_shift;
  return a.window > 0 ? std::min(all, a.window + (rows - 1) / a.G) : all;
}
// A block for each unit, and no join, up to 1024 visible tokens (whole / dealt out: 16 sequences of
// 1000 on 8 heads 13.5 / 19 us, 64 of them 18 / 28; one of 2000 on one head 17.5 / 15), and up
// to 4096 where there is a unit for every 16 of them (16 sequences of 2000 on 8 heads 18 / 22
// us, 128 of 4000 118 / 130; 8 of 4000 31 / 21).  (Times of calls, 11 us at least.)  Else
// the granules are dealt out.
bool attn_few_whole(const AttnArgs &a) {
  const int64_t span = attn_span(a, 64);
  return span <= 1024 || (span <= 4096 && span <= (int64_t)16 * a.B * a.Hkv);
}
// Two blocks for each of the 256 compute units, never more than there can be granules.
int64_t attn_few_blocks(const AttnArgs &a) {
  return std::min<int64_t>((int64_t)a.B * a.Hkv * (ceil_div(attn_span(a, 64), kGran) + 1), kAttnFewBlocks);
}

// Eight threads to a row where a unit can have 16 pieces or more, else four (one head of 50000, 391
// pieces, a graph of calls: 19.7 -> 15.7 us a call; 2 heads of 64 elements over 20000: 14.8 -> 12.8;
// 16 pieces, 4 sequences of 6000 on 8 heads: 19.1 both ways).
template <int D, int NB>
static hipError_t join(const AttnArgs &a, hipStream_t st) {
  if (attn_few_blocks(a) >= (int64_t)16 * a.B * a.Hkv)
    k_attn_join<D, NB, 8><<<(unsigned)attn_join_blocks<D, NB, 8>(a), 256, 0, st>>>(a);
  else
    k_attn_join<D, NB, 4><<<(unsigned)attn_join_blocks<D, NB, 4>(a), 256, 0, st>>>(a);
  return hipGetLastError();
}

template <int D, bool kFp8, int NB>
static hipError_t few(const AttnArgs &a, hipStream_t st) {
  if (attn_few_whole(a)) {
    k_attn_few<D, kFp8, NB, true><<<(unsigned)(a.B * a.Hkv), 256, 0, st>>>(a);
    return hipGetLastError();
  }
  // (one block to a compute unit where the registers or LDS hold no second one: 6 tokens of two
  // sequences of 24000, 32 heads of 128 on 4, e4m3: 46 -> 36 us a call.  Its kernel takes 27 us for
  // the 50 MB and 30 for the 98 of bf16: four waves to a compute unit keep few loads in flight.)
  constexpr int64_t kAtOnce = (NB == 4 && D == 128) || attn_few_lds<D, kFp8, NB>() > 80 * 1024 ? 256 : kAttnFewBlocks;
  k_attn_few<D, kFp8, NB, false><<<(unsigned)std::min(attn_few_blocks(a), kAtOnce), 256, 0, st>>>(a);
  return join<D, NB>(a, st);
}

hipError_t launch_attn_join(const AttnArgs &a, int D, int NB, hipStream_t st) {
  return D == 64 ? (NB == 1 ? join<64, 1> : join<64, 2>)(a, st) : (NB == 1 ? join<128, 1> : join<128, 2>)(a, st);
}

hipError_t launch_attn_few(const AttnArgs &a, int D, bool fp8, int NB, hipStream_t st) {
  using F = hipError_t (*)(const AttnArgs &, hipStream_t);
  static constexpr F f[2][2][3] = {{{few<64, false, 1>, few<64, false, 2>, few<64, false, 4>},
                                    {few<64, true, 1>, few<64, true, 2>, few<64, true, 4>}},
                                   {{few<128, false, 1>, few<128, false, 2>, few<128, false, 4>},
                                    {few<128, true, 1>, few<128, true, 2>, few<128, true, 4>}}};
  return f[D == 128][fp8][NB == 1 ? 0 : NB == 2 ? 1 : 2](a, st);
}

}  // namespace lcvq
