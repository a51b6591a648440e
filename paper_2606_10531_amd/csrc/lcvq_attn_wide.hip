// Attention of new tokens over a paged cache, many rows per sequence (a chunk of a prompt).
// The mathematics, operand forms and row order are those of lcvq_attn.hip.
//
// A unit is (sequence, 128 of its rows, cached head), rows in order of token and then query
// head; a block takes a unit, or one of `splits` parts of its visible tokens (wide_plan).  Its
// four waves have 32 rows each and share tiles of 64 tokens in LDS as bf16, K and V in two
// buffers each: 64 KiB for D = 128, so that two blocks stand on a compute unit, and one
// can multiply while the other is at its softmax.  (One block of 256 rows with the softmax of a
// tile woven between the products of the next takes 9 % longer at 512 tokens over 8192; one of
// 512 threads and 256 rows 5 % less there, but 4 % more on prompts and 50 % on mixed batches.)
//
// Tiles get to LDS through registers, tile i + 2 under way from the cache while tile i is
// multiplied and i + 1 is written: an 8-bit cache's entries are converted with their scales on
// the way, once per block, and with direct loads in flight the compiler waits for all of them
// before each transposing read.  The stores lie between the second product's instructions.
//
// Bound: the vector units and the matrix cores, which overlap in small part.  A wave's 32 rows
// and 64 tokens are 64 instructions of 8.4 ns (the rate that the chip holds) at D = 128 and 32
// exponentials per lane with as many multiplications, sums, maxima and conversions.  512 tokens
// over 8192 in e4m3, of whose cycles the matrix cores are busy in 0.40 and the vector units in 0.46
// at 64 heads of 128 on 8 (133 GFLOP): 128 to 134 us once the clock has settled (two cards; 150 the
// first dozen calls) and 9 for the join, 1.0 PFLOP/s; 0.24 and 0.45 at 32 heads of 64 (33 GFLOP, but half as many
// exponentials): 50 and 5 us, 0.66 PFLOP/s.  Three blocks of D = 64 on a compute unit (168
// registers) are no faster than two.
//
// The running maximum follows only when a row's has grown by 8 in log2 units, so that
// probabilities reach at most 2^8 and the rescaling branch is rare.  (Under the true maximum the
// largest probability is 1, which bf16 holds; under a lagging one it is rounded like the others.)
//
// Blocks of one cached head follow one another every Hkv blocks, so that with 8 (16, ..)
// heads an XCD's L2 holds its own head's entries.  The sequences go from last to first, and of each
// the last rows, which see most, come first: a long sequence in front begins late.
#include <algorithm>
#include <type_traits>
#include <utility>

#include "lcvq_attn_few.hpp"

namespace lcvq {

constexpr int kWideTok = 64;           // tokens of a tile
constexpr int kRing = 3;               // operands under way from LDS, and the one in use
constexpr float kWideSlack = 8.0f;     // log2 units that a row's maximum may lag

template <int... I, class F>
__device__ __forceinline__ void wide_for(std::integer_sequence<int, I...>, F f) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void wide_for(F f) {
  wide_for(std::make_integer_sequence<int, N>{}, f);
}

// v_maximum3_f32: unlike the maximum that skips a NaN it needs no instruction that quiets its
// operands (a NaN score makes its row NaN in any case)
__device__ __forceinline__ float wide_max(float a, float b) { return __builtin_elementwise_maximum(a, b); }

__device__ __forceinline__ int64_t seq_tiles(const AttnArgs &a, const AttnSeq &s) {
  const int64_t rows = (int64_t)s.nq * a.G;
  return s.nq <= 0 || rows <= a.few_rows ? 0 : (rows + kAttnWideRows - 1) / kAttnWideRows;
}

template <int D>
__device__ __forceinline__ constexpr int64_t wide_part_floats() {
  return (int64_t)kAttnWideRows * (D + 2);
}

// LDS of a block: K0 K1 V0 V1.
template <int D>
__host__ __device__ __forceinline__ constexpr int attn_wide_lds() {
  return 4 * kWideTok * 2 * D;
}

template <int D, bool kFp8>
__device__ __forceinline__ void attn_wide(const AttnArgs &a, char *lds, int block, int splits) {
  constexpr int NB = 2;
  constexpr int kSrc = kFp8 ? D : 2 * D;        // bytes of an entry in the cache
  constexpr int kRow = 2 * D, kChunks = kRow / 16;  // of an entry in LDS
  constexpr int kTileB = kWideTok * kRow;
  constexpr int kPer = kSrc / 16, kPass = 256 / kPer;  // 16-byte chunks of an entry, entries per pass of the block
  constexpr int kC = kWideTok / kPass;          // passes: chunks of K, and of V, per thread
  constexpr int kPuts = D / 16;                 // stores into LDS per thread and tile
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, c16 = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = block % a.Hkv, rest = block / a.Hkv, split = rest % splits, item = rest / splits;
  const AttnPlace pl = attn_place(
      a, [&](const AttnSeq &q) { return seq_tiles(a, q); }, [&](int64_t total) { return total - 1 - item; }, -1);
  const int b = pl.b, r0 = (int)(pl.total - 1 - item - pl.at) * kAttnWideRows;
  if (splits > 1 && h == 0 && split == 0 && tid == 0) {  // for k_attn_wide_join
    a.items[2 * item] = b;
    a.items[2 * item + 1] = r0;
  }
  if (b < 0) return;
  const AttnSeq sq = attn_uni(attn_seq(a, b));
  const int rows = sq.nq * a.G;
  const int r1 = min(rows, r0 + kAttnWideRows);

  bf16x8 qf[NB][D / 32];
  int lo[NB], hi[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    const int r = r0 + 32 * wave + 16 * n + c16, i = r / a.G, gq = r - i * a.G;
    const bool live = r < rows;
    attn_range(a, sq, live ? i : sq.nq - 1, lo[n], hi[n]);
    const uint16_t *qp = a.q + (int64_t)(sq.q0 + (live ? i : 0)) * a.q_token + (int64_t)(h * a.G + (live ? gq : 0)) * a.q_head;
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks) {
      const u32x4 w = live ? *reinterpret_cast<const u32x4 *>(qp + 32 * ks + 8 * g) : u32x4{0, 0, 0, 0};
      qf[n][ks] = __builtin_bit_cast(bf16x8, w);
    }
  }
  // tokens that some row of the block sees, and that every row of the wave sees
  int seen_lo, seen_hi, all_lo, all_hi, none;
  attn_range(a, sq, r0 / a.G, seen_lo, none);
  attn_range(a, sq, (r1 - 1) / a.G, none, seen_hi);
  attn_range(a, sq, min(r0 + 32 * wave, rows - 1) / a.G, none, all_hi);
  attn_range(a, sq, min(r0 + 32 * wave + 31, rows - 1) / a.G, all_lo, none);
  const int tile0 = seen_lo / kWideTok, tiles_all = max(0, (seen_hi + kWideTok - 1) / kWideTok - tile0);
  const int ta = (int)((int64_t)tiles_all * split / splits), tb = (int)((int64_t)tiles_all * (split + 1) / splits);
  const int tiles = tb - ta, tok0 = (tile0 + ta) * kWideTok;

  floatx4 acc[D / 16][NB];
  // mc: c m, or 0 where that is far and the exponents are c (x - m); far: some row's is
  bool far = true;
  float m[NB], mc[NB], l[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    m[n] = kAttnLow;
    mc[n] = attn_far(kAttnLow, a.c) ? 0.0f : kAttnLow * a.c;
    l[n] = 0.0f;
#pragma unroll
    for (int db = 0; db < D / 16; ++db) acc[db][n] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  }

  // ---- staging.  The pages of a tile's four 16-token groups: that of group l % 4 in lane l.
  const int32_t *table = a.table + (int64_t)b * a.width;
  auto page_of = [&](int i) __attribute__((always_inline)) {  // (some token is visible: len > 0)
    return table[min(tok0 + i * kWideTok + (lane & 3) * 16, sq.len - 1) >> a.page_shift];
  };
  // tokens that every row of the block sees
  int blk_lo, blk_hi;
  attn_range(a, sq, r0 / a.G, none, blk_hi);
  attn_range(a, sq, (r1 - 1) / a.G, blk_lo, none);
  bool odd = false;        // values have been left out
  u32x4 hold[2][kC];       // chunks of K and V under way
  uint32_t hold_s[2][kC];  // e4m3: their scale bytes
  // thread t takes chunk t % kPer of entry t / kPer + kPass j of the tile
  const int crow = tid / kPer, cchunk = tid % kPer;
  // chunk j of K (which = 0) or V (1) of tile i on the pages `ids`
  auto fetch = [&](int which, int j, int i, int ids) __attribute__((always_inline)) {
    const char *src = which ? a.v : a.k;
    const uint8_t *scale = which ? a.vs : a.ks;
    // the wave's entries lie in one group: the cache row of its first token and how many tokens
    // there are (0: no such page, or past the end), in scalar registers
    const int u = (wave * (kPass / 4) + j * kPass) / 16, id = __builtin_amdgcn_readlane(ids, u);
    const int t = tok0 + i * kWideTok + 16 * u, r = (crow + j * kPass) & 15;
    const bool there = (i < tiles) & (t < sq.len) & ((uint32_t)id < (uint32_t)a.pages);
    const int64_t row = (((int64_t)(there ? id : 0) * a.Hkv + h) << a.page_shift) + (t & ((1 << a.page_shift) - 1));
    const int left = there ? min(16, sq.len - t) : 0;
    hold[which][j] = __builtin_amdgcn_raw_buffer_load_b128(make_rsrc(src + row * kSrc, left * kSrc), r * kSrc + 16 * cchunk, 0, 0);
    if constexpr (kFp8) hold_s[which][j] = __builtin_amdgcn_raw_buffer_load_b8(make_rsrc(scale + row, left), r, 0, 0);
  };
  auto fetch_all = [&](int which, int i, int ids) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < kC; ++j) fetch(which, j, i, ids);
    __builtin_amdgcn_sched_barrier(0);
  };
  // store w of the kPuts: K first
  auto put = [&](auto w_c, int kbuf, int vbuf) __attribute__((always_inline)) {
    constexpr int w = decltype(w_c)::value, which = w / (kPuts / 2), x = w % (kPuts / 2), j = kFp8 ? x >> 1 : x;
    const int r = crow + j * kPass, c = kFp8 ? 2 * cchunk + (x & 1) : cchunk;
    char *at = lds + (which ? 2 + vbuf : kbuf) * kTileB + r * kRow + ((c ^ attn_swz<kChunks>(r)) << 4);
    if constexpr (kFp8) {
      const uint32_t w0 = hold[which][j][2 * (x & 1)], w1 = hold[which][j][2 * (x & 1) + 1];
      *reinterpret_cast<bf16x8 *>(at) = e4m3_to_bf16x8(w0, w1, kv_scale(hold_s[which][j]));
    } else {
      *reinterpret_cast<u32x4 *>(at) = hold[which][j];
    }
  };
  // V of tile i, which some rows may not see, without values that are no numbers
  auto sift = [&](int i) __attribute__((always_inline)) {
    const int t0 = tok0 + i * kWideTok;
    if ((t0 >= blk_lo) & (t0 + kWideTok <= blk_hi)) return;
    bool any = false;
#pragma unroll
    for (int j = 0; j < kC; ++j) any |= attn_odd<kFp8>(hold[1][j]) || (kFp8 && hold_s[1][j] > kKvByteTop);
    if (__ballot(any) == 0) return;
    odd = true;
#pragma unroll
    for (int j = 0; j < kC; ++j) {
      hold[1][j] = attn_without_odd<kFp8>(hold[1][j]);
      if (kFp8 && hold_s[1][j] > kKvByteTop) {
        hold[1][j] = u32x4{0u, 0u, 0u, 0u};
        hold_s[1][j] = 127;
      }
    }
  };
  // ---- operands
  auto k_operand = [&](int buf, int u, int ks) __attribute__((always_inline)) {
    return *reinterpret_cast<const bf16x8 *>(lds + buf * kTileB + (16 * u + c16) * kRow + (((4 * ks + g) ^ attn_swz<kChunks>(c16)) << 4));
  };
  auto v_operand = [&](int buf, int k, int db) __attribute__((always_inline)) {
    return attn_v_operand<D, false>(lds + (2 + buf) * kTileB + k * 32 * kRow, lane, db);
  };
  auto hide = [&](int i, int ids, floatx4 (&s)[4][NB]) __attribute__((always_inline)) {
    const int t0 = tok0 + i * kWideTok;
    const uint32_t there = (uint32_t)__ballot((uint32_t)ids < (uint32_t)a.pages) & 15u;  // (past the end hi hides)
    if ((t0 >= all_lo) & (t0 + kWideTok <= all_hi) & (there == 15u)) return;
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int t = t0 + 16 * u + 4 * g + e;
#pragma unroll
        for (int n = 0; n < NB; ++n) s[u][n][e] = (t >= lo[n]) & (t < hi[n]) & ((there >> u) & 1) ? s[u][n][e] : -__builtin_inff();
      }
  };
  // mx: maxima of a tile's scores over the lane's tokens.  New running maxima where a row's has
  // grown by more than the slack.
  auto follow = [&](float (&mx)[NB]) __attribute__((always_inline)) {
    float over = (mx[0] - m[0]) * a.c;
#pragma unroll
    for (int n = 1; n < NB; ++n) over = fmaxf(over, (mx[n] - m[n]) * a.c);
    if (__ballot(over > kWideSlack) == 0) return;
    bool any_far = false;
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const float mn = fmaxf(m[n], attn_max4(mx[n])), f = __builtin_amdgcn_exp2f((m[n] - mn) * a.c);
      m[n] = mn;
      mc[n] = attn_far(mn, a.c) ? 0.0f : mn * a.c;
      any_far |= attn_far(mn, a.c);
      l[n] *= f;
#pragma unroll
      for (int db = 0; db < D / 16; ++db) acc[db][n] *= f;
    }
    far = __ballot(any_far) != 0;
  };

  constexpr int kKs = D / 32, kDb = D / 16;
  // Tile i on the pages id0.  K(i + 1) and V(i + 1) are under way; those of i + 2, on id2, take
  // their registers.
  auto body = [&](auto par_c, int i, int id0, int id2) __attribute__((always_inline)) {
    constexpr int par = decltype(par_c)::value;
    floatx4 s[4][NB];
    bf16x8 kf[kRing];
    wide_for<kRing - 1>([&](auto f) __attribute__((always_inline)) { kf[f] = k_operand(par, f / kKs, f % kKs); });
    wide_for<4 * kKs>([&](auto f_c) __attribute__((always_inline)) {
      constexpr int f = decltype(f_c)::value, u = f / kKs, ks = f % kKs, fn = f + kRing - 1;
      if constexpr (fn < 4 * kKs) kf[fn % kRing] = k_operand(par, fn / kKs, fn % kKs);
#pragma unroll
      for (int n = 0; n < NB; ++n)
        s[u][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[f % kRing], qf[n][ks], ks == 0 ? floatx4{0.0f, 0.0f, 0.0f, 0.0f} : s[u][n], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    });
    hide(i, id0, s);
    float mx[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      mx[n] = s[0][n][0];
#pragma unroll
      for (int j = 1; j < 16; ++j) mx[n] = wide_max(mx[n], s[j >> 2][n][j & 3]);
    }
    follow(mx);
    if (far) {
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        const float off = attn_far(m[n], a.c) ? m[n] : 0.0f;
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[u][n][e] -= off;
      }
    }
    bf16x8 pf[2][NB];
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        float p[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = __builtin_amdgcn_exp2f(fmaf(s[2 * k + (j >> 2)][n][j & 3], a.c, -mc[n]));
#pragma unroll
        for (int j = 0; j < 8; ++j) l[n] += p[j];
        const u32x4 w = {pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7])};
        pf[k][n] = __builtin_bit_cast(bf16x8, w);
      }
    __builtin_amdgcn_sched_barrier(0);
    sift(i + 1);
    bf16x8 vf[kRing];
    wide_for<kRing - 1>([&](auto f) __attribute__((always_inline)) { vf[f] = v_operand(par, 0, f); });
    __builtin_amdgcn_s_setprio(1);  // (the other block's wave on the SIMD has its softmax then: 3 % at 512 tokens over 8192)
    wide_for<2 * kDb>([&](auto f_c) __attribute__((always_inline)) {
      constexpr int f = decltype(f_c)::value, k = f / kDb, db = f % kDb, fn = f + kRing - 1;
      if constexpr (fn < 2 * kDb) vf[fn % kRing] = v_operand(par, fn / kDb, fn % kDb);
#pragma unroll
      for (int n = 0; n < NB; ++n) acc[db][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[f % kRing], pf[k][n], acc[db][n], 0, 0, 0);
      constexpr int kGap = 2 * kDb / kPuts;
      if constexpr (f % kGap == kGap - 1) {
        constexpr int w = f / kGap, which = w / (kPuts / 2), x = w % (kPuts / 2);
        put(std::integral_constant<int, w>{}, 1 - par, 1 - par);
        if constexpr (!kFp8 || (x & 1)) fetch(which, kFp8 ? x >> 1 : x, i + 2, id2);
      }
      __builtin_amdgcn_sched_barrier(0);
    });
    __builtin_amdgcn_s_setprio(0);
    LCVQ_WAIT_LGKM0();
    LCVQ_BARRIER();
  };

  if (tiles > 0) {
    int id0 = page_of(0), id1 = page_of(1), id2 = page_of(2), id3 = page_of(3);
    fetch_all(0, 0, id0);
    fetch_all(1, 0, id0);
    sift(0);
    wide_for<kPuts>([&](auto w) __attribute__((always_inline)) { put(w, 0, 0); });
    fetch_all(0, 1, id1);
    fetch_all(1, 1, id1);
    LCVQ_WAIT_LGKM0();
    LCVQ_BARRIER();
    // in pairs (no way out between the two: the loads under way would be waited for at the join)
    int i = 0;
    for (; i + 1 < tiles; i += 2) {
      const int id4 = page_of(i + 4);
      body(std::integral_constant<int, 0>{}, i, id0, id2);
      const int id5 = page_of(i + 5);
      body(std::integral_constant<int, 1>{}, i + 1, id1, id3);
      id0 = id2;
      id1 = id3;
      id2 = id4;
      id3 = id5;
    }
    if (i < tiles) body(std::integral_constant<int, 0>{}, i, id0, id2);
  }

#pragma unroll
  for (int n = 0; n < NB; ++n) {
    l[n] = attn_sum4(l[n]);
    const int r = r0 + 32 * wave + 16 * n + c16;
    if (r >= rows) continue;
    if (splits == 1) {
#pragma unroll
      for (int db = 0; db < D / 16; ++db) attn_store(a, sq, h, r, 16 * db + 4 * g, D, acc[db][n], m[n], l[n]);
    } else {
      float *part = a.part_wide + (((int64_t)item * a.Hkv + h) * splits + split) * wide_part_floats<D>();
#pragma unroll
      for (int db = 0; db < D / 16; ++db) *reinterpret_cast<floatx4 *>(part + (int64_t)(r - r0) * D + 16 * db + 4 * g) = acc[db][n];
      if (g == 0) {
        part[kAttnWideRows * D + r - r0] = m[n];
        part[kAttnWideRows * D + kAttnWideRows + r - r0] = l[n];
      }
    }
  }
  uint32_t *flags = reinterpret_cast<uint32_t *>(lds);  // (the tiles are read)
  if (lane == 0) flags[wave] = odd ? 1u : 0u;
  __syncthreads();
  if ((flags[0] | flags[1] | flags[2] | flags[3]) != 0) {
    float *part = a.part_wide + (((int64_t)item * a.Hkv + h) * splits + split) * wide_part_floats<D>();
    attn_put_odd<D, kFp8, kWideTok>(a, sq, b, h, r0, r1, tok0, tok0 + tiles * kWideTok, blk_lo, blk_hi, [&](int r, int d, float sum) {
      if (splits == 1)
        attn_put_out<D>(a, sq, h, r, d, sum);
      else
        part[(int64_t)(r - r0) * D + d] += sum;
    });
  }
}

template <int D, bool kFp8>
__global__ __launch_bounds__(256, 2) void k_attn_wide(AttnArgs a, int splits) {
  __shared__ __attribute__((aligned(1024))) char lds[attn_wide_lds<D>()];
  attn_wide<D, kFp8>(a, lds, (int)blockIdx.x, splits);
}

// Both kinds of sequence in one launch: the first `few` blocks stream the cache for the
// sequences with few rows (kWhole: a unit each; else one on a compute unit) while those behind
// them multiply.  (Both in turn, eight blocks at a time, takes longer: 32 tokens beside a chunk
// of 1000 under a window of 2048 54 us, few rows first 48.)  One stage where two would fill the
// compute unit's LDS with one block.
template <int D, bool kFp8>
constexpr int kMixedStages = attn_few_lds<D, kFp8, 2>() > 80 * 1024 ? 1 : 2;
template <int D, bool kFp8, int NB, bool kWhole>
__global__ __launch_bounds__(256, 2) void k_attn_mixed(AttnArgs a, int few, int splits) {
  constexpr int kStages = kMixedStages<D, kFp8>;
  constexpr int kF = attn_few_lds<D, kFp8, NB, kStages>(), kW = attn_wide_lds<D>();
  static_assert(kF <= 80 * 1024, "two blocks on a compute unit");
  __shared__ __attribute__((aligned(1024))) char lds[kF > kW ? kF : kW];
  if ((int)blockIdx.x < few)
    attn_few<D, kFp8, NB, kWhole, kStages>(a, lds, (int)blockIdx.x, few);
  else
    attn_wide<D, kFp8>(a, lds, (int)blockIdx.x - few, splits);
}

// Joins the parts of the units' tokens (up to 64); the first `few` blocks those of the sequences with few
// rows (NB 0: none).  kShare 4 for more than four parts (27 parts of 140 tokens over 7000, two
// cached heads: 17 -> 5.6 us), else 1 (two parts of 512 tokens over 8192, 8 cached heads: 9.3 us,
// 15.2 with four threads to a row, half of them idle).
template <int D, int NB, int kShare>
__global__ __launch_bounds__(256) void k_attn_wide_join(AttnArgs a, int few, int splits) {
  __shared__ __attribute__((aligned(16))) char lds[attn_join_lds<D, 4>()];
  constexpr int kR = attn_join_rows<D, kShare>();
  int block = (int)blockIdx.x;
  if constexpr (NB != 0) {
    if (block < few) {
      attn_join_few<D, NB>(a, lds, block);
      return;
    }
    block -= few;
  }
  const int unit = block / (kAttnWideRows / kR), h = unit % a.Hkv, item = unit / a.Hkv;
  const int b = a.items[2 * item], r0 = a.items[2 * item + 1];
  if (b < 0) return;
  const AttnSeq sq = attn_seq(a, b);
  const int r = block % (kAttnWideRows / kR) * kR + (int)threadIdx.x / (D / 4) % kR, rows = sq.nq * a.G - r0;
  const float *part = a.part_wide + ((int64_t)item * a.Hkv + h) * splits * wide_part_floats<D>();
  attn_join<D, kShare, kAttnWideRows>(a, lds, sq, h, min(r, rows - 1), r0 + r, r < rows, splits,
                                      [&](int i) { return part + i * wide_part_floats<D>(); });
}

// ---------------------------------------------------------------- launch ---
struct WidePlan {
  int64_t units;  // at most that many (row tile, cached head)
  int splits;
};
// Parts: the number that takes least time by this model, whose unit is a tile of a block with
// another one on its compute unit (1.9 us; 1.2 for D = 64), for as many sequences of max_q new
// tokens as T has room for.  512 blocks run at once, and up to 256, one to a compute unit, take
// 0.65 of the time (0.8 for D = 64 with nothing else to run, whose tiles are shorter than the
// loads' way); a block begins and ends in 3 tiles' time, the join in another 3, and 512 parts
// are written and read in 7 (5).  Blocks for single tokens beside them are not counted.  (900 tokens over 4096, 64 heads on 8: 456 units whole 131 us, in two
// parts 152.  1500 over 8000, 32 heads of 64: 376 units whole 152 us, in two parts 145.)
static WidePlan wide_plan(const AttnArgs &a, int D, bool alone) {
  const double one = D == 64 && alone ? 0.8 : 0.65, parts = D == 64 ? 5.0 : 7.0;
  const int64_t per = ceil_div((int64_t)a.max_q * a.G, kAttnWideRows), steps = ceil_div(attn_span(a, kAttnWideRows), kWideTok);
  const int64_t likely = std::max<int64_t>(a.T / a.max_q, 1) * per * a.Hkv;
  WidePlan p;
  p.units = std::min<int64_t>((int64_t)a.T * a.G / kAttnWideRows + a.B, (int64_t)a.B * per) * a.Hkv;
  p.splits = 1;
  const int most = (int)std::min<int64_t>({64, 2 * kAttnWideUnits / p.units, steps / 2});
  double best = 0.0;
  for (int s = 1; s <= std::max(most, 1); ++s) {
    const int64_t blocks = likely * s, rest = blocks % 512;
    const double rounds = (double)(blocks / 512) + (rest == 0 ? 0.0 : rest <= 256 ? one : 1.0);
    const double time = rounds * ((double)steps / s + 3.0) + (s > 1 ? 3.0 + parts * (double)blocks / 512 : 0.0);
    if (s == 1 || time < best) {
      best = time;
      p.splits = s;
    }
  }
  return p;
}

template <int D, int NB>
static void wide_join(const AttnArgs &a, const WidePlan &p, hipStream_t st) {
  const unsigned few = NB != 0 ? (unsigned)attn_join_blocks<D, NB>(a) : 0;
  auto go = [&](auto share) {
    constexpr int kShare = decltype(share)::value;
    const unsigned blocks = few + (unsigned)p.units * (kAttnWideRows / attn_join_rows<D, kShare>());
    k_attn_wide_join<D, NB, kShare><<<blocks, 256, 0, st>>>(a, (int)few, p.splits);
  };
  if (p.splits > 4)
    go(std::integral_constant<int, 4>{});
  else
    go(std::integral_constant<int, 1>{});
}

template <int D, bool kFp8>
static hipError_t wide(const AttnArgs &a, int NB, hipStream_t st) {
  // (NB 4 would leave one block to a compute unit)
  const bool both = NB != 0 && NB < 4;
  const WidePlan p = wide_plan(a, D, !both);
  if (both) {
    const bool whole = attn_few_whole(a);
    const int few = whole ? a.B * a.Hkv : (int)std::min<int64_t>(attn_few_blocks(a), 256);
    auto k = NB == 1 ? (whole ? k_attn_mixed<D, kFp8, 1, true> : k_attn_mixed<D, kFp8, 1, false>)
                     : (whole ? k_attn_mixed<D, kFp8, 2, true> : k_attn_mixed<D, kFp8, 2, false>);
    k<<<(unsigned)(few + p.units * p.splits), 256, 0, st>>>(a, few, p.splits);
    if (p.splits > 1)
      (whole ? wide_join<D, 0> : NB == 1 ? wide_join<D, 1> : wide_join<D, 2>)(a, p, st);
    else if (!whole)
      return launch_attn_join(a, D, NB, st);
    return hipGetLastError();
  }
  if (NB != 0) {
    const hipError_t e = launch_attn_few(a, D, kFp8, NB, st);
    if (e != hipSuccess) return e;
  }
  k_attn_wide<D, kFp8><<<(unsigned)(p.units * p.splits), 256, 0, st>>>(a, p.splits);
  if (p.splits > 1) wide_join<D, 0>(a, p, st);
  return hipGetLastError();
}

hipError_t launch_attn_wide(const AttnArgs &a, int D, bool fp8, int NB, hipStream_t st) {
  auto go = D == 64 ? (fp8 ? wide<64, true> : wide<64, false>) : (fp8 ? wide<128, true> : wide<128, false>);
  return go(a, NB, st);
}

}  // namespace lcvq
