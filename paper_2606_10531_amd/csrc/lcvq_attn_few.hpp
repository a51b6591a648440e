// The block program of k_attn_few (lcvq_attn.hip, which has the mathematics), shared with the
// kernel that runs it beside the wide one.
#pragma once

#include <algorithm>

#include "lcvq_attn.hpp"

namespace lcvq {

constexpr int kGran = 128;  // tokens per granule: 32 for each of the four waves

// Granules of a sequence in this kernel: at least one for a sequence with rows (somebody
// writes them), none for those with more than `rows` rows, which the wide kernel takes.
__device__ __forceinline__ int64_t seq_granules(const AttnArgs &a, const AttnSeq &s, int rows) {
  if (s.nq <= 0 || s.nq * a.G > rows) return 0;
  const int n = (s.len + kGran - 1) / kGran - s.first(a) / kGran;
  return n < 1 ? 1 : n;
}

// First granule of block p when `total` of them are dealt out to at most `blocks` blocks, none
// of which stays empty between others.
__device__ __forceinline__ int64_t attn_share(int64_t total, int blocks, int p) {
  const int64_t n = min(total, (int64_t)blocks);
  return p >= n ? total : total * p / n;
}

// One partial result: 16 NB rows of D sums, then their maxima, then their sums.
template <int D, int NB>
__device__ __forceinline__ constexpr int64_t part_floats() {
  return (int64_t)16 * NB * (D + 2);
}

// LDS of a block: kStages tiles of K and V for each wave, or the waves' sums; then their
// statistics and flags.
template <int D, bool kFp8, int NB, int kStages>
__host__ __device__ __forceinline__ constexpr int attn_few_data() {
  const int stage = 4 * kStages * 2 * 32 * (kFp8 ? D : 2 * D), merge = 4 * 16 * NB * ((NB == 4 ? D / 2 : D) + 4) * 4;
  return stage > merge ? stage : merge;
}
template <int D, bool kFp8, int NB, int kStages = 2>
__host__ __device__ __forceinline__ constexpr int attn_few_lds() {
  return attn_few_data<D, kFp8, NB, kStages>() + 2 * 4 * 16 * NB * 4 + 16;
}

// Block p of `blocks`.  kWhole: block (b, h) takes the whole unit, and there is nothing to join.
// kStages 2: the next tile is under way while one is multiplied; 1 leaves that to another block.
template <int D, bool kFp8, int NB, bool kWhole, int kStages = 2>
__device__ __forceinline__ void attn_few(const AttnArgs &a, char *lds, int p, int blocks) {
  constexpr int kRow = kFp8 ? D : 2 * D;      // bytes of an entry
  constexpr int kChunks = kRow / 16;          // 16-byte chunks of an entry
  constexpr int kTileB = 32 * kRow;           // bytes of a wave's tile
  constexpr int kLoads = kRow / 64;           // direct loads of a 16-token group
  constexpr int kRowsL = 64 / kChunks;        // entries per load
  constexpr int kRows = 16 * NB;
  constexpr int kHalf = NB == 4 ? 2 : 1;      // the waves' sums are added in that many parts of D
  constexpr int kDh = D / kHalf;
  constexpr int kData = attn_few_data<D, kFp8, NB, kStages>();
  float (&s_m)[4][kRows] = *reinterpret_cast<float (*)[4][kRows]>(lds + kData);
  float (&s_l)[4][kRows] = *reinterpret_cast<float (*)[4][kRows]>(lds + kData + 4 * kRows * 4);
  uint32_t *s_odd = reinterpret_cast<uint32_t *>(lds + kData + 2 * 4 * kRows * 4);
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, c16 = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  char *stage = lds + wave * 2 * kStages * kTileB;

  // Of lane l: the page of 16-token group l % 2, this wave's part, of granule id0 + l / 2 of 32.
  int b, ids = 0, id0 = 0;
  AttnSeq sq;
  int64_t at, pos, end, nb_;  // granules before the sequence, the block's, the sequence's per unit
  if constexpr (kWhole) {
    b = p / a.Hkv;
    const int t = (lane >> 1) * kGran + wave * 32 + (lane & 1) * 16;
    if (t < a.width << a.page_shift)
      ids = a.table[(int64_t)b * a.width + (t >> a.page_shift)];  // (before its length is known)
    sq = attn_uni(attn_seq(a, b));
    nb_ = seq_granules(a, sq, kRows);
    if (nb_ == 0) return;
    at = pos = 0;
    end = nb_;
  } else {
    const AttnPlace pl = attn_place(
        a, [&](const AttnSeq &q) { return seq_granules(a, q, kRows) * a.Hkv; },
        [&](int64_t total) { return attn_share(total, blocks, p); }, -1);
    pos = attn_share(pl.total, blocks, p);
    end = attn_share(pl.total, blocks, p + 1);
    if (pos >= end || pl.b < 0) return;
    b = pl.b;
    at = pl.at;
    sq = attn_uni(attn_seq(a, b));
    nb_ = seq_granules(a, sq, kRows);
  }
  bool first_piece = true;

  // lane-constant offsets: direct loads (chunk swizzled by the row), K operand, V operand
  uint32_t goff[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int r = i * kRowsL + lane / kChunks, pos16 = lane % kChunks;
    goff[i] = (uint32_t)(r * kRow + ((pos16 ^ attn_swz<kChunks>(r)) << 4));
  }

  while (pos < end) {
    while (!kWhole && pos >= at + nb_ * a.Hkv) {  // next sequence with granules (there is one: pos < end <= total)
      at += nb_ * a.Hkv;
      ++b;
      sq = attn_uni(attn_seq(a, b));
      nb_ = seq_granules(a, sq, kRows);
    }
    const int h = kWhole ? p - b * a.Hkv : (int)((pos - at) / nb_);
    const int64_t unit0 = kWhole ? 0 : at + h * nb_;
    const int64_t stop = min(end, unit0 + nb_);
    const int gran0 = sq.first(a) / kGran;
    const int ga = gran0 + (int)(pos - unit0), gb = gran0 + (int)(stop - unit0);
    const int rows = sq.nq * a.G;

    // ---- rows: Q operand and the visible range of each
    bf16x8 qf[NB][D / 32];
    int lo[NB], hi[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const int r = 16 * n + c16, i = r / a.G, gq = r - i * a.G;
      const bool live = r < rows;
      attn_range(a, sq, live ? i : 0, lo[n], hi[n]);
      const uint16_t *qp = a.q + (int64_t)(sq.q0 + (live ? i : 0)) * a.q_token + (int64_t)(h * a.G + (live ? gq : 0)) * a.q_head;
#pragma unroll
      for (int ks = 0; ks < D / 32; ++ks) {
        const int e0 = kFp8 ? 64 * (ks >> 1) + 16 * g + 8 * (ks & 1) : 32 * ks + 8 * g;
        const u32x4 w = live ? *reinterpret_cast<const u32x4 *>(qp + e0) : u32x4{0, 0, 0, 0};
        qf[n][ks] = __builtin_bit_cast(bf16x8, w);
      }
    }
    // tokens that every row sees: no mask is needed inside
    int all_lo, all_hi, none;
    attn_range(a, sq, 0, none, all_hi);
    attn_range(a, sq, sq.nq - 1, all_lo, none);

    floatx4 acc[D / 16][NB];
    float m[NB], mc[NB], l[NB];  // mc: c m, or 0 where that is far and the exponents are c (x - m)
    uint32_t far = (1u << NB) - 1;  // the n some of whose rows are far
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      m[n] = kAttnLow;
      mc[n] = attn_far(kAttnLow, a.c) ? 0.0f : kAttnLow * a.c;
      l[n] = 0.0f;
#pragma unroll
      for (int db = 0; db < D / 16; ++db) acc[db][n] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    const int tok0 = ga * kGran + wave * 32, tok_end = min(gb * kGran, sq.len);
    const int steps = tok_end > tok0 ? (tok_end - tok0 + kGran - 1) / kGran : 0;
    auto load_pages = [&](int i0) __attribute__((always_inline)) {
      if (kWhole && ga + min(steps, i0 + 32) <= 32) return;  // they are there
      id0 = ga + i0;
      const int t = tok0 + (i0 + (lane >> 1)) * kGran + (lane & 1) * 16;
      ids = t < sq.len ? a.table[(int64_t)b * a.width + (t >> a.page_shift)] : -1;
    };
    auto page_id = [&](int i, int u) __attribute__((always_inline)) {
      return __builtin_amdgcn_readlane(ids, 2 * ((ga + i - id0) & 31) + u);
    };
    bool odd = false;  // the wave has left values out
    uint32_t ksc[2][2], vsc[2][2];
    // Loads of step i (of `steps`; a step past them loads nothing: the buffers are empty)
    auto issue = [&](int buf, int i) __attribute__((always_inline)) {
      LCVQ_WAIT_LGKM0();  // what was read from the buffer has arrived
      __builtin_amdgcn_sched_barrier(0);
      uint32_t base = (uint32_t)(wave * 2 * kStages * kTileB + buf * 2 * kTileB);
      asm volatile("" : "+s"(base));
      int64_t row[2];
      int left[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int id = page_id(i, u), t = tok0 + i * kGran + u * 16;
        const bool there = (uint32_t)id < (uint32_t)a.pages && i < steps && t < sq.len;
        row[u] = (((int64_t)(there ? id : 0) * a.Hkv + h) << a.page_shift) + (t & ((1 << a.page_shift) - 1));
        left[u] = there ? min(16, sq.len - t) : 0;
        if constexpr (kFp8) {
          ksc[buf][u] = __builtin_amdgcn_raw_buffer_load_b32(make_rsrc(a.ks + row[u], there ? 16 : 0), 4 * g, 0, 0);
          vsc[buf][u] = __builtin_amdgcn_raw_buffer_load_b32(make_rsrc(a.vs + row[u], there ? 16 : 0), 4 * g, 0, 0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const __amdgpu_buffer_rsrc_t rk = make_rsrc(a.k + row[u] * kRow, left[u] * kRow);
        const __amdgpu_buffer_rsrc_t rv = make_rsrc(a.v + row[u] * kRow, left[u] * kRow);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
          buffer_to_lds16(rk, (lds_void *)(lds + base + (u * kLoads + j) * 1024), goff[j]);
          buffer_to_lds16(rv, (lds_void *)(lds + base + kTileB + (u * kLoads + j) * 1024), goff[j]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    auto step = [&](int buf, int i) __attribute__((always_inline)) {
      const char *kt = stage + buf * 2 * kTileB, *vt = kt + kTileB;
      const int t0 = tok0 + i * kGran;
      floatx4 s[2][NB];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int n = 0; n < NB; ++n) s[u][n] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int u = 0; u < 2; ++u) attn_scores<D, kFp8, NB>(kt, 16 * u + c16, g, qf, s[u]);
      float ks8[8], vs8[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        ks8[j] = kFp8 ? kv_scale((ksc[buf][j >> 2] >> (8 * (j & 3))) & 0xffu) : 1.0f;
        vs8[j] = kFp8 ? kv_scale((vsc[buf][j >> 2] >> (8 * (j & 3))) & 0xffu) : 1.0f;
      }
      const bool page0 = (uint32_t)page_id(i, 0) < (uint32_t)a.pages;
      const bool page1 = (uint32_t)page_id(i, 1) < (uint32_t)a.pages;
      const bool masked = !((t0 >= all_lo) & (t0 + 32 <= all_hi) & page0 & page1);
      bf16x8 pf[NB];
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        float x[8];
        uint32_t seen = 0xffu;
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = kFp8 ? s[j >> 2][n][j & 3] * ks8[j] : s[j >> 2][n][j & 3];
        if (masked) {
          seen = 0;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int u = j >> 2, t = t0 + 16 * u + 4 * g + (j & 3);
            const bool on = (t >= lo[n]) & (t < hi[n]) & (u ? page1 : page0);
            seen |= on ? 1u << j : 0u;
            x[j] = on ? x[j] : -__builtin_inff();
          }
        }
        float mx = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
        mx = attn_max4(mx);
        if (__ballot(mx > m[n])) {
          const float mn = fmaxf(m[n], mx), f = __builtin_amdgcn_exp2f((m[n] - mn) * a.c);
          m[n] = mn;
          mc[n] = attn_far(mn, a.c) ? 0.0f : mn * a.c;
          far = __ballot(attn_far(mn, a.c)) != 0 ? far | 1u << n : far & ~(1u << n);
          l[n] *= f;
#pragma unroll
          for (int db = 0; db < D / 16; ++db) acc[db][n] *= f;
        }
        if (far >> n & 1) {  // (rows that are not keep their bits)
          const float off = attn_far(m[n], a.c) ? m[n] : 0.0f;
#pragma unroll
          for (int j = 0; j < 8; ++j) x[j] -= off;
        }
        float pr[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          pr[j] = __builtin_amdgcn_exp2f(fmaf(x[j], a.c, -mc[n]));
          l[n] += pr[j];
          if (kFp8) pr[j] *= vs8[j];
          if (masked) pr[j] = (seen >> j) & 1 ? pr[j] : 0.0f;
        }
        const u32x4 w = {pack_bf16x2(pr[0], pr[1]), pack_bf16x2(pr[2], pr[3]), pack_bf16x2(pr[4], pr[5]),
                         pack_bf16x2(pr[6], pr[7])};
        pf[n] = __builtin_bit_cast(bf16x8, w);
      }
      if (masked) {  // hidden tokens' values that are no numbers (those of missing pages are zeros)
        u32x4 *w = reinterpret_cast<u32x4 *>(lds + wave * 2 * kStages * kTileB + buf * 2 * kTileB + kTileB) + lane;
        bool any = false;
#pragma unroll
        for (int j = 0; j < 2 * kLoads; ++j) any |= attn_odd<kFp8>(w[64 * j]);
        if (__ballot(any) != 0 && !((t0 >= all_lo) & (t0 + 32 <= all_hi))) {
#pragma unroll
          for (int j = 0; j < 2 * kLoads; ++j) w[64 * j] = attn_without_odd<kFp8>(w[64 * j]);
          odd = true;
        }
      }
#pragma unroll
      for (int db = 0; db < D / 16; ++db) {
        const bf16x8 va = attn_v_operand<D, kFp8>(vt, lane, db);
#pragma unroll
        for (int n = 0; n < NB; ++n) acc[db][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pf[n], acc[db][n], 0, 0, 0);
      }
    };
    constexpr int kFlight = 4 * kLoads + (kFp8 ? 4 : 0);  // loads of a stage
    // Steps in pairs, the last of an odd number behind the loop; no way out between the loads
    // and the step that they belong to, or the compiler waits for all of them at the join.
    for (int i0 = 0; i0 < steps; i0 += 32) {
      load_pages(i0);
      const int i1 = min(steps, i0 + 32);
      if constexpr (kStages == 1) {
        for (int i = i0; i < i1; ++i) {
          issue(0, i);
          attn_wait_vm<0>();
          step(0, i);
        }
        continue;
      }
      issue(0, i0);
      int i = i0;
      for (; i + 1 < i1; i += 2) {
        issue(1, i + 1);
        attn_wait_vm<kFlight>();
        step(0, i);
        issue(0, i + 2 < i1 ? i + 2 : steps);
        attn_wait_vm<kFlight>();
        step(1, i + 1);
      }
      attn_wait_vm<0>();
      if (i < i1) step(0, i);
    }

    // ---- the waves' sums
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      l[n] = attn_sum4(l[n]);
      if (g == 0) {
        s_m[wave][16 * n + c16] = m[n];
        s_l[wave][16 * n + c16] = l[n];
      }
    }
    if (lane == 0) s_odd[wave] = odd ? 1u : 0u;
    __syncthreads();  // (also: every wave has read its last tile)
    float f[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const int r = 16 * n + c16;
      f[n] = __builtin_amdgcn_exp2f((m[n] - fmaxf(fmaxf(s_m[0][r], s_m[1][r]), fmaxf(s_m[2][r], s_m[3][r]))) * a.c);
    }
    const bool whole = kWhole || (pos == unit0 && stop == unit0 + nb_);
    if (!kWhole && tid == 0) {  // where the unit's pieces are, for k_attn_join
      int32_t *u = a.units + 2 * ((int64_t)b * a.Hkv + h);
      if (pos == unit0) u[0] = 2 * p + (first_piece ? 0 : 1);
      if (stop == unit0 + nb_) u[1] = p;
    }
    float *part = a.part + (2 * (int64_t)p + (first_piece ? 0 : 1)) * part_floats<D, NB>();
    float *red = reinterpret_cast<float *>(lds);
#pragma unroll
    for (int half = 0; half < kHalf; ++half) {
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int db = 0; db < kDh / 16; ++db)
          *reinterpret_cast<floatx4 *>(red + (wave * kRows + 16 * n + c16) * (kDh + 4) + 16 * db + 4 * g) =
              acc[half * (kDh / 16) + db][n] * f[n];
      __syncthreads();
      for (int it = tid; it < rows * (kDh / 4); it += 256) {
        const int r = it / (kDh / 4), d0 = 4 * (it - r * (kDh / 4));
        floatx4 v = *reinterpret_cast<const floatx4 *>(red + r * (kDh + 4) + d0);
#pragma unroll
        for (int w = 1; w < 4; ++w) v += *reinterpret_cast<const floatx4 *>(red + (w * kRows + r) * (kDh + 4) + d0);
        const float mx = fmaxf(fmaxf(s_m[0][r], s_m[1][r]), fmaxf(s_m[2][r], s_m[3][r]));
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) sum += s_l[w][r] * __builtin_amdgcn_exp2f((s_m[w][r] - mx) * a.c);
        const int d = half * kDh + d0;
        if (whole) {
          attn_store(a, sq, h, r, d, D, v, mx, sum);
        } else {
          *reinterpret_cast<floatx4 *>(part + (int64_t)r * D + d) = v;
          if (d == 0) {
            part[kRows * D + r] = mx;
            part[kRows * D + kRows + r] = sum;
          }
        }
      }
      __syncthreads();
    }
    if ((s_odd[0] | s_odd[1] | s_odd[2] | s_odd[3]) != 0)
      attn_put_odd<D, kFp8, 32>(a, sq, b, h, 0, rows, ga * kGran, tok_end, all_lo, all_hi, [&](int r, int d, float sum) {
        if (whole)
          attn_put_out<D>(a, sq, h, r, d, sum);
        else
          part[(int64_t)r * D + d] += sum;
      });
    __syncthreads();  // (s_odd is read)
    if constexpr (kWhole) return;
    first_piece = false;
    pos = stop;
  }
}

// ---- joining the pieces of a unit: their sums, maxima and sums of exponentials.
// kShare groups of threads take the same rows of different pieces and add up in LDS, so that
// 27 pieces are 7 rounds of loads.
template <int D, int kShare>
__host__ __device__ __forceinline__ constexpr int attn_join_rows() {  // rows of a block
  return 256 / (D / 4 * kShare);
}
template <int D, int kShare>
__host__ __device__ __forceinline__ constexpr int attn_join_lds() {
  return 256 * 16 + 2 * kShare * attn_join_rows<D, kShare>() * 4;
}
// Row rl of the block, row r of the unit's pieces (kPiece of them in each; `piece(i)` of n), which
// is row r_out of the sequence.
template <int D, int kShare, int kPiece, class Piece>
__device__ __forceinline__ void attn_join(const AttnArgs &a, char *lds, const AttnSeq &sq, int h, int r, int r_out, bool live, int n,
                                          Piece piece) {
  constexpr int kT = D / 4, kR = attn_join_rows<D, kShare>();
  const int tid = threadIdx.x, share = tid / (kT * kR), rl = tid / kT % kR, d0 = 4 * (tid % kT);
  float m = -__builtin_inff(), l = 0.0f;
  floatx4 v = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int i = share; i < n; i += kShare) {
    const float *part = piece(i);
    const floatx4 x = *reinterpret_cast<const floatx4 *>(part + (int64_t)r * D + d0);
    const float pm = part[kPiece * D + r], psum = part[kPiece * D + kPiece + r];
    const float mn = fmaxf(m, pm), f = __builtin_amdgcn_exp2f((m - mn) * a.c), fp = __builtin_amdgcn_exp2f((pm - mn) * a.c);
    v = v * f + x * fp;
    l = l * f + psum * fp;
    m = mn;
  }
  if constexpr (kShare > 1) {
    floatx4(&red)[kShare][kR][kT] = *reinterpret_cast<floatx4(*)[kShare][kR][kT]>(lds);
    float(&s_m)[kShare][kR] = *reinterpret_cast<float(*)[kShare][kR]>(lds + 256 * 16);
    float(&s_l)[kShare][kR] = *reinterpret_cast<float(*)[kShare][kR]>(lds + 256 * 16 + kShare * kR * 4);
    red[share][rl][tid % kT] = v;
    if (tid % kT == 0) {
      s_m[share][rl] = m;
      s_l[share][rl] = l;
    }
    __syncthreads();
    if (share != 0) return;
    m = s_m[0][rl];
#pragma unroll
    for (int i = 1; i < kShare; ++i) m = fmaxf(m, s_m[i][rl]);
    l = 0.0f;
    v = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < kShare; ++i) {
      const float f = __builtin_amdgcn_exp2f((s_m[i][rl] - m) * a.c);
      v += red[i][rl][tid % kT] * f;
      l += s_l[i][rl] * f;
    }
  }
  if (live) attn_store(a, sq, h, r_out, d0, D, v, m, l);
}

// Blocks and program of the join of attn_few's split units: the first piece lies at slot u[0],
// the others at the first slots of the blocks behind it up to u[1].
template <int D, int NB, int kShare = 4>
static int64_t attn_join_blocks(const AttnArgs &a) {
  return (int64_t)a.B * a.Hkv * ceil_div(std::min(16 * NB, a.max_q * a.G), attn_join_rows<D, kShare>());
}
template <int D, int NB, int kShare = 4>
__device__ __forceinline__ void attn_join_few(const AttnArgs &a, char *lds, int block) {
  constexpr int kRows = 16 * NB, kR = attn_join_rows<D, kShare>();
  const int unit = block % (a.B * a.Hkv), row0 = block / (a.B * a.Hkv) * kR, b = unit / a.Hkv, h = unit - b * a.Hkv;
  // (read beside the lengths; of a unit without rows in this kernel nobody wrote them, or uses them)
  const int s0 = attn_uni(a.units[2 * (int64_t)unit]), p1 = attn_uni(a.units[2 * (int64_t)unit + 1]);
  const AttnSeq sq = attn_seq(a, b);
  const int rows = sq.nq * a.G;
  if (rows <= row0 || rows > kRows) return;
  const int p0 = s0 >> 1, n = p1 - p0 + 1;
  if (n == 1) return;  // finished by its block
  const int r = row0 + (int)threadIdx.x / (D / 4) % kR, rr = min(r, rows - 1);
  attn_join<D, kShare, kRows>(a, lds, sq, h, rr, r, r < rows, n,
                              [&](int i) { return a.part + (int64_t)(i == 0 ? s0 : 2 * (p0 + i)) * part_floats<D, NB>(); });
}

}  // namespace lcvq
