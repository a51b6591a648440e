// Layer output from 4-bit weights with a scale, and a zero point, per row and group of
// columns, for few tokens:
//
//   Y[t, r] = sum_k s[k, r] ( sum_{c in group k} code[r, c] X[t, c]  -  z[k, r] sum_{c in group k} X[t, c] )
//
// on v_mfma_f32_16x16x32_bf16 with 16 weight rows on M and up to 16 tokens on N.  A code c
// becomes the bf16 value 16 + c by one shift and one and-or (the four bits stand at the top
// of the mantissa of [16, 32)), exactly; the 16 joins the zero point, and the group's sum of
// X comes from one more product with ones.  Products of bf16 are exact in fp32, groups are
// summed in fp32, and each group's sum is scaled once.  (16 rather than 128 + c, which
// needs no shift for the first of four: the sums that cancel are eight times smaller.)
//
// The word of eight columns gives its codes in pairs (i, i + 4), i = 0..3, so X is taken
// in that order (four byte permutes per eight columns and lane, shared by the row blocks).
//
// Block: 16 MR weight rows; its waves split K in steps of 128 columns (w, w + kW, ..) and add
// their tiles in LDS at the end, in wave order.  Few rows over a long K are split over
// blocks as well (k_int4_sum adds those).  Each wave has two stages: the loads of the next
// step are in flight while the current one is multiplied.
//
// Scales and zero points come in either order (strides): by row, as quantisers make them, a
// step takes 2 kU bytes of a line of each row, which costs the first-level cache more lookups than
// the codes do; by group its rows lie side by side.  By row / by group, a graph of calls:
// 28672 x 8192 with zero points at one token 34.3 / 30.4 us, in groups of 32 41.0 / 37.8; 8192 x
// 28672 in groups of 64 at 16 tokens 39.8 / 36.4; up to 11008 columns and rows no difference.
//
// Bound: HBM, the codes once (0.5 byte per weight, and 2 or 4 bytes per group); at 16 tokens
// also X from the L2, as many bytes as the codes of 64 rows.  28672 x 8192 with zero points by row, one
// token: 35 us, 3.6 TB/s; 8192 x 28672 in groups of 64 by row, 16 tokens: 39 us, 3.2 TB/s, and 5 for
// the spans; 4096 x 4096, one token: 5 us, of which the codes at a copy's rate are 1.7 and the
// launch the most.
#include <algorithm>

#include "lcvq_mfma.hpp"
#include "lcvq_prep.hpp"
#include "lcvq_serve.hpp"

namespace lcvq {

template <int N>
__device__ __forceinline__ void int4_wait_vm() {
  LCVQ_WAIT_VM(N);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Eight codes -> bf16 16 + code, in the order 0 4 1 5 2 6 3 7.
__device__ __forceinline__ bf16x8 int4_operand(uint32_t w) {
  const u32x4 v = {((w << 3) & 0x00780078u) | 0x41804180u, ((w >> 1) & 0x00780078u) | 0x41804180u,
                   ((w >> 5) & 0x00780078u) | 0x41804180u, ((w >> 9) & 0x00780078u) | 0x41804180u};
  return __builtin_bit_cast(bf16x8, v);
}
// Eight columns of X (four dwords) in that order.
__device__ __forceinline__ bf16x8 int4_x(const u32x4 &x) {
  const u32x4 v = {__builtin_amdgcn_perm(x[2], x[0], 0x05040100u), __builtin_amdgcn_perm(x[2], x[0], 0x07060302u),
                   __builtin_amdgcn_perm(x[3], x[1], 0x05040100u), __builtin_amdgcn_perm(x[3], x[1], 0x07060302u)};
  return __builtin_bit_cast(bf16x8, v);
}

// Which of a step's sixteen words of eight columns lane group q takes for its product i:
// the 32 columns of a product lie in one group of kG columns.
template <int kG>
__device__ __forceinline__ int int4_word(int i, int q) {
  return kG == 128 ? 4 * q + i : kG == 64 ? 8 * (i >> 1) + 2 * q + (i & 1) : 4 * i + q;
}

// Scale (and zero point) of row r and group k: element r s_row + k s_group.  kTok: tokens staged, 4 or 16.  kG: columns that a product's sum may span (32, 64, 128; larger groups are multiples of
// 128).  kSplit: block (x, y) takes the steps [y span, (y + 1) span) and stores its sums in
// `part` (span y, token, row).
template <int MR, int kW, int kTok, int kG, bool kZero, bool kSplit>
__global__ __launch_bounds__(64 * kW, MR > 4 ? 1 : 2) void k_int4(const uint8_t *__restrict__ packed, const uint16_t *__restrict__ scales,
                                                     const uint16_t *__restrict__ zeros, int64_t m, int64_t n, int64_t groups, uint32_t s_row,
                                                     uint32_t s_group, uint64_t per_step, int KT,
                                                     const uint16_t *__restrict__ X, int Nc, void *__restrict__ Y, int y_bf16,
                                                     int span, float *__restrict__ part) {
  constexpr int kU = 128 / kG;                                   // groups of a step
  constexpr int kS = (MR * kU + 3) / 4, kP = kZero ? 2 : 1;      // loads of a step's scales, and of its zero points
  constexpr int kX = MR * 1024 + kP * kS * 256, kStage = kX + kTok * 256;  // X behind codes and scales
  constexpr int kLoads = kTok / 4 + kP * kS + MR;
  __shared__ __attribute__((aligned(1024))) char lds[2 * kW * kStage];
  const int tid = threadIdx.x, lane = tid & 63, q = lane >> 4, c16 = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // Blocks i, i + 8, .. run on one XCD: they take neighbouring rows, whose scales share lines.
  const uint32_t xcd = blockIdx.x & 7, per = gridDim.x >> 3, more = gridDim.x & 7;
  const int64_t r0 = (int64_t)(xcd * per + min(xcd, more) + (blockIdx.x >> 3)) * 16 * MR, ldb = n / 2;
  const int j0 = kSplit ? (int)blockIdx.y * span : 0;
  if constexpr (kSplit) KT = min(KT, j0 + span);
  const __amdgpu_buffer_rsrc_t rsA = make_rsrc(packed + r0 * ldb, (m - r0 < 16 * MR ? m - r0 : 16 * MR) * ldb);
  const __amdgpu_buffer_rsrc_t rsX = make_rsrc(X, (int64_t)Nc * n * 2);
  const int lrow = lane >> 2, lpiece = (lane & 3) ^ ((lrow >> 1) & 3);
  const uint32_t aoff = (uint32_t)(lrow * ldb + 16 * lpiece), astep = (uint32_t)(16 * ldb);
  const int64_t s0 = r0 * s_row, s_bytes = (groups * m - s0) * 2;
  const __amdgpu_buffer_rsrc_t rsS = make_rsrc(scales + s0, s_bytes);
  const __amdgpu_buffer_rsrc_t rsZ = make_rsrc(kZero ? zeros + s0 : scales, kZero ? s_bytes : 0);

  const uint32_t soff = 2u * ((uint32_t)(lane % kU) * s_group + (uint32_t)(lane / kU) * s_row);

  // A step past the end loads zeros; no load is behind a branch, so that their number is known.
  auto load = [&](int u, int j) __attribute__((always_inline)) {
    LCVQ_WAIT_LGKM0();  // what was read from the stage has arrived
    __builtin_amdgcn_sched_barrier(0);
    const bool on = j < KT;
    uint32_t base = (uint32_t)((wave * 2 + u) * kStage);
    asm volatile("" : "+s"(base));
    // X: a token's 128 columns are 16 chunks, chunk c of token t at place c ^ t
#pragma unroll
    for (int i = 0; i < kTok / 4; ++i) {
      const int t = 4 * i + (lane >> 4), c = j * 128 + 8 * ((lane & 15) ^ t);
      buffer_to_lds16(rsX, (lds_void *)(lds + base + kX + i * 1024),
                      on & (t < Nc) & (c < (int)n) ? (uint32_t)(t * (int)n + c) * 2u : kOffNone);
    }
    // The block's scales, one to a dword of LDS, a row's groups side by side: lanes of one row read
    // one line where the scales are in rows, lanes of one group where they are in groups.  (Of
    // rows past m what lies there, or zeros: not stored.  A group of 128 / kU columns, or of
    // several steps: j / (group / 128) as a product.)
    const uint32_t g0 = kU > 1 ? (uint32_t)(j * kU) : (uint32_t)(((uint64_t)(uint32_t)j * per_step) >> 32);
    const uint32_t at = on & (j * 128 + (lane % kU) * kG < (int)n) ? 2u * (g0 * s_group) + soff : kOffNone;
#pragma unroll
    for (int i = 0; i < kS; ++i) {
      const uint32_t off = lane < 16 * MR * kU - 64 * i ? at + (uint32_t)(128 / kU * i) * s_row : kOffNone;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsS, (lds_void *)(lds + base + MR * 1024 + i * 256), 2, (int)off, 0, 0, 0);
      if constexpr (kZero)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsZ, (lds_void *)(lds + base + MR * 1024 + (kS + i) * 256), 2, (int)off, 0, 0, 0);
    }
    // a row's words past its end are its neighbour's, or zeros: they meet zeros of X
#pragma unroll
    for (int rb = 0; rb < MR; ++rb)
      buffer_to_lds16(rsA, (lds_void *)(lds + base + rb * 1024), on ? aoff + rb * astep + 64u * (uint32_t)j : kOffNone);
    __builtin_amdgcn_sched_barrier(0);
  };
  floatx4 y[MR];
#pragma unroll
  for (int rb = 0; rb < MR; ++rb) y[rb] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  bf16x8 ones;
#pragma unroll
  for (int i = 0; i < 8; ++i) ones[i] = (__bf16)1.0f;
  auto step = [&](int u) __attribute__((always_inline)) {
    uint32_t base = (uint32_t)((wave * 2 + u) * kStage);
    asm volatile("" : "+s"(base));  // the addresses are made here: held over the loop, they crowd out the rest
    const floatx4 none = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    const int tok = kTok == 16 ? c16 : c16 & 3;  // (what a lane past the last token adds up is not stored)
    const char *xrow = lds + base + kX + tok * 256;
    bf16x8 xf[4];
    float off[kU];  // (16 + zero point, or 24) times the group's sum of X
#pragma unroll
    for (int k = 0; k < kU; ++k) {
      floatx4 xs = none;
#pragma unroll
      for (int i = k * (4 / kU); i < (k + 1) * (4 / kU); ++i) {
        xf[i] = int4_x(*reinterpret_cast<const u32x4 *>(xrow + ((int4_word<kG>(i, q) ^ tok) << 4)));
        xs = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, xf[i], xs, 0, 0, 0);
      }
      off[k] = kZero ? xs[0] : 24.0f * xs[0];
    }
    const char *st = lds + base + c16 * 64;
    const int swz = (c16 >> 1) & 3;
#pragma unroll
    for (int rb = 0; rb < MR; ++rb) {
      uint32_t w[4];
      if constexpr (kG == 128) {
        const u32x4 v = *reinterpret_cast<const u32x4 *>(st + rb * 1024 + ((q ^ swz) << 4));
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = v[i];
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int wd = int4_word<kG>(i, q);
          w[i] = *reinterpret_cast<const uint32_t *>(st + rb * 1024 + (((wd >> 2) ^ swz) << 4) + 4 * (wd & 3));
        }
      }
      const u32x4 *vec = reinterpret_cast<const u32x4 *>(lds + base + MR * 1024 + (16 * rb + 4 * q) * kU * 4);
      u32x4 sv[kU], zv[kU];  // of the lane's four rows and their groups: row e, group k in dword e kU + k
#pragma unroll
      for (int k = 0; k < kU; ++k) {
        sv[k] = vec[k];
        zv[k] = kZero ? vec[k + kS * 16] : u32x4{0u, 0u, 0u, 0u};
      }
#pragma unroll
      for (int k = 0; k < kU; ++k) {
        floatx4 acc = none;
#pragma unroll
        for (int i = k * (4 / kU); i < (k + 1) * (4 / kU); ++i)
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(int4_operand(w[i]), xf[i], acc, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t se = sv[(e * kU + k) / 4][(e * kU + k) % 4], ze = zv[(e * kU + k) / 4][(e * kU + k) % 4];
          const float t = kZero ? fmaf(-16.0f - bf16_to_f32((uint16_t)ze), off[k], acc[e]) : acc[e] - off[k];
          y[rb][e] = fmaf(bf16_to_f32((uint16_t)se), t, y[rb][e]);
        }
      }
      // two row blocks in registers at a time, and their sums made here, not where they are needed
      asm volatile("" : "+v"(y[rb]));
      if (rb & 1) __builtin_amdgcn_sched_barrier(0);
    }
  };
  int j = j0 + wave;
  load(0, j);
  for (; j + kW < KT; j += 2 * kW) {
    load(1, j + kW);
    int4_wait_vm<kLoads>();
    step(0);
    load(0, j + 2 * kW);
    int4_wait_vm<kLoads>();
    step(1);
  }
  LCVQ_WAIT_ALL();
  __builtin_amdgcn_sched_barrier(0);
  if (j < KT) step(0);

  // ------------------------------------------------------------ the waves' sums
  __syncthreads();
  floatx4 *red = reinterpret_cast<floatx4 *>(lds);  // [wave][row block][lane]
#pragma unroll
  for (int rb = 0; rb < MR; ++rb) red[(wave * MR + rb) * 64 + lane] = y[rb];
  __syncthreads();
  for (int rb = wave; rb < MR; rb += kW) {
    floatx4 v = red[rb * 64 + lane];
#pragma unroll
    for (int w = 1; w < kW; ++w) v += red[(w * MR + rb) * 64 + lane];
    const int64_t row = r0 + 16 * rb + 4 * q;
    if (c16 >= Nc) continue;
    const int64_t o = (int64_t)c16 * m + row;
    if constexpr (kSplit) {
      float *dst = part + (int64_t)blockIdx.y * Nc * m + o;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (row + e < m) dst[e] = v[e];
    } else if ((m & 3) == 0) {  // four rows of a token are one aligned store
      if (row >= m) continue;
      if (y_bf16) {
        *reinterpret_cast<u32x2 *>(reinterpret_cast<uint16_t *>(Y) + o) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
      } else {
        *reinterpret_cast<floatx4 *>(reinterpret_cast<float *>(Y) + o) = v;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (row + e < m) {
          if (y_bf16) {
            reinterpret_cast<uint16_t *>(Y)[o + e] = (uint16_t)pack_bf16x2(v[e], 0.0f);
          } else {
            reinterpret_cast<float *>(Y)[o + e] = v[e];
          }
        }
    }
  }
}

// The spans' sums, in order; one output per thread.
__global__ __launch_bounds__(256) void k_int4_sum(const float *__restrict__ part, int spans, int64_t total, void *__restrict__ Y,
                                                  int y_bf16) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= total) return;
  float v = 0.0f;
#pragma unroll 4
  for (int s = 0; s < spans; ++s) v += part[s * total + i];
  if (y_bf16) {
    reinterpret_cast<uint16_t *>(Y)[i] = (uint16_t)pack_bf16x2(v, 0.0f);
  } else {
    reinterpret_cast<float *>(Y)[i] = v;
  }
}

// ---------------------------------------------------------------- launch ---
// Rows per block: 16 MR with the fewest rounds of blocks over the 256 compute units and
// those rounds full, MR at most 3 up to four tokens and 8 above, where a block's X counts
// (28672 x 8192 at 16 tokens, 7 row blocks and four waves 33 us a call, 2 and eight 41); but 2
// where four tokens or fewer meet more than 16384 rows (28672 x 8192 with zero points at one
// token: 3 row blocks 28.9 us a call, 2 27.6, 1 28.4.  Graphs of calls, 3 / 2 / 1 row blocks, by
// group: 32000 x 4096 in groups of 32 30.2 / 23.5 / 25.5, 20000 x 8192 in groups of 64 23.9 / 23.6 /
// 23.2, 17000 x 4096 12.8 / 13.1 / 12.7, 65536 x 2048 23.0 / 23.5 / 28.0, 128256 x 4096 55.8 / 58.9 /
// 65.4; by row 41.5 / 35.1 / 34.0 for the first and 30.1 / 23.9 / 24.7 for the second).
//
// K is split over blocks, whose sums a second launch adds,
//  - where there are fewer than 128 blocks of 16 rows, to fill the chip;
//  - above four tokens where up to 8192 rows meet 128 steps or more: 64 rows a block read a
//    quarter of the X that 16 do (8192 x 28672 at 16 tokens: 32 rows 36.1 us a call, 64 rows
//    and two spans 33.8.  Graphs of calls, whole K in the best of 16, 32 and 64 rows / 64 rows and
//    spans, by group: 5120 x 27648 26.0 / 21.3, 4096 x 16384 15.1 / 14.3, 2048 x 16384 14.8 / 10.7, but
//    6000 x 19968 in groups of 32 30.8 / 31.6 and, at the rule's end, 8192 x 16384 22.1 / 23.6).
Int4Plan int4_plan(int64_t m, int64_t n, bool many, int most_mr) {
  Int4Plan p{};
  const int64_t rb = ceil_div(m, 16), rounds = ceil_div(rb, 256 * most_mr);
  p.KT = (int)ceil_div(n, 128);
  p.mr = rb > 0 ? (int)ceil_div(rb, 256 * rounds) : 1;
  if (!many && rb > 1024) p.mr = 2;
  int64_t spans = 1;
  if (rb < 128 && p.KT >= 32) {
    p.mr = 1;
    spans = std::min<int64_t>(256 / std::max<int64_t>(rb, 1), p.KT / 8);
  } else if (many && rb <= 512 && p.KT >= 128) {
    p.mr = 4;
    spans = 1024 / rb;
  }
  p.span = (int)ceil_div(p.KT, std::max<int64_t>(spans, 1));
  p.spans = p.span > 0 ? (int)ceil_div(p.KT, p.span) : 1;
  return p;
}
int64_t int4_bytes(int64_t N, int64_t m, int64_t n) {
  int64_t bytes = 0;
  for (int many = 0; many <= (N > 4 ? 1 : 0); ++many) {
    const Int4Plan p = int4_plan(m, n, many, many ? 8 : 3);
    if (p.spans > 1) bytes = std::max<int64_t>(bytes, p.spans * std::min<int64_t>(N, many ? 16 : 4) * m * 4);
  }
  return bytes;
}

template <int kTok, int kG, bool kZero>
static hipError_t launch(const Int4Args &a, const uint16_t *X, int Nc, char *Y, hipStream_t st) {
  constexpr bool kMany = kTok == 16;
  constexpr int kMost = kMany ? 8 : 3;
  const Int4Plan p = int4_plan(a.m, a.n, kMany, kMost);
  const int64_t groups = a.n / a.group;
  // ceil(2^32 / (group / 128)): exact for fewer than 2^14 steps
  const uint64_t per_step = ((1ull << 32) + std::max(a.group / 128, 1) - 1) / std::max(a.group / 128, 1);
  using K = decltype(&k_int4<1, 8, kTok, kG, kZero, false>);
  K f;
  int waves = 8;
  if (p.spans > 1) {
    f = k_int4<1, 8, kTok, kG, kZero, true>;
    if constexpr (kMany)
      if (p.mr == 4) f = k_int4<4, 8, kTok, kG, kZero, true>;
  } else if constexpr (kMany) {  // (eight waves' X and more than three row blocks do not fit in the LDS)
    static constexpr K k[8] = {k_int4<1, 8, kTok, kG, kZero, false>, k_int4<2, 8, kTok, kG, kZero, false>,
                               k_int4<3, 8, kTok, kG, kZero, false>, k_int4<4, 4, kTok, kG, kZero, false>,
                               k_int4<5, 4, kTok, kG, kZero, false>, k_int4<6, 4, kTok, kG, kZero, false>,
                               k_int4<7, 4, kTok, kG, kZero, false>, k_int4<8, 4, kTok, kG, kZero, false>};
    f = k[p.mr - 1];
    waves = p.mr > 3 ? 4 : 8;
  } else {
    static constexpr K k[3] = {k_int4<1, 8, kTok, kG, kZero, false>, k_int4<2, 8, kTok, kG, kZero, false>,
                               k_int4<3, 8, kTok, kG, kZero, false>};
    f = k[p.mr - 1];
  }
  f<<<dim3((unsigned)ceil_div(a.m, 16 * p.mr), (unsigned)p.spans), 64 * waves, 0, st>>>(
      a.packed, a.scales, a.zeros, a.m, a.n, groups, (uint32_t)(a.by_row ? groups : 1), (uint32_t)(a.by_row ? 1 : a.m), per_step, p.KT, X, Nc, Y, a.y_bf16 ? 1 : 0, p.span, a.part);
  if (p.spans > 1)
    k_int4_sum<<<(unsigned)ceil_div(a.m * Nc, 256), 256, 0, st>>>(a.part, p.spans, a.m * Nc, Y, a.y_bf16 ? 1 : 0);
  return hipGetLastError();
}

template <int kTok>
static hipError_t launch_group(const Int4Args &a, const uint16_t *X, int Nc, char *Y, hipStream_t st) {
  const bool z = a.zeros != nullptr;
  auto go = a.group == 32 ? (z ? launch<kTok, 32, true> : launch<kTok, 32, false>)
            : a.group == 64 ? (z ? launch<kTok, 64, true> : launch<kTok, 64, false>)
                            : (z ? launch<kTok, 128, true> : launch<kTok, 128, false>);
  return go(a, X, Nc, Y, st);
}

hipError_t launch_int4(const Int4Args &a, const uint16_t *X, int Nc, char *Y, hipStream_t st) {
  return Nc <= 4 ? launch_group<4>(a, X, Nc, Y, st) : launch_group<16>(a, X, Nc, Y, st);
}

}  // namespace lcvq
