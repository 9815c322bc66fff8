// mx4_gemm.hpp -- the large products C = sum over pairs (i, j) of A_i B_j^T behind the MXFP4 calls,
// one kernel for three kinds of operands, all rows of the reduction:
//   GEMM_FP4   both sides MXFP4 codes with their scales (32 x 32 x 64 scaled products);
//   GEMM_BF16, GEMM_F16   both sides 16-bit numbers (32 x 32 x 16 products);
//   GEMM_MIX   A bfloat16, B MXFP4 codes, turned into bfloat16 in registers;
//   GEMM_MIXH  A binary16, B MXFP4 codes, turned into binary16 in registers: a row of B is taken
//              relative to its largest scale, the power of two goes to the result's column.  36
//              binades below that scale are exact in binary16; a tile with a number further down
//              (which the rows' pass over the scales finds) splits A into two bfloat16 pieces
//              instead, in registers, at half the rate.
// The operands of one instruction are 16 bytes a lane in every kind, and it takes as long (32
// cycles of a SIMD at the full rate), so the kinds share tiles, staging and schedule.
//
// A workgroup computes BM x BN outputs, WM x WN wavefronts TM x TN tiles of 32 x 32 each.  A step
// is 128 bytes of every row of A (256 codes or 64 16-bit numbers) and as much of the reduction of
// B.  Steps go into a ring of S LDS buffers by direct loads (no registers in between), S - 1 steps
// ahead of the products; one barrier a step.  Chunk c (16 bytes) of row r lies at position
// c ^ (r / 2 mod 8) of its row: 16 neighbouring rows' chunks c lie in 16 different groups of four of
// the 64 banks.
//
// What bounds it.  Large tiles: the schedule.  The matrix instructions are busy 56% (FP4) and 60% (MIX)
// of the cycles; two wavefronts a SIMD, two buffers and one barrier a step that all eight wavefronts
// meet leave 29% of the wavefronts' cycles waiting at it and for loads.  LDS is busy a quarter of the
// time (a wavefront of 128 x 64 outputs reads 6 KiB of it for 8 instructions).  The power limit holds
// the clock at 1.7 to 2.0 GHz; under it a loop of the scaled instruction alone reaches 6.55 PFLOP/s.
// 8192^3 FP4 262 to 272 us, 4.1 PFLOP/s; 4096^3 MIX 102 us, 1.34 PFLOP/s, where a library product of
// plain bfloat16 takes 98; 4096^3 MIXH 107 us, 5 of them the pass over the scales.  Grids of about 256
// small tiles: a step takes 0.36 to 0.6 us whatever it multiplies, its loads' and reads' latency
// (4096 x 4096 by 256 rows: MIX 22 us, FP4 12, where bytes and operations need 6 and 2).
#pragma once

#include "mcf_internal.hpp"
#include "mx4.hpp"

namespace mcf {

enum GemmKind { GEMM_FP4 = 0, GEMM_BF16 = 1, GEMM_F16 = 2, GEMM_MIX = 3, GEMM_MIXH = 4 };

struct GemmArgs {
  const char *a, *b;              // pieces' planes of rows
  int64_t a_plane, b_plane;       // bytes from plane to plane
  int64_t a_ld, b_ld;             // bytes of a row
  const uint32_t *as, *bs;        // scales [plane][groups][rows]
  int64_t groups;
  const uint8_t *top, *wide;      // MIXH: the largest scale of each row of B, and for every 64 rows
                                  // whether a number lies too far below it
  void *c;                        // [M][N]
  const void *bias;               // [N] or null
  float *partial;                 // [slices][M][N], with more than one slice
  int64_t M, N;
  int steps, total, slices;       // steps of a pair, of all pairs; slices of the reduction
  int pairs;                      // at most 16
  uint64_t pa, pb;                // the planes of pair p, 4 bits each
};

// 16 (4) bytes a lane from base + off straight into LDS at `to` + 16 (4) lane.  The loads are
// asm so that the compiler does not wait for them in front of every LDS read; gemm_wait does.
// m0 holds the LDS address, and a load that reads it follows its write by a wait state.  The compiler
// sets m0 where it needs it and allots it to nothing, which it says of a clobber.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ inline void lds_load16(uint32_t to, uint32_t off, const void *base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(__builtin_amdgcn_readfirstlane(to)), "v"(off), "s"(base) : "m0", "memory");
}
__device__ inline void lds_load4(uint32_t to, uint32_t off, const void *base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(__builtin_amdgcn_readfirstlane(to)), "v"(off), "s"(base) : "m0", "memory");
}
#pragma clang diagnostic pop
__device__ inline const char *uniform(const void *p) {
  const uint64_t u = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)u), hi = __builtin_amdgcn_readfirstlane((uint32_t)(u >> 32));
  return (const char *)((uint64_t)hi << 32 | lo);
}
// All but the youngest LEFT loads of this wavefront have landed and its LDS reads are done; then
// the workgroup's barrier.
template <int LEFT>
__device__ inline void gemm_wait() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}

__device__ inline uint32_t lds_address(const void *p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void *)p;
}

// Workgroup id -> tile.  Ids go to the 8 XCDs in turn; each XCD takes a contiguous run of tiles, and
// a run walks 8 rows of tiles column by column, so that the tiles an XCD works on share operands
// in its L2.
__device__ inline void gemm_tile(uint32_t id, uint32_t gm, uint32_t gn, uint32_t *tm, uint32_t *tn) {
  const uint32_t n = gm * gn, q = n / 8, rest = n % 8, x = id % 8, l = id / 8;
  const uint32_t t = x < rest ? x * (q + 1) + l : rest * (q + 1) + (x - rest) * q + l;
  const uint32_t band = t / (8 * gn), first = band * 8, rows = gm - first < 8 ? gm - first : 8, in = t - first * gn;
  *tm = first + in % rows;
  *tn = in / rows;
}

template <bool B>
struct Flag {
  static constexpr bool value = B;
};

// A wavefront's tiles to `to`, its first element in the M x N result; `rows` and `cols` are what is
// left of the result there.  Lane (r, g) holds column r of a tile, rows 8 (e / 4) + 4 g + e mod 4.
// A row's start is scalar arithmetic, the lane's part a 32-bit offset.  SHIFT: the columns' powers
// of two.
template <typename T, bool SHIFT, int TM, int TN>
__device__ inline void gemm_store(const f32x16 (&acc)[TM][TN], T *to, const T *bias, const int (&shift)[TN], int64_t ld,
                                  int rows, int cols) {
  const int lane = threadIdx.x & 63, r = lane & 31, g = lane >> 5;
  const uint32_t off = (uint32_t)(4 * g * ld + r);
  const auto store = [&](auto whole) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int m = i * 32 + (e >> 2) * 8 + (e & 3);
        T *row = to + m * ld;
#pragma unroll
        for (int j = 0; j < TN; ++j)
          if (decltype(whole)::value || (m + 4 * g < rows && j * 32 + r < cols)) {
            float v = acc[i][j][e];
            if constexpr (SHIFT) v = ldexpf(v, shift[j]);
            row[off + j * 32] = (T)(bias ? v + (float)bias[j * 32 + r] : v);
          }
      }
  };
  // apart, so that a whole tile's stores carry no tests (15 us of the 8192 x 8192 result)
  if (rows >= 32 * TM && cols >= 32 * TN)
    store(Flag<true>());
  else
    store(Flag<false>());
}

constexpr bool gemm_mixed(GemmKind k) { return k == GEMM_MIX || k == GEMM_MIXH; }

template <GemmKind KIND, int TM, int TN>
struct Operands {
  u32x4 a[TM], b[gemm_mixed(KIND) ? 1 : TN];
};
template <GemmKind KIND, int TM, int TN>
struct Scales {
  uint32_t a[KIND == GEMM_FP4 ? 2 : 1][TM], b[KIND == GEMM_FP4 ? 2 : 1][TN];
  u32x4 codes[gemm_mixed(KIND) ? TN : 1];
  float scale[TN];
};
__device__ inline i32x8 widen(u32x4 v) {
  const i32x4 w = __builtin_bit_cast(i32x4, v);
  return __builtin_shufflevector(w, w, 0, 1, 2, 3, -1, -1, -1, -1);
}

// LDS of a workgroup: S stages.
template <GemmKind KIND, int BM, int BN>
struct alignas(128) GemmStage {
  char a[BM * 128];
  char b[BN * (gemm_mixed(KIND) ? 32 : 128)];
  uint32_t as[KIND == GEMM_FP4 ? 2 * BM : 1], bs[KIND == GEMM_FP4 ? 2 * BN : (gemm_mixed(KIND) ? BN : 1)];
};

// One workgroup: tile `tile` of slice `slice`.
template <GemmKind KIND, typename T, int WM, int WN, int TM, int TN, int S>
__device__ __forceinline__ void gemm_body(const GemmArgs &a, char *lds, uint32_t tile, int slice) {
  constexpr int BM = WM * TM * 32, BN = WN * TN * 32, NW = WM * WN;
  constexpr bool MIX = gemm_mixed(KIND);
  constexpr int BB = MIX ? 32 : 128;  // bytes of a row of B in a step
  constexpr bool SCALED_A = KIND == GEMM_FP4, SCALED_B = KIND == GEMM_FP4 || MIX;
  constexpr int SG = KIND == GEMM_FP4 ? 2 : 1;     // words of scales of a row in a step
  using Stage = GemmStage<KIND, BM, BN>;
  Stage *const st = reinterpret_cast<Stage *>(lds);

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t tm, tn;
  gemm_tile(tile, (uint32_t)((a.M + BM - 1) / BM), (uint32_t)((a.N + BN - 1) / BN), &tm, &tn);
  const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
  const int s_begin = (int)((int64_t)a.total * slice / a.slices), s_end = (int)((int64_t)a.total * (slice + 1) / a.slices);

  // what this lane loads in a step: rows past the end repeat the last one
  constexpr int NB = BN * BB / 1024, LA = BM / 8 / NW, LB = (NB + NW - 1) / NW;
  constexpr int LOADS_A = LA + (SCALED_A ? (SG * BM / 64 + NW - 1) / NW : 0);
  constexpr int LOADS = LOADS_A + LB + (SCALED_B ? (SG * BN / 64 + NW - 1) / NW : 0);
  static_assert(LOADS * (S - 1) < 64, "vmcnt counts to 63");
  static_assert(LA % 2 == 0 && (BB != 128 || LB % 2 == 0), "rows of a load start at a multiple of 16 or 8 past one");
  static_assert(BM % (8 * NW) == 0 && (BB != 128 || NB % NW == 0), "whole loads a wavefront");
  uint32_t offa[LA], offb[LB];
  const int64_t la = a.M - m0 < BM ? a.M - m0 : BM, lb = a.N - n0 < BN ? a.N - n0 : BN;  // rows left
#pragma unroll
  for (int i = 0; i < LA; ++i) {
    const int r = (wave * LA + i) * 8 + (lane >> 3), c = (lane & 7) ^ ((r >> 1) & 7);
    offa[i] = (uint32_t)((r < la ? r : la - 1) * a.a_ld) + c * 16;
  }
#pragma unroll
  for (int i = 0; i < LB; ++i) {
    int r, c;
    if constexpr (BB == 128) {
      r = (wave * LB + i) * 8 + (lane >> 3), c = (lane & 7) ^ ((r >> 1) & 7);
    } else {
      r = (wave * LB + i) % NB * 32 + (lane >> 1), c = lane & 1;  // past the last one: again
    }
    offb[i] = (uint32_t)((r < lb ? r : lb - 1) * a.b_ld) + c * 16;
  }

  // 64 where this lane's even-numbered (odd-numbered) loads are of a row's upper half
  const uint32_t upper[2] = {((uint32_t)lane & 4) * 16, (~(uint32_t)lane & 4) * 16};
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_address(&st[0]));
  // A step is step k of a pair.
  struct At {
    int pair, k;
  };
  const auto next = [&](At s, bool go) {
    const bool wrap = s.k + 1 == a.steps;
    return At{go && wrap ? s.pair + 1 : s.pair, go ? (wrap ? 0 : s.k + 1) : s.k};
  };
  // The loads of a step of A, and of B, each with its scales.
  const auto load_a = [&](int buf, At s) {
    const int k = s.k, ia = (int)(a.pa >> (4 * s.pair)) & 15;
    const uint32_t to = lds0 + buf * (uint32_t)sizeof(Stage);
    const char *pa = uniform(a.a + ia * a.a_plane + m0 * a.a_ld + (int64_t)k * 128);
    // FP4, an odd group count: the last step's upper half re-reads the lower one and counts for
    // nothing (its scales are taken as 0 on both sides, and 2^-254 times 36 is 0)
    const bool whole = KIND != GEMM_FP4 || 2 * k + 1 < a.groups;
    const uint32_t back[2] = {whole ? 0 : upper[0], whole ? 0 : upper[1]};
#pragma unroll
    for (int i = 0; i < LA; ++i)
      lds_load16(to + offsetof(Stage, a) + (wave * LA + i) * 1024, KIND == GEMM_FP4 ? offa[i] - back[i & 1] : offa[i], pa);
    // Words of scales, 64 a load; a wavefront past the last one repeats a load, with the same data.
    if constexpr (SCALED_A) {
      constexpr int N = SG * BM / 64;
#pragma unroll
      for (int i = 0; i < (N + NW - 1) / NW; ++i) {
        const int e = (wave + i * NW) % N * 64, g = e / BM, r = e % BM + lane;
        const int64_t grp = 2 * k + g < a.groups ? 2 * k + g : a.groups - 1;
        lds_load4(to + offsetof(Stage, as) + e * 4, (uint32_t)(r < la ? r : la - 1) * 4,
                  uniform(a.as + (ia * a.groups + grp) * a.M + m0));
      }
    }
  };
  const auto load_b = [&](int buf, At s) {
    const int k = s.k, ib = (int)(a.pb >> (4 * s.pair)) & 15;
    const uint32_t to = lds0 + buf * (uint32_t)sizeof(Stage);
    const char *pb = uniform(a.b + ib * a.b_plane + n0 * a.b_ld + (int64_t)k * BB);
    const bool whole = KIND != GEMM_FP4 || 2 * k + 1 < a.groups;
    const uint32_t back[2] = {whole ? 0 : upper[0], whole ? 0 : upper[1]};
#pragma unroll
    for (int i = 0; i < LB; ++i)
      lds_load16(to + offsetof(Stage, b) + (wave * LB + i) % NB * 1024, KIND == GEMM_FP4 ? offb[i] - back[i & 1] : offb[i], pb);
    if constexpr (SCALED_B) {
      constexpr int N = SG * BN / 64;
#pragma unroll
      for (int i = 0; i < (N + NW - 1) / NW; ++i) {
        const int e = (wave + i * NW) % N * 64, g = e / BN, r = e % BN + lane;
        int64_t grp = KIND == GEMM_FP4 ? 2 * k + g : k >> 1;
        if (grp >= a.groups) grp = a.groups - 1;
        lds_load4(to + offsetof(Stage, bs) + e * 4, (uint32_t)(r < lb ? r : lb - 1) * 4,
                  uniform(a.bs + (ib * a.groups + grp) * a.N + n0));
      }
    }
  };

  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;

  const int r = lane & 31, g = lane >> 5, wm = (wave / WN) * TM * 32, wn = (wave % WN) * TN * 32;
  // The operands of quarter q of a step, of which a lane holds chunk 4 g + q (16-bit kinds) or
  // 2 q + g (FP4) of its rows, and what multiplies them.
  Operands<KIND, TM, TN> op[2];
  Scales<KIND, TM, TN> sc, sc_next;
  // MIXH: a column's power of two, and whether this tile needs the wide form
  int shift_of[TN];
  bool any_wide = false;
#pragma unroll
  for (int j = 0; j < TN; ++j) {
    shift_of[j] = 0;
    if constexpr (KIND == GEMM_MIXH) {
      const int64_t n = n0 + wn + j * 32 + r;
      shift_of[j] = (int)a.top[n < a.N ? n : a.N - 1] - 140;
    }
  }
  if constexpr (KIND == GEMM_MIXH) {
    for (int64_t n = n0; n < n0 + lb; n += 64) any_wide = any_wide || a.wide[n / 64] != 0;
  }
  const auto read = [&](int buf, int q, Operands<KIND, TM, TN> &o) {
    const Stage &B = st[buf];
    const int c = ((KIND == GEMM_FP4 ? 2 * q + g : 4 * g + q) ^ ((r >> 1) & 7)) * 16;
#pragma unroll
    for (int i = 0; i < TM; ++i) o.a[i] = *reinterpret_cast<const u32x4 *>(B.a + (wm + r + i * 32) * 128 + c);
    if constexpr (!MIX) {
#pragma unroll
      for (int j = 0; j < TN; ++j) o.b[j] = *reinterpret_cast<const u32x4 *>(B.b + (wn + r + j * 32) * 128 + c);
    }
  };
  const auto read_scales = [&](int buf, int k, Scales<KIND, TM, TN> &sc, auto wide) {
    const Stage &B = st[buf];
    if constexpr (KIND == GEMM_FP4) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t keep = h == 0 || 2 * k + 1 < a.groups ? 0xffffffffu : 0u;
#pragma unroll
        for (int i = 0; i < TM; ++i) sc.a[h][i] = (B.as[h * BM + wm + i * 32 + r] & keep) >> (8 * g);
#pragma unroll
        for (int j = 0; j < TN; ++j) sc.b[h][j] = (B.bs[h * BN + wn + j * 32 + r] & keep) >> (8 * g);
      }
    }
    if constexpr (MIX) {
      // lane group g takes block g of the step's two: the reduction runs over them side by side
      const int shift = 8 * (2 * (k & 1) + g);
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        sc.codes[j] = *reinterpret_cast<const u32x4 *>(B.b + (wn + r + j * 32) * BB + g * 16);
        uint32_t byte = (B.bs[wn + j * 32 + r] >> shift) & 255u;
        if constexpr (KIND == GEMM_MIXH && !decltype(wide)::value) {
          // relative to the row's largest scale, which becomes 2^13: 6 2^13 is below binary16's end
          const int rel = (int)byte - shift_of[j];
          byte = byte == 255 ? 255 : (rel > 0 ? rel : 0);
        }
        sc.scale[j] = mx_scale(byte);
      }
    }
  };
  const auto multiply = [&](int q, const Operands<KIND, TM, TN> &o, auto wide) {
    u32x4 fb[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      if constexpr (KIND == GEMM_MIXH && !decltype(wide)::value)
        fb[j] = __builtin_bit_cast(u32x4, mx_f16(sc.codes[j][q], sc.scale[j]));
      else if constexpr (MIX)
        fb[j] = __builtin_bit_cast(u32x4, mx_bf16(sc.codes[j][q], sc.scale[j]));
      else
        fb[j] = o.b[j];
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      bf16x8 piece[2];
      if constexpr (KIND == GEMM_MIXH && decltype(wide)::value)
        mx_cut8<_Float16, 2>(__builtin_bit_cast(Raw8<_Float16>, o.a[i]), piece);
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        f32x16 &c = acc[i][j];
        if constexpr (KIND == GEMM_FP4) {
          const i32x8 x = widen(o.a[i]), y = widen(fb[j]);
          const int sa = (int)sc.a[q >> 1][i], sb = (int)sc.b[q >> 1][j];
          if ((q & 1) == 0)
            c = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 4, 0, sa, 0, sb);
          else
            c = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 4, 2, sa, 2, sb);
        } else if constexpr (KIND == GEMM_MIXH && decltype(wide)::value) {
#pragma unroll
          for (int p = 0; p < 2; ++p)
            c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(piece[p], __builtin_bit_cast(bf16x8, fb[j]), c, 0, 0, 0);
        } else if constexpr (KIND == GEMM_F16 || KIND == GEMM_MIXH) {
          c = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, o.a[i]), __builtin_bit_cast(f16x8, fb[j]), c, 0, 0, 0);
        } else {
          c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, o.a[i]), __builtin_bit_cast(bf16x8, fb[j]), c, 0, 0, 0);
        }
      }
    }
  };
  // Reads of the next quarter between the products of this one.
  const auto weave = [&]() {
    constexpr int READS = TM + (MIX ? 0 : TN), EACH = TM * TN / READS > 0 ? TM * TN / READS : 1;
#pragma unroll
    for (int i = 0; i < READS; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, EACH, 0);
    }
  };

  const auto run = [&](auto wide) {
    const int last = s_end - 1;
    At here = {s_begin / a.steps, s_begin % a.steps}, ahead = here;
    int k = here.k, buf = 0;
#pragma unroll
    for (int i = 0; i < S; ++i) {
      load_a(i, ahead);
      if (i + 1 == S) break;  // its B comes with the first step's products
      load_b(i, ahead);
      ahead = next(ahead, s_begin + i < last);
    }
    gemm_wait<LOADS * (S - 2) + LOADS_A>();
    read_scales(0, k, sc, wide);
    read(0, 0, op[0]);
    for (int step = s_begin; step < s_end; ++step) {
      const int then = buf + 1 == S ? 0 : buf + 1, before = buf == 0 ? S - 1 : buf - 1;
      load_b(before, ahead);
      ahead = next(ahead, step + S - 1 < last);
      read(buf, 1, op[1]);
      // a wavefront in its products goes before one at its loads (2 to 4% of the 16-bit kinds; the
      // scaled products lose 1%)
      if constexpr (KIND != GEMM_FP4) __builtin_amdgcn_s_setprio(1);
      multiply(0, op[0], wide);
      weave();
      read(buf, 2, op[0]);
      multiply(1, op[1], wide);
      weave();
      read(buf, 3, op[1]);
      multiply(2, op[0], wide);
      weave();
      if constexpr (KIND != GEMM_FP4) __builtin_amdgcn_s_setprio(0);
      // Every read of this buffer is out.  Once all wavefronts are here the next step's buffer has
      // landed and this one is free; the last quarter's products cover the first reads.  Past the
      // end the last step is loaded and read again, and not multiplied.
      gemm_wait<LOADS * (S - 2)>();
      load_a(buf, ahead);
      if (step < last) k = k + 1 == a.steps ? 0 : k + 1;
      read_scales(then, k, sc_next, wide);
      read(then, 0, op[0]);
      multiply(3, op[1], wide);
      weave();
      sc = sc_next;
      buf = then;
    }
    gemm_wait<0>();  // no load may land after the workgroup has left
  };
  if (s_begin < s_end) {
    if (KIND == GEMM_MIXH && any_wide)
      run(Flag<KIND == GEMM_MIXH>());
    else
      run(Flag<false>());
  }

  const int64_t at = (m0 + wm) * a.N + n0 + wn;
  constexpr bool SHIFT = KIND == GEMM_MIXH;
  if (any_wide) {
#pragma unroll
    for (int j = 0; j < TN; ++j) shift_of[j] = 0;
  }
  if (a.slices > 1)
    gemm_store<float, SHIFT, TM, TN>(acc, a.partial + slice * a.M * a.N + at, nullptr, shift_of, a.N, (int)la - wm,
                                     (int)lb - wn);
  else
    gemm_store<T, SHIFT, TM, TN>(acc, reinterpret_cast<T *>(a.c) + at,
                                 a.bias ? reinterpret_cast<const T *>(a.bias) + n0 + wn : nullptr, shift_of, a.N,
                                 (int)la - wm, (int)lb - wn);
}

template <GemmKind KIND, typename T, int WM, int WN, int TM, int TN, int S>
__global__ __launch_bounds__(64 * WM * WN, 1) void mx_gemm_kernel(GemmArgs a) {
  __shared__ __attribute__((aligned(128))) char lds[sizeof(GemmStage<KIND, WM * TM * 32, WN * TN * 32>) * S];
  gemm_body<KIND, T, WM, WN, TM, TN, S>(a, lds, blockIdx.x, blockIdx.y);
}

// Two products in one launch, of 16-bit operands: workgroups [0, n) are the first's tiles, slice by
// slice, the others the second's.  Their loads and products overlap where one grid alone leaves the
// chip half empty: the gradients of a 4096 x 1024 -> 1024 binary16 layer take 34 us so, 45 us as two
// launches.
template <GemmKind K1, GemmKind K2, typename T, int WM, int WN, int TM, int TN, int S>
__global__ __launch_bounds__(64 * WM * WN, 1) void mx_gemm_two_kernel(GemmArgs a, GemmArgs b, uint32_t n, uint32_t tiles_a,
                                                                     uint32_t tiles_b) {
  static_assert(!gemm_mixed(K1) && K1 != GEMM_FP4 && !gemm_mixed(K2) && K2 != GEMM_FP4, "one size of LDS");
  __shared__ __attribute__((aligned(128))) char lds[sizeof(GemmStage<K1, WM * TM * 32, WN * TN * 32>) * S];
  if (blockIdx.x < n)
    gemm_body<K1, T, WM, WN, TM, TN, S>(a, lds, blockIdx.x % tiles_a, blockIdx.x / tiles_a);
  else
    gemm_body<K2, T, WM, WN, TM, TN, S>(b, lds, (blockIdx.x - n) % tiles_b, (blockIdx.x - n) / tiles_b);
}

// The slices' sums, in the slices' order; eight slices are asked for at a time.
template <typename T>
__global__ __launch_bounds__(256) void mx_gemm_sum_kernel(GemmArgs a) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, n = a.M * a.N;
  if (i >= n) return;
  float v = 0.0f;
  for (int s0 = 0; s0 < a.slices; s0 += 8) {
    float p[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) p[u] = s0 + u < a.slices ? a.partial[(s0 + u) * n + i] : 0.0f;
#pragma unroll
    for (int u = 0; u < 8; ++u) v += p[u];
  }
  // n stays below 2^26 with more than one slice
  if (a.bias) v += (float)reinterpret_cast<const T *>(a.bias)[(uint32_t)i % (uint32_t)a.N];
  reinterpret_cast<T *>(a.c)[i] = (T)v;
}

// src [rows][cols] -> dst [P][rows][ld], zeros from cols to ld: the pieces of binary32, 16-bit numbers as
// they are.
template <typename T>
__global__ __launch_bounds__(256) void mx_stage_kernel(const T *src, uint16_t *dst, int64_t rows, int64_t cols,
                                                       int64_t ld, int64_t first) {
  constexpr int P = sizeof(T) == 4 ? mx_pieces<T>() : 1;
  const int64_t per_row = ld / 8, id = (first + blockIdx.x) * 256 + threadIdx.x;
  if (id >= rows * per_row) return;
  const int64_t row = id <= 0xffffffffll ? (int64_t)((uint32_t)id / (uint32_t)per_row) : id / per_row;
  const int64_t col = (id - row * per_row) * 8;
  const Raw8<T> r = load8_tail(src + row * cols + col, cols - col);
  bf16x8 f[P];
  mx_cut8<T, P>(r, f);
#pragma unroll
  for (int k = 0; k < P; ++k) *reinterpret_cast<bf16x8 *>(dst + ((int64_t)k * rows + row) * ld + col) = f[k];
}

inline void gemm_pair(GemmArgs &a, int i, int j) {
  a.pa |= (uint64_t)i << (4 * a.pairs);
  a.pb |= (uint64_t)j << (4 * a.pairs++);
}

struct GemmPlan {
  int tile;    // 256, 128 or 64: outputs a side of a workgroup
  int slices;  // of the reduction
};

// Tile and slices for an M x N product of `total` steps: the least time by this model, a function of
// the sizes alone.  Measured (us): a step of a grid of 256 workgroups, and of one of 512, which two
// of the smaller tiles' workgroups a CU share; and what a launch costs besides its steps.  One row of
// times serves all kinds, which are a third apart: it gives 227 us for 8192^3 FP4, which takes 265, and
// 118 for 4096^3 MIX, which takes 102.
struct GemmRow {
  int tile;
  double step1, step2, fixed;
};
constexpr GemmRow GEMM_ROWS[3] = {{256, 1.7, 3.4, 9.0}, {128, 0.6, 1.0, 5.0}, {64, 0.36, 0.52, 3.0}};
constexpr int GEMM_SLICES[8] = {1, 2, 3, 4, 6, 8, 12, 16};

inline int64_t gemm_tiles(int64_t M, int64_t N, int64_t tile) {
  return ((M + tile - 1) / tile) * ((N + tile - 1) / tile);
}
// A slice keeps four steps or more; the partial sums stay below 2^28 bytes.
inline bool gemm_slices_fit(int64_t M, int64_t N, int64_t total, int slices) {
  return slices == 1 || (total >= 4 * slices && (double)M * (double)N * slices <= 67108864.0);
}
// The slices' sum: a launch, and its reads and writes at 4 TB/s.
inline double gemm_sum_time(int64_t M, int64_t N, int slices) {
  return slices == 1 ? 0.0 : 3.0 + (double)M * (double)N * (4.0 * slices + 4.0) / 4e6;
}

inline GemmPlan gemm_plan(int64_t M, int64_t N, int64_t total, double *time = nullptr) {
  GemmPlan best = {64, 1};
  double least = 1e300;
  for (const GemmRow &r : GEMM_ROWS)
    for (int slices : GEMM_SLICES) {
      if (!gemm_slices_fit(M, N, total, slices)) break;
      const int64_t n = gemm_tiles(M, N, r.tile) * slices, full = n / 512, rest = n % 512;
      // a tile of no steps takes one's time too: its workgroups and stores, and a large result in
      // small tiles would pass the 2^32 threads of a launch
      const double steps = total == 0 ? 1.0 : (double)((total + slices - 1) / slices);
      const double t = r.fixed + gemm_sum_time(M, N, slices) +
                       steps * ((double)full * r.step2 + (rest > 256 ? r.step2 : (rest > 0 ? r.step1 : 0.0)));
      if (t < least) {
        least = t;
        best = {r.tile, slices};
      }
    }
  if (time) *time = least;
  return best;
}

// The same for two products in one launch: their workgroups share the chip, 512 at a time at the
// larger grids' rate, and the longer chain of steps is a lower bound.  tile = 0 where two launches
// are faster by the model.
struct GemmTwoPlan {
  int tile, slices1, slices2;
};
inline GemmTwoPlan gemm_two_plan(int64_t M1, int64_t N1, int64_t total1, int64_t M2, int64_t N2, int64_t total2) {
  double t1, t2;
  GemmTwoPlan best = {0, gemm_plan(M1, N1, total1, &t1).slices, gemm_plan(M2, N2, total2, &t2).slices};
  if (M1 == 0 || N1 == 0 || total1 == 0 || M2 == 0 || N2 == 0 || total2 == 0) return best;
  double least = t1 + t2;
  for (const GemmRow &r : GEMM_ROWS) {
    // by slices of one product: its workgroups, its steps, the time of its slices' sum
    struct Choice {
      double n, steps, sum;
    } c[2][8];
    int count[2] = {0, 0};
    const int64_t sizes[2][3] = {{M1, N1, total1}, {M2, N2, total2}};
    for (int p = 0; p < 2; ++p) {
      const int64_t M = sizes[p][0], N = sizes[p][1], total = sizes[p][2];
      const double tiles = (double)gemm_tiles(M, N, r.tile);
      for (int i = 0; i < 8 && gemm_slices_fit(M, N, total, GEMM_SLICES[i]); ++i) {
        const int k = GEMM_SLICES[i];
        c[p][count[p]++] = {tiles * k, (double)(((int)total + k - 1) / k), gemm_sum_time(M, N, k)};
      }
    }
    for (int i = 0; i < count[0]; ++i)
      for (int j = 0; j < count[1]; ++j) {
        const Choice &a = c[0][i], &b = c[1][j];
        const double n = a.n + b.n, chain = a.steps > b.steps ? a.steps : b.steps;
        const double work = (a.n * a.steps + b.n * b.steps) * (r.step2 / 512.0);
        const double alone = chain * (n > 256.0 ? r.step2 : r.step1);
        const double t = r.fixed + (work > alone ? work : alone) + a.sum + b.sum;
        if (n < 2147483648.0 && t < least) {
          least = t;
          best = {r.tile, GEMM_SLICES[i], GEMM_SLICES[j]};
        }
      }
  }
  return best;
}

inline int64_t gemm_slices_bytes(int64_t M, int64_t N, int slices) { return slices > 1 ? slices * M * N * 4 : 0; }
inline int64_t gemm_partial_bytes(int64_t M, int64_t N, int64_t total) {
  return gemm_slices_bytes(M, N, gemm_plan(M, N, total).slices);
}

template <typename T>
void gemm_sum(const GemmArgs &a, hipStream_t stream) {
  if (a.slices > 1) mx_gemm_sum_kernel<T><<<(unsigned)((a.M * a.N + 255) / 256), 256, 0, stream>>>(a);
}

// Both products by one launch at the plan's tile; a and b are complete but for total and slices.
template <GemmKind K1, GemmKind K2, typename T>
hipError_t gemm_two(GemmArgs &a, GemmArgs &b, const GemmTwoPlan &p, hipStream_t stream) {
  a.total = a.steps * a.pairs;
  b.total = b.steps * b.pairs;
  a.slices = p.slices1;
  b.slices = p.slices2;
  const uint32_t ta = (uint32_t)gemm_tiles(a.M, a.N, p.tile), tb = (uint32_t)gemm_tiles(b.M, b.N, p.tile);
  const uint32_t n = ta * (uint32_t)a.slices;
  const dim3 grid(n + tb * (uint32_t)b.slices);
  if (p.tile == 256)
    mx_gemm_two_kernel<K1, K2, T, 2, 4, 4, 2, 2><<<grid, 512, 0, stream>>>(a, b, n, ta, tb);
  else if (p.tile == 128)
    mx_gemm_two_kernel<K1, K2, T, 2, 2, 2, 2, 2><<<grid, 256, 0, stream>>>(a, b, n, ta, tb);
  else
    mx_gemm_two_kernel<K1, K2, T, 2, 2, 1, 1, 4><<<grid, 256, 0, stream>>>(a, b, n, ta, tb);
  gemm_sum<T>(a, stream);
  gemm_sum<T>(b, stream);
  return hipGetLastError();
}

template <GemmKind KIND, typename T>
hipError_t gemm(GemmArgs &a, const GemmPlan &p, hipStream_t stream) {
  a.total = a.steps * a.pairs;
  a.slices = p.slices;
  const dim3 grid((unsigned)(((a.M + p.tile - 1) / p.tile) * ((a.N + p.tile - 1) / p.tile)), (unsigned)p.slices);
  if (p.tile == 256)
    mx_gemm_kernel<KIND, T, 2, 4, 4, 2, 2><<<grid, 512, 0, stream>>>(a);
  else if (p.tile == 128)
    mx_gemm_kernel<KIND, T, 2, 2, 2, 2, 2><<<grid, 256, 0, stream>>>(a);
  else
    mx_gemm_kernel<KIND, T, 2, 2, 1, 1, 4><<<grid, 256, 0, stream>>>(a);
  gemm_sum<T>(a, stream);
  return hipGetLastError();
}

template <GemmKind KIND, typename T>
hipError_t gemm(GemmArgs &a, hipStream_t stream) {
  return gemm<KIND, T>(a, gemm_plan(a.M, a.N, a.steps * a.pairs), stream);
}

}  // namespace mcf
