// Gradients of attention in a window (attn_kernel_window.h).
//
// With P = exp(scale S - lse) over the visible pairs, S = Q K^T, dP = dO V^T, delta = rowsum(dO * O):
//   dS = P * (dP - delta),  dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO.
// Two kernels, each of which forms S and dP once: one owns queries and goes over their keys (dQ, and delta on the way),
// one owns keys and goes over the queries that see them, of all query heads that share them (dK, dV).  Seven products
// instead of five, but no sum goes through atomics: the same inputs give the same bits.
//
// Both are the same shape.  A wave owns 32 columns (its queries, or its keys) as second operands; tiles of 32 rows of two
// matrices (K and V, or Q and dO) pass through LDS, read row-wise for S^T and dP^T (first operand: rows of the tile) and
// transposed for the products that add up, whose second operands are P and dS as they lie in registers.  Two waves per SIMD.
//
// A wave issues in order, an instruction every four cycles at best, and an MFMA that finds the matrix pipe busy holds up
// what stands behind it.  So the work on 32 rows is written as a stream of GAPS: an MFMA, the read of the first operand of
// three gaps later, a share of the vector work (exponentials beside dP and what follows it, dS behind them), a scheduling
// barrier; the second wave of the SIMD fills what one leaves.  Us of dQ, and of dK and dV, for 16 380 tokens, 8 query heads
// on 4 key heads, D = 128, nine frames of 780 and the first: scheduled by the compiler, 64 columns to a wave, one wave per
// SIMD 930 and 2660 (it gathers reads and vector work and spills), the same in gaps 787 and 1253 (half its cycles waits),
// this form 642 and 940.  Of a gap's about 125 cycles (dQ) and 142 (dK, dV) on a CU, its eight waves' MFMAs take 64 of each
// SIMD, and their operands, 1 KB a wave and 1.25 KB with K's, 64 and 80 of LDS: 32 columns to a wave feed no more.
#pragma once
#include "attn_kernel_window.h"

namespace calibatt_dev {

// Swizzle of 16-byte chunks for tiles that are read both ways: 16 consecutive rows at one chunk column, and four
// consecutive rows times four neighbouring chunks, each land on 16 distinct chunks of a 256-byte line.
template <int D>
__device__ __forceinline__ int both_swz(int row) {
  constexpr int CH = D / 8;
  const int u = row / (16 / CH);
  return CH == 16 ? ((u & 3) << 2) | ((u >> 2) & 3) : ((u & 1) << 2) | ((u >> 1) & 3);
}

// fp16 has few exponents: probabilities are kept times 2^15, which takes 1 to 32768, and dS times a power of two F that follows
// the data (bf16 needs neither).  As out is a mean of rows of V, |dS| <= P (|dP| + |delta|) <= 2 |dO| |V|, and F is the largest
// power of two that keeps twice that bound within 2^16: no dS leaves the type, whatever the scale of dO (a loss that was
// scaled, say), and of a bound of one, dS down to 2^-28 keep their precision.  dQ's columns are queries, so F is a query's own
// there; dK's are keys, whose sums need one F for all queries, that of the largest |dO| of the key head.
template <typename T> struct GradScale { static constexpr float P_LOG2 = 0.f, P_UNIT = 1.f; static constexpr bool FOLLOWS = false; };
template <> struct GradScale<F16> { static constexpr float P_LOG2 = 15.f, P_UNIT = 1.f / 32768.f; static constexpr bool FOLLOWS = true; };

// F for squares of |dO| and of |V|
__device__ __forceinline__ float grad_factor(float do_square, float v_square) {
  const float bound = 2.f * sqrtf(do_square * v_square);  // (squares of up to 128 * 65504^2, products within fp32)
  return bound > 0.f ? ldexpf(1.f, 15 - __builtin_amdgcn_frexp_expf(bound)) : 1.f;
}

// out (+)= a b.  Written out, because the compiler, given 512 registers, keeps every accumulator of an MFMA in AGPRs, from
// where S and dP are copied element by element, and then moves the sums around them (700 copies per 128 MFMAs).  Here S
// and dP are VGPRs (IN_V) and the sums AGPRs.  What the compiler does not know of an asm's MFMA is kept by hand: the
// operands may just have been written by vector instructions (two wait states in front), and a result is read by others
// only behind settle() (csrc/check_mfma_waits.py).
// B_A: the second operand is in AGPRs as well.
template <typename T, bool IN_V, bool FRESH, bool B_A = false>
__device__ __forceinline__ void mfma_gap(f32x16 &out, const u32x4 a, const u32x4 b) {
#define CALIBATT_GAP(op)                                                                                                  \
  if constexpr (FRESH && B_A) asm volatile("s_nop 1\n\t" op " %0, %1, %2, 0" : "=&v"(out) : "v"(a), "a"(b));              \
  else if constexpr (FRESH) asm volatile("s_nop 1\n\t" op " %0, %1, %2, 0" : "=&v"(out) : "v"(a), "v"(b));                \
  else if constexpr (IN_V && B_A) asm volatile("s_nop 1\n\t" op " %0, %1, %2, %0" : "+v"(out) : "v"(a), "a"(b));          \
  else if constexpr (IN_V) asm volatile("s_nop 1\n\t" op " %0, %1, %2, %0" : "+v"(out) : "v"(a), "v"(b));                 \
  else asm volatile("s_nop 1\n\t" op " %0, %1, %2, %0" : "+a"(out) : "v"(a), "v"(b));
  if constexpr (std::is_same<T, Bf16>::value) {
    CALIBATT_GAP("v_mfma_f32_32x32x16_bf16")
  } else {
    CALIBATT_GAP("v_mfma_f32_32x32x16_f16")
  }
#undef CALIBATT_GAP
}
// Everything read behind this sees the results of the MFMAs in front of it.
template <bool IN_V>
__device__ __forceinline__ void settle(f32x16 &x) {
  if constexpr (IN_V) asm volatile("s_nop 15" : "+v"(x));
  else asm volatile("s_nop 15" : "+a"(x));
}

template <int D, typename T, int NT_>
struct GradTile {
  static constexpr int NT = NT_, COLS = 32, BLOCK = NT / 64 * COLS;  // columns of a wave, of the workgroup
  static constexpr int ROWS = 32, ROWB = D * 2, CH = D / 8, DS = D / 16, DB = D / 32;
  static constexpr int TILE = ROWS * ROWB, PAIR = 2 * TILE;      // bytes of one matrix's tile, of both
  // Load instructions of a wave for a pair of tiles: ITERS for each matrix, or, where one instruction of half the waves
  // fills a tile, one for the matrix of its half.
  static constexpr int ITERS = ROWS * CH / NT, LOADS = ITERS ? 2 * ITERS : 1, RPI = NT / CH;
  static_assert((ITERS && RPI % 16 == 0) || 2 * ROWS * CH == NT, "the swizzle of an instruction's rows is the same for every one");

  // A phase (S, dP, or one of the products that add up) has PH gaps.  The UNITS of vector work of 32 rows, pairs of a lane's
  // values, by their gap behind the start of dP: exponentials over 22/16 of a phase, then each pair's dS, in dK and dV's
  // kernel over 18/16, in dQ's over the 10/16 that are left before S of the next rows.  In the former the first halves are
  // needed half a phase before the second ones: probabilities from gap PH on (dV), dS from gap 2 PH on (dK).
  static constexpr int AHEAD = 3, RA = AHEAD + 1;  // gaps between the read of a first operand and its use
  static constexpr int PH = DS, UNITS = 8, EXP_GAPS = 22 * PH / 16;
  static_assert(DS == 2 * DB, "phases of the same length");
  static constexpr int exp_gap(int u) { return u * EXP_GAPS / UNITS; }
  static constexpr int ds_gap(int u) { return EXP_GAPS + u * (18 * PH / 16) / UNITS; }
  static constexpr int dq_ds_gap(int u) { return EXP_GAPS + u * (2 * PH - EXP_GAPS) / UNITS; }
  static_assert(exp_gap(UNITS / 2 - 1) < PH && exp_gap(UNITS - 1) < PH + PH / 2, "probabilities are there before dV");
  static_assert(EXP_GAPS >= PH && ds_gap(UNITS / 2 - 1) < 2 * PH && ds_gap(UNITS - 1) < 2 * PH + PH / 2, "dS is there before dK");
  static_assert(dq_ds_gap(UNITS - 1) < 2 * PH, "S of the next rows takes the place of this one's");

  int tid, lane, wave, l32, g;
  uint32_t row_addr;     // row-wise reads: chunk column s at row_addr ^ (s << 5)
  uint32_t col_addr[2];  // transposed reads: d block db at col_addr[t] ^ (db << 6), slab j at + 16 j * ROWB
  uint32_t second_addr;  // operands of columns that stay in LDS: chunk column s at second_addr ^ (s << 5)
  uint32_t lds_base, lds_wave;
  int load_row, load_chunk;  // what this lane loads of a tile

  __device__ __forceinline__ explicit GradTile(char *lds) {
    tid = threadIdx.x;
    lane = tid & 63;
    wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    l32 = lane & 31;
    g = lane >> 5;
    lds_base = (uint32_t)(uintptr_t)(LDS_PTR(char))lds;  // a multiple of 1024
    lds_wave = __builtin_amdgcn_readfirstlane(lds_base + wave * 1024);  // (of a pair, where a load is half a pair)
    load_row = tid / CH % ROWS;
    load_chunk = (tid % CH) ^ both_swz<D>(load_row);
    const int row = (l32 & 0x13) | ((l32 & 4) << 1) | ((l32 & 8) >> 1);  // so that a lane's eight values are of consecutive rows
    row_addr = row * ROWB + ((g ^ both_swz<D>(row)) << 4);
    second_addr = l32 * ROWB + ((g ^ both_swz<D>(l32)) << 4);
    const int L16 = lane & 15, blk = lane >> 4;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int r = 8 * (blk >> 1) + (L16 >> 2) + 4 * t;
      col_addr[t] = r * ROWB + (((2 * (blk & 1) + ((L16 & 3) >> 1)) ^ both_swz<D>(r)) << 4) + (L16 & 1) * 8;
    }
  }
  // rows [row0, row0 + 32) of two matrices into the pair of tiles at LDS byte `at`
  __device__ __forceinline__ void issue(const u32x4 first, const u32x4 second, int row0, uint32_t at, uint32_t first_bytes, uint32_t second_bytes) const {
    if constexpr (ITERS > 0) {
#pragma unroll
      for (int it = 0; it < ITERS; ++it)
        dma_16B_per_lane<true>(first, load_row * first_bytes + load_chunk * 16, (uint32_t)(row0 + it * RPI) * first_bytes, lds_wave + at + it * NT * 16);
#pragma unroll
      for (int it = 0; it < ITERS; ++it)
        dma_16B_per_lane<true>(second, load_row * second_bytes + load_chunk * 16, (uint32_t)(row0 + it * RPI) * second_bytes, lds_wave + at + TILE + it * NT * 16);
    } else if (wave < NT / 128) {
      dma_16B_per_lane<true>(first, load_row * first_bytes + load_chunk * 16, (uint32_t)row0 * first_bytes, lds_wave + at);
    } else {
      dma_16B_per_lane<true>(second, load_row * second_bytes + load_chunk * 16, (uint32_t)row0 * second_bytes, lds_wave + at);
    }
  }
  // a column's D elements as second operand
  __device__ __forceinline__ void operand(const uint16_t *row, u32x4 (&x)[DS]) const {
#pragma unroll
    for (int s = 0; s < DS; ++s) x[s] = *reinterpret_cast<const u32x4 *>(row + 16 * s + 8 * g);
  }
  // waits for the loads of operands here, and not inside the loop, where tiles are on their way as well
  template <bool IN_A = false>
  static __device__ __forceinline__ void arrive(u32x4 (&x)[DS]) {
#pragma unroll
    for (int s = 0; s < DS; ++s) {
      if constexpr (IN_A) asm volatile("" : "+a"(x[s]));
      else asm volatile("" : "+v"(x[s]));
    }
  }
  // First operands: slab s of a tile's rows, and their transpose's 16-row slab j and 32-wide d block db.  `at`: LDS address
  // of this lane's piece of a pair of tiles (see Places), `off`: of the tile in the pair.
  static __device__ __forceinline__ u32x4 rows_of(uint32_t at, int off, int s) {
    return *(LDS_PTR(const u32x4))(uintptr_t)((at ^ (s << 5)) + off);
  }
  static __device__ __forceinline__ u32x4 cols_of(const uint32_t (&at)[2], int off, int j, int db) {
    off += 16 * j * ROWB;
    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(uintptr_t)((at[0] ^ (db << 6)) + off)));
    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(uintptr_t)((at[1] ^ (db << 6)) + off)));
    return u32x4{lo[0], lo[1], hi[0], hi[1]};
  }
  // Addresses of a pair of tiles.  They pass through an empty asm, so that the many that are derived from them are formed
  // where they are used (one instruction) instead of kept in registers.
  struct Places {
    uint32_t rows, cols[2];
    __device__ __forceinline__ Places(const GradTile &t, uint32_t pair) : rows(t.row_addr + pair), cols{t.col_addr[0] + pair, t.col_addr[1] + pair} {
      asm volatile("" : "+v"(rows), "+v"(cols[0]), "+v"(cols[1]));
    }
  };
  // a column's D sums times f, rounded, to its row in memory; zeros for a row that is not `there`
  static __device__ __forceinline__ void store(const f32x16 (&sum)[DB], float f, bool there, uint16_t *row, int g) {
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const u32x2 x = {T::pack(sum[db][4 * a] * f, sum[db][4 * a + 1] * f), T::pack(sum[db][4 * a + 2] * f, sum[db][4 * a + 3] * f)};
        *reinterpret_cast<u32x2 *>(row + 32 * db + 8 * a + 4 * g) = there ? x : u32x2{0, 0};
      }
  }
};

// dP - delta in units of dS beside P as kept
__device__ __forceinline__ float ds_factor(float dp, float ds_of_p, float dl) { return __builtin_fmaf(dp, ds_of_p, -dl); }

// The queries that see keys [j0, j1) (j1 within k_len): of the window between two positions, of the sinks all from the
// first on.
struct WindowQueries {
  int begin, end;
  // first query that sees key j, last + 1 that does
  static __device__ __forceinline__ int first_of(const WindowDims &p, const WindowEntry &e, int j) {
    if (p.right < 0) return 0;
    const long long pos = ((long long)(j / p.frame) - p.right) * p.frame - e.start;
    return (int)min(max(pos, 0ll), (long long)e.q_len);
  }
  static __device__ __forceinline__ int end_of(const WindowDims &p, const WindowEntry &e, int j) {
    if (p.left < 0 || j < p.sinks) return e.q_len;
    const long long pos = ((long long)(j / p.frame) + p.left + 1) * p.frame - e.start;
    return (int)min(max(pos, 0ll), (long long)e.q_len);
  }
  __device__ __forceinline__ WindowQueries(const WindowDims &p, const WindowEntry &e, int j0, int j1) {
    begin = first_of(p, e, j0);
    end = j0 < p.sinks ? e.q_len : end_of(p, e, j1 - 1);
  }
};

// ---- sizes of dO and V --------------------------------------------------------------------------------------
// Largest squares of the norms of a key head's rows of dO (of the query heads that share it) and of V, of each in as many
// pieces as there are slots.  Rows that meet nothing do not count, they may hold anything, nor do rows that are not finite:
// those spoil what they meet, and nothing else.  Maxima: the order does not matter.  Bound by its chain of loads, of which
// eight rows a lane are in flight: 14 us of the 483 of a pass of 12 heads of 8190 tokens, D = 128, 16 of 2167 for 16 380 tokens,
// 8 query heads on 4.
constexpr int SIZE_ROWS = 128, SIZE_MAX_SLOTS = 128;  // rows of a piece at least, pieces of either tensor at most

template <int D>
__global__ __launch_bounds__(256) void window_attn_sizes_kernel(const uint16_t *__restrict__ gdo, const uint16_t *__restrict__ gv, const WindowDims p) {
  constexpr int LANES = D / 8, ROWS = 256 / LANES, FLIGHT = 8;
  __shared__ float most[4];
  const int slots = p.do_slots + p.v_slots, bh = blockIdx.x / slots, slot = blockIdx.x - bh * slots, b = bh / p.Hkv, hk = bh - b * p.Hkv;
  const int G = p.Hq / p.Hkv, c = 8 * (threadIdx.x % LANES);
  const bool of_do = slot < p.do_slots;
  // G Nq and Nk rows, each within 31 bits, but not what is stepped beyond them
  const int rows = of_do ? G * p.Nq : p.Nk, piece = of_do ? slot : slot - p.do_slots, pieces = of_do ? p.do_slots : p.v_slots;
  const int first = (int)((long long)rows * piece / pieces), last = (int)((long long)rows * (piece + 1) / pieces);
  const WindowEntry e(p, b);
  float m = 0.f;
  const uint16_t *const do_group = gdo + (size_t)b * p.dout.b + (size_t)hk * G * p.dout.h, *const v_head = gv + (size_t)b * p.kv.b + (size_t)hk * p.kv.h;
  for (long long r0 = (long long)first + threadIdx.x / LANES; r0 < last; r0 += FLIGHT * ROWS) {
    u32x4 raw[FLIGHT];
    bool seen[FLIGHT];
#pragma unroll
    for (int n = 0; n < FLIGHT; ++n) {
      const int r = (int)min(r0 + n * ROWS, (long long)last - 1);
      const uint16_t *row;
      if (of_do) {
        const int g = r / p.Nq, i = r - g * p.Nq;
        int lo, hi;
        e.interval(p, i, lo, hi);
        seen[n] = i < e.q_len && (lo < hi || min(p.sinks, hi) > 0);
        row = do_group + (size_t)g * p.dout.h + (size_t)i * p.dout.n;
      } else {
        seen[n] = r < e.k_len && WindowQueries::first_of(p, e, r) < WindowQueries::end_of(p, e, r);
        row = v_head + (size_t)r * p.kv.n;
      }
      raw[n] = *reinterpret_cast<const u32x4 *>(row + c);
    }
#pragma unroll
    for (int n = 0; n < FLIGHT; ++n) {
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t two = raw[n][k];
        float x[2];
        F16::unpack(two, x);
        s = __builtin_fmaf(x[0], x[0], __builtin_fmaf(x[1], x[1], s));
      }
#pragma unroll
      for (int k = 1; k < LANES; k *= 2) s += __shfl_xor(s, k);  // (all lanes of a row are in the loop together)
      m = seen[n] && s <= FLT_MAX ? fmaxf(m, s) : m;
    }
  }
#pragma unroll
  for (int k = LANES; k < 64; k *= 2) m = fmaxf(m, __shfl_xor(m, k));
  if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6] = m;
  __syncthreads();
  if (threadIdx.x == 0) p.sizes[blockIdx.x] = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
}

// The largest of a key head's pieces, the same in every lane.
__device__ __forceinline__ void largest_squares(const WindowDims &p, int b, int hk, float &of_do, float &of_v) {
  const int lane = threadIdx.x & 63;
  const float *const at = p.sizes + ((size_t)b * p.Hkv + hk) * (p.do_slots + p.v_slots);
  float d = 0.f, v = 0.f;
  for (int i = lane; i < p.do_slots; i += 64) d = fmaxf(d, at[i]);
  for (int i = lane; i < p.v_slots; i += 64) v = fmaxf(v, at[p.do_slots + i]);
#pragma unroll
  for (int k = 1; k < 64; k *= 2) {
    d = fmaxf(d, __shfl_xor(d, k));
    v = fmaxf(v, __shfl_xor(v, k));
  }
  of_do = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, d)));
  of_v = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v)));
}

// ---- dQ -----------------------------------------------------------------------------------------------------
// 128 queries to a workgroup, two workgroups per CU: eight waves of one workgroup on the same tiles read them half as often,
// but wait for each other (655 us two, 700 one, also with a barrier for every second tile and three tiles on their way).
// The tiles lie in a ring of four: in its turn tile t is read for dP, t - 1 for dQ and t + 1 for S, while t + 2 is on its way.
template <int D, typename T>
using DqTile = GradTile<D, T, 256>;
template <int D, typename T>
constexpr int dq_lds_bytes() { return 4 * DqTile<D, T>::PAIR; }

template <int D, typename T>
__global__ __launch_bounds__(256, 2) void window_attn_dq_kernel(
    const uint16_t *__restrict__ gdo, const uint16_t *__restrict__ gq, const uint16_t *__restrict__ gk,
    const uint16_t *__restrict__ gv, const uint16_t *__restrict__ gout, const float *__restrict__ lse,
    uint16_t *__restrict__ gdq, float *__restrict__ stats, const WindowDims p) {
  using Tile = DqTile<D, T>;
  using Tiles = WindowTiles<Tile::ROWS>;
  constexpr int BQ = Tile::BLOCK, DS = Tile::DS, DB = Tile::DB, AHEAD = Tile::AHEAD, RA = Tile::RA;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int nbq = (p.Nq + BQ - 1) / BQ;
  const int unit = window_unit(p.B * p.Hq * nbq * p.dq_parts);
  if (unit < 0) return;
  const int part = unit % p.dq_parts, of_q = unit / p.dq_parts;
  const int x = of_q / nbq, r = nbq - 1 - (of_q - x * nbq);
  int b, h;
  window_head(x, p.B, p.Hq / p.Hkv, b, h);
  const int bh = b * p.Hq + h;
  const WindowEntry e(p, b);
  const Tile w(lds);
  const int i0 = r * BQ, i1 = min(i0 + BQ, e.q_len), col = i0 + w.wave * Tile::COLS + w.l32;
  const size_t row0 = (size_t)bh * p.Nq;
  f32x16 dq[DB];
  float ds_unit = 1.f;  // what dQ's sums are to be multiplied by: 1 / F
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) dq[db][v] = 0.f;
  if (i0 < i1) {
    float most_do = 0.f, most_v = 0.f;
    if constexpr (GradScale<T>::FOLLOWS) largest_squares(p, b, h / (p.Hq / p.Hkv), most_do, most_v);
    const Tiles tiles(p, e, i0, i1);
    // tiles [t0, t0 + n) of the block, counted from 0 below
    const int t0 = (int)((long long)tiles.n * part / p.dq_parts), n_tiles = (int)((long long)tiles.n * (part + 1) / p.dq_parts) - t0;
    const size_t kv_head = (size_t)b * p.kv.b + (size_t)(h / (p.Hq / p.Hkv)) * p.kv.h;
    const uint32_t row_bytes = (uint32_t)p.kv.n * 2;
    u32x4 Kres = head_rsrc(gk + kv_head, 0), Vres = head_rsrc(gv + kv_head, 0);
    auto issue = [&](int t) {  // a tile behind the last one reads nothing
      const int end = t < n_tiles ? tiles.end(t0 + t) : 0;
      Kres[2] = Vres[2] = __builtin_amdgcn_readfirstlane(end > 0 ? (uint32_t)(end - 1) * row_bytes + Tile::ROWB : 0u);
      const int first = __builtin_amdgcn_readfirstlane(t < n_tiles ? tiles.row(t0 + t) : 0);
      w.issue(Kres, Vres, first, (uint32_t)(t & 3) * Tile::PAIR, row_bytes, row_bytes);
    };
    issue(0);
    u32x4 q[DS], dout[DS];
    int lo, hi;
    const int row = min(col, i1 - 1);  // columns behind the last query: its values, not stored
    e.interval(p, row, lo, hi);
    w.operand(gq + (size_t)b * p.q.b + (size_t)h * p.q.h + (size_t)row * p.q.n, q);
    w.operand(gdo + (size_t)b * p.dout.b + (size_t)h * p.dout.h + (size_t)row * p.dout.n, dout);
    const float z = lse[row0 + row];
    // a query that sees nothing: exponents of -inf, and no dO, as a probability of zero does not outweigh what is not finite
    const bool sees = z != -INFINITY;
    const float lse2 = sees ? z * 1.4426950408889634f - GradScale<T>::P_LOG2 : INFINITY;
#pragma unroll
    for (int s = 0; s < DS; ++s) dout[s] = sees ? dout[s] : u32x4{0, 0, 0, 0};
    float dl = 0.f, ds_of_p = 1.f;  // ds_of_p: factor of dP - delta beside P as kept
    {
      float square = 0.f;
      u32x4 o[DS];
      w.operand(gout + (size_t)b * p.out.b + (size_t)h * p.out.h + (size_t)row * p.out.n, o);
#pragma unroll
      for (int s = 0; s < DS; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t x = dout[s][i], y = o[s][i];
          float x2[2], y2[2];
          T::unpack(x, x2);
          T::unpack(y, y2);
          dl = __builtin_fmaf(x2[0], y2[0], dl);
          dl = __builtin_fmaf(x2[1], y2[1], dl);
          if constexpr (GradScale<T>::FOLLOWS) square = __builtin_fmaf(x2[0], x2[0], __builtin_fmaf(x2[1], x2[1], square));
        }
      dl = sum_with_other_half(dl);
      float dl_keys = dl;
      if constexpr (GradScale<T>::FOLLOWS) {
        const float f = grad_factor(sum_with_other_half(square), most_v);
        ds_unit = 1.f / f;
        ds_of_p = f * GradScale<T>::P_UNIT;
        dl_keys = dl * (grad_factor(most_do, most_v) * GradScale<T>::P_UNIT);
        dl *= ds_of_p;
      }
      if (w.g == 0 && col < i1 && part == 0) {  // for dK and dV: [head][lse2, delta][query]
        stats[2 * row0 + col] = lse2;
        stats[2 * row0 + p.Nq + col] = dl_keys;
      }
    }
    // dO in AGPRs, beside dQ: the compiler halves the registers, and the VGPRs are for the rest
    Tile::arrive(q);
    Tile::template arrive<true>(dout);
    // the logit of an unseen key: -inf behind its product with the scale, which is not zero
    const float sc = p.scale_log2e == 0.f ? 1e-30f : p.scale_log2e, unseen = sc < 0.f ? INFINITY : -INFINITY;
    f32x16 s, dp;
    u32x4 ds[2], ds_before[2], a[RA];
    ds_before[0] = ds_before[1] = u32x4{0, 0, 0, 0};
    issue(1);
    asm volatile("s_waitcnt vmcnt(%0)" : : "n"(Tile::LOADS) : "memory");
    __syncthreads();
    auto place_of = [&](int t) { return typename Tile::Places(w, w.lds_base + (uint32_t)(t & 3) * Tile::PAIR); };
    typename Tile::Places before = place_of(0);  // (dS before tile 0 is zero)
    static_unroll<DS>([&](auto k) {
      a[0] = Tile::rows_of(before.rows, 0, k);
      mfma_gap<T, true, k == 0>(s, a[0], q[k]);
    });
    static_unroll<AHEAD>([&](auto i) { a[i] = Tile::rows_of(before.rows, Tile::TILE, i); });
    for (int t = 0; t < n_tiles; ++t) {
      // dP, dQ of tile t - 1, S of tile t + 1; exponentials and dS beside the first two
      const typename Tile::Places at = place_of(t), next = place_of(t + 1);
      constexpr int N = 3 * DS;
      static_assert(N % RA == 0, "the operands' places go on with the next tile");
      auto fetch = [&](auto q) {  // the operand of gap q (behind the last one: of tile t + 1)
        constexpr int i = q;
        if constexpr (i < DS) a[i % RA] = Tile::rows_of(at.rows, Tile::TILE, i);
        else if constexpr (i < 2 * DS) a[i % RA] = Tile::cols_of(before.cols, 0, (i - DS) / DB, (i - DS) % DB);
        else if constexpr (i < N) a[i % RA] = Tile::rows_of(next.rows, 0, i - 2 * DS);
        else a[i % RA] = Tile::rows_of(next.rows, Tile::TILE, i - N);
      };
      static_unroll<N>([&](auto gap) {
        constexpr int g = gap;
        if constexpr (g == 2 * DS - AHEAD) {
          asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
          __syncthreads();  // tile t + 1 is there, and every wave is done with tile t - 2, whose place t + 2 takes
          issue(t + 2);
        }
        fetch(std::integral_constant<int, g + AHEAD>{});
        if constexpr (g < DS) mfma_gap<T, true, g == 0, true>(dp, a[g % RA], dout[g]);
        else if constexpr (g < 2 * DS) mfma_gap<T, false, false>(dq[(g - DS) % DB], a[g % RA], ds_before[(g - DS) / DB]);
        else mfma_gap<T, true, g == 2 * DS>(s, a[g % RA], q[g - 2 * DS]);
        if constexpr (g == 0) {
          settle<true>(s);
          if (!tiles.whole(t0 + t)) {  // the keys that a query does not see: a probability of 2^-inf
            int from, end;
            tile_interval(tiles, t0 + t, lo, hi, from, end);
            const uint32_t span = (uint32_t)max(end - from, 0);
            from = tiles.row(t0 + t) + 8 * w.g - from;
#pragma unroll
            for (int v = 0; v < 16; ++v) s[v] = (uint32_t)(from + 16 * (v >> 3) + (v & 7)) < span ? s[v] : unseen;
          }
        }
        if constexpr (g == Tile::EXP_GAPS) settle<true>(dp);
        static_unroll<Tile::UNITS>([&](auto u) {
          constexpr int v = 2 * u;
          if constexpr (Tile::exp_gap(u) == g) {
            s[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[v], sc, -lse2));
            s[v + 1] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[v + 1], sc, -lse2));
          }
          if constexpr (Tile::dq_ds_gap(u) == g)
            ds[v >> 3][(v >> 1) & 3] = T::pack(s[v] * ds_factor(dp[v], ds_of_p, dl), s[v + 1] * ds_factor(dp[v + 1], ds_of_p, dl));
        });
        __builtin_amdgcn_sched_barrier(0);
      });
      before = at;
      ds_before[0] = ds[0];
      ds_before[1] = ds[1];
    }
    settle<true>(s);  // nothing reads the last S, but its registers are written again
    if (n_tiles > 0)
      static_unroll<DS>([&](auto k) {
        a[0] = Tile::cols_of(before.cols, 0, k / DB, k % DB);
        mfma_gap<T, false, false>(dq[k % DB], a[0], ds_before[k / DB]);
      });
    asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
#pragma unroll
    for (int db = 0; db < DB; ++db) settle<false>(dq[db]);
  }
  if (col >= p.Nq) return;
  if (p.dq_parts > 1) {
    float *const to = p.part_dq + ((size_t)part * ((size_t)p.B * p.Hq * p.Nq) + row0 + col) * D + 4 * w.g;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int a = 0; a < 4; ++a)
        *reinterpret_cast<f32x4 *>(to + 32 * db + 8 * a) =
            f32x4{dq[db][4 * a] * ds_unit, dq[db][4 * a + 1] * ds_unit, dq[db][4 * a + 2] * ds_unit, dq[db][4 * a + 3] * ds_unit};
  } else {
    Tile::store(dq, p.scale * ds_unit, col < i1, gdq + (size_t)b * p.dq.b + (size_t)h * p.dq.h + (size_t)col * p.dq.n, w.g);
  }
}

// ---- dK, dV -------------------------------------------------------------------------------------------------
// Units of work of one key head: the blocks that hold sinks in bwd_sink_parts parts each, the others in bwd_parts.
__device__ __forceinline__ int grad_units(const WindowDims &p, int n_blocks) {
  return p.n_sink_blocks * p.bwd_sink_parts + (n_blocks - p.n_sink_blocks) * p.bwd_parts;
}

// At D = 128 the sums, K and V of 32 columns are 192 of a wave's 256 registers, and what is left spills; so the operands of
// K stay in LDS there, where reading them takes the reads of 32 rows from 32 to 40 KB a wave.
template <int D>
constexpr bool DKV_K_IN_LDS = D == 128;
constexpr int DKV_RING = 4;  // two tiles that are read, two on their way
template <int D, typename T>
using DkvTile = GradTile<D, T, 512>;
template <int D, typename T>
constexpr int dkv_lds_bytes() {
  using Tile = DkvTile<D, T>;
  return DKV_RING * Tile::PAIR + DKV_RING * 256 + (DKV_K_IN_LDS<D> ? Tile::BLOCK * Tile::ROWB : 0);
}

template <int D, typename T>
__global__ __launch_bounds__(512, 2) void window_attn_dkv_kernel(
    const uint16_t *__restrict__ gdo, const uint16_t *__restrict__ gq, const uint16_t *__restrict__ gk,
    const uint16_t *__restrict__ gv, const float *__restrict__ stats,
    uint16_t *__restrict__ gdk, uint16_t *__restrict__ gdv, const WindowDims p) {
  using Tile = DkvTile<D, T>;
  constexpr int BKV = Tile::BLOCK, DS = Tile::DS, DB = Tile::DB, ROWS = Tile::ROWS, AHEAD = Tile::AHEAD, RA = Tile::RA;
  constexpr bool K_LDS = DKV_K_IN_LDS<D>;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  // [ring][Q, dO tiles], [ring][lse2 of 32 rows, delta of 32 rows], K of the block
  constexpr int STATS = DKV_RING * Tile::PAIR, KEYS = STATS + DKV_RING * 256;
  const int nkb = (p.Nk + BKV - 1) / BKV, per_head = grad_units(p, nkb);
  const int unit = window_unit(p.B * p.Hkv * per_head);
  if (unit < 0) return;
  const int x = unit / per_head;
  int b, hk, rest = unit - x * per_head, block, part, parts;
  window_head(x, p.B, 1, b, hk);
  const int bh = b * p.Hkv + hk;
  const bool sink_block = rest < p.n_sink_blocks * p.bwd_sink_parts;
  if (sink_block) {
    parts = p.bwd_sink_parts;
    block = rest / parts;
    part = rest - block * parts;
  } else {
    parts = p.bwd_parts;
    rest -= p.n_sink_blocks * p.bwd_sink_parts;
    block = rest / parts;
    part = rest - block * parts;
    block += p.n_sink_blocks;
  }
  const WindowEntry e(p, b);
  const Tile w(lds);
  const int j0 = block * BKV, j1 = min(j0 + BKV, e.k_len), G = p.Hq / p.Hkv, col = j0 + w.wave * Tile::COLS + w.l32;
  f32x16 dk[DB], dv[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) dk[db][v] = dv[db][v] = 0.f;
  float ds_unit = 1.f;  // what dK's sums are to be multiplied by: 1 / F
  if (j0 < j1) {
    const WindowQueries seen(p, e, j0, j1);
    const int n_tiles = max(0, seen.end - seen.begin + ROWS - 1) / ROWS;
    const int u0 = (int)((long long)G * n_tiles * part / parts), u1 = (int)((long long)G * n_tiles * (part + 1) / parts);
    if (u0 < u1) {
      float ds_of_p = 1.f;
      if constexpr (GradScale<T>::FOLLOWS) {
        float most_do, most_v;
        largest_squares(p, b, hk, most_do, most_v);
        const float f = grad_factor(most_do, most_v);
        ds_unit = 1.f / f;
        ds_of_p = f * GradScale<T>::P_UNIT;
      }
      const uint32_t q_bytes = (uint32_t)p.q.n * 2, do_bytes = (uint32_t)p.dout.n * 2;
      const uint32_t q_limit = (uint32_t)(seen.end - 1) * q_bytes + Tile::ROWB, do_limit = (uint32_t)(seen.end - 1) * do_bytes + Tile::ROWB;
      // the tile that is asked for next: its head's rows, and the first of them
      int next_row = __builtin_amdgcn_readfirstlane(seen.begin + ROWS * (u0 % n_tiles));
      const int h0 = __builtin_amdgcn_readfirstlane(hk * G + u0 / n_tiles);
      const uint16_t *next_q = gq + (size_t)b * p.q.b + (size_t)h0 * p.q.h, *next_do = gdo + (size_t)b * p.dout.b + (size_t)h0 * p.dout.h;
      const float *next_stats = stats + 2 * ((size_t)b * p.Hq + h0) * p.Nq;
      const uint32_t stats_limit = (uint32_t)p.Nq * 8;  // bytes of a head's, 2^28 at most as its rows are within 2^32
      auto issue = [&](int u) {  // a tile behind the last one reads nothing
        const bool there = u < u1;
        const u32x4 Qres = head_rsrc(next_q, __builtin_amdgcn_readfirstlane(there ? q_limit : 0u));
        const u32x4 Dres = head_rsrc(next_do, __builtin_amdgcn_readfirstlane(there ? do_limit : 0u));
        w.issue(Qres, Dres, next_row, (uint32_t)(u % DKV_RING) * Tile::PAIR, q_bytes, do_bytes);
        if (w.wave == 0) {  // lanes 0..31 lse2 of the rows, lanes 32..63 delta; zeros behind the last query
          const u32x4 Sres = head_rsrc(reinterpret_cast<const uint16_t *>(next_stats), __builtin_amdgcn_readfirstlane(there ? stats_limit : 0u));
          const int row = next_row + w.l32;
          dma_4B_per_lane(Sres, row < seen.end ? (uint32_t)(row + (w.g ? p.Nq : 0)) * 4 : 0xfffffff0u,  // (behind every limit)
                          __builtin_amdgcn_readfirstlane(w.lds_base + STATS + (uint32_t)(u % DKV_RING) * 256));
        }
        next_row += ROWS;
        if (next_row >= seen.end) {
          next_row = seen.begin;
          next_q += p.q.h;
          next_do += p.dout.h;
          next_stats += 2 * (size_t)p.Nq;
        }
      };
      int first = next_row;
      issue(u0);
      issue(u0 + 1);
      u32x4 k[DS], v[DS];  // (k: unused where it stays in LDS)
      const int key = min(col, j1 - 1);
      const size_t kv_head = (size_t)b * p.kv.b + (size_t)hk * p.kv.h;
      uint32_t at_k = 0;
      if constexpr (K_LDS) {  // the wave's own rows, in pieces of 1 KB
        const uint32_t kv_bytes = (uint32_t)p.kv.n * 2, keys = KEYS + w.wave * Tile::COLS * Tile::ROWB;
        const u32x4 Kres = head_rsrc(gk + kv_head, __builtin_amdgcn_readfirstlane((uint32_t)(j1 - 1) * kv_bytes + Tile::ROWB));
        constexpr int PER = 64 / Tile::CH;  // rows of an instruction
        const uint32_t to_lds = __builtin_amdgcn_readfirstlane(w.lds_base + keys);
        const int row0 = __builtin_amdgcn_readfirstlane(j0 + w.wave * Tile::COLS);
#pragma unroll
        for (int it = 0; it < Tile::COLS / PER; ++it) {
          const int row = it * PER + w.lane / Tile::CH, c = (w.lane % Tile::CH) ^ both_swz<D>(row);
          dma_16B_per_lane<true>(Kres, (uint32_t)(w.lane / Tile::CH) * kv_bytes + c * 16, (uint32_t)(row0 + it * PER) * kv_bytes, to_lds + it * 1024);
        }
        at_k = w.second_addr + w.lds_base + keys;
      } else {
        w.operand(gk + kv_head + (size_t)key * p.kv.n, k);
        Tile::arrive(k);
      }
      w.operand(gv + kv_head + (size_t)key * p.kv.n, v);
      // queries that see the column's key, and those that see every key of the wave
      const int from = WindowQueries::first_of(p, e, key), to = col < j1 ? WindowQueries::end_of(p, e, key) : from;
      const int jw0 = __builtin_amdgcn_readfirstlane(j0 + w.wave * Tile::COLS), jw1 = jw0 + Tile::COLS;
      const int from_max = jw1 <= j1 ? WindowQueries::first_of(p, e, jw1 - 1) : INT_MAX;
      const int to_min = jw1 <= p.sinks ? e.q_len : WindowQueries::end_of(p, e, max(jw0, p.sinks));
      // no V for a key that nothing sees: it may hold anything, and dS = P (dP - delta) is zero only for a finite dP
#pragma unroll
      for (int s = 0; s < DS; ++s) v[s] = from < to ? v[s] : u32x4{0, 0, 0, 0};
      Tile::arrive(v);
      const float sc = p.scale_log2e == 0.f ? 1e-30f : p.scale_log2e, unseen = sc < 0.f ? INFINITY : -INFINITY;
      for (int u = u0; u < u1; ++u) {
        if (((u - u0) & 1) == 0) {
          asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
          __syncthreads();  // tiles u and u + 1 (and K) are there, and every wave is done with the two before, whose places
          issue(u + 2);     // the next two take
          issue(u + 3);
        }
        // S, dP, dV, dK; exponentials and dS beside them from dP on
        constexpr int PH = Tile::PH, N = 4 * DS;
        constexpr int RING = D == 128 ? 4 : 8, STAT_AHEAD = 3;  // pairs of lse2, then of delta, on their way
        f32x16 s, dp;
        u32x4 pp[2], ds[2], a[RA], second[RA];
        f32x2 row_stat[RING];
        const typename Tile::Places at(w, w.lds_base + (uint32_t)(u % DKV_RING) * Tile::PAIR);
        uint32_t at_second = at_k;
        asm volatile("" : "+v"(at_second));
        const float *const row_stats = reinterpret_cast<const float *>(lds + STATS + (u % DKV_RING) * 256) + 8 * w.g;
        auto fetch = [&](auto q) {
          constexpr int i = q;
          if constexpr (i < DS) {
            a[i % RA] = Tile::rows_of(at.rows, 0, i);
            if constexpr (K_LDS) second[i % RA] = Tile::rows_of(at_second, 0, i);
          } else if constexpr (i < 2 * DS) {
            a[i % RA] = Tile::rows_of(at.rows, Tile::TILE, i - DS);
          } else {
            constexpr int n = (i - 2 * DS) % DS;
            a[i % RA] = Tile::cols_of(at.cols, i < 3 * DS ? Tile::TILE : 0, n / DB, n % DB);
          }
        };
        static_unroll<AHEAD>(fetch);
        static_unroll<N>([&](auto gap) {
          constexpr int g = gap;
          if constexpr (g + AHEAD < N) fetch(std::integral_constant<int, g + AHEAD>{});
          static_unroll<16>([&](auto r) {
            constexpr auto use_of = [](int x) { return PH + (x < 8 ? Tile::exp_gap(x) : Tile::ds_gap(x % 8)); };
            constexpr int pair = r % 8, use = use_of(r);
            static_assert(r < RING || use_of(r - RING) < use - STAT_AHEAD, "the place of a pair of rows is free again");
            if constexpr (use - STAT_AHEAD == g)
              row_stat[r % RING] = *reinterpret_cast<const f32x2 *>(row_stats + (r < 8 ? 0 : 32) + 16 * (pair >> 2) + 2 * (pair & 3));
          });
          if constexpr (g < DS) {
            if constexpr (K_LDS) mfma_gap<T, true, g == 0>(s, a[g % RA], second[g % RA]);
            else mfma_gap<T, true, g == 0>(s, a[g % RA], k[g]);
          } else if constexpr (g < 2 * DS) {
            mfma_gap<T, true, g == DS>(dp, a[g % RA], v[g - DS]);
          } else if constexpr (g < 3 * DS) {
            mfma_gap<T, false, false>(dv[(g - 2 * DS) % DB], a[g % RA], pp[(g - 2 * DS) / DB]);
          } else {
            mfma_gap<T, false, false>(dk[(g - 3 * DS) % DB], a[g % RA], ds[(g - 3 * DS) / DB]);
          }
          if constexpr (g == PH) {
            settle<true>(s);
            if (!(first >= from_max && first + ROWS <= to_min)) {  // queries that do not see the column's key
              const int begin = first + 8 * w.g - from;
              const uint32_t span = (uint32_t)max(to - from, 0);
#pragma unroll
              for (int n = 0; n < 16; ++n) s[n] = (uint32_t)(begin + 16 * (n >> 3) + (n & 7)) < span ? s[n] : unseen;
            }
          }
          if constexpr (g == PH + Tile::EXP_GAPS) settle<true>(dp);
          static_unroll<Tile::UNITS>([&](auto u_) {
            constexpr int n = 2 * u_;
            if constexpr (PH + Tile::exp_gap(u_) == g) {
              const f32x2 lse2 = row_stat[u_ % RING];
              s[n] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n], sc, -lse2[0]));
              s[n + 1] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n + 1], sc, -lse2[1]));
              pp[n >> 3][(n >> 1) & 3] = T::pack(s[n], s[n + 1]);
            }
            if constexpr (PH + Tile::ds_gap(u_) == g) {
              const f32x2 dl = row_stat[(8 + u_) % RING];
              ds[n >> 3][(n >> 1) & 3] = T::pack(s[n] * ds_factor(dp[n], ds_of_p, dl[0]), s[n + 1] * ds_factor(dp[n + 1], ds_of_p, dl[1]));
            }
          });
          __builtin_amdgcn_sched_barrier(0);
        });
        first += ROWS;
        if (first >= seen.end) first = seen.begin;
      }
      asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        settle<false>(dk[db]);
        settle<false>(dv[db]);
      }
    }
  }
  if (col >= p.Nk) return;
  if (parts > 1) {
    // sums of a part: [part][dk, dv][key rows][D], the blocks with sinks behind all others
    const size_t rows = (size_t)p.B * p.Hkv * p.Nk, sink_rows = (size_t)p.B * p.Hkv * p.n_sink_blocks * BKV;
    const size_t before = p.bwd_parts > 1 && sink_block ? (size_t)p.bwd_parts * 2 * rows : 0;
    const size_t n = sink_block ? sink_rows : rows;
    const size_t row = sink_block ? (size_t)bh * p.n_sink_blocks * BKV + col : (size_t)bh * p.Nk + col;
    float *const to_k = p.part_dkv + (before + (size_t)(2 * part) * n + row) * D + 4 * w.g, *const to_v = to_k + n * D;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        *reinterpret_cast<f32x4 *>(to_k + 32 * db + 8 * a) =
            f32x4{dk[db][4 * a] * ds_unit, dk[db][4 * a + 1] * ds_unit, dk[db][4 * a + 2] * ds_unit, dk[db][4 * a + 3] * ds_unit};
        *reinterpret_cast<f32x4 *>(to_v + 32 * db + 8 * a) = f32x4{dv[db][4 * a], dv[db][4 * a + 1], dv[db][4 * a + 2], dv[db][4 * a + 3]};
      }
    return;
  }
  const bool there = col < j1;  // rows behind the keys: zeros, their columns repeat the last key
  const size_t at = (size_t)b * p.dkv.b + (size_t)hk * p.dkv.h + (size_t)col * p.dkv.n;
  Tile::store(dk, p.scale * ds_unit, there, gdk + at, w.g);
  Tile::store(dv, GradScale<T>::P_UNIT, there, gdv + at, w.g);
}

// Sums of the parts of every key's row, and behind them of every query's, in the order of the parts, rounded once.
template <int D, typename T>
__global__ __launch_bounds__(256) void window_attn_grad_sum_kernel(uint16_t *__restrict__ gdq, uint16_t *__restrict__ gdk,
                                                                   uint16_t *__restrict__ gdv, const WindowDims p) {
  using Tile = DkvTile<D, T>;
  constexpr int LANES = D / 8, BKV = Tile::BLOCK;
  const size_t rows = (size_t)p.B * p.Hkv * p.Nk;
  // with whole blocks beside those with sinks, only the rows of the latter are left to be added up
  const int cut = p.bwd_parts > 1 ? p.Nk : p.bwd_sink_parts > 1 ? min(p.Nk, p.n_sink_blocks * BKV) : 0;
  const long long item = (long long)blockIdx.x * (256 / LANES) + threadIdx.x / LANES, of_keys = 2ll * p.B * p.Hkv * cut;
  const int c = 8 * (threadIdx.x % LANES);
  const float *from;
  size_t step;
  int parts, b;
  uint16_t *to;
  float f = p.scale;
  bool there;
  if (item < of_keys) {
    const int which = (int)(item & 1), key = (int)((item >> 1) % cut), bh = (int)((item >> 1) / cut), hk = bh % p.Hkv;
    const bool sink = key < p.n_sink_blocks * BKV;
    const size_t n = sink ? (size_t)p.B * p.Hkv * p.n_sink_blocks * BKV : rows;
    const size_t first = sink && p.bwd_parts > 1 ? (size_t)p.bwd_parts * 2 * rows : 0;
    const size_t row = sink ? (size_t)bh * p.n_sink_blocks * BKV + key : (size_t)bh * p.Nk + key;
    from = p.part_dkv + (first + which * n + row) * D;
    step = 2 * n * D;
    parts = sink ? p.bwd_sink_parts : p.bwd_parts;
    b = bh / p.Hkv;
    to = (which ? gdv : gdk) + (size_t)b * p.dkv.b + (size_t)hk * p.dkv.h + (size_t)key * p.dkv.n;
    if (which) f = GradScale<T>::P_UNIT;
    there = key < (p.k_len ? min(p.k_len[b], p.Nk) : p.Nk);
  } else {
    const long long row = item - of_keys, n = (long long)p.B * p.Hq * p.Nq;
    if (p.dq_parts == 1 || row >= n) return;
    const int i = (int)(row % p.Nq), bh = (int)(row / p.Nq);
    from = p.part_dq + (size_t)row * D;
    step = (size_t)n * D;
    parts = p.dq_parts;
    b = bh / p.Hq;
    to = gdq + (size_t)b * p.dq.b + (size_t)(bh % p.Hq) * p.dq.h + (size_t)i * p.dq.n;
    there = i < (p.q_len ? min(p.q_len[b], p.Nq) : p.Nq);
  }
  float x[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = 0.f;
#pragma unroll 4
  for (int s = 0; s < parts; ++s, from += step) {
    const f32x4 u = *reinterpret_cast<const f32x4 *>(from + c), v = *reinterpret_cast<const f32x4 *>(from + c + 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] += u[j], x[4 + j] += v[j];
  }
  u32x4 out;
#pragma unroll
  for (int j = 0; j < 4; ++j) out[j] = there ? T::pack(x[2 * j] * f, x[2 * j + 1] * f) : 0u;
  *reinterpret_cast<u32x4 *>(to + c) = out;
}

}  // namespace calibatt_dev
