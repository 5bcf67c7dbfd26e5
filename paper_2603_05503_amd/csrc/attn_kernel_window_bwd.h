// Gradients of attention in a window (attn_kernel_window.h).
//
// With P = exp(scale S - lse) over the visible pairs, S = Q K^T, dP = dO V^T, delta = rowsum(dO * O):
//   dS = P * (dP - delta),  dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO.
// Two kernels, each of which forms S and dP once: one owns queries and goes over their keys (dQ, and delta on the way),
// one owns keys and goes over the queries that see them, of all query heads that share them (dK, dV).  Seven products
// instead of five, but no sum goes through atomics: the same inputs give the same bits.
//
// Both are the same shape.  A wave owns NB blocks of 32 columns (its queries, or its keys) as second operands in
// registers; tiles of 64 rows of two matrices (K and V, or Q and dO) pass through LDS, read row-wise for S^T and dP^T
// (first operand: rows of the tile) and transposed for the products that add up, whose second operands are P and dS as
// they lie in registers.  With NB = 2 a wave holds 512 registers and is alone on its SIMD, every LDS read feeds two MFMAs,
// and it hides its vector work behind its own MFMAs: exponentials beside dP, dS beside the products with P.
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

// fp16 has few exponents: probabilities are kept times 2^15, which takes 1 to 32768, and dS times 2^4 (up to 2^12 with its
// precision down to 2^-18); bf16 needs neither.
template <typename T> struct GradScale { static constexpr float P_LOG2 = 0.f, DS = 1.f; };
template <> struct GradScale<F16> { static constexpr float P_LOG2 = 15.f, DS = 16.f; };

template <int D, int NB, typename T>
struct GradTile {
  static constexpr int NT = 256, ROWS = 64, ROWB = D * 2, CH = D / 8, DS = D / 16, DB = D / 32;
  static constexpr int TILE = ROWS * ROWB;           // bytes of one matrix's tile
  static constexpr int RPI = NT / CH, ITERS = ROWS / RPI;
  static_assert(RPI % 16 == 0, "the swizzle of an instruction's rows is the same for every one");
  static constexpr int LDS_BYTES = 4 * TILE;         // two buffers of two matrices
  static constexpr int COLS = NB * 32;               // columns of a wave
  static constexpr float P_UNIT = GradScale<T>::P_LOG2 == 0.f ? 1.f : 1.f / 32768.f;   // what P_LOG2 stands for
  static constexpr float DS_OF_P = GradScale<T>::DS * P_UNIT;                          // factor of dP - delta beside P as kept

  int tid, lane, wave, l32, g;
  uint32_t row_addr;     // row-wise reads: chunk column s at row_addr ^ (s << 5), 32 rows on at + 32 * ROWB
  uint32_t col_addr[2];  // transposed reads: d block db at col_addr[t] ^ (db << 6), slab j at + 16 j * ROWB
  uint32_t lds_wave;

  __device__ __forceinline__ explicit GradTile(char *lds) {
    tid = threadIdx.x;
    lane = tid & 63;
    wave = tid >> 6;
    l32 = lane & 31;
    g = lane >> 5;
    const uint32_t base = (uint32_t)(uintptr_t)(LDS_PTR(char))lds;
    lds_wave = __builtin_amdgcn_readfirstlane(base + wave * 1024);
    const int row = (l32 & 0x13) | ((l32 & 4) << 1) | ((l32 & 8) >> 1);  // so that a lane's eight values are of consecutive rows
    row_addr = row * ROWB + ((g ^ both_swz<D>(row)) << 4);
    const int L16 = lane & 15, blk = lane >> 4;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int r = 8 * (blk >> 1) + (L16 >> 2) + 4 * t;
      col_addr[t] = r * ROWB + (((2 * (blk & 1) + ((L16 & 3) >> 1)) ^ both_swz<D>(r)) << 4) + (L16 & 1) * 8;
    }
  }
  // rows [row0, row0 + 64) of a matrix into the tile at LDS byte `at`
  __device__ __forceinline__ void issue(const u32x4 rsrc, int row0, uint32_t at, uint32_t row_bytes) const {
    const int row = tid / CH, c = (tid % CH) ^ both_swz<D>(row);
    const uint32_t voff = row * row_bytes + c * 16;
#pragma unroll
    for (int it = 0; it < ITERS; ++it)
      dma_16B_per_lane<true>(rsrc, voff, (uint32_t)(row0 + it * RPI) * row_bytes, lds_wave + at + it * NT * 16);
  }
  // a column's D elements as second operand
  __device__ __forceinline__ void operand(const uint16_t *row, u32x4 (&x)[DS]) const {
#pragma unroll
    for (int s = 0; s < DS; ++s) x[s] = *reinterpret_cast<const u32x4 *>(row + 16 * s + 8 * g);
  }
  // out[c] = (rows [32 half, 32 half + 32) of the tile) . columns
  __device__ __forceinline__ void products(const char *tile, int half, const u32x4 (&x)[NB][DS], f32x16 (&out)[NB]) const {
#pragma unroll
    for (int c = 0; c < NB; ++c)
#pragma unroll
      for (int v = 0; v < 16; ++v) out[c][v] = 0.f;
#pragma unroll
    for (int s = 0; s < DS; ++s) {
      const u32x4 a = *reinterpret_cast<const u32x4 *>(tile + half * 32 * ROWB + (row_addr ^ (s << 5)));
#pragma unroll
      for (int c = 0; c < NB; ++c) out[c] = T::mfma(a, x[c][s], out[c]);
    }
  }
  // sum[c][db] += (rows [32 half, + 32) of the tile)^T . weights, weights as packed pairs of the rows' values
  __device__ __forceinline__ void add(const char *tile, int half, const uint32_t (&w)[NB][8], f32x16 (&sum)[NB][DB]) const {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const char *const at = tile + (half * 32 + 16 * j) * ROWB;
        const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(at + (col_addr[0] ^ (db << 6)))));
        const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(at + (col_addr[1] ^ (db << 6)))));
        const u32x4 a = {lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
        for (int c = 0; c < NB; ++c) sum[c][db] = T::mfma(a, u32x4{w[c][4 * j], w[c][4 * j + 1], w[c][4 * j + 2], w[c][4 * j + 3]}, sum[c][db]);
      }
  }
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

// ---- dQ -----------------------------------------------------------------------------------------------------
template <int D, int NB, typename T>
__global__ __launch_bounds__(256, NB == 2 ? 1 : 2) void window_attn_dq_kernel(
    const uint16_t *__restrict__ gdo, const uint16_t *__restrict__ gq, const uint16_t *__restrict__ gk,
    const uint16_t *__restrict__ gv, const uint16_t *__restrict__ gout, const float *__restrict__ lse,
    uint16_t *__restrict__ gdq, float *__restrict__ delta, const WindowDims p) {
  using Tile = GradTile<D, NB, T>;
  using Tiles = WindowTiles<64>;
  constexpr int BQ = 4 * Tile::COLS, DS = Tile::DS, DB = Tile::DB;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int nbq = (p.Nq + BQ - 1) / BQ;
  const int unit = window_unit(p.B * p.Hq * nbq);
  if (unit < 0) return;
  const int bh = unit / nbq, r = nbq - 1 - (unit - bh * nbq), b = bh / p.Hq, h = bh - b * p.Hq;
  const WindowEntry e(p, b);
  const Tile w(lds);
  const int i0 = r * BQ, i1 = min(i0 + BQ, e.q_len);
  const size_t row0 = (size_t)bh * p.Nq;
  uint16_t *const dq_head = gdq + (size_t)b * p.dq.b + (size_t)h * p.dq.h;
  f32x16 dq[NB][DB];
  int col[NB];
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    col[c] = i0 + w.wave * Tile::COLS + 32 * c + w.l32;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) dq[c][db][v] = 0.f;
  }
  if (i0 < i1) {
    const Tiles tiles(p, e, i0, i1);
    const size_t kv_head = (size_t)b * p.kv.b + (size_t)(h / (p.Hq / p.Hkv)) * p.kv.h;
    const uint32_t row_bytes = (uint32_t)p.kv.n * 2;
    u32x4 Kres = head_rsrc(gk + kv_head, 0), Vres = head_rsrc(gv + kv_head, 0);
    auto issue = [&](int t) {  // a tile behind the last one reads nothing
      const int end = t < tiles.n ? tiles.end(t) : 0;
      Kres[2] = Vres[2] = __builtin_amdgcn_readfirstlane(end > 0 ? (uint32_t)(end - 1) * row_bytes + Tile::ROWB : 0u);
      const int first = __builtin_amdgcn_readfirstlane(t < tiles.n ? tiles.row(t) : 0);
      const uint32_t at = (t & 1) * 2 * Tile::TILE;
      w.issue(Kres, first, at, row_bytes);
      w.issue(Vres, first, at + Tile::TILE, row_bytes);
    };
    issue(0);
    u32x4 q[NB][DS], dout[NB][DS];
    float lse2[NB], dl[NB];
    int lo[NB], hi[NB];
#pragma unroll
    for (int c = 0; c < NB; ++c) {
      const int row = min(col[c], i1 - 1);  // columns behind the last query: its values, not stored
      e.interval(p, row, lo[c], hi[c]);
      w.operand(gq + (size_t)b * p.q.b + (size_t)h * p.q.h + (size_t)row * p.q.n, q[c]);
      w.operand(gdo + (size_t)b * p.dout.b + (size_t)h * p.dout.h + (size_t)row * p.dout.n, dout[c]);
      u32x4 o[DS];
      w.operand(gout + (size_t)b * p.out.b + (size_t)h * p.out.h + (size_t)row * p.out.n, o);
      const float z = lse[row0 + row];
      float sum = 0.f;
#pragma unroll
      for (int s = 0; s < DS; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t x = dout[c][s][i], y = o[s][i];
          float x2[2], y2[2];
          T::unpack(x, x2);
          T::unpack(y, y2);
          sum = __builtin_fmaf(x2[0], y2[0], sum);
          sum = __builtin_fmaf(x2[1], y2[1], sum);
        }
      dl[c] = sum_with_other_half(sum);
      // a query that sees nothing: exponents of -inf
      lse2[c] = z == -INFINITY ? INFINITY : z * 1.4426950408889634f - GradScale<T>::P_LOG2;
      if (w.g == 0 && col[c] < i1) delta[row0 + col[c]] = dl[c];
      dl[c] *= Tile::DS_OF_P;
    }
    const float sc = p.scale_log2e;
    for (int t = 0; t < tiles.n; ++t) {
      asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
      __syncthreads();  // tile t is there, and every wave is done with tile t - 1
      issue(t + 1);
      const char *const kt = lds + (t & 1) * 2 * Tile::TILE, *const vt = kt + Tile::TILE;
      const bool whole = tiles.whole(t);
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        f32x16 s[NB], dp[NB];
        uint32_t ds[NB][8];
        w.products(kt, half, q, s);
        w.products(vt, half, dout, dp);
#pragma unroll
        for (int c = 0; c < NB; ++c) {
          if (!whole) {
            int a, z;
            tile_interval(tiles, t, lo[c], hi[c], a, z);
            const int first = tiles.row(t) + 32 * half + 8 * w.g - a;
            const uint32_t span = (uint32_t)max(z - a, 0);
#pragma unroll
            for (int v = 0; v < 16; ++v) s[c][v] = (uint32_t)(first + 16 * (v >> 3) + (v & 7)) < span ? s[c][v] * sc : -INFINITY;
          } else {
#pragma unroll
            for (int v = 0; v < 16; ++v) s[c][v] *= sc;
          }
#pragma unroll
          for (int v = 0; v < 16; v += 2) {
            const float p0 = __builtin_amdgcn_exp2f(s[c][v] - lse2[c]), p1 = __builtin_amdgcn_exp2f(s[c][v + 1] - lse2[c]);
            ds[c][v >> 1] = T::pack(p0 * __builtin_fmaf(dp[c][v], Tile::DS_OF_P, -dl[c]),
                                    p1 * __builtin_fmaf(dp[c][v + 1], Tile::DS_OF_P, -dl[c]));
          }
        }
        w.add(kt, half, ds, dq);
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
  }
  const float f = p.scale / GradScale<T>::DS;
#pragma unroll
  for (int c = 0; c < NB; ++c)
    if (col[c] < p.Nq) Tile::store(dq[c], f, col[c] < i1, dq_head + (size_t)col[c] * p.dq.n, w.g);
}

// ---- dK, dV -------------------------------------------------------------------------------------------------
// The queries that see keys [j0, j1) (j1 within k_len): of the window between two positions, of the sinks all from the
// first on.
struct WindowQueries {
  int begin, end;
  static __device__ __forceinline__ int floor_div(int x, int y) {
    const int f = x / y;
    return f - (f * y > x);
  }
  // first query that sees key j, last + 1 that does
  static __device__ __forceinline__ int first_of(const WindowDims &p, const WindowEntry &e, int j) {
    if (p.right < 0) return 0;
    const long long pos = ((long long)j / p.frame - p.right) * p.frame - e.start;
    return (int)min(max(pos, 0ll), (long long)e.q_len);
  }
  static __device__ __forceinline__ int end_of(const WindowDims &p, const WindowEntry &e, int j) {
    if (p.left < 0 || j < p.sinks) return e.q_len;
    const long long pos = ((long long)j / p.frame + p.left + 1) * p.frame - e.start;
    return (int)min(max(pos, 0ll), (long long)e.q_len);
  }
  __device__ __forceinline__ WindowQueries(const WindowDims &p, const WindowEntry &e, int j0, int j1) {
    begin = first_of(p, e, j0);
    end = j0 < p.sinks ? e.q_len : end_of(p, e, j1 - 1);
  }
};

// Units of work of one key head: the blocks that hold sinks in bwd_sink_parts parts each, the others in bwd_parts.
__device__ __forceinline__ int grad_units(const WindowDims &p, int n_blocks) {
  return p.n_sink_blocks * p.bwd_sink_parts + (n_blocks - p.n_sink_blocks) * p.bwd_parts;
}

template <int D, int NB, typename T>
__global__ __launch_bounds__(256, NB == 2 ? 1 : 2) void window_attn_dkv_kernel(
    const uint16_t *__restrict__ gdo, const uint16_t *__restrict__ gq, const uint16_t *__restrict__ gk,
    const uint16_t *__restrict__ gv, const float *__restrict__ lse, const float *__restrict__ delta,
    uint16_t *__restrict__ gdk, uint16_t *__restrict__ gdv, const WindowDims p) {
  using Tile = GradTile<D, NB, T>;
  constexpr int BKV = 4 * Tile::COLS, DS = Tile::DS, DB = Tile::DB;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  float *const stats = reinterpret_cast<float *>(lds + Tile::LDS_BYTES);  // [2 buffers][lse2 of 64 rows, delta of 64 rows]
  const int nkb = (p.Nk + BKV - 1) / BKV, per_head = grad_units(p, nkb);
  const int unit = window_unit(p.B * p.Hkv * per_head);
  if (unit < 0) return;
  const int bh = unit / per_head, b = bh / p.Hkv, hk = bh - b * p.Hkv;
  int rest = unit - bh * per_head, block, part, parts;
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
  const int j0 = block * BKV, j1 = min(j0 + BKV, e.k_len), G = p.Hq / p.Hkv;
  f32x16 dk[NB][DB], dv[NB][DB];
  int col[NB];
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    col[c] = j0 + w.wave * Tile::COLS + 32 * c + w.l32;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) dk[c][db][v] = dv[c][db][v] = 0.f;
  }
  if (j0 < j1) {
    const WindowQueries seen(p, e, j0, j1);
    const int n_tiles = max(0, seen.end - seen.begin + 63) / 64;
    const int u0 = (int)((long long)G * n_tiles * part / parts), u1 = (int)((long long)G * n_tiles * (part + 1) / parts);
    if (u0 < u1) {
      const uint32_t q_bytes = (uint32_t)p.q.n * 2, do_bytes = (uint32_t)p.dout.n * 2;
      const uint32_t q_limit = (uint32_t)(seen.end - 1) * q_bytes + Tile::ROWB, do_limit = (uint32_t)(seen.end - 1) * do_bytes + Tile::ROWB;
      float stat = 0.f;  // of row tid & 63 of the tile that is on its way: threads 0..63 lse, 64..127 delta
      auto issue = [&](int u) {
        const int h = hk * G + u / n_tiles, first = seen.begin + 64 * (u % n_tiles), at = (u & 1) * 2 * Tile::TILE;
        const bool there = u < u1;
        const u32x4 Qres = head_rsrc(gq + (size_t)b * p.q.b + (size_t)(there ? h : 0) * p.q.h, there ? q_limit : 0u);
        const u32x4 Dres = head_rsrc(gdo + (size_t)b * p.dout.b + (size_t)(there ? h : 0) * p.dout.h, there ? do_limit : 0u);
        w.issue(Qres, __builtin_amdgcn_readfirstlane(first), at, q_bytes);
        w.issue(Dres, __builtin_amdgcn_readfirstlane(first), at + Tile::TILE, do_bytes);
        if (w.wave < 2) {
          const int row = first + w.lane;
          stat = w.wave == 0 ? INFINITY : 0.f;  // a row that is not there, or sees nothing: exponents of -inf
          if (there && row < seen.end) {
            const size_t from = ((size_t)b * p.Hq + h) * p.Nq + row;
            if (w.wave == 0) {
              const float z = lse[from];
              if (z != -INFINITY) stat = z * 1.4426950408889634f - GradScale<T>::P_LOG2;
            } else {
              stat = delta[from] * Tile::DS_OF_P;
            }
          }
        }
      };
      auto leave_stat = [&](int u) {
        if (w.wave < 2) stats[(u & 1) * 128 + w.wave * 64 + w.lane] = stat;
      };
      issue(u0);
      u32x4 k[NB][DS], v[NB][DS];
      int from[NB], to[NB];  // queries that see the column's key
#pragma unroll
      for (int c = 0; c < NB; ++c) {
        const int row = min(col[c], j1 - 1);
        w.operand(gk + (size_t)b * p.kv.b + (size_t)hk * p.kv.h + (size_t)row * p.kv.n, k[c]);
        w.operand(gv + (size_t)b * p.kv.b + (size_t)hk * p.kv.h + (size_t)row * p.kv.n, v[c]);
        from[c] = WindowQueries::first_of(p, e, row);
        to[c] = col[c] < j1 ? WindowQueries::end_of(p, e, row) : from[c];
      }
      // every key of the wave is seen by the queries [from_max, to_min)
      const int jw0 = j0 + __builtin_amdgcn_readfirstlane(w.wave) * Tile::COLS, jw1 = jw0 + Tile::COLS;
      const int from_max = jw1 <= j1 ? WindowQueries::first_of(p, e, jw1 - 1) : INT_MAX;
      const int to_min = jw1 <= p.sinks ? e.q_len : WindowQueries::end_of(p, e, max(jw0, p.sinks));
      leave_stat(u0);
      const float sc = p.scale_log2e;
      for (int u = u0; u < u1; ++u) {
        asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
        __syncthreads();  // tile u and its rows' lse and delta are there, and every wave is done with tile u - 1
        issue(u + 1);
        const char *const qt = lds + (u & 1) * 2 * Tile::TILE, *const dt = qt + Tile::TILE;
        const float *const st = stats + (u & 1) * 128;
        const int first = seen.begin + 64 * (u % n_tiles);
        const bool whole = first >= from_max && first + 64 <= to_min;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          f32x16 s[NB], dp[NB];
          uint32_t pp[NB][8], ds[NB][8];
          float lse2[16], dl[16];
          w.products(qt, half, k, s);
          w.products(dt, half, v, dp);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int at = 32 * half + 16 * (i >> 1) + 8 * w.g + 4 * (i & 1);
            const f32x4 x = *reinterpret_cast<const f32x4 *>(st + at), y = *reinterpret_cast<const f32x4 *>(st + 64 + at);
#pragma unroll
            for (int n = 0; n < 4; ++n) lse2[4 * i + n] = x[n], dl[4 * i + n] = y[n];
          }
#pragma unroll
          for (int c = 0; c < NB; ++c) {
            if (!whole) {
              const int at = first + 32 * half + 8 * w.g - from[c];
              const uint32_t span = (uint32_t)max(to[c] - from[c], 0);
#pragma unroll
              for (int n = 0; n < 16; ++n) s[c][n] = (uint32_t)(at + 16 * (n >> 3) + (n & 7)) < span ? s[c][n] * sc : -INFINITY;
            } else {
#pragma unroll
              for (int n = 0; n < 16; ++n) s[c][n] *= sc;
            }
#pragma unroll
            for (int n = 0; n < 16; n += 2) {
              const float p0 = __builtin_amdgcn_exp2f(s[c][n] - lse2[n]), p1 = __builtin_amdgcn_exp2f(s[c][n + 1] - lse2[n + 1]);
              pp[c][n >> 1] = T::pack(p0, p1);
              ds[c][n >> 1] = T::pack(p0 * __builtin_fmaf(dp[c][n], Tile::DS_OF_P, -dl[n]),
                                      p1 * __builtin_fmaf(dp[c][n + 1], Tile::DS_OF_P, -dl[n + 1]));
            }
          }
          w.add(dt, half, pp, dv);
          w.add(qt, half, ds, dk);
        }
        leave_stat(u + 1);
      }
      asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
    }
  }
  const float fk = p.scale / GradScale<T>::DS, fv = Tile::P_UNIT;
  if (parts > 1) {
    // sums of a part: [part][dk, dv][key rows][D], the blocks with sinks behind all others
    const size_t rows = (size_t)p.B * p.Hkv * p.Nk, sink_rows = (size_t)p.B * p.Hkv * p.n_sink_blocks * BKV;
    const size_t first = p.bwd_parts > 1 && sink_block ? (size_t)p.bwd_parts * 2 * rows : 0;
    const size_t n = sink_block ? sink_rows : rows;
#pragma unroll
    for (int c = 0; c < NB; ++c)
      if (col[c] < p.Nk) {
        const size_t row = sink_block ? (size_t)bh * p.n_sink_blocks * BKV + col[c] : (size_t)bh * p.Nk + col[c];
        float *const to_k = p.part_dkv + (first + (size_t)(2 * part) * n + row) * D + 4 * w.g, *const to_v = to_k + n * D;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int a = 0; a < 4; ++a) {
            *reinterpret_cast<f32x4 *>(to_k + 32 * db + 8 * a) = f32x4{dk[c][db][4 * a], dk[c][db][4 * a + 1], dk[c][db][4 * a + 2], dk[c][db][4 * a + 3]};
            *reinterpret_cast<f32x4 *>(to_v + 32 * db + 8 * a) = f32x4{dv[c][db][4 * a], dv[c][db][4 * a + 1], dv[c][db][4 * a + 2], dv[c][db][4 * a + 3]};
          }
      }
    return;
  }
#pragma unroll
  for (int c = 0; c < NB; ++c)
    if (col[c] < p.Nk) {
      const bool there = col[c] < j1;  // rows behind the keys: zeros, their columns repeat the last key
      const size_t at = (size_t)b * p.dkv.b + (size_t)hk * p.dkv.h + (size_t)col[c] * p.dkv.n;
      Tile::store(dk[c], fk, there, gdk + at, w.g);
      Tile::store(dv[c], fv, there, gdv + at, w.g);
    }
}

// Sums of the parts of every key's row, in the order of the parts, rounded once.
template <int D, int NB, typename T>
__global__ __launch_bounds__(256) void window_attn_dkv_sum_kernel(uint16_t *__restrict__ gdk, uint16_t *__restrict__ gdv,
                                                                  const WindowDims p) {
  using Tile = GradTile<D, NB, T>;
  constexpr int LANES = D / 8, BKV = 4 * Tile::COLS;
  const size_t rows = (size_t)p.B * p.Hkv * p.Nk;
  // with whole blocks beside those with sinks, only the rows of the latter are left to be added up
  const int cut = p.bwd_parts > 1 ? p.Nk : min(p.Nk, p.n_sink_blocks * BKV);
  const long long item = (long long)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  if (item >= 2ll * p.B * p.Hkv * cut) return;
  const int which = (int)(item & 1), key = (int)((item >> 1) % cut), bh = (int)((item >> 1) / cut);
  const bool sink = key < p.n_sink_blocks * BKV;
  const size_t n = sink ? (size_t)p.B * p.Hkv * p.n_sink_blocks * BKV : rows;
  const size_t first = sink && p.bwd_parts > 1 ? (size_t)p.bwd_parts * 2 * rows : 0;
  const size_t row = sink ? (size_t)bh * p.n_sink_blocks * BKV + key : (size_t)bh * p.Nk + key;
  const int parts = sink ? p.bwd_sink_parts : p.bwd_parts, c = 8 * (threadIdx.x % LANES);
  const float *from = p.part_dkv + (first + which * n + row) * D + c;
  float x[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = 0.f;
#pragma unroll 4
  for (int s = 0; s < parts; ++s, from += 2 * n * D) {
    const f32x4 u = *reinterpret_cast<const f32x4 *>(from), v = *reinterpret_cast<const f32x4 *>(from + 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] += u[j], x[4 + j] += v[j];
  }
  const int b = bh / p.Hkv, hk = bh - b * p.Hkv;
  const WindowEntry e(p, b);
  const float f = which ? Tile::P_UNIT : p.scale / GradScale<T>::DS;
  u32x4 out;
#pragma unroll
  for (int j = 0; j < 4; ++j) out[j] = key < e.k_len ? T::pack(x[2 * j] * f, x[2 * j + 1] * f) : 0u;
  uint16_t *const to = which ? gdv : gdk;
  *reinterpret_cast<u32x4 *>(to + (size_t)b * p.dkv.b + (size_t)hk * p.dkv.h + (size_t)key * p.dkv.n + c) = out;
}

}  // namespace calibatt_dev
