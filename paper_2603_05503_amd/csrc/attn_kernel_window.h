// Attention in a window, with a few first keys that stay visible, forward.
//
// A query at position p is in frame f = floor(p / frame) and sees the keys of frames f - left .. f + right, and the
// first `sinks` keys as far as they are not ahead of that: [0, min(sinks, hi)) and [lo, hi) with
//   lo = max(0, (f - left) frame),  hi = min(k_len, (f + right + 1) frame)     (left, right < 0: 0 and k_len)
// out = softmax(scale q K^T) V over them, zeros where there is none; lse = log of the sum of exponentials, -inf there.
// A block of queries needs the keys of two ranges, the sinks' [0, s_end) and the window's [w_begin, w_end), which meet
// and never overlap: w_begin >= sinks.  So every tile of keys needs one interval per query for its mask, and tiles
// inside all of a block's intervals none.  Tiles start at the range and not at multiples of their size, and the buffer
// descriptors end with the range: a key that no query of the block sees is not read, whatever it holds.
#pragma once
#include <limits.h>

#include "attn_kernel_il.h"

namespace calibatt_dev {

struct WindowDims {
  int B, Hq, Hkv, Nq, Nk;
  int left, right, sinks, frame, offset;
  const int32_t *q_start, *q_len, *k_len;  // per batch entry, or NULL: offset, Nq, Nk
  float scale, scale_log2e;
  Strides q, kv, out;
  int parts;                               // pieces that a block's tiles are cut into
  float *part_rows, *part_ml;              // [parts][B Hq Nq][D] sums and [parts][B Hq Nq][2] references and row sums
  int dq_parts, bwd_parts, bwd_sink_parts, n_sink_blocks;  // of the gradients, see attn_kernel_window_bwd.h
  float *part_dq, *part_dkv;
  float *sizes;                            // [B Hkv][do_slots + v_slots], fp16: see GradScale
  int do_slots, v_slots;
  Strides dout, dq, dkv;
};

// One batch entry's lengths and the intervals of its queries.
struct WindowEntry {
  int start, q_len, k_len;
  __device__ __forceinline__ WindowEntry(const WindowDims &p, int b) {
    // positions within 2^30 either way: differences and sums with lengths stay in 32 bits
    start = __builtin_amdgcn_readfirstlane(min(max(p.q_start ? p.q_start[b] : p.offset, -(1 << 30)), 1 << 30));
    q_len = __builtin_amdgcn_readfirstlane(p.q_len ? min(max(p.q_len[b], 0), p.Nq) : p.Nq);
    k_len = __builtin_amdgcn_readfirstlane(p.k_len ? min(max(p.k_len[b], 0), p.Nk) : p.Nk);
  }
  // [lo, hi) of query i
  __device__ __forceinline__ void interval(const WindowDims &p, int i, int &lo, int &hi) const {
    const int pos = start + i;
    int f = pos;
    if (p.frame > 1) {
      f = pos / p.frame;
      f -= f * p.frame > pos;  // towards minus infinity
    }
    const long long l = ((long long)f - p.left) * p.frame, h = ((long long)f + p.right + 1) * p.frame;
    lo = p.left < 0 ? 0 : (int)min(max(l, 0ll), (long long)INT_MAX);
    hi = p.right < 0 ? k_len : (int)min(max(h, 0ll), (long long)k_len);
  }
};

// The tiles of `SUB` keys of queries [i0, i1): of the sinks first, then of the window.
template <int SUB>
struct WindowTiles {
  int s_end, w_begin, w_end, n_sink, n;
  int lo_max, hi_min;  // every query of the block sees [lo_max, hi_min), and the sinks below hi_min
  __device__ __forceinline__ WindowTiles(const WindowDims &p, const WindowEntry &e, int i0, int i1) {
    int lo0, hi0, lo1, hi1;
    e.interval(p, i0, lo0, hi0);
    e.interval(p, i1 - 1, lo1, hi1);
    s_end = min(p.sinks, hi1);
    w_begin = min(max(lo0, s_end), hi1);
    w_end = hi1;
    lo_max = lo1;
    hi_min = hi0;
    n_sink = (s_end + SUB - 1) / SUB;
    n = n_sink + (w_end - w_begin + SUB - 1) / SUB;
  }
  // First key row of tile t, and the end of its range; a tile behind the last one lies behind the window.
  __device__ __forceinline__ int row(int t) const { return t < n_sink ? t * SUB : t < n ? w_begin + (t - n_sink) * SUB : w_end; }
  __device__ __forceinline__ int end(int t) const { return t < n_sink ? s_end : w_end; }
  __device__ __forceinline__ bool whole(int t) const {
    const int r = row(t);
    return r + SUB <= min(hi_min, end(t)) && (t < n_sink || r >= lo_max);
  }
};

// The key range of tile t that a query with [lo, hi) sees.
template <typename Tiles>
__device__ __forceinline__ void tile_interval(const Tiles &tiles, int t, int lo, int hi, int &a, int &b) {
  a = t < tiles.n_sink ? 0 : lo;
  b = min(hi, tiles.end(t));
}

// Where workgroup i of 8 ceil(total / 8) works: every XCD takes a run of neighbouring units, so that the queries of one
// head, and the heads that share keys, read them through one L2.  -1: nothing.
__device__ __forceinline__ int window_unit(int total) {
  const int x = blockIdx.x & 7, j = blockIdx.x >> 3;
  const int first = (int)((long long)total * x / 8), last = (int)((long long)total * (x + 1) / 8);
  return j < last - first ? first + j : -1;
}

// Head x of all key heads (G = 1) or query heads in the order of the units: the heads that share keys next to each other,
// then the batch entries, whose lengths may differ much, dealt evenly over the XCDs by that.  (48 heads of three sequences
// of which one is empty, 1327 tokens: dK and dV 107 us with an entry's heads next to each other, 64 so.)
__device__ __forceinline__ void window_head(int x, int B, int G, int &b, int &h) {
  const int group = x / G, hk = group / B;
  b = group - hk * B;
  h = hk * G + (x - group * G);
}

// fp16 has few exponents, and long rows many small probabilities: they are kept times 2^15 (shared rows, blocks of 32) and 2^7 of
// what they are relative to the running reference, which the interleaved engine leaves up to 2^8 below a row's largest.
template <typename T> constexpr int BLOCKS_P_LOG2 = std::is_same<T, F16>::value ? 7 : 0;
template <typename T> constexpr int STEP_P_LOG2 = std::is_same<T, F16>::value ? 15 : 0;

// ---- blocks of 128 queries ----------------------------------------------------------------------------------
// The interleaved engine (attn_kernel_il.h) over the tiles of a block: its stages, its softmax beside the MFMAs, its
// two workgroups per CU.  What differs is where the tiles are, and that the mask is an interval per query.
template <int D, typename T>
struct WindowRow : IlRow<D, 128, 64, T, true, BLOCKS_P_LOG2<T>> {
  using Base = IlRow<D, 128, 64, T, true, BLOCKS_P_LOG2<T>>;
  using Base::EL;
  using Base::V_S;
  using Base::Base;
  // keys of the sub-tile in S buffer PAR outside [a, b) (relative to this lane's first key) become -inf
  template <int PAR>
  __device__ __forceinline__ void mask_interval(int a, int b) {
    const uint32_t span = (uint32_t)max(b - a, 0);
    static_unroll<EL>([&](auto e) {
      constexpr int key = 32 * (e / 16) + 16 * ((e % 16) >> 3) + (e & 7);
      float s;
      asm volatile("v_mov_b32 %0, v[%1]" : "=v"(s) : "n"(V_S + PAR * EL + e));
      s = (uint32_t)(key - a) < span ? s : -INFINITY;
      named_write<V_S + PAR * EL + e>(__builtin_bit_cast(uint32_t, s));
    });
  }
};

// Tiles [t0, t1) of a block, from its first loads to the last O += P V (see il_run_row, whose stages these are).
template <typename Row, typename Tiles>
__device__ __forceinline__ void window_run_row(Row &rb, const uint16_t *qrow_ptr, u32x4 Kres, u32x4 Vres, const Tiles &tiles,
                                               int t0, int t1, int lo, int hi, float scale_log2e) {
  constexpr int LOADS = Row::LOADS_PER_WAVE;
  rb.begin_row(qrow_ptr, scale_log2e);
  if (t0 >= t1) {
    wait_vmem<0>();
    return;
  }
  const uint32_t row_bytes = rb.kv_row_bytes;
  const int n_stream = max(t1 - t0, 2);
  // row and descriptor of tile k of the stream (rows behind the range read as zeros)
  auto row_of = [&](int k) {
    return __builtin_amdgcn_readfirstlane(t0 + k < t1 ? tiles.row(t0 + k) : tiles.w_end);
  };
  auto bytes_of = [&](int k) {
    const int end = t0 + k < t1 ? tiles.end(t0 + k) : 0;
    return (uint32_t)__builtin_amdgcn_readfirstlane(end > 0 ? (uint32_t)(end - 1) * row_bytes + Row::ROWB : 0u);
  };
  auto K_of = [&](int k) {
    Kres[2] = bytes_of(k);
    return Kres;
  };
  auto V_of = [&](int k) {
    Vres[2] = bytes_of(k);
    return Vres;
  };
  auto mask = [&](auto par, int k) {
    const int t = t0 + k;
    if (t < t1 && tiles.whole(t)) return;
    int a, b;
    tile_interval(tiles, t, lo, hi, a, b);
    if (t >= t1) b = a;  // a lone tile is padded with one of which nothing is seen
    const int first = tiles.row(t) + 8 * rb.g;
    rb.template mask_interval<decltype(par)::value>(a - first, b - first);
  };
  constexpr std::integral_constant<int, 0> even{};
  constexpr std::integral_constant<int, 1> odd{};
  rb.issue_k_sub(K_of(0), row_of(0), 0);
  rb.issue_k_sub(K_of(1), row_of(1), 1);
  rb.issue_v_sub(V_of(0), row_of(0), 0);
  wait_vmem<2 * LOADS>();
  rb.finish_q(scale_log2e);
  __syncthreads();
  rb.template stage<0, false, true, false>();
  mask(even, 0);
  wait_vmem<0>();
  __syncthreads();
  rb.issue_k_sub(K_of(2), row_of(2), 0);
  rb.template stage<1, false, true, true>();
  mask(odd, 1);
  wait_vmem<0>();
  __syncthreads();
  bool odd_end = false;
  for (int k = 2; k < n_stream; k += 2) {
    rb.template stage<0, true, true, true, true>(V_of(k - 1), row_of(k - 1), K_of(k + 1), row_of(k + 1));
    mask(even, k);
    wait_vmem<0>();
    __syncthreads();
    odd_end = k + 1 == n_stream;
    if (odd_end) break;
    rb.template stage<1, true, true, true, true>(V_of(k), row_of(k), K_of(k + 2), row_of(k + 2));
    mask(odd, k + 1);
    wait_vmem<0>();
    __syncthreads();
  }
  const int last = n_stream - 1;
  if (odd_end) {
    rb.issue_v_sub(V_of(last), row_of(last), 0);
    rb.template stage<1, true, false, true>();
    wait_vmem<0>();
    __syncthreads();
    rb.template stage<0, true, false, false>();
  } else {
    rb.issue_v_sub(V_of(last), row_of(last), 1);
    rb.template stage<0, true, false, true>();
    wait_vmem<0>();
    __syncthreads();
    rb.template stage<1, true, false, false>();
  }
}

template <int D, typename T>
__global__ __launch_bounds__(256, 2) __attribute__((amdgpu_num_vgpr(IL_VGPRS))) void window_attn_fwd_kernel(
    const uint16_t *__restrict__ gq, const uint16_t *__restrict__ gk, const uint16_t *__restrict__ gv,
    uint16_t *__restrict__ gout, float *__restrict__ lse, const WindowDims p) {
  using Row = WindowRow<D, T>;
  using Tiles = WindowTiles<Row::SUB>;
  constexpr int NT = Row::NT, ROWB = Row::ROWB, CH = Row::CH, OST = Row::OST, BQ = 128;
  il_claim_registers();
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int nbq = (p.Nq + BQ - 1) / BQ;
  const int unit = window_unit(p.B * p.Hq * nbq * p.parts);
  if (unit < 0) return;
  const int part = unit % p.parts, block = unit / p.parts;
  const int x = block / nbq, r = nbq - 1 - (block - x * nbq);  // later queries first: they see no fewer keys
  int b, h;
  window_head(x, p.B, p.Hq / p.Hkv, b, h);
  const int bh = b * p.Hq + h;
  const WindowEntry e(p, b);
  Row rb(lds, (uint32_t)p.kv.n * 2);
  const int i0 = r * BQ, i1 = min(i0 + BQ, e.q_len), i = i0 + rb.row_in_block();
  const uint16_t *const q_head = gq + (size_t)b * p.q.b + (size_t)h * p.q.h;
  const size_t kv_head = (size_t)b * p.kv.b + (size_t)(h / (p.Hq / p.Hkv)) * p.kv.h;
  int lo = 0, hi = 0;
  if (i0 < i1) {
    const Tiles tiles(p, e, i0, i1);
    const int row = min(i, i1 - 1);
    e.interval(p, row, lo, hi);
    const int t0 = (int)((long long)tiles.n * part / p.parts), t1 = (int)((long long)tiles.n * (part + 1) / p.parts);
    const u32x4 Kres = head_rsrc(gk + kv_head, 0), Vres = head_rsrc(gv + kv_head, 0);
    window_run_row(rb, q_head + (size_t)row * p.q.n, Kres, Vres, tiles, t0, t1, lo, hi, p.scale_log2e);
  } else {
    rb.begin_row(q_head, p.scale_log2e);  // no query of the block exists: its rows are empty
    wait_vmem<0>();
  }
  __syncthreads();  // every wave is done with the tile windows
  rb.m_run -= BLOCKS_P_LOG2<T>;  // what the sums are relative to
  const size_t row0 = ((size_t)bh * p.Nq) + i0;
  if (p.parts > 1) {
    if (i >= p.Nq) return;
    const size_t at = (size_t)part * ((size_t)p.B * p.Hq * p.Nq) + row0 + rb.row_in_block();
    const float l_tot = i < i1 ? sum_with_other_half(rb.l_run) : 0.f;
    if (rb.g == 0) *reinterpret_cast<f32x2 *>(p.part_ml + 2 * at) = f32x2{rb.m_run, l_tot};
    float *const row = p.part_rows + at * D + 4 * rb.g;
    static_unroll<4 * Row::DB>([&](auto q4) {
      constexpr int db = q4 / 4, a = q4 % 4, base = Row::A_O + 16 * db + 4 * a;
      *reinterpret_cast<f32x4 *>(row + 32 * db + 8 * a) =
          f32x4{acc_read<base>(), acc_read<base + 1>(), acc_read<base + 2>(), acc_read<base + 3>()};
    });
    return;
  }
  const float row_lse = rb.stage_rows(lds);
  __syncthreads();
  if (lse && rb.g == 0 && i < p.Nq) lse[row0 + rb.row_in_block()] = i < i1 ? row_lse : -INFINITY;
  uint16_t *const dst = gout + (size_t)b * p.out.b + (size_t)h * p.out.h + (size_t)i0 * p.out.n;
#pragma unroll 2
  for (int L = rb.tid; L < BQ * CH; L += NT) {
    const int row = L / CH, cc = L % CH;
    if (i0 + row < p.Nq) {
      u32x4 val = *reinterpret_cast<const u32x4 *>(lds + row * OST + cc * 16);
      if (i0 + row >= i1) val = u32x4{0, 0, 0, 0};
      *reinterpret_cast<u32x4 *>(dst + (size_t)row * p.out.n + cc * 8) = val;
    }
  }
}

// ---- few queries --------------------------------------------------------------------------------------------
// Up to 32 rows of queries share their keys: SHARED, the G query heads of a key head with Nq queries each, a single token of
// a stream above all; or a block of 32 queries of one head, where blocks of 128 would leave the GPU idle (forward_form).  What such a call costs is reading the visible keys and values once.  A workgroup takes a part of
// a (batch entry, key head)'s tiles of 32 keys, each of its four waves every fourth of them, in LDS of its own, so that
// the loop has no barrier: S^T = K Q^T and O^T += V^T P^T as in the engine for blocks, with all rows in one 32-column
// MFMA tile.  Two tiles of K and V per wave are in flight (64 KB a CU at D = 128), which is what HBM's latency asks for.
constexpr int STEP_KEYS = 32, STEP_WAVES = 4;

template <int D, typename T>
struct StepLds {
  static constexpr int TILE = STEP_KEYS * D * 2;
  static constexpr int WAVE = 4 * TILE;  // two buffers of K and V
  static constexpr int BYTES = STEP_WAVES * WAVE;
  static constexpr int JOIN_STRIDE = D + 4;  // floats of a row's sums when the waves join them
  static_assert(STEP_WAVES * 32 * (JOIN_STRIDE + 2) * 4 <= BYTES, "the joined sums do not fit");
};

template <int D, bool SHARED, typename T>
__global__ __launch_bounds__(STEP_WAVES * 64) void window_attn_step_kernel(
    const uint16_t *__restrict__ gq, const uint16_t *__restrict__ gk, const uint16_t *__restrict__ gv,
    uint16_t *__restrict__ gout, float *__restrict__ lse, const WindowDims p) {
  using Lds = StepLds<D, T>;
  using Tiles = WindowTiles<STEP_KEYS>;
  using LoadK = TileLoader<D, STEP_KEYS, 64, false>;
  using LoadV = TileLoader<D, STEP_KEYS, 64, true>;
  constexpr int ROWB = D * 2, DS = D / 16, DB = D / 32, ITERS = LoadK::ITERS;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int G = p.Hq / p.Hkv, blocks = SHARED ? 1 : (p.Nq + 31) / 32;
  const int unit = window_unit(p.B * (SHARED ? p.Hkv : p.Hq) * blocks * p.parts);
  if (unit < 0) return;
  const int part = unit % p.parts, x = unit / p.parts / blocks, block = blocks - 1 - (unit / p.parts - x * blocks);
  int b, h0;  // the first head of the rows
  window_head(x, p.B, SHARED ? 1 : G, b, h0);
  const int hk = SHARED ? h0 : h0 / G, i0 = 32 * block, R = SHARED ? G * p.Nq : min(32, p.Nq - i0);
  if (SHARED) h0 *= G;
  auto head_of = [&](int row) { return SHARED ? h0 + row / p.Nq : h0; };
  auto query_of = [&](int row) { return SHARED ? row % p.Nq : i0 + row; };
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, g = lane >> 5;
  const WindowEntry e(p, b);
  const int row = min(l32, R - 1), h = head_of(row);
  f32x16 o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[db][v] = 0.f;
  float m_run = -FLT_MAX, l_run = 0.f;
  if (i0 < e.q_len) {
    const Tiles tiles(p, e, i0, SHARED ? e.q_len : min(i0 + 32, e.q_len));
    int lo, hi;
    const int row_q = min(query_of(row), e.q_len - 1);
    e.interval(p, row_q, lo, hi);
    const int t0 = (int)((long long)tiles.n * part / p.parts), t1 = (int)((long long)tiles.n * (part + 1) / p.parts);
    const size_t kv_head = (size_t)b * p.kv.b + (size_t)hk * p.kv.h;
    u32x4 Kres = head_rsrc(gk + kv_head, 0), Vres = head_rsrc(gv + kv_head, 0);
    const uint32_t row_bytes = (uint32_t)p.kv.n * 2;
    const uint32_t lds_base = (uint32_t)(uintptr_t)(LDS_PTR(char))lds;
    const uint32_t lds_wave = __builtin_amdgcn_readfirstlane(lds_base + wave * Lds::WAVE);
    char *const mine = lds + wave * Lds::WAVE;
    auto issue = [&](int t, int buf) {  // tile t into buffer buf; a tile behind the part reads nothing
      const int end = t < t1 ? tiles.end(t) : 0;
      const uint32_t bytes = __builtin_amdgcn_readfirstlane(end > 0 ? (uint32_t)(end - 1) * row_bytes + ROWB : 0u);
      const int r0 = __builtin_amdgcn_readfirstlane(t < t1 ? tiles.row(t) : 0);
      Kres[2] = Vres[2] = bytes;
#pragma unroll
      for (int it = 0; it < ITERS; ++it)
        LoadK::template issue_one<true>(it, Kres, r0, lds_wave + buf * 2 * Lds::TILE, lane, LoadK::lane_offset(lane, it, row_bytes), row_bytes);
#pragma unroll
      for (int it = 0; it < ITERS; ++it)
        LoadV::template issue_one<true>(it, Vres, r0, lds_wave + (buf * 2 + 1) * Lds::TILE, lane, LoadV::lane_offset(lane, it, row_bytes), row_bytes);
    };
    issue(t0 + wave, 0);
    issue(t0 + wave + STEP_WAVES, 1);
    // Q^T as the second operand: lane (row l32, half g) holds d = 16 s + 8 g + [0, 8)
    u32x4 q[DS];
    const uint16_t *const qp = gq + (size_t)b * p.q.b + (size_t)h * p.q.h + (size_t)row_q * p.q.n + 8 * g;
#pragma unroll
    for (int s = 0; s < DS; ++s) q[s] = *reinterpret_cast<const u32x4 *>(qp + 16 * s);
    // operand addresses as in RowBlock
    const int krow = (l32 & 0x13) | ((l32 & 4) << 1) | ((l32 & 8) >> 1);
    const uint32_t k_addr = krow * ROWB + ((g ^ k_swz<D>(krow)) << 4);
    const int L16 = lane & 15, blk = lane >> 4, v_row = 8 * (blk >> 1) + (L16 >> 2);
    uint32_t v_addr[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
      v_addr[db] = v_row * ROWB + (((4 * db + 2 * (blk & 1) + ((L16 & 3) >> 1)) ^ v_swz<D>(v_row)) << 4) + (L16 & 1) * 8;
    const float sc = p.scale_log2e;
    int buf = 0;
    for (int t = t0 + wave; t < t1; t += STEP_WAVES, buf ^= 1) {
      // the loads of this tile are there when only those of the next one are in flight
      asm volatile("s_waitcnt vmcnt(%0)" : : "n"(2 * ITERS) : "memory");
      const char *const kt = mine + buf * 2 * Lds::TILE, *const vt = kt + Lds::TILE;
      f32x16 s;
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = 0.f;
#pragma unroll
      for (int d = 0; d < DS; ++d) s = T::mfma(*reinterpret_cast<const u32x4 *>(kt + (k_addr ^ (d << 5))), q[d], s);
      int a, z;
      tile_interval(tiles, t, lo, hi, a, z);
      const int first = tiles.row(t) + 8 * g;
      const bool whole = tiles.whole(t);
      const uint32_t span = (uint32_t)max(z - a, 0);
      float m_loc = -INFINITY;
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int key = first + 16 * (v >> 3) + (v & 7);
        s[v] = whole || (uint32_t)(key - a) < span ? s[v] * sc : -INFINITY;
        m_loc = fmaxf(m_loc, s[v]);
      }
      const float m_new = fmaxf(m_run, max_with_other_half(m_loc));  // finite: leading keys at -inf have no weight
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      const float ref = m_new - STEP_P_LOG2<T>;
      l_run *= alpha;
      uint32_t pk[8];
#pragma unroll
      for (int v = 0; v < 16; v += 2) {
        const float p0 = __builtin_amdgcn_exp2f(s[v] - ref), p1 = __builtin_amdgcn_exp2f(s[v + 1] - ref);
        l_run += p0 + p1;
        pk[v >> 1] = T::pack(p0, p1);
      }
      if (__any(alpha != 1.0f)) {
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int v = 0; v < 16; ++v) o[db][v] *= alpha;
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const u32x4 pw = {pk[4 * j], pk[4 * j + 1], pk[4 * j + 2], pk[4 * j + 3]};
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const char *at = vt + v_addr[db] + 16 * j * ROWB;
          const u32x2 first4 = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(at)));
          const u32x2 next4 = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(at + 4 * ROWB)));
          o[db] = T::mfma(u32x4{first4[0], first4[1], next4[0], next4[1]}, pw, o[db]);
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");  // the buffer is read before it is filled again
      issue(t + 2 * STEP_WAVES, buf);
    }
    asm volatile("s_waitcnt vmcnt(0)" : : : "memory");  // nothing is written to LDS behind this
  }
  l_run = sum_with_other_half(l_run);
  m_run -= STEP_P_LOG2<T>;  // what the sums are relative to
  __syncthreads();
  // join the waves' sums: rows [wave][32][JOIN_STRIDE], then their references and row sums
  float *const rows = reinterpret_cast<float *>(lds), *const ml = rows + STEP_WAVES * 32 * Lds::JOIN_STRIDE;
  float *const my_row = rows + (wave * 32 + l32) * Lds::JOIN_STRIDE + 4 * g;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int a = 0; a < 4; ++a)
      *reinterpret_cast<f32x4 *>(my_row + 32 * db + 8 * a) =
          f32x4{o[db][4 * a], o[db][4 * a + 1], o[db][4 * a + 2], o[db][4 * a + 3]};
  if (g == 0) *reinterpret_cast<f32x2 *>(ml + 2 * (wave * 32 + l32)) = f32x2{m_run, l_run};
  __syncthreads();
  constexpr int LANES = D / 8;  // 8 channels each
  for (int L = threadIdx.x; L < R * LANES; L += STEP_WAVES * 64) {
    const int rr = L / LANES, c = 8 * (L % LANES);
    const int head = head_of(rr), qi = query_of(rr);
    float m = -FLT_MAX, l = 0.f, x[8];
#pragma unroll
    for (int w = 0; w < STEP_WAVES; ++w) m = fmaxf(m, ml[2 * (w * 32 + rr)]);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = 0.f;
#pragma unroll
    for (int w = 0; w < STEP_WAVES; ++w) {
      const float f = __builtin_amdgcn_exp2f(ml[2 * (w * 32 + rr)] - m);
      l = __builtin_fmaf(f, ml[2 * (w * 32 + rr) + 1], l);
      const float *const from = rows + (w * 32 + rr) * Lds::JOIN_STRIDE + c;
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = __builtin_fmaf(f, from[j], x[j]);
    }
    const bool there = qi < e.q_len;
    if (!there) l = 0.f;
    const size_t out_row = ((size_t)b * p.Hq + head) * p.Nq + qi;
    if (p.parts > 1) {
      const size_t at = (size_t)part * ((size_t)p.B * p.Hq * p.Nq) + out_row;
      *reinterpret_cast<f32x4 *>(p.part_rows + at * D + c) = f32x4{x[0], x[1], x[2], x[3]};
      *reinterpret_cast<f32x4 *>(p.part_rows + at * D + c + 4) = f32x4{x[4], x[5], x[6], x[7]};
      if (c == 0) *reinterpret_cast<f32x2 *>(p.part_ml + 2 * at) = f32x2{m, l};
    } else {
      const float inv = l == 0.f ? 0.f : 1.0f / l;
      u32x4 w;
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = there ? T::pack(x[2 * j] * inv, x[2 * j + 1] * inv) : 0u;
      *reinterpret_cast<u32x4 *>(gout + (size_t)b * p.out.b + (size_t)head * p.out.h + (size_t)qi * p.out.n + c) = w;
      if (lse && c == 0) lse[out_row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
    }
  }
}

// ---- rows that were cut -------------------------------------------------------------------------------------
// Relative to the largest reference M of a row's parts: O = sum_s 2^(m_s - M) O_s, and likewise the row sums.  A part
// without a visible key has a row sum of zero, and its O is not read.
// A workgroup takes ROWS rows, of each row 256 / (ROWS LANES) lanes every so many parts: one row where there are few, so that
// its parts are read at once and not one after the other (112 rows of 31 parts, D = 128: 4.2 us, the whole call of 56 heads
// on 7, two streams of 7904 keys 38 -> 26 us).
template <int D, int ROWS, typename T>
__global__ __launch_bounds__(256) void window_attn_merge_kernel(uint16_t *__restrict__ gout, float *__restrict__ lse, const WindowDims p) {
  constexpr int LANES = D / 8, GROUPS = 256 / (ROWS * LANES);
  __shared__ float sums[GROUPS > 1 ? GROUPS : 1][GROUPS > 1 ? ROWS * D : 1], shares[GROUPS][ROWS][2];
  const long long total = (long long)p.B * p.Hq * p.Nq;
  const int place = threadIdx.x / LANES, group = place / ROWS, in_wg = place % ROWS, c = 8 * (threadIdx.x % LANES);
  const long long row = (long long)blockIdx.x * ROWS + in_wg;
  const bool there = row < total;
  float m = -FLT_MAX, l = 0.f, x[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = 0.f;
  if (there) {
#pragma unroll 4
    for (int s = group; s < p.parts; s += GROUPS) {
      const f32x2 ml = *reinterpret_cast<const f32x2 *>(p.part_ml + 2 * (s * total + row));
      if (ml[1] != 0.f) m = fmaxf(m, ml[0]);
    }
#pragma unroll 4
    for (int s = group; s < p.parts; s += GROUPS) {
      const size_t at = (size_t)(s * total + row);
      const f32x2 ml = *reinterpret_cast<const f32x2 *>(p.part_ml + 2 * at);
      if (ml[1] == 0.f) continue;
      const float f = __builtin_amdgcn_exp2f(ml[0] - m);
      l = __builtin_fmaf(f, ml[1], l);
      const f32x4 u = *reinterpret_cast<const f32x4 *>(p.part_rows + at * D + c),
                  v = *reinterpret_cast<const f32x4 *>(p.part_rows + at * D + c + 4);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[j] = __builtin_fmaf(f, u[j], x[j]);
        x[4 + j] = __builtin_fmaf(f, v[j], x[4 + j]);
      }
    }
  }
  if constexpr (GROUPS > 1) {  // the groups' sums, in their order, relative to the largest of their references
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[group][in_wg * D + c + j] = x[j];
    if (c == 0) {
      shares[group][in_wg][0] = m;
      shares[group][in_wg][1] = l;
    }
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) m = fmaxf(m, shares[g][in_wg][0]);
    l = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = 0.f;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      const float f = __builtin_amdgcn_exp2f(shares[g][in_wg][0] - m);
      l = __builtin_fmaf(f, shares[g][in_wg][1], l);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = __builtin_fmaf(f, sums[g][in_wg * D + c + j], x[j]);
    }
  }
  if (!there) return;
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  u32x4 w;
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = T::pack(x[2 * j] * inv, x[2 * j + 1] * inv);
  const int i = (int)(row % p.Nq), bh = (int)(row / p.Nq), b = bh / p.Hq, h = bh - b * p.Hq;
  *reinterpret_cast<u32x4 *>(gout + (size_t)b * p.out.b + (size_t)h * p.out.h + (size_t)i * p.out.n + c) = w;
  if (lse && c == 0) lse[row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

}  // namespace calibatt_dev
