// Kernels over the rows of q, k and of a layer's input: rotary positions with several axes, and layer
// norm with its gradients.  All of them move a row's channels through registers once; what they cost is
// the bytes that they read and write.
#pragma once
#include "attn_common.h"

namespace calibatt_dev {

// ---- elements -----------------------------------------------------------------------------------------------
// Element types of rows: how many lie in 16 bytes, and their conversion from and to fp32 (to nearest even).
struct RowBf16 {
  typedef uint16_t type;
  static constexpr int PER16 = 8;
  static __device__ __forceinline__ float get(uint16_t x) { return __builtin_bit_cast(float, (uint32_t)x << 16); }
  static __device__ __forceinline__ uint16_t put(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
  static __device__ __forceinline__ void unpack(const u32x4 raw, float *x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __builtin_bit_cast(float, raw[i] << 16);
      x[2 * i + 1] = __builtin_bit_cast(float, raw[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ u32x4 pack(const float *x) {
    u32x4 raw;
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[i] = Bf16::pack(x[2 * i], x[2 * i + 1]);
    return raw;
  }
};
struct RowF16 {
  typedef uint16_t type;
  static constexpr int PER16 = 8;
  static __device__ __forceinline__ float get(uint16_t x) { return (float)__builtin_bit_cast(_Float16, x); }
  static __device__ __forceinline__ uint16_t put(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }
  static __device__ __forceinline__ void unpack(const u32x4 raw, float *x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t word = raw[i];  // (a bit cast of the vector's element itself reads element 0)
      const f16x2 two = __builtin_bit_cast(f16x2, word);
      x[2 * i] = (float)two[0];
      x[2 * i + 1] = (float)two[1];
    }
  }
  static __device__ __forceinline__ u32x4 pack(const float *x) {
    u32x4 raw;
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[i] = F16::pack(x[2 * i], x[2 * i + 1]);
    return raw;
  }
};
struct RowF32 {
  typedef float type;
  static constexpr int PER16 = 4;
  static __device__ __forceinline__ float get(float x) { return x; }
  static __device__ __forceinline__ float put(float x) { return x; }
  static __device__ __forceinline__ void unpack(const u32x4 raw, float *x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t word = raw[i];
      x[i] = __builtin_bit_cast(float, word);
    }
  }
  static __device__ __forceinline__ u32x4 pack(const float *x) {
    u32x4 raw;
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[i] = __builtin_bit_cast(uint32_t, x[i]);
    return raw;
  }
};

// ---- rotary positions ---------------------------------------------------------------------------------------
// The first 2 * pairs channels of a head are pairs; the pairs are dealt to the axes in order, pair i of axis a turns by
// pos_a * frequency(a, i), whose cosine and sine stand in a table of [length of the axis][pairs of the axis].  The
// gradient is the same with the sines negated, as the inverse of a rotation is its transpose.
constexpr int ROPE_MAX_AXES = 4;

struct RopeTensor {
  const void *x;
  void *out;
  Strides in, out_s;
  int H;
};
struct RopeDims {
  int N, pairs, n_axes;
  int end[ROPE_MAX_AXES];     // pairs of the axes so far
  int length[ROPE_MAX_AXES];  // positions that an axis's table has
  int at[ROPE_MAX_AXES];      // first entry of its table
  int grid[ROPE_MAX_AXES], start[ROPE_MAX_AXES];  // without positions: token grid (row-major) and its first positions
  long long pos_b;            // positions: distance between batch entries (0: the same for all)
  int n_grid;                 // tokens of the grid; the ones behind it are not turned
  int heads_per_wg, tokens_per_wg, units;
  float sign;                 // -1: inverse
};

// A thread owns a UNIT of one token: 8 consecutive channels (interleaved pairs), or 8 channels and the 8 that lie
// `pairs` behind them (halves); it finds the cosines and sines of the unit's pairs once and goes over the heads of its
// share, so table reads are spread over up to heads_per_wg heads of q and k.  A workgroup holds 256 / units tokens:
// whole 16-byte accesses, consecutive lanes on consecutive channels.  Bound by HBM; four heads are in flight per thread.
template <typename T, bool HALVES>
__global__ __launch_bounds__(256) void rope_axes_kernel(const RopeTensor q, const RopeTensor k, const float2 *__restrict__ table,
                                                        const int *__restrict__ positions, const RopeDims p) {
  constexpr int LOADS = 8 / T::PER16;        // 16-byte loads for 8 channels
  constexpr int NP = HALVES ? 8 : 4;         // pairs of a unit
  constexpr int PARTS = HALVES ? 2 : 1;
  typedef typename T::type E;
  const int unit = threadIdx.x % p.units;
  const int slot = threadIdx.x / p.units;
  const int n = blockIdx.x * p.tokens_per_wg + slot;
  if (slot >= p.tokens_per_wg || n >= p.N) return;
  const int b = blockIdx.z;
  // channels of the unit: [c0, c0 + 8) and, in halves, [c0 + pairs, c0 + pairs + 8); units behind the pairs are copied
  const int n_turning = HALVES ? p.pairs / 8 : p.pairs / 4;
  const bool turning = unit < n_turning;
  const int c0 = turning ? 8 * unit : 2 * p.pairs + 8 * (unit - n_turning);
  float co[NP], si[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) co[i] = 1.f, si[i] = 0.f;
  if (turning) {
    int pos[ROPE_MAX_AXES];
    if (positions) {
      const int *at = positions + b * p.pos_b + (long long)n * p.n_axes;
#pragma unroll
      for (int a = 0; a < ROPE_MAX_AXES; ++a) pos[a] = a < p.n_axes ? at[a] : -1;
    } else {
      int rest = n;
#pragma unroll
      for (int a = ROPE_MAX_AXES - 1; a >= 0; --a) {
        pos[a] = -1;
        if (a < p.n_axes) {
          const int up = rest / p.grid[a];
          pos[a] = n < p.n_grid ? p.start[a] + rest - up * p.grid[a] : -1;
          rest = up;
        }
      }
    }
    const int p0 = NP * unit;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      int axis_at = 0, axis_pos = -1, first = 0, n_pairs = 0, length = 0;
#pragma unroll
      for (int a = ROPE_MAX_AXES - 1; a >= 0; --a)
        if (a < p.n_axes && p0 + i < p.end[a]) {  // the first axis whose pairs end behind this one
          first = a ? p.end[a - 1] : 0;
          n_pairs = p.end[a] - first;
          axis_at = p.at[a];
          axis_pos = pos[a];
          length = p.length[a];
        }
      if (axis_pos >= length) {  // not in the table: no angle
        co[i] = si[i] = __builtin_nanf("");
      } else if (axis_pos >= 0) {
        const float2 t = table[axis_at + (long long)axis_pos * n_pairs + p0 + i - first];
        co[i] = t.x;
        si[i] = t.y * p.sign;
      }
    }
  }
  const int h0 = blockIdx.y * p.heads_per_wg, h1 = min(h0 + p.heads_per_wg, q.H + k.H);
  auto place = [&](int h, const E *&from, E *&to) {
    const bool of_q = h < q.H;
    const RopeTensor &t = of_q ? q : k;
    const int hh = of_q ? h : h - q.H;
    from = reinterpret_cast<const E *>(t.x) + b * t.in.b + hh * t.in.h + n * t.in.n + c0;
    to = reinterpret_cast<E *>(t.out) + b * t.out_s.b + hh * t.out_s.h + n * t.out_s.n + c0;
  };
  auto turn_and_store = [&](const u32x4 (&raw)[PARTS][LOADS], E *to) {
    float x[PARTS * 8];
#pragma unroll
    for (int s = 0; s < PARTS; ++s)
#pragma unroll
      for (int l = 0; l < LOADS; ++l) T::unpack(raw[s][l], x + 8 * s + T::PER16 * l);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int u = HALVES ? i : 2 * i, v = HALVES ? 8 + i : 2 * i + 1;
      const float a = x[u], c = x[v];
      x[u] = a * co[i] - c * si[i];
      x[v] = a * si[i] + c * co[i];
    }
#pragma unroll
    for (int s = 0; s < PARTS; ++s)
      if (s == 0 || turning)
#pragma unroll
        for (int l = 0; l < LOADS; ++l)
          *reinterpret_cast<u32x4 *>(to + s * p.pairs + T::PER16 * l) = T::pack(x + 8 * s + T::PER16 * l);
  };
  auto load = [&](const E *from, u32x4 (&raw)[PARTS][LOADS]) {
#pragma unroll
    for (int s = 0; s < PARTS; ++s)
#pragma unroll
      for (int l = 0; l < LOADS; ++l)  // the second half of a unit that is only copied does not exist
        raw[s][l] = s == 0 || turning ? *reinterpret_cast<const u32x4 *>(from + s * p.pairs + T::PER16 * l) : u32x4{0, 0, 0, 0};
  };
  constexpr int FLIGHT = HALVES || LOADS > 1 ? 2 : 4;  // heads in flight
  int h = h0;
  for (; h + FLIGHT <= h1; h += FLIGHT) {
    u32x4 raw[FLIGHT][PARTS][LOADS];
    E *to[FLIGHT];
#pragma unroll
    for (int i = 0; i < FLIGHT; ++i) {
      const E *from;
      place(h + i, from, to[i]);
      load(from, raw[i]);
    }
#pragma unroll
    for (int i = 0; i < FLIGHT; ++i) turn_and_store(raw[i], to[i]);
  }
  for (; h < h1; ++h) {
    u32x4 raw[PARTS][LOADS];
    const E *from;
    E *to;
    place(h, from, to);
    load(from, raw);
    turn_and_store(raw, to);
  }
}

// ---- layer norm ---------------------------------------------------------------------------------------------
// y = (x - mean) rstd w + b with rstd = 1 / sqrt(mean((x - mean)^2) + eps); without `center` the mean is taken as 0.
// With h = (x - mean) rstd and g = dy w:
//   dx = rstd (g - mean(g) - h mean(g h))  (without center no mean(g)),  dw = sum over rows of dy h,  db = sum of dy.
// The statistics are taken from the row as it lies in registers, the deviations from the mean and not from a difference
// of large sums; the gradients find them again instead of reading what the forward would have had to store.
struct NormDims {
  int rows, n1, n2;          // row r = (r / (n1 n2), r / n2 % n1, r % n2)
  Strides x, dy, y;          // b, h, n: distances of the three indices; y: of the output (y or dx)
  int C;
  float eps;
  int center, weight_f32;
};

template <int LPR>
__device__ __forceinline__ float group_sum(float x) {
  auto dpp = [](float v, auto ctrl) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value,
                                                                 0xf, 0xf, false));
  };
  x += dpp(x, std::integral_constant<int, 0xB1>{});
  x += dpp(x, std::integral_constant<int, 0x4E>{});
  x += dpp(x, std::integral_constant<int, 0x141>{});
  if constexpr (LPR >= 16) x += dpp(x, std::integral_constant<int, 0x140>{});
  if constexpr (LPR >= 32) {
    float a = x, b = x;
    asm volatile("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(a), "+v"(b));
    x = a + b;
  }
  if constexpr (LPR >= 64) x = sum_with_other_half(x);
  return x;
}

// Sum over the LPR lanes of a row; with 256 lanes over the four waves through LDS.  `slot` is never that of the sum before,
// over the rows as well: a wave that is a sum ahead writes elsewhere than where others still read, and can't be two ahead,
// as one barrier stands in every sum.
template <int LPR>
__device__ __forceinline__ void row_sums(float &a, float &b, float *red, int slot) {
  a = group_sum<LPR < 64 ? LPR : 64>(a);
  b = group_sum<LPR < 64 ? LPR : 64>(b);
  if constexpr (LPR > 64) {
    float *const at = red + slot * 8;
    if ((threadIdx.x & 63) == 0) {
      at[threadIdx.x >> 6] = a;
      at[4 + (threadIdx.x >> 6)] = b;
    }
    __syncthreads();
    a = (at[0] + at[1]) + (at[2] + at[3]);
    b = (at[4] + at[5]) + (at[6] + at[7]);
  }
}

// LPR lanes hold a row, NV pieces of VEC elements each (16 bytes, or single elements where a row is not a whole number
// of aligned 16-byte pieces).
template <typename T, int VEC, int LPR, int NV>
struct NormRow {
  typedef typename T::type E;
  typedef std::conditional_t<(VEC > 1), u32x4, E> Raw;
  static constexpr int GROUPS = 256 / LPR;
  const int lane = threadIdx.x % LPR;

  __device__ __forceinline__ int column(int v) const { return (v * LPR + lane) * VEC; }
  __device__ __forceinline__ void load(const E *row, int C, Raw (&raw)[NV]) const {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = column(v);
      raw[v] = Raw{};
      if (c < C) raw[v] = *reinterpret_cast<const Raw *>(row + c);
    }
  }
  static __device__ __forceinline__ void unpack(const Raw &raw, float *x) {
    if constexpr (VEC > 1) T::unpack(raw, x);
    else x[0] = T::get(raw);
  }
  static __device__ __forceinline__ void store(E *at, const float *x) {
    if constexpr (VEC > 1) *reinterpret_cast<u32x4 *>(at) = T::pack(x);
    else *at = T::put(x[0]);
  }
  // weights or biases of this lane's columns
  __device__ __forceinline__ void parameters(const void *from, bool f32, int C, float other, float (&w)[NV * VEC]) const {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = column(v);
#pragma unroll
      for (int e = 0; e < VEC; ++e) w[v * VEC + e] = other;
      if (!from || c >= C) continue;
      if constexpr (VEC == 1) {
        w[v] = f32 ? ((const float *)from)[c] : T::get(((const E *)from)[c]);
      } else if (f32) {
#pragma unroll
        for (int e = 0; e < VEC; e += 4) RowF32::unpack(*reinterpret_cast<const u32x4 *>((const float *)from + c + e), w + v * VEC + e);
      } else {
        T::unpack(*reinterpret_cast<const u32x4 *>((const E *)from + c), w + v * VEC);
      }
    }
  }
};

__device__ __forceinline__ long long norm_offset(const NormDims &p, const Strides &s, int r) {
  if (p.n1 == 1 && p.n2 == 1) return (long long)r * s.b;  // one run of rows
  const int q = r / p.n2, i2 = r - q * p.n2, i0 = q / p.n1;
  return i0 * s.b + (long long)(q - i0 * p.n1) * s.h + i2 * s.n;
}

template <typename T, int VEC, int LPR, int NV>
__global__ __launch_bounds__(256) void layer_norm_fwd_kernel(const typename T::type *__restrict__ x, const void *__restrict__ weight,
                                                             const void *__restrict__ bias, typename T::type *__restrict__ y,
                                                             const NormDims p) {
  using Row = NormRow<T, VEC, LPR, NV>;
  __shared__ float red[24];
  const Row r;
  const int step = gridDim.x * Row::GROUPS, first = blockIdx.x * Row::GROUPS + threadIdx.x / LPR;
  float w[NV * VEC], b[NV * VEC];
  if constexpr (VEC > 1) {
    r.parameters(weight, p.weight_f32, p.C, 1.f, w);
    r.parameters(bias, p.weight_f32, p.C, 0.f, b);
  }
  const float inv = 1.0f / p.C;
  typename Row::Raw next[NV];
  int slot = 1;  // of the only sum that a row without a mean has: 1 and 2 in turn
  if (first < p.rows) r.load(x + norm_offset(p, p.x, first), p.C, next);
  for (int row = first; row < p.rows; row += step) {
    float xs[NV * VEC];
    float sum = 0.f, unused = 0.f, sq = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) Row::unpack(next[v], xs + v * VEC);
    if (row + step < p.rows) r.load(x + norm_offset(p, p.x, row + step), p.C, next);
    float mean = 0.f;
    if (p.center) {
#pragma unroll
      for (int i = 0; i < NV * VEC; ++i) sum += xs[i];
      row_sums<LPR>(sum, unused, red, 0);
      mean = sum * inv;
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const bool in = r.column(v) < p.C;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        xs[v * VEC + e] -= mean;
        const float d = in ? xs[v * VEC + e] : 0.f;
        sq = __builtin_fmaf(d, d, sq);
      }
    }
    row_sums<LPR>(sq, unused, red, slot);
    slot ^= 3;
    const float rstd = 1.0f / sqrtf(__builtin_fmaf(sq, inv, p.eps));
    typename T::type *const out = y + norm_offset(p, p.y, row);
    if constexpr (VEC == 1) {  // too many columns for registers beside the row's, and cached
      r.parameters(weight, p.weight_f32, p.C, 1.f, w);
      r.parameters(bias, p.weight_f32, p.C, 0.f, b);
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const int i = v * VEC + e;
        xs[i] = __builtin_fmaf(xs[i] * rstd, w[i], b[i]);
      }
      if (r.column(v) < p.C) Row::store(out + r.column(v), xs + v * VEC);
    }
  }
}

// Gradients.  A workgroup goes over the rows with steps of the grid and keeps its share of dw and db in registers; at
// the end it leaves them as row blockIdx.x of `partial` ([gridDim.x][2][C]), which layer_norm_params_kernel adds up: a
// fixed order of additions, no atomics.  A single workgroup's shares are the sums, and go to gdw and gdb (NULL: not
// asked for).
template <typename T, int VEC, int LPR, int NV>
__global__ __launch_bounds__(256) void layer_norm_bwd_kernel(const typename T::type *__restrict__ dy, const typename T::type *__restrict__ x,
                                                             const void *__restrict__ weight, typename T::type *__restrict__ dx,
                                                             float *__restrict__ partial, void *gdw, void *gdb, const NormDims p) {
  using Row = NormRow<T, VEC, LPR, NV>;
  constexpr int EL = NV * VEC;
  __shared__ float red[24];
  extern __shared__ float shares[];  // [GROUPS][LPR * EL] where a workgroup holds more than one row
  const Row r;
  const int step = gridDim.x * Row::GROUPS, group = threadIdx.x / LPR, first = blockIdx.x * Row::GROUPS + group;
  float w[EL], dw[EL], db[EL];
  if constexpr (VEC > 1) r.parameters(weight, p.weight_f32, p.C, 1.f, w);
#pragma unroll
  for (int i = 0; i < EL; ++i) dw[i] = db[i] = 0.f;
  const float inv = 1.0f / p.C;
  typename Row::Raw next_x[NV], next_dy[NV];
  if (first < p.rows) {
    r.load(x + norm_offset(p, p.x, first), p.C, next_x);
    r.load(dy + norm_offset(p, p.dy, first), p.C, next_dy);
  }
  for (int row = first; row < p.rows; row += step) {
    float h[EL], g[EL];
    float unused = 0.f, mean = 0.f, sq = 0.f, sum_g = 0.f, sum_gh = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      Row::unpack(next_x[v], h + v * VEC);
      Row::unpack(next_dy[v], g + v * VEC);
    }
    if (row + step < p.rows) {
      r.load(x + norm_offset(p, p.x, row + step), p.C, next_x);
      r.load(dy + norm_offset(p, p.dy, row + step), p.C, next_dy);
    }
    if constexpr (VEC == 1) r.parameters(weight, p.weight_f32, p.C, 1.f, w);
    if (p.center) {
#pragma unroll
      for (int i = 0; i < EL; ++i) mean += h[i];
      row_sums<LPR>(mean, unused, red, 0);
      mean *= inv;
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const bool in = r.column(v) < p.C;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const int i = v * VEC + e;
        h[i] = in ? h[i] - mean : 0.f;
        sq = __builtin_fmaf(h[i], h[i], sq);
      }
    }
    unused = 0.f;
    row_sums<LPR>(sq, unused, red, 1);
    const float rstd = 1.0f / sqrtf(__builtin_fmaf(sq, inv, p.eps));
#pragma unroll
    for (int i = 0; i < EL; ++i) {
      h[i] *= rstd;
      dw[i] = __builtin_fmaf(g[i], h[i], dw[i]);
      db[i] += g[i];
      g[i] *= w[i];
      sum_g += g[i];
      sum_gh = __builtin_fmaf(g[i], h[i], sum_gh);
    }
    row_sums<LPR>(sum_g, sum_gh, red, 2);
    const float mean_g = p.center ? sum_g * inv : 0.f, mean_gh = sum_gh * inv;
    typename T::type *const out = dx + norm_offset(p, p.y, row);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const int i = v * VEC + e;
        g[i] = rstd * (g[i] - mean_g - h[i] * mean_gh);
      }
      if (r.column(v) < p.C) Row::store(out + r.column(v), g + v * VEC);
    }
  }
  if (!gdw && !gdb) return;
  const bool alone = gridDim.x == 1;
  auto put = [&](void *sums, int which, int c, float s) {
    if (!alone) partial[((size_t)blockIdx.x * 2 + which) * p.C + c] = s;
    else if (sums && p.weight_f32) ((float *)sums)[c] = s;
    else if (sums) ((typename T::type *)sums)[c] = T::put(s);
  };
  auto leave = [&](const float (&share)[EL], void *sums, int which) {
    if constexpr (Row::GROUPS == 1) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = r.column(v);
        if (c >= p.C) continue;
        if (VEC > 1 && !alone) {  // (single floats, 32 bytes apart from lane to lane, took a fifth of the kernel's time)
#pragma unroll
          for (int e = 0; e < VEC; e += 4)
            *reinterpret_cast<u32x4 *>(partial + ((size_t)blockIdx.x * 2 + which) * p.C + c + e) = RowF32::pack(share + v * VEC + e);
        } else {
#pragma unroll
          for (int e = 0; e < VEC; ++e) put(sums, which, c + e, share[v * VEC + e]);
        }
      }
    } else {
      constexpr int W = LPR * EL;
      __syncthreads();
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < VEC; ++e) shares[group * W + r.column(v) + e] = share[v * VEC + e];
      __syncthreads();
      for (int c = threadIdx.x; c < p.C; c += 256) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < Row::GROUPS; ++i) s += shares[i * W + c];
        put(sums, which, c, s);
      }
    }
  };
  leave(dw, gdw, 0);
  leave(db, gdb, 1);
}

// Columns of `partial` ([n][2][C]) added up: COLS columns per workgroup, its 256 / COLS slices of the n rows one after
// the other in registers and joined in LDS.
template <typename T, int COLS>
__global__ __launch_bounds__(256) void layer_norm_params_kernel(const float *__restrict__ partial, int n, int C, int f32,
                                                                void *dw, void *db) {
  constexpr int SLICES = 256 / COLS;
  __shared__ float sums[SLICES][COLS];
  const int col = threadIdx.x % COLS, slice = threadIdx.x / COLS, c = blockIdx.x * COLS + col;
  float s = 0.f;
  if (c < 2 * C) {
#pragma unroll 8
    for (int i = slice; i < n; i += SLICES) s += partial[(size_t)i * 2 * C + c];
  }
  sums[slice][col] = s;
  __syncthreads();
  if (slice == 0 && c < 2 * C) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < SLICES; ++i) s += sums[i][col];
    void *const to = c < C ? dw : db;
    const int at = c < C ? c : c - C;
    if (!to) return;
    if (f32) ((float *)to)[at] = s;
    else ((typename T::type *)to)[at] = T::put(s);
  }
}

}  // namespace calibatt_dev
