// Host launchers and C entry points of the kernels over rows (row_kernels.h): rotary positions with several
// axes, layer norm and its gradients.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "calibatt.h"
#include "launch.h"
#include "row_kernels.h"

namespace {
using namespace calibatt_dev;
using namespace calibatt_host;

int element_bytes(int dtype) { return dtype == CALIBATT_F32 ? 4 : 2; }
bool element_type_ok(int dtype) { return dtype == CALIBATT_BF16 || dtype == CALIBATT_F16 || dtype == CALIBATT_F32; }

// compute units of the current device, looked up once
int device_cus(int &cus) {
  static DevInfo info;
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return CALIBATT_ERR_LAUNCH;
  cus = info.slots[dev].load(std::memory_order_acquire);
  if (cus > 0) return CALIBATT_OK;
  if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0)
    return CALIBATT_ERR_LAUNCH;
  info.slots[dev].store(cus, std::memory_order_release);
  return CALIBATT_OK;
}

// ---- rotary positions ---------------------------------------------------------------------------------------
// Strides of a tensor; those of an axis of one entry are never stepped along.  No two rows of an output may overlap.
bool rope_strides(const calibatt_strides *given, int B, int H, int N, int D, bool output, Strides &s) {
  s = given ? Strides{given->b, given->h, given->n} : Strides{(int64_t)H * N * D, (int64_t)N * D, D};
  const int64_t sizes[3] = {B, H, N}, steps[3] = {s.b, s.h, s.n};
  if (output && !rows_apart(sizes, steps, D)) return false;
  if (B == 1) s.b = 0;
  if (H == 1) s.h = 0;
  if (N == 1) s.n = D;
  return s.n >= D && s.b >= 0 && s.h >= 0 && s.n % 8 == 0 && s.h % 8 == 0 && s.b % 8 == 0;
}

// Entries of the tables of all axes, or -1 where they are more than 32-bit indices reach.
long long rope_entries(int n_axes, const int32_t *dims, const int32_t *length) {
  long long n = 0;
  for (int a = 0; a < n_axes; ++a) n += (long long)(dims[a] / 2) * length[a];
  return n <= 0x3fffffff ? n : -1;
}

int rope_axes_ok(int n_axes, const int32_t *dims, const int32_t *length) {
  if (n_axes < 1 || n_axes > ROPE_MAX_AXES) return CALIBATT_ERR_UNSUPPORTED;
  long long channels = 0;
  for (int a = 0; a < n_axes; ++a) {
    if (dims[a] < 0 || dims[a] % 2 || length[a] <= 0) return CALIBATT_ERR_SHAPE;
    channels += dims[a];
  }
  if (channels == 0 || channels > 1024) return CALIBATT_ERR_SHAPE;
  return rope_entries(n_axes, dims, length) < 0 ? CALIBATT_ERR_SHAPE : CALIBATT_OK;
}

// ---- layer norm ---------------------------------------------------------------------------------------------
constexpr int NORM_MAX_C = 8192;

struct NormTensors {
  const void *x, *dy;
  void *y;
};

// Rows in the order of memory, and as few indices as they need: the indices by falling distance in x, neighbours
// joined where every tensor's distances allow it.
void norm_dims(const int64_t n[3], const calibatt_strides *const s[3], int C, float eps, int center, int weight_f32,
               NormDims &p) {
  struct Index {
    int64_t n, s[3];
  } list[3];
  int m = 0;
  for (int i = 0; i < 3; ++i) {
    if (n[i] == 1) continue;
    Index x = {n[i], {0, 0, 0}};
    for (int t = 0; t < 3; ++t) x.s[t] = i == 0 ? s[t]->b : i == 1 ? s[t]->h : s[t]->n;
    list[m++] = x;
  }
  std::stable_sort(list, list + m, [](const Index &a, const Index &b) { return a.s[0] > b.s[0]; });
  for (int i = m - 2; i >= 0; --i) {
    bool one = true;
    for (int t = 0; t < 3; ++t) one = one && list[i].s[t] == list[i + 1].n * list[i + 1].s[t];
    if (!one) continue;
    const int64_t both = list[i].n * list[i + 1].n;
    list[i] = list[i + 1];
    list[i].n = both;
    for (int j = i + 1; j + 1 < m; ++j) list[j] = list[j + 1];
    --m;
  }
  const Index none = {1, {0, 0, 0}};
  const Index i0 = m > 0 ? list[0] : none, i1 = m > 2 ? list[1] : none, i2 = m > 1 ? list[m - 1] : none;
  p.rows = (int)(n[0] * n[1] * n[2]);
  p.n1 = (int)i1.n;
  p.n2 = (int)i2.n;
  Strides *const to[3] = {&p.x, &p.dy, &p.y};
  for (int t = 0; t < 3; ++t) *to[t] = Strides{i0.s[t], i1.s[t], i2.s[t]};
  p.C = C;
  p.eps = eps;
  p.center = center ? 1 : 0;
  p.weight_f32 = weight_f32;
}

// How a row of C elements lies in lanes: pieces of 16 bytes where they can be had, few lanes for short rows (several
// rows to a wave), the whole workgroup for long ones.
template <typename T, typename F>
int norm_layout(bool wide, int C, F &&f) {
#define CALIBATT_NORM(vec, lpr, nv) f(std::integral_constant<int, vec>{}, std::integral_constant<int, lpr>{}, std::integral_constant<int, nv>{})
  if (wide) {
    constexpr int V = T::PER16;
    const int pieces = C / V;
    if (pieces <= 8) return CALIBATT_NORM(V, 8, 1);
    if (pieces <= 16) return CALIBATT_NORM(V, 16, 1);
    if (pieces <= 32) return CALIBATT_NORM(V, 32, 1);
    if (pieces <= 64) return CALIBATT_NORM(V, 64, 1);
    if (pieces <= 128) return CALIBATT_NORM(V, 64, 2);
    if (pieces <= 256) return CALIBATT_NORM(V, 64, 4);
    if (pieces <= 512) return CALIBATT_NORM(V, 256, 2);
    if (pieces <= 768) return CALIBATT_NORM(V, 256, 3);
    if (pieces <= 1024) return CALIBATT_NORM(V, 256, 4);
    if constexpr (V == 4) {
      if (pieces <= 1536) return CALIBATT_NORM(V, 256, 6);
      return CALIBATT_NORM(V, 256, 8);
    }
    return CALIBATT_ERR_UNSUPPORTED;
  }
  if (C <= 64) return CALIBATT_NORM(1, 64, 1);
  if (C <= 256) return CALIBATT_NORM(1, 64, 4);
  if (C <= 1024) return CALIBATT_NORM(1, 256, 4);
  if (C <= 4096) return CALIBATT_NORM(1, 256, 16);
  return CALIBATT_NORM(1, 256, 32);
#undef CALIBATT_NORM
}

// whether every row of a tensor is made of aligned pieces of 16 bytes
bool norm_wide(const void *ptr, const calibatt_strides &s, int C, int bytes) {
  return ((uintptr_t)ptr & 15) == 0 && (C * bytes) % 16 == 0 && (s.b * bytes) % 16 == 0 && (s.h * bytes) % 16 == 0 &&
         (s.n * bytes) % 16 == 0;
}

int norm_check(int64_t B, int64_t H, int64_t N, int C, int dtype, int weight_dtype, float eps) {
  if (B <= 0 || H <= 0 || N <= 0 || C <= 0 || !(eps >= 0.f)) return CALIBATT_ERR_SHAPE;
  if (B > 0x3fffffff || H > 0x3fffffff || N > 0x3fffffff || B * H > 0x3fffffff || B * H * N > 0x3fffffff) return CALIBATT_ERR_SHAPE;
  if (!element_type_ok(dtype) || (weight_dtype != dtype && weight_dtype != CALIBATT_F32) || C > NORM_MAX_C)
    return CALIBATT_ERR_UNSUPPORTED;
  return CALIBATT_OK;
}
// `row`: C for an output, whose rows must not overlap, 0 for an input, whose rows may be one
bool norm_tensor_ok(const void *ptr, const int64_t n[3], const calibatt_strides &s, int bytes, int row) {
  const int64_t step[3] = {s.b, s.h, s.n};
  for (int i = 0; i < 3; ++i)
    if (step[i] < 0) return false;
  if (row && !rows_apart(n, step, row)) return false;
  return ((uintptr_t)ptr & (bytes - 1)) == 0;
}

// Workgroups of the gradients' kernel at most, and rows of the workspace: two for every CU.  Each leaves a share of dw
// and db that is written and read again, so more of them cost more (5120 columns, 32 760 rows: 21 MB of shares beside
// 1 007 MB); fewer keep too few rows in flight.
constexpr int NORM_BWD_WGS_PER_CU = 2;
// Rounds of rows that one workgroup takes by itself, and adds up without a second launch (16 rows of 88: 17 us with one,
// 14 without).
constexpr int NORM_BWD_ALONE = 8;

template <typename T>
int launch_norm_fwd(const NormTensors &t, const void *weight, const void *bias, bool wide, const NormDims &p, hipStream_t stream) {
  int cus = 0;
  if (int st = device_cus(cus)) return st;
  return norm_layout<T>(wide, p.C, [&](auto vec, auto lpr, auto nv) {
    constexpr int GROUPS = 256 / lpr;
    const int grid = std::min((p.rows + GROUPS - 1) / GROUPS, cus * 8);
    typedef typename T::type E;
    return launch_kernel(layer_norm_fwd_kernel<T, vec, lpr, nv>, (unsigned)grid, 256, 0, stream, (const E *)t.x, weight,
                         bias, (E *)t.y, p);
  });
}

template <typename T>
int launch_norm_bwd(const NormTensors &t, const void *weight, bool wide, const NormDims &p, void *dweight, void *dbias,
                    float *partial, hipStream_t stream) {
  int cus = 0, grid = 0;
  if (int st = device_cus(cus)) return st;
  const int st = norm_layout<T>(wide, p.C, [&](auto vec, auto lpr, auto nv) {
    constexpr int GROUPS = 256 / lpr;
    constexpr int SMEM = GROUPS == 1 ? 0 : 256 * vec * nv * 4;
    grid = std::min((p.rows + GROUPS - 1) / GROUPS, cus * NORM_BWD_WGS_PER_CU);
    if (grid <= NORM_BWD_ALONE) grid = 1;
    typedef typename T::type E;
    return launch_kernel(layer_norm_bwd_kernel<T, vec, lpr, nv>, (unsigned)grid, 256, SMEM, stream, (const E *)t.dy,
                         (const E *)t.x, weight, (E *)t.y, partial, dweight, dbias, p);
  });
  if (st != CALIBATT_OK || grid == 1 || !(dweight || dbias)) return st;
  // few columns: narrow pieces of them, so that many lanes share the rows of each
  if (p.C <= 512)
    return launch_kernel(layer_norm_params_kernel<T, 8>, (unsigned)((2 * p.C + 7) / 8), 256, 0, stream, (const float *)partial,
                         grid, p.C, p.weight_f32, dweight, dbias);
  return launch_kernel(layer_norm_params_kernel<T, 32>, (unsigned)((2 * p.C + 31) / 32), 256, 0, stream, (const float *)partial,
                       grid, p.C, p.weight_f32, dweight, dbias);
}

}  // namespace

extern "C" int calibatt_rope_table(int n_axes, const int32_t *dims, const int32_t *length, const double *scale, double theta,
                                   float *table, int64_t capacity, int64_t *entries) {
  if (!dims || !length || !entries) return CALIBATT_ERR_NULL;
  if (int st = rope_axes_ok(n_axes, dims, length)) return st;
  if (!(theta > 0.0) || !isfinite(theta)) return CALIBATT_ERR_SHAPE;
  for (int a = 0; scale && a < n_axes; ++a)
    if (!isfinite(scale[a])) return CALIBATT_ERR_SHAPE;
  *entries = rope_entries(n_axes, dims, length);
  if (!table) return CALIBATT_OK;
  if (capacity < *entries) return CALIBATT_ERR_BUFFER_TOO_SMALL;
  float *to = table;
  for (int a = 0; a < n_axes; ++a)
    for (int pos = 0; pos < length[a]; ++pos)
      for (int i = 0; i < dims[a] / 2; ++i) {
        // in 64 bits: an angle of many turns keeps its place in the turn
        const double angle = pos * (scale ? scale[a] : 1.0) * pow(theta, -2.0 * i / dims[a]);
        *to++ = (float)cos(angle);
        *to++ = (float)sin(angle);
      }
  return CALIBATT_OK;
}

extern "C" int calibatt_rope_axes(const void *q, void *q_out, const void *k, void *k_out, int B, int Hq, int Hk, int N, int D,
                                  const calibatt_rope *rope, const calibatt_rope_place *place,
                                  const calibatt_strides *q_strides, const calibatt_strides *q_out_strides,
                                  const calibatt_strides *k_strides, const calibatt_strides *k_out_strides, int dtype,
                                  int inverse, void *stream) {
  if (!q || !q_out || !rope || !rope->table || !place || (k && !k_out)) return CALIBATT_ERR_NULL;
  if (!k) Hk = 0;
  if (B <= 0 || Hq <= 0 || N <= 0 || D <= 0 || (k && Hk <= 0)) return CALIBATT_ERR_SHAPE;
  if (B > 65535 || Hq > 0xffff || Hk > 0xffff || N > 1 << 30) return CALIBATT_ERR_SHAPE;
  if (!element_type_ok(dtype) || D % 8 || D > 1024) return CALIBATT_ERR_UNSUPPORTED;
  if (int st = rope_axes_ok(rope->n_axes, rope->dims, rope->length)) return st;
  RopeDims p = {};
  p.N = N;
  p.n_axes = rope->n_axes;
  p.sign = inverse ? -1.f : 1.f;
  int at = 0;
  for (int a = 0; a < p.n_axes; ++a) {
    p.pairs += rope->dims[a] / 2;
    p.end[a] = p.pairs;
    p.length[a] = rope->length[a];
    p.at[a] = at;
    at += rope->dims[a] / 2 * rope->length[a];
  }
  if (2 * p.pairs > D) return CALIBATT_ERR_SHAPE;
  const bool halves = !rope->interleaved;
  if (p.pairs % (halves ? 8 : 4)) return CALIBATT_ERR_UNSUPPORTED;  // whole 16-byte pieces
  if (place->positions) {
    if (((uintptr_t)place->positions & 3) || place->positions_b < 0) return CALIBATT_ERR_SHAPE;
    p.pos_b = place->positions_b;
  } else {
    long long n_grid = 1;
    for (int a = 0; a < p.n_axes; ++a) {
      if (place->grid[a] <= 0 || place->start[a] < 0 || (long long)place->start[a] + place->grid[a] > p.length[a])
        return CALIBATT_ERR_SHAPE;
      p.grid[a] = place->grid[a];
      p.start[a] = place->start[a];
      n_grid *= place->grid[a];
      if (n_grid > N) return CALIBATT_ERR_SHAPE;
    }
    p.n_grid = (int)n_grid;
  }
  const calibatt_strides *const given[4] = {q_strides, q_out_strides, k_strides, k_out_strides};
  Strides s[4] = {};
  for (int i = 0; i < (k ? 4 : 2); ++i)
    if (!rope_strides(given[i], B, i < 2 ? Hq : Hk, N, D, i & 1, s[i])) return CALIBATT_ERR_SHAPE;
  if (((uintptr_t)q | (uintptr_t)q_out | (uintptr_t)k | (uintptr_t)(k ? k_out : nullptr)) & 15) return CALIBATT_ERR_SHAPE;
  if ((uintptr_t)rope->table & 7) return CALIBATT_ERR_SHAPE;
  const RopeTensor tq = {q, q_out, s[0], s[1], Hq}, tk = {k, k_out, s[2], s[3], Hk};
  p.units = halves ? p.pairs / 8 + (D - 2 * p.pairs) / 8 : D / 8;
  p.tokens_per_wg = 256 / p.units;
  if (N / p.tokens_per_wg >= 0xffffff) return CALIBATT_ERR_SHAPE;  // a launch has less than 2^32 threads along an axis
  // Heads of one workgroup: as many as leave every CU eight workgroups, at most 16 (the tables are then read for one
  // byte in sixteen that is moved).
  const long long wgs = (long long)B * ((N + p.tokens_per_wg - 1) / p.tokens_per_wg);
  int cus = 0;
  if (int st = device_cus(cus)) return st;
  const int heads = Hq + Hk;
  p.heads_per_wg = (int)std::min<long long>(16, std::max<long long>(1, wgs * heads / (8LL * cus)));
  const dim3 grid((N + p.tokens_per_wg - 1) / p.tokens_per_wg, (heads + p.heads_per_wg - 1) / p.heads_per_wg, B);
  if (grid.y > 65535) return CALIBATT_ERR_SHAPE;
  auto go = [&](auto type, auto h) {
    const float2 *table = (const float2 *)rope->table;
    const int *positions = place->positions;
    void *argv[] = {(void *)&tq, (void *)&tk, (void *)&table, (void *)&positions, (void *)&p};
    return hipLaunchKernel((const void *)rope_axes_kernel<decltype(type), decltype(h)::value>, grid, dim3(256), argv, 0,
                           (hipStream_t)stream) == hipSuccess ? CALIBATT_OK : CALIBATT_ERR_LAUNCH;
  };
  auto typed = [&](auto type) { return halves ? go(type, std::true_type{}) : go(type, std::false_type{}); };
  return dtype == CALIBATT_BF16 ? typed(RowBf16{}) : dtype == CALIBATT_F16 ? typed(RowF16{}) : typed(RowF32{});
}

extern "C" int calibatt_layer_norm_fwd(const void *x, const void *weight, const void *bias, void *y, int64_t B, int64_t H,
                                       int64_t N, int C, const calibatt_strides *x_strides, const calibatt_strides *y_strides,
                                       float eps, int center, int dtype, int weight_dtype, void *stream) {
  if (!x || !y || (bias && !weight)) return CALIBATT_ERR_NULL;
  if (int st = norm_check(B, H, N, C, dtype, weight_dtype, eps)) return st;
  const calibatt_strides packed = {H * N * C, N * C, C};
  const calibatt_strides &sx = x_strides ? *x_strides : packed, &sy = y_strides ? *y_strides : packed;
  const int bytes = element_bytes(dtype), wbytes = element_bytes(weight_dtype);
  const int64_t n[3] = {B, H, N};
  if (!norm_tensor_ok(x, n, sx, bytes, 0) || !norm_tensor_ok(y, n, sy, bytes, C)) return CALIBATT_ERR_SHAPE;
  if (((uintptr_t)weight | (uintptr_t)bias) & (wbytes - 1)) return CALIBATT_ERR_SHAPE;
  const calibatt_strides *const s[3] = {&sx, &sx, &sy};
  NormDims p;
  norm_dims(n, s, C, eps, center, weight_dtype == CALIBATT_F32, p);
  const bool wide = norm_wide(x, sx, C, bytes) && norm_wide(y, sy, C, bytes) && (((uintptr_t)weight | (uintptr_t)bias) & 15) == 0;
  const NormTensors t = {x, nullptr, y};
  hipStream_t hs = (hipStream_t)stream;
  return dtype == CALIBATT_BF16  ? launch_norm_fwd<RowBf16>(t, weight, bias, wide, p, hs)
         : dtype == CALIBATT_F16 ? launch_norm_fwd<RowF16>(t, weight, bias, wide, p, hs)
                                 : launch_norm_fwd<RowF32>(t, weight, bias, wide, p, hs);
}

extern "C" int calibatt_layer_norm_bwd_workspace_bytes(int C, int64_t *bytes) {
  if (!bytes) return CALIBATT_ERR_NULL;
  if (C <= 0) return CALIBATT_ERR_SHAPE;
  if (C > NORM_MAX_C) return CALIBATT_ERR_UNSUPPORTED;
  int cus = 0;
  if (int st = device_cus(cus)) return st;
  *bytes = (int64_t)cus * NORM_BWD_WGS_PER_CU * 2 * C * 4;
  return CALIBATT_OK;
}

extern "C" int calibatt_layer_norm_bwd(const void *dy, const void *x, const void *weight, void *dx, void *dweight, void *dbias,
                                       int64_t B, int64_t H, int64_t N, int C, const calibatt_strides *dy_strides,
                                       const calibatt_strides *x_strides, const calibatt_strides *dx_strides, float eps,
                                       int center, int dtype, int weight_dtype, float *workspace, int64_t workspace_bytes,
                                       void *stream) {
  if (!dy || !x || !dx || ((dweight || dbias) && (!weight || !workspace))) return CALIBATT_ERR_NULL;
  if (int st = norm_check(B, H, N, C, dtype, weight_dtype, eps)) return st;
  const calibatt_strides packed = {H * N * C, N * C, C};
  const calibatt_strides &sg = dy_strides ? *dy_strides : packed, &sx = x_strides ? *x_strides : packed,
                         &sd = dx_strides ? *dx_strides : packed;
  const int bytes = element_bytes(dtype), wbytes = element_bytes(weight_dtype);
  const int64_t n[3] = {B, H, N};
  if (!norm_tensor_ok(dy, n, sg, bytes, 0) || !norm_tensor_ok(x, n, sx, bytes, 0) || !norm_tensor_ok(dx, n, sd, bytes, C))
    return CALIBATT_ERR_SHAPE;
  if (((uintptr_t)weight | (uintptr_t)dweight | (uintptr_t)dbias) & (wbytes - 1)) return CALIBATT_ERR_SHAPE;
  const bool params = dweight || dbias;
  if (params) {
    int64_t need = 0;
    if (int st = calibatt_layer_norm_bwd_workspace_bytes(C, &need)) return st;
    if ((uintptr_t)workspace & 3) return CALIBATT_ERR_SHAPE;
    if (workspace_bytes < need) return CALIBATT_ERR_BUFFER_TOO_SMALL;
  }
  const calibatt_strides *const s[3] = {&sx, &sg, &sd};
  NormDims p;
  norm_dims(n, s, C, eps, center, weight_dtype == CALIBATT_F32, p);
  const bool wide = norm_wide(x, sx, C, bytes) && norm_wide(dy, sg, C, bytes) && norm_wide(dx, sd, C, bytes) &&
                    (((uintptr_t)weight | (uintptr_t)workspace) & 15) == 0;
  const NormTensors t = {x, dy, dx};
  hipStream_t hs = (hipStream_t)stream;
  float *const partial = params ? workspace : nullptr;
  return dtype == CALIBATT_BF16  ? launch_norm_bwd<RowBf16>(t, weight, wide, p, dweight, dbias, partial, hs)
         : dtype == CALIBATT_F16 ? launch_norm_bwd<RowF16>(t, weight, wide, p, dweight, dbias, partial, hs)
                                 : launch_norm_bwd<RowF32>(t, weight, wide, p, dweight, dbias, partial, hs);
}
