// Host launcher and C entry points of attention in a window (attn_kernel_window.h).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "attn_kernel_window.h"
#include "attn_kernel_window_bwd.h"
#include "calibatt.h"
#include "launch.h"

namespace {
using namespace calibatt_dev;
using namespace calibatt_host;

constexpr int WINDOW_CUS = 256;        // plans are functions of the sizes alone
constexpr int WINDOW_MAX_PARTS = 64;
constexpr int64_t MAX_GRID = 0x7ffff0;  // workgroups: a launch has less than 2^32 threads, 512 to a workgroup at most

// Keys that n neighbouring queries see at most, without the sinks.
int64_t window_span(const calibatt_window &w, int n, int Nk) {
  if (w.left < 0 || w.right < 0) return Nk;
  // their frames are at most (n - 1) / frame + 2
  const int64_t frames = (int64_t)(n - 1) / w.frame + 2 + w.left + w.right;
  return std::min<int64_t>(Nk, frames * w.frame);
}
int64_t window_tiles(const calibatt_window &w, int n, int Nk, int tile) {
  return (std::min<int64_t>(w.sinks, Nk) + tile - 1) / tile + (window_span(w, n, Nk) + tile - 1) / tile;
}

// Which kernel a forward goes through.
enum ForwardForm { BLOCKS_128 = CALIBATT_WINDOW_BLOCKS_128, BLOCKS_32 = CALIBATT_WINDOW_BLOCKS_32, SHARED_ROWS = CALIBATT_WINDOW_SHARED_ROWS };
// Workgroups of the kernel for few queries that the GPU holds (its LDS, 128 KB at D = 128).
int64_t step_slots(int D) { return D == 128 ? WINDOW_CUS : 2 * WINDOW_CUS; }
ForwardForm forward_form(int B, int Hq, int Hkv, int Nq, int Nk, int D, const calibatt_window &w) {
  // few enough rows of queries to a key head to read the keys once for all of them
  if ((int64_t)(Hq / Hkv) * Nq <= 32) return SHARED_ROWS;
  // Calls whose blocks of 128 queries leave most of the GPU idle wait for one chain of tiles after the other; blocks of 32,
  // whose four waves take a fourth of the keys each, have four times as many chains of half the length, but read every key
  // four times as often.  They are faster where they all run at once, for up to about 48 tiles each.  Us, D = 64 / 128, all
  // keys so far, blocks of 128 (in parts) and of 32: 2 heads of 128 queries on 1024 keys 16 and 12 / 18 and 16; 8 heads of
  // 1024 17 and 12 / 22 and 17; 8 of 1024 on 4096 27.5 and 27.8 / 33 and 54; 16 of 1024 19 and 15 / 26 and 22, on 3000 30 and
  // 34 / 40 and 64.  (At D = 128 the 512 blocks of 16 heads are two rounds, which the rule leaves to blocks of 128: 4 us more
  // on 1024 keys, 24 less on 3000.)
  const int64_t units = (int64_t)B * Hq * ((Nq + 31) / 32);
  if (units <= step_slots(D) && units * window_tiles(w, 32, Nk, STEP_KEYS) <= 48 * step_slots(D)) return BLOCKS_32;
  return BLOCKS_128;
}

// Pieces that the tiles of every block of queries are cut into.
int forward_parts(ForwardForm form, int B, int Hq, int Hkv, int Nq, int Nk, int D, const calibatt_window &w) {
  if (form != BLOCKS_128) {
    const bool shared = form == SHARED_ROWS;
    const int64_t units = shared ? (int64_t)B * Hkv : (int64_t)B * Hq * ((Nq + 31) / 32);
    const int64_t tiles = window_tiles(w, shared ? Nq : 32, Nk, STEP_KEYS);
    if (tiles <= 8 * STEP_WAVES) return 1;  // a second launch costs more than eight rounds of the waves
    // (few rows of one key head wait for HBM, and have two workgroups per CU one after the other)
    const int64_t fill = std::max<int64_t>(1, (shared ? 2 * WINDOW_CUS : step_slots(D)) / units);
    return (int)std::max<int64_t>(1, std::min<int64_t>({fill, (tiles + 2 * STEP_WAVES - 1) / (2 * STEP_WAVES), WINDOW_MAX_PARTS}));
  }
  const int64_t units = (int64_t)B * Hq * ((Nq + 127) / 128), tiles = window_tiles(w, 128, Nk, 64);
  // As many as fill the GPU, of eight tiles at least: 4 heads of 3000 tokens, all keys, 54 us whole, 37 in five parts; 16 heads
  // of 1024, D = 64, on 8192 keys 114 and, in four, 51, on 1024 keys 19.1 whole, 19.4 in two.
  const int64_t fill = 2 * WINDOW_CUS / units;
  return (int)std::max<int64_t>(1, std::min<int64_t>({fill, tiles / 8, WINDOW_MAX_PARTS}));
}

int64_t forward_bytes(int parts, int B, int Hq, int Nq, int D) {
  return parts > 1 ? (int64_t)parts * B * Hq * Nq * (D + 2) * 4 : 0;
}

int window_check(int B, int Hq, int Hkv, int Nq, int Nk, int D, const calibatt_window &w) {
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || Nq <= 0 || Nk <= 0 || D <= 0 || Hq % Hkv) return CALIBATT_ERR_SHAPE;
  if (Nq > 1 << 30 || Nk > 1 << 30 || w.left < -1 || w.right < -1 || w.sinks < 0 || w.frame <= 0) return CALIBATT_ERR_SHAPE;
  if (w.offset > 1 << 30 || w.offset < -(1 << 30)) return CALIBATT_ERR_SHAPE;
  if ((int64_t)B * Hq > 1 << 24 || (int64_t)B * Hq * Nq > 0x7fffffffLL || (int64_t)B * Hkv * Nk > 0x7fffffffLL) return CALIBATT_ERR_SHAPE;
  if (((uintptr_t)w.q_start | (uintptr_t)w.q_len | (uintptr_t)w.k_len) & 3) return CALIBATT_ERR_SHAPE;
  if (D != 64 && D != 128) return CALIBATT_ERR_UNSUPPORTED;
  return CALIBATT_OK;
}

// Strides of a tensor; those of an axis of one entry are never stepped along.  No two rows of an output may overlap.
bool window_strides(const calibatt_strides *given, int B, int H, int N, int D, bool output, Strides &s) {
  s = given ? Strides{given->b, given->h, given->n} : Strides{(int64_t)H * N * D, (int64_t)N * D, D};
  const int64_t sizes[3] = {B, H, N}, steps[3] = {s.b, s.h, s.n};
  if (output && !rows_apart(sizes, steps, D)) return false;
  if (B == 1) s.b = 0;
  if (H == 1) s.h = 0;
  if (N == 1) s.n = D;
  if (s.n < D || s.n > 0x7fffffff || s.b < 0 || s.h < 0 || s.n % 8 || s.h % 8 || s.b % 8) return false;
  // The kernels address the rows of one head with 32-bit byte offsets, also those behind the last one that a tile or a block
  // of 256 still has: they have to lie behind a descriptor's end, and not past 2^32 at the head's first rows again.
  return ((unsigned long long)N + 256) * (unsigned long long)s.n * 2 <= 0xffffffffULL;
}

void window_dims(int B, int Hq, int Hkv, int Nq, int Nk, const calibatt_window &w, float scale, WindowDims &p) {
  p = WindowDims{};
  p.B = B;
  p.Hq = Hq;
  p.Hkv = Hkv;
  p.Nq = Nq;
  p.Nk = Nk;
  p.left = w.left;
  p.right = w.right;
  p.sinks = std::min(w.sinks, Nk);
  p.frame = w.frame;
  p.offset = w.offset;
  p.q_start = w.q_start;
  p.q_len = w.q_len;
  p.k_len = w.k_len;
  p.scale = scale;
  p.scale_log2e = scale * 1.4426950408889634f;
  p.parts = 1;
}

template <int D, typename T>
int launch_forward(ForwardForm form, const uint16_t *q, const uint16_t *k, const uint16_t *v, uint16_t *out, float *lse,
                   const WindowDims &p, hipStream_t stream) {
  const int block = form == BLOCKS_128 ? 128 : 32;
  const int64_t units = (int64_t)p.B * (form == SHARED_ROWS ? p.Hkv : (int64_t)p.Hq * ((p.Nq + block - 1) / block)) * p.parts;
  if (units > MAX_GRID) return CALIBATT_ERR_SHAPE;
  const unsigned grid = (unsigned)(8 * ((units + 7) / 8));
  static DevInfo info[3];
  auto go = [&](auto kernel, int threads, int smem) {
    int unused = 0;
    const int st = prepare(kernel, threads, smem, info[form], unused);
    return st ? st : launch_kernel(kernel, grid, threads, smem, stream, q, k, v, out, lse, p);
  };
  constexpr int STEP_LDS = StepLds<D, T>::BYTES;
  const int st = form == SHARED_ROWS ? go(window_attn_step_kernel<D, true, T>, STEP_WAVES * 64, STEP_LDS)
                 : form == BLOCKS_32 ? go(window_attn_step_kernel<D, false, T>, STEP_WAVES * 64, STEP_LDS)
                                     : go(window_attn_fwd_kernel<D, T>, 256, WindowRow<D, T>::LDS_BYTES);
  if (st || p.parts == 1) return st;
  const int64_t rows = (int64_t)p.B * p.Hq * p.Nq;
  constexpr int PER_WG = 256 / (D / 8);
  if (rows <= 2 * WINDOW_CUS)
    return launch_kernel(window_attn_merge_kernel<D, 1, T>, (unsigned)rows, 256, 0, stream, out, lse, p);
  return launch_kernel(window_attn_merge_kernel<D, PER_WG, T>, (unsigned)((rows + PER_WG - 1) / PER_WG), 256, 0, stream, out, lse, p);
}

// ---- gradients ----------------------------------------------------------------------------------------------
// How the queries that see a block of 256 keys are cut into parts.  A block with sinks is seen by all later queries, so it
// gets parts as long as the others'.
struct GradPlan {
  int dq_parts, parts, sink_parts, sink_blocks;
  int do_slots, v_slots;  // pieces whose largest rows of dO and V are found apart (fp16)
  int64_t sums_bytes;     // of lse and delta of every query, and the sums of the parts
  int64_t bytes;          // of the workspace: those, and the sizes of the pieces
};
GradPlan grad_plan(int B, int Hq, int Hkv, int Nq, int Nk, int D, const calibatt_window &w) {
  GradPlan g;
  constexpr int BLOCK = 256, ROWS = 32, SLOTS = WINDOW_CUS;
  const int64_t blocks = (Nk + BLOCK - 1) / BLOCK, G = Hq / Hkv, heads = (int64_t)B * Hkv;
  g.sink_blocks = w.left < 0 ? 0 : (std::min(w.sinks, Nk) + BLOCK - 1) / BLOCK;
  const int64_t all = G * ((Nq + ROWS - 1) / ROWS);
  int64_t one = all;  // tiles of queries that see a block, without sinks
  if (w.left >= 0 && w.right >= 0) one = std::min<int64_t>(all, G * ((window_span(w, BLOCK, Nq) + ROWS - 1) / ROWS));
  // Rounds of workgroups times the length of a part, which costs so many tiles beside its own (its start, its sums to
  // memory and back).  All gradients, us, by parts: 8 heads on 4 of 16 380 tokens, nine frames of 780 and the first, 1 1900,
  // 2 1696, 3 1615, 4 1616 (chosen), 8 1671; 8 on 2 of 5027, 870 keys, 1 268, 4 132, 6 124 (chosen), 8 153; 4 of 3000, all
  // keys, 1 196, 4 109, 5 106 (chosen), 6 133; 40 of 1500 1 154 (chosen), 2 177.
  constexpr int64_t PART_COST = 12, ALONE = 4;
  double best = 0.0;
  g.parts = 0;
  for (int64_t parts = 1; parts <= WINDOW_MAX_PARTS && (parts == 1 || one / parts >= 8); ++parts) {
    const int64_t length = (one + parts - 1) / parts;
    const int64_t sink_parts = std::min<int64_t>(WINDOW_MAX_PARTS, (all + length - 1) / length);
    const int64_t sink_length = (all + sink_parts - 1) / sink_parts, longest = g.sink_blocks ? std::max(length, sink_length) : length;
    const int64_t units = heads * (g.sink_blocks * sink_parts + (blocks - g.sink_blocks) * parts);
    const double cost = (double)((units + SLOTS - 1) / SLOTS) * (double)(longest + (parts > 1 ? PART_COST : ALONE));
    if (g.parts && cost >= 0.97 * best) continue;
    best = cost;
    g.parts = (int)parts;
    g.sink_parts = (int)std::max<int64_t>(1, sink_parts);
  }
  // dQ: of a few blocks of queries the tiles of keys are cut, to eight at least (all gradients of 6 heads of 1801 tokens, all
  // keys so far: 107 us whole, 82 in four parts; 8 heads of 875, three frames of 134, D = 64: 51 and, in two, 45)
  const int64_t q_rows = (int64_t)B * Hq * Nq, q_units = (int64_t)B * Hq * ((Nq + 127) / 128);
  g.dq_parts = (int)std::max<int64_t>(1, std::min<int64_t>({2 * WINDOW_CUS / q_units, window_tiles(w, 128, Nk, ROWS) / 8, WINDOW_MAX_PARTS}));
  g.sums_bytes = (q_rows + 1) / 2 * 16 + (g.dq_parts > 1 ? g.dq_parts * q_rows * D * 4 : 0);
  const int64_t row = 2 * D * 4;
  if (g.parts > 1) g.sums_bytes += g.parts * heads * Nk * row;
  if (g.sink_blocks && g.sink_parts > 1) g.sums_bytes += g.sink_parts * heads * g.sink_blocks * BLOCK * row;
  g.do_slots = (int)std::min<int64_t>(SIZE_MAX_SLOTS, (G * Nq + SIZE_ROWS - 1) / SIZE_ROWS);
  g.v_slots = (int)std::min<int64_t>(SIZE_MAX_SLOTS, (Nk + SIZE_ROWS - 1) / SIZE_ROWS);
  g.bytes = g.sums_bytes + heads * (g.do_slots + g.v_slots) * 4;
  return g;
}

struct GradTensors {
  const uint16_t *dout, *q, *k, *v, *out;
  const float *lse;
  uint16_t *dq, *dk, *dv;
  float *stats;  // lse and delta as the second kernel wants them, [head][2][query]
};

template <int D, typename T>
int launch_backward(const GradTensors &t, const WindowDims &p, hipStream_t stream) {
  constexpr int BLOCK_Q = DqTile<D, T>::BLOCK, BLOCK = DkvTile<D, T>::BLOCK, DQ_LDS = dq_lds_bytes<D, T>(), DKV_LDS = dkv_lds_bytes<D, T>();
  static DevInfo dq_info, dkv_info;
  int unused = 0;
  if (int st = prepare(window_attn_dq_kernel<D, T>, 256, DQ_LDS, dq_info, unused)) return st;
  if (int st = prepare(window_attn_dkv_kernel<D, T>, 512, DKV_LDS, dkv_info, unused)) return st;
  const int64_t q_units = (int64_t)p.B * p.Hq * ((p.Nq + BLOCK_Q - 1) / BLOCK_Q) * p.dq_parts, blocks = (p.Nk + BLOCK - 1) / BLOCK;
  const int64_t k_units = (int64_t)p.B * p.Hkv * (p.n_sink_blocks * p.bwd_sink_parts + (blocks - p.n_sink_blocks) * p.bwd_parts);
  const int64_t cut = p.bwd_parts > 1 ? p.Nk : p.bwd_sink_parts > 1 ? std::min(p.Nk, p.n_sink_blocks * BLOCK) : 0;
  const int64_t sums = 2 * cut * p.B * p.Hkv + (p.dq_parts > 1 ? (int64_t)p.B * p.Hq * p.Nq : 0);
  const int64_t per_wg = 256 / (D / 8), sum_wgs = (sums + per_wg - 1) / per_wg;
  if (q_units > MAX_GRID || k_units > MAX_GRID || sum_wgs > MAX_GRID) return CALIBATT_ERR_SHAPE;
  if constexpr (GradScale<T>::FOLLOWS) {
    const int64_t pieces = (int64_t)p.B * p.Hkv * (p.do_slots + p.v_slots);
    if (pieces > MAX_GRID) return CALIBATT_ERR_SHAPE;
    if (int st = launch_kernel(window_attn_sizes_kernel<D>, (unsigned)pieces, 256, 0, stream, t.dout, t.v, p)) return st;
  }
  if (int st = launch_kernel(window_attn_dq_kernel<D, T>, (unsigned)(8 * ((q_units + 7) / 8)), 256, DQ_LDS, stream, t.dout, t.q, t.k,
                             t.v, t.out, t.lse, t.dq, t.stats, p))
    return st;
  if (int st = launch_kernel(window_attn_dkv_kernel<D, T>, (unsigned)(8 * ((k_units + 7) / 8)), 512, DKV_LDS, stream, t.dout, t.q,
                             t.k, t.v, (const float *)t.stats, t.dk, t.dv, p))
    return st;
  return sum_wgs ? launch_kernel(window_attn_grad_sum_kernel<D, T>, (unsigned)sum_wgs, 256, 0, stream, t.dq, t.dk, t.dv, p) : CALIBATT_OK;
}

}  // namespace

extern "C" int calibatt_window_attn_workspace_bytes(int B, int Hq, int Hkv, int Nq, int Nk, int D,
                                                    const calibatt_window *window, int64_t *forward, int64_t *backward) {
  if (!window || !forward || !backward) return CALIBATT_ERR_NULL;
  if (int st = window_check(B, Hq, Hkv, Nq, Nk, D, *window)) return st;
  const ForwardForm form = forward_form(B, Hq, Hkv, Nq, Nk, D, *window);
  *forward = forward_bytes(forward_parts(form, B, Hq, Hkv, Nq, Nk, D, *window), B, Hq, Nq, D);
  *backward = grad_plan(B, Hq, Hkv, Nq, Nk, D, *window).bytes;
  return CALIBATT_OK;
}

extern "C" int calibatt_window_attn_form(int B, int Hq, int Hkv, int Nq, int Nk, int D, const calibatt_window *window,
                                         calibatt_window_form *form) {
  if (!window || !form) return CALIBATT_ERR_NULL;
  if (int st = window_check(B, Hq, Hkv, Nq, Nk, D, *window)) return st;
  const ForwardForm forward = forward_form(B, Hq, Hkv, Nq, Nk, D, *window);
  const GradPlan g = grad_plan(B, Hq, Hkv, Nq, Nk, D, *window);
  *form = calibatt_window_form{forward, forward_parts(forward, B, Hq, Hkv, Nq, Nk, D, *window), g.dq_parts, g.parts, g.sink_parts,
                               g.sink_blocks};
  return CALIBATT_OK;
}

extern "C" int calibatt_window_attn_fwd(const void *q, const void *k, const void *v, void *out, float *lse, int B, int Hq,
                                        int Hkv, int Nq, int Nk, int D, const calibatt_window *window, float scale,
                                        const calibatt_strides *q_strides, const calibatt_strides *kv_strides,
                                        const calibatt_strides *out_strides, int dtype, void *workspace,
                                        int64_t workspace_bytes, void *stream) {
  if (!q || !k || !v || !out || !window) return CALIBATT_ERR_NULL;
  if (int st = window_check(B, Hq, Hkv, Nq, Nk, D, *window)) return st;
  if (dtype != CALIBATT_BF16 && dtype != CALIBATT_F16) return CALIBATT_ERR_UNSUPPORTED;
  if (out == q || out == k || out == v || !(scale - scale == 0.f)) return CALIBATT_ERR_SHAPE;
  WindowDims p;
  window_dims(B, Hq, Hkv, Nq, Nk, *window, scale, p);
  if (!window_strides(q_strides, B, Hq, Nq, D, false, p.q) || !window_strides(kv_strides, B, Hkv, Nk, D, false, p.kv) ||
      !window_strides(out_strides, B, Hq, Nq, D, true, p.out))
    return CALIBATT_ERR_SHAPE;
  if ((((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)out | (uintptr_t)workspace) & 15) || ((uintptr_t)lse & 3))
    return CALIBATT_ERR_SHAPE;
  const ForwardForm form = forward_form(B, Hq, Hkv, Nq, Nk, D, *window);
  if (workspace) {
    p.parts = forward_parts(form, B, Hq, Hkv, Nq, Nk, D, *window);
    if (workspace_bytes < forward_bytes(p.parts, B, Hq, Nq, D)) return CALIBATT_ERR_BUFFER_TOO_SMALL;
    p.part_rows = (float *)workspace;
    p.part_ml = p.part_rows + (size_t)p.parts * B * Hq * Nq * D;
  }
  const uint16_t *const q_ = (const uint16_t *)q, *const k_ = (const uint16_t *)k, *const v_ = (const uint16_t *)v;
  uint16_t *const o_ = (uint16_t *)out;
  hipStream_t s = (hipStream_t)stream;
  if (D == 128)
    return dtype == CALIBATT_BF16 ? launch_forward<128, Bf16>(form, q_, k_, v_, o_, lse, p, s)
                                  : launch_forward<128, F16>(form, q_, k_, v_, o_, lse, p, s);
  return dtype == CALIBATT_BF16 ? launch_forward<64, Bf16>(form, q_, k_, v_, o_, lse, p, s)
                                : launch_forward<64, F16>(form, q_, k_, v_, o_, lse, p, s);
}

extern "C" int calibatt_window_attn_bwd(const void *dout, const void *q, const void *k, const void *v, const void *out,
                                        const float *lse, void *dq, void *dk, void *dv, int B, int Hq, int Hkv, int Nq, int Nk,
                                        int D, const calibatt_window *window, float scale, const calibatt_strides *dout_strides,
                                        const calibatt_strides *q_strides, const calibatt_strides *kv_strides,
                                        const calibatt_strides *out_strides, const calibatt_strides *dq_strides,
                                        const calibatt_strides *dkv_strides, int dtype, void *workspace,
                                        int64_t workspace_bytes, void *stream) {
  if (!dout || !q || !k || !v || !out || !lse || !dq || !dk || !dv || !window || !workspace) return CALIBATT_ERR_NULL;
  if (int st = window_check(B, Hq, Hkv, Nq, Nk, D, *window)) return st;
  if (dtype != CALIBATT_BF16 && dtype != CALIBATT_F16) return CALIBATT_ERR_UNSUPPORTED;
  if (!(scale - scale == 0.f) || dk == dv) return CALIBATT_ERR_SHAPE;
  // the second kernel reads what the first has read, so no result may lie where an input does
  const void *const inputs[] = {dout, q, k, v, out, lse};
  for (const void *x : inputs)
    if (x == dq || x == dk || x == dv || x == workspace) return CALIBATT_ERR_SHAPE;
  if (dq == dk || dq == dv) return CALIBATT_ERR_SHAPE;
  WindowDims p;
  window_dims(B, Hq, Hkv, Nq, Nk, *window, scale, p);
  if (!window_strides(dout_strides, B, Hq, Nq, D, false, p.dout) || !window_strides(q_strides, B, Hq, Nq, D, false, p.q) ||
      !window_strides(kv_strides, B, Hkv, Nk, D, false, p.kv) || !window_strides(out_strides, B, Hq, Nq, D, false, p.out) ||
      !window_strides(dq_strides, B, Hq, Nq, D, true, p.dq) || !window_strides(dkv_strides, B, Hkv, Nk, D, true, p.dkv))
    return CALIBATT_ERR_SHAPE;
  uintptr_t at = 0;
  for (const void *x : {dout, q, k, v, out, (const void *)dq, (const void *)dk, (const void *)dv, (const void *)workspace}) at |= (uintptr_t)x;
  if ((at & 15) || ((uintptr_t)lse & 3)) return CALIBATT_ERR_SHAPE;
  const GradPlan g = grad_plan(B, Hq, Hkv, Nq, Nk, D, *window);
  if (workspace_bytes < g.bytes) return CALIBATT_ERR_BUFFER_TOO_SMALL;
  p.dq_parts = g.dq_parts;
  p.bwd_parts = g.parts;
  p.bwd_sink_parts = g.sink_parts;
  p.n_sink_blocks = g.sink_blocks;
  p.part_dq = (float *)workspace + ((int64_t)B * Hq * Nq + 1) / 2 * 4;
  p.part_dkv = p.part_dq + (g.dq_parts > 1 ? (int64_t)g.dq_parts * B * Hq * Nq * D : 0);
  p.sizes = (float *)((char *)workspace + g.sums_bytes);
  p.do_slots = g.do_slots;
  p.v_slots = g.v_slots;
  const GradTensors t = {(const uint16_t *)dout, (const uint16_t *)q, (const uint16_t *)k, (const uint16_t *)v,
                         (const uint16_t *)out, lse, (uint16_t *)dq, (uint16_t *)dk, (uint16_t *)dv, (float *)workspace};
  hipStream_t s = (hipStream_t)stream;
  if (D == 128) return dtype == CALIBATT_BF16 ? launch_backward<128, Bf16>(t, p, s) : launch_backward<128, F16>(t, p, s);
  return dtype == CALIBATT_BF16 ? launch_backward<64, Bf16>(t, p, s) : launch_backward<64, F16>(t, p, s);
}
