// Attention over a shared prefix and own caches: the join of the pieces, accumulated weights, and the entry points (kernels: prefix_attn.h).
#include "prefix_attn.h"

#include <cmath>

// ---------------------------------------------------------------------------------------------
// Join.  Bound by latency: launch, statistics, pieces, result (64 requests x 32 heads of 16 pieces of 64 dims, with the weights of 2048 own keys each, 42
// MB in all: 10 us; 32 x 32 heads of 7 pieces of 32 dims 3.5 us).  Threads are (piece, four dims): a thread weighs its pieces against the maximum of its
// own, four of them asked for at a time, before it is known how many there are (what counts is how many latencies follow on each other).  FEW pieces: W
// threads take a row by themselves.  Otherwise a workgroup does, and its threads of equal dims are added up against the row's maximum in a fixed order.
// ---------------------------------------------------------------------------------------------
// Pieces that the items left of the rows of request b from `in` on (a row of the request's): as prefix_item() cuts them.
__device__ __forceinline__ int prefix_pieces(const PrefixArgs& a, int b, int in, int kt, int row_tile) {
  const int tile0 = in / row_tile * row_tile;
  const int own_n = own_visible(own_len(a, b), a.L, (min(tile0 + row_tile, a.own_rows) - 1) / a.g);
  const int own_tiles = (own_n + kt - 1) / kt + (a.joint ? a.p_tiles : 0);
  return (a.joint ? 0 : a.p_chunks) + (own_tiles + a.o_chunk - 1) / a.o_chunk;
}
// The workgroups behind those of the rows add up the weights of 1024 own keys of a request each, from the scores that the items kept; the row
// statistics they need they join themselves.
__device__ void prefix_join_weights(const PrefixArgs& a, int kt, int row_tile, long long id) {
  __shared__ float lse2[32];
  const int per = (a.own_max + 1023) / 1024;
  const int bh = static_cast<int>(id / per), b = bh / a.h_kv, hk = bh - b * a.h_kv, first = static_cast<int>(id - static_cast<long long>(bh) * per) * 1024;
  const int n = own_len(a, b), lane = threadIdx.x & 63;
  if (first >= n) return;
  const int key = first + static_cast<int>(threadIdx.x) * 4;
  const PrefixScores early = prefix_scores(a, bh, 0, min(key, a.own_pad - 4));
  const floatx4 before = prefix_weights_before(a, bh, key, n);
  for (int r = threadIdx.x >> 6; r < a.own_rows; r += 4) {
    const float2* const ml = reinterpret_cast<const float2*>(a.part_ml) + (static_cast<long long>(hk) * a.rows + b * a.own_rows + r) * a.slots;
    const int pieces = prefix_pieces(a, b, r, kt, row_tile);
    float m = -INFINITY, l = 0.f;
    for (int i = lane; i < pieces; i += 64) {
      const float2 x = ml[i];
      const float top = fmaxf(m, x.x), ref = top == -INFINITY ? 0.f : top;
      l = l * __builtin_amdgcn_exp2f(m - ref) + x.y * __builtin_amdgcn_exp2f(x.x - ref);
      m = top;
    }
    const float top = wave_max(m), ref = top == -INFINITY ? 0.f : top;
    l = wave_sum(l * __builtin_amdgcn_exp2f(m - ref));
    if (lane == 0) lse2[r] = l == 0.f ? INFINITY : ref + __builtin_amdgcn_logf(l);
  }
  __syncthreads();
  if (key < n) prefix_weigh(a, bh, early, before, lse2, n, key);
}
template <int W, bool FEW>      // threads of a piece: kp_vo / 4 rounded up to a power of two
__global__ __launch_bounds__(256) void prefix_join_kernel(const PrefixArgs a, int kt, int row_tile, unsigned row_blocks) {
  constexpr int GROUPS = FEW ? 1 : 256 / W;      // threads of a row / W
  if (blockIdx.x >= row_blocks) return prefix_join_weights(a, kt, row_tile, blockIdx.x - row_blocks);
  const long long at = FEW ? static_cast<long long>(blockIdx.x) * (256 / W) + threadIdx.x / W : blockIdx.x;
  if (FEW && at >= static_cast<long long>(a.h_kv) * a.rows) return;
  const int hk = static_cast<int>(at / a.rows), row = static_cast<int>(at - static_cast<long long>(hk) * a.rows);
  const int token = row / a.g, b = token / a.L, head = hk * a.g + (row - token * a.g);
  const float2* const ml = reinterpret_cast<const float2*>(a.part_ml) + at * a.slots;
  const int grp = FEW ? 0 : threadIdx.x / W, lane = threadIdx.x % W, d = min(lane * 4, a.kv - 4);
  const float* const po = a.part_o + at * a.slots * a.kv + d;
  float m = -INFINITY, l = 0.f;
  floatx4 o = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = grp; i0 < a.slots; i0 += 4 * GROUPS) {
    float2 x[4];
    floatx4 p[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = min(i0 + j * GROUPS, a.slots - 1);
      x[j] = ml[i];
      p[j] = *reinterpret_cast<const floatx4*>(po + static_cast<long long>(i) * a.kv);
    }
    const int n = prefix_pieces(a, b, row - b * a.own_rows, kt, row_tile);
    float top = m;
#pragma unroll
    for (int j = 0; j < 4; ++j) {      // slots that no item wrote hold anything
      if (i0 + j * GROUPS >= n) x[j] = float2{-INFINITY, 0.f};
      top = fmaxf(top, x[j].x);
    }
    const float ref = top == -INFINITY ? 0.f : top, f = __builtin_amdgcn_exp2f(m - ref);
    m = top;
    l *= f;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] *= f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (x[j].y == 0.f) continue;      // no key seen; not by the maximum, which is -inf where all scores are NaN too
      const float w = __builtin_amdgcn_exp2f(x[j].x - ref);
      l += w * x[j].y;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += w * p[j][e];
    }
  }
  if constexpr (!FEW) {
    __shared__ floatx4 so[GROUPS][W];
    __shared__ float sm[GROUPS], sl[GROUPS];
    so[grp][lane] = o;
    if (lane == 0) { sm[grp] = m; sl[grp] = l; }
    __syncthreads();
    if (grp > 0) return;
    m = sm[0];
#pragma unroll
    for (int i = 1; i < GROUPS; ++i) m = fmaxf(m, sm[i]);
    const float ref = m == -INFINITY ? 0.f : m;
    l = 0.f;
    o = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      const float w = __builtin_amdgcn_exp2f(sm[i] - ref);
      const floatx4 p = so[i][lane];
      l += w * sl[i];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += w * p[e];
    }
  }
  if (lane * 4 < a.kv) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] *= inv;
    *reinterpret_cast<bf16x4_t*>(a.o + token * a.ld_o + static_cast<long long>(head) * a.kv + d) = __builtin_convertvector(o, bf16x4_t);
  }
  if (lane == 0 && a.lse)
    a.lse[(static_cast<long long>(b) * a.h + head) * a.L + (token - b * a.L)] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * LN2;
}

// ---------------------------------------------------------------------------------------------
// Weights: w_out[j] = w_in[j] + sum over the rows of the request that see own key j of exp(s_j - lse).  Keys stay in registers while the rows pass by from
// the first that sees a key, 32 at a time, the next ones on their way; S^T = K Q^T, so that the sum over rows is a sum over lanes, taken once at the end.
// MANY rows: 64 keys a workgroup, its wavefronts take the rows in turn.  Otherwise 32 keys a wavefront, and no key is read twice.  Bound by the latency
// of the rows' reads, then by the exponentials: 16 x 509 tokens of 32 heads on their own 509 keys 36 us, the attention itself 620.
// ---------------------------------------------------------------------------------------------
template <int DQ, bool MANY>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void prefix_weights_kernel(const PrefixArgs a, const float* lse, const float* w_in,
                                                                                                     float* w_out, int cap) {
  constexpr int KT = MANY ? 2 : 1, STEP = MANY ? 128 : 32;      // tiles of 32 keys; rows from one of a wavefront's tiles to its next
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), hh = lane >> 5, l32 = lane & 31;
  const int b = blockIdx.y / a.h_kv, hk = blockIdx.y - b * a.h_kv;
  const int n = own_len(a, b), k0 = MANY ? blockIdx.x * 64 : (blockIdx.x * 4 + wave) * 32;
  if (k0 >= n) return;
  const bf16_t* const kb = a.k + b * a.k_sb + hk * a.k_sh;
  bf16x8_t kf[KT][DQ / 16];
#pragma unroll
  for (int u = 0; u < KT; ++u)
#pragma unroll
    for (int c = 0; c < DQ / 16; ++c)
      kf[u][c] = *reinterpret_cast<const bf16x8_t*>(kb + min(k0 + 32 * u + l32, n - 1) * a.k_st + min(16 * c + 8 * hh, a.kq - 8));
  const int first = max(k0 - (n - a.L), 0) * a.g;      // the first token that sees key k0
  const int start = first + (MANY ? 32 * wave : 0) + l32, step_t = STEP / a.g, step_i = STEP - step_t * a.g;
  int t = start / a.g, i = start - t * a.g;      // the lane's row: token and query head of the group
  const auto load = [&](u32x4 (&x)[DQ / 16], float& ref) __attribute__((always_inline)) {      // rows behind the last: the last one
    const int head = hk * a.g + (t < a.L ? i : a.g - 1), tt = min(t, a.L - 1);
    const bf16_t* const src = a.q + (static_cast<long long>(b) * a.L + tt) * a.ld_q + static_cast<long long>(head) * a.kq;
#pragma unroll
    for (int c = 0; c < DQ / 16; ++c) x[c] = *reinterpret_cast<const u32x4*>(src + min(16 * c + 8 * hh, a.kq - 8));
    ref = lse[(static_cast<long long>(b) * a.h + head) * a.L + tt];
  };
  float sum[KT][16] = {};
  u32x4 next[DQ / 16];
  float next_ref;
  load(next, next_ref);
  for (int r0 = start - l32; r0 < a.own_rows; r0 += STEP) {
    bf16x8_t qf[DQ / 16];
#pragma unroll
    for (int c = 0; c < DQ / 16; ++c) qf[c] = __builtin_bit_cast(bf16x8_t, 16 * c + 8 * hh < a.kq ? next[c] : u32x4{0u, 0u, 0u, 0u});
    const float ref = next_ref * LOG2E;
    const int left = (t < a.L ? own_visible(n, a.L, t) : 0) - k0;      // keys from k0 on that the row sees
    t += step_t;
    i += step_i;
    while (i >= a.g) { i -= a.g; ++t; }
    if (r0 + STEP < a.own_rows) load(next, next_ref);
    const bool whole = __builtin_amdgcn_ballot_w64(left < 32 * KT) == 0ull;
#pragma unroll
    for (int u = 0; u < KT; ++u) {
      floatx16 s = {};
#pragma unroll
      for (int c = 0; c < DQ / 16; ++c) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[u][c], qf[c], s, 0, 0, 0);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], a.sc, -ref));
        sum[u][e] += whole || 32 * u + 8 * (e / 4) + 4 * hh + e % 4 < left ? p : 0.f;
      }
    }
  }
  float total = 0.f;      // without MANY: lane e of either half keeps the sum of register e
  __shared__ float all[4][32 * KT];
#pragma unroll
  for (int u = 0; u < KT; ++u)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float x = row16_sum(sum[u][e]);
      const float y = x + __shfl_xor(x, 16);
      if (!MANY) total = l32 == e ? y : total;
      else if (l32 == 0) all[wave][32 * u + 8 * (e / 4) + 4 * hh + e % 4] = y;
    }
  int j = k0 + 8 * (l32 / 4) + 4 * hh + l32 % 4;
  bool writes = l32 < 16;
  if constexpr (MANY) {
    __syncthreads();
    j = k0 + lane;
    writes = wave == 0;
    total = (all[0][lane] + all[1][lane]) + (all[2][lane] + all[3][lane]);
  }
  const long long at = static_cast<long long>(blockIdx.y) * cap + j;
  if (writes && j < n) w_out[at] = (w_in ? w_in[at] : 0.f) + total;
}

// ---------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------
static int prefix_width(int kp) { return kp <= 32 ? 32 : (kp <= 64 ? 64 : 128); }
static int rows_of(int kind) { return 16 << kind; }
static int kind_of(int rows) { return rows <= 16 ? ROWS_16 : (rows <= 32 ? ROWS_32 : (rows <= 64 ? ROWS_64 : ROWS_128)); }
static int keys_of(int kind) { return kind >= ROWS_64 ? 64 : 32; }       // keys of a tile
static int tiles_at_once(int kind) { return kind >= ROWS_64 ? 1 : 4; }   // tiles that a workgroup works on

struct PrefixPlan {
  int dq, dv, own, prefix;
  unsigned grid, weigh;      // workgroups of the items, and of the weights in the join
  size_t part_o, part_ml, lse, scores;      // bytes of workspace
};

// What the items of a call cost, in ns, for the choice between ways to cut it.  Constants as measured: an item's start and end 3 us, a step's least time (a
// latency of memory and what a compute unit can take in, or a tile of a wavefront that has a SIMD for itself: 1.4 us for 32 rows of 64 + 64 dims), 5.5
// bytes/ps of memory over all workgroups (`share` of them read the same keys), and a row and key of a tile on a compute unit (heads of 64 + 64 dims 0.08
// ns; the unused rows of a tile cost as much).  keys: of the item; active: workgroups at work, `alike` of them such items.  How good the choice is: with
// the chunks of the prefix forced to other counts (8 to 48, 1 and 2 of own keys) it is the best for 12 x 5 tokens on 8191 and for 8 on 2000, within 1 % for
// 64 on 32768, but 5 % off the best with weights (15 chosen, 12 best), and 8 % off for 32 on 4096 (6 chosen, 3 best): the model has no term for a last
// round of workgroups that is partly filled.  Joint items or items apart forced over 200 random shapes: 1.4 % lost in the mean, 39 % at most.
struct ItemCost { double step, item; };
static ItemCost item_cost(const PrefixArgs& a, const PrefixPlan& p, int kind, double steps, double keys, double active, double alike, double share) {
  const double per_cu = std::ceil(alike / 256), step_keys = keys_of(kind) * tiles_at_once(kind);
  const double pair = (0.02 + 0.0005 * (p.dq + p.dv)) * (kind == ROWS_256 ? 0.92 : 1);
  const double memory = active * (keys < step_keys ? keys : step_keys) * (a.kq + a.kv) * 2 / (5500 * share);
  const double compute = per_cu * rows_of(kind) * step_keys * pair;
  const double of_kind = kind == ROWS_64 ? 0.7 : (kind == ROWS_128 ? 1 : 1.7);
  double step = kind >= ROWS_64 ? of_kind * (600 + 6 * (p.dq + p.dv)) : std::fmax(700, 7 * (a.kq + a.kv));      // a wavefront by itself
  if (memory > step) step = memory;
  if (compute > step) step = compute;
  return {step, 3000 + steps * step};
}
static double join_cost(const PrefixArgs& a, int slots) {
  return slots > 1 ? 4000 + static_cast<double>(a.h_kv) * a.rows * slots * (a.kv + 2) * 8 / 5000 : 0;
}
static inline long long ceil_div(long long x, long long y) { return (x + y - 1) / y; }

// LDS of an item whose wavefronts take `steps` tiles each, as PrefixShape has it (an upper bound on the stages will do).
static int lds_of(const PrefixPlan& p, int kind, long long steps, int stages) {
  return static_cast<int>(steps < stages ? (steps > 0 ? steps : 1) : stages) * keys_of(kind) * tiles_at_once(kind) * (p.dq + p.dv) * 2;
}
// Workgroups at work at once, by LDS and by the registers of their kind.  Items of a single step hold one stage, which leaves room for twice as many (60
// x 4 tokens on 4 own keys, 16 heads of 128 + 128 dims, 15.8 -> 9.8 us; 89 tokens on 49 + 1 keys, 32 heads of 48 + 48 dims, 23.9 -> 16.4).
static long long resident_of(const PrefixPlan& p, int kind, int lds) {
  const int dims = p.dq + p.dv, by_lds = lds > 0 ? 160 * 1024 / lds : 4;
  const int by_regs = kind == ROWS_256 ? 2 : (kind == ROWS_128 ? (dims <= 64 ? 4 : (dims <= 128 ? 3 : 2)) : (dims <= 128 ? 4 : (kind == ROWS_32 ? 2 : 3)));
  const int n = by_lds < by_regs ? by_lds : by_regs;
  return 256ll * (n > 0 ? n : 1);
}

// Items that run over the prefix and then the own keys of their request: `chunks` of them per tile of rows.
static double plan_joint(PrefixArgs& a, PrefixPlan& p, bool set) {
  const int kt = keys_of(p.own), at_once = tiles_at_once(p.own);
  const long long pairs = static_cast<long long>(a.B) * a.h_kv * a.o_row_tiles;
  const long long tiles = ceil_div(a.P, kt) + ceil_div(a.own_max, kt), steps = ceil_div(tiles, at_once);
  double best = 0;
  long long best_chunk = 0;
  for (long long chunks = 1; chunks <= 64 && (chunks == 1 || ceil_div(steps, chunks) >= 2); chunks += (chunks < 8 ? 1 : chunks / 4)) {
    const long long chunk = steps > 0 ? ceil_div(steps, chunks) : 1, n = steps > 0 ? ceil_div(steps, chunk) : 1, wgs = pairs * n;
    const long long resident = resident_of(p, p.own, lds_of(p, p.own, chunk, 2));
    const double active = static_cast<double>(wgs < resident ? wgs : resident), rounds = wgs <= resident ? 1 : static_cast<double>(wgs) / resident + 0.15;
    const ItemCost c = item_cost(a, p, p.own, static_cast<double>(chunk), static_cast<double>(a.P + a.own_max) / n, active, active, a.o_row_tiles);
    const double cost = rounds * c.item + join_cost(a, static_cast<int>(n));
    if (best_chunk == 0 || cost < best) { best = cost; best_chunk = chunk; }
  }
  if (set) {
    p.prefix = p.own;
    a.joint = 1;
    a.p_items = a.p_chunks = a.p_chunk = a.p_row_tiles = 0;
    a.p_tiles = static_cast<int>(ceil_div(a.P, kt));
    a.o_chunk = static_cast<int>(best_chunk * at_once);
    a.o_chunks = tiles > 0 ? static_cast<int>(ceil_div(tiles, a.o_chunk)) : 1;
    a.slots = a.o_chunks > 1 ? a.o_chunks : 0;
    a.o_stages = a.p_stages = static_cast<int>(best_chunk < 4 ? best_chunk : 4);
  }
  return best;
}
// Items of the prefix for the rows of all requests, and items of own keys.
static double plan_apart(PrefixArgs& a, PrefixPlan& p, bool set) {
  const int prefix = kind_of(a.rows) < p.own ? p.own : kind_of(a.rows), kt_p = keys_of(prefix), at_once_p = tiles_at_once(prefix);
  const int kt = keys_of(p.own), at_once = tiles_at_once(p.own);
  const long long row_tiles = ceil_div(a.rows, rows_of(prefix)), pairs = static_cast<long long>(a.B) * a.h_kv * a.o_row_tiles;
  const long long p_steps = ceil_div(ceil_div(a.P, kt_p), at_once_p), o_steps = ceil_div(ceil_div(a.own_max, kt), at_once);
  double best = 0;
  long long best_p = 0, best_o = 0;
  for (long long pc = 1; pc <= 128 && (pc == 1 || ceil_div(p_steps, pc) >= 2); pc += (pc < 8 ? 1 : pc / 4))
    for (long long oc = 1; oc <= 32 && (oc == 1 || ceil_div(o_steps, oc) >= 2); oc *= 2) {
      const long long p_chunk = ceil_div(p_steps, pc), o_chunk = o_steps > 0 ? ceil_div(o_steps, oc) : 1;
      const long long p_n = ceil_div(p_steps, p_chunk), o_n = ceil_div(o_steps, o_chunk);
      const double p_wgs = static_cast<double>(a.h_kv * row_tiles * p_n), o_wgs = static_cast<double>(pairs * o_n), wgs = p_wgs + o_wgs;
      const int lds_p = lds_of(p, prefix, p_chunk, prefix >= ROWS_64 && p.own < ROWS_64 ? 4 : 2), lds_o = lds_of(p, p.own, o_chunk, 2);
      const long long resident = resident_of(p, prefix, lds_p > lds_o ? lds_p : lds_o);
      const double active = wgs < resident ? wgs : static_cast<double>(resident);
      const double p_keys = static_cast<double>(a.P) / p_n, o_keys = static_cast<double>(a.own_max) / (o_n > 0 ? o_n : 1);
      const ItemCost cp = item_cost(a, p, prefix, static_cast<double>(p_chunk), p_keys, active, active * p_wgs / wgs, static_cast<double>(row_tiles));
      const ItemCost co = item_cost(a, p, p.own, static_cast<double>(o_chunk), o_keys, active, active * o_wgs / wgs, 1);
      const double longest = cp.item > co.item ? cp.item : co.item, all = (p_wgs * cp.item + o_wgs * co.item) / resident;
      const double cost = (all > longest ? all + longest / 4 : longest) + join_cost(a, static_cast<int>(p_n + o_n));
      if (best_p == 0 || cost < best) { best = cost; best_p = p_chunk; best_o = o_chunk; }
    }
  if (set) {
    p.prefix = prefix;
    a.joint = 0;
    a.p_tiles = static_cast<int>(ceil_div(a.P, kt_p));
    a.p_row_tiles = static_cast<int>(row_tiles);
    a.p_chunk = static_cast<int>(best_p * at_once_p);
    a.p_chunks = static_cast<int>(ceil_div(a.p_tiles, a.p_chunk));
    a.p_items = a.p_chunks * a.p_row_tiles * a.h_kv;
    a.o_chunk = static_cast<int>(best_o * at_once);
    a.o_chunks = static_cast<int>(ceil_div(ceil_div(a.own_max, kt), a.o_chunk));
    a.slots = a.p_chunks + a.o_chunks;
    a.p_stages = static_cast<int>(best_p < 4 ? best_p : 4);
    a.o_stages = static_cast<int>(best_o < 4 ? best_o : 4);
    if (prefix == p.own && a.o_stages < a.p_stages) a.o_stages = a.p_stages;
  }
  return best;
}

// Fills the item fields of `a` (shapes are set) and the plan.
static bool prefix_plan(PrefixArgs& a, PrefixPlan& p, bool weights) {
  p.dq = prefix_width(a.kq);
  p.dv = prefix_width(a.kv);
  p.own = kind_of(a.own_rows);
  a.o_row_tiles = static_cast<int>(ceil_div(a.own_rows, rows_of(p.own)));
  const long long rows = static_cast<long long>(a.h_kv) * a.rows;
  if (static_cast<long long>(a.B) * a.h_kv * a.o_row_tiles * 64 > 0x7fffffffll || rows * 128 > 0x7fffffffll * 64) return false;
  // Rows of a request that fill a tile of their own, a batch of one or no prefix: nothing to gain by putting requests together.
  const bool only_joint = a.B == 1 || a.P == 0 || p.own >= ROWS_64;
  // Wide heads apart: own tiles for every wavefront take so much LDS that one workgroup is left to a compute unit; shared tiles leave two, and a
  // wavefront with the few rows keeps up with memory (12 x 5 tokens on 8191, 96 and 128 dims: 49 -> 44 us; 64 and 64 dims: no difference).
  const int own = p.own, apart_own = prefix_wide(p.dq, p.dv) ? ROWS_64 : p.own;
  const double joint = only_joint ? 0 : plan_joint(a, p, false);
  p.own = apart_own;
  if (!only_joint && plan_apart(a, p, false) < joint) {
    plan_apart(a, p, true);
  } else {
    p.own = own;
    plan_joint(a, p, true);
    // Prompts: 64 rows a wavefront halve the reads of LDS, where narrow heads leave the registers.  A compute unit holds two such workgroups.  From two
    // rounds of them on, at equal padding, against items of 128 rows: 0.93 to 0.95 of the time with 64 + 64 dims and 4096 prefix keys or more, 0.94 to
    // 0.97 with 96 in all, 0.95 to 1.01 with 1000; but 1.06 with 500 + 250 keys; with 32 + 32 dims 1.06 with 1000, 0.98 to 1.01 with 4096, 0.98 with 8192.
    // One more of the 128-row tiles padded is lost (300 rows, 2000 + 400 keys: 265 us against 180).  Under two rounds it depends on how full the last is (509
    // tokens of 4 query heads on 8192 keys, 512 / 640 / 768 / 896 / 960 workgroups: 0.92 / 1.10 / 0.95 / 1.03 / 0.94): left with 128.
    const long long tiles_256 = ceil_div(a.own_rows, 256), keys = static_cast<long long>(a.P) + a.own_max;
    if (own == ROWS_128 && !prefix_wide(p.dq, p.dv) && a.slots == 0 && static_cast<long long>(a.B) * a.h_kv * tiles_256 >= 2 * 2 * 256 &&
        a.o_row_tiles == 2 * tiles_256 && keys >= (p.dq + p.dv > 64 ? 1024 : 4096)) {
      p.own = ROWS_256;
      a.o_row_tiles = static_cast<int>(tiles_256);
      plan_joint(a, p, true);
    }
  }
  // Keys that no other item reads, and more of them than the last cache (256 MB) keeps until a next call, by own_max where lengths are on the device
  // (short caches under a far larger own_max give up what the cache would have kept: the header says so): their loads pass the caches by.  Own
  // caches of 134 MB 27.5 -> 23.9 us, 100 MB 21.6 -> 19.9, 268 MB 51.4 -> 44.5; a prefix of 268 MB 55.0 -> 48.0.  With 67 MB it depends on what
  // passes between two calls: 17.2 -> 15.2 where the cache had lost them, 14.0 -> 14.9 where it had not.
  const auto once = [&](double heads, double keys, int row_tiles) { return row_tiles == 1 && heads * keys * (a.kq + a.kv) * 2 > 96e6; };
  a.own_once = once(static_cast<double>(a.B) * a.h_kv, a.own_max, a.o_row_tiles);
  a.prefix_once = once(a.h_kv, a.P, a.joint ? a.B * a.o_row_tiles : a.p_row_tiles);
  // the kernels cut the keys as the plan did
  if (a.p_tiles != ceil_div(a.P, keys_of(p.prefix)) || p.prefix < p.own) return false;
  const auto held = [](int stages, int chunk, int kind) { return stages >= 4 || ceil_div(chunk, tiles_at_once(kind)) <= stages; };
  if (!held(a.o_stages, a.o_chunk, p.own) || !held(p.prefix == p.own ? a.o_stages : a.p_stages, a.p_chunk, p.prefix)) return false;
  // The weights need every own score against a sum that is complete only at the end.  Kept scores are written and read, 8 bytes a row and key;
  // without them the keys are read a second time, 2 kp_qk bytes a key, in a launch of its own.
  const bool keep = weights && a.own_rows <= 32 && a.own_max > 0 && 4 * a.own_rows <= a.kq;
  const long long weigh = keep && a.slots ? static_cast<long long>(a.B) * a.h_kv * ceil_div(a.own_max, 1024) : 0;
  const long long grid = a.p_items + static_cast<long long>(a.B) * a.h_kv * a.o_row_tiles * a.o_chunks;
  if (grid > 0x7fffffffll || rows + weigh > 0x7fffffffll || static_cast<long long>(a.p_chunks) * a.p_row_tiles * a.h_kv > 0x7fffffffll) return false;
  p.grid = static_cast<unsigned>(grid);
  p.weigh = static_cast<unsigned>(weigh);
  const size_t pieces = static_cast<size_t>(rows) * a.slots;
  p.part_o = pieces * a.kv * sizeof(float);
  p.part_ml = pieces * 2 * sizeof(float);
  a.own_pad = static_cast<int>(ceil_div(a.own_max, 64) * 64);
  p.scores = keep ? static_cast<size_t>(rows) * a.own_pad * sizeof(float) : 0;
  p.lse = weights && !keep ? static_cast<size_t>(a.B) * a.L * a.h * sizeof(float) : 0;
  return true;
}

#define JOIN_INSTANTIATE(W)                                                             \
  template __global__ void prefix_join_kernel<W, false>(const PrefixArgs, int, int, unsigned); \
  template __global__ void prefix_join_kernel<W, true>(const PrefixArgs, int, int, unsigned);
JOIN_INSTANTIATE(8) JOIN_INSTANTIATE(16) JOIN_INSTANTIATE(32)
#undef JOIN_INSTANTIATE
template <int W>
static void prefix_join_launch(const PrefixArgs& a, const PrefixPlan& p, hipStream_t st) {
  const long long rows = static_cast<long long>(a.h_kv) * a.rows;
  // Few pieces, or enough rows that W threads each keep the chip busy (32 requests, 32 heads, 7 pieces: 22.6 -> 21.0 us for the call; 60 tokens, 32
  // heads, 11 pieces of 128 dims 44.1 -> 42.8; but 256 rows of 10 pieces 9.5 -> 10.3, and 2048 rows of 28 pieces 41.3 -> 42.8).
  const bool few = a.slots <= 4 || (a.slots <= 16 && rows >= 1024);
  const unsigned blocks = static_cast<unsigned>(few ? (rows + 256 / W - 1) / (256 / W) : rows);
  const auto kern = few ? prefix_join_kernel<W, true> : prefix_join_kernel<W, false>;
  hipLaunchKernelGGL(kern, dim3(blocks + p.weigh), dim3(256), 0, st, a, keys_of(p.own), rows_of(p.own), blocks);
}
template __global__ void prefix_weights_kernel<32, false>(const PrefixArgs, const float*, const float*, float*, int);
template __global__ void prefix_weights_kernel<32, true>(const PrefixArgs, const float*, const float*, float*, int);
template __global__ void prefix_weights_kernel<64, false>(const PrefixArgs, const float*, const float*, float*, int);
template __global__ void prefix_weights_kernel<64, true>(const PrefixArgs, const float*, const float*, float*, int);
template __global__ void prefix_weights_kernel<128, false>(const PrefixArgs, const float*, const float*, float*, int);
template __global__ void prefix_weights_kernel<128, true>(const PrefixArgs, const float*, const float*, float*, int);

int ecospa_cache_check(const ecospa_cache* c) {
  if (!c || !c->k || !c->v || !c->lens || (c->P > 0 && (!c->pk || !c->pv))) return ECOSPA_ERR_NULL;
  if (c->dtype != ECOSPA_BF16) return ECOSPA_ERR_DTYPE;
  if (c->B < 1 || c->h_kv < 1 || c->h < c->h_kv || c->h % c->h_kv || c->cap < 1 || c->own_max < 0 || c->own_max > c->cap || c->P < 0) return ECOSPA_ERR_SHAPE;
  if (c->kp_qk < 16 || c->kp_qk > 128 || c->kp_qk % 16 || c->kp_vo < 16 || c->kp_vo > 128 || c->kp_vo % 16) return ECOSPA_ERR_SHAPE;
  if (!(c->scale > 0.f) || c->scale > 2.0e38f) return ECOSPA_ERR_SHAPE;
  const long long rows[4] = {c->k_st, c->v_st, c->P > 0 ? c->pk_st : 1ll << 20, c->P > 0 ? c->pv_st : 1ll << 20};
  for (int i = 0; i < 4; ++i)      // 64 rows of a tile stay within 32 bits of bytes
    if (rows[i] < (i & 1 ? c->kp_vo : c->kp_qk) || rows[i] >= 1ll << 25) return ECOSPA_ERR_SHAPE;
  if (c->k_sb < 0 || c->k_sh < 0 || c->v_sb < 0 || c->v_sh < 0 || (c->P > 0 && (c->pk_sh < 0 || c->pv_sh < 0))) return ECOSPA_ERR_SHAPE;
  if (!aligned16(c->k) || !aligned16(c->v) || (c->k_sb | c->k_sh | c->k_st | c->v_sb | c->v_sh | c->v_st) % 8) return ECOSPA_ERR_ALIGN;
  if (c->P > 0 && (!aligned16(c->pk) || !aligned16(c->pv) || (c->pk_sh | c->pk_st | c->pv_sh | c->pv_st) % 8)) return ECOSPA_ERR_ALIGN;
  return ECOSPA_OK;
}
static int prefix_args(const ecospa_cache* c, int L, PrefixArgs& a, PrefixPlan& p, bool weights) {
  if (L < 1 || static_cast<long long>(c->B) * L * c->h > (1ll << 30) || static_cast<long long>(c->B) * c->h_kv > 65535) return ECOSPA_ERR_SHAPE;
  memset(&a, 0, sizeof(a));
  memset(&p, 0, sizeof(p));
  a.k = static_cast<const bf16_t*>(c->k); a.v = static_cast<const bf16_t*>(c->v);
  a.pk = static_cast<const bf16_t*>(c->P > 0 ? c->pk : c->k); a.pv = static_cast<const bf16_t*>(c->P > 0 ? c->pv : c->v);
  a.lens = c->lens;
  a.k_sb = c->k_sb; a.k_sh = c->k_sh; a.k_st = c->k_st; a.v_sb = c->v_sb; a.v_sh = c->v_sh; a.v_st = c->v_st;
  if (c->P > 0) { a.pk_sh = c->pk_sh; a.pk_st = c->pk_st; a.pv_sh = c->pv_sh; a.pv_st = c->pv_st; }
  a.B = c->B; a.L = L; a.h = c->h; a.h_kv = c->h_kv; a.g = c->h / c->h_kv; a.kq = c->kp_qk; a.kv = c->kp_vo; a.P = c->P; a.own_max = c->own_max;
  a.sc = c->scale * LOG2E;
  a.own_rows = L * a.g;
  a.rows = c->B * a.own_rows;
  return prefix_plan(a, p, weights) ? ECOSPA_OK : ECOSPA_ERR_SHAPE;
}

// How the launches cut a call (for tests): the fields in the order below; 0 where the call would be refused.
int prefix_attn_cut(const ecospa_cache& cache, int L, int weights, int* out) {
  PrefixArgs a;
  PrefixPlan p;
  if (ecospa_cache_check(&cache) != ECOSPA_OK || prefix_args(&cache, L, a, p, weights != 0) != ECOSPA_OK) return 0;
  const int fields[] = {a.joint, a.p_tiles, a.p_chunks, a.p_chunk, a.p_row_tiles, a.p_items, a.o_chunks, a.o_chunk, a.o_row_tiles, a.slots, p.own, p.prefix,
                        static_cast<int>(p.grid), static_cast<int>(p.weigh), a.own_pad, p.scores > 0};
  for (size_t i = 0; i < sizeof(fields) / sizeof(fields[0]); ++i) out[i] = fields[i];
  return static_cast<int>(sizeof(fields) / sizeof(fields[0]));
}

extern "C" size_t ecospa_prefix_attn_workspace_bytes(const ecospa_cache* cache, int L, int with_weights) {
  PrefixArgs a;
  PrefixPlan p;
  if (ecospa_cache_check(cache) != ECOSPA_OK || prefix_args(cache, L, a, p, with_weights != 0) != ECOSPA_OK) return 0;
  return align_up(p.part_o, 256) + align_up(p.part_ml, 256) + align_up(p.lse, 256) + align_up(p.scores, 256);
}

extern "C" int ecospa_prefix_attn(ecospa_ctx* ctx, const ecospa_cache* cache, int L, const void* q, long long ld_q, void* o, long long ld_o,
                                  float* lse, const float* weights_in, float* weights_out) {
  if (!ctx || !q || !o || (weights_in && !weights_out)) return ECOSPA_ERR_NULL;
  int rc = ecospa_cache_check(cache);
  if (rc != ECOSPA_OK) return rc;
  PrefixArgs a;
  PrefixPlan p;
  rc = prefix_args(cache, L, a, p, weights_out != nullptr);
  if (rc != ECOSPA_OK) return rc;
  if (ld_q < static_cast<long long>(a.h) * a.kq || ld_o < static_cast<long long>(a.h) * a.kv) return ECOSPA_ERR_SHAPE;
  if (!aligned16(q) || !aligned16(o) || ld_q % 8 || ld_o % 8) return ECOSPA_ERR_ALIGN;
  WsCarver ws(ctx->ws, ctx->ws_bytes);
  if (p.part_o) {
    a.part_o = static_cast<float*>(ws.take(p.part_o));
    a.part_ml = static_cast<float*>(ws.take(p.part_ml));
  }
  if (p.scores) a.scores = static_cast<float*>(ws.take(p.scores));
  if (p.lse && !lse) lse = static_cast<float*>(ws.take(p.lse));
  if (ws.off > 0 && !ws.ok()) return ECOSPA_ERR_WORKSPACE;
  a.q = static_cast<const bf16_t*>(q); a.ld_q = ld_q; a.o = static_cast<bf16_t*>(o); a.ld_o = ld_o; a.lse = lse;
  a.w_in = weights_in; a.w_out = weights_out; a.cap = cache->cap;
  const hipError_t e = p.dq == 32 ? prefix_launch_32(a, p.dv, p.own, p.prefix, p.grid, ctx->stream)
                     : p.dq == 64 ? prefix_launch_64(a, p.dv, p.own, p.prefix, p.grid, ctx->stream)
                                  : prefix_launch_128(a, p.dv, p.own, p.prefix, p.grid, ctx->stream);
  if (e != hipSuccess) return hip_fail(ctx, e, "prefix_attn_kernel");
  if (a.slots) {
    if (a.kv <= 32) prefix_join_launch<8>(a, p, ctx->stream);
    else if (a.kv <= 64) prefix_join_launch<16>(a, p, ctx->stream);
    else prefix_join_launch<32>(a, p, ctx->stream);
    ECOSPA_CHECK_LAUNCH(ctx, "prefix_join_kernel");
  }
  if (p.lse && a.own_max > 0) {
    // whole calls, MANY against not: 512 rows (8 x 8 heads, 128 tokens) 20.0 us / 24.1, 2048 rows 58.8 / 76.1, 512 rows of single heads 108.3 / 108.5; but
    // 256 rows of single heads 40.2 / 30.4 and 33 rows 25.9 / 18.1
    const bool many = a.own_rows >= 512;
    const dim3 grid((a.own_max + (many ? 63 : 127)) / (many ? 64 : 128), a.B * a.h_kv);
    const auto few_kern = p.dq == 32 ? prefix_weights_kernel<32, false> : (p.dq == 64 ? prefix_weights_kernel<64, false> : prefix_weights_kernel<128, false>);
    const auto many_kern = p.dq == 32 ? prefix_weights_kernel<32, true> : (p.dq == 64 ? prefix_weights_kernel<64, true> : prefix_weights_kernel<128, true>);
    const auto kern = many ? many_kern : few_kern;
    hipLaunchKernelGGL(kern, grid, dim3(256), 0, ctx->stream, a, lse, weights_in, weights_out, cache->cap);
    ECOSPA_CHECK_LAUNCH(ctx, "prefix_weights_kernel");
  }
  return ECOSPA_OK;
}
