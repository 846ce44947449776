// Attention of a few new tokens of B requests over a prefix that all of them share and over caches of their own, on compact heads.
//
// With s_j = scale q.k_j over the P prefix keys and the own keys that the query sees, o = sum_j exp(s_j - lse) v_j, lse = log sum_j exp(s_j).
// Both sums are carried over tiles of keys against a running maximum (m, l, O), and pieces of them over disjoint keys join exactly:
// (m, l, O) + (m', l', O') = (M, l e^(m-M) + l' e^(m'-M), O e^(m-M) + O' e^(m'-M)).
//
// The prefix is the same for every request, so the rows of a key/value head - query heads of its group x new tokens x requests - are one
// matrix and every prefix key is read once for all of them; the own caches are read once each for the rows of their request.  Work is cut
// into items (rows x range of keys, prefix or own); items of the same rows leave (m, l, O) in the workspace and a second launch joins them.
//
// Layout: scores are computed transposed on v_mfma_f32_16x16x32_bf16, S^T = K Q^T (16 keys x 16 rows): a row of the softmax is a lane's
// column, and the four result registers of two key tiles are, rounded to bf16, the B operand of O^T = V^T P^T without going through LDS.
// The matching V^T operand comes from transposing LDS reads.  Columns of 16 rather than 32: most calls have few rows (a token of a request
// is g = h / h_kv rows), and the exponentials of unused columns are the largest cost beside the memory.
//
// Rounding: scores, maxima, sums and accumulators are fp32; the probabilities enter the second product rounded to bf16 (the matrix
// unit's type), the denominator is summed from the unrounded ones, so that lse and the weights keep fp32 accuracy.
#include "attn_tile.h"

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));

struct PrefixArgs {
  const bf16_t *q, *k, *v, *pk, *pv;
  bf16_t* o;
  float* lse;              // [B, h, L] or null
  float *part_o, *part_ml;   // workspace: [h_kv][rows][slots][kp_vo] and [h_kv][rows][slots][2] (maximum in score * scale * log2 e, sum)
  const int* lens;
  long long ld_q, ld_o, k_sb, k_sh, k_st, v_sb, v_sh, v_st, pk_sh, pk_st, pv_sh, pv_st;
  int B, L, h, h_kv, g, kq, kv, P, own_max;
  float sc;                // scale * log2 e
  int rows;                // B * L * g rows of a key/value head
  int own_rows;            // L * g of them belong to a request
  int joint;               // items run over the prefix and then the request's own keys; otherwise over one of them
  int p_tiles;             // key tiles of the prefix, as the items that read it cut it
  int p_chunks, p_chunk, p_row_tiles;      // prefix items: chunks, key tiles of a chunk, tiles of rows
  int o_chunks, o_chunk, o_row_tiles;      // own (or joint) items
  int p_items;             // prefix items in front of the others in the grid
  int slots;               // pieces per row in the workspace; 0: every item is all of its rows
};

// own keys of request b that its new token t sees (the new tokens are the last L rows of the cache)
__device__ __forceinline__ int own_len(const PrefixArgs& a, int b) { return min(max(a.lens[b], 0), a.own_max); }
__device__ __forceinline__ int own_visible(int n, int L, int t) { return min(max(n - L + 1 + t, 0), n); }

// Direct global->LDS loads of [KT rows][D] tiles, by one wavefront (WAVES = 1) or shared out over the workgroup's four.  An instruction
// fills 64 / (D / 8) consecutive rows; the swizzle of the LDS tile is applied on the global side.  Rows beyond `valid` repeat the last valid one
// (nothing behind the end of a cache is read), dims beyond the kept width the last kept chunk: stand-ins that masks and zero operands keep out.
template <int D, int KT, int WAVES>
struct KvLoader {
  static constexpr int CPR = D / 8, RPI = 64 / CPR, PER = (KT / RPI) / WAVES, NC = D == 32 ? 1 : (D == 64 ? 2 : 4);
  static_assert(PER >= 1, "a tile is at least an instruction of every wavefront");
  unsigned col[NC];      // byte offset of the lane's chunk, by the parity of the instruction (the swizzle repeats every 16 rows)
  int row0, wave;
  __device__ __forceinline__ void init(int kp) {
    const int lane = threadIdx.x & 63;
    wave = WAVES == 1 ? 0 : static_cast<int>(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
    row0 = wave * (PER * RPI) + lane / CPR;
#pragma unroll
    for (int i = 0; i < NC; ++i) col[i] = static_cast<unsigned>(min(((lane % CPR) ^ nat_swz<D>(row0 + i * RPI)) * 8, kp - 8) * 2);
  }
  __device__ __forceinline__ void issue(bf16_t* tile, const char* base, unsigned ldb, int valid) const {
    lds_bf16_t* const dst = (lds_bf16_t*)tile + wave * (PER * 512);
    if (valid >= KT) {
      const unsigned at = static_cast<unsigned>(row0) * ldb;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        unsigned o = at + col[i % NC];
        asm volatile("" : "+v"(o));      // keeps the offset a lane register at the load
        __builtin_amdgcn_global_load_lds(reinterpret_cast<const void*>(base + static_cast<unsigned long long>(i * RPI) * ldb + o), dst + i * 512, 16, 0, 0);
      }
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        unsigned o = static_cast<unsigned>(min(row0 + i * RPI, valid - 1)) * ldb + col[i % NC];
        asm volatile("" : "+v"(o));
        __builtin_amdgcn_global_load_lds(reinterpret_cast<const void*>(base + o), dst + i * 512, 16, 0, 0);
      }
    }
  }
};
// at most VM direct loads of this wavefront are still under way
template <int VM>
__device__ __forceinline__ void loads_wait() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((VM & 15) | ((VM >> 4) << 14) | (7 << 4) | (15 << 8));
  asm volatile("" ::: "memory");
}

// V^T fragment of 32 keys x 16 dims: lane (dim l % 16, group l / 16) gets its dim of keys 4 group .. + 3 of both 16-key tiles.
template <int D>
__device__ __forceinline__ void trn_issue16(TrnRegs& r, const bf16_t* tile, int dim0, int s) {
  const int lane = threadIdx.x & 63, i = lane & 15;
  const int row = 4 * (lane >> 4) + (i >> 2), col = dim0 + 4 * (i & 3);      // rows 16 apart have the same swizzle: both offsets are constants
  const lds_bf16_t* t3 = (const lds_bf16_t*)tile;
  const unsigned at = static_cast<unsigned>(reinterpret_cast<uintptr_t>(t3 + nat_off<D>(row, col >> 3) + (col & 7)));
  asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(r.lo) : "v"(at), "i"(s * 64 * D) : "memory");
  asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(r.hi) : "v"(at), "i"(s * 64 * D + 32 * D) : "memory");
}
// maximum over the four 16-lane groups (a row's keys are spread over them), in every lane
__device__ __forceinline__ float groups_max(float v) {
  const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
  const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
}
__device__ __forceinline__ float groups_sum(float v) {
  const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(q[0]) + __uint_as_float(q[1]);
}

// State of the NR x 16 rows of a wavefront.
template <int DV, int NR>
struct RowState {
  floatx4 o[NR][DV / 16];
  float m[NR], l[NR];      // running reference of raw scores; this lane's share of the sum of exponentials
  __device__ __forceinline__ void init() {
#pragma unroll
    for (int c = 0; c < NR; ++c) {
      m[c] = -INFINITY;
      l[c] = 0.f;
#pragma unroll
      for (int u = 0; u < DV / 16; ++u) o[c][u] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
  }
};

// One tile of KT keys.  left[c]: keys of this tile that the lane's row of column group c sees (any value: beyond KT all, below 1 none);
// whole: every row sees all of the tile.
template <int DQ, int DV, int NR, int KT>
__device__ __forceinline__ void prefix_tile(const bf16_t* Kt, const bf16_t* Vt, const bf16x8_t (&qf)[NR][DQ / 32], RowState<DV, NR>& st, float sc,
                                            bool whole, const int (&left)[NR]) {
  const int lane = threadIdx.x & 63, grp = lane >> 4, l16 = lane & 15;
  floatx4 s[NR][KT / 16];
#pragma unroll
  for (int t = 0; t < KT / 16; ++t) {
    bf16x8_t kf[DQ / 32];
#pragma unroll
    for (int i = 0; i < DQ / 32; ++i) kf[i] = *reinterpret_cast<const bf16x8_t*>(Kt + nat_off<DQ>(16 * t + l16, 4 * i + grp));
#pragma unroll
    for (int c = 0; c < NR; ++c) {
      s[c][t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < DQ / 32; ++i) s[c][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[i], qf[c][i], s[c][t], 0, 0, 0);
    }
  }
  if (!whole) {
#pragma unroll
    for (int c = 0; c < NR; ++c)
#pragma unroll
      for (int t = 0; t < KT / 16; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) s[c][t][r] = 16 * t + 4 * grp + r < left[c] ? s[c][t][r] : -INFINITY;
  }
  // The reference only has to keep the exponentials in range: it moves, and the accumulators are rescaled, when some row's maximum has grown
  // by more than RESCALE_LOG2 binades since it was set (or the row sees its first key).
  bool grown = false;
  float m_new[NR];
#pragma unroll
  for (int c = 0; c < NR; ++c) {
    float mx = s[c][0][0];
#pragma unroll
    for (int t = 0; t < KT / 16; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[c][t][r]);
    m_new[c] = fmaxf(st.m[c], groups_max(mx));
    grown = grown || (m_new[c] - st.m[c]) * sc > RESCALE_LOG2 || (m_new[c] > st.m[c] && st.m[c] == -INFINITY);
  }
  if (__builtin_amdgcn_ballot_w64(grown) != 0ull) {
#pragma unroll
    for (int c = 0; c < NR; ++c) {
      const float alpha = st.m[c] == m_new[c] ? 1.f : __builtin_amdgcn_exp2f((st.m[c] - m_new[c]) * sc);
      st.m[c] = m_new[c];
      st.l[c] *= alpha;
#pragma unroll
      for (int u = 0; u < DV / 16; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r) st.o[c][u][r] *= alpha;
    }
  }
#pragma unroll
  for (int c = 0; c < NR; ++c) {
    const float msc = (st.m[c] == -INFINITY ? 0.f : st.m[c]) * sc;
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < KT / 16; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        s[c][t][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[c][t][r], sc, -msc));
        sum += s[c][t][r];
      }
    st.l[c] += sum;
  }
#pragma unroll
  for (int i = 0; i < KT / 32; ++i) {
    TrnRegs vr[DV / 16];
#pragma unroll
    for (int u = 0; u < DV / 16; ++u) trn_issue16<DV>(vr[u], Vt, 16 * u, i);
    bf16x8_t pf[NR];
#pragma unroll
    for (int c = 0; c < NR; ++c) {
      const floatx8 p = {s[c][2 * i][0], s[c][2 * i][1], s[c][2 * i][2], s[c][2 * i][3], s[c][2 * i + 1][0], s[c][2 * i + 1][1], s[c][2 * i + 1][2], s[c][2 * i + 1][3]};
      pf[c] = __builtin_convertvector(p, bf16x8_t);
    }
    trn_wait();
#pragma unroll
    for (int u = 0; u < DV / 16; ++u) {
      const bf16x8_t vf = trn_frag(vr[u]);
#pragma unroll
      for (int c = 0; c < NR; ++c) st.o[c][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[c], st.o[c][u], 0, 0, 0);
    }
  }
}

// What an item is.
struct Item {
  int hk, b;            // key/value head; request of its own keys (-1: none)
  int row0, n_rows;     // rows of the head
  int slot;
  int t0, t1, split;    // key tiles t0 .. t1 - 1; those from `split` on are own tiles
  int own_n;            // own rows that may be read
};
template <int KT>
__device__ __forceinline__ bool prefix_item(const PrefixArgs& a, int row_tile, Item& it) {
  int id = blockIdx.x;
  if (id < a.p_items) {
    const int chunk = id / (a.p_row_tiles * a.h_kv), r = id - chunk * (a.p_row_tiles * a.h_kv);
    it.hk = r / a.p_row_tiles;
    it.b = -1;
    it.row0 = (r - it.hk * a.p_row_tiles) * row_tile;
    it.n_rows = min(row_tile, a.rows - it.row0);
    it.slot = chunk;
    it.t0 = chunk * a.p_chunk;
    it.t1 = min(it.t0 + a.p_chunk, a.p_tiles);
    it.split = a.p_tiles;
    it.own_n = 0;
    return true;
  }
  id -= a.p_items;
  const int per = a.o_chunks * a.o_row_tiles;
  const int bh = id / per, r = id - bh * per, chunk = r / a.o_row_tiles, rt = r - chunk * a.o_row_tiles;
  it.b = bh / a.h_kv;
  it.hk = bh - it.b * a.h_kv;
  const int first = rt * row_tile;
  it.n_rows = min(row_tile, a.own_rows - first);
  it.row0 = it.b * a.own_rows + first;
  it.slot = (a.joint ? 0 : a.p_chunks) + chunk;
  it.split = a.joint ? a.p_tiles : 0;
  const int n = own_len(a, it.b);
  it.own_n = own_visible(n, a.L, (first + it.n_rows - 1) / a.g);      // of the last row
  it.t0 = chunk * a.o_chunk;
  it.t1 = min(it.t0 + a.o_chunk, it.split + (it.own_n + KT - 1) / KT);
  return it.t0 < it.t1 || a.slots == 0;      // without slots the item writes its rows even if they see nothing
}
template <int DQ, int DV, bool SHARE>
struct PrefixShape {
  static constexpr int KT = SHARE || DQ + DV <= 64 ? 64 : 32;
  static constexpr int NB = 2;
  static constexpr int lds(int nr) {
    const int loop = (SHARE ? 1 : 4) * NB * KT * (DQ + DV) * 2, join = SHARE ? 0 : 4 * nr * (DV * 16 + 32) * 4;
    return loop > join ? loop : join;
  }
};

// SHARE: the four wavefronts take NR * 16 rows each and share every key tile.  Otherwise they share the item's rows (at most NR * 16) and take
// the key tiles in turn, from LDS buffers of their own without a barrier, and join at the end.
template <int DQ, int DV, int NR, bool SHARE>
__device__ __forceinline__ void prefix_rows(const PrefixArgs& a, bf16_t* const lds_all) {
  typedef PrefixShape<DQ, DV, SHARE> Shape;
  constexpr int KT = Shape::KT, WAVES = SHARE ? 4 : 1, NB = Shape::NB;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), grp = lane >> 4, l16 = lane & 15;
  Item it;
  if (!prefix_item<KT>(a, (SHARE ? 4 : 1) * NR * 16, it)) return;
  bf16_t* const buf = lds_all + (SHARE ? 0 : wave * NB * KT * (DQ + DV));      // [NB][K tile, V tile]

  KvLoader<DQ, KT, WAVES> kl;
  KvLoader<DV, KT, WAVES> vl;
  kl.init(a.kq);
  vl.init(a.kv);
  const char* const pk = reinterpret_cast<const char*>(a.pk + it.hk * a.pk_sh);
  const char* const pv = reinterpret_cast<const char*>(a.pv + it.hk * a.pv_sh);
  const char* const ok = reinterpret_cast<const char*>(a.k + (it.b < 0 ? 0 : it.b) * a.k_sb + it.hk * a.k_sh);
  const char* const ov = reinterpret_cast<const char*>(a.v + (it.b < 0 ? 0 : it.b) * a.v_sb + it.hk * a.v_sh);
  const auto issue = [&](int j, int n) __attribute__((always_inline)) {
    const bool own = j >= it.split;
    const long long first = static_cast<long long>(own ? j - it.split : j) * KT;
    const int valid = (own ? it.own_n : a.P) - static_cast<int>(first);
    const long long ldk = 2 * (own ? a.k_st : a.pk_st), ldv = 2 * (own ? a.v_st : a.pv_st);
    bf16_t* const at = buf + n * (KT * (DQ + DV));
    kl.issue(at, (own ? ok : pk) + first * ldk, static_cast<unsigned>(ldk), valid);
    vl.issue(at + KT * DQ, (own ? ov : pv) + first * ldv, static_cast<unsigned>(ldv), valid);
  };
  constexpr int STEP = SHARE ? 1 : 4;
  const int first = it.t0 + (SHARE ? 0 : wave);
  if (first < it.t1) issue(first, 0);

  // the wavefront's rows: queries straight from memory, rows and dims outside are zero
  bf16x8_t qf[NR][DQ / 32];
  int seen[NR];      // own keys the row sees
#pragma unroll
  for (int c = 0; c < NR; ++c) {
    const int r = (SHARE ? wave * NR * 16 : 0) + c * 16 + l16, row = it.row0 + min(r, it.n_rows - 1);
    const int token = row / a.g;
    const bf16_t* const src = a.q + token * a.ld_q + static_cast<long long>(it.hk * a.g + (row - token * a.g)) * a.kq;
    seen[c] = it.b < 0 ? 0 : own_visible(own_len(a, it.b), a.L, token - it.b * a.L);
    u32x4 raw[DQ / 32];
#pragma unroll
    for (int i = 0; i < DQ / 32; ++i) raw[i] = *reinterpret_cast<const u32x4*>(src + min(32 * i + 8 * grp, a.kq - 8));
#pragma unroll
    for (int i = 0; i < DQ / 32; ++i)
      qf[c][i] = __builtin_bit_cast(bf16x8_t, r < it.n_rows && 32 * i + 8 * grp < a.kq ? raw[i] : u32x4{0u, 0u, 0u, 0u});
  }
  int least = seen[0];
#pragma unroll
  for (int c = 1; c < NR; ++c) least = min(least, seen[c]);
  least = static_cast<int>(wave_umin(static_cast<uint32_t>(least)));      // own keys that every row sees

  RowState<DV, NR> st;
  st.init();
  int cur = 0;
  for (int j = first; j < it.t1; j += STEP) {
    stream_wait();
    if (SHARE) __syncthreads();
    if (j + STEP < it.t1) issue(j + STEP, cur ^ 1);
    const bool own = j >= it.split;
    const int k0 = (own ? j - it.split : j) * KT;
    int left[NR];
#pragma unroll
    for (int c = 0; c < NR; ++c) left[c] = (own ? seen[c] : a.P) - k0;
    const bf16_t* const at = buf + cur * (KT * (DQ + DV));
    prefix_tile<DQ, DV, NR, KT>(at, at + KT * DQ, qf, st, a.sc, k0 + KT <= (own ? least : a.P), left);
    cur ^= 1;
  }
#pragma unroll
  for (int c = 0; c < NR; ++c) st.l[c] = groups_sum(st.l[c]);

  // this lane's four dims of block u of row r: normalised into the output, or a piece for the join
  const auto write = [&](int c, int u, const floatx4& acc, float m, float l, bool with_ml) __attribute__((always_inline)) {
    const int r = (SHARE ? wave * NR * 16 : 0) + c * 16 + l16, row = it.row0 + r;
    if (r >= it.n_rows) return;
    if (a.slots == 0) {
      const int token = row / a.g, head = it.hk * a.g + (row - token * a.g);
      if (16 * u < a.kv) {
        const float inv = l > 0.f ? 1.f / l : 0.f;
        floatx4 f;
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = acc[i] * inv;
        *reinterpret_cast<bf16x4_t*>(a.o + token * a.ld_o + static_cast<long long>(head) * a.kv + 16 * u + 4 * grp) = __builtin_convertvector(f, bf16x4_t);
      }
      if (with_ml && a.lse && grp == 0) {
        const int b = token / a.L;
        a.lse[(static_cast<long long>(b) * a.h + head) * a.L + (token - b * a.L)] = l > 0.f ? (m * a.sc + __builtin_amdgcn_logf(l)) * LN2 : -INFINITY;
      }
    } else {
      const long long at = (static_cast<long long>(it.hk) * a.rows + row) * a.slots + it.slot;
      if (16 * u < a.kv) *reinterpret_cast<floatx4*>(a.part_o + at * a.kv + 16 * u + 4 * grp) = acc;
      if (with_ml && grp == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * at) = float2{m * a.sc, l};
    }
  };
  if (SHARE) {
#pragma unroll
    for (int c = 0; c < NR; ++c)
#pragma unroll
      for (int u = 0; u < DV / 16; ++u) write(c, u, st.o[c][u], st.m[c], st.l[c], u == 0);
  } else {
    __syncthreads();
    float* const part = reinterpret_cast<float*>(lds_all);      // [4][NR][DV / 16][4][64]
    float* const ms = part + 4 * NR * DV * 16;                  // [4][NR][16] each
    float* const ls = ms + 4 * NR * 16;
#pragma unroll
    for (int c = 0; c < NR; ++c) {
#pragma unroll
      for (int u = 0; u < DV / 16; ++u)
        *reinterpret_cast<floatx4*>(part + (((wave * NR + c) * (DV / 16) + u) * 64 + lane) * 4) = st.o[c][u];
      if (grp == 0) {
        ms[(wave * NR + c) * 16 + l16] = st.m[c];
        ls[(wave * NR + c) * 16 + l16] = st.l[c];
      }
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < NR; ++c) {
      float m_all = ms[c * 16 + l16], al[4], l_all = 0.f;
#pragma unroll
      for (int w = 1; w < 4; ++w) m_all = fmaxf(m_all, ms[(w * NR + c) * 16 + l16]);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float m = ms[(w * NR + c) * 16 + l16];
        al[w] = m == m_all ? (m == -INFINITY ? 0.f : 1.f) : __builtin_amdgcn_exp2f((m - m_all) * a.sc);
        l_all += al[w] * ls[(w * NR + c) * 16 + l16];
      }
#pragma unroll
      for (int u0 = 0; u0 < DV / 16; u0 += 4) {
        const int u = u0 + wave;
        if (u >= DV / 16) break;
        floatx4 f = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const floatx4 x = *reinterpret_cast<const floatx4*>(part + (((w * NR + c) * (DV / 16) + u) * 64 + lane) * 4);
#pragma unroll
          for (int i = 0; i < 4; ++i) f[i] += al[w] * x[i];
        }
        write(c, u, f, m_all, l_all, u == 0);
      }
    }
  }
}


// Which rows an item has: ROWS_16, ROWS_32: up to 16 or 32, its key tiles shared out over the wavefronts; ROWS_128: 32 a wavefront.
enum { ROWS_16 = 0, ROWS_32 = 1, ROWS_128 = 2 };
// KIND: rows of every item; prefix items have ROWS_128 where PREFIX_128 says so.
// Two wavefronts a SIMD at least: the register file then has no accumulation half, and the scores need no moves between the halves.
template <int DQ, int DV, int KIND, bool PREFIX_128>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void prefix_attn_kernel(const PrefixArgs a) {
  extern __shared__ __attribute__((aligned(16))) bf16_t lds_all[];      // one object: see attn.hip
  if (PREFIX_128 && static_cast<int>(blockIdx.x) < a.p_items) prefix_rows<DQ, DV, 2, true>(a, lds_all);
  else prefix_rows<DQ, DV, KIND == ROWS_16 ? 1 : 2, KIND == ROWS_128>(a, lds_all);
}

// ---------------------------------------------------------------------------------------------
// Join: a workgroup puts the pieces of a row together.  Threads are (piece, four dims); a thread weighs its pieces against the maximum of its
// own, four of them asked for at a time (what counts is how many latencies follow on each other), then the threads of equal dims are added up
// against the row's maximum in a fixed order.
// ---------------------------------------------------------------------------------------------
template <int W>      // threads of a piece: kp_vo / 4 rounded up to a power of two
__global__ __launch_bounds__(256) void prefix_join_kernel(const PrefixArgs a, int kt, int row_tile) {
  constexpr int GROUPS = 256 / W;
  __shared__ floatx4 so[GROUPS][W];
  __shared__ float sm[GROUPS], sl[GROUPS];
  const long long at = blockIdx.x;
  const int hk = static_cast<int>(at / a.rows), row = static_cast<int>(at - static_cast<long long>(hk) * a.rows);
  const int token = row / a.g, b = token / a.L, head = hk * a.g + (row - token * a.g);
  // own pieces: as prefix_item() cuts them for the tile of rows that this row is in
  const int in = row - b * a.own_rows, tile0 = in / row_tile * row_tile;
  const int own_n = own_visible(own_len(a, b), a.L, (min(tile0 + row_tile, a.own_rows) - 1) / a.g);
  const int own_tiles = (own_n + kt - 1) / kt + (a.joint ? a.p_tiles : 0);
  const int n = (a.joint ? 0 : a.p_chunks) + (own_tiles + a.o_chunk - 1) / a.o_chunk;
  const float2* const ml = reinterpret_cast<const float2*>(a.part_ml) + at * a.slots;
  const int grp = threadIdx.x / W, lane = threadIdx.x % W, d = min(lane * 4, a.kv - 4);
  const float* const po = a.part_o + at * a.slots * a.kv + d;
  float m = -INFINITY, l = 0.f;
  floatx4 o = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = grp; i0 < n; i0 += 4 * GROUPS) {
    float2 x[4];
    floatx4 p[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = min(i0 + j * GROUPS, n - 1);
      x[j] = ml[i];
      p[j] = *reinterpret_cast<const floatx4*>(po + static_cast<long long>(i) * a.kv);
    }
    float top = m;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (i0 + j * GROUPS >= n) x[j].x = -INFINITY;
      top = fmaxf(top, x[j].x);
    }
    const float ref = top == -INFINITY ? 0.f : top, f = __builtin_amdgcn_exp2f(m - ref);
    m = top;
    l *= f;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] *= f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float w = x[j].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x[j].x - ref);
      l += w * x[j].y;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += w * p[j][e];
    }
  }
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
  if (lane * 4 < a.kv) {
    const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] *= inv;
    *reinterpret_cast<bf16x4_t*>(a.o + token * a.ld_o + static_cast<long long>(head) * a.kv + d) = __builtin_convertvector(o, bf16x4_t);
  }
  if (lane == 0 && a.lse)
    a.lse[(static_cast<long long>(b) * a.h + head) * a.L + (token - b * a.L)] = l > 0.f ? (m + __builtin_amdgcn_logf(l)) * LN2 : -INFINITY;
}

// ---------------------------------------------------------------------------------------------
// Weights: w_out[j] = w_in[j] + sum over the rows of the request that see own key j of exp(s_j - lse).  A wavefront takes 32 keys: their fragments
// stay in registers while the rows pass by, 16 at a time; the sum over a tile's rows is a sum over lanes.
// ---------------------------------------------------------------------------------------------
template <int DQ>
__global__ __launch_bounds__(256) void prefix_weights_kernel(const PrefixArgs a, const float* lse, const float* w_in, float* w_out, int cap) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), grp = lane >> 4, l16 = lane & 15;
  const int b = blockIdx.y / a.h_kv, hk = blockIdx.y - b * a.h_kv;
  const int n = own_len(a, b), k0 = (blockIdx.x * 4 + wave) * 32;
  if (k0 >= n) return;
  const bf16_t* const kb = a.k + b * a.k_sb + hk * a.k_sh;
  bf16x8_t kf[2][DQ / 32];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < DQ / 32; ++i)
      kf[t][i] = *reinterpret_cast<const bf16x8_t*>(kb + min(k0 + 16 * t + l16, n - 1) * a.k_st + min(32 * i + 8 * grp, a.kq - 8));
  float sum[2][4] = {};
  for (int r0 = 0; r0 < a.own_rows; r0 += 16) {
    const int r = min(r0 + l16, a.own_rows - 1), t = r / a.g, head = hk * a.g + (r - t * a.g);
    const long long token = static_cast<long long>(b) * a.L + t;
    const bf16_t* const src = a.q + token * a.ld_q + static_cast<long long>(head) * a.kq;
    bf16x8_t qf[DQ / 32];
#pragma unroll
    for (int i = 0; i < DQ / 32; ++i) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(src + min(32 * i + 8 * grp, a.kq - 8));
      qf[i] = __builtin_bit_cast(bf16x8_t, 32 * i + 8 * grp < a.kq ? x : u32x4{0u, 0u, 0u, 0u});
    }
    const float ref = lse[(static_cast<long long>(b) * a.h + head) * a.L + t] * LOG2E;
    const int left = (r0 + l16 < a.own_rows ? own_visible(n, a.L, t) : 0) - k0 - 4 * grp;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      floatx4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < DQ / 32; ++i) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[u][i], qf[i], s, 0, 0, 0);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], a.sc, -ref));
        sum[u][e] += 16 * u + e < left ? p : 0.f;
      }
    }
  }
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float x = row16_sum(sum[u][e]);
      const int j = k0 + 16 * u + 4 * grp + e;
      const long long at = static_cast<long long>(blockIdx.y) * cap + j;
      if (l16 == 0 && j < n) w_out[at] = (w_in ? w_in[at] : 0.f) + x;
    }
}

// ---------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------
static int prefix_width(int kp) { return kp <= 32 ? 32 : (kp <= 64 ? 64 : 128); }
static int rows_of(int kind) { return kind == ROWS_16 ? 16 : (kind == ROWS_32 ? 32 : 128); }

struct PrefixPlan {
  int dq, dv, kind, prefix_128, kt, join_row_tile;
  unsigned grid;
  size_t part_o, part_ml, lse;      // bytes of workspace
};
// Fills the item fields of `a` (shapes are set) and the plan.
static bool prefix_plan(PrefixArgs& a, PrefixPlan& p) {
  p.dq = prefix_width(a.kq);
  p.dv = prefix_width(a.kv);
  const bool small = p.dq + p.dv <= 64;
  const long long resident = 512;
  // Rows of a request that fill a tile of their own, a batch of one or no prefix: nothing to gain by putting requests together.
  const int kind_own = a.own_rows <= 16 ? ROWS_16 : (a.own_rows <= 32 ? ROWS_32 : ROWS_128);
  const int kt_own = kind_own == ROWS_128 || small ? 64 : 32;
  const int step_own = kind_own == ROWS_128 ? 1 : 4;      // key tiles that a workgroup works on at once
  a.o_row_tiles = (a.own_rows + rows_of(kind_own) - 1) / rows_of(kind_own);
  const long long pairs = static_cast<long long>(a.B) * a.h_kv * a.o_row_tiles;
  const long long own_steps = ((a.own_max + kt_own - 1) / kt_own + step_own - 1) / step_own;
  const long long p_steps_joint = ((a.P + kt_own - 1) / kt_own + step_own - 1) / step_own;
  a.joint = a.B == 1 || a.P == 0 || kind_own == ROWS_128 || pairs * p_steps_joint <= 2 * resident;
  p.kind = kind_own;
  p.prefix_128 = 0;
  a.p_items = a.p_chunks = a.p_chunk = a.p_row_tiles = 0;
  if (a.joint) {
    const int total_tiles = (a.P + kt_own - 1) / kt_own + (a.own_max + kt_own - 1) / kt_own;
    const long long steps = (total_tiles + step_own - 1) / step_own;
    long long chunk = (pairs * steps + 2 * resident - 1) / (2 * resident);
    chunk = chunk < 4 ? 4 : chunk;
    if (pairs >= resident || chunk >= steps) chunk = steps > 1 ? steps : 1;
    a.p_tiles = (a.P + kt_own - 1) / kt_own;
    a.o_chunk = static_cast<int>(chunk * step_own);
    a.o_chunks = total_tiles > 0 ? (total_tiles + a.o_chunk - 1) / a.o_chunk : 1;
    a.slots = a.o_chunks > 1 ? a.o_chunks : 0;
  } else {
    const int kind_p = a.rows <= 16 ? ROWS_16 : (a.rows <= 32 ? ROWS_32 : ROWS_128);
    p.prefix_128 = kind_p == ROWS_128;
    if (!p.prefix_128) p.kind = kind_p;      // the own items of few requests ride along
    const int kt_p = p.prefix_128 || small ? 64 : 32, step_p = p.prefix_128 ? 1 : 4;
    a.p_tiles = (a.P + kt_p - 1) / kt_p;
    a.p_row_tiles = (a.rows + rows_of(kind_p) - 1) / rows_of(kind_p);
    const long long p_steps = static_cast<long long>(a.h_kv) * a.p_row_tiles * ((a.p_tiles + step_p - 1) / step_p);
    long long chunk = (p_steps + pairs * own_steps + 2 * resident - 1) / (2 * resident);
    chunk = chunk < 4 ? 4 : chunk;
    a.p_chunk = static_cast<int>(chunk * step_p);
    a.p_chunks = (a.p_tiles + a.p_chunk - 1) / a.p_chunk;
    a.p_items = a.p_chunks * a.p_row_tiles * a.h_kv;
    a.o_chunk = static_cast<int>(chunk * step_own);
    const int o_tiles = (a.own_max + kt_own - 1) / kt_own;
    a.o_chunks = (o_tiles + a.o_chunk - 1) / a.o_chunk;
    a.slots = a.p_chunks + a.o_chunks;
  }
  p.kt = kt_own;
  p.join_row_tile = rows_of(p.kind);
  const long long grid = a.p_items + pairs * a.o_chunks;
  if (grid > 0x7fffffffll || static_cast<long long>(a.p_chunks) * a.p_row_tiles * a.h_kv > 0x7fffffffll) return false;
  p.grid = static_cast<unsigned>(grid);
  const size_t pieces = static_cast<size_t>(a.h_kv) * a.rows * a.slots;
  p.part_o = pieces * a.kv * sizeof(float);
  p.part_ml = pieces * 2 * sizeof(float);
  return true;
}

template <int DQ, int DV, int KIND, bool P128>
static hipError_t prefix_launch(const PrefixArgs& a, unsigned grid, hipStream_t st) {
  constexpr int own = PrefixShape<DQ, DV, KIND == ROWS_128>::lds(KIND == ROWS_16 ? 1 : 2), pre = P128 ? PrefixShape<DQ, DV, true>::lds(2) : 0;
  constexpr int lds = own > pre ? own : pre;
  const auto kern = prefix_attn_kernel<DQ, DV, KIND, P128>;
  static LdsAttrOnce attr_once;
  if (lds > 64 * 1024) {
    const hipError_t e = attr_once.ensure(reinterpret_cast<const void*>(kern), lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kern, dim3(grid), dim3(256), lds, st, a);
  return hipGetLastError();
}
#define PREFIX_INSTANTIATE(DQ, DV)                                                        \
  template __global__ void prefix_attn_kernel<DQ, DV, ROWS_16, false>(const PrefixArgs);  \
  template __global__ void prefix_attn_kernel<DQ, DV, ROWS_32, false>(const PrefixArgs);  \
  template __global__ void prefix_attn_kernel<DQ, DV, ROWS_128, false>(const PrefixArgs); \
  template __global__ void prefix_attn_kernel<DQ, DV, ROWS_16, true>(const PrefixArgs);   \
  template __global__ void prefix_attn_kernel<DQ, DV, ROWS_32, true>(const PrefixArgs);
#define PREFIX_WIDTHS(X) X(32, 32) X(32, 64) X(64, 32) X(64, 64) X(32, 128) X(64, 128) X(128, 32) X(128, 64) X(128, 128)
PREFIX_WIDTHS(PREFIX_INSTANTIATE)
#undef PREFIX_INSTANTIATE
template __global__ void prefix_join_kernel<8>(const PrefixArgs, int, int);
template __global__ void prefix_join_kernel<16>(const PrefixArgs, int, int);
template __global__ void prefix_join_kernel<32>(const PrefixArgs, int, int);
template __global__ void prefix_weights_kernel<32>(const PrefixArgs, const float*, const float*, float*, int);
template __global__ void prefix_weights_kernel<64>(const PrefixArgs, const float*, const float*, float*, int);
template __global__ void prefix_weights_kernel<128>(const PrefixArgs, const float*, const float*, float*, int);

int ecospa_cache_check(const ecospa_cache* c) {
  if (!c || !c->k || !c->v || !c->lens || (c->P > 0 && (!c->pk || !c->pv))) return ECOSPA_ERR_NULL;
  if (c->dtype != ECOSPA_BF16) return ECOSPA_ERR_DTYPE;
  if (c->B < 1 || c->h_kv < 1 || c->h < c->h_kv || c->h % c->h_kv || c->cap < 1 || c->own_max < 0 || c->own_max > c->cap || c->P < 0) return ECOSPA_ERR_SHAPE;
  if (c->kp_qk < 16 || c->kp_qk > 128 || c->kp_qk % 16 || c->kp_vo < 16 || c->kp_vo > 128 || c->kp_vo % 16) return ECOSPA_ERR_SHAPE;
  if (!(c->scale > 0.f) || c->scale > 3.0e38f) return ECOSPA_ERR_SHAPE;
  const long long rows[4] = {c->k_st, c->v_st, c->P > 0 ? c->pk_st : 1ll << 20, c->P > 0 ? c->pv_st : 1ll << 20};
  for (int i = 0; i < 4; ++i)      // 64 rows of a tile stay within 32 bits of bytes
    if (rows[i] < (i & 1 ? c->kp_vo : c->kp_qk) || rows[i] >= 1ll << 25) return ECOSPA_ERR_SHAPE;
  if (c->k_sb < 0 || c->k_sh < 0 || c->v_sb < 0 || c->v_sh < 0 || (c->P > 0 && (c->pk_sh < 0 || c->pv_sh < 0))) return ECOSPA_ERR_SHAPE;
  if (!aligned16(c->k) || !aligned16(c->v) || (c->k_sb | c->k_sh | c->k_st | c->v_sb | c->v_sh | c->v_st) % 8) return ECOSPA_ERR_ALIGN;
  if (c->P > 0 && (!aligned16(c->pk) || !aligned16(c->pv) || (c->pk_sh | c->pk_st | c->pv_sh | c->pv_st) % 8)) return ECOSPA_ERR_ALIGN;
  return ECOSPA_OK;
}
static int prefix_args(const ecospa_cache* c, int L, PrefixArgs& a, PrefixPlan& p, bool with_lse) {
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
  if (!prefix_plan(a, p)) return ECOSPA_ERR_SHAPE;
  p.lse = with_lse ? static_cast<size_t>(c->B) * L * c->h * sizeof(float) : 0;
  return ECOSPA_OK;
}

extern "C" size_t ecospa_prefix_attn_workspace_bytes(const ecospa_cache* cache, int L) {
  PrefixArgs a;
  PrefixPlan p;
  if (ecospa_cache_check(cache) != ECOSPA_OK || prefix_args(cache, L, a, p, true) != ECOSPA_OK) return 0;
  return align_up(p.part_o, 256) + align_up(p.part_ml, 256) + align_up(p.lse, 256);
}

extern "C" int ecospa_prefix_attn(ecospa_ctx* ctx, const ecospa_cache* cache, int L, const void* q, long long ld_q, void* o, long long ld_o,
                                  float* lse, const float* weights_in, float* weights_out) {
  if (!ctx || !q || !o || (weights_in && !weights_out)) return ECOSPA_ERR_NULL;
  int rc = ecospa_cache_check(cache);
  if (rc != ECOSPA_OK) return rc;
  PrefixArgs a;
  PrefixPlan p;
  rc = prefix_args(cache, L, a, p, weights_out && !lse);
  if (rc != ECOSPA_OK) return rc;
  if (ld_q < static_cast<long long>(a.h) * a.kq || ld_o < static_cast<long long>(a.h) * a.kv) return ECOSPA_ERR_SHAPE;
  if (!aligned16(q) || !aligned16(o) || ld_q % 8 || ld_o % 8) return ECOSPA_ERR_ALIGN;
  WsCarver ws(ctx->ws, ctx->ws_bytes);
  if (p.part_o) {
    a.part_o = static_cast<float*>(ws.take(p.part_o));
    a.part_ml = static_cast<float*>(ws.take(p.part_ml));
  }
  if (p.lse) lse = static_cast<float*>(ws.take(p.lse));
  if ((p.part_o || p.lse) && !ws.ok()) return ECOSPA_ERR_WORKSPACE;
  a.q = static_cast<const bf16_t*>(q); a.ld_q = ld_q; a.o = static_cast<bf16_t*>(o); a.ld_o = ld_o; a.lse = lse;
  hipError_t e = hipErrorInvalidValue;
#define PREFIX_CASE(Q, V)                                                                                          \
  if (p.dq == Q && p.dv == V) {                                                                                    \
    if (p.kind == ROWS_128) e = prefix_launch<Q, V, ROWS_128, false>(a, p.grid, ctx->stream);                      \
    else if (p.kind == ROWS_16 && !p.prefix_128) e = prefix_launch<Q, V, ROWS_16, false>(a, p.grid, ctx->stream);  \
    else if (p.kind == ROWS_32 && !p.prefix_128) e = prefix_launch<Q, V, ROWS_32, false>(a, p.grid, ctx->stream);  \
    else if (p.kind == ROWS_16) e = prefix_launch<Q, V, ROWS_16, true>(a, p.grid, ctx->stream);                    \
    else e = prefix_launch<Q, V, ROWS_32, true>(a, p.grid, ctx->stream);                                           \
  }
  PREFIX_WIDTHS(PREFIX_CASE)
#undef PREFIX_CASE
  if (e != hipSuccess) return hip_fail(ctx, e, "prefix_attn_kernel");
  if (a.slots) {
    const long long rows = static_cast<long long>(a.h_kv) * a.rows;
    const dim3 grid(static_cast<unsigned>(rows));
    if (a.kv <= 32) hipLaunchKernelGGL(prefix_join_kernel<8>, grid, dim3(256), 0, ctx->stream, a, p.kt, p.join_row_tile);
    else if (a.kv <= 64) hipLaunchKernelGGL(prefix_join_kernel<16>, grid, dim3(256), 0, ctx->stream, a, p.kt, p.join_row_tile);
    else hipLaunchKernelGGL(prefix_join_kernel<32>, grid, dim3(256), 0, ctx->stream, a, p.kt, p.join_row_tile);
    ECOSPA_CHECK_LAUNCH(ctx, "prefix_join_kernel");
  }
  if (weights_out && a.own_max > 0) {
    const dim3 grid((a.own_max + 127) / 128, a.B * a.h_kv);
    const auto kern = p.dq == 32 ? prefix_weights_kernel<32> : (p.dq == 64 ? prefix_weights_kernel<64> : prefix_weights_kernel<128>);
    hipLaunchKernelGGL(kern, grid, dim3(256), 0, ctx->stream, a, lse, weights_in, weights_out, cache->cap);
    ECOSPA_CHECK_LAUNCH(ctx, "prefix_weights_kernel");
  }
  return ECOSPA_OK;
}
