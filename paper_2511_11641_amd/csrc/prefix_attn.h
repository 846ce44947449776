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
// Layout: scores are computed transposed, S^T = K Q^T (keys x rows): a row of the softmax is a lane's column, and result registers are, rounded
// to bf16, the B operand of O^T = V^T P^T without going through LDS.  The matching V^T operand comes from transposing LDS reads.  Few rows go
// on v_mfma_f32_16x16x32_bf16, columns of 16 (Rows16): most calls have few (a token of a request is g = h / h_kv rows), and the exponentials of
// unused columns are the largest cost beside the memory.  Many rows go on v_mfma_f32_32x32x16_bf16 (Rows32): half the matrix instructions and
// half the steps of a maximum across lanes.
//
// What bounds it (heads of 64 + 64 dims): one token a request on own caches alone, memory - 64 x 8 heads x 2048 keys, 268 MB, 44.7 us, 6.0 TB/s of the
// 6.3 that a plain read reaches.  Rows of many requests on a prefix, the vector unit: an exponential takes a SIMD about as long as the matrix products
// of its score, and maximum, scaling, sum and conversion as long again - 256 rows x 8 heads on 32768 keys 41 us, 417 TFLOP/s with its join; 16 x 509 tokens on 8192 keys and their own 620 us, 909
// TFLOP/s by the pairs that see each other, at the clock that power allows (1.9 GHz).  Both at once, 64 requests on 32768 + 2048 keys with weights: 65 us.  A single short request, latency: 61 + 33 keys 4.5 us.
//
// Only a row that sees no key has a sum of exponentials of zero; it is told by that.  A row that meets a score that is not a number, or +inf, has a sum,
// an output, a log-sum-exp and weights that are not numbers, in whatever piece the key lies (its maximum may say -inf: maxima pass over NaN).
//
// Rounding: scores, maxima, sums and accumulators are fp32; the probabilities enter the second product rounded to bf16 (the matrix
// unit's type), the denominator is summed from the unrounded ones, so that lse and the weights keep fp32 accuracy.
#pragma once
#include "attn_tile.h"

#include <type_traits>

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
  int p_stages, o_stages;  // LDS stages that such an item comes to use (no more than its tiles of a wavefront)
  int p_items;             // prefix items in front of the others in the grid
  int own_once, prefix_once;      // keys that one item reads, too many to stay in the last cache: their loads pass the caches by
  int slots;               // pieces per row in the workspace; 0: every item is all of its rows
  float* scores;           // workspace: [B][h_kv][own_rows][own_pad] scores of the own keys times scale * log2 e, null: not wanted
  int own_pad;
  const float* w_in;       // with scores: the weights before and after
  float* w_out;
  int cap;
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
  template <int AUX>      // 0, or 2: past the caches
  __device__ __forceinline__ void issue(bf16_t* tile, const char* base, unsigned ldb, int valid) const {
    lds_bf16_t* const dst = (lds_bf16_t*)tile + wave * (PER * 512);
    if (valid >= KT) {
      const unsigned at = static_cast<unsigned>(row0) * ldb;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        unsigned o = at + col[i % NC];
        asm volatile("" : "+v"(o));      // keeps the offset a lane register at the load
        __builtin_amdgcn_global_load_lds(reinterpret_cast<const void*>(base + static_cast<unsigned long long>(i * RPI) * ldb + o), dst + i * 512, 16, 0, AUX);
      }
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        unsigned o = static_cast<unsigned>(min(row0 + i * RPI, valid - 1)) * ldb + col[i % NC];
        asm volatile("" : "+v"(o));
        __builtin_amdgcn_global_load_lds(reinterpret_cast<const void*>(base + o), dst + i * 512, 16, 0, AUX);
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

// The rows of a wavefront: queries, accumulators and running softmax.  m: running reference of raw scores, l: this lane's share of the sum of
// exponentials (keys are spread over the lanes of a column).  chunk(c, q): four dims from dim(q) on of the row in column group c.
//
// The reference only has to keep the exponentials in range: it moves, and the accumulators are rescaled, when some row's maximum has grown by more
// than RESCALE_LOG2 binades since it was set (at a row's first key: infinitely).
template <int DQ, int DV, int NR>
struct Rows16 {
  static constexpr int COLS = NR, ROWS = 16 * NR, CHUNKS = DV / 16;
  bf16x8_t qf[NR][DQ / 32];
  floatx4 o[NR][DV / 16];
  float m[NR], l[NR];
  static __device__ __forceinline__ int lane() { return threadIdx.x & 63; }
  static __device__ __forceinline__ int row(int c) { return 16 * c + (lane() & 15); }
  static __device__ __forceinline__ int dim(int q) { return 16 * q + 4 * (lane() >> 4); }
  static __device__ __forceinline__ bool lead() { return lane() < 16; }      // of the lanes of a column
  __device__ __forceinline__ floatx4 chunk(int c, int q) const { return o[c][q]; }
  __device__ __forceinline__ void init() {
#pragma unroll
    for (int c = 0; c < NR; ++c) {
      m[c] = -INFINITY;
      l[c] = 0.f;
#pragma unroll
      for (int u = 0; u < DV / 16; ++u) o[c][u] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
  }
  __device__ __forceinline__ void load(int c, const bf16_t* src, int kq, bool there) {
    const int grp = lane() >> 4;
    u32x4 raw[DQ / 32];
#pragma unroll
    for (int i = 0; i < DQ / 32; ++i) raw[i] = *reinterpret_cast<const u32x4*>(src + min(32 * i + 8 * grp, kq - 8));
#pragma unroll
    for (int i = 0; i < DQ / 32; ++i) qf[c][i] = __builtin_bit_cast(bf16x8_t, there && 32 * i + 8 * grp < kq ? raw[i] : u32x4{0u, 0u, 0u, 0u});
  }
  __device__ __forceinline__ void finish() {
#pragma unroll
    for (int c = 0; c < NR; ++c) l[c] = groups_sum(l[c]);
  }
  // One tile of KT keys.  left[c]: keys of this tile that the lane's row of column group c sees (any value: beyond KT all, below 1 none);
  // whole: every row sees all of the tile.  keep: where the scores of the lane's rows go (column groups 16 keep_pitch apart; null: nowhere),
  // for the rows that `kept` has a bit for.
  template <int KT>
  __device__ __forceinline__ void tile(const bf16_t* Kt, const bf16_t* Vt, float sc, bool whole, const int (&left)[NR], float* keep, int keep_pitch, unsigned kept) {
    const int grp = lane() >> 4, l16 = lane() & 15;
    floatx4 s[NR][KT / 16];
    // Key fragments in groups of at most eight, all of a group read in front of its products, and products of the same 32 dims side by side: left
    // to itself the compiler reads and waits for two fragments at a time and lets each product wait for the one before it.
    constexpr int TG = KT / 16 < 8 / (DQ / 32) ? KT / 16 : 8 / (DQ / 32);
#pragma unroll
    for (int t0 = 0; t0 < KT / 16; t0 += TG) {
      bf16x8_t kf[TG][DQ / 32];
#pragma unroll
      for (int t = 0; t < TG; ++t)
#pragma unroll
        for (int i = 0; i < DQ / 32; ++i) kf[t][i] = *reinterpret_cast<const bf16x8_t*>(Kt + nat_off<DQ>(16 * (t0 + t) + l16, 4 * i + grp));
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < DQ / 32; ++i)
#pragma unroll
        for (int t = 0; t < TG; ++t)
#pragma unroll
          for (int c = 0; c < NR; ++c)
            s[c][t0 + t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[t][i], qf[c][i], i == 0 ? floatx4{0.f, 0.f, 0.f, 0.f} : s[c][t0 + t], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (!whole) {
#pragma unroll
      for (int c = 0; c < NR; ++c)
#pragma unroll
        for (int t = 0; t < KT / 16; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) s[c][t][r] = 16 * t + 4 * grp + r < left[c] ? s[c][t][r] : -INFINITY;
    }
    if (keep) {
#pragma unroll
      for (int c = 0; c < NR; ++c)
        if ((kept >> c) & 1u) {
#pragma unroll
          for (int t = 0; t < KT / 16; ++t) {
            floatx4 x;
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = s[c][t][r] * sc;
            *reinterpret_cast<floatx4*>(keep + static_cast<long long>(c) * 16 * keep_pitch + 16 * t + 4 * grp) = x;
          }
        }
    }
    bool grown = false;
    float m_new[NR];
#pragma unroll
    for (int c = 0; c < NR; ++c) {
      float mx = s[c][0][0];
#pragma unroll
      for (int t = 0; t < KT / 16; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[c][t][r]);
      m_new[c] = fmaxf(m[c], groups_max(mx));
      grown |= (m_new[c] - m[c]) * sc > RESCALE_LOG2;
    }
    if (__builtin_amdgcn_ballot_w64(grown) != 0ull) {
#pragma unroll
      for (int c = 0; c < NR; ++c) {
        const float alpha = m[c] == m_new[c] ? 1.f : __builtin_amdgcn_exp2f((m[c] - m_new[c]) * sc);
        m[c] = m_new[c];
        l[c] *= alpha;
#pragma unroll
        for (int u = 0; u < DV / 16; ++u)
#pragma unroll
          for (int r = 0; r < 4; ++r) o[c][u][r] *= alpha;
      }
    }
#pragma unroll
    for (int c = 0; c < NR; ++c) {
      const float msc = (m[c] == -INFINITY ? 0.f : m[c]) * sc;
#pragma unroll
      for (int t = 0; t < KT / 16; ++t) {
#pragma unroll
        for (int r = 0; r < 4; ++r) s[c][t][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[c][t][r], sc, -msc));
        l[c] += (s[c][t][0] + s[c][t][1]) + (s[c][t][2] + s[c][t][3]);
      }
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
        for (int c = 0; c < NR; ++c) o[c][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[c], o[c][u], 0, 0, 0);
      }
    }
  }
};
template <int DQ, int DV, int NR>
struct Rows32 {
  static constexpr int COLS = NR, ROWS = 32 * NR, CHUNKS = DV / 8;
  bf16x8_t qf[NR][DQ / 16];
  floatx16 o[NR][DV / 32];
  float m[NR], l[NR];
  static __device__ __forceinline__ int lane() { return threadIdx.x & 63; }
  static __device__ __forceinline__ int row(int c) { return 32 * c + (lane() & 31); }
  static __device__ __forceinline__ int dim(int q) { return 8 * q + 4 * (lane() >> 5); }
  static __device__ __forceinline__ bool lead() { return lane() < 32; }
  __device__ __forceinline__ floatx4 chunk(int c, int q) const {
    const floatx16& x = o[c][q >> 2];
    return floatx4{x[4 * (q & 3)], x[4 * (q & 3) + 1], x[4 * (q & 3) + 2], x[4 * (q & 3) + 3]};
  }
  __device__ __forceinline__ void init() {
#pragma unroll
    for (int c = 0; c < NR; ++c) {
      m[c] = -INFINITY;
      l[c] = 0.f;
#pragma unroll
      for (int u = 0; u < DV / 32; ++u)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[c][u][r] = 0.f;
    }
  }
  __device__ __forceinline__ void load(int c, const bf16_t* src, int kq, bool there) {
    const int hh = lane() >> 5;
    u32x4 raw[DQ / 16];
#pragma unroll
    for (int i = 0; i < DQ / 16; ++i) raw[i] = *reinterpret_cast<const u32x4*>(src + min(16 * i + 8 * hh, kq - 8));
#pragma unroll
    for (int i = 0; i < DQ / 16; ++i) qf[c][i] = __builtin_bit_cast(bf16x8_t, there && 16 * i + 8 * hh < kq ? raw[i] : u32x4{0u, 0u, 0u, 0u});
  }
  __device__ __forceinline__ void finish() {
#pragma unroll
    for (int c = 0; c < NR; ++c) {
      const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(l[c]), __float_as_uint(l[c]), false, false);
      l[c] = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    }
  }
  template <int KT>
  __device__ __forceinline__ void tile(const bf16_t* Kt, const bf16_t* Vt, float sc, bool whole, const int (&left)[NR], float*, int, unsigned) {
    const int hh = lane() >> 5, l32 = lane() & 31;
    floatx16 s[NR][KT / 32];
    constexpr int IG = DQ / 16 < 4 ? DQ / 16 : 4;      // 16 dims each: eight fragments of both key tiles in front of their products
#pragma unroll
    for (int i0 = 0; i0 < DQ / 16; i0 += IG) {
      bf16x8_t kf[KT / 32][IG];
#pragma unroll
      for (int i = 0; i < IG; ++i)
#pragma unroll
        for (int t = 0; t < KT / 32; ++t) kf[t][i] = *reinterpret_cast<const bf16x8_t*>(Kt + nat_off<DQ>(32 * t + l32, 2 * (i0 + i) + hh));
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < IG; ++i)
#pragma unroll
        for (int t = 0; t < KT / 32; ++t)
#pragma unroll
          for (int c = 0; c < NR; ++c)
            s[c][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[t][i], qf[c][i0 + i], i0 + i == 0 ? floatx16{} : s[c][t], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (!whole) {
#pragma unroll
      for (int c = 0; c < NR; ++c)
#pragma unroll
        for (int t = 0; t < KT / 32; ++t)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[c][t][r] = 32 * t + 8 * (r / 4) + 4 * hh + r % 4 < left[c] ? s[c][t][r] : -INFINITY;
    }
    bool grown = false;
    float m_new[NR];
#pragma unroll
    for (int c = 0; c < NR; ++c) {
      float mx = s[c][0][0];
#pragma unroll
      for (int t = 0; t < KT / 32; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[c][t][r]);
      const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
      m_new[c] = fmaxf(m[c], fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1])));
      grown |= (m_new[c] - m[c]) * sc > RESCALE_LOG2;
    }
    if (__builtin_amdgcn_ballot_w64(grown) != 0ull) {
#pragma unroll
      for (int c = 0; c < NR; ++c) {
        const float alpha = m[c] == m_new[c] ? 1.f : __builtin_amdgcn_exp2f((m[c] - m_new[c]) * sc);
        m[c] = m_new[c];
        l[c] *= alpha;
#pragma unroll
        for (int u = 0; u < DV / 32; ++u)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[c][u][r] *= alpha;
      }
    }
#pragma unroll
    for (int c = 0; c < NR; ++c) {
      const float msc = (m[c] == -INFINITY ? 0.f : m[c]) * sc;
#pragma unroll
      for (int t = 0; t < KT / 32; ++t)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
#pragma unroll
          for (int e = 0; e < 4; ++e) s[c][t][r + e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[c][t][r + e], sc, -msc));
          l[c] += (s[c][t][r] + s[c][t][r + 1]) + (s[c][t][r + 2] + s[c][t][r + 3]);
        }
    }
#pragma unroll
    for (int i = 0; i < KT / 32; ++i) {      // 32 keys: two products a block of dims
      TrnRegs vr[2][DV / 32];
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int u = 0; u < DV / 32; ++u) trn_issue<DV>(vr[e][u], Vt, 32 * u, 2 * i + e);
      bf16x8_t pf[NR][2];
#pragma unroll
      for (int c = 0; c < NR; ++c)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          floatx8 p;
#pragma unroll
          for (int r = 0; r < 8; ++r) p[r] = s[c][i][8 * e + r];
          pf[c][e] = __builtin_convertvector(p, bf16x8_t);
        }
      trn_wait();
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int u = 0; u < DV / 32; ++u) {
          const bf16x8_t vf = trn_frag(vr[e][u]);
#pragma unroll
          for (int c = 0; c < NR; ++c) o[c][u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[c][e], o[c][u], 0, 0, 0);
        }
    }
  }
};

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
// Kept scores of own keys j .. j + 3 for four rows from r0 on (rows beyond the last: the last one's).
struct PrefixScores { floatx4 x[4]; };
__device__ __forceinline__ PrefixScores prefix_scores(const PrefixArgs& a, long long bh, int r0, int j) {
  const float* const scores = a.scores + bh * a.own_rows * a.own_pad + j;
  PrefixScores s;
#pragma unroll
  for (int i = 0; i < 4; ++i) s.x[i] = *reinterpret_cast<const floatx4*>(scores + static_cast<long long>(min(r0 + i, a.own_rows - 1)) * a.own_pad);
  return s;
}
__device__ __forceinline__ floatx4 prefix_weights_before(const PrefixArgs& a, long long bh, int j, int n) {
  floatx4 w = {0.f, 0.f, 0.f, 0.f};
  if (a.w_in) {
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = a.w_in[bh * a.cap + min(j + e, n - 1)];
  }
  return w;
}
// Accumulated weights of own keys j .. j + 3 (those below n) of request and head bh, from the kept scores of its rows: w_out = w_in + sum over the rows of
// exp2(score - lse2), nothing where the score is -inf (the row does not see the key, whatever its lse2 is).  early: prefix_scores() of rows 0 .. 3, before: prefix_weights_before(), both asked for in front of what lse2 waits for.
__device__ __forceinline__ void prefix_weigh(const PrefixArgs& a, long long bh, PrefixScores early, const floatx4& before, const float* lse2, int n, int j) {
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  for (int r = 0; r < a.own_rows; r += 4) {
    if (r > 0) early = prefix_scores(a, bh, r, j);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float ref = r + i < a.own_rows ? lse2[r + i] : INFINITY;
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += early.x[i][e] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(early.x[i][e] - ref);
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (j + e < n) a.w_out[bh * a.cap + j + e] = before[e] + sum[e];
}

// Rows of an item: up to 16 or 32, its key tiles shared out over the wavefronts; up to 64, 128 or 256, 16, 32 or 64 a wavefront, and every tile shared.
enum { ROWS_16 = 0, ROWS_32 = 1, ROWS_64 = 2, ROWS_128 = 3, ROWS_256 = 4 };
// Key tiles, LDS buffers of NB stages and their bytes.  Shared tiles have 64 keys; a wavefront's own ones 32, so that two stages for four wavefronts take
// as much as four stages of shared tiles.
template <int DQ, int DV, int ROWS, int NB>
struct PrefixShape {
  static constexpr bool SHARE = ROWS >= ROWS_64;
  typedef std::conditional_t<ROWS >= ROWS_128, Rows32<DQ, DV, ROWS == ROWS_256 ? 2 : 1>, Rows16<DQ, DV, ROWS == ROWS_32 ? 2 : 1>> Rows;
  static constexpr int KT = SHARE ? 64 : 32, ROW_TILE = 16 << ROWS;
  static constexpr int stage = (SHARE ? 1 : 4) * KT * (DQ + DV) * 2, join = SHARE ? 0 : (4 * Rows::COLS * (DV * 16 + 32) + Rows::COLS * 16) * 4;
  static constexpr int lds(int stages) { return (stages < NB ? stages : NB) * stage > join ? (stages < NB ? stages : NB) * stage : join; }
};

// An item.  Shared tiles: the four wavefronts take their rows each.  Otherwise they share the item's rows and take the key tiles in turn, from
// LDS buffers of their own without a barrier, and join at the end.  NB stages: NB - 1 tiles are on their way; `stages` of them are there.
template <int DQ, int DV, int ROWS, int NB>
__device__ __forceinline__ void prefix_rows(const PrefixArgs& a, bf16_t* const lds_all, int stages) {
  typedef PrefixShape<DQ, DV, ROWS, NB> Shape;
  typedef typename Shape::Rows Rows;
  constexpr bool SHARE = Shape::SHARE;
  constexpr int KT = Shape::KT, WAVES = SHARE ? 4 : 1, COLS = Rows::COLS;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Item it;
  if (!prefix_item<KT>(a, Shape::ROW_TILE, it)) return;
  bf16_t* const buf = lds_all + (SHARE ? 0 : wave * stages * (KT * (DQ + DV)));      // [stages][K tile, V tile]

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
    const char *const kb = (own ? ok : pk) + first * ldk, *const vb = (own ? ov : pv) + first * ldv;
    if (own ? a.own_once : a.prefix_once) {
      kl.template issue<2>(at, kb, static_cast<unsigned>(ldk), valid);
      vl.template issue<2>(at + KT * DQ, vb, static_cast<unsigned>(ldv), valid);
    } else {
      kl.template issue<0>(at, kb, static_cast<unsigned>(ldk), valid);
      vl.template issue<0>(at + KT * DQ, vb, static_cast<unsigned>(ldv), valid);
    }
  };
  constexpr int STEP = SHARE ? 1 : 4;
  const int first = it.t0 + (SHARE ? 0 : wave);
#pragma unroll
  for (int i = 0; i < NB - 1; ++i)
    if (first + i * STEP < it.t1) issue(first + i * STEP, i);

  // the wavefront's rows: queries straight from memory, rows and dims outside are zero
  Rows st;
  st.init();
  const int first_row = SHARE ? wave * Rows::ROWS : 0;
  const bool idle = first_row >= it.n_rows;      // a wavefront without rows only loads
  int seen[COLS];                                // own keys the row sees
  unsigned kept = 0u;
#pragma unroll
  for (int c = 0; c < COLS; ++c) {
    const int r = first_row + Rows::row(c), row = it.row0 + min(r, it.n_rows - 1), token = row / a.g;
    st.load(c, a.q + token * a.ld_q + static_cast<long long>(it.hk * a.g + (row - token * a.g)) * a.kq, a.kq, r < it.n_rows);
    seen[c] = it.b < 0 ? 0 : own_visible(own_len(a, it.b), a.L, token - it.b * a.L);
    kept |= r < it.n_rows ? 1u << c : 0u;
  }
  int least = seen[0];
#pragma unroll
  for (int c = 1; c < COLS; ++c) least = min(least, seen[c]);
  least = static_cast<int>(wave_umin(static_cast<uint32_t>(least)));      // own keys that every row sees
  // scores of own keys are kept where the call wants weights (then an item has all rows of its request)
  float* const keep = a.scores && it.b >= 0 ? a.scores + (static_cast<long long>(it.b * a.h_kv + it.hk) * a.own_rows + first_row + Rows::row(0)) * a.own_pad : nullptr;

  int j = first;
  while (j < it.t1) {
#pragma unroll
    for (int n = 0; n < NB; ++n) {      // a stage's buffer is known to the compiler
      if (j >= it.t1) break;
      // of the operations issued since this tile's loads, at least those of the NB - 2 tiles behind it are loads that may still be under way
      if (NB > 2 && j + (NB - 2) * STEP < it.t1) loads_wait<(NB - 2) * (KvLoader<DQ, KT, WAVES>::PER + KvLoader<DV, KT, WAVES>::PER)>();
      else stream_wait();
      if (SHARE) __syncthreads();
      if (j + (NB - 1) * STEP < it.t1) issue(j + (NB - 1) * STEP, (n + NB - 1) % NB);
      if (!idle) {
        const bool own = j >= it.split;
        const int k0 = (own ? j - it.split : j) * KT;
        int left[COLS];
#pragma unroll
        for (int c = 0; c < COLS; ++c) left[c] = (own ? seen[c] : a.P) - k0;
        const bf16_t* const at = buf + n * (KT * (DQ + DV));
        st.template tile<KT>(at, at + KT * DQ, a.sc, k0 + KT <= (own ? least : a.P), left, own && keep ? keep + k0 : nullptr, a.own_pad, kept);
      }
      j += STEP;
    }
  }
  st.finish();

  // this lane's four dims of chunk q of its row: normalised into the output, or a piece for the join
  const auto write = [&](int c, int q, const floatx4& acc, float m, float l) __attribute__((always_inline)) {
    const int r = first_row + Rows::row(c), row = it.row0 + r, d = Rows::dim(q);
    if (r >= it.n_rows) return;
    if (a.slots == 0) {
      const int token = row / a.g, head = it.hk * a.g + (row - token * a.g);
      if (d < a.kv) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        floatx4 f;
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = acc[i] * inv;
        *reinterpret_cast<bf16x4_t*>(a.o + token * a.ld_o + static_cast<long long>(head) * a.kv + d) = __builtin_convertvector(f, bf16x4_t);
      }
      if (q == 0 && a.lse && Rows::lead()) {
        const int b = token / a.L;
        a.lse[(static_cast<long long>(b) * a.h + head) * a.L + (token - b * a.L)] = l == 0.f ? -INFINITY : (m * a.sc + __builtin_amdgcn_logf(l)) * LN2;
      }
    } else {
      const long long at = (static_cast<long long>(it.hk) * a.rows + row) * a.slots + it.slot;
      if (d < a.kv) *reinterpret_cast<floatx4*>(a.part_o + at * a.kv + d) = acc;
      if (q == 0 && Rows::lead()) *reinterpret_cast<float2*>(a.part_ml + 2 * at) = float2{m * a.sc, l};
    }
  };
  if constexpr (SHARE) {
#pragma unroll
    for (int c = 0; c < COLS; ++c)
#pragma unroll
      for (int q = 0; q < Rows::CHUNKS; ++q) write(c, q, st.chunk(c, q), st.m[c], st.l[c]);
  } else {
    constexpr int U = DV / 16;
    __syncthreads();
    float* const part = reinterpret_cast<float*>(lds_all);       // [4][COLS][U][64][4]
    float* const ms = part + 4 * COLS * DV * 16;                 // [4][COLS][16] each
    float* const ls = ms + 4 * COLS * 16;
    float* const lse2 = ls + 4 * COLS * 16;                      // [COLS][16]
    const int l16 = lane & 15;
#pragma unroll
    for (int c = 0; c < COLS; ++c) {
#pragma unroll
      for (int u = 0; u < U; ++u) *reinterpret_cast<floatx4*>(part + (((wave * COLS + c) * U + u) * 64 + lane) * 4) = st.chunk(c, u);
      if (Rows::lead()) {
        ms[(wave * COLS + c) * 16 + l16] = st.m[c];
        ls[(wave * COLS + c) * 16 + l16] = st.l[c];
      }
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < COLS; ++c) {
      float m_all = ms[c * 16 + l16], al[4], l_all = 0.f;
#pragma unroll
      for (int w = 1; w < 4; ++w) m_all = fmaxf(m_all, ms[(w * COLS + c) * 16 + l16]);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float m = ms[(w * COLS + c) * 16 + l16];
        al[w] = m == m_all ? (m == -INFINITY ? 0.f : 1.f) : __builtin_amdgcn_exp2f((m - m_all) * a.sc);
        l_all += al[w] * ls[(w * COLS + c) * 16 + l16];
      }
#pragma unroll
      for (int u0 = 0; u0 < U; u0 += 4) {
        const int u = u0 + wave;
        if (u >= U) break;
        floatx4 f = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const floatx4 x = *reinterpret_cast<const floatx4*>(part + (((w * COLS + c) * U + u) * 64 + lane) * 4);
#pragma unroll
          for (int i = 0; i < 4; ++i) f[i] += al[w] * x[i];
        }
        write(c, u, f, m_all, l_all);
      }
      if (a.slots == 0 && wave == 0 && Rows::lead()) lse2[c * 16 + l16] = l_all == 0.f ? INFINITY : m_all * a.sc + __builtin_amdgcn_logf(l_all);
    }
    if (a.slots == 0 && keep) {      // the item has seen all of its rows' keys: weights from the scores it kept
      __threadfence_block();
      __syncthreads();
      const long long bh = static_cast<long long>(it.b) * a.h_kv + it.hk;
      for (int k = threadIdx.x * 4; k < it.own_n; k += 1024)
        prefix_weigh(a, bh, prefix_scores(a, bh, 0, k), prefix_weights_before(a, bh, k, it.own_n), lse2, it.own_n, k);
    }
  }
}

// OWN: rows of the items of a request; PREFIX: of those of the prefix alone, in front of them in the grid (the same: all items are of one kind).
// Shared tiles have four stages beside own ones (whose LDS is there anyway), else few enough for several workgroups on a compute unit.
template <int DQ, int DV, int OWN, int PREFIX>
struct PrefixKernel {
  static constexpr int NB_S = DQ + DV <= 128 && OWN == ROWS_64 ? 3 : 2, NB_O = OWN >= ROWS_64 ? NB_S : 2, NB_P = PREFIX < ROWS_64 ? 2 : (OWN >= ROWS_64 ? NB_S : 4);
  static constexpr int lds(int o_stages, int p_stages) {      // a call of one kind has its prefix items in o_stages too
    const int own = PrefixShape<DQ, DV, OWN, NB_O>::lds(o_stages), pre = OWN == PREFIX ? 0 : PrefixShape<DQ, DV, PREFIX, NB_P>::lds(p_stages);
    return own > pre ? own : pre;
  }
};
// Two wavefronts a SIMD at least: the register file then has no accumulation half, and the scores need no moves between the halves.
template <int DQ, int DV, int OWN, int PREFIX>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void prefix_attn_kernel(const PrefixArgs a) {
  typedef PrefixKernel<DQ, DV, OWN, PREFIX> K;
  extern __shared__ __attribute__((aligned(16))) bf16_t lds_all[];      // one object: see attn.hip
  if (OWN != PREFIX && static_cast<int>(blockIdx.x) < a.p_items) prefix_rows<DQ, DV, PREFIX, K::NB_P>(a, lds_all, min(a.p_stages, K::NB_P));
  else prefix_rows<DQ, DV, OWN, K::NB_O>(a, lds_all, min(a.o_stages, K::NB_O));
}

// The pairs that are built: items of one kind for every width; apart, own tiles beside the prefix's for narrow heads, and shared ones for wide heads,
// where own tiles of every wavefront would leave a compute unit one workgroup (prefix_plan()).
#define PREFIX_KINDS_ALL(X, DQ, DV) X(DQ, DV, ROWS_16, ROWS_16) X(DQ, DV, ROWS_32, ROWS_32) X(DQ, DV, ROWS_64, ROWS_64) X(DQ, DV, ROWS_128, ROWS_128)
#define PREFIX_KINDS_NARROW(X, DQ, DV)                                                                 \
  X(DQ, DV, ROWS_16, ROWS_32) X(DQ, DV, ROWS_16, ROWS_64) X(DQ, DV, ROWS_32, ROWS_64)                  \
  X(DQ, DV, ROWS_16, ROWS_128) X(DQ, DV, ROWS_32, ROWS_128) X(DQ, DV, ROWS_256, ROWS_256)
#define PREFIX_KINDS_WIDE(X, DQ, DV) X(DQ, DV, ROWS_64, ROWS_128)
constexpr bool prefix_wide(int dq, int dv) { return dq + dv > 128; }
template <int DQ, int DV, int OWN, int PREFIX>
static hipError_t prefix_launch(const PrefixArgs& a, unsigned grid, hipStream_t st) {
  constexpr int most = PrefixKernel<DQ, DV, OWN, PREFIX>::lds(4, 4);
  const int lds = PrefixKernel<DQ, DV, OWN, PREFIX>::lds(a.o_stages, a.p_stages);
  const auto kern = prefix_attn_kernel<DQ, DV, OWN, PREFIX>;
  static LdsAttrOnce attr_once;
  if (most > 64 * 1024) {
    const hipError_t e = attr_once.ensure(reinterpret_cast<const void*>(kern), most);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kern, dim3(grid), dim3(256), lds, st, a);
  return hipGetLastError();
}
template <int DQ, int DV>
static hipError_t prefix_launch_width(const PrefixArgs& a, int own, int prefix, unsigned grid, hipStream_t st) {
#define PREFIX_KIND(Q, V, O, P) if (own == O && prefix == P) return prefix_launch<Q, V, O, P>(a, grid, st);
  PREFIX_KINDS_ALL(PREFIX_KIND, DQ, DV)
  if constexpr (prefix_wide(DQ, DV)) {
    PREFIX_KINDS_WIDE(PREFIX_KIND, DQ, DV)
  } else {
    PREFIX_KINDS_NARROW(PREFIX_KIND, DQ, DV)
  }
#undef PREFIX_KIND
  return hipErrorInvalidValue;
}
// by the width of the queries, a translation unit each
hipError_t prefix_launch_32(const PrefixArgs& a, int dv, int own, int prefix, unsigned grid, hipStream_t st);
hipError_t prefix_launch_64(const PrefixArgs& a, int dv, int own, int prefix, unsigned grid, hipStream_t st);
hipError_t prefix_launch_128(const PrefixArgs& a, int dv, int own, int prefix, unsigned grid, hipStream_t st);
