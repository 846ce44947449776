// Attention of new tokens over caches of 8-bit floats (not part of the C ABI).
//
// o = sum_j p_j v_j / sum_j p_j, p_j = exp(scale q.k_j - m), one pass over the keys with a running maximum.  An item is a request, a key/value head,
// 16 T of its queries and a piece of its keys; four wavefronts take the piece's groups of 32 keys in turn, each by itself, and meet in LDS at the end.
// Neither operand needs LDS:
//   scores^T = K Q^T   A: 16 keys x 32 dims.  A lane asks for the 8 (two steps: 16) bytes of its key that its slots of the contraction are given; which dims
//                      those are does not matter as long as the queries' fragments hold the same.  Codes become bf16 exactly.
//   o^T = V^T P^T      A: 16 dims x 32 keys.  A lane holds W neighbouring dims of eight keys: its part of W fragments, once the bytes of two keys are
//                      paired (a permutation instruction for two dims) and converted.  The eight keys are those whose scores the lane computed, so the
//                      probabilities go from accumulator to operand without leaving the lane.
// A key's scale multiplies its score.  A value's is split: its power of two (2^-100 for smaller scales: bf16 then holds every code times it) goes into the conversion, exactly,
// and what is left (1 for the scales that an append writes) into the probability.  Both are the same for 16 keys, a block or part of one.
// Bounds.  Single tokens: memory; 64 requests, 8 heads of 64 dims, 16384 keys: 715 MB in 131 to 136 us, 5.3 to 5.4 TB/s (a large read here 6.35).  Prompts: vector
// instructions, exponentials and the conversion of codes in front of 16 dense products each; 8 requests of 509 tokens, 32 heads of 64 dims on 8, over 4096 keys: 140 to 146 us,
// 0.56 to 0.58 PFLOP/s.  Behind it: accumulators in vector registers alone (moves to and from the other half of the register file were a fifth of all instructions), loads that
// are asked for without branches.
#pragma once
#include "quant_cache.h"

typedef __bf16 qa_bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 qa_bf16x2 __attribute__((ext_vector_type(2)));
typedef float qa_floatx4 __attribute__((ext_vector_type(4)));
typedef float qa_floatx8 __attribute__((ext_vector_type(8)));
typedef unsigned qa_uintx4 __attribute__((ext_vector_type(4)));
typedef unsigned qa_uintx2 __attribute__((ext_vector_type(2)));

#define QA_RESCALE 8.0f        // growth of a row's maximum, in binades, that brings its sums to the new one
#define QA_LN2 0.6931471805599453f
#define QA_LEAST (27u << 23)   // bits of 2^-100

// two codes times the power of two below `scale` (the instruction looks at its exponent alone)
template <bool HIGH>
__device__ __forceinline__ unsigned qa_pair(unsigned codes, float scale = 1.0f) { return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, HIGH)); }
// eight codes of a key to a fragment
__device__ __forceinline__ qa_bf16x8 qa_frag(unsigned lo, unsigned hi) {
  return __builtin_bit_cast(qa_bf16x8, qa_uintx4{qa_pair<false>(lo), qa_pair<true>(lo), qa_pair<false>(hi), qa_pair<true>(hi)});
}
// over the four groups of 16 lanes
__device__ __forceinline__ float qa_max4(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float qa_sum4(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// ONCE: past the caches
template <bool ONCE, typename V>
__device__ __forceinline__ V qa_load(const unsigned char* p) {
  if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
  else return *reinterpret_cast<const V*>(p);
}

// One group of 32 keys as it comes from memory.
template <int KQ, int W>
struct QaRaw {
  unsigned k[2][2 * KQ];            // two tiles of 16 keys
  unsigned v[8][W > 4 ? 2 : 1];     // keys 4 g .. + 3 and 16 + 4 g .. + 3
  float ks[2], vs[2];
};

// What is written for a row whose maximum (base 2), sum and weighted values over all keys are known; prior: the result over other keys, joined in.
__device__ __forceinline__ void qa_finish_row(float& m, float& l, float& in, const float* lse_in) {
  in = 0.f;
  if (lse_in) {
    const float p = *lse_in * 1.4426950408889634f;
    if (p != -INFINITY) {
      const float top = fmaxf(m, p), ref = top == -INFINITY ? 0.f : top;
      in = __builtin_amdgcn_exp2f(p - ref);
      const float own = __builtin_amdgcn_exp2f(m - ref);
      l = (l == 0.f ? 0.f : l * own) + in;
      m = ref;
    }
  }
}

template <int T, int KQ, int W, bool ONCE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(T == 1 ? (W < 8 && KQ < 4 ? 4 : 3) : 2)))
void quant_attn_kernel(const QuantAttnArgs a) {
  constexpr int WAVES = 4, ROWS = 16 * T, KV = 16 * W, PITCH = KV + 4;
  __shared__ __attribute__((aligned(16))) float lds_o[WAVES][16][PITCH];
  __shared__ float lds_m[WAVES][16], lds_l[WAVES][16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, g = lane >> 4;
  // the row blocks and pieces of a head's keys on one XCD
  const int per = a.row_blocks * a.pieces, j = blockIdx.x >> 3, group = j / per * 8 + (blockIdx.x & 7), in_group = j % per;
  if (group >= a.B * a.h_kv) return;
  const int b = group / a.h_kv, hk = group - b * a.h_kv, rb = in_group / a.pieces, piece = in_group - rb * a.pieces;
  const int len = min(max(a.lens[b], 0), a.own_max), row0 = rb * ROWS, row_last = min(row0 + ROWS, a.rows) - 1;
  // keys that the first and the last of these queries see
  const int sees_first = len - a.L + 1 + row0 / a.g, sees_last = len - a.L + 1 + row_last / a.g;
  // pieces of equal length, by the request's own number of keys: ragged lengths then make no empty ones (a multiple of the four wavefronts' groups)
  const int piece_keys = ((len + a.pieces - 1) / a.pieces + 127) & ~127, key0 = piece * piece_keys, key1 = min(key0 + piece_keys, sees_last);

  qa_bf16x8 qf[T][KQ];
  int sees[T];
#pragma unroll
  for (int t = 0; t < T; ++t) {
    const int row = min(row0 + t * 16 + l16, a.rows - 1), tok = row / a.g, head = hk * a.g + row - tok * a.g;
    sees[t] = len - a.L + 1 + tok;
    const bf16_t* const q = a.q + (static_cast<long long>(b) * a.L + tok) * a.ld_q + head * a.kq;
#pragma unroll
    for (int s = 0; s < KQ; ++s) {
      const int d = (s & ~1) * 32 + (s + 1 < KQ || (s & 1) ? 16 * g + 8 * (s & 1) : 8 * g);      // pairs of steps: 16 dims a lane; a last single one: 8
      qf[t][s] = d < a.kq ? *reinterpret_cast<const qa_bf16x8*>(q + d) : qa_bf16x8{};
    }
  }
  const unsigned char* const kb = a.k + b * a.k_sb + hk * a.k_sh;
  const unsigned char* const vb = a.v + b * a.v_sb + hk * a.v_sh;
  const float* const ksb = a.k_scale + static_cast<long long>(group) * a.blocks;
  const float* const vsb = a.v_scale + static_cast<long long>(group) * a.blocks;
  // dims beyond a head's width: the key's first ones again (against zeros of the query), the value's first ones again (never written)
  unsigned kd[(KQ + 1) / 2];
#pragma unroll
  for (int s = 0; s < KQ; s += 2) {
    const int d = s * 32 + (s + 1 < KQ ? 16 : 8) * g;
    kd[s / 2] = d < a.kq ? d : 0;
  }
  const unsigned vd = W * l16 < a.kv ? W * l16 : 0, kst = static_cast<unsigned>(a.k_st), vst = static_cast<unsigned>(a.v_st);

  const auto fetch = [&](const unsigned char* kp, const unsigned char* vp, auto&& krow, auto&& vrow, QaRaw<KQ, W>& x) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int s = 0; s < KQ; s += 2) {
        if (s + 1 < KQ) {
          const qa_uintx4 u = qa_load<ONCE, qa_uintx4>(krow(kp, i) + kd[s / 2]);
          x.k[i][2 * s] = u.x; x.k[i][2 * s + 1] = u.y;
          x.k[i][(2 * s + 2) % (2 * KQ)] = u.z; x.k[i][(2 * s + 3) % (2 * KQ)] = u.w;
        } else {
          const qa_uintx2 u = qa_load<ONCE, qa_uintx2>(krow(kp, i) + kd[s / 2]);
          x.k[i][2 * s] = u.x; x.k[i][2 * s + 1] = u.y;
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const unsigned char* const p = vrow(vp, e);
      if constexpr (W == 8) {
        const qa_uintx2 u = qa_load<ONCE, qa_uintx2>(p);
        x.v[e][0] = u.x; x.v[e][W > 4 ? 1 : 0] = u.y;
      } else if constexpr (W == 4) {
        x.v[e][0] = qa_load<ONCE, unsigned>(p);
      } else {
        x.v[e][0] = qa_load<ONCE, unsigned short>(p);
      }
    }
  };
  const unsigned klane = l16 * kst, vlane = 4 * g * vst + vd;
  const auto load = [&](int c, QaRaw<KQ, W>& x) __attribute__((always_inline)) {
    const int k0 = c * 32;
    const unsigned char* const kp = kb + static_cast<long long>(k0) * a.k_st;
    const unsigned char* const vp = vb + static_cast<long long>(k0) * a.v_st;
    if (k0 + 32 <= key1) {
      fetch(kp, vp, [&](const unsigned char* p, int i) __attribute__((always_inline)) { return p + 16 * i * a.k_st + klane; },
            [&](const unsigned char* p, int e) __attribute__((always_inline)) { return p + (16 * (e >> 2) + (e & 3)) * a.v_st + vlane; }, x);
    } else {      // rows beyond the last key repeat it: nothing behind a length is read
      const int most = key1 - 1 - k0;
      fetch(kp, vp, [&](const unsigned char* p, int i) __attribute__((always_inline)) { return p + static_cast<unsigned>(min(16 * i + l16, most)) * kst; },
            [&](const unsigned char* p, int e) __attribute__((always_inline)) { return p + (static_cast<unsigned>(min(16 * (e >> 2) + 4 * g + (e & 3), most)) * vst + vd); }, x);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int blk = min(k0 + 16 * i, key1 - 1) >> a.block_log2;
      x.ks[i] = ksb[blk];
      x.vs[i] = vsb[blk];
    }
  };

  qa_floatx4 o[T][W];
  float m[T], l[T];
#pragma unroll
  for (int t = 0; t < T; ++t) {
    m[t] = -INFINITY;
    l[t] = 0.f;
#pragma unroll
    for (int f = 0; f < W; ++f) o[t][f] = qa_floatx4{0.f, 0.f, 0.f, 0.f};
  }
  const auto step = [&](int c, const QaRaw<KQ, W>& x) __attribute__((always_inline)) {
    qa_bf16x8 vf[W];
    const unsigned vs[2] = {__float_as_uint(x.vs[0]), __float_as_uint(x.vs[1])};
    const float two_to[2] = {__uint_as_float(max(vs[0], QA_LEAST)), __uint_as_float(max(vs[1], QA_LEAST))};
#pragma unroll
    for (int f = 0; f < W; f += 2) {
      unsigned w[2][4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const unsigned two = __builtin_amdgcn_perm(x.v[2 * e + 1][f >> 2], x.v[2 * e][f >> 2], f & 2 ? 0x07030602u : 0x05010400u);
        w[0][e] = qa_pair<false>(two, two_to[e >> 1]);
        w[1][e] = qa_pair<true>(two, two_to[e >> 1]);
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) vf[f + u] = __builtin_bit_cast(qa_bf16x8, qa_uintx4{w[u][0], w[u][1], w[u][2], w[u][3]});
    }
    const bool powers = ((vs[0] | vs[1]) & 0x7fffffu) == 0u && min(vs[0], vs[1]) >= QA_LEAST;      // what an append writes
    qa_floatx4 s[T][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      qa_bf16x8 kf[KQ];
#pragma unroll
      for (int u = 0; u < KQ; ++u) kf[u] = qa_frag(x.k[i][2 * u], x.k[i][2 * u + 1]);
#pragma unroll
      for (int t = 0; t < T; ++t) {
        s[t][i] = qa_floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < KQ; ++u) s[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[u], qf[t][u], s[t][i], 0, 0, 0);
      }
    }
    // never 0, which a key's tiny scale makes: times the -inf of a masked key it would be NaN (the least number instead moves no score by 2^-21)
    const auto positive = [](float f) __attribute__((always_inline)) { return __uint_as_float(max(__float_as_uint(f), 1u)); };
    const float by[2] = {positive(x.ks[0] * a.scale_log2), positive(x.ks[1] * a.scale_log2)};
    if (c * 32 + 32 > sees_first) {
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int key = c * 32 + 16 * (e >> 2) + 4 * g + (e & 3);
          s[t][e >> 2][e & 3] = key < sees[t] && key < key1 ? s[t][e >> 2][e & 3] : -INFINITY;
        }
    }
    // the lane's own largest: a row's reference has to be near it, not equal to it, so the lanes of a row agree on new ones only where one falls behind
    float top[T];
    bool behind = false;
#pragma unroll
    for (int t = 0; t < T; ++t) {
      float most[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int e = 0; e < 8; ++e) most[e >> 2] = fmaxf(most[e >> 2], s[t][e >> 2][e & 3]);
      top[t] = fmaxf(most[0] * by[0], most[1] * by[1]);
      behind = behind || top[t] > m[t] + QA_RESCALE;
    }
    if (__any(behind)) {
#pragma unroll
      for (int t = 0; t < T; ++t) {
        const float up = fmaxf(m[t], qa_max4(top[t])), f0 = m[t] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[t] - up);
        m[t] = up;
        l[t] = l[t] == 0.f ? 0.f : l[t] * f0;
#pragma unroll
        for (int f = 0; f < W; ++f) o[t][f] *= f0;
      }
    }
#pragma unroll
    for (int t = 0; t < T; ++t) {
      const float ref = m[t] == -INFINITY ? 0.f : m[t];
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][e >> 2][e & 3], by[e >> 2], -ref));
      l[t] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
      if (!powers) {
        float rest[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) rest[i] = vs[i] >= QA_LEAST ? __uint_as_float((vs[i] & 0x807fffffu) | 0x3f800000u) : x.vs[i] * 0x1p100f;
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] *= rest[e >> 2];
      }
      qa_floatx8 w;
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = p[e];
      const qa_bf16x8 pf = __builtin_convertvector(w, qa_bf16x8);
#pragma unroll
      for (int f = 0; f < W; ++f) o[t][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[f], pf, o[t][f], 0, 0, 0);
    }
  };
  const int end = (key1 + 31) >> 5;      // groups up to here; key0 is a multiple of 128
  int c = (key0 >> 5) + wave;
  // The next group is on its way while one is computed, in two sets of registers in turn.  Behind the last one it is asked for again: a load that may or may not
  // have been issued makes the compiler wait for every other as well.
  if (c < end) {
    const int last = c + (end - 1 - c) / WAVES * WAVES;
    QaRaw<KQ, W> x;
    load(c, x);
    QaRaw<KQ, W> y;
    for (;;) {
      load(min(c + WAVES, last), y);
      step(c, x);
      if (c == last) break;
      c += WAVES;
      load(min(c + WAVES, last), x);
      step(c, y);
      if (c == last) break;
      c += WAVES;
    }
  }

  // The wavefronts meet, 16 queries at a time: lane (l16, g) holds query l16, dims W (4 g + r) + f.
  const int kv1 = a.kv;
#pragma unroll
  for (int t = 0; t < T; ++t) {
    if (t) __syncthreads();
    const float sum = qa_sum4(l[t]);
    if (g == 0) { lds_m[wave][l16] = m[t]; lds_l[wave][l16] = sum; }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int f = 0; f < W; ++f) lds_o[wave][l16][W * (4 * g + r) + f] = o[t][f][r];
    __syncthreads();
    const int rl = threadIdx.x >> 4, at = (threadIdx.x & 15) * W, row = row0 + t * 16 + rl;
    float top = -INFINITY, all = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) top = fmaxf(top, lds_m[w][rl]);
    const float ref = top == -INFINITY ? 0.f : top;
    float v[W], f0[WAVES];
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float lw = lds_l[w][rl];
      f0[w] = lw == 0.f ? 0.f : __builtin_amdgcn_exp2f(lds_m[w][rl] - ref);
      all += lw == 0.f ? 0.f : lw * f0[w];
    }
#pragma unroll
    for (int f = 0; f < W; ++f) {
      v[f] = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) v[f] += lds_o[w][rl][at + f] * f0[w];
    }
    if (row > row_last || at >= kv1) continue;
    if (a.part) {
      float* const p = a.part + ((static_cast<long long>(group) * a.row_blocks + rb) * a.pieces + piece) * (ROWS * (KV + 2ll)) + (t * 16 + rl) * (KV + 2);
#pragma unroll
      for (int f = 0; f < W; ++f) p[at + f] = v[f];
      if (at == 0) { p[KV] = top; p[KV + 1] = all; }
      continue;
    }
    const int tok = row / a.g, head = hk * a.g + row - tok * a.g;
    const long long flat = (static_cast<long long>(b) * a.h + head) * a.L + tok, orow = static_cast<long long>(b) * a.L + tok;
    float in = 0.f, mm = top, ll = all;
    qa_finish_row(mm, ll, in, a.lse_in ? a.lse_in + flat : nullptr);
    const float own = all == 0.f ? 0.f : __builtin_amdgcn_exp2f(top - (mm == -INFINITY ? 0.f : mm)), inv = ll == 0.f ? 0.f : 1.f / ll;
    if (a.lse && at == 0) a.lse[flat] = ll == 0.f ? -INFINITY : mm * QA_LN2 + logf(ll);
#pragma unroll
    for (int f = 0; f < W; ++f) {
      float y = v[f] * own;
      if (in != 0.f) y += in * bf16_to_f32(a.o_in[orow * a.ld_oi + head * a.kv + at + f]);
      a.o[orow * a.ld_o + head * a.kv + at + f] = f32_to_bf16(y * inv);
    }
  }
}

template <int T, int KQ, int W, bool ONCE>
static hipError_t quant_attn_launch(const QuantAttnArgs& a, hipStream_t st) {
  const int groups = (a.B * a.h_kv + 7) / 8 * 8;
  hipLaunchKernelGGL((quant_attn_kernel<T, KQ, W, ONCE>), dim3(static_cast<unsigned>(groups) * a.row_blocks * a.pieces), dim3(256), 0, st, a);
  return hipGetLastError();
}
template <int W>
static hipError_t quant_attn_dispatch(const QuantAttnArgs& a, int T, int KQ, bool once, hipStream_t st) {
#define QA_CASE(t, k) if constexpr (t <= quant_attn_tiles(k, W)) if (T == t && KQ == k) return t == 1 && once ? quant_attn_launch<t, k, W, t == 1>(a, st) : quant_attn_launch<t, k, W, false>(a, st);
  QA_CASE(1, 1) QA_CASE(1, 2) QA_CASE(1, 3) QA_CASE(1, 4) QA_CASE(2, 1) QA_CASE(2, 2) QA_CASE(2, 3) QA_CASE(2, 4) QA_CASE(4, 1) QA_CASE(4, 2) QA_CASE(4, 3) QA_CASE(4, 4)
#undef QA_CASE
  return hipErrorInvalidValue;
}
