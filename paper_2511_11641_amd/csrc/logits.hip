// Penalties, biases, temperature and masks on logits, with the best token and the log-sum-exp of every row.
//
// A workgroup takes a range of the vocabulary of one row.  It counts the row's history and bias entries that fall into its range in LDS
// (integer atomics: the order does not show), then passes over its logits once, 16 bytes a lane: load, transform, store, running maximum with
// its token and running sum of exponentials.  The ranges' results of a row are joined by a second launch (none where one range is the row).
// Nothing is added in an order that varies: results repeat bit for bit.
#include "common.h"

#define LOGITS_THREADS 256
#define LOGITS_BIAS_ONE (1 << 22)      // a counter holds occurrences in the history (22 bits) and, above them, bias entries (10 bits)

struct LogitsPart {
  float m, s;      // maximum and sum of exp(x - m)
  int at;          // its lowest token, -1: none
  int pad;
};
struct LogitsArgs {
  ecospa_logits q;
  LogitsPart* part;
  int range, ranges;      // tokens of a workgroup, a multiple of 8
};

// (m, at) of the better of two: larger value, then lower token
__device__ __forceinline__ void logits_join(float& m, float& s, int& at, float m2, float s2, int at2) {
  const float M = fmaxf(m, m2), ref = M == -INFINITY ? 0.f : M;
  const float f = m == M ? 1.f : __expf(m - ref), f2 = m2 == M ? 1.f : __expf(m2 - ref);
  s = (m == -INFINITY && s == 0.f ? 0.f : s * f) + (m2 == -INFINITY && s2 == 0.f ? 0.f : s2 * f2);
  if (at2 >= 0 && (at < 0 || m2 > m || (m2 == m && at2 < at))) at = at2;
  m = M;
}
__device__ __forceinline__ void logits_finish(const LogitsArgs& a, int b, float m, float s, int at) {
  if (a.q.pick) a.q.pick[b] = at;
  if (a.q.lse) a.q.lse[b] = m == INFINITY ? INFINITY : (m == -INFINITY ? 0.f : m) + logf(s);
}

template <typename T, typename U>
__global__ __launch_bounds__(LOGITS_THREADS) void logits_kernel(const LogitsArgs a) {
  extern __shared__ __attribute__((aligned(16))) int lds_logits[];
  int* const count = lds_logits;                                             // [range]
  float* const bias = reinterpret_cast<float*>(lds_logits + a.range);        // [range], set where the counter holds bias entries
  const ecospa_logits& q = a.q;
  const int b = blockIdx.y, v0 = blockIdx.x * a.range, n = min(a.range, q.V - v0), tid = threadIdx.x;
  const int hist = q.history ? min(max(q.history_len ? q.history_len[b] : q.ld_history, 0), q.ld_history) : 0;
  const bool counted = hist > 0 || q.n_bias > 0;
  if (counted) {
    for (int i = tid * 4; i < a.range; i += LOGITS_THREADS * 4) *reinterpret_cast<int4*>(count + i) = int4{0, 0, 0, 0};
    __syncthreads();
    const int* const h = q.history + static_cast<long long>(b) * q.ld_history;
    for (int i = tid; i < hist; i += LOGITS_THREADS) {
      const unsigned v = static_cast<unsigned>(h[i] - v0);
      if (h[i] >= v0 && v < static_cast<unsigned>(n)) atomicAdd(&count[v], 1);
    }
    const int* const ids = q.bias_ids + static_cast<long long>(b) * q.n_bias;
    const float* const val = q.bias + static_cast<long long>(b) * q.n_bias;
    for (int i = tid; i < q.n_bias; i += LOGITS_THREADS)
      if (ids[i] >= v0 && ids[i] - v0 < n) atomicAdd(&count[ids[i] - v0], LOGITS_BIAS_ONE);
    __syncthreads();
    for (int i = tid; i < q.n_bias; i += LOGITS_THREADS) {
      const int id = ids[i];
      if (id < v0 || id - v0 >= n) continue;
      float sum = val[i];
      bool first = true;
      if (static_cast<unsigned>(count[id - v0]) >= 2u * LOGITS_BIAS_ONE) {      // listed more than once: its first entry adds them in order
        for (int j = 0; j < i; ++j) first = first && ids[j] != id;
        for (int j = i + 1; j < q.n_bias; ++j) sum = ids[j] == id ? sum + val[j] : sum;
      }
      if (first) bias[id - v0] = sum;
    }
    __syncthreads();
  }
  const float rep = q.repetition ? q.repetition[b] : 1.f, freq = q.frequency ? q.frequency[b] : 0.f, pres = q.presence ? q.presence[b] : 0.f;
  const float temp = q.temperature ? q.temperature[b] : 1.f;
  const int mr = q.mask ? q.mask_row[b] : -1;
  const unsigned* const mask = mr >= 0 && mr < q.n_masks ? q.mask + mr * q.ld_mask : nullptr;
  const T* const row = static_cast<const T*>(q.logits) + b * q.ld;
  U* const out = q.out ? static_cast<U*>(q.out) + b * q.ld_out : nullptr;
  float m = -INFINITY, s = 0.f;
  int at = -1;
  for (int i = tid * 8; i < n; i += LOGITS_THREADS * 8) {
    const int v = v0 + i, left = n - i;
    float x[8];
    if (left >= 8) {
      if constexpr (sizeof(T) == 2) {
        const uint4 u = *reinterpret_cast<const uint4*>(row + v);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) { x[2 * e] = __uint_as_float(w[e] << 16); x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u); }
      } else {
        const float4 u = *reinterpret_cast<const float4*>(row + v), w = *reinterpret_cast<const float4*>(row + v + 4);
        x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w; x[4] = w.x; x[5] = w.y; x[6] = w.z; x[7] = w.w;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = e < left ? load_f32<T>(row + v + e) : -INFINITY;
    }
    if (counted) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = count[i + e], past = c & (LOGITS_BIAS_ONE - 1);
        if (past) {
          x[e] = x[e] > 0.f ? x[e] / rep : x[e] * rep;
          x[e] = __fsub_rn(__fsub_rn(x[e], __fmul_rn(freq, static_cast<float>(past))), pres);
        }
        if (static_cast<unsigned>(c) >= static_cast<unsigned>(LOGITS_BIAS_ONE)) x[e] += bias[i + e];
      }
    }
    if (q.temperature) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = x[e] / temp;
    }
    if (mask) {
      const unsigned bits = mask[v >> 5] >> (v & 31);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = (bits >> e) & 1u ? x[e] : -INFINITY;
    }
    if (out) {
      if (left >= 8) {
        if constexpr (sizeof(U) == 2) {
          typedef float floatx8 __attribute__((ext_vector_type(8)));
          typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
          floatx8 f;
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] = x[e];
          *reinterpret_cast<uint4*>(out + v) = __builtin_bit_cast(uint4, __builtin_convertvector(f, bf16x8));
        } else {
          *reinterpret_cast<float4*>(out + v) = float4{x[0], x[1], x[2], x[3]};
          *reinterpret_cast<float4*>(out + v + 4) = float4{x[4], x[5], x[6], x[7]};
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < left) store_f32<U>(out + v + e, x[e]);
      }
    }
    float mx = m;
#pragma unroll
    for (int e = 0; e < 8; ++e) mx = fmaxf(mx, x[e]);
    if (mx > m) {
      s *= m == -INFINITY ? 0.f : __expf(m - mx);
      m = mx;
#pragma unroll
      for (int e = 7; e >= 0; --e) at = x[e] == m ? v + e : at;
    }
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int e = 0; e < 8; ++e) s += e < left ? __expf(x[e] - ref) : 0.f;
  }
  __shared__ LogitsPart red[LOGITS_THREADS / 64];
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) logits_join(m, s, at, __shfl_xor(m, o, 64), __shfl_xor(s, o, 64), __shfl_xor(at, o, 64));
  if ((tid & 63) == 0) red[tid >> 6] = LogitsPart{m, s, at, 0};
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < LOGITS_THREADS / 64; ++w) logits_join(m, s, at, red[w].m, red[w].s, red[w].at);
    if (a.ranges == 1) logits_finish(a, b, m, s, at);
    else a.part[static_cast<long long>(b) * a.ranges + blockIdx.x] = LogitsPart{m, s, at, 0};
  }
}
// a wavefront joins the ranges of a row
__global__ __launch_bounds__(256) void logits_join_kernel(const LogitsArgs a) {
  const int b = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (b >= a.q.B) return;
  float m = -INFINITY, s = 0.f;
  int at = -1;
  for (int i = lane; i < a.ranges; i += 64) {
    const LogitsPart p = a.part[static_cast<long long>(b) * a.ranges + i];
    logits_join(m, s, at, p.m, p.s, p.at);
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) logits_join(m, s, at, __shfl_xor(m, o, 64), __shfl_xor(s, o, 64), __shfl_xor(at, o, 64));
  if (lane == 0) logits_finish(a, b, m, s, at);
}

// Tokens of a workgroup.
static int logits_range(int B, int V) {
  int r = 4096;
  while (r > 2048 && static_cast<long long>(B) * ((V + r - 1) / r) < 512) r >>= 1;
  return r;
}
extern "C" size_t ecospa_logits_workspace_bytes(int B, int V) {
  if (B < 1 || V < 1 || B > 65535 || V > (1 << 24)) return 0;
  const int r = logits_range(B, V), n = (V + r - 1) / r;
  return n > 1 ? align_up(static_cast<size_t>(B) * n * sizeof(LogitsPart), 256) : 0;
}
extern "C" int ecospa_logits_process(ecospa_ctx* ctx, const ecospa_logits* q) {
  if (!ctx || !q || !q->logits || (!q->out && !q->pick && !q->lse) || (q->n_bias > 0 && (!q->bias_ids || !q->bias)) || (q->mask && !q->mask_row))
    return ECOSPA_ERR_NULL;
  if (!dtype_ok(q->dtype) || (q->out && !dtype_ok(q->out_dtype))) return ECOSPA_ERR_DTYPE;
  if (q->B < 1 || q->V < 1 || q->B > 65535 || q->V > (1 << 24) || q->ld < q->V || (q->out && q->ld_out < q->V)) return ECOSPA_ERR_SHAPE;
  if (q->n_bias < 0 || q->n_bias > 1023 || (q->history && (q->ld_history < 0 || q->ld_history >= LOGITS_BIAS_ONE)) ||
      (q->mask && (q->n_masks < 1 || q->ld_mask < (q->V + 31) / 32)))
    return ECOSPA_ERR_SHAPE;
  if (!aligned16(q->logits) || q->ld % 8 || (q->out && (!aligned16(q->out) || q->ld_out % 8))) return ECOSPA_ERR_ALIGN;
  LogitsArgs a;
  memset(&a, 0, sizeof(a));
  a.q = *q;
  a.range = logits_range(q->B, q->V);
  a.ranges = (q->V + a.range - 1) / a.range;
  if (a.ranges > 1) {
    WsCarver ws(ctx->ws, ctx->ws_bytes);
    a.part = static_cast<LogitsPart*>(ws.take(static_cast<size_t>(q->B) * a.ranges * sizeof(LogitsPart)));
    if (!ws.ok()) return ECOSPA_ERR_WORKSPACE;
  }
  const dim3 grid(a.ranges, q->B), block(LOGITS_THREADS);
  const int lds = a.range * (q->n_bias > 0 ? 8 : 4);
  const bool out_bf = q->out && q->out_dtype == ECOSPA_BF16;
  const auto kern = q->dtype == ECOSPA_BF16 ? (out_bf ? logits_kernel<bf16_t, bf16_t> : logits_kernel<bf16_t, float>)
                                            : (out_bf ? logits_kernel<float, bf16_t> : logits_kernel<float, float>);
  hipLaunchKernelGGL(kern, grid, block, lds, ctx->stream, a);
  ECOSPA_CHECK_LAUNCH(ctx, "logits_kernel");
  if (a.ranges > 1) {
    hipLaunchKernelGGL(logits_join_kernel, dim3((q->B + 3) / 4), dim3(256), 0, ctx->stream, a);
    ECOSPA_CHECK_LAUNCH(ctx, "logits_join_kernel");
  }
  return ECOSPA_OK;
}
