// Penalties, biases, temperature and masks on logits, with the best token and the log-sum-exp of every row.
//
// A workgroup takes a range of the vocabulary of one row.  It asks for all of its logits first - 8, 16 or 32 a thread stay in registers - and for
// the head of the history, and counts, while the logits travel, the row's history and bias entries that fall into its range in LDS (integer
// atomics: the order does not show).  Then every thread transforms and stores its logits; maximum, its lowest token and the sum of
// exponentials come from the registers, without a second look at memory.  The ranges' results of a row are joined by a second launch (none where
// one range is the row).  Nothing is added in an order that varies: results repeat bit for bit.
//
// The penalties, a temperature and the exponential are about 50 vector instructions a logit, beside 4 to 8 bytes of memory: 256 x 131072 fp32 with
// histories of 8192, which every one of 16 ranges looks through, take 64.8 us, 4.1 TB/s, the vector unit 77 % busy; with histories of 100 55.2 us,
// 4.9 TB/s (calls one behind the other, the join among them).  Few rows are bound by latencies: 1 x 32000 bf16 5.9 us.
#include "common.h"

#include <type_traits>

#define LOGITS_COUNTS 22               // a counter's low bits: occurrences in the history; above them: the last bias entry of the token, from 1
#define LOGITS_MAX_BIAS 1023

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));

struct LogitsPart {
  float m, s;      // maximum and sum of exp(x - m)
  int at;          // its lowest token, -1: none
  int pad;
};
struct LogitsArgs {
  ecospa_logits q;
  LogitsPart* part;
  int range, ranges;      // tokens of a workgroup (a multiple of 8), workgroups of a row
};

// x / d for a divisor whose rounded reciprocal r is at hand: the product with it and one correction by its exact remainder, half the
// division's instructions (which are what bounds these kernels beside memory); infinite x keep the plain product.  plain: d and r are finite, as nearly
// always.  Otherwise (plain is false) nothing is corrected where the remainder is no number, and a subnormal d, which can lack a finite reciprocal,
// is taken 2^64 times as large, the quotient after it.
struct LogitsDivisor {
  float d, r, after;
  bool plain;
};
__device__ __forceinline__ LogitsDivisor logits_divisor(float d) {
  const float after = fabsf(d) < 1.17549435e-38f ? 18446744073709551616.f : 1.f, r = 1.f / (d * after);
  return {d * after, r, after, after == 1.f && fabsf(d) < INFINITY};
}
template <bool PLAIN>
__device__ __forceinline__ float logits_div(float x, const LogitsDivisor& by) {
  const float y = x * by.r, e = __builtin_fmaf(-y, by.d, x);
  if (PLAIN) return __builtin_fmaf(fabsf(e) < INFINITY ? e : 0.f, by.r, y);
  return (fabsf(e) < INFINITY ? __builtin_fmaf(e, by.r, y) : y) * by.after;
}
__device__ __forceinline__ void logits_finish(const LogitsArgs& a, int b, float m, float s, int at) {
  if (a.q.pick) a.q.pick[b] = at;
  if (a.q.lse) a.q.lse[b] = (m == -INFINITY ? 0.f : m) + logf(s);
}

// Eight wavefronts a SIMD with 16 logits a thread: left to itself the compiler takes 4 registers more than they have (256 x 131072 fp32 77 -> 72 us).
template <typename T, typename U, int THREADS, int EACH>
__global__ __launch_bounds__(THREADS) __attribute__((amdgpu_waves_per_eu(EACH == 16 ? 8 : 4))) void logits_kernel(const LogitsArgs a) {
  constexpr int CHUNKS = EACH / 8, WAVES = THREADS / 64, EARLY = 8;      // entries of the history that a thread asks for together
  extern __shared__ __attribute__((aligned(16))) int lds_logits[];
  int* const count = lds_logits;                                                 // [range]
  float* const bias = reinterpret_cast<float*>(lds_logits + a.range);            // [n_bias]: the value of the last entry of every token listed
  __shared__ float red_m[WAVES], red_s[WAVES];
  __shared__ int red_at[WAVES], twice;
  const ecospa_logits& q = a.q;
  const int b = blockIdx.y, v0 = blockIdx.x * a.range, n = min(a.range, q.V - v0), full = n >> 3, tid = threadIdx.x;
  const T* const row = static_cast<const T*>(q.logits) + b * q.ld + v0;
  // chunk c of a thread: tokens 8 (c THREADS + tid) .. + 7 of the range; one beyond the last whole chunk is asked for at the last (and dropped)
  uint4 raw[CHUNKS][sizeof(T) / 2];
  if (full > 0) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const uint4* const src = reinterpret_cast<const uint4*>(row + min(c * THREADS + tid, full - 1) * 8);
#pragma unroll
      for (int e = 0; e < static_cast<int>(sizeof(T) / 2); ++e) raw[c][e] = src[e];
    }
  }
  const int hist = q.history ? min(max(q.history_len ? q.history_len[b] : q.ld_history, 0), q.ld_history) : 0;
  const bool counted = hist > 0 || q.n_bias > 0;
  const int* const h = q.history + static_cast<long long>(b) * q.ld_history;
  int id[EARLY];
#pragma unroll
  for (int e = 0; e < EARLY; ++e) id[e] = hist > 0 ? h[min(e * THREADS + tid, hist - 1)] : -1;
  const float rep = q.repetition ? q.repetition[b] : 1.f, freq = q.frequency ? q.frequency[b] : 0.f, pres = q.presence ? q.presence[b] : 0.f;
  const LogitsDivisor by_rep = logits_divisor(rep), by_temp = logits_divisor(q.temperature ? q.temperature[b] : 1.f);
  const int mr = q.mask ? q.mask_row[b] : -1;
  const unsigned* const mask = mr >= 0 && mr < q.n_masks ? q.mask + mr * q.ld_mask : nullptr;
  unsigned allowed[CHUNKS];
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    const int v = v0 + min((c * THREADS + tid) * 8, n - 1) / 8 * 8;
    allowed[c] = mask ? mask[v >> 5] >> (v & 31) : 0xffu;
  }
  if (counted) {
    for (int i = tid * 4; i < a.range; i += THREADS * 4) *reinterpret_cast<int4*>(count + i) = int4{0, 0, 0, 0};
    if (tid == 0) twice = 0;
    __syncthreads();
    if (q.n_bias > 0) {
      const int* const ids = q.bias_ids + static_cast<long long>(b) * q.n_bias;
      const float* const val = q.bias + static_cast<long long>(b) * q.n_bias;
      for (int i = tid; i < q.n_bias; i += THREADS) {
        const int at = ids[i] - v0;
        bias[i] = val[i];
        if (ids[i] >= v0 && at < n) atomicMax(reinterpret_cast<unsigned*>(&count[at]), static_cast<unsigned>(i + 1) << LOGITS_COUNTS);
      }
      __syncthreads();
      for (int i = tid; i < q.n_bias; i += THREADS) {
        const int at = ids[i] - v0;
        if (ids[i] >= v0 && at < n && static_cast<unsigned>(count[at]) >> LOGITS_COUNTS != static_cast<unsigned>(i + 1)) twice = 1;
      }
      __syncthreads();
      if (twice) {      // tokens listed more than once: the last entry takes the sum, in the order of the list
        for (int i = tid; i < q.n_bias; i += THREADS) {
          const int at = ids[i] - v0;
          if (ids[i] < v0 || at >= n || static_cast<unsigned>(count[at]) >> LOGITS_COUNTS != static_cast<unsigned>(i + 1)) continue;
          float sum = 0.f;
          for (int j = 0; j <= i; ++j) sum = ids[j] == ids[i] ? sum + val[j] : sum;
          bias[i] = sum;
        }
      }
    }
    for (int i0 = 0; i0 < hist; i0 += THREADS * EARLY) {
      if (i0 > 0) {
        const int* const p = h + i0;
        const int most = hist - 1 - i0;
#pragma unroll
        for (int e = 0; e < EARLY; ++e) id[e] = p[min(e * THREADS + tid, most)];
      }
      const int there = hist - i0;
#pragma unroll
      for (int e = 0; e < EARLY; ++e) {
        const unsigned at = static_cast<unsigned>(id[e] - v0);      // below v0: beyond any n
        if (at < static_cast<unsigned>(n) && e * THREADS + tid < there) atomicAdd(&count[at], 1);
      }
    }
    __syncthreads();
  }
  U* const out = q.out ? static_cast<U*>(q.out) + b * q.ld_out + v0 : nullptr;
  float x[CHUNKS][8], m = -INFINITY;
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    const int ch = c * THREADS + tid, i = ch * 8, left = n - i;      // tokens from this chunk on
    if (ch < full) {
      if constexpr (sizeof(T) == 2) {
        const uint32_t w[4] = {raw[c][0].x, raw[c][0].y, raw[c][0].z, raw[c][0].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) { x[c][2 * e] = __uint_as_float(w[e] << 16); x[c][2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u); }
      } else {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint4 u = raw[c][sizeof(T) / 2 - 2 + e];
          x[c][4 * e] = __uint_as_float(u.x); x[c][4 * e + 1] = __uint_as_float(u.y);
          x[c][4 * e + 2] = __uint_as_float(u.z); x[c][4 * e + 3] = __uint_as_float(u.w);
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[c][e] = e < left ? load_f32<T>(row + i + e) : -INFINITY;
      if (left <= 0) continue;
    }
    if (counted) {
      int k[8];
      *reinterpret_cast<int4*>(k) = *reinterpret_cast<const int4*>(count + i);
      *reinterpret_cast<int4*>(k + 4) = *reinterpret_cast<const int4*>(count + i + 4);
      if (k[0] | k[1] | k[2] | k[3] | k[4] | k[5] | k[6] | k[7]) {
        unsigned entries = 0u;
        const auto penalise = [&](auto plain) __attribute__((always_inline)) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {      // without branches: among 512 tokens of a wavefront some are in any history
            const int past = k[e] & ((1 << LOGITS_COUNTS) - 1);
            entries |= static_cast<unsigned>(k[e]);
            const bool up = x[c][e] > 0.f;      // x / rep as logits_div(), otherwise x rep
            float y;
            if (plain()) {
              const float f = up ? by_rep.r : rep, y0 = x[c][e] * f, r0 = __builtin_fmaf(-y0, rep, x[c][e]);
              y = __builtin_fmaf(up && fabsf(r0) < INFINITY ? r0 : 0.f, f, y0);
            } else {
              y = up ? logits_div<false>(x[c][e], by_rep) : x[c][e] * rep;
            }
            const float z = __fsub_rn(__fsub_rn(y, __fmul_rn(freq, static_cast<float>(past))), pres);
            x[c][e] = past ? z : x[c][e];
          }
        };
        if (by_rep.plain) penalise(std::true_type{});
        else penalise(std::false_type{});
        if (entries >> LOGITS_COUNTS) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const unsigned entry = static_cast<unsigned>(k[e]) >> LOGITS_COUNTS;
            if (entry) x[c][e] += bias[entry - 1];
          }
        }
      }
    }
    if (q.temperature) {
      if (by_temp.plain) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[c][e] = logits_div<true>(x[c][e], by_temp);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[c][e] = logits_div<false>(x[c][e], by_temp);
      }
    }
    if (mask) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {      // a set bit keeps the value: a bit-field extraction and a bitwise selection
        const unsigned t = static_cast<unsigned>(__builtin_amdgcn_sbfe(static_cast<int>(allowed[c]), e, 1));
        x[c][e] = __uint_as_float((t & __float_as_uint(x[c][e])) | (~t & 0xff800000u));
      }
    }
    if (out) {      // past the caches: the rows are read once and written once (256 x 131072 fp32 72 -> 64.5 us, 128 x 32000 bf16 11.0 -> 10.4)
      if (ch < full) {
        if constexpr (sizeof(U) == 2) {
          floatx8 f;
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] = x[c][e];
          __builtin_nontemporal_store(__builtin_bit_cast(uintx4, __builtin_convertvector(f, bf16x8)), reinterpret_cast<uintx4*>(out + i));
        } else {
          __builtin_nontemporal_store(floatx4{x[c][0], x[c][1], x[c][2], x[c][3]}, reinterpret_cast<floatx4*>(out + i));
          __builtin_nontemporal_store(floatx4{x[c][4], x[c][5], x[c][6], x[c][7]}, reinterpret_cast<floatx4*>(out + i + 4));
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < left) store_f32<U>(out + i + e, x[c][e]);
      }
    }
    if (left < 8) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[c][e] = e < left ? x[c][e] : -INFINITY;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) m = fmaxf(m, x[c][e]);
  }
  const float own_m = m;
  m = wave_max(m);
  if ((tid & 63) == 0) red_m[tid >> 6] = m;
  __syncthreads();
  m = red_m[0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) m = fmaxf(m, red_m[w]);
  // against +inf nothing could be told from what is not a number: the largest finite value in its place makes a sum of +inf, or NaN beside a NaN
  const float ref = m == -INFINITY ? 0.f : fminf(m, 3.402823466e38f);
  float s = 0.f;
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
    for (int e = 0; e < 8; ++e) s += __builtin_amdgcn_exp2f((x[c][e] - ref) * 1.4426950408889634f);      // the difference first: large logits lose nothing
  uint32_t at = 0xffffffffu;
  if (own_m == m) {
#pragma unroll
    for (int c = CHUNKS - 1; c >= 0; --c)
#pragma unroll
      for (int e = 7; e >= 0; --e) at = x[c][e] == m ? static_cast<uint32_t>((c * THREADS + tid) * 8 + e) : at;
  }
  s = wave_sum(s);
  at = wave_umin(at);
  if ((tid & 63) == 0) { red_s[tid >> 6] = s; red_at[tid >> 6] = static_cast<int>(at); }
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < WAVES; ++w) { s += red_s[w]; at = min(at, static_cast<uint32_t>(red_at[w])); }
    const int token = m == -INFINITY || at == 0xffffffffu ? -1 : v0 + static_cast<int>(at);
    if (a.ranges == 1) logits_finish(a, b, m, s, token);
    else a.part[static_cast<long long>(b) * a.ranges + blockIdx.x] = LogitsPart{m, s, token, 0};
  }
}
// A wavefront joins the ranges of a row, in their order.
__global__ __launch_bounds__(256) void logits_join_kernel(const LogitsArgs a) {
  const int b = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (b >= a.q.B) return;
  const LogitsPart* const p = a.part + static_cast<long long>(b) * a.ranges;
  LogitsPart x = p[min(lane, a.ranges - 1)];      // up to 64 ranges are read once
  float m = x.m;
  for (int i = lane + 64; i < a.ranges; i += 64) m = fmaxf(m, p[i].m);
  m = wave_max(m);
  const float ref = m == -INFINITY ? 0.f : m;
  float s = 0.f;
  uint32_t at = 0xffffffffu;
  for (int i = lane; i < a.ranges; i += 64) {
    if (i > lane) x = p[i];
    s += x.s * (x.m == m && m != -INFINITY ? 1.f : __expf(x.m - ref));
    if (x.m == m && x.at >= 0) at = min(at, static_cast<uint32_t>(x.at));
  }
  s = wave_sum(s);
  at = wave_umin(at);
  if (lane == 0) logits_finish(a, b, m, s, at == 0xffffffffu ? -1 : static_cast<int>(at));
}

// Threads, logits a thread and tokens of a workgroup. A vocabulary that one workgroup holds needs no join (256 x 9000 bf16, histories of 2000:
// one range of 1024 threads 7.4 us, two of 512 and the join 9.9).  Else 16 logits a thread in workgroups of 512, of which a compute unit holds four (256 x
// 131072 fp32, histories of 8192 / 100: workgroups of 512 64.4 / 55.6 us, of 1024 65.8 / 61.4; 32 logits a thread were 5 %, 8 were 25 % slower), and 8 in
// workgroups of 256 while all of them are resident at once and shorter passes end sooner (1 x 32000: 5.8 us against 7.0; 64 x 32000 8.6 against 8.7).
// Rows of up to 32768 bf16 logits for most compute units, but not more than one each: a workgroup a row, 32 logits a thread, which saves the join and
// reads the history once.  Against 16 a thread, seven vocabularies from 16500 to 32768, histories of 1000: 160 rows 0.92 to 1.04 of the time, 192 0.83 to
// 0.96, 224 and 256 0.82 to 0.89 (histories of 8000 0.71 to 0.79); but 272 rows 1.25 to 1.36, 128 rows 0.98 to 1.13.  In fp32 256 rows 19.9 us against 16.8.
struct LogitsPlan { int threads, each, range, ranges; };
static LogitsPlan logits_plan(int B, int V, bool bf) {
  LogitsPlan p;
  const bool twice = V > 1024 * 16 && V <= 1024 * 32 && bf && B >= 160 && B <= 256, one = V <= 1024 * 16 || twice, few = !one && static_cast<long long>(B) * V <= 1 << 21;
  p.each = few ? 8 : (twice ? 32 : 16);
  p.threads = few ? 256 : (!one ? 512 : (V <= 256 * 16 ? 256 : (V <= 512 * 16 ? 512 : 1024)));
  p.ranges = (V + p.threads * p.each - 1) / (p.threads * p.each);
  p.range = ((V + p.ranges - 1) / p.ranges + 31) / 32 * 32;
  p.ranges = (V + p.range - 1) / p.range;
  return p;
}
template <typename T, typename U, int THREADS, int EACH>
static hipError_t logits_launch_as(const LogitsArgs& a, hipStream_t st) {
  constexpr int most = (THREADS * EACH + LOGITS_MAX_BIAS) * 4;
  const int lds = (a.range + a.q.n_bias) * 4;
  const auto kern = logits_kernel<T, U, THREADS, EACH>;
  static LdsAttrOnce attr_once;
  if (most > 60 * 1024) {      // beside the static part
    const hipError_t e = attr_once.ensure(reinterpret_cast<const void*>(kern), most);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kern, dim3(a.ranges, a.q.B), dim3(THREADS), lds, st, a);
  return hipGetLastError();
}
template <typename T, typename U>
static hipError_t logits_launch(const LogitsArgs& a, const LogitsPlan& p, hipStream_t st) {
  if constexpr (sizeof(T) == 2)
    if (p.each == 32) return logits_launch_as<T, U, 1024, 32>(a, st);
  if (p.each == 8) return logits_launch_as<T, U, 256, 8>(a, st);
  return p.threads == 256 ? logits_launch_as<T, U, 256, 16>(a, st) : (p.threads == 512 ? logits_launch_as<T, U, 512, 16>(a, st) : logits_launch_as<T, U, 1024, 16>(a, st));
}
#define LOGITS_INSTANTIATE(T, U)                                                                                                          \
  template __global__ void logits_kernel<T, U, 256, 8>(const LogitsArgs); template __global__ void logits_kernel<T, U, 256, 16>(const LogitsArgs); \
  template __global__ void logits_kernel<T, U, 512, 16>(const LogitsArgs); template __global__ void logits_kernel<T, U, 1024, 16>(const LogitsArgs);
LOGITS_INSTANTIATE(bf16_t, bf16_t) LOGITS_INSTANTIATE(bf16_t, float) LOGITS_INSTANTIATE(float, bf16_t) LOGITS_INSTANTIATE(float, float)
template __global__ void logits_kernel<bf16_t, bf16_t, 1024, 32>(const LogitsArgs);
template __global__ void logits_kernel<bf16_t, float, 1024, 32>(const LogitsArgs);
#undef LOGITS_INSTANTIATE

extern "C" size_t ecospa_logits_workspace_bytes(int B, int V) {
  if (B < 1 || V < 1 || B > 65535 || V > (1 << 24)) return 0;
  const LogitsPlan p = logits_plan(B, V, false);      // the types are not known: the plan with more ranges
  return p.ranges > 1 ? align_up(static_cast<size_t>(B) * p.ranges * sizeof(LogitsPart), 256) : 0;
}
extern "C" int ecospa_logits_process(ecospa_ctx* ctx, const ecospa_logits* q) {
  if (!ctx || !q || !q->logits || (!q->out && !q->pick && !q->lse) || (q->n_bias > 0 && (!q->bias_ids || !q->bias)) || (q->mask && !q->mask_row))
    return ECOSPA_ERR_NULL;
  if (!dtype_ok(q->dtype) || (q->out && !dtype_ok(q->out_dtype))) return ECOSPA_ERR_DTYPE;
  if (q->B < 1 || q->V < 1 || q->B > 65535 || q->V > (1 << 24) || q->ld < q->V || (q->out && q->ld_out < q->V)) return ECOSPA_ERR_SHAPE;
  if (q->n_bias < 0 || q->n_bias > LOGITS_MAX_BIAS || (q->history && (q->ld_history < 0 || q->ld_history >= 1 << LOGITS_COUNTS)) ||
      (q->mask && (q->n_masks < 1 || q->ld_mask < (q->V + 31) / 32)))
    return ECOSPA_ERR_SHAPE;
  if (!aligned16(q->logits) || q->ld % 8 || (q->out && (!aligned16(q->out) || q->ld_out % 8))) return ECOSPA_ERR_ALIGN;
  LogitsArgs a;
  memset(&a, 0, sizeof(a));
  a.q = *q;
  const LogitsPlan p = logits_plan(q->B, q->V, q->dtype == ECOSPA_BF16);
  a.range = p.range;
  a.ranges = p.ranges;
  if (a.ranges > 1) {
    WsCarver ws(ctx->ws, ctx->ws_bytes);
    a.part = static_cast<LogitsPart*>(ws.take(static_cast<size_t>(q->B) * a.ranges * sizeof(LogitsPart)));
    if (!ws.ok()) return ECOSPA_ERR_WORKSPACE;
  }
  hipError_t e;
  const bool bf = q->dtype == ECOSPA_BF16, out_bf = q->out ? q->out_dtype == ECOSPA_BF16 : bf;
  if (bf) e = out_bf ? logits_launch<bf16_t, bf16_t>(a, p, ctx->stream) : logits_launch<bf16_t, float>(a, p, ctx->stream);
  else e = out_bf ? logits_launch<float, bf16_t>(a, p, ctx->stream) : logits_launch<float, float>(a, p, ctx->stream);
  if (e != hipSuccess) return hip_fail(ctx, e, "logits_kernel");
  if (a.ranges > 1) {
    hipLaunchKernelGGL(logits_join_kernel, dim3((q->B + 3) / 4), dim3(256), 0, ctx->stream, a);
    ECOSPA_CHECK_LAUNCH(ctx, "logits_join_kernel");
  }
  return ECOSPA_OK;
}
