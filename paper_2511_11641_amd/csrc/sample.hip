// A token drawn for every row of logits by a given random number, after temperature, top-k, top-p and min-p.
//
// A token of logit x weighs 2^(t - e), t = x log2(e) / T, with e the whole number at or above the row's largest t; weights are held as whole numbers of
// 2^-42, so that sums are exact in any order and results repeat.  All three restrictions keep a leading part of the tokens in order (larger logits
// first, equal ones by index), so what is kept is everything up to one token, the border.  Nothing is sorted:
//   scan    A workgroup takes a range of a row, once through memory: its largest logit, the weights relative to its own binade (a shift brings them to the
//           row's later on), their sums over chunks of 512 tokens, and a histogram of counts and weights in bins of an eighth of a binade.
//   draw    A workgroup a row: the ranges' histograms are added, the bin with the border is found, and the chunks that reach up to that bin are read again
//           (they are in the last-level cache): weights above it are summed by chunk, the tokens in it go to a list in LDS, where the border is found digit by digit
//           of (logit, index).  Then the chunk that the random number falls into, and the token in it.
// Weights decide on whole tokens next to borders, so they are good to 2^-42: a table of 64 powers and four terms of the series in 64 bits, which run at the rate
// of 32 bits here (some 25 instructions a token, at fp32 about as long as the memory takes).
#include "common.h"

typedef unsigned long long smp_u64;

#define SMP_BITS 42
#define SMP_BINS (SMP_BITS * 8 + 16)     // an eighth of a binade each; the least weight, 1, is rounded from half a binade below 2^0
#define SMP_CHUNK 512                    // tokens of a chunk: 8 a lane
#define SMP_MAX_V (1 << 20)              // 42 bits of a weight and 20 of a vocabulary: sums below 2^62
#define SMP_MAX_RANGES 512
#define SMP_LIST 4096
#define SMP_DRAW 1024

struct SamplePart {
  double e;              // binade that the range's weights are relative to
  float top;             // largest logit, -inf: none
  int at;                // its lowest token
  int bins;              // histogram bins in use
};
struct SampleArgs {
  ecospa_sample_args q;
  SamplePart* part;      // [B][ranges]
  float* chunk_top;      // [B][chunks]
  smp_u64* chunk_sum;    // [B][chunks], relative to their range
  smp_u64* bin_sum;      // [B][ranges][SMP_BINS]
  unsigned* bin_count;   // [B][ranges][SMP_BINS]
  int range, ranges, chunks;      // tokens of a range (a multiple of SMP_CHUNK)
};

constexpr double smp_power(int j) {      // 2^(j / 64)
  const double x = j * (0.69314718055994530942 / 64.0);
  double s = 1.0, t = 1.0;
  for (int i = 1; i < 24; ++i) { t *= x / i; s += t; }
  return s;
}
struct SamplePowers { double p[64]; };
constexpr SamplePowers smp_powers() {
  SamplePowers t{};
  for (int j = 0; j < 64; ++j) t.p[j] = smp_power(j);
  return t;
}
__device__ const SamplePowers SMP_POWERS = smp_powers();

// The binade of a range whose largest logit is `top`, and the place of that logit, 64 (t - e).  (A temperature so small that a place has no fraction left: 0.)
__device__ __forceinline__ double smp_binade(float top, double c64) {
  return fabsf(top) == INFINITY ? 0.0 : __builtin_ceil(static_cast<double>(top) * c64 * (1.0 / 64.0));
}
__device__ __forceinline__ double smp_base(float top, double c64, double e) {
  return fabsf(top) == INFINITY || __builtin_fabs(e) > 1e13 ? 0.0 : __builtin_fma(static_cast<double>(top), c64, -64.0 * e);
}
// 64 (t - e) of a logit of that range, from its distance to `top`, which 64 bits hold; what has no weight (NaN, -inf, a finite one beside +inf) is far below
__device__ __forceinline__ double smp_place(float x, float top, double c64, double base) {
  const double u = x == top ? base : __builtin_fma(static_cast<double>(x) - static_cast<double>(top), c64, base);
  return __builtin_fmax(u, -64.0 * (SMP_BITS + 4));
}
// its weight times 2^42, not rounded; k: the place in whole 64ths (<= 0 but for a rounding)
__device__ __forceinline__ double smp_weight(double u, const double* powers, int& k) {
  const double w = __builtin_rint(u), r = (u - w) * (0.69314718055994530942 / 64.0);
  k = static_cast<int>(w);
  double p = __builtin_fma(r, 1.0 / 24.0, 1.0 / 6.0);
  p = __builtin_fma(p, r, 0.5);
  p = __builtin_fma(p, r, 1.0);
  p = __builtin_fma(p, r, 1.0);
  return __builtin_ldexp(p * powers[k & 63], SMP_BITS + (k >> 6));
}
__device__ __forceinline__ smp_u64 smp_whole(double w) {      // nearest whole number of w < 2^51: the low bits of 2^52 + w
  return __builtin_bit_cast(smp_u64, w + 4503599627370496.0) & 0xfffffffffffffull;
}
__device__ __forceinline__ int smp_bin(int k) { return min(max(-k, 0) >> 3, SMP_BINS - 1); }
// larger logits first: ascending numbers, -0 with +0 (NaN has no weight and is never asked for)
__device__ __forceinline__ unsigned smp_rank(float x) {
  const unsigned b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? b : 0x7fffffffu - b;
}
// sums over the wavefront, v < 2^45: two halves through lane permutations
__device__ __forceinline__ unsigned smp_add64(unsigned v) {
#define SMP_DPP(ctrl) v += static_cast<unsigned>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), (ctrl), 0xF, 0xF, true))
  SMP_DPP(0xB1); SMP_DPP(0x4E); SMP_DPP(0x141); SMP_DPP(0x140);
#undef SMP_DPP
  const auto row = [&](int l) __attribute__((always_inline)) { return static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(v), l)); };
  return (row(0) + row(16)) + (row(32) + row(48));
}
__device__ __forceinline__ smp_u64 smp_wave_sum(smp_u64 v) {
  return (static_cast<smp_u64>(smp_add64(static_cast<unsigned>(v >> 25))) << 25) + smp_add64(static_cast<unsigned>(v) & 0x1ffffffu);
}
template <typename T>
__device__ __forceinline__ float smp_scalar(const T* p, int i) { return load_f32<T>(p + i); }
// eight tokens of a lane; those at and beyond `left` are -inf and are not read
template <typename T>
__device__ __forceinline__ void smp_load(const T* p, int left, float (&x)[8]) {
  if (left >= 8) {
    if constexpr (sizeof(T) == 2) {
      const uint4 u = *reinterpret_cast<const uint4*>(p);
      const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) { x[2 * e] = __uint_as_float(w[e] << 16); x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u); }
    } else {
      const float4 lo = *reinterpret_cast<const float4*>(p), hi = *reinterpret_cast<const float4*>(p + 4);
      x[0] = lo.x; x[1] = lo.y; x[2] = lo.z; x[3] = lo.w; x[4] = hi.x; x[5] = hi.y; x[6] = hi.z; x[7] = hi.w;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = e < left ? smp_scalar(p, e) : -INFINITY;
  }
}
// What a row asks for.
struct SampleRow {
  bool greedy, by_k, by_p, by_min;
  double c64;
  int k;
  float p, min_p;
};
__device__ __forceinline__ SampleRow smp_row(const ecospa_sample_args& q, int b) {
  SampleRow r;
  const float t = q.temperature ? q.temperature[b] : 1.f;
  r.k = q.top_k ? q.top_k[b] : 0;
  r.p = q.top_p ? q.top_p[b] : 1.f;
  r.min_p = q.min_p ? fminf(q.min_p[b], 1.f) : 0.f;
  if (q.min_p && !(q.min_p[b] == q.min_p[b])) r.min_p = 0.f;
  r.greedy = !(t > 0.f);
  r.by_k = r.k >= 1 && r.k < q.V;
  r.by_p = r.p < 1.f;
  r.by_min = r.min_p > 0.f;
  r.c64 = 64.0 * 1.4426950408889634074 / static_cast<double>(r.greedy ? 1.f : t);
  return r;
}

// ---------------------------------------------------------------------------------------------
// scan
// ---------------------------------------------------------------------------------------------
template <typename T, int THREADS, int EACH>
__global__ __launch_bounds__(THREADS) void sample_scan_kernel(const SampleArgs a) {
  constexpr int WAVES = THREADS / 64, CH = EACH / 8;
  __shared__ smp_u64 sum[SMP_BINS];
  __shared__ unsigned count[SMP_BINS];
  __shared__ double powers[64];
  __shared__ float red_top[WAVES];
  __shared__ int red_at[WAVES], used;
  const ecospa_sample_args& q = a.q;
  const int b = blockIdx.y, v0 = blockIdx.x * a.range, n = min(a.range, q.V - v0), tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const T* const row = static_cast<const T*>(q.logits) + b * q.ld + v0;
  float x[CH][8];
#pragma unroll
  for (int c = 0; c < CH; ++c) smp_load(row + (c * WAVES + wave) * SMP_CHUNK + lane * 8, n - (c * WAVES + wave) * SMP_CHUNK - lane * 8, x[c]);
  const SampleRow r = smp_row(q, b);
  const bool bins = !r.greedy && (r.by_k || r.by_p);
  if (tid < 64) powers[tid] = SMP_POWERS.p[tid];
  if (tid == 0) used = 0;
  if (bins) {
    for (int i = tid; i < SMP_BINS; i += THREADS) { sum[i] = 0; count[i] = 0; }
  }
  float top = -INFINITY;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    float m = -INFINITY;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = fmaxf(m, x[c][e]);
    m = wave_max(m);
    const int chunk = c * WAVES + wave;
    if (lane == 0 && chunk * SMP_CHUNK < n) a.chunk_top[static_cast<long long>(b) * a.chunks + blockIdx.x * (a.range / SMP_CHUNK) + chunk] = m;
    top = fmaxf(top, m);
  }
  if (lane == 0) red_top[wave] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < WAVES; ++w) top = fmaxf(top, red_top[w]);
  SamplePart* const part = a.part + static_cast<long long>(b) * a.ranges + blockIdx.x;
  if (r.greedy) {
    unsigned at = 0xffffffffu;
#pragma unroll
    for (int c = CH - 1; c >= 0; --c)
#pragma unroll
      for (int e = 7; e >= 0; --e) at = x[c][e] == top ? static_cast<unsigned>((c * WAVES + wave) * SMP_CHUNK + lane * 8 + e) : at;
    at = wave_umin(at);
    if (lane == 0) red_at[wave] = static_cast<int>(at);
    __syncthreads();
    if (tid == 0) {
#pragma unroll
      for (int w = 1; w < WAVES; ++w) at = min(at, static_cast<unsigned>(red_at[w]));
      *part = SamplePart{0.0, top, v0 + static_cast<int>(at), 0};
    }
    return;
  }
  const double e = smp_binade(top, r.c64), base = smp_base(top, r.c64, e);
  int most = 0;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    smp_u64 s = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      int k;
      const smp_u64 w = smp_whole(smp_weight(smp_place(x[c][i], top, r.c64, base), powers, k));
      s += w;
      if (bins && w != 0) {
        const int bin = smp_bin(k);
        atomicAdd(&sum[bin], w);
        if (r.by_k) atomicAdd(&count[bin], 1u);
        most = max(most, bin + 1);
      }
    }
    s = smp_wave_sum(s);
    const int chunk = c * WAVES + wave;
    if (lane == 0 && chunk * SMP_CHUNK < n) a.chunk_sum[static_cast<long long>(b) * a.chunks + blockIdx.x * (a.range / SMP_CHUNK) + chunk] = s;
  }
  if (bins && most > 0) atomicMax(&used, most);
  __syncthreads();
  if (tid == 0) *part = SamplePart{e, top, 0, used};
  if (bins) {
    const long long at = (static_cast<long long>(b) * a.ranges + blockIdx.x) * SMP_BINS;
    for (int i = tid; i < used; i += THREADS) {
      a.bin_sum[at + i] = sum[i];
      if (r.by_k) a.bin_count[at + i] = count[i];
    }
  }
}

// ---------------------------------------------------------------------------------------------
// draw
// ---------------------------------------------------------------------------------------------
struct SampleShared {
  smp_u64 chunk[SMP_MAX_V / SMP_CHUNK];      // kept weight by chunk
  smp_u64 list_key[SMP_LIST], list_w[SMP_LIST];
  smp_u64 sum[SMP_BINS];
  unsigned count[SMP_BINS];
  smp_u64 digit_sum[256];
  unsigned digit_count[256];
  double powers[64], base[SMP_MAX_RANGES];
  float top[SMP_MAX_RANGES];
  int shift[SMP_MAX_RANGES];                 // binades below the row's; 63: no weight
  smp_u64 scan[SMP_DRAW / 64];
  smp_u64 out[4];
  int flag[4];
  float red_f[SMP_DRAW / 64];
  double red_d[SMP_DRAW / 64];
  int listed;
};
__device__ __forceinline__ smp_u64 smp_inclusive(smp_u64 v) {      // over the lanes of a wavefront
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const smp_u64 u = __shfl_up(v, off, 64);
    if ((threadIdx.x & 63) >= static_cast<unsigned>(off)) v += u;
  }
  return v;
}
// One wavefront: the first of n bins where the running sum of v reaches `need` (the last bin that holds anything if none does), into out[0]; out[1], out[2]: sums of v
// and of w over the bins in front of it; out[3]: 1 where `need` is reached.
template <typename V, typename W>
__device__ __forceinline__ void smp_find(int n, smp_u64 need, V&& v, W&& w, smp_u64* out) {
  const int lane = threadIdx.x & 63, per = (n + 63) / 64;
  smp_u64 mine = 0, other = 0;
  int last = -1;
  for (int i = 0; i < per; ++i) {
    const int bin = lane * per + i;
    if (bin >= n) break;
    mine += v(bin);
    other += w(bin);
    if (v(bin) != 0) last = bin;
  }
  const smp_u64 upto = smp_inclusive(mine), upto_w = smp_inclusive(other);
  const unsigned long long reached = __ballot(upto >= need), some = __ballot(last >= 0);
  if (some == 0) {
    if (lane == 0) { out[0] = 0; out[1] = out[2] = out[3] = 0; }
    return;
  }
  const int from = reached ? __ffsll(reached) - 1 : 63 - __clzll(some);
  if (lane == from) {
    smp_u64 front = upto - mine, front_w = upto_w - other;
    int bin = lane * per;
    if (reached) {
      for (; front + v(bin) < need; ++bin) { front += v(bin); front_w += w(bin); }
    } else {
      for (; bin < last; ++bin) { front += v(bin); front_w += w(bin); }
    }
    out[0] = static_cast<smp_u64>(bin);
    out[1] = front;
    out[2] = front_w;
    out[3] = reached ? 1 : 0;
  }
}

template <typename T>
struct SampleWalk {
  const SampleArgs& a;
  SampleShared& sh;
  const T* row;
  const float* chunk_top;
  double c64;
  int per_range;             // chunks
  // place of a logit of range r relative to the row's binade
  __device__ __forceinline__ double place(float x, int r) const {
    return smp_place(x, sh.top[r], c64, sh.base[r]);
  }
  // f(chunk, range, logits of the lane's eight tokens) for the wavefront's chunks that reach bin `least` or above it, AHEAD of them on their way together
  template <int AHEAD, typename F, typename G>
  __device__ __forceinline__ void chunks(int least, F&& f, G&& skipped) const {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int c0 = wave; c0 < a.chunks; c0 += AHEAD * (SMP_DRAW / 64)) {
      float x[AHEAD][8];
      bool on[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const int c = c0 + i * (SMP_DRAW / 64);
        on[i] = c < a.chunks;
        if (on[i]) {
          const int r = c / per_range, s = sh.shift[r];
          const double u = place(chunk_top[c], r);
          on[i] = s < 63 && smp_bin(static_cast<int>(__builtin_rint(u))) + 8 * s <= least;
        }
        on[i] = __builtin_amdgcn_readfirstlane(on[i]) != 0;
        if (on[i]) smp_load(row + c * SMP_CHUNK + lane * 8, a.q.V - c * SMP_CHUNK - lane * 8, x[i]);
      }
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const int c = c0 + i * (SMP_DRAW / 64);
        if (on[i]) f(c, c / per_range, x[i]);
        else if (c < a.chunks) skipped(c);
      }
    }
  }
};
__device__ __forceinline__ smp_u64 smp_key(float x, int v) { return (static_cast<smp_u64>(smp_rank(x)) << 20) | static_cast<unsigned>(v); }

// The border among the tokens of one bin: the least key such that the tokens up to it hold `need` (tokens if `counted`, else weight).  each(f) calls
// f(key, weight) for every token of the bin, over the threads of the workgroup.  -> the key; taken: weight up to it.
template <typename E>
__device__ __forceinline__ smp_u64 smp_border(SampleShared& sh, smp_u64 need, bool counted, E&& each, smp_u64& taken) {
  const int tid = threadIdx.x;
  if (tid == 0) { sh.out[0] = ~0ull; sh.out[1] = 0; }
  __syncthreads();
  smp_u64 lo = ~0ull, hi = 0;
  each([&](smp_u64 key, smp_u64) __attribute__((always_inline)) { lo = min(lo, key); hi = max(hi, key); });
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    lo = min(lo, static_cast<smp_u64>(__shfl_xor(lo, off, 64)));
    hi = max(hi, static_cast<smp_u64>(__shfl_xor(hi, off, 64)));
  }
  if ((tid & 63) == 0) { atomicMin(&sh.out[0], lo); atomicMax(&sh.out[1], hi); }
  __syncthreads();
  lo = sh.out[0];
  hi = sh.out[1];
  __syncthreads();
  taken = 0;
  if (lo > hi) return 0;      // no token of any weight
  int bits = 64 - __clzll((hi - lo) | 1ull), shift = max(bits - 8, 0);
  for (;;) {
    for (int i = tid; i < 256; i += SMP_DRAW) { sh.digit_sum[i] = 0; sh.digit_count[i] = 0; }
    __syncthreads();
    each([&](smp_u64 key, smp_u64 w) __attribute__((always_inline)) {
      if (key < lo || key > hi) return;
      const int d = static_cast<int>((key - lo) >> shift);
      atomicAdd(&sh.digit_sum[d], w);
      atomicAdd(&sh.digit_count[d], 1u);
    });
    __syncthreads();
    if (tid < 64) {
      const auto s = [&](int i) __attribute__((always_inline)) { return sh.digit_sum[i]; };
      const auto c = [&](int i) __attribute__((always_inline)) { return static_cast<smp_u64>(sh.digit_count[i]); };
      if (counted) smp_find(256, need, c, s, sh.out);
      else smp_find(256, need, s, c, sh.out);
    }
    __syncthreads();
    const int d = static_cast<int>(sh.out[0]);
    const smp_u64 front = sh.out[1], front_other = sh.out[2], in_sum = sh.digit_sum[d], in_count = sh.digit_count[d];
    __syncthreads();
    taken += counted ? front_other : front;
    need -= min(front, need);
    lo += static_cast<smp_u64>(d) << shift;
    hi = min(hi, lo + ((1ull << shift) - 1));
    if (in_count <= 1 || need >= (counted ? in_count : in_sum) || shift == 0) {
      taken += in_sum;
      return hi;
    }
    shift = max(shift - 8, 0);
  }
}

template <typename T>
__global__ __launch_bounds__(SMP_DRAW) void sample_draw_kernel(const SampleArgs a) {
  extern __shared__ __attribute__((aligned(16))) char lds_sample[];
  SampleShared& sh = *reinterpret_cast<SampleShared*>(lds_sample);
  const ecospa_sample_args& q = a.q;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  constexpr int WAVES = SMP_DRAW / 64;
  const SampleRow r = smp_row(q, b);
  const SamplePart* const part = a.part + static_cast<long long>(b) * a.ranges;
  if (tid < 64) sh.powers[tid] = SMP_POWERS.p[tid];
  // the row's largest logit and binade
  SamplePart mine{0.0, -INFINITY, 0, 0};
  if (tid < a.ranges) mine = part[tid];
  const float own_top = wave_max(mine.top);
  double e = mine.top == -INFINITY ? -__builtin_inf() : mine.e;
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) e = __builtin_fmax(e, __shfl_xor(e, off, 64));
  if (lane == 0) { sh.red_f[wave] = own_top; sh.red_d[wave] = e; }
  __syncthreads();
  float top = -INFINITY;
  for (int w = 0; w < WAVES; ++w) { top = fmaxf(top, sh.red_f[w]); e = __builtin_fmax(e, sh.red_d[w]); }
  if (top == -INFINITY) {      // nothing to draw from
    if (tid == 0) {
      q.token[b] = -1;
      if (q.prob) q.prob[b] = 0.f;
    }
    return;
  }
  if (r.greedy) {
    unsigned at = tid < a.ranges && mine.top == top ? static_cast<unsigned>(mine.at) : 0xffffffffu;
    at = wave_umin(at);
    if (lane == 0) sh.scan[wave] = at;
    __syncthreads();
    if (tid == 0) {
      for (int w = 0; w < WAVES; ++w) at = min(at, static_cast<unsigned>(sh.scan[w]));
      q.token[b] = static_cast<int>(at);
      if (q.prob) q.prob[b] = 1.f;
    }
    return;
  }
  const bool infinite = top == INFINITY;
  if (infinite) e = 0.0;
  if (tid < a.ranges) {
    const double below = e - mine.e;
    const bool none = mine.top == -INFINITY || (infinite && mine.top != INFINITY) || below > SMP_BITS + 1;
    sh.shift[tid] = none ? 63 : static_cast<int>(below);
    sh.top[tid] = mine.top;
    sh.base[tid] = smp_base(mine.top, r.c64, mine.e);
  }
  __syncthreads();
  const T* const row = static_cast<const T*>(q.logits) + b * q.ld;
  const SampleWalk<T> walk{a, sh, row, a.chunk_top + static_cast<long long>(b) * a.chunks, r.c64, a.range / SMP_CHUNK};
  // least place (64ths, relative to the row's binade) that min-p leaves
  const double least_place = r.by_min ? smp_base(top, r.c64, e) + 64.0 * log2(static_cast<double>(r.min_p)) : -1e30;

  int border_bin = SMP_BINS;      // tokens of lower bins are kept whole
  smp_u64 border = 0;             // and of this bin those with keys up to this
  if (r.by_k || r.by_p) {
    for (int i = tid; i < SMP_BINS; i += SMP_DRAW) {
      smp_u64 s = 0;
      unsigned c = 0;
      for (int g = 0; g < a.ranges; ++g) {
        const int by = sh.shift[g], from = i - 8 * by;
        if (by >= 63 || from < 0 || from >= part[g].bins) continue;
        const long long at = (static_cast<long long>(b) * a.ranges + g) * SMP_BINS + from;
        s += a.bin_sum[at] >> by;
        if (r.by_k) c += a.bin_count[at];
      }
      sh.sum[i] = s;
      sh.count[i] = c;
    }
    __syncthreads();
  }
  const auto bin_sum = [&](int i) __attribute__((always_inline)) { return sh.sum[i]; };
  const auto bin_count = [&](int i) __attribute__((always_inline)) { return static_cast<smp_u64>(sh.count[i]); };
  // weights above `bin` by chunk (where `sums`), and the tokens in it to the list
  const auto gather = [&](int bin, bool sums) __attribute__((always_inline)) {
    if (tid == 0) sh.listed = 0;
    __syncthreads();
    walk.template chunks<2>(bin, [&](int c, int g, const float (&x)[8]) __attribute__((always_inline)) {
      const int by = sh.shift[g];
      smp_u64 s = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const double u = walk.place(x[i], g);
        const int k = static_cast<int>(__builtin_rint(u)), at = smp_bin(k) + 8 * by;
        if (at > bin) continue;
        int k2;
        const smp_u64 w = smp_whole(smp_weight(u, sh.powers, k2)) >> by;
        if (w == 0) continue;
        if (at < bin) {
          if (u - 64.0 * by >= least_place) s += w;
        } else {
          const int slot = atomicAdd(&sh.listed, 1);
          if (slot < SMP_LIST) { sh.list_key[slot] = smp_key(x[i], c * SMP_CHUNK + lane * 8 + i); sh.list_w[slot] = w; }
        }
        __builtin_amdgcn_sched_barrier(0);      // one token behind the other: eight chains at once need more registers than there are
      }
      if (sums) {
        s = smp_wave_sum(s);
        if (lane == 0) sh.chunk[c] = s;
      }
    }, [&](int c) __attribute__((always_inline)) { if (sums && lane == 0) sh.chunk[c] = 0; });
    __syncthreads();
  };
  // every token of `bin`, from the list or, where it did not hold them, from the row
  const auto each_of = [&](int bin, auto&& f) __attribute__((always_inline)) {
    const int n = sh.listed;
    if (n <= SMP_LIST) {
      for (int i = tid; i < n; i += SMP_DRAW) f(sh.list_key[i], sh.list_w[i]);
    } else {
      walk.template chunks<1>(bin, [&](int c, int g, const float (&x)[8]) __attribute__((always_inline)) {
        const int by = sh.shift[g];
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[i];
#pragma unroll 1
        for (int i = 0; i < 8; ++i) {      // a loop: this is the rare path, and it stands here four times
          const float xi = y[0];
#pragma unroll
          for (int m = 0; m < 7; ++m) y[m] = y[m + 1];
          int k;
          const smp_u64 w = smp_whole(smp_weight(walk.place(xi, g), sh.powers, k)) >> by;
          if (w != 0 && smp_bin(k) + 8 * by == bin) f(smp_key(xi, c * SMP_CHUNK + lane * 8 + i), w);
        }
      }, [](int) __attribute__((always_inline)) {});
    }
  };
  // by the number of tokens first: what is kept then is what top-p is a part of
  smp_u64 total = 0;
  bool bordered = false;
  int phase = r.by_k ? 0 : (r.by_p ? 1 : (r.by_min ? 2 : 3));      // tokens, weight, min-p alone, nothing more
#pragma unroll 1
  while (phase < 3) {
    int bin = SMP_BINS;
    smp_u64 front = 0, front_sum = 0;
    bool reached = true;
    smp_u64 need = static_cast<smp_u64>(r.k);
    if (phase == 1) {
      if (!bordered) {
        if (tid < 64) {
          smp_u64 s = 0;
          for (int i = lane; i < SMP_BINS; i += 64) s += sh.sum[i];
          s = smp_inclusive(s);
          if (lane == 63) sh.out[0] = s;
        }
        __syncthreads();
        total = sh.out[0];
        __syncthreads();
      }
      // the least whole number of 2^-42 at or above top_p times the total
      const smp_u64 p = r.p > 0.f ? static_cast<smp_u64>(static_cast<double>(r.p) * 4294967296.0) : 0ull;
      const unsigned __int128 prod = static_cast<unsigned __int128>(total) * p;
      need = max(static_cast<smp_u64>(prod >> 32) + (static_cast<unsigned>(static_cast<smp_u64>(prod)) != 0u ? 1 : 0), 1ull);
    }
    if (phase < 2) {
      if (tid < 64) {
        if (phase == 0) smp_find(SMP_BINS, need, bin_count, bin_sum, sh.out);
        else smp_find(SMP_BINS, need, bin_sum, bin_count, sh.out);
      }
      __syncthreads();
      bin = static_cast<int>(sh.out[0]);
      front = sh.out[1];
      front_sum = phase == 0 ? sh.out[2] : front;
      reached = sh.out[3] != 0;
      __syncthreads();
    }
    if (phase == 0 && !reached) {      // fewer tokens than k weigh anything
      phase = r.by_p ? 1 : (r.by_min ? 2 : 3);
      continue;
    }
    gather(bin, phase != 0 || !r.by_p);
    if (phase == 2) break;
    smp_u64 taken;
    border = smp_border(sh, max(need - min(front, need), 1ull), phase == 0, [&](auto&& f) __attribute__((always_inline)) { each_of(bin, f); }, taken);
    border_bin = bin;
    bordered = true;
    total = front_sum + taken;
    phase = phase == 0 && r.by_p ? 1 : 3;
  }
  if (bordered) {
    // the kept tokens of the border's bin join their chunks' sums
    each_of(border_bin, [&](smp_u64 key, smp_u64 w) __attribute__((always_inline)) {
      if (key > border) return;
      const int v = static_cast<int>(key & 0xfffffu), g = v / a.range;
      if (r.by_min && walk.place(load_f32<T>(row + v), g) - 64.0 * sh.shift[g] < least_place) return;
      atomicAdd(&sh.chunk[v / SMP_CHUNK], w);
    });
    __syncthreads();
  }
  const bool whole = !bordered && !r.by_min;
  if (whole) {
    for (int c = tid; c < a.chunks; c += SMP_DRAW) {
      const int by = sh.shift[c / walk.per_range];
      sh.chunk[c] = by >= 63 ? 0 : a.chunk_sum[static_cast<long long>(b) * a.chunks + c] >> by;
    }
    __syncthreads();
  }

  // the chunk that the random number falls into
  constexpr int PER = SMP_MAX_V / SMP_CHUNK / SMP_DRAW;
  smp_u64 own[PER], all = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    own[i] = tid * PER + i < a.chunks ? sh.chunk[tid * PER + i] : 0;
    all += own[i];
  }
  const smp_u64 upto = smp_inclusive(all);
  if (lane == 63) sh.scan[wave] = upto;
  __syncthreads();
  smp_u64 front = 0;
  total = 0;
  for (int w = 0; w < WAVES; ++w) {
    front += w < wave ? sh.scan[w] : 0;
    total += sh.scan[w];
  }
  front += upto - all;
  const float uf = q.u[b];
  const smp_u64 u = uf > 0.f ? (uf < 1.f ? static_cast<smp_u64>(static_cast<double>(uf) * 4294967296.0) : 4294967295ull) : 0ull;
  smp_u64 target = static_cast<smp_u64>((static_cast<unsigned __int128>(total) * u) >> 32);
  if (!(uf < 1.f) && uf == uf) target = total - 1;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (target >= front && target < front + own[i]) {
      sh.out[0] = static_cast<smp_u64>(tid * PER + i);
      sh.out[1] = target - front;
    }
    front += own[i];
  }
  __syncthreads();
  if (tid >= 64) return;
  // the token
  const int c = static_cast<int>(sh.out[0]), g = c / walk.per_range, by = sh.shift[g];
  const smp_u64 into = whole ? sh.out[1] << by : sh.out[1];      // unrestricted sums are those of the range's own binade
  float x[8];
  smp_load(row + c * SMP_CHUNK + lane * 8, q.V - c * SMP_CHUNK - lane * 8, x);
  smp_u64 w[8], s = 0;
  double exact[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    int k;
    const double p = walk.place(x[i], g);
    exact[i] = smp_weight(p, sh.powers, k);
    w[i] = smp_whole(exact[i]) >> (whole ? 0 : by);
    const int at = smp_bin(k) + 8 * by;
    const bool kept = whole || ((at < border_bin || (at == border_bin && smp_key(x[i], c * SMP_CHUNK + lane * 8 + i) <= border)) && p - 64.0 * by >= least_place);
    w[i] = kept ? w[i] : 0;
    s += w[i];
  }
  smp_u64 before = smp_inclusive(s) - s;
  const unsigned long long have = __ballot(s != 0 && before <= into);      // the last lane that starts at or in front of the target
  if (lane != 63 - __clzll(have)) return;
  int at = -1;
  double weight = 0.0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (w[i] != 0 && before <= into) { at = i; weight = exact[i]; }
    before += w[i];
  }
  q.token[b] = c * SMP_CHUNK + lane * 8 + at;
  if (q.prob) q.prob[b] = static_cast<float>(fmin(__builtin_ldexp(weight, -by) / static_cast<double>(total), 1.0));
}

// ---------------------------------------------------------------------------------------------
// entry points
// ---------------------------------------------------------------------------------------------
// Ranges of 8192 tokens; of 2048 while there are few of them.
struct SamplePlan { int threads, range, ranges, chunks; };
static SamplePlan sample_plan(int B, int V) {
  SamplePlan p;
  const bool few = static_cast<long long>(B) * V <= 1 << 21;
  p.threads = few ? 256 : 512;
  p.range = few ? 2048 : 8192;
  p.ranges = (V + p.range - 1) / p.range;
  p.chunks = (V + SMP_CHUNK - 1) / SMP_CHUNK;
  return p;
}
static void sample_carve(SampleArgs& a, const SamplePlan& p, WsCarver& ws, int B) {
  const size_t n = static_cast<size_t>(B) * p.ranges, c = static_cast<size_t>(B) * p.chunks;
  a.part = static_cast<SamplePart*>(ws.take(n * sizeof(SamplePart)));
  a.bin_sum = static_cast<smp_u64*>(ws.take(n * SMP_BINS * sizeof(smp_u64)));
  a.bin_count = static_cast<unsigned*>(ws.take(n * SMP_BINS * sizeof(unsigned)));
  a.chunk_sum = static_cast<smp_u64*>(ws.take(c * sizeof(smp_u64)));
  a.chunk_top = static_cast<float*>(ws.take(c * sizeof(float)));
}
extern "C" size_t ecospa_sample_workspace_bytes(int B, int V) {
  if (B < 1 || V < 1 || B > 65535 || V > SMP_MAX_V) return 0;
  SampleArgs a;
  WsCarver ws(nullptr, 0);
  sample_carve(a, sample_plan(B, V), ws, B);
  return align_up(ws.off, 256);
}
template <typename T>
static hipError_t sample_launch(const SampleArgs& a, const SamplePlan& p, hipStream_t st) {
  const dim3 g(p.ranges, a.q.B);
  if (p.threads == 256) hipLaunchKernelGGL((sample_scan_kernel<T, 256, 8>), g, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((sample_scan_kernel<T, 512, 16>), g, dim3(512), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  static LdsAttrOnce attr_once;
  const auto kern = sample_draw_kernel<T>;
  e = attr_once.ensure(reinterpret_cast<const void*>(kern), static_cast<int>(sizeof(SampleShared)));
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kern, dim3(a.q.B), dim3(SMP_DRAW), sizeof(SampleShared), st, a);
  return hipGetLastError();
}
static_assert(sizeof(SampleShared) <= 120 * 1024, "LDS of a compute unit");
template __global__ void sample_draw_kernel<float>(const SampleArgs);
template __global__ void sample_draw_kernel<bf16_t>(const SampleArgs);

extern "C" int ecospa_sample(ecospa_ctx* ctx, const ecospa_sample_args* q) {
  if (!ctx || !q || !q->logits || !q->u || !q->token) return ECOSPA_ERR_NULL;
  if (!dtype_ok(q->dtype)) return ECOSPA_ERR_DTYPE;
  if (q->B < 1 || q->V < 1 || q->B > 65535 || q->V > SMP_MAX_V || q->ld < q->V) return ECOSPA_ERR_SHAPE;
  if (!aligned16(q->logits) || q->ld % 8) return ECOSPA_ERR_ALIGN;
  const void* const four[] = {q->u, q->temperature, q->top_k, q->top_p, q->min_p, q->token, q->prob};
  for (const void* p : four)
    if (reinterpret_cast<uintptr_t>(p) & 3u) return ECOSPA_ERR_ALIGN;
  SampleArgs a;
  memset(&a, 0, sizeof(a));
  a.q = *q;
  const SamplePlan p = sample_plan(q->B, q->V);
  a.range = p.range; a.ranges = p.ranges; a.chunks = p.chunks;
  WsCarver ws(ctx->ws, ctx->ws_bytes);
  sample_carve(a, p, ws, q->B);
  if (!ws.ok()) return ECOSPA_ERR_WORKSPACE;
  const hipError_t e = q->dtype == ECOSPA_BF16 ? sample_launch<bf16_t>(a, p, ctx->stream) : sample_launch<float>(a, p, ctx->stream);
  if (e != hipSuccess) return hip_fail(ctx, e, "sample_kernel");
  return ECOSPA_OK;
}
