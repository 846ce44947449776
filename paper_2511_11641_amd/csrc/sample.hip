// A token drawn for every row of logits by a given random number, after temperature, top-k, top-p and min-p.
//
// A token of logit x weighs 2^(t - e), t = x log2(e) / T, with e the whole number at or above the largest t; weights are held as whole numbers of
// 2^-42, so that sums are exact in any order and results repeat.  All three restrictions keep a leading part of the tokens in order (larger logits
// first, equal ones by index), so what is kept is everything up to one token, the border.  Nothing is sorted:
//   scan    A workgroup takes a range of a row, once through memory: its largest logit, the weights relative to its own binade (a shift brings them to the
//           row's later on), and a histogram of weights (and counts) in bins of a sixteenth of a binade.
//   draw    A workgroup a row: the ranges' histograms are added and the bin with the border is found; the row is read again (it is in the last-level cache), by
//           comparisons alone, for the tokens of that bin, which go to a list in LDS; there the border is found digit by digit of (logit, index).  The histograms
//           then say what every range keeps, hence the range that the random number falls into; only its weights are computed again.  Where top-k keeps few tokens, the
//           list takes all of them, and the rest is counted there.
// Weights decide on whole tokens next to borders, so they are good to 2^-42: a table of 64 powers and four terms of the series in 64 bits, which run at the rate
// of 32 bits here.
// 256 rows of 131072 fp32 logits with top-p and min-p: scan 46 us, bound by 33 vector instructions a token, the unit 82 % busy (134 MB alone would be 21); draw 40 us,
// where every row is read again from the last-level cache at up to 11 TB/s and the rest is some 20 dependent steps.  One bf16 row of 32000 with a top-k of 50 and top-p:
// scan 6.5, draw 15, a dozen dependent steps; 20 without the list of all that top-k keeps.  32 logits a lane and four wavefronts a range leave 6 wavefronts a SIMD
// (16 logits 50 us, eight wavefronts 49).
#include "common.h"

#include <type_traits>

typedef unsigned long long smp_u64;

#define SMP_BITS 42
#define SMP_BIN_LOG2 4                   // bins of a binade
#define SMP_LEAST (64 * (SMP_BITS + 4))  // places, in 64ths of a binade below e: further down is as far down as nothing
#define SMP_BINS ((SMP_LEAST >> (6 - SMP_BIN_LOG2)) + 4)
#define SMP_CHUNK 512                    // tokens of a chunk: 8 a lane
#define SMP_MAX_V (1 << 20)              // 42 bits of a weight and 20 of a vocabulary: sums below 2^63
#define SMP_RANGE_LOG2 13                // tokens of a range: 8192, or
#define SMP_FEW_LOG2 11                  // 2048 where a row has few (sample_plan), SMP_FEW_V at most
#define SMP_FEW_V (1 << 16)
#define SMP_MAX_RANGES 128
#define SMP_LIST 4096
#define SMP_SHORT 256
#define SMP_SCAN 256
#define SMP_DRAW 1024

struct SamplePart {
  double e;              // binade that the range's weights are relative to
  smp_u64 total;         // their sum
  float top;             // largest logit, -inf: none
  int at;                // its lowest token (greedy rows alone)
  int bins;              // histogram bins in use
  int pad;
};
struct SampleArgs {
  ecospa_sample_args q;
  SamplePart* part;      // [B][ranges]
  float* chunk_top;      // [B][chunks]
  smp_u64* bin_sum;      // [B][ranges][SMP_BINS]
  unsigned* bin_count;   // [B][ranges][SMP_BINS]
  int range, range_log2, ranges, chunks;      // tokens of a range (a multiple of SMP_CHUNK)
};

constexpr double smp_power(int j) {      // 2^(j / 64)
  const double x = j * (0.69314718055994530942 / 64.0);
  double s = 1.0, t = 1.0;
  for (int i = 1; i < 24; ++i) { t *= x / i; s += t; }
  return s;
}
struct SamplePowers { smp_u64 p[64]; };
constexpr SamplePowers smp_powers() {      // bits of 2^(j / 64 + 42), less j << 14 in the upper word: k << 14 brings it back for k's low bits, and whole binades with it
  SamplePowers t{};
  for (int j = 0; j < 64; ++j) t.p[j] = __builtin_bit_cast(smp_u64, smp_power(j) * (1ull << SMP_BITS)) - (static_cast<smp_u64>(j) << 46);
  return t;
}
__device__ const SamplePowers SMP_POWERS = smp_powers();

// Where a logit of a range lies, in 64ths of a binade relative to the range's e.  Ordinary: one fused step.  Where the largest is +inf (it alone, with its equals,
// weighs then), or a temperature so small that places have no fraction left: by the distance to the largest, which is at 0.
struct SampleScale {
  double c64, off;
  float top;
  bool plain;
};
__device__ __forceinline__ double smp_binade(float top, double c64) {
  return fabsf(top) == INFINITY ? 0.0 : __builtin_ceil(static_cast<double>(top) * c64 * (1.0 / 64.0));
}
__device__ __forceinline__ SampleScale smp_scale(float top, double c64, double e) {
  const bool plain = fabsf(top) < INFINITY && __builtin_fabs(e) < 1e12;
  return {c64, plain ? -64.0 * e : 0.0, top, plain};
}
template <bool PLAIN>
__device__ __forceinline__ double smp_place_as(float x, const SampleScale& s) {      // no weight (NaN, -inf): far below
  if constexpr (PLAIN) return __builtin_fmax(__builtin_fma(static_cast<double>(x), s.c64, s.off), -1.0 * SMP_LEAST);
  else return x == s.top ? 0.0 : __builtin_fmax((static_cast<double>(x) - static_cast<double>(s.top)) * s.c64, -1.0 * SMP_LEAST);
}
__device__ __forceinline__ double smp_place(float x, const SampleScale& s) { return s.plain ? smp_place_as<true>(x, s) : smp_place_as<false>(x, s); }
// The weight times 2^42 of a place u as two factors: a power of the table, moved by whole binades, and the series.  k: u in whole 64ths (the low bits of u + 1.5 2^52).
struct SampleWeight {
  double power, series;
  int k;
};
struct SampleSeries {      // of the scan, kept in registers: literals are moved there again for every token
  double c4 = SMP_L * SMP_L * SMP_L * SMP_L / 24.0, c3 = SMP_L * SMP_L * SMP_L / 6.0, c2 = SMP_L * SMP_L / 2.0, c1 = SMP_L, whole = 4503599627370496.0;
  static constexpr double SMP_L = 0.69314718055994530942 / 64.0;
  __device__ __forceinline__ void keep() { asm volatile("" : "+v"(c4), "+v"(c3), "+v"(c2), "+v"(c1), "+v"(whole)); }
};
__device__ __forceinline__ SampleWeight smp_weight(double u, const smp_u64* powers, const SampleSeries& c) {
  constexpr double M = 6755399441055744.0;
  const double m = u + M, r = u - (m - M);
  SampleWeight w;
  w.k = static_cast<int>(__builtin_bit_cast(smp_u64, m));
  double p = __builtin_fma(r, c.c4, c.c3);
  p = __builtin_fma(p, r, c.c2);
  p = __builtin_fma(p, r, c.c1);
  w.series = __builtin_fma(p, r, 1.0);
  const smp_u64 t = powers[w.k & 63];
  const unsigned hi = static_cast<unsigned>(t >> 32) + (static_cast<unsigned>(w.k) << 14);
  w.power = __builtin_bit_cast(double, (static_cast<smp_u64>(hi) << 32) | static_cast<unsigned>(t));
  return w;
}
__device__ __forceinline__ smp_u64 smp_whole(const SampleWeight& w, const SampleSeries& c) {      // the nearest whole number: the low bits of 2^52 + the weight
  return __builtin_bit_cast(smp_u64, __builtin_fma(w.series, w.power, c.whole)) & 0xfffffffffffffull;
}
// the bin of a place: places are 0 or less but for a rounding of 2^-6 at most (e below 10^12), so k is 0 or less
__device__ __forceinline__ int smp_bin(int k) { return -k >> (6 - SMP_BIN_LOG2); }
// larger logits first: ascending numbers, -0 with +0 (NaN has no weight and is never asked for)
__device__ __forceinline__ unsigned smp_rank(float x) {
  const unsigned b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? b : 0x7fffffffu - b;
}
// sums over the wavefront, v < 2^51 (a lane of the scan adds up 32 tokens, 2^47 at most): two parts through lane permutations, whose sums of 64 lanes stay below 2^32
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
template <typename T, int EACH>
__global__ __launch_bounds__(SMP_SCAN) void sample_scan_kernel(const SampleArgs a) {
  constexpr int WAVES = SMP_SCAN / 64, CH = EACH / 8;
  __shared__ smp_u64 sum[SMP_BINS + 64];       // behind the bins a place a lane for what weighs nothing: no branch, and no address that many lanes add to
  __shared__ unsigned count[SMP_BINS + 64];
  __shared__ smp_u64 powers[64];
  __shared__ float red_top[WAVES];
  __shared__ int red_at[WAVES], used;
  __shared__ smp_u64 total;
  const ecospa_sample_args& q = a.q;
  const int b = blockIdx.y, v0 = blockIdx.x * a.range, n = min(a.range, q.V - v0), tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const T* const row = static_cast<const T*>(q.logits) + b * q.ld + v0;
  float x[CH][8];
  if (n == a.range) {
#pragma unroll
    for (int c = 0; c < CH; ++c) smp_load(row + (c * WAVES + wave) * SMP_CHUNK + lane * 8, 8, x[c]);
  } else {
#pragma unroll
    for (int c = 0; c < CH; ++c) smp_load(row + (c * WAVES + wave) * SMP_CHUNK + lane * 8, n - (c * WAVES + wave) * SMP_CHUNK - lane * 8, x[c]);
  }
  const SampleRow r = smp_row(q, b);
  const bool bins = !r.greedy && (r.by_k || r.by_p || r.by_min);
  if (tid < 64) powers[tid] = SMP_POWERS.p[tid];
  if (tid == 0) { used = 0; total = 0; }
  if (bins) {
    for (int i = tid; i < SMP_BINS; i += SMP_SCAN) { sum[i] = 0; count[i] = 0; }
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
      *part = SamplePart{0.0, 0, top, v0 + static_cast<int>(at), 0, 0};
    }
    return;
  }
  const double e = smp_binade(top, r.c64);
  const SampleScale scale = smp_scale(top, r.c64, e);
  smp_u64 s = 0;
  SampleSeries series;
  series.keep();
  // mode 0: weights alone, 1: their histogram, 2: and that of counts
  const auto weigh = [&](auto plain, auto mode) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float xi = x[c][i];
        asm volatile("" : "+v"(xi));      // its conversion stays here: made once for all modes, in front of them, it would take two registers a token
        const SampleWeight wt = smp_weight(smp_place_as<decltype(plain)::value>(xi, scale), powers, series);
        const smp_u64 w = smp_whole(wt, series);
        s += w;
        if constexpr (decltype(mode)::value > 0) {
          const int bin = w != 0 ? smp_bin(wt.k) : SMP_BINS + lane;
          atomicAdd(&sum[bin], w);
          if constexpr (decltype(mode)::value > 1) atomicAdd(&count[bin], 1u);
        }
      }
    }
  };
  using std::integral_constant;
  if (!scale.plain) weigh(std::false_type{}, integral_constant<int, 2>{});
  else if (!bins) weigh(std::true_type{}, integral_constant<int, 0>{});
  else if (r.by_k) weigh(std::true_type{}, integral_constant<int, 2>{});
  else weigh(std::true_type{}, integral_constant<int, 1>{});
  s = smp_wave_sum(s);
  if (lane == 0) atomicAdd(&total, s);
  __syncthreads();
  if (bins) {
    int most = 0;
    for (int i = tid; i < SMP_BINS; i += SMP_SCAN) most = sum[i] != 0 ? i + 1 : most;
    if (most) atomicMax(&used, most);
    __syncthreads();
  }
  if (tid == 0) *part = SamplePart{e, total, top, 0, used, 0};
  if (bins) {
    const long long at = (static_cast<long long>(b) * a.ranges + blockIdx.x) * SMP_BINS;
    for (int i = tid; i < used; i += SMP_SCAN) {
      a.bin_sum[at + i] = sum[i];
      if (r.by_k) a.bin_count[at + i] = count[i];
    }
  }
}

// ---------------------------------------------------------------------------------------------
// draw
// ---------------------------------------------------------------------------------------------
struct SampleShared {
  smp_u64 list_key[SMP_LIST], list_w[SMP_LIST];      // weights relative to their range
  smp_u64 kept[SMP_MAX_RANGES];                       // kept weight by range, relative to it
  smp_u64 sum[SMP_BINS];
  unsigned count[SMP_BINS];
  smp_u64 digit_sum[256];
  unsigned digit_count[256];
  smp_u64 powers[64];
  SampleScale scale[SMP_MAX_RANGES];
  int shift[SMP_MAX_RANGES], bins[SMP_MAX_RANGES];    // binades below the row's (63: no weight); histogram bins in use
  float lo[SMP_MAX_RANGES], hi[SMP_MAX_RANGES];       // logits that can fall into the bin that is looked for
  smp_u64 chunk[SMP_DRAW / 64], scan[SMP_DRAW / 64], scan_w[SMP_DRAW / 64], out[4];
  float red_f[SMP_DRAW / 64];
  double red_d[SMP_DRAW / 64];
  int listed;
};
static_assert(sizeof(SampleShared) <= 120 * 1024, "LDS of a compute unit");
static_assert(SMP_BINS <= SMP_DRAW, "a bin a thread");
static_assert(SMP_MAX_V >> SMP_RANGE_LOG2 <= SMP_MAX_RANGES && SMP_FEW_V >> SMP_FEW_LOG2 <= SMP_MAX_RANGES && SMP_MAX_RANGES <= SMP_DRAW, "ranges of a row");
// running sums over the lanes of a wavefront, by lane permutations; ROWS: over every 16 lanes
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ smp_u64 smp_moved(smp_u64 v) {      // 0 where a lane has no source
  const unsigned lo = static_cast<unsigned>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, ROW_MASK, 0xF, true));
  const unsigned hi = static_cast<unsigned>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v >> 32), CTRL, ROW_MASK, 0xF, true));
  return (static_cast<smp_u64>(hi) << 32) | lo;
}
template <bool ROWS = false>
__device__ __forceinline__ smp_u64 smp_inclusive(smp_u64 v) {
  v += smp_moved<0x111, 0xF>(v);
  v += smp_moved<0x112, 0xF>(v);
  v += smp_moved<0x114, 0xF>(v);
  v += smp_moved<0x118, 0xF>(v);
  if constexpr (!ROWS) {
    v += smp_moved<0x142, 0xA>(v);      // lane 15 of a row to the next row: rows 1 and 3
    v += smp_moved<0x143, 0xC>(v);      // lane 31 to rows 2 and 3
  }
  return v;
}
__device__ __forceinline__ smp_u64 smp_lane(smp_u64 v, int l) {
  const unsigned lo = static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(v), l)), hi = static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(v >> 32), l));
  return (static_cast<smp_u64>(hi) << 32) | lo;
}
// A value a wavefront, in LDS: the sum in front of this wavefront and that of all.  (A read a lane: sixteen reads of the whole wavefront would keep the LDS busy.)
static_assert(SMP_DRAW == 16 * 64, "a row of lanes holds a value a wavefront");
__device__ __forceinline__ smp_u64 smp_waves(const smp_u64* each, int wave, smp_u64& all) {
  const smp_u64 own = each[threadIdx.x & 15], upto = smp_inclusive<true>(own);
  all = smp_lane(upto, 15);
  return smp_lane(upto - own, wave);
}
// The workgroup: the first of n <= SMP_DRAW bins where the running sum of v reaches `need(the sum of all)` (the last bin that holds anything if none does): its index,
// the sums of v and of w over the bins in front of it, whether it is reached.  A bin a thread.  Every thread has left sh.scan, sh.scan_w and sh.out behind when it is called.
struct SampleFound {
  int bin;
  smp_u64 front, front_w, need;
  bool reached;
};
template <typename N, typename V, typename W>
__device__ __forceinline__ SampleFound smp_find(SampleShared& sh, int n, N&& need_, V&& v, W&& w) {
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));      // addresses are made here: kept over the phases of a draw they would not fit the registers
  const int lane = tid & 63, wave = tid >> 6;
  const smp_u64 own = tid < n ? v(tid) : 0, own_w = tid < n ? w(tid) : 0;
  smp_u64 upto = own, upto_w = own_w;
  if (wave * 64 < n) {
    upto = smp_inclusive(own);
    upto_w = smp_inclusive(own_w);
  }
  if (lane == 63) { sh.scan[wave] = upto; sh.scan_w[wave] = upto_w; }
  if (tid == 0) { sh.out[0] = 0; sh.out[1] = 0; sh.out[2] = 0; }
  __syncthreads();
  smp_u64 all, all_w;
  const int w_ = __builtin_amdgcn_readfirstlane(wave);
  upto += smp_waves(sh.scan, w_, all);
  upto_w += smp_waves(sh.scan_w, w_, all_w);
  SampleFound f;
  f.need = need_(all);
  f.reached = all >= f.need;
  if (own != 0 && (f.reached ? upto >= f.need && upto - own < f.need : upto == all)) {
    sh.out[0] = static_cast<smp_u64>(tid);
    sh.out[1] = upto - own;
    sh.out[2] = upto_w - own_w;
  }
  __syncthreads();
  f.bin = static_cast<int>(sh.out[0]);
  f.front = sh.out[1];
  f.front_w = sh.out[2];
  return f;
}
__device__ __forceinline__ smp_u64 smp_key(float x, int v) { return (static_cast<smp_u64>(smp_rank(x)) << 20) | static_cast<unsigned>(v); }
__device__ __forceinline__ float smp_logit(smp_u64 key) {
  const unsigned r = static_cast<unsigned>(key >> 20);
  return __uint_as_float(r & 0x80000000u ? r : 0x7fffffffu - r);
}
__device__ __forceinline__ int smp_token(smp_u64 key) { return static_cast<int>(key & 0xfffffu); }

// The border among the tokens of a short list (up to SMP_SHORT): every token's place in order is counted against all others, four lanes a token.
__device__ __forceinline__ smp_u64 smp_border_short(SampleShared& sh, int n, int range_log2, smp_u64 need, bool counted, smp_u64& taken) {
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  const int i = tid >> 2;
  if (tid < n) sh.digit_sum[tid] = sh.list_w[tid] >> sh.shift[smp_token(sh.list_key[tid]) >> range_log2];
  if (tid == 0) { sh.out[0] = ~0ull; sh.out[1] = 0; sh.out[2] = 0; }
  __syncthreads();
  if (i < n) {
    const smp_u64 key = sh.list_key[i], w = sh.digit_sum[i];
    smp_u64 front = 0;
    unsigned front_n = 0;
    for (int m = tid & 3; m < n; m += 4) {
      const smp_u64 x = sh.digit_sum[m];
      const bool in = sh.list_key[m] < key && x != 0;
      front += in ? x : 0;
      front_n += in ? 1u : 0u;
    }
    front += __shfl_xor(front, 1, 64);
    front_n += __shfl_xor(front_n, 1, 64);
    front += __shfl_xor(front, 2, 64);
    front_n += __shfl_xor(front_n, 2, 64);
    if ((tid & 3) == 0 && w != 0) {
      atomicMax(&sh.out[2], front + w);
      if (counted ? front_n + 1u == need : front < need && front + w >= need) { sh.out[0] = key; sh.out[1] = front + w; }
    }
  }
  __syncthreads();
  const smp_u64 key = sh.out[0];
  taken = key == ~0ull ? sh.out[2] : sh.out[1];      // fewer than asked for: all of them
  __syncthreads();
  return key;
}

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
  if ((tid & 63) == 0 && lo <= hi) { atomicMin(&sh.out[0], lo); atomicMax(&sh.out[1], hi); }
  __syncthreads();
  lo = sh.out[0];
  hi = sh.out[1];
  __syncthreads();
  taken = 0;
  if (lo > hi) return 0;      // no token of any weight
  int shift = max(64 - __clzll((hi - lo) | 1ull) - 8, 0);
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
    const auto s = [&](int i) __attribute__((always_inline)) { return sh.digit_sum[i]; };
    const auto c = [&](int i) __attribute__((always_inline)) { return static_cast<smp_u64>(sh.digit_count[i]); };
    const auto n = [&](smp_u64) __attribute__((always_inline)) { return need; };
    const SampleFound f = counted ? smp_find(sh, 256, n, c, s) : smp_find(sh, 256, n, s, c);
    const int d = f.bin;
    const smp_u64 front = f.front, front_other = f.front_w, in_sum = sh.digit_sum[d], in_count = sh.digit_count[d];
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

// x p for 0 < p < 1, cut to a whole number, and whether anything was cut off: an fp32 number is 24 bits and a shift, so the product is exact in 128 bits (x < 2^63)
__device__ __forceinline__ smp_u64 smp_times(smp_u64 x, float p, bool& more) {
  const unsigned bits = __float_as_uint(p), e = bits >> 23;
  const int shift = min(150 - static_cast<int>(max(e, 1u)), 127);      // 87 bits of a product: further down nothing is left
  const unsigned __int128 prod = static_cast<unsigned __int128>(x) * ((bits & 0x7fffffu) | (e ? 0x800000u : 0u)), whole = prod >> shift;
  more = (whole << shift) != prod;
  return static_cast<smp_u64>(whole);
}
// the least whole number of 2^-42 at or above top_p < 1 times the weight, 1 at least
__device__ __forceinline__ smp_u64 smp_share(smp_u64 weight, float top_p) {
  if (!(top_p > 0.f)) return 1ull;
  bool more;
  const smp_u64 whole = smp_times(weight, top_p, more);
  return max(whole + (more ? 1 : 0), 1ull);
}
// where a random number falls among `total`
__device__ __forceinline__ smp_u64 smp_target(float u, smp_u64 total) {
  if (u >= 1.f) return total - 1;
  bool more;
  return u > 0.f ? smp_times(total, u, more) : 0ull;
}
// The rest of a draw whose list holds every token that top-k can keep, SMP_SHORT at most: each is counted against all others, four lanes a token, in order of
// the logits for what is kept and in order of the vocabulary for the draw.
__device__ __forceinline__ void smp_draw_short(SampleShared& sh, const SampleArgs& a, const SampleRow& r, int n, double least_place, int b) {
  const ecospa_sample_args& q = a.q;
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  const int i = tid >> 2;
  if (tid < n) sh.digit_sum[tid] = sh.list_w[tid] >> sh.shift[smp_token(sh.list_key[tid]) >> a.range_log2];
  if (tid == 0) { sh.out[0] = 0; sh.out[1] = 0; }
  __syncthreads();
  const bool mine = i < n, first = mine && (tid & 3) == 0;
  const smp_u64 key = mine ? sh.list_key[i] : 0, w = mine ? sh.digit_sum[i] : 0;
  const int g = smp_token(key) >> a.range_log2, by = sh.shift[g];
  smp_u64 front = 0;
  unsigned front_n = 0;
  for (int m = tid & 3; m < n; m += 4) {
    const smp_u64 x = sh.digit_sum[m];
    const bool in = sh.list_key[m] < key && x != 0;
    front += in ? x : 0;
    front_n += in ? 1u : 0u;
  }
  front += __shfl_xor(front, 1, 64);
  front_n += __shfl_xor(front_n, 1, 64);
  front += __shfl_xor(front, 2, 64);
  front_n += __shfl_xor(front_n, 2, 64);
  bool keep = w != 0 && front_n < static_cast<unsigned>(r.k);
  if (first && keep) atomicAdd(&sh.out[0], w);
  __syncthreads();
  const double place = smp_place(smp_logit(key), sh.scale[g]);
  keep = keep && (!r.by_p || front < smp_share(sh.out[0], r.p)) && place - 64.0 * by >= least_place;
  if (first) {
    sh.list_w[i] = keep ? w : 0;
    if (keep) atomicAdd(&sh.out[1], w);
  }
  __syncthreads();
  const smp_u64 total = sh.out[1], target = smp_target(q.u[b], total);
  smp_u64 before = 0;
  for (int m = tid & 3; m < n; m += 4) before += smp_token(sh.list_key[m]) < smp_token(key) ? sh.list_w[m] : 0;
  before += __shfl_xor(before, 1, 64);
  before += __shfl_xor(before, 2, 64);
  if (first && keep && before <= target && target < before + w) {
    const SampleWeight exact = smp_weight(place, sh.powers, SampleSeries{});
    q.token[b] = smp_token(key);
    if (q.prob) q.prob[b] = static_cast<float>(fmin(__builtin_ldexp(exact.series * exact.power, -by) / static_cast<double>(total), 1.0));
  }
}

template <typename T>
__global__ __launch_bounds__(SMP_DRAW) void sample_draw_kernel(const SampleArgs a) {
  extern __shared__ __attribute__((aligned(16))) char lds_sample[];
  SampleShared& sh = *reinterpret_cast<SampleShared*>(lds_sample);
  const ecospa_sample_args& q = a.q;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  constexpr int WAVES = SMP_DRAW / 64;
  const SampleSeries series;
  const SampleRow r = smp_row(q, b);
  const SamplePart* const part = a.part + static_cast<long long>(b) * a.ranges;
  if (tid < 64) sh.powers[tid] = SMP_POWERS.p[tid];
  const float* const chunk_top = a.chunk_top + static_cast<long long>(b) * a.chunks;
  const float early_top = chunk_top[min(wave + lane * WAVES, a.chunks - 1)];      // the chunks that `walk` looks at first
  // the row's largest logit and binade
  SamplePart mine{0.0, 0, -INFINITY, 0, 0, 0};
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
    sh.bins[tid] = none ? 0 : mine.bins;
    sh.kept[tid] = none ? 0 : mine.total;
    sh.scale[tid] = smp_scale(mine.top, r.c64, mine.e);
  }
  __syncthreads();
  const T* const row = static_cast<const T*>(q.logits) + b * q.ld;
  const smp_u64* const bin_sums = a.bin_sum + static_cast<long long>(b) * a.ranges * SMP_BINS;
  const unsigned* const bin_counts = a.bin_count + static_cast<long long>(b) * a.ranges * SMP_BINS;
  const int per_log2 = a.range_log2 - 9;      // chunks of a range
  const bool bounded = r.by_k || r.by_p || r.by_min;
  // least place (relative to the row's binade) that min-p leaves, and its bin
  const double least_place = r.by_min ? smp_place(top, smp_scale(top, r.c64, e)) + 64.0 * log2(static_cast<double>(r.min_p)) : -1e30;
  const int least_bin = r.by_min ? smp_bin(static_cast<int>(__builtin_rint(__builtin_fmax(least_place, -1.0 * SMP_LEAST)))) : SMP_BINS;
  if (bounded) {      // the row's histogram, eight ranges on their way together
    for (int i = tid; i < SMP_BINS; i += SMP_DRAW) {
      smp_u64 s = 0;
      unsigned c = 0;
      for (int g0 = 0; g0 < a.ranges; g0 += 8) {
        smp_u64 x[8];
        unsigned y[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const int g = min(g0 + u, a.ranges - 1), from = i - (sh.shift[g] << SMP_BIN_LOG2);
          const bool in = g0 + u < a.ranges && from >= 0 && from < sh.bins[g];
          const int at = g * SMP_BINS + max(from, 0);      // read in any case: loads under a condition are waited for one by one
          x[u] = bin_sums[at] >> sh.shift[g];
          y[u] = r.by_k ? bin_counts[at] : 0;
          x[u] = in ? x[u] : 0;
          y[u] = in ? y[u] : 0;
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) { s += x[u]; c += y[u]; }
      }
      sh.sum[i] = s;
      sh.count[i] = c;
    }
  }
  const auto bin_sum = [&](int i) __attribute__((always_inline)) { return sh.sum[i]; };
  const auto bin_count = [&](int i) __attribute__((always_inline)) { return static_cast<smp_u64>(sh.count[i]); };
  // f(chunk, logits of the lane's eight tokens) for the wavefront's chunks that reach the bin that is looked for, AHEAD of them on their way together
  const auto walk = [&](auto ahead_, auto&& f) __attribute__((always_inline)) {
    constexpr int AHEAD = decltype(ahead_)::value;
    for (int c1 = wave; c1 < a.chunks; c1 += 64 * WAVES) {
      const int own = min(c1 + lane * WAVES, a.chunks - 1);      // a lane knows one chunk
      const float own_most = c1 == wave ? early_top : chunk_top[own];
      unsigned long long left = __ballot(c1 + lane * WAVES < a.chunks && own_most >= sh.lo[own >> per_log2]);
      while (left) {
        float x[AHEAD][8];
        int c[AHEAD];
        bool on[AHEAD], whole = true;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
          on[i] = left != 0;
          c[i] = on[i] ? c1 + __builtin_ctzll(left) * WAVES : c[0];      // none left: read again, to no use (a load under a condition is waited for by itself)
          left &= left - 1;
          whole = whole && (c[i] + 1) * SMP_CHUNK <= q.V;
        }
        if (whole) {
#pragma unroll
          for (int i = 0; i < AHEAD; ++i) smp_load(row + c[i] * SMP_CHUNK + lane * 8, 8, x[i]);
        } else {
#pragma unroll
          for (int i = 0; i < AHEAD; ++i) smp_load(row + c[i] * SMP_CHUNK + lane * 8, q.V - c[i] * SMP_CHUNK - lane * 8, x[i]);
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
          if (on[i]) f(c[i], x[i]);
      }
    }
  };
  // the tokens of `bin` (and of those above it) to the list: those whose logit can be in it first, then what they weigh
  const auto gather = [&](int bin, bool above) __attribute__((always_inline)) {
    if (tid == 0) sh.listed = 0;
    if (tid < a.ranges) {
      const SampleScale& s = sh.scale[tid];
      const int by = sh.shift[tid], width = 1 << (6 - SMP_BIN_LOG2);
      float lo = INFINITY, hi = -INFINITY;
      if (by < 63) {
        lo = -INFINITY;
        hi = INFINITY;
        if (s.plain && s.c64 > 0.0) {      // places of the bin, and a little on both sides
          const double u1 = 64.0 * by - width * bin, xl = (u1 - width - s.off) / s.c64, xh = (u1 + 1.0 - s.off) / s.c64;
          lo = static_cast<float>(xl - (__builtin_fabs(xl) * 1e-6 + 1e-36));
          hi = bin == 0 || above ? INFINITY : static_cast<float>(xh + (__builtin_fabs(xh) * 1e-6 + 1e-36));
        }
      }
      sh.lo[tid] = lo;
      sh.hi[tid] = hi;
    }
    __syncthreads();
    walk(std::integral_constant<int, sizeof(T) == 2 ? 4 : 2>{}, [&](int c, const float (&x)[8]) __attribute__((always_inline)) {
      const float lo = sh.lo[c >> per_log2], hi = sh.hi[c >> per_log2];
      const int v = c * SMP_CHUNK + lane * 8;
      // few of them are: a bit each, then one token a lane and turn
      float y[8];
      unsigned bits = 0u;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        y[i] = x[i];
        asm volatile("" : "+v"(y[i]));      // a register: chosen among by selects, not through memory
        bits |= y[i] >= lo && y[i] <= hi ? 1u << i : 0u;
      }
#pragma unroll 1
      while (bits) {
        const int i = __builtin_ctz(bits);
        float yi = y[0];
#pragma unroll
        for (int m = 1; m < 8; ++m) yi = i == m ? y[m] : yi;
        const int slot = atomicAdd(&sh.listed, 1);
        if (slot < SMP_LIST) sh.list_key[slot] = smp_key(yi, v + i);
        bits &= bits - 1;
      }
    });
    __syncthreads();
    for (int i = tid; i < min(sh.listed, SMP_LIST); i += SMP_DRAW) {
      const smp_u64 key = sh.list_key[i];
      const int g = smp_token(key) >> a.range_log2, by = sh.shift[g];
      const SampleWeight w = smp_weight(smp_place(smp_logit(key), sh.scale[g]), sh.powers, series);
      const int at = smp_bin(w.k) + (by << SMP_BIN_LOG2);
      sh.list_w[i] = at == bin || (above && at < bin) ? smp_whole(w, series) : 0;
    }
    __syncthreads();
  };
  // f(key, weight relative to its range, its shift) for every token of `bin`, from the list or, where it did not hold them, from the row
  const auto each_of = [&](int bin, auto&& f) __attribute__((always_inline)) {
    const int n = sh.listed;
    if (n <= SMP_LIST) {
      for (int i = tid; i < n; i += SMP_DRAW) {
        const smp_u64 key = sh.list_key[i], w = sh.list_w[i];
        const int by = sh.shift[smp_token(key) >> a.range_log2];
        if (w >> by) f(key, w, by);
      }
    } else {
      walk(std::integral_constant<int, 1>{}, [&](int c, const float (&x)[8]) __attribute__((always_inline)) {
        const int g = c >> per_log2, by = sh.shift[g];
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[i];
#pragma unroll 1
        for (int i = 0; i < 8; ++i) {      // a loop: this is the rare path, and it stands here four times
          const float xi = y[0];
#pragma unroll
          for (int m = 0; m < 7; ++m) y[m] = y[m + 1];
          if (!(xi >= sh.lo[g] && xi <= sh.hi[g])) continue;
          const SampleWeight wt = smp_weight(smp_place(xi, sh.scale[g]), sh.powers, series);
          const smp_u64 w = smp_whole(wt, series);
          if ((w >> by) != 0 && smp_bin(wt.k) + (by << SMP_BIN_LOG2) == bin) f(smp_key(xi, c * SMP_CHUNK + lane * 8 + i), w, by);
        }
      });
    }
  };
  int border_bin = SMP_BINS;      // tokens of lower bins are kept whole
  smp_u64 border = ~0ull;         // and of this bin those with keys up to this
  // by the number of tokens first: what is kept then is what top-p is a part of; min-p last
  smp_u64 total = 0;
  bool bordered = false;
  int phase = r.by_k ? 0 : (r.by_p ? 1 : (r.by_min ? 2 : 3));
  __syncthreads();
#pragma unroll 1
  while (phase < 3) {
    int bin = least_bin;
    smp_u64 front = 0, front_sum = 0, need = 0;
    bool reached = true, few = false;
    if (phase < 2) {
      const smp_u64 k = static_cast<smp_u64>(r.k);
      const auto of_all = [&](smp_u64 all) __attribute__((always_inline)) { return smp_share(bordered ? total : all, r.p); };
      const SampleFound f = phase == 0 ? smp_find(sh, SMP_BINS, [&](smp_u64) __attribute__((always_inline)) { return k; }, bin_count, bin_sum)
                                       : smp_find(sh, SMP_BINS, of_all, bin_sum, bin_count);
      bin = f.bin;
      front = f.front;
      need = f.need;
      front_sum = phase == 0 ? f.front_w : front;
      reached = f.reached;
      few = phase == 0 && reached && front + sh.count[bin] <= SMP_SHORT;
      __syncthreads();
    } else if (border_bin <= least_bin) {      // min-p cuts behind the border or in its bin, whose list is there
      break;
    }
    const int next = phase == 0 && r.by_p ? 1 : (phase < 2 && r.by_min ? 2 : 3);
    if (phase == 0 && !reached) {      // fewer tokens than k weigh anything
      phase = next;
      continue;
    }
    if (few) {      // all that top-k can keep: one list for everything that follows
      gather(bin, true);
      if (sh.listed <= SMP_SHORT) {
        smp_draw_short(sh, a, r, sh.listed, least_place, b);
        return;
      }
      __syncthreads();
    }
    if (next == 2 && bin > least_bin) {      // min-p cuts in front of it: where exactly it lies doesn't matter
      border_bin = bin;
      phase = next;
      continue;
    }
    gather(bin, false);
    border = ~0ull;
    if (phase < 2) {
      smp_u64 taken;
      const smp_u64 rest = max(need - min(front, need), 1ull);
      if (sh.listed <= SMP_SHORT)
        border = smp_border_short(sh, sh.listed, a.range_log2, rest, phase == 0, taken);
      else
        border = smp_border(sh, rest, phase == 0,
                          [&](auto&& f) __attribute__((always_inline)) { each_of(bin, [&](smp_u64 key, smp_u64 w, int by) __attribute__((always_inline)) { f(key, w >> by); }); }, taken);
      total = front_sum + taken;
      bordered = true;
    }
    border_bin = bin;
    phase = next;
  }
  const bool cut = border_bin < SMP_BINS;
  const auto kept_there = [&](smp_u64 key, double place, int by) __attribute__((always_inline)) { return key <= border && place - 64.0 * by >= least_place; };
  if (cut) {
    // what every range keeps: its bins above the border's, and the border's tokens
    for (int g = wave; g < a.ranges; g += WAVES) {
      const int end = min(border_bin - (sh.shift[g] << SMP_BIN_LOG2), sh.bins[g]);
      smp_u64 s = 0;
      for (int i = lane; i < end; i += 64) s += bin_sums[g * SMP_BINS + i];
#pragma unroll
      for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off, 64);
      if (lane == 0) sh.kept[g] = s;
    }
    __syncthreads();
    each_of(border_bin, [&](smp_u64 key, smp_u64 w, int by) __attribute__((always_inline)) {
      const int g = smp_token(key) >> a.range_log2;
      if (kept_there(key, smp_place(smp_logit(key), sh.scale[g]), by)) atomicAdd(&sh.kept[g], w);
    });
    __syncthreads();
  }

  // the range that the random number falls into
  const smp_u64 own = tid < a.ranges && sh.shift[tid] < 63 ? sh.kept[tid] >> sh.shift[tid] : 0, upto = smp_inclusive(own);
  if (lane == 63) sh.scan[wave] = upto;
  __syncthreads();
  const smp_u64 front = smp_waves(sh.scan, wave, total) + upto - own;
  const smp_u64 target = smp_target(q.u[b], total);
  if (target >= front && target < front + own) {
    sh.out[0] = static_cast<smp_u64>(tid);
    sh.out[1] = (target - front) << sh.shift[tid];      // relative to the range from here on
  }
  __syncthreads();
  const int g = static_cast<int>(sh.out[0]), by = sh.shift[g], n_chunks = 1 << per_log2, c = (g << per_log2) + wave;
  smp_u64 into = sh.out[1], w[8], s = 0;
  double exact[8];
  if (wave < n_chunks) {      // a wavefront a chunk
    float x[8];
    smp_load(row + c * SMP_CHUNK + lane * 8, q.V - c * SMP_CHUNK - lane * 8, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const double p = smp_place(x[i], sh.scale[g]);
      const SampleWeight wt = smp_weight(p, sh.powers, series);
      const int at = smp_bin(wt.k) + (by << SMP_BIN_LOG2);
      // a token of the border's bin that weighs nothing in the row's binade is not kept: it was not counted
      const bool kept = !cut || at < border_bin || (at == border_bin && (smp_whole(wt, series) >> by) != 0 && kept_there(smp_key(x[i], c * SMP_CHUNK + lane * 8 + i), p, by));
      exact[i] = wt.series * wt.power;
      w[i] = kept ? smp_whole(wt, series) : 0;
      s += w[i];
    }
    const smp_u64 all = smp_wave_sum(s);
    if (lane == 0) sh.chunk[wave] = all;
  }
  __syncthreads();
  if (wave >= n_chunks) return;
  smp_u64 before = 0;
  int last = 0;      // the last chunk that starts at or in front of the target and holds anything
  for (int i = 0; i < n_chunks; ++i) {
    if (sh.chunk[i] != 0 && before <= into) last = i;
    before += sh.chunk[i];
  }
  if (wave != last) return;
  for (int i = 0; i < wave; ++i) into -= sh.chunk[i];
  before = smp_inclusive(s) - s;
  const unsigned long long have = __ballot(s != 0 && before <= into);      // the last lane, likewise
  if (lane != 63 - __clzll(have)) return;
  int at = 0;
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
// Ranges of 8192 tokens; of 2048 where a row has few and the rows don't fill the card (both kernels, fp32 with top-p, us, 2048 against 8192: 1 row of 32000 21.5 : 24.4,
// 1 of 131072 32 : 27, 64 of 32000 33.6 : 34.3, 128 of 32000 39 : 36).
struct SamplePlan { int range_log2, ranges, chunks; };
static SamplePlan sample_plan(int B, int V) {
  SamplePlan p;
  const bool few = V <= SMP_FEW_V && static_cast<long long>(B) * V <= 1 << 21;
  p.range_log2 = few ? SMP_FEW_LOG2 : SMP_RANGE_LOG2;
  p.ranges = (V + (1 << p.range_log2) - 1) >> p.range_log2;
  p.chunks = (V + SMP_CHUNK - 1) / SMP_CHUNK;
  return p;
}
static void sample_carve(SampleArgs& a, const SamplePlan& p, WsCarver& ws, int B) {
  const size_t n = static_cast<size_t>(B) * p.ranges;
  a.part = static_cast<SamplePart*>(ws.take(n * sizeof(SamplePart)));
  a.bin_sum = static_cast<smp_u64*>(ws.take(n * SMP_BINS * sizeof(smp_u64)));
  a.bin_count = static_cast<unsigned*>(ws.take(n * SMP_BINS * sizeof(unsigned)));
  a.chunk_top = static_cast<float*>(ws.take(static_cast<size_t>(B) * p.chunks * sizeof(float)));
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
  if (p.range_log2 == SMP_FEW_LOG2) hipLaunchKernelGGL((sample_scan_kernel<T, 8>), g, dim3(SMP_SCAN), 0, st, a);
  else hipLaunchKernelGGL((sample_scan_kernel<T, 32>), g, dim3(SMP_SCAN), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  static LdsAttrOnce attr_once;
  const auto kern = sample_draw_kernel<T>;
  e = attr_once.ensure(reinterpret_cast<const void*>(kern), static_cast<int>(sizeof(SampleShared)));
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kern, dim3(a.q.B), dim3(SMP_DRAW), sizeof(SampleShared), st, a);
  return hipGetLastError();
}
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
  a.range = 1 << p.range_log2; a.range_log2 = p.range_log2; a.ranges = p.ranges; a.chunks = p.chunks;
  WsCarver ws(ctx->ws, ctx->ws_bytes);
  sample_carve(a, p, ws, q->B);
  if (!ws.ok()) return ECOSPA_ERR_WORKSPACE;
  const hipError_t e = q->dtype == ECOSPA_BF16 ? sample_launch<bf16_t>(a, p, ctx->stream) : sample_launch<float>(a, p, ctx->stream);
  if (e != hipSuccess) return hip_fail(ctx, e, "sample_kernel");
  return ECOSPA_OK;
}
