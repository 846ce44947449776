// Products of 8-bit integers with a scale for each row of either operand: rows brought to 8 bits, and the contraction's entry point (its
// kernels are those of gemm_ring.h, gemm_flow.h and gemm_share.h).
#include "gemm.h"

typedef unsigned i8_uintx2 __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------------------------------------
// Rows to 8 bits: s = max |x| / 127, q = x / s to the nearest whole number (half to even), the quotients those of a division.  The row stays in
// registers between its maximum and its codes: up to EACH pieces of 8 elements a thread; wider rows are read again.  The maximum is taken
// of the bits without the sign, as integers, above which infinity and NaN rank: such a row has a scale of NaN, so that products with it say so.
// ---------------------------------------------------------------------------------------------
struct QuantArgs {
  const void* x;
  signed char* q;
  float* scale;
  long long ld, ld_q;
  int rows, cols;
};
template <typename T>
__device__ __forceinline__ void quant_load(const T* p, float (&f)[8]) {
  if constexpr (sizeof(T) == 2) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
  } else {
    const float4 lo = *reinterpret_cast<const float4*>(p), hi = *reinterpret_cast<const float4*>(p + 4);
    f[0] = lo.x; f[1] = lo.y; f[2] = lo.z; f[3] = lo.w; f[4] = hi.x; f[5] = hi.y; f[6] = hi.z; f[7] = hi.w;
  }
}
__device__ __forceinline__ unsigned quant_top(const float (&f)[8], unsigned top) {
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
  return top;
}
// x / s from the rounded reciprocal and one correction by the exact remainder; tiny scales, whose reciprocal can be infinite, by division
__device__ __forceinline__ i8_uintx2 quant_codes(const float (&f)[8], float s, float r, bool tiny) {
  unsigned w[2] = {0u, 0u};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float y = f[i] * r;
    y = __builtin_fmaf(__builtin_fmaf(-y, s, f[i]), r, y);
    if (tiny) y = fminf(fmaxf(f[i] / s, -127.f), 127.f);      // a subnormal scale is a coarse one
    w[i >> 2] |= (static_cast<unsigned>(static_cast<int>(rintf(y))) & 0xffu) << (8 * (i & 3));
  }
  return i8_uintx2{w[0], w[1]};
}
template <typename T, int THREADS, int EACH>
__global__ __launch_bounds__(256) void quant_rows_kernel(const QuantArgs a) {
  constexpr int ROWS = 256 / THREADS;
  const int row = blockIdx.x * ROWS + threadIdx.x / THREADS, t = threadIdx.x % THREADS, pieces = a.cols >> 3;
  const bool in = row < a.rows;
  const T* const x = static_cast<const T*>(a.x) + static_cast<long long>(in ? row : 0) * a.ld;
  float f[EACH][8];
  unsigned top = 0u;
#pragma unroll
  for (int c = 0; c < EACH; ++c) quant_load(x + static_cast<long long>(min(c * THREADS + t, pieces - 1)) * 8, f[c]);
#pragma unroll
  for (int c = 0; c < EACH; ++c) top = quant_top(f[c], top);
  for (int p = EACH * THREADS + t; p < pieces; p += THREADS) {
    float g[8];
    quant_load(x + static_cast<long long>(p) * 8, g);
    top = quant_top(g, top);
  }
  top = ~wave_umin(~top);
  if constexpr (THREADS > 64) {
    __shared__ unsigned red[4];
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
    __syncthreads();
    top = max(max(red[0], red[1]), max(red[2], red[3]));
  }
  if (!in) return;
  const bool fine = top < 0x7f800000u, tiny = top < 0x0d800000u;      // 2^-100
  const float s = fine ? __uint_as_float(top) / 127.f : __uint_as_float(0x7fc00000u);
  const bool zero = s == 0.f || !fine;
  const float d = zero ? 1.f : s, r = 1.f / d;
  if (t == 0) a.scale[row] = s;
  signed char* const q = a.q + static_cast<long long>(row) * a.ld_q;
  const auto put = [&](int p, const float (&g)[8]) __attribute__((always_inline)) {
    const i8_uintx2 w = quant_codes(g, d, r, tiny);
    *reinterpret_cast<i8_uintx2*>(q + static_cast<long long>(p) * 8) = zero ? i8_uintx2{0u, 0u} : w;
  };
#pragma unroll
  for (int c = 0; c < EACH; ++c)
    if (c * THREADS + t < pieces) put(c * THREADS + t, f[c]);
  for (int p = EACH * THREADS + t; p < pieces; p += THREADS) {
    float g[8];
    quant_load(x + static_cast<long long>(p) * 8, g);
    put(p, g);
  }
}

template <typename T>
static void quant_launch(const QuantArgs& a, hipStream_t st) {
  const int pieces = a.cols >> 3;
  // a workgroup a row while rows are few (64 rows of 2048: 2.9 us against 3.3 for a wavefront a row), a wavefront a row where they are many (16384 rows of 512: 6 us against
  // 14, of 2048 16 against 26: 100 MB at 6.1 TB/s, out of the last-level cache)
  const dim3 wide(a.rows), four((a.rows + 3) / 4);
  if (a.rows <= 1024 || pieces > 64 * 8) {
    if (pieces <= 256) hipLaunchKernelGGL((quant_rows_kernel<T, 256, 1>), wide, dim3(256), 0, st, a);
    else if (pieces <= 512) hipLaunchKernelGGL((quant_rows_kernel<T, 256, 2>), wide, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((quant_rows_kernel<T, 256, 8>), wide, dim3(256), 0, st, a);
  } else if (pieces <= 128) hipLaunchKernelGGL((quant_rows_kernel<T, 64, 2>), four, dim3(256), 0, st, a);
  else if (pieces <= 256) hipLaunchKernelGGL((quant_rows_kernel<T, 64, 4>), four, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((quant_rows_kernel<T, 64, 8>), four, dim3(256), 0, st, a);
}

extern "C" int ecospa_quant_rows(ecospa_ctx* ctx, int rows, int cols, int dtype, const void* x, long long ld, void* q, long long ld_q, float* scale) {
  if (!ctx || !x || !q || !scale) return ECOSPA_ERR_NULL;
  if (!dtype_ok(dtype)) return ECOSPA_ERR_DTYPE;
  if (rows < 1 || rows > 1 << 30 || cols < 8 || cols % 8 || ld < cols || ld_q < cols) return ECOSPA_ERR_SHAPE;
  if (!aligned16(x) || !aligned16(q) || ld % 8 || ld_q % 16 || (reinterpret_cast<uintptr_t>(scale) & 3u)) return ECOSPA_ERR_ALIGN;
  QuantArgs a;
  a.ld = ld; a.ld_q = ld_q; a.cols = cols;
  // a launch takes fewer than 2^32 work-items, 2^24 workgroups
  constexpr int most = 1 << 23;
  for (int row = 0; row < rows; row += most) {
    a.x = static_cast<const char*>(x) + row * ld * (dtype == ECOSPA_BF16 ? 2 : 4); a.q = static_cast<signed char*>(q) + row * ld_q; a.scale = scale + row;
    a.rows = rows - row < most ? rows - row : most;
    if (dtype == ECOSPA_BF16) quant_launch<bf16_t>(a, ctx->stream);
    else quant_launch<float>(a, ctx->stream);
    ECOSPA_CHECK_LAUNCH(ctx, "quant_rows_kernel");
  }
  return ECOSPA_OK;
}

extern "C" int ecospa_contract_quant(ecospa_ctx* ctx, int M, int N, int K, const void* A, long long lda, const float* sa, const void* B, long long ldb,
                                  const float* sb, const void* bias, int act, void* C, long long ldc) {
  if (!ctx || !A || !B || !C || !sa || !sb) return ECOSPA_ERR_NULL;
  const bool gated = act == ECOSPA_ACT_SWIGLU;
  if (act < ECOSPA_ACT_NONE || act > ECOSPA_ACT_SWIGLU) return ECOSPA_ERR_DTYPE;
  // 131071 products of two -128 are the most that a 32-bit sum is sure to hold; tiles are addressed by 32-bit offsets
  if (M < 1 || N < 8 || K < 16 || K > 131056 || lda < K || ldb < K || ldc < (gated ? N / 2 : N) || lda >= 1 << 24 || ldb >= 1 << 24 || ldc >= 1 << 23) return ECOSPA_ERR_SHAPE;
  if (K % 16 || N % (gated ? 16 : 8) || lda % 16 || ldb % 16 || ldc % 8 || !aligned16(A) || !aligned16(B) || !aligned16(C) || !aligned16(sb) || (reinterpret_cast<uintptr_t>(sa) & 3u) ||
      (bias && !aligned16(bias))) return ECOSPA_ERR_ALIGN;
  GemmDesc d;
  memset(&d, 0, sizeof(d));
  d.M = M; d.N = N; d.K = K / 2;
  d.A = A; d.lda = lda / 2; d.B = B; d.ldb = ldb / 2;
  d.epi.h = sa; d.epi.rope_cos = sb; d.epi.bias = bias; d.epi.act = act;
  d.epi.kind = gated ? EPI_SWIGLU : (act == ECOSPA_ACT_NONE ? EPI_STORE : EPI_ACT);
  if (gated) { d.epi.c2 = C; d.epi.ldc2 = ldc; }
  else { d.epi.c = C; d.epi.ldc = ldc; }
  return ecospa_gemm_i8(ctx, d);
}
