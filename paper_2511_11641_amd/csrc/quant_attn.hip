// Attention over caches of 8-bit floats: how a call is cut into items, the join of a row's pieces, the entry points.  The items: quant_attn.h.
#include "quant_cache.h"

// One wavefront a query: its pieces, in their order, and what came in from other keys.
__global__ __launch_bounds__(256) void quant_attn_join_kernel(const QuantAttnArgs a, int rows_of_block, int pitch) {
  const long long id = static_cast<long long>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (id >= static_cast<long long>(a.B) * a.h_kv * a.rows) return;
  const int group = static_cast<int>(id / a.rows), row = static_cast<int>(id - static_cast<long long>(group) * a.rows);
  const int b = group / a.h_kv, hk = group - b * a.h_kv, rb = row / rows_of_block, rl = row - rb * rows_of_block;
  const float* const part = a.part + (static_cast<long long>(group) * a.row_blocks + rb) * a.pieces * (static_cast<long long>(rows_of_block) * pitch) + rl * pitch;
  const long long next = static_cast<long long>(rows_of_block) * pitch;
  float top = -INFINITY;
  for (int i = lane; i < a.pieces; i += 64) top = fmaxf(top, part[i * next + pitch - 2]);
  top = wave_max(top);
  const float ref = top == -INFINITY ? 0.f : top;
  float all = 0.f, v0 = 0.f, v1 = 0.f;
  const int d0 = min(lane, a.kv - 1), d1 = min(lane + 64, a.kv - 1);
  // a lane a piece for its factor, then eight pieces' values on their way together
  for (int i0 = 0; i0 < a.pieces; i0 += 64) {
    const int i = i0 + lane;
    const float l = i < a.pieces ? part[i * next + pitch - 1] : 0.f, f = l == 0.f ? 0.f : __builtin_amdgcn_exp2f(part[i * next + pitch - 2] - ref);
    all += wave_sum(l == 0.f ? 0.f : l * f);
    const int here = min(a.pieces - i0, 64);
    for (int j0 = 0; j0 < here; j0 += 8) {
      float x0[8], x1[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float* const p = part + (i0 + min(j0 + j, here - 1)) * next;
        x0[j] = p[d0];
        x1[j] = a.kv > 64 ? p[d1] : 0.f;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float fj = __shfl(f, min(j0 + j, 63), 64);
        const bool on = j0 + j < here && fj != 0.f;      // a piece without keys has no values (NaN factors are kept)
        v0 += on ? x0[j] * fj : 0.f;
        v1 += on ? x1[j] * fj : 0.f;
      }
    }
  }
  const int tok = row / a.g, head = hk * a.g + row - tok * a.g;
  const long long flat = (static_cast<long long>(b) * a.h + head) * a.L + tok, orow = static_cast<long long>(b) * a.L + tok;
  float mm = top, in = 0.f, own = 1.f;
  if (a.lse_in) {
    const float p = a.lse_in[flat] * 1.4426950408889634f;
    if (p != -INFINITY) {
      mm = fmaxf(top, p);
      const float r = mm == -INFINITY ? 0.f : mm;
      in = __builtin_amdgcn_exp2f(p - r);
      own = all == 0.f ? 0.f : __builtin_amdgcn_exp2f(ref - r);
      all = all == 0.f ? in : all * own + in;
    }
  }
  const float inv = all == 0.f ? 0.f : 1.f / all;
  if (a.lse && lane == 0) a.lse[flat] = all == 0.f ? -INFINITY : (mm == -INFINITY ? 0.f : mm) * 0.6931471805599453f + logf(all);
  for (int u = 0; u < 2; ++u) {
    const int d = lane + 64 * u;
    if (d >= a.kv) break;
    float y = (u ? v1 : v0) * own;
    if (in != 0.f) y += in * bf16_to_f32(a.o_in[orow * a.ld_oi + head * a.kv + d]);
    a.o[orow * a.ld_o + head * a.kv + d] = f32_to_bf16(y * inv);
  }
}

// Tiles of 16 queries a wavefront takes, and how many pieces the keys of a head are cut into.  More tiles read and convert a key less often, fewer make more
// workgroups: as many as the rows fill while there are 512 workgroups, two a compute unit (us, heads of 64 dims, four queries' heads a key's: 64 requests of 16384
// keys and 16 tokens, 4 : 1 tiles 192 : 251; 16 requests of 4096 and 8 tokens, 2 : 1 tiles 20.8 : 17.8.  Less than 512, here 256, costs 16 requests of 16 tokens
// 26.5 : 21.2, more, 1024, 64 requests of 5 tokens 174 : 152).  Where one tile each leaves room, keys are cut, into a piece for each 512 that a request may hold (256: the
// same; 1024: one request of 4096 keys 12.4 : 11.0), which a request's own keys then share in whole 128s; 1024 keys in one piece, which needs no join (one request of 1000 keys
// 7.8 : 10.8, of 2048 11.8 : 10.4).
#define QA_ITEMS 512
struct QuantPlan { int T, row_blocks, pieces, W; };
static QuantPlan quant_plan(const ecospa_quant_cache* c, int L) {
  QuantPlan p;
  const int rows = c->h / c->h_kv * L;
  p.W = c->kp_vo <= 32 ? 2 : (c->kp_vo <= 64 ? 4 : 8);
  const long long groups = static_cast<long long>(c->B) * c->h_kv;
  const int widest = quant_attn_tiles((c->kp_qk + 31) / 32, p.W);
  p.T = rows <= 16 ? 1 : (rows <= 32 || widest == 2 ? 2 : 4);
  while (p.T > 1 && groups * ((rows + 16 * p.T - 1) / (16 * p.T)) < QA_ITEMS) p.T /= 2;
  p.row_blocks = (rows + 16 * p.T - 1) / (16 * p.T);
  const long long items = groups * p.row_blocks;
  const int most = c->own_max <= 1024 ? 1 : (c->own_max + 511) / 512;
  long long want = items >= QA_ITEMS ? 1 : (QA_ITEMS + items - 1) / items;
  if (want > most) want = most;
  if (want < 1) want = 1;
  p.pieces = static_cast<int>(want);
  return p;
}
static size_t quant_part_bytes(const ecospa_quant_cache* c, const QuantPlan& p) {
  if (p.pieces <= 1) return 0;
  return static_cast<size_t>(c->B) * c->h_kv * p.row_blocks * p.pieces * (16 * p.T) * (16 * p.W + 2) * sizeof(float);
}
static bool quant_call_ok(const ecospa_quant_cache* c, int L) { return L >= 1 && static_cast<long long>(c->B) * L * c->h <= (1ll << 30); }

extern "C" size_t ecospa_quant_cache_attn_workspace_bytes(const ecospa_quant_cache* c, int L) {
  if (ecospa_quant_cache_check(c) != ECOSPA_OK || !quant_call_ok(c, L)) return 0;
  return align_up(quant_part_bytes(c, quant_plan(c, L)), 256);
}
extern "C" int ecospa_quant_cache_attn(ecospa_ctx* ctx, const ecospa_quant_cache* c, int L, const void* q, long long ld_q, const void* o_in, long long ld_oi,
                                       const float* lse_in, void* o, long long ld_o, float* lse) {
  if (!ctx || !q || !o || !o_in != !lse_in) return ECOSPA_ERR_NULL;
  const int rc = ecospa_quant_cache_check(c);
  if (rc != ECOSPA_OK) return rc;
  const int nq = c->h * c->kp_qk, no = c->h * c->kp_vo;
  if (!quant_call_ok(c, L) || ld_q < nq || ld_o < no || (o_in && ld_oi < no)) return ECOSPA_ERR_SHAPE;
  if (!aligned16(q) || !aligned16(o) || !aligned16(o_in) || ld_q % 8 || ld_o % 8 || (o_in && ld_oi % 8) || (reinterpret_cast<uintptr_t>(lse) & 3u) ||
      (reinterpret_cast<uintptr_t>(lse_in) & 3u))
    return ECOSPA_ERR_ALIGN;
  const QuantPlan p = quant_plan(c, L);
  QuantAttnArgs a;
  memset(&a, 0, sizeof(a));
  if (p.pieces > 1) {
    WsCarver ws(ctx->ws, ctx->ws_bytes);
    a.part = static_cast<float*>(ws.take(quant_part_bytes(c, p)));
    if (!ws.ok()) return ECOSPA_ERR_WORKSPACE;
  }
  a.q = static_cast<const bf16_t*>(q); a.o = static_cast<bf16_t*>(o); a.lse = lse; a.o_in = static_cast<const bf16_t*>(o_in); a.lse_in = lse_in;
  a.k = static_cast<const unsigned char*>(c->k); a.v = static_cast<const unsigned char*>(c->v); a.k_scale = c->k_scale; a.v_scale = c->v_scale; a.lens = c->lens;
  a.ld_q = ld_q; a.ld_o = ld_o; a.ld_oi = ld_oi; a.k_sb = c->k_sb; a.k_sh = c->k_sh; a.k_st = c->k_st; a.v_sb = c->v_sb; a.v_sh = c->v_sh; a.v_st = c->v_st;
  a.B = c->B; a.L = L; a.h = c->h; a.h_kv = c->h_kv; a.g = c->h / c->h_kv; a.rows = a.g * L; a.kq = c->kp_qk; a.kv = c->kp_vo; a.own_max = c->own_max;
  a.block_log2 = 31 - __builtin_clz(static_cast<unsigned>(c->block));
  a.blocks = (c->cap + c->block - 1) / c->block;
  a.row_blocks = p.row_blocks; a.pieces = p.pieces;
  a.scale_log2 = c->scale * 1.4426950408889634f;
  if (static_cast<long long>((c->B * c->h_kv + 7) / 8 * 8) * p.row_blocks * p.pieces * 256 >= 1ll << 32) return ECOSPA_ERR_SHAPE;      // a launch takes no more work-items
  const int KQ = (c->kp_qk + 31) / 32;
  // keys that one workgroup reads, and more of them than the last-level cache (256 MB) keeps until a next call: past the caches (64 requests of 16384 keys 132 : 138 us,
  // 5.4 : 5.2 TB/s; out of the cache 134 MB 26 : 20)
  const bool once = p.row_blocks == 1 && static_cast<long long>(c->B) * c->h_kv * c->own_max * (c->kp_qk + c->kp_vo) > 256ll << 20;
  const hipError_t e = p.W == 2 ? quant_attn_launch_w2(a, p.T, KQ, once, ctx->stream) : p.W == 4 ? quant_attn_launch_w4(a, p.T, KQ, once, ctx->stream) : quant_attn_launch_w8(a, p.T, KQ, once, ctx->stream);
  if (e != hipSuccess) return hip_fail(ctx, e, "quant_attn_kernel");
  if (p.pieces > 1) {
    const long long rows = static_cast<long long>(c->B) * c->h_kv * a.rows;
    hipLaunchKernelGGL(quant_attn_join_kernel, dim3(static_cast<unsigned>((rows + 3) / 4)), dim3(256), 0, ctx->stream, a, 16 * p.T, 16 * p.W + 2);
    ECOSPA_CHECK_LAUNCH(ctx, "quant_attn_join_kernel");
  }
  return ECOSPA_OK;
}
