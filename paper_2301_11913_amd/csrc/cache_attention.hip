// Attention of new tokens over the paged int8 cache.
//
// One wavefront per (row, query head), 64 cached tokens at a time: a lane makes one token's score, then owns d_head / 64 elements of
// the output.  One pass with the running maximum and sum of the softmax.
#include "cache.h"

namespace swarm {
namespace {

struct AttnArgs {
  CacheArgs c;
  const void* q;
  void* out;
  const uint64_t* tree;
  size_t q_pitch, out_pitch;
  bool s16;
};

template <typename T, int DH>
__global__ __launch_bounds__(64) void cache_attention_kernel(AttnArgs a) {
  __shared__ float qs[DH];
  __shared__ float ps[64];
  __shared__ int pages[64];
  const int lane = threadIdx.x, h = blockIdx.x % a.c.H, row = blockIdx.x / a.c.H;
  const int b = row / a.c.tokens, t = row - b * a.c.tokens, g = h / (a.c.H / a.c.KV);
  const Span s = span_of(a.c, b);
  if (t >= s.fresh) return;
  for (int d = lane; d < DH; d += 64) qs[d] = Elem<T>::load((const T*)a.q + (size_t)row * a.q_pitch + (size_t)h * DH + d);
  __syncthreads();
  const uint64_t tree = a.tree ? a.tree[row] : 0;
  const float c = (DH == 64 ? 0.125f : 0.08838834764831845f) * 1.4426950408889634f;
  const int n = s.past + s.fresh, P1 = (1 << a.c.page_shift) - 1;
  float m = -INFINITY, l = 0.f, o[DH / 64] = {};
  for (int j0 = 0; j0 < n; j0 += 64) {
    const int j = j0 + lane, u = j - s.past;
    const int page = j < n ? page_of(a.c, b, j) : -1;
    const bool sees = page >= 0 && (u < 0 || (a.tree ? (tree >> u) & 1 : u <= t));
    float x = -INFINITY;
    if (sees) {
      const int8_t* k = a.c.k_codes + codes_at<DH>(a.c, page, g) + (size_t)(j & P1) * DH;
      x = 0.f;
      for (int blk = 0; blk < DH / 64; ++blk) {
        float dot = 0.f;
        for (int d = 0; d < 64; ++d) dot = fmaf((float)k[blk * 64 + d], qs[blk * 64 + d], dot);
        x = fmaf(dot, block_scale_load(a.c.k_scales, scales_at<DH>(a.c, page, g) + ((size_t)blk << a.c.page_shift) + (j & P1), a.s16), x);
      }
      x *= c;
    }
    const float mn = fmaxf(m, wave_max(x)), top = mn == -INFINITY ? 0.f : mn;
    const float keep = exp2f(m - top), p = exp2f(x - top);
    l = l * keep + wave_sum(p);
    m = mn;
    __syncthreads();
    ps[lane] = sees ? p : 0.f;
    pages[lane] = sees ? page : -1;
    __syncthreads();
    for (int blk = 0; blk < DH / 64; ++blk) {
      float acc = o[blk] * keep;
      for (int e = 0; e < 64; ++e) {
        const int pg = pages[e], place = (j0 + e) & P1;
        if (pg < 0) continue;
        const float v = (float)a.c.v_codes[codes_at<DH>(a.c, pg, g) + ((size_t)(blk * 64 + lane) << a.c.page_shift) + place];
        acc = fmaf(ps[e] * v, block_scale_load(a.c.v_scales, scales_at<DH>(a.c, pg, g) + ((size_t)blk << a.c.page_shift) + place, a.s16), acc);
      }
      o[blk] = acc;
    }
  }
  for (int blk = 0; blk < DH / 64; ++blk)
    Elem<T>::store((T*)a.out + (size_t)row * a.out_pitch + (size_t)h * DH + blk * 64 + lane, l == 0.f ? 0.f : o[blk] / l);
}

}  // namespace

size_t cache_attention_scratch_bytes(const swarm_cache_config*, int, int) { return 0; }

swarm_status cache_attention_launch(const swarm_cache_config* c, const CacheArgs& args, int, const void* q, size_t q_pitch,
                                    const uint64_t* tree, void* out, size_t out_pitch, void*, hipStream_t st) {
  const AttnArgs a{args, q, out, tree, q_pitch, out_pitch, c->scale_bits == 16};
  const long long blocks = (long long)c->batch * args.tokens * c->n_heads;
  if (blocks > 0x7FFFFFFF) return SWARM_ERR_SHAPE;
  const dim3 grid((unsigned)blocks), block(64);
  if (c->dtype == SWARM_BF16) {
    if (c->d_head == 64) hipLaunchKernelGGL((cache_attention_kernel<bf16_raw, 64>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((cache_attention_kernel<bf16_raw, 128>), grid, block, 0, st, a);
  } else {
    if (c->d_head == 64) hipLaunchKernelGGL((cache_attention_kernel<float, 64>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((cache_attention_kernel<float, 128>), grid, block, 0, st, a);
  }
  return launch_status();
}

}  // namespace swarm

using namespace swarm;

extern "C" size_t swarm_cache_attention_workspace_bytes(const swarm_cache_config* cfg, int32_t tokens, int32_t max_len) {
  if (cache_config_status(cfg, tokens) != SWARM_OK || max_len < 0) return 0;
  return cache_attention_scratch_bytes(cfg, tokens, max_len);
}

extern "C" swarm_status swarm_cache_attention(const swarm_cache_config* cfg, const swarm_cache* cache, const int32_t* page_table,
                                              const int32_t* past, const int32_t* fresh, int32_t tokens, int32_t max_len,
                                              const void* q, size_t q_pitch, const uint64_t* tree, void* out, size_t out_pitch,
                                              void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!cfg || !cache_pointers_ok(cache) || !page_table || !past || !q || !out) return SWARM_ERR_NULL;
  const swarm_status bad = cache_config_status(cfg, tokens);
  if (bad != SWARM_OK) return bad;
  const size_t width = (size_t)cfg->n_heads * cfg->d_head;
  if (max_len < 0 || (tree && tokens > 64) || q == out || !cache_aligned(cache) || !pitch_ok(q, q_pitch, width, cfg->dtype) ||
      !pitch_ok(out, out_pitch, width, cfg->dtype) || ((uintptr_t)tree & 7) || ((uintptr_t)workspace & 255))
    return SWARM_ERR_SHAPE;
  const size_t need = cache_attention_scratch_bytes(cfg, tokens, max_len);
  if (need && !workspace) return SWARM_ERR_NULL;
  if (need > workspace_bytes) return SWARM_ERR_WORKSPACE;
  return cache_attention_launch(cfg, cache_args(cfg, cache, page_table, past, fresh, tokens), max_len, q, q_pitch, tree, out,
                                out_pitch, workspace, (hipStream_t)hip_stream);
}
