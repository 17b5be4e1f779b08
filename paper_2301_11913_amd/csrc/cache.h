// What the kernels of the key / value cache share: the pool's layout, the sequences' lengths, argument checks.
#pragma once
#include "kernels.h"
#include "swarm_cache.h"

namespace swarm {

// A cache and the new tokens of a call as a kernel takes them.
struct CacheArgs {
  int8_t *k_codes, *v_codes;
  void *k_scales, *v_scales;
  const int32_t* table;
  const int32_t *past, *fresh;   // fresh == nullptr: `tokens` of every sequence
  int H, KV, page_shift, n_pages, B, table_pages, tokens;
};

struct Span {
  int past, fresh;
};
// Lengths of sequence b; out of range: nothing new, and nothing before it either.
__device__ __forceinline__ Span span_of(const CacheArgs& a, int b) {
  Span s{a.past[b], a.fresh ? a.fresh[b] : a.tokens};
  const bool ok = s.past >= 0 && s.fresh >= 0 && s.fresh <= a.tokens &&
                  (long long)s.past + s.fresh <= ((long long)a.table_pages << a.page_shift);
  return ok ? s : Span{0, 0};
}
// Page of token j (within the table) of sequence b, -1 where it is out of range.
__device__ __forceinline__ int page_of(const CacheArgs& a, int b, int j) {
  const int p = a.table[(size_t)b * a.table_pages + (j >> a.page_shift)];
  return (unsigned)p < (unsigned)a.n_pages ? p : -1;
}
// Start of a page's codes (keys or values) and scales of head g, in elements.
template <int DH>
__device__ __forceinline__ size_t codes_at(const CacheArgs& a, int page, int g) {
  return (((size_t)page * a.KV + g) << a.page_shift) * DH;
}
template <int DH>
__device__ __forceinline__ size_t scales_at(const CacheArgs& a, int page, int g) {
  return (((size_t)page * a.KV + g) << a.page_shift) * (DH / 64);
}

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
// Values rounded to bf16 by the unit's own conversion, which leaves what is no number one whatever its bits.
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

__device__ __forceinline__ void store_rounded(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_rounded(bf16_raw* p, float v) { *p = __builtin_bit_cast(bf16_raw, (__bf16)v); }

// 8 consecutive elements <-> fp32
template <typename T> struct Row8;
template <> struct Row8<bf16_raw> {
  static __device__ __forceinline__ void load(const bf16_raw* p, float (&x)[8]) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ void store(bf16_raw* p, const float (&x)[8]) {
    uint4 v;
    v.x = pack2(x[0], x[1]); v.y = pack2(x[2], x[3]); v.z = pack2(x[4], x[5]); v.w = pack2(x[6], x[7]);
    *reinterpret_cast<uint4*>(p) = v;
  }
};
template <> struct Row8<float> {
  static __device__ __forceinline__ void load(const float* p, float (&x)[8]) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
  static __device__ __forceinline__ void store(float* p, const float (&x)[8]) {
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
  }
};

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
// Whether rows of `width` elements, `pitch` apart, hold together and start on 16 bytes.
inline bool pitch_ok(const void* p, size_t pitch, size_t width, int dtype) {
  return aligned16(p) && pitch >= width && pitch <= ((size_t)1 << 24) && (pitch * (dtype == SWARM_BF16 ? 2 : 4)) % 16 == 0;
}

// The checks that every call begins with.  SWARM_OK, or what to return.
inline swarm_status cache_config_status(const swarm_cache_config* c, int tokens) {
  if (!c) return SWARM_ERR_NULL;
  if (c->dtype != SWARM_F32 && c->dtype != SWARM_BF16) return SWARM_ERR_DTYPE;
  if (c->n_kv_heads < 1 || c->n_heads < 1 || c->n_heads > 1024 || c->n_heads % c->n_kv_heads) return SWARM_ERR_SHAPE;
  if (c->d_head != 64 && c->d_head != 128) return SWARM_ERR_SHAPE;
  if (c->page_tokens < 16 || c->page_tokens > 65536 || (c->page_tokens & (c->page_tokens - 1))) return SWARM_ERR_SHAPE;
  if (c->n_pages < 1 || c->batch < 1 || c->table_pages < 1) return SWARM_ERR_SHAPE;
  if ((long long)c->table_pages * c->page_tokens > (1ll << 30)) return SWARM_ERR_SHAPE;
  if (c->scale_bits != 32 && c->scale_bits != 16) return SWARM_ERR_SHAPE;
  if (tokens < 1 || (long long)c->batch * tokens > (1ll << 24)) return SWARM_ERR_SHAPE;
  return SWARM_OK;
}
inline bool cache_pointers_ok(const swarm_cache* c) { return c && c->k_codes && c->v_codes && c->k_scales && c->v_scales; }
inline bool cache_aligned(const swarm_cache* c) {
  return aligned16(c->k_codes) && aligned16(c->v_codes) && aligned16(c->k_scales) && aligned16(c->v_scales);
}
inline CacheArgs cache_args(const swarm_cache_config* c, const swarm_cache* k, const int32_t* table, const int32_t* past,
                            const int32_t* fresh, int tokens) {
  return CacheArgs{k->k_codes, k->v_codes, k->k_scales, k->v_scales, table, past, fresh, c->n_heads, c->n_kv_heads,
                   __builtin_ctz((unsigned)c->page_tokens), c->n_pages, c->batch, c->table_pages, tokens};
}

// rows of one key / value head (tokens x query heads of it) that a kernel counts in 32 bits
inline bool cache_attention_shape_ok(const swarm_cache_config* c, int tokens) {
  return (long long)tokens * (c->n_heads / c->n_kv_heads) <= (1ll << 24);
}
// Attention over a cache (checked arguments); `scratch` holds cache_attention_scratch_bytes of it.
size_t cache_attention_scratch_bytes(const swarm_cache_config* c, int tokens, int max_len);
swarm_status cache_attention_launch(const swarm_cache_config* c, const CacheArgs& a, int max_len, const void* q, size_t q_pitch,
                                    const uint64_t* tree, void* out, size_t out_pitch, void* scratch, hipStream_t st);
swarm_status cache_append_launch(const swarm_cache_config* c, const CacheArgs& a, const void* q, const void* k, const void* v,
                                 size_t pitch, const int32_t* positions, bool rotary, void* q_out, size_t q_out_pitch,
                                 hipStream_t st);

}  // namespace swarm
