// Attention of many new tokens over the paged int8 cache, bf16: drafted trees, prompts.
//
// The codes are whole numbers of 8 bits, which bf16 holds exactly: a tile of 64 tokens is read once per workgroup, turned into bf16 on
// the way into LDS (one conversion per code, one byte permutation per two) and contracted with the queries on v_mfma_f32_16x16x32_bf16.  The
// scales never touch the codes: a score is the sum over the blocks of 64 elements of (products) * (key's scale), and the weight of a
// value is p_j times its scale, so the only roundings beyond fp32 are those of the weights to bf16.
//   scores  S^T [token][query] = K Q^T: a lane owns one query column, so maximum and sum need no more than two exchanges between lanes;
//           row 4 a + i of key tile (h, u) is token 32 h + 8 a + 4 u + i, which leaves a lane eight consecutive tokens' weights:
//   output  O^T [element][query] = V^T P^T takes them as its operand without an exchange, and the transposed values of the cache are
//           V^T as it lies.
// The running maximum is raised only when a score passes it by 2^8.  LDS holds two stages; chunks of 16 bytes are XOR-swizzled so that a
// fragment's 16 rows fall on different banks.
#include "cache_attention.h"

namespace swarm {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;

constexpr int kThreads = 256, kWaves = 4;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
// four codes as bf16: whole numbers of 8 bits, so the upper half of their fp32 form is all there is
__device__ __forceinline__ uint2 codes4(uint32_t w) {
  const uint32_t a = __float_as_uint((float)(int8_t)w), b = __float_as_uint((float)(int8_t)(w >> 8));
  const uint32_t c = __float_as_uint((float)(int8_t)(w >> 16)), d = __float_as_uint((float)(int8_t)(w >> 24));
  return make_uint2(__builtin_amdgcn_perm(b, a, 0x07060302u), __builtin_amdgcn_perm(d, c, 0x07060302u));
}

template <int DH> struct Tiles {
  static constexpr int NB = DH / 64;
  static constexpr int KCH = DH / 8;                       // 16-byte chunks of a key row
  static constexpr int PIECES = 64 * DH / 16 / kThreads;   // pieces of 16 codes per thread, of keys and of values
  struct Stage {
    uint4 k[64 * KCH];
    uint4 v[DH * 8];
    float ks[NB][64], vs[NB][64];                          // keys' with the factor of the scores in them
  };
  static __device__ __forceinline__ int k_at(int key, int chunk) {
    if constexpr (DH == 128) return key * KCH + (chunk ^ (((key >> 1) & 12) | (key & 3)));
    return key * KCH + (chunk ^ (((key >> 1) & 4) | (key & 3)));
  }
  static __device__ __forceinline__ int v_at(int d, int chunk) { return d * 8 + (chunk ^ (d & 7)); }
};

template <int DH, int NQ, bool S16>
__global__ __launch_bounds__(kThreads, 2) void cache_attention_rows_kernel(AttnArgs a) {
  using T = Tiles<DH>;
  constexpr int NB = T::NB, DT = DH / 16, KK = DH / 32, Q = kWaves * 16 * NQ;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  typename T::Stage* stage = reinterpret_cast<typename T::Stage*>(lds);
  const int lane = threadIdx.x & 63, n = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // workgroups go to the 8 XCDs in turn: all units of a sequence and head to one, which keeps its tiles in that XCD's L2; the last
  // rows, which see the most, first
  const int per_pair = a.row_groups * a.splits, x = blockIdx.x >> 3;
  const int pair = x / per_pair * 8 + (blockIdx.x & 7);
  if (pair >= a.c.B * a.c.KV) return;
  const int which = x % per_pair, rg = a.row_groups - 1 - which / a.splits, split = which % a.splits;
  const int b = pair / a.c.KV, g = pair - b * a.c.KV;
  const Span s = span_of(a.c, b);
  const int r0 = rg * Q, rows = s.fresh * a.group;
  if (r0 >= rows) return;
  const int len = a.tree ? s.past + s.fresh : s.past + (min(r0 + Q, rows) - 1) / a.group + 1;
  const int tiles = (len + kAttnTile - 1) / kAttnTile;
  const int first = split * a.chunk, end = split + 1 == a.splits ? tiles : min(tiles, first + a.chunk);

  // ---- this wavefront's queries, and up to where each sees
  bf16x8 qf[NQ][KK];
  uint64_t among[NQ];                    // which of the new tokens (tree)
  int limit[NQ];                         // tokens below it are seen (the past; without a tree the row's own too)
  const int w0 = r0 + wave * 16 * NQ;
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    const int r = w0 + q * 16 + n;
    const bool real = r < rows;
    const int t = real ? r / a.group : 0, h = real ? r - t * a.group : 0;
    const bf16_raw* src = reinterpret_cast<const bf16_raw*>(a.q) + ((size_t)b * a.c.tokens + t) * a.q_pitch + (size_t)(g * a.group + h) * DH;
#pragma unroll
    for (int k = 0; k < KK; ++k) {
      const uint4 v = real ? *reinterpret_cast<const uint4*>(src + k * 32 + lg * 8) : make_uint4(0, 0, 0, 0);
      qf[q][k] = __builtin_bit_cast(bf16x8, v);
    }
    among[q] = 0;
    if (a.tree && real) among[q] = a.tree[(size_t)b * a.c.tokens + t] & (s.fresh >= 64 ? ~0ull : (1ull << s.fresh) - 1);
    limit[q] = a.tree ? s.past : s.past + t + 1;
  }
  // tiles below `inner` are seen whole by all rows; without a tree, tiles from `outer` on by none of this wavefront's
  const int inner = a.tree ? s.past : s.past + min(w0, rows - 1) / a.group + 1;
  const int outer = w0 >= rows ? 0 : a.tree ? len : s.past + (min(w0 + 16 * NQ, rows) - 1) / a.group + 1;

  f32x4 o[NQ][DT];
  float m[NQ], l[NQ];
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    m[q] = -INFINITY; l[q] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[q][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // ---- staging: pages of a tile's four times 16 tokens (scalar), codes and scales in registers, then bf16 in LDS
  const int P1 = (1 << a.c.page_shift) - 1, last16 = (len - 1) & ~15;
  const int32_t* table = a.c.table + (size_t)b * a.c.table_pages;
  struct Pages { int p[4]; };
  auto pages_of = [&](int tile) {
    Pages r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = table[min(tile * kAttnTile + 16 * i, last16) >> a.c.page_shift];
      r.p[i] = (unsigned)p < (unsigned)a.c.n_pages ? p : -1;
    }
    return r;
  };
  auto valid_of = [&](int tile, const Pages& pg) {
    const int left = len - tile * kAttnTile;
    uint64_t v = left >= 64 ? ~0ull : (1ull << left) - 1;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (pg.p[i] < 0) v &= ~(0xFFFFull << (16 * i));
    return v;
  };
  auto pick = [&](const Pages& pg, int i) { return i == 0 ? pg.p[0] : i == 1 ? pg.p[1] : i == 2 ? pg.p[2] : pg.p[3]; };
  uint4 kc[T::PIECES], vc[T::PIECES];
  float sc = 0.f;
  constexpr int KP = DH / 16;                                // pieces of a key row
  auto load = [&](int tile, const Pages& pg) {
    const int j0 = tile * kAttnTile;
#pragma unroll
    for (int i = 0; i < T::PIECES; ++i) {
      const int idx = threadIdx.x + i * kThreads, key = idx / KP, piece = idx % KP;
      const int place = min(j0 + key, last16 + 15) & P1;
      kc[i] = *reinterpret_cast<const uint4*>(a.c.k_codes + codes_at<DH>(a.c, max(pick(pg, key >> 4), 0), g) + (size_t)place * DH + piece * 16);
    }
#pragma unroll
    for (int i = 0; i < T::PIECES; ++i) {
      const int idx = threadIdx.x + i * kThreads, d = idx >> 2, piece = idx & 3;
      const int place = min(j0 + piece * 16, last16) & P1;
      vc[i] = *reinterpret_cast<const uint4*>(a.c.v_codes + codes_at<DH>(a.c, max(pick(pg, piece), 0), g) + ((size_t)d << a.c.page_shift) + place);
    }
    if (threadIdx.x < 2 * NB * 64) {
      const int key = threadIdx.x & 63, blk = (threadIdx.x >> 6) % NB;
      const int page = pick(pg, key >> 4), place = min(j0 + key, last16 + 15) & P1;
      const size_t at = scales_at<DH>(a.c, max(page, 0), g) + ((size_t)blk << a.c.page_shift) + place;
      sc = block_scale_load(threadIdx.x < NB * 64 ? a.c.k_scales : a.c.v_scales, at, S16);
    }
  };
  const float factor = (DH == 64 ? 0.125f : 0.08838834764831845f) * kLog2e;
  auto store = [&](typename T::Stage& st) {
#pragma unroll
    for (int i = 0; i < T::PIECES; ++i) {
      const int idx = threadIdx.x + i * kThreads, key = idx / KP, piece = idx % KP;
      const uint2 w0 = codes4(kc[i].x), w1 = codes4(kc[i].y), w2 = codes4(kc[i].z), w3 = codes4(kc[i].w);
      st.k[T::k_at(key, 2 * piece)] = make_uint4(w0.x, w0.y, w1.x, w1.y);
      st.k[T::k_at(key, 2 * piece + 1)] = make_uint4(w2.x, w2.y, w3.x, w3.y);
    }
#pragma unroll
    for (int i = 0; i < T::PIECES; ++i) {
      const int idx = threadIdx.x + i * kThreads, d = idx >> 2, piece = idx & 3;
      const uint2 w0 = codes4(vc[i].x), w1 = codes4(vc[i].y), w2 = codes4(vc[i].z), w3 = codes4(vc[i].w);
      st.v[T::v_at(d, 2 * piece)] = make_uint4(w0.x, w0.y, w1.x, w1.y);
      st.v[T::v_at(d, 2 * piece + 1)] = make_uint4(w2.x, w2.y, w3.x, w3.y);
    }
    if (threadIdx.x < 2 * NB * 64) {
      const int key = threadIdx.x & 63, blk = (threadIdx.x >> 6) % NB;
      if (threadIdx.x < NB * 64) st.ks[blk][key] = sc * factor;
      else st.vs[blk][key] = sc;
    }
  };

  if (first < end) {
    Pages pg = pages_of(first);
    uint64_t valid = valid_of(first, pg);
    load(first, pg);
    store(stage[0]);
    if (first + 1 < end) pg = pages_of(first + 1);
    __syncthreads();
    for (int tile = first; tile < end; ++tile) {
      const bool more = tile + 1 < end;
      uint64_t valid_next = 0;
      if (more) {
        load(tile + 1, pg);
        valid_next = valid_of(tile + 1, pg);
        if (tile + 2 < end) pg = pages_of(tile + 2);
      }
      const int j0 = tile * kAttnTile;
      if (j0 < outer) {
        const typename T::Stage& st = stage[(tile - first) & 1];
        // ---- scores
        float p[NQ][16];
#pragma unroll
        for (int hu = 0; hu < 4; ++hu) {
          const int h = hu >> 1, u = hu & 1, key = 32 * h + 8 * (n >> 2) + 4 * u + (n & 3);
          f32x4 acc[NQ][NB];
#pragma unroll
          for (int q = 0; q < NQ; ++q)
#pragma unroll
            for (int blk = 0; blk < NB; ++blk) acc[q][blk] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = 0; k < KK; ++k) {
            const bf16x8 kf = __builtin_bit_cast(bf16x8, st.k[T::k_at(key, k * 4 + lg)]);
#pragma unroll
            for (int q = 0; q < NQ; ++q) acc[q][k / 2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[q][k], acc[q][k / 2], 0, 0, 0);
          }
          float4 ks[NB];
#pragma unroll
          for (int blk = 0; blk < NB; ++blk) ks[blk] = *reinterpret_cast<const float4*>(&st.ks[blk][32 * h + 8 * lg + 4 * u]);
#pragma unroll
          for (int q = 0; q < NQ; ++q) {
            float* to = p[q] + h * 8 + u * 4;
            to[0] = acc[q][0][0] * ks[0].x; to[1] = acc[q][0][1] * ks[0].y; to[2] = acc[q][0][2] * ks[0].z; to[3] = acc[q][0][3] * ks[0].w;
            if constexpr (NB == 2) {
              to[0] = fmaf(acc[q][1][0], ks[1].x, to[0]); to[1] = fmaf(acc[q][1][1], ks[1].y, to[1]);
              to[2] = fmaf(acc[q][1][2], ks[1].z, to[2]); to[3] = fmaf(acc[q][1][3], ks[1].w, to[3]);
            }
          }
        }
        const bool whole = valid == ~0ull && j0 + kAttnTile <= inner;
        uint64_t sees[NQ];
#pragma unroll
        for (int q = 0; q < NQ; ++q) sees[q] = ~0ull;
        if (!whole) {
#pragma unroll
          for (int q = 0; q < NQ; ++q) {
            const int below = limit[q] - j0;
            uint64_t v = below >= 64 ? ~0ull : below <= 0 ? 0ull : (1ull << below) - 1;
            const int shift = j0 - s.past;                       // of the first new token's bit
            if (shift > -64 && shift < 64) v |= shift >= 0 ? among[q] >> shift : among[q] << -shift;
            sees[q] = v & valid;
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (!((sees[q] >> (32 * (e >> 3) + 8 * lg + (e & 7))) & 1)) p[q][e] = -INFINITY;
          }
        }
        // ---- softmax
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          float top = p[q][0];
#pragma unroll
          for (int e = 1; e < 16; ++e) top = fmaxf(top, p[q][e]);
          if (__ballot(top > m[q] + 8.0f)) {
            top = fmaxf(top, __shfl_xor(top, 16, 64));
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float mn = fmaxf(m[q], top);
            const float keep = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[q] - mn);
            m[q] = mn;
            l[q] *= keep;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[q][d] *= keep;
          }
          const float ref = m[q] == -INFINITY ? 0.f : m[q];
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            p[q][e] = __builtin_amdgcn_exp2f(p[q][e] - ref);
            l[q] += p[q][e];
          }
        }
        // ---- output
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          bf16x8 pf[NQ][NB];
#pragma unroll
          for (int blk = 0; blk < NB; ++blk) {
            const float4 s0 = *reinterpret_cast<const float4*>(&st.vs[blk][32 * h + 8 * lg]);
            const float4 s1 = *reinterpret_cast<const float4*>(&st.vs[blk][32 * h + 8 * lg + 4]);
            const float vs[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll
            for (int q = 0; q < NQ; ++q) {
              float w[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) w[e] = p[q][h * 8 + e] * vs[e];
              if (!whole) {                                      // a scale that is no number, of a token that is not seen
#pragma unroll
                for (int e = 0; e < 8; ++e)
                  if (!((sees[q] >> (32 * h + 8 * lg + e)) & 1)) w[e] = 0.f;
              }
              pf[q][blk] = __builtin_bit_cast(bf16x8, make_uint4(pack2(w[0], w[1]), pack2(w[2], w[3]), pack2(w[4], w[5]), pack2(w[6], w[7])));
            }
          }
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            const bf16x8 vf = __builtin_bit_cast(bf16x8, st.v[T::v_at(d * 16 + n, h * 4 + lg)]);
#pragma unroll
            for (int q = 0; q < NQ; ++q) o[q][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[q][d / 4], o[q][d], 0, 0, 0);
          }
        }
      }
      if (more) store(stage[(tile + 1 - first) & 1]);
      valid = valid_next;
      __syncthreads();
    }
  }

#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    float total = l[q];
    total += __shfl_xor(total, 16, 64);
    total += __shfl_xor(total, 32, 64);
    const int r = w0 + q * 16 + n;
    if (r >= rows) continue;
    if (a.splits == 1) {
      const int t = r / a.group, h = r - t * a.group;
      bf16_raw* to = reinterpret_cast<bf16_raw*>(a.out) + ((size_t)b * a.c.tokens + t) * a.out_pitch + (size_t)(g * a.group + h) * DH + 4 * lg;
      const float f = total == 0.f ? 0.f : 1.0f / total;
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const f32x4 y = o[q][d];
        *reinterpret_cast<uint2*>(to + d * 16) =
            total == 0.f ? make_uint2(0, 0) : make_uint2(pack2(y[0] * f, y[1] * f), pack2(y[2] * f, y[3] * f));
      }
    } else {
      const size_t at = ((((size_t)b * a.row_groups + rg) * a.c.KV + g) * a.splits + split) * Q + (r - r0);
#pragma unroll
      for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4*>(a.part_o + at * DH + d * 16 + 4 * lg) = o[q][d];
      if (lg == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * at) = make_float2(m[q], total);
    }
  }
}

template <int DH, int NQ, bool S16>
swarm_status launch(const AttnArgs& a, hipStream_t st) {
  static LdsOptIn opted;
  constexpr size_t bytes = 2 * sizeof(typename Tiles<DH>::Stage);
  const swarm_status ok = lds_opt_in(reinterpret_cast<const void*>(&cache_attention_rows_kernel<DH, NQ, S16>), bytes, opted);
  if (ok != SWARM_OK) return ok;
  const long long pairs = ((long long)a.c.B * a.c.KV + 7) / 8 * 8, blocks = pairs * a.row_groups * a.splits;
  if (blocks > 0x7FFFFFFF) return SWARM_ERR_SHAPE;
  hipLaunchKernelGGL((cache_attention_rows_kernel<DH, NQ, S16>), dim3((unsigned)blocks), dim3(kThreads), bytes, st, a);
  return launch_status();
}

}  // namespace

swarm_status cache_attention_rows_launch(const AttnArgs& a, int dh, int tiles, hipStream_t st) {
  if (dh == 64) {
    if (tiles == 1) return a.s16 ? launch<64, 1, true>(a, st) : launch<64, 1, false>(a, st);
    return a.s16 ? launch<64, 2, true>(a, st) : launch<64, 2, false>(a, st);
  }
  if (tiles == 1) return a.s16 ? launch<128, 1, true>(a, st) : launch<128, 1, false>(a, st);
  return a.s16 ? launch<128, 2, true>(a, st) : launch<128, 2, false>(a, st);
}

}  // namespace swarm
