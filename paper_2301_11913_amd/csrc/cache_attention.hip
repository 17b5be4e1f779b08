// Attention of new tokens over the paged int8 cache, for few rows per key / value head and for fp32: products of whole numbers.
//
// The cache's codes go to the matrix cores as they are.  q is a block's power of two times a whole number of 30 bits, and that is a sum of 4
// signed bytes times 256^i: four rows of an int8 MFMA (v_mfma_i32_16x16x64_i8, whose 64 steps of the contraction are exactly one block
// of the codec) hold one query's bytes, a tile of 16 rows four queries.  The products and their sums are exact; a block's sum is put together
// from its bytes' sums in fp32 and multiplied by q's power of two and the keys' scales.
// The weights p_j = 2^(s_j - m) go the same way: p_j times the value's scale, as a whole number of 30 bits relative to the largest that the
// query has among the 64 tokens, contracted with their value codes.  Where the tokens' scales lie further apart than 2^5, what those 30 bits
// leave of a weight goes through a second time (60 bits of the largest): a value's elements are not all large, and where its code is 0 the
// others' are all there is.  Nothing is converted per cached element, and one query uses the matrix cores no worse than four.
//   keys    column n of tile c is token 4 n + c: a lane then holds the weights of four consecutive tokens, one word per byte row.
//   values  lie transposed in the cache: a lane's operand is 16 consecutive tokens of one element, one load.
// What a wavefront reads goes straight into registers, the next 64 tokens' keys while this tile's softmax runs, the next values behind its
// last product.  Bound by reading the cache while a key / value head has few rows: 17 KB per 64 tokens at d_head 128 against
// 506 vector instructions for four rows (32 sequences of up to 8192 tokens, 32 heads of 128: 1.26 GB in 215 us, 5.9 TB/s; the vector
// units are busy for 30 % of that).  The four wavefronts of a workgroup take tiles in turn; long sequences are spread over
// workgroups (splits of `chunk` tiles), whose partial sums a second kernel joins.
#include "cache_attention.h"

namespace swarm {
namespace {

typedef __attribute__((ext_vector_type(4))) int i32x4;

constexpr int kThreads = 256, kWaves = 4;
constexpr int kTile = kAttnTile;
constexpr int kRowPitch = 20;          // 32-bit words of a row of weights' bytes: 16, and 4 against bank conflicts
constexpr int kBits = 30;
constexpr int kSpread = 5;             // exponents of the scales that one pass does for
constexpr float kLog2e = 1.4426950408889634f;

// Reductions over the 16 lanes of a row of the register file
template <int N>
__device__ __forceinline__ uint32_t turned(uint32_t v) { return __builtin_amdgcn_mov_dpp(v, 0x120 + N, 0xF, 0xF, true); }
__device__ __forceinline__ float max16(float v) {
  v = fmaxf(v, __uint_as_float(turned<8>(__float_as_uint(v))));
  v = fmaxf(v, __uint_as_float(turned<4>(__float_as_uint(v))));
  v = fmaxf(v, __uint_as_float(turned<2>(__float_as_uint(v))));
  return fmaxf(v, __uint_as_float(turned<1>(__float_as_uint(v))));
}
__device__ __forceinline__ uint32_t umax16(uint32_t v) {
  v = max(v, turned<8>(v)); v = max(v, turned<4>(v)); v = max(v, turned<2>(v));
  return max(v, turned<1>(v));
}
__device__ __forceinline__ uint32_t umin16(uint32_t v) { return ~umax16(~v); }
__device__ __forceinline__ float sum16(float v) {
  v += __uint_as_float(turned<8>(__float_as_uint(v))); v += __uint_as_float(turned<4>(__float_as_uint(v)));
  v += __uint_as_float(turned<2>(__float_as_uint(v)));
  return v + __uint_as_float(turned<1>(__float_as_uint(v)));
}

// A number below 2^kBits in magnitude as bytes: sum of (signed byte i) * 256^i.
__device__ __forceinline__ uint32_t digits(int x) { return ((uint32_t)x + 0x80808080u) ^ 0x80808080u; }
// and back, from the sums over the bytes
__device__ __forceinline__ float joined(const i32x4& a) {
  return fmaf((float)((a[3] << 8) + a[2]), 65536.0f, (float)((a[1] << 8) + a[0]));
}

template <bool S16>
__device__ __forceinline__ float4 scales4(const void* p, size_t i) {
  if constexpr (S16) {
    const uint2 v = *reinterpret_cast<const uint2*>(reinterpret_cast<const uint16_t*>(p) + i);
    return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xFFFF0000u), __uint_as_float(v.y << 16),
                       __uint_as_float(v.y & 0xFFFF0000u));
  } else {
    return *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p) + i);
  }
}

// RT tiles of four rows; a row is (token t, query head of the group): r = t * group + head.
template <typename T, int DH, int RT, bool S16>
__global__ __launch_bounds__(kThreads) void cache_attention_bytes_kernel(AttnArgs a) {
  constexpr int NB = DH / 64, Q = 4 * RT, DT = DH / 16;
  constexpr int kQBytes = Q * 4 * DH, kOBytes = kWaves * Q * (DH + 2) * 4, kPBytes = kWaves * NB * 16 * kRowPitch * 4;
  __shared__ __attribute__((aligned(16))) char lds[kQBytes + kPBytes > kOBytes ? kQBytes + kPBytes : kOBytes];
  __shared__ float q_scale[Q][NB];
  const int lane = threadIdx.x & 63, n = lane & 15, lg = lane >> 4;
  // Said to be the same for all lanes, which makes the loop over tiles a scalar one.  Without it the compiler (ROCm 7.2) masks the loop by
  // lanes and has been seen to give the registers of the values' scales to their maximum (v_max_u32 v9, v8, v9) with the scales still to be
  // read (v_ldexp_f32 v6, v9, v6), of source that reads one array twice and writes it nowhere between.
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int unit = blockIdx.x;
  const int split = unit % a.splits; unit /= a.splits;
  const int g = unit % a.c.KV; unit /= a.c.KV;
  const int rg = unit % a.row_groups, b = unit / a.row_groups;
  const Span s = span_of(a.c, b);
  const int r0 = rg * Q, rows = s.fresh * a.group;
  if (r0 >= rows) return;
  const int t_last = min(r0 + Q, rows) - 1;
  const int len = a.tree ? s.past + s.fresh : s.past + t_last / a.group + 1;     // tokens that any of these rows sees
  const int tiles = (len + kTile - 1) / kTile;
  const int first = split * a.chunk, end = split + 1 == a.splits ? tiles : min(tiles, first + a.chunk);

  // ---- the queries' bytes: 16 lanes make one block of one row
  {
    uint8_t* qd = reinterpret_cast<uint8_t*>(lds);
    for (int i = threadIdx.x; i < Q * NB * 16; i += kThreads) {
      const int e = i & 15, blk = (i >> 4) % NB, q = (i >> 4) / NB, r = r0 + q;
      float x[4] = {0.f, 0.f, 0.f, 0.f};
      if (r < rows) {
        const T* src = reinterpret_cast<const T*>(a.q) + ((size_t)b * a.c.tokens + r / a.group) * a.q_pitch +
                       (size_t)(g * a.group + r % a.group) * DH + blk * 64 + e * 4;
#pragma unroll
        for (int u = 0; u < 4; ++u) x[u] = Elem<T>::load(src + u);
      }
      uint32_t top = 0;                 // magnitudes compare as whole numbers, what is no number above all
#pragma unroll
      for (int u = 0; u < 4; ++u) top = max(top, __float_as_uint(x[u]) & 0x7FFFFFFFu);
      top = umax16(top);
      const int ex = (int)(top >> 23) - 126;                  // magnitudes are below 2^ex
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const uint32_t w = digits((int)rintf(ldexpf(x[u], kBits - ex)));
#pragma unroll
        for (int k = 0; k < 4; ++k) qd[(q * 4 + k) * DH + blk * 64 + e * 4 + u] = (uint8_t)(w >> (8 * k));
      }
      const float c = (DH == 64 ? 0.125f : 0.08838834764831845f) * kLog2e;
      if (e == 0) q_scale[q][blk] = top >= 0x7F800000u ? __uint_as_float(0x7FC00000u) : ldexpf(c, ex - kBits);
    }
  }
  __syncthreads();
  i32x4 qf[RT][NB];
  float qs[RT][NB];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int blk = 0; blk < NB; ++blk) {
      qf[rt][blk] = *reinterpret_cast<const i32x4*>(lds + (rt * 16 + n) * DH + blk * 64 + lg * 16);
      qs[rt][blk] = q_scale[rt * 4 + lg][blk];
    }
  uint32_t* weights = reinterpret_cast<uint32_t*>(lds + kQBytes) + wave * NB * 16 * kRowPitch;

  float m[RT], l[RT], o[RT][DT];
  uint64_t see[RT];
  int my_t[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    m[rt] = -INFINITY; l[rt] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[rt][d] = 0.f;
    const int r = r0 + rt * 4 + lg;
    my_t[rt] = r < rows ? r / a.group : 0;
    see[rt] = a.tree && r < rows ? a.tree[(size_t)b * a.c.tokens + my_t[rt]] : 0;
  }

  const int P1 = (1 << a.c.page_shift) - 1;
  const int last_k = (len - 1) & ~3, last_v = (len - 1) & ~15;
  // pages of the tokens that this lane loads of a tile: keys 4 n .. 4 n + 3, values 16 lg .. 16 lg + 15; past the end the last ones
  auto page_k = [&](int tile) { return page_of(a.c, b, min(tile * kTile + 4 * n, last_k)); };
  auto page_v = [&](int tile) { return page_of(a.c, b, min(tile * kTile + 16 * lg, last_v)); };
  uint4 kf[4][NB], vf[DT];
  float4 ks[NB], vs[NB];
  auto load_keys = [&](int tile, int page) {
    const int place = min(tile * kTile + 4 * n, last_k) & P1;
    const int8_t* base = a.c.k_codes + codes_at<DH>(a.c, max(page, 0), g) + (size_t)place * DH + lg * 16;
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int blk = 0; blk < NB; ++blk) kf[c][blk] = *reinterpret_cast<const uint4*>(base + c * DH + blk * 64);
    const size_t at = scales_at<DH>(a.c, max(page, 0), g) + place;
#pragma unroll
    for (int blk = 0; blk < NB; ++blk) ks[blk] = scales4<S16>(a.c.k_scales, at + ((size_t)blk << a.c.page_shift));
  };
  auto load_values = [&](int tile, int page, int k_page) {
    const int place = min(tile * kTile + 16 * lg, last_v) & P1;
    const int8_t* base = a.c.v_codes + codes_at<DH>(a.c, max(page, 0), g) + ((size_t)n << a.c.page_shift) + place;
#pragma unroll
    for (int d = 0; d < DT; ++d) vf[d] = *reinterpret_cast<const uint4*>(base + ((size_t)d << (a.c.page_shift + 4)));
    const size_t at = scales_at<DH>(a.c, max(k_page, 0), g) + (min(tile * kTile + 4 * n, last_k) & P1);
#pragma unroll
    for (int blk = 0; blk < NB; ++blk) vs[blk] = scales4<S16>(a.c.v_scales, at + ((size_t)blk << a.c.page_shift));
  };

  int tile = first + wave;
  int pk = -1, pk_next = -1, pv_next = -1;
  if (tile < end) {
    pk = page_k(tile);
    const int pv = page_v(tile);
    load_keys(tile, pk);
    load_values(tile, pv, pk);
    if (tile + kWaves < end) { pk_next = page_k(tile + kWaves); pv_next = page_v(tile + kWaves); }
  }
  for (; tile < end; tile += kWaves) {
    const bool more = tile + kWaves < end;
    // ---- scores
    float p[RT][4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) p[rt][c] = 0.f;
#pragma unroll
      for (int blk = 0; blk < NB; ++blk) {
        const float k = c == 0 ? ks[blk].x : c == 1 ? ks[blk].y : c == 2 ? ks[blk].z : ks[blk].w;
        const i32x4 kv = __builtin_bit_cast(i32x4, kf[c][blk]);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          const i32x4 acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(qf[rt][blk], kv, i32x4{0, 0, 0, 0}, 0, 0, 0);
          p[rt][c] = fmaf(joined(acc), k * qs[rt][blk], p[rt][c]);
        }
      }
    }
    const int pk_now = pk;
    if (more) {
      pk = pk_next;
      load_keys(tile + kWaves, pk);
    }
    // ---- which of them count; the values' scales of what does not may be anything
    const int j0 = tile * kTile;
    const bool inner = j0 + kTile <= s.past && __ballot(pk_now < 0) == 0;
    float vn[NB][4];
#pragma unroll
    for (int blk = 0; blk < NB; ++blk) { vn[blk][0] = vs[blk].x; vn[blk][1] = vs[blk].y; vn[blk][2] = vs[blk].z; vn[blk][3] = vs[blk].w; }
    if (!inner) {
      bool any[4] = {false, false, false, false};
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int j = j0 + 4 * n + c, u = j - s.past;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          const bool sees = pk_now >= 0 && (u < 0 || (u < s.fresh && (a.tree ? (see[rt] >> u) & 1 : u <= my_t[rt])));
          if (!sees) p[rt][c] = -INFINITY;
          any[c] |= sees;
        }
        // a token that this lane's rows do not see may be seen by the other lane groups' rows
        any[c] |= __shfl_xor((int)any[c], 16, 64) != 0;
        any[c] |= __shfl_xor((int)any[c], 32, 64) != 0;
#pragma unroll
        for (int blk = 0; blk < NB; ++blk) vn[blk][c] = any[c] ? vn[blk][c] : 0.f;
      }
    }
    // ---- whether the values' scales lie apart
    bool apart = false;
#pragma unroll
    for (int blk = 0; blk < NB; ++blk) {
      uint32_t sc[4];                  // magnitudes compare as whole numbers; what is no number comes out on top
#pragma unroll
      for (int c = 0; c < 4; ++c) sc[c] = __float_as_uint(vn[blk][c]) & 0x7FFFFFFFu;
      uint32_t top = umax16(max(max(sc[0], sc[1]), max(sc[2], sc[3])));
      if (__ballot(top >= 0x7F800000u)) {      // an infinite value or none: for its block of the rows that see it, and no others
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          uint32_t hit = 0;
#pragma unroll
          for (int c = 0; c < 4; ++c) hit |= sc[c] >= 0x7F800000u && p[rt][c] != -INFINITY;
          hit = umax16(hit);
#pragma unroll
          for (int d = 4 * blk; d < 4 * blk + 4; ++d) o[rt][d] = hit ? __uint_as_float(0x7FC00000u) : o[rt][d];
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          if (sc[c] < 0x7F800000u) continue;
          vn[blk][c] = 0.f;
          sc[c] = 0;
        }
        top = umax16(max(max(sc[0], sc[1]), max(sc[2], sc[3])));
      }
      const uint32_t least = umin16(min(min(sc[0] - 1, sc[1] - 1), min(sc[2] - 1, sc[3] - 1))) + 1;      // of those that are not 0
      apart |= top != 0 && (top >> 23) >= (least >> 23) + kSpread;
    }
    const bool again = __ballot(apart) != 0;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      // ---- softmax of this tile
      const float mn = max16(fmaxf(fmaxf(m[rt], fmaxf(p[rt][0], p[rt][1])), fmaxf(p[rt][2], p[rt][3])));
      const float top = mn == -INFINITY ? 0.f : mn;
      const float keep = __builtin_amdgcn_exp2f(m[rt] - top);
      m[rt] = mn;
      l[rt] *= keep;
      float w[NB][4];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const float x = __builtin_amdgcn_exp2f(p[rt][c] - top);
        l[rt] += x;
#pragma unroll
        for (int blk = 0; blk < NB; ++blk) w[blk][c] = x * vn[blk][c];
      }
      float kept = keep;
#pragma nounroll
      for (int pass = 0;; ++pass) {
        float back[NB];
#pragma unroll
        for (int blk = 0; blk < NB; ++blk) {
          const float most = max16(fmaxf(fmaxf(fabsf(w[blk][0]), fabsf(w[blk][1])), fmaxf(fabsf(w[blk][2]), fabsf(w[blk][3]))));
          const int ex = max(__builtin_amdgcn_frexp_expf(most), -110);      // all are below 2^ex; the way back, 2^(ex - kBits), is a number
          back[blk] = ldexpf(1.0f, ex - kBits);
          uint32_t d[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const float r = rintf(ldexpf(w[blk][c], kBits - ex));
            d[c] = digits((int)r);
            w[blk][c] -= r * back[blk];                                     // exact
          }
          // byte i of four tokens to a word of row 4 q + i
          const uint32_t a0 = __builtin_amdgcn_perm(d[1], d[0], 0x05010400u), a1 = __builtin_amdgcn_perm(d[3], d[2], 0x05010400u);
          const uint32_t b0 = __builtin_amdgcn_perm(d[1], d[0], 0x07030602u), b1 = __builtin_amdgcn_perm(d[3], d[2], 0x07030602u);
          uint32_t* to = weights + blk * 16 * kRowPitch + lg * 4 * kRowPitch + n;
          to[0] = __builtin_amdgcn_perm(a1, a0, 0x05040100u);
          to[kRowPitch] = __builtin_amdgcn_perm(a1, a0, 0x07060302u);
          to[2 * kRowPitch] = __builtin_amdgcn_perm(b1, b0, 0x05040100u);
          to[3 * kRowPitch] = __builtin_amdgcn_perm(b1, b0, 0x07060302u);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        i32x4 pf[NB];
#pragma unroll
        for (int blk = 0; blk < NB; ++blk)
          pf[blk] = *reinterpret_cast<const i32x4*>(weights + blk * 16 * kRowPitch + n * kRowPitch + lg * 4);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const i32x4 acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(pf[d / 4], __builtin_bit_cast(i32x4, vf[d]), i32x4{0, 0, 0, 0}, 0, 0, 0);
          o[rt][d] = fmaf(o[rt][d], kept, joined(acc) * back[d / 4]);
        }
        if (__builtin_expect(!again || pass, 1)) break;
        kept = 1.0f;
      }
    }
    if (more) {
      load_values(tile + kWaves, pv_next, pk);
      if (tile + 2 * kWaves < end) { pk_next = page_k(tile + 2 * kWaves); pv_next = page_v(tile + 2 * kWaves); }
    }
  }

  // ---- the wavefronts' results, one after the other in a fixed order
  __syncthreads();
  float* ow = reinterpret_cast<float*>(lds);                  // [wave][row][d_head]
  float* ml = ow + kWaves * Q * DH;                           // [wave][row][2]
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const float total = sum16(l[rt]);
    const int q = wave * Q + rt * 4 + lg;
    if (n == 0) { ml[2 * q] = m[rt]; ml[2 * q + 1] = total; }
#pragma unroll
    for (int d = 0; d < DT; ++d) ow[q * DH + d * 16 + n] = o[rt][d];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < Q * DH; i += kThreads) {
    const int q = i / DH, d = i - q * DH, r = r0 + q;
    if (r >= rows) continue;
    float mw[kWaves], top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) { mw[w] = ml[2 * (w * Q + q)]; top = fmaxf(top, mw[w]); }
    const float ref = top == -INFINITY ? 0.f : top;
    float total = 0.f, x = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(mw[w] - ref);
      total = fmaf(ml[2 * (w * Q + q) + 1], f, total);
      x = fmaf(ow[(w * Q + q) * DH + d], f, x);
    }
    if (a.splits == 1) {
      store_rounded(reinterpret_cast<T*>(a.out) + ((size_t)b * a.c.tokens + r / a.group) * a.out_pitch +
                    (size_t)(g * a.group + r % a.group) * DH + d, total == 0.f ? 0.f : x / total);
    } else {
      const size_t at = (size_t)blockIdx.x * Q + q;
      a.part_o[at * DH + d] = x;
      if (d == 0) { a.part_ml[2 * at] = top; a.part_ml[2 * at + 1] = total; }
    }
  }
}

// The splits of a row and head joined.  d_head / 4 threads hold a row's elements; `slices` of them (a power of two, no more than
// there are splits) share a row, each takes every slices-th split, and the slices are added up in order.  Many splits: one row per
// workgroup; two: as many as fit.
template <typename T, int DH>
__global__ __launch_bounds__(kThreads) void cache_attention_join_kernel(AttnArgs a, int Q, int slices) {
  constexpr int LANES = DH / 4, SLICES = kThreads / LANES;
  __shared__ float4 sums[SLICES][LANES];
  __shared__ float tops[SLICES], totals[SLICES];
  const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES, slice = slot & (slices - 1), per = SLICES / slices;
  const long long unit = (long long)blockIdx.x * per + slot / slices;          // (row, head)
  const int h = (int)(unit % a.c.H);
  const long long row = unit / a.c.H;
  const int b = (int)(row / a.c.tokens), t = (int)(row - (long long)b * a.c.tokens), g = h / a.group;
  const bool real = b < a.c.B && t < span_of(a.c, min(b, a.c.B - 1)).fresh;
  const int r = t * a.group + h - g * a.group, rg = r / Q;
  const size_t at = (((size_t)b * a.row_groups + rg) * a.c.KV + g) * a.splits * Q + (r - rg * Q);
  float top = -INFINITY;
  if (real)
    for (int p = slice + lane * slices; p < a.splits; p += LANES * slices) top = fmaxf(top, a.part_ml[2 * (at + (size_t)p * Q)]);
#pragma unroll
  for (int d = LANES / 2; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
  if (lane == 0) tops[slot] = top;
  __syncthreads();
  for (int i = 0; i < slices; ++i) top = fmaxf(top, tops[slot - slice + i]);
  const float ref = top == -INFINITY ? 0.f : top;
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  float total = 0.f;
  if (real) {
#pragma unroll 4
    for (int p = slice; p < a.splits; p += slices) {
      const size_t k = at + (size_t)p * Q;
      const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + 2 * k);
      const float4 o = *reinterpret_cast<const float4*>(a.part_o + k * DH + lane * 4);
      const float f = __builtin_amdgcn_exp2f(ml.x - ref);
      total = fmaf(ml.y, f, total);
      x.x = fmaf(o.x, f, x.x); x.y = fmaf(o.y, f, x.y); x.z = fmaf(o.z, f, x.z); x.w = fmaf(o.w, f, x.w);
    }
  }
  sums[slot][lane] = x;
  if (lane == 0) totals[slot] = total;
  __syncthreads();
  if (slice || !real) return;
  for (int i = 1; i < slices; ++i) {
    const float4 y = sums[slot + i][lane];
    x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
    total += totals[slot + i];
  }
  T* to = reinterpret_cast<T*>(a.out) + (size_t)row * a.out_pitch + (size_t)h * DH + lane * 4;
  const float f = total == 0.f ? 0.f : 1.0f / total;
  const float y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) store_rounded(to + i, total == 0.f ? 0.f : y[i] * f);
}

// How the rows and the tokens of a call are cut.
struct Cut {
  bool many;           // the kernel of many rows
  int row_tiles;       // tiles of four rows per workgroup (of 32 where there are many)
  int rows;            // rows of a workgroup
  int row_groups, splits, chunk;
};
Cut cut_of(const swarm_cache_config* c, int tokens, int max_len) {
  Cut k{};
  const int rows = tokens * (c->n_heads / c->n_kv_heads);
  // bf16, 8 sequences of 4000 tokens, 32 heads, with 4 / 5 / 8 / 9 / 16 / 32 rows each: the kernel of bytes 58 / 77 / 78 / 105 / 107 / 174 us
  // at d_head 128 and 32 / 36 / 36 / 45 / 46 / 70 at 64, the kernel of many rows 76 / 72 / 72 / 73 / 76 / 78 and 40 / 40 / 41 / 41 / 41 / 43
  k.many = c->dtype == SWARM_BF16 && rows > (c->d_head == 64 ? 8 : 4);
  if (k.many) {
    k.row_tiles = rows <= 64 ? 2 : 4;
    k.rows = 32 * k.row_tiles;
  } else {
    // fp32, the same with 16 heads and 9 / 32 rows: 8 rows at a time 28 / 42 us at d_head 64 and 69 / 109 at 128, 16 rows 27 / 41 and 63 / 100;
    // a call with 9 rows over 4 x 500 tokens, 4 heads of 64, 10.3 and 10.9
    k.row_tiles = rows <= 4 ? 1 : rows <= 8 || c->d_head == 64 ? 2 : 4;
    k.rows = 4 * k.row_tiles;
  }
  k.row_groups = (rows + k.rows - 1) / k.rows;
  const long long cap = (long long)c->table_pages * c->page_tokens;
  const long long len = max_len > 0 ? std::min<long long>(max_len, cap) : cap;
  const long long tiles = (len + kTile - 1) / kTile, whole = (long long)c->batch * c->n_kv_heads * k.row_groups;
  // As many workgroups as are resident, each of four tiles at least (one for every wavefront): 512, with many rows of d_head 64 768.
  // 32 sequences of up to 8192 tokens / one of 131072 with 8 heads: 215 / 59 us; with 256 215 / 61, 1024 215 / 62, 2048 252 / 72, 4096 281 / 90.
  // Trees of 33 over 2011 tokens / 32 rows over 8 x 4000, d_head 128: 49 / 78 us; with 256 60 / 109, 768 54 / 90, 1024 55 / 86.
  // 32 rows over 8 x 4000 tokens at d_head 64: 43 us; with 256 70, 512 50, 1024 53.
  const long long target = k.many && c->d_head == 64 ? 768 : 512;
  const long long chunk = std::max(4ll, std::min<long long>(1ll << 24, (whole * tiles + target - 1) / target));
  k.splits = (int)std::max(1ll, (tiles + chunk - 1) / chunk);
  k.chunk = (int)chunk;
  return k;
}
size_t partial_rows(const swarm_cache_config* c, const Cut& k) {
  return (size_t)c->batch * c->n_kv_heads * k.row_groups * k.splits * k.rows;
}

}  // namespace

size_t cache_attention_scratch_bytes(const swarm_cache_config* c, int tokens, int max_len) {
  const Cut k = cut_of(c, tokens, max_len);
  return k.splits == 1 ? 0 : (partial_rows(c, k) * (c->d_head + 2) * 4 + 255) & ~(size_t)255;
}

namespace {
template <typename T, int DH, int RT>
void launch_bytes(const AttnArgs& a, unsigned blocks, hipStream_t st) {
  if (a.s16) hipLaunchKernelGGL((cache_attention_bytes_kernel<T, DH, RT, true>), dim3(blocks), dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL((cache_attention_bytes_kernel<T, DH, RT, false>), dim3(blocks), dim3(kThreads), 0, st, a);
}
template <typename T, int DH>
swarm_status launch(const AttnArgs& a, const Cut& k, hipStream_t st) {
  const long long blocks = (long long)a.c.B * a.c.KV * k.row_groups * k.splits, joins = (long long)a.c.B * a.c.tokens * a.c.H;
  if (blocks > 0x7FFFFFFF || (k.splits > 1 && joins > 0x7FFFFFFF)) return SWARM_ERR_SHAPE;
  if (k.many) {
    const swarm_status st1 = cache_attention_rows_launch(a, DH, k.row_tiles, st);
    if (st1 != SWARM_OK) return st1;
  } else if (k.row_tiles == 1) {
    launch_bytes<T, DH, 1>(a, (unsigned)blocks, st);
  } else {
    if constexpr (sizeof(T) == 4 || DH == 64)
      if (k.row_tiles == 2) launch_bytes<T, DH, 2>(a, (unsigned)blocks, st);
    if constexpr (sizeof(T) == 4 && DH == 128)
      if (k.row_tiles == 4) launch_bytes<T, DH, 4>(a, (unsigned)blocks, st);
  }
  if (k.splits > 1) {
    int slices = 1024 / DH;
    while (slices > 1 && slices > k.splits) slices >>= 1;
    const int per = 1024 / DH / slices;
    hipLaunchKernelGGL((cache_attention_join_kernel<T, DH>), dim3((unsigned)((joins + per - 1) / per)), dim3(kThreads), 0, st, a, k.rows, slices);
  }
  return launch_status();
}
}  // namespace

swarm_status cache_attention_launch(const swarm_cache_config* c, const CacheArgs& args, int max_len, const void* q, size_t q_pitch,
                                    const uint64_t* tree, void* out, size_t out_pitch, void* scratch, hipStream_t st) {
  const Cut k = cut_of(c, args.tokens, max_len);
  AttnArgs a{args, q, out, tree, q_pitch, out_pitch, nullptr, nullptr, c->n_heads / c->n_kv_heads, k.row_groups, k.splits, k.chunk,
             c->scale_bits == 16};
  if (k.splits > 1) {
    a.part_o = (float*)scratch;
    a.part_ml = a.part_o + partial_rows(c, k) * c->d_head;
  }
  if (c->dtype == SWARM_BF16) return c->d_head == 64 ? launch<bf16_raw, 64>(a, k, st) : launch<bf16_raw, 128>(a, k, st);
  return c->d_head == 64 ? launch<float, 64>(a, k, st) : launch<float, 128>(a, k, st);
}

}  // namespace swarm

using namespace swarm;

extern "C" size_t swarm_cache_attention_workspace_bytes(const swarm_cache_config* cfg, int32_t tokens, int32_t max_len) {
  if (cache_config_status(cfg, tokens) != SWARM_OK || max_len < 0 || !cache_attention_shape_ok(cfg, tokens)) return 0;
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
  if (max_len < 0 || !cache_attention_shape_ok(cfg, tokens) || (tree && tokens > 64) || q == out || !cache_aligned(cache) || !pitch_ok(q, q_pitch, width, cfg->dtype) ||
      !pitch_ok(out, out_pitch, width, cfg->dtype) || ((uintptr_t)tree & 7) || ((uintptr_t)workspace & 255))
    return SWARM_ERR_SHAPE;
  const size_t need = cache_attention_scratch_bytes(cfg, tokens, max_len);
  if (need && !workspace) return SWARM_ERR_NULL;
  if (need > workspace_bytes) return SWARM_ERR_WORKSPACE;
  return cache_attention_launch(cfg, cache_args(cfg, cache, page_table, past, fresh, tokens), max_len, q, q_pitch, tree, out,
                                out_pitch, workspace, (hipStream_t)hip_stream);
}
