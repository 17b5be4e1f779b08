// Attention of many new tokens over the paged int8 cache, bf16: drafted trees, prompts.
//
// The codes are whole numbers of 8 bits, which bf16 and fp16 hold exactly: a tile of 64 tokens is read once per workgroup, and on the way
// into LDS the keys turn into bf16, as the queries are, and the values into fp16.  The products are v_mfma_f32_32x32x16.  The scales never
// touch the codes: a score is the sum over the blocks of 64 elements of (products) * (key's scale), and the weight of a value is p_j times
// its scale, so the only roundings beyond fp32 are those of the weights.  These are held in fp16 (a rounding of 2^-11, where bf16's 2^-8 would
// be as large as the output's own) relative to a power of two, which is the unit of the query's sums as well.  The unit puts a tile's scales
// between 2^-3 and 2^7, the largest from 4 on, so a weight has an error of half an fp16 step or, if that is more, of 2^-27 of what it would
// be with p_j = 1 and the largest scale (2^-22 of that with its own scale, where that is the smallest possible).  The unit follows the tiles
// up and down, up no further than a query's own weights ask for.  A tile whose scales other than 0 lie further apart than 2^10 is gone
// through once for each range of 2^10 that a block has tokens in.  So a value that a row does not see, or sees with next to no weight,
// costs the others none of their digits.
// 4 prompts of 2048 tokens, 32 heads of 128, on one state after the other: 273 us, with scales times a random 2^+-3 274, 2^+-12 1950.
//   scores  S^T [token][query] = K Q^T, 32 tokens x 32 queries: a lane owns one query column, so a maximum or a sum needs one exchange
//           between lanes; row 8 a + 4 b + i of the keys' operand is token 16 (a / 2) + 8 b + 4 (a % 2) + i, which leaves a lane eight
//           consecutive tokens' weights twice:
//   output  O^T [element][query] = V^T P^T takes them as its operand without an exchange, and the transposed values of the cache are
//           V^T as it lies.
// RW wavefronts of a workgroup take 32 rows each; with KW = 2 two wavefronts share rows and take 32 of a tile's 64 tokens each
// (few rows, where the tile's conversion and the wait for it would outweigh them), joined at the end.
// 4 prompts of 2048 tokens, 32 heads of 128: 224 to 238 us, 578 to 615 TFLOP/s; 461 vector instructions per wavefront and tile keep the
// vector units busy for 54 % of that, the products the matrix cores for 27 %, and two wavefronts per SIMD (240 registers) overlap little of
// the two.
// The running maximum is raised only when a score passes it by 2^8.  LDS holds two stages; 16-byte chunks are XOR-swizzled so that the 16
// rows of a fragment that are read together fall on different banks.
#include "cache_attention.h"

namespace swarm {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kNoExp = -100000;        // no unit yet
constexpr int kRange = 10;             // exponents of the scales that go together: 2^-3 to 2^7 units
constexpr int kLeast = 124;            // the biased exponent of a scale of 2^-3 units, less the unit's exponent
// How far below its largest weight the unit of a query's sums may be.  A weight is below 2^15 units (2^8 by the running maximum, 2^7 by the
// scale), a code is below 2^7 and there are up to 2^30 tokens, so sums are numbers down to a unit of 2^-72 of that weight's.
constexpr int kFall = 72;
// 4 prompts of 2048 tokens, 32 heads of 128, on one state after the other: 265 us; 4 pairs at a time 263, 2 286, one 298, all 16 of an XCD 262
constexpr int kPairs = 8;

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
__device__ __forceinline__ uint32_t pack2_f16(float a, float b) {
  f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
}
// four codes as fp16: 0x6400 + u is 1024 + u for a byte u, here the code + 128
__device__ __forceinline__ uint2 codes4_f16(uint32_t w) {
  const f16x2 back = {(_Float16)-1152.0f, (_Float16)-1152.0f};
  w ^= 0x80808080u;
  const f16x2 a = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u)) + back;
  const f16x2 b = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u)) + back;
  return make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b));
}
// the largest of a wavefront's values (not negative, as whole numbers), the same for all lanes
template <int N>
__device__ __forceinline__ uint32_t turned(uint32_t v) { return __builtin_amdgcn_mov_dpp(v, 0x120 + N, 0xF, 0xF, true); }
__device__ __forceinline__ uint32_t wave_umax(uint32_t v) {
  v = max(v, turned<8>(v)); v = max(v, turned<4>(v)); v = max(v, turned<2>(v)); v = max(v, turned<1>(v));
  return max(max((uint32_t)__builtin_amdgcn_readlane(v, 0), (uint32_t)__builtin_amdgcn_readlane(v, 16)),
             max((uint32_t)__builtin_amdgcn_readlane(v, 32), (uint32_t)__builtin_amdgcn_readlane(v, 48)));
}
__device__ __forceinline__ uint32_t wave_umin(uint32_t v) { return ~wave_umax(~v); }
// four codes as bf16: whole numbers of 8 bits, so the upper half of their fp32 form is all there is
__device__ __forceinline__ uint2 codes4(uint32_t w) {
  const uint32_t a = __float_as_uint((float)(int8_t)w), b = __float_as_uint((float)(int8_t)(w >> 8));
  const uint32_t c = __float_as_uint((float)(int8_t)(w >> 16)), d = __float_as_uint((float)(int8_t)(w >> 24));
  return make_uint2(__builtin_amdgcn_perm(b, a, 0x07060302u), __builtin_amdgcn_perm(d, c, 0x07060302u));
}

template <int DH> struct Stage {
  static constexpr int NB = DH / 64, CH = DH / 8;          // 16-byte chunks of a key row
  uint4 k[64 * CH];
  uint4 v[DH * 8];
  float ks[NB][64], vs[NB][64];                            // keys' with the factor of the scores in them, values' over 2^unit
  float none[64];                                          // zeros
  // .x: the unit times 4, and 2 where the scales lie apart: unit[] holds one for each token then, and 1 where .y, .z are not 0: the tokens, by
  // bits, whose value's scale is no finite number (0 stands in its place)
  uint4 about[NB];
  int unit[NB][64];
  static __device__ __forceinline__ int k_at(int key, int chunk) {
    return key * CH + (chunk ^ (DH == 128 ? key & 15 : (key >> 1) & 7));
  }
  static __device__ __forceinline__ int v_at(int d, int chunk) { return d * 8 + (chunk ^ ((d >> 1) & 7)); }
};

template <int DH, int RW, int KW, bool S16>
__global__ __launch_bounds__(64 * RW * KW, 2) void cache_attention_rows_kernel(AttnArgs a) {
  using St = Stage<DH>;
  constexpr int THREADS = 64 * RW * KW;
  constexpr int NB = DH / 64, DT = DH / 32, KK = DH / 16, Q = 32 * RW;
  constexpr int PIECES = 64 * DH / 16 / THREADS;           // pieces of 16 codes per thread, of keys and of values
  constexpr int SCALES = 2 * NB * 64;
  static_assert(SCALES <= THREADS, "a thread holds one scale of a tile");
  extern __shared__ __attribute__((aligned(16))) char lds[];
  St* stage = reinterpret_cast<St*>(lds);
  const int lane = threadIdx.x & 63, n = lane & 31, lh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row_wave = wave % RW, key_wave = wave / RW;
  // Workgroups go to the 8 XCDs in turn: all units of a sequence and head to one, kPairs of these at a time, so that its L2 holds what
  // they read; among them the last rows, which see the most, first.
  const int per_pair = a.row_groups * a.splits, mine = (a.c.B * a.c.KV + 7) >> 3, x = blockIdx.x >> 3;
  const int turn = x / (kPairs * per_pair), left = x - turn * kPairs * per_pair, width = min(kPairs, mine - turn * kPairs);
  const int which = left / width, pair = (turn * kPairs + left % width) * 8 + (blockIdx.x & 7);
  if (pair >= a.c.B * a.c.KV) return;
  const int rg = a.row_groups - 1 - which / a.splits, split = which % a.splits;
  const int b = pair / a.c.KV, g = pair - b * a.c.KV;
  const Span s = span_of(a.c, b);
  const int r0 = rg * Q, rows = s.fresh * a.group;
  if (r0 >= rows) return;
  const int len = a.tree ? s.past + s.fresh : s.past + (min(r0 + Q, rows) - 1) / a.group + 1;
  const int tiles = (len + kAttnTile - 1) / kAttnTile;
  const int first = split * a.chunk, end = split + 1 == a.splits ? tiles : min(tiles, first + a.chunk);

  // ---- this wavefront's queries, and up to where each sees
  const int w0 = r0 + row_wave * 32, r = w0 + n;
  const bool real = r < rows;
  const int t = real ? r / a.group : 0, head = g * a.group + (real ? r - t * a.group : 0);
  const size_t row = (size_t)b * a.c.tokens + t;
  bf16x8 qf[KK];
  {
    const bf16_raw* src = reinterpret_cast<const bf16_raw*>(a.q) + row * a.q_pitch + (size_t)head * DH + lh * 8;
#pragma unroll
    for (int k = 0; k < KK; ++k)
      qf[k] = __builtin_bit_cast(bf16x8, real ? *reinterpret_cast<const uint4*>(src + k * 16) : make_uint4(0, 0, 0, 0));
  }
  // which of the new tokens it sees (tree), and the tokens below `limit` (the past; without a tree up to the row's own)
  const uint64_t among = a.tree && real ? a.tree[row] & (s.fresh >= 64 ? ~0ull : (1ull << s.fresh) - 1) : 0;
  const int limit = a.tree ? s.past : s.past + t + 1;
  // tokens below `inner` are seen by all rows of this wavefront; from `outer` on by none
  const int inner = a.tree ? s.past : s.past + min(w0, rows - 1) / a.group + 1;
  const int outer = w0 >= rows ? 0 : a.tree ? len : s.past + (min(w0 + 32, rows) - 1) / a.group + 1;

  f32x16 o[DT];
  float ref = 0.f, l = 0.f;              // weights are 2^(score - ref)
  float most = -INFINITY;                // what a score may exceed ref by: nothing before the first, then 8
  int v_exp[NB], v_top[NB];              // the query's o is in units of 2^v_exp; its largest weight was about 2^v_top
#pragma unroll
  for (int blk = 0; blk < NB; ++blk) v_exp[blk] = v_top[blk] = kNoExp;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[d][e] = 0.f;

  // ---- staging: codes and scales of a tile in registers, then bf16 in LDS
  const int shift = a.c.page_shift, P1 = (1 << shift) - 1, last16 = (len - 1) & ~15;
  const int32_t* table = a.c.table + (size_t)b * a.c.table_pages;
  // Pages of a tile's four times 16 tokens, past the end the last ones; as they stand in the table, and looked at a tile later, so that
  // nothing waits for them.
  struct Pages { int p[4]; };
  auto is_page = [&](int p) { return (unsigned)p < (unsigned)a.c.n_pages; };
  auto pages_of = [&](int tile) {
    Pages out;
    if (shift >= 6) {
      out.p[0] = out.p[1] = out.p[2] = out.p[3] = table[(tile * kAttnTile) >> shift];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) out.p[i] = table[min(tile * kAttnTile + 16 * i, last16) >> shift];
    }
    return out;
  };
  auto valid_of = [&](int tile, const Pages& pg) {
    const int left = len - tile * kAttnTile;
    uint64_t v = left >= 64 ? ~0ull : (1ull << left) - 1;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (!is_page(pg.p[i])) v &= ~(0xFFFFull << (16 * i));
    return v;
  };
  auto pick = [&](const Pages& pg, int i) {
    const int p = i == 0 ? pg.p[0] : i == 1 ? pg.p[1] : i == 2 ? pg.p[2] : pg.p[3];
    return is_page(p) ? p : 0;
  };
  uint4 kc[PIECES], vc[PIECES];
  float sc;
  constexpr int KP = DH / 16;                                // pieces of a key row
  // The addresses first and one set of loads for both cases: with loads in the branches the merge would wait for them.
  auto load = [&](int tile, const Pages& pg) {
    const int j0 = tile * kAttnTile;
    size_t k_from[PIECES], v_from[PIECES], s_from;
    if (shift >= 6) {                                        // one page: its start is the same for all threads
      const size_t page0 = codes_at<DH>(a.c, pick(pg, 0), g), scale0 = scales_at<DH>(a.c, pick(pg, 0), g);
      const int place = j0 & P1;                             // the rest of the page is there, whether written or not
      const size_t k0 = page0 + (size_t)place * DH, v0 = page0 + place;
#pragma unroll
      for (int i = 0; i < PIECES; ++i) k_from[i] = k0 + (threadIdx.x + i * THREADS) * 16;
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const uint32_t idx = threadIdx.x + i * THREADS;
        v_from[i] = v0 + (((idx >> 2) << shift) + (idx & 3) * 16);
      }
      s_from = scale0 + (((threadIdx.x >> 6) % NB) << shift) + place + (threadIdx.x & 63);
    } else {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const int idx = threadIdx.x + i * THREADS, key = idx / KP, piece = idx % KP, place = min(j0 + key, last16 + 15) & P1;
        k_from[i] = codes_at<DH>(a.c, pick(pg, key >> 4), g) + place * DH + piece * 16;
      }
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const int idx = threadIdx.x + i * THREADS, d = idx >> 2, piece = idx & 3, place = min(j0 + piece * 16, last16) & P1;
        v_from[i] = codes_at<DH>(a.c, pick(pg, piece), g) + (d << shift) + place;
      }
      const int key = threadIdx.x & 63, blk = (threadIdx.x >> 6) % NB, place = min(j0 + key, last16 + 15) & P1;
      s_from = scales_at<DH>(a.c, pick(pg, key >> 4), g) + (blk << shift) + place;
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i) kc[i] = *reinterpret_cast<const uint4*>(a.c.k_codes + k_from[i]);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) vc[i] = *reinterpret_cast<const uint4*>(a.c.v_codes + v_from[i]);
    sc = block_scale_load(wave < NB ? a.c.k_scales : a.c.v_scales, s_from, S16);              // of threads beyond SCALES: in bounds, of no use
  };
  const float factor = (DH == 64 ? 0.125f : 0.08838834764831845f) * kLog2e;
  int v_now = kNoExp;                                        // of the wavefronts that stage values' scales
  auto store = [&](St& st, uint64_t valid) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int idx = threadIdx.x + i * THREADS, key = idx / KP, piece = idx % KP;
      const uint2 w0 = codes4(kc[i].x), w1 = codes4(kc[i].y), w2 = codes4(kc[i].z), w3 = codes4(kc[i].w);
      st.k[St::k_at(key, 2 * piece)] = make_uint4(w0.x, w0.y, w1.x, w1.y);
      st.k[St::k_at(key, 2 * piece + 1)] = make_uint4(w2.x, w2.y, w3.x, w3.y);
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int idx = threadIdx.x + i * THREADS, d = idx >> 2, piece = idx & 3;
      const uint2 w0 = codes4_f16(vc[i].x), w1 = codes4_f16(vc[i].y), w2 = codes4_f16(vc[i].z), w3 = codes4_f16(vc[i].w);
      st.v[St::v_at(d, 2 * piece)] = make_uint4(w0.x, w0.y, w1.x, w1.y);
      st.v[St::v_at(d, 2 * piece + 1)] = make_uint4(w2.x, w2.y, w3.x, w3.y);
    }
    const int key = threadIdx.x & 63, blk = wave % NB;       // a wavefront's 64 lanes are the 64 tokens of one block
    if (wave < NB) {
      st.ks[blk][key] = sc * factor;
    } else if (wave < 2 * NB) {
      const bool there = (valid >> key) & 1, fine = (__float_as_uint(sc) & 0x7FFFFFFFu) < 0x7F800000u;
      const uint64_t bad = __ballot(there && !fine);
      const float v = there && fine ? sc : 0.f;
      const uint32_t bits = __float_as_uint(v) & 0x7FFFFFFFu;
      const int ex = (int)(bits >> 23), place = ex - kLeast - v_now;       // v is from 2^(ex - 127) to below 2^(ex - 126)
      bool apart = false;
      if (__ballot(bits != 0 && (uint32_t)place >= (uint32_t)kRange) || (__ballot(place >= kRange / 2) == 0 && __ballot(bits != 0))) {
        const int hi = (int)(wave_umax(bits) >> 23), lo = (int)((wave_umin(bits - 1) + 1) >> 23);    // of those that are not 0
        apart = lo == 0 || hi - lo >= kRange;
        if (!apart) v_now = (hi - lo == kRange - 1 ? hi : hi + 1) - kRange + 1 - kLeast;        // room for a scale twice as large, if there is
      }
      const int unit = apart && bits != 0 ? ex - ex % kRange - kLeast : v_now;
      st.vs[blk][key] = ldexpf(v, -unit);
      if (apart) st.unit[blk][key] = unit;
      if (key == 0) st.about[blk] = make_uint4((uint32_t)(v_now * 4 + (apart ? 2 : 0) + (bad ? 1 : 0)), (uint32_t)bad, (uint32_t)(bad >> 32), 0);
    }
  };

  // 32 tokens of a tile: scores, weights, output
  const int k_row = (n & 16) | ((n & 4) << 1) | ((n & 8) >> 1) | (n & 3);       // the token of this lane's row of the keys' operand
  // odd: not all queries' sums are in the tile's unit, or it has several, or there is a bad value: for the block `which` alone then, and
  // tokens of one unit
  auto half = [&](const St& st, int j0, int kh, uint64_t valid, bool odd, int which, int unit, bool bad_ones) {
    f32x16 acc[NB];
#pragma unroll
    for (int blk = 0; blk < NB; ++blk)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[blk][e] = 0.f;
#pragma unroll
    for (int k = 0; k < KK; ++k) {
      const bf16x8 kf = __builtin_bit_cast(bf16x8, st.k[St::k_at(32 * kh + k_row, 2 * k + lh)]);
      acc[k / 4] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[k], acc[k / 4], 0, 0, 0);
    }
    float p[16];                                             // tokens 32 kh + 16 (e / 8) + 8 lh + e % 8
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      const int at = 32 * kh + 16 * (e >> 3) + 8 * lh + (e & 4);
      const float4 k0 = *reinterpret_cast<const float4*>(&st.ks[0][at]);
      p[e] = fmaf(acc[0][e], k0.x, -ref); p[e + 1] = fmaf(acc[0][e + 1], k0.y, -ref);
      p[e + 2] = fmaf(acc[0][e + 2], k0.z, -ref); p[e + 3] = fmaf(acc[0][e + 3], k0.w, -ref);
      if constexpr (NB == 2) {
        const float4 k1 = *reinterpret_cast<const float4*>(&st.ks[NB - 1][at]);
        p[e] = fmaf(acc[NB - 1][e], k1.x, p[e]); p[e + 1] = fmaf(acc[NB - 1][e + 1], k1.y, p[e + 1]);
        p[e + 2] = fmaf(acc[NB - 1][e + 2], k1.z, p[e + 2]); p[e + 3] = fmaf(acc[NB - 1][e + 3], k1.w, p[e + 3]);
      }
    }
    const int h0 = j0 + 32 * kh;
    const bool whole = (uint32_t)(valid >> (32 * kh)) == 0xFFFFFFFFu && h0 + 32 <= inner;
    uint32_t sees = 0xFFFFFFFFu;                             // of the lane's query, by token
    if (!whole) {
      const int below = limit - h0;
      sees = below >= 32 ? 0xFFFFFFFFu : below <= 0 ? 0u : (1u << below) - 1;
      const int u0 = h0 - s.past;                            // of the first of them among the new tokens
      if (u0 > -32 && u0 < 64) sees |= u0 >= 0 ? (uint32_t)(among >> u0) : (uint32_t)(among << -u0);
      sees = (sees & (uint32_t)(valid >> (32 * kh))) >> (8 * lh);
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (!((sees >> (16 * (e >> 3) + (e & 7))) & 1)) p[e] = -INFINITY;
    }
    float top = fmaxf(p[0], p[1]);
#pragma unroll
    for (int e = 2; e < 16; ++e) top = fmaxf(top, p[e]);
    if (__ballot(top > most)) {
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      if (top > -INFINITY) {
        const bool fresh = most == -INFINITY;
        const float next = fresh ? top : ref + fmaxf(top, 0.f), up = next - ref;
        const float keep = fresh ? 1.f : __builtin_amdgcn_exp2f(-up);        // fresh: there is nothing yet
#pragma unroll
        for (int blk = 0; blk < NB; ++blk) v_top[blk] -= fresh ? 0 : (int)fminf(up, 1000.f);
        ref = next;
        most = 8.0f;
        l *= keep;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] *= keep;
#pragma unroll
        for (int e = 0; e < 16; ++e) p[e] -= up;
      }
    }
    const float* vs[NB];
#pragma unroll
    for (int blk = 0; blk < NB; ++blk) vs[blk] = odd && blk != which ? st.none : st.vs[blk];
    float counted = 1.0f;                                    // what makes a weight one of the sum l
    if (odd) {
      // a value that is infinite or none goes to its block of all the rows that see it, and to no others
      float none = 0.f;
      if (bad_ones) {
        const uint32_t bad = kh == 0 ? st.about[which].y : st.about[which].z;
        if (sees & (bad >> (8 * lh)) & 0x00FF00FFu) none = __uint_as_float(0x7FC00000u);
        none += __shfl_xor(none, 32, 64);
      }
      // The sums to the unit, or to that of the query's largest weight here where that is less but more than the sums' own (a query
      // without weights here adds zeros in any unit); the weights to what they are in that unit.  What is too far below the sums is left out.
      const float* mine = which == 0 ? st.vs[0] : st.vs[NB - 1];
      float top = -INFINITY;                                 // of those that have a value other than 0
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, mine[32 * kh + 16 * (e >> 3) + 8 * lh + (e & 7)] != 0.f ? p[e] : -INFINITY);
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      const bool any = top > -126.0f;
      const int up = (int)ceilf(any ? top : 0.f);            // the weights are 2^up at most
      int by = 0;
#pragma unroll
      for (int blk = 0; blk < NB; ++blk) {
        if (blk != which) continue;
        const int next = unit;
        const bool first = v_top[blk] < kNoExp / 2;          // the sums are 0 yet, in no unit
        const int have = first ? kNoExp : v_exp[blk];
        const bool counts = next >= have || next >= v_top[blk] - kFall;
        const int at = !real || (first && !any) ? next : !any || !counts ? v_exp[blk] : next < have ? next : min(next, max(next + max(up, -100), have));
        const float less = (first ? 0.f : ldexpf(1.0f, have - at)) + none;
#pragma unroll
        for (int d = 2 * blk; d < 2 * blk + 2; ++d) o[d] *= less;
        by = !any ? 0 : counts ? next - at : -60;            // 2^-60: nothing in fp16
        v_exp[blk] = at;
        v_top[blk] = any && counts ? max(v_top[blk], next + up) : v_top[blk];
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) p[e] += (float)by;
      counted = which == 0 ? ldexpf(1.0f, -by) : 0.f;
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      p[e] = __builtin_amdgcn_exp2f(p[e]);
      l = fmaf(p[e], counted, l);
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      f16x8 pf[NB];
#pragma unroll
      for (int blk = 0; blk < NB; ++blk) {
        const float4 s0 = *reinterpret_cast<const float4*>(vs[blk] + 32 * kh + 16 * c + 8 * lh);
        const float4 s1 = *reinterpret_cast<const float4*>(vs[blk] + 32 * kh + 16 * c + 8 * lh + 4);
        const float* w = p + 8 * c;
        pf[blk] = __builtin_bit_cast(f16x8, make_uint4(pack2_f16(w[0] * s0.x, w[1] * s0.y), pack2_f16(w[2] * s0.z, w[3] * s0.w),
                                                       pack2_f16(w[4] * s1.x, w[5] * s1.y), pack2_f16(w[6] * s1.z, w[7] * s1.w)));
      }
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const f16x8 vf = __builtin_bit_cast(f16x8, st.v[St::v_at(d * 32 + n, 4 * kh + 2 * c + lh)]);
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, pf[d / 2], o[d], 0, 0, 0);
      }
    }
  };

  if (first < end) {                     // (no write to LDS without tiles: nothing would keep it from the results that are joined there)
    if (threadIdx.x < 128) stage[threadIdx.x >> 6].none[threadIdx.x & 63] = 0.f;
    Pages pg = pages_of(first);
    uint64_t valid = valid_of(first, pg);
    load(first, pg);
    store(stage[0], valid);
    if (first + 1 < end) pg = pages_of(first + 1);
    __syncthreads();
    for (int tile = first; tile < end; ++tile) {
      const bool more = tile + 1 < end;
      const St& st = stage[(tile - first) & 1];
      int head[NB];                                          // asked for here, looked at behind the next tile's loads
#pragma unroll
      for (int blk = 0; blk < NB; ++blk) head[blk] = (int)st.about[blk].x;
      uint64_t valid_next = 0;
      if (more) {
        load(tile + 1, pg);
        valid_next = valid_of(tile + 1, pg);
        if (tile + 2 < end) pg = pages_of(tile + 2);
      }
      const int j0 = tile * kAttnTile;
      int flags = 0;
      bool moves = false;
#pragma unroll
      for (int blk = 0; blk < NB; ++blk) {
        head[blk] = __builtin_amdgcn_readfirstlane(head[blk]);
        flags |= head[blk] & 3;
        if (tile == first && !(head[blk] & 2)) v_exp[blk] = head[blk] >> 2;     // of sums that are 0 yet
        moves |= v_exp[blk] != head[blk] >> 2;
      }
      const bool odd = flags != 0 || __ballot(moves) != 0;
      if (__builtin_expect(!odd, 1)) {
        if constexpr (KW == 1) {
          if (j0 < outer) half(st, j0, 0, valid, false, 0, 0, false);
          if (j0 + 32 < outer) half(st, j0, 1, valid, false, 0, 0, false);
        } else {
          if (j0 + 32 * key_wave < outer) half(st, j0, key_wave, valid, false, 0, 0, false);
        }
      }
#pragma unroll
      for (int blk = 0; blk < NB; ++blk) v_top[blk] = odd && most > -INFINITY ? max(v_top[blk], v_exp[blk]) : v_top[blk];
#pragma nounroll
      for (int which = 0; __builtin_expect(odd && which < NB, 0); ++which) {
        const int mine = which == 0 ? head[0] : head[NB - 1];
        // the tokens that are left; the same for all lanes, as the loop over their units has to know
        uint64_t rest = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(valid >> 32)) << 32 |
                        (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)valid);
#pragma nounroll
        while (rest) {
          uint64_t now = rest;
          int unit = mine >> 2;
          if (mine & 2) {
            const int theirs = st.unit[which][lane];
            unit = __builtin_amdgcn_readlane(theirs, __builtin_ctzll(rest));
            now &= __ballot(theirs == unit);
          }
          rest &= ~now;
#pragma nounroll
          for (int i = 0; i < (KW == 1 ? 2 : 1); ++i) {
            const int kh = KW == 1 ? i : key_wave;
            if (j0 + 32 * kh < outer) half(st, j0, kh, now, true, which, unit, flags & 1);
          }
        }
      }
      if (more) store(stage[(tile + 1 - first) & 1], valid_next);
      valid = valid_next;
      __syncthreads();
    }
  }

#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[d][e] = ldexpf(o[d][e], v_exp[d / 2]);
  l += __shfl_xor(l, 32, 64);
  float m = most == -INFINITY ? -INFINITY : ref;
  if constexpr (KW == 2) {                                   // the second half's results through LDS: [row wavefront][register][lane]
    float* other = reinterpret_cast<float*>(lds) + row_wave * (DT * 16 + 2) * 64 + lane;
    if (key_wave == 1) {
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) other[(d * 16 + e) * 64] = o[d][e];
      other[DT * 16 * 64] = m;
      other[(DT * 16 + 1) * 64] = l;
    }
    __syncthreads();
    if (key_wave == 1) return;
    const float m1 = other[DT * 16 * 64], mn = fmaxf(m, m1), ref = mn == -INFINITY ? 0.f : mn;
    const float f0 = __builtin_amdgcn_exp2f(m - ref), f1 = __builtin_amdgcn_exp2f(m1 - ref);
    m = mn;
    l = fmaf(other[(DT * 16 + 1) * 64], f1, l * f0);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[d][e] = fmaf(other[(d * 16 + e) * 64], f1, o[d][e] * f0);
  }
  if (!real) return;
  if (a.splits == 1) {
    bf16_raw* to = reinterpret_cast<bf16_raw*>(a.out) + row * a.out_pitch + (size_t)head * DH + 4 * lh;
    const float f = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *reinterpret_cast<uint2*>(to + d * 32 + 2 * e) =
            l == 0.f ? make_uint2(0, 0) : make_uint2(pack2(o[d][e] * f, o[d][e + 1] * f), pack2(o[d][e + 2] * f, o[d][e + 3] * f));
  } else {
    const size_t at = ((((size_t)b * a.row_groups + rg) * a.c.KV + g) * a.splits + split) * Q + (r - r0);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *reinterpret_cast<float4*>(a.part_o + at * DH + d * 32 + 2 * e + 4 * lh) = make_float4(o[d][e], o[d][e + 1], o[d][e + 2], o[d][e + 3]);
    if (lh == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * at) = make_float2(m, l);
  }
}

template <int DH, int RW, int KW, bool S16>
swarm_status launch(const AttnArgs& a, hipStream_t st) {
  static LdsOptIn opted;
  constexpr size_t bytes = 2 * sizeof(Stage<DH>);
  static_assert(KW == 1 || RW * (DH / 2 + 2) * 64 * 4 <= (int)bytes, "the second half's results fit where the tiles were");
  const swarm_status ok = lds_opt_in(reinterpret_cast<const void*>(&cache_attention_rows_kernel<DH, RW, KW, S16>), bytes, opted);
  if (ok != SWARM_OK) return ok;
  const long long pairs = ((long long)a.c.B * a.c.KV + 7) / 8 * 8, blocks = pairs * a.row_groups * a.splits;
  if (blocks > 0x7FFFFFFF) return SWARM_ERR_SHAPE;
  hipLaunchKernelGGL((cache_attention_rows_kernel<DH, RW, KW, S16>), dim3((unsigned)blocks), dim3(64 * RW * KW), bytes, st, a);
  return launch_status();
}
template <int DH, bool S16>
swarm_status launch_rows(const AttnArgs& a, int row_waves, hipStream_t st) {
  return row_waves == 2 ? launch<DH, 2, 2, S16>(a, st) : launch<DH, 4, 1, S16>(a, st);
}

}  // namespace

swarm_status cache_attention_rows_launch(const AttnArgs& a, int dh, int row_waves, hipStream_t st) {
  if (dh == 64) return a.s16 ? launch_rows<64, true>(a, row_waves, st) : launch_rows<64, false>(a, row_waves, st);
  return a.s16 ? launch_rows<128, true>(a, row_waves, st) : launch_rows<128, false>(a, row_waves, st);
}

}  // namespace swarm
