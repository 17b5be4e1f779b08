// The paged int8 cache of keys and values: append (rotation and quantisation in one pass), read, and the move that keeps the accepted
// tokens of a draft.  All three are streaming kernels: append reads a row element once and writes its code, read the reverse.
//
// Keys lie as rows, page[head][token][d_head]: the 8 (d_head 64) or 16 (128) threads of a row make its codes from 8 elements each,
// the block absmax being a butterfly over 8 lanes as in the boundary codec.  Values lie transposed, page[head][d_head][token]:
// a workgroup quantises 64 consecutive tokens of one head, turns the codes in LDS (four tokens to a 32-bit word) and writes
// 16 tokens of one element at a time, so that no store is shorter than 16 bytes except at the ends of the new tokens.
// 4 x 2048 tokens of 32 x 128, rotated: append 82 us for 339 MB, read 42 for 205 MB (a copy moves 5.2 TB/s).
#include "cache.h"

namespace swarm {
namespace {

constexpr int kThreads = 256;
constexpr int kTokens = 16;      // tokens of a workgroup of rows (queries, keys)
constexpr int kTile = 64;        // tokens of a workgroup of values
constexpr int kPitch = 17;       // 32-bit words per element row of a turned tile: 16, and one against bank conflicts

__device__ __forceinline__ int code_of(float x, const BlockDivisor& s) {
  return (int)fminf(fmaxf(rintf(s.quotient(x)), -127.0f), 127.0f);
}

// Codes of 8 of the 64 elements of a block whose other 56 the lanes of the octet hold; returns the scale as it is stored.
__device__ __forceinline__ float encode8(const float (&x)[8], int (&c)[8], bool s16) {
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(x[i]));
  m = fmaxf(m, __shfl_xor(m, 1, 64));
  m = fmaxf(m, __shfl_xor(m, 2, 64));
  m = fmaxf(m, __shfl_xor(m, 4, 64));
  const float scale = block_scale_rounded(m / 127.0f, s16);
  const BlockDivisor div(scale);
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = scale == 0.0f ? 0 : code_of(x[i], div);
  return scale;
}

__device__ __forceinline__ uint32_t bytes4(int a, int b, int c, int d) {
  return (uint32_t)(a & 0xFF) | ((uint32_t)(b & 0xFF) << 8) | ((uint32_t)(c & 0xFF) << 16) | ((uint32_t)d << 24);
}

struct AppendArgs {
  CacheArgs c;
  const void *q, *k, *v;
  void* q_out;
  const int32_t* positions;
  size_t pitch, q_out_pitch;
  int row_tiles, head_groups, heads_per_group, value_tiles;
  int row_blocks;          // workgroups of rows; those of values follow
  bool s16;
};

// Rows of queries (rotated into q_out) and keys (rotated, quantised): 16 tokens of one sequence, some of the heads.  The angles'
// cosines and sines are made once per token and pair for all of these heads, in 64 bits, in LDS.
template <typename T, int DH, bool ROT>
__device__ __forceinline__ void append_rows(const AppendArgs& a, int block, double2* turn) {
  const int group = block % a.head_groups, rest = block / a.head_groups;
  const int b = rest / a.row_tiles, t0 = (rest - b * a.row_tiles) * kTokens;
  const Span s = span_of(a.c, b);
  if (t0 >= s.fresh) return;
  const int n = min(kTokens, s.fresh - t0);
  const size_t row0 = (size_t)b * a.c.tokens + t0;
  if constexpr (ROT) {
    constexpr int HALF = DH / 2;
    for (int i = threadIdx.x; i < n * HALF; i += kThreads) {
      const int t = i / HALF, pair = i - t * HALF;
      const int pos = a.positions ? a.positions[row0 + t] : s.past + t0 + t;
      const double inv = exp2(-(double)pair / (double)HALF * 13.287712379549449);   // log2(10000)
      double sn, cs;
      sincos((double)pos * inv, &sn, &cs);
      turn[i] = make_double2(cs, sn);
    }
    __syncthreads();
  }
  // A pass: HS heads of the tile's tokens, one chunk of 8 elements per thread; U passes' loads are on their way together.  Threads beyond
  // the last token or head do the last one's work over again, without writing it.
  constexpr int C = DH / 8, HS = kThreads / (kTokens * C), U = 4;
  const int q_heads = ROT ? a.c.H : 0, heads = q_heads + a.c.KV;
  const int h0 = group * a.heads_per_group, h1 = min(heads, h0 + a.heads_per_group);
  const int chunk = threadIdx.x % C, mine = threadIdx.x / C % kTokens, t = min(mine, n - 1);
  const int hh = __builtin_amdgcn_readfirstlane(threadIdx.x / (C * kTokens));
  const int j = s.past + t0 + t, page = page_of(a.c, b, j), place = j & ((1 << a.c.page_shift) - 1);
  for (int hb = h0 + hh; hb < h1; hb += U * HS) {
    float x[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = min(hb + u * HS, h1 - 1);
      const T* src = reinterpret_cast<const T*>(h < q_heads ? a.q : a.k) + (row0 + t) * a.pitch + (size_t)(h < q_heads ? h : h - q_heads) * DH;
      Row8<T>::load(src + chunk * 8, x[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = hb + u * HS;
      if (h >= h1) break;
      const bool is_q = h < q_heads;
      const int head = is_q ? h : h - q_heads;
      if constexpr (ROT) {
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          const double2 w = turn[t * (DH / 2) + chunk * 4 + p];
          const double e = x[u][2 * p], o = x[u][2 * p + 1];
          x[u][2 * p] = (float)(e * w.x - o * w.y);
          x[u][2 * p + 1] = (float)(e * w.y + o * w.x);
        }
        if (is_q) {
          if (mine < n) Row8<T>::store(reinterpret_cast<T*>(a.q_out) + (row0 + t) * a.q_out_pitch + (size_t)head * DH + chunk * 8, x[u]);
          continue;
        }
      }
      int c[8];
      const float scale = encode8(x[u], c, a.s16);
      if (mine >= n || page < 0) continue;
      *reinterpret_cast<uint2*>(a.c.k_codes + codes_at<DH>(a.c, page, head) + (size_t)place * DH + chunk * 8) =
          make_uint2(bytes4(c[0], c[1], c[2], c[3]), bytes4(c[4], c[5], c[6], c[7]));
      if ((chunk & 7) == 0)
        block_scale_store(a.c.k_scales, scales_at<DH>(a.c, page, head) + ((size_t)(chunk >> 3) << a.c.page_shift) + place, scale, a.s16);
    }
  }
}

// The values of one head at 64 consecutive places of a sequence, as far as they are new.
template <typename T, int DH>
__device__ __forceinline__ void append_values(const AppendArgs& a, int block, uint32_t* turned) {
  const int head = block % a.c.KV, rest = block / a.c.KV;
  const int b = rest / a.value_tiles, tile = rest - b * a.value_tiles;
  const Span s = span_of(a.c, b);
  if (s.fresh == 0) return;                      // there is no nearest new token to load in place of the others
  const int base = (s.past / kTile + tile) * kTile, end = s.past + s.fresh;      // places base .. base + 63
  if (base >= end || base + kTile <= s.past) return;
  constexpr int C = DH / 8;
  const int chunk = threadIdx.x % C, quad = threadIdx.x / C;                     // d_head 64: half of the threads have no tokens
  if (quad < kTile / 4) {
    uint32_t words[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    float x[4][8];
    int pages[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {                  // all loads first; places that are not new take the nearest one that is
      const int j = min(max(base + quad * 4 + u, s.past), end - 1);
      Row8<T>::load(reinterpret_cast<const T*>(a.v) + ((size_t)b * a.c.tokens + (j - s.past)) * a.pitch + (size_t)head * DH + chunk * 8, x[u]);
      pages[u] = page_of(a.c, b, j);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int j = base + quad * 4 + u;
      int c[8];
      const float scale = encode8(x[u], c, a.s16);
#pragma unroll
      for (int i = 0; i < 8; ++i) words[i] |= (uint32_t)(c[i] & 0xFF) << (8 * u);
      if ((chunk & 7) == 0 && pages[u] >= 0 && j >= s.past && j < end)
        block_scale_store(a.c.v_scales, scales_at<DH>(a.c, pages[u], head) + ((size_t)(chunk >> 3) << a.c.page_shift) +
                          (j & ((1 << a.c.page_shift) - 1)), scale, a.s16);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) turned[(chunk * 8 + i) * kPitch + quad] = words[i];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < DH * 4; i += kThreads) {
    const int d = i >> 2, j0 = base + (i & 3) * 16;
    if (j0 >= end || j0 + 16 <= s.past) continue;
    const int page = page_of(a.c, b, j0);
    if (page < 0) continue;
    int8_t* to = a.c.v_codes + codes_at<DH>(a.c, page, head) + ((size_t)d << a.c.page_shift) + (j0 & ((1 << a.c.page_shift) - 1));
    const uint32_t* w = turned + d * kPitch + (i & 3) * 4;
    if (j0 >= s.past && j0 + 16 <= end) {
      *reinterpret_cast<uint4*>(to) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
      for (int e = max(0, s.past - j0); e < min(16, end - j0); ++e) to[e] = (int8_t)(w[e >> 2] >> (8 * (e & 3)));
    }
  }
}

template <typename T, int DH, bool ROT>
__global__ __launch_bounds__(kThreads) void cache_append_kernel(AppendArgs a) {
  __shared__ __attribute__((aligned(16))) char lds[ROT ? kTokens * DH / 2 * sizeof(double2) : DH * kPitch * 4];
  static_assert(sizeof(double2) * kTokens / 2 >= kPitch * 4, "a turned tile fits where the angles do");
  if ((int)blockIdx.x < a.row_blocks)
    append_rows<T, DH, ROT>(a, blockIdx.x, reinterpret_cast<double2*>(lds));
  else
    append_values<T, DH>(a, blockIdx.x - a.row_blocks, reinterpret_cast<uint32_t*>(lds));
}

struct ReadArgs {
  CacheArgs c;
  void *k, *v;
  int row_tiles, value_tiles, key_blocks;
  bool s16;
};

template <typename T, int DH>
__device__ __forceinline__ void read_keys(const ReadArgs& a, int block) {
  const int head = block % a.c.KV, rest = block / a.c.KV;
  const int b = rest / a.row_tiles, t0 = (rest - b * a.row_tiles) * kTile;
  const Span s = span_of(a.c, b);
  constexpr int C = DH / 8;
  for (int i = threadIdx.x; i < kTile * C; i += kThreads) {
    const int t = t0 + i / C, chunk = i % C;
    if (t >= s.fresh) return;
    const int j = s.past + t, page = page_of(a.c, b, j), place = j & ((1 << a.c.page_shift) - 1);
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (page >= 0) {
      const uint2 w = *reinterpret_cast<const uint2*>(a.c.k_codes + codes_at<DH>(a.c, page, head) + (size_t)place * DH + chunk * 8);
      const float scale = block_scale_load(a.c.k_scales, scales_at<DH>(a.c, page, head) + ((size_t)(chunk >> 3) << a.c.page_shift) + place, a.s16);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = (float)(int8_t)((e < 4 ? w.x : w.y) >> (8 * (e & 3))) * scale;
    }
    Row8<T>::store(reinterpret_cast<T*>(a.k) + (((size_t)b * a.c.tokens + t) * a.c.KV + head) * DH + chunk * 8, x);
  }
}

template <typename T, int DH>
__device__ __forceinline__ void read_values(const ReadArgs& a, int block, uint32_t* turned) {
  const int head = block % a.c.KV, rest = block / a.c.KV;
  const int b = rest / a.value_tiles, tile = rest - b * a.value_tiles;
  const Span s = span_of(a.c, b);
  if (s.fresh == 0) return;
  const int base = (s.past / kTile + tile) * kTile, end = s.past + s.fresh;
  if (base >= end || base + kTile <= s.past) return;
  for (int i = threadIdx.x; i < DH * 4; i += kThreads) {
    const int d = i >> 2, j0 = base + (i & 3) * 16;
    uint4 w = make_uint4(0, 0, 0, 0);
    if (j0 < end && j0 + 16 > s.past) {
      const int page = page_of(a.c, b, j0);
      if (page >= 0)
        w = *reinterpret_cast<const uint4*>(a.c.v_codes + codes_at<DH>(a.c, page, head) + ((size_t)d << a.c.page_shift) +
                                            (j0 & ((1 << a.c.page_shift) - 1)));
    }
    uint32_t* to = turned + d * kPitch + (i & 3) * 4;
    to[0] = w.x; to[1] = w.y; to[2] = w.z; to[3] = w.w;
  }
  __syncthreads();
  constexpr int C = DH / 8;
  const int chunk = threadIdx.x % C, quad = threadIdx.x / C;
  if (quad >= kTile / 4) return;
  uint32_t words[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) words[i] = turned[(chunk * 8 + i) * kPitch + quad];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int j = base + quad * 4 + u;
    if (j < s.past || j >= end) continue;
    const int page = page_of(a.c, b, j);
    const float scale = page < 0 ? 0.f
        : block_scale_load(a.c.v_scales, scales_at<DH>(a.c, page, head) + ((size_t)(chunk >> 3) << a.c.page_shift) +
                           (j & ((1 << a.c.page_shift) - 1)), a.s16);
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)(int8_t)(words[i] >> (8 * u)) * scale;
    Row8<T>::store(reinterpret_cast<T*>(a.v) + (((size_t)b * a.c.tokens + (j - s.past)) * a.c.KV + head) * DH + chunk * 8, x);
  }
}

template <typename T, int DH>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(ReadArgs a) {
  __shared__ uint32_t turned[DH * kPitch];
  if ((int)blockIdx.x < a.key_blocks) read_keys<T, DH>(a, blockIdx.x);
  else read_values<T, DH>(a, blockIdx.x - a.key_blocks, turned);
}

// One head of one sequence: everything that moves is read into LDS before anything is written, so the order of `kept` is free.
constexpr int kDraft = 64;
constexpr int kDraftBytes = 84;        // 79 places (64, starting anywhere in 16) and padding to an odd number of words
template <int DH>
__global__ __launch_bounds__(kThreads) void cache_keep_kernel(CacheArgs a, const int32_t* __restrict__ kept, bool s16) {
  __shared__ uint4 keys[kDraft * DH / 16];
  __shared__ uint32_t values[DH * kDraftBytes / 4];
  __shared__ float scales[2][DH / 64][kDraft];
  __shared__ int from[kDraft];
  __shared__ __attribute__((aligned(16))) uint8_t place_from[80];   // where the value that goes to a place lies among the values read
  const int b = blockIdx.x / a.KV, head = blockIdx.x - b * a.KV;
  const Span s = span_of(a, b);                 // fresh: how many are kept
  if (s.fresh == 0) return;
  const int P1 = (1 << a.page_shift) - 1;
  const long long cap = (long long)a.table_pages << a.page_shift;
  const int base = s.past & ~15, off = s.past - base;
  if (threadIdx.x < 80) {
    const int j = (int)threadIdx.x - off;
    int u = -1;
    if (j >= 0 && j < s.fresh) {
      u = kept[(size_t)b * a.tokens + j];
      if (u < 0 || u >= a.tokens || (long long)s.past + u >= cap || page_of(a, b, s.past + u) < 0) u = -1;
      from[j] = u;
    }
    place_from[threadIdx.x] = (uint8_t)(u < 0 ? (int)threadIdx.x : off + u);
  }
  // places of the draft that the table can hold, in chunks of 16
  const int last = (int)min((long long)s.past + a.tokens, cap), chunks = (last - base + 15) >> 4;
  for (int i = threadIdx.x; i < DH * chunks; i += kThreads) {
    const int d = i / chunks, c = i - d * chunks, j0 = base + 16 * c, page = page_of(a, b, j0);
    if (page < 0) continue;
    const uint4 w = *reinterpret_cast<const uint4*>(a.v_codes + codes_at<DH>(a, page, head) + ((size_t)d << a.page_shift) + (j0 & P1));
    uint32_t* to = values + (d * kDraftBytes >> 2) + 4 * c;
    to[0] = w.x; to[1] = w.y; to[2] = w.z; to[3] = w.w;
  }
  __syncthreads();
  constexpr int KC = DH / 16;
  for (int i = threadIdx.x; i < s.fresh * KC; i += kThreads) {
    const int j = i / KC, c = i - j * KC, u = from[j];
    if (u < 0) continue;
    const int at = s.past + u, page = page_of(a, b, at);
    keys[i] = *reinterpret_cast<const uint4*>(a.k_codes + codes_at<DH>(a, page, head) + (size_t)(at & P1) * DH + c * 16);
  }
  for (int i = threadIdx.x; i < s.fresh * 2 * (DH / 64); i += kThreads) {
    const int j = i % s.fresh, what = i / s.fresh, u = from[j];
    if (u < 0) continue;
    const int at = s.past + u, page = page_of(a, b, at);
    scales[what & 1][what >> 1][j] = block_scale_load(what & 1 ? a.v_scales : a.k_scales, scales_at<DH>(a, page, head) +
                                                      ((size_t)(what >> 1) << a.page_shift) + (at & P1), s16);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < s.fresh * KC; i += kThreads) {
    const int j = i / KC, c = i - j * KC, at = s.past + j, page = page_of(a, b, at);
    if (from[j] < 0 || page < 0) continue;
    *reinterpret_cast<uint4*>(a.k_codes + codes_at<DH>(a, page, head) + (size_t)(at & P1) * DH + c * 16) = keys[i];
  }
  for (int i = threadIdx.x; i < s.fresh * 2 * (DH / 64); i += kThreads) {
    const int j = i % s.fresh, what = i / s.fresh, at = s.past + j, page = page_of(a, b, at);
    if (from[j] < 0 || page < 0) continue;
    block_scale_store(what & 1 ? a.v_scales : a.k_scales, scales_at<DH>(a, page, head) + ((size_t)(what >> 1) << a.page_shift) +
                      (at & P1), scales[what & 1][what >> 1][j], s16);
  }
  // a chunk of 16 places per wavefront at a time: its sources are the same for all elements
  const int to_chunks = (off + s.fresh + 15) >> 4, d = threadIdx.x % DH;
  for (int c = threadIdx.x / DH; c < to_chunks; c += kThreads / DH) {
    const int j0 = base + 16 * c, page = page_of(a, b, j0);
    if (page < 0) continue;
    const uint8_t* row = reinterpret_cast<const uint8_t*>(values) + d * kDraftBytes;
    const uint4 at = *reinterpret_cast<const uint4*>(place_from + 16 * c);
    const uint32_t src[4] = {at.x, at.y, at.z, at.w};
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 16; ++e) w[e >> 2] |= (uint32_t)row[(src[e >> 2] >> (8 * (e & 3))) & 0xFF] << (8 * (e & 3));
    *reinterpret_cast<uint4*>(a.v_codes + codes_at<DH>(a, page, head) + ((size_t)d << a.page_shift) + (j0 & P1)) =
        make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// 64-place tiles that `tokens` consecutive tokens can touch
int tiles_touched(int tokens) { return (tokens + kTile - 2) / kTile + 1; }

template <typename T, int DH>
swarm_status append_as(AppendArgs a, bool rot, int blocks, hipStream_t st) {
  if (rot) hipLaunchKernelGGL((cache_append_kernel<T, DH, true>), dim3(blocks), dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL((cache_append_kernel<T, DH, false>), dim3(blocks), dim3(kThreads), 0, st, a);
  return launch_status();
}

}  // namespace

swarm_status cache_append_launch(const swarm_cache_config* c, const CacheArgs& args, const void* q, const void* k, const void* v,
                                 size_t pitch, const int32_t* positions, bool rotary, void* q_out, size_t q_out_pitch,
                                 hipStream_t st) {
  AppendArgs a{};
  a.c = args; a.q = q; a.k = k; a.v = v; a.q_out = q_out; a.positions = positions; a.pitch = pitch; a.q_out_pitch = q_out_pitch;
  a.s16 = c->scale_bits == 16;
  a.row_tiles = (args.tokens + kTokens - 1) / kTokens;
  a.value_tiles = tiles_touched(args.tokens);
  const int heads = (rotary ? c->n_heads : 0) + c->n_kv_heads;
  const long long tiles = (long long)c->batch * a.row_tiles;
  // heads are spread over workgroups until there are four of these per compute unit, eight heads each at least: every workgroup
  // makes its own angles
  const int groups = (int)std::max(1ll, std::min<long long>((heads + 7) / 8, 1024 / tiles));
  a.heads_per_group = (heads + groups - 1) / groups;
  a.head_groups = (heads + a.heads_per_group - 1) / a.heads_per_group;
  const long long rows = tiles * a.head_groups, blocks = rows + (long long)c->batch * a.value_tiles * c->n_kv_heads;
  if (blocks > 0x7FFFFFFF) return SWARM_ERR_SHAPE;
  a.row_blocks = (int)rows;
  if (c->dtype == SWARM_BF16)
    return c->d_head == 64 ? append_as<bf16_raw, 64>(a, rotary, (int)blocks, st) : append_as<bf16_raw, 128>(a, rotary, (int)blocks, st);
  return c->d_head == 64 ? append_as<float, 64>(a, rotary, (int)blocks, st) : append_as<float, 128>(a, rotary, (int)blocks, st);
}

}  // namespace swarm

using namespace swarm;

extern "C" swarm_status swarm_cache_append(const swarm_cache_config* cfg, const swarm_cache* cache, const int32_t* page_table,
                                           const int32_t* past, const int32_t* fresh, int32_t tokens, const void* q, const void* k,
                                           const void* v, size_t row_pitch, const int32_t* positions, int32_t rotary, void* q_out,
                                           size_t q_out_pitch, void* hip_stream) {
  if (!cfg || !cache_pointers_ok(cache) || !page_table || !past || !k || !v) return SWARM_ERR_NULL;
  if (rotary && (!q || !q_out)) return SWARM_ERR_NULL;
  const swarm_status bad = cache_config_status(cfg, tokens);
  if (bad != SWARM_OK) return bad;
  if (!rotary && (q || q_out || positions)) return SWARM_ERR_SHAPE;
  const size_t kv = (size_t)cfg->n_kv_heads * cfg->d_head, qw = (size_t)cfg->n_heads * cfg->d_head;
  if (!cache_aligned(cache) || !pitch_ok(k, row_pitch, kv, cfg->dtype) || !pitch_ok(v, row_pitch, kv, cfg->dtype)) return SWARM_ERR_SHAPE;
  if (rotary && (!pitch_ok(q, row_pitch, qw, cfg->dtype) || !pitch_ok(q_out, q_out_pitch, qw, cfg->dtype) ||
                 (q == q_out && row_pitch != q_out_pitch)))
    return SWARM_ERR_SHAPE;
  return cache_append_launch(cfg, cache_args(cfg, cache, page_table, past, fresh, tokens), q, k, v, row_pitch, positions, rotary != 0,
                             q_out, q_out_pitch, (hipStream_t)hip_stream);
}

extern "C" swarm_status swarm_cache_read(const swarm_cache_config* cfg, const swarm_cache* cache, const int32_t* page_table,
                                         const int32_t* first, const int32_t* count, int32_t tokens, void* k_out, void* v_out,
                                         void* hip_stream) {
  if (!cfg || !cache_pointers_ok(cache) || !page_table || !first || !k_out || !v_out) return SWARM_ERR_NULL;
  const swarm_status bad = cache_config_status(cfg, tokens);
  if (bad != SWARM_OK) return bad;
  if (!cache_aligned(cache) || !aligned16(k_out) || !aligned16(v_out) || k_out == v_out) return SWARM_ERR_SHAPE;
  ReadArgs a{};
  a.c = cache_args(cfg, cache, page_table, first, count, tokens); a.k = k_out; a.v = v_out; a.s16 = cfg->scale_bits == 16;
  a.row_tiles = (tokens + kTile - 1) / kTile;
  a.value_tiles = tiles_touched(tokens);
  const long long keys = (long long)cfg->batch * a.row_tiles * cfg->n_kv_heads;
  const long long blocks = keys + (long long)cfg->batch * a.value_tiles * cfg->n_kv_heads;
  if (blocks > 0x7FFFFFFF) return SWARM_ERR_SHAPE;
  a.key_blocks = (int)keys;
  const dim3 grid((unsigned)blocks), block(kThreads);
  hipStream_t st = (hipStream_t)hip_stream;
  if (cfg->dtype == SWARM_BF16) {
    if (cfg->d_head == 64) hipLaunchKernelGGL((cache_read_kernel<bf16_raw, 64>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((cache_read_kernel<bf16_raw, 128>), grid, block, 0, st, a);
  } else {
    if (cfg->d_head == 64) hipLaunchKernelGGL((cache_read_kernel<float, 64>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((cache_read_kernel<float, 128>), grid, block, 0, st, a);
  }
  return launch_status();
}

extern "C" swarm_status swarm_cache_keep(const swarm_cache_config* cfg, const swarm_cache* cache, const int32_t* page_table,
                                         const int32_t* past, const int32_t* kept, const int32_t* n_kept, int32_t tokens,
                                         void* hip_stream) {
  if (!cfg || !cache_pointers_ok(cache) || !page_table || !past || !kept || !n_kept) return SWARM_ERR_NULL;
  const swarm_status bad = cache_config_status(cfg, tokens);
  if (bad != SWARM_OK) return bad;
  if (tokens > kDraft || !cache_aligned(cache) || (long long)cfg->batch * cfg->n_kv_heads > 0x7FFFFFFF) return SWARM_ERR_SHAPE;
  const CacheArgs a = cache_args(cfg, cache, page_table, past, n_kept, tokens);
  const dim3 grid((unsigned)(cfg->batch * cfg->n_kv_heads)), block(kThreads);
  if (cfg->d_head == 64) hipLaunchKernelGGL((cache_keep_kernel<64>), grid, block, 0, (hipStream_t)hip_stream, a, kept, cfg->scale_bits == 16);
  else hipLaunchKernelGGL((cache_keep_kernel<128>), grid, block, 0, (hipStream_t)hip_stream, a, kept, cfg->scale_bits == 16);
  return launch_status();
}
