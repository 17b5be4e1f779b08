// Rules on rows of logits: penalties for tokens that a row's history holds, biases, a mask of allowed tokens.
//
// One pass over the logits.  A workgroup owns kColumns columns of one row: it counts the history's tokens that fall among them in
// LDS (whole numbers, so the order of the additions does not matter), adds up the biases that do, and then rewrites its columns.  The
// history is read by every workgroup of the row (from cache: 8 KB for 2048 tokens), which costs less than a pass of its own over
// the logits to mark it.
#include "kernels.h"
#include "swarm_head.h"

namespace swarm {
namespace {

constexpr int kThreads = 256;
constexpr int kColumns = 2048;
constexpr int kMaxBias = 1024;

struct LogitsArgs {
  swarm_logits_rules r;
  const void* logits;
  float* out;
  size_t pitch, out_pitch;
};

template <typename T>
__global__ __launch_bounds__(kThreads) void logits_adjust_kernel(LogitsArgs a) {
  __shared__ int count[kColumns];
  __shared__ float bias[kColumns];
  __shared__ uint32_t biased[kColumns / 32];
  const int row = blockIdx.y, c0 = blockIdx.x * kColumns, n = min(kColumns, a.r.vocab - c0);
  const int said = a.r.history ? min(max(a.r.history_len[row], 0), a.r.history_max) : 0;
  const int given = a.r.bias_ids ? min(max(a.r.bias_len[row], 0), a.r.bias_max) : 0;
  for (int i = threadIdx.x; i < kColumns; i += kThreads) count[i] = 0;
  if (threadIdx.x < kColumns / 32) biased[threadIdx.x] = 0;
  __syncthreads();
  const int32_t* history = a.r.history + (size_t)row * a.r.history_max;
  for (int i = threadIdx.x; i < said; i += kThreads) {
    const int v = history[i] - c0;
    if ((unsigned)v < (unsigned)n) atomicAdd(&count[v], 1);
  }
  const int32_t* ids = a.r.bias_ids + (size_t)row * a.r.bias_max;
  for (int i = threadIdx.x; i < given; i += kThreads) {
    const int id = ids[i], v = id - c0;
    if ((unsigned)v >= (unsigned)n) continue;
    bool first = true;                    // the first entry of an id adds up all of them, in order
    for (int e = 0; e < i; ++e) first &= ids[e] != id;
    if (!first) continue;
    float sum = 0.0f;
    for (int e = i; e < given; ++e)
      if (ids[e] == id) sum += a.r.bias[(size_t)row * a.r.bias_max + e];
    bias[v] = sum;
    atomicOr(&biased[v >> 5], 1u << (v & 31));
  }
  __syncthreads();
  const float rep = a.r.repetition ? a.r.repetition[row] : 1.0f;
  const float freq = a.r.frequency ? a.r.frequency[row] : 0.0f, pres = a.r.presence ? a.r.presence[row] : 0.0f;
  const T* in = reinterpret_cast<const T*>(a.logits) + (size_t)row * a.pitch + c0;
  float* out = a.out + (size_t)row * a.out_pitch + c0;
  const uint32_t* allowed = a.r.allowed ? a.r.allowed + (size_t)row * ((a.r.vocab + 31) >> 5) + (c0 >> 5) : nullptr;
  for (int i = threadIdx.x; i < n; i += kThreads) {
    float x = Elem<T>::load(in + i);
    const int times = count[i];
    if (times > 0) {
      x = x > 0.0f ? x / rep : x * rep;
      x = x - freq * (float)times - pres;
    }
    if ((biased[i >> 5] >> (i & 31)) & 1) x += bias[i];
    if (allowed && !((allowed[i >> 5] >> (i & 31)) & 1)) x = -INFINITY;
    out[i] = x;
  }
}

}  // namespace
}  // namespace swarm

using namespace swarm;

extern "C" swarm_status swarm_logits_adjust(const swarm_logits_rules* r, const void* logits, int32_t dtype, size_t logits_pitch,
                                            float* out, size_t out_pitch, void* hip_stream) {
  if (!r || !logits || !out) return SWARM_ERR_NULL;
  if ((r->history && !r->history_len) || (r->bias_ids && (!r->bias || !r->bias_len))) return SWARM_ERR_NULL;
  if (dtype != SWARM_F32 && dtype != SWARM_BF16) return SWARM_ERR_DTYPE;
  if (r->rows < 1 || r->rows > 65535 || r->vocab < 1 || r->vocab > (1 << 24)) return SWARM_ERR_SHAPE;
  if (r->history_max < 0 || r->history_max > (1 << 24) || r->bias_max < 0 || r->bias_max > kMaxBias) return SWARM_ERR_SHAPE;
  if (logits_pitch < (size_t)r->vocab || out_pitch < (size_t)r->vocab) return SWARM_ERR_SHAPE;
  if (((uintptr_t)logits & (dtype == SWARM_BF16 ? 1 : 3)) || ((uintptr_t)out & 3)) return SWARM_ERR_SHAPE;
  if (logits == out && (dtype != SWARM_F32 || logits_pitch != out_pitch)) return SWARM_ERR_SHAPE;
  const LogitsArgs a{*r, logits, out, logits_pitch, out_pitch};
  const dim3 grid((r->vocab + kColumns - 1) / kColumns, r->rows), block(kThreads);
  if (dtype == SWARM_BF16) hipLaunchKernelGGL(logits_adjust_kernel<bf16_raw>, grid, block, 0, (hipStream_t)hip_stream, a);
  else hipLaunchKernelGGL(logits_adjust_kernel<float>, grid, block, 0, (hipStream_t)hip_stream, a);
  return launch_status();
}
