// Expert layer of a few tokens on the physical instances a plan names (definition in topoep.h).
//
// Bound by memory: every block that some id names is read once, 6 * hidden * ffn bytes, and meets
// at most a few tokens.
#include <algorithm>
#include <new>

#include "layer_common.cuh"

namespace topoep {

namespace {

constexpr int kAnyThreads = 256;

struct ExpertsParams {
  const __nv_bfloat16* main;
  const __nv_bfloat16* replica;
  const __nv_bfloat16* x;
  __nv_bfloat16* y;
  const int32_t* ids;
  const float* weights;
  float* h;
  uint32_t* status;
  long long x_stride, y_stride;
  int tokens, k, H, F, e_loc, slots, instances;
};

__device__ __forceinline__ const __nv_bfloat16* block_of(const ExpertsParams& p, int inst) {
  const int s = p.e_loc + p.slots, r = inst / s, l = inst - r * s;
  const long long per = 3ll * p.H * p.F;
  return l < p.e_loc ? p.main + (long long)(r * p.e_loc + l) * per
                     : p.replica + (long long)(r * p.slots + l - p.e_loc) * per;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Any sizes and alignment: one warp for an (assignment, row of gate and up).
__global__ void __launch_bounds__(kAnyThreads) experts_gate_any_kernel(const ExpertsParams p) {
  const int lane = threadIdx.x & 31, a = blockIdx.y, f = blockIdx.x * (kAnyThreads / 32) + (threadIdx.x >> 5);
  const int inst = p.ids[a];
  if (inst < 0 || inst >= p.instances) {
    if (inst != -1 && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(p.status, TOPOEP_FLAG_BAD_ID);
    return;
  }
  if (f >= p.F) return;
  const __nv_bfloat16* blk = block_of(p, inst);
  const __nv_bfloat16 *wg = blk + (long long)f * p.H, *wu = wg + (long long)p.F * p.H;
  const __nv_bfloat16* x = p.x + (a / p.k) * p.x_stride;
  float g = 0.0f, u = 0.0f;
  for (int i = lane; i < p.H; i += 32) {
    const float v = to_f32(x[i]);
    g += v * to_f32(wg[i]);
    u += v * to_f32(wu[i]);
  }
  g = warp_sum(g);
  u = warp_sum(u);
  if (lane == 0) p.h[(long long)a * p.F + f] = g / (1.0f + expf(-g)) * u;
}

__global__ void __launch_bounds__(kAnyThreads) experts_down_any_kernel(const ExpertsParams p) {
  const int lane = threadIdx.x & 31, t = blockIdx.y, c = blockIdx.x * (kAnyThreads / 32) + (threadIdx.x >> 5);
  if (c >= p.H) return;
  float y = 0.0f;
  for (int j = 0; j < p.k; ++j) {
    const int a = t * p.k + j, inst = p.ids[a];
    if (inst < 0 || inst >= p.instances) continue;
    const __nv_bfloat16* wd = block_of(p, inst) + 2ll * p.F * p.H + (long long)c * p.F;
    const float* h = p.h + (long long)a * p.F;
    float s = 0.0f;
    for (int i = lane; i < p.F; i += 32) s += h[i] * to_f32(wd[i]);
    y += p.weights[a] * warp_sum(s);
  }
  if (lane == 0) p.y[t * p.y_stride + c] = __float2bfloat16_rn(y);
}

constexpr size_t kAlign = 256;
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

}  // namespace

}  // namespace topoep

using namespace topoep;

struct topoep_experts_ctx {
  int ranks, e_loc, slots, instances, hidden, ffn, top_k, max_tokens;
  const void* main;
  const void* replica;
  bool have_params;
  unsigned char* ws;
  size_t ws_bytes, off_h;
};

extern "C" int topoep_experts_create(topoep_experts_t* out, int ranks, int experts_per_rank,
                                     int slots_per_rank, int hidden, int ffn, int top_k,
                                     int max_tokens) {
  if (!out) return TOPOEP_ERR_NULL;
  if (ranks < 1 || experts_per_rank < 0 || slots_per_rank < 0 || hidden < 1 || hidden > 65536 ||
      ffn < 1 || ffn > 65536 || top_k < 1 || top_k > 16 || max_tokens < 1 || max_tokens > 128)
    return TOPOEP_ERR_CONFIG;
  const long long s = (long long)experts_per_rank + slots_per_rank;
  if (s < 1 || s > 8192 || s * ranks > 8192) return TOPOEP_ERR_CONFIG;
  topoep_experts_ctx* h = new (std::nothrow) topoep_experts_ctx();
  if (!h) return TOPOEP_ERR_CONFIG;
  h->ranks = ranks;
  h->e_loc = experts_per_rank;
  h->slots = slots_per_rank;
  h->instances = (int)(s * ranks);
  h->hidden = hidden;
  h->ffn = ffn;
  h->top_k = top_k;
  h->max_tokens = max_tokens;
  h->off_h = kAlign;
  h->ws_bytes = h->off_h + align_up((size_t)4 * max_tokens * top_k * ffn);
  *out = h;
  return TOPOEP_OK;
}

extern "C" void topoep_experts_destroy(topoep_experts_t h) { delete h; }

extern "C" size_t topoep_experts_workspace_bytes(topoep_experts_t h) { return h ? h->ws_bytes : 0; }

extern "C" int topoep_experts_set_workspace(topoep_experts_t h, void* dev_ptr, size_t bytes) {
  if (!h || !dev_ptr) return TOPOEP_ERR_NULL;
  if (bytes < h->ws_bytes || !aligned_to(dev_ptr, kAlign)) return TOPOEP_ERR_WORKSPACE;
  h->ws = nullptr;
  cudaError_t e = cudaMemset(dev_ptr, 0, kAlign);
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  if (e != cudaSuccess) return TOPOEP_ERR_CUDA;
  h->ws = static_cast<unsigned char*>(dev_ptr);
  return TOPOEP_OK;
}

extern "C" int topoep_experts_set_params(topoep_experts_t h, const void* dev_main_params,
                                         const void* dev_replica_buf) {
  if (!h) return TOPOEP_ERR_NULL;
  if ((h->e_loc > 0 && !dev_main_params) || (h->slots > 0 && !dev_replica_buf)) return TOPOEP_ERR_NULL;
  if (!aligned_to(dev_main_params, 16) || !aligned_to(dev_replica_buf, 16)) return TOPOEP_ERR_ALIGN;
  h->main = dev_main_params;
  h->replica = dev_replica_buf;
  h->have_params = true;
  return TOPOEP_OK;
}

extern "C" int topoep_experts_forward(topoep_experts_t h, const void* dev_x, int64_t x_row_stride,
                                      const int32_t* dev_ids, const float* dev_weights, int tokens,
                                      void* dev_y, int64_t y_row_stride, topoep_stream_t stream) {
  if (!h) return TOPOEP_ERR_NULL;
  if (!h->ws) return TOPOEP_ERR_WORKSPACE;
  if (!h->have_params) return TOPOEP_ERR_NULL;
  if (tokens < 0 || tokens > h->max_tokens || x_row_stride < h->hidden ||
      y_row_stride < h->hidden || x_row_stride > (1ll << 32) || y_row_stride > (1ll << 32))
    return TOPOEP_ERR_SIZE;
  if (tokens == 0) return TOPOEP_OK;
  if (!dev_x || !dev_ids || !dev_weights || !dev_y) return TOPOEP_ERR_NULL;
  if (!aligned_to(dev_x, 2) || !aligned_to(dev_y, 2) || !aligned_to(dev_ids, 4) || !aligned_to(dev_weights, 4))
    return TOPOEP_ERR_ALIGN;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  ExpertsParams p = {};
  p.main = static_cast<const __nv_bfloat16*>(h->main);
  p.replica = static_cast<const __nv_bfloat16*>(h->replica);
  p.x = static_cast<const __nv_bfloat16*>(dev_x);
  p.y = static_cast<__nv_bfloat16*>(dev_y);
  p.ids = dev_ids;
  p.weights = dev_weights;
  p.h = reinterpret_cast<float*>(h->ws + h->off_h);
  p.status = reinterpret_cast<uint32_t*>(h->ws);
  p.x_stride = x_row_stride;
  p.y_stride = y_row_stride;
  p.tokens = tokens;
  p.k = h->top_k;
  p.H = h->hidden;
  p.F = h->ffn;
  p.e_loc = h->e_loc;
  p.slots = h->slots;
  p.instances = h->instances;
  const int per = kAnyThreads / 32;
  experts_gate_any_kernel<<<dim3((p.F + per - 1) / per, tokens * p.k), kAnyThreads, 0, st>>>(p);
  experts_down_any_kernel<<<dim3((p.H + per - 1) / per, tokens), kAnyThreads, 0, st>>>(p);
  return cudaGetLastError() == cudaSuccess ? TOPOEP_OK : TOPOEP_ERR_CUDA;
}

extern "C" int topoep_experts_read_status(topoep_experts_t h, uint32_t* host_flags) {
  if (!h || !host_flags) return TOPOEP_ERR_NULL;
  if (!h->ws) return TOPOEP_ERR_WORKSPACE;
  cudaError_t e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = cudaMemcpy(host_flags, h->ws, 4, cudaMemcpyDeviceToHost);
  if (e == cudaSuccess) e = cudaMemset(h->ws, 0, 4);
  return e == cudaSuccess ? TOPOEP_OK : TOPOEP_ERR_CUDA;
}
