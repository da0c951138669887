// Router of an MoE layer: scores of a token's experts -> ids and weights of the chosen ones, and
// the gradient of the scores.  The definitions stand in topoep.h.
#include <cmath>
#include <climits>

#include "layer_common.cuh"

namespace topoep {

namespace {

constexpr int kRouterThreads = 128;
constexpr float kSigmoidEps = 1e-20f;

struct RouterParams {
  const void* logits;
  const float* bias;
  const uint8_t* mask;
  int32_t* ids;
  float* weights;
  const float* grad_weights;
  void* grad;
  long long stride, grad_stride, tokens;
  int E, k;
  float scale;
};

__device__ __forceinline__ float sigmoid_of(float l) { return 1.0f / (1.0f + expf(-l)); }

// Orders floats like unsigned integers; what may never be chosen (-inf, NaN) is 0.
__device__ __forceinline__ unsigned order_key(float c) {
  if (!(c > -INFINITY)) return 0u;
  const unsigned u = __float_as_uint(c == 0.0f ? 0.0f : c);   // -0 and +0 tie
  return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Ids and weights of one token whose j-th choice is in lane j (id -1: none left); z is the logit of
// the choice, all_sum the softmax denominator over all experts relative to the first choice.
template <bool SIGMOID, bool NORM>
__device__ __forceinline__ float weight_of(int id, float z, float all_sum, float scale) {
  const float top = __shfl_sync(0xffffffffu, z, 0);
  float w;
  if (SIGMOID) {
    w = id >= 0 ? sigmoid_of(z) : 0.0f;
    if (NORM) w = w / (warp_sum(w) + kSigmoidEps);
  } else {
    w = id >= 0 ? expf(z - top) : 0.0f;
    w = w / (NORM ? warp_sum(w) : all_sum);
  }
  return id >= 0 ? w * scale : 0.0f;
}

// Any number of experts: one warp a token, k rounds over the row, each taking the largest
// (choice, -id) below the one taken before.  The row is read from L1/L2 after the first round.
template <typename T, bool SIGMOID, bool NORM>
__global__ void __launch_bounds__(kRouterThreads) router_forward_any_kernel(const RouterParams p) {
  const int lane = threadIdx.x & 31;
  const long long t = (long long)blockIdx.x * (kRouterThreads / 32) + (threadIdx.x >> 5);
  if (t >= p.tokens) return;
  const T* row = static_cast<const T*>(p.logits) + t * p.stride;
  const bool masked = p.mask && p.mask[t] == 0;
  unsigned long long last = ~0ull;
  int my_id = -1;
  for (int j = 0; j < p.k && !masked; ++j) {
    unsigned long long best = 0;
    for (int i = lane; i < p.E; i += 32) {
      const float l = to_f32(row[i]);
      unsigned key = order_key(l);
      if (p.bias && key) key = order_key(sigmoid_of(l) + p.bias[i]);
      const unsigned long long full = key ? ((unsigned long long)key << 32) | (0xffffffffu - i) : 0ull;
      if (full < last && full > best) best = full;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      const unsigned long long other = __shfl_xor_sync(0xffffffffu, best, o);
      best = other > best ? other : best;
    }
    if (best == 0) break;
    if (lane == j) my_id = (int)(0xffffffffu - (unsigned)best);
    last = best;
  }
  const float z = my_id >= 0 ? to_f32(row[my_id]) : 0.0f;
  float all = 0.0f;
  if (!SIGMOID && !NORM) {
    const float top = __shfl_sync(0xffffffffu, z, 0);
    for (int i = lane; i < p.E; i += 32) all += expf(to_f32(row[i]) - top);
    all = warp_sum(all);
  }
  const float w = weight_of<SIGMOID, NORM>(my_id, z, all, p.scale);
  if (lane < p.k) {
    p.ids[t * p.k + lane] = my_id;
    p.weights[t * p.k + lane] = w;
  }
}

template <typename T, bool SIGMOID, bool NORM>
__global__ void __launch_bounds__(kRouterThreads) router_backward_any_kernel(const RouterParams p) {
  const int lane = threadIdx.x & 31;
  const long long t = (long long)blockIdx.x * (kRouterThreads / 32) + (threadIdx.x >> 5);
  if (t >= p.tokens) return;
  const T* row = static_cast<const T*>(p.logits) + t * p.stride;
  T* grad = static_cast<T*>(p.grad) + t * p.grad_stride;
  int id = lane < p.k ? p.ids[t * p.k + lane] : -1;
  if (id >= p.E) id = -1;
  const bool taken = id >= 0;
  const float w = taken ? p.weights[t * p.k + lane] : 0.0f;
  const float dw = taken ? p.grad_weights[t * p.k + lane] : 0.0f;
  const float wdw = w * dw;
  const float m = warp_sum(wdw) / p.scale;
  float part = NORM ? w * (dw - m) : wdw;
  if (SIGMOID && taken) part = part / (1.0f + expf(to_f32(row[id])));
  if (!SIGMOID && !NORM && __any_sync(0xffffffffu, taken)) {
    float top = -INFINITY;
    for (int i = lane; i < p.E; i += 32) top = fmaxf(top, to_f32(row[i]));
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    float sum = 0.0f;
    for (int i = lane; i < p.E; i += 32) sum += expf(to_f32(row[i]) - top);
    sum = warp_sum(sum);
    const float c = -m * p.scale / sum;
    for (int i = lane; i < p.E; i += 32) grad[i] = from_f32<T>(expf(to_f32(row[i]) - top) * c);
    if (taken) part += expf(to_f32(row[id]) - top) * c;
  } else {
    for (int i = lane; i < p.E; i += 32) grad[i] = from_f32<T>(0.0f);
  }
  __syncwarp();   // the chosen places are written after the row
  if (taken) grad[id] = from_f32<T>(part);
}

template <typename T, bool SIGMOID, bool NORM>
cudaError_t launch_forward(const RouterParams& p, cudaStream_t stream) {
  const long long blocks = (p.tokens + kRouterThreads / 32 - 1) / (kRouterThreads / 32);
  router_forward_any_kernel<T, SIGMOID, NORM><<<(unsigned)blocks, kRouterThreads, 0, stream>>>(p);
  return cudaGetLastError();
}

template <typename T, bool SIGMOID, bool NORM>
cudaError_t launch_backward(const RouterParams& p, cudaStream_t stream) {
  const long long blocks = (p.tokens + kRouterThreads / 32 - 1) / (kRouterThreads / 32);
  router_backward_any_kernel<T, SIGMOID, NORM><<<(unsigned)blocks, kRouterThreads, 0, stream>>>(p);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_typed(const RouterParams& p, bool sigmoid, bool norm, bool forward, cudaStream_t s) {
  if (forward)
    return sigmoid ? (norm ? launch_forward<T, true, true>(p, s) : launch_forward<T, true, false>(p, s))
                   : (norm ? launch_forward<T, false, true>(p, s) : launch_forward<T, false, false>(p, s));
  return sigmoid ? (norm ? launch_backward<T, true, true>(p, s) : launch_backward<T, true, false>(p, s))
                 : (norm ? launch_backward<T, false, true>(p, s) : launch_backward<T, false, false>(p, s));
}

int launch(const topoep_router_config* cfg, const RouterParams& p, bool forward, cudaStream_t s) {
  const bool sigmoid = cfg->score == TOPOEP_SCORE_SIGMOID, norm = cfg->normalize != 0;
  cudaError_t e;
  switch (cfg->dtype) {
    case TOPOEP_DTYPE_F32: e = launch_typed<float>(p, sigmoid, norm, forward, s); break;
    case TOPOEP_DTYPE_BF16: e = launch_typed<__nv_bfloat16>(p, sigmoid, norm, forward, s); break;
    default: e = launch_typed<__half>(p, sigmoid, norm, forward, s); break;
  }
  return e == cudaSuccess ? TOPOEP_OK : TOPOEP_ERR_CUDA;
}

int check(const topoep_router_config* c, int64_t row_stride, int64_t tokens) {
  if (!c) return TOPOEP_ERR_NULL;
  if (c->experts < 1 || c->experts > 16384 || c->top_k < 1 || c->top_k > 32 ||
      c->top_k > c->experts)
    return TOPOEP_ERR_CONFIG;
  if (!dtype_known(c->dtype) || (c->score != TOPOEP_SCORE_SOFTMAX && c->score != TOPOEP_SCORE_SIGMOID) ||
      (c->normalize != 0 && c->normalize != 1) || !(c->scale > 0.0f) || !std::isfinite(c->scale))
    return TOPOEP_ERR_ARG;
  // one block index per group of tokens, 64-bit element offsets
  if (tokens < 0 || tokens > (1ll << 31) || row_stride < c->experts || row_stride > (1ll << 32))
    return TOPOEP_ERR_SIZE;
  return TOPOEP_OK;
}

}  // namespace

}  // namespace topoep

using namespace topoep;

extern "C" int topoep_router_forward(const topoep_router_config* cfg, const void* dev_logits,
                                     int64_t row_stride, int64_t tokens, const float* dev_bias,
                                     const uint8_t* dev_token_mask, int32_t* dev_topk_ids,
                                     float* dev_weights, topoep_stream_t stream) {
  const int rc = check(cfg, row_stride, tokens);
  if (rc != TOPOEP_OK) return rc;
  if (dev_bias && cfg->score != TOPOEP_SCORE_SIGMOID) return TOPOEP_ERR_ARG;
  if (tokens == 0) return TOPOEP_OK;
  if (!dev_logits || !dev_topk_ids || !dev_weights) return TOPOEP_ERR_NULL;
  if (!aligned_to(dev_logits, dtype_bytes(cfg->dtype)) || !aligned_to(dev_topk_ids, 4) ||
      !aligned_to(dev_weights, 4) || !aligned_to(dev_bias, 4))
    return TOPOEP_ERR_ALIGN;
  RouterParams p = {};
  p.logits = dev_logits;
  p.stride = row_stride;
  p.tokens = tokens;
  p.bias = dev_bias;
  p.mask = dev_token_mask;
  p.ids = dev_topk_ids;
  p.weights = dev_weights;
  p.E = cfg->experts;
  p.k = cfg->top_k;
  p.scale = cfg->scale;
  return launch(cfg, p, true, static_cast<cudaStream_t>(stream));
}

extern "C" int topoep_router_backward(const topoep_router_config* cfg, const void* dev_logits,
                                      int64_t row_stride, int64_t tokens,
                                      const int32_t* dev_topk_ids, const float* dev_weights,
                                      const float* dev_grad_weights, void* dev_grad_logits,
                                      int64_t grad_row_stride, topoep_stream_t stream) {
  const int rc = check(cfg, row_stride, tokens);
  if (rc != TOPOEP_OK) return rc;
  if (grad_row_stride < cfg->experts || grad_row_stride > (1ll << 32)) return TOPOEP_ERR_SIZE;
  if (tokens == 0) return TOPOEP_OK;
  if (!dev_logits || !dev_topk_ids || !dev_weights || !dev_grad_weights || !dev_grad_logits)
    return TOPOEP_ERR_NULL;
  if (!aligned_to(dev_logits, dtype_bytes(cfg->dtype)) || !aligned_to(dev_topk_ids, 4) ||
      !aligned_to(dev_grad_logits, dtype_bytes(cfg->dtype)) || !aligned_to(dev_weights, 4) ||
      !aligned_to(dev_grad_weights, 4))
    return TOPOEP_ERR_ALIGN;
  RouterParams p = {};
  p.logits = dev_logits;
  p.stride = row_stride;
  p.tokens = tokens;
  p.ids = const_cast<int32_t*>(dev_topk_ids);
  p.weights = const_cast<float*>(dev_weights);
  p.grad_weights = dev_grad_weights;
  p.grad = dev_grad_logits;
  p.grad_stride = grad_row_stride;
  p.E = cfg->experts;
  p.k = cfg->top_k;
  p.scale = cfg->scale;
  return launch(cfg, p, false, static_cast<cudaStream_t>(stream));
}
