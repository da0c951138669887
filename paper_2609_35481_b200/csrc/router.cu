// Router of an MoE layer: scores of a token's experts -> ids and weights of the chosen ones, and
// the gradient of the scores.  The definitions stand in topoep.h.
#include <algorithm>
#include <cfloat>
#include <climits>
#include <cmath>

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
  bool sigmoid, norm;
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

// ------------------------------------------------------------------ up to 512 experts, forward
//
// One warp a token, VPL logits in the registers of each lane.  262144 tokens of 256 experts leave about 190 instructions a token at the speed of
// the memory, so the choice is made in few of them:
//   1. every lane's largest choice value; k rounds of a warp maximum give the k-th largest t of the
//      32 lane maxima.  At least k values are >= t, so nothing below t is chosen, and seldom more
//      than a few others are: about nine candidates for k = 8 of 256.
//   2. the candidates' ids are compacted into shared memory, one a lane;
//   3. a candidate's place is the number of candidates before it in (value, id) order, which it
//      counts itself; the lanes with a place below k write it.
// More than 32 candidates (many equal logits) take k rounds over the registers instead.

template <typename T, int N> struct Row;   // N adjacent elements
template <> struct Row<float, 1> { using type = float; };
template <> struct Row<float, 2> { using type = float2; };
template <> struct Row<float, 4> { using type = float4; };
template <> struct Row<__nv_bfloat16, 1> { using type = __nv_bfloat16; };
template <> struct Row<__nv_bfloat16, 2> { using type = uint32_t; };
template <> struct Row<__nv_bfloat16, 4> { using type = uint2; };
template <> struct Row<__nv_bfloat16, 8> { using type = uint4; };
template <> struct Row<__half, 1> { using type = __half; };
template <> struct Row<__half, 2> { using type = uint32_t; };
template <> struct Row<__half, 4> { using type = uint2; };
template <> struct Row<__half, 8> { using type = uint4; };

// Lane's element i of a row is expert expert_of<W>(i, lane): vectors of W, lanes side by side.  Rows
// that cannot be read as vectors are read element by element into the same places, so that the
// order of every sum, and with it every bit, is the same.
template <typename T, int VPL> constexpr int kVecOf = VPL * sizeof(T) <= 16 ? VPL : 16 / (int)sizeof(T);

template <int W>
__device__ __forceinline__ int expert_of(int i, int lane) { return i / W * (32 * W) + lane * W + i % W; }

template <typename T, int VPL, bool VEC>
__device__ __forceinline__ void load_row(const T* row, int E, int lane, float (&x)[VPL]) {
  constexpr int W = kVecOf<T, VPL>;
#pragma unroll
  for (int v = 0; v < VPL / W; ++v) {
    const int at = expert_of<W>(v * W, lane);
    if (VEC && at < E) {   // E is a multiple of W
      const typename Row<T, W>::type raw = *reinterpret_cast<const typename Row<T, W>::type*>(row + at);
      const T* e = reinterpret_cast<const T*>(&raw);
#pragma unroll
      for (int i = 0; i < W; ++i) x[v * W + i] = to_f32(e[i]);
    } else {
#pragma unroll
      for (int i = 0; i < W; ++i) x[v * W + i] = !VEC && at + i < E ? to_f32(row[at + i]) : -INFINITY;
    }
  }
}

__device__ __forceinline__ float warp_max(float v) {   // of the values that are not NaN
  float r;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}

// k rounds over the registers, any number of candidates: lane j returns the j-th choice.
template <int VPL, int W>
__device__ __forceinline__ int choose_slowly(const float (&c)[VPL], int k, int lane) {
  unsigned long long last = ~0ull;
  int mine = -1;
#pragma unroll 1
  for (int j = 0; j < k; ++j) {
    unsigned long long best = 0;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      const unsigned key = order_key(c[i]);
      const unsigned long long full = key ? ((unsigned long long)key << 32) | (0xffffffffu - expert_of<W>(i, lane)) : 0ull;
      if (full < last && full > best) best = full;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      const unsigned long long other = __shfl_xor_sync(0xffffffffu, best, o);
      best = other > best ? other : best;
    }
    if (best == 0) break;
    if (lane == j) mine = (int)(0xffffffffu - (unsigned)best);
    last = best;
  }
  return mine;
}

template <typename T, int VPL, bool VEC>
__global__ void __launch_bounds__(kRouterThreads) router_forward_kernel(const RouterParams p) {
  constexpr int W = kVecOf<T, VPL>;
  __shared__ __align__(16) float values[kRouterThreads / 32][32];   // of the candidates
  __shared__ int numbers[kRouterThreads / 32][32];
  const int lane = threadIdx.x & 31;
  float* value = values[threadIdx.x >> 5];
  int* number = numbers[threadIdx.x >> 5];
  const int step = gridDim.x * (kRouterThreads / 32), k = p.k;
  long long t = (long long)blockIdx.x * (kRouterThreads / 32) + (threadIdx.x >> 5);
  const T* row = static_cast<const T*>(p.logits) + t * p.stride;
  int32_t* out_id = p.ids + t * k + lane;
  float* out_w = p.weights + t * k + lane;
  for (; t < p.tokens; t += step, row += step * p.stride, out_id += step * k, out_w += step * k) {
    float x[VPL];
    load_row<T, VPL, VEC>(row, p.E, lane, x);
    if (p.bias) {
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        const int e = expert_of<W>(i, lane);
        if (e < p.E && x[i] != -INFINITY) x[i] = sigmoid_of(x[i]) + __ldg(p.bias + e);
      }
    }
    // comparisons with a NaN are false and a maximum passes it over: it is never a candidate
    float left = x[0], at_least = -INFINITY;
#pragma unroll
    for (int i = 1; i < VPL; ++i) left = fmaxf(left, x[i]);
    const float top = warp_max(fmaxf(left, -INFINITY));
    if (VPL > 1) {
      at_least = top;
#pragma unroll 7
      for (int j = 1; j < k; ++j) {
        if (left == at_least) left = -INFINITY;
        at_least = warp_max(left);
      }
    }
    at_least = fmaxf(at_least, -FLT_MAX);   // -inf is no candidate
    unsigned mine = 0;
#pragma unroll
    for (int i = 0; i < VPL; ++i)
      if (x[i] >= at_least) mine |= 1u << i;
    if (p.mask && p.mask[t] == 0) mine = 0;
    int n = 0;
    value[lane] = -INFINITY;
    for (unsigned some = __ballot_sync(0xffffffffu, mine != 0); some; some = __ballot_sync(0xffffffffu, mine != 0)) {
      const int at = n + __popc(some & ((1u << lane) - 1));
      if (mine && at < 32) number[at] = expert_of<W>(__ffs(mine) - 1, lane);
      mine &= mine - 1;
      n += __popc(some);
    }
    int id = -1;
    float z = 0.0f;
    __syncwarp();
    if (n <= 32) {
      float c = -INFINITY;
      if (lane < n) {
        id = number[lane];
        c = z = to_f32(row[id]);
        if (p.bias) c = sigmoid_of(z) + __ldg(p.bias + id);
        value[lane] = c;
      }
      __syncwarp();
      int place = 0;
      for (int j = 0; j < n; j += 4) {
        const float4 other = *reinterpret_cast<const float4*>(value + j);
        place += (other.x > c) + (other.y > c) + (other.z > c) + (other.w > c);
      }
      if (lane >= n) place = lane;
      // equal values share a place and leave another empty: then ids count too
      if (__reduce_or_sync(0xffffffffu, 1u << place) != 0xffffffffu && lane < n) {
        place = 0;
        for (int j = 0; j < n; ++j) place += value[j] > c || (value[j] == c && number[j] < id);
      }
      __syncwarp();
      if (lane < n) {
        value[place] = z;
        number[place] = id;
      }
      __syncwarp();
      id = -1;
      if (lane < min(n, k)) {   // lane j now has the j-th choice
        z = value[lane];
        id = number[lane];
      }
      __syncwarp();
    } else {
      id = choose_slowly<VPL, W>(x, k, lane);
      if (id >= 0) z = to_f32(row[id]);
    }
    float w = 0.0f;
    if (p.sigmoid) {
      if (id >= 0) w = sigmoid_of(z);
      if (p.norm) w = __fdividef(w, warp_sum(w) + kSigmoidEps);
    } else {
      if (id >= 0) w = expf(z - top);
      float sum = w;
      if (!p.norm) {   // over all experts
        sum = 0.0f;
#pragma unroll
        for (int i = 0; i < VPL; ++i) sum += __expf(x[i] - top);
      }
      w = __fdividef(w, warp_sum(sum));
    }
    if (lane < k) {
      *out_id = id;
      *out_w = id >= 0 ? w * p.scale : 0.0f;
    }
  }
}

// Enough warps for every SM to be full, or one a token.
unsigned router_blocks(long long tokens, int sms, int threads_per_token, int blocks_per_sm) {
  const long long per = kRouterThreads / threads_per_token, wanted = (tokens + per - 1) / per;
  return (unsigned)std::min(wanted, (long long)sms * blocks_per_sm);
}

template <typename T, int VPL>
cudaError_t launch_forward_rows(const RouterParams& p, int sms, cudaStream_t stream) {
  constexpr int W = kVecOf<T, VPL>;
  const unsigned blocks = router_blocks(p.tokens, sms, 32, 2048 / kRouterThreads);
  if (p.E % W == 0 && aligned_to(p.logits, W * sizeof(T)) && (p.tokens == 1 || p.stride % W == 0))
    router_forward_kernel<T, VPL, true><<<blocks, kRouterThreads, 0, stream>>>(p);
  else
    router_forward_kernel<T, VPL, false><<<blocks, kRouterThreads, 0, stream>>>(p);
  return cudaGetLastError();
}

template <typename T, bool SIGMOID, bool NORM>
cudaError_t launch_forward(const RouterParams& p, int sms, cudaStream_t stream) {
  if (p.E <= 32) return launch_forward_rows<T, 1>(p, sms, stream);
  if (p.E <= 64) return launch_forward_rows<T, 2>(p, sms, stream);
  if (p.E <= 128) return launch_forward_rows<T, 4>(p, sms, stream);
  if (p.E <= 256) return launch_forward_rows<T, 8>(p, sms, stream);
  if (p.E <= 512) return launch_forward_rows<T, 16>(p, sms, stream);
  const long long blocks = (p.tokens + kRouterThreads / 32 - 1) / (kRouterThreads / 32);
  router_forward_any_kernel<T, SIGMOID, NORM><<<(unsigned)blocks, kRouterThreads, 0, stream>>>(p);
  return cudaGetLastError();
}

template <typename T, bool SIGMOID, bool NORM>
cudaError_t launch_backward(const RouterParams& p, int, cudaStream_t stream) {
  const long long blocks = (p.tokens + kRouterThreads / 32 - 1) / (kRouterThreads / 32);
  router_backward_any_kernel<T, SIGMOID, NORM><<<(unsigned)blocks, kRouterThreads, 0, stream>>>(p);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_typed(const RouterParams& p, bool sigmoid, bool norm, bool forward, int sms, cudaStream_t s) {
  if (forward)
    return sigmoid ? (norm ? launch_forward<T, true, true>(p, sms, s) : launch_forward<T, true, false>(p, sms, s))
                   : (norm ? launch_forward<T, false, true>(p, sms, s) : launch_forward<T, false, false>(p, sms, s));
  return sigmoid ? (norm ? launch_backward<T, true, true>(p, sms, s) : launch_backward<T, true, false>(p, sms, s))
                 : (norm ? launch_backward<T, false, true>(p, sms, s) : launch_backward<T, false, false>(p, sms, s));
}

int launch(const topoep_router_config* cfg, RouterParams& p, bool forward, cudaStream_t s) {
  const bool sigmoid = cfg->score == TOPOEP_SCORE_SIGMOID, norm = cfg->normalize != 0;
  p.sigmoid = sigmoid;
  p.norm = norm;
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return TOPOEP_ERR_CUDA;
  switch (cfg->dtype) {
    case TOPOEP_DTYPE_F32: e = launch_typed<float>(p, sigmoid, norm, forward, sms, s); break;
    case TOPOEP_DTYPE_BF16: e = launch_typed<__nv_bfloat16>(p, sigmoid, norm, forward, sms, s); break;
    default: e = launch_typed<__half>(p, sigmoid, norm, forward, sms, s); break;
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
