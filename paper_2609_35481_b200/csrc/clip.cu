// Global norm of many gradient tensors and clipping (definition in topoep.h).
//
// Bound by memory: every element is read for the norm, then read again and written for the
// scaling.  The list of tensors is cut into chunks of kChunk elements of one tensor; blocks walk
// the chunks blockIdx.x, blockIdx.x + gridDim.x, ...
#include <climits>
#include <cmath>
#include <new>
#include <vector>

#include "layer_common.cuh"

namespace topoep {

namespace {

constexpr int kClipThreads = 512;
constexpr int kChunk = 16384;           // elements of a chunk
constexpr int kMaxBlocks = 2048;        // partial results in the workspace
constexpr float kClipEps = 1e-6f;

struct ClipTensor {
  const void* src;
  void* dst;
  long long cols, src_stride, dst_stride, elements;
  long long first_chunk;
  int dtype, pad;
};

struct ClipParams {
  const ClipTensor* tensors;
  double* partial;
  float* norm;
  long long chunks;
  int count, kind, blocks;
  float max_norm;
};

// Index of the tensor that holds chunk c: the last one whose first chunk is not above c.
__device__ __forceinline__ int tensor_of(const ClipParams& p, long long c) {
  int lo = 0, hi = p.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (p.tensors[mid].first_chunk <= c) lo = mid; else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ long long offset_of(const ClipTensor& t, long long i, long long stride) {
  return stride == t.cols ? i : i / t.cols * stride + i % t.cols;
}

__device__ __forceinline__ double join(double a, double b, int kind) {
  if (kind == 0) return a + b;
  return isnan(a) ? a : isnan(b) ? b : fmax(a, b);
}

template <typename T>
__device__ __forceinline__ void add_chunk(const ClipTensor& t, long long first, int kind, double* sum) {
  const T* src = static_cast<const T*>(t.src);
  const long long last = min(first + (long long)kChunk, t.elements);
  for (long long i = first + threadIdx.x; i < last; i += kClipThreads) {
    const float g = to_f32(src[offset_of(t, i, t.src_stride)]);
    if (kind == 0) *sum += (double)g * g;
    else *sum = join(*sum, fabs((double)g), kind);
  }
}

// Sum (or maximum) over the block in a fixed order; the result is in every thread of warp 0.
__device__ double block_join(double v, int kind, double* shared) {
  for (int o = 16; o; o >>= 1) v = join(v, __shfl_xor_sync(0xffffffffu, v, o), kind);
  if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
  __syncthreads();
  v = (threadIdx.x & 31) < kClipThreads / 32 ? shared[threadIdx.x & 31] : 0.0;
  for (int o = 16; o; o >>= 1) v = join(v, __shfl_xor_sync(0xffffffffu, v, o), kind);
  __syncthreads();
  return v;
}

__global__ void __launch_bounds__(kClipThreads) clip_norm_kernel(const ClipParams p) {
  __shared__ double shared[32];
  double sum = 0.0;
  for (long long c = blockIdx.x; c < p.chunks; c += gridDim.x) {
    const ClipTensor t = p.tensors[tensor_of(p, c)];
    const long long first = (c - t.first_chunk) * kChunk;
    if (t.dtype == TOPOEP_DTYPE_F32) add_chunk<float>(t, first, p.kind, &sum);
    else if (t.dtype == TOPOEP_DTYPE_BF16) add_chunk<__nv_bfloat16>(t, first, p.kind, &sum);
    else add_chunk<__half>(t, first, p.kind, &sum);
  }
  sum = block_join(sum, p.kind, shared);
  if (threadIdx.x == 0) p.partial[blockIdx.x] = sum;
}

template <typename T>
__device__ __forceinline__ void scale_chunk(const ClipTensor& t, long long first, float factor) {
  const T* src = static_cast<const T*>(t.src);
  T* dst = static_cast<T*>(t.dst);
  const long long last = min(first + (long long)kChunk, t.elements);
  for (long long i = first + threadIdx.x; i < last; i += kClipThreads)
    dst[offset_of(t, i, t.dst_stride)] = from_f32<T>(to_f32(src[offset_of(t, i, t.src_stride)]) * factor);
}

__global__ void __launch_bounds__(kClipThreads) clip_scale_kernel(const ClipParams p, int scale) {
  __shared__ double shared[32];
  __shared__ float factor_shared;
  double sum = 0.0;
  for (int i = threadIdx.x; i < p.blocks; i += kClipThreads) sum = join(sum, p.partial[i], p.kind);
  sum = block_join(sum, p.kind, shared);
  if (threadIdx.x == 0) {
    const float norm = (float)(p.kind == 0 ? sqrt(sum) : sum);
    if (blockIdx.x == 0) *p.norm = norm;
    const float f = p.max_norm / (norm + kClipEps);
    factor_shared = f > 1.0f ? 1.0f : f;   // a NaN stays
  }
  __syncthreads();
  if (!scale) return;
  const float factor = factor_shared;
  for (long long c = blockIdx.x; c < p.chunks; c += gridDim.x) {
    const ClipTensor t = p.tensors[tensor_of(p, c)];
    const long long first = (c - t.first_chunk) * kChunk;
    if (t.dtype == TOPOEP_DTYPE_F32) scale_chunk<float>(t, first, factor);
    else if (t.dtype == TOPOEP_DTYPE_BF16) scale_chunk<__nv_bfloat16>(t, first, factor);
    else scale_chunk<__half>(t, first, factor);
  }
}

constexpr size_t kAlign = 256;
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

}  // namespace

}  // namespace topoep

using namespace topoep;

struct topoep_clip_ctx {
  std::vector<ClipTensor> tensors;
  long long chunks;
  unsigned char* ws;
  size_t off_tensors, ws_bytes;
  int sms;
};

extern "C" int topoep_clip_create(topoep_clip_t* out, int64_t count, const topoep_grad_tensor* tensors) {
  if (!out || (count > 0 && !tensors)) return TOPOEP_ERR_NULL;
  if (count < 0 || count > (1 << 24)) return TOPOEP_ERR_SIZE;
  topoep_clip_ctx* h = new (std::nothrow) topoep_clip_ctx();
  if (!h) return TOPOEP_ERR_CONFIG;
  int rc = TOPOEP_OK;
  try {
    h->chunks = 0;
    for (int64_t i = 0; i < count && rc == TOPOEP_OK; ++i) {
      const topoep_grad_tensor& g = tensors[i];
      if (!dtype_known(g.dtype)) { rc = TOPOEP_ERR_ARG; break; }
      if (g.rows < 0 || g.cols < 0 || (g.cols > 0 && g.rows > (1ll << 48) / g.cols)) { rc = TOPOEP_ERR_SIZE; break; }
      if (g.rows == 0 || g.cols == 0) continue;
      if (!g.src) { rc = TOPOEP_ERR_NULL; break; }
      const bool in_place = !g.dst || g.dst == g.src;
      if (g.rows > 1 && (g.src_row_stride < g.cols || g.src_row_stride > (1ll << 40))) { rc = TOPOEP_ERR_SIZE; break; }
      const int64_t dst_stride = g.dst ? g.dst_row_stride : g.src_row_stride;
      if (g.rows > 1 && (dst_stride < g.cols || dst_stride > (1ll << 40))) { rc = TOPOEP_ERR_SIZE; break; }
      if (in_place && g.rows > 1 && g.src_row_stride != dst_stride) { rc = TOPOEP_ERR_ARG; break; }
      const size_t bytes = dtype_bytes(g.dtype);
      if (!aligned_to(g.src, bytes) || !aligned_to(g.dst, bytes)) { rc = TOPOEP_ERR_ALIGN; break; }
      ClipTensor t = {};
      t.src = g.src;
      t.dst = in_place ? const_cast<void*>(g.src) : g.dst;
      t.cols = g.cols;
      t.src_stride = g.rows > 1 ? g.src_row_stride : g.cols;
      t.dst_stride = g.rows > 1 ? dst_stride : g.cols;
      t.elements = g.rows * g.cols;
      t.first_chunk = h->chunks;
      t.dtype = g.dtype;
      h->chunks += (t.elements + kChunk - 1) / kChunk;
      h->tensors.push_back(t);
    }
  } catch (...) {
    rc = TOPOEP_ERR_CONFIG;
  }
  if (rc != TOPOEP_OK) { delete h; return rc; }
  h->off_tensors = align_up(sizeof(double) * kMaxBlocks);
  h->ws_bytes = h->off_tensors + align_up(sizeof(ClipTensor) * h->tensors.size());
  *out = h;
  return TOPOEP_OK;
}

extern "C" void topoep_clip_destroy(topoep_clip_t h) { delete h; }

extern "C" size_t topoep_clip_workspace_bytes(topoep_clip_t h) { return h ? h->ws_bytes : 0; }

extern "C" int topoep_clip_set_workspace(topoep_clip_t h, void* dev_ptr, size_t bytes) {
  if (!h || !dev_ptr) return TOPOEP_ERR_NULL;
  if (bytes < h->ws_bytes || !aligned_to(dev_ptr, kAlign)) return TOPOEP_ERR_WORKSPACE;
  h->ws = nullptr;
  unsigned char* ws = static_cast<unsigned char*>(dev_ptr);
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&h->sms, cudaDevAttrMultiProcessorCount, dev);
  if (e == cudaSuccess && !h->tensors.empty())
    e = cudaMemcpy(ws + h->off_tensors, h->tensors.data(), sizeof(ClipTensor) * h->tensors.size(),
                   cudaMemcpyHostToDevice);
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  if (e != cudaSuccess) return TOPOEP_ERR_CUDA;
  h->ws = ws;
  return TOPOEP_OK;
}

static int enqueue_clip(topoep_clip_t h, int kind, float max_norm, float* dev_norm, int scale,
                        cudaStream_t stream) {
  if (!h) return TOPOEP_ERR_NULL;
  if (!h->ws) return TOPOEP_ERR_WORKSPACE;
  if (kind != 0 && kind != 1) return TOPOEP_ERR_ARG;
  if (!(max_norm >= 0.0f)) return TOPOEP_ERR_ARG;
  if (!dev_norm) return TOPOEP_ERR_NULL;
  if (!aligned_to(dev_norm, 4)) return TOPOEP_ERR_ALIGN;
  ClipParams p = {};
  p.tensors = reinterpret_cast<const ClipTensor*>(h->ws + h->off_tensors);
  p.partial = reinterpret_cast<double*>(h->ws);
  p.norm = dev_norm;
  p.chunks = h->chunks;
  p.count = (int)h->tensors.size();
  p.kind = kind;
  p.max_norm = max_norm;
  long long blocks = 4ll * h->sms;
  if (blocks > kMaxBlocks) blocks = kMaxBlocks;
  if (blocks > h->chunks) blocks = h->chunks;
  if (blocks < 1) blocks = 1;
  p.blocks = (int)blocks;
  clip_norm_kernel<<<(unsigned)blocks, kClipThreads, 0, stream>>>(p);
  clip_scale_kernel<<<scale ? (unsigned)blocks : 1u, kClipThreads, 0, stream>>>(p, scale);
  return cudaGetLastError() == cudaSuccess ? TOPOEP_OK : TOPOEP_ERR_CUDA;
}

extern "C" int topoep_clip_norm(topoep_clip_t h, int kind, float* dev_norm, topoep_stream_t stream) {
  return enqueue_clip(h, kind, 0.0f, dev_norm, 0, static_cast<cudaStream_t>(stream));
}

extern "C" int topoep_clip_run(topoep_clip_t h, int kind, float max_norm, float* dev_norm,
                               topoep_stream_t stream) {
  return enqueue_clip(h, kind, max_norm, dev_norm, 1, static_cast<cudaStream_t>(stream));
}
