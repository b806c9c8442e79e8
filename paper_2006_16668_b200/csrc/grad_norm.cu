// The norm of many gradients together, norm = sqrt(sum g^2), and their clipping to a bound:
// out = g min(1, max_norm / norm).
//
// The list of tensors travels in the launch's own parameters (up to 1024 tensors per launch), so a call copies nothing to
// the device and can be captured.  A block takes chunks of 16384 elements of the concatenated tensors, in a fixed
// order, so the sums have the same bits from run to run.  Bound by HBM: the norm reads every gradient once, the
// clipping reads and writes it once (4e8 elements of both types, 0.99 GB: 554 us for both calls, 5.4 TB/s).
// Squares of 16 bytes are added in fp32 where their largest lies between 2^-40 and 2^60 (nothing overflows, and what
// underflows is below 2^-24 of it), otherwise in fp64; everything beyond 16 bytes is added in fp64.
#include <algorithm>

#include "checks.cuh"
#include "pack.cuh"
#include "plan.cuh"

namespace gshard {

namespace {

constexpr int kChunk = 16384;                  // elements per work item
constexpr int kThreads = 256;
constexpr int kBlocksPerSm = 8;
constexpr int kMaxBlocks = 148 * kBlocksPerSm;    // the grid does not depend on the GPU: neither do the sums

// count: elements times 2, plus 1 for bf16
template <int N> struct GradTable {
  const void* in[N];
  void* out[N];
  long long count[N];
  int first[N + 1];                            // first chunk of each tensor
  int n;
};

// Elements that p lies behind a 16-byte boundary.
template <typename T>
__host__ __device__ __forceinline__ int skew(const T* p) { return (int)((reinterpret_cast<uintptr_t>(p) & 15u) / sizeof(T)); }

// A tensor's chunks are cut at 16-byte boundaries of its memory, so that single elements occur at its ends only.
struct Range { long long begin, end; };
template <typename T>
__device__ __forceinline__ Range range_of(const T* p, int chunk, long long count) {
  const long long at = (long long)chunk * kChunk - skew(p);
  return {max(0ll, at), min(count, at + kChunk)};
}

// the tensor that owns a chunk
template <int N>
__device__ __forceinline__ int owner_of(const GradTable<N>& t, int chunk) {
  int lo = 0, hi = t.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.first[mid] <= chunk) lo = mid; else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ double square(float v) { return (double)v * (double)v; }

template <typename T, int W>
__device__ __forceinline__ double squares(const Pack<T, W>& p) {
  float top = 0.f, s = 0.f;
#pragma unroll
  for (int j = 0; j < W; ++j) {
    const float v = p.get(j);
    top = fmaxf(top, fabsf(v));
    s = fmaf(v, v, s);
  }
  if (top == 0.f || (top > 0x1p-40f && top < 0x1p60f)) {
    if (s == s) return (double)s;              // a NaN hides from the maximum
  }
  double d = 0.0;
#pragma unroll
  for (int j = 0; j < W; ++j) d += square(p.get(j));
  return d;
}

// f(pack or element, index) over [begin, end) of a tensor: 16-byte packs where the address allows, single elements around
// them (and throughout where `other`, the tensor written, is aligned differently).
template <typename T, typename FP, typename FE>
__device__ __forceinline__ void walk(const T* p, const void* other, long long begin, long long end, FP on_pack, FE on_element) {
  constexpr int W = 16 / (int)sizeof(T);
  const bool packs = ((reinterpret_cast<uintptr_t>(p) ^ reinterpret_cast<uintptr_t>(other)) & 15u) == 0;
  const int off = skew(p + begin);
  const long long head = packs ? min(end, begin + (off ? W - off : 0)) : end;
  const long long tail = head + (end - head) / W * W;
  for (long long i = begin + threadIdx.x; i < head; i += kThreads) on_element(i);
  constexpr int U = 8;                         // packs in flight
  for (long long i = head + (long long)threadIdx.x * W; i < tail; i += (long long)kThreads * W * U) {
    Pack<T, W> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + (long long)u * kThreads * W < tail) v[u].load_once(p + i + (long long)u * kThreads * W);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + (long long)u * kThreads * W < tail) on_pack(v[u], i + (long long)u * kThreads * W);
  }
  for (long long i = tail + threadIdx.x; i < end; i += kThreads) on_element(i);
}

template <typename T>
__device__ __forceinline__ double sum_chunk(const T* p, int chunk, long long count) {
  constexpr int W = 16 / (int)sizeof(T);
  const Range r = range_of(p, chunk, count);
  double s = 0.0;
  walk(p, p, r.begin, r.end, [&](const Pack<T, W>& v, long long) { s += squares<T, W>(v); }, [&](long long i) { s += square(to_f32(p[i])); });
  return s;
}

__device__ __forceinline__ double block_sum(double s) {
  __shared__ double part[kThreads / 32];
#pragma unroll
  for (int off = 16; off; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
  __syncthreads();
  s = 0.0;
#pragma unroll
  for (int i = 0; i < kThreads / 32; ++i) s += part[i];
  return s;
}

template <int N>
__global__ void __launch_bounds__(kThreads) grad_sum_kernel(const __grid_constant__ GradTable<N> t, double* partial) {
  double s = 0.0;
  for (int chunk = blockIdx.x; chunk < t.first[t.n]; chunk += gridDim.x) {
    const int i = owner_of(t, chunk);
    s += t.count[i] & 1 ? sum_chunk(static_cast<const __nv_bfloat16*>(t.in[i]), chunk - t.first[i], t.count[i] >> 1)
                        : sum_chunk(static_cast<const float*>(t.in[i]), chunk - t.first[i], t.count[i] >> 1);
  }
  s = block_sum(s);
  if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

__global__ void __launch_bounds__(kThreads) grad_sum_finish_kernel(const double* partial, int n, double* sumsq) {
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += kThreads) s += partial[i];
  s = block_sum(s);
  if (threadIdx.x == 0) *sumsq = s;
}

// The factor is a * b: a = 1, or 2^-126 where the factor lies below the normal numbers, of which fp32 keeps few bits or none, though
// the products may be any number.  (What v a loses to underflow is below half of fp32's smallest number in the product.  fp64 products on that
// branch made the call 8 % slower for everyone.)
template <typename T>
__device__ __forceinline__ void scale_chunk(const T* p, T* q, int chunk, long long count, float a, float b) {
  constexpr int W = 16 / (int)sizeof(T);
  const Range r = range_of(p, chunk, count);
  walk(p, q, r.begin, r.end,
       [&](const Pack<T, W>& v, long long i) {
         if (b == 1.f) {                    // a copy, bit by bit: also of what is no number
           *reinterpret_cast<uint4*>(q + i) = v.raw;
           return;
         }
         float f[W];
#pragma unroll
         for (int j = 0; j < W; ++j) f[j] = v.get(j) * a * b;
         store_pack<T, W>(q + i, f);
       },
       [&](long long i) { q[i] = b == 1.f ? p[i] : from_f32<T>(to_f32(p[i]) * a * b); });
}

template <int N>
__global__ void __launch_bounds__(kThreads) grad_clip_kernel(const __grid_constant__ GradTable<N> t, const double* sumsq, float max_norm,
                                                             float* norm_out) {
  const double norm = sqrt(*sumsq);
  // a norm that the caller sees as infinite or NaN leaves the gradients unchanged: finite ones whose norm is beyond fp32 among them
  const double value = norm > (double)max_norm && (float)norm < INFINITY ? (double)max_norm / norm : 1.0;
  const bool low = value < 0x1p-126;
  const float a = low ? 0x1p-126f : 1.f, b = low ? fminf((float)(value * 0x1p126), 0x1.fffffep-1f) : (float)value;      // b == 1: a copy
  if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
  // from the end: the norm has read the last chunks last, and L2 still holds them
  for (int chunk = t.first[t.n] - 1 - (int)blockIdx.x; chunk >= 0; chunk -= gridDim.x) {
    const int i = owner_of(t, chunk);
    if (b == 1.f && t.in[i] == t.out[i]) continue;
    if (t.count[i] & 1)
      scale_chunk(static_cast<const __nv_bfloat16*>(t.in[i]), static_cast<__nv_bfloat16*>(t.out[i]), chunk - t.first[i], t.count[i] >> 1, a, b);
    else
      scale_chunk(static_cast<const float*>(t.in[i]), static_cast<float*>(t.out[i]), chunk - t.first[i], t.count[i] >> 1, a, b);
  }
}

int grad_validate(const gshard_grad_list* l, bool clip) {
  if (!l || l->n < 0) return GSHARD_ERR_INVALID_ARG;
  if (l->n == 0) return GSHARD_OK;
  if (!l->grads || !l->counts || !l->dtypes || (clip && !l->outs)) return GSHARD_ERR_INVALID_ARG;
  for (int i = 0; i < l->n; ++i) {
    if (l->dtypes[i] != GSHARD_F32 && l->dtypes[i] != GSHARD_BF16) return GSHARD_ERR_INVALID_ARG;
    if (l->counts[i] < 0) return GSHARD_ERR_INVALID_ARG;
    if (l->counts[i] > (1ll << 38)) return GSHARD_ERR_UNSUPPORTED_SHAPE;
    const uintptr_t es = l->dtypes[i] == GSHARD_BF16 ? 2 : 4;
    if (l->counts[i] && (!l->grads[i] || reinterpret_cast<uintptr_t>(l->grads[i]) % es)) return GSHARD_ERR_INVALID_ARG;
    if (clip && l->counts[i] && (!l->outs[i] || reinterpret_cast<uintptr_t>(l->outs[i]) % es)) return GSHARD_ERR_INVALID_ARG;
  }
  return GSHARD_OK;
}

// Calls f(table, blocks) for runs of the list's tensors; every table holds fewer than 2^30 chunks.
template <int N, typename F>
void for_tables(const gshard_grad_list& l, bool clip, F f) {
  GradTable<N> t;
  int i = 0;
  while (i < l.n) {
    t.n = 0;
    long long chunks = 0;
    for (; i < l.n && t.n < N; ++i) {
      if (!l.counts[i]) continue;
      const long long off = l.dtypes[i] == GSHARD_BF16 ? skew(static_cast<const __nv_bfloat16*>(l.grads[i])) : skew(static_cast<const float*>(l.grads[i]));
      const long long more = (l.counts[i] + off + kChunk - 1) / kChunk;
      if (t.n && chunks + more >= (1 << 30)) break;
      t.in[t.n] = l.grads[i];
      t.out[t.n] = clip ? l.outs[i] : nullptr;
      t.count[t.n] = l.counts[i] * 2 + (l.dtypes[i] == GSHARD_BF16);
      t.first[t.n++] = (int)chunks;
      chunks += more;
    }
    t.first[t.n] = (int)chunks;
    if (chunks) f(t, (int)std::min<long long>(chunks, kMaxBlocks));
  }
}

// A table is passed to its kernel by value: the small one for lists that fit it.
constexpr int kSmallTable = 64, kLargeTable = 1024;
template <typename F>
void for_tables_of(const gshard_grad_list& l, bool clip, F f) {
  if (l.n <= kSmallTable) for_tables<kSmallTable>(l, clip, f);
  else for_tables<kLargeTable>(l, clip, f);
}

int partial_sums(const gshard_grad_list& l) {
  int n = 0;
  for_tables_of(l, false, [&](const auto&, int blocks) { n += blocks; });
  return n;
}

}  // namespace

}  // namespace gshard

using namespace gshard;

extern "C" {

size_t gshard_grad_norm_workspace_bytes(const gshard_grad_list* list) {
  if (grad_validate(list, false) != GSHARD_OK) return 0;
  return align_up((size_t)partial_sums(*list) * sizeof(double) + 1);
}

int gshard_grad_norm(const gshard_grad_list* list, double* sumsq, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  launch_counter().n = 0;
  GS_CHECK(grad_validate(list, false));
  if (!sumsq || reinterpret_cast<uintptr_t>(sumsq) % 8) return GSHARD_ERR_INVALID_ARG;
  GS_CHECK_WORKSPACE(workspace, workspace_bytes, gshard_grad_norm_workspace_bytes(list));
  GS_CHECK(check_device());
  NvtxRange range("gshard.grad_norm");
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  double* partial = static_cast<double*>(workspace);
  int n = 0;
  for_tables_of(*list, false, [&](const auto& table, int blocks) {
    grad_sum_kernel<<<blocks, kThreads, 0, st>>>(table, partial + n);
    count_launch();
    n += blocks;
  });
  grad_sum_finish_kernel<<<1, kThreads, 0, st>>>(partial, n, sumsq);
  count_launch();
  return cudaGetLastError() == cudaSuccess ? GSHARD_OK : GSHARD_ERR_CUDA;
}

int gshard_grad_clip(const gshard_grad_list* list, const double* sumsq, float max_norm, float* norm, void* cuda_stream) {
  launch_counter().n = 0;
  GS_CHECK(grad_validate(list, true));
  if (!sumsq || reinterpret_cast<uintptr_t>(sumsq) % 8 || reinterpret_cast<uintptr_t>(norm) % 4) return GSHARD_ERR_INVALID_ARG;
  if (!(max_norm >= 0.f)) return GSHARD_ERR_INVALID_ARG;
  GS_CHECK(check_device());
  NvtxRange range("gshard.grad_clip");
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  for_tables_of(*list, true, [&](const auto& table, int blocks) {
    grad_clip_kernel<<<blocks, kThreads, 0, st>>>(table, sumsq, max_norm, norm);
    norm = nullptr;                            // the first launch has written it
    count_launch();
  });
  if (norm) {                                  // an empty list: the norm alone
    GradTable<kSmallTable> none;
    none.n = 0;
    none.first[0] = 0;
    grad_clip_kernel<<<1, kThreads, 0, st>>>(none, sumsq, max_norm, norm);
    count_launch();
  }
  return cudaGetLastError() == cudaSuccess ? GSHARD_OK : GSHARD_ERR_CUDA;
}

}  // extern "C"
