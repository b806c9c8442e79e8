// Cross attention: entry points, argument checks and the row sums of the backward pass.
#include "attention.cuh"
#include "checks.cuh"
#include "pack.cuh"
#include "plan.cuh"

namespace gshard {

namespace {

// delta[b, h, t] = sum over d of dout o in fp32, one warp per row
__global__ void __launch_bounds__(256) attention_delta_kernel(const AttentionArgs a, float* delta, long long rows) {
  const int lane = threadIdx.x & 31;
  for (long long r = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); r < rows; r += (long long)gridDim.x * 8) {
    const float* o = static_cast<const float*>(a.o) + r * a.D;
    const float* g = static_cast<const float*>(a.dout) + r * a.D;
    float s = 0.f;
    const int c = lane * 4;
    if (c < a.D) {
      float x[4], y[4];
      load_pack<float, 4>(o + c, x);
      load_pack<float, 4>(g + c, y);
#pragma unroll
      for (int j = 0; j < 4; ++j) s = fmaf(x[j], y[j], s);
    }
#pragma unroll
    for (int off = 16; off; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
    if (lane == 0) {
      const long long token = r / a.H;
      const int h = (int)(r % a.H);
      delta[(token / a.Tq * a.H + h) * a.Tq + token % a.Tq] = s;
    }
  }
}

int attention_validate(const gshard_attention_config* c) {
  if (!c || c->batch < 0 || c->q_len < 0 || c->k_len < 0 || c->heads <= 0 || c->kv_heads <= 0 || c->head_dim <= 0)
    return GSHARD_ERR_INVALID_ARG;
  if (c->dtype != GSHARD_F32 && c->dtype != GSHARD_BF16) return GSHARD_ERR_INVALID_ARG;
  if (!(c->scale >= 1e-20f && c->scale <= 1e20f)) return GSHARD_ERR_INVALID_ARG;     // lse / scale is a finite number
  if (c->heads % c->kv_heads) return GSHARD_ERR_INVALID_ARG;
  if (c->head_dim % 8 || c->head_dim > 128) return GSHARD_ERR_UNSUPPORTED_SHAPE;
  const int64_t q_row = (int64_t)c->heads * c->head_dim, k_row = (int64_t)c->kv_heads * c->head_dim;
  if (c->q_stride < q_row || c->k_stride < k_row || c->v_stride < k_row) return GSHARD_ERR_INVALID_ARG;
  const int align = c->dtype == GSHARD_BF16 ? 8 : 4;
  if ((c->q_stride | c->k_stride | c->v_stride) % align) return GSHARD_ERR_INVALID_ARG;
  // tensor map strides in bytes and tile counts in 31 bits
  const int64_t far = 1ll << 36;
  if (c->q_stride >= far || c->k_stride >= far || c->v_stride >= far || c->heads > 65535) return GSHARD_ERR_UNSUPPORTED_SHAPE;
  const int64_t most = std::max(c->q_len, c->k_len);
  if (most > (1 << 30) || (most + 63) / 64 * c->heads >= (1ll << 31) || (most + 63) / 64 * c->heads * c->batch >= (1ll << 31))
    return GSHARD_ERR_UNSUPPORTED_SHAPE;
  // by division: the products may pass 63 bits
  auto spans_too_much = [](int64_t tokens, int64_t stride) { return tokens > 0 && stride > ((1ll << 38) - 1) / tokens; };
  if (spans_too_much(c->q_len, c->q_stride) || spans_too_much(c->k_len, std::max(c->k_stride, c->v_stride))) return GSHARD_ERR_UNSUPPORTED_SHAPE;
  return GSHARD_OK;
}

AttentionArgs attention_args(const gshard_attention_config& c, const void* q, const void* k, const void* v, const int32_t* lengths) {
  AttentionArgs a{};
  a.q = q; a.k = k; a.v = v; a.lengths = lengths;
  a.B = c.batch; a.Tq = c.q_len; a.Tk = c.k_len; a.H = c.heads; a.Hkv = c.kv_heads; a.D = c.head_dim;
  a.scale = c.scale;
  a.q_stride = c.q_stride; a.k_stride = c.k_stride; a.v_stride = c.v_stride;
  return a;
}

struct AttentionPlan { size_t status, delta, scratch, total; };

AttentionPlan attention_plan(const gshard_attention_config& c, bool backward) {
  const AttentionArgs a = attention_args(c, nullptr, nullptr, nullptr, nullptr);
  const bool bf16 = c.dtype == GSHARD_BF16;
  Carver w;
  AttentionPlan p{};
  p.status = w.take(256);
  if (backward) {
    if (!bf16) p.delta = w.take(4 * (size_t)c.batch * c.heads * c.q_len);
    p.scratch = w.take(4 * (bf16 ? attention_umma_backward_floats(a) : attention_simt_backward_floats(a)));
  } else if (!attention_is_few(bf16, a.B, a.Tq, a.Tk, a.H, a.Hkv, a.D)) {
    p.scratch = w.take(4 * (bf16 ? attention_umma_forward_floats(a) : attention_simt_forward_floats(a)));
  }
  p.total = w.off;
  return p;
}

int clear_status(void* workspace, cudaStream_t st) {
  if (cudaMemsetAsync(workspace, 0, sizeof(int), st) == cudaSuccess) return GSHARD_OK;
  cudaGetLastError();
  return GSHARD_ERR_CUDA;
}

}  // namespace

}  // namespace gshard

using namespace gshard;

extern "C" {

size_t gshard_cross_attention_workspace_bytes(const gshard_attention_config* config, int for_backward) {
  if (attention_validate(config) != GSHARD_OK) return 0;
  return attention_plan(*config, for_backward != 0).total;
}

int gshard_cross_attention_forward(const gshard_attention_config* config, const void* q, const void* k, const void* v,
                                   const int32_t* k_lengths, void* o, float* lse, void* workspace, size_t workspace_bytes,
                                   void* cuda_stream) {
  launch_counter().n = 0;
  GS_CHECK(attention_validate(config));
  const gshard_attention_config& c = *config;
  if (c.batch == 0 || c.q_len == 0) return GSHARD_OK;
  GS_CHECK_PTR(q); GS_CHECK_PTR(o); GS_CHECK_OPTIONAL_PTR(lse);
  if (c.k_len) { GS_CHECK_PTR(k); GS_CHECK_PTR(v); }
  if (reinterpret_cast<uintptr_t>(k_lengths) % 4) return GSHARD_ERR_INVALID_ARG;
  if (o == q || o == k || o == v || o == lse) return GSHARD_ERR_INVALID_ARG;
  const AttentionPlan pl = attention_plan(c, false);
  GS_CHECK_WORKSPACE(workspace, workspace_bytes, pl.total);
  GS_CHECK(check_device());
  NvtxRange range("gshard.attention");
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  AttentionArgs a = attention_args(c, q, k, v, k_lengths);
  a.o = o; a.lse = lse; a.status = static_cast<int*>(workspace);
  const bool bf16 = c.dtype == GSHARD_BF16;
  if (attention_is_few(bf16, a.B, a.Tq, a.Tk, a.H, a.Hkv, a.D)) return launch_attention_few(a, bf16, st);
  GS_CHECK(clear_status(workspace, st));
  float* scratch = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + pl.scratch);
  return bf16 ? launch_attention_umma_forward(a, scratch, st) : launch_attention_simt_forward(a, scratch, st);
}

int gshard_cross_attention_backward(const gshard_attention_config* config, const void* q, const void* k, const void* v,
                                    const int32_t* k_lengths, const void* o, const float* lse, const void* dout, void* dq, void* dk,
                                    void* dv, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  launch_counter().n = 0;
  GS_CHECK(attention_validate(config));
  const gshard_attention_config& c = *config;
  if (c.batch == 0 || (c.q_len == 0 && c.k_len == 0)) return GSHARD_OK;
  if (c.q_len) { GS_CHECK_PTR(q); GS_CHECK_PTR(o); GS_CHECK_PTR(lse); GS_CHECK_PTR(dout); GS_CHECK_PTR(dq); }
  if (c.k_len) { GS_CHECK_PTR(k); GS_CHECK_PTR(v); GS_CHECK_PTR(dk); GS_CHECK_PTR(dv); }
  if (reinterpret_cast<uintptr_t>(k_lengths) % 4) return GSHARD_ERR_INVALID_ARG;
  const void* in[] = {q, k, v, o, lse, dout};
  const void* out[] = {dq, dk, dv};
  for (int i = 0; i < 3; ++i) {
    for (const void* p : in)
      if (out[i] && out[i] == p) return GSHARD_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (out[i] && out[i] == out[j]) return GSHARD_ERR_INVALID_ARG;
  }
  const AttentionPlan pl = attention_plan(c, true);
  GS_CHECK_WORKSPACE(workspace, workspace_bytes, pl.total);
  GS_CHECK(check_device());
  NvtxRange range("gshard.attention.backward");
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  AttentionArgs a = attention_args(c, q, k, v, k_lengths);
  float* scratch = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + pl.scratch);
  float* delta = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + pl.delta);
  a.o = const_cast<void*>(o); a.lse = const_cast<float*>(lse); a.dout = dout; a.delta = delta;
  a.dq = dq; a.dk = dk; a.dv = dv; a.status = static_cast<int*>(workspace);
  GS_CHECK(clear_status(workspace, st));
  if (c.dtype == GSHARD_BF16) return launch_attention_umma_backward(a, scratch, st);
  const long long rows = (long long)c.batch * c.q_len * c.heads;
  if (rows) {
    attention_delta_kernel<<<grid_for_rows(rows), 256, 0, st>>>(a, delta, rows);
    count_launch();
  }
  return launch_attention_simt_backward(a, scratch, st);
}

}  // extern "C"
