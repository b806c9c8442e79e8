// Shared by the cross-attention kernels.
//
//   s = scale q.k over the keys below the source's length, p = softmax(s), o = p v, lse = log sum exp(s)
//   backward, with o and lse as the forward kept them: P = exp(s - lse), delta = sum over d of dout o,
//   dS = scale P (dout v^T - delta), dq = dS k, dk = dS^T q, dv = P^T dout; heads that share a key head add up.
#pragma once
#include "common.cuh"
#include "tensor_map.cuh"

namespace gshard {

struct AttentionArgs {
  const void* q; const void* k; const void* v;       // [B, Tq, H, D], [B, Tk, Hkv, D]: tokens at the strides below
  const int32_t* lengths;                            // [B] keys of each source, or nullptr: Tk
  void* o; float* lse;                               // [B, Tq, H, D] packed, [B, H, Tq]; lse may be nullptr in the forward
  const void* dout; const float* delta;              // like o, like lse
  void* dq; void* dk; void* dv;                      // laid out like q, k, v
  int B, Tq, Tk, H, Hkv, D;
  float scale;
  long long q_stride, k_stride, v_stride;            // elements from one token to the next; batches are dense
  int* status;
};

__device__ __forceinline__ int source_length(const AttentionArgs& a, int b) {
  return a.lengths ? min(max(__ldg(a.lengths + b), 0), a.Tk) : a.Tk;
}

// Division of 31-bit numbers by a divisor known at launch: a multiplication and a shift (Granlund and Montgomery, 1994) where the
// hardware's takes some twenty instructions, which in the thread that issues MMAs cost the tensor core.
struct Divisor {
  uint32_t d, mul, shift;
  Divisor() = default;
  explicit Divisor(int divisor) : d((uint32_t)divisor), shift(0) {
    while ((1ull << shift) < d) ++shift;
    mul = (uint32_t)(((1ull << 32) * ((1ull << shift) - d)) / d + 1);
  }
  __device__ __forceinline__ int quotient(int n) const { return (int)((__umulhi(mul, (uint32_t)n) + (uint32_t)n) >> shift); }
  // quotient; n becomes the remainder
  __device__ __forceinline__ int split(int& n) const {
    const int q = quotient(n);
    n -= q * (int)d;
    return q;
  }
};

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// attention_few.cu: up to 8 rows (queries x heads) per key head, in one launch
bool attention_is_few(bool bf16, int B, int Tq, int Tk, int H, int Hkv);
int launch_attention_few(const AttentionArgs& a, bool bf16, cudaStream_t st);

// attention_simt.cu: fp32 on the CUDA cores
int launch_attention_simt_forward(const AttentionArgs& a, cudaStream_t st);
int launch_attention_simt_backward(const AttentionArgs& a, cudaStream_t st);

// attention_umma.cu, attention_backward.cu: bf16 on the tensor cores.  scratch, stats: attention_parts_floats() and
// attention_stats_floats() floats
size_t attention_parts_floats(int B, int Tq, int Tk, int H, int Hkv, int D);
int launch_attention_umma_forward(const AttentionArgs& a, float* scratch, cudaStream_t st);
size_t attention_stats_floats(int B, int Tq, int H);
int launch_attention_umma_backward(const AttentionArgs& a, float* stats, cudaStream_t st);

// Tensor map of k or v.  A batch of sources without tokens gets a valid map that nothing reads through.
inline bool make_source_map(CUtensorMap* map, const AttentionArgs& a, const void* base, long long stride, int box_tokens) {
  return a.Tk > 0 ? make_token_map(map, base, a.D, a.Hkv, a.Tk, a.B, stride, box_tokens)
                  : make_token_map(map, a.q, a.D, 1, 1, 1, stride, box_tokens);
}

}  // namespace gshard
