// Shared by the cross-attention kernels.
//
//   s = scale q.k over the keys below the source's length, p = softmax(s), o = p v, lse = log sum exp(s)
//   backward, with o and lse as the forward kept them: P = exp(s - lse), delta = sum over d of dout o,
//   dS = scale P (dout v^T - delta), dq = dS k, dk = dS^T q, dv = P^T dout; heads that share a key head add up.
#pragma once
#include <algorithm>

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

// A long axis of `units` tiles is cut into parts where the `blocks` that walk it leave many of the GPU's `slots` idle, all the time or
// in the last round: every part leaves its sums in fp32 (about one tile's time), and a second launch adds them in order (about two).
// Measured, backward in bf16: 4096 queries of 16 heads on 400 keys of 2 heads of 128, 448 us whole and 107 in parts; 64 queries of one
// head on 32768 keys, 335 and 49; where the rounds are even, the same (2 x 1024 x 1024, 8 heads: 51 us).
struct Parts { int parts, each; };
inline Parts parts_of(long long blocks, int units, int slots) {
  Parts best{1, std::max(units, 1)};
  auto rounds = [&](long long n) { return (n + slots - 1) / slots; };
  long long least = rounds(blocks) * (best.each + 1ll);
  for (int n = 2; n * std::max(blocks, 1ll) <= 4ll * slots && n * 4 <= units; ++n) {      // at least four tiles each
    const int each = ceil_div(units, n), parts = ceil_div(units, each);    // none is empty
    const long long cost = rounds(parts * blocks) * (each + 1ll) + 2;
    if (cost < least) { best = {parts, each}; least = cost; }
  }
  return best;
}

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// attention_few.cu: up to 8 rows (queries x heads) per key head, in one launch
bool attention_is_few(bool bf16, int B, int Tq, int Tk, int H, int Hkv, int D);
int launch_attention_few(const AttentionArgs& a, bool bf16, cudaStream_t st);

// The kernels by type: attention_simt.cu, fp32 on the CUDA cores; attention_umma.cu and attention_backward.cu, bf16 on the tensor
// cores.  scratch: so many floats, 256-byte aligned.
size_t attention_simt_forward_floats(const AttentionArgs& a);
size_t attention_simt_backward_floats(const AttentionArgs& a);
size_t attention_umma_forward_floats(const AttentionArgs& a);
size_t attention_umma_backward_floats(const AttentionArgs& a);
int launch_attention_simt_forward(const AttentionArgs& a, float* scratch, cudaStream_t st);
int launch_attention_simt_backward(const AttentionArgs& a, float* scratch, cudaStream_t st);
int launch_attention_umma_forward(const AttentionArgs& a, float* scratch, cudaStream_t st);
int launch_attention_umma_backward(const AttentionArgs& a, float* scratch, cudaStream_t st);

// attention_join.cu.  o and lse from the outputs part_o [parts][B, Tq, H, D] and (powers of two) part_lse [parts][B, Tq, H] of the
// parts of every source; a part without keys has lse -inf and an o that is not read.
int launch_join_outputs(const AttentionArgs& a, bool bf16, const float* part_o, const float* part_lse, int parts, cudaStream_t st);
// dq, dk or dv from the sums of parts, [B, tokens, heads, D] each and `pitch` floats apart: out = factor times their sum.  part_keys > 0: part i is there for
// sources of more than i * part_keys keys (dq); else tokens are keys, and those from the source's length on have none (dk, dv).
int launch_join_gradient(const AttentionArgs& a, bool bf16, const float* part, int parts, int part_keys, void* out, int tokens, int heads,
                         long long stride, float factor, cudaStream_t st, size_t pitch);

// Tensor map of k or v.  A batch of sources without tokens gets a valid map that nothing reads through.
inline bool make_source_map(CUtensorMap* map, const AttentionArgs& a, const void* base, long long stride, int box_tokens) {
  return a.Tk > 0 ? make_token_map(map, base, a.D, a.Hkv, a.Tk, a.B, stride, box_tokens)
                  : make_token_map(map, a.q, a.D, 1, 1, 1, stride, box_tokens);
}

}  // namespace gshard
