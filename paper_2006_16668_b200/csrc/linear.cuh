// Shared by the linear operator's kernels.
#pragma once
#include "activation.cuh"
#include "kernels.cuh"
#include "pack.cuh"

namespace gshard {

// linear_few.cu: the whole operator in one launch for up to 8 rows; also clears the status word.
int launch_linear_few(int n, int K, int cols, bool bf16, bool out_f32, const void* x, const void* w, void* y,
                      const LinearEpilogue& lin, int* status, cudaStream_t st);

// linear_mid.cu: a product whose output tiles run at once, with the operator's epilogue, in one launch (operands
// as in UmmaGemm: bf16 output with at most two planes together, fp32 output with one or three each).  bn == 0: too many tiles, or too deep for them.
struct MidShape { int bn, splits; };
MidShape linear_mid_shape(long long rows, int cols, long long depth, int passes, bool out_f32);
int launch_linear_mid(const UmmaGemm& g, const LinearEpilogue& lin, MidShape shape, bool clear_status, int* status, cudaStream_t st);

// The operator's epilogue on four neighbouring sums at element `off` (column `col`) of the output.
template <typename TY>
__device__ __forceinline__ void linear_epilogue4(const LinearEpilogue& lin, void* y, long long off, int col, float4 s) {
  float f[4] = {s.x, s.y, s.z, s.w};
  if (lin.bias) {
    const float4 b = __ldg(reinterpret_cast<const float4*>(lin.bias + col));
    f[0] += b.x; f[1] += b.y; f[2] += b.z; f[3] += b.w;
  }
  if (lin.pre) store_pack<TY, 4>(static_cast<TY*>(lin.pre) + off, f);
#pragma unroll
  for (int j = 0; j < 4; ++j) f[j] = activation_value(f[j], lin.act);
  if (lin.residual) {
    float r[4];
    load_pack<TY, 4>(static_cast<const TY*>(lin.residual) + off, r);
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] += r[j];
  }
  store_pack<TY, 4>(static_cast<TY*>(y) + off, f);
}

}  // namespace gshard
