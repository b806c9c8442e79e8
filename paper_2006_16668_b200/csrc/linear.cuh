// Shared by the linear operator's kernels.
#pragma once
#include "activation.cuh"
#include "kernels.cuh"
#include "pack.cuh"

namespace gshard {

// linear_few.cu: the whole operator in one launch for up to 8 rows; also clears the status word.  gated: the gated linear operator
// with cols columns of w, cols / 2 of y (typed like x).
int launch_linear_few(int n, int K, int cols, bool bf16, bool out_f32, const void* x, const void* w, void* y,
                      const LinearEpilogue& lin, int* status, cudaStream_t st, bool gated = false);

// linear_mid.cu: a product whose output tiles run at once, with the operator's epilogue, in one launch (operands
// as in UmmaGemm: bf16 output with at most two planes together, fp32 output with one or three each).  bn == 0: too many tiles, or too deep for them.
struct MidShape { int bn, splits; };
MidShape linear_mid_shape(long long rows, int cols, long long depth, int passes, bool out_f32);
int launch_linear_mid(const UmmaGemm& g, const LinearEpilogue& lin, MidShape shape, bool clear_status, int* status, cudaStream_t st);

// linear.cu: regions of the workspace and how the products are run.
struct LinearPlan {
  size_t status, xp, wp, dpre, colsum, join, total;
  int planes, chunks, chunk, splits, dx_splits, dw_splits;
  MidShape mid, dx_mid, dw_mid;          // bn > 0: the product goes to linear_mid.cu
};

LinearPlan linear_plan(int64_t n, int K, int cols, int dtype, int out_dtype, bool backward);
int linear_validate(int64_t n, int32_t K, int32_t cols, int32_t dtype, int32_t out_dtype);
// Three bf16 planes of one or two fp32 tensors (the second may have no elements), one behind the other.
void linear_split_planes(const void* src0, void* dst0, long long n0, const void* src1, void* dst1, long long n1, cudaStream_t st);
// y = act(x . w + bias) + residual on checked arguments.
int linear_run_forward(int64_t n_rows, int K, int cols, int dtype, int out_dtype, const LinearEpilogue& lin, const void* x,
                       const void* w, void* y, const LinearPlan& pl, unsigned char* ws, cudaStream_t st);
// dx = dpre . w^T and dw = x^T . dpre (either may be nullptr) from `planes` bf16 planes of dpre [n_rows, cols] (3: fp32).
// cleared: an earlier kernel of the call has cleared the status word.
int linear_run_gradients(int64_t n_rows, int K, int cols, bool fp32, int planes, const void* x, const void* w, const void* dpre,
                         void* dx, void* dw, const LinearPlan& pl, unsigned char* ws, bool cleared, cudaStream_t st);

// The three bf16 planes of fp32 values: hi takes the top 8 bits of the significand, mid the next 8, lo the last 8,
// each by truncation, so that hi + mid + lo is the value exactly (below 2^-110 to half a step of 2^-133) and nothing overflows.
__device__ __forceinline__ void split3(const float* f, float* hi, float* mid, float* lo, int n) {
#pragma unroll
  for (int j = 0; j < n; ++j) {
    hi[j] = __uint_as_float(__float_as_uint(f[j]) & 0xffff0000u);
    const float r = f[j] - hi[j];
    mid[j] = __uint_as_float(__float_as_uint(r) & 0xffff0000u);
    lo[j] = r - mid[j];
  }
}
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

// The gated linear operator's epilogue on four neighbouring sums of both factors, column `col` of row `row` of h [n, cols].
template <typename TY>
__device__ __forceinline__ void gated_epilogue4(const LinearEpilogue& lin, void* h, long long row, int cols, int col, float4 gate, float4 up) {
  const float g[4] = {gate.x, gate.y, gate.z, gate.w}, u[4] = {up.x, up.y, up.z, up.w};
  if (lin.pre) {
    TY* pre = static_cast<TY*>(lin.pre) + row * 2 * cols + col;
    store_pack<TY, 4>(pre, g);
    store_pack<TY, 4>(pre + cols, u);
  }
  float f[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) f[j] = (sizeof(TY) == 2 ? activation_value_fast(g[j], lin.act) : activation_value(g[j], lin.act)) * u[j];
  store_pack<TY, 4>(static_cast<TY*>(h) + row * cols + col, f);
}

}  // namespace gshard
