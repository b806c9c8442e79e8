// The first half of a gated feed-forward block: pre = x . w, h = act(gate) up, where the first `cols` columns of
// w [K, 2 cols] make the gate and the last the other factor (with silu and gelu the SwiGLU and GEGLU of Shazeer's "GLU
// variants improve Transformer", 2020; no bias, as in the experts' feed-forward), and its backward pass:
//   dgate = dh up act'(gate), dup = dh act(gate), dx = dpre . w^T, dw = x^T . dpre
// The second half, h . wo, is the linear operator.
// Bound by the tensor pipe and, at training size, the power cap: 16384 x 1024 -> 8192 bf16, gelu, projections kept, 411 us at 76 % tensor
// activity (the epilogue writes three bf16 values per pair of sums); 65536 rows 2000 to 2150 us.  Backward, 30011 rows, 2095 us.
#include <algorithm>

#include "activation.cuh"
#include "checks.cuh"
#include "linear.cuh"
#include "pack.cuh"
#include "plan.cuh"
#include "umma_epilogue.cuh"

namespace gshard {

namespace {

// h = act(gate) up from fp32 projections, 8 columns per thread; keeps them as T where pre is given.
template <typename T, int ACT>
__global__ void __launch_bounds__(256) gated_value_kernel(const float* __restrict__ acc, T* __restrict__ h, T* pre, long long n8, int cols) {
  constexpr bool FAST = sizeof(T) == 2;
  const int c8 = cols / 8;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n8; i += (long long)gridDim.x * 256) {
    const long long row = i / c8;
    const int col = (int)(i % c8) * 8;
    const long long at = row * 2 * cols + col;
    float g[8], u[8], y[8];
#pragma unroll
    for (int j = 0; j < 8; j += 4) {
      load_pack<float, 4>(acc + at + j, g + j);
      load_pack<float, 4>(acc + at + cols + j, u + j);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = (FAST ? activation_value_fast(g[j], ACT) : activation_value(g[j], ACT)) * u[j];
    constexpr int W = 16 / (int)sizeof(T);
#pragma unroll
    for (int j = 0; j < 8; j += W) {
      store_pack<T, W>(h + row * cols + col + j, y + j);
      if (pre) {
        store_pack<T, W>(pre + at + j, g + j);
        store_pack<T, W>(pre + at + cols + j, u + j);
      }
    }
  }
}

// dpre of 8 columns per thread as PLANES bf16 planes of [n, 2 cols] (1: rounded; 2: rounded, and what the rounding left;
// 3: fp32).  Also clears the status word for the products that follow.
template <typename T, int PLANES, int ACT>
__global__ void __launch_bounds__(256) gated_dpre_kernel(const T* __restrict__ dh, const T* __restrict__ pre, __nv_bfloat16* __restrict__ dpre,
                                                         int* status, long long n8, int cols, long long plane) {
  constexpr bool FAST = PLANES < 3;
  constexpr int W = 16 / (int)sizeof(T), P = 8 / W;
  if (blockIdx.x == 0 && threadIdx.x == 0) *status = 0;
  const int c8 = cols / 8;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n8; i += (long long)gridDim.x * 256) {
    const long long row = i / c8;
    const int col = (int)(i % c8) * 8;
    const long long at = row * 2 * cols + col;
    Pack<T, W> pg[P], pu[P], pd[P];
#pragma unroll
    for (int j = 0; j < P; ++j) {
      pd[j].load_once(dh + row * cols + col + j * W);
      pg[j].load_once(pre + at + j * W);
      pu[j].load_once(pre + at + cols + j * W);
    }
    float d[2][8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float g = pg[j / W].get(j % W), u = pu[j / W].get(j % W), y = pd[j / W].get(j % W);
      d[0][j] = y * u * (FAST ? activation_slope_fast(g, ACT) : activation_slope(g, ACT));
      d[1][j] = y * (FAST ? activation_value_fast(g, ACT) : activation_value(g, ACT));
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      __nv_bfloat16* out = dpre + at + half * cols;
      if (PLANES == 1) {
        store_pack<__nv_bfloat16, 8>(out, d[half]);
      } else if (PLANES == 2) {
        float hi[8], lo[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          hi[j] = __bfloat162float(__float2bfloat16_rn(d[half][j]));
          lo[j] = fabsf(hi[j]) == INFINITY ? 0.f : d[half][j] - hi[j];        // an infinity is all in the first plane
        }
        store_pack<__nv_bfloat16, 8>(out, hi);
        store_pack<__nv_bfloat16, 8>(out + plane, lo);
      } else {
        float hi[8], mid[8], lo[8];
        split3(d[half], hi, mid, lo, 8);
        store_pack<__nv_bfloat16, 8>(out, hi);
        store_pack<__nv_bfloat16, 8>(out + plane, mid);
        store_pack<__nv_bfloat16, 8>(out + 2 * plane, lo);
      }
    }
  }
}

int gated_grid(long long items) {
  return (int)std::max<long long>(1, std::min<long long>((items + 255) / 256, (long long)device_sms() * 16));
}

#define GSHARD_FOR_ACTIVATION(act, CASE) \
  switch (act) {                         \
    CASE(GSHARD_ACT_NONE)                \
    CASE(GSHARD_ACT_RELU)                \
    CASE(GSHARD_ACT_GELU)                \
    CASE(GSHARD_ACT_GELU_TANH)           \
    CASE(GSHARD_ACT_SILU)                \
  }

template <typename T>
void launch_value(const float* acc, void* h, void* pre, long long n, int cols, int act, cudaStream_t st) {
  const long long n8 = n * cols / 8;
#define GSHARD_CASE(A) \
  case A: gated_value_kernel<T, A><<<gated_grid(n8), 256, 0, st>>>(acc, static_cast<T*>(h), static_cast<T*>(pre), n8, cols); break;
  GSHARD_FOR_ACTIVATION(act, GSHARD_CASE)
#undef GSHARD_CASE
  count_launch();
}

template <typename T, int PLANES>
void launch_gated_dpre(const void* dh, const void* pre, void* dpre, int* status, long long n, int cols, int act, cudaStream_t st) {
  const long long n8 = n * cols / 8;
#define GSHARD_CASE(A)                                                                                                            \
  case A:                                                                                                                         \
    gated_dpre_kernel<T, PLANES, A><<<gated_grid(n8), 256, 0, st>>>(static_cast<const T*>(dh), static_cast<const T*>(pre),       \
                                                                    static_cast<__nv_bfloat16*>(dpre), status, n8, cols, n * 2 * cols); \
    break;
  GSHARD_FOR_ACTIVATION(act, GSHARD_CASE)
#undef GSHARD_CASE
  count_launch();
}

int gated_validate(int64_t n, int32_t K, int32_t cols, int32_t dtype) {
  if (cols <= 0) return GSHARD_ERR_INVALID_ARG;
  if (cols % 8 || cols > (1 << 23)) return GSHARD_ERR_UNSUPPORTED_SHAPE;
  return linear_validate(n, K, 2 * cols, dtype, dtype);
}

// How a forward runs.
//   FEW      w streams through the CUDA cores in one launch (linear_few.cu): up to 4 rows, 8 of fp32, whose planes would first be
//            written.  1024 -> 4096, bf16, us, few / tiles / project: 1 row 6.7 / 14.2 / 7.5, 4 rows 8.7 / 12.6 / 9.7, 8 rows
//            11.0 / 12.6 / 9.8; fp32, 8 rows 12.4 / 58.8 / 14.3.
//   TILES    one launch on CTA pairs, both factors of a tile side by side in tensor memory (umma2_gemm.cu).  One tile takes
//            about 8.6 us + 4.3 us per 1024 of the contraction (fp32 22 + 29), so it wants enough tiles to fill the pairs.
//   PROJECT  the product in the linear operator's forms, which cut the contraction, and the projections meet in a second launch.
//            Better where that product is one launch (linear_mid.cu; 4096 -> 1024, bf16: 64 rows 25.9 / 10.7), or the tiles
//            are few: 4096 -> 1024, 512 rows (16 tiles) 26.3 / 21.9, 1024 rows (32 tiles) 27.0 / 28.6; 2048 -> 2048, 512 rows (32 tiles)
//            18.0 / 23.0; fp32: 32 tiles 81.5 / 63.1, 64 tiles 88.9 / 94.4.
enum class GatedForm { FEW, TILES, PROJECT };
GatedForm gated_form(int64_t n, int K, int cols, bool bf16) {
  if (n <= (bf16 ? 4 : 8)) return GatedForm::FEW;
  if (linear_mid_shape(n, 2 * cols, K, bf16 ? 1 : umma_epi::kPasses3, true).bn) return GatedForm::PROJECT;
  const int64_t tiles = (n + 255) / 256 * ((cols + 127) / 128);
  return tiles >= (bf16 ? 24 : 48) ? GatedForm::TILES : GatedForm::PROJECT;
}

struct GatedPlan {
  GatedForm form;
  LinearPlan lin;            // backward, PROJECT
  size_t xp, wp, acc, total;
};

GatedPlan gated_plan(int64_t n, int K, int cols, int dtype, bool backward) {
  GatedPlan p{};
  Carver w;
  if (backward) {
    p.lin = linear_plan(n, K, 2 * cols, dtype, dtype, true);
    p.total = p.lin.total;
    return p;
  }
  p.form = gated_form(n, K, cols, dtype == GSHARD_BF16);
  if (p.form == GatedForm::PROJECT) {
    p.lin = linear_plan(n, K, 2 * cols, dtype, GSHARD_F32, false);
    w.take(p.lin.total);
    p.acc = w.take((size_t)n * 2 * cols * 4);
  } else {
    w.take(256);             // status word
    if (p.form == GatedForm::TILES && dtype == GSHARD_F32) {
      p.xp = w.take((size_t)n * K * 6);
      p.wp = w.take((size_t)K * 2 * cols * 6);
    }
  }
  p.total = w.off;
  return p;
}

}  // namespace

}  // namespace gshard

using namespace gshard;

extern "C" {

size_t gshard_gated_linear_workspace_bytes(int64_t n_rows, int32_t K, int32_t cols, int32_t dtype, int for_backward) {
  if (gated_validate(n_rows, K, cols, dtype) != GSHARD_OK) return 0;
  return gated_plan(n_rows, K, cols, dtype, for_backward != 0).total;
}

int gshard_gated_linear_forward(int64_t n_rows, int32_t K, int32_t cols, int32_t dtype, int32_t activation, const void* x, const void* w,
                                void* h, void* pre, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  launch_counter().n = 0;
  GS_CHECK(gated_validate(n_rows, K, cols, dtype));
  if (activation < GSHARD_ACT_NONE || activation > GSHARD_ACT_SILU) return GSHARD_ERR_INVALID_ARG;
  if (n_rows == 0) return GSHARD_OK;
  GS_CHECK_PTR(x); GS_CHECK_PTR(w); GS_CHECK_PTR(h); GS_CHECK_OPTIONAL_PTR(pre);
  if (h == x || h == w || (pre && (pre == x || pre == w || pre == h))) return GSHARD_ERR_INVALID_ARG;
  const GatedPlan pl = gated_plan(n_rows, K, cols, dtype, false);
  GS_CHECK_WORKSPACE(workspace, workspace_bytes, pl.total);
  GS_CHECK(check_device());
  NvtxRange range("gshard.gated_linear");
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  int* status = reinterpret_cast<int*>(ws);
  const bool bf16 = dtype == GSHARD_BF16;
  if (pl.form == GatedForm::FEW) {
    const LinearEpilogue lin{nullptr, nullptr, pre, activation};
    GS_CHECK(launch_linear_few((int)n_rows, K, 2 * cols, bf16, !bf16, x, w, h, lin, status, st, true));
  } else if (pl.form == GatedForm::TILES) {
    GatedGemm g{x, w, h, pre, (int)n_rows, cols, K, 1, activation};
    if (!bf16) {
      linear_split_planes(x, ws + pl.xp, n_rows * K, w, ws + pl.wp, (long long)K * 2 * cols, st);
      g.A = ws + pl.xp; g.B = ws + pl.wp; g.planes = 3;
    }
    GS_CHECK(launch_umma2_gated(g, status, st));
  } else {
    float* acc = reinterpret_cast<float*>(ws + pl.acc);
    GS_CHECK(linear_run_forward(n_rows, K, 2 * cols, dtype, GSHARD_F32, LinearEpilogue{}, x, w, acc, pl.lin, ws, st));
    if (bf16) launch_value<__nv_bfloat16>(acc, h, pre, n_rows, cols, activation, st);
    else launch_value<float>(acc, h, pre, n_rows, cols, activation, st);
  }
  return cudaGetLastError() == cudaSuccess ? GSHARD_OK : GSHARD_ERR_CUDA;
}

int gshard_gated_linear_backward(int64_t n_rows, int32_t K, int32_t cols, int32_t dtype, int32_t activation, const void* x, const void* w,
                                 const void* pre, const void* dh, void* dx, void* dw, void* workspace, size_t workspace_bytes,
                                 void* cuda_stream) {
  launch_counter().n = 0;
  GS_CHECK(gated_validate(n_rows, K, cols, dtype));
  if (activation < GSHARD_ACT_NONE || activation > GSHARD_ACT_SILU) return GSHARD_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  GS_CHECK_OPTIONAL_PTR(dx); GS_CHECK_OPTIONAL_PTR(dw);
  if (dx && dx == dw) return GSHARD_ERR_INVALID_ARG;
  const bool fp32 = dtype == GSHARD_F32;
  if (n_rows == 0) {                              // no rows: the weight gradient is an empty sum
    if (!dw) return GSHARD_OK;
    GS_CHECK(check_device());
    if (cudaMemsetAsync(dw, 0, (size_t)K * 2 * cols * (fp32 ? 4 : 2), st) == cudaSuccess) return GSHARD_OK;
    cudaGetLastError();
    return GSHARD_ERR_CUDA;
  }
  GS_CHECK_PTR(dh); GS_CHECK_PTR(pre);
  if (dx) GS_CHECK_PTR(w);
  if (dw) GS_CHECK_PTR(x);
  for (const void* p : {x, w, pre, dh})
    if (p && (p == dx || p == dw)) return GSHARD_ERR_INVALID_ARG;
  const GatedPlan pl = gated_plan(n_rows, K, cols, dtype, true);
  GS_CHECK_WORKSPACE(workspace, workspace_bytes, pl.total);
  GS_CHECK(check_device());
  NvtxRange range("gshard.gated_linear.backward");
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  int* status = reinterpret_cast<int*>(ws);
  const int planes = pl.lin.planes;
  void* dpre = ws + pl.lin.dpre;
  if (fp32) launch_gated_dpre<float, 3>(dh, pre, dpre, status, n_rows, cols, activation, st);
  else if (planes == 2) launch_gated_dpre<__nv_bfloat16, 2>(dh, pre, dpre, status, n_rows, cols, activation, st);
  else launch_gated_dpre<__nv_bfloat16, 1>(dh, pre, dpre, status, n_rows, cols, activation, st);
  return linear_run_gradients(n_rows, K, 2 * cols, fp32, planes, x, w, dpre, dx, dw, pl.lin, ws, true, st);
}

}  // extern "C"
