// The distillation loss sum w |y_hat - y| and its gradient for gfx950: kernels and host layer of rehyat_distill_loss.
//
// Bound by HBM: y_hat and y are read and the gradient written once, three flops an element.  Workgroups take contiguous
// pieces; each leaves one fp64 sum, and a second launch of one workgroup adds those in a fixed order, so that results
// are the same from call to call.
#include <cmath>

#include "rehyat_elem.h"
#include "rehyat_host.h"

namespace rehyat {
namespace {

constexpr int kThreads = 256;

struct LossArgs {
  const uint16_t* y_hat;
  const void* y;
  const float* weight;   // [B, N] or null
  uint16_t* grad;
  double* partial;       // [rows, pieces]
  float scale;
  int64_t row;           // elements of a row of pieces: N d of one (b, h), or everything where there are no weights
  int64_t piece;         // elements of a piece
  int H, N, d;
};

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
  for (int i = 32; i; i >>= 1) x += __shfl_xor(x, i);
  return x;
}

template <int THREADS>
__device__ __forceinline__ double block_sum(double x) {   // on thread 0
  __shared__ double part[THREADS / kWave];
  x = wave_sum(x);
  if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = x;
  __syncthreads();
  if (threadIdx.x == 0)
    for (int i = 1; i < THREADS / kWave; ++i) x += part[i];
  return x;
}

// |D| w and the gradient of one element; `up` and `down` are the gradient's two values
__device__ __forceinline__ float element(float y_hat, float y, float w, uint16_t up, uint16_t down, uint16_t* g) {
  const float diff = y_hat - y;
  if (w == 0.f) {
    *g = 0;
    return 0.f;
  }
  *g = diff > 0.f ? up : diff < 0.f ? down : diff == 0.f ? (uint16_t)0 : (uint16_t)0x7fc0;
  return __builtin_fabsf(diff) * w;
}

template <typename E>
__global__ __launch_bounds__(kThreads) void loss_kernel(LossArgs a) {
  typedef typename E::store T;
  const int64_t lo = blockIdx.x * a.piece, hi = lo + a.piece < a.row ? lo + a.piece : a.row;
  const int64_t base = blockIdx.y * a.row;
  const float* weight = a.weight ? a.weight + (int64_t)(blockIdx.y / a.H) * a.N : nullptr;
  double sum = 0;
  for (int64_t i = lo + threadIdx.x; i < hi; i += kThreads) {
    const float w = weight ? weight[(uint32_t)i / (uint32_t)a.d] : 1.f;
    const float up = weight ? w * a.scale : a.scale;
    uint16_t g;
    sum += element(Bf16::get(a.y_hat[base + i]), E::get(((const T*)a.y)[base + i]), w, Bf16::put(up), Bf16::put(-up), &g);
    a.grad[base + i] = g;
  }
  sum = block_sum<kThreads>(sum);
  if (threadIdx.x == 0) a.partial[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = sum;
}

__global__ __launch_bounds__(1024) void loss_finish_kernel(const double* partial, int n, float scale, float* loss) {
  double sum = 0;
  for (int i = threadIdx.x; i < n; i += 1024) sum += partial[i];
  sum = block_sum<1024>(sum);
  if (threadIdx.x == 0) *loss = (float)(sum * scale);
}

// How a loss of `rows` rows is cut: pieces of at least 2,048 elements, about 4,096 of them in all.
void cut(int64_t rows, int64_t row, int64_t* piece, int64_t* pieces) {
  int64_t want = 4096 / rows;
  if (want < 1) want = 1;
  int64_t p = (row + want - 1) / want;
  p = (p + 2047) / 2048 * 2048;
  *piece = p;
  *pieces = (row + p - 1) / p;
}

bool sizes_ok(int B, int H, int N, int d) {
  return B >= 1 && H >= 1 && N >= 1 && d >= 1 && (int64_t)B * H <= 65535 && (int64_t)N < ((int64_t)1 << 31) / d;
}

}  // namespace
}  // namespace rehyat

using namespace rehyat;

extern "C" {

size_t rehyat_distill_loss_workspace_bytes(int B, int H, int N, int d) {
  if (!sizes_ok(B, H, N, d)) return 0;
  int64_t piece, whole, rows;
  cut(1, (int64_t)B * H * N * d, &piece, &whole);
  cut((int64_t)B * H, (int64_t)N * d, &piece, &rows);
  rows *= (int64_t)B * H;
  return align256((size_t)(whole > rows ? whole : rows) * sizeof(double));
}

int rehyat_distill_loss(const void* y_hat, const void* y, int type, const float* weight, float scale, void* grad,
                        float* loss, int B, int H, int N, int d, void* workspace, size_t workspace_bytes, void* stream) {
  if (!y_hat || !y || !grad || !loss || !workspace) return REHYAT_E_NULL;
  if (!sizes_ok(B, H, N, d) || !valid_type(type) || !std::isfinite(scale)) return REHYAT_E_SHAPE;
  if (!aligned16(y_hat) || !aligned16(y) || !aligned16(grad) || !aligned4(loss) || (weight && !aligned4(weight)))
    return REHYAT_E_SHAPE;
  if (!aligned(workspace, 256) || workspace_bytes < rehyat_distill_loss_workspace_bytes(B, H, N, d))
    return REHYAT_E_WORKSPACE;
  LossArgs a;
  a.y_hat = (const uint16_t*)y_hat;
  a.y = y;
  a.weight = weight;
  a.grad = (uint16_t*)grad;
  a.partial = (double*)workspace;
  a.scale = scale;
  a.H = H;
  a.N = N;
  a.d = d;
  const int64_t rows = weight ? (int64_t)B * H : 1;
  a.row = weight ? (int64_t)N * d : (int64_t)B * H * N * d;
  int64_t pieces;
  cut(rows, a.row, &a.piece, &pieces);
  const dim3 grid((unsigned)pieces, (unsigned)rows);
  hipStream_t st = (hipStream_t)stream;
  switch (type) {
    case REHYAT_BF16: loss_kernel<Bf16><<<grid, kThreads, 0, st>>>(a); break;
    case REHYAT_FP16: loss_kernel<Fp16><<<grid, kThreads, 0, st>>>(a); break;
    default: loss_kernel<Fp32><<<grid, kThreads, 0, st>>>(a);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(e, "loss kernel launch");
  loss_finish_kernel<<<1, 1024, 0, st>>>(a.partial, (int)(pieces * rows), scale, loss);
  e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(e, "loss sum kernel launch");
  return REHYAT_OK;
}

}  // extern "C"
