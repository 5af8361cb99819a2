// The distillation loss sum w |y_hat - y| and its gradient for gfx950: kernels and host layer of rehyat_distill_loss.
//
// Bound by HBM: y_hat and y are read and the gradient written once, three flops an element.  Workgroups take contiguous
// pieces, eight elements a thread at a time, two of them in flight; each leaves one fp64 sum, and a second launch of one
// workgroup adds those in a fixed order, so that results are the same from call to call.  480p (302 MB): 50.3 us, of them
// 4.6 for the second launch, 6.0 TB/s; a padded pair at 320x480 against an fp32 teacher (605 MB) 104 us, 5.8 TB/s (an
// element a thread 129 and 212 us).
#include <cmath>

#include "rehyat_elem.h"
#include "rehyat_host.h"

namespace rehyat {
namespace {

constexpr int kThreads = 256;
// Elements and rows up to which one workgroup does it all, in one launch instead of two.  In a graph, one and two: 8,192
// elements 3.1 and 4.4 us, 32,768 4.7 and 4.7, 65,536 7.1 and 4.6; a call by itself has 2.5 us less to enqueue.
constexpr int kSmall = 32768, kSmallRows = 4;

struct LossArgs {
  const uint16_t* y_hat;
  const void* y;
  const float* weight;   // [B, N] or null
  uint16_t* grad;
  double* partial;       // [rows, pieces]
  float* loss;
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

// Eight elements of a row: their part of the sum, and their gradients.  Rows of (b, h)s of an odd size begin anywhere.
constexpr int kVec = 8;
template <typename E, bool NT>
struct Eight {
  typedef uint16_t u16x8 __attribute__((ext_vector_type(8), aligned(2)));
  typedef typename E::store teacher __attribute__((ext_vector_type(8), aligned(sizeof(typename E::store))));
  u16x8 y_hat;
  teacher y;
  float w;
  __device__ __forceinline__ float run(float scale, uint16_t* grad) const {
    const float up = w * scale;
    const uint16_t gu = Bf16::put(up), gd = Bf16::put(-up);
    u16x8 g;
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
      uint16_t one;
      sum += element(Bf16::get(y_hat[k]), E::get(y[k]), w, gu, gd, &one);
      g[k] = one;
    }
    if (NT) __builtin_nontemporal_store(g, (u16x8*)grad);
    else *(u16x8*)grad = g;
    return sum;
  }
};

// A workgroup takes elements [lo, hi) of row `r`; its sum on thread 0.
template <typename E, int THREADS, bool NT>
__device__ __forceinline__ double loss_piece(const LossArgs& a, int64_t r, int64_t lo, int64_t hi) {
  typedef typename E::store T;
  typedef Eight<E, NT> V;
  const uint16_t* const y_hat = a.y_hat + r * a.row;
  const T* const y = (const T*)a.y + r * a.row;
  uint16_t* const grad = a.grad + r * a.row;
  const float* const weight = a.weight ? a.weight + (int64_t)((uint32_t)r / (uint32_t)a.H) * a.N : nullptr;
  auto weight_of = [&](int64_t i) { return weight ? weight[(uint32_t)i / (uint32_t)a.d] : 1.f; };
  double sum = 0;
  int64_t i = lo;
  if (!weight || a.d % kVec == 0) {   // eight elements have one weight (lo is a multiple of 8)
    constexpr int kStep = THREADS * kVec;
    auto fetch = [&](int64_t at) {
      V x;
      x.y_hat = *(const typename V::u16x8*)(y_hat + at);
      const typename V::teacher* const t = (const typename V::teacher*)(y + at);
      x.y = NT ? __builtin_nontemporal_load(t) : *t;
      x.w = weight_of(at);
      return x;
    };
    int64_t at = lo + threadIdx.x * kVec;
    for (; at + kStep + kVec <= hi; at += 2 * kStep) {   // two in flight
      const V x = fetch(at), z = fetch(at + kStep);
      sum += x.run(a.scale, grad + at);
      sum += z.run(a.scale, grad + at + kStep);
    }
    if (at + kVec <= hi) sum += fetch(at).run(a.scale, grad + at);
    i = lo + (hi - lo) / kVec * kVec;
  }
  for (i += threadIdx.x; i < hi; i += THREADS) {
    const float w = weight_of(i), up = w * a.scale;
    uint16_t g;
    sum += element(Bf16::get(y_hat[i]), E::get(y[i]), w, Bf16::put(up), Bf16::put(-up), &g);
    grad[i] = g;
  }
  return block_sum<THREADS>(sum);
}

template <typename E, bool NT>
__global__ __launch_bounds__(kThreads) void loss_kernel(LossArgs a) {
  const int64_t lo = blockIdx.x * a.piece, hi = lo + a.piece < a.row ? lo + a.piece : a.row;
  const double sum = loss_piece<E, kThreads, NT>(a, blockIdx.y, lo, hi);
  if (threadIdx.x == 0) a.partial[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = sum;
}

// Few elements: one workgroup, one launch.
template <typename E>
__global__ __launch_bounds__(1024) void loss_small_kernel(LossArgs a, int rows) {
  double sum = 0;
  for (int r = 0; r < rows; ++r) {
    sum += loss_piece<E, 1024, false>(a, r, 0, a.row);
    __syncthreads();   // the sums' shared memory
  }
  if (threadIdx.x == 0) *a.loss = (float)(sum * a.scale);
}

__global__ __launch_bounds__(1024) void loss_finish_kernel(const double* partial, int n, float scale, float* loss) {
  double sum = 0;
  constexpr int kDepth = 8;   // in flight
  for (int i = threadIdx.x; i < n; i += kDepth * 1024) {
    double x[kDepth];
#pragma unroll
    for (int k = 0; k < kDepth; ++k) x[k] = i + k * 1024 < n ? partial[i + k * 1024] : 0.0;
#pragma unroll
    for (int k = 0; k < kDepth; ++k) sum += x[k];
  }
  sum = block_sum<1024>(sum);
  if (threadIdx.x == 0) *loss = (float)(sum * scale);
}

// How a loss of `rows` rows is cut: pieces of at least 2,048 elements (eight a thread), at most about 16,384 of them in all
// (480p: 52.2 us, of 8,192 52.8, of 4,096 53.5, before their sums were read eight at a time, which is 2 us less; with an
// fp32 teacher 106, 109, 115).
void cut(int64_t rows, int64_t row, int64_t* piece, int64_t* pieces) {
  int64_t want = 16384 / rows;
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
  const int64_t n = (int64_t)B * H * N * d;
  if (!ranges_apart(grad, 2 * n, y_hat, 2 * n) || !ranges_apart(grad, 2 * n, y, n * (int64_t)type_bytes(type)) ||
      (weight && !ranges_apart(grad, 2 * n, weight, (int64_t)4 * B * N)))
    return REHYAT_E_SHAPE;
  const size_t need = rehyat_distill_loss_workspace_bytes(B, H, N, d);
  if (!aligned(workspace, 256) || workspace_bytes < need) return REHYAT_E_WORKSPACE;
  const struct {
    const void* at;
    int64_t bytes;
  } used[] = {{y_hat, 2 * n}, {grad, 2 * n}, {y, n * (int64_t)type_bytes(type)}};
  for (const auto& u : used)
    if (!ranges_apart(loss, 4, u.at, u.bytes) || !ranges_apart(workspace, (int64_t)need, u.at, u.bytes)) return REHYAT_E_SHAPE;
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
  a.row = weight ? (int64_t)N * d : n;
  a.loss = loss;
  hipStream_t st = (hipStream_t)stream;
  hipError_t e;
  if (rows * a.row <= kSmall && rows <= kSmallRows) {
    switch (type) {
      case REHYAT_BF16: loss_small_kernel<Bf16><<<1, 1024, 0, st>>>(a, (int)rows); break;
      case REHYAT_FP16: loss_small_kernel<Fp16><<<1, 1024, 0, st>>>(a, (int)rows); break;
      default: loss_small_kernel<Fp32><<<1, 1024, 0, st>>>(a, (int)rows);
    }
    e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(e, "loss kernel launch");
    return REHYAT_OK;
  }
  int64_t pieces;
  cut(rows, a.row, &a.piece, &pieces);
  const dim3 grid((unsigned)pieces, (unsigned)rows);
  // The teacher's output is read once, the gradient not before a pass over as much again: past the caches where they do
  // not hold it all (480p, 302 MB: 50 us against 57; the whole gradient step is the same either way).
  const bool nt = past_caches(rows * a.row * (4 + (int64_t)type_bytes(type)));
  auto* const kernel = type == REHYAT_BF16   ? (nt ? loss_kernel<Bf16, true> : loss_kernel<Bf16, false>)
                       : type == REHYAT_FP16 ? (nt ? loss_kernel<Fp16, true> : loss_kernel<Fp16, false>)
                                             : (nt ? loss_kernel<Fp32, true> : loss_kernel<Fp32, false>);
  kernel<<<grid, kThreads, 0, st>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(e, "loss kernel launch");
  loss_finish_kernel<<<1, 1024, 0, st>>>(a.partial, (int)(pieces * rows), scale, loss);
  e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(e, "loss sum kernel launch");
  return REHYAT_OK;
}

}  // extern "C"
