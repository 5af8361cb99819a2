// AdamW over many tensors at once for gfx950: kernels and host layer of rehyat_adamw_*.
//
// Bound by HBM: gradient, weight and both moments are read once, weight and moments written once; some thirty flops an
// element stand against 18 (moments in 8 bits) to 30 bytes.  A table in device memory, written when the tensors are
// named, cuts all of them into items of 4,096 elements, so that one launch serves any number of tensors of any size
// without the host touching them again.
//
// Moments in 8 bits: groups of 32 elements share an exponent, a power of two, so scaling is exact and every rounding is
// one of the format's own.  m is e4m3 (what the card converts to and from in hardware); v has no sign and needs range
// more than m does: 5 bits of exponent, 3 of mantissa, no zero exponent, which is the leading 11 bits of an fp32
// number less a constant of the group, so that both directions are a few integer instructions.  Rounded to nearest it
// keeps 1/16 of v, 1/32 of the square root that divides the update.  v that is not 0 keeps a code of at least 1: a
// divisor that fell to 0 beside an m that did not would make the update unbounded.
#include <algorithm>
#include <cmath>
#include <new>

#include "rehyat_elem.h"
#include "rehyat_host.h"

namespace rehyat {
namespace {

constexpr int kThreads = 256;
constexpr int kItem = 4096;    // elements of an item: a multiple of the group
constexpr int kGroup = 32;

struct Header {
  int64_t step;      // updates made (the caller may see and set it)
  uint32_t arrived;  // workgroups of the running step that are done
  uint32_t n_tensors;
  int64_t items;
  int64_t pad[5];
};
static_assert(sizeof(Header) == 64, "the tensors' descriptions follow at 64 bytes");

struct Desc {
  void* param;
  float* master;
  const void* grad;
  void *m, *v;
  uint8_t *m_exp, *v_exp;
  int64_t n;
  int32_t first_item, param_type, grad_type, pad;
};
static_assert(sizeof(Desc) == 80, "");

__host__ __device__ inline size_t map_offset(int n_tensors) { return sizeof(Header) + sizeof(Desc) * (size_t)n_tensors; }

// ---- the table ----------------------------------------------------------------------------------------------------

constexpr int kPrepare = 40;   // descriptions a launch carries in its arguments (3.3 KB of them)
struct PrepareArgs {
  Desc desc[kPrepare];
  Header header;
  char* table;
  int first, count;
};

__global__ __launch_bounds__(kThreads) void adamw_prepare_kernel(PrepareArgs a) {
  const Desc& d = a.desc[blockIdx.x];
  const int i = a.first + blockIdx.x;
  if (threadIdx.x == 0) {
    ((Desc*)(a.table + sizeof(Header)))[i] = d;
    if (i == 0) *(Header*)a.table = a.header;
  }
  int32_t* map = (int32_t*)(a.table + map_offset(a.header.n_tensors)) + d.first_item;
  const int64_t items = (d.n + kItem - 1) / kItem;
  for (int64_t k = threadIdx.x; k < items; k += kThreads) map[k] = i;
}

// ---- 8-bit moments ------------------------------------------------------------------------------------------------

__device__ __forceinline__ float power_of_two(int e) { return __builtin_bit_cast(float, (uint32_t)e << 23); }   // 2^(e - 127)

// exponent of a group whose largest magnitude has the bits `top`; `least` keeps factors and codes in range
__device__ __forceinline__ int group_exponent(uint32_t top, int least) {
  const int e = (int)(top >> 23);
  return e >= 254 ? 255 : e < least ? least : e;
}
constexpr int kLeastM = 8, kLeastV = 31;

__device__ __forceinline__ float decode_m(uint32_t code, int e) {
  if (e == 255) return __builtin_nanf("");
  return __builtin_amdgcn_cvt_f32_fp8((int)code, 0) * power_of_two((e < kLeastM ? kLeastM : e) - 7);
}
__device__ __forceinline__ uint32_t encode_m(float m, int e) {
  if (e == 255) return 0;
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(m * power_of_two(261 - e), 0.f, 0, false) & 255;
}
__device__ __forceinline__ float decode_v(uint32_t code, int e) {
  if (e == 255) return __builtin_nanf("");
  return code == 0 ? 0.f : __builtin_bit_cast(float, (code + ((uint32_t)((e < kLeastV ? kLeastV : e) - 30) << 3)) << 20);
}
__device__ __forceinline__ uint32_t encode_v(float v, int e) {
  const uint32_t bits = __builtin_bit_cast(uint32_t, v);
  if (e == 255 || bits == 0) return 0;
  const int code = (int)((bits + 0x7ffffu + ((bits >> 20) & 1)) >> 20) - ((e - 30) << 3);
  return code < 1 ? 1 : code > 255 ? 255 : code;
}

__device__ __forceinline__ float load(int type, const void* p, int64_t i) {
  return type == REHYAT_FP32 ? ((const float*)p)[i]
         : type == REHYAT_BF16 ? Bf16::get(((const uint16_t*)p)[i]) : Fp16::get(((const uint16_t*)p)[i]);
}
__device__ __forceinline__ void store(int type, void* p, int64_t i, float x) {
  if (type == REHYAT_FP32) ((float*)p)[i] = x;
  else ((uint16_t*)p)[i] = type == REHYAT_BF16 ? Bf16::put(x) : Fp16::put(x);
}

// ---- the step -----------------------------------------------------------------------------------------------------

struct StepArgs {
  char* table;
  const float* lr_device;
  double lr, weight_decay, log_beta1, log_beta2;
  float beta1, rest1, beta2, rest2, eps;   // rest = 1 - beta
};

template <int BITS>
__global__ __launch_bounds__(kThreads) void adamw_kernel(StepArgs a) {
  Header* const header = (Header*)a.table;
  const Desc* const descs = (const Desc*)(a.table + sizeof(Header));
  const int32_t* const map = (const int32_t*)(a.table + map_offset(header->n_tensors));
  const int64_t step = header->step + 1;
  const double lr = a.lr_device ? (double)*a.lr_device : a.lr;
  // 1 - beta^t, with log(beta) from the host
  const float rate = (float)(lr / -expm1((double)step * a.log_beta1));
  const float root = (float)(1.0 / sqrt(-expm1((double)step * a.log_beta2)));
  const float keep = (float)(1.0 - lr * a.weight_decay);
  for (int64_t item = blockIdx.x; item < header->items; item += gridDim.x) {
    const Desc d = descs[map[item]];
    const int64_t base = (item - d.first_item) * kItem;
    for (int k = threadIdx.x; k < kItem; k += kThreads) {
      const int64_t i = base + k;
      const bool in = i < d.n;
      float g = 0.f, m = 0.f, v = 0.f, p = 0.f;
      if (in) {
        g = load(d.grad_type, d.grad, i);
        p = d.master ? d.master[i] : load(d.param_type, d.param, i);
      }
      if (BITS == 32) {
        if (in) {
          m = ((const float*)d.m)[i];
          v = ((const float*)d.v)[i];
        }
        m = a.beta1 * m + a.rest1 * g;
        v = a.beta2 * v + a.rest2 * (g * g);
        if (in) {
          ((float*)d.m)[i] = m;
          ((float*)d.v)[i] = v;
        }
      } else {
        if (in) {
          m = decode_m(((const uint8_t*)d.m)[i], d.m_exp[i / kGroup]);
          v = decode_v(((const uint8_t*)d.v)[i], d.v_exp[i / kGroup]);
        }
        // in 64 bits, where products of 24-bit numbers are exact: m, v are the true sums rounded once, so that what
        // lies half way between two codes is decided by the numbers and not by how they were added
        m = (float)fma((double)a.beta1, (double)m, (double)a.rest1 * (double)g);
        v = (float)fma((double)a.beta2, (double)v, (double)a.rest2 * ((double)g * (double)g));
        uint32_t top_m = __builtin_bit_cast(uint32_t, m) & 0x7fffffffu, top_v = __builtin_bit_cast(uint32_t, v) & 0x7fffffffu;
#pragma unroll
        for (int x = 16; x; x >>= 1) {
          const uint32_t om = __shfl_xor(top_m, x), ov = __shfl_xor(top_v, x);
          top_m = om > top_m ? om : top_m;
          top_v = ov > top_v ? ov : top_v;
        }
        const int em = group_exponent(top_m, kLeastM), ev = group_exponent(top_v, kLeastV);
        if (i < (d.n + kGroup - 1) / kGroup * kGroup) {
          ((uint8_t*)d.m)[i] = encode_m(m, em);
          ((uint8_t*)d.v)[i] = encode_v(v, ev);
          if (i % kGroup == 0) {
            d.m_exp[i / kGroup] = em;
            d.v_exp[i / kGroup] = ev;
          }
        }
      }
      p = p * keep - rate * (m / (sqrtf(v) * root + a.eps));
      if (in) {
        if (d.master) d.master[i] = p;
        store(d.param_type, d.param, i, p);
      }
    }
  }
  // the last workgroup counts the update: by then every workgroup has read the count
  __syncthreads();
  if (threadIdx.x == 0 &&
      __hip_atomic_fetch_add(&header->arrived, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1) {
    header->arrived = 0;
    header->step = step;
  }
}

__global__ __launch_bounds__(kThreads) void adamw_moments_kernel(const uint8_t* m, const uint8_t* m_exp, const uint8_t* v,
                                                                 const uint8_t* v_exp, float* m_out, float* v_out,
                                                                 int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= n) return;
  m_out[i] = decode_m(m[i], m_exp[i / kGroup]);
  v_out[i] = decode_v(v[i], v_exp[i / kGroup]);
}

// ---- host ---------------------------------------------------------------------------------------------------------

struct Range {
  uintptr_t lo, hi;
  bool written;
};

// Whether no written range overlaps another range.  `r` is sorted here.
bool apart(Range* r, size_t n) {
  std::sort(r, r + n, [](const Range& x, const Range& y) { return x.lo < y.lo; });
  uintptr_t any = 0, written = 0;   // ends of what came before
  for (size_t i = 0; i < n; ++i) {
    if (r[i].lo < (r[i].written ? any : written)) return false;
    any = std::max(any, r[i].hi);
    if (r[i].written) written = std::max(written, r[i].hi);
  }
  return true;
}

bool fraction(double x) { return x >= 0.0 && x < 1.0; }
bool not_negative(double x) { return std::isfinite(x) && x >= 0.0; }

}  // namespace
}  // namespace rehyat

using namespace rehyat;

extern "C" {

size_t rehyat_adamw_table_bytes(const int64_t* sizes, int n_tensors) {
  if (!sizes || n_tensors < 1) return 0;
  int64_t items = 0;
  for (int i = 0; i < n_tensors; ++i) {
    if (sizes[i] < 0 || sizes[i] >= ((int64_t)1 << 40)) return 0;
    items += (sizes[i] + kItem - 1) / kItem;
    if (items >= ((int64_t)1 << 31)) return 0;
  }
  return align256(map_offset(n_tensors) + (size_t)items * sizeof(int32_t));
}

int rehyat_adamw_prepare(const rehyat_adamw_tensor* tensors, int n_tensors, int state_bits, int64_t step, void* table,
                         size_t table_bytes, rehyat_adamw_plan* plan, void* stream) {
  if (!tensors || !table || !plan) return REHYAT_E_NULL;
  if (n_tensors < 1 || (state_bits != 32 && state_bits != 8) || step < 0) return REHYAT_E_SHAPE;
  if (!aligned(table, 256)) return REHYAT_E_WORKSPACE;
  Range* const ranges = new (std::nothrow) Range[(size_t)n_tensors * 7 + 1];
  if (!ranges) return REHYAT_E_WORKSPACE;
  size_t nr = 0;
  auto range = [&](const void* p, int64_t bytes, bool written) {
    ranges[nr++] = {(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes, written};
  };
  int64_t items = 0;
  int rc = REHYAT_OK;
  for (int i = 0; i < n_tensors && rc == REHYAT_OK; ++i) {
    const rehyat_adamw_tensor& t = tensors[i];
    if (t.n < 0 || t.n >= ((int64_t)1 << 40) || !valid_type(t.param_type) || !valid_type(t.grad_type)) rc = REHYAT_E_SHAPE;
    else if (t.n > 0) {
      const size_t ps = type_bytes(t.param_type), gs = type_bytes(t.grad_type);
      if (!t.param || !t.grad || !t.m || !t.v || (state_bits == 8 && (!t.m_exp || !t.v_exp))) rc = REHYAT_E_NULL;
      else if (!aligned(t.param, ps) || !aligned(t.grad, gs) || !aligned16(t.m) || !aligned16(t.v) ||
               (t.master && !aligned4(t.master)))
        rc = REHYAT_E_SHAPE;
      const int64_t groups = (t.n + kGroup - 1) / kGroup, state = state_bits == 32 ? 4 * t.n : kGroup * groups;
      range(t.param, t.n * ps, true);
      range(t.grad, t.n * gs, false);
      range(t.m, state, true);
      range(t.v, state, true);
      if (t.master) range(t.master, 4 * t.n, true);
      if (state_bits == 8) {
        range(t.m_exp, groups, true);
        range(t.v_exp, groups, true);
      }
      items += (t.n + kItem - 1) / kItem;
      if (items >= ((int64_t)1 << 31)) rc = REHYAT_E_SHAPE;
    }
  }
  const size_t need = align256(map_offset(n_tensors) + (size_t)items * sizeof(int32_t));
  if (rc == REHYAT_OK && items == 0) rc = REHYAT_E_SHAPE;
  if (rc == REHYAT_OK && table_bytes < need) rc = REHYAT_E_WORKSPACE;
  if (rc == REHYAT_OK) {
    range(table, (int64_t)need, true);
    if (!apart(ranges, nr)) rc = REHYAT_E_SHAPE;
  }
  delete[] ranges;
  if (rc != REHYAT_OK) return rc;

  PrepareArgs a{};
  a.header.step = step;
  a.header.n_tensors = (uint32_t)n_tensors;
  a.header.items = items;
  a.table = (char*)table;
  int64_t at = 0;
  for (int first = 0; first < n_tensors; first += kPrepare) {
    a.first = first;
    a.count = std::min(kPrepare, n_tensors - first);
    for (int i = 0; i < a.count; ++i) {
      const rehyat_adamw_tensor& t = tensors[first + i];
      a.desc[i] = {t.param, t.master, t.grad, t.m, t.v, (uint8_t*)t.m_exp, (uint8_t*)t.v_exp, t.n, (int32_t)at,
                   t.param_type, t.grad_type, 0};
      at += (t.n + kItem - 1) / kItem;
    }
    adamw_prepare_kernel<<<a.count, kThreads, 0, (hipStream_t)stream>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(e, "AdamW table kernel launch");
  }
  plan->table = table;
  plan->items = items;
  plan->n_tensors = n_tensors;
  plan->state_bits = state_bits;
  return REHYAT_OK;
}

int rehyat_adamw_step(const rehyat_adamw_plan* plan, const rehyat_adamw_hyper* hyper, void* stream) {
  if (!plan || !hyper || !plan->table) return REHYAT_E_NULL;
  if (plan->items < 1 || plan->n_tensors < 1 || (plan->state_bits != 32 && plan->state_bits != 8)) return REHYAT_E_SHAPE;
  if (!aligned(plan->table, 256)) return REHYAT_E_WORKSPACE;
  if (!not_negative(hyper->lr) || !not_negative(hyper->weight_decay) || !not_negative(hyper->eps) ||
      !((float)hyper->eps > 0.f) || !fraction(hyper->beta1) || !fraction(hyper->beta2))
    return REHYAT_E_SHAPE;
  if (hyper->lr_device && !aligned4(hyper->lr_device)) return REHYAT_E_SHAPE;
  StepArgs a;
  a.table = (char*)plan->table;
  a.lr_device = hyper->lr_device;
  a.lr = hyper->lr;
  a.weight_decay = hyper->weight_decay;
  a.log_beta1 = std::log(hyper->beta1);
  a.log_beta2 = std::log(hyper->beta2);
  a.beta1 = (float)hyper->beta1;
  a.rest1 = (float)(1.0 - hyper->beta1);
  a.beta2 = (float)hyper->beta2;
  a.rest2 = (float)(1.0 - hyper->beta2);
  a.eps = (float)hyper->eps;
  const int grid = (int)std::min<int64_t>(plan->items, 2048);
  if (plan->state_bits == 32) adamw_kernel<32><<<grid, kThreads, 0, (hipStream_t)stream>>>(a);
  else adamw_kernel<8><<<grid, kThreads, 0, (hipStream_t)stream>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(e, "AdamW kernel launch");
  return REHYAT_OK;
}

int rehyat_adamw_moments(const void* m, const void* m_exp, const void* v, const void* v_exp, float* m_out, float* v_out,
                         int64_t n, void* stream) {
  if (!m || !m_exp || !v || !v_exp || !m_out || !v_out) return REHYAT_E_NULL;
  if (n < 1 || n >= ((int64_t)1 << 38)) return REHYAT_E_SHAPE;
  if (!aligned16(m) || !aligned16(v) || !aligned16(m_out) || !aligned16(v_out)) return REHYAT_E_SHAPE;
  adamw_moments_kernel<<<(unsigned)((n + kThreads - 1) / kThreads), kThreads, 0, (hipStream_t)stream>>>(
      (const uint8_t*)m, (const uint8_t*)m_exp, (const uint8_t*)v, (const uint8_t*)v_exp, m_out, v_out, n);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(e, "AdamW moments kernel launch");
  return REHYAT_OK;
}

}  // extern "C"
