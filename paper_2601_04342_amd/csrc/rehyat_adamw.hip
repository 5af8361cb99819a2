// AdamW over many tensors at once for gfx950: kernels and host layer of rehyat_adamw_*.
//
// Bound by HBM: gradient, weight and both moments are read once, weight and moments written once; some thirty flops an
// element stand against 18 (moments in 8 bits) to 30 bytes.  A table in device memory, written when the tensors are
// named, cuts all of them into items of 1,024 elements, so that one launch serves any number of tensors of any size
// without the host touching them again.  The eight tensors of one block (71 MB, half in the caches) take 14.1 us, those of
// 25 blocks (1,778 MB) 302 us, 5.9 TB/s; with 8-bit moments (1,075 MB) 186 us, 5.8 TB/s, and 83 us to read those back.
//
// Moments in 8 bits: groups of 32 elements share an exponent, a power of two, so scaling is exact and every rounding is
// one of the format's own.  m is e4m3 (what the card converts to and from in hardware); v has no sign and needs range
// more than m does: 5 bits of exponent, 3 of mantissa, no zero exponent, which is the leading 11 bits of an fp32
// number less a constant of the group, so that both directions are a few integer instructions.  v that is not 0 keeps a
// code of at least 1: a divisor that fell to 0 beside an m that did not would make the update unbounded.
//
// A step of these formats is 1/8 to 1/16 of the value, an update changes v by 1/1000 of it at beta2 = 0.999: rounded to
// nearest, nearly every change would be lost, and v would neither follow the mean of g^2 up (a quarter of it after 3,000
// updates with normal gradients) nor fall when gradients do (13 times it, 5,000 updates after they fell to a tenth).  So
// codes are rounded at random, up with the probability that leaves the mean where it was: v is then right in the mean and
// off by 0.2 of itself, which makes the update's rms 1.03 of what it is with 32 bits.  The random bits are a hash of the
// update's number and the element's place, so runs and replays agree.  The first updates change v by more than a step, and
// are rounded to nearest (hyper.nearest_steps).
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <new>

#include "rehyat_elem.h"
#include "rehyat_host.h"

namespace rehyat {
namespace {

constexpr int kThreads = 256;
constexpr int kItem = 4 * kThreads;    // elements of an item: four a thread
constexpr int kGroup = 32;

// Workgroups a CU holds at most (see adamw_kernel), of 256 CUs.
constexpr int kWaves32 = 4, kWaves8 = 6;

// Workgroups of a step say that they have read `step`, each to one of up to kCounters counters in a cache line of its own,
// as many as arrive at each, and the last of each to `arrived`: atomics on one address are done one after the other, 45 ns
// each, and the step of one block's eight tensors (71 MB) took 97 us with all of 2,048 workgroups on one counter, at its
// end; now, of 1,024 on 32, 14 us.
constexpr int kCounters = 40;
static_assert(kCounters * kCounters >= 256 * kWaves32 && kCounters * kCounters >= 256 * kWaves8, "for the largest grid");
struct Header {
  int64_t step;      // updates made (the caller may see and set it)
  uint32_t arrived;  // counters that are full
  uint32_t pad[29];
  struct {
    uint32_t arrived, pad[31];
  } counter[kCounters];
};
static_assert(sizeof(Header) == 128 * (1 + kCounters), "lines of 128 bytes; the tensors' descriptions follow");

struct Desc {
  void* param;
  float* master;
  const void* grad;
  void *m, *v;
  uint8_t *m_exp, *v_exp;
  int64_t n;
  int32_t first_item, param_type, grad_type, pad;
};

__host__ __device__ inline size_t map_offset(int n_tensors) { return sizeof(Header) + sizeof(Desc) * (size_t)n_tensors; }

// ---- the table ----------------------------------------------------------------------------------------------------

constexpr int kPrepare = 40;   // descriptions a launch carries in its arguments (3.3 KB of them)
struct PrepareArgs {
  Desc desc[kPrepare];
  char* table;
  int64_t step;
  int first, n_tensors;
};

__global__ __launch_bounds__(kThreads) void adamw_prepare_kernel(PrepareArgs a) {
  const Desc& d = a.desc[blockIdx.x];
  const int i = a.first + blockIdx.x;
  if (threadIdx.x == 0) ((Desc*)(a.table + sizeof(Header)))[i] = d;
  if (i == 0) {
    Header* const h = (Header*)a.table;
    if (threadIdx.x == 0) {
      h->step = a.step;
      h->arrived = 0;
    }
    for (int k = threadIdx.x; k < kCounters; k += kThreads) h->counter[k].arrived = 0;
  }
  int32_t* map = (int32_t*)(a.table + map_offset(a.n_tensors)) + d.first_item;
  const int64_t items = (d.n + kItem - 1) / kItem;
  for (int64_t k = threadIdx.x; k < items; k += kThreads) map[k] = i;
}

// ---- 8-bit moments ------------------------------------------------------------------------------------------------

// (of a value, not of a vector's element in place: this compiler's bit cast of one takes the vector's first)
__device__ __forceinline__ uint32_t bits_of(float x) { return __builtin_bit_cast(uint32_t, x); }
__device__ __forceinline__ float power_of_two(int e) { return __builtin_bit_cast(float, (uint32_t)e << 23); }   // 2^(e - 127)

// exponent of a group whose largest magnitude has the bits `top`; `least` keeps factors and codes in range
__device__ __forceinline__ int group_exponent(uint32_t top, int least) {
  const int e = (int)(top >> 23);
  return e >= 254 ? 255 : e < least ? least : e;
}
constexpr int kLeastM = 8, kLeastV = 31;

// four codes of one group at a time, as they stand in a word
__device__ __forceinline__ f32x4 decode_m(uint32_t codes, int e) {
  const float f = e == 255 ? __builtin_nanf("") : power_of_two((e < kLeastM ? kLeastM : e) - 7);
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
  return f32x4{lo[0] * f, lo[1] * f, hi[0] * f, hi[1] * f};
}
__device__ __forceinline__ uint32_t encode_m(f32x4 m, int e) {
  const float f = power_of_two(261 - e);
  int codes = __builtin_amdgcn_cvt_pk_fp8_f32(m[0] * f, m[1] * f, 0, false);
  codes = __builtin_amdgcn_cvt_pk_fp8_f32(m[2] * f, m[3] * f, codes, true);
  return e == 255 ? 0u : (uint32_t)codes;
}
// (a group whose exponent is 255 has codes of 255, which under 254 are not numbers)
__device__ __forceinline__ f32x4 decode_v(uint32_t codes, int e) {
  const uint32_t least = (uint32_t)((e < kLeastV ? kLeastV : e > 254 ? 254 : e) - 30) << 3;
  f32x4 x;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t c = codes >> (8 * k) & 255;
    x[k] = c == 0 ? 0.f : __builtin_bit_cast(float, (c + least) << 20);
  }
  return x;
}
// one code of v, of an fp32 number's bits and what is added to them before those beyond the code are cut off
__device__ __forceinline__ uint32_t code_v(uint32_t bits, uint32_t more, int e) {
  int c = (int)((bits + more) >> 20) - ((e - 30) << 3);
  c = c < 1 ? 1 : c > 255 ? 255 : c;
  return bits == 0 ? 0u : (uint32_t)c;
}
__device__ __forceinline__ uint32_t encode_v(f32x4 v, int e) {
  uint32_t codes = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t bits = bits_of(v[k]);
    codes |= code_v(bits, 0x7ffffu + ((bits >> 20) & 1), e) << (8 * k);
  }
  return e == 255 ? ~0u : codes;
}

// 32 bits of x's that differ in any way: two rounds of folding the upper half down and multiplying, with the fractions of
// the roots of 2 and 3 as odd factors.
__device__ __forceinline__ uint32_t scatter(uint32_t x) {
  x ^= x >> 16;
  x *= 0x6a09e667u;
  x ^= x >> 15;
  x *= 0xbb67ae85u;
  return x ^ x >> 16;
}
// Codes rounded up with a probability of how far the value is on its way there: 20 random bits are added to the 20 that the
// code does not keep of v, and 16 (with half of the last) to those that it does not keep of m.  An element's two share the
// four bits that count least for v.  For m the card has an instruction, which adds the upper 20 bits of its second
// operand (below e4m3's least exponent to the bits behind its least step); with integers instead 25 blocks take 4 us more.
// Four elements share a hash, each with a byte of its own in front (a hash for each: 3 us more).
__device__ __forceinline__ void encode_random(f32x4 m, f32x4 v, int em, int ev, uint32_t hash, uint32_t* cm, uint32_t* cv) {
  const float f = power_of_two(261 - em);
  const uint32_t r[4] = {hash, hash << 8 | hash >> 24, hash << 16 | hash >> 16, hash << 24 | hash >> 8};
  auto bits_m = [&](int k) { return (int)(r[k] << 16 | 0x8000); };
  int x = __builtin_amdgcn_cvt_sr_fp8_f32(m[0] * f, bits_m(0), 0, 0);
  x = __builtin_amdgcn_cvt_sr_fp8_f32(m[1] * f, bits_m(1), x, 1);
  x = __builtin_amdgcn_cvt_sr_fp8_f32(m[2] * f, bits_m(2), x, 2);
  x = __builtin_amdgcn_cvt_sr_fp8_f32(m[3] * f, bits_m(3), x, 3);
  uint32_t y = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) y |= code_v(bits_of(v[k]), r[k] >> 12, ev) << (8 * k);
  *cm = em == 255 ? 0u : (uint32_t)x;
  *cv = ev == 255 ? ~0u : y;
}
// largest over the eight lanes that hold a group: neighbours, pairs, then the two halves mirrored
__device__ __forceinline__ uint32_t group_max(uint32_t x) {
  auto other = [](uint32_t y, auto ctrl) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)y, decltype(ctrl)::value, 0xf, 0xf, true);
  };
  uint32_t y = other(x, std::integral_constant<int, 0xb1>{});    // quad_perm 1 0 3 2
  x = y > x ? y : x;
  y = other(x, std::integral_constant<int, 0x4e>{});             // quad_perm 2 3 0 1
  x = y > x ? y : x;
  y = other(x, std::integral_constant<int, 0x141>{});            // lanes 0 .. 7 reversed
  return y > x ? y : x;
}

// Four elements from i on; a caller's tensor may begin at any element, and end inside the four (`left` of them are there).
// The pointers come out of the table, where the compiler cannot see that they are to global memory; `p` is the same for
// the whole workgroup and i a 32-bit index from it (one register of offsets instead of two of address for each tensor).
typedef f32x4 f32x4_e __attribute__((aligned(4)));
typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
typedef u16x4 u16x4_e __attribute__((aligned(2)));
template <typename T>
using global = __attribute__((address_space(1))) T;
template <typename T>
__device__ __forceinline__ global<T>* at(const void* p, uint32_t i) { return (global<T>*)(T*)p + i; }
// NT: past the caches, see past_caches.
template <bool NT, typename E, typename V>
__device__ __forceinline__ f32x4 load4(const void* p, uint32_t i, int left) {
  const global<typename E::store>* const q = at<typename E::store>(p, i);
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  if (left >= 4) {
    const V y = NT ? __builtin_nontemporal_load((const global<V>*)q) : *(const global<V>*)q;
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = E::get(y[k]);
  } else {
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (k < left) x[k] = E::get(q[k]);
  }
  return x;
}
template <bool NT, typename E, typename V>
__device__ __forceinline__ void store4(void* p, uint32_t i, int left, f32x4 x) {
  global<typename E::store>* const q = at<typename E::store>(p, i);
  if (left >= 4) {
    V y;
#pragma unroll
    for (int k = 0; k < 4; ++k) y[k] = E::put(x[k]);
    if (NT) __builtin_nontemporal_store(y, (global<V>*)q);
    else *(global<V>*)q = y;
  } else {
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (k < left) q[k] = E::put(x[k]);
  }
}
template <bool NT>
__device__ __forceinline__ f32x4 load(int type, const void* p, uint32_t i, int left) {
  if (type == REHYAT_FP32) return load4<NT, Fp32, f32x4_e>(p, i, left);
  if (type == REHYAT_BF16) return load4<NT, Bf16, u16x4_e>(p, i, left);
  return load4<NT, Fp16, u16x4_e>(p, i, left);
}
template <bool NT>
__device__ __forceinline__ void store(int type, void* p, uint32_t i, int left, f32x4 x) {
  if (type == REHYAT_FP32) store4<NT, Fp32, f32x4_e>(p, i, left, x);
  else if (type == REHYAT_BF16) store4<NT, Bf16, u16x4_e>(p, i, left, x);
  else store4<NT, Fp16, u16x4_e>(p, i, left, x);
}

// ---- the step -----------------------------------------------------------------------------------------------------

struct StepArgs {
  char* table;
  const float* lr_device;
  double lr, weight_decay, log_beta1, log_beta2;
  float beta1, rest1, beta2, rest2, eps;   // rest = 1 - beta
  double exact[4];                         // the first four in 64 bits
  float keep;                              // 1 - lr weight_decay
  int32_t n_tensors, counters;
  int64_t items, nearest_steps;
};

// Root and, in the step, reciprocal are the hardware's approximations, off by one in the last place: the update keeps 21
// bits and more, and with exact ones, 18 instructions an element more, a step of 25 blocks with 8-bit moments took 11 us
// longer, of 245, and with 32 bits a step of one block 0.6 us longer, of 12.7.  The root's argument is scaled out of the
// denormals, which the instruction takes for 0; divisors are normal numbers, since eps is.
__device__ __forceinline__ float root_of(float v) {
  const bool small = v < 0x1p-96f;
  return __builtin_amdgcn_sqrtf(small ? v * 0x1p32f : v) * (small ? 0x1p-16f : 1.f);
}

// One item: where it begins in each tensor.
struct Piece {
  void* param;
  float* master;
  const void* grad;
  void *m, *v;
  uint8_t *m_exp, *v_exp;
  int32_t left;                   // elements from there to the end of the tensors, at most kItem
  int32_t param_type, grad_type;
};
template <int BITS>
__device__ __forceinline__ Piece piece_of(const Desc& d, int64_t item) {
  const int64_t lo = (item - d.first_item) * kItem;
  Piece c;
  c.param = (char*)d.param + lo * (d.param_type == REHYAT_FP32 ? 4 : 2);
  c.master = d.master ? d.master + lo : nullptr;
  c.grad = (const char*)d.grad + lo * (d.grad_type == REHYAT_FP32 ? 4 : 2);
  c.m = (char*)d.m + lo * (BITS / 8);
  c.v = (char*)d.v + lo * (BITS / 8);
  c.m_exp = d.m_exp + lo / kGroup;
  c.v_exp = d.v_exp + lo / kGroup;
  c.left = d.n - lo < kItem ? (int)(d.n - lo) : kItem;
  c.param_type = d.param_type;
  c.grad_type = d.grad_type;
  return c;
}

// What a thread holds of an item: four elements.
template <int BITS>
struct Quad {
  f32x4 g, p;
  f32x4 m, v;            // 32 bits
  uint32_t cm, cv;       // 8 bits: codes, and the group's exponents
  int em, ev;
};

// Workgroups a CU holds (kWaves32, kWaves8), which is also waves a SIMD: one round of them walks over all items.  Shared
// memory that nobody uses keeps further ones out, so that no CU gets more of the round than another.  Of 3 / 4 / 5 / 6 the
// 200 tensors of 25 blocks take 400 / 316 / 319 / 324 us (more of them open more rows of memory than it holds); 8-bit
// moments, with more arithmetic to hide, 473 / 316 / 303 / 299, their values' reading included (before their codes went
// through the caches, with which 6 take 278).
template <int BITS, bool NT>
__global__ __launch_bounds__(kThreads, BITS == 32 ? kWaves32 : kWaves8) void adamw_kernel(StepArgs a) {
  Header* const header = (Header*)a.table;
  const Desc* const descs = (const Desc*)(a.table + sizeof(Header));
  const int32_t* const map = (const int32_t*)(a.table + map_offset(a.n_tensors));
  const uint32_t i = 4 * threadIdx.x;   // the thread's first element of an item
  // whether the thread has a part in an item; with 8 bits the lanes of a group stay together, whose codes reach to its end
  auto active = [&](const Piece& c) { return (int)(BITS == 32 ? i : i / kGroup * kGroup) < c.left; };
  Piece c;
  Quad<BITS> x;
  auto fetch = [&](int64_t item) {
    c = piece_of<BITS>(descs[map[item]], item);
    if (!active(c)) return;
    const int left = c.left - (int)i;
    x.g = load<NT>(c.grad_type, c.grad, i, left);
    x.p = c.master ? load4<NT, Fp32, f32x4_e>(c.master, i, left) : load<NT>(c.param_type, c.param, i, left);
    if (BITS == 32) {
      x.m = load4<NT, Fp32, f32x4>(c.m, i, left);
      x.v = load4<NT, Fp32, f32x4>(c.v, i, left);
    } else {
      x.cm = *at<uint32_t>(c.m, i / 4);
      x.cv = *at<uint32_t>(c.v, i / 4);
      x.em = *at<uint8_t>(c.m_exp, i / kGroup);
      x.ev = *at<uint8_t>(c.v_exp, i / kGroup);
    }
  };
  fetch(blockIdx.x);

  // factors of this update, and the workgroup's arrival (its answer is not looked at before the end)
  __shared__ float factors[3];
  __shared__ int64_t count;
  __shared__ uint32_t rounding[2];   // whether to nearest; otherwise what the update's number adds to the hash
  uint32_t before = 0;
  const uint32_t counters = a.counters, mine = blockIdx.x % counters;
  if (threadIdx.x < 2) {   // 1 - beta^t of either beta, with log(beta) from the host
    const int64_t step = header->step + 1;
    if (threadIdx.x == 0) count = step;
    const float lr = a.lr_device ? *a.lr_device : (float)a.lr;
    const float c = -expm1f((float)((double)step * (threadIdx.x ? a.log_beta2 : a.log_beta1)));
    factors[threadIdx.x] = threadIdx.x ? 1.f / sqrtf(c) : lr / c;
    factors[2] = a.lr_device ? (float)(1.0 - (double)lr * a.weight_decay) : a.keep;
    rounding[0] = step <= a.nearest_steps;
    rounding[1] = scatter((uint32_t)step * 0x9e3779b9u + (uint32_t)(step >> 32));   // the golden ratio's fraction
  }
  __syncthreads();
  if (threadIdx.x == 0)
    before = __hip_atomic_fetch_add(&header->counter[mine].arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  // (in scalar registers, and the count in shared memory: the others are just as many as six waves may have, and with three
  // of them spilled a million parameters took 8.1 us instead of 7.7)
  auto scalar = [](uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); };
  auto factor = [&](int k) { return __builtin_bit_cast(float, scalar(bits_of(factors[k]))); };
  const float rate = factor(0), root = factor(1), keep = factor(2);
  const bool nearest = scalar(rounding[0]);
  const uint32_t key = scalar(rounding[1]);

  for (int64_t item = blockIdx.x; item < a.items; ) {
    const Piece e = c;
    const Quad<BITS> y = x;
    const int64_t place = item * kThreads;   // of the item's first four elements among all
    item += gridDim.x;
    if (item < a.items) fetch(item);   // in flight behind what follows
    if (!active(e)) continue;
    const int left = e.left - (int)i;
    f32x4 m, v, p = y.p;
    if (BITS == 32) {
      m = a.beta1 * y.m + a.rest1 * y.g;
      v = a.beta2 * y.v + a.rest2 * (y.g * y.g);
      store4<NT, Fp32, f32x4>(e.m, i, left, m);
      store4<NT, Fp32, f32x4>(e.v, i, left, v);
    } else {
      m = decode_m(y.cm, y.em);
      v = decode_v(y.cv, y.ev);
      if (nearest) {
        // in 64 bits, where products of 24-bit numbers are exact: sums rounded once there and once to fp32, so that what
        // lies half way between two codes is decided by the numbers and not by how they were added
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const double g = y.g[k];
          m[k] = (float)fma(a.exact[0], (double)m[k], a.exact[1] * g);
          v[k] = (float)fma(a.exact[2], (double)v[k], a.exact[3] * (g * g));
        }
      } else {
        m = a.beta1 * m + a.rest1 * y.g;
        v = a.beta2 * v + a.rest2 * (y.g * y.g);
      }
      uint32_t top_m = 0, top_v = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t bm = bits_of(m[k]) & 0x7fffffffu, bv = bits_of(v[k]) & 0x7fffffffu;
        top_m = bm > top_m ? bm : top_m;
        top_v = bv > top_v ? bv : top_v;
      }
      const int em = group_exponent(group_max(top_m), kLeastM), ev = group_exponent(group_max(top_v), kLeastV);
      uint32_t cm, cv;
      if (nearest) cm = encode_m(m, em), cv = encode_v(v, ev);
      else   // (what does not fit 32 bits of the four elements' place changes the key)
        encode_random(m, v, em, ev, scatter(((uint32_t)place + threadIdx.x) ^ (key + (uint32_t)(place >> 32) * 0x9e3779b9u)), &cm,
                      &cv);
      *at<uint32_t>(e.m, i / 4) = cm;
      *at<uint32_t>(e.v, i / 4) = cv;
      if (threadIdx.x % (kGroup / 4) == 0) {
        *at<uint8_t>(e.m_exp, i / kGroup) = em;
        *at<uint8_t>(e.v_exp, i / kGroup) = ev;
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) p[k] = p[k] * keep - rate * (m[k] * __builtin_amdgcn_rcpf(root_of(v[k]) * root + a.eps));
    if (e.master) store4<NT, Fp32, f32x4_e>(e.master, i, left, p);
    store<NT>(e.param_type, e.param, i, left, p);
  }

  // the last to have read the count writes the next one
  if (threadIdx.x == 0 && before == (gridDim.x - mine + counters - 1) / counters - 1 &&
      __hip_atomic_fetch_add(&header->arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == counters - 1) {
    for (uint32_t k = 0; k < counters; ++k)
      __hip_atomic_store(&header->counter[k].arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(&header->arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(&header->step, count, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
}

template <bool NT>
__global__ __launch_bounds__(kThreads) void adamw_moments_kernel(const uint8_t* m, const uint8_t* m_exp, const uint8_t* v,
                                                                 const uint8_t* v_exp, float* m_out, float* v_out,
                                                                 int64_t n) {
  const uint32_t i = 4 * (blockIdx.x * kThreads + threadIdx.x);   // n is 2^32 at most
  if (i >= n) return;
  const int left = n - i < 4 ? (int)(n - i) : 4;
  store4<NT, Fp32, f32x4>(m_out, i, left, decode_m(*(const uint32_t*)(m + i), m_exp[i / kGroup]));
  store4<NT, Fp32, f32x4>(v_out, i, left, decode_v(*(const uint32_t*)(v + i), v_exp[i / kGroup]));
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
bool not_negative(double x) { return x >= 0.0 && x <= FLT_MAX; }

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
  a.step = step;
  a.n_tensors = n_tensors;
  a.table = (char*)table;
  int64_t at = 0;
  for (int first = 0; first < n_tensors; first += kPrepare) {
    a.first = first;
    const int count = std::min(kPrepare, n_tensors - first);
    for (int i = 0; i < count; ++i) {
      const rehyat_adamw_tensor& t = tensors[first + i];
      a.desc[i] = {t.param, t.master, t.grad, t.m, t.v, (uint8_t*)t.m_exp, (uint8_t*)t.v_exp, t.n, (int32_t)at,
                   t.param_type, t.grad_type, 0};
      at += (t.n + kItem - 1) / kItem;
    }
    adamw_prepare_kernel<<<count, kThreads, 0, (hipStream_t)stream>>>(a);
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
      !((float)hyper->eps >= FLT_MIN) || !fraction(hyper->beta1) || !fraction(hyper->beta2) || hyper->nearest_steps < 0)
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
  a.exact[0] = a.beta1;
  a.exact[1] = a.rest1;
  a.exact[2] = a.beta2;
  a.exact[3] = a.rest2;
  a.eps = (float)hyper->eps;
  a.keep = (float)(1.0 - hyper->lr * hyper->weight_decay);
  a.n_tensors = plan->n_tensors;
  a.items = plan->items;
  a.nearest_steps = hyper->nearest_steps;
  const int waves = plan->state_bits == 32 ? kWaves32 : kWaves8, lds = (160 * 1024 / waves - 64) & ~1023;
  const int grid = (int)std::min<int64_t>(plan->items, 256 * waves);
  a.counters = 1;   // as many as arrive at each
  while (a.counters * a.counters < grid) ++a.counters;
  // past the caches 1,778 MB take 316 us against 338, through them 71 MB 14.1 against 15.2; codes of 8-bit moments, half a
  // line to a wave's instruction, always go through them (278 us against 299)
  const bool nt = past_caches(plan->items * kItem * (plan->state_bits == 32 ? 30 : 18));
  auto* const kernel = plan->state_bits == 32 ? (nt ? adamw_kernel<32, true> : adamw_kernel<32, false>)
                                              : (nt ? adamw_kernel<8, true> : adamw_kernel<8, false>);
  kernel<<<grid, kThreads, lds, (hipStream_t)stream>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(e, "AdamW kernel launch");
  return REHYAT_OK;
}

int rehyat_adamw_moments(const void* m, const void* m_exp, const void* v, const void* v_exp, float* m_out, float* v_out,
                         int64_t n, void* stream) {
  if (!m || !m_exp || !v || !v_exp || !m_out || !v_out) return REHYAT_E_NULL;
  if (n < 1 || n >= ((int64_t)1 << 38)) return REHYAT_E_SHAPE;
  if (!aligned16(m) || !aligned16(v) || !aligned16(m_out) || !aligned16(v_out)) return REHYAT_E_SHAPE;
  const int64_t groups = (n + kGroup - 1) / kGroup;
  Range ranges[] = {{(uintptr_t)m, (uintptr_t)m + kGroup * groups, false}, {(uintptr_t)v, (uintptr_t)v + kGroup * groups, false},
                    {(uintptr_t)m_exp, (uintptr_t)m_exp + groups, false}, {(uintptr_t)v_exp, (uintptr_t)v_exp + groups, false},
                    {(uintptr_t)m_out, (uintptr_t)m_out + 4 * n, true}, {(uintptr_t)v_out, (uintptr_t)v_out + 4 * n, true}};
  if (!apart(ranges, 6)) return REHYAT_E_SHAPE;
  auto* const kernel = past_caches(10 * n) ? adamw_moments_kernel<true> : adamw_moments_kernel<false>;
  // elements of a launch, as its threads, are counted in 32 bits
  for (int64_t lo = 0, most = (int64_t)1 << 32; lo < n; lo += most) {
    const int64_t count = std::min(n - lo, most);
    kernel<<<(unsigned)((count + kItem - 1) / kItem), kThreads, 0, (hipStream_t)stream>>>(
        (const uint8_t*)m + lo, (const uint8_t*)m_exp + lo / kGroup, (const uint8_t*)v + lo,
        (const uint8_t*)v_exp + lo / kGroup, m_out + lo, v_out + lo, count);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(e, "AdamW moments kernel launch");
  }
  return REHYAT_OK;
}

}  // extern "C"
