// Rotary positions of queries and keys for gfx950: kernel and host layer of rehyat_rope.
//
// Pair i of a head row turns by angle = position * frequency.  Frequencies come as 2^-64 parts of a turn a position, so
// the 64-bit product, which wraps, IS the angle modulo a turn; its upper 32 bits (2^-32 of a turn is 1.5e-9 rad) give the
// quadrant and an angle within an eighth of a turn, where short series for cos and sin serve.  No reduction adds to what a
// far position makes of the frequency's own rounding: position times 2^-64 turns at most, which 2^32 positions take to that
// cut-off (what a double is off by is some hundred times as much, at one radian a position).
//
// Bound by HBM: each element is read and written once, and needs 3 flops.  A thread keeps the cos and sin of its one or
// two pairs and walks over the heads of its token with them, since they are the same for every head, four heads in
// flight.  q and k of a 480p layer, 403 MB: 73.4 us, 5.5 TB/s; the gradient of a guidance pair, 805 MB, 142 us, 5.7 TB/s;
// half of each head in fp16, 126 MB, 24.8 us.  One head at a time they took 110, 222 and 62 us; with 16 bytes a
// thread, four and eight pairs of angles, 77.5, 150 and 29.  Stored past the caches the first takes 6 us less, and the
// attention behind it, which then finds nothing there, 14 us more.
#include <cmath>
#include <initializer_list>

#include "rehyat_elem.h"
#include "rehyat_host.h"

namespace rehyat {
namespace {

// Heads a thread walks over, at most, and the waves a launch should have for it: many heads share their angles, but few
// waves do not fill the chip.  q and k of (sequences, heads, tokens, width), half layout, with 1,024 / 2,048 / 4,096 /
// 16,384 waves wanted: (1, 12, 512, 128) 4.0 / 3.8 / 4.7 / 4.7 us, (2, 12, 1560, 128) 7.9 / 7.9 / 7.5 / 11.0,
// (1, 12, 4096, 128) 9.5 / 9.5 / 9.5 / 13.2.  At most 8 heads instead of 16: the gradient of a pair 157 us, not 142.
constexpr int kMostHeads = 16, kWaves = 2048;

struct RopeOperand {
  const void* x;
  void* out;
  int64_t xb, xh, xn, ob, oh, on;
  int heads;
};

struct RopeArgs {
  RopeOperand op[2];
  int groups0;                   // blockIdx.y below it: heads of op[0], from it on: of op[1]
  int group;                     // heads of a group
  const uint64_t* turns;
  const void* pos;               // explicit positions, or null
  int64_t pos_b, pos_n;
  uint64_t start;
  int pos_bits;
  uint32_t items, slots;         // B * N * slots; pieces of a row
  uint32_t N, frame, cols;       // frame: tokens of one step of the first axis
  int d, rot, axes, sec1, sec2;  // pairs from sec1 on belong to axis 1, from sec2 on to axis 2
  uint32_t copies_from;          // slots from here on copy
  float scale, sign;
};

// cos and sin of an angle given in 2^-32 turns: within an eighth of a turn of the nearest quarter, the series in the
// angle (the first term left out is 2.5e-9 of the result at most), then the quarter turns.
__device__ __forceinline__ void cos_sin(uint32_t t, float* c, float* s) {
  const uint32_t quarter = (t + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(t - (quarter << 30)) * 1.46291807926715968e-9f;   // 2 pi 2^-32
  const float y = x * x;
  const float sn = x + x * y * (-1.f / 6 + y * (1.f / 120 + y * (-1.f / 5040 + y * (1.f / 362880))));
  const float cs = 1.f + y * (-0.5f + y * (1.f / 24 + y * (-1.f / 720 + y * (1.f / 40320 + y * (-1.f / 3628800)))));
  const float a = quarter & 1 ? sn : cs, b = quarter & 1 ? cs : sn;
  *c = quarter == 1 || quarter == 2 ? -a : a;
  *s = quarter >= 2 ? -b : b;
}

// V elements of a row that stand together, loaded and stored as one; rows begin at any element (the first of them one, two
// or four elements off 16 bytes: 32.3 us where 31.4 are taken otherwise).
template <typename E, int V>
struct Vec {
  typedef typename E::store raw __attribute__((ext_vector_type(V), aligned(sizeof(typename E::store))));
  static __device__ __forceinline__ raw load(const typename E::store* p) { return *(const raw*)p; }
  static __device__ __forceinline__ void store(typename E::store* p, raw x) { *(raw*)p = x; }
  static __device__ __forceinline__ float get(raw x, int i) { return E::get(x[i]); }
};
template <typename E>
struct Vec<E, 1> {
  typedef typename E::store raw;
  static __device__ __forceinline__ raw load(const raw* p) { return *p; }
  static __device__ __forceinline__ void store(raw* p, raw x) { *p = x; }
  static __device__ __forceinline__ float get(raw x, int) { return E::get(x); }
};
template <typename E, int V>
__device__ __forceinline__ typename Vec<E, V>::raw round_all(const float* x) {
  typename Vec<E, V>::raw r;
  if constexpr (V == 1) {
    r = E::put(x[0]);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) r[i] = E::put(x[i]);
  }
  return r;
}

// A thread holds V pairs' worth of a row: with the half layout V elements of either half, otherwise V elements in a row.
// Beyond the rotated part it holds as many elements, which it copies: `keep`.
template <typename E, int LAYOUT, int V>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  typedef typename E::store T;
  typedef Vec<E, V> W;
  typedef typename W::raw R;
  constexpr bool kHalf = LAYOUT == REHYAT_ROPE_HALF;
  constexpr int kPairs = kHalf ? V : V / 2;
  const uint32_t i = blockIdx.x * 256 + threadIdx.x;
  if (i >= a.items) return;
  const uint32_t token = i / a.slots, slot = i - token * a.slots;
  const uint32_t b = token / a.N, n = token - b * a.N;
  const bool second = (int)blockIdx.y >= a.groups0;
  const RopeOperand& op = second ? a.op[1] : a.op[0];
  const int h0 = ((int)blockIdx.y - (second ? a.groups0 : 0)) * a.group;
  const int h1 = h0 + a.group < op.heads ? h0 + a.group : op.heads;

  const bool keep = slot >= a.copies_from;
  uint32_t first, other = 0;
  if (kHalf) {
    first = keep ? a.rot + 2 * V * (slot - a.copies_from) : V * slot;
    other = keep ? first + V : first + a.rot / 2;
    if (other >= (uint32_t)a.d) other = first;   // an odd number of copied pieces: the last twice
  } else {
    first = V * slot;
  }
  const T* x = (const T*)op.x + b * op.xb + n * op.xn + h0 * op.xh + first;
  T* out = (T*)op.out + b * op.ob + n * op.on + h0 * op.oh + first;
  const int64_t to_other = (int64_t)other - first;

  float c[kPairs], s[kPairs];
  if (!keep) {
    uint64_t pos[3];   // modulo 2^64
    if (a.pos) {
      const int64_t at = b * a.pos_b + n * a.pos_n;
#pragma unroll
      for (int x = 0; x < 3; ++x)
        if (x < a.axes) pos[x] = a.pos_bits == 64 ? ((const int64_t*)a.pos)[at + x] : (int64_t)((const int32_t*)a.pos)[at + x];
    } else {
      const uint32_t f = n / a.frame, r = n - f * a.frame, y = r / a.cols;
      pos[0] = a.start + f;
      pos[1] = a.axes == 2 ? r : y;
      pos[2] = r - y * a.cols;
    }
    const uint32_t pair0 = kPairs * slot;
#pragma unroll
    for (int k = 0; k < kPairs; ++k) {
      const int pair = pair0 + k;
      const uint64_t p = pair >= a.sec2 ? pos[2] : pair >= a.sec1 ? pos[1] : pos[0];
      cos_sin((uint32_t)((p * a.turns[pair]) >> 32), &c[k], &s[k]);
      c[k] *= a.scale;
      s[k] *= a.scale * a.sign;
    }
  }
  constexpr int kDepth = 4;   // heads in flight
  for (int h = h0; h < h1; h += kDepth, x += kDepth * op.xh, out += kDepth * op.oh) {
    R u[kDepth], v[kDepth];
#pragma unroll
    for (int k = 0; k < kDepth; ++k)
      if (h + k < h1) {
        u[k] = W::load(x + k * op.xh);
        if (kHalf) v[k] = W::load(x + k * op.xh + to_other);
      }
#pragma unroll
    for (int k = 0; k < kDepth; ++k)
      if (h + k < h1) {
        if (!keep) {
          float lo[V], hi[V];
#pragma unroll
          for (int j = 0; j < kPairs; ++j) {
            const float p = kHalf ? W::get(u[k], j) : W::get(u[k], 2 * j), q = kHalf ? W::get(v[k], j) : W::get(u[k], 2 * j + 1);
            const float rp = p * c[j] - q * s[j], rq = q * c[j] + p * s[j];
            if (kHalf) lo[j] = rp, hi[j] = rq;
            else lo[2 * j] = rp, lo[2 * j + 1] = rq;
          }
          u[k] = round_all<E, V>(lo);
          if (kHalf) v[k] = round_all<E, V>(hi);
        }
        W::store(out + k * op.oh, u[k]);
        if (kHalf) W::store(out + k * op.oh + to_other, v[k]);
      }
  }
}

template <typename E>
void launch(const RopeArgs& a, int layout, int v, dim3 grid, hipStream_t st) {
  if (layout == REHYAT_ROPE_INTERLEAVED) rope_kernel<E, REHYAT_ROPE_INTERLEAVED, 2><<<grid, 256, 0, st>>>(a);
  else if (v == 2) rope_kernel<E, REHYAT_ROPE_HALF, 2><<<grid, 256, 0, st>>>(a);
  else rope_kernel<E, REHYAT_ROPE_HALF, 1><<<grid, 256, 0, st>>>(a);
}

// The rows of a tensor: where they begin, in bytes, and how they lie.
struct Rows {
  uintptr_t base;
  int64_t stride[3], extent[3];   // over sequences, heads, tokens
};

// Dimensions of more than one step, by falling stride; how many.
int by_stride(const Rows& r, int order[3]) {
  int n = 0;
  for (int i = 0; i < 3; ++i)
    if (r.extent[i] > 1) {
      int j = n++;
      for (; j > 0 && r.stride[order[j - 1]] < r.stride[i]; --j) order[j] = order[j - 1];
      order[j] = i;
    }
  return n;
}

// Elements from the first to the last of all rows; 0 where rows may overlap, that is where a dimension does not step over
// all that the smaller ones span.
int64_t span_of(const Rows& r, int64_t d) {
  int order[3];
  int64_t span = d;
  for (int n = by_stride(r, order); n-- > 0;) {
    const int i = order[n];
    if (r.stride[i] < span) return 0;
    span += r.stride[i] * (r.extent[i] - 1);
  }
  return span;
}

// Whether `delta` elements, from an output's row to another tensor's, are the difference of two of their rows.
bool meets(int64_t delta, const Rows& out, const Rows& other, const int* order, int n, int64_t d) {
  if (n == 0) return delta > -d && delta < d;
  const int64_t s = out.stride[*order], q = delta >= 0 ? delta / s : -((s - 1 - delta) / s);
  for (int64_t k = q; k <= q + 1; ++k)   // what the smaller strides make up is less than this one
    if (k < out.extent[*order] && k > -other.extent[*order] && meets(delta - k * s, out, other, order + 1, n - 1, d)) return true;
  return false;
}

// Whether writing `out` leaves `other` alone.  Tensors of one layout may lie between each other's rows, as queries and keys
// of one projection do; of tensors with different strides, one within the range of the other is taken to overlap it.
bool apart(const Rows& out, const Rows& other, int64_t d, size_t es) {
  const int64_t own = span_of(out, d);
  int64_t theirs = d;
  for (int i = 0; i < 3; ++i) theirs += other.stride[i] * (other.extent[i] - 1);
  if (out.base + (uintptr_t)own * es <= other.base || other.base + (uintptr_t)theirs * es <= out.base) return true;
  Rows both = out;
  for (int i = 0; i < 3; ++i) {
    both.extent[i] = out.extent[i] > other.extent[i] ? out.extent[i] : other.extent[i];
    if (both.extent[i] > 1 && out.stride[i] != other.stride[i]) return false;
  }
  if (!span_of(both, d)) return false;
  const int64_t bytes = (int64_t)(other.base - out.base);
  if (bytes % (int64_t)es) return false;
  int order[3];
  const int n = by_stride(both, order);
  return !meets(bytes / (int64_t)es, out, other, order, n, d);
}

}  // namespace
}  // namespace rehyat

using namespace rehyat;

extern "C" {

int rehyat_rope_turns(const double* radians, int n, uint64_t* turns) {
  if (!radians || !turns) return REHYAT_E_NULL;
  if (n < 1) return REHYAT_E_SHAPE;
  for (int i = 0; i < n; ++i)
    if (!std::isfinite(radians[i])) return REHYAT_E_SHAPE;
  for (int i = 0; i < n; ++i) {
    long double t = (long double)radians[i] / 6.28318530717958647692528676655900577L;
    t -= std::floor(t);                       // in [0, 1]: 1 where a tiny negative one rounds up
    t = std::rint(std::ldexp(t, 64));
    turns[i] = t >= 18446744073709551616.0L ? 0 : (uint64_t)t;
  }
  return REHYAT_OK;
}

int rehyat_rope(const rehyat_rope_operand* operands, int n_operands, const rehyat_rope_plan* plan,
                const rehyat_rope_positions* positions, int B, int N, int type, int inverse, void* stream) {
  if (!operands || !plan || !positions || !plan->turns) return REHYAT_E_NULL;
  if (n_operands < 1 || n_operands > 2 || B < 1 || N < 1 || !valid_type(type)) return REHYAT_E_SHAPE;
  if (inverse != 0 && inverse != 1) return REHYAT_E_SHAPE;
  const int d = plan->d, rot = plan->rot, axes = plan->axes;
  if (d < 2 || d > 512 || d % 2 || rot < 2 || rot > d || rot % 2) return REHYAT_E_SHAPE;
  if (plan->layout != REHYAT_ROPE_INTERLEAVED && plan->layout != REHYAT_ROPE_HALF) return REHYAT_E_SHAPE;
  if (axes < 1 || axes > 3 || !std::isfinite(plan->scale)) return REHYAT_E_SHAPE;
  int64_t pairs = 0;
  for (int x = 0; x < axes; ++x) {
    if (plan->section[x] < 1) return REHYAT_E_SHAPE;
    pairs += plan->section[x];
  }
  if (pairs != rot / 2) return REHYAT_E_SHAPE;
  if (!aligned(plan->turns, 8)) return REHYAT_E_SHAPE;
  if ((int64_t)B * N >= ((int64_t)1 << 31) / d) return REHYAT_E_SHAPE;
  const size_t es = type_bytes(type);

  RopeArgs a{};
  if (positions->data) {
    if (positions->bits != 32 && positions->bits != 64) return REHYAT_E_SHAPE;
    if (!aligned(positions->data, positions->bits / 8)) return REHYAT_E_SHAPE;
    if (positions->stride_b < 0 || positions->stride_b > ((int64_t)1 << 46) / B || positions->stride_n < 0 ||
        positions->stride_n > ((int64_t)1 << 46) / N)
      return REHYAT_E_SHAPE;
    a.pos = positions->data;
    a.pos_bits = positions->bits;
    a.pos_b = positions->stride_b;
    a.pos_n = positions->stride_n;
    a.frame = a.cols = 1;
  } else {
    int64_t frame = 1;
    if (axes > 1) {
      if (positions->cols < 1 || (axes == 3 && positions->rows < 1)) return REHYAT_E_SHAPE;
      frame = (int64_t)positions->cols * (axes == 3 ? positions->rows : 1);
    }
    a.frame = frame < N ? (uint32_t)frame : (uint32_t)N;   // a larger frame holds every token as well
    a.cols = axes > 1 ? (uint32_t)positions->cols : 1;
    a.start = (uint64_t)positions->start;
  }
  Rows in[2], out[2];
  for (int i = 0; i < n_operands; ++i) {
    const rehyat_rope_operand& o = operands[i];
    if (!o.x || !o.out) return REHYAT_E_NULL;
    if (o.heads < 1 || o.heads > 65535) return REHYAT_E_SHAPE;
    if (!aligned(o.x, es) || !aligned(o.out, es)) return REHYAT_E_SHAPE;
    in[i] = {(uintptr_t)o.x, {o.x_stride_b, o.x_stride_h, o.x_stride_n}, {B, o.heads, N}};
    out[i] = {(uintptr_t)o.out, {o.out_stride_b, o.out_stride_h, o.out_stride_n}, {B, o.heads, N}};
    for (int k = 0; k < 3; ++k)
      for (int64_t v : {in[i].stride[k], out[i].stride[k]})
        if (v < 0 || v > ((int64_t)1 << 46) / in[i].extent[k]) return REHYAT_E_SHAPE;   // sums of products fit 64 bits
    if (!span_of(out[i], d)) return REHYAT_E_SHAPE;
    if (a.pos && !ranges_apart(o.out, span_of(out[i], d) * (int64_t)es, a.pos,
                               ((B - 1) * a.pos_b + (N - 1) * a.pos_n + axes) * (a.pos_bits / 8)))
      return REHYAT_E_SHAPE;
    a.op[i] = {o.x, o.out, o.x_stride_b, o.x_stride_h, o.x_stride_n, o.out_stride_b, o.out_stride_h, o.out_stride_n, o.heads};
  }
  for (int i = 0; i < n_operands; ++i)
    for (int j = 0; j < n_operands; ++j) {
      const bool in_place = i == j && in[i].base == out[i].base && [&] {
        for (int k = 0; k < 3; ++k)
          if (in[i].extent[k] > 1 && in[i].stride[k] != out[i].stride[k]) return false;
        return true;
      }();
      if (!in_place && !apart(out[i], in[j], d, es)) return REHYAT_E_SHAPE;
      if (i != j && !apart(out[i], out[j], d, es)) return REHYAT_E_SHAPE;
    }
  a.turns = plan->turns;
  a.rot = rot;
  a.axes = axes;
  a.sec1 = axes > 1 ? plan->section[0] : rot;
  a.sec2 = axes > 2 ? plan->section[0] + plan->section[1] : rot;
  a.scale = plan->scale;
  a.sign = inverse ? -1.f : 1.f;
  const bool half = plan->layout == REHYAT_ROPE_HALF, in_place = [&] {
    for (int i = 0; i < n_operands; ++i) {
      const RopeOperand& o = a.op[i];
      if (o.x != o.out || o.xb != o.ob || o.xh != o.oh || o.xn != o.on) return false;
    }
    return true;
  }();
  const int part = half ? rot / 2 : rot, rest = d - rot;
  const int v = half && part % 2 ? 1 : 2;   // (rot and d are even, and so is `rest`)
  a.d = d;
  a.copies_from = part / v;
  a.slots = a.copies_from + (in_place ? 0 : half ? (rest / v + 1) / 2 : rest / v);
  a.N = N;
  a.items = (uint32_t)B * N * a.slots;
  // Heads a thread walks over: many, since they share their angles, unless that leaves too few waves.
  const int64_t waves = (a.items + 63) / 64;
  auto groups_of = [&](int group) {
    int n = 0;
    for (int i = 0; i < n_operands; ++i) n += (a.op[i].heads + group - 1) / group;
    return n;
  };
  a.group = kMostHeads;
  while (a.group > 1 && waves * groups_of(a.group) < kWaves && groups_of(a.group / 2) <= 65535) a.group /= 2;
  while (groups_of(a.group) > 65535) a.group *= 2;
  a.groups0 = (a.op[0].heads + a.group - 1) / a.group;
  const int groups = groups_of(a.group);
  const dim3 grid((a.items + 255) / 256, groups);
  hipStream_t st = (hipStream_t)stream;
  switch (type) {
    case REHYAT_BF16: launch<Bf16>(a, plan->layout, v, grid, st); break;
    case REHYAT_FP16: launch<Fp16>(a, plan->layout, v, grid, st); break;
    default: launch<Fp32>(a, plan->layout, v, grid, st);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(e, "rotary position kernel launch");
  return REHYAT_OK;
}

}  // extern "C"
