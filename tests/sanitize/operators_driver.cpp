// Runs the host layers of the operators around the attention (rotary positions, distillation loss, AdamW) under
// AddressSanitizer / UndefinedBehaviorSanitizer.  No call below reaches the GPU: every one is rejected, or answered, before
// the first HIP call.  Pointers are fake, aligned, non-null values that are never dereferenced.
#include <climits>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <vector>

#include "../../include/rehyat.h"

#define CHECK(c) do { if (!(c)) { printf("FAILED line %d: %s\n", __LINE__, #c); return 1; } } while (0)

int main() {
  void* const A = (void*)0x1000;

  // frequencies, into an exactly sized array (ASan guards its ends)
  for (int n : {1, 2, 63, 64, 256}) {
    std::vector<double> f((size_t)n);
    for (int i = 0; i < n; ++i) f[(size_t)i] = (i % 2 ? -1.0 : 1.0) * std::pow(10.0, 40.0 - 80.0 * i / n);
    std::vector<uint64_t> t((size_t)n);
    CHECK(rehyat_rope_turns(f.data(), n, t.data()) == REHYAT_OK);
    f[(size_t)n - 1] = INFINITY;
    CHECK(rehyat_rope_turns(f.data(), n, t.data()) == REHYAT_E_SHAPE);
  }

  // rotary positions: extreme sizes and strides, all refused
  rehyat_rope_plan plan = {(const uint64_t*)A, 64, 64, REHYAT_ROPE_HALF, 1, {32, 0, 0}, 1.f};
  rehyat_rope_positions pos = {};
  for (int64_t s : {(int64_t)-1, (int64_t)63, INT64_MAX, INT64_MIN, (int64_t)1 << 45})
    for (int which = 0; which < 3; ++which) {
      rehyat_rope_operand op = {A, (void*)0x100000000, 1536, 512, 64, 1536, 512, 64, 3};
      (which == 0 ? op.out_stride_b : which == 1 ? op.out_stride_h : op.out_stride_n) = s;
      if (which == 0 && s == (int64_t)1 << 45) op.heads = 0;
      CHECK(rehyat_rope(&op, 1, &plan, &pos, 2, 8, REHYAT_BF16, 0, nullptr) == REHYAT_E_SHAPE);
    }
  {
    const rehyat_rope_operand op = {A, (void*)((uintptr_t)A + 128), 1536, 512, 64, 1536, 512, 64, 3};
    for (int B : {0, -1, INT_MAX, INT_MIN})
      for (int N : {0, -1, INT_MAX, INT_MIN})
        CHECK(rehyat_rope(&op, 1, &plan, &pos, B, N, REHYAT_BF16, 0, nullptr) == REHYAT_E_SHAPE);
    CHECK(rehyat_rope(&op, 1, &plan, &pos, 2, 8, REHYAT_BF16, 0, nullptr) == REHYAT_E_SHAPE);
    CHECK(rehyat_rope(&op, INT_MAX, &plan, &pos, 2, 8, REHYAT_BF16, 0, nullptr) == REHYAT_E_SHAPE);
    CHECK(rehyat_rope(nullptr, 1, &plan, &pos, 2, 8, REHYAT_BF16, 0, nullptr) == REHYAT_E_NULL);
    rehyat_rope_plan bad = plan;
    bad.axes = 3;
    bad.section[0] = INT_MAX, bad.section[1] = INT_MAX, bad.section[2] = INT_MAX;
    CHECK(rehyat_rope(&op, 1, &bad, &pos, 2, 8, REHYAT_BF16, 0, nullptr) == REHYAT_E_SHAPE);
    bad = plan;
    bad.axes = 3;
    bad.section[0] = 12, bad.section[1] = 10, bad.section[2] = 10;
    pos.rows = INT_MAX, pos.cols = INT_MAX, pos.start = INT64_MIN;      // a frame of any size; refused for the overlap
    CHECK(rehyat_rope(&op, 1, &bad, &pos, 2, 8, REHYAT_BF16, 0, nullptr) == REHYAT_E_SHAPE);
    pos.data = A, pos.bits = 64, pos.stride_b = INT64_MAX;
    CHECK(rehyat_rope(&op, 1, &plan, &pos, 2, 8, REHYAT_BF16, 0, nullptr) == REHYAT_E_SHAPE);
  }

  // loss: workspace arithmetic over a sweep of shapes, then rejections
  for (int B : {1, 3, 255, 65535})
    for (int H : {1, 12, 257})
      for (int N : {1, 32760, 16777215})
        for (int d : {1, 17, 64, 128}) {
          const bool ok = (int64_t)B * H <= 65535 && N < ((int64_t)1 << 31) / d;
          const size_t need = rehyat_distill_loss_workspace_bytes(B, H, N, d);
          CHECK(ok ? need > 0 && need % 256 == 0 && need <= (size_t)1 << 20 : need == 0);
          CHECK(rehyat_distill_loss(A, A, REHYAT_FP32, nullptr, 1.f, A, (float*)A, B, H, N, d, A, need, nullptr) == REHYAT_E_SHAPE);
        }
  CHECK(rehyat_distill_loss_workspace_bytes(INT_MAX, INT_MAX, INT_MAX, INT_MAX) == 0);
  CHECK(rehyat_distill_loss_workspace_bytes(1, 1, INT_MIN, 64) == 0);

  // AdamW: tables, tensors read from an exactly sized array, overlaps among many ranges
  for (int n : {1, 2, 41, 500}) {
    std::vector<int64_t> sizes((size_t)n, 100000);
    const size_t need = rehyat_adamw_table_bytes(sizes.data(), n);
    CHECK(need > 0 && need % 256 == 0);
    std::vector<rehyat_adamw_tensor> t((size_t)n);
    for (int i = 0; i < n; ++i) {
      char* const at = (char*)0x100000000 + (int64_t)i * 0x1000000;
      t[(size_t)i] = {at, (float*)(at + 0x100000), at + 0x200000, at + 0x300000, at + 0x400000, at + 0x500000, at + 0x600000,
                      100000, REHYAT_BF16, REHYAT_FP32};
    }
    rehyat_adamw_plan p;
    CHECK(rehyat_adamw_prepare(t.data(), n, 8, 0, A, need - 1, &p, nullptr) == REHYAT_E_WORKSPACE);
    t[(size_t)n - 1].v = t[0].m;
    CHECK(rehyat_adamw_prepare(t.data(), n, 8, 0, A, need, &p, nullptr) == REHYAT_E_SHAPE);
    t[(size_t)n - 1].n = INT64_MAX;
    CHECK(rehyat_adamw_prepare(t.data(), n, 32, 0, A, need, &p, nullptr) == REHYAT_E_SHAPE);
    t[(size_t)n - 1].n = INT64_MIN;
    CHECK(rehyat_adamw_prepare(t.data(), n, 32, INT64_MIN, A, need, &p, nullptr) == REHYAT_E_SHAPE);
    sizes[(size_t)n - 1] = INT64_MAX;
    CHECK(rehyat_adamw_table_bytes(sizes.data(), n) == 0);
  }
  CHECK(rehyat_adamw_moments(A, A, A, A, (float*)A, (float*)A, INT64_MAX, nullptr) == REHYAT_E_SHAPE);
  CHECK(rehyat_adamw_moments(A, A, A, A, (float*)A, (float*)A, 64, nullptr) == REHYAT_E_SHAPE);
  {
    const rehyat_adamw_plan p = {A, INT64_MAX, INT_MAX, 16};
    const rehyat_adamw_hyper h = {NAN, NAN, NAN, NAN, NAN, nullptr};
    CHECK(rehyat_adamw_step(&p, &h, nullptr) == REHYAT_E_SHAPE);
  }
  printf("operators sanitize ok\n");
  return 0;
}
