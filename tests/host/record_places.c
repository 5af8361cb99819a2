/* What calls launch without a GPU, by size and by where their arguments are; output as of record_operators.c, whose runtime
 * entry points these are.  Pointers are fake and never dereferenced.
 *   record_places LIB moments ELEMENTS
 *   record_places LIB positions BITS AXES B N STRIDE_B STRIDE_N DATA OUT SECOND_OUT    (3 heads of 64, head-major)
 *   record_places LIB loss TYPE B H N D Y_HAT Y WEIGHT GRAD LOSS WORKSPACE */
#define main record_operators
#include "record_operators.c"
#undef main

int main(int argc, char** argv) {
  if (argc < 4) return 2;
  void* const lib = dlopen(argv[1], RTLD_NOW);
  if (!lib) return 2;
  int rc = -100;
  arg = argv + 3;
  if (!strcmp(argv[2], "moments")) {
    int (*const moments)(const void*, const void*, const void*, const void*, float*, float*, int64_t, void*) =
        dlsym(lib, "rehyat_adamw_moments");
    char* const at = (char*)0x10000000000;
    const long long n = next(), room = (4 * n + 4095) / 256 * 256;
    rc = moments(at, at + room, at + 2 * room, at + 3 * room, (float*)(at + 4 * room), (float*)(at + 5 * room), n, NULL);
  } else if (!strcmp(argv[2], "positions")) {
    int (*const rope)(const rehyat_rope_operand*, int, const rehyat_rope_plan*, const rehyat_rope_positions*, int, int, int,
                      int, void*) = dlsym(lib, "rehyat_rope");
    const int bits = (int)next(), axes = (int)next(), B = (int)next(), N = (int)next(), d = 64;
    rehyat_rope_plan plan = {(const uint64_t*)0x1000, d, d, REHYAT_ROPE_HALF, axes, {axes == 1 ? 32 : 12, axes == 2 ? 20 : 10, 10}, 1.f};
    rehyat_rope_positions pos = {0};
    pos.bits = bits, pos.stride_b = next(), pos.stride_n = next(), pos.data = (const void*)next();
    rehyat_rope_operand op[2];
    for (int i = 0; i < 2; ++i)
      op[i] = (rehyat_rope_operand){(const void*)(0x100000000000 + i * 0x10000000000), (void*)next(), 3LL * N * d, (int64_t)N * d, d,
                                    3LL * N * d, (int64_t)N * d, d, 3};
    rc = rope(op, op[1].out ? 2 : 1, &plan, &pos, B, N, REHYAT_BF16, 0, NULL);
  } else if (!strcmp(argv[2], "loss")) {
    size_t (*const bytes)(int, int, int, int) = dlsym(lib, "rehyat_distill_loss_workspace_bytes");
    int (*const loss)(const void*, const void*, int, const float*, float, void*, float*, int, int, int, int, void*, size_t,
                      void*) = dlsym(lib, "rehyat_distill_loss");
    const int type = (int)next(), B = (int)next(), H = (int)next(), N = (int)next(), d = (int)next();
    void* p[6];
    for (int i = 0; i < 6; ++i) p[i] = (void*)next();
    rc = loss(p[0], p[1], type, p[2], 1.f, p[3], p[4], B, H, N, d, p[5], bytes(B, H, N, d), NULL);
  }
  printf("status %d\n", rc);
  return 0;
}
