/* What rehyat_rope, rehyat_distill_loss and rehyat_adamw_* launch, without a GPU: as in record_launches.c the runtime entry
 * points that a launch passes through are defined here.
 *   record_operators LIB rope TYPE LAYOUT B N D ROT N_OPERANDS { X OUT HEADS XB XH XN OB OH ON } ...
 *   record_operators LIB loss TYPE WEIGHTED B H N D
 *   record_operators LIB adamw BITS N_TENSORS ELEMENTS
 * One line per launch (grid x y z, kernel), then "status S".  Pointers are fake and never dereferenced. */
#include <dlfcn.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "../../include/rehyat.h"

typedef struct { unsigned x, y, z; } dim3;

static struct { const void* host; const char* name; } kernels[256];
static int n_kernels;
static dim3 cfg_grid, cfg_block;
static size_t cfg_shared;

void** __hipRegisterFatBinary(const void* data) {
  static void* handle;
  (void)data;
  return &handle;
}
void __hipUnregisterFatBinary(void** modules) { (void)modules; }
void __hipRegisterFunction(void** modules, const void* host, char* device, const char* name, unsigned limit, void* tid,
                           void* bid, void* block, void* grid, int* wsize) {
  (void)modules, (void)device, (void)limit, (void)tid, (void)bid, (void)block, (void)grid, (void)wsize;
  if (n_kernels < 256) kernels[n_kernels].host = host, kernels[n_kernels++].name = name;
}
void __hipRegisterVar(void** modules, void* var, char* host, char* device, int ext, size_t size, int constant, int global) {
  (void)modules, (void)var, (void)host, (void)device, (void)ext, (void)size, (void)constant, (void)global;
}
int __hipPushCallConfiguration(dim3 grid, dim3 block, size_t shared, void* stream) {
  (void)stream;
  cfg_grid = grid, cfg_block = block, cfg_shared = shared;
  return 0;
}
int __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* shared, void** stream) {
  *grid = cfg_grid, *block = cfg_block, *shared = cfg_shared, *stream = NULL;
  return 0;
}
int hipLaunchKernel(const void* host, dim3 grid, dim3 block, void** args, size_t shared, void* stream) {
  const char* name = "?";
  (void)block, (void)args, (void)shared, (void)stream;
  for (int i = 0; i < n_kernels; ++i)
    if (kernels[i].host == host) name = kernels[i].name;
  printf("%u %u %u %s\n", grid.x, grid.y, grid.z, name);
  return 0;
}
int hipGetLastError(void) { return 0; }

static char** arg;
static long long next(void) { return *arg ? strtoll(*arg++, NULL, 0) : 0; }

int main(int argc, char** argv) {
  if (argc < 4) return 2;
  void* const lib = dlopen(argv[1], RTLD_NOW);
  if (!lib) {
    fprintf(stderr, "%s\n", dlerror());
    return 2;
  }
  void* const A = (void*)0x1000;
  int rc = -100;
  arg = argv + 3;
  if (!strcmp(argv[2], "rope")) {
    int (*const rope)(const rehyat_rope_operand*, int, const rehyat_rope_plan*, const rehyat_rope_positions*, int, int, int,
                      int, void*) = dlsym(lib, "rehyat_rope");
    const int type = (int)next(), layout = (int)next(), B = (int)next(), N = (int)next(), d = (int)next(), rot = (int)next(),
              n = (int)next();
    rehyat_rope_plan plan = {(const uint64_t*)A, d, rot, layout, 1, {rot / 2, 0, 0}, 1.f};
    rehyat_rope_positions pos = {0};
    rehyat_rope_operand op[2] = {{0}};
    for (int i = 0; i < n && i < 2; ++i) {
      op[i].x = (const void*)next(), op[i].out = (void*)next(), op[i].heads = (int)next();
      op[i].x_stride_b = next(), op[i].x_stride_h = next(), op[i].x_stride_n = next();
      op[i].out_stride_b = next(), op[i].out_stride_h = next(), op[i].out_stride_n = next();
    }
    rc = rope(op, n, &plan, &pos, B, N, type, 0, NULL);
  } else if (!strcmp(argv[2], "loss")) {
    size_t (*const bytes)(int, int, int, int) = dlsym(lib, "rehyat_distill_loss_workspace_bytes");
    int (*const loss)(const void*, const void*, int, const float*, float, void*, float*, int, int, int, int, void*, size_t,
                      void*) = dlsym(lib, "rehyat_distill_loss");
    const int type = (int)next(), weighted = (int)next(), B = (int)next(), H = (int)next(), N = (int)next(), d = (int)next();
    char* const far = (char*)0x10000000000;
    rc = loss(far, far + 0x10000000000, type, weighted ? (const float*)A : NULL, 1.f, far + 0x20000000000,
              (float*)A, B, H, N, d, A, bytes(B, H, N, d), NULL);
  } else {
    int (*const prepare)(const rehyat_adamw_tensor*, int, int, int64_t, void*, size_t, rehyat_adamw_plan*, void*) =
        dlsym(lib, "rehyat_adamw_prepare");
    int (*const step)(const rehyat_adamw_plan*, const rehyat_adamw_hyper*, void*) = dlsym(lib, "rehyat_adamw_step");
    const int bits = (int)next(), n = (int)next();
    const long long elements = next();
    rehyat_adamw_tensor* const t = calloc((size_t)n, sizeof(*t));
    char* at = (char*)0x10000000000;
    for (int i = 0; i < n; ++i) {
      void** const p[7] = {&t[i].param, (void**)&t[i].master, (void**)&t[i].grad, &t[i].m, &t[i].v, &t[i].m_exp, &t[i].v_exp};
      for (int k = 0; k < 7; ++k) *p[k] = at, at += (4 * elements + 511) / 256 * 256;
      t[i].n = elements, t[i].param_type = REHYAT_BF16, t[i].grad_type = REHYAT_FP32;
    }
    rehyat_adamw_plan plan = {0};
    const rehyat_adamw_hyper hyper = {1e-3, 0.9, 0.999, 1e-8, 0.01, NULL};
    rc = prepare(t, n, bits, 0, (void*)0x1000, (size_t)1 << 39, &plan, NULL);
    if (rc == 0) {
      printf("items %lld\n", (long long)plan.items);
      rc = step(&plan, &hyper, NULL);
    }
    free(t);
  }
  printf("status %d\n", rc);
  return 0;
}
