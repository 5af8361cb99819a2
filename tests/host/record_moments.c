/* What rehyat_adamw_moments launches, without a GPU: record_moments LIB - ELEMENTS.  Output as of record_operators.c, whose
 * runtime entry points these are. */
#define main record_operators
#include "record_operators.c"
#undef main

int main(int argc, char** argv) {
  if (argc != 4) return 2;
  void* const lib = dlopen(argv[1], RTLD_NOW);
  if (!lib) return 2;
  int (*const moments)(const void*, const void*, const void*, const void*, float*, float*, int64_t, void*) =
      dlsym(lib, "rehyat_adamw_moments");
  char* const at = (char*)0x10000000000;
  const long long n = strtoll(argv[3], NULL, 0), room = 4 * n + 4096;
  const int rc = moments(at, at + room, at + 2 * room, at + 3 * room, (float*)(at + (4 * room & ~255LL)),
                         (float*)(at + (6 * room & ~255LL)), n, NULL);
  printf("status %d\n", rc);
  return 0;
}
