/* The part of the HIP runtime that libmixkv.so's host code launches kernels with, as a recorder: nothing runs, every launch is written down.  Loaded into a process of its own
 * (RTLD_GLOBAL) in front of libmixkv.so. */
#include <stddef.h>
#include <stdint.h>
#include <string.h>

typedef struct { uint32_t x, y, z; } dim;
typedef struct { uint32_t grid[3], block[3]; const char *name; } launch;

enum { MOST_KERNELS = 4096, MOST_LAUNCHES = 65536 };
static struct { const void *host; const char *name; } kernels[MOST_KERNELS];
static launch launches[MOST_LAUNCHES];
static int n_kernels, n_launches;
static struct { dim grid, block; size_t shared; void *stream; } next;

void recorder_clear(void) { n_launches = 0; }
int recorder_count(void) { return n_launches; }
const launch *recorder_launch(int i) { return i >= 0 && i < n_launches && i < MOST_LAUNCHES ? &launches[i] : NULL; }

void **__hipRegisterFatBinary(const void *data) { static void *handle; (void)data; return &handle; }
void __hipUnregisterFatBinary(void **handle) { (void)handle; }
void __hipRegisterVar(void **modules, void *var, char *host, const char *device, int ext, size_t size, int constant, int global) {
  (void)modules; (void)var; (void)host; (void)device; (void)ext; (void)size; (void)constant; (void)global;
}
void __hipRegisterFunction(void **modules, const void *host, char *device, const char *name, unsigned limit, void *tid, void *bid, dim *block, dim *grid, int *warp) {
  (void)modules; (void)device; (void)limit; (void)tid; (void)bid; (void)block; (void)grid; (void)warp;
  if (n_kernels == MOST_KERNELS) return;
  kernels[n_kernels].host = host;
  kernels[n_kernels++].name = name;
}
int __hipPushCallConfiguration(dim grid, dim block, size_t shared, void *stream) {
  next.grid = grid; next.block = block; next.shared = shared; next.stream = stream;
  return 0;
}
int __hipPopCallConfiguration(dim *grid, dim *block, size_t *shared, void **stream) {
  *grid = next.grid; *block = next.block; *shared = next.shared; *stream = next.stream;
  return 0;
}
int hipLaunchKernel(const void *host, dim grid, dim block, void **args, size_t shared, void *stream) {
  launch l = {{0, 0, 0}, {0, 0, 0}, "?"};
  int i;
  (void)args; (void)shared; (void)stream;
  l.grid[0] = grid.x; l.grid[1] = grid.y; l.grid[2] = grid.z;
  l.block[0] = block.x; l.block[1] = block.y; l.block[2] = block.z;
  for (i = 0; i < n_kernels; ++i)
    if (kernels[i].host == host) l.name = kernels[i].name;
  if (n_launches < MOST_LAUNCHES) launches[n_launches] = l;
  ++n_launches;
  return 0;
}
int hipGetLastError(void) { return 0; }
