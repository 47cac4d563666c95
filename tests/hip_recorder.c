/* Stands in for the HIP calls of a kernel launch, so that what the library's
 * host side asks for can be looked at without a GPU: nothing is launched. */
#include <stddef.h>
#include <stdint.h>

typedef struct {
  uint32_t x, y, z;
} dim3;
typedef struct {
  const void* func; /* the kernel's handle */
  int64_t limit;    /* of dynamic shared memory: set to this (>= 0), or -1: a launch */
  int64_t shared;   /* the launch's dynamic shared memory */
  int64_t blocks, threads;
} record;

record records[4096];
int n_records = 0;

static dim3 grid, block;
static size_t shared_bytes;
static void* stream_of;

static void add(const void* f, int64_t limit, int64_t shared, int64_t blocks, int64_t threads) {
  if (n_records < 4096) {
    record r = {f, limit, shared, blocks, threads};
    records[n_records++] = r;
  }
}

int hipFuncSetAttribute(const void* func, int attribute, int value) {
  (void)attribute;
  add(func, value, 0, 0, 0);
  return 0;
}
int __hipPushCallConfiguration(dim3 g, dim3 b, size_t shared, void* stream) {
  grid = g, block = b, shared_bytes = shared, stream_of = stream;
  return 0;
}
int __hipPopCallConfiguration(dim3* g, dim3* b, size_t* shared, void** stream) {
  *g = grid, *b = block, *shared = shared_bytes, *stream = stream_of;
  return 0;
}
int hipLaunchKernel(const void* func, dim3 g, dim3 b, void** args, size_t shared, void* stream) {
  (void)args, (void)stream;
  add(func, -1, (int64_t)shared, (int64_t)g.x * g.y * g.z, (int64_t)b.x * b.y * b.z);
  return 0;
}
int hipGetDevice(int* d) {
  *d = 0;
  return 0;
}
int hipDeviceGetAttribute(int* v, int attribute, int device) {
  (void)attribute, (void)device;
  *v = 256;
  return 0;
}
int hipOccupancyMaxActiveBlocksPerMultiprocessor(int* n, const void* func, int threads, size_t shared) {
  (void)func, (void)threads, (void)shared;
  *n = 2;
  return 0;
}
int hipGetLastError(void) { return 0; }
