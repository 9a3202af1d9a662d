/* The part of the HIP runtime that libpodrollout.so calls to launch kernels, without a device: launches are printed with their
 * kernel, grid, workgroup and dynamic LDS instead, and refused as the runtime refuses them.  256 compute units (what the library
 * assumes where it cannot ask). */
#include <stddef.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

typedef struct { uint32_t x, y, z; } dim3_t;
enum { kOk = 0, kInvalidValue = 1, kInvalidConfiguration = 9, kNotSupported = 801 };

static struct { const void *host; char name[512]; } kernels[4096];
static int n_kernels, last_error;
static struct { dim3_t grid, block; size_t lds; void *stream; } pushed;

void **__hipRegisterFatBinary(const void *data) { static void *module; (void)data; return &module; }
void __hipUnregisterFatBinary(void **module) { (void)module; }
void __hipRegisterVar(void **m, void *v, char *h, char *d, int e, size_t s, int c, int g) {
  (void)m, (void)v, (void)h, (void)d, (void)e, (void)s, (void)c, (void)g;
}
void __hipRegisterFunction(void **m, const void *host, char *fn, const char *name, unsigned t, void *a, void *b, void *c, void *d, int *w) {
  (void)m, (void)fn, (void)t, (void)a, (void)b, (void)c, (void)d, (void)w;
  if (n_kernels == 4096) abort();
  kernels[n_kernels].host = host;
  snprintf(kernels[n_kernels++].name, sizeof kernels[0].name, "%s", name);
  if (getenv("RECORDER_LISTS_KERNELS")) printf("kernel %s\n", name);
}
int __hipPushCallConfiguration(dim3_t grid, dim3_t block, size_t lds, void *stream) {
  pushed.grid = grid, pushed.block = block, pushed.lds = lds, pushed.stream = stream;
  return kOk;
}
int __hipPopCallConfiguration(dim3_t *grid, dim3_t *block, size_t *lds, void **stream) {
  *grid = pushed.grid, *block = pushed.block, *lds = pushed.lds, *stream = pushed.stream;
  return kOk;
}
int hipLaunchKernel(const void *f, dim3_t g, dim3_t b, void **args, size_t lds, void *stream) {
  const char *name = "?";
  (void)args, (void)stream;
  for (int i = 0; i < n_kernels; ++i)
    if (kernels[i].host == f) name = kernels[i].name;
  const int fits = g.x && g.y && g.z && b.x && b.y && b.z && (uint64_t)g.x * b.x <= UINT32_MAX && (uint64_t)g.y * b.y <= UINT32_MAX &&
                   (uint64_t)g.z * b.z <= UINT32_MAX && g.y <= 65535 && g.z <= 65535 && (uint64_t)b.x * b.y * b.z <= 1024 && lds <= 163840;
  printf("launch %s %u %u %u %u %u %u %zu\n", name, g.x, g.y, g.z, b.x, b.y, b.z, lds);
  return fits ? kOk : (last_error = kInvalidConfiguration);
}
int hipGetLastError(void) { const int e = last_error; last_error = kOk; return e; }
int hipGetDevice(int *device) { *device = 0; return kOk; }
int hipGetDevicePropertiesR0600(void *p, int device) { (void)p, (void)device; return kNotSupported; }
/* An error that is returned and nowhere else to be found. */
int hipFuncSetAttribute(const void *f, int attribute, int value) {
  (void)f, (void)attribute, (void)value;
  return getenv("RECORDER_REFUSES_ATTRIBUTES") ? kInvalidValue : kOk;
}
int hipGetSymbolAddress(void **p, const void *symbol) { (void)p, (void)symbol; return kNotSupported; }
int hipMemcpyAsync(void *d, const void *s, size_t n, int kind, void *st) { (void)d, (void)s, (void)n, (void)kind, (void)st; return kNotSupported; }
int hipMemsetAsync(void *d, int v, size_t n, void *st) { (void)d, (void)v, (void)n, (void)st; return kNotSupported; }
int hipStreamIsCapturing(void *st, int *status) { (void)st; *status = 0; return kOk; }
int hipStreamSynchronize(void *st) { (void)st; return kOk; }
