/* Stands in for the HIP runtime under libbsa.so (tests/launch_checks.py): launches are reported, nothing runs and no
 * device is needed. */
#include <stddef.h>
#include <stdlib.h>

typedef struct { unsigned x, y, z; } dim3;
typedef void (*report_t)(const char* kernel, const unsigned* grid, const unsigned* block, void** args);

static struct { const void* host; const char* name; } kernels[4096];
static int n_kernels;
static dim3 grid_, block_;
static size_t shared_;
static void* stream_;
static report_t report;

void launch_stub_report(report_t f) { report = f; }

void** __hipRegisterFatBinary(const void* data) { (void)data; return (void**)&kernels; }
void __hipUnregisterFatBinary(void** m) { (void)m; }
void __hipRegisterVar(void** m, void* var, char* host, char* device, int ext, size_t size, int constant, int global) {
  (void)m, (void)var, (void)host, (void)device, (void)ext, (void)size, (void)constant, (void)global;
}
void __hipRegisterFunction(void** m, const void* host, char* device, const char* name, unsigned limit, void* tid, void* bid,
                           dim3* bdim, dim3* gdim, int* wsize) {
  (void)m, (void)device, (void)limit, (void)tid, (void)bid, (void)bdim, (void)gdim, (void)wsize;
  if (n_kernels == 4096) abort();
  kernels[n_kernels].host = host;
  kernels[n_kernels++].name = name;
}
int __hipPushCallConfiguration(dim3 grid, dim3 block, size_t shared, void* stream) {
  grid_ = grid, block_ = block, shared_ = shared, stream_ = stream;
  return 0;
}
int __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* shared, void** stream) {
  *grid = grid_, *block = block_, *shared = shared_, *stream = stream_;
  return 0;
}
int hipLaunchKernel(const void* host, dim3 grid, dim3 block, void** args, size_t shared, void* stream) {
  (void)shared, (void)stream;
  const char* name = "";
  for (int i = 0; i < n_kernels; ++i)
    if (kernels[i].host == host) name = kernels[i].name;
  if (report) report(name, &grid.x, &block.x, args);
  return 0;
}
int hipGetLastError(void) { return 0; }
