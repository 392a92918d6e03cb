/* A CUDA runtime that does nothing, for the library's host code without a GPU: preloaded, it stands in for the functions that
 * libgambit.so takes from libcudart.  Launches and copies succeed, but for the one that fake_fail_at names, which fails as in
 * the runtime: its error is returned, and kept for cudaGetLastError. */
#include <cuda_runtime_api.h>

static int fail_at = -1, calls = 0, regs = 255;
static cudaError_t last = cudaSuccess;

void fake_fail_at(int n) { fail_at = n, calls = 0; }
int fake_calls(void) { return calls; }
void fake_regs(int n) { regs = n; }

static cudaError_t work(void) { return calls++ == fail_at ? (last = cudaErrorInvalidValue) : cudaSuccess; }

void** __cudaRegisterFatBinary(void* x) { static void* h; return (void)x, &h; }
void __cudaRegisterFatBinaryEnd(void** x) { (void)x; }
void __cudaUnregisterFatBinary(void** x) { (void)x; }
void __cudaRegisterFunction(void** a, const char* b, char* c, const char* d, int e, void* f, void* g, void* h, void* i, int* j) {
  (void)a, (void)b, (void)c, (void)d, (void)e, (void)f, (void)g, (void)h, (void)i, (void)j;
}
void __cudaRegisterVar(void** a, char* b, char* c, const char* d, int e, size_t f, int g, int h) {
  (void)a, (void)b, (void)c, (void)d, (void)e, (void)f, (void)g, (void)h;
}
cudaError_t __cudaGetKernel(cudaKernel_t* k, const void* f) { return *k = (cudaKernel_t)f, cudaSuccess; }
cudaError_t __cudaLaunchKernel(cudaKernel_t k, dim3 g, dim3 b, void** a, size_t m, cudaStream_t s) {
  return (void)k, (void)g, (void)b, (void)a, (void)m, (void)s, work();
}
unsigned __cudaPushCallConfiguration(dim3 g, dim3 b, size_t m, struct CUstream_st* s) { return (void)g, (void)b, (void)m, (void)s, 0; }
cudaError_t __cudaPopCallConfiguration(dim3* g, dim3* b, size_t* m, void* s) {
  *g = *b = (dim3){1, 1, 1};
  *m = 0;
  *(cudaStream_t*)s = 0;
  return cudaSuccess;
}
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t* c, const void* f, void** a) { return (void)c, (void)f, (void)a, work(); }
cudaError_t cudaMemsetAsync(void* p, int x, size_t n, cudaStream_t s) { return (void)p, (void)x, (void)n, (void)s, work(); }
cudaError_t cudaMemcpyAsync(void* d, const void* p, size_t n, enum cudaMemcpyKind k, cudaStream_t s) {
  return (void)d, (void)p, (void)n, (void)k, (void)s, work();
}
cudaError_t cudaDeviceGetAttribute(int* x, enum cudaDeviceAttr a, int d) { return (void)a, (void)d, *x = 152, cudaSuccess; }
cudaError_t cudaGetDevice(int* d) { return *d = 0, cudaSuccess; }
cudaError_t cudaFuncGetAttributes(struct cudaFuncAttributes* a, const void* f) {
  static const struct cudaFuncAttributes none;
  (void)f;
  *a = none;
  a->numRegs = regs;
  return cudaSuccess;
}
cudaError_t cudaFuncSetAttribute(const void* f, enum cudaFuncAttribute a, int x) { return (void)f, (void)a, (void)x, cudaSuccess; }
cudaError_t cudaEventRecordWithFlags(cudaEvent_t e, cudaStream_t s, unsigned f) { return (void)e, (void)s, (void)f, cudaSuccess; }
const char* cudaGetErrorString(cudaError_t e) { return (void)e, "an error of the fake"; }
cudaError_t cudaGetLastError(void) {
  const cudaError_t e = last;
  last = cudaSuccess;
  return e;
}
cudaError_t cudaGetSymbolAddress(void** p, const void* s) { return (void)s, *p = 0, cudaErrorInvalidSymbol; }
static int encode(void) { return 0; }
cudaError_t cudaGetDriverEntryPointByVersion(const char* n, void** f, unsigned v, unsigned long long x, enum cudaDriverEntryPointQueryResult* q) {
  return (void)n, (void)v, (void)x, *f = (void*)encode, *q = cudaDriverEntryPointSuccess, cudaSuccess;
}
cudaError_t cudaStreamGetCaptureInfo(cudaStream_t s, enum cudaStreamCaptureStatus* c, unsigned long long* id, cudaGraph_t* g,
                                     const cudaGraphNode_t** d, const cudaGraphEdgeData** e, size_t* n) {
  (void)s, (void)id, (void)g, (void)d, (void)e, (void)n;
  *c = cudaStreamCaptureStatusNone;
  return cudaSuccess;
}
cudaError_t cudaStreamIsCapturing(cudaStream_t s, enum cudaStreamCaptureStatus* c) { return (void)s, *c = cudaStreamCaptureStatusNone, cudaSuccess; }
cudaError_t cudaStreamSynchronize(cudaStream_t s) { return (void)s, cudaSuccess; }
