// fake_cudart.cpp -- a CUDA runtime of two imaginary GPUs for tests of the
// library's host code on a machine without one.  It is linked with the
// library's objects in the real runtime's place.  Nothing runs: launches are
// checked the way the runtime checks them (the dynamic shared memory that a
// kernel was allowed on the current device) and logged.
//
// fake_log() lists the calls since the last fake_reset(), a line each, with
// the device they were made on.
#include <cuda_runtime_api.h>
#include <dlfcn.h>

#include <cstdio>
#include <cstring>
#include <map>
#include <string>

namespace {

constexpr int kDevices = 2;
int g_device = 0;
cudaError_t g_last = cudaSuccess;
std::string g_log, g_fail;                    // g_fail: the call that fails once
std::map<const void *, std::string> g_names;  // host stub -> kernel
std::map<std::pair<int, const void *>, int> g_smem;   // allowed, by device and kernel
struct Pushed {
    dim3 grid, block;
    size_t smem;
    cudaStream_t stream;
} g_pushed;

void log(const char *what, const std::string &rest) {
    char head[64];
    snprintf(head, sizeof head, "%s dev=%d ", what, g_device);
    g_log += head + rest + "\n";
}
bool failing(const char *what) {
    if (g_fail != what) return false;
    g_fail.clear();
    return true;
}
cudaError_t done(cudaError_t e) {
    if (e != cudaSuccess) g_last = e;
    return e;
}
std::string hex(const void *p) {
    char s[32];
    snprintf(s, sizeof s, "%p", p);
    return s;
}
cudaError_t launch(const void *func, size_t smem) {
    log("launch", g_names[func] + " smem=" + std::to_string(smem));
    if (failing("launch")) return done(cudaErrorLaunchOutOfResources);
    const auto it = g_smem.find({g_device, func});
    const size_t allowed = it == g_smem.end() ? 49152 : (size_t)it->second;
    return done(smem > allowed ? cudaErrorInvalidValue : cudaSuccess);
}
int fake_encode() { return 0; }   // of a tensor map

}  // namespace

extern "C" {

void fake_reset(int device) {
    g_device = device;
    g_last = cudaSuccess;
    g_log.clear();
    g_fail.clear();
}
void fake_fail_once(const char *what) { g_fail = what; }
const char *fake_log() { return g_log.c_str(); }

// ---- devices and errors ----
cudaError_t cudaGetDevice(int *d) {
    *d = g_device;
    return cudaSuccess;
}
cudaError_t cudaDeviceGetAttribute(int *v, cudaDeviceAttr attr, int) {
    if (failing("cudaDeviceGetAttribute")) return done(cudaErrorInitializationError);
    // as many SMs as the device's number says, so that a count kept from the
    // other device shows
    *v = attr == cudaDevAttrMultiProcessorCount ? 100 + 10 * g_device : 0;
    return cudaSuccess;
}
cudaError_t cudaGetLastError() {
    const cudaError_t e = g_last;
    g_last = cudaSuccess;
    return e;
}
const char *cudaGetErrorName(cudaError_t) { return "fake"; }
const char *cudaGetErrorString(cudaError_t) { return "fake"; }

// ---- kernels ----
cudaError_t cudaFuncSetAttribute(const void *func, cudaFuncAttribute attr, int value) {
    if (failing("cudaFuncSetAttribute")) return done(cudaErrorMemoryAllocation);
    if (attr == cudaFuncAttributeMaxDynamicSharedMemorySize) g_smem[{g_device, func}] = value;
    return cudaSuccess;
}
cudaError_t cudaFuncGetAttributes(cudaFuncAttributes *a, const void *) {
    memset(a, 0, sizeof *a);
    return cudaSuccess;
}
cudaError_t cudaOccupancyMaxActiveBlocksPerMultiprocessorWithFlags(int *n, const void *, int,
                                                                   size_t, unsigned) {
    if (failing("cudaOccupancyMaxActiveBlocksPerMultiprocessor")) return done(cudaErrorUnknown);
    *n = 1;
    return cudaSuccess;
}
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t *c, const void *func, void **) {
    return launch(func, c->dynamicSmemBytes);
}
unsigned __cudaPushCallConfiguration(dim3 grid, dim3 block, size_t smem, cudaStream_t st) {
    g_pushed = {grid, block, smem, st};
    return 0;
}
cudaError_t __cudaPopCallConfiguration(dim3 *grid, dim3 *block, size_t *smem, void *st) {
    *grid = g_pushed.grid;
    *block = g_pushed.block;
    *smem = g_pushed.smem;
    *static_cast<cudaStream_t *>(st) = g_pushed.stream;
    return cudaSuccess;
}
cudaError_t __cudaGetKernel(cudaKernel_t *k, const void *func) {
    *k = (cudaKernel_t) const_cast<void *>(func);
    return cudaSuccess;
}
cudaError_t __cudaLaunchKernel(cudaKernel_t k, dim3, dim3, void **, size_t smem, cudaStream_t) {
    return launch((const void *)k, smem);
}
void **__cudaRegisterFatBinary(void *) {
    static void *handle;
    return &handle;
}
void __cudaRegisterFatBinaryEnd(void **) {}
void __cudaUnregisterFatBinary(void **) {}
void __cudaRegisterFunction(void **, const char *func, char *, const char *name, int, void *,
                            void *, void *, void *, int *) {
    g_names[func] = name;
}
void __cudaRegisterVar(void **, char *, char *, const char *, int, size_t, int, int) {}

// ---- memory: a symbol lies a gigabyte apart on each device ----
cudaError_t cudaGetSymbolAddress(void **p, const void *symbol) {
    if (failing("cudaGetSymbolAddress")) return done(cudaErrorInvalidSymbol);
    *p = (char *)symbol + ((size_t)g_device << 30);
    log("symbol", hex(*p));
    return cudaSuccess;
}
cudaError_t cudaMalloc(void **, size_t) { return done(cudaErrorMemoryAllocation); }
cudaError_t cudaFree(void *) { return cudaSuccess; }
cudaError_t cudaMemset(void *, int, size_t) { return cudaSuccess; }
cudaError_t cudaMemcpy(void *, const void *, size_t, cudaMemcpyKind) { return cudaSuccess; }
cudaError_t cudaMemsetAsync(void *p, int, size_t n, cudaStream_t) {
    log("memset", hex(p) + " bytes=" + std::to_string(n));
    return cudaSuccess;
}
cudaError_t cudaMemcpyAsync(void *, const void *src, size_t n, cudaMemcpyKind, cudaStream_t) {
    log("copy", hex(src) + " bytes=" + std::to_string(n));
    return cudaSuccess;
}
cudaError_t cudaPointerGetAttributes(cudaPointerAttributes *, const void *) {
    return done(cudaErrorInvalidValue);
}
cudaError_t cudaGetDriverEntryPointByVersion(const char *, void **fn, unsigned, unsigned long long,
                                             cudaDriverEntryPointQueryResult *q) {
    if (failing("cudaGetDriverEntryPointByVersion")) return done(cudaErrorInitializationError);
    *fn = (void *)&fake_encode;
    *q = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}

// ---- streams and graphs: not reached by the tests ----
cudaError_t cudaDeviceSynchronize() { return cudaSuccess; }
cudaError_t cudaStreamSynchronize(cudaStream_t) { return cudaSuccess; }
cudaError_t cudaStreamCreateWithFlags(cudaStream_t *, unsigned) { return done(cudaErrorUnknown); }
cudaError_t cudaStreamDestroy(cudaStream_t) { return cudaSuccess; }
cudaError_t cudaStreamBeginCapture(cudaStream_t, cudaStreamCaptureMode) {
    return done(cudaErrorUnknown);
}
cudaError_t cudaStreamEndCapture(cudaStream_t, cudaGraph_t *) { return done(cudaErrorUnknown); }
cudaError_t cudaGraphInstantiate(cudaGraphExec_t *, cudaGraph_t, unsigned long long) {
    return done(cudaErrorUnknown);
}
cudaError_t cudaGraphLaunch(cudaGraphExec_t, cudaStream_t) { return done(cudaErrorUnknown); }
cudaError_t cudaGraphExecDestroy(cudaGraphExec_t) { return cudaSuccess; }
cudaError_t cudaGraphDestroy(cudaGraph_t) { return cudaSuccess; }

}  // extern "C"
