/* A CUDA runtime of recorded calls, for tests of the library's host side without a GPU: linked with the library's objects in place of
 * the real one. Several devices of compute capability 10.0; nothing runs, nothing is allocated. Test doubles only. */
#include <cuda_runtime_api.h>
#include <stdio.h>
#include <string.h>

#define N_DEV 4
#define N_FUNC 1024
static int g_device, g_sms[N_DEV] = {148, 148, 148, 148}, g_fit[N_DEV] = {148, 148, 148, 148};
static struct { const void* fn; char name[160]; int smem[N_DEV]; } g_func[N_FUNC];
static int g_n_func, g_n_launch;
static struct { char name[160]; unsigned grid, block, cluster; size_t smem; int device, allowed; } g_launch[64];

static int find(const void* fn) {
  for (int i = 0; i < g_n_func; ++i)
    if (g_func[i].fn == fn) return i;
  return -1;
}
void fake_set_device(int d) { g_device = d; }
void fake_set_fit(int d, int ctas) { g_fit[d] = ctas; } /* CTAs of clusters that device d holds at once */
int fake_launches(void) { return g_n_launch; }
void fake_clear_launches(void) { g_n_launch = 0; }
/* launch i: kernel name into `name`; grid, block, cluster, dynamic shared memory, what the kernel may take of it, device */
int fake_launch(int i, char* name, int n, long long* out) {
  if (i < 0 || i >= g_n_launch || i >= 64) return -1;
  snprintf(name, (size_t)n, "%s", g_launch[i].name);
  out[0] = g_launch[i].grid, out[1] = g_launch[i].block, out[2] = g_launch[i].cluster;
  out[3] = (long long)g_launch[i].smem, out[4] = g_launch[i].allowed, out[5] = g_launch[i].device;
  return 0;
}
/* kernels whose name holds `part` and that device d has been told about */
int fake_prepared(int d, const char* part) {
  int n = 0;
  for (int i = 0; i < g_n_func; ++i) n += strstr(g_func[i].name, part) != NULL && g_func[i].smem[d] != 0;
  return n;
}

void** __cudaRegisterFatBinary(void* p) { static void* h[1]; (void)p; return h; }
void __cudaRegisterFatBinaryEnd(void** h) { (void)h; }
void __cudaUnregisterFatBinary(void** h) { (void)h; }
void __cudaRegisterFunction(void** h, const char* fn, char* dev, const char* name, int lim, void* a, void* b, void* c, void* d, int* w) {
  (void)h, (void)dev, (void)lim, (void)a, (void)b, (void)c, (void)d, (void)w;
  if (g_n_func < N_FUNC) {
    g_func[g_n_func].fn = fn;
    snprintf(g_func[g_n_func++].name, sizeof g_func[0].name, "%s", name);
  }
}
void __cudaRegisterVar(void** h, char* v, char* a, const char* n, int e, size_t s, int c, int g) { (void)h, (void)v, (void)a, (void)n, (void)e, (void)s, (void)c, (void)g; }
unsigned __cudaPushCallConfiguration(dim3 g, dim3 b, size_t s, void* st) { (void)g, (void)b, (void)s, (void)st; return 0; }
cudaError_t __cudaPopCallConfiguration(dim3* g, dim3* b, size_t* s, void* st) { (void)g, (void)b, (void)s, (void)st; return cudaSuccess; }

cudaError_t cudaGetDevice(int* d) { *d = g_device; return cudaSuccess; }
cudaError_t cudaSetDevice(int d) { g_device = d; return cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int* v, enum cudaDeviceAttr a, int d) {
  *v = a == cudaDevAttrComputeCapabilityMajor ? 10 : a == cudaDevAttrMultiProcessorCount ? g_sms[d] : 0;
  return cudaSuccess;
}
cudaError_t cudaFuncSetAttribute(const void* fn, enum cudaFuncAttribute a, int v) {
  const int i = find(fn);
  if (i < 0) return cudaErrorInvalidDeviceFunction;
  if (a == cudaFuncAttributeMaxDynamicSharedMemorySize) g_func[i].smem[g_device] = v;
  return cudaSuccess;
}
static unsigned cluster_of(const cudaLaunchConfig_t* c) {
  for (unsigned i = 0; i < c->numAttrs; ++i)
    if (c->attrs[i].id == cudaLaunchAttributeClusterDimension) return c->attrs[i].val.clusterDim.x;
  return 1;
}
cudaError_t cudaOccupancyMaxActiveClusters(int* n, const void* fn, const cudaLaunchConfig_t* c) {
  if (find(fn) < 0) return cudaErrorInvalidDeviceFunction;
  *n = g_fit[g_device] / (int)cluster_of(c);
  return cudaSuccess;
}
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t* c, const void* fn, void** args) {
  const int i = find(fn);
  (void)args;
  if (i < 0) return cudaErrorInvalidDeviceFunction;
  if (g_n_launch < 64) {
    snprintf(g_launch[g_n_launch].name, sizeof g_launch[0].name, "%s", g_func[i].name);
    g_launch[g_n_launch].grid = c->gridDim.x, g_launch[g_n_launch].block = c->blockDim.x, g_launch[g_n_launch].cluster = cluster_of(c);
    g_launch[g_n_launch].smem = c->dynamicSmemBytes, g_launch[g_n_launch].device = g_device;
    g_launch[g_n_launch++].allowed = g_func[i].smem[g_device];
  }
  return cudaSuccess;
}
static int encode(void) { return 0; }
cudaError_t cudaGetDriverEntryPoint(const char* s, void** fn, unsigned long long f, enum cudaDriverEntryPointQueryResult* r) {
  (void)s, (void)f;
  *fn = (void*)encode;
  *r = cudaDriverEntryPointSuccess;
  return cudaSuccess;
}
const char* cudaGetErrorString(cudaError_t e) { return e == cudaSuccess ? "no error" : "an error of the fake runtime"; }
cudaError_t cudaGetLastError(void) { return cudaSuccess; }
/* everything else that the library links to: refused */
int fake_unused(void) { return cudaErrorNotSupported; }
