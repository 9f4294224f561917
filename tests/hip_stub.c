/* The HIP calls that libtensile.so makes, without a GPU: what is launched is only written down.  Loaded in front of libtensile.so
 * by host_calls.py, so that the entry points' checks and the choice of a kernel can be tested on any machine. */
#include <stdint.h>
#include <string.h>

typedef struct { uint32_t x, y, z; } dim3;

enum { kMost = 4096 };
static struct { const void *host; const char *name; } functions[kMost];
static int n_functions;
static struct { const char *name; uint32_t grid, block; } launches[kMost];
static int n_launches;
static dim3 grid_, block_;
static size_t shared_;
static void *stream_;
static char modules[64];
static int n_modules;
static uintptr_t next_address = 0x700000000000;

void **__hipRegisterFatBinary(const void *data) { (void)data; return (void **)&modules[n_modules++ % 64]; }
void __hipUnregisterFatBinary(void **m) { (void)m; }
void __hipRegisterVar(void **m, void *var, char *host, char *device, int ext, size_t size, int constant, int global) {
    (void)m; (void)var; (void)host; (void)device; (void)ext; (void)size; (void)constant; (void)global;
}
void __hipRegisterFunction(void **m, const void *host, char *device, const char *name, unsigned limit, void *tid, void *bid, void *bdim, void *gdim, int *wsize) {
    (void)m; (void)device; (void)limit; (void)tid; (void)bid; (void)bdim; (void)gdim; (void)wsize;
    if (n_functions < kMost) {
        functions[n_functions].host = host;
        functions[n_functions++].name = name;
    }
}
int __hipPushCallConfiguration(dim3 grid, dim3 block, size_t shared, void *stream) {
    grid_ = grid; block_ = block; shared_ = shared; stream_ = stream;
    return 0;
}
int __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *shared, void **stream) {
    *grid = grid_; *block = block_; *shared = shared_; *stream = stream_;
    return 0;
}
int hipLaunchKernel(const void *host, dim3 grid, dim3 block, void **args, size_t shared, void *stream) {
    (void)args; (void)shared; (void)stream;
    for (int k = 0; k < n_functions; ++k)
        if (functions[k].host == host && n_launches < kMost) {
            launches[n_launches].name = functions[k].name;
            launches[n_launches].grid = grid.x;
            launches[n_launches++].block = block.x;
            break;
        }
    return 0;
}

int hipGetDevice(int *device) { *device = 0; return 0; }
int hipDeviceGetAttribute(int *value, int attribute, int device) { (void)attribute; (void)device; *value = 256; return 0; }   /* (asked for the CUs alone) */
int hipDeviceSynchronize(void) { return 0; }
int hipGetLastError(void) { return 0; }
const char *hipGetErrorString(int e) { (void)e; return "stub"; }
int hipMalloc(void **p, size_t n) {
    *p = (void *)next_address;
    next_address += (n + 4095) / 4096 * 4096;
    return 0;
}
int hipFree(void *p) { (void)p; return 0; }

/* what host_calls.py asks for */
void stub_forget(void) { n_launches = 0; }
int stub_launches(void) { return n_launches; }
const char *stub_name(int k) { return launches[k].name; }
unsigned stub_grid(int k) { return launches[k].grid; }
unsigned stub_block(int k) { return launches[k].block; }
