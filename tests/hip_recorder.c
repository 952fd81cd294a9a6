/* A HIP runtime with two devices and no GPU: it keeps the calling thread's
 * current device, and notes every launch instead of running it.  Loaded before
 * libpccl.so so that the library's host code can be tested without a GPU. */
#include <stdint.h>
#include <stdlib.h>
#include <string.h>

typedef struct { uint32_t x, y, z; } dim3_t;
typedef struct { uint32_t grid[3], block[3]; int32_t device, pad; uint64_t arg[6]; } launch_t;

launch_t launches[4096];
int n_launches, current_device, launch_error, n_set_device;

int hipGetDeviceCount(int *n) { *n = 2; return 0; }
int hipGetDevice(int *d) { *d = current_device; return 0; }
int hipSetDevice(int d) { current_device = d; n_set_device++; return 0; }
int hipGetLastError(void) { int e = launch_error; launch_error = 0; return e; }
int hipFuncSetAttribute(const void *f, int what, int value) { (void)f; (void)what; (void)value; return 0; }
int hipGetSymbolAddress(void **p, const void *s) { *p = (void *)s; return 0; }
int hipHostMalloc(void **p, size_t n, unsigned flags) { (void)flags; *p = calloc(1, n); return *p ? 0 : 2; }
int hipHostFree(void *p) { free(p); return 0; }
int hipEventCreate(void **e) { *e = NULL; return 0; }
int hipEventDestroy(void *e) { (void)e; return 0; }

static __thread struct { dim3_t grid, block; size_t lds; void *stream; } call;

int __hipPushCallConfiguration(dim3_t grid, dim3_t block, size_t lds, void *stream)
{
    call.grid = grid;
    call.block = block;
    call.lds = lds;
    call.stream = stream;
    return 0;
}

int __hipPopCallConfiguration(dim3_t *grid, dim3_t *block, size_t *lds, void **stream)
{
    *grid = call.grid;
    *block = call.block;
    *lds = call.lds;
    *stream = call.stream;
    return 0;
}

int hipLaunchKernel(const void *f, dim3_t grid, dim3_t block, void **args, size_t lds, void *stream)
{
    (void)f;
    (void)lds;
    (void)stream;
    if (n_launches < 4096) {
        launch_t *l = &launches[n_launches++];
        l->grid[0] = grid.x, l->grid[1] = grid.y, l->grid[2] = grid.z;
        l->block[0] = block.x, l->block[1] = block.y, l->block[2] = block.z;
        l->device = current_device;
        memcpy(l->arg, args[0], sizeof l->arg);   /* the kernels' first argument is a structure of at least that size */
    }
    return 0;
}
