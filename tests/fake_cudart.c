/* A stand-in for the CUDA runtime that runs nothing and writes down what it is asked, with the
 * device that is current then: the host side of the libraries can be tested on a machine without a
 * GPU, or with more devices than it has.  Device memory is addresses that nobody reads; a copy to
 * the host delivers zeros. */
#include <stdint.h>
#include <string.h>

#include <cuda.h>
#include <cuda_runtime_api.h>

#define DEVICES 4
#define SMS 148

typedef struct {
    char what[40];
    int device;
    void *stream;
    unsigned grid[3], threads;
} record;

static record entries[4096];
static int count, current;
static uintptr_t next_address = 1u << 20;
static struct { dim3 grid, block; size_t smem; void *stream; } pushed;

static cudaError_t note(const char *what, void *stream, const dim3 *grid, const dim3 *block)
{
    record *r = &entries[count];
    if (count == 4096) return cudaErrorUnknown;
    ++count;
    memset(r, 0, sizeof(*r));
    strncpy(r->what, what, sizeof(r->what) - 1);
    r->device = current;
    r->stream = stream;
    if (grid) r->grid[0] = grid->x, r->grid[1] = grid->y, r->grid[2] = grid->z, r->threads = block->x * block->y * block->z;
    return cudaSuccess;
}

int fake_count(void) { return count; }
void fake_clear(void) { count = 0; }
const char *fake_what(int i) { return entries[i].what; }
int fake_device(int i) { return entries[i].device; }
void *fake_stream(int i) { return entries[i].stream; }
unsigned fake_blocks(int i) { return entries[i].grid[0] * entries[i].grid[1] * entries[i].grid[2]; }

cudaError_t cudaGetDevice(int *device) { *device = current; return cudaSuccess; }
cudaError_t cudaSetDevice(int device)
{
    if (device < 0 || device >= DEVICES) return cudaErrorInvalidDevice;
    current = device;
    return cudaSuccess;
}
cudaError_t cudaDeviceGetAttribute(int *v, enum cudaDeviceAttr a, int device)
{
    (void)device;
    *v = a == cudaDevAttrMultiProcessorCount ? SMS : 0;
    return cudaSuccess;
}
cudaError_t cudaGetDeviceProperties(struct cudaDeviceProp *p, int device)
{
    (void)device;
    memset(p, 0, sizeof(*p));
    p->multiProcessorCount = SMS;
    return cudaSuccess;
}
cudaError_t cudaDeviceGetStreamPriorityRange(int *least, int *greatest) { *least = *greatest = 0; return cudaSuccess; }
cudaError_t cudaGetLastError(void) { return cudaSuccess; }

cudaError_t cudaMalloc(void **p, size_t bytes)
{
    *p = (void *)next_address;
    next_address += (bytes + 511) & ~(size_t)255;
    return note("malloc", 0, 0, 0);
}
cudaError_t cudaFree(void *p) { return p ? note("free", 0, 0, 0) : cudaSuccess; }
cudaError_t cudaMemset(void *p, int v, size_t n) { (void)p, (void)v, (void)n; return note("memset", 0, 0, 0); }
cudaError_t cudaMemsetAsync(void *p, int v, size_t n, cudaStream_t s) { (void)p, (void)v, (void)n; return note("memset", s, 0, 0); }
cudaError_t cudaMemcpy(void *d, const void *s, size_t n, enum cudaMemcpyKind k)
{
    (void)s;
    if (k == cudaMemcpyDeviceToHost) memset(d, 0, n);
    return note("memcpy", 0, 0, 0);
}
cudaError_t cudaMemcpyAsync(void *d, const void *s, size_t n, enum cudaMemcpyKind k, cudaStream_t stream)
{
    (void)s;
    if (k == cudaMemcpyDeviceToHost) memset(d, 0, n);
    return note("memcpy", stream, 0, 0);
}
cudaError_t cudaStreamSynchronize(cudaStream_t s) { return note("synchronize", s, 0, 0); }
cudaError_t cudaEventCreate(cudaEvent_t *e) { *e = 0; return note("event", 0, 0, 0); }
cudaError_t cudaEventDestroy(cudaEvent_t e) { (void)e; return note("event", 0, 0, 0); }
cudaError_t cudaEventRecord(cudaEvent_t e, cudaStream_t s) { (void)e; return note("event", s, 0, 0); }
cudaError_t cudaEventSynchronize(cudaEvent_t e) { (void)e; return note("event", 0, 0, 0); }
cudaError_t cudaEventElapsedTime(float *ms, cudaEvent_t a, cudaEvent_t b) { (void)a, (void)b; *ms = 1.0f; return cudaSuccess; }

cudaError_t cudaFuncSetAttribute(const void *f, enum cudaFuncAttribute a, int v) { (void)f, (void)a, (void)v; return note("attribute", 0, 0, 0); }
cudaError_t cudaFuncGetAttributes(struct cudaFuncAttributes *a, const void *f) { (void)f; memset(a, 0, sizeof(*a)); return cudaSuccess; }
cudaError_t cudaOccupancyMaxActiveClusters(int *n, const void *f, const cudaLaunchConfig_t *c) { (void)f, (void)c; *n = SMS / 2; return cudaSuccess; }
cudaError_t cudaOccupancyMaxActiveBlocksPerMultiprocessorWithFlags(int *n, const void *f, int t, size_t s, unsigned flags)
{
    (void)f, (void)t, (void)s, (void)flags;
    *n = 1;
    return cudaSuccess;
}
cudaError_t cudaGetSymbolAddress(void **p, const void *symbol) { (void)symbol; return cudaMalloc(p, 256); }

static CUresult encode(CUtensorMap *m, CUtensorMapDataType t, cuuint32_t rank, void *base, const cuuint64_t *dims, const cuuint64_t *strides,
                       const cuuint32_t *box, const cuuint32_t *steps, CUtensorMapInterleave i, CUtensorMapSwizzle s,
                       CUtensorMapL2promotion l, CUtensorMapFloatOOBfill f)
{
    (void)t, (void)rank, (void)base, (void)dims, (void)strides, (void)box, (void)steps, (void)i, (void)s, (void)l, (void)f;
    memset(m, 0, sizeof(*m));
    return CUDA_SUCCESS;
}
cudaError_t cudaGetDriverEntryPoint(const char *name, void **fn, unsigned long long flags, enum cudaDriverEntryPointQueryResult *q)
{
    (void)name, (void)flags;
    *fn = (void *)encode;
    *q = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}

cudaError_t cudaLaunchKernel(const void *f, dim3 grid, dim3 block, void **args, size_t smem, cudaStream_t s)
{
    (void)f, (void)args, (void)smem;
    return note("launch", s, &grid, &block);
}
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t *c, const void *f, void **args)
{
    (void)f, (void)args;
    return note("launch", c->stream, &c->gridDim, &c->blockDim);
}
unsigned __cudaPushCallConfiguration(dim3 grid, dim3 block, size_t smem, void *stream)
{
    pushed.grid = grid, pushed.block = block, pushed.smem = smem, pushed.stream = stream;
    return 0;
}
cudaError_t __cudaPopCallConfiguration(dim3 *grid, dim3 *block, size_t *smem, void *stream)
{
    *grid = pushed.grid, *block = pushed.block, *smem = pushed.smem, *(void **)stream = pushed.stream;
    return cudaSuccess;
}
void **__cudaRegisterFatBinary(void *image) { static void *handle; (void)image; return &handle; }
void __cudaRegisterFatBinaryEnd(void **h) { (void)h; }
void __cudaUnregisterFatBinary(void **h) { (void)h; }
void __cudaRegisterFunction(void **h, const char *f, char *d, const char *n, int l, void *a, void *b, void *c, void *e, int *w)
{
    (void)h, (void)f, (void)d, (void)n, (void)l, (void)a, (void)b, (void)c, (void)e, (void)w;
}
void __cudaRegisterVar(void **h, char *v, char *a, const char *n, int ext, size_t size, int constant, int global)
{
    (void)h, (void)v, (void)a, (void)n, (void)ext, (void)size, (void)constant, (void)global;
}
