/* A stand-in for what the operators on device tensors ask of the CUDA runtime, preloaded before libisc.so: kernels do nothing,
 * launches are recorded with their grids, tensor maps are always made, and the kernels' device variables are words of the host. */
#include <cuda_runtime_api.h>
#include <pthread.h>
#include <string.h>

#define MAX_FUNCS 512
#define MAX_VARS 64
#define MAX_LAUNCHES 4096

static struct { const void *host; const char *name; } funcs[MAX_FUNCS];
static struct { const void *host; const char *name; int word; } vars[MAX_VARS];
static struct { const char *name; dim3 grid, block; } launches[MAX_LAUNCHES];
static int n_funcs, n_vars, n_launches, device;
static pthread_mutex_t lock = PTHREAD_MUTEX_INITIALIZER;
static __thread struct { dim3 grid, block; size_t smem; void *stream; } pending;

/* what the tests ask and set */
void fake_reset(void) { n_launches = 0; }
int fake_launches(void) { return n_launches; }
const char *fake_launch_name(int i) { return launches[i].name; }
unsigned fake_launch_blocks(int i) { return launches[i].grid.x; }
void fake_set_device(int d) { device = d; }
/* `n` more waits have run out in the kernels of the file'th file that counts them; returns how many files do */
int fake_timeouts(int file, int n)
{
    int found = 0;
    for (int i = 0; i < n_vars; ++i)
        if (strstr(vars[i].name, "timeout") && found++ == file) vars[i].word += n;
    return found;
}

void **__cudaRegisterFatBinary(void *image) { static void *handle; (void)image; return &handle; }
void __cudaRegisterFatBinaryEnd(void **h) { (void)h; }
void __cudaUnregisterFatBinary(void **h) { (void)h; }
void __cudaRegisterVar(void **h, char *host, char *dev, const char *name, int ext, size_t size, int constant, int global)
{
    (void)h; (void)dev; (void)ext; (void)size; (void)constant; (void)global;
    if (n_vars < MAX_VARS) { vars[n_vars].host = host; vars[n_vars].name = name; ++n_vars; }
}
void __cudaRegisterFunction(void **h, const char *host, char *dev, const char *name, int limit, uint3 *t, uint3 *b, dim3 *bd, dim3 *gd, int *w)
{
    (void)h; (void)dev; (void)limit; (void)t; (void)b; (void)bd; (void)gd; (void)w;
    if (n_funcs < MAX_FUNCS) { funcs[n_funcs].host = host; funcs[n_funcs].name = name; ++n_funcs; }
}
unsigned __cudaPushCallConfiguration(dim3 grid, dim3 block, size_t smem, void *stream)
{
    pending.grid = grid; pending.block = block; pending.smem = smem; pending.stream = stream;
    return 0;
}
cudaError_t __cudaPopCallConfiguration(dim3 *grid, dim3 *block, size_t *smem, void *stream)
{
    *grid = pending.grid; *block = pending.block; *smem = pending.smem; *(void **)stream = pending.stream;
    return cudaSuccess;
}

static cudaError_t record(const void *func, dim3 grid, dim3 block)
{
    cudaError_t e = cudaErrorInvalidDeviceFunction;
    pthread_mutex_lock(&lock);
    for (int i = 0; i < n_funcs; ++i)
        if (funcs[i].host == func && n_launches < MAX_LAUNCHES) {
            launches[n_launches].name = funcs[i].name;
            launches[n_launches].grid = grid;
            launches[n_launches++].block = block;
            e = cudaSuccess;
            break;
        }
    pthread_mutex_unlock(&lock);
    return e;
}
cudaError_t cudaLaunchKernel(const void *func, dim3 grid, dim3 block, void **args, size_t smem, cudaStream_t st)
{
    (void)args; (void)smem; (void)st;
    return record(func, grid, block);
}
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t *config, const void *func, void **args) { (void)args; return record(func, config->gridDim, config->blockDim); }
cudaError_t cudaFuncSetAttribute(const void *func, enum cudaFuncAttribute attr, int value) { (void)func; (void)attr; (void)value; return cudaSuccess; }

static cudaError_t copy(const void *symbol, void *at, size_t n, int back)
{
    cudaError_t e = cudaErrorInvalidSymbol;
    pthread_mutex_lock(&lock);
    for (int i = 0; i < n_vars; ++i)
        if (vars[i].host == symbol && n == sizeof(vars[i].word)) {
            memcpy(back ? (void *)&vars[i].word : at, back ? at : (void *)&vars[i].word, n);
            e = cudaSuccess;
        }
    pthread_mutex_unlock(&lock);
    return e;
}
cudaError_t cudaMemcpyFromSymbolAsync(void *dst, const void *symbol, size_t n, size_t offset, enum cudaMemcpyKind kind, cudaStream_t st)
{
    (void)offset; (void)kind; (void)st;
    return copy(symbol, dst, n, 0);
}
cudaError_t cudaMemcpyToSymbolAsync(const void *symbol, const void *src, size_t n, size_t offset, enum cudaMemcpyKind kind, cudaStream_t st)
{
    (void)offset; (void)kind; (void)st;
    return copy(symbol, (void *)src, n, 1);
}

cudaError_t cudaGetLastError(void) { return cudaSuccess; }
const char *cudaGetErrorString(cudaError_t e) { return e == cudaSuccess ? "no error" : "fake error"; }
cudaError_t cudaGetDevice(int *d) { *d = device; return cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int *value, enum cudaDeviceAttr attr, int d)
{
    (void)d;
    *value = attr == cudaDevAttrMultiProcessorCount ? 148 : 0;
    return cudaSuccess;
}
static int encode(void) { return 0; }
cudaError_t cudaGetDriverEntryPoint(const char *symbol, void **fn, unsigned long long flags, enum cudaDriverEntryPointQueryResult *r)
{
    (void)symbol; (void)flags;
    *fn = (void *)encode;
    *r = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}
cudaError_t cudaStreamSynchronize(cudaStream_t st) { (void)st; return cudaSuccess; }
