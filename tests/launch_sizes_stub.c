/* launch_stub.c, and a launch that the runtime does not take (2^32 work-items or more in a dimension, 2^16 workgroups or more in the second
   or third) fails as it does there.  The name of the last launch's kernel is kept. */
#include <string.h>
#define hipLaunchKernel counted_launch
#include "launch_stub.c"
#undef hipLaunchKernel

static struct {
    const void *kernel;
    const char *name;
} kernels[1 << 14];
static int known;
static const char *last_name;

void __hipRegisterFunction(void **modules, const void *kernel, char *stub_name, const char *name, unsigned limit, void *tid, void *bid, void *block_dim,
                           void *grid_dim, int *words)
{
    (void)modules, (void)stub_name, (void)limit, (void)tid, (void)bid, (void)block_dim, (void)grid_dim, (void)words;
    if (known < 1 << 14) {
        kernels[known].kernel = kernel;
        kernels[known++].name = name;
    }
}
const char *launch_stub_kernel(void) { return last_name; }
int launch_stub_known(void) { return known; }
const char *launch_stub_kernel_of(int i) { return kernels[i].name; }
uint64_t launch_stub_workgroups(void) { return (uint64_t)grid.x * grid.y * grid.z; }
uint32_t launch_stub_row(void) { return grid.x; }

int hipLaunchKernel(const void *kernel, dim3_t g, dim3_t b, void **args, size_t shared, void *stream)
{
    const int status = counted_launch(kernel, g, b, args, shared, stream);
    last_name = "";
    for (int i = 0; i < known; ++i)
        if (kernels[i].kernel == kernel) last_name = kernels[i].name;
    if (status) return status;
    const uint64_t most = 1ull << 32;
    if (!g.x || !g.y || !g.z || (uint64_t)g.x * b.x >= most || (uint64_t)g.y * b.y >= most || (uint64_t)g.z * b.z >= most || g.y >= 1 << 16 || g.z >= 1 << 16)
        return last_error = 9;   /* hipErrorInvalidConfiguration */
    return 0;
}
