/* Stand-ins for the CUDA runtime calls that the library's host code makes, for tests of that code without a GPU:
 * device memory is host memory, launches are written down and not made, and the n-th launch can be told to fail. */
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

typedef struct { unsigned x, y, z; } dim3_;
typedef struct { dim3_ grid, block; size_t smem; void *stream; void *attrs; unsigned n_attrs; } config_;

static char text[1 << 16];
static size_t used;
static int launches, failing = -1, stale = -1, mallocs, no_room = -1, last;

static void note(const char *line) {
    if (used + strlen(line) + 2 < sizeof text) used += (size_t)sprintf(text + used, "%s\n", line);
}

const char *fake_log(void) { return text; }
void fake_reset(int fail_launch) { text[0] = 0; used = 0; launches = 0; failing = fail_launch; stale = -1; mallocs = last = 0; no_room = -1; }
/* after the n-th launch an error of somebody else's is found */
void fake_stale_error(int after_launch) { stale = after_launch; }

/* the n-th allocation from now on finds no memory; errors are kept until they are asked for, as the runtime keeps them */
void fake_no_room(int allocation) { mallocs = 0; no_room = allocation; }

static int launch(dim3_ g) {
    char line[96];
    const int fails = launches++ == failing;
    snprintf(line, sizeof line, "%s %u %u %u", fails ? "failed-launch" : "launch", g.x, g.y, g.z);
    note(line);
    return fails ? last = 701 : 0;
}

int cudaLaunchKernelExC(const config_ *c, const void *f, void **args) { (void)f; (void)args; return launch(c->grid); }
int cudaLaunchKernel(const void *f, dim3_ g, dim3_ b, void **args, size_t smem, void *st) {
    (void)f; (void)b; (void)args; (void)smem; (void)st;
    return launch(g);
}
int cudaFuncSetAttribute(const void *f, int attr, int value) { (void)f; (void)attr; (void)value; return 0; }
int cudaGetLastError(void) {
    const int e = launches - 1 == stale ? 9 : last;
    last = 0;
    return e;
}
int cudaGetDevice(int *d) { *d = 0; return 0; }
int cudaDeviceGetAttribute(int *v, int attr, int d) { (void)attr; (void)d; *v = 148; return 0; }
int cudaMalloc(void **p, size_t n) {
    *p = mallocs++ == no_room ? NULL : aligned_alloc(256, (n + 255) / 256 * 256);
    return *p ? 0 : (last = 2);
}
int cudaFree(void *p) { free(p); return 0; }
int cudaMemset(void *p, int v, size_t n) {
    memset(p, v, n);
    note("memset on the default stream");
    return 0;
}
int cudaMemsetAsync(void *p, int v, size_t n, void *st) {
    char line[96];
    memset(p, v, n);
    snprintf(line, sizeof line, "memset %d %zu on %zu", v, n, (size_t)(uintptr_t)st);
    note(line);
    return 0;
}
int cudaStreamSynchronize(void *st) {
    note((uintptr_t)st <= 1 ? "wait for the default stream" : "wait for another stream");   /* (1: cudaStreamLegacy) */
    return 0;
}
