/* fake_hip.c with the number of threads of every launch in its text, in place of the LDS that it asks for. */
#define hipLaunchKernel unused_hipLaunchKernel
#include "fake_hip.c"
#undef hipLaunchKernel

int hipLaunchKernel(const void *f, dim3 g, dim3 b, void **args, size_t lds, void *s) {
    (void)args; (void)lds; (void)s;
    note("launch", name_of(f), (long long)g.x * b.x * ((long long)g.y * b.y) * ((long long)g.z * b.z));
    return 0;
}
