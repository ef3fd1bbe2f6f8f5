// A stand-in for the HIP calls that start kernels, for tests without a GPU:
// loaded before libnlb.so, it takes the library's launches and records them
// instead of running them.  fail_at: the launch (from 0) that is refused, -1
// for none.
#include <cstddef>
#include <cstdint>

namespace {
struct Dim3 {
    uint32_t x, y, z;
};
struct Launch {
    Dim3 grid, block;
    size_t lds;
};
Launch launches[256], pushed;
int count = 0, error = 0;
void *pushed_stream = nullptr;
}  // namespace

extern "C" {
int fail_at = -1;
int launched() { return count; }
void launch_sizes(int i, uint64_t *out) {
    const Launch &l = launches[i];
    const uint64_t v[6] = {l.grid.x, l.grid.y, l.grid.z, l.block.x, l.block.y, l.block.z};
    for (int k = 0; k < 6; k++) out[k] = v[k];
}
void forget() { count = error = 0; }
void leave_error(int e) { error = e; }

int hipGetDevice(int *d) { return *d = 0; }
int hipGetDeviceCount(int *n) {
    *n = 1;
    return 0;
}
int hipSetDevice(int) { return 0; }
int hipFuncSetAttribute(const void *, int, int) { return 0; }
int hipGetLastError() {
    const int e = error;
    error = 0;
    return e;
}
int hipLaunchKernel(const void *, Dim3 grid, Dim3 block, void **, size_t lds, void *) {
    if (count < 256) launches[count] = {grid, block, lds};
    if (count++ != fail_at) return 0;
    return error = 1;                                         // hipErrorInvalidValue
}
int __hipPushCallConfiguration(Dim3 grid, Dim3 block, size_t lds, void *stream) {
    pushed = {grid, block, lds};
    pushed_stream = stream;
    return 0;
}
int __hipPopCallConfiguration(Dim3 *grid, Dim3 *block, size_t *lds, void **stream) {
    *grid = pushed.grid;
    *block = pushed.block;
    *lds = pushed.lds;
    *stream = pushed_stream;
    return 0;
}
}
