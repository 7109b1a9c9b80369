// A CUDA runtime that launches nothing: it stands in for the real one under the cache's host code, keeps each device's
// shared-memory limits, refuses launches above them as the real one does, and notes what would have run.
#include <cuda_runtime_api.h>

#include <map>
#include <string>
#include <utility>

namespace {
int device = 0, sms[4] = {152, 152, 152, 152}, fail_attribute = 0, launches = 0;
std::map<std::pair<int, const void *>, int> limits;
std::map<const void *, std::string> names;
std::string last_name;
unsigned last_grid[3];
struct { dim3 grid, block; size_t smem; void *stream; } pushed;

int launch(const void *f, dim3 grid, size_t smem) {
    const auto it = limits.find({device, f});
    if (static_cast<int>(smem) > (it == limits.end() ? 48 * 1024 : it->second)) return cudaErrorInvalidValue;
    if (names[f].find("join") == std::string::npos) {
        last_name = names[f];
        last_grid[0] = grid.x;
        last_grid[1] = grid.y;
        last_grid[2] = grid.z;
    }
    ++launches;
    return cudaSuccess;
}
}  // namespace

namespace qe {
unsigned *device_error_word() {
    static unsigned word[4];
    return &word[device];
}
}  // namespace qe

extern "C" {
void fake_device(int d, int count) { device = d; sms[d] = count; }
void fake_fail_attribute(int n) { fail_attribute = n; }
int fake_launches() { return launches; }
const char *fake_kernel() { return last_name.c_str(); }
unsigned fake_grid(int i) { return last_grid[i]; }

cudaError_t cudaGetDevice(int *d) { *d = device; return cudaSuccess; }
cudaError_t cudaGetLastError(void) { return cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int *v, cudaDeviceAttr, int d) { *v = sms[d]; return cudaSuccess; }
cudaError_t cudaFuncSetAttribute(const void *f, cudaFuncAttribute, int bytes) {
    if (fail_attribute > 0) {
        --fail_attribute;
        return cudaErrorInvalidValue;
    }
    limits[{device, f}] = bytes;
    return cudaSuccess;
}
cudaError_t cudaMallocAsync(void **p, size_t, cudaStream_t) { *p = reinterpret_cast<void *>(0x100000); return cudaSuccess; }
cudaError_t cudaFreeAsync(void *, cudaStream_t) { return cudaSuccess; }
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t *c, const void *f, void **) {
    return static_cast<cudaError_t>(launch(f, c->gridDim, c->dynamicSmemBytes));
}

// what compiled launches call
void **__cudaRegisterFatBinary(void *) { static void *handle; return &handle; }
void __cudaRegisterFatBinaryEnd(void **) {}
void __cudaUnregisterFatBinary(void **) {}
void __cudaRegisterFunction(void **, const char *host, char *, const char *name, int, void *, void *, void *, void *, int *) { names[host] = name; }
unsigned __cudaPushCallConfiguration(dim3 grid, dim3 block, size_t smem, void *stream) {
    pushed = {grid, block, smem, stream};
    return 0;
}
int __cudaPopCallConfiguration(dim3 *grid, dim3 *block, size_t *smem, void *stream) {
    *grid = pushed.grid;
    *block = pushed.block;
    *smem = pushed.smem;
    *static_cast<void **>(stream) = pushed.stream;
    return 0;
}
int __cudaGetKernel(void **kernel, const void *f) { *kernel = const_cast<void *>(f); return 0; }
int __cudaLaunchKernel(void *kernel, dim3 grid, dim3, void **, size_t smem, void *) { return launch(kernel, grid, smem); }
}
