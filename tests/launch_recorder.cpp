// Stands in for the HIP runtime in front of the library, so that its host code runs without a GPU: launches are written down instead
// of made, and the call that a test names fails.  Loaded into the global scope ahead of liblccrf.so (test_encoder_launches.py).
#include <stddef.h>
#include <stdint.h>

#include <vector>

struct Dim { uint32_t x, y, z; };

namespace {
struct Launch { Dim grid, block; };
std::vector<Launch> launches;
Dim pushed_grid, pushed_block;
size_t pushed_shared;
void* pushed_stream;
int fail_launch = -1, fail_attribute = 0, last_error = 0;
constexpr int kInvalidConfiguration = 9, kLaunchFailure = 719;
int set(int e) {
    if (e) last_error = e;
    return e;
}
bool launchable(uint32_t grid, uint32_t block) { return grid && block && static_cast<uint64_t>(grid) * block < uint64_t{1} << 32; }
}  // namespace

extern "C" {

// The launch that fails (counted from 0; none below 0), and whether kernels may not have their LDS.
void recorder_reset(int launch, int attribute) {
    launches.clear();
    fail_launch = launch;
    fail_attribute = attribute;
    last_error = 0;
}
int recorder_count() { return static_cast<int>(launches.size()); }
void recorder_get(int i, uint32_t* out) {
    const Launch& l = launches[i];
    const uint32_t v[6] = {l.grid.x, l.grid.y, l.grid.z, l.block.x, l.block.y, l.block.z};
    for (int k = 0; k < 6; ++k) out[k] = v[k];
}

int __hipPushCallConfiguration(Dim grid, Dim block, size_t shared, void* stream) {
    pushed_grid = grid;
    pushed_block = block;
    pushed_shared = shared;
    pushed_stream = stream;
    return 0;
}
int __hipPopCallConfiguration(Dim* grid, Dim* block, size_t* shared, void** stream) {
    *grid = pushed_grid;
    *block = pushed_block;
    *shared = pushed_shared;
    *stream = pushed_stream;
    return 0;
}
int hipLaunchKernel(const void*, Dim grid, Dim block, void**, size_t, void*) {
    const int k = static_cast<int>(launches.size());
    launches.push_back({grid, block});
    if (!launchable(grid.x, block.x) || !launchable(grid.y, block.y) || !launchable(grid.z, block.z)) return set(kInvalidConfiguration);
    return set(k == fail_launch ? kLaunchFailure : 0);
}
int hipGetLastError() {
    const int e = last_error;
    last_error = 0;
    return e;
}
int hipGetDevice(int* device) {
    *device = 0;
    return 0;
}
int hipFuncSetAttribute(const void*, int, int) { return set(fail_attribute ? kLaunchFailure : 0); }

}  // extern "C"
