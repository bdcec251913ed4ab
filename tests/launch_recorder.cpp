// The few calls of the HIP runtime that launches of liblshbeam.so go through, answered without a GPU: a launch is written down
// instead of made.  Loaded with its symbols global before the library, these stand in front of the runtime's.
#include <cstddef>
#include <cstdint>
#include <vector>

struct Dim3 { uint32_t x, y, z; };
struct Launch { uint64_t grid, block, lds; };

static std::vector<Launch> launches;
static Launch pushed;
static Dim3 pushed_grid, pushed_block;
static void* pushed_stream;
static int refuse_above = -1, last_error = 0;   // bytes of LDS above which hipFuncSetAttribute gives an error (-1: never)
constexpr int kInvalidValue = 1;

extern "C" {

int hipGetDevice(int* dev) { *dev = 0; return 0; }
int hipFuncSetAttribute(const void*, int, int value) {
    if (refuse_above < 0 || value <= refuse_above) return 0;
    return last_error = kInvalidValue;
}
int hipGetLastError() { const int e = last_error; last_error = 0; return e; }
int hipPeekAtLastError() { return last_error; }
int __hipPushCallConfiguration(Dim3 grid, Dim3 block, size_t lds, void* stream) {
    pushed_grid = grid; pushed_block = block; pushed.lds = lds; pushed_stream = stream;
    return 0;
}
int __hipPopCallConfiguration(Dim3* grid, Dim3* block, size_t* lds, void** stream) {
    *grid = pushed_grid; *block = pushed_block; *lds = pushed.lds; *stream = pushed_stream;
    return 0;
}
int hipLaunchKernel(const void*, Dim3 grid, Dim3 block, void**, size_t lds, void*) {
    launches.push_back(Launch{(uint64_t)grid.x * grid.y * grid.z, (uint64_t)block.x * block.y * block.z, lds});
    return 0;
}

// for the tests
void recorder_begin(int refuse) { launches.clear(); refuse_above = refuse; last_error = 0; }
int recorder_count() { return (int)launches.size(); }
void recorder_get(int i, uint64_t* to) { to[0] = launches[i].grid; to[1] = launches[i].block; to[2] = launches[i].lds; }

}  // extern "C"
