// Takes the place of the HIP runtime's launch calls under a libheadkv.so that is
// loaded after it: notes the grids and launches nothing.
#include <hip/hip_runtime.h>

namespace {

struct Launch {
    unsigned grid, block;
};
constexpr int kMost = 4096;
Launch seen[kMost];
int count = 0;
dim3 next_grid, next_block;
size_t next_lds;
hipStream_t next_stream;

}  // namespace

extern "C" {

hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t stream) {
    next_grid = grid, next_block = block, next_lds = lds, next_stream = stream;
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* stream) {
    *grid = next_grid, *block = next_block, *lds = next_lds, *stream = next_stream;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void*, dim3 grid, dim3 block, void**, size_t, hipStream_t) {
    if (count < kMost) seen[count] = {grid.x, block.x};
    ++count;
    return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }

int fake_launches() { return count; }
void fake_launch(int i, unsigned* grid, unsigned* block) {
    *grid = seen[i].grid;
    *block = seen[i].block;
}
void fake_clear() { count = 0; }

}  // extern "C"
