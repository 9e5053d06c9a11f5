// stand_in_hip.cpp, which also notes how large what is asked for is: bytes of device memory, and the work items of a launch's widest dimension.
#define hipMalloc stand_in_unused_malloc
#define hipLaunchKernel stand_in_unused_launch
#define __hipPushCallConfiguration stand_in_unused_push
#define __hipPopCallConfiguration stand_in_unused_pop
#include "stand_in_hip.cpp"
#undef hipMalloc
#undef hipLaunchKernel
#undef __hipPushCallConfiguration
#undef __hipPopCallConfiguration

static size_t bytes_held, most_items, most_groups;
static dim3 next_grid, next_block;

extern "C" {
size_t stand_in_bytes() { return bytes_held; }   // of every hipMalloc so far
size_t stand_in_items() { return most_items; }   // of the widest dimension of any launch so far
size_t stand_in_groups() { return most_groups; } // workgroups of the second or third dimension of any launch so far, the most

hipError_t hipMalloc(void** p, size_t n) {
    bytes_held += n;
    return stand_in_unused_malloc(p, n);
}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t) {
    next_grid = grid;
    next_block = block;
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* stream) {
    *grid = next_grid;
    *block = next_block;
    *lds = 0;
    *stream = nullptr;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void* fn, dim3 grid, dim3 block, void** args, size_t lds, hipStream_t stream) {
    const size_t items[3] = {(size_t)grid.x * block.x, (size_t)grid.y * block.y, (size_t)grid.z * block.z};
    for (size_t n : items) most_items = n > most_items ? n : most_items;
    most_groups = grid.y > most_groups ? grid.y : most_groups;
    most_groups = grid.z > most_groups ? grid.z : most_groups;
    return stand_in_unused_launch(fn, grid, block, args, lds, stream);
}
}
