// Launch helpers of the cache operators.
#pragma once
#include <cuda_runtime.h>

namespace tts {

// Every kernel of the cache operators is launched as a programmatic dependent of whatever precedes it in
// the stream: its blocks may become resident while the predecessor drains.  grid_dependency_wait() is each
// kernel's first statement before it touches memory (it returns when the predecessor has completed and its
// writes are visible), so the order of the stream holds; grid_launch_dependents() lets the successor start
// its own launch.  Blocks that are resident while the predecessor still writes must not read what it writes through the
// read-only path, so none of these kernels' pointers is __restrict__.  Two of these in a row cost about 2 us less than two plain launches.
__device__ __forceinline__ void grid_dependency_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void grid_launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

template <typename... KArgs, typename... Args>
cudaError_t launch_dependent(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid; cfg.blockDim = block; cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// The context's device for the span of a call, whichever device is current in the calling thread.
class OnDevice {
public:
    explicit OnDevice(int device) : back_(-1), err_(cudaSuccess) {
        int now = device;
        err_ = cudaGetDevice(&now);
        if (err_ == cudaSuccess && now != device) { err_ = cudaSetDevice(device); if (err_ == cudaSuccess) back_ = now; }
    }
    ~OnDevice() { if (back_ >= 0) cudaSetDevice(back_); }
    OnDevice(const OnDevice&) = delete;
    OnDevice& operator=(const OnDevice&) = delete;
    cudaError_t error() const { return err_; }
private:
    int back_;
    cudaError_t err_;
};

}  // namespace tts
