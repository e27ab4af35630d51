// Products in 8 bits for many rows a group: the kernels of matmul_f8_tiles.h, but for activations into short rows of h (matmul_f8_ties.hip).
#include "matmul_f8_tiles.h"

namespace emoe {
namespace {

template <int EPI>
__global__ __launch_bounds__(64 * NW) void tiled_kernel(F8Product p, float* __restrict__ partials, int n_tiles, int XCDS) {
    tiles<EPI, false>(p, partials, n_tiles, XCDS);
}

}  // namespace

hipError_t launch_f8_tiled(const F8Product& p, F8Epilogue epilogue, float* partials, hipStream_t st) {
    if (epilogue != kF8Plain && p.lay.nb <= kTieBlocksTiled) return launch_f8_ties(p, epilogue, partials, st);
    DeviceShape shape;
    const hipError_t e = device_shape(&shape);
    if (e != hipSuccess) return e;
    switch (epilogue) {
        case kF8Swiglu: return launch_tiles<kF8Swiglu, false, tiled_kernel<kF8Swiglu>>(p, partials, shape, st);
        case kF8Relu: return launch_tiles<kF8Relu, false, tiled_kernel<kF8Relu>>(p, partials, shape, st);
        default: return launch_tiles<kF8Plain, false, tiled_kernel<kF8Plain>>(p, partials, shape, st);
    }
}

}  // namespace emoe
