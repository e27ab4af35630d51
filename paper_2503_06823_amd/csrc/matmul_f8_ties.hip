// Products in 8 bits for many rows a group, activations into rows of h of up to kTieBlocksTiled blocks: the kernels of matmul_f8_tiles.h, which also note the
// elements near ties of two codes (see kNearTie), and a launch that sums those once more.
#include "matmul_f8_tiles.h"

namespace emoe {
namespace {

template <int EPI>
__global__ __launch_bounds__(64 * NW) void tiled_ties(F8Product p, float* __restrict__ partials, int n_tiles, int XCDS) {
    tiles<EPI, true>(p, partials, n_tiles, XCDS);
}

// The elements of h that store_h() found near ties, once more, those that matter to their row: in the tiles themselves nobody would multiply meanwhile, and the
// other blocks of a row are not known.  A thread looks at 64 outputs of a row at a time; of what a workgroup finds a thread each asks whether it matters,
// and half wavefronts sum what does.  All of it is memory latencies, one after the other: so workgroups are large, and no more than there are CUs.
// A row is at least as large as the square root of the sum of the squares of its blocks' largest elements, each 224 and more under its power.  An element matters
// if its two codes, 32 apart from 256 on and 16 below, are more than 1 / 16 of that apart.
constexpr float kMatters32 = 5.22f, kMatters16 = 1.306f;  // (32 * 16 / 224)^2, (16 * 16 / 224)^2: what the row's squares have to stay below, in this block's power
constexpr int kNearThreads = 512, kNearAtOnce = 16;      // of a workgroup; words of 64 outputs that a thread looks at in one go
constexpr int kNearList = 2048;                          // elements that a workgroup lists at once
struct NearElement {  // of a list: (round * threads + thread) * 64 + bit
    int row, nb, n;
    __device__ NearElement(uint32_t entry, uint32_t word0, uint32_t stride, uint32_t rows) {
        const uint32_t word = word0 + entry / (64 * kNearThreads) * stride + entry / 64 % kNearThreads;  // [block][half][row]
        const int half_block = (int)(word / rows), bit = entry & 63;
        row = (int)(word % rows);
        nb = half_block >> 1;
        n = half_block * 64 + ((bit >> 2) & 3) * 16 + (bit >> 4) * 4 + (bit & 3);  // 16 a quad of the lanes that found them
    }
};
template <int M>
__global__ __launch_bounds__(kNearThreads) void near_ties_kernel(F8Product p) {
    __shared__ uint32_t list[kNearList], matters[kNearList];
    __shared__ int counts[kNearThreads / 64], how_many;
    const int thread = threadIdx.x, lane = thread & 63, wave = thread >> 6, half = thread & 31;
    const uint32_t words = 2u * p.lay.nb * p.rows, stride = gridDim.x * kNearThreads;
    // a lane of a half wavefront knows two groups
    int begin_of[2] = {0, 0}, end_of[2] = {half == 0 ? p.rows : 0, 0}, end = p.rows;
    if (p.offsets != nullptr) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            begin_of[i] = half + 32 * i < p.groups ? p.offsets[half + 32 * i] : 0;
            end_of[i] = half + 32 * i < p.groups ? p.offsets[half + 32 * i + 1] : 0;
        }
        end = p.offsets[p.groups];
    }
    auto code_of = [&](const NearElement& e) { return p.h.codes + (size_t)e.row * p.h.row_step + (size_t)(e.n >> 4) * p.h.piece_step + (e.n & 15); };
    auto power_of = [&](const NearElement& e) { return (uint32_t)reinterpret_cast<const uint8_t*>(p.h.scales + (size_t)(e.nb >> 2) * p.h.rows + e.row)[e.nb & 3]; };
    for (uint32_t word0 = blockIdx.x * kNearThreads; word0 < words; word0 += kNearAtOnce * stride) {
        uint64_t near[kNearAtOnce];
        int mine = 0;
#pragma unroll
        for (int r = 0; r < kNearAtOnce; ++r) {
            const uint32_t word = word0 + r * stride + thread;
            near[r] = word < words ? reinterpret_cast<const uint64_t*>(p.near)[word] : 0;
        }
#pragma unroll
        for (int r = 0; r < kNearAtOnce; ++r) {
            if (near[r] != 0 && (int)((word0 + r * stride + thread) % (uint32_t)p.rows) >= end) near[r] = 0;  // (behind the last group nobody wrote)
            mine += __popcll(near[r]);
        }
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int below = __shfl_up(upto, o);
            upto += lane >= o ? below : 0;
        }
        if (lane == 63) counts[wave] = upto;
        __syncthreads();
        int total = 0, first = upto - mine;
#pragma unroll
        for (int w = 0; w < kNearThreads / 64; ++w) {
            first += w < wave ? counts[w] : 0;
            total += counts[w];
        }
        for (int base = 0; base < total; base += kNearList) {
            int at = first - base;
#pragma unroll
            for (int r = 0; r < kNearAtOnce; ++r)
                for (uint64_t bits = near[r]; bits != 0; bits &= bits - 1, ++at)
                    if (at >= 0 && at < kNearList) list[at] = (uint32_t)(r * kNearThreads + thread) * 64 + __builtin_ctzll(bits);
            if (thread == 0) how_many = 0;
            __syncthreads();
            const int count = total - base < kNearList ? total - base : kNearList;
            for (int i = thread; i < count; i += kNearThreads) {
                const NearElement e(list[i], word0, stride, (uint32_t)p.rows);
                const uint32_t code = *code_of(e) & 127u;
                const int power = (int)power_of(e);
                uint32_t powers[(kTieBlocksTiled + 3) / 4];
#pragma unroll
                for (int j = 0; j < (kTieBlocksTiled + 3) / 4; ++j) powers[j] = 4 * j < p.lay.nb ? p.h.scales[(size_t)j * p.h.rows + e.row] : 0;
                float squares = 0.0f;  // of the row's blocks' powers, over this one's
#pragma unroll
                for (int j = 0; j < kTieBlocksTiled; ++j)
                    if (j < p.lay.nb) squares += ldexpf(1.0f, 2 * ((int)((powers[j >> 2] >> (8 * (j & 3))) & 255u) - power));
                if (squares < (code >= 0x78u ? kMatters32 : kMatters16)) matters[atomicAdd(&how_many, 1)] = list[i];  // (0x78: 256.  In any order: each is one's own)
            }
            __syncthreads();
            for (int i = thread >> 5; i < how_many; i += kNearThreads / 32) {
                const NearElement e(matters[i], word0, stride, (uint32_t)p.rows);
                const uint32_t power = power_of(e), x_row = p.perm != nullptr ? (uint32_t)p.perm[e.row] / (uint32_t)p.k : (uint32_t)e.row;
                const uint32_t low = (uint32_t)(__ballot(begin_of[0] <= e.row && e.row < end_of[0]) >> (lane & 32));
                const uint32_t high = (uint32_t)(__ballot(begin_of[1] <= e.row && e.row < end_of[1]) >> (lane & 32));
                if ((low | high) == 0) continue;
                const int group = low != 0 ? __builtin_ctz(low) : 32 + __builtin_ctz(high);
                const uint8_t* matrix[M];
                matrix[0] = p.w0 + (size_t)group * p.matrix_bytes;
                if constexpr (M == 2) matrix[1] = p.w1 + (size_t)group * p.matrix_bytes;
                const float h = f8_h<M, 32>(p.lay, matrix, e.n, F8RowInMemory(p.x, x_row));
                if (half == 0) *code_of(e) = (uint8_t)f8_codes(h, 0.0f, 0.0f, 0.0f, f8_inverse(power));
            }
            __syncthreads();
        }
        __syncthreads();
    }
}

template <int EPI>
hipError_t launch(const F8Product& p, float* partials, hipStream_t st) {
    DeviceShape shape;
    hipError_t e = device_shape(&shape);
    if (e == hipSuccess) e = launch_tiles<EPI, true, tiled_ties<EPI>>(p, partials, shape, st);
    if (e != hipSuccess) return e;
    const long long all = (2ll * p.lay.nb * p.rows + kNearThreads - 1) / kNearThreads;
    near_ties_kernel<EPI == kF8Swiglu ? 2 : 1><<<(unsigned)(all < shape.groups ? all : shape.groups), kNearThreads, 0, st>>>(p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_f8_ties(const F8Product& p, F8Epilogue epilogue, float* partials, hipStream_t st) {
    return epilogue == kF8Swiglu ? launch<kF8Swiglu>(p, partials, st) : launch<kF8Relu>(p, partials, st);
}

}  // namespace emoe
