// Conversions to and from 8 bits under a power of two a block of 128: matrices once when a model is read, rows of activations
// before every product.  All of it is exact but the one rounding to a code, so the bits depend on nothing but the input.
// Bound by memory: an element is read and written once.  Packing 14336 x 4096 of bf16 takes 42 us (4.2 TB/s) and reading it back 27 (6.5 TB/s, of it what was packed
// from caches), rows of 8192 x 4096 21 to 24 us (4.2 to 4.8 TB/s); a copy reaches 5.1.
#include "matrix_f8.h"

namespace emoe {
namespace {

// Eight elements from memory, as numbers; zeros where there are none.
__device__ __forceinline__ void load8(const bf16_t* p, bool there, float (&v)[8]) {
    f8_widened(there ? *reinterpret_cast<const uint4*>(p) : make_uint4(0, 0, 0, 0), v);
}
__device__ __forceinline__ void load8(const float* p, bool there, float (&v)[8]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const float4 r = there ? *reinterpret_cast<const float4*>(p + 4 * h) : make_float4(0, 0, 0, 0);
        v[4 * h] = r.x; v[4 * h + 1] = r.y; v[4 * h + 2] = r.z; v[4 * h + 3] = r.w;
    }
}
__device__ __forceinline__ void store8(bf16_t* p, const float (&v)[8]) {
    uint32_t w[4];  // (the numbers have four significant bits: nothing is rounded)
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (__float_as_uint(v[2 * i]) >> 16) | (__float_as_uint(v[2 * i + 1]) & 0xffff0000u);
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}

// A workgroup takes a block.  Pass i covers rows 16 i .. 16 i + 15, a thread eight columns of one row: reads are whole
// lines of a row, and the block's order in memory keeps the 16 threads' codes of a column group together.
struct BlockPlace {
    int row, column;  // of pass 0, in the block
    int code;         // byte of its eight codes
};
__device__ __forceinline__ BlockPlace block_place(int t) {
    const int r = t >> 4, c = t & 15;
    return {r, c * 8, (c >> 3) * 1024 + ((c >> 1) & 3) * 256 + r * 16 + (c & 1) * 8};
}

template <class E>
__global__ __launch_bounds__(256) void pack_kernel(const E* __restrict__ w, int64_t stride, uint8_t* __restrict__ matrix, F8Layout lay,
                                                   size_t codes, size_t bytes, int N, int K) {
    __shared__ uint32_t tops[4];
    const int kb = blockIdx.x % lay.kb, nb = blockIdx.x / lay.kb;
    const E* from = w + (size_t)blockIdx.y * N * stride;
    uint8_t* to = matrix + (size_t)blockIdx.y * bytes;
    const BlockPlace at = block_place(threadIdx.x);
    const int k = kb * kF8Block + at.column, n0 = nb * kF8Block + at.row;
    float v[8][8];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int n = n0 + 16 * i;
        load8(from + (size_t)(n < N ? n : 0) * stride + (k < K ? k : 0), n < N && k < K, v[i]);
        top = umax(top, f8_top(v[i]));
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) top = umax(top, (uint32_t)__shfl_xor((int)top, o));
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
    const uint32_t byte = f8_scale_byte(umax(umax(tops[0], tops[1]), umax(tops[2], tops[3])));
    const float inverse = f8_inverse(byte);
    uint8_t* block = to + (size_t)(nb * lay.kb + kb) * kF8BlockBytes + at.code;
#pragma unroll
    for (int i = 0; i < 8; ++i) *reinterpret_cast<uint2*>(block + i * kF8Strip) = f8_codes(v[i], inverse);
    // the scale, and zeros for the columns behind the last block that share its dword
    if ((int)threadIdx.x < 4 && (kb == lay.kb - 1 || threadIdx.x == 0) && kb + (int)threadIdx.x < 4 * lay.kg)
        to[codes + (size_t)nb * 4 * lay.kg + kb + threadIdx.x] = threadIdx.x == 0 ? (uint8_t)byte : 0;
    if (blockIdx.x == gridDim.x - 1) {  // and to whole 256 bytes
        const size_t scales = codes + (size_t)lay.nb * 4 * lay.kg;
        if (scales + threadIdx.x < bytes) to[scales + threadIdx.x] = 0;
    }
}

template <class E>
__global__ __launch_bounds__(256) void unpack_kernel(const uint8_t* __restrict__ matrix, E* __restrict__ w, int64_t stride, F8Layout lay,
                                                     size_t codes, size_t bytes, int N, int K) {
    const int kb = blockIdx.x % lay.kb, nb = blockIdx.x / lay.kb;
    const uint8_t* from = matrix + (size_t)blockIdx.y * bytes;
    E* to = w + (size_t)blockIdx.y * N * stride;
    const BlockPlace at = block_place(threadIdx.x);
    const int k = kb * kF8Block + at.column, n0 = nb * kF8Block + at.row;
    if (k >= K) return;
    const uint32_t byte = from[codes + (size_t)nb * 4 * lay.kg + kb];
    const float scale = byte == 255u ? __uint_as_float(0x7fc00000u) : byte == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(byte << 23);
    const uint8_t* block = from + (size_t)(nb * lay.kb + kb) * kF8BlockBytes + at.code;
    uint2 q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = *reinterpret_cast<const uint2*>(block + i * kF8Strip);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int n = n0 + 16 * i;
        if (n >= N) break;
        float v[8];
        v[0] = __builtin_amdgcn_cvt_f32_fp8(q[i].x, 0); v[1] = __builtin_amdgcn_cvt_f32_fp8(q[i].x, 1);
        v[2] = __builtin_amdgcn_cvt_f32_fp8(q[i].x, 2); v[3] = __builtin_amdgcn_cvt_f32_fp8(q[i].x, 3);
        v[4] = __builtin_amdgcn_cvt_f32_fp8(q[i].y, 0); v[5] = __builtin_amdgcn_cvt_f32_fp8(q[i].y, 1);
        v[6] = __builtin_amdgcn_cvt_f32_fp8(q[i].y, 2); v[7] = __builtin_amdgcn_cvt_f32_fp8(q[i].y, 3);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= scale;
        store8(to + (size_t)n * stride + k, v);
    }
}

// Rows of a product's left operand.  A wavefront takes four blocks of a row, one dword of scales: 16 lanes a block, eight elements a lane.
__global__ __launch_bounds__(256) void rows_kernel(const bf16_t* __restrict__ x, int64_t stride, int K, F8Rows to, int kb, int kg, long long units,
                                                   const int32_t* __restrict__ perm, int k_of, const int32_t* __restrict__ end) {
    const long long unit = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (unit >= units) return;
    const int lane = threadIdx.x & 63;
    const int row = (int)(unit / kg), group = (int)(unit % kg);
    long long from = row;
    if (perm != nullptr) {
        if (row >= *end) return;  // (perm is not set there)
        from = (uint32_t)perm[row] / (uint32_t)k_of;
    }
    const int k = group * 4 * kF8Block + lane * 8;
    float v[8];
    load8(x + from * stride + (k < K ? k : 0), k < K, v);
    uint32_t top = f8_top(v);
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) top = umax(top, (uint32_t)__shfl_xor((int)top, o));
    uint32_t byte = f8_scale_byte(top);
    if (k < kb * kF8Block)
        *reinterpret_cast<uint2*>(to.codes + (size_t)row * to.row_step + (size_t)(k >> 4) * to.piece_step + (k & 8)) = f8_codes(v, f8_inverse(byte));
    byte <<= 8 * (lane >> 4);
    byte |= (uint32_t)__shfl_xor((int)byte, 16);
    byte |= (uint32_t)__shfl_xor((int)byte, 32);
    if (lane == 0) to.scales[(size_t)group * to.rows + row] = byte;
}

}  // namespace

hipError_t launch_f8_rows(const void* x, int64_t stride, int K, const F8Rows& to, const int32_t* perm, int k, const int32_t* end, hipStream_t st) {
    const F8Layout lay = f8_layout(1, K);
    const long long units = (long long)to.rows * lay.kg;
    rows_kernel<<<(unsigned)((units + 3) / 4), 256, 0, st>>>(static_cast<const bf16_t*>(x), stride, K, to, lay.kb, lay.kg, units, perm, k, end);
    return hipGetLastError();
}

hipError_t launch_matrix_pack(int count, int N, int K, int dtype, const void* w, int64_t stride, void* matrix, hipStream_t st) {
    const F8Layout lay = f8_layout(N, K);
    const dim3 grid((unsigned)(lay.nb * lay.kb), (unsigned)count);
    auto run = [&](auto* from) {
        pack_kernel<<<grid, 256, 0, st>>>(from, stride, static_cast<uint8_t*>(matrix), lay, lay.codes(), lay.bytes(), N, K);
        return hipGetLastError();
    };
    return dtype == EMOE_F32 ? run(static_cast<const float*>(w)) : run(static_cast<const bf16_t*>(w));
}

hipError_t launch_matrix_unpack(int count, int N, int K, int dtype, const void* matrix, void* w, int64_t stride, hipStream_t st) {
    const F8Layout lay = f8_layout(N, K);
    const dim3 grid((unsigned)(lay.nb * lay.kb), (unsigned)count);
    auto run = [&](auto* to) {
        unpack_kernel<<<grid, 256, 0, st>>>(static_cast<const uint8_t*>(matrix), to, stride, lay, lay.codes(), lay.bytes(), N, K);
        return hipGetLastError();
    };
    return dtype == EMOE_F32 ? run(static_cast<float*>(w)) : run(static_cast<bf16_t*>(w));
}

}  // namespace emoe
