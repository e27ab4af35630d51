// Matrices in 8 bits: how they lie in memory, the conversion, and the launchers of what works with them.
#pragma once
#include "common.h"

namespace emoe {

constexpr int kF8Block = 128;                          // rows and columns that share a power of two; of a row of x or h, elements
constexpr int kF8BlockBytes = kF8Block * kF8Block;     // of a block's codes
constexpr int kF8Strip = 16 * kF8Block;                // of 16 rows of a block: what one matrix instruction multiplies

// A packed matrix [N][K] (see emoe.h): codes [nb][kb][8][2][64][16], then scale bytes [nb][4 kg].
struct F8Layout {
    int nb, kb, kg;  // blocks of rows, of columns, and those in fours (a dword of scales)
    __host__ __device__ size_t codes() const { return (size_t)nb * kb * kF8BlockBytes; }
    __host__ __device__ size_t bytes() const { return codes() + (((size_t)nb * kg * 4 + 255) & ~(size_t)255); }
};
inline F8Layout f8_layout(int N, int K) {
    const int nb = (N + kF8Block - 1) / kF8Block, kb = (K + kF8Block - 1) / kF8Block;
    return {nb, kb, (kb + 3) / 4};
}

// Rows in 8 bits: codes, in pieces of 16 in one of two orders, and scales [kg][rows], a dword for four blocks of 128 elements.
// By rows, [rows][kb 8][16], as tiles are brought to LDS; by pieces, [kb 8][rows][16], where a matrix instruction's operand goes from
// memory to registers: neighbouring lanes, which hold neighbouring rows, then read neighbouring bytes (64 rows times 6144 x 4096: 15.3 us
// by rows, where each lane of a load has a line of its own, 12.5 by pieces).
struct F8Rows {
    uint8_t* codes;
    uint32_t* scales;
    int rows;
    int row_step, piece_step;  // bytes from a row to the next, and from a piece of a row to the next
};
inline size_t f8_rows_scale_bytes(long long rows, int K) { return (size_t)rows * f8_layout(1, K).kg * 4; }

// The product of grouped rows with their group's matrix (offsets NULL: one group of all rows), and what becomes of it:
// plain: bf16 rows of out; SwiGLU, ReLU: the activation's result as rows in 8 bits, h.
enum F8Epilogue { kF8Plain = 0, kF8Swiglu = 1, kF8Relu = 2 };
struct F8Product {
    F8Rows x;
    const int32_t* perm;  // (tiles, and `from`) grouped row r is row perm[r] / k of x; NULL: r
    int k;
    const int32_t* offsets;
    int groups;
    int rows;  // grouped rows, those behind the last group included
    const uint8_t* w0;
    const uint8_t* w1;  // SwiGLU: the other factor's matrices
    F8Layout lay;       // of a matrix
    size_t matrix_bytes;
    int N;
    bf16_t* out;
    int64_t out_stride;
    const int32_t* out_perm;  // row r is stored as row out_perm[r]; NULL: r
    F8Rows h;
    const bf16_t* from;  // (streaming) NULL, or the rows themselves, x not being there: workgroups convert them
    int64_t from_stride;
    int K;
};
// Whether streaming converts the rows itself, every workgroup all of its own: what a launch costs, against work that each repeats.  Measured in a graph
// (us, converted by the workgroups / by a launch before): 6144 x 4096, 1 row 7.5 / 9.7, 4 rows 9.2 / 9.9; 6144 x 1024, 16 rows 6.8 / 6.8; 4096 x 14336, 1 row
// 13.4 / 15.9; 16 rows of 16 groups of 2816 x 1024 10.7 / 13.3; one token's experts of 14336 x 4096 60.2 / 62.9.
constexpr int kF8OwnBlocks = 128;
inline bool f8_own_rows(long long rows, int K) { return rows <= 16 && rows * f8_layout(1, K).kb <= kF8OwnBlocks; }

// Row r of `to` is row r of x, or with perm row perm[r] / k; of these only the rows before *end.
hipError_t launch_f8_rows(const void* x, int64_t stride, int K, const F8Rows& to, const int32_t* perm, int k, const int32_t* end, hipStream_t st);
// x by pieces, a row of it for each grouped row; or `from`
hipError_t launch_f8_stream(const F8Product& p, F8Epilogue epilogue, hipStream_t st);
// partials: kTiledPartialBytes.  x by rows; at least two blocks of columns.
hipError_t launch_f8_tiled(const F8Product& p, F8Epilogue epilogue, float* partials, hipStream_t st);

hipError_t launch_matrix_pack(int count, int N, int K, int dtype, const void* w, int64_t stride, void* matrix, hipStream_t st);
hipError_t launch_matrix_unpack(int count, int N, int K, int dtype, const void* matrix, void* w, int64_t stride, hipStream_t st);

// The layer's calls with dtype EMOE_F8.
int validate_f8_layer(const emoe_layer_desc& d);  // what the limits of rows and matrices in whole blocks add to validate_desc()
size_t ffn_f8_ws_bytes(const emoe_layer_desc& d);
size_t f8_matrix_bytes(int N, int K);
hipError_t launch_ffn_f8(const emoe_layer_desc& d, const void* x_perm, RowGather gather, const int32_t* offsets, const void* w1,
                         const void* w3, const void* w2, void* y_perm, void* ws, int passes, hipStream_t st);

#ifdef __HIPCC__
// The scale byte (exponent + 127) of a block whose largest magnitude has the bits `top`: the smallest 2^e >= 2^-126 with top <= 448 * 2^e =
// 1.75 * 2^(e + 8), 2^119 if that is less (the numbers stay finite); 255, NaN, if the block holds an infinity or a NaN (whose bits are the largest).
__device__ __forceinline__ uint32_t f8_scale_byte(uint32_t top) {
    if (top >= 0x7f800000u) return 255u;
    const int byte = (int)((top + 0x1fffffu) >> 23) - 8;  // (carries where the mantissa is above 1.75)
    return (uint32_t)(byte < 1 ? 1 : byte > 246 ? 246 : byte);
}
// 1 / 2^e as a factor, exact; anything for 255
__device__ __forceinline__ float f8_inverse(uint32_t byte) { return __uint_as_float((254u - (byte & 0xffu)) << 23); }
// Four numbers under a block's factor to codes: the nearest, ties to the even code, 448 beyond (under 2^119 only)
__device__ __forceinline__ uint32_t f8_codes(float a, float b, float c, float d, float inverse) {
    auto in = [&](float v) { return __builtin_amdgcn_fmed3f(v * inverse, -448.0f, 448.0f); };
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(in(a), in(b), 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(in(c), in(d), w, true);
    return (uint32_t)w;
}
__device__ __forceinline__ uint32_t f8_magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }
// The same of eight at once
__device__ __forceinline__ void f8_widened(uint4 bf16s, float (&v)[8]) {
    const uint32_t w[4] = {bf16s.x, bf16s.y, bf16s.z, bf16s.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint32_t f8_top(const float (&v)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = umax(m, f8_magnitude(v[i]));
    return m;
}
__device__ __forceinline__ uint2 f8_codes(const float (&v)[8], float inverse) {
    return make_uint2(f8_codes(v[0], v[1], v[2], v[3], inverse), f8_codes(v[4], v[5], v[6], v[7], inverse));
}
#endif

}  // namespace emoe
