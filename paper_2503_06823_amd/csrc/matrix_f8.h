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
// Blocks of a row of h up to which elements near ties of two codes are summed again (see kNearTie), by tiles and by streaming
constexpr int kTieBlocksTiled = 5, kTieBlocks = 20;
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
    uint16_t* near;  // (tiles) which elements of h are near ties of two codes, [lay.nb][2][rows][4], see near_ties_kernel
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
// K tiles (blocks of columns) from which leftover tiles are cut into pieces: the pieces' sums and the launch that adds them cost as much as some 24 of them.
// Cut / not, us: 8 blocks 39.4 / 27.3 (2048 rows times 4096 x 1024); 11 57.7 / 48.2 (24 groups of 300 rows times 2048 x 1408); 16 82.4 / 84.2, 39.8 / 31.8; 23 101.2 /
// 99.4; 25 49.9 / 48.8 (1024 rows times 6144 x 3200), 57.2 / 52.0 (2048 times 4096 x 3200); 26 46.7 / 49.4 (2100 times 1040 x 3208); 32 56.3 / 58.3 (1024 times
// 6144 x 4096), 63.6 / 62.1, 106.5 / 112.8 (5120 times 4096 x 4096), of experts 177.9 / 173.0; 112 1186 / 1227 (4096 tokens' experts of 14336).
constexpr int kF8LeastCut = 24;
// partials: f8_partial_bytes(p.lay.kb).  x by rows; at least two blocks of columns.
inline size_t f8_partial_bytes(int kb) { return kb >= kF8LeastCut ? kTiledPartialBytes : kTiledPlanBytes; }
hipError_t launch_f8_tiled(const F8Product& p, F8Epilogue epilogue, float* partials, hipStream_t st);
hipError_t launch_f8_ties(const F8Product& p, F8Epilogue epilogue, float* partials, hipStream_t st);  // (its part for activations into short rows of h)

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

// ---- elements of h near a tie of two codes ------------------------------------------------------------------------------
// The matrix cores' sums are 1e-5 to 5e-5 off (see matmul_f8_stream.hip), a thousandth of a code's step, and of an element that near a tie of two codes
// they decide which of the two it gets.  Of the elements that are large in their block (128 and more, of up to 448) the codes are up to an eighth of the
// element apart: where such an element is most of its row of h, an output row changes by as much (1368 tokens, d 1216, f 200: one row 9 %, all outputs 5.8e-3;
// with those elements summed again 0.8 % and 2.5e-3).  So a large element within kNearTie of a tie that matters to its row, its step being more than 1 / 16 of it,
// gets its sums once more, products exact and added in fp32, and the code of these, whichever kernel makes h.  (1e-4 to 3e-4 of all elements are near ties.)
// Where blocks share a power, a step is at most 1 / 16 of rows of more than five blocks (a block's largest element is 224 or more under its power, a step 32), and a
// code on the other side of a tie changes them by no more than the rounding of each of their elements to four bits.  So tiles look for such elements in rows of up to
// five blocks, at 10 us a call (16384 rows of d 1216, f 200 78 -> 88; 6000 of f 640, ReLU, 56 -> 66), and streaming, where few rows are much of a call's result, up to
// 20 (64 tokens' 24 experts of f 1408 63.3 -> 65.1, 500 tokens' of f 512 32.4 -> 36.1, 1368 of f 200 44.4 -> 49.0; beyond, 64 tokens' of f 14336 190 -> 203).
// Tiles up to 20 blocks: 8192 tokens' 24 experts of f 1408 472 -> 505 us; of any length: 4096 tokens' of 14336 1172 -> 1215.
// A call takes longer for it with such elements: a microsecond or two of a half or whole wavefront each, which is felt where most rows have many.
// What is left: one in some 100 sums of large elements is off by more than kNearTie (2e-4 to 1e-4 of the element, where terms of the sum cancel); smaller elements
// have what the matrix cores say, a step of theirs being at most a thirtieth of the block's largest.
constexpr uint32_t kNearTie = 1573;  // 0.0015 steps, a step being 2^20 of a float's last places
// near * 2 + whether a number under its block's factor is one of them.  Codes have three places after the point: a tie is where the other 20 say one half, from
// 136 on, the first of the large ones; smaller numbers leave bit 30.  (By signs: a comparison would take scalar registers, and two wait states.)
__device__ __forceinline__ uint32_t f8_near_ties(uint32_t near, float scaled) {
    const uint32_t over = __float_as_uint(scaled) - (0x43080000u - kNearTie);
    return __builtin_amdgcn_alignbit(near, (over & 0x400fffffu) - 2 * kNearTie, 31);
}

// 16 products of codes, exact, and their sum
__device__ __forceinline__ float f8_dot16(uint4 a, uint4 b) {
    const int u[4] = {(int)a.x, (int)a.y, (int)a.z, (int)a.w}, v[4] = {(int)b.x, (int)b.y, (int)b.z, (int)b.w};
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        sum = fmaf(__builtin_amdgcn_cvt_f32_fp8(u[i], 0), __builtin_amdgcn_cvt_f32_fp8(v[i], 0), sum);
        sum = fmaf(__builtin_amdgcn_cvt_f32_fp8(u[i], 1), __builtin_amdgcn_cvt_f32_fp8(v[i], 1), sum);
        sum = fmaf(__builtin_amdgcn_cvt_f32_fp8(u[i], 2), __builtin_amdgcn_cvt_f32_fp8(v[i], 2), sum);
        sum = fmaf(__builtin_amdgcn_cvt_f32_fp8(u[i], 3), __builtin_amdgcn_cvt_f32_fp8(v[i], 3), sum);
    }
    return sum;
}
// A row of x in 8 bits: its pieces of 16 codes and its powers
struct F8RowInMemory {
    const uint8_t* codes;
    const uint8_t* powers;
    size_t piece_step, fours_step;  // bytes from a piece to the next; from four powers to the next four
    __device__ F8RowInMemory(const F8Rows& x, size_t row)
        : codes(x.codes + row * x.row_step), powers(reinterpret_cast<const uint8_t*>(x.scales + row)), piece_step(x.piece_step), fours_step((size_t)x.rows * 4) {}
    __device__ uint4 piece(int q) const { return *reinterpret_cast<const uint4*>(codes + q * piece_step); }
    __device__ int power(int b) const { return powers[(b >> 2) * fours_step + (b & 3)]; }
};
// Element n of h for row x, by LANES lanes that stand together: a lane takes pieces lane, lane + LANES, ...  M: 2 for SwiGLU, 1 for ReLU.
template <int M, int LANES, class Row>
__device__ __forceinline__ float f8_h(const F8Layout& lay, const uint8_t* const (&matrix)[M], int n, const Row& x) {
    const size_t w_at = (size_t)(n >> 7) * lay.kb * kF8BlockBytes + ((n >> 4) & 7) * kF8Strip + (n & 15) * 16;
    const size_t power_at = lay.codes() + (size_t)(n >> 7) * lay.kg * 4;
    constexpr int AHEAD = 4;  // a lane's pieces on their way together
    const int pieces = lay.kb * 8;
    float sum[M] = {};
    for (int q0 = threadIdx.x & (LANES - 1); q0 < pieces; q0 += AHEAD * LANES) {
        uint4 xc[AHEAD], wc[M][AHEAD];
        int power[M][AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int q = q0 + i * LANES < pieces ? q0 + i * LANES : q0, b = q >> 3;
            xc[i] = x.piece(q);
            const int x_power = x.power(b);
#pragma unroll
            for (int m = 0; m < M; ++m) {
                wc[m][i] = *reinterpret_cast<const uint4*>(matrix[m] + w_at + (size_t)b * kF8BlockBytes + ((q >> 2) & 1) * 1024 + (q & 3) * 256);
                power[m][i] = x_power + matrix[m][power_at + b];
            }
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
#pragma unroll
            for (int m = 0; m < M; ++m) sum[m] += q0 + i * LANES < pieces ? ldexpf(f8_dot16(wc[m][i], xc[i]), power[m][i] - 254) : 0.0f;
    }
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1)
#pragma unroll
        for (int m = 0; m < M; ++m) sum[m] += __shfl_xor(sum[m], o);
    if constexpr (M == 2) return sum[0] / (1.0f + __expf(-sum[0])) * sum[M - 1];
    else return sum[0] < 0.0f ? 0.0f : sum[0];
}
#endif

}  // namespace emoe
