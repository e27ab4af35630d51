// Products in 8 bits for few rows a group (a decode step): the cost is reading each matrix that has rows once.
//
// A workgroup (4 wavefronts) owns 128 rows of a matrix - of the SwiGLU product the same 128 rows of both - and all of K, so that it
// has whole blocks of 128 outputs, which is what the activation's result needs to be brought to 8 bits.  The wavefronts take every fourth block
// of 128 columns.  Matrices lie in memory in the order in which the matrix instruction (v_mfma_scale_f32_16x16x128_f8f6f4) wants them, so
// they go from memory to registers and nowhere else, a contiguous KiB a load, and no wavefront waits for another before the end of K.  The matrix's
// rows are the instruction's row operand, 16 tokens its columns; the powers of two are operands of the instruction.
// The four partial sums meet in LDS, added in wavefront order.
//
// The instruction adds the products of eight consecutive elements with what lies 2^-14 below the largest one's power of two cut off, and all else in
// fp32: 1.5e-5 of a sum of random products, a hundredth of the rounding of the result to bf16.  (The bf16 instruction, on exact
// products of the same codes, has half the rate.)
#include "matrix_f8.h"

namespace emoe {
namespace {

typedef int intx8 __attribute__((ext_vector_type(8)));
typedef int intx4 __attribute__((ext_vector_type(4)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ intx8 two(const uint8_t* p, int second) {
    const intx4 a = *reinterpret_cast<const intx4*>(p), b = *reinterpret_cast<const intx4*>(p + second);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

template <int EPI, int TB>
__global__ __launch_bounds__(256) void stream_kernel(F8Product p) {
    constexpr int NB = EPI == kF8Swiglu ? 16 : 8;  // 16-row blocks of a wavefront: 8 of each matrix
    constexpr int NQ = NB / 4;                     // of which each wavefront finishes a quarter
    constexpr int REGION = NQ * TB * 4 * 64;
    __shared__ float red[2][3][REGION];
    __shared__ uint32_t tops[4][16 * TB];

    const int nb = blockIdx.x % p.lay.nb, group = blockIdx.x / p.lay.nb;
    int row0 = 0, row_end = p.rows;
    if (p.offsets != nullptr) {
        row0 = p.offsets[group];
        row_end = p.offsets[group + 1];
        row0 = row0 > 0 ? row0 : 0;
        row_end = row_end < p.rows ? row_end : p.rows;
    }
    if (row_end <= row0) return;  // its matrix is never touched
    const int lane = threadIdx.x & 63, tok = lane & 15, quad = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

    const size_t at = (size_t)group * p.matrix_bytes + (size_t)nb * p.lay.kb * kF8BlockBytes;
    const uint8_t* w0 = p.w0 + at + lane * 16;
    const uint8_t* w1 = EPI == kF8Swiglu ? p.w1 + at + lane * 16 : nullptr;
    const size_t scales_at = (size_t)group * p.matrix_bytes + p.lay.codes() + (size_t)nb * p.lay.kg * 4;
    const uint32_t* s0 = reinterpret_cast<const uint32_t*>(p.w0 + scales_at);
    const uint32_t* s1 = EPI == kF8Swiglu ? reinterpret_cast<const uint32_t*>(p.w1 + scales_at) : nullptr;
    const int steps = (p.lay.kb - wave + 3) / 4;  // this wavefront's blocks of columns: wave, wave + 4, ...

    for (int tok0 = row0; tok0 < row_end; tok0 += 16 * TB) {
        const uint8_t* x[TB];
        const uint32_t* xs[TB];
#pragma unroll
        for (int t = 0; t < TB; ++t) {
            int r = tok0 + 16 * t + tok;
            r = r < row_end ? r : row_end - 1;  // (rows past the end are multiplied and not stored)
            if (p.perm != nullptr) r = (int)((uint32_t)p.perm[r] / (uint32_t)p.k);
            x[t] = p.x.codes + (size_t)r * p.x.stride + quad * 16;
            xs[t] = p.x.scales + r;
        }
        floatx4 acc[NB][TB];
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int t = 0; t < TB; ++t) acc[i][t] = floatx4{0, 0, 0, 0};

        intx8 w[NB], xf[TB];
        uint32_t xb[TB], b0 = 0, b1 = 0;
        auto load_w = [&](int i, int s) {
            const uint8_t* base = (i < 8 ? w0 : w1) + (size_t)(4 * s + wave) * kF8BlockBytes + (i & 7) * kF8Strip;
            w[i] = two(base, 1024);
        };
        auto load_x = [&](int s) {
#pragma unroll
            for (int t = 0; t < TB; ++t) {
                xf[t] = two(x[t] + (size_t)(4 * s + wave) * kF8Block, 64);
                xb[t] = xs[t][(size_t)s * p.x.rows] >> (8 * wave);
            }
            b0 = s0[s] >> (8 * wave);
            if (EPI == kF8Swiglu) b1 = s1[s] >> (8 * wave);
        };
        if (steps > 0) {
            load_x(0);
#pragma unroll
            for (int i = 0; i < NB; ++i) load_w(i, 0);
        }
        for (int s = 0; s < steps; ++s) {
            intx8 xc[TB];
            uint32_t xbc[TB];
            const uint32_t b0c = b0, b1c = b1;
#pragma unroll
            for (int t = 0; t < TB; ++t) { xc[t] = xf[t]; xbc[t] = xb[t]; }
            const int next = s + 1 < steps ? s + 1 : s;  // (the last step's once more, and unused)
            load_x(next);
#pragma unroll
            for (int i = 0; i < NB; ++i) {
#pragma unroll
                for (int t = 0; t < TB; ++t)
                    acc[i][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w[i], xc[t], acc[i][t], 0, 0, 0, (int)(i < 8 ? b0c : b1c), 0,
                                                                                 (int)xbc[t]);
                load_w(i, next);
            }
        }

        // ---- the four partial sums; wavefront q finishes rows 32 q .. 32 q + 31 of the 128 (of each matrix) -----------------
        floatx4 sum[NQ][TB];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float(*to)[REGION] = red[q & 1];
            auto block = [&](int j) { return j < 2 ? 2 * q + j : 8 + 2 * q + j - 2; };
            if (wave != q) {
                float* mine = to[wave < q ? wave : wave - 1] + lane;
#pragma unroll
                for (int j = 0; j < NQ; ++j)
#pragma unroll
                    for (int t = 0; t < TB; ++t)
#pragma unroll
                        for (int v = 0; v < 4; ++v) mine[((j * TB + t) * 4 + v) * 64] = acc[block(j)][t][v];
            }
            __syncthreads();
            if (wave == q) {
#pragma unroll
                for (int j = 0; j < NQ; ++j)
#pragma unroll
                    for (int t = 0; t < TB; ++t)
#pragma unroll
                        for (int v = 0; v < 4; ++v) {
                            float s = 0.0f;
#pragma unroll
                            for (int o = 0; o < 4; ++o)
                                s += o == q ? acc[block(j)][t][v] : to[o < q ? o : o - 1][lane + ((j * TB + t) * 4 + v) * 64];
                            sum[j][t][v] = s;
                        }
            }
        }

        // a lane holds token tok and outputs 4 quad .. 4 quad + 3 of two blocks of 16
        const int n0 = nb * kF8Block + wave * 32 + quad * 4;
        if constexpr (EPI == kF8Plain) {
#pragma unroll
            for (int t = 0; t < TB; ++t) {
                const int r = tok0 + 16 * t + tok;
                if (r >= row_end) continue;
                bf16_t* to = p.out + (size_t)(p.out_perm != nullptr ? p.out_perm[r] : r) * p.out_stride;
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    if (n0 + 16 * j < p.N) *reinterpret_cast<bf16x4*>(to + n0 + 16 * j) = __builtin_convertvector(sum[j][t], bf16x4);
            }
        } else {
#pragma unroll
            for (int t = 0; t < TB; ++t) {
                uint32_t top = 0;
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        float g = sum[j][t][v];
                        if constexpr (EPI == kF8Swiglu) g = g / (1.0f + __expf(-g)) * sum[2 + j][t][v];
                        else g = g < 0.0f ? 0.0f : g;  // (NaN stays)
                        sum[j][t][v] = g;
                        top = umax(top, f8_magnitude(g));
                    }
                top = umax(top, (uint32_t)__shfl_xor((int)top, 16));
                top = umax(top, (uint32_t)__shfl_xor((int)top, 32));
                if (quad == 0) tops[wave][16 * t + tok] = top;
            }
            __syncthreads();
#pragma unroll
            for (int t = 0; t < TB; ++t) {
                const int r = tok0 + 16 * t + tok, c = 16 * t + tok;
                const uint32_t byte = f8_scale_byte(umax(umax(tops[0][c], tops[1][c]), umax(tops[2][c], tops[3][c])));
                if (r >= row_end) continue;
                const float inverse = f8_inverse(byte);
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    *reinterpret_cast<uint32_t*>(p.h.codes + (size_t)r * p.h.stride + n0 + 16 * j) =
                        f8_codes(sum[j][t][0], sum[j][t][1], sum[j][t][2], sum[j][t][3], inverse);
                if (wave == 0 && quad == 0) reinterpret_cast<uint8_t*>(p.h.scales + (size_t)(nb >> 2) * p.h.rows + r)[nb & 3] = (uint8_t)byte;
            }
        }
        __syncthreads();  // red and tops are free again
    }
}

template <int EPI>
hipError_t launch(const F8Product& p, hipStream_t st) {
    const unsigned grid = (unsigned)(p.groups * p.lay.nb);
    const long long rows = (p.rows + p.groups - 1) / p.groups;
    if (p.rows <= 16 || rows <= 8) stream_kernel<EPI, 1><<<grid, 256, 0, st>>>(p);
    else if (rows <= 22) stream_kernel<EPI, 2><<<grid, 256, 0, st>>>(p);
    else stream_kernel<EPI, 4><<<grid, 256, 0, st>>>(p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_f8_stream(const F8Product& p, F8Epilogue epilogue, hipStream_t st) {
    switch (epilogue) {
        case kF8Swiglu: return launch<kF8Swiglu>(p, st);
        case kF8Relu: return launch<kF8Relu>(p, st);
        default: return launch<kF8Plain>(p, st);
    }
}

}  // namespace emoe
