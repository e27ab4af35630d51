// Rows of keys and values into the 4-bit cache, and back.
//
// Four lanes hold a block of 32 elements, eight each: one 16-byte load of bf16, the largest magnitude by two steps over the
// lanes (as integers: a NaN is larger than all numbers), a power of two as scale, and the converters of gfx950, whose rounding is to
// nearest even.  With the scale a power of two x / s is exact, so the codes depend on the input alone.  Bound by HBM at
// many tokens: 2 bytes of bf16 in and 17/32 out per element, or the other way round; by the launch at a decode step's.  Measured with
// 8 heads of 128 elements, as replayed graphs: 32768 tokens 36.9 us to write, 35.3 to read, 4.6 and 4.8 TB/s where a large copy reaches 5.1 (with
// the heads of a token in a workgroup 37.6 both; 32 heads of 64: 21.0 and 20.3 us against 23.6 and 25.4); 8192 tokens 9.4 and 8.5, in scattered slots
// 9.7 and 9.3; 64 tokens 2.2 and 2.1.  Two or four pieces a thread, with their loads together, took as long.
#include "kv_cache.h"

namespace emoe {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;

// Eight elements of a row as fp32.
__device__ __forceinline__ void load8(const float* p, float* x) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void load8(const bf16_t* p, float* x) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

// The larger of this lane's value and that of the lane CTRL leads to (quad_perm).
template <int CTRL>
__device__ __forceinline__ uint32_t larger(uint32_t v) {
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
    return v > o ? v : o;
}

// Where a slot's row of one head lies: codes, scales.
struct RowAt {
    size_t codes, scales;
};
__device__ __forceinline__ RowAt row_at(int slot, int head, int kv_heads, KvPage page, bool values, int dim) {
    const int p = slot >> page.log2_size, in_page = slot & ((1 << page.log2_size) - 1);
    const size_t base = ((size_t)p * kv_heads + head) * (size_t)(2 * (page.codes + page.scales));
    return {base + (values ? page.codes : 0) + (size_t)in_page * (dim / 2),
            base + 2 * page.codes + (values ? page.scales : 0) + (size_t)in_page * (dim / kKvBlock)};
}

// The four lanes of a block: their codes, and its scale byte.
__device__ __forceinline__ uint32_t quantise(const float* x, uint32_t* scale_byte) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t a = __float_as_uint(x[j]) & 0x7fffffffu;
        top = a > top ? a : top;
    }
    top = larger<0xB1>(top);  // lanes 1 0 3 2
    top = larger<0x4E>(top);  // lanes 2 3 0 1
    const bool finite = top < 0x7f800000u;
    // amax = 1.m * 2^(e - 127) <= 7 * 2^k = 1.75 * 2^(k + 2)
    int byte = (int)(top >> 23) - 2 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
    byte = byte < 1 ? 1 : byte > (int)kLastScale ? (int)kLastScale : byte;  // no code stands for what passes the range
    byte = finite ? byte : 255;
    const float scale = __uint_as_float((uint32_t)byte << 23);
    uint32_t codes = 0;
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[0], x[1], scale, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[2], x[3], scale, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[4], x[5], scale, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[6], x[7], scale, 3);
    *scale_byte = (uint32_t)byte;
    return finite ? codes : 0u;
}

// A thread: eight elements of a token's keys and the same of its values.  A workgroup: one head of 16 or 32 tokens, so that both sides are whole
// lines where the slots follow each other, with its neighbours at the other heads of these tokens.
struct Thread {
    uint32_t token, head, piece;
};
__device__ __forceinline__ Thread this_thread(int kv_heads, int log_pieces) {
    const uint32_t tokens = blockIdx.x / (uint32_t)kv_heads;
    return {tokens * (kThreads >> log_pieces) + (threadIdx.x >> log_pieces), blockIdx.x - tokens * kv_heads, threadIdx.x & ((1u << log_pieces) - 1)};
}

template <class E>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(const E* __restrict__ k, int64_t k_stride, const E* __restrict__ v,
                                                             int64_t v_stride, const int32_t* __restrict__ slots, uint8_t* __restrict__ cache,
                                                             int T, int kv_heads, int dim, int n_slots, KvPage page) {
    const int log_pieces = dim == 64 ? 3 : 4;
    const auto [t, head, piece] = this_thread(kv_heads, log_pieces);
    if (t >= (uint32_t)T) return;  // alike in the four lanes of a block
    const uint32_t e = (head << log_pieces) + piece;
    const int slot = slots[t];
    float x[2][8];
    load8(k + (int64_t)t * k_stride + e * 8, x[0]);
    load8(v + (int64_t)t * v_stride + e * 8, x[1]);
    if ((unsigned)slot >= (unsigned)n_slots) return;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        uint32_t byte;
        const uint32_t codes = quantise(x[w], &byte);
        const RowAt at = row_at(slot, head, kv_heads, page, w == 1, dim);
        *reinterpret_cast<uint32_t*>(cache + at.codes + piece * 4) = codes;
        if ((piece & 3) == 0) cache[at.scales + piece / 4] = (uint8_t)byte;
    }
}

__device__ __forceinline__ void store8(float* p, uint32_t codes, float scale) {
    floatx2 f[4];
    f[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0);
    f[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1);
    f[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2);
    f[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3);
    reinterpret_cast<float4*>(p)[0] = float4{f[0][0], f[0][1], f[1][0], f[1][1]};
    reinterpret_cast<float4*>(p)[1] = float4{f[2][0], f[2][1], f[3][0], f[3][1]};
}
__device__ __forceinline__ void store8(bf16_t* p, uint32_t codes, float scale) {
    uint4 o;
    o.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
    o.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
    o.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
    o.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
    *reinterpret_cast<uint4*>(p) = o;
}

template <class E>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(const uint8_t* __restrict__ cache, const int32_t* __restrict__ slots,
                                                           E* __restrict__ k, E* __restrict__ v, int T, int kv_heads, int dim, int n_slots,
                                                           KvPage page) {
    const int log_pieces = dim == 64 ? 3 : 4;
    const auto [t, head, piece] = this_thread(kv_heads, log_pieces);
    if (t >= (uint32_t)T) return;
    const size_t i = (((size_t)t * kv_heads + head) << log_pieces) + piece;
    const int slot = slots[t];
    uint32_t codes[2] = {0, 0}, byte[2] = {127, 127};
    if ((unsigned)slot < (unsigned)n_slots) {
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const RowAt at = row_at(slot, head, kv_heads, page, w == 1, dim);
            codes[w] = *reinterpret_cast<const uint32_t*>(cache + at.codes + piece * 4);
            byte[w] = cache[at.scales + piece / 4];
        }
    }
    store8(k + i * 8, codes[0], scale_of_byte(byte[0]));
    store8(v + i * 8, codes[1], scale_of_byte(byte[1]));
}

// At most 2^33 elements (emoe.h), 2048 a workgroup.
unsigned groups_of(const emoe_kv_desc& d, int T) {
    const long long tokens = kThreads * 8 / d.head_dim;
    return (unsigned)((T + tokens - 1) / tokens * d.kv_heads);
}

}  // namespace

hipError_t launch_kv_append(const emoe_kv_desc& d, int T, int dtype, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                            const int32_t* slot, void* cache, hipStream_t st) {
    auto run = [&](auto* kp, auto* vp) {
        kv_append_kernel<<<groups_of(d, T), kThreads, 0, st>>>(kp, k_stride, vp, v_stride, slot, static_cast<uint8_t*>(cache), T, d.kv_heads, d.head_dim,
                                                               d.pages * d.page_size, kv_page(d));
        return hipGetLastError();
    };
    if (dtype == EMOE_F32) return run(static_cast<const float*>(k), static_cast<const float*>(v));
    return run(static_cast<const bf16_t*>(k), static_cast<const bf16_t*>(v));
}

hipError_t launch_kv_read(const emoe_kv_desc& d, int T, int dtype, const void* cache, const int32_t* slot, void* k, void* v,
                          hipStream_t st) {
    auto run = [&](auto* kp, auto* vp) {
        kv_read_kernel<<<groups_of(d, T), kThreads, 0, st>>>(static_cast<const uint8_t*>(cache), slot, kp, vp, T, d.kv_heads, d.head_dim,
                                                             d.pages * d.page_size, kv_page(d));
        return hipGetLastError();
    };
    if (dtype == EMOE_F32) return run(static_cast<float*>(k), static_cast<float*>(v));
    return run(static_cast<bf16_t*>(k), static_cast<bf16_t*>(v));
}

}  // namespace emoe
