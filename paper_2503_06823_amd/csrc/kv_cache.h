// The paged 4-bit cache of keys and values: layout, and what its kernels share.
#pragma once
#include "common.h"

namespace emoe {

constexpr int kKvBlock = 32;                        // elements that share a scale
constexpr uint32_t kLastScale = 252;                // largest scale byte whose codes all fit in fp32 and bf16: 6 * 2^125
constexpr size_t kAttentionWsBytes = 64ull << 20;   // no call needs more

// Host-side checks; EMOE_OK or an error.
int validate_kv_desc(const emoe_kv_desc* d);
int validate_attention(const emoe_kv_desc* d, const emoe_attention_desc* a);

inline int log2_of(int v) {
    int n = 0;
    while ((1 << n) < v) ++n;
    return n;
}

// Bytes of one head's part of a page, and where its sections begin.
struct KvPage {
    int log2_size;   // tokens
    int codes;       // bytes of the codes of its keys, and of its values
    int scales;      // the same of the scales
    __host__ __device__ int bytes() const { return 2 * (codes + scales); }
};
inline KvPage kv_page(const emoe_kv_desc& d) {
    return {log2_of(d.page_size), d.page_size * d.head_dim / 2, d.page_size * d.head_dim / kKvBlock};
}

// A scale byte as the factor that the converters take: they look at the exponent alone; 255 becomes a NaN.
__device__ __forceinline__ float scale_of_byte(uint32_t b) { return __uint_as_float(__umul24(b, 0x808000u)); }

// Inclusive prefix sum of 64 lanes' values, by DPP: two instructions a step and half instead of two trips to LDS.
__device__ __forceinline__ long long wave_inclusive(long long v) {
#define EMOE_SCAN_STEP(ctrl, rows)                                                                                   \
    {                                                                                                                \
        const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, ctrl, rows, 0xf, false);         \
        const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(v >> 32), ctrl, rows, 0xf, false);           \
        v += (long long)((uint64_t)hi << 32 | lo);                                                                   \
    }
    EMOE_SCAN_STEP(0x111, 0xf)  // row_shr 1, 2, 4, 8
    EMOE_SCAN_STEP(0x112, 0xf)
    EMOE_SCAN_STEP(0x114, 0xf)
    EMOE_SCAN_STEP(0x118, 0xf)
    EMOE_SCAN_STEP(0x142, 0xa)  // row_bcast 15 to rows 1 and 3, 31 to rows 2 and 3
    EMOE_SCAN_STEP(0x143, 0xc)
#undef EMOE_SCAN_STEP
    return v;
}
__device__ __forceinline__ long long readlane(long long v, int lane) {
    const int lo = __builtin_amdgcn_readlane((int)v, lane), hi = __builtin_amdgcn_readlane((int)(v >> 32), lane);
    return ((long long)hi << 32) | (uint32_t)lo;
}

// The largest of a wavefront's values >= 0, in all lanes.
__device__ __forceinline__ int wave_top(int v) {
#define EMOE_TOP_STEP(ctrl, rows)                                                    \
    {                                                                                \
        const int o = __builtin_amdgcn_update_dpp(0, v, ctrl, rows, 0xf, false);      \
        v = o > v ? o : v;                                                           \
    }
    EMOE_TOP_STEP(0x111, 0xf)
    EMOE_TOP_STEP(0x112, 0xf)
    EMOE_TOP_STEP(0x114, 0xf)
    EMOE_TOP_STEP(0x118, 0xf)
    EMOE_TOP_STEP(0x142, 0xa)
    EMOE_TOP_STEP(0x143, 0xc)
#undef EMOE_TOP_STEP
    return __builtin_amdgcn_readlane(v, 63);
}

hipError_t launch_kv_plan(const emoe_kv_desc& d, int T, const int32_t* len, const int32_t* new_len, int32_t* table,
                          const int32_t* free_pages, const int64_t* counters, int32_t* cu_new, int32_t* slot, int32_t* position,
                          int32_t* seq_len, int64_t* counters_out, int32_t* refused, hipStream_t st);
hipError_t launch_kv_release(const emoe_kv_desc& d, const int32_t* len_before, const int32_t* len, const int32_t* ended, int window,
                             int sinks, const int32_t* table, int32_t* free_pages, const int64_t* counters, int64_t* counters_out,
                             hipStream_t st);
hipError_t launch_kv_advance(const emoe_kv_desc& d, const int32_t* seq_len, const int32_t* ended, int32_t* len, hipStream_t st);
hipError_t launch_kv_append(const emoe_kv_desc& d, int T, int dtype, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                            const int32_t* slot, void* cache, hipStream_t st);
hipError_t launch_kv_read(const emoe_kv_desc& d, int T, int dtype, const void* cache, const int32_t* slot, void* k, void* v,
                          hipStream_t st);

// What the attention kernels are told.
struct AttentionArgs {
    const void* q;
    const uint8_t* cache;
    const int32_t* table;
    const int32_t* seq_len;
    const int32_t* cu_new;
    void* out;
    uint8_t* ws;
    int64_t q_stride, out_stride;
    float scale_log2;  // scale * log2(e): the exponentials are powers of two
    int T, R, max_new, q_heads, kv_heads, group, width, pages, window, sinks;
    KvPage page;
    uint32_t group_inverse;
    int group_shift;

    // row / group of a row below 2^27: the inverse is too large by less than 2^-27 of itself
    void set_group(int heads) {
        group = heads;
        for (group_shift = 0; 1 << group_shift < heads; ++group_shift) {}
        group_inverse = (uint32_t)(((1ull << (27 + group_shift)) + heads - 1) / heads) << 4;
    }
    __device__ __forceinline__ int token_of(int row) const { return (int)(__umulhi(2u * (uint32_t)row, group_inverse) >> group_shift); }
};
size_t attention_ws_bytes(const emoe_kv_desc& d, const emoe_attention_desc& a);
hipError_t launch_attention(const emoe_kv_desc& d, const emoe_attention_desc& a, const AttentionArgs& args, hipStream_t st);

}  // namespace emoe
