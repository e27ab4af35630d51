// What the attention kernels share: which tokens a row of queries sees, how the work is cut, the fragments of the matrix
// instructions.
#pragma once
#include "kv_cache.h"

namespace emoe {

// Work that is cut along the keys: pieces leave their outputs (fp32, not divided by the sum), maxima and sums in slots of the workspace, and
// a launch at the end adds them.
constexpr int kFewRows = 16;      // rows of a slot of the kernel for few queries
// Workgroups of it that a CU holds, two slots each, by their registers.  With rows of 64 elements a workgroup has half the bytes on their way: 64 decodes
// of 500 to 8000 tokens on 16 heads 50 us with four, 52 with three; short calls 0 to 3 % the other way.  fp32 of 128: 32 of them to 4000 tokens on 8 heads 26 us
// with two, 28 with three, of which one waits for its place.
constexpr int few_per_cu(int dim, bool bf16) { return dim == 64 && bf16 ? 4 : dim == 64 || bf16 ? 3 : 2; }
constexpr int few_slots(int dim) { return 2 * few_per_cu(dim, true) * kMaxGroups; }
constexpr int kTileRows = 128;    // of the kernel for many
constexpr int kTileSlots = 2 * kMaxGroups;  // as many as run at the same time
struct Piece {
    int token0, row0, rows, kv_head;
    int piece, count;         // the how many-th of how many pieces; count 0: there is none in this slot
    int first, second, step;  // slots of the row's pieces: first, second, second + step, ...
    int pad[3];
};
struct AttentionWs {
    size_t few_records, few_sums, few_outputs;
    size_t tile_count, tile_records, tile_sums, tile_outputs;  // tile_count: slots in use
    size_t total;
};
// Which requests the kernel for few queries takes, by their rows (query tokens times the heads of a kv head): up to `always`, and up to `small` if
// little is gained (few_gain) on all that have more than `always`.  The kernel for many takes the others.
struct FewRule {
    int always, small;
};
hipError_t launch_attention_few(const emoe_kv_desc& d, int dtype, const AttentionArgs& a, FewRule rule, const AttentionWs& ws, int* slots,
                                hipStream_t st);
hipError_t launch_attention_tile(const emoe_kv_desc& d, const AttentionArgs& a, FewRule rule, const AttentionWs& ws, hipStream_t st);

// What the kernel for many queries saves on a request of 33 to 512 rows, in rows of 16 times tokens: it costs 3/2 such rows for a tile of 128
// rows and 1/2 for 32 of them, and starts later.  Below kFewGain for all such requests together the other one is faster (us, few / many queries'
// kernel, 32 heads on 8, requests times rows on tokens: 128 on 4000 19 / 22, on 16000 32 / 26; 512 on 2000 20 / 22, on 4000 31 / 26; 4 times 128 on
// 2000 22 / 25, 256 31 / 30; 16 times 40 on 4000 41 / 55, 64 times 128 / 128; 16 times 512 on 2000 164 / 78).
constexpr long long kFewGain = 500000;
__host__ __device__ constexpr long long few_gain(long long rows, long long seen) {
    return (rows + 15) / 16 * (seen + 256) - (3 * ((rows + 127) / 128) + (rows + 31) / 32) * (seen + 400) / 2;
}

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

constexpr float kLowest = -3.0e38f;  // of a running maximum: finite, so that nothing minus it is a NaN

// A value that all lanes hold alike, in a scalar register: what is computed from it costs no vector instruction, and addresses made of it
// no vector registers.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// An address made of a scalar base and a lane's offset, which a load adds itself if it finds the offset in 32 bits; widened ahead of a loop, as the
// compiler likes to, it takes 64-bit additions of the vector units (a prompt of 2048 tokens 53 us instead of 52).
__device__ __forceinline__ const uint8_t* lane_at(const uint8_t* base, uint32_t offset) {
    asm volatile("" : "+v"(offset));
    return base + offset;
}

// A request's queries and keys, from the lengths on the device, whatever these hold.
struct Request {
    int first;  // its first query's token
    int n;      // query tokens that are answered
    int seq;    // tokens that can be seen, positions 0 .. seq-1
    int len;    // one more than the last one's position: query i stands at len - n + i
};
__device__ __forceinline__ Request request(const AttentionArgs& a, int begin, int end, int len) {
    Request q;
    begin = begin < 0 ? 0 : begin < a.T ? begin : a.T;
    end = end < begin ? begin : end < a.T ? end : a.T;
    q.first = begin;
    q.n = end - begin < a.max_new ? end - begin : a.max_new;
    len = len < 0 ? 0 : len;
    const int most = a.width << a.page.log2_size;
    q.seq = len < most ? len : most;
    q.len = len - (end - begin - q.n);
    return q;
}
__device__ __forceinline__ Request request(const AttentionArgs& a, int r) { return request(a, a.cu_new[r], a.cu_new[r + 1], a.seq_len[r]); }
// r alike in a wavefront: through the scalar cache, for a vector load would wait for all that are on their way
typedef const __attribute__((address_space(4))) int32_t* ScalarInts;
__device__ __forceinline__ Request scalar_request(const AttentionArgs& a, int r) {
    const ScalarInts cu_new = (ScalarInts)(a.cu_new + r), seq_len = (ScalarInts)(a.seq_len + r);
    return request(a, cu_new[0], cu_new[1], seq_len[0]);
}

// The key tiles that queries at positions first .. last see: 0 .. sinks-1 and from .. to-1, the i-th of them.
struct Tiles {
    int sinks, from, to;
    __device__ int count() const { return sinks + (to > from ? to - from : 0); }
    __device__ int tile(int i) const { return i < sinks ? i : i - sinks + from; }
};
__device__ __forceinline__ Request uniform(Request q) { return {uniform(q.first), uniform(q.n), uniform(q.seq), uniform(q.len)}; }
__device__ __forceinline__ Tiles uniform(Tiles t) { return {uniform(t.sinks), uniform(t.from), uniform(t.to)}; }
template <int SIZE>
__device__ __forceinline__ Tiles tiles(const AttentionArgs& a, int seq, int first, int last) {
    Tiles t;
    const int end = last + 1 < seq ? last + 1 : seq;
    t.to = end > 0 ? (end + SIZE - 1) / SIZE : 0;
    t.sinks = t.from = 0;
    if (a.window > 0) {
        const long long lo = (long long)first - a.window + 1;
        t.from = lo > 0 ? (int)(lo / SIZE) : 0;
        const int s = a.sinks < end ? a.sinks : end;
        t.sinks = s > 0 ? (s + SIZE - 1) / SIZE : 0;
        if (t.sinks >= t.from) t.sinks = t.from = 0;  // one piece
    }
    return t;
}

// The most rows of a request that the kernel for few queries takes; every wavefront by itself, alike in both kernels.
__device__ __forceinline__ int few_rows(const AttentionArgs& a, FewRule rule) {
    if (rule.small <= rule.always) return rule.always;
    const int lane = threadIdx.x & 63;
    long long gain = 0;
#pragma unroll 4
    for (int r = lane; r < a.R; r += 64) {
        const Request q = request(a, r);
        const long long rows = (long long)q.n * a.group, reach = (long long)a.window + a.sinks + q.n;
        const long long seen = a.window > 0 && reach < q.seq ? reach : q.seq;
        if (rows > rule.always) gain += few_gain(rows, seen) * a.kv_heads;
    }
    gain = readlane(wave_inclusive(gain), 63);
    return gain <= kFewGain ? rule.small : rule.always;
}

// x over the four lanes that hold one query (lane, lane ^ 16, ^ 32, ^ 48).
template <class F>
__device__ __forceinline__ uint32_t over_groups(uint32_t x, F f) {
    const auto a = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    x = f(a[0], a[1]);
    const auto b = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return f(b[0], b[1]);
}
template <class F>
__device__ __forceinline__ float over_groups(float x, F f) {
    return __uint_as_float(over_groups(__float_as_uint(x), [&](uint32_t x, uint32_t y) {
        return __float_as_uint(f(__uint_as_float(x), __uint_as_float(y)));
    }));
}

// What a lane loads of 16 tokens' keys or values, D / 4 elements of one row: a word holds eight.
template <int D> struct Quarter { typedef uint32_t type __attribute__((ext_vector_type(4))); };
template <> struct Quarter<64> { typedef uint32_t type __attribute__((ext_vector_type(2))); };

// Eight elements of 4 bits as bf16: exact, a code has two significant bits.
__device__ __forceinline__ bf16x8 from_codes(uint32_t codes, float scale) {
    union {
        bf16x2 two[4];
        bf16x8 eight;
    } u;
    u.two[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
    u.two[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
    u.two[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
    u.two[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
    return u.eight;
}

// Eight fp32 numbers as one bf16 operand or, with PIECES 3, as three whose sum is exact to 24 bits.
template <int PIECES>
__device__ __forceinline__ void to_operands(const float* x, bf16x8* out) {
    float rest[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) rest[i] = x[i];
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            out[p][i] = (__bf16)rest[i];
            if (p + 1 < PIECES) rest[i] -= (float)out[p][i];
        }
}

// Eight elements of a bf16 query.  The sign of the scores' scale goes into them.
__device__ __forceinline__ bf16x8 signed_query(const uint4& raw, float scale) {
    const uint32_t sign = scale < 0.0f ? 0x80008000u : 0u;
    return __builtin_bit_cast(bf16x8, uint4{raw.x ^ sign, raw.y ^ sign, raw.z ^ sign, raw.w ^ sign});
}

// Four rows (tokens) of one column (element) from row-major bf16 in LDS: of the 16 lanes of a group, lane j names the eight
// bytes of columns 4 (j % 4) on of row j / 4, and receives column j of the four rows.
__device__ __forceinline__ shortx4 read_transposed(const bf16_t* p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4*)p);
}

__device__ __forceinline__ void store4(float* p, floatx4 v) { *reinterpret_cast<floatx4*>(p) = v; }
__device__ __forceinline__ void store4(bf16_t* p, floatx4 v) { *reinterpret_cast<bf16x4*>(p) = __builtin_convertvector(v, bf16x4); }

}  // namespace
}  // namespace emoe
