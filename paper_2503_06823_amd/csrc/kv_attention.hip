// Attention over the paged 4-bit cache: which kernel takes which requests, the workspace, and the sum of pieces.
#include "kv_attention.h"

namespace emoe {
namespace {

// The pieces of rows that were cut, in the pieces' order.  A workgroup for every piece; those of one cut take its rows in turn.  A team of
// lanes has four elements of a row each; where there are many pieces all teams share a row's, so that those of a long context are read side by
// side, else every team has a row of its own.  Bound by its launch and two dependent reads: 4.8 us after 64 decodes, 5.4 after one long
// one (96 pieces a row), 9 after two prompts of 512 tokens next to 14 decodes (25 MB of pieces).  More rows or pieces in flight a team, and 128 or 512
// threads, took as long or longer.
constexpr int kJoinThreads = 256;
constexpr int kOneTeam = 8;  // pieces that a team adds alone
constexpr float kRoom = 10.0f;   // log2 of more pieces than there are: their sum is no larger than the values
constexpr int kTileJoiners = 2;  // workgroups of a piece of the kernel for many, which has eight times the rows
template <class E, int D>
__global__ __launch_bounds__(kJoinThreads) void attention_join_kernel(AttentionArgs a, AttentionWs lay, int few_slots) {
    constexpr int LANES = D / 4, TEAMS = kJoinThreads / LANES;
    __shared__ floatx4 part[TEAMS][LANES];
    __shared__ float2 part_sums[TEAMS];
    const bool few = (int)blockIdx.x < few_slots;
    const int of_tiles = (int)blockIdx.x - few_slots, rows = few ? kFewRows : kTileRows;
    const int slot = few ? blockIdx.x : of_tiles / kTileJoiners, joiner = few ? 0 : of_tiles % kTileJoiners, joiners = few ? 1 : kTileJoiners;
    if (!few && slot >= *reinterpret_cast<const int*>(a.ws + lay.tile_count)) return;
    const Piece p = reinterpret_cast<const Piece*>(a.ws + (few ? lay.few_records : lay.tile_records))[slot];
    if (p.count == 0) return;
    auto row_of = [&](int n, int row) { return (size_t)(n == 0 ? p.first : p.second + (n - 1) * p.step) * rows + row; };
    const float2* sums = reinterpret_cast<const float2*>(a.ws + (few ? lay.few_sums : lay.tile_sums));
    const float* outputs = reinterpret_cast<const float*>(a.ws + (few ? lay.few_outputs : lay.tile_outputs));
    const int lane = threadIdx.x % LANES, team = threadIdx.x / LANES;
    const int shares = p.count > kOneTeam ? TEAMS : 1;  // teams of a row
    const int share = team % shares, side = team / shares, step = p.count * (TEAMS / shares);
    for (int row0 = p.piece + joiner * step; row0 < p.rows; row0 += step * joiners) {
        const int row = row0 + side * p.count;
        floatx4 v = {0.0f, 0.0f, 0.0f, 0.0f};
        float top = kLowest, all = 0.0f;
        if (row < p.rows) {
#pragma unroll 4
            for (int n = share; n < p.count; n += shares) {  // one pass: nothing is loaded that waits for another load but the record
                const size_t at = row_of(n, row);
                const float2 s = sums[at];
                const floatx4 o = *reinterpret_cast<const floatx4*>(outputs + at * D + 4 * lane);
                const float up = fmaxf(top, s.x), f = __builtin_amdgcn_exp2f(top - up), g = __builtin_amdgcn_exp2f(s.x - up - kRoom);
                top = up;
                all = all * f + s.y * g;
                v = v * f + o * g;
            }
        }
        if (shares > 1) {
            part[team][lane] = v;
            if (lane == 0) part_sums[team] = float2{top, all};
            __syncthreads();
            if (share == 0) {
                for (int s = 1; s < TEAMS; ++s) top = fmaxf(top, part_sums[s].x);
                v = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
                all = 0.0f;
                for (int s = 0; s < TEAMS; ++s) {
                    const float f = __builtin_amdgcn_exp2f(part_sums[s].x - top);
                    all += part_sums[s].y * f;
                    v += part[s][lane] * f;
                }
            }
            __syncthreads();  // the sums are read
        }
        if (share == 0 && row < p.rows) {
            const int m = p.row0 + row, token = a.token_of(m);
            const float by = all == 0.0f ? 0.0f : 1.0f / all;
            store4(static_cast<E*>(a.out) + (int64_t)(p.token0 + token) * a.out_stride +
                       (int64_t)(p.kv_head * a.group + m - token * a.group) * D + 4 * lane, v * by);
        }
    }
}

size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

AttentionWs attention_ws(int dim, bool tiles) {
    AttentionWs w;
    w.few_records = 0;
    const size_t slots = few_slots(dim);
    w.few_sums = align256(slots * sizeof(Piece));
    w.few_outputs = align256(w.few_sums + slots * kFewRows * 8);
    w.tile_count = align256(w.few_outputs + slots * kFewRows * dim * 4);
    w.tile_records = w.tile_count + 256;
    w.tile_sums = align256(w.tile_records + kTileSlots * sizeof(Piece));
    w.tile_outputs = align256(w.tile_sums + (size_t)kTileSlots * kTileRows * 8);
    w.total = tiles ? align256(w.tile_outputs + (size_t)kTileSlots * kTileRows * dim * 4) : w.tile_count;
    return w;
}

// Requests of up to this many rows go to the kernel for few queries always, of up to the other where little is gained.
constexpr int kAlwaysFewRows = 32, kSmallFewRows = 512;

// The tile kernel is for bf16: fp32 queries would take three times the matrix work and registers there, and are for verification.  A gain that is
// small at the table's full width is small: it is at most 9/16 of the rows of 16 times what they see.
bool with_tiles(const emoe_kv_desc& d, const emoe_attention_desc& a) {
    const long long rows = (long long)a.max_new * (a.q_heads / d.kv_heads);
    if (a.dtype != EMOE_BF16 || rows <= kAlwaysFewRows) return false;
    const long long row_tiles = ((long long)a.T * a.q_heads / d.kv_heads + 15) / 16 + d.rows;  // at most, of 16 rows
    return rows > kSmallFewRows || row_tiles * d.kv_heads * ((long long)d.table_width * d.page_size + 256) / 16 * 9 > kFewGain;
}

}  // namespace

size_t attention_ws_bytes(const emoe_kv_desc& d, const emoe_attention_desc& a) {
    return attention_ws(d.head_dim, with_tiles(d, a)).total;
}

hipError_t launch_attention(const emoe_kv_desc& d, const emoe_attention_desc& at, const AttentionArgs& a, hipStream_t st) {
    // Lengths are on the device: both kernels are launched unless the host knows that one will find nothing.
    const bool tiles = with_tiles(d, at);
    FewRule rule = {0x7fffffff, 0};
    bool few = true;
    if (tiles) {
        const bool large = (long long)a.T * a.q_heads / 128 * few_gain(128, 0) > kFewGain;  // if all the tokens are there, whatever they see
        rule = {kAlwaysFewRows, large ? 0 : kSmallFewRows};
        if (a.R == 1 && (large || a.max_new * (long long)a.group > kSmallFewRows)) {  // one request, which goes there whatever it brings
            rule = {0, 0};
            few = false;
        }
    }
    const AttentionWs ws = attention_ws(d.head_dim, tiles);
    static_assert(few_slots(64) / 2 <= 1 << (int)kRoom && few_slots(128) / 2 <= 1 << (int)kRoom, "a piece a workgroup");
    static_assert((size_t)few_slots(64) * (sizeof(Piece) + kFewRows * (8 + 128 * 4)) + (size_t)kTileSlots * (sizeof(Piece) + kTileRows * (8 + 128 * 4)) +
                          8 * 256 <= kAttentionWsBytes, "as include/emoe.h promises");
    int few_slots = 0;
    if (tiles) {
        hipError_t e = launch_attention_tile(d, a, rule, ws, st);
        if (e != hipSuccess) return e;
    }
    if (few) {
        hipError_t e = launch_attention_few(d, at.dtype, a, rule, ws, &few_slots, st);
        if (e != hipSuccess) return e;
    }
    const int groups = few_slots + (tiles ? kTileSlots * kTileJoiners : 0);
    if (groups == 0) return hipSuccess;
    auto join = [&](auto element, auto dim) {
        attention_join_kernel<decltype(element), decltype(dim)::value><<<(unsigned)groups, kJoinThreads, 0, st>>>(a, ws, few_slots);
        return hipGetLastError();
    };
    if (at.dtype == EMOE_F32)
        return d.head_dim == 64 ? join(float(), std::integral_constant<int, 64>()) : join(float(), std::integral_constant<int, 128>());
    return d.head_dim == 64 ? join(bf16_t(), std::integral_constant<int, 64>()) : join(bf16_t(), std::integral_constant<int, 128>());
}

}  // namespace emoe
