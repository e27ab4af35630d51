// Attention over the paged 4-bit cache for requests of few queries: a decode step, one token a request.
//
//   S^T = K Q^T,  P^T = exp2(S^T - max),  O^T += V^T P^T,  with one pass over the keys and values, the running maximum and sum.
//
// Bound by reading the cache once: 2 * D * 17/32 bytes a token and kv head, against 4 * D flop for each of the heads that share
// it.  A workgroup has 16 rows (query token, query head) of one kv head, padded, and a piece of the request's keys;
// its four wavefronts take tiles of 32 tokens in turn, each with a maximum, a sum and an output of its own, so that nothing waits in
// the walk; they meet once, at its end.  The matrix instructions' token and element orders are free as long as both operands
// agree, and are chosen so that no data moves between lanes but V's:
//   - K becomes bf16 in registers, which is exact, and so are its products with bf16 queries; fp32 queries and weights are three bf16 operands each,
//     exact to fp32.  Lane (row = lane % 16, group = lane / 16) holds D / 4 consecutive elements of one token's key, which lie in one
//     block; step s multiplies its eight elements s, of all groups, with q's.  The scaled matrix instructions, which take K in 4 bits, want q in 8:
//     two such numbers under a scale lose what a channel has 2^-14 below the largest, and are no faster (64 decodes 68.6 us either way, 1024 of 20 to
//     600 tokens 84 with bf16, 91 with them).
//   - Weights of bf16 calls are rounded to bf16: one product instead of three, with the bits that the result keeps.
//   - P^T comes out of S^T in the registers in which the second product wants it: lane (query, group) holds tokens 4 group .. +3
//     of each 16, and V's rows are taken in that order.
//   - V: converted to bf16 where its scale is one per lane, through LDS (a wavefront's own), read back transposed.
//
// Split: all rows' key tiles make one line, of which every workgroup that the chip holds takes an equal part (Stretch).  A row that is cut
// leaves its pieces (fp32 output, maximum, sum) in the workspace, and a second launch adds them in the pieces' order.  A workgroup has two
// slots there: the piece that its share ends in is the first of its row, the one that it begins in is not.
//
// Keys and values are loaded in the order of memory: 16 bytes a lane at the stride of a token's row took an L1 access a lane.  What is alike in
// a wavefront is held in scalar registers (page numbers, addresses): in vector registers it took 16 of them and half the
// instructions, and the lookup of a page waited for the tiles on their way.
//
// Measured (32 heads on 8 of 128 elements; with the sum of pieces): 64 requests of 500 to 16383 tokens 68 to 71 us (322 MB), one of 131072 37 to 39
// (143 MB), 32 behind windows of 4096 31 to 32 (116 MB).  The walk itself reads 6.1 to 6.9 TB/s, where a plain read stream reaches 6.9; the
// same launches without the walk take 15 us (20 with 64 requests: more beginnings): two launches 4, from the lengths to the first tiles
// 5, the end of a stretch 3, the sum of pieces 3.  All three wavefronts of a SIMD together spend 1.5 us of instructions on a round of
// tiles that memory brings in 1.9.  A fourth wavefront a SIMD, and V's fragments read before
// the exponentials, brought nothing.
#include <math.h>

#include "kv_attention.h"

namespace emoe {
namespace {

constexpr int kTok = 32;      // tokens of a tile
constexpr int kRows = kFewRows;  // of a workgroup
constexpr int kLogWaves = 2, kWaves = 1 << kLogWaves;
// See Stretch.
constexpr int kFixed = 2;       // units that a stretch's beginning and end take time for
constexpr int kLeastUnits = 3;  // of a workgroup's share
constexpr int kSnap = 1;
constexpr float kLazy = 8.0f;   // log2 of what a weight may grow to before the maximum is taken up

template <class E> struct Pieces { static constexpr int n = 1; };
template <> struct Pieces<float> { static constexpr int n = 3; };

// The work as one line of units: requests in order, of a request its kv heads, of a head its tiles of 16 rows, of those (a stretch) kFixed
// units for its beginning and end and then the rounds of key tiles that the longest row sees, at least one.  Every workgroup takes an
// equal part of the line, so that all of them end together whatever the lengths; a boundary within kSnap rounds of a stretch's beginning or
// end moves there, or nothing would be left whole.  A round is kWaves << shift tiles: more than one a wavefront only where the line would not
// fit 31 bits.
struct Stretch {
    int row_tiles;  // of a request
    int rounds;     // of one of its stretches
    __device__ int all(int kv_heads) const { return row_tiles * kv_heads * (kFixed + rounds); }
};
__device__ __forceinline__ Stretch stretch(const AttentionArgs& a, const Request& q, int most_rows, int shift) {
    const int rows = q.n * a.group;
    if (rows == 0 || rows > most_rows) return {0, 0};
    const int n = (tiles<kTok>(a, q.seq, q.len - q.n, q.len - 1).count() + (kWaves << shift) - 1) >> shift >> kLogWaves;
    return {(int)((uint32_t)(rows + kRows - 1) / kRows), n > 0 ? n : 1};
}

// total units in `groups` shares, the first `longer` of them one unit longer.
struct Shares {
    int total, each, longer, groups;
    __device__ __forceinline__ int begin(int w) const { return w * each + (w < longer ? w : longer); }
    __device__ __forceinline__ int owner(int u) const {
        const int of_longer = longer * (each + 1);
        return u < of_longer ? (uint32_t)u / (uint32_t)(each + 1) : longer + (uint32_t)(u - of_longer) / (uint32_t)each;
    }
};

// The shares, and the request in which this workgroup's begins; every wavefront by itself.  A lane sums R / 64 requests that follow each other,
// whose lengths come together; those of the lane in which the share begins are then summed one by one.  (64 requests a trip, twice: 1024 decodes of
// 20 to 600 tokens 104 us.)
struct Start {
    Shares shares;
    int r;
    int before;  // units of the requests before r
    Request request;
    Stretch stretch;
};
__device__ __forceinline__ bool find_start(const AttentionArgs& a, int most_rows, int shift, Start* s) {
    const int lane = threadIdx.x & 63, per_lane = (a.R + 63) / 64;
    Request mine;
    Stretch its;
    auto units_of = [&](int r) {
        mine = {0, 0, 0, 0};
        if (r < a.R) mine = request(a, r);
        its = stretch(a, mine, most_rows, shift);
        return its.all(a.kv_heads);
    };
    long long all = 0;
#pragma unroll 4
    for (int j = 0; j < per_lane; ++j) all += units_of(lane * per_lane + j);
    all = wave_inclusive(all);
    if (readlane(all, 63) > 0x7fffffff) return false;  // there are more queries than T: cu_new is not a list of offsets
    int upto = (int)all;
    const int total = __builtin_amdgcn_readlane(upto, 63);
    const int most = (uint32_t)(total + kLeastUnits - 1) / kLeastUnits;
    s->shares.total = total;
    s->shares.groups = most < (int)gridDim.x ? most : (int)gridDim.x;
    if ((int)blockIdx.x >= s->shares.groups) return false;
    s->shares.each = (uint32_t)total / (uint32_t)s->shares.groups;
    s->shares.longer = total - s->shares.each * s->shares.groups;
    const int begin = s->shares.begin(blockIdx.x);
    int at = __builtin_ctzll(__ballot(upto > begin));
    s->before = at > 0 ? __builtin_amdgcn_readlane(upto, at - 1) : 0;
    s->r = at;
    if (per_lane > 1) {
        const int first = at * per_lane, end = first + per_lane;
        for (int r0 = first;; r0 += 64) {
            const int r = r0 + lane;
            upto = (int)wave_inclusive((long long)units_of(r < end ? r : a.R));
            const int sum = __builtin_amdgcn_readlane(upto, 63);
            if (begin - s->before < sum || r0 + 64 >= end) {
                at = __builtin_ctzll(__ballot(upto > begin - s->before) | 1ull << 63);
                if (at > 0) s->before += __builtin_amdgcn_readlane(upto, at - 1);
                s->r = r0 + at;
                break;
            }
            s->before += sum;
        }
    }
    s->request = {__builtin_amdgcn_readlane(mine.first, at), __builtin_amdgcn_readlane(mine.n, at), __builtin_amdgcn_readlane(mine.seq, at),
                  __builtin_amdgcn_readlane(mine.len, at)};
    s->stretch = {__builtin_amdgcn_readlane(its.row_tiles, at), __builtin_amdgcn_readlane(its.rounds, at)};
    return true;
}

// ONE_PAGE: pages of kTok tokens or more, so that a tile lies in one and takes one lookup (decodes 1 % faster, with rows of 64 elements 4).
template <class E, int D, bool ONE_PAGE>
__global__ __launch_bounds__(64 * kWaves, few_per_cu(D, sizeof(E) == 2)) void attention_few_kernel(AttentionArgs a, FewRule rule, int shift, AttentionWs lay) {
    constexpr int PIECES = Pieces<E>::n, STEPS = D / 32, BLOCKS = D / 16;
    constexpr int V_STRIDE = D + 16;  // elements; 32 bytes past the row: 16 rows of 32 bytes fall on all banks alike
    constexpr int V_BYTES = kTok * V_STRIDE * 2, WAVE_BYTES = V_BYTES + kTok * D / 2;  // V as bf16, K as it comes
    static_assert(WAVE_BYTES % 16 == 0 && BLOCKS * 1024 <= WAVE_BYTES, "the outputs take V's place at the end");
    __shared__ __align__(16) char lds[kWaves * WAVE_BYTES];
    __shared__ float sums[kWaves][kRows][2];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int col = lane & 15, group = lane >> 4;

    const int most_rows = uniform(few_rows(a, rule));
    Start start;
    const bool some = find_start(a, most_rows, shift, &start);
    Piece* records = reinterpret_cast<Piece*>(a.ws + lay.few_records) + 2 * (size_t)blockIdx.x;
    bool used[2] = {false, false};
    const int share_end = some ? start.shares.begin(blockIdx.x + 1) : 0;
    int r = uniform(start.r), before = start.before;
    Request q = start.request;
    Stretch here = start.stretch;
    for (int unit = some ? start.shares.begin(blockIdx.x) : 0; unit < share_end;) {
        if (unit - before >= here.all(a.kv_heads)) {
            before += here.all(a.kv_heads);
            q = scalar_request(a, ++r);
            here = stretch(a, q, most_rows, shift);
            continue;
        }
        const int rounds = uniform(here.rounds), units = kFixed + rounds, nth = uniform((uint32_t)(unit - before) / (uint32_t)units);
        const int first_unit = before + nth * units;
        const int snap = kSnap < rounds / 2 ? kSnap : rounds / 2;
        auto round_at = [&](int u) {
            const int k = u - first_unit < units ? u - first_unit - kFixed : rounds;
            return uniform(k <= snap ? 0 : k >= rounds - snap ? rounds : k);
        };
        const int u_begin = round_at(unit), u_end = round_at(share_end);
        unit = first_unit + units;
        if (u_begin >= u_end) continue;
        const int kv_head = uniform((uint32_t)nth / (uint32_t)here.row_tiles), row_tile = nth - kv_head * here.row_tiles;
        const int rows = q.n * a.group, row0 = row_tile * kRows, last_row = row0 + kRows < rows ? row0 + kRows - 1 : rows - 1;
        const int p_first = q.len - q.n + a.token_of(row0), p_last = q.len - q.n + a.token_of(last_row);

        const int row = row0 + col, token = a.token_of(row), head = kv_head * a.group + row - token * a.group;
        const int position = row < rows ? q.len - q.n + token : -1;  // -1 sees nothing

        const E* q_at = static_cast<const E*>(a.q) + (int64_t)(q.first + token) * a.q_stride + (int64_t)head * D;
        bf16x8 query[PIECES][STEPS];
        if constexpr (PIECES == 1) {  // sent for before the first tiles are
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                uint4 raw = {0, 0, 0, 0};
                if (row < rows) raw = *reinterpret_cast<const uint4*>(q_at + group * (D / 4) + 8 * s);
                query[0][s] = __builtin_bit_cast(bf16x8, raw);
            }
        }

        const Tiles seen = uniform(tiles<kTok>(a, q.seq, q.len - q.n, q.len - 1));
        const int i_begin = u_begin * (kWaves << shift), i_all = seen.count();
        int i_end = u_end < rounds ? u_end * (kWaves << shift) : i_all;
        // What is added to the maximum, so that all weights together are below 1 and outputs no larger than the values: of at most 2^lift / 2^kLazy tokens.
        const float lift = kLazy + 5.0f + (float)(32 - __builtin_clz((uint32_t)(i_end > i_begin ? i_end - i_begin : 1)));
        while (i_end > 0 && seen.tile(i_end - 1) * kTok > p_last) --i_end;  // no row of this tile sees so far
        const ScalarInts table = (ScalarInts)(a.table + (size_t)r * a.width);
        const int page_mask = (1 << a.page.log2_size) - 1;
        const uint32_t head_bytes = (uint32_t)a.page.bytes(), page_stride = head_bytes * (uint32_t)a.kv_heads;
        const uint8_t* cache = a.cache + (size_t)kv_head * head_bytes;
        bf16_t* v_lds = reinterpret_cast<bf16_t*>(lds + wave * WAVE_BYTES);
        char* k_lds = lds + wave * WAVE_BYTES + V_BYTES;

        // Both are loaded in the order of memory, quarter lane % 4 of token lane / 4 (16 bytes a lane at a stride of 64 took an access of the
        // L1 cache per lane).  Keys go through LDS, where quarter q of token t lies in place q ^ swizzle(t), to lane (token, quarter).
        const int in_tok = lane >> 2, quarter = lane & 3;
        const uint32_t in_at = in_tok * (D / 2) + quarter * (D / 8), v_scale_at = in_tok * (D / 32) + quarter * (D / 4) / 32;
        const uint32_t k_scale_at = col * (D / 32) + group * (D / 4) / 32;
        auto swizzle = [](int t) { return (t >> (D == 128 ? 2 : 3)) & 3; };
        char* k_to = k_lds + in_tok * (D / 2) + (quarter ^ swizzle(in_tok)) * (D / 8);
        const char* k_from = k_lds + col * (D / 2) + (group ^ swizzle(col)) * (D / 8);
        bf16_t* v_to = v_lds + in_tok * V_STRIDE + quarter * (D / 4);
        const bf16_t* v_from = v_lds + (4 * group + (col >> 2)) * V_STRIDE + 4 * (col & 3);

        // Where a tile's two halves of 16 tokens lie: codes and scales of their keys.  Pages of nobody are read as page 0, and masked.
        struct Place {
            const uint8_t *codes0, *codes1, *scales0, *scales1;
            int t0;
            bool owned0, owned1;
        };
        auto place = [&](int i) {
            Place p;
            p.t0 = seen.tile(i) * kTok;
            auto half = [&](int t, const uint8_t*& codes, const uint8_t*& scales, bool& owned) {
                const int b = t >> a.page.log2_size, in_page = t & page_mask;
                const uint32_t page = (uint32_t)table[b < a.width ? b : a.width - 1];
                owned = page < (uint32_t)a.pages && b < a.width;
                const uint8_t* head = cache + (uint64_t)(owned ? page : 0u) * page_stride;
                codes = head + in_page * (D / 2);
                scales = head + 2 * a.page.codes + in_page * (D / 32);
            };
            half(p.t0, p.codes0, p.scales0, p.owned0);
            if constexpr (ONE_PAGE) {
                p.codes1 = p.codes0 + 16 * (D / 2);
                p.scales1 = p.scales0 + 16 * (D / 32);
                p.owned1 = p.owned0;
            } else {
                half(p.t0 + 16, p.codes1, p.scales1, p.owned1);
            }
            return p;
        };
        typedef typename Quarter<D>::type Words;
        Words k0, k1, v0, v1;
        uint32_t k_scale0, k_scale1, v_scale0, v_scale1;
        auto load_keys = [&](const Place& p) {
            k0 = *reinterpret_cast<const Words*>(lane_at(p.codes0, in_at));
            k1 = *reinterpret_cast<const Words*>(lane_at(p.codes1, in_at));
            k_scale0 = *lane_at(p.scales0, k_scale_at);
            k_scale1 = *lane_at(p.scales1, k_scale_at);
        };
        auto load_values = [&](const Place& p) {
            v0 = *reinterpret_cast<const Words*>(lane_at(p.codes0 + a.page.codes, in_at));
            v1 = *reinterpret_cast<const Words*>(lane_at(p.codes1 + a.page.codes, in_at));
            v_scale0 = *lane_at(p.scales0 + a.page.scales, v_scale_at);
            v_scale1 = *lane_at(p.scales1 + a.page.scales, v_scale_at);
        };

        floatx4 out[BLOCKS];
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) out[b] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
        float most = kLowest, sum = 0.0f;
        uint32_t bad = 0;  // quarters of this lane's query that a block of NaN values among its tokens has reached

        // Tile i + 4's values and keys are on their way from where tile i's have been used on, and its page is looked up a tile earlier.  The first
        // tile's are sent for before the queries are.
        int i = i_begin + wave;
        const int last = i_end - 1;  // past the end: the last tile again, unused
        Place now, next;
        if (i < i_end) {
            now = place(i);
            load_values(now);
            load_keys(now);
            next = place(i + kWaves < i_end ? i + kWaves : last);
        }
        // Scores are compared before they are scaled: the scale is positive, its sign goes into q.  A scale of zero becomes next to nothing, so
        // that it does not meet an infinity.
        const float scale = fmaxf(fabsf(a.scale_log2), 1e-37f);
        if constexpr (PIECES == 1) {
#pragma unroll
            for (int s = 0; s < STEPS; ++s) query[0][s] = signed_query(__builtin_bit_cast(uint4, query[0][s]), a.scale_log2);
        } else {
            float x[8];
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = 0.0f;
                if (row < rows) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = q_at[group * (D / 4) + s * 8 + i] * (a.scale_log2 < 0.0f ? -1.0f : 1.0f);
                }
                bf16x8 o[PIECES];
                to_operands<PIECES>(x, o);
#pragma unroll
                for (int p = 0; p < PIECES; ++p) query[p][s] = o[p];
            }
        }

        for (; i < i_end; i += kWaves) {
            const Place after = place(i + 2 * kWaves < i_end ? i + 2 * kWaves : last);
            const int t0 = now.t0;
            // every row sees every token of the tile
            const bool whole = now.owned0 & now.owned1 & (t0 + kTok - 1 <= p_first) &
                               ((a.window == 0) | (t0 > p_last - a.window) | (t0 + kTok <= a.sinks));
            if (!whole) {  // what was never written: any number will do
                if (!(t0 + in_tok < q.seq && now.owned0)) v_scale0 = 127;
                if (!(t0 + 16 + in_tok < q.seq && now.owned1)) v_scale1 = 127;
            }
            const unsigned long long nan0 = __ballot(v_scale0 > kLastScale), nan1 = __ballot(v_scale1 > kLastScale);
            auto write_values = [&](const Words& words, uint32_t byte, bf16_t* to) {
                const float scale = scale_of_byte(byte > kLastScale ? 127 : byte);
#pragma unroll
                for (int e = 0; e < D / 32; ++e) *reinterpret_cast<bf16x8*>(to + 8 * e) = from_codes(words[e], scale);
            };
            write_values(v0, v_scale0, v_to);
            write_values(v1, v_scale1, v_to + 16 * V_STRIDE);
            load_values(next);
            *reinterpret_cast<Words*>(k_to) = k0;
            *reinterpret_cast<Words*>(k_to + 16 * D / 2) = k1;
            const float scale0 = scale_of_byte(k_scale0), scale1 = scale_of_byte(k_scale1);
            load_keys(next);
            auto scores = [&](const char* from, float by) {
                const Words words = *reinterpret_cast<const Words*>(from);
                floatx4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int st = 0; st < STEPS; ++st) {
                    const bf16x8 key = from_codes(words[st], by);
#pragma unroll
                    for (int p = PIECES - 1; p >= 0; --p) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key, query[p][st], s, 0, 0, 0);
                }
                return s;
            };
            const floatx4 z0 = scores(k_from, scale0), z1 = scores(k_from + 16 * D / 2, scale1);
            float z[8] = {z0[0], z0[1], z0[2], z0[3], z1[0], z1[1], z1[2], z1[3]};
            if (!whole) {
                const int from = a.window > 0 && position >= a.window ? position - a.window + 1 : 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int j = t0 + 16 * (e / 4) + 4 * group + e % 4;
                    const bool sees = (j <= position) & ((j >= from) | (j < a.sinks)) & (e < 4 ? now.owned0 : now.owned1);
                    z[e] = sees ? z[e] : -INFINITY;
                }
            }
            if ((nan0 | nan1) != 0) {
                // bit 4 t + quarter of nan0: the value of token t is none, or may be infinite.  V holds numbers there; what sees it becomes NaN at the end
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    bad |= z[e] != -INFINITY ? (uint32_t)((e < 4 ? nan0 : nan1) >> (16 * group + 4 * (e % 4))) & 15u : 0u;
            }
            float top = z[0];
#pragma unroll
            for (int e = 1; e < 8; ++e) top = fmaxf(top, z[e]);
            top = over_groups(top, [](float x, float y) { return fmaxf(x, y); }) * scale;
            if (__any(top > most + (kLazy - lift))) {  // the weights stay below 2^8 of the first ones: a maximum that rises by less is not worth a pass over the output
                const float up = fmaxf(most, top + lift), f = __builtin_amdgcn_exp2f(most - up);
                most = up;
                sum *= f;
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b) out[b] *= f;
            }
            float w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = __builtin_amdgcn_exp2f(fmaf(z[e], scale, -most));
            bf16x8 weight[PIECES];
            to_operands<PIECES>(w, weight);
            if constexpr (PIECES == 1) {  // as they are multiplied with: what rounding does to all alike is divided out
                union {
                    bf16x8 all;
                    bf16x2 two[4];
                } u;
                u.all = weight[0];
                const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
                for (int e = 0; e < 4; ++e) sum = __builtin_amdgcn_fdot2_f32_bf16(u.two[e], ones, sum, false);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += w[e];
            }
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                union {
                    shortx4 half[2];
                    bf16x8 all;
                } f;
                f.half[0] = read_transposed(v_from + 16 * b);
                f.half[1] = read_transposed(v_from + 16 * V_STRIDE + 16 * b);
#pragma unroll
                for (int p = PIECES - 1; p >= 0; --p) out[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.all, weight[p], out[b], 0, 0, 0);
            }
            now = next;
            next = after;
        }

        // the four wavefronts' outputs, to the largest of their maxima
        sum = over_groups(sum, [](float x, float y) { return x + y; });
        if (__any(bad != 0)) {
            bad |= (uint32_t)__shfl_xor((int)bad, 16);
            bad |= (uint32_t)__shfl_xor((int)bad, 32);
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b)
                if (bad >> (b * 16 / (D / 4)) & 1u) out[b] = floatx4{NAN, NAN, NAN, NAN};
        }
        floatx4* part = reinterpret_cast<floatx4*>(lds);
        constexpr int WAVE_PARTS = WAVE_BYTES / 16;
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) part[wave * WAVE_PARTS + b * 64 + lane] = out[b];
        if (group == 0) {
            sums[wave][col][0] = most;
            sums[wave][col][1] = sum;
        }
        __syncthreads();
        float top = kLowest, all = 0.0f, factor[kWaves];
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sums[w][col][0]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            factor[w] = __builtin_amdgcn_exp2f(sums[w][col][0] - top);
            all += sums[w][col][1] * factor[w];
        }
        const bool cut = u_begin > 0 || u_end < rounds;
        const int which = u_begin == 0 ? 1 : 0;
        const size_t slot = 2 * (size_t)blockIdx.x + which;
#pragma unroll
        for (int n = 0; n < BLOCKS / kWaves; ++n) {
            const int b = wave * (BLOCKS / kWaves) + n;
            floatx4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < kWaves; ++w) v += part[w * WAVE_PARTS + b * 64 + lane] * factor[w];
            const int d = 16 * b + 4 * group;
            if (row >= rows) continue;
            if (cut) {
                float* to = reinterpret_cast<float*>(a.ws + lay.few_outputs) + (slot * kRows + col) * D + d;
                *reinterpret_cast<floatx4*>(to) = v;
            } else {
                const float by = all == 0.0f ? 0.0f : 1.0f / all;
                store4(static_cast<E*>(a.out) + (int64_t)(q.first + token) * a.out_stride + (int64_t)head * D + d, v * by);
            }
        }
        if (cut) {
            used[which] = true;
            if (wave == 0 && group == 0) {
                float* to = reinterpret_cast<float*>(a.ws + lay.few_sums) + (slot * kRows + col) * 2;
                to[0] = top;
                to[1] = all;
                if (col == 0) {
                    // whose share holds a unit, boundaries as they are after snapping
                    const int w0 = start.shares.owner(first_unit + kFixed + snap), w1 = start.shares.owner(first_unit + units - snap - 1);
                    records[which] = Piece{q.first, row0, rows - row0 < kRows ? rows - row0 : kRows, kv_head, (int)blockIdx.x - w0, w1 - w0 + 1,
                                           2 * w0 + 1, 2 * (w0 + 1), 2, {}};
                }
            }
        }
        __syncthreads();  // the outputs are read: the next stretch's tiles may take their place
    }
    if (threadIdx.x == 0) {
        if (!used[0]) records[0].count = 0;
        if (!used[1]) records[1].count = 0;
    }
}

}  // namespace

// *slots: of the workspace that can hold a piece.
hipError_t launch_attention_few(const emoe_kv_desc& d, int dtype, const AttentionArgs& a, FewRule rule, const AttentionWs& ws, int* slots,
                                hipStream_t st) {
    DeviceShape shape;
    hipError_t e = device_shape(&shape);
    if (e != hipSuccess) return e;
    // As many workgroups as the chip holds at once, or as many as there can be shares for, by the tokens and the requests.
    const int most_rows = rule.always > rule.small ? rule.always : rule.small;
    const long long rows = (long long)a.max_new * a.group < most_rows ? (long long)a.max_new * a.group : most_rows;
    const long long per_request = (rows + kRows - 1) / kRows, by_tokens = (long long)a.T * a.group / kRows + a.R;
    const long long row_tiles = per_request * a.R < by_tokens ? per_request * a.R : by_tokens;
    // A round's tiles are doubled until a stretch has no more rounds than leave the line in 31 bits (row tiles of all heads: below 2^25).
    const long long stretches = row_tiles * a.kv_heads, most_tiles = (((long long)a.width << a.page.log2_size) + kTok - 1) / kTok;
    int shift = 0;
    auto rounds_of = [&] { return ((most_tiles - 1) >> shift >> kLogWaves) + 1; };
    while (rounds_of() > 1 && stretches * (kFixed + rounds_of()) > 0x7fffffff - kLeastUnits) ++shift;
    const long long most_rounds = rounds_of(), line = stretches * (kFixed + most_rounds), shares = (line + kLeastUnits - 1) / kLeastUnits;
    const int at_once = few_per_cu(d.head_dim, dtype == EMOE_BF16) * shape.groups, groups = shares < at_once ? (int)shares : at_once;
    *slots = most_rounds > 2 * kSnap + 1 ? 2 * groups : 0;  // none if no stretch is long enough to be cut
    auto run = [&](auto element, auto dim) {
        auto* kernel = d.page_size >= kTok ? attention_few_kernel<decltype(element), decltype(dim)::value, true>
                                           : attention_few_kernel<decltype(element), decltype(dim)::value, false>;
        kernel<<<(unsigned)groups, 64 * kWaves, 0, st>>>(a, rule, shift, ws);
        return hipGetLastError();
    };
    if (dtype == EMOE_F32)
        return d.head_dim == 64 ? run(float(), std::integral_constant<int, 64>()) : run(float(), std::integral_constant<int, 128>());
    return d.head_dim == 64 ? run(bf16_t(), std::integral_constant<int, 64>()) : run(bf16_t(), std::integral_constant<int, 128>());
}

}  // namespace emoe
