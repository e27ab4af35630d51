// Attention over the paged 4-bit cache for bf16 requests of many queries: prompts, and pieces of them.
//
//   S^T = K Q^T,  P^T = exp2(S^T - max),  O^T += V^T P^T,  one pass over the keys and values, as for few queries.
//
// Bound by the matrix cores (4 * D flop a query, head and visible token), next to them by the exponentials and by LDS.  A workgroup
// has 128 rows (query token, query head) of one kv head, 32 a wavefront, and walks the keys in tiles of 64; two workgroups share a
// CU, so that one's exponentials run under the other's products.
//   - K and V are converted to bf16, exactly, once for the workgroup on their way into LDS; V is read back transposed.  K in 4 bits on the scaled
//     matrix instructions takes a quarter of its LDS bytes and no conversion (a prompt of 8192 tokens 474 us instead of 528), but wants q in 8
//     bits: two such numbers under a scale lose what a channel has 2^-14 below the largest, and scores far more than that where keys are weak in the large
//     channels.
//   - P^T comes out of S^T in the registers in which the second product wants it, rounded to bf16: one product, with the bits that the result keeps.
// The tile after the next is on its way from memory while a tile is multiplied, the next one is written to the other half of LDS under the
// scores' products; one barrier a tile.
//
// Split: a workgroup takes a row tile's keys whole, the longest first, where there are enough row tiles; else pieces of them (find_job), which
// leave fp32 outputs, maxima and sums in the workspace for a second launch to add.
//
// Measured: a prompt of 8192 tokens (32 heads on 8 of 128 elements) 515 to 525 us, 1.05 to 1.07 PFLOP/s of what the mask leaves.  The matrix cores are
// busy for 49 % of the cycles, the vector units for 45 % and LDS for 46 %, the first two hardly at the same time.  Prompts of 512, 1024, 2048 and 4096
// tokens: 20, 30, 51 and 150 us (2048: 56 if the last of two row tiles for a CU does not go with the first).  Tried with K in 4 bits: scores of the
// next tile ahead of this one's exponentials (519 us against 504 then), a third wavefront a SIMD (633: it spilled); a higher priority in the products
// changed nothing.
#include <math.h>

#include "kv_attention.h"

namespace emoe {
namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));

constexpr int kTok = 64;    // tokens of a tile
constexpr int kRows = kTileRows;
constexpr int kWaves = 4;
// Of a lane's weights, before the maximum is looked for again: a row's two lanes have 1 together, so that its outputs are no larger than the values.
constexpr float kMostSum = 0.5f;
constexpr float kLift = 16.0f;  // log2 of what the largest weight then is below 1: contexts of 2^15 tokens before their sum alone asks for it

// A request's row tiles, the key tiles that all its queries see together, which are those of its longest row tile but for a window, and those of its
// first row tile.
struct Rows {
    int row_tiles, longest, shortest;
};
__device__ __forceinline__ Rows rows_of(const AttentionArgs& a, const Request& q, int least_rows) {
    const long long rows = (long long)q.n * a.group;
    if (rows == 0 || rows < least_rows) return {0, 0, 0};
    const int n = (int)((rows + kRows - 1) / kRows);
    const int p0 = q.len - q.n, first = kRows / a.group < q.n ? kRows / a.group : q.n;
    const int whole = tiles<kTok>(a, q.seq, p0, q.len - 1).count(), start = tiles<kTok>(a, q.seq, p0, p0 + first - 1).count();
    return {n, whole > 0 ? whole : 1, start > 0 ? start : 1};
}

// A piece of work: a row tile, and the how many-th of its pieces of `each` key tiles.
struct Job {
    int r, row_tile, kv_head, piece, pieces, each, slot, all_slots;
    bool found;
    Request q;
};

// How row tiles are cut: so that the work is over soonest, in the time that a lone workgroup of a CU takes for a key tile.  Two on a CU take
// kTwo times as long as one (one's products and the other's exponentials hardly overlap).  Whole row tiles take the longest one's tiles, or a CU's share
// of all of them if that is more.  Else the longest is divided by 2 to 64, an estimate a lane: pieces of c tiles take c if every CU has one at
// most, kTwo c if it has two, and if there are more the longer of c and a CU's share, kUneven for what is not even and kBegin for a second beginning; a
// piece of a row tile that is cut needs a slot, costs 64 KiB (of 64 elements: 32) written and read again, a tile's time for kPerTile of them, and kCut
// for the first.  The constants were fitted at 128 elements.
// Every wavefront by itself, 64 requests a trip.
constexpr float kTwo = 1.65f, kCut = 3.0f, kPerTile = 43.0f, kUneven = 1.1f, kBegin = 3.0f;
constexpr int kLeastCut = 6;  // key tiles
constexpr int kAhead = 4;     // times 64 requests' lengths come together
// Workgroups beyond the places and the row tiles, for pieces of a row tile that is longer than all others: four prompts of 512 tokens on 100 to 8000
// take 117 us with them, 169 without.  As they take some 1 us where none is cut, and more where each reads many lengths, only for few requests.
__device__ __host__ __forceinline__ int extra_places(const AttentionArgs& a, int places) { return a.R <= 64 ? places / 4 : 0; }
// Requests come in the order of their longest row tiles where they are at most 64 with rows for this kernel (else as they are): `list` holds those of
// this wavefront.
__device__ __forceinline__ Job find_job(const AttentionArgs& a, int least_rows, int places, int want, bool to_the_end, int* list) {
    const int lane = threadIdx.x & 63;
    Request mine;
    Rows rows;
    int id;
    auto lengths = [&](int r) { return r < a.R ? request(a, r) : Request{0, 0, 0, 0}; };
    auto take = [&](int r, const Request& q) {
        id = r;
        mine = q;
        rows = rows_of(a, q, least_rows);
    };
    int longest = 0, active = 0;
    long long work = 0, row_tiles = 0;  // work: twice the key tiles of all
    auto add = [&] {
        longest = rows.longest > longest ? rows.longest : longest;
        work += (long long)rows.row_tiles * (rows.longest + rows.shortest);
        row_tiles += rows.row_tiles;
        const unsigned long long some = __ballot(rows.row_tiles > 0);
        if (a.R > 64 && rows.row_tiles > 0) {
            const int at = active + __builtin_popcountll(some & ((1ull << lane) - 1));
            if (at < 64) list[at] = id;
        }
        active += __builtin_popcountll(some);
    };
    if (a.R <= 64) {
        take(lane, lengths(lane));
        add();
    } else {
        for (int r0 = 0; r0 < a.R; r0 += 64 * kAhead) {
            Request ahead[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) ahead[k] = lengths(r0 + 64 * k + lane);
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                take(r0 + 64 * k + lane, ahead[k]);
                add();
            }
        }
    }
    longest = wave_top(longest);
    work = readlane(wave_inclusive(work), 63) * a.kv_heads;
    row_tiles = readlane(wave_inclusive(row_tiles), 63) * a.kv_heads;
    Job job;
    job.found = false;
    job.all_slots = 0;
    if (longest == 0 || row_tiles > 0x7fffffff) return job;  // so many only if cu_new is not a list of offsets
    const int cus = places / 2;
    const float share = 0.5f * kTwo * (float)work * 0.5f / (float)cus;
    const bool may_cut = longest > kLeastCut && (float)longest > share;
    const long long limit = (row_tiles > places ? row_tiles : places) + extra_places(a, places);
    if (want >= (may_cut ? limit : row_tiles) && !to_the_end) return job;
    const bool at_hand = active <= 64;
    if (at_hand && a.R > 64) {
        const int r = lane < active ? list[lane] : a.R;
        take(r, lengths(r));
    }
    if (at_hand && active > 1) {
        const unsigned long long some = __ballot(rows.row_tiles > 0), below = (1ull << lane) - 1;
        int rank = active + __builtin_popcountll(~some & below);
        if (rows.row_tiles > 0) rank = 0;
        for (unsigned long long left = some; left != 0; left &= left - 1) {
            const int at = __builtin_ctzll(left), other = __builtin_amdgcn_readlane(rows.longest, at);
            if (rows.row_tiles > 0) rank += (other > rows.longest) | ((other == rows.longest) & (at < lane));
        }
        auto sorted = [&](int v) { return __builtin_amdgcn_ds_permute(4 * rank, v); };
        id = sorted(id);
        mine = {sorted(mine.first), sorted(mine.n), sorted(mine.seq), sorted(mine.len)};
        rows = {sorted(rows.row_tiles), sorted(rows.longest), sorted(rows.shortest)};
    }
    const int end = at_hand ? 1 : a.R;  // of the trips
    int each = longest;
    long long count = row_tiles;
    if (may_cut) {
        const int c = (longest + lane) / (lane + 1);  // this lane's estimate
        long long pieces = 0, cut = 0;
        for (int r0 = 0; r0 < end; r0 += 64) {
            if (!at_hand) take(r0 + lane, lengths(r0 + lane));
            for (unsigned long long some = __ballot(rows.row_tiles > 0); some != 0; some &= some - 1) {
                const int at = __builtin_ctzll(some), k = (__builtin_amdgcn_readlane(rows.longest, at) + c - 1) / c;
                const long long here = (long long)(__builtin_amdgcn_readlane(rows.row_tiles, at) * a.kv_heads) * k;
                pieces += here;
                if (k > 1) cut += here;
            }
        }
        float time = fmaxf((float)c, share);
        if (lane > 0) time = (pieces <= cus ? (float)c : pieces <= places ? kTwo * (float)c : kUneven * time + kBegin) + kCut + (float)cut / kPerTile;
        // the longest pieces of those that take least, to an eighth of a tile's time
        const int saved = cut > places || pieces > (limit < gridDim.x ? limit : gridDim.x) ? 0 : 0x7fffffff - (int)fminf(8.0f * time, 1e9f);
        const int best = __builtin_ctzll(__ballot(saved == wave_top(saved)));
        each = __builtin_amdgcn_readlane(c, best);
        count = readlane(pieces, best);
    }
    if (want >= count && !to_the_end) return job;
    // The longest row tiles come first.  With two for a CU at most the last of them comes second, for the CU with the longest.
    if (count <= places && want >= cus) want = want < count ? (int)count - 1 - (want - cus) : 0x7fffffff;

    int jobs = 0, slots = 0;
    for (int r0 = 0; r0 < end; r0 += 64) {
        if (!at_hand) take(r0 + lane, lengths(r0 + lane));
        const int k = rows.row_tiles > 0 ? (rows.longest + each - 1) / each : 0;
        const int here = rows.row_tiles * a.kv_heads * k, cut_here = k > 1 ? here : 0;
        const int upto = (int)wave_inclusive((long long)here), cut_upto = (int)wave_inclusive((long long)cut_here);
        const int total = __builtin_amdgcn_readlane(upto, 63);
        if (!job.found && want - jobs < total) {
            const int at = __builtin_ctzll(__ballot(upto > want - jobs));
            const int row_tiles = __builtin_amdgcn_readlane(rows.row_tiles, at);
            int local = want - jobs - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(here, at));
            // kv heads side by side: workgroups of one head then share an XCD's L2 where the heads are a multiple of the XCDs; the longest row
            // tiles first, for the short ones fill the gaps at the end
            job.kv_head = local % a.kv_heads;
            local /= a.kv_heads;
            job.row_tile = row_tiles - 1 - local % row_tiles;
            job.piece = local / row_tiles;
            job.r = __builtin_amdgcn_readlane(id, at);
            job.pieces = __builtin_amdgcn_readlane(k, at);
            job.each = each;
            job.slot = slots + __builtin_amdgcn_readlane(cut_upto, at) - __builtin_amdgcn_readlane(cut_here, at) +
                       (job.row_tile * a.kv_heads + job.kv_head) * job.pieces + job.piece;
            job.q = {__builtin_amdgcn_readlane(mine.first, at), __builtin_amdgcn_readlane(mine.n, at), __builtin_amdgcn_readlane(mine.seq, at),
                     __builtin_amdgcn_readlane(mine.len, at)};
            job.found = true;
        }
        jobs += total;
        slots += __builtin_amdgcn_readlane(cut_upto, 63);
        if (job.found && !to_the_end) break;
    }
    job.all_slots = slots;
    return job;
}

template <int D>
__global__ __launch_bounds__(64 * kWaves, 2) void attention_tile_kernel(AttentionArgs a, FewRule rule, int places, AttentionWs lay) {
    constexpr int STEPS = D / 16, BLOCKS = D / 32, SCALES = D / 32;
    constexpr int ROW = 2 * D;  // bytes of a token's keys or values in LDS
    typedef typename Quarter<D>::type Words;
    struct Half {
        __attribute__((aligned(16))) char v[kTok * ROW];  // bf16
        __attribute__((aligned(16))) char k[kTok * ROW];
        // of a wavefront's 16 tokens: 1, some block of values is NaN or may be infinite; 2, their page is nobody's.  Which blocks: bit 4 t + quarter.  Eight copies,
        // so that all lanes can write without a branch.
        __attribute__((aligned(16))) int odd[8][kWaves];
        unsigned long long nan[8][kWaves];
    };
    __shared__ Half halves[2];
    __shared__ int list[kWaves][64];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int col = lane & 31, group = lane >> 5;

    const Job job = find_job(a, uniform(few_rows(a, rule)) + 1, places, blockIdx.x, blockIdx.x == 0, list[wave]);
    if (blockIdx.x == 0 && threadIdx.x == 0) *reinterpret_cast<int*>(a.ws + lay.tile_count) = job.all_slots;
    if (!job.found) return;
    const int r = uniform(job.r), kv_head = uniform(job.kv_head), row_tile = uniform(job.row_tile), pieces = uniform(job.pieces);
    const Request q = uniform(job.q);
    const int rows = q.n * a.group, row0 = row_tile * kRows, p0 = q.len - q.n;
    const int last_row = row0 + kRows < rows ? row0 + kRows - 1 : rows - 1;
    // the wavefront's own rows
    const int w_row0 = row0 + 32 * wave, w_last = w_row0 + 31 < rows ? w_row0 + 31 : rows - 1;
    const bool w_any = w_row0 < rows;
    const int w_first_p = uniform(p0 + a.token_of(w_row0)), w_last_p = uniform(p0 + a.token_of(w_last));

    const Tiles seen = uniform(tiles<kTok>(a, q.seq, p0 + a.token_of(row0), p0 + a.token_of(last_row)));
    const int i_all = seen.count(), each = uniform(job.each);
    const int i_begin = uniform(job.piece) * each;
    int i_end = i_begin + each < i_all ? i_begin + each : i_all;
    if (job.piece + 1 == job.pieces) i_end = i_all;

    const ScalarInts table = (ScalarInts)(a.table + (size_t)r * a.width);
    const int page_mask = (1 << a.page.log2_size) - 1;
    const uint32_t head_bytes = (uint32_t)a.page.bytes(), page_stride = head_bytes * (uint32_t)a.kv_heads;
    const uint8_t* cache = a.cache + (size_t)kv_head * head_bytes;

    // A wavefront brings 16 tokens of a tile, which lie in one page: quarter lane % 4 of token lane / 4, in the order of memory.
    const int in_tok = 16 * wave + (lane >> 2), quarter = lane & 3;
    const uint32_t in_at = (lane >> 2) * (D / 2) + quarter * (D / 8), scale_at = (lane >> 2) * SCALES + quarter * (D / 4) / 32;
    struct Place {
        const uint8_t *codes, *scales;
        int t0;
        bool owned;
    };
    auto place = [&](int i) {
        Place p;
        p.t0 = seen.tile(i) * kTok;
        const int t = p.t0 + 16 * wave, b = t >> a.page.log2_size;
        const uint32_t page = (uint32_t)table[b < a.width ? b : a.width - 1];
        p.owned = page < (uint32_t)a.pages && b < a.width;
        const uint8_t* head = cache + (uint64_t)(p.owned ? page : 0u) * page_stride;
        p.codes = head + (t & page_mask) * (D / 2);
        p.scales = head + 2 * a.page.codes + (t & page_mask) * SCALES;
        return p;
    };
    Words k_in, v_in;
    uint32_t k_byte, v_byte;
    auto load = [&](const Place& p) {
        k_in = *reinterpret_cast<const Words*>(lane_at(p.codes, in_at));
        v_in = *reinterpret_cast<const Words*>(lane_at(p.codes + a.page.codes, in_at));
        k_byte = *lane_at(p.scales, scale_at);
        v_byte = *lane_at(p.scales + a.page.scales, scale_at);
    };
    // In LDS the 64-byte piece b of V's row t lies in place b ^ v_swizzle(t), so that the four rows of a transposed read fall on all banks, and
    // in odd rows the 16-byte pieces of a pair are swapped, so that the two rows that eight lanes write do; the 16-byte chunk c of K's
    // row t lies in k_place(c) ^ k_swizzle(t), so that a chunk of eight or sixteen rows does, and what eight lanes write (1 % faster than c ^ t % 16).
    auto v_swizzle = [](int t) { return D == 128 ? t & 3 : (t >> 1) & 1; };
    auto k_swizzle = [](int t) { return D == 128 ? (t & 1) << 2 | (t >> 1 & 3) | (t & 8) : t & 7; };
    const int v_to = in_tok * ROW + (((quarter * (D / 4) / 32) ^ v_swizzle(in_tok)) * 64) + (D == 128 ? 0 : (quarter & 1) * 32);
    const int v_even = v_to + (in_tok & 1) * 16, v_odd = v_to + 16 - (in_tok & 1) * 16;
    const int k_to = in_tok * ROW, k_turn = k_swizzle(in_tok);
    auto k_place = [](int chunk) { return D == 128 ? chunk >> 2 | (chunk & 3) << 2 : chunk; };
    auto write = [&](Half& h, const Place& p) {
        const bool there = p.owned & (p.t0 + in_tok < q.seq);
        uint32_t byte = there ? v_byte : 127u;  // never written: any number will do
        const unsigned long long nan = __ballot(byte > kLastScale);
        h.nan[lane & 7][wave] = nan;
        h.odd[lane & 7][wave] = (nan != 0 ? 1 : 0) | (p.owned ? 0 : 2);
        const float k_scale = scale_of_byte(k_byte);
#pragma unroll
        for (int e = 0; e < D / 32; ++e) *reinterpret_cast<bf16x8*>(h.k + k_to + ((k_place(quarter * (D / 32) + e) ^ k_turn) * 16)) = from_codes(k_in[e], k_scale);
        const float scale = scale_of_byte(byte > kLastScale ? 127u : byte);
#pragma unroll
        for (int e = 0; e < D / 32; ++e) *reinterpret_cast<bf16x8*>(h.v + (e % 2 == 0 ? v_even : v_odd) + 32 * (e / 2)) = from_codes(v_in[e], scale);
    };

    Place ahead, after;
    if (i_begin < i_end) {
        const Place first = place(i_begin);
        load(first);
        ahead = place(i_begin + 1 < i_end ? i_begin + 1 : i_end - 1);
        write(halves[0], first);
        load(ahead);
        after = place(i_begin + 2 < i_end ? i_begin + 2 : i_end - 1);
    }

    // Lane (col, group) holds elements 16 s + 8 group .. +7 of its row.
    const int row = w_row0 + col, token = a.token_of(row), head = kv_head * a.group + row - token * a.group;
    const int position = row < rows ? p0 + token : -1;  // -1 sees nothing
    bf16x8 query[STEPS];
    {
        const bf16_t* at = static_cast<const bf16_t*>(a.q) + (int64_t)(q.first + token) * a.q_stride + (int64_t)head * D + group * 8;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            uint4 raw = {0, 0, 0, 0};
            if (row < rows) raw = *reinterpret_cast<const uint4*>(at + 16 * s);
            query[s] = signed_query(raw, a.scale_log2);
        }
    }

    floatx16 out[BLOCKS];
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) out[b][e] = 0.0f;
    float most = kLowest, sum = 0.0f;  // the weights are 2^(scaled score - most)
    uint32_t bad = 0;  // quarters of this lane's query that a block of NaN values has reached

    // fragment addresses: K's row is the lane's column index; V's rows 4 group + (lane % 16) / 4 of every eight, four columns each
    const int sub = (lane >> 4) & 1, v_row = 4 * group + ((lane & 15) >> 2);
    const int k_from = col * ROW, k_from_turn = k_swizzle(col);  // 32 rows further on it is the same
    int v_from[BLOCKS];
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) v_from[b] = v_row * ROW + ((b ^ v_swizzle(v_row)) * 64) + sub * 32 + ((((lane & 3) >> 1) ^ (v_row & 1)) * 16) + (lane & 1) * 8;

    auto barrier = [] {
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };
    barrier();

    // Scores are compared before they are scaled: the scale is positive, its sign went into q.  A scale of zero becomes next to nothing, so
    // that it does not meet an infinity.
    const float scale = fmaxf(fabsf(a.scale_log2), 1e-37f);
    auto scores = [&](const Half& h, int tb) {
        floatx16 z;
#pragma unroll
        for (int e = 0; e < 16; ++e) z[e] = 0.0f;
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
            const bf16x8 key = *reinterpret_cast<const bf16x8*>(h.k + k_from + 32 * tb * ROW + ((k_place(2 * st + group) ^ k_from_turn) * 16));
            z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key, query[st], z, 0, 0, 0);
        }
        return z;
    };
    // masks 32 tokens' scores, and notes blocks of NaN values among the tokens seen: V holds numbers there
    auto look_closely = [&](floatx16& z, const Half& h, int4 odd4, int t0, int tb) {
        const int odd[2] = {tb == 0 ? odd4.x : odd4.z, tb == 0 ? odd4.y : odd4.w};
        // token 8 (e / 4) + 4 group + e % 4 of these 32, compared as 8 (e / 4) + e % 4: numbers that an instruction holds
        const int base = t0 + 32 * tb + 4 * group, last = position - base, first_sink = a.sinks - base;
        const int first = a.window > 0 && position >= a.window ? position - a.window + 1 - base : -base;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int j = 8 * (e / 4) + e % 4;
            const bool sees = (j <= last) & ((j >= first) | (j < first_sink)) & ((odd[e / 8] & 2) == 0);
            z[e] = sees ? z[e] : -INFINITY;
        }
        if (((odd[0] | odd[1]) & 1) != 0) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const uint32_t* eights = reinterpret_cast<const uint32_t*>(&h.nan[0][2 * tb + e / 8]);
                const uint32_t tokens = (uint32_t)uniform((int)eights[e / 4 % 2]) >> (16 * group);
                bad |= z[e] != -INFINITY ? tokens >> (4 * (e % 4)) & 15u : 0u;
            }
        }
    };
    auto largest = [&](const floatx16& z) {
        float top = z[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) top = fmaxf(top, z[e]);
        const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
        return fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
    };
    // The weights are taken against the largest score of the row's first tile, whatever comes later: they are floating-point numbers, and none
    // loses a bit until their sum comes near 1.  Only then is the maximum looked for, for all rows of the wavefront.
    auto weigh = [&](const floatx16* z, bf16x8* w) {
        union {
            bf16x2 two[16];
            bf16x8 eight[4];
        } u;
#pragma unroll
        for (int e = 0; e < 32; ++e) u.eight[e / 8][e % 8] = (__bf16)__builtin_amdgcn_exp2f(fmaf(z[e / 16][e % 16], scale, -most));
        const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
        float added[2] = {0.0f, 0.0f};
#pragma unroll
        for (int e = 0; e < 16; ++e) added[e % 2] = __builtin_amdgcn_fdot2_f32_bf16(u.two[e], ones, added[e % 2], false);
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = u.eight[k];
        return added[0] + added[1];
    };
    // One tile.  `under` runs under the scores' products: no branch between it and them.
    auto step = [&](const Half& here, int t0, bool closely, int4 odd, auto under) {
        floatx16 z[2];
        z[0] = scores(here, 0);
        z[1] = scores(here, 1);
        under();
        if (closely) {
            look_closely(z[0], here, odd, t0, 0);
            look_closely(z[1], here, odd, t0, 1);
        }
        bf16x8 w[4];
        float added = weigh(z, w);
        if (__any(sum + added > kMostSum)) {
            const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
            const float so_far = most + __builtin_amdgcn_logf(fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])));
            const float up = fmaxf(most, fmaxf(fmaxf(largest(z[0]), largest(z[1])) * scale, so_far) + kLift), f = __builtin_amdgcn_exp2f(most - up);
            most = up;
            sum *= f;
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) out[b] *= f;
            added = weigh(z, w);
        }
        sum += added;
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                union {
                    shortx4 half[2];
                    bf16x8 all;
                } f;
                f.half[0] = read_transposed(reinterpret_cast<const bf16_t*>(here.v + v_from[b] + (16 * k) * ROW));
                f.half[1] = read_transposed(reinterpret_cast<const bf16_t*>(here.v + v_from[b] + (16 * k + 8) * ROW));
                out[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.all, w[k], out[b], 0, 0, 0);
            }
    };
    int at = 0;
    // the next tile into the half that held the one before: all have passed the barrier after it
    auto stage = [&](int i, int next_at) {
        write(halves[next_at], ahead);
        load(after);
        const int next_t0 = ahead.t0;
        ahead = after;
        after = place(i + 3 < i_end ? i + 3 : i_end - 1);
        return next_t0;
    };
    if (w_any && i_begin < i_end) {
        int t0 = seen.tile(i_begin) * kTok;
        for (int i = i_begin; i < i_end; ++i) {
            const int next_at = at ^ 1;
            const Half& h = halves[at];
            const int4 odd = *reinterpret_cast<const int4*>(h.odd[0]);
            const bool closely = (uniform(odd.x | odd.y | odd.z | odd.w) != 0) | (t0 + kTok - 1 > w_first_p) |
                                 ((a.window > 0) & (t0 <= w_last_p - a.window) & (t0 + kTok > a.sinks));
            int next_t0;
            step(h, t0, closely, odd, [&] { next_t0 = stage(i, next_at); });
            barrier();
            t0 = next_t0;
            at = next_at;
        }
    } else {
        for (int i = i_begin; i < i_end; ++i) {  // a wavefront without rows brings its part of the tiles
            at ^= 1;
            stage(i, at);
            barrier();
        }
    }

    if (row >= rows) return;
    {
        const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
        sum = __uint_as_float(both[0]) + __uint_as_float(both[1]);
    }
    bad |= (uint32_t)__shfl_xor((int)bad, 32);
    const bool cut = pieces > 1;
    const float by = cut ? 1.0f : sum == 0.0f ? 0.0f : 1.0f / sum;
    const size_t slot_row = (size_t)uniform(job.slot) * kRows + 32 * wave + col;
    float* piece_to = reinterpret_cast<float*>(a.ws + lay.tile_outputs) + slot_row * D;
    bf16_t* to = static_cast<bf16_t*>(a.out) + (int64_t)(q.first + token) * a.out_stride + (int64_t)head * D;
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int d = 32 * b + 8 * e + 4 * group;
            floatx4 v = {out[b][4 * e], out[b][4 * e + 1], out[b][4 * e + 2], out[b][4 * e + 3]};
            v *= by;
            if (bad >> (D == 128 ? b : 2 * b) & (D == 128 ? 1u : 3u)) v = floatx4{NAN, NAN, NAN, NAN};
            if (cut) *reinterpret_cast<floatx4*>(piece_to + d) = v;
            else *reinterpret_cast<bf16x4*>(to + d) = __builtin_convertvector(v, bf16x4);
        }
    if (cut && group == 0) {
        *reinterpret_cast<float2*>(a.ws + lay.tile_sums + slot_row * 8) = float2{most, sum};
        if (threadIdx.x == 0) {
            const int n = rows - row0 < kRows ? rows - row0 : kRows;
            const int first = uniform(job.slot) - uniform(job.piece);
            reinterpret_cast<Piece*>(a.ws + lay.tile_records)[uniform(job.slot)] =
                Piece{q.first, row0, n, kv_head, uniform(job.piece), pieces, first, first + 1, 1};
        }
    }
}

}  // namespace

hipError_t launch_attention_tile(const emoe_kv_desc& d, const AttentionArgs& a, FewRule rule, const AttentionWs& lay, hipStream_t st) {
    DeviceShape shape;
    hipError_t e = device_shape(&shape);
    if (e != hipSuccess) return e;
    // Row tiles at most: n rows have (n - 1) / kRows + 1, and there are no more requests than of the fewest rows that come here.
    const long long least = rule.always + 1, all_rows = (long long)a.T * a.group, requests = all_rows / least < a.R ? all_rows / least : a.R;
    const long long per_request = ((long long)a.max_new * a.group + kRows - 1) / kRows, by_rows = requests + (all_rows - requests) / kRows;
    const long long row_tiles = per_request * a.R < by_rows ? per_request * a.R : by_rows;
    // whole row tiles, or pieces of them
    const int places = 2 * shape.groups;
    static_assert(2 * kMaxGroups <= kTileSlots, "a slot for every piece");
    const long long jobs = row_tiles * a.kv_heads, groups = jobs < places ? places : jobs + extra_places(a, places);
    if (groups > 0x7fffffff / 256) return hipErrorInvalidValue;
    if (d.head_dim == 64) attention_tile_kernel<64><<<(unsigned)groups, 64 * kWaves, 0, st>>>(a, rule, places, lay);
    else attention_tile_kernel<128><<<(unsigned)groups, 64 * kWaves, 0, st>>>(a, rule, places, lay);
    return hipGetLastError();
}

}  // namespace emoe
