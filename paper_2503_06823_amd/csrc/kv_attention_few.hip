// Attention over the paged 4-bit cache for requests of few queries: a decode step, one token a request.
//
//   S^T = K Q^T,  P^T = exp2(S^T - max),  O^T += V^T P^T,  with one pass over the keys and values, the running maximum and sum.
//
// Bound by reading the cache once: 2 * D * 17/32 bytes a token and kv head, against 4 * D flop for each of the heads that share
// it.  A workgroup has 16 rows (query token, query head) of one kv head, padded, and a piece of the request's keys;
// its four wavefronts take tiles of 32 tokens in turn, each with a maximum, a sum and an output of its own, so that nothing waits in
// the walk; they meet once, at its end.  The matrix instructions' token and element orders are free as long as both operands
// agree, and are chosen so that no data moves between lanes but V's:
//   - K: lane (row = lane % 16, group = lane / 16) holds D / 4 consecutive elements of one token, one 16-byte load (D = 128),
//     which all lie in one block and share one scale; step s multiplies its eight elements s, of all groups, with q's.
//   - P^T comes out of S^T in the registers in which the second product wants it: lane (query, group) holds tokens 4 group .. +3
//     of each 16, and V's rows are taken in that order.
//   - V: converted to bf16 where its scale is one per lane, through LDS (a wavefront's own), read back transposed.
// fp32 queries and weights are three bf16 operands each, which is exact to fp32; a 4-bit number is exact in bf16.
//
// Split: pieces of c tiles, so that all requests and heads together are about as many pieces as the chip holds workgroups; c
// follows from the lengths, which every wavefront reads for itself.  A row that is cut leaves its pieces (fp32 output, maximum, sum) in
// the workspace, and a second launch adds them in the pieces' order.
#include "kv_attention.h"

namespace emoe {
namespace {

constexpr int kTok = 32;      // tokens of a tile
constexpr int kRows = 16;     // rows of a workgroup
constexpr int kWaves = 4;
constexpr int kLeastTiles = 8;  // of a piece
constexpr float kLazy = 8.0f;   // log2 of what a weight may grow to before the maximum is taken up

// Workspace: [0] number of pieces, records, maxima and sums, outputs.
struct Piece {
    int token0, row0, rows, kv_head, piece, count, pad0, pad1;
};
struct FewWs {
    size_t records, sums, outputs, total;
};
FewWs few_ws(int most_pieces, int dim) {
    FewWs w;
    w.records = 256;
    w.sums = w.records + (size_t)most_pieces * sizeof(Piece);
    w.outputs = w.sums + (size_t)most_pieces * kRows * 8;
    w.total = w.outputs + (size_t)most_pieces * kRows * dim * 4;
    return w;
}

template <class E> struct Pieces { static constexpr int n = 1; };
template <> struct Pieces<float> { static constexpr int n = 3; };

__device__ __forceinline__ void load8(const float* p, float* x) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = p[i];
}
__device__ __forceinline__ void load8(const bf16_t* p, float* x) {
    const bf16x8 v = *reinterpret_cast<const bf16x8*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
}
__device__ __forceinline__ void store4(float* p, floatx4 v) { *reinterpret_cast<floatx4*>(p) = v; }
__device__ __forceinline__ void store4(bf16_t* p, floatx4 v) { *reinterpret_cast<bf16x4*>(p) = __builtin_convertvector(v, bf16x4); }

// The piece of work of a workgroup.
struct Job {
    int r, row_tile, kv_head, piece, pieces, tiles_each, slot;
};

// Finds job `want` of the requests with at most most_rows rows; every wavefront by itself, 64 requests a trip.  false: there is none.
// all_slots (if not null) receives the number of pieces of rows that are cut.
__device__ bool find_job(const AttentionArgs& a, int most_rows, int at_once, int want, Job* job, int* all_slots) {
    const int lane = threadIdx.x & 63;
    auto of_row = [&](int r, int* tiles_r, int* row_tiles) {
        *tiles_r = *row_tiles = 0;
        if (r >= a.R) return;
        const Request q = request(a, r);
        const long long rows = (long long)q.n * a.group;
        if (rows == 0 || rows > most_rows) return;
        *row_tiles = (int)((rows + kRows - 1) / kRows);
        *tiles_r = tiles<kTok>(a, q.seq, q.len - q.n, q.len - 1).count();
    };
    int tiles_r, row_tiles;
    long long units = 0;
    for (int r0 = 0; r0 < a.R; r0 += 64) {
        of_row(r0 + lane, &tiles_r, &row_tiles);
        units += (long long)tiles_r * row_tiles * a.kv_heads;
    }
#pragma unroll
    for (int s = 32; s > 0; s /= 2) {
        const int lo = __shfl_xor((int)units, s), hi = __shfl_xor((int)(units >> 32), s);
        units += ((long long)hi << 32) | (uint32_t)lo;
    }
    long long c = (units + at_once - 1) / at_once;
    c = (c + kWaves - 1) / kWaves * kWaves;
    const int each = c < kLeastTiles ? kLeastTiles : (int)c;
    int jobs = 0, slots = 0;
    bool found = false;
    for (int r0 = 0; r0 < a.R; r0 += 64) {
        if (a.R > 64) of_row(r0 + lane, &tiles_r, &row_tiles);
        const int pieces = tiles_r > each ? (tiles_r + each - 1) / each : 1;
        const int mine = row_tiles * a.kv_heads * pieces, cut = pieces > 1 ? mine : 0;
        const int upto = wave_inclusive(mine), cut_upto = wave_inclusive(cut);
        const int total = __builtin_amdgcn_readlane(upto, 63);
        if (!found && want - jobs < total) {
            const int at = __builtin_ctzll(__ballot(upto > want - jobs));
            const int p = __builtin_amdgcn_readlane(pieces, at), rt = __builtin_amdgcn_readlane(row_tiles, at);
            int local = want - jobs - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(mine, at));
            job->r = r0 + at;
            job->pieces = p;
            job->tiles_each = each;
            job->row_tile = local % rt;
            local /= rt;
            job->kv_head = local % a.kv_heads;
            job->piece = local / a.kv_heads;
            job->slot = slots + __builtin_amdgcn_readlane(cut_upto, at) - __builtin_amdgcn_readlane(cut, at) +
                        (job->kv_head * rt + job->row_tile) * p + job->piece;
            found = true;
        }
        jobs += total;
        slots += __builtin_amdgcn_readlane(cut_upto, 63);
        if (found && all_slots == nullptr) break;
    }
    if (all_slots != nullptr) *all_slots = slots;
    return found;
}

template <int D> struct KeyLoad { typedef uint4 type; };
template <> struct KeyLoad<64> { typedef uint2 type; };

// A tile on its way: what one lane loads of it.
template <int D>
struct Tile {
    static constexpr int V_LOADS = kTok * D / 2 / 1024;  // 16 bytes a lane
    union {
        typename KeyLoad<D>::type load;
        uint32_t step[D / 32];
    } k[2];
    uint4 v[V_LOADS];
    uint32_t k_scale[2], v_scale[V_LOADS];
};

template <class E, int D>
__global__ __launch_bounds__(64 * kWaves) void attention_few_kernel(AttentionArgs a, int most_rows, int at_once, int most_pieces, FewWs lay) {
    constexpr int PIECES = Pieces<E>::n, STEPS = D / 32, BLOCKS = D / 16;
    constexpr int V_STRIDE = D + 16;  // elements; 32 bytes past the row: 16 rows of 32 bytes fall on all banks alike
    constexpr int V_PER_TOKEN = D / 32;
    constexpr int WAVE_BYTES = kTok * V_STRIDE * 2;
    static_assert(BLOCKS * 1024 <= WAVE_BYTES, "the outputs take V's place at the end");
    __shared__ __align__(16) char lds[kWaves * WAVE_BYTES];
    __shared__ float sums[kWaves][kRows][2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, group = lane >> 4;

    Job job;
    int slots = 0;
    const bool found = find_job(a, most_rows, at_once, blockIdx.x, &job, blockIdx.x == 0 ? &slots : nullptr);
    if (blockIdx.x == 0 && threadIdx.x == 0) *reinterpret_cast<int*>(a.ws) = slots;
    if (!found) return;
    const int r = __builtin_amdgcn_readfirstlane(job.r), kv_head = __builtin_amdgcn_readfirstlane(job.kv_head);
    const Request q = request(a, r);
    const int rows = q.n * a.group, row0 = job.row_tile * kRows;
    const int row = row0 + col, token = row / a.group, head = kv_head * a.group + row % a.group;
    const int position = row < rows ? q.len - q.n + token : -1;  // -1 sees nothing
    const int last_row = row0 + kRows < rows ? row0 + kRows - 1 : rows - 1;
    const int p_first = q.len - q.n + row0 / a.group, p_last = q.len - q.n + last_row / a.group;

    bf16x8 query[PIECES][STEPS];
    {
        float x[8];
        const E* at = static_cast<const E*>(a.q) + (int64_t)(q.first + token) * a.q_stride + (int64_t)head * D + group * (D / 4);
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = 0.0f;
            if (row < rows) load8(at + s * 8, x);
            bf16x8 o[PIECES];
            to_operands<PIECES>(x, o);
#pragma unroll
            for (int p = 0; p < PIECES; ++p) query[p][s] = o[p];
        }
    }

    const Tiles seen = tiles<kTok>(a, q.seq, q.len - q.n, q.len - 1);
    int i_end = (job.piece + 1) * job.tiles_each, i_all = seen.count();
    i_end = i_end < i_all ? i_end : i_all;
    while (i_end > 0 && seen.tile(i_end - 1) * kTok > p_last) --i_end;  // no row of this tile sees so far
    const int32_t* table = a.table + (size_t)r * a.width;
    const size_t page_bytes = (size_t)a.page.bytes();
    bf16_t* v_lds = reinterpret_cast<bf16_t*>(lds + wave * WAVE_BYTES);

    auto page_of = [&](int i, int half) {
        const int b = (seen.tile(i) * kTok + 16 * half) >> a.page.log2_size;
        return b < a.width ? __builtin_amdgcn_readfirstlane(table[b]) : -1;
    };
    auto load = [&](Tile<D>& t, int i, const int* pages) {
        const uint8_t* base[2];
        int in_page[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int pg = (unsigned)pages[h] < (unsigned)a.pages ? pages[h] : 0;
            base[h] = a.cache + ((size_t)pg * a.kv_heads + kv_head) * page_bytes;
            in_page[h] = (seen.tile(i) * kTok + 16 * h) & ((1 << a.page.log2_size) - 1);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int tk = in_page[h] + col;
            t.k[h].load = *reinterpret_cast<const typename KeyLoad<D>::type*>(base[h] + tk * (D / 2) + group * (D / 8));
            t.k_scale[h] = base[h][2 * a.page.codes + tk * (D / 32) + group * (D / 4) / 32];
        }
#pragma unroll
        for (int n = 0; n < Tile<D>::V_LOADS; ++n) {
            const int chunk = n * 64 + lane, tok = chunk / V_PER_TOKEN, h = D == 128 ? n : tok / 16;
            const uint8_t* from = D == 128 ? base[n] : h ? base[1] : base[0];
            const int tk = (D == 128 ? in_page[n] : h ? in_page[1] : in_page[0]) + tok % 16;
            t.v[n] = *reinterpret_cast<const uint4*>(from + a.page.codes + tk * (D / 2) + chunk % V_PER_TOKEN * 16);
            t.v_scale[n] = from[2 * a.page.codes + a.page.scales + tk * (D / 32) + chunk % V_PER_TOKEN];
        }
    };

    floatx4 out[BLOCKS];
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) out[b] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    float most = kLowest, sum = 0.0f;

    auto multiply = [&](const Tile<D>& t, int i, const int* pages) {
        const int t0 = seen.tile(i) * kTok;
        const bool owned[2] = {(unsigned)pages[0] < (unsigned)a.pages, (unsigned)pages[1] < (unsigned)a.pages};
        // every row sees every token of the tile
        const bool whole = owned[0] && owned[1] && t0 + kTok - 1 <= p_first &&
                           (a.window == 0 || t0 > p_last - a.window || t0 + kTok <= a.sinks);
        bool nan = false;
#pragma unroll
        for (int n = 0; n < Tile<D>::V_LOADS; ++n) {
            const int chunk = n * 64 + lane, tok = chunk / V_PER_TOKEN;
            uint32_t byte = t.v_scale[n];
            if (!whole && (t0 + tok >= q.seq || !(tok < 16 ? owned[0] : owned[1]))) byte = 127;  // never written: any number will do
            nan |= byte == 255;
            const float scale = scale_of_byte(byte);
            bf16_t* to = v_lds + tok * V_STRIDE + chunk % V_PER_TOKEN * 32;
            *reinterpret_cast<bf16x8*>(to) = from_codes(t.v[n].x, scale);
            *reinterpret_cast<bf16x8*>(to + 8) = from_codes(t.v[n].y, scale);
            *reinterpret_cast<bf16x8*>(to + 16) = from_codes(t.v[n].z, scale);
            *reinterpret_cast<bf16x8*>(to + 24) = from_codes(t.v[n].w, scale);
        }
        float z[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            floatx4 s = {0.0f, 0.0f, 0.0f, 0.0f};
            const float scale = scale_of_byte(t.k_scale[h]);
#pragma unroll
            for (int st = 0; st < STEPS; ++st) {
                const bf16x8 key = from_codes(t.k[h].step[st], scale);
#pragma unroll
                for (int p = PIECES - 1; p >= 0; --p) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key, query[p][st], s, 0, 0, 0);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) z[4 * h + e] = s[e] * a.scale_log2;
        }
        if (!whole) {
            const int from = a.window > 0 && position >= a.window ? position - a.window + 1 : 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int j = t0 + 16 * (e / 4) + 4 * group + e % 4;
                const bool sees = j <= position && (j >= from || j < a.sinks) && owned[e / 4];
                z[e] = sees ? z[e] : -INFINITY;
            }
        }
        float top = z[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) top = fmaxf(top, z[e]);
        top = over_groups(top, [](float x, float y) { return fmaxf(x, y); });
        if (__any(top > most + kLazy)) {  // the weights stay below 2^8: a maximum that rises by less is not worth a pass over the output
            const float next = fmaxf(most, top), f = __builtin_amdgcn_exp2f(most - next);
            most = next;
            sum *= f;
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) out[b] *= f;
        }
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            w[e] = __builtin_amdgcn_exp2f(z[e] - most);
            sum += w[e];
        }
        bf16x8 weight[PIECES];
        to_operands<PIECES>(w, weight);
        const bf16_t* v_at = v_lds + (4 * group + (col >> 2)) * V_STRIDE + 4 * (col & 3);
        union VFragment {
            shortx4 half[2];
            bf16x8 all;
        };
        if (__any(nan)) {
            // blocks of NaN: what sees them becomes NaN, what does not stays as it is
            bf16x8 sees;
#pragma unroll
            for (int e = 0; e < 8; ++e) sees[e] = (__bf16)(z[e] == -INFINITY ? 0.0f : 1.0f);
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                VFragment f;
                f.half[0] = read_transposed(v_at + 16 * b);
                f.half[1] = read_transposed(v_at + 16 * V_STRIDE + 16 * b);
                bf16x8 bad;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const bool is = f.all[e] != f.all[e];
                    bad[e] = (__bf16)(is ? 1.0f : 0.0f);
                    f.all[e] = is ? (__bf16)0.0f : f.all[e];
                }
                floatx4 hit = {0.0f, 0.0f, 0.0f, 0.0f};
                hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bad, sees, hit, 0, 0, 0);
#pragma unroll
                for (int p = PIECES - 1; p >= 0; --p) out[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.all, weight[p], out[b], 0, 0, 0);
#pragma unroll
                for (int e = 0; e < 4; ++e) out[b][e] = hit[e] > 0.0f ? __uint_as_float(0x7fc00000u) : out[b][e];
            }
            return;
        }
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            VFragment f;
            f.half[0] = read_transposed(v_at + 16 * b);
            f.half[1] = read_transposed(v_at + 16 * V_STRIDE + 16 * b);
#pragma unroll
            for (int p = PIECES - 1; p >= 0; --p) out[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.all, weight[p], out[b], 0, 0, 0);
        }
    };

    // tile i + 4 is on its way while tile i is multiplied, and the page of tile i + 8 is looked up
    int i = job.piece * job.tiles_each + wave;
    if (i < i_end) {
        Tile<D> now;
        int pages[2], pages_next[2] = {-1, -1};
#pragma unroll
        for (int h = 0; h < 2; ++h) pages[h] = page_of(i, h);
        if (i + kWaves < i_end) {
#pragma unroll
            for (int h = 0; h < 2; ++h) pages_next[h] = page_of(i + kWaves, h);
        }
        load(now, i, pages);
        for (; i < i_end; i += kWaves) {
            Tile<D> next = now;
            int pages_after[2] = {-1, -1};
            if (i + kWaves < i_end) load(next, i + kWaves, pages_next);
            if (i + 2 * kWaves < i_end) {
#pragma unroll
                for (int h = 0; h < 2; ++h) pages_after[h] = page_of(i + 2 * kWaves, h);
            }
            multiply(now, i, pages);
            now = next;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                pages[h] = pages_next[h];
                pages_next[h] = pages_after[h];
            }
        }
    }

    // the four wavefronts' outputs, to the largest of their maxima
    sum = over_groups(sum, [](float x, float y) { return x + y; });
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
    const bool cut = job.pieces > 1;
    if (row >= rows && !cut) return;
    const int slot = job.slot < most_pieces ? job.slot : most_pieces - 1;
#pragma unroll
    for (int n = 0; n < BLOCKS / kWaves; ++n) {
        const int b = wave * (BLOCKS / kWaves) + n;
        floatx4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) v += part[w * WAVE_PARTS + b * 64 + lane] * factor[w];
        const int d = 16 * b + 4 * group;
        if (cut) {
            float* to = reinterpret_cast<float*>(a.ws + lay.outputs) + ((size_t)slot * kRows + col) * D + d;
            if (row < rows) *reinterpret_cast<floatx4*>(to) = v;
        } else {
            const float by = all == 0.0f ? 0.0f : 1.0f / all;
            store4(static_cast<E*>(a.out) + (int64_t)(q.first + token) * a.out_stride + (int64_t)head * D + d, v * by);
        }
    }
    if (cut && wave == 0 && group == 0) {
        float* to = reinterpret_cast<float*>(a.ws + lay.sums) + ((size_t)slot * kRows + col) * 2;
        to[0] = top;
        to[1] = all;
        if (col == 0) {
            const int n = rows - row0 < kRows ? rows - row0 : kRows;
            reinterpret_cast<Piece*>(a.ws + lay.records)[slot] = Piece{q.first, row0, n, kv_head, job.piece, job.pieces, 0, 0};
        }
    }
}

// The pieces of rows that were cut, in the pieces' order.  A workgroup for every piece; those of one row share its elements.
template <class E, int D>
__global__ __launch_bounds__(256) void attention_join_kernel(AttentionArgs a, FewWs lay) {
    const int slots = *reinterpret_cast<const int*>(a.ws);
    if ((int)blockIdx.x >= slots) return;
    const Piece p = reinterpret_cast<const Piece*>(a.ws + lay.records)[blockIdx.x];
    const size_t first = blockIdx.x - p.piece;
    const float* sums = reinterpret_cast<const float*>(a.ws + lay.sums) + first * kRows * 2;
    const float* outputs = reinterpret_cast<const float*>(a.ws + lay.outputs) + first * kRows * D;
    for (int e = p.piece * 256 + threadIdx.x; e < p.rows * D; e += p.count * 256) {
        const int row = e / D, d = e % D;
        float top = kLowest;
        for (int n = 0; n < p.count; ++n) top = fmaxf(top, sums[(n * kRows + row) * 2]);
        float all = 0.0f, v = 0.0f;
#pragma unroll 4
        for (int n = 0; n < p.count; ++n) {
            const float f = __builtin_amdgcn_exp2f(sums[(n * kRows + row) * 2] - top);
            all += sums[(n * kRows + row) * 2 + 1] * f;
            v += outputs[((size_t)n * kRows + row) * D + d] * f;
        }
        const int m = p.row0 + row;
        store_from_f32(static_cast<E*>(a.out), (size_t)((int64_t)(p.token0 + m / a.group) * a.out_stride +
                                                        (int64_t)(p.kv_head * a.group + m % a.group) * D + d), all == 0.0f ? 0.0f : v / all);
    }
}

constexpr int kPerCu = 4;  // workgroups that a CU holds

}  // namespace

size_t attention_few_ws_bytes(const emoe_kv_desc& d) { return few_ws(2 * kPerCu * kMaxGroups, d.head_dim).total; }

hipError_t launch_attention_few(const emoe_kv_desc& d, const emoe_attention_desc& at, const AttentionArgs& a, int most_rows, hipStream_t st) {
    DeviceShape shape;
    hipError_t e = device_shape(&shape);
    if (e != hipSuccess) return e;
    const int at_once = kPerCu * shape.groups, most_pieces = 2 * at_once;
    const FewWs lay = few_ws(most_pieces, d.head_dim);
    // row tiles that there can be, by the tokens and by the requests
    const long long per_request = ((long long)(a.max_new * (long long)a.group < most_rows ? a.max_new * (long long)a.group : most_rows) + kRows - 1) / kRows;
    const long long by_tokens = (long long)a.T * a.group / kRows + a.R;
    const long long row_tiles = per_request * a.R < by_tokens ? per_request * a.R : by_tokens;
    const long long groups = row_tiles * a.kv_heads + at_once;  // no more pieces than that
    if (groups > 0x7fffffff / 256) return hipErrorInvalidValue;
    auto run = [&](auto element, auto dim) {
        typedef decltype(element) E;
        constexpr int D = decltype(dim)::value;
        attention_few_kernel<E, D><<<(unsigned)groups, 64 * kWaves, 0, st>>>(a, most_rows, at_once, most_pieces, lay);
        hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
        attention_join_kernel<E, D><<<(unsigned)most_pieces, 256, 0, st>>>(a, lay);
        return hipGetLastError();
    };
    if (at.dtype == EMOE_F32)
        return d.head_dim == 64 ? run(float(), std::integral_constant<int, 64>()) : run(float(), std::integral_constant<int, 128>());
    return d.head_dim == 64 ? run(bf16_t(), std::integral_constant<int, 64>()) : run(bf16_t(), std::integral_constant<int, 128>());
}

size_t attention_ws_bytes(const emoe_kv_desc& d, const emoe_attention_desc&) { return attention_few_ws_bytes(d); }

hipError_t launch_attention(const emoe_kv_desc& d, const emoe_attention_desc& at, const AttentionArgs& a, hipStream_t st) {
    return launch_attention_few(d, at, a, 0x7fffffff, st);
}

}  // namespace emoe
