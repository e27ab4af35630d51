// Products in 8 bits for few rows a group (a decode step): the cost is reading each matrix that has rows once.
//
// A workgroup takes a unit: the rows of a group's matrix that share a power of two, 128, of the SwiGLU product those of both matrices -
// whole blocks of 128 outputs, which is what the activation's result needs to be brought to 8 bits - or fewer of a plain product, and all of K, times
// up to 64 rows of x.  A wavefront has STRIPS strips of 16 of the matrix's rows and every SPLIT-th block of 128 columns.  Matrices lie in memory in the
// order in which the matrix instruction (v_mfma_scale_f32_16x16x128_f8f6f4) wants them, so they go from memory to registers and nowhere else, a
// contiguous KiB a load, eight strips (16 KiB) on their way a wavefront, and no wavefront waits for another before the end of K.  The matrix's rows are
// the instruction's row operand, 16 rows of x its columns; the powers of two are operands of the instruction.
// The partial sums meet in LDS, added in wavefront order.  Few short rows are converted to 8 bits here, by each workgroup for itself, while the matrix's
// first strips are on their way; other rows by a launch before.
//
// One token's experts (two of 14336 x 4096, SwiGLU): 234 MB in 36 us, 6.5 TB/s, and 117 MB in 21 (the read stream: 6.9 TB/s, with some 2 us to begin and
// end); a whole matrix of 6144 x 4096 in 6.8.  64 rows: x, read once by each workgroup, is what bounds: 50 MB through the L1 caches for a matrix
// of 25 MB, 15 us with the conversion's launch.
//
// The instruction adds the products of eight consecutive elements in units of 2^-13 of the largest pair's power of two, and all else in
// fp32: 1.5e-5 of a sum of random products, a hundredth of the rounding of the result to bf16.  (The bf16 instruction, on exact
// products of the same codes, has half the rate.)
#include "matrix_f8.h"

namespace emoe {
namespace {

typedef int intx8 __attribute__((ext_vector_type(8)));
typedef unsigned int uintx4 __attribute__((ext_vector_type(4)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

// Blocks of columns of a wavefront on their way, eight strips: with the rows of x what the registers of two wavefronts a SIMD hold
constexpr int ring(int tb, int strips) { return tb == 4 && strips == 2 ? 3 : 8 / strips; }

__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void* base, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)bytes, 0x00020000);
}
// 16 bytes at `lane + at` and 16 at `second` bytes from there: an offset of the lane's, and a scalar one
template <int POLICY>  // of caches: 2, not kept: a matrix is read once; 0
__device__ __forceinline__ intx8 two(__amdgpu_buffer_rsrc_t from, uint32_t lane, uint32_t at, int second) {
    const uintx4 a = __builtin_amdgcn_raw_buffer_load_b128(from, (int)lane, (int)at, POLICY);
    const uintx4 b = __builtin_amdgcn_raw_buffer_load_b128(from, (int)lane + second, (int)at, POLICY);
    return __builtin_bit_cast(intx8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Row groups of a unit: the activation's results want 128 rows
constexpr int row_groups(int epilogue, int strips) { return epilogue == kF8Plain ? 1 : 8 / strips; }
constexpr int matrices(int epilogue) { return epilogue == kF8Swiglu ? 2 : 1; }

// A workgroup's rows of x where it converts them itself: codes [row][kb][128], and the powers [row][kb] as bytes
struct OwnRows {
    uint8_t codes[kF8OwnBlocks * kF8Block];
    uint8_t powers[kF8OwnBlocks];
};
// Their conversion, 16 lanes a block and eight elements a lane, in two parts: the loads, and once the matrix's first loads are on their way the rest
template <int WAVES>
struct RowsInFlight {
    static constexpr int kRounds = kF8OwnBlocks * 16 / (64 * WAVES);
    uint4 raw[kRounds];
    __device__ __forceinline__ void request(const F8Product& p, int row0, int row_end) {
        const int kb = p.lay.kb, units = (row_end - row0) * kb * 16;
        const uint32_t inverse = 65536u / (uint32_t)kb + 1u;  // (block * inverse) >> 16 is block / kb up to kF8OwnBlocks
        uint32_t row[kRounds];
        int k[kRounds];
#pragma unroll
        for (int i = 0; i < kRounds; ++i) {
            const int u = i * 64 * WAVES + threadIdx.x, block = u >> 4, r = (int)((uint32_t)block * inverse >> 16);
            k[i] = u < units ? (block - r * kb) * kF8Block + (u & 15) * 8 : p.K;
            row[i] = u < units ? row0 + r : row0;
        }
        if (p.perm != nullptr) {
#pragma unroll
            for (int i = 0; i < kRounds; ++i) row[i] = (uint32_t)p.perm[row[i]];
#pragma unroll
            for (int i = 0; i < kRounds; ++i) row[i] /= (uint32_t)p.k;
        }
#pragma unroll
        for (int i = 0; i < kRounds; ++i) {
            raw[i] = make_uint4(0, 0, 0, 0);
            if (k[i] < p.K) raw[i] = *reinterpret_cast<const uint4*>(p.from + (int64_t)row[i] * p.from_stride + k[i]);
        }
    }
    __device__ __forceinline__ void convert(const F8Product& p, int row0, int row_end, OwnRows& own) const {
        const int units = (row_end - row0) * p.lay.kb * 16;
#pragma unroll
        for (int i = 0; i < kRounds; ++i) {
            if (i * 64 * WAVES >= units) break;
            const int u = i * 64 * WAVES + threadIdx.x;
            float v[8];
            f8_widened(raw[i], v);
            uint32_t top = f8_top(v);
#pragma unroll
            for (int o = 1; o < 16; o <<= 1) top = umax(top, (uint32_t)__shfl_xor((int)top, o));
            const uint32_t byte = f8_scale_byte(top);
            if (u < units) {
                *reinterpret_cast<uint2*>(own.codes + u * 8) = f8_codes(v, f8_inverse(byte));
                if ((u & 15) == 0) own.powers[u >> 4] = (uint8_t)byte;
            }
        }
        // a barrier for LDS alone: the matrix's loads stay on their way
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
    }
};

// As F8RowInMemory, of OwnRows
struct OwnRow {
    const uint8_t *codes, *powers;
    __device__ uint4 piece(int q) const { return *reinterpret_cast<const uint4*>(codes + q * 16); }
    __device__ int power(int b) const { return powers[b]; }
};

// Rows row0 .. row_end - 1 of x, 16 TB at most, times a unit of their group's matrix.  OWN: x is converted here.
template <int EPI, int TB, int STRIPS, int WAVES, bool OWN>
__device__ __forceinline__ void multiply_unit(const F8Product& p, int unit, int group, int row0, int row_end, floatx4 (&red)[WAVES][STRIPS][64],
                                              uint32_t (&tops)[WAVES][64], OwnRows* own) {
    static_assert(!OWN || TB == 1, "at most 16 rows");
    constexpr int M = matrices(EPI), H = row_groups(EPI, STRIPS), SPLIT = WAVES / (M * H);
    static_assert(SPLIT >= 1 && SPLIT * M * H == WAVES, "every wavefront has a part");
    constexpr int DEPTH = ring(TB, STRIPS);
    constexpr int ALL = STRIPS * H;       // strips of a unit, of one matrix
    constexpr int FINAL = ALL >= WAVES ? ALL / WAVES : 1;  // that a wavefront finishes
    const int lane = threadIdx.x & 63, tok = lane & 15, quad = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int part = wave % SPLIT, half = wave / SPLIT % H;
    const int nb = unit * ALL / 8, strip0 = unit * ALL % 8;  // its block of 128 rows, and place in it

    const uint8_t* matrix = (M == 2 && wave >= SPLIT * H ? p.w1 : p.w0) + (size_t)group * p.matrix_bytes;
    const uint32_t codes = (uint32_t)p.lay.codes();
    const __amdgpu_buffer_rsrc_t w_rsrc = make_rsrc(matrix, codes);
    const uint32_t x_bytes = (uint32_t)p.x.rows * (uint32_t)p.lay.kb * kF8Block;
    const __amdgpu_buffer_rsrc_t x_rsrc = make_rsrc(p.x.codes, x_bytes);
    const uint32_t xs_bytes = (uint32_t)p.x.rows * (uint32_t)p.lay.kg * 4u;
    const __amdgpu_buffer_rsrc_t xs_rsrc = make_rsrc(p.x.scales, xs_bytes);
    const uint32_t x_block = 8u * (uint32_t)p.x.piece_step;  // bytes from a block of columns to the next
    const uint32_t* w_scales = reinterpret_cast<const uint32_t*>(matrix + codes + (size_t)nb * p.lay.kg * 4);
    const uint32_t w_at = (uint32_t)nb * p.lay.kb * kF8BlockBytes + (strip0 + half * STRIPS) * kF8Strip;
    const int mine = (p.lay.kb - part + SPLIT - 1) / SPLIT;  // this wavefront's blocks of columns: part, part + SPLIT, ...

    uint32_t x_lane[TB], xs_lane[TB];
#pragma unroll
    for (int t = 0; t < TB; ++t) {
        int r = row0 + 16 * t + tok;
        r = r < row_end ? r : row_end - 1;  // (rows past the end are multiplied and not stored)
        if constexpr (OWN) {
            xs_lane[t] = (uint32_t)((r - row0) * p.lay.kb);  // its first block
            x_lane[t] = xs_lane[t] * kF8Block + quad * 16;
        } else {
            x_lane[t] = (uint32_t)r * p.x.row_step + (uint32_t)quad * p.x.piece_step;
            xs_lane[t] = (uint32_t)r * 4;
        }
    }
    intx8 w[DEPTH][STRIPS], x[DEPTH][TB];
    uint32_t xb[DEPTH][TB], wb[DEPTH];
    // the wavefront's j-th block of columns; behind its last one out of range: zeros, and nothing is read
    auto load_w = [&](int slot, int j) {
        const bool there = j < mine;
        const uint32_t b = there ? part + j * SPLIT : part, lane_at = there ? lane * 16u : codes;
#pragma unroll
        for (int i = 0; i < STRIPS; ++i) w[slot][i] = two<2>(w_rsrc, lane_at, w_at + b * kF8BlockBytes + i * kF8Strip, 1024);
        wb[slot] = w_scales[b >> 2];
    };
    auto load_x = [&](int slot, int j) {
        const bool there = j < mine;
        const int b = there ? part + j * SPLIT : part;
#pragma unroll
        for (int t = 0; t < TB; ++t) {
            if constexpr (OWN) {  // (behind the last block the first one again: its products are with zeros)
                const int at = there ? b : 0;
                const uintx4* from = reinterpret_cast<const uintx4*>(own->codes + x_lane[t] + at * kF8Block);
                x[slot][t] = __builtin_bit_cast(intx8, __builtin_shufflevector(from[0], from[4], 0, 1, 2, 3, 4, 5, 6, 7));
                xb[slot][t] = own->powers[xs_lane[t] + at];
                continue;
            }
            x[slot][t] = two<0>(x_rsrc, there ? x_lane[t] : x_bytes, (uint32_t)b * x_block, (int)(x_block / 2));
            xb[slot][t] = __builtin_amdgcn_raw_buffer_load_b32(xs_rsrc, (int)(there ? xs_lane[t] : xs_bytes), (b >> 2) * p.x.rows * 4, 0);
        }
    };
    if constexpr (OWN) {
        RowsInFlight<WAVES> rows;
        rows.request(p, row0, row_end);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) load_w(d, d);
        __builtin_amdgcn_sched_barrier(0);
        rows.convert(p, row0, row_end, *own);
    }
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
        if constexpr (!OWN) load_w(d, d);
        load_x(d, d);
    }
    floatx4 acc[STRIPS][TB];
#pragma unroll
    for (int i = 0; i < STRIPS; ++i)
#pragma unroll
        for (int t = 0; t < TB; ++t) acc[i][t] = floatx4{0, 0, 0, 0};
    for (int j = 0; j < mine; j += DEPTH) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            __builtin_amdgcn_sched_barrier(0);
            const int shift = 8 * ((part + (j + d) * SPLIT) & 3);
            uint32_t xbc[TB];
            const uint32_t wbc = j + d < mine ? wb[d] >> shift : 127u;  // (zeros times any power but NaN)
#pragma unroll
            for (int t = 0; t < TB; ++t) xbc[t] = OWN ? xb[d][t] : xb[d][t] >> shift;
#pragma unroll
            for (int i = 0; i < STRIPS; ++i)
#pragma unroll
                for (int t = 0; t < TB; ++t)
                    acc[i][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w[d][i], x[d][t], acc[i][t], 0, 0, 0, (int)wbc, 0, (int)xbc[t]);
            load_w(d, j + d + DEPTH);
            load_x(d, j + d + DEPTH);
        }
    }

    // ---- the partial sums, 16 rows of x at a time; wavefront q finishes the strips from q FINAL on ------------------
    floatx4 sum[M][FINAL][TB];
#pragma unroll
    for (int t = 0; t < TB; ++t) {
#pragma unroll
        for (int i = 0; i < STRIPS; ++i) red[wave][i][lane] = acc[i][t];
        __syncthreads();
        if (ALL >= WAVES || wave < ALL) {
#pragma unroll
            for (int m = 0; m < M; ++m)
#pragma unroll
                for (int f = 0; f < FINAL; ++f) {
                    const int i = wave * FINAL + f, from = (m * H + i / STRIPS) * SPLIT;
                    floatx4 v = red[from][i % STRIPS][lane];
#pragma unroll
                    for (int o = 1; o < SPLIT; ++o) v += red[from + o][i % STRIPS][lane];
                    sum[m][f][t] = v;
                }
        }
        __syncthreads();
    }

    // a lane holds row tok of x and outputs 4 quad .. 4 quad + 3 of its wavefront's strips
    const int n0 = nb * kF8Block + (strip0 + wave * FINAL) * 16 + quad * 4;
    if constexpr (EPI == kF8Plain) {
        if (ALL >= WAVES || wave < ALL) {
#pragma unroll
            for (int t = 0; t < TB; ++t) {
                const int r = row0 + 16 * t + tok;
                if (r >= row_end) continue;
                bf16_t* to = p.out + (size_t)(p.out_perm != nullptr ? p.out_perm[r] : r) * p.out_stride + n0;
#pragma unroll
                for (int f = 0; f < FINAL; ++f)
                    if (n0 + 16 * f < p.N) *reinterpret_cast<bf16x4*>(to + 16 * f) = __builtin_convertvector(sum[0][f][t], bf16x4);
            }
        }
    } else {
#pragma unroll
        for (int t = 0; t < TB; ++t) {
            uint32_t top = 0;
#pragma unroll
            for (int f = 0; f < FINAL; ++f)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    float g = sum[0][f][t][v];
                    if constexpr (EPI == kF8Swiglu) g = g / (1.0f + __expf(-g)) * sum[M - 1][f][t][v];
                    else g = g < 0.0f ? 0.0f : g;  // (NaN stays)
                    sum[0][f][t][v] = g;
                    top = umax(top, f8_magnitude(g));
                }
            top = umax(top, (uint32_t)__shfl_xor((int)top, 16));
            top = umax(top, (uint32_t)__shfl_xor((int)top, 32));
            if (quad == 0) tops[wave][16 * t + tok] = top;
        }
        __syncthreads();
        uint32_t near[TB], top_of[TB];
#pragma unroll
        for (int t = 0; t < TB; ++t) {
            const int r = row0 + 16 * t + tok, c = 16 * t + tok;
            uint32_t top = tops[0][c];
#pragma unroll
            for (int o = 1; o < WAVES; ++o) top = umax(top, tops[o][c]);
            const uint32_t byte = f8_scale_byte(top);
            const float inverse = f8_inverse(byte);
            near[t] = 0;
            top_of[t] = top;
            if (r >= row_end) continue;
#pragma unroll
            for (int f = FINAL - 1; f >= 0; --f) {
                const floatx4& h = sum[0][f][t];
                *reinterpret_cast<uint32_t*>(p.h.codes + (size_t)r * p.h.row_step + (size_t)((n0 >> 4) + f) * p.h.piece_step + quad * 4) = f8_codes(h[0], h[1], h[2], h[3], inverse);
#pragma unroll
                for (int v = 3; v >= 0; --v) near[t] = f8_near_ties(near[t], h[v] * inverse);
            }
            if (byte == 255u || p.lay.nb > kTieBlocks) near[t] = 0;
            if (wave == 0 && quad == 0) reinterpret_cast<uint8_t*>(p.h.scales + (size_t)(nb >> 2) * p.h.rows + r)[nb & 3] = (uint8_t)byte;
        }
#pragma unroll 1
        for (int t = 0; t < TB; ++t) {
            uint32_t its_near = near[0], its_top = top_of[0];
#pragma unroll
            for (int i = 1; i < TB; ++i) {
                its_near = t == i ? near[i] : its_near;
                its_top = t == i ? top_of[i] : its_top;
            }
            for (uint64_t left = __ballot(its_near != 0); left != 0; left &= left - 1) {
                const int who = __builtin_amdgcn_readfirstlane(__builtin_ctzll(left)), row = row0 + 16 * t + (who & 15);
                const float inverse = f8_inverse(f8_scale_byte((uint32_t)__builtin_amdgcn_readlane((int)its_top, who)));
                const uint8_t* both[M];
                both[0] = p.w0 + (size_t)group * p.matrix_bytes;
                if constexpr (M == 2) both[1] = p.w1 + (size_t)group * p.matrix_bytes;
                for (uint32_t bits = (uint32_t)__builtin_amdgcn_readlane((int)its_near, who); bits != 0; bits &= bits - 1) {
                    const int bit = __builtin_ctz(bits), n = nb * kF8Block + (strip0 + wave * FINAL + (bit >> 2)) * 16 + (who >> 4) * 4 + (bit & 3);
                    float h;
                    if constexpr (OWN) h = f8_h<M, 64>(p.lay, both, n, OwnRow{own->codes + (row - row0) * p.lay.kb * kF8Block, own->powers + (row - row0) * p.lay.kb});
                    else h = f8_h<M, 64>(p.lay, both, n, F8RowInMemory(p.x, row));
                    if (lane == who)  // (which stored the element before)
                        p.h.codes[(size_t)row * p.h.row_step + (size_t)(n >> 4) * p.h.piece_step + (n & 15)] = (uint8_t)f8_codes(h, 0.0f, 0.0f, 0.0f, inverse);
                }
            }
        }
    }
}

// MOST: blocks of 16 rows that a workgroup has at most, 1 or 4.  Workgroups go through the units of an item, then of the next: with MOST 1 items are groups, otherwise
// 64 rows of a group or what is left of it, counted through the groups (there are fewer than there are workgroups for).
template <int EPI, int MOST, int STRIPS, int WAVES, bool OWN>
__global__ __launch_bounds__(64 * WAVES, 2) void stream_kernel(F8Product p, int n_units) {
    __shared__ floatx4 red[WAVES][STRIPS][64];
    __shared__ uint32_t tops[WAVES][64];
    OwnRows* own = nullptr;
    if constexpr (OWN) {
        __shared__ __align__(16) OwnRows rows;
        own = &rows;
    }
    const int unit = blockIdx.x % n_units, item = blockIdx.x / n_units;
    int group = 0, row0 = 0, row_end = p.rows;
    if (MOST == 1 || p.groups == 1) {
        if (MOST == 1) group = item;
        if (p.offsets != nullptr) {
            row0 = p.offsets[group];
            row_end = p.offsets[group + 1];
            row0 = row0 > 0 ? row0 : 0;
            row_end = row_end < p.rows ? row_end : p.rows;
        }
        if (MOST > 1) row0 += item * 16 * MOST;
    } else {
        const int lane = threadIdx.x & 63;
        int begin = 0, end = 0;
        if (lane < p.groups) {
            begin = p.offsets[lane];
            end = p.offsets[lane + 1];
            begin = begin > 0 ? begin : 0;
            end = end < p.rows ? end : p.rows;
        }
        const int items = end > begin ? (end - begin + 16 * MOST - 1) / (16 * MOST) : 0;
        int upto = items;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int below = __shfl_up(upto, o);
            upto += lane >= o ? below : 0;
        }
        const uint64_t behind = __ballot(upto > item);
        if (behind == 0) return;
        group = __builtin_amdgcn_readfirstlane(__builtin_ctzll(behind));
        row0 = __builtin_amdgcn_readlane(begin, group) + (item - __builtin_amdgcn_readlane(upto - items, group)) * 16 * MOST;
        row_end = __builtin_amdgcn_readlane(end, group);
    }
    if (row_end <= row0) return;  // its matrix is never touched
    if (MOST > 1) row_end = row_end < row0 + 16 * MOST ? row_end : row0 + 16 * MOST;
    if (MOST == 1 || row_end - row0 <= 16) multiply_unit<EPI, 1, STRIPS, WAVES, OWN>(p, unit, group, row0, row_end, red, tops, own);
    else if (row_end - row0 <= 32) multiply_unit<EPI, MOST == 1 ? 1 : 2, STRIPS, WAVES, OWN>(p, unit, group, row0, row_end, red, tops, own);
    else multiply_unit<EPI, MOST, STRIPS, WAVES, OWN>(p, unit, group, row0, row_end, red, tops, own);
}

template <int EPI, int MOST, int STRIPS, int WAVES>
hipError_t launch_shape(const F8Product& p, hipStream_t st) {
    constexpr int all = STRIPS * row_groups(EPI, STRIPS);
    const int n_units = (p.N + 16 * all - 1) / (16 * all);
    const long long chunks = MOST == 1 ? p.groups : p.groups == 1 ? (p.rows + 16 * MOST - 1) / (16 * MOST) : p.groups + p.rows / (16 * MOST);
    const unsigned grid = (unsigned)(chunks * n_units);
    if constexpr (MOST == 1) {
        if (p.from != nullptr) {
            stream_kernel<EPI, MOST, STRIPS, WAVES, true><<<grid, 64 * WAVES, 0, st>>>(p, n_units);
            return hipGetLastError();
        }
    }
    stream_kernel<EPI, MOST, STRIPS, WAVES, false><<<grid, 64 * WAVES, 0, st>>>(p, n_units);
    return hipGetLastError();
}

// A wavefront's strips by the strips that there are: more of them a wavefront read x less often, fewer leave no CU without work.  Measured with matrices from
// HBM, plain products of 17 to 64 rows a stretch (us, two strips / four): 128 strips 13.1 / 14.3 (64 rows times 2048 x 4096), 384 15.5 / 16.7 (6144 x 4096), 512
// 16.4 / 17.4, 768 23.8 / 19.6, two stretches of 384 23.8 / 18.5, 1040 12.0 / 10.0 (16 groups of 1032 x 776), 2048 103 / 100 (8 of 4096 x 14336); eight wavefronts
// of four strips were up to a fifth slower.  Up to 16 rows (one strip / two / four): 64 strips 4.5 / 5.3 / 6.7 (one row times 1024 x 4096), 256 5.9 / 7.1 / 8.7, 384
// 8.3 / 7.5 / 9.3, 512 27.2 / 25.8 / 29.6 (2 of 4096 x 14336), 520 6.3 / 5.6 / 4.5 (8 of 1032 x 776), 768 12.4 / 12.7 / 11.6, 2000 28.0 / 27.6 / 26.2, 2048 23.9 / 15.1 /
// 13.4 (16 rows of 16 of 2048 x 1408); with eight wavefronts one or two strips 10.1 and 7.2 at 384, 36.9 and 27.7 at 2000.  The activations' products want 128 rows a unit; four wavefronts / eight: 20 rows of 6 groups of 14336 x 4096 121 / 121
// (SwiGLU), 71 / 74 (ReLU), one row of 32 of 512 x 512 9.5 / 10.2, 7.9 / 9.0; with eight strips a wavefront 130, 72, 9.9, 7.9.
template <int EPI>
hipError_t launch(const F8Product& p, hipStream_t st) {
    const long long groups = p.groups < p.rows ? p.groups : p.rows;  // that can have rows
    const bool few = p.rows <= 16;
    if constexpr (EPI == kF8Plain) {
        const long long stretches = (p.rows + 63) / 64, strips = (groups > stretches ? groups : stretches) * ((p.N + 15) / 16);
        if (strips > 512) return few ? launch_shape<EPI, 1, 4, 4>(p, st) : launch_shape<EPI, 4, 4, 4>(p, st);
        if (!few) return launch_shape<EPI, 4, 2, 4>(p, st);
        return strips > 256 ? launch_shape<EPI, 1, 2, 4>(p, st) : launch_shape<EPI, 1, 1, 4>(p, st);
    } else {
        return few ? launch_shape<EPI, 1, 4, 4>(p, st) : launch_shape<EPI, 4, 4, 4>(p, st);
    }
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
