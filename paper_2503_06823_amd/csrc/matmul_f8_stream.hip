// Products in 8 bits for few rows a group (a decode step): the cost is reading each matrix that has rows once.
//
// The work is one line of steps: the groups that have rows, of a group its blocks of 128 matrix rows, of those the passes of 16 TB rows of
// x, and of these (a unit) K in steps of 512 columns.  Every workgroup (4 wavefronts) takes an equal part of the line, so that all end
// together whatever the groups are.  Of the SwiGLU product a unit has the same 128 rows of both matrices: whole blocks of 128 outputs, which is what the
// activation's result needs to be brought to 8 bits.
// A step is a block of 128 columns for each wavefront.  Matrices lie in memory in the order in which the matrix instruction
// (v_mfma_scale_f32_16x16x128_f8f6f4) wants them, so they go from memory to registers and nowhere else, a contiguous KiB a load: a
// register that was multiplied is loaded again at once, with what comes RING strips of 16 rows later, across units too, and no wavefront waits for another before a
// unit's end.  The matrix's rows are the instruction's row operand, 16 rows of x its columns; the powers of two are operands of the
// instruction.  At a unit's end the four partial sums meet in LDS, added in wavefront order.
// A unit that is cut leaves its pieces in the workspace; who brings the last one adds them in their order and finishes the unit.  Pieces are
// written and read past the caches that workgroups do not share, and each is in memory before it is counted.
//
// The instruction adds the products of eight consecutive elements in units of 2^-13 of the largest pair's power of two, and all else in
// fp32: 1.5e-5 of a sum of random products, a hundredth of the rounding of the result to bf16.  (The bf16 instruction, on exact
// products of the same codes, has half the rate.)
#include "matrix_f8.h"

namespace emoe {
namespace {

typedef int intx8 __attribute__((ext_vector_type(8)));
typedef int intx4 __attribute__((ext_vector_type(4)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

constexpr int kLeastSteps = 2; // of a workgroup's part of the line

typedef unsigned int uintx4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void* base, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)bytes, 0x00020000);
}
// 16 bytes at `lane + at` and 16 at `second` bytes from there: an offset of the lane's, and a scalar one
template <int POLICY>
__device__ __forceinline__ intx8 two(__amdgpu_buffer_rsrc_t from, uint32_t lane, uint32_t at, int second) {
    const uintx4 a = __builtin_amdgcn_raw_buffer_load_b128(from, (int)lane, (int)at, POLICY);
    const uintx4 b = __builtin_amdgcn_raw_buffer_load_b128(from, (int)lane + second, (int)at, POLICY);
    return __builtin_bit_cast(intx8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Barrier for what lies in LDS; loads on their way stay there.
__device__ __forceinline__ void barrier_lds() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Groups in registers: lane g holds group g's rows and the number of its first unit.
struct Groups {
    int begin, end, first;
    int units;  // all (uniform)
};
__device__ __forceinline__ Groups find_groups(const F8Product& p, int rows_a_pass, int lane) {
    Groups g;
    g.begin = g.end = 0;
    if (lane < p.groups) {
        g.begin = p.offsets != nullptr ? p.offsets[lane] : 0;
        g.end = p.offsets != nullptr ? p.offsets[lane + 1] : p.rows;
        g.begin = g.begin > 0 ? g.begin : 0;
        g.end = g.end < p.rows ? g.end : p.rows;
        g.end = g.end > g.begin ? g.end : g.begin;
    }
    const int mine = (g.end - g.begin + rows_a_pass - 1) / rows_a_pass * p.lay.nb;
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int v = __shfl_up(upto, o);
        if (lane >= o) upto += v;
    }
    g.first = upto - mine;
    g.units = __builtin_amdgcn_readlane(upto, 63);
    return g;
}

struct Unit {
    int group, nb, row0, row_end;
};
__device__ __forceinline__ Unit unit_at(const Groups& g, const F8Product& p, int rows_a_pass, int lane, int u) {
    // the last group that begins at or before u: one without rows begins where its successor does
    const int at = __popcll(__ballot(lane < p.groups && g.first <= u)) - 1;
    const int begin = __builtin_amdgcn_readlane(g.begin, at), end = __builtin_amdgcn_readlane(g.end, at);
    const int passes = (end - begin + rows_a_pass - 1) / rows_a_pass;
    const int in = u - __builtin_amdgcn_readlane(g.first, at);
    const int nb = in / passes, row0 = begin + (in - nb * passes) * rows_a_pass;
    return {at, nb, row0, row0 + rows_a_pass < end ? row0 + rows_a_pass : end};
}

// The line's steps in `groups` equal parts, the first `longer` of them one step longer.
struct Shares {
    int each, longer, groups;
    __device__ __forceinline__ int begin(int w) const { return w * each + (w < longer ? w : longer); }
    __device__ __forceinline__ int owner(int step) const {
        const int of_longer = longer * (each + 1);
        return step < of_longer ? (int)((uint32_t)step / (uint32_t)(each + 1)) : longer + (int)((uint32_t)(step - of_longer) / (uint32_t)each);
    }
};

// Workgroups that a CU holds, by the registers that they take
constexpr int per_cu(int epilogue, int tb) { return (epilogue == kF8Swiglu && tb >= 2) || tb == 4 ? 1 : 2; }

template <int EPI, int TB>
__global__ __launch_bounds__(256, per_cu(EPI, TB)) void stream_kernel(F8Product p, float* __restrict__ pieces, int* __restrict__ counters) {
    constexpr int NB = EPI == kF8Swiglu ? 16 : 8;  // 16-row strips of a wavefront: 8 of each matrix
    constexpr int NQ = NB / 4;                     // of which each wavefront finishes a quarter
    constexpr int RING = EPI == kF8Swiglu && TB <= 2 && per_cu(EPI, TB) == 1 ? 16 : 8;  // strips of a wavefront on their way
    constexpr int ROWS = 16 * TB;
    __shared__ floatx4 red[4][NB][64];
    __shared__ uint32_t tops[4][ROWS];
    __shared__ int last_of;

    const int lane = threadIdx.x & 63, tok = lane & 15, quad = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Groups table = find_groups(p, ROWS, lane);
    const int KG = p.lay.kg;
    const int steps = table.units * KG;
    Shares shares;
    shares.groups = (steps + kLeastSteps - 1) / kLeastSteps;
    shares.groups = shares.groups < (int)gridDim.x ? shares.groups : (int)gridDim.x;
    if ((int)blockIdx.x >= shares.groups) return;
    shares.each = steps / shares.groups;
    shares.longer = steps - shares.each * shares.groups;
    const int line0 = shares.begin(blockIdx.x), line_end = shares.begin(blockIdx.x + 1);

    // ---- where a step's operands are ----------------------------------------------------------------------------
    struct Place {
        const uint8_t *w0, *w1;  // the group's matrices
        uint32_t at;             // bytes from there to this wavefront's block of 128 columns of step 0
        uint32_t scales;         // and to the powers
    };
    auto place_of = [&](const Unit& u) {
        Place o;
        o.w0 = p.w0 + (size_t)u.group * p.matrix_bytes;
        o.w1 = EPI == kF8Swiglu ? p.w1 + (size_t)u.group * p.matrix_bytes : o.w0;
        o.at = ((uint32_t)u.nb * p.lay.kb + wave) * kF8BlockBytes;
        o.scales = (uint32_t)p.lay.codes() + (uint32_t)u.nb * KG * 4;
        return o;
    };
    auto rows_of = [&](const Unit& u, uint32_t (&row)[TB]) {
#pragma unroll
        for (int t = 0; t < TB; ++t) {
            const int r = u.row0 + 16 * t + tok;
            const int at = r < u.row_end ? r : u.row_end - 1;  // (rows past the end are multiplied and not stored)
            row[t] = p.perm != nullptr ? (uint32_t)p.perm[at] : (uint32_t)at;
        }
    };
    const uint32_t divisor = p.perm != nullptr ? (uint32_t)p.k : 1u;
    // (a wavefront beyond K's last block takes that block once more, times zeros)
    auto block_of = [&](int s) { return 4 * s + wave < p.lay.kb ? 4 * s : p.lay.kb - 1 - wave; };

    const uint32_t matrix_codes = (uint32_t)p.lay.codes();
    const __amdgpu_buffer_rsrc_t x_rsrc = make_rsrc(p.x.codes, (uint32_t)p.x.rows * (uint32_t)p.x.stride);
    const __amdgpu_buffer_rsrc_t xs_rsrc = make_rsrc(p.x.scales, (uint32_t)p.x.rows * (uint32_t)KG * 4u);
    const uint32_t w_lane = lane * 16;
    intx8 w[RING], xf[TB];
    uint32_t xb[TB], b0 = 0, b1 = 0;        // powers, those of four blocks of columns together
    uint32_t x_lane[TB], xs_lane[TB];       // this lane's rows
    auto load_w = [&](int slot, const Place& o, int block, int i) {
        const uint8_t* base = o.w0;
        if (EPI == kF8Swiglu && i >= 8) base = o.w1;
        w[slot] = two<0>(make_rsrc(base, matrix_codes), w_lane, o.at + (uint32_t)block * kF8BlockBytes + (i & 7) * kF8Strip, 1024);
    };
    auto load_x = [&](const Place& o, int s, int block) {
#pragma unroll
        for (int t = 0; t < TB; ++t) {
            xf[t] = two<0>(x_rsrc, x_lane[t], (uint32_t)(block + wave) * kF8Block, 64);
            xb[t] = __builtin_amdgcn_raw_buffer_load_b32(xs_rsrc, (int)xs_lane[t], s * p.x.rows * 4, 0);
        }
        b0 = *reinterpret_cast<const uint32_t*>(o.w0 + o.scales + s * 4);
        if (EPI == kF8Swiglu) b1 = *reinterpret_cast<const uint32_t*>(o.w1 + o.scales + s * 4);
    };
    auto take_rows = [&](const uint32_t (&row)[TB]) {
#pragma unroll
        for (int t = 0; t < TB; ++t) {
            const uint32_t r = row[t] / divisor;
            x_lane[t] = r * (uint32_t)p.x.stride + quad * 16;
            xs_lane[t] = r * 4;
        }
    };

    int u = line0 / KG, s = line0 - u * KG;
    int line = line0;
    Unit cur = unit_at(table, p, ROWS, lane, u);
    Place at = place_of(cur);
    uint32_t next_row[TB];
    const int block0 = block_of(s);
#pragma unroll
    for (int i = 0; i < RING; ++i) load_w(i, at, block0, i);
    rows_of(cur, next_row);
    take_rows(next_row);
    load_x(at, s, block0);

    while (line < line_end) {
        const int begin = s;                                                       // this workgroup's steps of the unit
        const int end = KG - s < line_end - line ? KG : s + line_end - line;
        const bool more = line + (end - begin) < line_end;                         // there is another unit
        const Unit nxt = more ? unit_at(table, p, ROWS, lane, u + 1) : cur;
        const Place next_at = more ? place_of(nxt) : at;
        rows_of(nxt, next_row);

        floatx4 acc[NB][TB];
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int t = 0; t < TB; ++t) acc[i][t] = floatx4{0, 0, 0, 0};
#pragma unroll 1
        for (; s < end; ++s) {
            const bool turn = s + 1 == end;
            const int then = !turn ? s + 1 : more ? 0 : s;  // (behind the last step: it once more, unused)
            const int block = block_of(s), then_block = block_of(then);
            Place then_at = at;
            if (turn) then_at = next_at;
            intx8 xc[TB];
            uint32_t xbc[TB];
            const int shift = 8 * (block + wave - 4 * s);
            const uint32_t b0c = b0 >> shift, b1c = b1 >> shift;
#pragma unroll
            for (int t = 0; t < TB; ++t) { xc[t] = xf[t]; xbc[t] = xb[t] >> shift; }
            if (4 * s + wave >= p.lay.kb) {
#pragma unroll
                for (int t = 0; t < TB; ++t) xc[t] = intx8{0, 0, 0, 0, 0, 0, 0, 0};
            }
            if (turn) take_rows(next_row);
            __builtin_amdgcn_sched_barrier(0);
            load_x(then_at, then, then_block);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < NB; ++i) {
#pragma unroll
                for (int t = 0; t < TB; ++t)
                    acc[i][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w[i % RING], xc[t], acc[i][t], 0, 0, 0, (int)(i < 8 ? b0c : b1c), 0,
                                                                                 (int)xbc[t]);
                if (i + RING < NB) load_w(i % RING, at, block, i + RING);
                else load_w(i % RING, then_at, then_block, (i + RING) % NB);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        line += end - begin;

        // ---- the four partial sums, 16 rows of x at a time; wavefront q finishes rows 32 q .. 32 q + 31 of the 128 (of each matrix) ----
        floatx4 sum[NQ][TB];
#pragma unroll
        for (int t = 0; t < TB; ++t) {
#pragma unroll
            for (int i = 0; i < NB; ++i) red[wave][i][lane] = acc[i][t];
            barrier_lds();
#pragma unroll
            for (int j = 0; j < NQ; ++j) {
                const int i = 2 * wave + j % 2 + j / 2 * 8;
                sum[j][t] = red[0][i][lane] + red[1][i][lane] + red[2][i][lane] + red[3][i][lane];
            }
            barrier_lds();
        }

        bool finish = true;
        if (begin > 0 || end < KG) {
            // A piece: a workgroup has two places, for the unit that its part ends in (whose first piece that may be) and the one that it begins in.
            constexpr int VALUES = NQ * TB * 4;
            auto piece = [&](int group, bool first) { return pieces + ((size_t)group * 2 + (first ? 1 : 0)) * (VALUES * 256) + threadIdx.x; };
            float* mine = piece(blockIdx.x, begin == 0);
#pragma unroll
            for (int t = 0; t < TB; ++t) {
                if (cur.row0 + 16 * t + tok >= cur.row_end) continue;
#pragma unroll
                for (int j = 0; j < NQ; ++j)
#pragma unroll
                    for (int v = 0; v < 4; ++v)
                        __hip_atomic_store(mine + ((j * TB + t) * 4 + v) * 256, sum[j][t][v], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            const int first = shares.owner(u * KG), last = shares.owner(u * KG + KG - 1);
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // in memory, before it is counted
            barrier_lds();
            if (threadIdx.x == 0) {
                const int before = __hip_atomic_fetch_add(counters + u, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                last_of = before == last - first;
                if (before == last - first) __hip_atomic_store(counters + u, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // for the next launch
            }
            barrier_lds();
            finish = __builtin_amdgcn_readfirstlane(last_of) != 0;
            if (finish) {
#pragma unroll
                for (int j = 0; j < NQ; ++j)
#pragma unroll
                    for (int t = 0; t < TB; ++t) sum[j][t] = floatx4{0, 0, 0, 0};
                for (int g = first; g <= last; ++g) {  // (its own among them, at its place)
                    const float* from = piece(g, g == first);
#pragma unroll
                    for (int t = 0; t < TB; ++t) {
                        if (cur.row0 + 16 * t + tok >= cur.row_end) continue;
                        floatx4 v[NQ];
#pragma unroll
                        for (int j = 0; j < NQ; ++j)
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                v[j][i] = __hip_atomic_load(from + ((j * TB + t) * 4 + i) * 256, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
                        for (int j = 0; j < NQ; ++j) sum[j][t] += v[j];
                    }
                }
            }
        }

        // a lane holds row tok of x and outputs 4 quad .. 4 quad + 3 of two strips of 16
        const int n0 = cur.nb * kF8Block + wave * 32 + quad * 4;
        if (!finish) {
        } else if constexpr (EPI == kF8Plain) {
#pragma unroll
            for (int t = 0; t < TB; ++t) {
                const int r = cur.row0 + 16 * t + tok;
                if (r >= cur.row_end) continue;
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
            barrier_lds();
#pragma unroll
            for (int t = 0; t < TB; ++t) {
                const int r = cur.row0 + 16 * t + tok, c = 16 * t + tok;
                const uint32_t byte = f8_scale_byte(umax(umax(tops[0][c], tops[1][c]), umax(tops[2][c], tops[3][c])));
                if (r >= cur.row_end) continue;
                const float inverse = f8_inverse(byte);
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    *reinterpret_cast<uint32_t*>(p.h.codes + (size_t)r * p.h.stride + n0 + 16 * j) =
                        f8_codes(sum[j][t][0], sum[j][t][1], sum[j][t][2], sum[j][t][3], inverse);
                if (wave == 0 && quad == 0) reinterpret_cast<uint8_t*>(p.h.scales + (size_t)(cur.nb >> 2) * p.h.rows + r)[cur.nb & 3] = (uint8_t)byte;
            }
        }
        barrier_lds();  // red, tops and last_of are free again
        cur = nxt;
        at = next_at;
        ++u;
        s = 0;
    }
}

template <int EPI, int TB>
hipError_t launch_tb(const F8Product& p, const F8StreamWs& ws, hipStream_t st) {
    DeviceShape shape;
    hipError_t e = device_shape(&shape);
    if (e != hipSuccess) return e;
    static_assert(kF8StreamPieceBytes >= (size_t)kMaxGroups * per_cu(EPI, TB) * 2 * (EPI == kF8Swiglu ? 16 : 8) * TB * 4 * 64 * 4, "two places a workgroup");
    // as many as the line can have parts, if each group with rows has its passes
    const long long passes = (p.rows + 16 * TB - 1) / (16 * TB) + (p.groups < p.rows ? p.groups : p.rows);
    const long long most = (passes * p.lay.nb * p.lay.kg + kLeastSteps - 1) / kLeastSteps;
    const long long at_once = (long long)shape.groups * per_cu(EPI, TB);
    stream_kernel<EPI, TB><<<(unsigned)(most < at_once ? most : at_once), 256, 0, st>>>(p, ws.pieces, ws.counters);
    return hipGetLastError();
}

template <int EPI>
hipError_t launch(const F8Product& p, const F8StreamWs& ws, hipStream_t st) {
    const long long rows = (p.rows + p.groups - 1) / p.groups;
    if (p.rows <= 16 || rows <= 8) return launch_tb<EPI, 1>(p, ws, st);
    if (rows <= 22) return launch_tb<EPI, 2>(p, ws, st);
    return launch_tb<EPI, 4>(p, ws, st);
}

}  // namespace

hipError_t launch_f8_stream(const F8Product& p, F8Epilogue epilogue, const F8StreamWs& ws, hipStream_t st) {
    switch (epilogue) {
        case kF8Swiglu: return launch<kF8Swiglu>(p, ws, st);
        case kF8Relu: return launch<kF8Relu>(p, ws, st);
        default: return launch<kF8Plain>(p, ws, st);
    }
}

}  // namespace emoe
