// Products in 8 bits for many rows a group: grouped GEMM on the scaled matrix instructions of gfx950.
//
// Tile: a workgroup of 4 wavefronts (2 x 2, one per SIMD) owns 256 rows x 256 matrix rows - of the SwiGLU product 128 rows of one
// matrix and the same 128 of the other, so that a lane holds gate and up of the same output - and each wavefront accumulates 128 x
// 128 as 8 x 8 blocks of v_mfma_scale_f32_16x16x128_f8f6f4 in 256 accumulator registers.  The matrix's rows are the instruction's row operand, 16
// rows of x its columns; the powers of two are operands of the instruction and cost nothing.  K is walked in tiles of 128, a tile row
// of either operand being one whole cache line, and one tile is one matrix instruction a block.
//
// Data movement: operand tiles (32 KiB each) go from memory straight into LDS, two of each.  Rows of x, which are gathered, lie there
// as rows whose 16-byte chunk c stands at place c ^ ((row >> 1) & 7), which makes the fragment reads free of bank conflicts; a packed matrix lies in memory
// in the order of the fragments and is copied as it is.  A tile has two phases, each with half of the matrix rows and a barrier at its
// end.  In phase 1 a wavefront reads the other half's fragments and requests rows and first half of the tile after next; in phase 2 it reads the next tile's rows and
// first half and requests the second half of the tile after next.  So whatever is requested has one and a half tiles, 3000 cycles, to arrive in, with 128 KiB of LDS.
// The powers of a row's next four tiles come as one dword, by the same kind of load.
//
// The stream of operand tiles does not stop between output tiles: the last two K tiles request the next item's first two.
// Rows are spread evenly over a group's tiles in blocks of 16, and the K loop is compiled for 0 .. 8 blocks a wavefront (tile_plan.h).  Tiles that
// do not fill a round of the chip are cut along K, and a second launch adds the pieces in order.
//
// 8192 rows times 6144 x 4096: 177 us a call, 22 to 25 of them the conversion, so some 152 for the product, 2.7 PFLOP/s (under the tracer 158 to 184; a library's
// product of the same extents, with one factor a matrix, 164 to 171).  The SwiGLU product of 8192 assignments over four experts of 14336 x 4096 in 745 to 777 us, 2.5
// PFLOP/s.  What bounds it is the power that the matrix cores draw: they are busy in 63 to 71 % of the cycles at a clock that they push down to 1.9 to 2.0 GHz; without
// any LDS reads it would be 7 to 10 % faster.  LDS is busy in 19 % of the cycles.  A tile of K takes 1.3 to 1.5 us; an item's end 4 us, of the SwiGLU product 10 (activation
// 5.6, codes and stores 3.4, the next item's beginning 1).
//
// The activation's result leaves as rows in 8 bits: h replaces the gate's accumulators, its largest magnitude over the 128 columns is joined between
// lanes and, of SwiGLU, between the two wavefronts that share the columns, and a lane's codes are exchanged so that 16 of a row are stored at once.
#pragma once
#include <atomic>
#include <type_traits>

#include "matrix_f8.h"
#include "mfma_agpr.h"
#include "tile_plan.h"

namespace emoe {
namespace {

typedef int intx8 __attribute__((ext_vector_type(8)));
typedef int intx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef unsigned int uintx4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void;
typedef const int32_t __attribute__((address_space(1)))* global_i32;
typedef const __attribute__((address_space(1))) void global_void;

constexpr int NW = 4, WN = 2;
constexpr int TS = 8;                         // 16-row blocks of x of a wavefront
constexpr int WB = 8;                         // 16-row blocks of the matrix of a wavefront
constexpr int BM = 256;                       // rows of a tile
constexpr int TILE_BYTES = BM * kF8Block;     // 32 KiB per operand
constexpr int HALF_BYTES = TILE_BYTES / 2;
constexpr int LPW = 8;                        // load instructions of a wavefront for a tile of rows (half as many for half a matrix tile)
constexpr int kPending = LPW + LPW / 2 + LPW / 2;  // of one phase 1 and one phase 2: what may be in flight at a barrier
// LDS: matrix tiles, row tiles, then the powers
constexpr int kRowsAt = 2 * TILE_BYTES;
constexpr int kScalesAt = 4 * TILE_BYTES;     // of 256 rows, two groups of four K tiles
constexpr int kScaleGroup = BM * 4;
constexpr int kMatrixScalesAt = kScalesAt + 2 * kScaleGroup;  // 256 bytes a wavefront, two groups
constexpr int kTopsAt = kMatrixScalesAt + 2 * NW * 256;       // magnitudes of 128 rows a wavefront
constexpr size_t LDS_BYTES = kTopsAt + NW * 128 * 4;
constexpr int kPieceTiles = 4;                // K tiles (512 elements) of a piece of a leftover tile, at least
constexpr int kFixupGroups = (kMaxGroups - 1) * TS;  // workgroups of the fix-up launch: the most units there can be
constexpr int kPlanFloats = kTiledPlanBytes / 4;     // the plan sits ahead of the partial sums

#define INLINE __attribute__((always_inline))  // of closures, whose captures otherwise end up in memory
// f(i) for i = B .. E - 1, each i a constant of the type system: no loop that the compiler would have to unroll first
template <int B, int E, class F>
__device__ __forceinline__ void unrolled(F&& f) {
    if constexpr (B < E) {
        f(std::integral_constant<int, B>{});
        unrolled<B + 1, E>(f);
    }
}
template <int N>
using Number = std::integral_constant<int, N>;
typedef std::integral_constant<int, 0> First;   // half of a matrix tile
typedef std::integral_constant<int, 1> Second;

constexpr int wait_imm(int n) { return (n & 0xf) | ((n >> 4) << 14) | (0x7 << 4) | (0x0 << 8); }
// Workgroup barrier once at most N of this wavefront's loads are pending and all its LDS reads have returned.
template <int N>
__device__ __forceinline__ void barrier_keep_loads() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(wait_imm(N));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void* base, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)bytes, 0x00020000);
}
__device__ __forceinline__ int opaque(int v) {
    asm volatile("" : "+v"(v));
    return v;
}

// The scaled matrix instruction with its accumulators in AGPRs (see mfma_agpr.h, whose rules hold here too).  Powers are byte 0 of their
// registers; the first one of a phase comes behind wait states, for the powers are the results of shifts.
__device__ __forceinline__ void mfma_f8(floatx4& acc, const intx8& w, const intx8& x, uint32_t ws, uint32_t xs) {
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0]" : "+a"(acc) : "v"(w), "v"(x), "v"(ws), "v"(xs));
}
__device__ __forceinline__ void mfma_f8_first(floatx4& acc, const intx8& w, const intx8& x, uint32_t ws, uint32_t xs) {
    asm volatile("s_nop 1\n\tv_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, 0, %3, %4 op_sel_hi:[0,0,0]" : "=a"(acc) : "v"(w), "v"(x), "v"(ws), "v"(xs));
}
// a number where an accumulator was
__device__ __forceinline__ float acc_written(float v) {
    float a;
    asm volatile("v_accvgpr_write_b32 %0, %1" : "=a"(a) : "v"(v));
    return a;
}

// The 16 x 16 output blocks of a wavefront for its row block ts: from accumulators or from sums of pieces.  get(block, v) is a value.
// h of one row block: activation into put(block, v, h); -> the largest magnitude of the lane's
template <int EPI, class Get, class Put>
__device__ __forceinline__ uint32_t activate(Get get, Put put) {
    constexpr int NB = EPI == kF8Swiglu ? WB / 2 : WB;
    uint32_t top = 0;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            float g = get(b, v);
            if constexpr (EPI == kF8Swiglu) g = g * __builtin_amdgcn_rcpf(1.0f + __expf(-g)) * get(b + NB, v);  // (rcp: an ulp, 2^-20 of a code's step)
            else g = g < 0.0f ? 0.0f : g;  // (NaN stays)
            put(b, v, g);
            top = umax(top, f8_magnitude(g));
        }
    top = umax(top, (uint32_t)__shfl_xor((int)top, 16));
    return umax(top, (uint32_t)__shfl_xor((int)top, 32));
}
// Four blocks' codes of a row (64 columns), exchanged so that a lane has the 16 of block lane / 16
__device__ __forceinline__ uintx4 codes_of(const float (&h)[4][4], float inverse) {
    uint32_t c[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) c[b] = f8_codes(h[b][0], h[b][1], h[b][2], h[b][3], inverse);
    const auto p = __builtin_amdgcn_permlane16_swap(c[0], c[1], false, false), q = __builtin_amdgcn_permlane16_swap(c[2], c[3], false, false);
    const auto u = __builtin_amdgcn_permlane32_swap(p[0], q[0], false, false), v = __builtin_amdgcn_permlane32_swap(p[1], q[1], false, false);
    return uintx4{u[0], v[0], u[1], v[1]};
}
// Rows of h: `row` < 0 writes nothing.  TIES: and which elements are near ties (see kNearTie), for near_ties_kernel
template <int EPI, bool TIES, class Get>
__device__ __forceinline__ void store_h(const F8Product& p, Get get, uint32_t top, int row, int nt, int wn, int lane) {
    constexpr int HALVES = EPI == kF8Swiglu ? 1 : 2;  // of a block of 128 outputs, that a wavefront has
    const int nb = EPI == kF8Swiglu ? nt : 2 * nt + wn, half0 = EPI == kF8Swiglu ? wn : 0;
    const uint32_t byte = f8_scale_byte(top);
    const float inverse = f8_inverse(byte);
    uintx4 val[HALVES];
    uint32_t near[HALVES] = {};
#pragma unroll
    for (int i = 0; i < HALVES; ++i) {
        float h[4][4];
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int v = 0; v < 4; ++v) h[b][v] = get(4 * i + b, v);
        if constexpr (TIES) {
#pragma unroll
            for (int j = 15; j >= 0; --j) near[i] = f8_near_ties(near[i], h[j >> 2][j & 3] * inverse);
        }
        val[i] = codes_of(h, inverse);
    }
    if (row < 0 || nb >= p.lay.nb) return;
    uint8_t* to = p.h.codes + (size_t)row * p.h.row_step + (size_t)(nb * 8 + 4 * half0 + (lane >> 4)) * p.h.piece_step;
#pragma unroll
    for (int i = 0; i < HALVES; ++i) *reinterpret_cast<uintx4*>(to + (size_t)(4 * i) * p.h.piece_step) = val[i];
    if constexpr (TIES) {  // a line of 16 rows
        uint16_t* near_to = p.near + ((size_t)(2 * nb + half0) * p.rows + row) * 4 + (lane >> 4);
#pragma unroll
        for (int i = 0; i < HALVES; ++i) near_to[(size_t)(4 * i) * p.rows] = byte == 255u ? 0 : (uint16_t)near[i];
    }
    if (half0 == 0 && lane < 16) reinterpret_cast<uint8_t*>(p.h.scales + (size_t)(nb >> 2) * p.h.rows + row)[nb & 3] = (uint8_t)byte;
}
// bf16 rows of out; `row` < 0 writes nothing.  Two neighbouring blocks' columns are exchanged so that a lane has eight that follow each other.
template <class Get>
__device__ __forceinline__ void store_out(const F8Product& p, Get get, int row, int nt, int wn, int lane) {
    bf16_t* to = p.out + (size_t)(row < 0 ? 0 : row) * p.out_stride;
    const int col0 = nt * 256 + wn * 128 + ((lane >> 4) & 1) * 16 + (lane >> 5) * 8;
#pragma unroll
    for (int b = 0; b < WB; b += 2) {
        uint32_t two[2][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const bf16x4 o = __builtin_convertvector((floatx4{get(b + i, 0), get(b + i, 1), get(b + i, 2), get(b + i, 3)}), bf16x4);
            __builtin_memcpy(two[i], &o, 8);
        }
        const auto lo = __builtin_amdgcn_permlane16_swap(two[0][0], two[1][0], false, false);
        const auto hi = __builtin_amdgcn_permlane16_swap(two[0][1], two[1][1], false, false);
        const int n = col0 + b * 16;
        if (row >= 0 && n < p.N) *reinterpret_cast<uintx4*>(to + n) = uintx4{lo[0], hi[0], lo[1], hi[1]};
    }
}

__device__ __forceinline__ SlotTable group_table(const F8Product& p, int n_tiles, int lane) {
    int begin = 0, end = 0;
    if (lane < p.groups) {
        begin = p.offsets != nullptr ? p.offsets[lane] : 0;
        end = p.offsets != nullptr ? p.offsets[lane + 1] : p.rows;
        begin = begin > 0 ? begin : 0;
        end = end < p.rows ? end : p.rows;
        end = end > begin ? end : begin;
    }
    return make_slot_table(begin, end, n_tiles, lane);
}
// K tiles of the pieces of a tile begin at whole fours, which share a dword of powers
__device__ __forceinline__ int piece_begin(int KB, int splits, int sp) {
    return sp == splits ? KB : (int)((long long)KB * sp / splits) & ~3;
}

template <int EPI, bool TIES>
__device__ __forceinline__ void tiles(const F8Product& p, float* __restrict__ partials, int n_tiles, int XCDS) {
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int KB = p.lay.kb;  // K tiles, at least two
    const int G = gridDim.x;
    const SlotTable table = group_table(p, n_tiles, lane);
    const Plan plan = make_plan(table.total, KB, G, KB < kF8LeastCut ? KB : kPieceTiles);
    if (blockIdx.x == 0 && threadIdx.x == 0) *reinterpret_cast<int4*>(partials) = make_int4(plan.tiles, plan.rounds, plan.left, plan.splits);
    const int xcd = blockIdx.x % XCDS, cu = blockIdx.x / XCDS, per_xcd = G / XCDS;
    const int sk_item = xcd * per_xcd + cu;

    struct Item {
        int slot, row0, row_end, nt, slot_tiles;
        int kb, kt;  // its K tiles
        int piece;   // -1: a whole tile; else the number of the K piece of a leftover tile
    };
    auto item_at = [&](int idx, Item& it) INLINE {
        int L;
        it.kb = 0;
        it.kt = KB;
        it.piece = -1;
        if (idx < plan.rounds) {
            L = idx * G + xcd * per_xcd + cu;
        } else {
            if (idx > plan.rounds || sk_item >= plan.left * plan.splits) return false;
            L = plan.rounds * G + sk_item / plan.splits;
            if (plan.splits > 1) {
                const int sp = sk_item % plan.splits;
                it.kb = piece_begin(KB, plan.splits, sp);
                it.kt = piece_begin(KB, plan.splits, sp + 1) - it.kb;
                it.piece = sk_item;
            }
        }
        decode_tile(table, p.groups, n_tiles, lane, L, it.slot, it.row0, it.row_end, it.nt, it.slot_tiles);
        return true;
    };

    // ---- memory -> LDS ---------------------------------------------------------------------------------------
    const uint32_t x_bytes = (uint32_t)p.x.rows * (uint32_t)p.x.row_step;
    const __amdgpu_buffer_rsrc_t x_rsrc = make_rsrc(p.x.codes, x_bytes);
    const uint32_t xs_bytes = (uint32_t)p.x.rows * (uint32_t)p.lay.kg * 4u;
    const __amdgpu_buffer_rsrc_t xs_rsrc = make_rsrc(p.x.scales, xs_bytes);
    // A wavefront loads 64 rows of a tile: a lane looks up where row 64 wave + lane comes from
    auto load_perm = [&](const Item& it) INLINE {
        int r = it.row0 + 64 * wave + lane;
        r = r >= it.row_end ? it.row_end - 1 : r;
        return p.perm != nullptr ? global_i32(p.perm)[r] : r;
    };
    const uint32_t perm_div = p.perm != nullptr ? (uint32_t)p.k : 1u;
    uint32_t x_voff[LPW], xs_voff;
    auto row_addr = [&](const Item& it, int perm_entry) INLINE {
        const int l = opaque(lane);
        const uint32_t x_row = (uint32_t)perm_entry / perm_div;
        xs_voff = it.row0 + 64 * wave + l >= it.row_end ? xs_bytes : x_row * 4u;
#pragma unroll
        for (int i = 0; i < LPW; ++i) {
            const int tr = 64 * wave + 8 * i + (l >> 3);
            const uint32_t row = (uint32_t)__shfl((int)x_row, 8 * i + (l >> 3));
            const int v = opaque((int)(row * (uint32_t)p.x.row_step + ((l & 7) ^ ((tr >> 1) & 7)) * 16));
            x_voff[i] = it.row0 + tr >= it.row_end ? x_bytes : (uint32_t)v;  // out of range: zeros without memory traffic
        }
    };
    // where an item's matrix halves begin, and its powers (bytes from the group's matrix); this wavefront loads blocks 2 (wave % 2) and the next
    // of those of wavefront column wave / 2
    struct Panel {
        const uint8_t *first, *second;
        uint32_t at, at_apart;  // of the first half, and from there to the second
        const uint8_t* s0;
        int64_t s_apart;
    };
    uint32_t w_voff = lane * 16;
    auto panel_of = [&](const Item& it) INLINE {
        Panel o;
        o.first = p.w0 + (size_t)it.slot * p.matrix_bytes;
        o.second = EPI == kF8Swiglu ? p.w1 + (size_t)it.slot * p.matrix_bytes : o.first;
        const int mine = wave & 1, column = wave >> 1;
        const int last = p.lay.nb - 1;
        if (EPI == kF8Swiglu) {
            o.at = (uint32_t)it.nt * KB * kF8BlockBytes + (column * 4 + mine * 2) * kF8Strip;
            o.at_apart = 0;
            o.s0 = o.first + p.lay.codes() + (size_t)it.nt * p.lay.kg * 4;
            o.s_apart = o.second - o.first;
        } else {
            const int from = 2 * it.nt + column < last ? 2 * it.nt + column : last;
            o.at = (uint32_t)from * KB * kF8BlockBytes + mine * 2 * kF8Strip;
            o.at_apart = 4 * kF8Strip;
            const int nb = 2 * it.nt + wn < last ? 2 * it.nt + wn : last;
            o.s0 = o.first + p.lay.codes() + (size_t)nb * p.lay.kg * 4;
            o.s_apart = 0;
        }
        return o;
    };
    const uint32_t w_bytes = (uint32_t)p.lay.codes();
    auto issue_x = [&](int i, int to_place, int kb) INLINE {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(x_rsrc, (lds_void*)(lds + kRowsAt + to_place + (LPW * wave + i) * 1024), 16,
                                                 (int)x_voff[i], kb * kF8Block, 0, 0);
    };
    auto issue_w = [&](const Panel& o, auto half_c, int i, int to_place, int kb) INLINE {
        constexpr int half = decltype(half_c)::value;
        const uint8_t* from = o.first;
        if constexpr (half == 1) from = o.second;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(make_rsrc(from, w_bytes),
                                                 (lds_void*)(lds + to_place + half * HALF_BYTES + wave * 4096 + i * 1024), 16,
                                                 (int)w_voff, (int)(o.at + half * o.at_apart + (uint32_t)kb * kF8BlockBytes + i * 1024), 0, 0);
    };
    auto issue_scales = [&](const Panel& o, int parity, int kb) INLINE {
        const int group = kb >> 2;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(xs_rsrc, (lds_void*)(lds + kScalesAt + parity * kScaleGroup + wave * 256), 4, (int)xs_voff,
                                                 group * p.x.rows * 4, 0, 0);
        const uint8_t* s = o.s0 + (lane & 1) * o.s_apart + group * 4;
        __builtin_amdgcn_global_load_lds((global_void*)s, (lds_void*)(lds + kMatrixScalesAt + (parity * NW + wave) * 256), 4, 0, 0);
    };

    Item cur, nxt;
    if (!item_at(0, cur)) return;
    int perm_entry = load_perm(cur);
    row_addr(cur, perm_entry);
    Panel panel = panel_of(cur);
    int wanted = cur.kb;                // the K tile that is requested next: of this item up to its last, then of the next one
    bool there = true;                  // whether there is a tile to request
    int scale_put = 0, scale_get = 1;   // which of two places the next group of powers takes, and which the last one that was read has
    int kb_next = 0;                    // the K tile after the one that is multiplied
    int place = 0;                      // of the tile that is multiplied in LDS: 0 or TILE_BYTES
    // the first two tiles
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int kb = __builtin_amdgcn_readfirstlane(wanted);
        if ((kb & 3) == 0) {
            issue_scales(panel, scale_put, kb);
            scale_put ^= 1;
        }
#pragma unroll
        for (int i = 0; i < LPW; ++i) issue_x(i, t * TILE_BYTES, kb);
#pragma unroll
        for (int i = 0; i < LPW / 2; ++i) issue_w(panel, First{}, i, t * TILE_BYTES, kb);
#pragma unroll
        for (int i = 0; i < LPW / 2; ++i) issue_w(panel, Second{}, i, t * TILE_BYTES, kb);
        kb_next = kb;
        ++wanted;
    }
    barrier_keep_loads<0>();

    for (int idx = 0;; ++idx) {
        // the perm entries of the next item, which have this whole item to arrive in, and (with the combine folded in) the output rows of
        // this one: register h of a lane holds that of row 64 h + lane of this wavefront's 128
        const bool have_nxt = item_at(idx + 1, nxt);
        if (have_nxt) perm_entry = load_perm(nxt);
        int out_entry[2] = {0, 0};
        if (EPI == kF8Plain && p.out_perm != nullptr) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = cur.row0 + token_row(wm, 4 * h + (lane >> 4)) + (lane & 15);
                out_entry[h] = global_i32(p.out_perm)[r < cur.row_end ? r : cur.row_end - 1];
            }
        }

        // Everything that touches the matrix cores is compiled for NB = 0 .. TS row blocks; the accumulators live and die inside one instance.
        auto do_item = [&](auto nb_c) INLINE {
            constexpr int NB = decltype(nb_c)::value;
            floatx4 acc[WB][TS];
            mfma_settle();
            // fragments of this and the next tile; of the two halves of the matrix rows.  Powers of this and the next tile.
            intx8 xf[2][TS], wf[2][WB / 2];
            uint32_t sx[TS], sw[2];
            // This lane's place in the tile that is read: row lane % 16 of a block and of it chunks lane / 16 and 4 + lane / 16 of 16 bytes; 16 consecutive
            // bytes of a half strip; the powers.  (Opaque: none of it is to be held in registers from item to item.)
            const int l = opaque(lane), f_row = l & 15;
            int xo = kRowsAt + (token_row(wm, 0) + f_row) * kF8Block + ((l >> 4) ^ ((f_row >> 1) & 7)) * 16 + place;
            int wo = wn * 8192 + l * 16 + place;
            const int sx_off = kScalesAt + (token_row(wm, 0) + f_row) * 4, sw_off = kMatrixScalesAt + wave * 256;
            auto read = [&](int at, int second) INLINE {
                const intx4 a = *reinterpret_cast<const intx4*>(lds + at), b = *reinterpret_cast<const intx4*>(lds + second);
                return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
            };
            auto read_x = [&](auto to_c, auto f_c) INLINE {
                constexpr int to = decltype(to_c)::value, f = decltype(f_c)::value;
                if constexpr (f < NB) xf[to][f] = read(xo + token_row(0, f) * kF8Block, (xo ^ 64) + token_row(0, f) * kF8Block);
            };
            auto read_w = [&](auto half_c, auto b_c) INLINE {
                constexpr int half = decltype(half_c)::value, b = decltype(b_c)::value;
                if constexpr (NB > 0) wf[half][b] = read(wo + half * HALF_BYTES + b * kF8Strip, wo + half * HALF_BYTES + b * kF8Strip + 1024);
            };
            // The powers of the next tile, read once the tile that is multiplied no longer needs a register: number j of row block j, then of the two
            // halves of the matrix rows.  They come with those of three other tiles and are shifted behind the barrier.
            auto take_scale = [&](auto j_c) INLINE {
                constexpr int j = decltype(j_c)::value;
                if constexpr (j >= TS) sw[j - TS] = *reinterpret_cast<const uint32_t*>(lds + sw_off + scale_get * NW * 256 + 4 * (j - TS));
                else if constexpr (j < NB) sx[j] = *reinterpret_cast<const uint32_t*>(lds + sx_off + scale_get * kScaleGroup + token_row(0, j) * 4);
            };
            auto shift_scales = [&](int kb) INLINE {
                const int shift = (kb & 3) * 8;
#pragma unroll
                for (int j = 0; j < NB; ++j) sx[j] >>= shift;
                sw[0] >>= shift;
                sw[1] >>= shift;
            };
            // Blocks FROM .. TO - 1 of half of the matrix rows times all rows of x; behind a matrix instruction goes what work(i), i < WORK, does at
            // its place, and behind that of row block mi what done(mi) does.
            auto phase = [&](auto first_c, auto half_c, auto now_c, auto from_c, auto to_c, auto work_c, auto&& work, auto&& done) INLINE {
                constexpr int FROM = decltype(from_c)::value, TO = decltype(to_c)::value, WORK = decltype(work_c)::value, MF = (TO - FROM) * NB;
                if constexpr (NB == 0) {
                    unrolled<0, WORK>(work);
                } else {
                    unrolled<0, MF>([&](auto m_c) INLINE {
                        constexpr int m = decltype(m_c)::value, ni = FROM + m / NB;
                        constexpr int mi = (ni & 1) ? NB - 1 - m % NB : m % NB;  // back and forth: only one operand changes
                        constexpr int half = decltype(half_c)::value, now = decltype(now_c)::value;
                        floatx4& a = acc[half * (WB / 2) + ni][mi];
                        if constexpr (decltype(first_c)::value) mfma_f8_first(a, wf[half][ni], xf[now][mi], sw[half], sx[mi]);
                        else mfma_f8(a, wf[half][ni], xf[now][mi], sw[half], sx[mi]);
                        unrolled<(m * WORK + MF - 1) / MF, ((m + 1) * WORK + MF - 1) / MF>(work);
                        done(std::integral_constant<int, mi>{});
                    });
                }
            };

            // ---- main loop -------------------------------------------------------------------------------------
            // `now`: which registers the tile has.  A barrier lets pass once all but the kPending newest loads have landed: what the phase
            // behind it reads was requested three phases before.
            auto k_tile = [&](auto first_c, auto now_c, bool last) INLINE {
                constexpr int now = decltype(now_c)::value, other = now ^ 1;
                const auto nothing = [](auto) INLINE {};
                const int kb = __builtin_amdgcn_readfirstlane(wanted);
                if (there && (kb & 3) == 0) {
                    issue_scales(panel, scale_put, kb);
                    scale_put ^= 1;
                }
                __builtin_amdgcn_sched_barrier(0);
                phase(first_c, First{}, now_c, Number<0>{}, Number<4>{}, Number<4 + LPW + LPW / 2>{}, [&](auto i_c) INLINE {
                    constexpr int i = decltype(i_c)::value;
                    if constexpr (i < 4) read_w(Second{}, i_c);
                    else if constexpr (i < 4 + LPW) issue_x(i - 4, place, kb);
                    else issue_w(panel, First{}, i - 4 - LPW, place, kb);
                }, nothing);
                __builtin_amdgcn_sched_barrier(0);
                barrier_keep_loads<kPending>();
                __builtin_amdgcn_sched_barrier(0);
                xo ^= TILE_BYTES;
                wo ^= TILE_BYTES;
                phase(first_c, Second{}, now_c, Number<0>{}, Number<3>{}, Number<4 + TS>{}, [&](auto i_c) INLINE {
                    constexpr int i = decltype(i_c)::value;
                    if constexpr (i < 4) read_w(First{}, i_c);
                    else read_x(Number<other>{}, Number<i - 4>{});
                }, nothing);
                __builtin_amdgcn_sched_barrier(0);
                if (!last && (kb_next & 3) == 0) scale_get ^= 1;  // (the next item turns to its first for itself)
                __builtin_amdgcn_sched_barrier(0);
                take_scale(Number<TS>{});
                phase(first_c, Second{}, now_c, Number<3>{}, Number<4>{}, Number<LPW / 2>{},
                      [&](auto i_c) INLINE { issue_w(panel, Second{}, decltype(i_c)::value, place, kb); }, take_scale);
                take_scale(Number<TS + 1>{});
                __builtin_amdgcn_sched_barrier(0);
                const int kb_then = kb_next;
                kb_next = kb;
                place ^= TILE_BYTES;
                ++wanted;
                barrier_keep_loads<kPending>();
                __builtin_amdgcn_sched_barrier(0);
                shift_scales(kb_then);
                asm volatile("s_nop 1");  // before matrix instructions that the compiler does not see
                __builtin_amdgcn_sched_barrier(0);
            };
            // the last two K tiles request the next item's first two
            auto turn_to_next = [&]() INLINE {
                wanted = 0;
                there = have_nxt;
                if (have_nxt) {
                    row_addr(nxt, perm_entry);
                    panel = panel_of(nxt);
                    wanted = nxt.kb;
                } else {  // none: they go on, out of range: zeros land where nobody reads any more
#pragma unroll
                    for (int i = 0; i < LPW; ++i) x_voff[i] = x_bytes;
                    w_voff = w_bytes;
                }
                __builtin_amdgcn_sched_barrier(0);
            };

            unrolled<0, TS>([&](auto f) INLINE { read_x(First{}, f); });
            unrolled<0, WB / 2>([&](auto b) INLINE { read_w(First{}, b); });
            scale_get ^= 1;
            unrolled<0, TS + 2>(take_scale);  // (an item begins at a whole four: nothing to shift)
            barrier_keep_loads<63>();  // read by everyone: phase 1 requests into these places
            __builtin_amdgcn_sched_barrier(0);
            int left = cur.kt;
            if (left == 2) {
                __builtin_amdgcn_s_waitcnt(wait_imm(0));  // nothing has waited for the next item's perm entries yet
                turn_to_next();
            }
            k_tile(std::true_type{}, std::integral_constant<int, 0>{}, false);
            --left;
#pragma unroll 1
            for (; left >= 2; left -= 2) {
                if (left == 2) turn_to_next();
                k_tile(std::false_type{}, std::integral_constant<int, 1>{}, false);
                if (left == 3) turn_to_next();
                k_tile(std::false_type{}, std::integral_constant<int, 0>{}, left == 2);
            }
            if (left == 1) k_tile(std::false_type{}, std::integral_constant<int, 1>{}, true);
            mfma_settle();

            if (cur.piece >= 0) {  // a K piece of a leftover tile: raw accumulators to the workspace, [register][thread]
                float* dst = partials + kPlanFloats + (size_t)cur.piece * (BM * BM) + threadIdx.x;
#pragma unroll
                for (int i = 0; i < WB; ++i)
#pragma unroll
                    for (int j = 0; j < NB; ++j)  // (the fix-up skips blocks without rows)
#pragma unroll
                        for (int v = 0; v < 4; ++v) dst[((i * TS + j) * 4 + v) * (64 * NW)] = acc_read(acc[i][j][v]);
            } else if constexpr (EPI == kF8Plain) {
#pragma unroll
                for (int ts = 0; ts < NB; ++ts) {
                    int row = cur.row0 + token_row(wm, ts) + (lane & 15);
                    const bool ok = row < cur.row_end;
                    if (p.out_perm != nullptr) row = __shfl(out_entry[ts >> 2], (ts & 3) * 16 + (lane & 15));
                    store_out(p, [&](int b, int v) INLINE { return acc_read(acc[b][ts][v]); }, ok ? row : -1, cur.nt, wn, lane);
                    __builtin_amdgcn_sched_barrier(0);  // a block at a time: the accumulators stay where they are until used
                }
            } else if constexpr (EPI == kF8Relu) {
#pragma unroll
                for (int ts = 0; ts < NB; ++ts) {
                    float h[WB][4];
                    const uint32_t top = activate<EPI>([&](int b, int v) { return acc_read(acc[b][ts][v]); }, [&](int b, int v, float x) { h[b][v] = x; });
                    const int row = cur.row0 + token_row(wm, ts) + (lane & 15);
                    store_h<EPI, TIES>(p, [&](int b, int v) { return h[b][v]; }, top, row < cur.row_end ? row : -1, cur.nt, wn, lane);
                    __builtin_amdgcn_sched_barrier(0);
                }
            } else {
                uint32_t tops[TS];
                uint32_t* shared_tops = reinterpret_cast<uint32_t*>(lds + kTopsAt);
#pragma unroll
                for (int ts = 0; ts < NB; ++ts) {
                    tops[ts] = activate<EPI>([&](int b, int v) { return acc_read(acc[b][ts][v]); },
                                             [&](int b, int v, float h) { acc[b][ts][v] = acc_written(h); });
                    if (lane < 16) shared_tops[wave * 128 + ts * 16 + lane] = tops[ts];
                    __builtin_amdgcn_sched_barrier(0);
                }
                barrier_keep_loads<63>();
#pragma unroll
                for (int ts = 0; ts < NB; ++ts) {
                    const uint32_t top = umax(tops[ts], shared_tops[(wave ^ 1) * 128 + ts * 16 + (lane & 15)]);
                    const int row = cur.row0 + token_row(wm, ts) + (lane & 15);
                    store_h<EPI, TIES>(p, [&](int b, int v) { return acc_read(acc[b][ts][v]); }, top, row < cur.row_end ? row : -1, cur.nt, wn, lane);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        };
        // Blocks without rows are skipped in groups of up to kBlockM tiles (one block of tile_in_slot); in a taller one the ragged tile multiplies its
        // padding and stays in step with the others, with whom it shares operand panels in L2.
        const int my_blocks = cur.slot_tiles > kSkipBlocksUpToTiles ? TS : blocks_of_wavefront(cur.row0, cur.row_end, wm);
        if (my_blocks >= 8) do_item(std::integral_constant<int, 8>{});
        else if (my_blocks == 7) do_item(std::integral_constant<int, 7>{});
        else if (my_blocks == 6) do_item(std::integral_constant<int, 6>{});
        else if (my_blocks == 5) do_item(std::integral_constant<int, 5>{});
        else if (my_blocks == 4) do_item(std::integral_constant<int, 4>{});
        else if (my_blocks == 3) do_item(std::integral_constant<int, 3>{});
        else if (my_blocks == 2) do_item(std::integral_constant<int, 2>{});
        else if (my_blocks == 1) do_item(std::integral_constant<int, 1>{});
        else do_item(std::integral_constant<int, 0>{});
        if (!have_nxt) break;
        cur = nxt;
    }
    barrier_keep_loads<0>();  // the surplus loads must not outlive the workgroup's LDS
}

// Adds the K pieces of each leftover tile in piece order and finishes it.  A workgroup takes the row blocks ts of both wavefront rows of a
// tile, in the places of the wavefronts that left them.  The plan is read from the head of the workspace: where nothing was
// cut, every workgroup exits after one load.
template <int EPI, bool TIES>
__global__ __launch_bounds__(64 * NW) void fixup_kernel(F8Product p, const float* __restrict__ partials, int n_tiles, int G) {
    __shared__ uint32_t shared_tops[NW][16];
    const int4 hdr = *reinterpret_cast<const int4*>(partials);
    const Plan plan{hdr.x, hdr.y, hdr.z, hdr.w};
    if (plan.splits <= 1) return;
    const int u = blockIdx.x;
    if (u >= plan.left * TS) return;
    const int tile = u / TS, ts = u % TS;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / WN, wn = wave % WN;
    int slot, row0, row_end, nt, slot_tiles;
    const SlotTable table = group_table(p, n_tiles, lane);
    decode_tile(table, p.groups, n_tiles, lane, plan.rounds * G + tile, slot, row0, row_end, nt, slot_tiles);
    const bool rows = row0 + token_row(wm, ts) < row_end;  // else nothing was written
    float sum[WB][4];
#pragma unroll
    for (int b = 0; b < WB; ++b)
#pragma unroll
        for (int v = 0; v < 4; ++v) sum[b][v] = 0.0f;
    for (int sp = 0; rows && sp < plan.splits; ++sp) {
        const float* src = partials + kPlanFloats + (size_t)(tile * plan.splits + sp) * (BM * BM) + threadIdx.x;
        float g[WB][4];  // all loads of a piece in flight together, then the adds
#pragma unroll
        for (int b = 0; b < WB; ++b)
#pragma unroll
            for (int v = 0; v < 4; ++v) g[b][v] = src[((b * TS + ts) * 4 + v) * (64 * NW)];
#pragma unroll
        for (int b = 0; b < WB; ++b)
#pragma unroll
            for (int v = 0; v < 4; ++v) sum[b][v] += g[b][v];
    }
    const int r = row0 + token_row(wm, ts) + (lane & 15);
    auto get = [&](int b, int v) { return sum[b][v]; };
    if constexpr (EPI == kF8Plain) {
        store_out(p, get, r < row_end ? (p.out_perm != nullptr ? p.out_perm[r] : r) : -1, nt, wn, lane);
    } else {
        uint32_t top = activate<EPI>(get, [&](int b, int v, float h) { sum[b][v] = h; });
        if constexpr (EPI == kF8Swiglu) {
            if (lane < 16) shared_tops[wave][lane] = top;
            __syncthreads();
            top = umax(top, shared_tops[wave ^ 1][lane & 15]);
        }
        store_h<EPI, TIES>(p, get, top, r < row_end ? r : -1, nt, wn, lane);
    }
}

// The product by KERNEL, an instance of tiles<EPI, TIES>, and its leftover tiles
template <int EPI, bool TIES, auto KERNEL>
hipError_t launch_tiles(const F8Product& p, float* partials, const DeviceShape& shape, hipStream_t st) {
    static std::atomic<uint64_t> devices_set{0};  // set once per kernel and device; setting it twice from two threads is harmless
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return e;
    const uint64_t bit = 1ull << (device & 63);
    if (!(devices_set.load(std::memory_order_acquire) & bit)) {
        e = hipFuncSetAttribute(reinterpret_cast<const void*>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, (int)LDS_BYTES);
        if (e != hipSuccess) return e;
        devices_set.fetch_or(bit, std::memory_order_release);
    }
    const int n_tiles = EPI == kF8Swiglu ? p.lay.nb : (p.lay.nb + 1) / 2;
    KERNEL<<<shape.groups, 64 * NW, LDS_BYTES, st>>>(p, partials, n_tiles, shape.xcds);
    if (p.lay.kb >= kF8LeastCut) fixup_kernel<EPI, TIES><<<kFixupGroups, 64 * NW, 0, st>>>(p, partials, n_tiles, shape.groups);
    return hipGetLastError();
}

}  // namespace
}  // namespace emoe
