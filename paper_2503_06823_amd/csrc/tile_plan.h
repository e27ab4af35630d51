// Which workgroup of a persistent launch takes which output tiles of a grouped product, for the kernels with tiles of 256 rows by four
// wavefronts (2 x 2): groups' sizes live on the device, and every workgroup derives its tiles from the offsets.
#pragma once
#include "common.h"

namespace emoe {
namespace {

constexpr int kTileRows = 256;
constexpr int kMaxSplits = 8;  // K pieces per leftover tile, at most

// ---- work distribution ------------------------------------------------------------------------
// The launch is persistent: one workgroup per CU.  Output tiles are numbered in (slot, n-tile,
// m-tile) order of tile_in_slot.  The first `rounds * G` tiles are dealt out whole, `rounds` per
// workgroup, so that the 32 workgroups of an XCD hold 32 consecutive tiles at any time (one weight
// panel and the slot's token panels stay in that XCD's L2).  Round r covers tiles r*G .. (r+1)*G-1,
// 32 for each XCD: every XCD works its way through all slots, so slots whose tiles cost less (fewer
// rows than a tile holds) do not leave some XCDs idle while others still work (a contiguous range of
// tiles per XCD took 4-7 % longer at 250-500 rows per slot).  The `left` tiles that do not fill a
// round are split along K into `splits` pieces each, so that they too occupy (nearly) every CU: a
// piece writes its fp32 accumulators to the workspace and a small second kernel adds the pieces in
// order and applies the epilogue.  Everything is derived from slot_offsets on the device.
struct Plan {
    int tiles;   // output tiles in total
    int rounds;  // whole tiles per workgroup
    int left;    // tiles beyond rounds * G
    int splits;  // K pieces per leftover tile (1 = none)
};

// `least`: K tiles of a piece
__device__ __forceinline__ Plan make_plan(int tiles, int k_tiles, int G, int least) {
    Plan p;
    p.tiles = tiles;
    p.rounds = p.tiles / G;
    p.left = p.tiles - p.rounds * G;
    int sp = p.left > 0 ? G / p.left : 1;
    const int by_k = k_tiles / least;
    sp = sp < by_k ? sp : by_k;
    sp = sp > kMaxSplits ? kMaxSplits : sp;
    p.splits = sp < 1 ? 1 : sp;
    return p;
}

// Order of a slot's m_tiles x n_tiles output tiles.  The 32 workgroups of an XCD hold 32 consecutive
// tiles at any time and their L2 has to supply one operand panel per distinct m-tile and per
// distinct n-tile among them, so consecutive tiles should form compact blocks: the n-tiles are
// taken four at a time, and inside such a group of columns the m-tiles eight at a time, m fastest
// (12 panels for 32 tiles; m fastest over a whole tall slot would need up to 33).
// rem = number of the tile within the slot -> its m-tile and n-tile.
constexpr int kBlockM = 8, kBlockN = 4;
constexpr int kSkipBlocksUpToTiles = kBlockM;  // see the K loop's dispatch
__device__ __forceinline__ void tile_in_slot(int rem, int m_tiles, int n_tiles, int& mt, int& nt) {
    const int group = rem / (m_tiles * kBlockN);  // group of up to four n-tiles
    const int gn = n_tiles - group * kBlockN < kBlockN ? n_tiles - group * kBlockN : kBlockN;
    int r = rem - group * (m_tiles * kBlockN);
    const int full = m_tiles / kBlockM;           // whole blocks of eight m-tiles
    int mb = kBlockM, m0 = 0;
    if (r < full * kBlockM * gn) {
        m0 = (r / (kBlockM * gn)) * kBlockM;
        r %= kBlockM * gn;
    } else {
        r -= full * kBlockM * gn;
        m0 = full * kBlockM;
        mb = m_tiles - m0;
    }
    mt = m0 + r % mb;
    nt = group * kBlockN + r / mb;
}

// Rows per m-tile of a slot of `rows` rows cut into `tiles` tiles: the rows are spread evenly (in
// whole 16-row MFMA blocks), so that a slot of 257 rows becomes tiles of 144 and 113 rows instead of
// 256 and 1.  A tile costs a pass over its weight panel whatever it holds; what is saved is the
// matrix work of the blocks without rows, which both tiles then skip.
__device__ __forceinline__ int rows_per_tile(int rows, int tiles) {
    const int even = (rows + tiles - 1) / (tiles > 0 ? tiles : 1);
    return (even + 15) & ~15;  // <= kTileRows, so tile number `tiles - 1` still starts inside the slot
}

// Which wavefronts multiply which of a tile's 16-row token blocks: the blocks alternate between
// the two wavefront rows, so that both finish together whatever the number of blocks that hold rows.
// -> first tile row of block j of wavefront row wm, and the number of its blocks that hold rows.
__device__ __forceinline__ int token_row(int wm, int j) { return (2 * j + wm) * 16; }
__device__ __forceinline__ int blocks_of_wavefront(int row0, int row_end, int wm) {
    return ((row_end - row0 + 15) / 16 - wm + 1) / 2;
}

// The slot table in registers: lane s of every wavefront holds slot s's row range and the number of
// the first output tile of that slot, so that finding a tile's slot is one ballot and three lane
// reads instead of a walk over slot_offsets in memory (a few thousand cycles per tile).
struct SlotTable {
    int begin, end;  // rows of slot `lane`
    int tiles;       // m-tiles of slot `lane`
    int first;       // number of the slot's first output tile (exclusive prefix of tiles * n_tiles)
    int total;       // all output tiles (uniform)
};

__device__ __forceinline__ SlotTable make_slot_table(int begin, int end, int n_tiles, int lane) {
    SlotTable t;
    t.begin = begin;
    t.end = end;
    t.tiles = (t.end - t.begin + kTileRows - 1) / kTileRows;
    const int span = t.tiles * n_tiles;
    int incl = span;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int up = __shfl_up(incl, off);
        if (lane >= off) incl += up;
    }
    t.first = incl - span;
    t.total = __builtin_amdgcn_readlane(incl, 63);
    return t;
}

__device__ __forceinline__ SlotTable make_slot_table(const int32_t* __restrict__ offsets, int S, int n_tiles, int lane) {
    return make_slot_table(lane < S ? offsets[lane] : 0, lane < S ? offsets[lane + 1] : 0, n_tiles, lane);
}

__device__ __forceinline__ void decode_tile(const SlotTable& t, int S, int n_tiles, int lane, int L, int& slot,
                                            int& row0, int& row_end, int& nt, int& slot_tiles) {
    // slots are in tile order and an empty slot starts where its successor does: the last slot that
    // starts at or before L is the non-empty one that holds it
    const unsigned long long m = __ballot(lane < S && t.first <= L);
    slot = __popcll(m) - 1;
    const int rem = L - __builtin_amdgcn_readlane(t.first, slot);
    const int tiles = __builtin_amdgcn_readlane(t.tiles, slot);
    int mt;
    tile_in_slot(rem, tiles, n_tiles, mt, nt);
    const int b = __builtin_amdgcn_readlane(t.begin, slot), e = __builtin_amdgcn_readlane(t.end, slot);
    const int rpt = rows_per_tile(e - b, tiles);
    row0 = b + mt * rpt;
    row_end = row0 + rpt < e ? row0 + rpt : e;
    slot_tiles = tiles;
}

}  // namespace
}  // namespace emoe
