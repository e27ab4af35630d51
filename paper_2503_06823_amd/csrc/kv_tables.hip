// Block tables, slot maps and the ring of free pages of the paged cache, from the requests' lengths, without the host
// (Section 3.5's scheduler decides on the host who runs; where their tokens go is decided here).
//
// Both operators are a prefix sum over the requests followed by a copy, bound by the time of one launch and of a few dependent
// reads, not by bytes.  So each is one launch: every workgroup makes the prefix sums it needs for itself, 1024 rows a trip,
// instead of a launch for the sums and one for the copies.  A workgroup of emoe_kv_plan owns 1024 tokens, finds the rows that
// they belong to by a running maximum over the places where rows begin, and the token that is first on a new page writes the
// table's entry.  A workgroup of emoe_kv_release owns 16 rows, a wavefront each.  Prefix sums within a wavefront go by DPP, not through
// LDS.  Measured: a plan of 64 requests with a token each 4.0 us, of 1000 requests with 16240 tokens 5.9; a release of 64 requests
// 3.2 us, of 1000 with windows 4.1; a launch that does nothing takes 2.
#include "kv_cache.h"

namespace emoe {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kReleaseRows = kWaves;
constexpr int kAdvanceThreads = 256;

// Inclusive prefix sums over the workgroup of N values a thread, and the sums of all.
template <int N>
__device__ __forceinline__ void block_scan(long long (&v)[N], long long (*totals)[kWaves], long long (&sums)[N]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = wave_inclusive(v[n]);
    __syncthreads();  // the totals of an earlier scan are read
    if (lane == 63) {
#pragma unroll
        for (int n = 0; n < N; ++n) totals[n][wave] = v[n];
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {  // 16 wavefronts' totals in 16 lanes
        const long long all = wave_inclusive(lane < kWaves ? totals[n][lane < kWaves ? lane : 0] : 0ll);
        sums[n] = readlane(all, kWaves - 1);
        v[n] += wave > 0 ? readlane(all, wave > 0 ? wave - 1 : 0) : 0ll;
    }
}

__device__ __forceinline__ int ring_index(int start, long long by, int pages) {
    long long i = start + by;
    while (i >= pages) i -= pages;
    return (int)i;
}

__global__ __launch_bounds__(kThreads) void kv_plan_kernel(int R, int T, int pages, int width, int log2_page,
                                                           const int32_t* __restrict__ len, const int32_t* __restrict__ new_len,
                                                           int32_t* table, const int32_t* __restrict__ free_pages,
                                                           const int64_t* __restrict__ counters, int32_t* __restrict__ cu_new,
                                                           int32_t* __restrict__ slot, int32_t* __restrict__ position,
                                                           int32_t* __restrict__ seq_len, int64_t* __restrict__ counters_out,
                                                           int32_t* __restrict__ refused) {
    __shared__ long long totals[2][kWaves];
    __shared__ int row_at[kThreads], pos0_at[kThreads], have_at[kThreads], base_at[kThreads];  // of the row that begins at this token
    __shared__ int last_of_wave[kWaves], refusals;
    const int i = threadIdx.x, lane = i & 63, wave = __builtin_amdgcn_readfirstlane(i >> 6);
    const int s0 = blockIdx.x * kThreads;
    const long long s1 = (long long)s0 + kThreads;
    const bool rows_too = blockIdx.x == 0;  // this workgroup writes what there is one of per row
    row_at[i] = -1;
    if (i == 0) refusals = 0;
    const long long head = counters[0], tail = counters[1];
    const long long free_now = tail - head < 0 ? 0 : tail - head > pages ? pages : tail - head;
    const long long P = 1ll << log2_page;

    long long tokens = 0, wanted = 0, taken = 0;  // of the rows of the trips before
    for (int r0 = 0; r0 < R && (rows_too || tokens < s1); r0 += kThreads) {
        const int r = r0 + i;
        const bool there = r < R;
        const int l_in = there ? len[r] : 0, n_in = there ? new_len[r] : 0;
        const long long l = l_in > 0 ? l_in : 0, n = n_in > 0 ? n_in : 0;
        const long long have = (l + P - 1) >> log2_page, want = (l + n + P - 1) >> log2_page;
        bool fits = want <= width;
        // tokens and pages in one go, as if all tokens found a place: a second scan only where some do not
        long long upto[2] = {n, fits ? want - have : 0}, sum[2];
        block_scan<2>(upto, totals, sum);
        const long long cu_end = tokens + upto[0], cu = cu_end - n;
        if (tokens + sum[0] > T) {
            fits &= cu_end <= T;
            long long again[1] = {fits ? want - have : 0}, again_sum[1];
            block_scan<1>(again, totals, again_sum);
            upto[1] = again[0];
            sum[1] = again_sum[0];
        }
        tokens += sum[0];
        const long long need = fits ? want - have : 0, all_upto = wanted + upto[1], base = all_upto - need;
        wanted += sum[1];
        const bool ok = fits && (need == 0 || all_upto <= free_now);
        if (rows_too) {
            if (wanted <= free_now) taken = wanted;
            else {
                long long got[1] = {ok ? need : 0}, got_sum[1];
                block_scan<1>(got, totals, got_sum);
                taken += got_sum[0];
            }
            if (there) {
                constexpr long long most = 0x7fffffff;
                if (r == 0) cu_new[0] = 0;
                cu_new[r + 1] = (int)(cu_end < most ? cu_end : most);
                seq_len[r] = ok ? (int)(l + n) : 0;
                if (!ok) atomicAdd(&refusals, 1);
            }
        }
        if (n > 0 && cu < s1 && cu_end > s0) {
            const int at = cu > s0 ? (int)(cu - s0) : 0;
            row_at[at] = r;
            pos0_at[at] = (int)(l - cu);  // the position of token t is pos0 + t: l and cu are below 2^31
            have_at[at] = ok ? (int)have : -1;
            base_at[at] = ok ? (int)base : 0;
        }
    }
    __syncthreads();
    if (rows_too && i == 0) {
        if (R == 0) cu_new[0] = 0;
        counters_out[0] = head + taken;
        counters_out[1] = tail;
        *refused = refusals;
    }
    // the row of a token: the last one that begins at it or before it
    int from = row_at[i] >= 0 ? i : -1;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
        const int o = __shfl_up(from, s);
        if (lane >= s && o > from) from = o;
    }
    if (lane == 63) last_of_wave[wave] = from;
    __syncthreads();
    for (int w = 0; w < wave; ++w) from = last_of_wave[w] > from ? last_of_wave[w] : from;
    const long long t = (long long)s0 + i;
    if (t >= T) return;
    if (from < 0 || t >= tokens) {
        slot[t] = position[t] = -1;
        return;
    }
    const int row = row_at[from], have = have_at[from], pos = pos0_at[from] + (int)t;
    const int start = (int)((unsigned long long)head % (unsigned)pages);
    position[t] = pos;
    if (have < 0) {
        slot[t] = -1;
        return;
    }
    const int b = pos >> log2_page, in_page = pos & (int)(P - 1);
    int32_t* entry = table + (size_t)row * width + b;
    int page;
    if (b < have) page = *entry;
    else {
        page = free_pages[ring_index(start, (long long)base_at[from] + b - have, pages)];
        if (in_page == 0) *entry = page;  // the first token of a new page is always among the new ones
    }
    slot[t] = (unsigned)page < (unsigned)pages ? (page << log2_page) + in_page : -1;
}

// The pages that a row gives back: 0 .. first-1 and from .. to-1.
struct Leaving {
    int first, from, to;
    __device__ int count() const { return first + (to > from ? to - from : 0); }
};

__device__ __forceinline__ Leaving leaving(int before, int now, bool ended, int window, int sinks, int log2_page) {
    const long long P = 1ll << log2_page;
    const int have = (int)((((long long)(now > 0 ? now : 0)) + P - 1) >> log2_page);
    if (window == 0) return {0, 0, ended ? have : 0};
    const int kept = (int)(((long long)sinks + P - 1) >> log2_page), first = kept < have ? kept : have;
    // pages before this one hold no token that a query at position n or later sees, but for the sinks'
    auto dropped = [&](int n) {
        const long long d = ((long long)n - window + 1) >> log2_page;
        return d < first ? first : d < have ? (int)d : have;
    };
    return {ended ? first : 0, dropped(before), ended ? have : dropped(now)};
}

__global__ __launch_bounds__(kThreads) void kv_release_kernel(int R, int pages, int width, int log2_page, int window, int sinks,
                                                              const int32_t* __restrict__ len_before, const int32_t* __restrict__ len,
                                                              const int32_t* __restrict__ ended, const int32_t* __restrict__ table,
                                                              int32_t* __restrict__ free_pages, const int64_t* __restrict__ counters,
                                                              int64_t* __restrict__ counters_out) {
    __shared__ long long totals[1][kWaves];
    __shared__ long long base_of[kReleaseRows];
    __shared__ Leaving rows[kReleaseRows];
    const int i = threadIdx.x, lane = i & 63, wave = __builtin_amdgcn_readfirstlane(i >> 6);
    const int own = blockIdx.x * kReleaseRows;
    const bool last = blockIdx.x == gridDim.x - 1;
    const long long tail = counters[1];
    long long before = 0;
    for (int r0 = 0; r0 < R && (r0 < own + kReleaseRows || last); r0 += kThreads) {
        const int r = r0 + i;
        Leaving l = {0, 0, 0};
        if (r < R) {
            const int held = len_before != nullptr ? len_before[r] : 0, now = len[r];
            l = leaving(held, now > held ? now : held, ended != nullptr && ended[r] != 0, window, sinks, log2_page);
            if (l.to > width) l.to = width;  // a length that the table cannot hold
            if (l.first > width) l.first = width;
        }
        long long upto[1] = {l.count()}, sum[1];
        block_scan<1>(upto, totals, sum);
        if (r >= own && r < own + kReleaseRows) {
            rows[r - own] = l;
            base_of[r - own] = before + upto[0] - l.count();
        }
        before += sum[0];
    }
    __syncthreads();
    if (last && i == 0) {
        counters_out[0] = counters[0];
        counters_out[1] = tail + before;
    }
    const int r = own + wave;
    if (r >= R) return;
    const Leaving l = rows[wave];
    const int n = l.count(), start = (int)(((unsigned long long)tail + (unsigned long long)base_of[wave]) % (unsigned)pages);
    const int32_t* row = table + (size_t)r * width;
    for (int k = lane; k < n; k += 64) free_pages[ring_index(start, k, pages)] = row[k < l.first ? k : l.from + k - l.first];
}

__global__ __launch_bounds__(kAdvanceThreads) void kv_advance_kernel(int R, const int32_t* __restrict__ seq_len, const int32_t* __restrict__ ended,
                                                                     int32_t* __restrict__ len) {
    const int r = blockIdx.x * kAdvanceThreads + threadIdx.x;
    if (r >= R) return;
    const int held = len[r], now = seq_len[r];
    len[r] = ended != nullptr && ended[r] != 0 ? 0 : now > held ? now : held;
}

}  // namespace

hipError_t launch_kv_plan(const emoe_kv_desc& d, int T, const int32_t* len, const int32_t* new_len, int32_t* table,
                          const int32_t* free_pages, const int64_t* counters, int32_t* cu_new, int32_t* slot, int32_t* position,
                          int32_t* seq_len, int64_t* counters_out, int32_t* refused, hipStream_t st) {
    const unsigned groups = T > 0 ? (unsigned)(((long long)T + kThreads - 1) / kThreads) : 1u;
    kv_plan_kernel<<<groups, kThreads, 0, st>>>(d.rows, T, d.pages, d.table_width, log2_of(d.page_size), len, new_len, table, free_pages,
                                                counters, cu_new, slot, position, seq_len, counters_out, refused);
    return hipGetLastError();
}

hipError_t launch_kv_release(const emoe_kv_desc& d, const int32_t* len_before, const int32_t* len, const int32_t* ended, int window,
                             int sinks, const int32_t* table, int32_t* free_pages, const int64_t* counters, int64_t* counters_out,
                             hipStream_t st) {
    const unsigned groups = d.rows > 0 ? (unsigned)((d.rows + kReleaseRows - 1) / kReleaseRows) : 1u;
    kv_release_kernel<<<groups, kThreads, 0, st>>>(d.rows, d.pages, d.table_width, log2_of(d.page_size), window, sinks, len_before, len,
                                                   ended, table, free_pages, counters, counters_out);
    return hipGetLastError();
}

hipError_t launch_kv_advance(const emoe_kv_desc& d, const int32_t* seq_len, const int32_t* ended, int32_t* len, hipStream_t st) {
    kv_advance_kernel<<<(unsigned)((d.rows + kAdvanceThreads - 1) / kAdvanceThreads), kAdvanceThreads, 0, st>>>(d.rows, seq_len, ended, len);
    return hipGetLastError();
}

}  // namespace emoe
