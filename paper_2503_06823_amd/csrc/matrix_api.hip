// C ABI of the matrices in 8 bits and of the products with them: host-side argument checks, workspace layout, and the experts' FFN
// in that form.  The operations are documented in include/emoe.h.
#include "matrix_f8.h"

namespace emoe {
namespace {

constexpr long long kMostExtent = 1ll << 31;
bool unaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }
int status_of(hipError_t e) { return e == hipSuccess ? EMOE_OK : EMOE_ERR_DEVICE; }
long long whole(long long n) { return (n + kF8Block - 1) / kF8Block * kF8Block; }
size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

int validate_matrix(int32_t N, int32_t K) {
    if (N <= 0 || K <= 0) return EMOE_ERR_SHAPE;
    if (N % 8 != 0 || K % 8 != 0) return EMOE_ERR_UNSUPPORTED;
    if (whole(N) * whole(K) >= kMostExtent) return EMOE_ERR_SHAPE;
    return EMOE_OK;
}

int validate_matrices(int32_t count, int32_t N, int32_t K, int32_t dtype, int64_t stride) {
    int rc = validate_matrix(N, K);
    if (rc != EMOE_OK) return rc;
    if (dtype != EMOE_F32 && dtype != EMOE_BF16) return EMOE_ERR_UNSUPPORTED;
    if (count < 0 || stride < K) return EMOE_ERR_SHAPE;
    if (count > 65535 || stride % 8 != 0) return EMOE_ERR_UNSUPPORTED;
    return EMOE_OK;
}

int validate_matmul(const emoe_matmul_desc* d) {
    if (d == nullptr) return EMOE_ERR_NULL;
    int rc = validate_matrix(d->N, d->K);
    if (rc != EMOE_OK) return rc;
    if (d->dtype != EMOE_BF16 || d->reserved != 0) return EMOE_ERR_UNSUPPORTED;
    if (d->rows < 0 || d->groups <= 0 || d->x_stride < d->K || d->out_stride < d->N) return EMOE_ERR_SHAPE;
    if (d->groups > kMaxExperts || d->x_stride % 8 != 0 || d->out_stride % 8 != 0) return EMOE_ERR_UNSUPPORTED;
    if ((d->rows + 2ll) * (whole(d->N) > whole(d->K) ? whole(d->N) : whole(d->K)) > kMostExtent) return EMOE_ERR_SHAPE;
    return EMOE_OK;
}

// Rows in 8 bits at `at`, and what follows them.
F8Rows rows_at(uint8_t* ws, size_t* at, long long rows, int K) {
    F8Rows r = {};
    r.codes = ws + *at;
    r.rows = (int)rows;
    *at = align256(*at + (size_t)rows * whole(K));
    r.scales = reinterpret_cast<uint32_t*>(ws + *at);
    *at = align256(*at + f8_rows_scale_bytes(rows, K));
    return r;
}

// Which kernel multiplies, by the rows (how many each group has lives on the device: half a stretch of 64 more than they fill is what groups of unequal
// sizes have on average).  Streaming reads a matrix once for every 64 rows of a group, from caches after the first; tiles of 256 x 256 read it once, but cost some 10 us
// more and leave CUs without work where they are few.  So streaming it is where one reading does, and where its workgroups are few or short.  Measured with matrices
// from HBM (us, streaming / tiles): one of 6144 x 4096 64 rows 15.7 / 25.9, 256 28.4 / 37.6, 512 40.1 / 41.1; 32000 x 4096 64 rows 33.0 / 47.9, 80
// 53.8 / 47.7; 1024 x 1024 1024 rows 10.9 / 23.4; 8 of 14336 x 4096 64 rows each 104 / 109, 80 185 / 109; 8 of 2048 x 2048 128 23.8 / 29.2, 256 35.1 / 36.5, 320
// 47.0 / 32.3; 24 of 2048 x 1408 64 31.0 / 27.0, 80 41.0 / 28.0.  SwiGLU's two: 6 groups of 14336 x 4096 64 rows 144 / 146, 80 254 / 156; 4 of 4096 x 1024
// 128 21.0 / 23.6; one of 14336 x 4096 128 51.3 / 50.2, 160 79.5 / 50.0; ReLU 128 30.7 / 36.8, 160 43.6 / 37.9; 16 of 2816 x 1032 64 24.3 / 23.1, 80
// 35.1 / 24.4.  Tiles take at least two blocks of columns.  What goes by averages is wrong about a group that has most of the rows: 3000 of 64 groups of 6144 x
// 4096 stream in 371 us spread evenly, in 426 with half of them in one group, in 226 with all of them there, which tiles of one group take 91 for.
bool is_tiled(long long rows, int groups, int N, int K, F8Epilogue epilogue) {
    if (K <= kF8Block || rows <= (groups == 1 ? 64ll : 48ll) * groups) return false;
    const bool plain = epilogue == kF8Plain;
    const long long stretches = groups == 1 ? (rows + 63) / 64 : (rows + 32ll * groups) / 64;
    const long long workgroups = stretches * (plain ? (N + 63) / 64 : (N + 127) / 128);
    return plain ? workgroups > 512 || workgroups * K > 1ll << 21 : workgroups > 384 || workgroups * K > 1ll << 20;
}
bool first_is_tiled(const emoe_layer_desc& d) {
    return is_tiled((long long)d.T * d.k, d.S, d.d_ff, d.d_model, d.act == EMOE_ACT_SWIGLU ? kF8Swiglu : kF8Relu);
}
bool second_is_tiled(const emoe_layer_desc& d) { return is_tiled((long long)d.T * d.k, d.S, d.d_model, d.d_ff, kF8Plain); }

// In the order that the kernel which multiplies them reads
F8Rows ordered(F8Rows r, int K, bool by_rows) {
    r.row_step = by_rows ? (int)whole(K) : 16;
    r.piece_step = by_rows ? 16 : r.rows * 16;
    return r;
}

struct MatmulWs {
    F8Rows x;
    float* partials;  // of the tiles
    size_t total;
};
MatmulWs matmul_ws(const emoe_matmul_desc& d, void* ws) {
    MatmulWs w;
    w.total = 0;
    w.x = rows_at(static_cast<uint8_t*>(ws), &w.total, d.rows, d.K);
    w.partials = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + w.total);
    if (is_tiled(d.rows, d.groups, d.N, d.K, kF8Plain)) w.total += f8_partial_bytes(f8_layout(d.N, d.K).kb);
    return w;
}

struct FfnF8Ws {
    F8Rows h, x;
    uint16_t* near;  // of the tiles, see F8Product
    float* partials;
    size_t total;
};
// (x has A rows where the caller grouped them)
FfnF8Ws ffn_ws(const emoe_layer_desc& d, void* ws) {
    FfnF8Ws w;
    const long long A = (long long)d.T * d.k;
    w.total = 0;
    w.h = rows_at(static_cast<uint8_t*>(ws), &w.total, A, d.d_ff);
    w.x = rows_at(static_cast<uint8_t*>(ws), &w.total, A, d.d_model);
    w.near = reinterpret_cast<uint16_t*>(static_cast<uint8_t*>(ws) + w.total);
    if (first_is_tiled(d) && whole(d.d_ff) <= kTieBlocksTiled * kF8Block) w.total = align256(w.total + (size_t)A * whole(d.d_ff) / 8);
    w.partials = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + w.total);
    const size_t first = first_is_tiled(d) ? f8_partial_bytes(f8_layout(d.d_ff, d.d_model).kb) : 0;
    const size_t second = second_is_tiled(d) ? f8_partial_bytes(f8_layout(d.d_model, d.d_ff).kb) : 0;
    w.total += first > second ? first : second;  // (one after the other)
    return w;
}

void own_rows(F8Product& p, const void* x, int64_t stride, int K) {
    p.from = static_cast<const bf16_t*>(x);
    p.from_stride = stride;
    p.K = K;
}

hipError_t multiply(bool tiled, const F8Product& p, F8Epilogue epilogue, float* partials, hipStream_t st) {
    return tiled ? launch_f8_tiled(p, epilogue, partials, st) : launch_f8_stream(p, epilogue, st);
}

}  // namespace

// Beside validate_desc(): 32-bit byte offsets into rows of whole blocks.
int validate_f8_layer(const emoe_layer_desc& d) {
    const long long A = (long long)d.T * d.k, m = whole(d.d_model), f = whole(d.d_ff);
    if ((A + 2) * (m > f ? m : f) > kMostExtent || m * f >= kMostExtent) return EMOE_ERR_SHAPE;
    return EMOE_OK;
}

size_t ffn_f8_ws_bytes(const emoe_layer_desc& d) {
    const size_t n = ffn_ws(d, nullptr).total;
    return n > 0 ? n : 256;
}

size_t f8_matrix_bytes(int N, int K) { return f8_layout(N, K).bytes(); }

hipError_t launch_ffn_f8(const emoe_layer_desc& d, const void* x_perm, RowGather gather, const int32_t* offsets, const void* w1,
                         const void* w3, const void* w2, void* y_perm, void* ws, int passes, hipStream_t st) {
    const FfnF8Ws lay = ffn_ws(d, ws);
    const int A = d.T * d.k;
    const bool swiglu = d.act == EMOE_ACT_SWIGLU;
    const bool second_tiled = second_is_tiled(d);
    const F8Rows h = ordered(lay.h, d.d_ff, second_tiled);
    hipError_t e = hipSuccess;
    F8Product p = {};
    p.offsets = offsets;
    p.groups = d.S;
    p.rows = A;
    p.k = 1;
    if (passes & 1) {
        const bool tiled = first_is_tiled(d);
        p.x = lay.x;
        // tiles gather the rows themselves, so that each is read and converted once
        if (tiled && gather.perm != nullptr) {
            p.x.rows = d.T;
            p.perm = gather.perm;
            p.k = gather.k;
        }
        p.x = ordered(p.x, d.d_model, tiled);
        p.w0 = static_cast<const uint8_t*>(w1);
        p.w1 = static_cast<const uint8_t*>(w3);
        p.lay = f8_layout(d.d_ff, d.d_model);
        p.matrix_bytes = p.lay.bytes();
        p.N = d.d_ff;
        p.h = h;
        p.near = lay.near;
        if (!tiled && f8_own_rows(A, d.d_model)) {
            own_rows(p, x_perm, d.d_model, d.d_model);
            p.perm = gather.perm;
            p.k = gather.k;
        } else {
            e = launch_f8_rows(x_perm, d.d_model, d.d_model, p.x, tiled ? nullptr : gather.perm, gather.k, offsets + d.S, st);
        }
        if (e == hipSuccess) e = multiply(tiled, p, swiglu ? kF8Swiglu : kF8Relu, lay.partials, st);
    }
    if (e != hipSuccess || !(passes & 2)) return e;
    p.x = h;
    p.from = nullptr;
    p.perm = nullptr;
    p.k = 1;
    p.w0 = static_cast<const uint8_t*>(w2);
    p.w1 = nullptr;
    p.lay = f8_layout(d.d_model, d.d_ff);
    p.matrix_bytes = p.lay.bytes();
    p.N = d.d_model;
    p.out = static_cast<bf16_t*>(y_perm);
    p.out_stride = d.d_model;
    p.out_perm = gather.out_perm;
    return multiply(second_tiled, p, kF8Plain, lay.partials, st);
}

}  // namespace emoe

using namespace emoe;

extern "C" {

int emoe_matrix_bytes(int32_t N, int32_t K, size_t* bytes) {
    int rc = validate_matrix(N, K);
    if (rc != EMOE_OK) return rc;
    if (!bytes) return EMOE_ERR_NULL;
    *bytes = f8_matrix_bytes(N, K);
    return EMOE_OK;
}

int emoe_matrix_pack(int32_t count, int32_t N, int32_t K, int32_t dtype, const void* w, int64_t w_stride, void* matrices, void* stream) {
    int rc = validate_matrices(count, N, K, dtype, w_stride);
    if (rc != EMOE_OK) return rc;
    if (count == 0) return EMOE_OK;
    if (!w || !matrices) return EMOE_ERR_NULL;
    if (unaligned(w) || unaligned(matrices)) return EMOE_ERR_UNSUPPORTED;
    if (w == matrices) return EMOE_ERR_SHAPE;
    return status_of(launch_matrix_pack(count, N, K, dtype, w, w_stride, matrices, static_cast<hipStream_t>(stream)));
}

int emoe_matrix_unpack(int32_t count, int32_t N, int32_t K, int32_t dtype, const void* matrices, void* w, int64_t w_stride, void* stream) {
    int rc = validate_matrices(count, N, K, dtype, w_stride);
    if (rc != EMOE_OK) return rc;
    if (count == 0) return EMOE_OK;
    if (!w || !matrices) return EMOE_ERR_NULL;
    if (unaligned(w) || unaligned(matrices)) return EMOE_ERR_UNSUPPORTED;
    if (w == matrices) return EMOE_ERR_SHAPE;
    return status_of(launch_matrix_unpack(count, N, K, dtype, matrices, w, w_stride, static_cast<hipStream_t>(stream)));
}

int emoe_matmul_workspace_bytes(const emoe_matmul_desc* desc, size_t* bytes) {
    int rc = validate_matmul(desc);
    if (rc != EMOE_OK) return rc;
    if (!bytes) return EMOE_ERR_NULL;
    *bytes = matmul_ws(*desc, nullptr).total;
    return EMOE_OK;
}

int emoe_matmul(const emoe_matmul_desc* desc, const void* x, const int32_t* group_offsets, const void* matrices, void* out, void* ws,
                size_t ws_bytes, void* stream) {
    int rc = validate_matmul(desc);
    if (rc != EMOE_OK) return rc;
    if (desc->rows == 0) return EMOE_OK;
    if (!x || !matrices || !out) return EMOE_ERR_NULL;
    if (desc->groups > 1 && !group_offsets) return EMOE_ERR_NULL;
    if (unaligned(x) || unaligned(matrices) || unaligned(out) || unaligned(ws)) return EMOE_ERR_UNSUPPORTED;
    if (out == x || out == matrices || ws == x || ws == matrices || ws == out) return EMOE_ERR_SHAPE;
    const MatmulWs lay = matmul_ws(*desc, ws);
    if (!ws || ws_bytes < lay.total) return EMOE_ERR_WORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    F8Product p = {};
    const bool tiled = is_tiled(desc->rows, desc->groups, desc->N, desc->K, kF8Plain);
    p.x = ordered(lay.x, desc->K, tiled);
    if (!tiled && f8_own_rows(desc->rows, desc->K)) own_rows(p, x, desc->x_stride, desc->K);
    else if (launch_f8_rows(x, desc->x_stride, desc->K, p.x, nullptr, 1, nullptr, st) != hipSuccess) return EMOE_ERR_DEVICE;
    p.k = 1;
    p.offsets = group_offsets;
    p.groups = desc->groups;
    p.rows = desc->rows;
    p.w0 = static_cast<const uint8_t*>(matrices);
    p.lay = f8_layout(desc->N, desc->K);
    p.matrix_bytes = p.lay.bytes();
    p.N = desc->N;
    p.out = static_cast<bf16_t*>(out);
    p.out_stride = desc->out_stride;
    return status_of(multiply(tiled, p, kF8Plain, lay.partials, st));
}

}  // extern "C"
