// Host side of the block operators: argument checks and launch sequences.  See include/fmtc.h.
#include "fmtc_block.h"

namespace {

using namespace fmtc;

fmtc_status hip_status(hipError_t e, const char* what) {
    return e == hipSuccess ? FMTC_OK : set_error(FMTC_EHIP, "%s: %s", what, hipGetErrorString(e));
}

bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }
bool dtype_ok(int t) { return t == FMTC_F32 || t == FMTC_BF16 || t == FMTC_F16; }
size_t dtype_size(int t) { return t == FMTC_F32 ? 4 : 2; }
int64_t blocks_of(int64_t n) { return (n + kF8Block - 1) / kF8Block; }

constexpr int64_t kMaxSide = (int64_t)1 << 31;  // rows, columns, depth
constexpr int64_t kMaxLd = (int64_t)1 << 40;
constexpr int64_t kMaxGroups = 0x7fffffff;      // workgroups of a launch

bool side_ok(int64_t n, int64_t least) { return n >= least && n < kMaxSide; }

// a matrix of `type` the caller owns; rows == 0: never touched
fmtc_status check_values(const char* who, const char* what, const void* p, int type, int64_t rows, int64_t cols, int64_t ld) {
    if (rows == 0) return FMTC_OK;
    if (!p) return set_error(FMTC_EINVAL, "%s: %s is NULL", who, what);
    if (!aligned(p, dtype_size(type))) return set_error(FMTC_EINVAL, "%s: %s is not aligned to its type", who, what);
    if (ld < cols || ld > kMaxLd) return set_error(FMTC_EINVAL, "%s: row stride %lld of %s, %lld columns", who, (long long)ld, what, (long long)cols);
    return FMTC_OK;
}

fmtc_status check_f8(const char* who, const char* what, const fmtc_f8* q) {
    if (!q) return set_error(FMTC_EINVAL, "%s: %s is NULL", who, what);
    if (!side_ok(q->rows, 0) || !side_ok(q->depth, 1))
        return set_error(FMTC_EINVAL, "%s: %s is %lld x %lld", who, what, (long long)q->rows, (long long)q->depth);
    if (q->format != FMTC_E4M3 && q->format != FMTC_E5M2) return set_error(FMTC_EINVAL, "%s: format %d of %s", who, q->format, what);
    if (q->scale != FMTC_SCALE_F32 && q->scale != FMTC_SCALE_E8M0) return set_error(FMTC_EINVAL, "%s: kind of scale %d of %s", who, q->scale, what);
    if (q->block_rows != 1 && q->block_rows != kF8Block) return set_error(FMTC_EINVAL, "%s: blocks of %d rows in %s", who, q->block_rows, what);
    if (q->rows == 0) return FMTC_OK;
    if (!q->d_codes || !q->d_scales) return set_error(FMTC_EINVAL, "%s: codes or scales of %s are NULL", who, what);
    if (!aligned(q->d_codes, 16) || (q->scale == FMTC_SCALE_F32 && !aligned(q->d_scales, 4)))
        return set_error(FMTC_EINVAL, "%s: codes of %s need 16-byte alignment, f32 scales 4-byte", who, what);
    if (q->ld % 16 != 0 || q->ld < blocks_of(q->depth) * kF8Block || q->ld > kMaxLd)
        return set_error(FMTC_EINVAL, "%s: row stride %lld of %s: a multiple of 16, at least the depth rounded up to 128", who, (long long)q->ld, what);
    if (q->ld_scales < (q->rows + q->block_rows - 1) / q->block_rows || q->ld_scales > kMaxLd)
        return set_error(FMTC_EINVAL, "%s: stride %lld between the scales of %s", who, (long long)q->ld_scales, what);
    return FMTC_OK;
}

fmtc_status check_workspace(const char* who, const void* p, size_t bytes, size_t need) {
    if (need == 0) return FMTC_OK;
    if (!p || !aligned(p, 256)) return set_error(FMTC_EINVAL, "%s: workspace is NULL or not 256-byte aligned", who);
    if (bytes < need) return set_error(FMTC_EBUFSIZE, "%s: workspace of %zu bytes, %zu needed", who, bytes, need);
    return FMTC_OK;
}

#define CHECK(call)                                   \
    do {                                              \
        const fmtc_status st_ = (call);               \
        if (st_ != FMTC_OK) return st_;               \
    } while (0)

fmtc_status check_norm(const char* who, const fmtc_norm* a) {
    if (!a) return set_error(FMTC_EINVAL, "%s: args is NULL", who);
    if (!side_ok(a->rows, 0) || a->C < 1 || a->C > 16384)
        return set_error(FMTC_EINVAL, "%s: %lld rows of %d channels (1 to 16384)", who, (long long)a->rows, a->C);
    if (!dtype_ok(a->type) || (a->weight_type != FMTC_F32 && a->weight_type != a->type))
        return set_error(FMTC_EINVAL, "%s: type %d, weights of type %d (f32 or the same)", who, a->type, a->weight_type);
    if (a->rows > 0 && !a->d_y && (a->d_w_post || a->d_gate)) return set_error(FMTC_EINVAL, "%s: w_post and gate need y", who);
    if (a->d_gate && a->rows_per_gate < 1) return set_error(FMTC_EINVAL, "%s: rows_per_gate %lld", who, (long long)a->rows_per_gate);
    const size_t w = dtype_size(a->weight_type);
    if (!aligned(a->d_w_post, w) || !aligned(a->d_w_pre, w) || !aligned(a->d_gate, w))
        return set_error(FMTC_EINVAL, "%s: weights or gate are not aligned to their type", who);
    if (a->d_y) CHECK(check_values(who, "y", a->d_y, a->type, a->rows, a->C, a->ld_y));
    return FMTC_OK;
}

}  // namespace

extern "C" {

fmtc_status fmtc_f8_quantize(const void* d_x, fmtc_dtype type, int64_t rows, int64_t cols, int64_t ld_x,
                             const fmtc_f8* by_rows, const fmtc_f8* by_cols, void* hip_stream) {
    const char* who = "fmtc_f8_quantize";
    if (!dtype_ok(type)) return set_error(FMTC_EINVAL, "%s: type %d", who, (int)type);
    if (!side_ok(rows, 0) || !side_ok(cols, 1)) return set_error(FMTC_EINVAL, "%s: %lld x %lld values", who, (long long)rows, (long long)cols);
    if (!by_rows && !by_cols) return set_error(FMTC_EINVAL, "%s: no output", who);
    if (rows == 0) return FMTC_OK;
    CHECK(check_values(who, "x", d_x, type, rows, cols, ld_x));
    if (by_rows) {
        CHECK(check_f8(who, "by_rows", by_rows));
        if (by_rows->rows != rows || by_rows->depth != cols) return set_error(FMTC_EINVAL, "%s: by_rows has another shape", who);
    }
    if (by_cols) {
        CHECK(check_f8(who, "by_cols", by_cols));
        if (by_cols->rows != cols || by_cols->depth != rows) return set_error(FMTC_EINVAL, "%s: by_cols has another shape", who);
    }
    if (by_rows && by_cols &&
        (by_rows->format != by_cols->format || by_rows->scale != by_cols->scale || by_rows->block_rows != by_cols->block_rows))
        return set_error(FMTC_EINVAL, "%s: the outputs' format, kind of scale and block_rows differ", who);
    if (rows * blocks_of(cols) > kMaxGroups) return set_error(FMTC_EINVAL, "%s: %lld x %lld values are too many", who, (long long)rows, (long long)cols);
    return hip_status(launch_f8_quantize(d_x, type, rows, cols, ld_x, by_rows, by_cols, nullptr, (hipStream_t)hip_stream), who);
}

size_t fmtc_f8_matmul_workspace_size(int64_t M, int64_t N, int64_t K) {
    return side_ok(M, 1) && side_ok(N, 1) && side_ok(K, 1) ? matmul_f8_workspace(M, N, K) : 0;
}

fmtc_status fmtc_f8_matmul(const fmtc_f8* a, const fmtc_f8* b, const float* d_bias, void* d_out, fmtc_dtype out_type,
                           int64_t ld_out, int accumulate, void* d_workspace, size_t ws_bytes, void* hip_stream) {
    const char* who = "fmtc_f8_matmul";
    CHECK(check_f8(who, "a", a));
    CHECK(check_f8(who, "b", b));
    if (a->depth != b->depth) return set_error(FMTC_EINVAL, "%s: depths %lld and %lld", who, (long long)a->depth, (long long)b->depth);
    if (a->block_rows != 1) return set_error(FMTC_EINVAL, "%s: a has blocks of %d rows", who, a->block_rows);
    if (a->scale != b->scale) return set_error(FMTC_EINVAL, "%s: a and b have different kinds of scale", who);
    if (b->format != FMTC_E4M3) return set_error(FMTC_EINVAL, "%s: b has to be E4M3", who);
    if (!dtype_ok(out_type)) return set_error(FMTC_EINVAL, "%s: type %d", who, (int)out_type);
    if (accumulate && out_type != FMTC_F32) return set_error(FMTC_EINVAL, "%s: accumulate needs an f32 output", who);
    if (!aligned(d_bias, 4)) return set_error(FMTC_EINVAL, "%s: bias is not aligned to its type", who);
    if (a->rows == 0 || b->rows == 0) return FMTC_OK;
    CHECK(check_values(who, "out", d_out, out_type, a->rows, b->rows, ld_out));
    if (((a->rows + 15) / 16) * ((b->rows + 15) / 16) > kMaxGroups) return set_error(FMTC_EINVAL, "%s: the output is too large", who);
    CHECK(check_workspace(who, d_workspace, ws_bytes, matmul_f8_workspace(a->rows, b->rows, a->depth)));
    return hip_status(launch_f8_matmul(*a, *b, d_bias, d_out, out_type, ld_out, accumulate, d_workspace, (hipStream_t)hip_stream), who);
}

}  // extern "C"

namespace {

// Workspace of fmtc_f8_matmul_backward: dy as codes by rows and by columns, the column sums of its blocks of rows, and what
// the two products need (one after the other).
struct BackwardSpace {
    size_t row_codes, row_scales, col_codes, col_scales, sums, product, product_bytes, total;
};
BackwardSpace backward_space(int64_t P, int64_t K, int64_t O) {
    BackwardSpace w;
    size_t o = 0;
    auto take = [&](size_t bytes) {
        const size_t here = o;
        o = align_up(o + bytes, 256);
        return here;
    };
    w.row_codes = take((size_t)P * blocks_of(O) * kF8Block);
    w.row_scales = take(sizeof(float) * (size_t)P * blocks_of(O));
    w.col_codes = take((size_t)O * blocks_of(P) * kF8Block);
    w.col_scales = take(sizeof(float) * (size_t)O * blocks_of(P));
    w.sums = take(sizeof(float) * (size_t)O * blocks_of(P));
    const size_t dx = matmul_f8_workspace(P, K, O), dw = matmul_f8_workspace(O, K, P);
    w.product_bytes = dx > dw ? dx : dw;
    w.product = take(w.product_bytes);
    w.total = o;
    return w;
}

}  // namespace

extern "C" {

size_t fmtc_f8_matmul_backward_workspace_size(int64_t P, int64_t K, int64_t O) {
    return side_ok(P, 1) && side_ok(K, 1) && side_ok(O, 1) ? backward_space(P, K, O).total : 0;
}

fmtc_status fmtc_f8_matmul_backward(const void* d_dy, fmtc_dtype dy_type, int64_t P, int64_t O, int64_t ld_dy,
                                    const fmtc_f8* w_t, const fmtc_f8* x_t, fmtc_f8_format format, fmtc_f8_scale scale,
                                    void* d_dx, fmtc_dtype dx_type, int64_t ld_dx, float* d_dw, int64_t ld_dw,
                                    float* d_dbias, int accumulate, void* d_workspace, size_t ws_bytes,
                                    void* hip_stream) {
    const char* who = "fmtc_f8_matmul_backward";
    hipStream_t s = (hipStream_t)hip_stream;
    if (!dtype_ok(dy_type) || !dtype_ok(dx_type)) return set_error(FMTC_EINVAL, "%s: types %d and %d", who, (int)dy_type, (int)dx_type);
    if (!side_ok(P, 0) || !side_ok(O, 1)) return set_error(FMTC_EINVAL, "%s: %lld x %lld gradients", who, (long long)P, (long long)O);
    if ((format != FMTC_E4M3 && format != FMTC_E5M2) || (scale != FMTC_SCALE_F32 && scale != FMTC_SCALE_E8M0))
        return set_error(FMTC_EINVAL, "%s: format %d, kind of scale %d", who, (int)format, (int)scale);
    if (!d_dx && !d_dw && !d_dbias) return set_error(FMTC_EINVAL, "%s: no output", who);
    CHECK(check_values(who, "dy", d_dy, dy_type, P, O, ld_dy));
    int64_t K = 1;
    if (d_dx) {
        CHECK(check_f8(who, "w_t", w_t));
        if (w_t->depth != O || w_t->format != FMTC_E4M3 || w_t->scale != (int)scale || w_t->block_rows != kF8Block)
            return set_error(FMTC_EINVAL, "%s: w_t has to be [K][%lld], E4M3, 128 x 128 blocks, the same kind of scale", who, (long long)O);
        K = w_t->rows;
        if (K < 1) return set_error(FMTC_EINVAL, "%s: w_t has no rows", who);
        CHECK(check_values(who, "dx", d_dx, dx_type, P, K, ld_dx));
    }
    if (d_dw) {
        // (no rows: x_t has no columns, and nothing of it is read)
        if (P > 0) CHECK(check_f8(who, "x_t", x_t));
        else if (!x_t || !side_ok(x_t->rows, 1)) return set_error(FMTC_EINVAL, "%s: x_t is NULL or has no rows", who);
        if (P > 0 && (x_t->depth != P || x_t->format != FMTC_E4M3 || x_t->scale != (int)scale || x_t->block_rows != 1))
            return set_error(FMTC_EINVAL, "%s: x_t has to be [K][%lld], E4M3, 1 x 128 blocks, the same kind of scale", who, (long long)P);
        if (d_dx && x_t->rows != K) return set_error(FMTC_EINVAL, "%s: w_t has %lld rows, x_t %lld", who, (long long)K, (long long)x_t->rows);
        K = x_t->rows;
        if (K < 1) return set_error(FMTC_EINVAL, "%s: x_t has no rows", who);
        CHECK(check_values(who, "dw", d_dw, FMTC_F32, O, K, ld_dw));
    }
    if (!aligned(d_dbias, 4)) return set_error(FMTC_EINVAL, "%s: dbias is not aligned to its type", who);
    if (P * blocks_of(O) > kMaxGroups || ((P + 15) / 16) * ((K + 15) / 16) > kMaxGroups || ((O + 15) / 16) * ((K + 15) / 16) > kMaxGroups)
        return set_error(FMTC_EINVAL, "%s: %lld x %lld gradients of %lld columns are too many", who, (long long)P, (long long)O, (long long)K);
    if (P == 0) {
        hipError_t e = hipSuccess;
        if (!accumulate) {
            if (d_dw) e = launch_fill_rows(d_dw, O, K, ld_dw, s);
            if (e == hipSuccess && d_dbias) e = launch_fill_rows(d_dbias, 1, O, O, s);
        }
        return hip_status(e, who);
    }
    const BackwardSpace w = backward_space(P, K, O);
    CHECK(check_workspace(who, d_workspace, ws_bytes, w.total));
    char* ws = static_cast<char*>(d_workspace);
    const fmtc_f8 by_rows{ws + w.row_codes, ws + w.row_scales, P, O, blocks_of(O) * kF8Block, P, (int)format, (int)scale, 1};
    const fmtc_f8 by_cols{ws + w.col_codes, ws + w.col_scales, O, P, blocks_of(P) * kF8Block, O, (int)format, (int)scale, 1};
    float* sums = d_dbias ? reinterpret_cast<float*>(ws + w.sums) : nullptr;
    hipError_t e = launch_f8_quantize(d_dy, dy_type, P, O, ld_dy, d_dx ? &by_rows : nullptr, d_dw || d_dbias ? &by_cols : nullptr, sums, s);
    if (e == hipSuccess && d_dx) e = launch_f8_matmul(by_rows, *w_t, nullptr, d_dx, dx_type, ld_dx, 0, ws + w.product, s);
    if (e == hipSuccess && d_dw) e = launch_f8_matmul(by_cols, *x_t, nullptr, d_dw, FMTC_F32, ld_dw, accumulate, ws + w.product, s);
    if (e == hipSuccess && d_dbias) e = launch_column_sums(sums, blocks_of(P), O, d_dbias, accumulate, s);
    return hip_status(e, who);
}

fmtc_status fmtc_block_norm(const fmtc_norm* args, void* d_h_out, int64_t ld_h_out, void* d_n, int64_t ld_n,
                            const fmtc_f8* n_codes, float* d_stats, void* hip_stream) {
    const char* who = "fmtc_block_norm";
    CHECK(check_norm(who, args));
    if (!(args->eps >= 0.f)) return set_error(FMTC_EINVAL, "%s: eps is negative or not a number", who);
    CHECK(check_values(who, "h", args->d_h, args->type, args->rows, args->C, args->ld_h));
    if (args->rows == 0) return FMTC_OK;
    if (!d_h_out && !d_n && !n_codes) return set_error(FMTC_EINVAL, "%s: no output", who);
    if ((d_n || n_codes) && !args->d_w_pre) return set_error(FMTC_EINVAL, "%s: n needs w_pre", who);
    if (d_h_out) CHECK(check_values(who, "h_out", d_h_out, args->type, args->rows, args->C, ld_h_out));
    if (d_n) CHECK(check_values(who, "n", d_n, args->type, args->rows, args->C, ld_n));
    if (n_codes) {
        CHECK(check_f8(who, "n_codes", n_codes));
        if (n_codes->rows != args->rows || n_codes->depth != args->C || n_codes->block_rows != 1)
            return set_error(FMTC_EINVAL, "%s: n_codes has to be [%lld][%d] in 1 x 128 blocks", who, (long long)args->rows, args->C);
    }
    if (!aligned(d_stats, 4)) return set_error(FMTC_EINVAL, "%s: stats is not aligned to its type", who);
    return hip_status(launch_block_norm(*args, d_h_out, ld_h_out, d_n, ld_n, n_codes, d_stats, (hipStream_t)hip_stream), who);
}

size_t fmtc_block_norm_workspace_size(int64_t rows, int C, int64_t rows_per_gate) {
    return side_ok(rows, 1) && C >= 1 && C <= 16384 && rows_per_gate >= 0 ? block_norm_workspace(rows, C, rows_per_gate) : 0;
}

fmtc_status fmtc_block_norm_backward(const fmtc_norm* args, const float* d_stats, const void* d_dn, int64_t ld_dn,
                                     const void* d_dh, int64_t ld_dh, void* d_dy, int64_t ld_dy, void* d_dh_in,
                                     int64_t ld_dh_in, float* d_dw_post, float* d_dw_pre, float* d_dgate,
                                     void* d_workspace, size_t ws_bytes, void* hip_stream) {
    const char* who = "fmtc_block_norm_backward";
    hipStream_t s = (hipStream_t)hip_stream;
    CHECK(check_norm(who, args));
    if (args->rows == 0) {
        if (!aligned(d_dw_post, 4) || !aligned(d_dw_pre, 4)) return set_error(FMTC_EINVAL, "%s: dw_post or dw_pre are not aligned to their type", who);
        hipError_t e = hipSuccess;
        if (d_dw_post) e = launch_fill_rows(d_dw_post, 1, args->C, args->C, s);
        if (e == hipSuccess && d_dw_pre) e = launch_fill_rows(d_dw_pre, 1, args->C, args->C, s);
        return hip_status(e, who);
    }
    if (!d_dy && !d_dh_in && !d_dw_post && !d_dw_pre && !d_dgate) return set_error(FMTC_EINVAL, "%s: no output", who);
    if (d_dn && !args->d_w_pre) return set_error(FMTC_EINVAL, "%s: dn needs w_pre", who);
    if (d_dw_pre && !args->d_w_pre) return set_error(FMTC_EINVAL, "%s: dw_pre needs w_pre", who);
    if (d_dy && !args->d_y) return set_error(FMTC_EINVAL, "%s: dy needs y", who);
    if (d_dw_post && !args->d_w_post) return set_error(FMTC_EINVAL, "%s: dw_post needs w_post", who);
    if (d_dgate && !args->d_gate) return set_error(FMTC_EINVAL, "%s: dgate needs a gate", who);
    if (!aligned(d_stats, 4) || !aligned(d_dw_post, 4) || !aligned(d_dw_pre, 4) || !aligned(d_dgate, 4))
        return set_error(FMTC_EINVAL, "%s: stats, dw_post, dw_pre or dgate are not aligned to their type", who);
    if (!d_stats) return set_error(FMTC_EINVAL, "%s: stats is NULL", who);
    if (d_dn) {
        CHECK(check_values(who, "h", args->d_h, args->type, args->rows, args->C, args->ld_h));
        CHECK(check_values(who, "dn", d_dn, args->type, args->rows, args->C, ld_dn));
    }
    if (d_dh) CHECK(check_values(who, "dh", d_dh, args->type, args->rows, args->C, ld_dh));
    if (d_dy) CHECK(check_values(who, "dy", d_dy, args->type, args->rows, args->C, ld_dy));
    if (d_dh_in) CHECK(check_values(who, "dh_in", d_dh_in, args->type, args->rows, args->C, ld_dh_in));
    CHECK(check_workspace(who, d_workspace, ws_bytes,
                          block_norm_workspace(args->rows, args->C, args->d_gate ? args->rows_per_gate : 0)));
    return hip_status(launch_block_norm_backward(*args, d_stats, d_dn, ld_dn, d_dh, ld_dh, d_dy, ld_dy, d_dh_in, ld_dh_in, d_dw_post,
                                                 d_dw_pre, d_dgate, d_workspace, s), who);
}

}  // extern "C"

namespace {

constexpr int64_t kMaxI8Depth = 131071;  // 128 * 128 * depth fits 32 bits

fmtc_status check_i8(const char* who, const char* what, const fmtc_i8* q) {
    if (!q) return set_error(FMTC_EINVAL, "%s: %s is NULL", who, what);
    if (!side_ok(q->rows, 0) || q->depth < 1 || q->depth > kMaxI8Depth)
        return set_error(FMTC_EINVAL, "%s: %s is %lld x %lld (depth 1 to %lld)", who, what, (long long)q->rows, (long long)q->depth, (long long)kMaxI8Depth);
    if (q->rows == 0) return FMTC_OK;
    if (!q->d_codes || !q->d_scales) return set_error(FMTC_EINVAL, "%s: codes or scales of %s are NULL", who, what);
    if (!aligned(q->d_codes, 16) || !aligned(q->d_scales, 4))
        return set_error(FMTC_EINVAL, "%s: codes of %s need 16-byte alignment, scales 4-byte", who, what);
    if (q->ld % 16 != 0 || q->ld < blocks_of(q->depth) * kF8Block || q->ld > kMaxLd)
        return set_error(FMTC_EINVAL, "%s: row stride %lld of %s: a multiple of 16, at least the depth rounded up to 128", who, (long long)q->ld, what);
    return FMTC_OK;
}

fmtc_status check_i8_product(const char* who, int64_t M, int64_t N, const float* d_bias, const void* d_out, fmtc_dtype out_type, int64_t ld_out) {
    if (!dtype_ok(out_type)) return set_error(FMTC_EINVAL, "%s: type %d", who, (int)out_type);
    if (!aligned(d_bias, 4)) return set_error(FMTC_EINVAL, "%s: bias is not aligned to its type", who);
    if (M == 0 || N == 0) return FMTC_OK;
    CHECK(check_values(who, "out", d_out, out_type, M, N, ld_out));
    if (((M + 15) / 16) * ((N + 15) / 16) > kMaxGroups) return set_error(FMTC_EINVAL, "%s: the output is too large", who);
    return FMTC_OK;
}

// Workspace of fmtc_i8_linear: x as codes, its scales, and what the product needs
struct LinearSpace { size_t codes, scales, product, product_bytes, total; };
LinearSpace linear_space(int64_t M, int64_t N, int64_t K) {
    if (i8_linear_is_one(M, K)) return {0, 0, 0, 0, 0};
    LinearSpace w;
    w.codes = 0;
    w.scales = align_up((size_t)M * blocks_of(K) * kF8Block, 256);
    w.product = align_up(w.scales + sizeof(float) * (size_t)M, 256);
    w.product_bytes = matmul_i8_workspace(M, N, K);
    w.total = w.product + w.product_bytes;
    return w;
}
bool i8_depth_ok(int64_t K) { return K >= 1 && K <= kMaxI8Depth; }

fmtc_status check_gnorm(const char* who, const fmtc_gnorm* a) {
    if (!a) return set_error(FMTC_EINVAL, "%s: args is NULL", who);
    if (!side_ok(a->samples, 0) || !side_ok(a->rows_per_sample, 0) || !side_ok(a->samples * a->rows_per_sample, 0))
        return set_error(FMTC_EINVAL, "%s: %lld samples of %lld rows", who, (long long)a->samples, (long long)a->rows_per_sample);
    if (a->C < 1 || a->C > 8192 || a->groups < 1 || a->C % a->groups != 0)
        return set_error(FMTC_EINVAL, "%s: %d channels (1 to 8192) in %d groups", who, a->C, a->groups);
    if (!dtype_ok(a->type) || (a->weight_type != FMTC_F32 && a->weight_type != a->type))
        return set_error(FMTC_EINVAL, "%s: type %d, weights of type %d (f32 or the same)", who, a->type, a->weight_type);
    if (a->act != FMTC_ACT_NONE && a->act != FMTC_ACT_RELU && a->act != FMTC_ACT_SILU) return set_error(FMTC_EINVAL, "%s: activation %d", who, a->act);
    if (!aligned(a->d_weight, dtype_size(a->weight_type)) || !aligned(a->d_bias, dtype_size(a->weight_type)))
        return set_error(FMTC_EINVAL, "%s: weight or bias are not aligned to their type", who);
    return check_values(who, "x", a->d_x, a->type, a->samples * a->rows_per_sample, a->C, a->ld_x);
}
bool gnorm_size_ok(int64_t samples, int64_t rows, int C, int groups) {
    return side_ok(samples, 1) && side_ok(rows, 1) && side_ok(samples * rows, 1) && C >= 1 && C <= 8192 && groups >= 1 && C % groups == 0;
}
// an array of a call that may be another one of it only as it is
fmtc_status check_in_place(const char* who, const char* what, const void* out, int64_t ld_out, const char* of, const void* in, int64_t ld_in) {
    if (out && out == in && ld_out != ld_in) return set_error(FMTC_EINVAL, "%s: %s is %s with another row stride", who, what, of);
    return FMTC_OK;
}

}  // namespace

extern "C" {

fmtc_status fmtc_i8_quantize(const void* d_x, fmtc_dtype type, int64_t rows, int64_t cols, int64_t ld_x, const fmtc_i8* out, void* hip_stream) {
    const char* who = "fmtc_i8_quantize";
    if (!dtype_ok(type)) return set_error(FMTC_EINVAL, "%s: type %d", who, (int)type);
    if (!side_ok(rows, 0) || !i8_depth_ok(cols)) return set_error(FMTC_EINVAL, "%s: %lld x %lld values", who, (long long)rows, (long long)cols);
    CHECK(check_i8(who, "out", out));
    if (out->rows != rows || out->depth != cols) return set_error(FMTC_EINVAL, "%s: out has another shape", who);
    CHECK(check_values(who, "x", d_x, type, rows, cols, ld_x));
    if (rows == 0) return FMTC_OK;
    return hip_status(launch_i8_quantize(d_x, type, rows, cols, ld_x, *out, (hipStream_t)hip_stream), who);
}

size_t fmtc_i8_matmul_workspace_size(int64_t M, int64_t N, int64_t K) {
    return side_ok(M, 1) && side_ok(N, 1) && i8_depth_ok(K) ? matmul_i8_workspace(M, N, K) : 0;
}

fmtc_status fmtc_i8_matmul(const fmtc_i8* a, const fmtc_i8* b, const float* d_bias, void* d_out, fmtc_dtype out_type,
                           int64_t ld_out, void* d_workspace, size_t ws_bytes, void* hip_stream) {
    const char* who = "fmtc_i8_matmul";
    CHECK(check_i8(who, "a", a));
    CHECK(check_i8(who, "b", b));
    if (a->depth != b->depth) return set_error(FMTC_EINVAL, "%s: depths %lld and %lld", who, (long long)a->depth, (long long)b->depth);
    CHECK(check_i8_product(who, a->rows, b->rows, d_bias, d_out, out_type, ld_out));
    if (a->rows == 0 || b->rows == 0) return FMTC_OK;
    CHECK(check_workspace(who, d_workspace, ws_bytes, matmul_i8_workspace(a->rows, b->rows, a->depth)));
    return hip_status(launch_i8_matmul(*a, *b, d_bias, d_out, out_type, ld_out, d_workspace, (hipStream_t)hip_stream), who);
}

size_t fmtc_i8_linear_workspace_size(int64_t rows, int64_t N, int64_t K) {
    return side_ok(rows, 1) && side_ok(N, 1) && i8_depth_ok(K) ? linear_space(rows, N, K).total : 0;
}

fmtc_status fmtc_i8_linear(const void* d_x, fmtc_dtype type, int64_t rows, int64_t ld_x, const fmtc_i8* w, const float* d_bias,
                           void* d_out, fmtc_dtype out_type, int64_t ld_out, void* d_workspace, size_t ws_bytes, void* hip_stream) {
    const char* who = "fmtc_i8_linear";
    hipStream_t s = (hipStream_t)hip_stream;
    if (!dtype_ok(type)) return set_error(FMTC_EINVAL, "%s: type %d", who, (int)type);
    CHECK(check_i8(who, "w", w));
    if (!side_ok(rows, 0)) return set_error(FMTC_EINVAL, "%s: %lld rows", who, (long long)rows);
    CHECK(check_values(who, "x", d_x, type, rows, w->depth, ld_x));
    CHECK(check_i8_product(who, rows, w->rows, d_bias, d_out, out_type, ld_out));
    if (rows == 0 || w->rows == 0) return FMTC_OK;
    const LinearSpace at = linear_space(rows, w->rows, w->depth);
    CHECK(check_workspace(who, d_workspace, ws_bytes, at.total));
    if (i8_linear_is_one(rows, w->depth)) return hip_status(launch_i8_linear_one(d_x, type, rows, ld_x, *w, d_bias, d_out, out_type, ld_out, s), who);
    char* ws = static_cast<char*>(d_workspace);
    const fmtc_i8 x{ws + at.codes, reinterpret_cast<float*>(ws + at.scales), rows, w->depth, blocks_of(w->depth) * kF8Block};
    hipError_t e = launch_i8_quantize(d_x, type, rows, w->depth, ld_x, x, s);
    if (e == hipSuccess) e = launch_i8_matmul(x, *w, d_bias, d_out, out_type, ld_out, ws + at.product, s);
    return hip_status(e, who);
}

size_t fmtc_group_norm_workspace_size(int64_t samples, int64_t rows_per_sample, int C, int groups, fmtc_dtype type, int to_codes) {
    return gnorm_size_ok(samples, rows_per_sample, C, groups) && dtype_ok(type) ? group_norm_workspace(samples, rows_per_sample, C, groups, type, to_codes) : 0;
}

fmtc_status fmtc_group_norm(const fmtc_gnorm* args, void* d_y, int64_t ld_y, const fmtc_i8* codes, float* d_stats, void* d_workspace,
                            size_t ws_bytes, void* hip_stream) {
    const char* who = "fmtc_group_norm";
    CHECK(check_gnorm(who, args));
    if (!(args->eps >= 0.f)) return set_error(FMTC_EINVAL, "%s: eps is negative or not a number", who);
    const int64_t rows = args->samples * args->rows_per_sample;
    if (codes) {
        CHECK(check_i8(who, "codes", codes));
        if (codes->rows != rows || codes->depth != args->C) return set_error(FMTC_EINVAL, "%s: codes has to be [%lld][%d]", who, (long long)rows, args->C);
    }
    if (!aligned(d_stats, 4)) return set_error(FMTC_EINVAL, "%s: stats is not aligned to its type", who);
    if (rows == 0) return FMTC_OK;
    if (!d_y && !codes && !d_stats) return set_error(FMTC_EINVAL, "%s: no output", who);
    if (d_y && codes) return set_error(FMTC_EINVAL, "%s: y and codes, one of them at most", who);
    if (d_y) {
        CHECK(check_values(who, "y", d_y, args->type, rows, args->C, ld_y));
        CHECK(check_in_place(who, "y", d_y, ld_y, "x", args->d_x, args->ld_x));
    }
    CHECK(check_workspace(who, d_workspace, ws_bytes, group_norm_workspace(args->samples, args->rows_per_sample, args->C, args->groups, args->type, codes)));
    return hip_status(launch_group_norm(*args, d_y, ld_y, codes, d_stats, d_workspace, (hipStream_t)hip_stream), who);
}

size_t fmtc_group_norm_backward_workspace_size(int64_t samples, int64_t rows_per_sample, int C, int groups, fmtc_dtype type) {
    return gnorm_size_ok(samples, rows_per_sample, C, groups) && dtype_ok(type) ? group_norm_backward_workspace(samples, rows_per_sample, C, groups, type) : 0;
}

fmtc_status fmtc_group_norm_backward(const fmtc_gnorm* args, const float* d_stats, const void* d_dy, int64_t ld_dy, void* d_dx,
                                     int64_t ld_dx, float* d_dweight, float* d_dbias, void* d_workspace, size_t ws_bytes,
                                     void* hip_stream) {
    const char* who = "fmtc_group_norm_backward";
    hipStream_t s = (hipStream_t)hip_stream;
    CHECK(check_gnorm(who, args));
    if (!aligned(d_stats, 4) || !aligned(d_dweight, 4) || !aligned(d_dbias, 4))
        return set_error(FMTC_EINVAL, "%s: stats, dweight or dbias are not aligned to their type", who);
    const int64_t rows = args->samples * args->rows_per_sample;
    if (rows == 0) {
        hipError_t e = hipSuccess;
        if (d_dweight) e = launch_fill_rows(d_dweight, 1, args->C, args->C, s);
        if (e == hipSuccess && d_dbias) e = launch_fill_rows(d_dbias, 1, args->C, args->C, s);
        return hip_status(e, who);
    }
    if (!d_dx && !d_dweight && !d_dbias) return set_error(FMTC_EINVAL, "%s: no output", who);
    if (!d_stats) return set_error(FMTC_EINVAL, "%s: stats is NULL", who);
    CHECK(check_values(who, "dy", d_dy, args->type, rows, args->C, ld_dy));
    if (d_dx) {
        CHECK(check_values(who, "dx", d_dx, args->type, rows, args->C, ld_dx));
        CHECK(check_in_place(who, "dx", d_dx, ld_dx, "x", args->d_x, args->ld_x));
        CHECK(check_in_place(who, "dx", d_dx, ld_dx, "dy", d_dy, ld_dy));
    }
    CHECK(check_workspace(who, d_workspace, ws_bytes, group_norm_backward_workspace(args->samples, args->rows_per_sample, args->C, args->groups, args->type)));
    return hip_status(launch_group_norm_backward(*args, d_stats, d_dy, ld_dy, d_dx, ld_dx, d_dweight, d_dbias, d_workspace, s), who);
}

}  // extern "C"

namespace {

constexpr int64_t kMaxValues = (int64_t)1 << 40;  // of a list together

fmtc_status check_list(const char* who, const fmtc_tensor* list, int64_t count) {
    if (count < 0 || (count > 0 && !list)) return set_error(FMTC_EINVAL, "%s: list of %lld arrays is NULL or has no such length", who, (long long)count);
    int64_t total = 0, written = 0, full = 0;
    for (int64_t i = 0; i < count; i++) {
        const fmtc_tensor& t = list[i];
        if (t.n < 0 || t.n > kMaxValues || (total += t.n) > kMaxValues) return set_error(FMTC_EINVAL, "%s: array %lld has %lld values", who, (long long)i, (long long)t.n);
        if (!dtype_ok(t.type) || (t.d_out && !dtype_ok(t.out_type)))
            return set_error(FMTC_EINVAL, "%s: array %lld has type %d, out_type %d", who, (long long)i, t.type, t.out_type);
        if (t.n == 0) continue;
        full++;
        written += t.d_out != nullptr;
        if (!t.d_in) return set_error(FMTC_EINVAL, "%s: array %lld is NULL", who, (long long)i);
        if (!aligned(t.d_in, dtype_size(t.type)) || (t.d_out && !aligned(t.d_out, dtype_size(t.out_type))))
            return set_error(FMTC_EINVAL, "%s: array %lld is not aligned to its type", who, (long long)i);
        if (t.d_out == t.d_in && t.out_type != t.type) return set_error(FMTC_EINVAL, "%s: array %lld is written in place in another type", who, (long long)i);
    }
    if (written != 0 && written != full) return set_error(FMTC_EINVAL, "%s: %lld of %lld arrays have an output", who, (long long)written, (long long)full);
    return FMTC_OK;
}

}  // namespace

extern "C" {

size_t fmtc_clip_workspace_size(const fmtc_tensor* h_list, int64_t count) {
    return check_list("fmtc_clip_workspace_size", h_list, count) == FMTC_OK ? clip_workspace(h_list, count) : 0;
}

fmtc_status fmtc_clip(const fmtc_tensor* h_list, int64_t count, double max_norm, double scale, double eps, float* d_norm,
                      void* d_workspace, size_t ws_bytes, void* hip_stream) {
    const char* who = "fmtc_clip";
    CHECK(check_list(who, h_list, count));
    if (!(max_norm >= 0.0)) return set_error(FMTC_EINVAL, "%s: max_norm is negative or not a number", who);
    if (!(scale >= 0.0 && scale <= 3.402823466385288e38) || !(eps >= 0.0 && eps <= 3.402823466385288e38))
        return set_error(FMTC_EINVAL, "%s: scale or eps are negative or not finite", who);
    if (!aligned(d_norm, 4)) return set_error(FMTC_EINVAL, "%s: norm is not aligned to its type", who);
    bool write = false, any = false;
    for (int64_t i = 0; i < count; i++) {
        any = any || h_list[i].n > 0;
        write = write || (h_list[i].d_out && h_list[i].n > 0);
    }
    if (!write && !d_norm) return any ? set_error(FMTC_EINVAL, "%s: no output", who) : FMTC_OK;
    CHECK(check_workspace(who, d_workspace, ws_bytes, clip_workspace(h_list, count)));
    return hip_status(launch_clip(h_list, count, max_norm, scale, eps, d_norm, d_workspace, (hipStream_t)hip_stream), who);
}

}  // extern "C"
