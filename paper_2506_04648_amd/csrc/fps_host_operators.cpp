// Host side of the operators around the attention: validation of views, norms and rotations, the rotation's
// table, and the extern "C" entry points.
#include "fps_mx4.h"

#include <math.h>
#include <string.h>

namespace fps {

// A view of [B, heads, rows, cols] (0: any) whose rows start at multiples of `align` bytes.
static int check_view(const fps_view* v, const char* name, long long B, long long heads, long long rows, long long cols,
                      int align, bool output) {
    if (!v) { set_error("%s is NULL", name); return FPS_ERR_INVALID_ARG; }
    FPS_TRY(check_ptr(v->data, name));
    if (v->dt != FPS_OUT_BF16 && v->dt != FPS_OUT_F32) {
        set_error("%s has invalid type %d", name, (int)v->dt);
        return FPS_ERR_INVALID_ARG;
    }
    const int64_t size[4] = {v->cols, v->rows, v->heads, v->B}, stride[4] = {1, v->stride_r, v->stride_h, v->stride_b};
    const long long want[4] = {cols, rows, heads, B};
    for (int i = 0; i < 4; ++i)
        if (size[i] <= 0 || (want[i] && size[i] != want[i])) {
            set_error("%s is [%d,%d,%d,%d], not [%lld,%lld,%lld,%lld]", name, v->B, v->heads, v->rows, v->cols, B, heads, rows, cols);
            return FPS_ERR_INVALID_ARG;
        }
    const int bytes = v->dt == FPS_OUT_F32 ? 4 : 2;
    int64_t s[4], n[4];                                   // the axes of more than one element, by falling stride
    int axes = 0;
    for (int i = 0; i < 4; ++i) {
        if (size[i] == 1) continue;
        if (stride[i] < 0 || stride[i] > ((int64_t)1 << 40)) {
            set_error("%s has a stride of %lld elements", name, (long long)stride[i]);
            return FPS_ERR_INVALID_ARG;
        }
        if (i > 0 && stride[i] * bytes % align) {
            set_error("%s has rows that are not %d-byte aligned", name, align);
            return FPS_ERR_INVALID_ARG;
        }
        int j = axes++;
        for (; j > 0 && s[j - 1] < stride[i]; --j) { s[j] = s[j - 1]; n[j] = n[j - 1]; }
        s[j] = stride[i];
        n[j] = size[i];
    }
    int64_t extent = 0;                                   // the last element's place
    for (int j = axes - 1; j >= 0; --j) {
        if (output && s[j] <= extent) {
            set_error("%s has elements that share a place", name);
            return FPS_ERR_INVALID_ARG;
        }
        extent += (n[j] - 1) * s[j];
        if (extent > ((int64_t)1 << 44)) { set_error("%s is too large", name); return FPS_ERR_INVALID_ARG; }
    }
    return FPS_OK;
}

static int check_norm(const fps_norm* n) {
    if (!n) return FPS_OK;
    if (n->weight) FPS_TRY(check_ptr(n->weight, "norm.weight"));
    uint32_t bits;                                        // compared as such: the library is built without regard to NaN
    memcpy(&bits, &n->eps, 4);
    if (bits < 0x00800000u || bits > 0x7F7FFFFFu) {
        set_error("norm.eps must be a normal float above 0");
        return FPS_ERR_INVALID_ARG;
    }
    return FPS_OK;
}

static int check_pairs(const fps_rotation* r) {
    if (r->pairs_t < 0 || r->pairs_h < 0 || r->pairs_w < 0 || r->pairs_t > kHeadDim / 2 || r->pairs_h > kHeadDim / 2 ||
        r->pairs_w > kHeadDim / 2 || r->pairs_t + r->pairs_h + r->pairs_w > kHeadDim / 2) {
        set_error("rotation of %d + %d + %d pairs: at most %d together", r->pairs_t, r->pairs_h, r->pairs_w, kHeadDim / 2);
        return FPS_ERR_INVALID_ARG;
    }
    return check_enum(r->pairing, FPS_PAIRS_HALVES, "rotation.pairing");
}

static size_t table_floats(const fps_shape* s, const fps_rotation* r) {
    return 2 * ((size_t)s->T * r->pairs_t + (size_t)s->H * r->pairs_h + (size_t)s->W * r->pairs_w);
}

static int check_rotation(const fps_shape* shape, const fps_rotation* r) {
    if (!r) return FPS_OK;
    FPS_TRY(check_pairs(r));
    if (table_floats(shape, r) != 0) FPS_TRY(check_ptr(r->table, "rotation.table"));
    if (table_floats(shape, r) > 0x7FFFFFFFu) { set_error("a rotation table of 2^31 floats or more"); return FPS_ERR_UNSUPPORTED; }
    if (r->stride_b < 0 || r->stride_b % 2 || r->stride_b > ((int64_t)1 << 40)) {
        set_error("rotation.stride_b of %lld floats", (long long)r->stride_b);
        return FPS_ERR_INVALID_ARG;
    }
    return FPS_OK;
}

// x and what is of its size: [B, heads, tokens, 128], rows of whole 16-byte chunks
static int check_tokens(const fps_shape* shape, const fps_view* v, const char* name, bool output) {
    const long long tokens = (long long)shape->T * shape->H * shape->W;
    if (tokens > 0x7FFFFFFF) { set_error("more than 2^31 - 1 tokens"); return FPS_ERR_UNSUPPORTED; }
    return check_view(v, name, shape->B, shape->heads, tokens, kHeadDim, 16, output);
}

// a view as a matrix of B*rows rows and heads*cols columns
static int check_matrix(const fps_view* v, const char* name, bool output) {
    FPS_TRY(check_view(v, name, 0, 0, 0, 0, 1, output));
    if (v->heads > 1 && v->cols % 32) { set_error("%s has several heads of %d columns, not a multiple of 32", name, v->cols); return FPS_ERR_INVALID_ARG; }
    if (mx4_bytes((long long)v->B * v->rows, (long long)v->heads * v->cols) == 0) {
        set_error("%s is too large a matrix", name);
        return FPS_ERR_UNSUPPORTED;
    }
    return FPS_OK;
}

}  // namespace fps

using namespace fps;

extern "C" {

size_t fps_rotation_floats(const fps_shape* shape, const fps_rotation* rot) {
    if (check_shape(shape, nullptr) != FPS_OK) return 0;
    if (!rot) { set_error("rot is NULL"); return 0; }
    return check_pairs(rot) == FPS_OK ? table_floats(shape, rot) : 0;
}

int fps_rotation_table_host(const fps_shape* shape, const fps_rotation* rot, const int64_t start[3], double base, float* table) {
    FPS_TRY(check_shape(shape, nullptr));
    if (!rot || !start || !table) { set_error("rot, start or table is NULL"); return FPS_ERR_INVALID_ARG; }
    FPS_TRY(check_pairs(rot));
    uint64_t bits;
    memcpy(&bits, &base, 8);
    if (bits == 0 || bits >= 0x7FF0000000000000u) { set_error("base must be finite and above 0"); return FPS_ERR_INVALID_ARG; }
    const int size[3] = {shape->T, shape->H, shape->W}, pairs[3] = {rot->pairs_t, rot->pairs_h, rot->pairs_w};
    float* out = table;
    for (int axis = 0; axis < 3; ++axis) {
        if (start[axis] > ((int64_t)1 << 52) || start[axis] < -((int64_t)1 << 52)) {
            set_error("start[%d] is beyond 2^52", axis);
            return FPS_ERR_INVALID_ARG;
        }
        for (int at = 0; at < size[axis]; ++at)
            for (int i = 0; i < pairs[axis]; ++i) {
                const double angle = (double)(start[axis] + at) * pow(base, -(double)i / pairs[axis]);
                *out++ = (float)cos(angle);
                *out++ = (float)sin(angle);
            }
    }
    return FPS_OK;
}

int fps_norm_rotate(const fps_shape* shape, const fps_view* x, const fps_norm* norm, const fps_rotation* rot,
                    const fps_view* y, void* stream) {
    Geom g;
    FPS_TRY(check_shape(shape, &g));
    FPS_TRY(check_tokens(shape, x, "x", false));
    FPS_TRY(check_tokens(shape, y, "y", true));
    FPS_TRY(check_norm(norm));
    FPS_TRY(check_rotation(shape, rot));
    return launch_norm_rotate(g, *x, norm, rot, *y, (hipStream_t)stream);
}

int fps_norm_rotate_operand(const fps_shape* shape, const fps_view* x, const fps_norm* norm, const fps_rotation* rot,
                            fps_role role, fps_precision prec, void* xq_out, float* scales_out, void* stream) {
    Geom g;
    FPS_TRY(check_shape(shape, &g));
    FPS_TRY(check_tokens(shape, x, "x", false));
    FPS_TRY(check_norm(norm));
    FPS_TRY(check_rotation(shape, rot));
    FPS_TRY(check_enum(role, FPS_ROLE_K, "role"));
    FPS_TRY(check_enum(prec, FPS_PREC_FP8, "prec"));
    FPS_TRY(check_ptr(xq_out, "xq_out"));
    if (prec == FPS_PREC_FP8) FPS_TRY(check_ptr(scales_out, "scales_out"));
    return launch_norm_rotate_operand(g, *x, norm, rot, role, prec, xq_out, scales_out, (hipStream_t)stream);
}

size_t fps_norm_rotate_bwd_bytes(const fps_shape* shape, const fps_norm* norm) {
    Geom g;
    if (check_shape(shape, &g) != FPS_OK || check_norm(norm) != FPS_OK) return 0;
    return norm_rotate_bwd_bytes(g, shape->heads, norm && norm->per_head);
}

int fps_norm_rotate_bwd(const fps_shape* shape, const fps_view* x, const fps_norm* norm, const fps_rotation* rot,
                        const fps_view* dy, const fps_view* dx, float* dweight, void* workspace, size_t workspace_bytes,
                        void* stream) {
    Geom g;
    FPS_TRY(check_shape(shape, &g));
    FPS_TRY(check_tokens(shape, x, "x", false));
    FPS_TRY(check_tokens(shape, dy, "dy", false));
    FPS_TRY(check_tokens(shape, dx, "dx", true));
    if (dy->dt != x->dt || dx->dt != x->dt) { set_error("x, dy and dx must have one type"); return FPS_ERR_INVALID_ARG; }
    FPS_TRY(check_norm(norm));
    FPS_TRY(check_rotation(shape, rot));
    if (dweight) {
        if (!norm || !norm->weight) { set_error("dweight without a norm's weight"); return FPS_ERR_INVALID_ARG; }
        FPS_TRY(check_ptr(dweight, "dweight"));
        FPS_TRY(check_ptr(workspace, "workspace"));
        const size_t need = norm_rotate_bwd_bytes(g, shape->heads, norm->per_head != 0);
        if (workspace_bytes < need) {
            set_error("workspace of %zu bytes, %zu needed", workspace_bytes, need);
            return FPS_ERR_WORKSPACE;
        }
    }
    return launch_norm_rotate_bwd(g, *x, norm, rot, *dy, *dx, dweight, (float*)workspace, (hipStream_t)stream);
}

int fps_dequantize(const fps_shape* shape, const void* xq, const float* scales, fps_role role, fps_vscale vscale,
                   fps_out_dtype dt, void* x_raster, void* stream) {
    Geom g;
    FPS_TRY(check_shape(shape, &g));
    FPS_TRY(check_enum(role, FPS_ROLE_V, "role"));
    FPS_TRY(check_enum(vscale, FPS_VSCALE_CHANNEL, "vscale"));
    FPS_TRY(check_enum(dt, FPS_OUT_F32, "dt"));
    FPS_TRY(check_ptr(xq, "xq"));
    FPS_TRY(check_ptr(scales, "scales"));
    FPS_TRY(check_ptr(x_raster, "x_raster"));
    return launch_dequantize(g, xq, scales, role, role == FPS_ROLE_V && vscale == FPS_VSCALE_CHANNEL, dt == FPS_OUT_F32,
                             x_raster, (hipStream_t)stream);
}

size_t fps_mx4_bytes(int64_t rows, int64_t cols) {
    const size_t n = mx4_bytes(rows, cols);
    if (n == 0) set_error("a matrix of %lld x %lld elements cannot be packed", (long long)rows, (long long)cols);
    return n;
}

int fps_mx4_quantize(const fps_view* x, void* packed, void* stream) {
    FPS_TRY(check_matrix(x, "x", false));
    FPS_TRY(check_ptr(packed, "packed"));
    return launch_mx4_quantize(*x, packed, (hipStream_t)stream);
}

int fps_mx4_dequantize(const void* packed, const fps_view* y, void* stream) {
    FPS_TRY(check_ptr(packed, "packed"));
    FPS_TRY(check_matrix(y, "y", true));
    return launch_mx4_dequantize(packed, *y, (hipStream_t)stream);
}

static int check_product(int64_t K, const void* b, const char* name, const float* bias, const fps_view* y) {
    FPS_TRY(check_matrix(y, "y", true));
    FPS_TRY(check_ptr(b, name));
    if (bias) FPS_TRY(check_ptr(bias, "bias"));
    if (mx4_bytes((long long)y->B * y->rows, K) == 0 || mx4_bytes((long long)y->heads * y->cols, K) == 0) {
        set_error("rows of %lld elements cannot be packed", (long long)K);
        return FPS_ERR_INVALID_ARG;
    }
    return FPS_OK;
}

int fps_mx4_matmul(int64_t K, const void* a, const void* b, const float* bias, const fps_view* y, void* stream) {
    FPS_TRY(check_product(K, b, "b", bias, y));
    FPS_TRY(check_ptr(a, "a"));
    return launch_mx4_matmul((int)K, a, b, bias, *y, (hipStream_t)stream);
}

size_t fps_mx4_linear_bytes(int64_t rows, int64_t K) { return fps_mx4_bytes(rows, K); }

int fps_mx4_linear(const fps_view* x, const void* w, const float* bias, const fps_view* y, void* workspace,
                   size_t workspace_bytes, void* stream) {
    FPS_TRY(check_matrix(x, "x", false));
    const int64_t M = (int64_t)x->B * x->rows, K = (int64_t)x->heads * x->cols;
    FPS_TRY(check_product(K, w, "w", bias, y));
    if ((int64_t)y->B * y->rows != M) {
        set_error("y has %lld rows, x %lld", (long long)y->B * y->rows, (long long)M);
        return FPS_ERR_INVALID_ARG;
    }
    FPS_TRY(check_ptr(workspace, "workspace"));
    if (workspace_bytes < mx4_bytes(M, K)) {
        set_error("workspace of %zu bytes, %zu needed", workspace_bytes, mx4_bytes(M, K));
        return FPS_ERR_WORKSPACE;
    }
    return launch_mx4_linear(*x, w, bias, *y, workspace, (hipStream_t)stream);
}

}  // extern "C"
