// Microscaled 4-bit matrices: the packed layout, and views as matrices.
//
// Packed layout of [rows, K], the operand order of v_mfma_scale_f32_32x32x64_f8f6f4: rows in tiles of 32, K in steps of 256, both padded
// with zeros.  Of a tile's step, 4 KB of codes: 16-byte chunk (q*64 + 32h + n) = the 32 codes (low half of a byte first) of row n,
// k = 64q + 32h + 0..31; and, behind the codes of all tiles, 256 bytes of scales: byte q of word 32h + n is that chunk's.  A lane's
// chunk is one scale block, and the instruction picks the byte of its lane's word: nothing is moved between loading and multiplying.
#pragma once
#include "fps_internal.h"

namespace fps {

constexpr int kMxRows = 32, kMxStep = 256, kMxStepBytes = 4096, kMxScaleBytes = 256;

__host__ __device__ inline int mx4_tiles(long long rows) { return (int)((rows + kMxRows - 1) / kMxRows); }
__host__ __device__ inline int mx4_steps(long long K) { return (int)((K + kMxStep - 1) / kMxStep); }

// 0: too large, or no matrix
inline size_t mx4_bytes(long long rows, long long cols) {
    if (rows < 1 || cols < 1 || rows > 0x7FFFFFFF || cols > 0x7FFFFFFF - kMxStep) return 0;
    const long long steps = (long long)mx4_tiles(rows) * mx4_steps(cols);
    return steps > 0x3FFFFFFF ? 0 : (size_t)steps * (kMxStepBytes + kMxScaleBytes);
}

struct Packed {
    const uint4* codes;          // [tile][step][4][64]
    const uint32_t* scales;      // [tile][step][64]
    int tiles, steps;
    Packed(const void* p, long long rows, long long K)
        : codes((const uint4*)p), tiles(mx4_tiles(rows)), steps(mx4_steps(K)) {
        scales = (const uint32_t*)((const char*)p + (size_t)tiles * steps * kMxStepBytes);
    }
};

// A view as a matrix: element (row, column) is at row / rows, row % rows, column / cols, column % cols
struct Matrix {
    char* data;
    long long stride_b, stride_h, stride_r;        // bytes
    int rows, cols, B, heads;
    uint32_t rc_rows, rc_cols;
    explicit Matrix(const fps_view& v) : data((char*)v.data), rows(v.rows), cols(v.cols), B(v.B), heads(v.heads), rc_cols(reciprocal(v.cols)) {
        const long long e = v.dt == FPS_OUT_F32 ? 4 : 2;
        if (B > 1 && (rows == 1 || v.stride_b == rows * v.stride_r)) {        // batches that follow each other are one
            stride_b = 0;
            stride_r = (rows == 1 ? v.stride_b : v.stride_r) * e;
            rows *= B;
            B = 1;
            stride_h = v.heads > 1 ? v.stride_h * e : 0;
            rc_rows = reciprocal(rows);
            return;
        }
        rc_rows = reciprocal(rows);
        stride_b = v.B > 1 ? v.stride_b * e : 0;
        stride_h = v.heads > 1 ? v.stride_h * e : 0;
        stride_r = v.rows > 1 ? v.stride_r * e : 0;
    }
    __host__ __device__ int all_rows() const { return B * rows; }
    __host__ __device__ int all_cols() const { return heads * cols; }
    __device__ char* row(int r) const {
        if (B == 1) return data + r * stride_r;
        const int b = quotient(r, rows, rc_rows);
        return data + b * stride_b + (r - b * rows) * stride_r;
    }
    // offset of column c in its row
    template <int BYTES> __device__ long long column(int c) const {
        if (heads == 1) return (long long)c * BYTES;
        const int h = quotient(c, cols, rc_cols);
        return h * stride_h + (long long)(c - h * cols) * BYTES;
    }
};

// the product in tiles of 256 x 256 or 128 x 128, operands copied ahead into LDS (fps_mx4_matmul.hip); K below 2^30
int launch_mx4_tiles(int edge, const void* a, const void* b, int K, const float* bias, const fps_view& y, hipStream_t st);

}  // namespace fps
