// Rows to microscaled 4-bit floating point and back, and the products of few rows or small matrices.
#include "fps_mx4.h"

namespace fps {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// 2^e of a scale byte e + 127; NaN for 255
__device__ __forceinline__ float scale_value(uint32_t byte) {
    return __uint_as_float(byte == 0 ? 0x00400000u : byte == 255 ? 0x7FC00000u : byte << 23);
}

// ---- quantisation -------------------------------------------------------------------------------
// A wave takes a step of 256 columns of a tile of 32 rows: a lane four blocks of 32 elements of its row, which need no other
// lane.  Bound by HBM: reads 2 (4) bytes an element and writes 17/32.
template <bool F32>
struct Block { uint4 v[F32 ? 8 : 4]; };

template <bool F32>
__device__ __forceinline__ Block<F32> load_block(const char* p, int n) {          // n elements of it, the rest zero
    constexpr int E = F32 ? 4 : 2;
    Block<F32> b;
    if (n >= 32) {
        __builtin_memcpy(&b, p, sizeof(b));                  // rows start anywhere: the loads need no alignment
    } else {
        uint32_t* w = reinterpret_cast<uint32_t*>(&b);
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            uint32_t x = 0;
            if (i < n) x = F32 ? *reinterpret_cast<const uint32_t*>(p + i * E) : *reinterpret_cast<const uint16_t*>(p + i * E);
            if (F32)        w[i] = x;
            else if (i & 1) w[i >> 1] |= x << 16;
            else            w[i >> 1] = x;
        }
    }
    return b;
}

// codes and scale byte of a block
template <bool F32>
__device__ __forceinline__ uint4 encode_block(const Block<F32>& b, uint32_t* byte) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(&b);
    uint32_t top = 0;                                        // magnitudes order like their bits
#pragma unroll
    for (int i = 0; i < (F32 ? 32 : 16); ++i) {
        if (F32) {
            const uint32_t m = w[i] & 0x7FFFFFFFu;
            top = m > top ? m : top;
        } else {
            const uint32_t lo = w[i] << 16 & 0x7FFF0000u, hi = w[i] & 0x7FFF0000u;
            top = lo > top ? lo : top;
            top = hi > top ? hi : top;
        }
    }
    const int e = (int)(top >> 23);
    *byte = e == 255 ? 255u : top == 0 ? 127u : e > 2 ? (uint32_t)(e - 2) : 0u;
    const float scale = __uint_as_float(e == 255 ? 0x3F800000u : *byte == 0 ? 0x00400000u : *byte << 23);
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t r = 0;
        if (F32) {
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(w[8 * i]), __uint_as_float(w[8 * i + 1]), scale, 0);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(w[8 * i + 2]), __uint_as_float(w[8 * i + 3]), scale, 1);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(w[8 * i + 4]), __uint_as_float(w[8 * i + 5]), scale, 2);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(w[8 * i + 6]), __uint_as_float(w[8 * i + 7]), scale, 3);
        } else {
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w[4 * i]), scale, 0);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w[4 * i + 1]), scale, 1);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w[4 * i + 2]), scale, 2);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w[4 * i + 3]), scale, 3);
        }
        o[i] = r;
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
}

template <bool F32>
__global__ __launch_bounds__(256) void mx4_quantize_kernel(Matrix x, uint4* __restrict__ codes, uint32_t* __restrict__ scales, int steps,
                                                           int waves) {
    const int wave = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (wave >= waves) return;
    const int tile = wave / steps, step = wave - tile * steps;
    const int r = tile * kMxRows + (lane & 31), K = x.all_cols();
    const bool real = r < x.all_rows();
    const char* row = x.row(real ? r : 0);
    uint32_t word = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int k = step * kMxStep + 64 * q + 32 * (lane >> 5);
        const int n = real && k < K ? K - k : 0;
        const Block<F32> b = load_block<F32>(row + (n > 0 ? x.column<F32 ? 4 : 2>(k) : 0), n);
        uint32_t byte;
        codes[((long long)wave * 4 + q) * 64 + lane] = encode_block<F32>(b, &byte);
        word |= byte << (8 * q);
    }
    scales[(long long)wave * 64 + lane] = word;
}

template <bool F32>
__global__ __launch_bounds__(256) void mx4_dequantize_kernel(Packed p, Matrix y, int waves) {
    const int wave = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (wave >= waves) return;
    const int tile = wave / p.steps, step = wave - tile * p.steps;
    const int r = tile * kMxRows + (lane & 31), K = y.all_cols();
    if (r >= y.all_rows()) return;
    char* row = y.row(r);
    const uint32_t word = p.scales[(long long)wave * 64 + lane];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int k = step * kMxStep + 64 * q + 32 * (lane >> 5);
        if (k >= K) break;
        const uint4 c = p.codes[((long long)wave * 4 + q) * 64 + lane];
        const uint32_t w[4] = {c.x, c.y, c.z, c.w};
        const float scale = scale_value(word >> (8 * q) & 255u);
        float f[32];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], 1.0f, 1);
            const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], 1.0f, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], 1.0f, 3);
            const float v[8] = {a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
#pragma unroll
            for (int j = 0; j < 8; ++j) f[8 * i + j] = v[j] * scale;
        }
        char* dst = row + y.column<F32 ? 4 : 2>(k);
        Block<F32> o;
        uint32_t* ow = reinterpret_cast<uint32_t*>(&o);
#pragma unroll
        for (int i = 0; i < (F32 ? 32 : 16); ++i)
            ow[i] = F32 ? __float_as_uint(f[i]) : __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{f[2 * i], f[2 * i + 1]}, bf16x2));
        if (k + 32 <= K) {
            __builtin_memcpy(dst, &o, sizeof(o));
        } else {
#pragma unroll
            for (int i = 0; i < 31; ++i)
                if (k + i < K) {
                    if (F32) reinterpret_cast<uint32_t*>(dst)[i] = ow[i];
                    else     reinterpret_cast<uint16_t*>(dst)[i] = (uint16_t)(ow[i >> 1] >> (16 * (i & 1)));
                }
        }
    }
}

// ---- products -----------------------------------------------------------------------------------
// A workgroup of KW waves takes 32 MT rows and 32 NT columns; its waves share the steps of K and read the operands straight into
// the matrix instructions' registers, then add up their sums in LDS.  The result's transpose is computed, so that a lane's four
// consecutive registers are four columns of a row.
__device__ __forceinline__ v8i operand(const uint4& c) { return v8i{(int)c.x, (int)c.y, (int)c.z, (int)c.w, 0, 0, 0, 0}; }

template <int MT, int NT, int KW, bool F32>
__global__ __launch_bounds__(64 * KW) void mx4_matmul_kernel(Packed a, Packed b, const float* __restrict__ bias, Matrix y, int columns) {
    constexpr int PITCH = 36;                                // floats; rows 16 bytes further along the banks
    __shared__ __attribute__((aligned(16))) float red[KW][32][PITCH];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int mt0 = blockIdx.x / columns * MT, nt0 = blockIdx.x % columns * NT;
    v16f acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
    const uint4 *pa[MT], *pb[NT];
    const uint32_t *ps[MT], *pt[NT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {                           // tiles beyond the last: the last one again
        const long long at = (long long)min_of(mt0 + i, a.tiles - 1) * a.steps;
        pa[i] = a.codes + at * 256 + lane;
        ps[i] = a.scales + at * 64 + lane;
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const long long at = (long long)min_of(nt0 + j, b.tiles - 1) * b.steps;
        pb[j] = b.codes + at * 256 + lane;
        pt[j] = b.scales + at * 64 + lane;
    }
    for (int s = wave; s < a.steps; s += KW) {
        uint4 ca[MT][4], cb[NT][4];
        uint32_t sa[MT], sb[NT];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
#pragma unroll
            for (int q = 0; q < 4; ++q) ca[i][q] = pa[i][s * 256 + q * 64];
            sa[i] = ps[i][s * 64];
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) {
#pragma unroll
            for (int q = 0; q < 4; ++q) cb[j][q] = pb[j][s * 256 + q * 64];
            sb[j] = pt[j][s * 64];
        }
        auto multiply = [&](auto q_tag) __attribute__((always_inline)) {
            constexpr int q = decltype(q_tag)::value;
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(cb[j][q]), operand(ca[i][q]), acc[i][j], 4, 4, q,
                                                                                (int)sb[j], q, (int)sa[i]);
        };
        multiply(Count<0>{}); multiply(Count<1>{}); multiply(Count<2>{}); multiply(Count<3>{});
    }
    const int M = y.all_rows(), N = y.all_cols(), h = lane >> 5;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            if (i + j > 0) __syncthreads();
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<float4*>(&red[wave][lane & 31][8 * q + 4 * h]) =
                    make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
            __syncthreads();
            for (int t = threadIdx.x; t < 256; t += 64 * KW) {
                const int m = t >> 3, n = 4 * (t & 7);
                float4 s = *reinterpret_cast<const float4*>(&red[0][m][n]);
#pragma unroll
                for (int k = 1; k < KW; ++k) {
                    const float4 o = *reinterpret_cast<const float4*>(&red[k][m][n]);
                    s.x += o.x; s.y += o.y; s.z += o.z; s.w += o.w;
                }
                const int row = (mt0 + i) * 32 + m, col = (nt0 + j) * 32 + n;
                if (row >= M || col >= N) continue;
                float v[4] = {s.x, s.y, s.z, s.w};
                char* dst = y.row(row) + y.column<F32 ? 4 : 2>(col);
                const int left = N - col;
                if (bias) {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (k < left) v[k] += bias[col + k];
                }
                if (left >= 4) {
                    if (F32) {
                        __builtin_memcpy(dst, v, 16);
                    } else {
                        const uint2 o = make_uint2(__builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{v[0], v[1]}, bf16x2)),
                                                   __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{v[2], v[3]}, bf16x2)));
                        __builtin_memcpy(dst, &o, 8);
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < 3; ++k)
                        if (k < left) {
                            if (F32) reinterpret_cast<float*>(dst)[k] = v[k];
                            else     reinterpret_cast<__bf16*>(dst)[k] = (__bf16)v[k];
                        }
                }
            }
        }
}

// ---- launches -----------------------------------------------------------------------------------
int launch_mx4_quantize(const fps_view& v, void* packed, hipStream_t st) {
    const Matrix x(v);
    const Packed p(packed, x.all_rows(), x.all_cols());
    const int waves = p.tiles * p.steps, grid = (waves + 3) / 4;
    if (v.dt == FPS_OUT_F32) mx4_quantize_kernel<true><<<grid, 256, 0, st>>>(x, (uint4*)p.codes, (uint32_t*)p.scales, p.steps, waves);
    else                     mx4_quantize_kernel<false><<<grid, 256, 0, st>>>(x, (uint4*)p.codes, (uint32_t*)p.scales, p.steps, waves);
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? FPS_OK : hip_fail(e, "mx4_quantize launch");
}

int launch_mx4_dequantize(const void* packed, const fps_view& v, hipStream_t st) {
    const Matrix y(v);
    const Packed p(packed, y.all_rows(), y.all_cols());
    const int waves = p.tiles * p.steps, grid = (waves + 3) / 4;
    if (v.dt == FPS_OUT_F32) mx4_dequantize_kernel<true><<<grid, 256, 0, st>>>(p, y, waves);
    else                     mx4_dequantize_kernel<false><<<grid, 256, 0, st>>>(p, y, waves);
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? FPS_OK : hip_fail(e, "mx4_dequantize launch");
}

template <int MT, int NT, int KW>
static int launch_direct(const Packed& a, const Packed& b, const float* bias, const fps_view& v, hipStream_t st) {
    const int columns = (b.tiles + NT - 1) / NT;
    const long long grid = (long long)((a.tiles + MT - 1) / MT) * columns;
    if (grid > 0x7FFFFFFF) { set_error("more tiles than a launch has workgroups for"); return FPS_ERR_UNSUPPORTED; }
    if (v.dt == FPS_OUT_F32) mx4_matmul_kernel<MT, NT, KW, true><<<(int)grid, 64 * KW, 0, st>>>(a, b, bias, Matrix(v), columns);
    else                     mx4_matmul_kernel<MT, NT, KW, false><<<(int)grid, 64 * KW, 0, st>>>(a, b, bias, Matrix(v), columns);
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? FPS_OK : hip_fail(e, "mx4_matmul launch");
}

int launch_mx4_matmul(int K, const void* a, const void* b, const float* bias, const fps_view& v, hipStream_t st) {
    const Packed pa(a, (long long)v.B * v.rows, K), pb(b, (long long)v.heads * v.cols, K);
    if (pa.steps < (1 << 22) && (long long)((pa.tiles + 7) / 8) * ((pb.tiles + 7) / 8) >= 128) return launch_mx4_large(a, b, K, bias, v, st);
    if (pa.tiles == 1) return launch_direct<1, 1, 8>(pa, pb, bias, v, st);
    return launch_direct<2, 2, 4>(pa, pb, bias, v, st);
}

}  // namespace fps
