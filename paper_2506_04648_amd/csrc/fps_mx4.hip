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

// the scale of a block whose largest magnitude has the bits `top`
struct BlockScale { uint32_t byte; float value; };
__device__ __forceinline__ BlockScale block_scale(uint32_t top) {
    const int e = (int)(top >> 23);
    const uint32_t byte = e == 255 ? 255u : top == 0 ? 127u : e > 2 ? (uint32_t)(e - 2) : 0u;
    return BlockScale{byte, __uint_as_float(e == 255 ? 0x3F800000u : byte == 0 ? 0x00400000u : byte << 23)};
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
    const BlockScale s = block_scale(top);
    const float scale = s.value;
    *byte = s.byte;
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

// codes and scale byte of the lane's block of quarter q of a step: row lane % 32 of the tile, 32 columns of lane / 32
template <bool F32>
__device__ __forceinline__ Block<F32> load_quarter(const Matrix& x, const char* row, bool real, int step, int q, int lane) {
    const int k = step * kMxStep + 64 * q + 32 * (lane >> 5), K = x.all_cols(), n = real && k < K ? K - k : 0;
    return load_block<F32>(row + (n > 0 ? x.column<F32 ? 4 : 2>(k) : 0), n);
}
// QS: quarters of a step that a wave takes, one or all four
template <bool F32, int QS>
__global__ __launch_bounds__(256) void mx4_quantize_kernel(Matrix x, uint4* __restrict__ codes, uint32_t* __restrict__ scales, int steps,
                                                           int waves) {
    const int wave = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (wave >= waves) return;
    const int at = QS == 4 ? wave : wave >> 2, q0 = QS == 4 ? 0 : wave & 3, tile = at / steps, step = at - tile * steps;
    const int r = tile * kMxRows + (lane & 31);
    const bool real = r < x.all_rows();
    const char* row = x.row(real ? r : 0);
    uint32_t word = 0;
#pragma unroll
    for (int q = q0; q < q0 + QS; ++q) {
        uint32_t byte;
        codes[((long long)at * 4 + q) * 64 + lane] = encode_block<F32>(load_quarter<F32>(x, row, real, step, q, lane), &byte);
        word |= byte << (8 * q);
        if (QS == 1) reinterpret_cast<uint8_t*>(scales)[((long long)at * 64 + lane) * 4 + q] = (uint8_t)byte;
    }
    if (QS == 4) scales[(long long)at * 64 + lane] = word;
}

// The same for matrices beyond the caches, read past them, which then keep the codes for the product: four lanes hold a block, 16 of them the
// 128 columns of a row, so that each load is whole lines (a lane's 64 bytes above are four loads of a line that has to stay); the codes
// go by way of the wave's own part of the LDS, whose instructions are carried out in their order.
template <bool F32>
__global__ __launch_bounds__(256) void mx4_quantize_rows_kernel(Matrix x, uint4* __restrict__ codes, uint32_t* __restrict__ scales, int steps,
                                                                int waves) {
    constexpr int E = F32 ? 4 : 2, WORDS = 2 * E, AT_ONCE = F32 ? 1 : 2, GROUP = 32 * 16 + 64, CODES = 8 * GROUP;     // 64 bytes: other banks
    __shared__ __attribute__((aligned(16))) uint8_t stage[4][CODES + kMxScaleBytes];
    const int wave = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (wave >= waves) return;
    uint8_t* const mine = stage[threadIdx.x >> 6];
    const int tile = wave / steps, step = wave - tile * steps, piece = lane & 3, blk = (lane >> 2) & 3, r4 = lane >> 4;
    const int M = x.all_rows(), K = x.all_cols();
    const char* row[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) row[i] = x.row(min_of(tile * kMxRows + 4 * i + r4, M - 1));
    typedef uint32_t words __attribute__((ext_vector_type(F32 ? 8 : 4)));
#pragma unroll
    for (int h0 = 0; h0 < 2; h0 += AT_ONCE) {
        words w[AT_ONCE][8];
#pragma unroll
        for (int half = 0; half < AT_ONCE; ++half) {
            const int k = step * kMxStep + 128 * (h0 + half) + 32 * blk + 8 * piece;
            const long long col = k < K ? x.column<E>(k) : 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int n = tile * kMxRows + 4 * i + r4 < M ? K - k : 0;
                words v = 0;
                if (n >= 8) {
                    typedef uint32_t chunk __attribute__((ext_vector_type(4), aligned(2)));       // rows start anywhere
#pragma unroll
                    for (int j = 0; j < WORDS / 4; ++j) {
                        const chunk c = __builtin_nontemporal_load(reinterpret_cast<const chunk*>(row[i] + col) + j);
                        v[4 * j] = c.x; v[4 * j + 1] = c.y; v[4 * j + 2] = c.z; v[4 * j + 3] = c.w;
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 7; ++j)
                        if (j < n) {
                            if (F32) v[j & 7] = reinterpret_cast<const uint32_t*>(row[i] + col)[j];
                            else     v[j >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(row[i] + col)[j] << (16 * (j & 1));
                        }
                }
                w[half][i] = v;
            }
        }
#pragma unroll
        for (int half = 0; half < AT_ONCE; ++half)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const words v = w[half][i];
                uint32_t top = 0;
#pragma unroll
                for (int j = 0; j < WORDS; ++j) {
                    const uint32_t lo = F32 ? v[j] & 0x7FFFFFFFu : v[j] << 16 & 0x7FFF0000u, hi = F32 ? 0u : v[j] & 0x7FFF0000u;
                    top = lo > top ? lo : top;
                    top = hi > top ? hi : top;
                }
                auto other = [&](auto ctrl) __attribute__((always_inline)) {
                    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, decltype(ctrl)::value, 0xf, 0xf, false);
                    top = o > top ? o : top;
                };
                other(Count<0xB1>{});
                other(Count<0x4E>{});
                const BlockScale s = block_scale(top);
                uint32_t r = 0;
                if constexpr (F32) {
                    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(v[0]), __uint_as_float(v[1]), s.value, 0);
                    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(v[2]), __uint_as_float(v[3]), s.value, 1);
                    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(v[4]), __uint_as_float(v[5]), s.value, 2);
                    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(v[6]), __uint_as_float(v[7]), s.value, 3);
                } else {
                    const uint32_t w0 = v[0], w1 = v[1], w2 = v[2], w3 = v[3];       // a cast of an element itself takes the first one
                    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w0), s.value, 0);
                    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w1), s.value, 1);
                    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w2), s.value, 2);
                    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w3), s.value, 3);
                }
                const int b4 = 4 * (h0 + half) + blk, n = 4 * i + r4;                // block of the step: quarter b4 / 2, half b4 % 2
                *reinterpret_cast<uint32_t*>(mine + b4 * GROUP + 16 * n + 4 * piece) = r;
                if (piece == 0) mine[CODES + (32 * (b4 & 1) + n) * 4 + (b4 >> 1)] = (uint8_t)s.byte;
            }
    }
    asm volatile("" ::: "memory");                           // the wave's reads stay behind its writes
#pragma unroll
    for (int q = 0; q < 4; ++q)
        codes[((long long)wave * 4 + q) * 64 + lane] = *reinterpret_cast<const uint4*>(mine + (2 * q + (lane >> 5)) * GROUP + 16 * (lane & 31));
    scales[(long long)wave * 64 + lane] = *reinterpret_cast<const uint32_t*>(mine + CODES + 4 * lane);
}

// Eight elements a lane, so that its 32 lanes store a row's 256 in a run; a wave two rows at a time, whose codes lie about the step's 4 KB.
template <bool F32>
__global__ __launch_bounds__(256) void mx4_dequantize_kernel(Packed p, Matrix y, int waves) {
    const int wave = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (wave >= waves) return;
    const int tile = wave / p.steps, step = wave - tile * p.steps, c = lane & 31, q = c >> 3, h = (c >> 2) & 1;
    const int k = step * kMxStep + 8 * c, K = y.all_cols(), M = y.all_rows(), r0 = tile * kMxRows + (lane >> 5);
    const uint32_t* codes = reinterpret_cast<const uint32_t*>(p.codes + (long long)wave * 256) + (q * 64 + 32 * h + (lane >> 5)) * 4 + (c & 3);
    const uint8_t* scales = reinterpret_cast<const uint8_t*>(p.scales + (long long)wave * 64) + (32 * h + (lane >> 5)) * 4 + q;
    constexpr int E = F32 ? 4 : 2;
    const long long col = k < K ? y.column<E>(k) : 0;
    uint32_t w[16], byte[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) { w[i] = codes[8 * i]; byte[i] = scales[8 * i]; }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int r = r0 + 2 * i;
        if (r >= M || k >= K) break;
        const float scale = scale_value(byte[i]);
        float f[8];
        auto two = [&](int j, const f32x2 v) __attribute__((always_inline)) { f[2 * j] = v[0] * scale; f[2 * j + 1] = v[1] * scale; };
        two(0, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], 1.0f, 0));
        two(1, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], 1.0f, 1));
        two(2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], 1.0f, 2));
        two(3, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], 1.0f, 3));
        uint32_t o[F32 ? 8 : 4];
#pragma unroll
        for (int j = 0; j < (F32 ? 8 : 4); ++j)
            o[j] = F32 ? __float_as_uint(f[j]) : __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{f[(2 * j) & 7], f[(2 * j + 1) & 7]}, bf16x2));
        char* dst = y.row(r) + col;
        if (k + 8 <= K) {
            __builtin_memcpy(dst, o, sizeof(o));
        } else {
#pragma unroll
            for (int j = 0; j < 7; ++j)
                if (k + j < K) {
                    if (F32) reinterpret_cast<uint32_t*>(dst)[j] = o[j & 7];
                    else     reinterpret_cast<uint16_t*>(dst)[j] = (uint16_t)(o[(j >> 1) & 3] >> (16 * (j & 1)));
                }
        }
    }
}

// ---- products -----------------------------------------------------------------------------------
// A workgroup of KW waves takes 32 rows and 32 columns; its waves share the steps of K, read the operands straight into the matrix
// instructions' registers, the next step's before they multiply this one's, and add up their sums in LDS.  The result's transpose is
// computed, so that a lane's four consecutive registers are four columns of a row.
__device__ __forceinline__ v8i operand(const uint4& c) { return v8i{(int)c.x, (int)c.y, (int)c.z, (int)c.w, 0, 0, 0, 0}; }

template <int KW, bool F32>
__global__ __launch_bounds__(64 * KW) void mx4_matmul_kernel(Packed a, Packed b, const float* __restrict__ bias, Matrix y) {
    constexpr int PITCH = 36;                                // floats: rows 16 bytes further along the banks
    __shared__ __attribute__((aligned(16))) float red[KW][32][PITCH];
    const int lane = threadIdx.x & 63, kw = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const int mt = blockIdx.x / b.tiles, nt = blockIdx.x - mt * b.tiles, m = threadIdx.x >> 3, col = nt * 32 + 4 * (threadIdx.x & 7);
    const int M = y.all_rows(), N = y.all_cols();
    const long long at_a = (long long)mt * a.steps, at_b = (long long)nt * b.steps;
    const uint4 *pa = a.codes + at_a * 256 + lane, *pb = b.codes + at_b * 256 + lane;
    const uint32_t *ps = a.scales + at_a * 64 + lane, *pt = b.scales + at_b * 64 + lane;
    struct Operands { uint4 a[4], b[4]; uint32_t sa, sb; };
    auto fetch = [&](Operands& o, int s) __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < 4; ++q) o.b[q] = pb[s * 256LL + q * 64];
        o.sb = pt[s * 64LL];
#pragma unroll
        for (int q = 0; q < 4; ++q) o.a[q] = pa[s * 256LL + q * 64];
        o.sa = ps[s * 64LL];
    };
    v16f acc = {};
    auto multiply = [&](const Operands& o) __attribute__((always_inline)) {
        auto quarter = [&](auto q_tag) __attribute__((always_inline)) {
            constexpr int q = decltype(q_tag)::value;
            acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(o.b[q]), operand(o.a[q]), acc, 4, 4, q, (int)o.sb, q, (int)o.sa);
        };
        quarter(Count<0>{}); quarter(Count<1>{}); quarter(Count<2>{}); quarter(Count<3>{});
    };
    Operands one, other;
    if (kw < a.steps) fetch(one, kw);
    float add[4];                                            // the bias of the thread's columns
#pragma unroll
    for (int k = 0; k < 4; ++k) add[k] = bias && col + k < N ? bias[col + k] : 0.0f;
    for (int s = kw; s < a.steps; s += 2 * KW) {
        if (s + KW < a.steps) fetch(other, s + KW);
        multiply(one);
        if (s + KW >= a.steps) break;
        if (s + 2 * KW < a.steps) fetch(one, s + 2 * KW);
        multiply(other);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4*>(&red[kw][lane & 31][8 * q + 4 * h]) = make_float4(acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]);
    __syncthreads();
    if (m >= 32 || mt * 32 + m >= M || col >= N) return;
    float4 s = *reinterpret_cast<const float4*>(&red[0][m][4 * (threadIdx.x & 7)]);
#pragma unroll
    for (int k = 1; k < KW; ++k) {
        const float4 o = *reinterpret_cast<const float4*>(&red[k][m][4 * (threadIdx.x & 7)]);
        s.x += o.x; s.y += o.y; s.z += o.z; s.w += o.w;
    }
    const float v[4] = {s.x + add[0], s.y + add[1], s.z + add[2], s.w + add[3]};
    char* dst = y.row(mt * 32 + m) + y.column<F32 ? 4 : 2>(col);
    const int left = N - col;
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

// ---- launches -----------------------------------------------------------------------------------
// Fewer than 1024 tiles' steps: a quarter of a step a wave, and four times as many waves.  851 x 1536 in bf16 7.2 -> 3.7 us.  More than the Infinity
// Cache's 256 MB: past the caches.  75600 x 5120 in bf16 184 -> 155 us (6.3 TB/s), from heads 182 -> 161, and the product behind it 875 -> 890;
// 32760 x 1536, which the cache holds, 20.4 us (6.2 TB/s), past the caches 22.4.
int launch_mx4_quantize(const fps_view& v, void* packed, hipStream_t st) {
    const Matrix x(v);
    const Packed p(packed, x.all_rows(), x.all_cols());
    const int at = p.tiles * p.steps;
    FPS_TRY(check_launch((at + 3) / 4, 256, "mx4_quantize"));
    auto launch = [&](auto f32, auto qs) {
        constexpr int QS = decltype(qs)::value;
        const int waves = QS == 4 ? at : 4 * at;
        mx4_quantize_kernel<decltype(f32)::value, QS><<<(waves + 3) / 4, 256, 0, st>>>(x, (uint4*)p.codes, (uint32_t*)p.scales, p.steps, waves);
    };
    auto typed = [&](auto f32) {
        constexpr bool F32 = decltype(f32)::value;
        if ((long long)x.all_rows() * x.all_cols() * (F32 ? 4 : 2) > (256LL << 20))
            mx4_quantize_rows_kernel<F32><<<(at + 3) / 4, 256, 0, st>>>(x, (uint4*)p.codes, (uint32_t*)p.scales, p.steps, at);
        else if (at < 1024) launch(f32, Count<1>{});
        else                launch(f32, Count<4>{});
    };
    if (v.dt == FPS_OUT_F32) typed(std::true_type{});
    else                     typed(std::false_type{});
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? FPS_OK : hip_fail(e, "mx4_quantize launch");
}

int launch_mx4_dequantize(const void* packed, const fps_view& v, hipStream_t st) {
    const Matrix y(v);
    const Packed p(packed, y.all_rows(), y.all_cols());
    const int waves = p.tiles * p.steps, grid = (waves + 3) / 4;
    FPS_TRY(check_launch(grid, 256, "mx4_dequantize"));
    if (v.dt == FPS_OUT_F32) mx4_dequantize_kernel<true><<<grid, 256, 0, st>>>(p, y, waves);
    else                     mx4_dequantize_kernel<false><<<grid, 256, 0, st>>>(p, y, waves);
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? FPS_OK : hip_fail(e, "mx4_dequantize launch");
}

template <int KW>
static int launch_direct(const Packed& a, const Packed& b, const float* bias, const fps_view& v, hipStream_t st) {
    const long long grid = (long long)a.tiles * b.tiles;
    FPS_TRY(check_launch(grid, 64 * KW, "mx4_matmul"));
    if (v.dt == FPS_OUT_F32) mx4_matmul_kernel<KW, true><<<(int)grid, 64 * KW, 0, st>>>(a, b, bias, Matrix(v));
    else                     mx4_matmul_kernel<KW, false><<<(int)grid, 64 * KW, 0, st>>>(a, b, bias, Matrix(v));
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? FPS_OK : hip_fail(e, "mx4_matmul launch");
}

// Which product.  us of the product alone, captured and replayed, rows x K x columns:
//   straight into registers (tiles of 32, K shared by 4 / 8 waves) against tiles of 128 by way of LDS, of which there are
//     1 x 5120 x 30720     13.4 / 13.3    14.6   240       300 x 1536 x 4608     5.5 /  6.4     6.0   108
//     128 x 5120 x 5120     6.4 /  6.3    10.9    40       64 x 5120 x 15360    11.6 / 12.7    11.4   120
//     96 x 20480 x 5120    17.5 / 19.2    33.2    40       400 x 1536 x 4608     6.0 /  7.9     6.1   144
//     256 x 5120 x 5120     9.6 /  9.5    11.1    80       33 x 5120 x 30720    25.1 / 24.9    15.3   240
//     1 x 20480 x 5120     11.9 / 11.3    32.6    40       851 x 1536 x 4608    10.8 / 14.1     7.0   252
//   so those of 128 from 112 of them on, with more rows than 32; eight waves only for few tiles and a long K;
//   tiles of 256, one a CU at a time, against tiles of 128, two a CU that take 1.7 of the time together (3.4 for 5 where there are many):
//     2048 x 5120 x 5120    33.8   34.3                     32760 x 1536 x 1536  54.5   52.3
//     4255 x 1536 x 4608    28.7   24.0                     8192 x 5120 x 5120    110    113
//     8000 x 1536 x 1536    18.0   16.6                     75600 x 5120 x 5120   887   1116
//   which the rounds of 256 tiles that the CUs make tell apart.
int launch_mx4_matmul(int K, const void* a, const void* b, const float* bias, const fps_view& v, hipStream_t st) {
    const Packed pa(a, (long long)v.B * v.rows, K), pb(b, (long long)v.heads * v.cols, K);
    const long long in_256 = (pa.tiles + 7LL) / 8 * ((pb.tiles + 7LL) / 8), in_128 = (pa.tiles + 3LL) / 4 * ((pb.tiles + 3LL) / 4);
    if (pa.tiles > 1 && in_128 >= 112 && pa.steps < (1 << 22)) {
        const bool large = 34 * ((in_256 + 255) / 256) <= 10 * ((in_128 + 255) / 256) + 3;
        return launch_mx4_tiles(large ? 256 : 128, a, b, K, bias, v, st);
    }
    if (pa.steps >= 16 && (long long)pa.tiles * pb.tiles <= 256) return launch_direct<8>(pa, pb, bias, v, st);
    return launch_direct<4>(pa, pb, bias, v, st);
}

int launch_mx4_linear(const fps_view& x, const void* w, const float* bias, const fps_view& v, void* workspace, hipStream_t st) {
    const int rc = launch_mx4_quantize(x, workspace, st);
    return rc == FPS_OK ? launch_mx4_matmul(x.heads * x.cols, workspace, w, bias, v, st) : rc;
}

}  // namespace fps
