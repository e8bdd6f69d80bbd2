// Each head's RMS norm of Q and K and the rotation by the token's place (t,h,w), in one pass: into the caller's layout, or
// straight into the packed operands of the attention; the gradient of both; and the values of packed E4M3 operands.
//
//   y = R(t,h,w) (x r w),  r = (mean x^2 + eps)^(-1/2),  R: 64 rotations of pairs of channels
//   g = R^T dy,  dw = sum g x r,  dx = r (g w - x r^2 mean(g w x))
//
// All of it is bound by HBM: some ten operations an element.  Eight lanes hold a row of 128 channels, 16 channels or 8
// pairs each, so that a row is one 16-byte load (two, four) of each lane, the sum over it three exchanges between neighbouring
// lanes, and a pair never leaves its lane.  The rotation's tables are as long as the axes: 20 KB at 720p, read from the caches.
#include "fps_device_common.h"

namespace fps {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}
__device__ __forceinline__ float low_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_bf16(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Strides of a tensor [B, heads, tokens, 128] in bytes
struct Rows {
    const char* data;
    long long b, h, r;
    __device__ const char* at(int bi, int hi, int n) const { return data + bi * b + hi * h + n * r; }
};

// What the norm and the rotation are, and where tokens stand
struct Turning {
    const float* weight;             // NULL: ones
    int weight_head;                 // floats from head to head: 128, or 0 if they share
    float eps;
    bool norm;
    const float* table;              // NULL: no rotation
    long long table_b;
    int ct, ch, cw;
    int T, H, W;
    uint32_t rc_plane, rc_row;       // reciprocals of H*W and W
};

// 8 pairs of channels of a row: unit u of 8.  Adjacent pairs: channels 16u..16u+15; halves: 8u..8u+7 and those + 64.
struct Pairs { float a[8], b[8]; };
template <bool F32> struct Chunks { uint4 v[F32 ? 4 : 2]; };

template <bool F32, bool HALVES>
__device__ __forceinline__ Chunks<F32> load_pairs(const char* row, int u) {
    constexpr int N = F32 ? 4 : 2, E = F32 ? 4 : 2;         // 16-byte loads; bytes an element
    Chunks<F32> c;
    const char* p = row + u * (HALVES ? 8 * E : 16 * E);
#pragma unroll
    for (int i = 0; i < N; ++i)
        c.v[i] = *reinterpret_cast<const uint4*>(p + (HALVES ? (i % (N / 2)) * 16 + (i / (N / 2)) * 64 * E : 16 * i));
    return c;
}
template <bool F32, bool HALVES>
__device__ __forceinline__ Pairs unpack(const Chunks<F32>& c) {
    Pairs p;
    float f[16];
    const uint32_t* w = reinterpret_cast<const uint32_t*>(c.v);
#pragma unroll
    for (int i = 0; i < 16; ++i) f[i] = F32 ? __uint_as_float(w[i]) : (i & 1) ? high_bf16(w[i >> 1]) : low_bf16(w[i >> 1]);
#pragma unroll
    for (int i = 0; i < 8; ++i) { p.a[i] = f[HALVES ? i : 2 * i]; p.b[i] = f[HALVES ? 8 + i : 2 * i + 1]; }
    return p;
}
template <bool F32, bool HALVES>
__device__ __forceinline__ void store_pairs(char* row, int u, const Pairs& p) {
    constexpr int N = F32 ? 4 : 2, E = F32 ? 4 : 2;
    float f[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) { f[HALVES ? i : 2 * i] = p.a[i]; f[HALVES ? 8 + i : 2 * i + 1] = p.b[i]; }
    Chunks<F32> c;
    uint32_t* w = reinterpret_cast<uint32_t*>(c.v);
#pragma unroll
    for (int i = 0; i < (F32 ? 16 : 8); ++i) w[i] = F32 ? __float_as_uint(f[i]) : pack_bf16(f[2 * i], f[2 * i + 1]);
    char* q = row + u * (HALVES ? 8 * E : 16 * E);
#pragma unroll
    for (int i = 0; i < N; ++i)
        *reinterpret_cast<uint4*>(q + (HALVES ? (i % (N / 2)) * 16 + (i / (N / 2)) * 64 * E : 16 * i)) = c.v[i];
}

// Cosines and sines of the unit's pairs 8u..8u+7 for token (t,h,w); pairs that do not turn: (1, 0)
struct Turn { float c[8], s[8]; };
__device__ __forceinline__ Turn load_turn(const Turning& k, const float2* table, int T, int H, int t, int h, int w, int u) {
    Turn r;                                                  // from a table of T places and H places before those of w
#pragma unroll
    for (int i = 0; i < 8; ++i) { r.c[i] = 1.0f; r.s[i] = 0.0f; }
    const int at_t = t * k.ct, at_h = T * k.ct + h * k.ch - k.ct, at_w = T * k.ct + H * k.ch + w * k.cw - k.ct - k.ch;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int p = 8 * u + i;
        if (p < k.ct + k.ch + k.cw) {                        // none without a rotation
            const float2 cs = table[(p < k.ct ? at_t : p < k.ct + k.ch ? at_h : at_w) + p];
            r.c[i] = cs.x;
            r.s[i] = cs.y;
        }
    }
    return r;
}
__device__ __forceinline__ Turn load_turn_of_token(const Turning& k, int b, int n, int u) {
    const int t = quotient(n, k.H * k.W, k.rc_plane), rem = n - t * (k.H * k.W), h = quotient(rem, k.W, k.rc_row);
    return load_turn(k, reinterpret_cast<const float2*>(k.table + b * k.table_b), k.T, k.H, t, h, rem - h * k.W, u);
}
template <bool HALVES>
__device__ __forceinline__ Pairs load_weight(const Turning& k, int h, int u) {
    if (k.weight) return unpack<true, HALVES>(load_pairs<true, HALVES>((const char*)(k.weight + h * k.weight_head), u));
    Pairs p;
#pragma unroll
    for (int i = 0; i < 8; ++i) p.a[i] = p.b[i] = 1.0f;
    return p;
}

// sum over the eight lanes of a row
__device__ __forceinline__ float row_sum(float x) {
    auto add = [&](auto ctrl) {
        x += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), decltype(ctrl)::value, 0xf, 0xf, false));
    };
    add(Count<0xB1>{});            // the neighbour of a pair of lanes
    add(Count<0x4E>{});            // the other pair of four
    add(Count<0x141>{});           // the other four of eight
    return x;
}
__device__ __forceinline__ float inverse_rms(const Turning& k, const Pairs& x) {
    if (!k.norm) return 1.0f;
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s = __builtin_fmaf(x.a[i], x.a[i], __builtin_fmaf(x.b[i], x.b[i], s));
    return __builtin_amdgcn_rsqf(row_sum(s) * (1.0f / 128.0f) + k.eps);
}
__device__ __forceinline__ Pairs norm_rotated(const Turning& k, const Pairs& x, const Pairs& w, const Turn& turn) {
    const float r = inverse_rms(k, x);
    Pairs y;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float a = x.a[i] * r * w.a[i], b = x.b[i] * r * w.b[i];
        y.a[i] = __builtin_fmaf(a, turn.c[i], -(b * turn.s[i]));
        y.b[i] = __builtin_fmaf(a, turn.s[i], b * turn.c[i]);
    }
    return y;
}

// ---- into the caller's layout -------------------------------------------------------------------
// A wave takes eight tokens; each of its rows' cosines and sines are read once for HC heads.
template <bool IN32, bool OUT32, bool HALVES, int HC>
__global__ __launch_bounds__(256) void norm_rotate_kernel(Rows x, Rows y, Turning k, int tokens, int heads, int parts) {
    const int blocks = (int)((tokens + 31u) >> 5), bp = blockIdx.x / blocks;        // tokens fastest
    const int u = threadIdx.x & 7, n = (blockIdx.x - bp * blocks) * 32 + (threadIdx.x >> 3);
    const int b = bp / parts, h0 = (bp - b * parts) * HC;
    if (n >= tokens) return;                                 // whole rows of lanes
    Chunks<IN32> c[HC];
#pragma unroll
    for (int i = 0; i < HC; ++i)
        if (h0 + i < heads) c[i] = load_pairs<IN32, HALVES>(x.at(b, h0 + i, n), u);
    const Turn turn = load_turn_of_token(k, b, n, u);
#pragma unroll
    for (int i = 0; i < HC; ++i) {
        if (h0 + i >= heads) break;
        const Pairs w = load_weight<HALVES>(k, h0 + i, u);
        store_pairs<OUT32, HALVES>(const_cast<char*>(y.at(b, h0 + i, n)), u, norm_rotated(k, unpack<IN32, HALVES>(c[i]), w, turn));
    }
}

// ---- into the packed operands -------------------------------------------------------------------
// As quantize_tiles_kernel (and pack_bf16_kernel): a workgroup is one scale group of up to three blocks, held in
// registers from the reading to the encoding; of larger groups a block, of which PASS 0 finds the maximum and PASS 1, which
// reads x again, encodes.
// A token's cosines and sines would be four times as many load instructions as its channels: where the entries of the
// group's planes, rows and columns are at most kStaged they are brought into LDS first.
constexpr int kWhole = -1, kStaged = 1024;
template <int BS, int THREADS, bool IN32, bool HALVES, bool FP8, int NB, int PASS>
__global__ __launch_bounds__(THREADS * NB) void norm_rotate_operand_kernel(Rows x, Turning k, uint8_t* __restrict__ xq,
                                                                           float* __restrict__ scales, int role, Geom g,
                                                                           int heads) {
    constexpr int U = BS * 8 / THREADS, WAVES = THREADS * NB / 64;
    __shared__ uint32_t red[WAVES];
    __shared__ float2 staged[kStaged];
    const int kb = NB > 1 ? (int)threadIdx.x / THREADS : 0, tid = threadIdx.x - kb * THREADS, u = tid & 7;
    const int blk = blockIdx.x * NB + kb;
    const BlockOrigin org = block_origin(g, blockIdx.x * NB);
    const int bh = quotient((int)org.tile_lin, g.M, g.rc_m), b = bh / heads, head = bh - b * heads;
    const int n0 = (int)(org.raster0 - (long long)bh * g.T * g.H * g.W);
    const Pairs weight = load_weight<HALVES>(k, head, u);

    Chunks<IN32> in[U];
    Offset token[U];                                         // from the group's first; t < 0: padding
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int slot = org.slot0 + kb * BS + (tid >> 3) + THREADS / 8 * i;
        token[i] = real_token(org.box, slot);
        if (slot < org.box.n) in[i] = load_pairs<IN32, HALVES>(x.at(b, head, n0 + (token[i].t * g.H + token[i].h) * g.W + token[i].w), u);
        else                  token[i].t = -1;
    }
    // the group's entries: its planes', rows' and columns' are three runs of the table
    const int t0 = quotient(n0, g.H * g.W, k.rc_plane), h0 = quotient(n0 - t0 * (g.H * g.W), g.W, k.rc_row), w0 = n0 - (t0 * g.H + h0) * g.W;
    const int et = org.box.n ? real_token(org.box, org.box.n - 1).t + 1 : 0, of_t = et * k.ct, of_h = org.box.eh * k.ch, of_w = org.box.ew * k.cw;
    const bool in_lds = of_t + of_h + of_w <= kStaged;
    const float2* table = reinterpret_cast<const float2*>(k.table + b * k.table_b);
    if (k.table && in_lds && et > 0) {
        for (int i = threadIdx.x; i < of_t + of_h + of_w; i += THREADS * NB)
            staged[i] = table[i < of_t ? t0 * k.ct + i
                                       : i < of_t + of_h ? g.T * k.ct + h0 * k.ch + i - of_t : g.T * k.ct + g.H * k.ch + w0 * k.cw + i - of_t - of_h];
    }
    __syncthreads();
    Pairs y[U];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < U; ++i) {
        if (token[i].t >= 0) {
            const Offset d = token[i];
            const Turn turn = in_lds ? load_turn(k, staged, et, org.box.eh, d.t, d.h, d.w, u)
                                     : load_turn(k, table, g.T, g.H, t0 + d.t, h0 + d.h, w0 + d.w, u);
            y[i] = norm_rotated(k, unpack<IN32, HALVES>(in[i]), weight, turn);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) y[i].a[j] = y[i].b[j] = 0.0f;
        }
        if (FP8 && PASS != 1) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {                    // magnitudes order like their bits, NaN above all
                const uint32_t ma = __float_as_uint(y[i].a[j]) & 0x7FFFFFFFu, mb = __float_as_uint(y[i].b[j]) & 0x7FFFFFFFu;
                top = top > ma ? top : ma;
                top = top > mb ? top : mb;
            }
        }
    }
    char* const dst = (char*)xq + (long long)blk * (BS * 128 * (FP8 ? 1 : 2));
    if constexpr (!FP8) {                                    // 8 channels are a chunk of 16 bytes
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int j = (tid >> 3) + THREADS / 8 * i;
            float f[16];
#pragma unroll
            for (int m = 0; m < 8; ++m) { f[HALVES ? m : 2 * m] = y[i].a[m]; f[HALVES ? 8 + m : 2 * m + 1] = y[i].b[m]; }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int c8 = HALVES ? u + 8 * half : 2 * u + half;
                int c = j * 16 + c8;
                if (role == FPS_ROLE_K) c = ((j >> 5) * 8 + (c8 >> 1)) * 64 + 32 * (c8 & 1) + (j & 31);
                uint4 o;
                o.x = pack_bf16(f[8 * half], f[8 * half + 1]);
                o.y = pack_bf16(f[8 * half + 2], f[8 * half + 3]);
                o.z = pack_bf16(f[8 * half + 4], f[8 * half + 5]);
                o.w = pack_bf16(f[8 * half + 6], f[8 * half + 7]);
                reinterpret_cast<uint4*>(dst)[c] = o;
            }
        }
        return;
    }
    if (PASS == 1) {
        top = __float_as_uint(scales[quotient(blockIdx.x, g.KBS, g.rc_kbs)]);
    } else {
        top = workgroup_max<WAVES>(top, red);
        if (PASS == 0) {
            if (threadIdx.x == 0) atomicMax((uint32_t*)&scales[quotient(blockIdx.x, g.KBS, g.rc_kbs)], top);
            return;
        }
    }
    const float amax = __uint_as_float(top), s = top == 0 ? 1.0f : amax / 448.0f;
    if (PASS == kWhole && threadIdx.x == 0) scales[blockIdx.x] = s;
    // a scale near the end of the range: its reciprocal would pass it
    const float up = s < 0x1p-60f ? 0x1p64f : 1.0f, rs = 1.0f / (s * up);
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int j = (tid >> 3) + THREADS / 8 * i;
        float f[16];
#pragma unroll
        for (int m = 0; m < 8; ++m) {
            f[HALVES ? m : 2 * m] = y[i].a[m] * up * rs;
            f[HALVES ? 8 + m : 2 * m + 1] = y[i].b[m] * up * rs;
        }
        uint32_t o[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) {                        // |x| <= amax: the product cannot reach the next code, 480
            int r = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * m], f[4 * m + 1], 0, false);
            o[m] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * m + 2], f[4 * m + 3], r, true);
        }
        // the 16-byte chunk of channels 16 c16.., of which a unit of halves has eight bytes each of two
        auto chunk = [&](int c16) {
            return role == FPS_ROLE_K ? (((j >> 5) * 2 + (c16 >> 2)) * 2 + (c16 & 1)) * 64 + 32 * ((c16 >> 1) & 1) + (j & 31)
                                      : j * 8 + c16;
        };
        if (HALVES) {
            *reinterpret_cast<uint2*>(dst + 16 * chunk(u >> 1) + 8 * (u & 1)) = make_uint2(o[0], o[1]);
            *reinterpret_cast<uint2*>(dst + 16 * chunk(4 + (u >> 1)) + 8 * (u & 1)) = make_uint2(o[2], o[3]);
        } else {
            reinterpret_cast<uint4*>(dst)[chunk(u)] = make_uint4(o[0], o[1], o[2], o[3]);
        }
    }
}

// ---- the gradient -------------------------------------------------------------------------------
// A workgroup takes 32 tokens at a time of HC heads (of one head, always the same, if they have weights of their own), reads the rows of all
// of them at once and their cosines and sines once, and keeps its lanes' share of dweight in registers; the workgroups' sums are
// added up by a second kernel, in a fixed order.
template <bool F32, bool HALVES, int HC>
__global__ __launch_bounds__(256) void norm_rotate_bwd_kernel(Rows x, Rows dy, Rows dx, Turning k, float* __restrict__ partial,
                                                              int tokens, int heads, int batches, int workgroups) {
    __shared__ float red[4][128];
    const int u = threadIdx.x & 7, row = threadIdx.x >> 3, parts = (int)((tokens + 31u) >> 5);
    const int group = blockIdx.x / workgroups, first = blockIdx.x - group * workgroups;
    const int own_head = k.weight_head ? group : -1, per = own_head >= 0 ? 1 : (heads + HC - 1) / HC;
    const long long items = (long long)batches * parts * per;               // (batch, token part, heads)
    Pairs dw;
#pragma unroll
    for (int i = 0; i < 8; ++i) dw.a[i] = dw.b[i] = 0.0f;
    for (long long item = first; item < items; item += workgroups) {
        const long long bp = item / per;
        const int h0 = own_head >= 0 ? own_head : (int)(item - bp * per) * HC, b = (int)(bp / parts);
        const int n = (int)(bp - (long long)b * parts) * 32 + row, last = own_head >= 0 ? h0 + 1 : heads;
        if (n >= tokens) continue;
        Chunks<F32> cx[HC], cy[HC];
#pragma unroll
        for (int i = 0; i < HC; ++i)
            if (h0 + i < last) {
                cx[i] = load_pairs<F32, HALVES>(x.at(b, h0 + i, n), u);
                cy[i] = load_pairs<F32, HALVES>(dy.at(b, h0 + i, n), u);
            }
        const Turn turn = load_turn_of_token(k, b, n, u);
        const Pairs w = load_weight<HALVES>(k, h0, u);                       // of all of them, or of the one
#pragma unroll
        for (int i = 0; i < HC; ++i) {
            if (h0 + i >= last) break;
            const Pairs xv = unpack<F32, HALVES>(cx[i]), g0 = unpack<F32, HALVES>(cy[i]);
            const float r = inverse_rms(k, xv);
            Pairs g;
            float dot = 0.0f;
#pragma unroll
            for (int m = 0; m < 8; ++m) {
                const float ga = __builtin_fmaf(g0.a[m], turn.c[m], g0.b[m] * turn.s[m]);
                const float gb = __builtin_fmaf(g0.b[m], turn.c[m], -(g0.a[m] * turn.s[m]));
                dw.a[m] = __builtin_fmaf(ga, xv.a[m] * r, dw.a[m]);
                dw.b[m] = __builtin_fmaf(gb, xv.b[m] * r, dw.b[m]);
                g.a[m] = ga * w.a[m];
                g.b[m] = gb * w.b[m];
                dot = __builtin_fmaf(g.a[m], xv.a[m], __builtin_fmaf(g.b[m], xv.b[m], dot));
            }
            const float back = k.norm ? row_sum(dot) * (1.0f / 128.0f) * r * r : 0.0f;
            Pairs d;
#pragma unroll
            for (int m = 0; m < 8; ++m) {
                d.a[m] = r * __builtin_fmaf(-xv.a[m], back, g.a[m]);
                d.b[m] = r * __builtin_fmaf(-xv.b[m], back, g.b[m]);
            }
            store_pairs<F32, HALVES>(const_cast<char*>(dx.at(b, h0 + i, n)), u, d);
        }
    }
    if (!partial) return;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int off = 8; off < 64; off <<= 1) {
            dw.a[i] += __shfl_xor(dw.a[i], off);
            dw.b[i] += __shfl_xor(dw.b[i], off);
        }
    if ((threadIdx.x & 63) < 8)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            red[threadIdx.x >> 6][HALVES ? 8 * u + i : 16 * u + 2 * i] = dw.a[i];
            red[threadIdx.x >> 6][HALVES ? 64 + 8 * u + i : 16 * u + 2 * i + 1] = dw.b[i];
        }
    __syncthreads();
    if (threadIdx.x < 128) {
        const int c = threadIdx.x;
        partial[(long long)blockIdx.x * 128 + c] = (red[0][c] + red[1][c]) + (red[2][c] + red[3][c]);
    }
}
// Eight channels a workgroup, 32 slices of the n partial sums
__global__ __launch_bounds__(256) void sum_partials_kernel(const float* __restrict__ partial, float* __restrict__ out, int n) {
    __shared__ float red[32][9];
    const int c = threadIdx.x & 7, slice = threadIdx.x >> 3, group = blockIdx.x >> 4, c0 = 8 * (blockIdx.x & 15);
    const float* p = partial + (long long)group * n * 128 + c0 + c;
    float s = 0.0f;
#pragma unroll 8
    for (int i = slice; i < n; i += 32) s += p[(long long)i * 128];
    red[slice][c] = s;
    __syncthreads();
    if (threadIdx.x < 8) {
        float t = 0.0f;
#pragma unroll
        for (int i = 0; i < 32; ++i) t += red[i][threadIdx.x];
        out[group * 128 + c0 + threadIdx.x] = t;
    }
}

// ---- the values of packed E4M3 operands ---------------------------------------------------------
// A workgroup takes a block of BS slots: sixteen lanes a token, 8 codes each, so that a row of bf16 is one store of its lanes; all of
// a thread's codes are requested at once.  V's block is turned back in LDS first.
template <int BS, bool F32, bool V>
__global__ __launch_bounds__(256) void dequantize_kernel(const uint8_t* __restrict__ xq, const float* __restrict__ scales,
                                                         int role, int per_channel, char* __restrict__ out, Geom g) {
    constexpr int U = BS * 16 / 256;                         // 8-byte units a thread
    __shared__ __attribute__((aligned(16))) uint8_t stage[V ? BS * 128 : 16];
    const BlockOrigin org = block_origin(g, blockIdx.x);
    const uint8_t* src = xq + (long long)blockIdx.x * (BS * 128);
    const int c8 = threadIdx.x & 15;
    uint2 codes[U];
    if (V) {
        uint4 v[(U + 1) / 2];
#pragma unroll
        for (int i = 0; i < (U + 1) / 2; ++i) {
            const int c = threadIdx.x + 256 * i;
            if (c < BS * 8) v[i] = reinterpret_cast<const uint4*>(src)[c];
        }
#pragma unroll
        for (int i = 0; i < (U + 1) / 2; ++i) {
            const int c = threadIdx.x + 256 * i, lane = c & 63, db = (c >> 6) & 3, kb = c >> 8, h = lane >> 5, n = lane & 31;
            if (c >= BS * 8) break;
            union { uint4 v; uint8_t b[16]; } o;
            o.v = v[i];
#pragma unroll
            for (int jj = 0; jj < 16; ++jj) stage[(32 * kb + 8 * (jj >> 2) + 4 * h + (jj & 3)) * 128 + 32 * db + n] = o.b[jj];
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int j = (threadIdx.x >> 4) + 16 * i, c16 = c8 >> 1;
        int at = j * 8 + c16;                                // 16-byte chunk of the block
        if (!V && role == FPS_ROLE_K) at = (((j >> 5) * 2 + (c16 >> 2)) * 2 + (c16 & 1)) * 64 + 32 * ((c16 >> 1) & 1) + (j & 31);
        codes[i] = *reinterpret_cast<const uint2*>((V ? stage : src) + 16 * at + 8 * (c8 & 1));
    }
    const int bh = quotient((int)org.tile_lin, g.M, g.rc_m);
    float s[8];
    if (V && per_channel) {
        const float4 lo = reinterpret_cast<const float4*>(scales + bh * 128)[2 * c8], hi = reinterpret_cast<const float4*>(scales + bh * 128)[2 * c8 + 1];
        s[0] = lo.x; s[1] = lo.y; s[2] = lo.z; s[3] = lo.w; s[4] = hi.x; s[5] = hi.y; s[6] = hi.z; s[7] = hi.w;
    } else {
        const float of_group = scales[quotient(blockIdx.x, g.KBS, g.rc_kbs)];
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k] = of_group;
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int slot = org.slot0 + (threadIdx.x >> 4) + 16 * i;
        if (slot >= org.box.n) break;
        const Offset d = real_token(org.box, slot);
        float f[8];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint32_t w = k ? codes[i].y : codes[i].x;
            const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
            f[4 * k] = lo[0] * s[4 * k];         f[4 * k + 1] = lo[1] * s[4 * k + 1];
            f[4 * k + 2] = hi[0] * s[4 * k + 2]; f[4 * k + 3] = hi[1] * s[4 * k + 3];
        }
        char* dst = out + (org.raster0 + ((long long)d.t * g.H + d.h) * g.W + d.w) * (F32 ? 512 : 256) + c8 * (F32 ? 32 : 16);
        if (F32) {
            reinterpret_cast<float4*>(dst)[0] = make_float4(f[0], f[1], f[2], f[3]);
            reinterpret_cast<float4*>(dst)[1] = make_float4(f[4], f[5], f[6], f[7]);
        } else {
            *reinterpret_cast<uint4*>(dst) = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
        }
    }
}

// ---- launches -----------------------------------------------------------------------------------
static Rows rows_of(const fps_view& v) {
    const long long e = v.dt == FPS_OUT_F32 ? 4 : 2;
    return Rows{(const char*)v.data, v.B > 1 ? v.stride_b * e : 0, v.heads > 1 ? v.stride_h * e : 0, v.rows > 1 ? v.stride_r * e : 0};
}
static Turning turning_of(const Geom& g, const fps_norm* norm, const fps_rotation* rot) {
    Turning k = {};
    if (norm) {
        k.norm = true;
        k.weight = norm->weight;
        k.weight_head = norm->weight && norm->per_head ? 128 : 0;
        k.eps = norm->eps;
    }
    if (rot && rot->pairs_t + rot->pairs_h + rot->pairs_w > 0) {
        k.table = rot->table;
        k.table_b = rot->stride_b;
        k.ct = rot->pairs_t; k.ch = rot->pairs_h; k.cw = rot->pairs_w;
    }
    k.T = g.T; k.H = g.H; k.W = g.W;
    k.rc_plane = reciprocal(g.H * g.W);
    k.rc_row = reciprocal(g.W);
    return k;
}
static bool halves(const fps_rotation* rot) { return rot && rot->pairing == FPS_PAIRS_HALVES; }

constexpr int kBwdHeads = 4;

// f(bool constants...) for run-time truth values
template <typename F> static void with(bool a, F&& f) { if (a) f(std::true_type{}); else f(std::false_type{}); }

int launch_norm_rotate(const Geom& g, const fps_view& x, const fps_norm* norm, const fps_rotation* rot, const fps_view& y,
                       hipStream_t st) {
    const Turning k = turning_of(g, norm, rot);
    const int tokens = x.rows;
    const long long blocks = (tokens + 31LL) / 32;
    const bool few = blocks * x.B * x.heads < 4096;
    const int parts = few ? x.heads : (x.heads + 3) / 4;
    const long long grid = blocks * x.B * parts;
    if (grid > 0x7FFFFFFF) { set_error("more rows than a launch has workgroups for"); return FPS_ERR_UNSUPPORTED; }
    with(x.dt == FPS_OUT_F32, [&](auto in32) { with(y.dt == FPS_OUT_F32, [&](auto out32) { with(halves(rot), [&](auto hv) { with(few, [&](auto one) {
        constexpr int HC = decltype(one)::value ? 1 : 4;
        norm_rotate_kernel<decltype(in32)::value, decltype(out32)::value, decltype(hv)::value, HC>
            <<<(int)grid, 256, 0, st>>>(rows_of(x), rows_of(y), k, tokens, x.heads, parts);
    }); }); }); });
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? FPS_OK : hip_fail(e, "norm_rotate launch");
}

template <int BS, bool IN32, bool HALVES>
static void launch_operand(const Geom& g, const Rows& x, const Turning& k, int heads, int role, int prec, uint8_t* xq, float* scales,
                           hipStream_t st) {
    constexpr int TH = BS == 128 ? 256 : 128;
    const int blocks = g.BH * g.M * g.KB, groups = g.BH * g.M * g.NS;
    if (prec != FPS_PREC_FP8) {
        norm_rotate_operand_kernel<BS, TH, IN32, HALVES, false, 1, kWhole><<<blocks, TH, 0, st>>>(x, k, xq, scales, role, g, heads);
        return;
    }
    auto whole = [&](auto nb) {
        constexpr int NB = decltype(nb)::value;
        norm_rotate_operand_kernel<BS, TH, IN32, HALVES, true, NB, kWhole><<<groups, TH * NB, 0, st>>>(x, k, xq, scales, role, g, heads);
    };
    if (g.KBS == 1)      whole(Count<1>{});
    else if (g.KBS == 2) whole(Count<2>{});
    else if (g.KBS == 3) whole(Count<3>{});
    else if constexpr (BS == 128) {                          // blocks of 32 are at most three a group
        clear_kernel<<<(groups + 255) / 256, 256, 0, st>>>((uint32_t*)scales, groups);
        norm_rotate_operand_kernel<BS, TH, IN32, HALVES, true, 1, 0><<<blocks, TH, 0, st>>>(x, k, xq, scales, role, g, heads);
        norm_rotate_operand_kernel<BS, TH, IN32, HALVES, true, 1, 1><<<blocks, TH, 0, st>>>(x, k, xq, scales, role, g, heads);
        amax_to_scale_kernel<<<(groups + 255) / 256, 256, 0, st>>>(scales, groups);
    }
}

int launch_norm_rotate_operand(const Geom& g, const fps_view& x, const fps_norm* norm, const fps_rotation* rot, int role,
                               int prec, void* xq, float* scales, hipStream_t st) {
    const Turning k = turning_of(g, norm, rot);
    with(g.BS == 128, [&](auto big) { with(x.dt == FPS_OUT_F32, [&](auto in32) { with(halves(rot), [&](auto hv) {
        launch_operand<decltype(big)::value ? 128 : 32, decltype(in32)::value, decltype(hv)::value>(g, rows_of(x), k, x.heads, role, prec, (uint8_t*)xq, scales, st);
    }); }); });
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? FPS_OK : hip_fail(e, "norm_rotate_operand launch");
}

// Workgroups of the gradient for each head, or for all where they share a weight
static int bwd_workgroups(const Geom& g, int heads, bool per_head) {
    const int batches = g.BH / heads;
    const long long parts = ((long long)g.T * g.H * g.W + 31) / 32, items = parts * batches * (per_head ? 1 : (heads + kBwdHeads - 1) / kBwdHeads);
    const long long most = per_head ? (1024 + heads - 1) / heads : 1024;
    return (int)(items < most ? items : most);
}
size_t norm_rotate_bwd_bytes(const Geom& g, int heads, bool per_head) {
    return (size_t)bwd_workgroups(g, heads, per_head) * (per_head ? heads : 1) * 128 * sizeof(float);
}
int launch_norm_rotate_bwd(const Geom& g, const fps_view& x, const fps_norm* norm, const fps_rotation* rot, const fps_view& dy,
                           const fps_view& dx, float* dweight, float* partial, hipStream_t st) {
    const Turning k = turning_of(g, norm, rot);
    const bool per_head = norm && norm->per_head && norm->weight;
    const int n = bwd_workgroups(g, x.heads, per_head), sums = per_head ? x.heads : 1;
    if (!dweight) partial = nullptr;
    with(x.dt == FPS_OUT_F32, [&](auto f32) { with(halves(rot), [&](auto hv) { with(per_head, [&](auto one) {
        norm_rotate_bwd_kernel<decltype(f32)::value, decltype(hv)::value, decltype(one)::value ? 1 : kBwdHeads>
            <<<n * sums, 256, 0, st>>>(rows_of(x), rows_of(dy), rows_of(dx), k, partial, x.rows, x.heads, x.B, n);
    }); }); });
    if (dweight) sum_partials_kernel<<<16 * sums, 256, 0, st>>>(partial, dweight, n);
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? FPS_OK : hip_fail(e, "norm_rotate_bwd launch");
}

int launch_dequantize(const Geom& g, const void* xq, const float* scales, int role, bool per_channel, bool f32, void* out,
                      hipStream_t st) {
    const int blocks = g.BH * g.M * g.KB;
    with(g.BS == 128, [&](auto big) { with(f32, [&](auto f) { with(role == FPS_ROLE_V, [&](auto v) {
        dequantize_kernel<decltype(big)::value ? 128 : 32, decltype(f)::value, decltype(v)::value>
            <<<blocks, 256, 0, st>>>((const uint8_t*)xq, scales, role, per_channel, (char*)out, g);
    }); }); });
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? FPS_OK : hip_fail(e, "dequantize launch");
}

}  // namespace fps
