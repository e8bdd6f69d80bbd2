// Each head's RMS norm of Q and K and the rotation by the token's place (t,h,w), in one pass: into the caller's layout, or
// straight into the packed operands of the attention; the gradient of both; and the values of packed E4M3 operands.
//
//   y = R(t,h,w) (x r w),  r = (mean x^2 + eps)^(-1/2),  R: 64 rotations of pairs of channels
//   n = x r,  g = R^T dy,  dw = sum g n,  dx = r (g w - n mean(g w n))
//
// All of it is bound by HBM: some ten operations an element.  Eight lanes hold a row of 128 channels, 16 channels or 8
// pairs each, so that a row is two (four) 16-byte loads of each lane, the sum over it three exchanges between neighbouring
// lanes, and a pair never leaves its lane.  The rotation's tables are as long as the axes: 24 KB at 720p, read from the caches.
#include "fps_device_common.h"

namespace fps {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

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

// The 16 channels of lane u of the eight that hold a row, so that each load and store of theirs is a run of 64 or 128 bytes: slot s is
// channel 64 (s / 8) + 8u + s % 8, or, BY4 (fp32 input), 32 (s / 4) + 4u + s % 4.  Pair i of 8: slots 2i and 2i + 1, or, halves,
// i and i + 8.  (Sixteen channels in a row to a lane, every load half of each line: 720p 350 us instead of 320, the gradient of
// 480p 70 instead of 61.)
typedef float f32x8 __attribute__((ext_vector_type(8)));
struct Pairs { f32x8 a, b; };                                // vectors: arrays end up in LDS where the compiler loses track of an index
template <bool BY4> __device__ __forceinline__ int channel_of(int u, int s) { return BY4 ? 32 * (s >> 2) + 4 * u + (s & 3) : 64 * (s >> 3) + 8 * u + (s & 7); }
template <bool BY4, bool HALVES> __device__ __forceinline__ int pair_of(int u, int i) {
    return HALVES ? channel_of<BY4>(u, i) : channel_of<BY4>(u, 2 * i) >> 1;
}
template <bool HALVES> __device__ __forceinline__ float slot_of(const Pairs& p, int s) {
    return HALVES ? (s < 8 ? p.a[s & 7] : p.b[s & 7]) : (s & 1) ? p.b[s >> 1] : p.a[s >> 1];
}
template <bool HALVES, typename F> __device__ __forceinline__ Pairs pairs_of(F&& slot) {
    Pairs p;
#pragma unroll
    for (int i = 0; i < 8; ++i) { p.a[i] = slot(HALVES ? i : 2 * i); p.b[i] = slot(HALVES ? 8 + i : 2 * i + 1); }
    return p;
}

// an input row's 16 channels, BY4 = F32
template <bool F32> struct Chunks { uint32_t __attribute__((ext_vector_type(F32 ? 16 : 8))) w; };
template <bool F32, bool PAST = false>                       // PAST: what is read does not stay in the caches
__device__ __forceinline__ Chunks<F32> load_row(const char* row, int u) {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    Chunks<F32> c;
#pragma unroll
    for (int i = 0; i < (F32 ? 4 : 2); ++i) {
        const u32x4* at = reinterpret_cast<const u32x4*>(row + 128 * i + 16 * u);
        const u32x4 v = PAST ? __builtin_nontemporal_load(at) : *at;
        c.w[4 * i] = v.x; c.w[4 * i + 1] = v.y; c.w[4 * i + 2] = v.z; c.w[4 * i + 3] = v.w;
    }
    return c;
}
template <bool F32, bool HALVES>
__device__ __forceinline__ Pairs unpack(const Chunks<F32>& c) {
    return pairs_of<HALVES>([&](int s) __attribute__((always_inline)) {
        if (F32) return __uint_as_float(c.w[s & (F32 ? 15 : 7)]);
        return (s & 1) ? high_bf16(c.w[s >> 1]) : low_bf16(c.w[s >> 1]);
    });
}
// PAST: what is stored does not stay in the caches
template <bool PAST>
__device__ __forceinline__ void store_16(char* at, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    if (PAST) __builtin_nontemporal_store(u32x4{x, y, z, w}, reinterpret_cast<u32x4*>(at));
    else      *reinterpret_cast<u32x4*>(at) = u32x4{x, y, z, w};
}
template <bool BY4, bool F32, bool HALVES, bool PAST>
__device__ __forceinline__ void store_row(char* row, int u, const Pairs& p) {
    auto f = [&](int s) __attribute__((always_inline)) { return slot_of<HALVES>(p, s); };
    auto two = [&](int s) __attribute__((always_inline)) { return pack_bf16(f(s), f(s + 1)); };
    if (F32) {
#pragma unroll
        for (int i = 0; i < 16; i += 4)
            store_16<PAST>(row + 4 * channel_of<BY4>(u, i), __float_as_uint(f(i)), __float_as_uint(f(i + 1)), __float_as_uint(f(i + 2)), __float_as_uint(f(i + 3)));
    } else if (BY4) {
#pragma unroll
        for (int i = 0; i < 16; i += 4) *reinterpret_cast<uint2*>(row + 2 * channel_of<BY4>(u, i)) = make_uint2(two(i), two(i + 2));
    } else {
#pragma unroll
        for (int i = 0; i < 16; i += 8) store_16<PAST>(row + 2 * channel_of<BY4>(u, i), two(i), two(i + 2), two(i + 4), two(i + 6));
    }
}

// Cosines and sines of the lane's pairs for token (t,h,w); pairs that do not turn: (1, 0)
struct Turn { f32x8 c, s; };
template <bool BY4, bool HALVES>
__device__ __forceinline__ Turn load_turn(const Turning& k, int b, int n, int u) {
    Turn r;
    if (!k.table) {
#pragma unroll
        for (int i = 0; i < 8; ++i) { r.c[i] = 1.0f; r.s[i] = 0.0f; }
        return r;
    }
    const int t = quotient(n, k.H * k.W, k.rc_plane), rem = n - t * (k.H * k.W), h = quotient(rem, k.W, k.rc_row), w = rem - h * k.W;
    const float2* table = reinterpret_cast<const float2*>(k.table + b * k.table_b);
    const int at_t = t * k.ct, at_h = k.T * k.ct + h * k.ch - k.ct, at_w = k.T * k.ct + k.H * k.ch + w * k.cw - k.ct - k.ch;
#pragma unroll
    for (int i = 0; i < 8; ++i) {                            // without a branch: those that stay read the first entry
        const int p = pair_of<BY4, HALVES>(u, i);
        const bool turns = p < k.ct + k.ch + k.cw;
        const float2 cs = table[turns ? (p < k.ct ? at_t : p < k.ct + k.ch ? at_h : at_w) + p : 0];
        r.c[i] = turns ? cs.x : 1.0f;
        r.s[i] = turns ? cs.y : 0.0f;
    }
    return r;
}
template <bool BY4, bool HALVES>
__device__ __forceinline__ Pairs load_weight(const Turning& k, int h, int u) {
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    f32x8 lo = 1.0f, hi = 1.0f;
    if (k.weight) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x4 v = *reinterpret_cast<const f32x4*>(k.weight + h * k.weight_head + channel_of<BY4>(u, 4 * i));
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (i < 2) lo[4 * i + j] = v[j];
                else       hi[4 * (i & 1) + j] = v[j];
            }
        }
    }
    return pairs_of<HALVES>([&](int s) __attribute__((always_inline)) { return s < 8 ? lo[s & 7] : hi[s & 7]; });
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
// the largest of m and two magnitudes; NaN if one of them is
__device__ __forceinline__ float max_magnitude(float m, float a, float b) {
    float r;
    asm("v_maximum3_f32 %0, %1, |%2|, |%3|" : "=v"(r) : "v"(m), "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ float inverse_rms(const Turning& k, const Pairs& x) {
    if (!k.norm) return 1.0f;
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s = __builtin_fmaf(x.a[i], x.a[i], __builtin_fmaf(x.b[i], x.b[i], s));
    return __builtin_amdgcn_rsqf(__builtin_fmaf(row_sum(s), 1.0f / 128.0f, k.eps));
}
// R w: what a pair of a normed row n = x r is multiplied with, y = (n_a x - n_b y, n_a z + n_b w).  r comes first, so that nothing that
// follows passes fp32's range, and a row whose squares do, r = 0, gives zeros.  Every kernel has these products and this order, so
// that a value has the same bits wherever it is asked for.
__device__ __forceinline__ float4 weighted(float wa, float wb, float cos, float sin) { return make_float4(wa * cos, wb * sin, wa * sin, wb * cos); }
__device__ __forceinline__ Pairs weighted_turned(const Pairs& n, const Pairs& w, const Turn& turn) {
    Pairs y;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float4 f = weighted(w.a[i], w.b[i], turn.c[i], turn.s[i]);
        y.a[i] = __builtin_fmaf(n.a[i], f.x, -(n.b[i] * f.y));
        y.b[i] = __builtin_fmaf(n.a[i], f.z, n.b[i] * f.w);
    }
    return y;
}
__device__ __forceinline__ Pairs times(const Pairs& y, float r) {
    Pairs z;
#pragma unroll
    for (int i = 0; i < 8; ++i) { z.a[i] = y.a[i] * r; z.b[i] = y.b[i] * r; }
    return z;
}

// the scale of a group whose largest magnitude has the bits `top`, NaN of a NaN; 1 where amax / 448 is nothing in fp32
__device__ __forceinline__ float scale_of(uint32_t top) {
    const float s = __uint_as_float(top) / 448.0f;
    return __float_as_uint(s) == 0 ? 1.0f : s;
}
__device__ __forceinline__ Pairs clamped(const Pairs& q) {
    Pairs z;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        z.a[i] = __builtin_amdgcn_fmed3f(q.a[i], -448.0f, 448.0f);
        z.b[i] = __builtin_amdgcn_fmed3f(q.b[i], -448.0f, 448.0f);
    }
    return z;
}
// x / s rounded once: rs is the rounded reciprocal, q a quotient to two half steps, and one step with its exact residual rounds it as a
// division does (P. Markstein, Computation of elementary functions on the IBM RISC System/6000 processor, 1990).  Three instructions an
// element instead of one, 480p 34.0 -> 35.7 us, 720p 215 -> 219, for the code of the quotient itself: y (r / s) had another one at some
// 1e-6 of the elements.
__device__ __forceinline__ Pairs quotients(const Pairs& x, float s, float rs) {
    auto divided = [&](float v) __attribute__((always_inline)) {
        const float q = v * rs;
        return __builtin_fmaf(__builtin_fmaf(-q, s, v), rs, q);
    };
    Pairs z;
#pragma unroll
    for (int i = 0; i < 8; ++i) { z.a[i] = divided(x.a[i]); z.b[i] = divided(x.b[i]); }
    return z;
}

// ---- into the caller's layout -------------------------------------------------------------------
// A wave takes eight tokens, whose cosines and sines are read once for HC heads.
template <bool IN32, bool OUT32, bool HALVES, int HC, bool PAST>
__global__ __launch_bounds__(256) void norm_rotate_kernel(Rows x, Rows y, Turning k, int tokens, int heads, int parts) {
    const int blocks = (int)((tokens + 31u) >> 5), bp = blockIdx.x / blocks;        // tokens fastest
    const int u = threadIdx.x & 7, n = (blockIdx.x - bp * blocks) * 32 + (threadIdx.x >> 3);
    const int b = bp / parts, h0 = (bp - b * parts) * HC;
    if (n >= tokens) return;                                 // whole rows of lanes
    Chunks<IN32> c[HC];
#pragma unroll
    for (int i = 0; i < HC; ++i)
        if (h0 + i < heads) c[i] = load_row<IN32, PAST>(x.at(b, h0 + i, n), u);
    const Turn turn = load_turn<IN32, HALVES>(k, b, n, u);
#pragma unroll
    for (int i = 0; i < HC; ++i) {
        if (h0 + i >= heads) break;
        const Pairs w = load_weight<IN32, HALVES>(k, h0 + i, u), v = unpack<IN32, HALVES>(c[i]);
        store_row<IN32, OUT32, HALVES, PAST>(const_cast<char*>(y.at(b, h0 + i, n)), u, weighted_turned(times(v, inverse_rms(k, v)), w, turn));
    }
}

// ---- into the packed operands -------------------------------------------------------------------
// As quantize_tiles_kernel (and pack_bf16_kernel): a workgroup is one scale group of up to four blocks, held in
// registers from the reading to the encoding; of larger groups a block, of which PASS 0 finds the maximum and PASS 1, which
// reads x again, encodes.
// A token's cosines and sines would be four times as many load instructions as its channels, and all the arithmetic is as long as the
// memory takes: where the entries of the group's planes, rows and columns, those of the columns filled up to 64 pairs, are at most
// kStaged (STAGED) they are brought into LDS first, multiplied by the pair's weights.  (Operands are, bit for bit, those of the raster
// tensor, in fp32 for FP8, in bf16 for BF16.)
constexpr int kWhole = -1, kStaged = 1024;
// Half of a wave's instructions find its tokens and stage the turns.  MANY: they are for kManyHeads heads, one after the other, of
// which the next one's rows are on their way while one is worked on.
constexpr int kManyHeads = 4;
struct Units { int heads, parts, count; uint32_t rc; };      // heads of a workgroup, workgroups for all heads; groups (blocks) of a head
template <int BS, int THREADS, bool IN32, bool HALVES, bool FP8, int NB, int PASS, bool STAGED, bool MANY, bool PAST, bool OWN>
__global__ __launch_bounds__(THREADS * NB) void norm_rotate_operand_kernel(Rows x, Turning k, uint8_t* __restrict__ xq,
                                                                           float* __restrict__ scales, int role, Geom g,
                                                                           int heads, Units units) {
    constexpr int U = BS * 8 / THREADS, WAVES = THREADS * NB / 64;
    __shared__ uint32_t red[2][WAVES];                        // of one head and the next
    __shared__ __attribute__((aligned(16))) float4 staged[STAGED ? kStaged : 1];
    __shared__ __attribute__((aligned(16))) float weights[OWN ? kManyHeads * 128 : 1];      // OWN: of the workgroup's heads, not in the staged turns
    const int kb = NB > 1 ? (int)threadIdx.x / THREADS : 0, tid = threadIdx.x - kb * THREADS, u = tid & 7;
    load_arguments<6>();
    const int bp = quotient(blockIdx.x, units.count, units.rc), b = bp / units.parts, head0 = (bp - b * units.parts) * units.heads;
    const int group0 = (b * heads + head0) * units.count + (blockIdx.x - bp * units.count), last_head = MANY ? min_of(head0 + units.heads, heads) - 1 : head0;
    const BlockOrigin org = block_origin(g, group0 * NB);
    const int n0 = (int)(org.raster0 - (long long)(b * heads + head0) * g.T * g.H * g.W);

    Chunks<IN32> ahead[U];                                   // the rows of the head to come
    Offset token[U];                                         // from the group's first; padding is zeros at the place of the last token
    const char* from[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int slot = org.slot0 + kb * BS + (tid >> 3) + THREADS / 8 * i;
        token[i] = real_token(org.box, slot < org.box.n ? slot : org.box.n > 0 ? org.box.n - 1 : 0);
        from[i] = x.at(b, head0, n0) + ((token[i].t * g.H + token[i].h) * g.W + token[i].w) * x.r;
        ahead[i].w = 0;
        if (slot < org.box.n) ahead[i] = load_row<IN32, PAST>(from[i], u);
    }
    // the group's entries: its planes' and rows' are runs of the table, its columns' each a run and as many (1, 0) as there are pairs left
    const int t0 = quotient(n0, g.H * g.W, k.rc_plane), h0 = quotient(n0 - t0 * (g.H * g.W), g.W, k.rc_row), w0 = n0 - (t0 * g.H + h0) * g.W;
    const int et = org.box.n ? real_token(org.box, org.box.n - 1).t + 1 : 0, rest = 64 - k.ct - k.ch;
    const int of_t = et * k.ct, of_h = org.box.eh * k.ch, of_w = org.box.ew * rest;
    if (STAGED) {                                            // a thread one pair's entries of every fourth (eighth, ..) place
        const int p = threadIdx.x & 63, axis = p < k.ct ? 0 : p < k.ct + k.ch ? 1 : 2;
        const int a = HALVES ? p : 2 * p, c = axis == 0 ? k.ct : axis == 1 ? k.ch : rest, q = axis == 0 ? p : axis == 1 ? p - k.ct : p - k.ct - k.ch;
        const int places = org.box.n == 0 ? 1 : axis == 0 ? et : axis == 1 ? org.box.eh : org.box.ew;
        const int from = axis == 0 ? t0 * k.ct : axis == 1 ? g.T * k.ct + h0 * k.ch : g.T * k.ct + g.H * k.ch + w0 * k.cw;
        const int step = axis == 2 ? k.cw : c, to = axis == 0 ? 0 : axis == 1 ? of_t : of_t + of_h;
        const bool turns = org.box.n > 0 && (axis < 2 || q < k.cw);
        const float2* table = reinterpret_cast<const float2*>(k.table + b * k.table_b);
        const float* w = k.weight + head0 * k.weight_head + a;
        const float wa = k.weight && !OWN ? w[0] : 1.0f, wb = k.weight && !OWN ? w[HALVES ? 64 : 1] : 1.0f;
        constexpr int R = THREADS * NB / 64, L = 4;          // places at a time, loads at a time
        for (int first = threadIdx.x >> 6; first < places; first += L * R) {
            float2 cs[L];
#pragma unroll
            for (int l = 0; l < L; ++l) {
                cs[l] = make_float2(1.0f, 0.0f);
                if (turns) cs[l] = table[from + min_of(first + l * R, places - 1) * step + q];
            }
#pragma unroll
            for (int l = 0; l < L; ++l)
                if (first + l * R < places)
                    staged[to + (first + l * R) * c + q] = weighted(wa, wb, cs[l].x, cs[l].y);
        }
    }
    if (OWN)
        for (int i = threadIdx.x; i < (last_head - head0 + 1) * 128; i += THREADS * NB) weights[i] = k.weight[head0 * 128 + i];
    if (STAGED) __syncthreads();
    auto turned = [&](const Pairs& v, const Offset& d, int head) __attribute__((always_inline)) {
        if (!STAGED) return weighted_turned(v, load_weight<IN32, HALVES>(k, head, u),
                                            load_turn<IN32, HALVES>(k, b, min_of(n0 + (d.t * g.H + d.h) * g.W + d.w, g.T * g.H * g.W - 1), u));
        const int at_t = d.t * k.ct, at_h = of_t + d.h * k.ch - k.ct, at_w = of_t + of_h + d.w * rest - k.ct - k.ch;
        Pairs by;
        if (OWN) by = pairs_of<HALVES>([&](int s) __attribute__((always_inline)) { return weights[(head - head0) * 128 + channel_of<IN32>(u, s)]; });
        Pairs y;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int p = pair_of<IN32, HALVES>(u, i);
            float4 f = staged[(p < k.ct ? at_t : p < k.ct + k.ch ? at_h : at_w) + p];
            if (OWN) f = weighted(by.a[i], by.b[i], f.x, f.y);
            y.a[i] = __builtin_fmaf(v.a[i], f.x, -(v.b[i] * f.y));
            y.b[i] = __builtin_fmaf(v.a[i], f.z, v.b[i] * f.w);
        }
        return y;
    };
    for (int head = head0; head <= last_head; ++head) {
        const int group = group0 + (head - head0) * units.count, blk = group * NB + kb;
        Chunks<IN32> now[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            now[i] = ahead[i];
            if (MANY && head < last_head) {
                from[i] += x.h;
                if (org.slot0 + kb * BS + (tid >> 3) + THREADS / 8 * i < org.box.n) ahead[i] = load_row<IN32, PAST>(from[i], u);
            }
        }
        Pairs y[U];
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            // a wave's rows of padding alone: tile (4,16,16) of 480p 70.7 -> 62.8 us, of 10 x 40 x 40 tokens of 20 heads 65.7 -> 62.4, BF16 of 480p 40.1 -> 38.8
            if (org.slot0 + kb * BS + (__builtin_amdgcn_readfirstlane(tid >> 6) << 3) + THREADS / 8 * i >= org.box.n) {
#pragma unroll
                for (int j = 0; j < 8; ++j) y[i].a[j] = y[i].b[j] = 0.0f;
                continue;
            }
            const Pairs x0 = unpack<IN32, HALVES>(now[i]), v = times(x0, inverse_rms(k, x0));
            y[i] = turned(v, token[i], head);
            if (FP8 && PASS != 1) {
#pragma unroll
                for (int j = 0; j < 8; ++j) m = max_magnitude(m, y[i].a[j], y[i].b[j]);
            }
        }
        uint32_t top = __float_as_uint(m) & 0x7FFFFFFFu;         // magnitudes order like their bits, NaN above all
        char* const dst = (char*)xq + (long long)blk * (BS * 128 * (FP8 ? 1 : 2));
        if constexpr (!FP8) {                                    // 8 channels are a chunk of 16 bytes
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int j = (tid >> 3) + THREADS / 8 * i;
                const Pairs& z = y[i];
                const bool real = org.slot0 + kb * BS + j < org.box.n;               // padding is 0, not -0
                auto two = [&](int s) __attribute__((always_inline)) { return real ? pack_bf16(slot_of<HALVES>(z, s & 15), slot_of<HALVES>(z, (s + 1) & 15)) : 0u; };
                auto chunk = [&](int c8) { return role == FPS_ROLE_K ? ((j >> 5) * 8 + (c8 >> 1)) * 64 + 32 * (c8 & 1) + (j & 31) : j * 16 + c8; };
#pragma unroll
                for (int m = 0; m < 16; m += IN32 ? 4 : 8) {
                    const int c = channel_of<IN32>(u, m);
                    char* at = dst + 16 * chunk(c >> 3) + 2 * (c & 7);
                    if (IN32) *reinterpret_cast<uint2*>(at) = make_uint2(two(m), two(m + 2));
                    else      *reinterpret_cast<uint4*>(at) = make_uint4(two(m), two(m + 2), two(m + 4), two(m + 6));
                }
            }
            continue;
        }
        if (PASS == 1) {
            top = __float_as_uint(scales[quotient(group, g.KBS, g.rc_kbs)]);
        } else {
            top = workgroup_max<WAVES>(top, red[(head - head0) & 1]);
            if (PASS == 0) {
                if (threadIdx.x == 0) atomicMax((uint32_t*)&scales[quotient(group, g.KBS, g.rc_kbs)], top);
                continue;
            }
        }
        const float s = scale_of(top);
        if (PASS == kWhole && threadIdx.x == 0) scales[group] = s;
        float by = s, rs = 1.0f / s;
        // A scale near the end of the range: its reciprocal would pass it, and one that has lost bits there leaves quotients beyond 448.  Such a
        // group's codes are written again: what stands before the others' conversions, or parts them from the quotients, costs 720p 3 to 15 us.
        const bool tiny = (uint32_t)__builtin_amdgcn_readfirstlane((int)top) < __builtin_bit_cast(uint32_t, 0x1p-52f);
        for (int again = 0;; again = 1) {
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int j = (tid >> 3) + THREADS / 8 * i;
                const Pairs z = quotients(y[i], by, rs);
                // the 16-byte chunk of channels 16 c16 ..
                auto chunk = [&](int c16) {
                    return role == FPS_ROLE_K ? (((j >> 5) * 2 + (c16 >> 2)) * 2 + (c16 & 1)) * 64 + 32 * ((c16 >> 1) & 1) + (j & 31) : j * 8 + c16;
                };
                uint32_t o[4];
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    const int w = __builtin_amdgcn_cvt_pk_fp8_f32(slot_of<HALVES>(z, 4 * m), slot_of<HALVES>(z, 4 * m + 1), 0, false);
                    o[m] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(slot_of<HALVES>(z, 4 * m + 2), slot_of<HALVES>(z, 4 * m + 3), w, true);
                    o[m] = org.slot0 + kb * BS + j < org.box.n ? o[m] : 0u;              // padding is 0, not -0
                }
#pragma unroll
                for (int m = 0; m < 4; m += IN32 ? 1 : 2) {
                    const int c = channel_of<IN32>(u, 4 * m);
                    char* at = dst + 16 * chunk(c >> 4) + (c & 15);
                    if (IN32) *reinterpret_cast<uint32_t*>(at) = o[m];
                    else if (PAST) __builtin_nontemporal_store(u32x2{o[m], o[(m + 1) & 3]}, reinterpret_cast<u32x2*>(at));
                    else           *reinterpret_cast<u32x2*>(at) = u32x2{o[m], o[(m + 1) & 3]};
                }
            }
            if (!tiny || again) break;
            by = s * 0x1p64f;
            rs = 1.0f / by;
#pragma unroll
            for (int i = 0; i < U; ++i) y[i] = clamped(quotients(times(y[i], 0x1p64f), by, rs));
            by = rs = 1.0f;                                  // divided already
        }
    }
}

// the maxima that PASS 0 found to scales
__global__ void scales_kernel(float* p, int n) {
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i < n) p[i] = scale_of(__float_as_uint(p[i]));
}

// ---- the gradient -------------------------------------------------------------------------------
// A workgroup takes 32 tokens of HC heads at a time, requests the rows of all of them at once and reads their cosines and sines once.  Its
// lanes' share of dweight stays in registers, that of each head (OWN: the workgroup's heads are then always the same) or one
// for all; the workgroups' sums are added up by a second kernel, in a fixed order.  (Requesting the next rows before these are worked
// on takes all registers and gains nothing: 720p 455 us, 450 without.)
template <bool F32, bool HALVES, int HC, bool OWN, bool PAST>
__global__ __launch_bounds__(256) void norm_rotate_bwd_kernel(Rows x, Rows dy, Rows dx, Turning k, float* __restrict__ partial,
                                                              int tokens, int heads, int batches, int workgroups) {
    constexpr int SUMS = OWN ? HC : 1;
    __shared__ float red[4][SUMS][128];
    const int u = threadIdx.x & 7, row = threadIdx.x >> 3, parts = (int)((tokens + 31u) >> 5);
    const int group = blockIdx.x / workgroups, first = blockIdx.x - group * workgroups;
    const int per = OWN ? 1 : (heads + HC - 1) / HC;
    const long long items = (long long)batches * parts * per;               // (batch, token part, heads)
    Pairs dw[SUMS];
#pragma unroll
    for (int j = 0; j < SUMS; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[j].a[i] = dw[j].b[i] = 0.0f;
    for (long long item = first; item < items; item += workgroups) {
        const long long bp = item / per;
        const int h0 = (OWN ? group : (int)(item - bp * per)) * HC, b = (int)(bp / parts), n = (int)(bp - (long long)b * parts) * 32 + row;
        if (n >= tokens) continue;
        Chunks<F32> cx[HC], cy[HC];
#pragma unroll
        for (int i = 0; i < HC; ++i)
            if (h0 + i < heads) {
                cx[i] = load_row<F32, PAST>(x.at(b, h0 + i, n), u);
                cy[i] = load_row<F32, PAST>(dy.at(b, h0 + i, n), u);
            }
        const Turn turn = load_turn<F32, HALVES>(k, b, n, u);
        Pairs w = load_weight<F32, HALVES>(k, h0, u);
#pragma unroll
        for (int i = 0; i < HC; ++i) {
            if (h0 + i >= heads) break;
            if (OWN && i > 0) w = load_weight<F32, HALVES>(k, h0 + i, u);
            const Pairs xv = unpack<F32, HALVES>(cx[i]), g0 = unpack<F32, HALVES>(cy[i]);
            Pairs& sum = dw[OWN ? i : 0];
            const float r = inverse_rms(k, xv);
            Pairs nv = times(xv, r);                         // at most the row's length: no product below passes fp32's range by x
            if (!k.norm) nv.a = nv.b = 0.0f;                 // R^T dy alone, whatever x holds
            Pairs g;
            float dot = 0.0f;
#pragma unroll
            for (int m = 0; m < 8; ++m) {
                const float ga = __builtin_fmaf(g0.a[m], turn.c[m], g0.b[m] * turn.s[m]);
                const float gb = __builtin_fmaf(g0.b[m], turn.c[m], -(g0.a[m] * turn.s[m]));
                sum.a[m] = __builtin_fmaf(ga, nv.a[m], sum.a[m]);
                sum.b[m] = __builtin_fmaf(gb, nv.b[m], sum.b[m]);
                g.a[m] = ga * w.a[m];
                g.b[m] = gb * w.b[m];
                dot = __builtin_fmaf(g.a[m], nv.a[m], __builtin_fmaf(g.b[m], nv.b[m], dot));
            }
            const float back = k.norm ? row_sum(dot) * (1.0f / 128.0f) : 0.0f;
            Pairs d;
#pragma unroll
            for (int m = 0; m < 8; ++m) {
                d.a[m] = r * __builtin_fmaf(-nv.a[m], back, g.a[m]);
                d.b[m] = r * __builtin_fmaf(-nv.b[m], back, g.b[m]);
            }
            store_row<F32, F32, HALVES, PAST>(const_cast<char*>(dx.at(b, h0 + i, n)), u, d);
        }
    }
    if (!partial) return;
#pragma unroll
    for (int j = 0; j < SUMS; ++j) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int off = 8; off < 64; off <<= 1) {
                dw[j].a[i] += __shfl_xor(dw[j].a[i], off);
                dw[j].b[i] += __shfl_xor(dw[j].b[i], off);
            }
        if ((threadIdx.x & 63) < 8) {
#pragma unroll
            for (int i = 0; i < 16; ++i) red[threadIdx.x >> 6][j][channel_of<F32>(u, i)] = slot_of<HALVES>(dw[j], i);
        }
    }
    __syncthreads();
    if (threadIdx.x < 128)
#pragma unroll
        for (int j = 0; j < SUMS; ++j) {                     // of a head its workgroups' sums follow each other
            const int c = threadIdx.x, head = group * HC + j;
            if (OWN && head >= heads) break;
            partial[((long long)(OWN ? head : 0) * workgroups + first) * 128 + c] = (red[0][j][c] + red[1][j][c]) + (red[2][j][c] + red[3][j][c]);
        }
}
// Eight channels a workgroup, 128 slices of the n partial sums: what bounds it is the loads that follow each other
__global__ __launch_bounds__(1024) void sum_partials_kernel(const float* __restrict__ partial, float* __restrict__ out, int n) {
    __shared__ float red[16][8];
    const int c = threadIdx.x & 7, slice = threadIdx.x >> 3, group = blockIdx.x >> 4, c0 = 8 * (blockIdx.x & 15);
    const float* p = partial + (long long)group * n * 128 + c0 + c;
    float s = 0.0f;
#pragma unroll 8
    for (int i = slice; i < n; i += 128) s += p[(long long)i * 128];
#pragma unroll
    for (int off = 8; off < 64; off <<= 1) s += __shfl_xor(s, off);
    if ((threadIdx.x & 63) < 8) red[threadIdx.x >> 6][c] = s;
    __syncthreads();
    if (threadIdx.x < 8) {
        float t = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) t += red[i][threadIdx.x];
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
// Input and output together beyond the Infinity Cache's 256 MB: the output does not push out what is there.  And what is read once
// goes past it too.  720p 303 -> 291 -> 278 us, its gradient 468 -> 458 by the latter; 480p, which the cache holds for what reads it next, 31.6 us, 37.4 past it.
constexpr long long kCaches = 256LL << 20;
static bool beyond_caches(const fps_view& x, const fps_view& y) {
    const long long n = (long long)x.B * x.heads * x.rows * kHeadDim;
    return n * ((x.dt == FPS_OUT_F32 ? 4 : 2) + (y.dt == FPS_OUT_F32 ? 4 : 2)) > kCaches;
}
static bool halves(const fps_rotation* rot) { return rot && rot->pairing == FPS_PAIRS_HALVES; }

// Heads a workgroup takes together.  us: forward, 720p of 40 heads, 480p of 12, 720p of 3: 2 292, 32.3, 20.3; 4 281, 31.4, 20.3; 8 286, 31.8,
// 22.3; 16 294, 34.6, 24.7.  The gradient with one weight for all, with its second kernel: 2 519, 68, 40; 4 468, 58, 36; 8 476, 67, 36; with
// weights of each head: 1 508, 70, 40; 2 469, 79, 51; 4 574, 119, 80.  Its workgroups, which stay: 512 468, 58.2, 36.7; 1024 468, 60.5, 35.4;
// 2048 467, 65, 38; with weights of each head 2048 552, 72, 37; 4096 508, 70, 40; 8192 489, 74, 46.  Weights of each head: one
// head a workgroup at every size, where two gain 8 % at 720p and lose 13 and 28 % at the others.
constexpr int kHeads = 4, kBwdHeads = 4, kBwdWorkgroups = 512, kOwnHeads = 1, kOwnWorkgroups = 4096;

// f(bool constants...) for run-time truth values
template <typename F> static void with(bool a, F&& f) { if (a) f(std::true_type{}); else f(std::false_type{}); }

int launch_norm_rotate(const Geom& g, const fps_view& x, const fps_norm* norm, const fps_rotation* rot, const fps_view& y,
                       hipStream_t st) {
    const Turning k = turning_of(g, norm, rot);
    const int tokens = x.rows;
    const long long blocks = (tokens + 31LL) / 32;
    // one head a workgroup, four: 128 tokens of 40 heads (160 parts of 32 rows) 3.2, 4.2 us; 1170 tokens of 40 heads (1480) 6.9, 6.5; 4255 of 12
    // (1596) 7.6, 6.8; 7800 of 12 (2928) 11.4, 9.9
    const bool few = blocks * x.B * x.heads < 1024;
    const int parts = few ? x.heads : (x.heads + kHeads - 1) / kHeads;
    const long long grid = blocks * x.B * parts;
    FPS_TRY(check_launch(grid, 256, "norm_rotate"));
    const bool past = beyond_caches(x, y);
    with(x.dt == FPS_OUT_F32, [&](auto in32) { with(y.dt == FPS_OUT_F32, [&](auto out32) { with(halves(rot), [&](auto hv) { with(past, [&](auto pa) {
        auto launch = [&](auto hc) {
            constexpr int HC = decltype(hc)::value;
            norm_rotate_kernel<decltype(in32)::value, decltype(out32)::value, decltype(hv)::value, HC, HC != 1 && decltype(pa)::value>
                <<<(int)grid, 256, 0, st>>>(rows_of(x), rows_of(y), k, tokens, x.heads, parts);
        };
        if (few) launch(Count<1>{});
        else     launch(Count<kHeads>{});
    }); }); }); });
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? FPS_OK : hip_fail(e, "norm_rotate launch");
}

template <int BS, bool IN32, bool HALVES, bool STAGED, bool MANY, bool PAST, bool OWN>
static int launch_operand(const Geom& g, const Rows& x, const Turning& k, int heads, int role, int prec, uint8_t* xq, float* scales,
                          hipStream_t st) {
    // two rows of a block a lane: with four 480p 37.7 us instead of 34.7, 720p 228 instead of 222, weights of each head 241 instead of 226; three
    // blocks of 128 would be more threads than a workgroup may have
    constexpr int TH = BS == 128 ? 512 : 128;
    struct Launch { Units units; int grid; };
    auto of_head = [&](int count, bool many) {
        const int each = many ? kManyHeads : 1, parts = (heads + each - 1) / each;
        return Launch{Units{each, parts, count, reciprocal(count)}, g.BH / heads * parts * count};
    };
    auto check = [](const Launch& l, int threads) { return check_launch(l.grid, threads, "norm_rotate_operand"); };
    const Launch blocks = of_head(g.M * g.KB, MANY);
    const int groups = g.BH * g.M * g.NS;
    if (prec != FPS_PREC_FP8) {
        FPS_TRY(check(blocks, TH));
        norm_rotate_operand_kernel<BS, TH, IN32, HALVES, false, 1, kWhole, STAGED, MANY, PAST, OWN><<<blocks.grid, TH, 0, st>>>(x, k, xq, scales, role, g, heads, blocks.units);
        return FPS_OK;
    }
    auto whole = [&](auto nb) {
        constexpr int NB = decltype(nb)::value, T = TH * NB > 1024 ? TH / 2 : TH;
        constexpr bool many = MANY && T == TH;               // twice the rows a lane: no registers for the next head's
        const Launch l = of_head(g.M * g.NS, many);
        FPS_TRY(check(l, T * NB));
        norm_rotate_operand_kernel<BS, T, IN32, HALVES, true, NB, kWhole, STAGED, many, many && PAST, many && OWN><<<l.grid, T * NB, 0, st>>>(x, k, xq, scales, role, g, heads, l.units);
        return (int)FPS_OK;
    };
    if (g.KBS == 1) return whole(Count<1>{});
    if (g.KBS == 2) return whole(Count<2>{});
    if (g.KBS == 3) return whole(Count<3>{});
    if constexpr (BS == 128) {                               // blocks of 32 are at most three a group
        if (g.KBS == 4) return whole(Count<4>{});            // 512 tokens, 1024 threads: one pass instead of two and three launches less
        FPS_TRY(check(blocks, TH));
        clear_kernel<<<(groups + 255) / 256, 256, 0, st>>>((uint32_t*)scales, groups);     // x is read twice: by way of the caches
        norm_rotate_operand_kernel<BS, TH, IN32, HALVES, true, 1, 0, STAGED, MANY, false, OWN><<<blocks.grid, TH, 0, st>>>(x, k, xq, scales, role, g, heads, blocks.units);
        norm_rotate_operand_kernel<BS, TH, IN32, HALVES, true, 1, 1, STAGED, MANY, false, OWN><<<blocks.grid, TH, 0, st>>>(x, k, xq, scales, role, g, heads, blocks.units);
        scales_kernel<<<(groups + 255) / 256, 256, 0, st>>>(scales, groups);
    }
    return FPS_OK;
}

int launch_norm_rotate_operand(const Geom& g, const fps_view& x, const fps_norm* norm, const fps_rotation* rot, int role,
                               int prec, void* xq, float* scales, hipStream_t st) {
    const Turning k = turning_of(g, norm, rot);
    const bool staged = (long long)g.Qt * k.ct + (long long)g.Qh * k.ch + (long long)g.Qw * (64 - k.ct - k.ch) <= kStaged;
    // past the caches: 720p of 40 heads 231 -> 222 us (BF16 307 -> 300); 480p of 12, which they hold, 34.6, 37.7
    const bool past = (long long)x.B * x.heads * x.rows * kHeadDim * (prec == FPS_PREC_FP8 ? 3 : 4) > kCaches;
    // Several heads a workgroup where there are 1024 blocks of 128 slots or more (bf16; fp32 rows leave no registers).  us with one head,
    // with four: 480p of 12 heads 34.5, 34.7 (BF16 40.6, 38.8), in tiles (4,16,16) 67, 63, 720p of 40 heads 247, 222 (306, 300), of 3 heads 21.9,
    // 21.9; 4255 tokens of 12 heads, 540 blocks of 128, 9.6, 12.3.  With weights of each head, which the staged turns then do not hold, beyond the
    // caches: 720p 248, 226 (306, 300); 480p 34.8, 38.7
    const bool own = k.weight_head != 0, many = staged && x.heads > 1 && (!own || past) && (long long)g.BH * g.M * g.KB * g.BS >= 128 * 1024;
    int rc = FPS_OK;
    auto launch = [&](auto big, auto in32, auto hv, auto sg, auto mn, auto pa, auto ow) {
        rc = launch_operand<decltype(big)::value ? 128 : 32, decltype(in32)::value, decltype(hv)::value, decltype(sg)::value, decltype(mn)::value, decltype(pa)::value, decltype(ow)::value>(
            g, rows_of(x), k, x.heads, role, prec, (uint8_t*)xq, scales, st);
    };
    with(g.BS == 128, [&](auto big) { with(halves(rot), [&](auto hv) {
        const std::true_type yes;
        const std::false_type no;
        if (x.dt == FPS_OUT_F32) with(staged, [&](auto sg) { launch(big, yes, hv, sg, no, no, no); });
        else if (many && own)    launch(big, no, hv, yes, yes, yes, yes);
        else if (many)           with(past, [&](auto pa) { launch(big, no, hv, yes, yes, pa, no); });
        else                     with(staged, [&](auto sg) { launch(big, no, hv, sg, no, no, no); });
    }); });
    if (rc != FPS_OK) return rc;
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? FPS_OK : hip_fail(e, "norm_rotate_operand launch");
}

// Workgroups of the gradient for each group of heads that have weights of their own, or for all where they share one
static int bwd_workgroups(const Geom& g, int heads, bool per_head) {
    const long long parts = ((long long)g.T * g.H * g.W + 31) / 32 * (g.BH / heads);
    const int at_once = per_head ? kOwnHeads : kBwdHeads, groups = (heads + at_once - 1) / at_once;
    const long long items = per_head ? parts : parts * groups, most = per_head ? (kOwnWorkgroups + groups - 1) / groups : kBwdWorkgroups;
    return (int)(items < most ? items : most);
}
size_t norm_rotate_bwd_bytes(const Geom& g, int heads, bool per_head) {
    return (size_t)bwd_workgroups(g, heads, per_head) * (per_head ? heads : 1) * 128 * sizeof(float);
}
int launch_norm_rotate_bwd(const Geom& g, const fps_view& x, const fps_norm* norm, const fps_rotation* rot, const fps_view& dy,
                           const fps_view& dx, float* dweight, float* partial, hipStream_t st) {
    const Turning k = turning_of(g, norm, rot);
    const bool per_head = norm && norm->per_head && norm->weight;
    const int n = bwd_workgroups(g, x.heads, per_head), grid = n * (per_head ? (x.heads + kOwnHeads - 1) / kOwnHeads : 1);
    if (!dweight) partial = nullptr;
    else if (per_head) FPS_TRY(check_launch(16LL * x.heads, 1024, "norm_rotate_bwd"));
    with(x.dt == FPS_OUT_F32, [&](auto f32) { with(halves(rot), [&](auto hv) { with(per_head, [&](auto own) { with(beyond_caches(x, dx), [&](auto pa) {
        norm_rotate_bwd_kernel<decltype(f32)::value, decltype(hv)::value, decltype(own)::value ? kOwnHeads : kBwdHeads, decltype(own)::value, decltype(pa)::value>
            <<<grid, 256, 0, st>>>(rows_of(x), rows_of(dy), rows_of(dx), k, partial, x.rows, x.heads, x.B, n);
    }); }); }); });
    if (dweight) sum_partials_kernel<<<16 * (per_head ? x.heads : 1), 1024, 0, st>>>(partial, dweight, n);
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? FPS_OK : hip_fail(e, "norm_rotate_bwd launch");
}

int launch_dequantize(const Geom& g, const void* xq, const float* scales, int role, bool per_channel, bool f32, void* out,
                      hipStream_t st) {
    const int blocks = g.BH * g.M * g.KB;
    FPS_TRY(check_launch(blocks, 256, "dequantize"));
    with(g.BS == 128, [&](auto big) { with(f32, [&](auto f) { with(role == FPS_ROLE_V, [&](auto v) {
        dequantize_kernel<decltype(big)::value ? 128 : 32, decltype(f)::value, decltype(v)::value>
            <<<blocks, 256, 0, st>>>((const uint8_t*)xq, scales, role, per_channel, (char*)out, g);
    }); }); });
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? FPS_OK : hip_fail(e, "dequantize launch");
}

}  // namespace fps
