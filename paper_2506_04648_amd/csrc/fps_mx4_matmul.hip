// Products of large microscaled 4-bit matrices.
//
// A workgroup of four waves, one on each SIMD of a CU, takes 256 x 256 elements of the result, a wave 128 x 128 of them in 256
// accumulation registers; it stays on its CU and goes from tile to tile.  Half a step of both operands, 128 columns in 32 KB,
// is a slot of a ring of four in the LDS; a slot is filled again as soon as it is read, three of them before it is needed, across the
// end of a tile as well.
#include "fps_mx4.h"

namespace fps {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kTileEdge = 256, kEdgeTiles = kTileEdge / kMxRows;
constexpr int kHalf = kMxStepBytes / 2, kSlot = 2 * kEdgeTiles * kHalf, kSlots = 4;              // bytes; of 16 row tiles half a step
constexpr int kScales = kSlots * kSlot, kScaleSlot = 2 * kEdgeTiles * kMxScaleBytes;               // behind them, two steps' scales
constexpr int kPieces = kScales + 2 * kScaleSlot;
constexpr int kPiecePitch = 64 * 2 + 16, kPiece = 32 * kPiecePitch;       // 32 rows of 64 columns in bf16, on their way out

struct TileMap { int tiles_m, tiles_n, total, workgroups; };

// From device memory to LDS, lane i's 16 bytes to dst + 16 i: 1 KB from a wave-uniform src (FAR bytes further on), or from the lanes'
// own addresses.  Inline assembly, so that the compiler does not wait for the copies before it reads other parts of the LDS.
// The instruction's offset counts on both sides, so dst is given FAR less.
template <int FAR>
__device__ __forceinline__ void copy_1k(const void* src, uint32_t lane_off, uint32_t dst, int dst_more) {
    asm volatile("s_add_i32 m0, %2, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 offset:%4"
                 : : "v"(lane_off), "s"(src), "s"(dst), "n"(dst_more - FAR), "n"(FAR) : "memory", "m0", "scc");
}
__device__ __forceinline__ void copy_lanes(const void* src, uint32_t dst) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(src), "s"(dst) : "memory", "m0");
}
// Waits until at most N of the wave's copies (and stores) are under way and all it has read from LDS is there; then for the other waves
template <int N>
__device__ __forceinline__ void meet() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(N) : "memory");
}

__device__ __forceinline__ v8i operand(const uint4& c) { return v8i{(int)c.x, (int)c.y, (int)c.z, (int)c.w, 0, 0, 0, 0}; }

// Where tile i of the result lies.  An XCD's workgroups, every eighth, take a contiguous part of the order, in which eight tiles down
// come before the next column: what its 32 CUs multiply at one time is 8 x 4 tiles, 12 panels of operands for its L2.
struct Place { int m, n; };
__device__ __forceinline__ Place place_of(const TileMap& t, int i) {
    const int band = 8 * t.tiles_n, g = i / band, rem = i - g * band;
    const int down = min_of(8, t.tiles_m - 8 * g), col = rem / down;
    return Place{8 * g + rem - col * down, col};
}

template <bool F32>
__global__ __launch_bounds__(256, 1) void mx4_large_kernel(Packed a, Packed b, const float* __restrict__ bias, Matrix y, TileMap map) {
    __shared__ __attribute__((aligned(1024))) uint8_t lds[kPieces + 4 * kPiece];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1, h = lane >> 5;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
    const int steps = a.steps;

    // this workgroup's tiles: first, first + stride, .. < end
    const int xcd = blockIdx.x & 7, per_xcd = (map.total + 7) >> 3, stride = map.workgroups >> 3;
    const int end = min_of(map.total, (xcd + 1) * per_xcd);
    int tile = xcd * per_xcd + (blockIdx.x >> 3);
    if (tile >= end) return;

    // copying: where the step that is copied next lies; wave w copies operand w / 2's row tiles 4 (w % 2) ..
    const Packed& mine = wave < 2 ? a : b;
    int copy_tile = tile, copy_step = 0;
    const char* codes_at[4];                                 // of the four row tiles
    const char* scales_at;                                   // of the lane's share of their scales
    auto locate = [&]() __attribute__((always_inline)) {
        const Place p = place_of(map, copy_tile);
        const int first = (wave < 2 ? p.m : p.n) * kEdgeTiles + 4 * (wave & 1);
#pragma unroll
        for (int i = 0; i < 4; ++i)                          // beyond the last row tile: the last one again
            codes_at[i] = (const char*)mine.codes + (long long)min_of(first + i, mine.tiles - 1) * steps * kMxStepBytes;
        scales_at = (const char*)mine.scales + (long long)min_of(first + (lane >> 4), mine.tiles - 1) * steps * kMxScaleBytes + 16 * (lane & 15);
    };
    locate();
    const uint32_t lane_off = 16 * lane, code_slots = lds0 + 4 * wave * kHalf, scale_slots = lds0 + kScales + 4 * wave * kMxScaleBytes;
    // one of the eight copies of half a step: kilobyte n % 2 of row tile n / 2; par: parity of the step
    auto copy_codes = [&](int par, auto half_tag, auto n_tag) __attribute__((always_inline)) {
        constexpr int half = decltype(half_tag)::value, n = decltype(n_tag)::value, far = half * kHalf + (n & 1) * 1024;
        copy_1k<far>(codes_at[n >> 1], lane_off, code_slots + par * (2 * kSlot), half * kSlot + (n >> 1) * kHalf + (n & 1) * 1024);
    };
    auto copy_scales = [&](int par) __attribute__((always_inline)) { copy_lanes(scales_at, scale_slots + par * kScaleSlot); };
    // to the next step; behind the last tile of the result the last one's again, or what follows it, which nobody reads
    auto advance = [&]() __attribute__((always_inline)) {
        const bool more = ++copy_step < steps;
        const int by = more ? 1 : 1 - steps;                 // without a further tile: from the start
        if (!more) {
            copy_step = 0;
            copy_tile += stride;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) codes_at[i] += (long long)by * kMxStepBytes;
        scales_at += (long long)by * kMxScaleBytes;
        if (!more && copy_tile < end) locate();
    };

    uint4 ca[2][4], cb[2][4];
    uint32_t sa[4], sb[4], sa_next[4], sb_next[4];
    const uint8_t* const read_a = lds + 4 * wm * kHalf + 16 * lane;
    const uint8_t* const read_b = lds + (kEdgeTiles + 4 * wn) * kHalf + 16 * lane;
    const uint8_t* const read_sa = lds + kScales + 4 * wm * kMxScaleBytes + 4 * lane;
    const uint8_t* const read_sb = lds + kScales + (kEdgeTiles + 4 * wn) * kMxScaleBytes + 4 * lane;
    // one of the eight operands of quarter q (0 or 1) of a slot, in the order of their use
    auto read = [&](int set, int slot, int q, int n) __attribute__((always_inline)) {
        const int at_slot = slot * kSlot + q * 1024;
        if (n == 1 || n > 4) ca[set][n > 4 ? n - 4 : 0] = *reinterpret_cast<const uint4*>(read_a + at_slot + (n > 4 ? n - 4 : 0) * kHalf);
        else                 cb[set][n ? n - 1 : 0] = *reinterpret_cast<const uint4*>(read_b + at_slot + (n ? n - 1 : 0) * kHalf);
    };
    auto read_scales = [&](int slot, int i) __attribute__((always_inline)) {
        sa_next[i] = *reinterpret_cast<const uint32_t*>(read_sa + slot * kScaleSlot + i * kMxScaleBytes);
        sb_next[i] = *reinterpret_cast<const uint32_t*>(read_sb + slot * kScaleSlot + i * kMxScaleBytes);
    };
    v16f acc[4][4];
    auto multiply = [&](auto q_tag, int n, bool first) __attribute__((always_inline)) {     // rows 32 (n / 4) .., columns 32 (n % 4) ..
        constexpr int q = decltype(q_tag)::value, set = q & 1;
        const v16f zero = {};
        const int i = n >> 2, j = n & 3;
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(cb[set][j]), operand(ca[set][i]), first ? zero : acc[i][j], 4, 4, q,
                                                                    (int)sb[j], q, (int)sa[i]);
    };

    // steps 0 and 1 of the sequence: nine copies a wave for the first half of a step, eight for the second
    auto copy_half = [&](int par, auto half_tag) __attribute__((always_inline)) {
        copy_codes(par, half_tag, Count<0>{}); copy_codes(par, half_tag, Count<1>{}); copy_codes(par, half_tag, Count<2>{});
        copy_codes(par, half_tag, Count<3>{}); copy_codes(par, half_tag, Count<4>{}); copy_codes(par, half_tag, Count<5>{});
        copy_codes(par, half_tag, Count<6>{}); copy_codes(par, half_tag, Count<7>{});
    };
    copy_scales(0);
    copy_half(0, Count<0>{});
    copy_half(0, Count<1>{});
    advance();
    copy_scales(1);
    copy_half(1, Count<0>{});
    copy_half(1, Count<1>{});
    meet<25>();
    int parity = 0;                                          // of the step: its slots are 2 parity and 2 parity + 1
#pragma unroll
    for (int n = 0; n < 8; ++n) read(0, 0, 0, n);
#pragma unroll
    for (int i = 0; i < 4; ++i) read_scales(0, i);
    uint8_t* const piece = lds + kPieces + wave * kPiece;
    const int M = y.all_rows(), N = y.all_cols();
    for (; tile < end; tile += stride) {
        // The order is as written.  A multiplication takes the matrix unit 32 cycles or more and the wave is alone on its SIMD: what else
        // there is to issue, the operands of the next 64 columns and the copies, stands between the multiplications, one at a time.
        auto step = [&](bool first) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) { sa[i] = sa_next[i]; sb[i] = sb_next[i]; }
            advance();                                       // before all else: behind a branch the multiplications would wait for it
            __builtin_amdgcn_sched_barrier(0);
            auto half = [&](auto h_tag) __attribute__((always_inline)) {
                constexpr int hf = decltype(h_tag)::value;
                const int slot = 2 * parity + hf, next = hf ? 2 * (parity ^ 1) : slot + 1;
#pragma unroll
                for (int n = 0; n < 16; ++n) {
                    multiply(Count<2 * hf>{}, n, first && hf == 0);
                    if (n < 8) read(1, slot, 1, n);
                    __builtin_amdgcn_sched_barrier(0);
                }
                meet<17>();                                  // the next slot has landed, of two more the copies go on; this one is read
                auto copying = [&](auto n_tag) __attribute__((always_inline)) {
                    constexpr int n = decltype(n_tag)::value;
                    multiply(Count<2 * hf + 1>{}, n, false);
                    if (n < 8) read(0, next, 0, n);
                    else copy_codes(parity, h_tag, Count<(n & 7)>{});          // of the step after the next, into this slot
                    if (n == 7 && !hf) copy_scales(parity);
                    if (n >= 4 && n < 8 && hf) read_scales(parity ^ 1, n & 3);
                    __builtin_amdgcn_sched_barrier(0);
                };
                copying(Count<0>{}); copying(Count<1>{}); copying(Count<2>{}); copying(Count<3>{});
                copying(Count<4>{}); copying(Count<5>{}); copying(Count<6>{}); copying(Count<7>{});
                copying(Count<8>{}); copying(Count<9>{}); copying(Count<10>{}); copying(Count<11>{});
                copying(Count<12>{}); copying(Count<13>{}); copying(Count<14>{}); copying(Count<15>{});
            };
            half(Count<0>{});
            half(Count<1>{});
            parity ^= 1;
        };
        step(true);
        for (int s = 1; s < steps; ++s) step(false);
        // out: pieces of 32 rows and 64 columns by way of the wave's own part of the LDS, rows of 128 bytes
        const Place p = place_of(map, tile);
        const int row0 = p.m * kTileEdge + wm * 128, col0 = p.n * kTileEdge + wn * 128;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int jj = 0; jj < 4; jj += F32 ? 1 : 2) {
#pragma unroll
                for (int j = jj; j < jj + (F32 ? 1 : 2); ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        float v[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) v[k] = acc[i][j][4 * q + k];
                        if (bias) {
                            const int c = col0 + 32 * j + 8 * q + 4 * h;
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                if (c + k < N) v[k] += bias[c + k];
                        }
                        uint8_t* const at_piece = piece + (lane & 31) * kPiecePitch + ((j - jj) * 32 + 8 * q + 4 * h) * (F32 ? 4 : 2);
                        if (F32) *reinterpret_cast<float4*>(at_piece) = make_float4(v[0], v[1], v[2], v[3]);
                        else *reinterpret_cast<uint2*>(at_piece) =
                                 make_uint2(__builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{v[0], v[1]}, bf16x2)),
                                            __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{v[2], v[3]}, bf16x2)));
                    }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const int m = 8 * t + (lane >> 3), c = lane & 7;
                    const uint4 v = *reinterpret_cast<const uint4*>(piece + m * kPiecePitch + 16 * c);
                    constexpr int E = F32 ? 4 : 2, W = 16 / E;       // bytes an element, elements a lane
                    const int row = row0 + 32 * i + m, col = col0 + 32 * jj + W * c;
                    if (row >= M || col >= N) continue;
                    char* dst = y.row(row) + y.column<E>(col);
                    if (col + W <= N) {
                        __builtin_memcpy(dst, &v, 16);
                    } else {
                        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                        for (int k = 0; k < W - 1; ++k)
                            if (col + k < N) {
                                if (F32) reinterpret_cast<uint32_t*>(dst)[k] = w[k];
                                else     reinterpret_cast<uint16_t*>(dst)[k] = (uint16_t)(w[k >> 1] >> (16 * (k & 1)));
                            }
                    }
                }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // read before the next piece is written
            }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // no copy is on its way to LDS that is another workgroup's by then
}

int launch_mx4_large(const void* pa, const void* pb, int K, const float* bias, const fps_view& v, hipStream_t st) {
    const Matrix y(v);
    const Packed a(pa, y.all_rows(), K), b(pb, y.all_cols(), K);
    TileMap map;
    map.tiles_m = (y.all_rows() + kTileEdge - 1) / kTileEdge;
    map.tiles_n = (y.all_cols() + kTileEdge - 1) / kTileEdge;
    const long long total = (long long)map.tiles_m * map.tiles_n;
    if (total > 0x0FFFFFFF) { set_error("more tiles than a launch has workgroups for"); return FPS_ERR_UNSUPPORTED; }
    map.total = (int)total;
    map.workgroups = 256;
    if (v.dt == FPS_OUT_F32) mx4_large_kernel<true><<<map.workgroups, 256, 0, st>>>(a, b, bias, y, map);
    else                     mx4_large_kernel<false><<<map.workgroups, 256, 0, st>>>(a, b, bias, y, map);
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? FPS_OK : hip_fail(e, "mx4_matmul launch");
}

}  // namespace fps
