// Products of large microscaled 4-bit matrices.
//
// A workgroup of four waves, one on each SIMD of a CU, takes 256 x 256 elements of the result, a wave 128 x 128 of them in 256
// accumulation registers; it stays on its CU and goes from tile to tile.  A step of 256 columns of both operands, 68 KB, is
// copied into one half of the LDS while the other is multiplied, across the end of a tile as well.
#include "fps_mx4.h"

namespace fps {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kTileEdge = 256, kEdgeTiles = kTileEdge / kMxRows;
constexpr int kStageScales = 2 * kEdgeTiles * kMxStepBytes, kStage = kStageScales + 2 * kEdgeTiles * kMxScaleBytes;   // bytes
constexpr int kPiecePitch = 64 * 2 + 16, kPiece = 32 * kPiecePitch;       // 32 rows of 64 columns in bf16, on their way out

struct TileMap { int tiles_m, tiles_n, total, workgroups; };

// 4 KB (a tile's step of codes) and 256 bytes (its scales) from device memory to LDS, by one wave; src and dst are wave-uniform.
// Inline assembly, so that the compiler does not wait for the copies before it reads other parts of the LDS.
__device__ __forceinline__ const void* uniform(const void* p) {
    const uint64_t v = reinterpret_cast<uint64_t>(p);
    return reinterpret_cast<const void*>((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v) |
                                         ((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(v >> 32)) << 32));
}
__device__ __forceinline__ void copy_codes(const void* src, uint32_t lane_off, uint32_t dst) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\t"
                 "global_load_lds_dwordx4 %0, %1\n\tglobal_load_lds_dwordx4 %0, %1 offset:1024\n\t"
                 "global_load_lds_dwordx4 %0, %1 offset:2048\n\tglobal_load_lds_dwordx4 %0, %1 offset:3072"
                 : : "v"(lane_off), "s"(uniform(src)), "s"(__builtin_amdgcn_readfirstlane((int)dst)) : "memory", "m0");
}
__device__ __forceinline__ void copy_scales(const void* src, uint32_t lane_off, uint32_t dst) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1"
                 : : "v"(lane_off), "s"(uniform(src)), "s"(__builtin_amdgcn_readfirstlane((int)dst)) : "memory", "m0");
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
    __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * kStage + 4 * kPiece];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1, h = lane >> 5;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
    const int steps = a.steps;

    // this workgroup's tiles: first, first + stride, .. < end
    const int xcd = blockIdx.x & 7, per_xcd = (map.total + 7) >> 3, stride = map.workgroups >> 3;
    const int end = min_of(map.total, (xcd + 1) * per_xcd);
    int tile = xcd * per_xcd + (blockIdx.x >> 3);
    if (tile >= end) return;

    // copying: the tile and step that are copied next; wave w copies operand w / 2's row tiles 4 (w % 2) ..
    const Packed& mine = wave < 2 ? a : b;
    int copy_tile = tile, copy_step = 0, stage = 0;
    long long at[4];                                         // step 0 of the wave's row tiles, in steps
    auto locate = [&]() __attribute__((always_inline)) {
        const Place p = place_of(map, copy_tile);
        const int first = (wave < 2 ? p.m : p.n) * kEdgeTiles + 4 * (wave & 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) at[i] = (long long)min_of(first + i, mine.tiles - 1) * steps;    // beyond the last: the last
    };
    locate();
    // row tile i of the wave's share; behind the last tile of the result the last one's again, which nobody reads
    auto copy = [&](int i) __attribute__((always_inline)) {
        const long long s = at[i] + copy_step;
        const uint32_t base = lds0 + stage * kStage;
        copy_codes((const char*)mine.codes + s * kMxStepBytes, 16 * lane, base + (4 * wave + i) * kMxStepBytes);
        copy_scales((const char*)mine.scales + s * kMxScaleBytes, 4 * lane, base + kStageScales + (4 * wave + i) * kMxScaleBytes);
    };
    auto copied = [&]() __attribute__((always_inline)) {
        stage ^= 1;
        if (++copy_step == steps) {
            copy_step = 0;
            copy_tile += stride;
            if (copy_tile < end) locate();
        }
    };

    uint4 ca[2][4], cb[2][4];
    uint32_t sa[4], sb[4], sa_next[4], sb_next[4];
    const uint8_t* const read_a = lds + 4 * wm * kMxStepBytes + 16 * lane;
    const uint8_t* const read_b = lds + (kEdgeTiles + 4 * wn) * kMxStepBytes + 16 * lane;
    const uint8_t* const read_sa = lds + kStageScales + 4 * wm * kMxScaleBytes + 4 * lane;
    const uint8_t* const read_sb = lds + kStageScales + (kEdgeTiles + 4 * wn) * kMxScaleBytes + 4 * lane;
    auto read = [&](int set, int from, int q) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            ca[set][i] = *reinterpret_cast<const uint4*>(read_a + from * kStage + i * kMxStepBytes + q * 1024);
            cb[set][i] = *reinterpret_cast<const uint4*>(read_b + from * kStage + i * kMxStepBytes + q * 1024);
        }
    };
    auto read_scales = [&](int from) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            sa_next[i] = *reinterpret_cast<const uint32_t*>(read_sa + from * kStage + i * kMxScaleBytes);
            sb_next[i] = *reinterpret_cast<const uint32_t*>(read_sb + from * kStage + i * kMxScaleBytes);
        }
    };
    v16f acc[4][4];
    auto multiply = [&](auto q_tag, int i, bool first) __attribute__((always_inline)) {     // rows 32 i .. of the wave's
        constexpr int q = decltype(q_tag)::value, set = q & 1;
        const v16f zero = {};
#pragma unroll
        for (int j = 0; j < 4; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(cb[set][j]), operand(ca[set][i]), first ? zero : acc[i][j], 4,
                                                                        4, q, (int)sb[j], q, (int)sa[i]);
    };

#pragma unroll
    for (int i = 0; i < 4; ++i) copy(i);
    copied();
#pragma unroll
    for (int i = 0; i < 4; ++i) copy(i);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // of both: once a launch
    __syncthreads();
    int from = 0;
    read(0, 0, 0);
    read_scales(0);
    uint8_t* const piece = lds + 2 * kStage + wave * kPiece;
    const int M = y.all_rows(), N = y.all_cols();
    for (; tile < end; tile += stride) {
        // the order is as written: the operands of the next 64 columns are requested before these are multiplied
        auto step = [&](bool first) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) { sa[i] = sa_next[i]; sb[i] = sb_next[i]; }
            copied();                                        // before all else: behind a branch the multiplications would wait for it
            __builtin_amdgcn_sched_barrier(0);
            auto quarter = [&](auto q_tag) __attribute__((always_inline)) {
                constexpr int q = decltype(q_tag)::value;
                read((q + 1) & 1, from, q + 1);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < 4; ++i) multiply(q_tag, i, first && q == 0);
                __builtin_amdgcn_sched_barrier(0);
            };
            quarter(Count<0>{});
            quarter(Count<1>{});
            quarter(Count<2>{});
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); // the next step, whose copy began a step ago
            __syncthreads();                                 // all waves have read this one: the one after the next takes its place
            from ^= 1;
            read(0, from, 0);
            read_scales(from);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                multiply(Count<3>{}, i, false);
                __builtin_amdgcn_sched_barrier(0);
                copy(i);
                __builtin_amdgcn_sched_barrier(0);
            }
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
