// Products of large microscaled 4-bit matrices.
//
// A workgroup of four waves, one on each SIMD of a CU, takes 256 x 256 elements of the result, a wave 128 x 128 of them in 256
// accumulation registers; it stays on its CU and goes from tile to tile.  Half a step of both operands, 128 columns in 32 KB,
// is a slot of a ring of four in the LDS; a slot is filled again as soon as it is read, three of them before it is needed, across the
// end of a tile as well.  Of results with fewer tiles, 128 x 128 elements in the same manner, two workgroups a CU.
//
// 75600 x 5120 x 5120 887 us, 4.5 PFLOP/s; 16384 x 16384 x 16384 1.80 ms, 4.9.  The matrix unit is busy in 62 % (71 %) of the cycles, at the 1.5 to
// 1.6 GHz that the chip's power leaves it (at 2.4 GHz its peak is 10 PFLOP/s); in the others its wave waits.  Of memory
// 0.90 GB (1.72) are read, 4 (6) times the operands.  (A whole step copied ahead instead of the
// ring, 16384^3 1.93 ms; the result stored between the tiles instead of among the next one's multiplications, 32760 x 1536 x 4608 166 us instead of 143.
// So are results in fp32, or in rows that are not multiples of 8 elements: 75600 x 5120 x 5120 1042 and 955 us, 32760 x 1536 x 4608 221 and 165.)
#include "fps_mx4.h"

namespace fps {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kHalf = kMxStepBytes / 2, kSlots = 4;

// A workgroup's tile is 64 W rows and columns, a wave's 32 W; its LDS, in bytes
template <int W, bool F32>
struct Tile {
    static constexpr int EDGE = 64 * W, TILES = 2 * W;                        // of 32 rows, of each operand
    static constexpr int SLOT = 2 * TILES * kHalf, SCALES = kSlots * SLOT, SCALE_SLOT = 2 * TILES * kMxScaleBytes;
    static constexpr int PIECES = SCALES + 2 * SCALE_SLOT;                    // on the way out 32 rows of 128 bytes a wave, or of 64 so that
    static constexpr int ROW = W == 4 || F32 ? 128 : 64, PITCH = ROW + 16, PIECE = 32 * PITCH;     // two workgroups have room on a CU
    static constexpr int BIAS = PIECES + 4 * PIECE, BYTES = BIAS + (W == 4 && !F32 ? 4 * EDGE * 4 : 0);
};

struct TileMap { int tiles_m, tiles_n, total, workgroups; };

// From device memory to LDS, lane i's 16 bytes to dst + 16 i: 1 KB from a wave-uniform src (FAR bytes further on), or from the lanes'
// own addresses.  Inline assembly, so that the compiler does not wait for the copies before it reads other parts of the LDS.
// The instruction's offset counts on both sides, so dst is given FAR less.
template <int FAR>
__device__ __forceinline__ void copy_1k(const void* src, uint32_t lane_off, uint32_t dst, int dst_more) {
    asm volatile("s_add_i32 m0, %2, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 offset:%4"
                 : : "v"(lane_off), "s"(src), "s"(dst), "n"(dst_more - FAR), "n"(FAR) : "memory", "m0", "scc");
}
__device__ __forceinline__ void copy_lanes(const void* src, uint32_t lane_off, uint32_t dst) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(lane_off), "s"(src), "s"(dst) : "memory", "m0");
}
__device__ __forceinline__ void copy_lanes(const void* src, uint32_t dst) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(src), "s"(dst) : "memory", "m0");
}
// The lane's number, worked out anew: what follows from it is then not kept in registers where every one is taken
__device__ __forceinline__ int lane_anew() {
    int l;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(l));
    return l;
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

template <int WT, bool F32, bool HIDDEN, bool PAST>
__global__ __launch_bounds__(256, WT == 4 ? 1 : 2) void mx4_large_kernel(Packed a, Packed b, const float* __restrict__ bias, Matrix y, TileMap map) {
    static_assert(!HIDDEN || (WT == 4 && !F32), "a result on its way among the next tile's multiplications is in bf16");
    static_assert(!PAST || HIDDEN, "only those stores pass the caches");
    using L = Tile<WT, F32>;
    constexpr int QUARTER = WT * WT, COPIES = 2 * WT;        // multiplications of 64 columns; copies of half a step, without scales
    __shared__ __attribute__((aligned(1024))) uint8_t lds[L::BYTES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1, h = lane >> 5;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
    const int steps = a.steps;

    // this workgroup's tiles: first, first + stride, .. < end
    const int xcd = blockIdx.x & 7, per_xcd = (map.total + 7) >> 3, stride = map.workgroups >> 3;
    const int end = min_of(map.total, (xcd + 1) * per_xcd);
    int tile = xcd * per_xcd + (blockIdx.x >> 3);
    if (tile >= end) return;

    // copying: where the step that is copied next lies; wave w copies operand w / 2's row tiles WT (w % 2) .., and scales of four
    const Packed& mine = wave < 2 ? a : b;
    int copy_tile = tile, copy_step = 0;
    const char* codes_at[WT];                                // of the row tiles
    const char* scales_at;                                   // of their scales,
    uint32_t scales_off;                                     // the lane's share of which is 16 bytes of tile lane / 16
    auto locate = [&]() __attribute__((always_inline)) {
        const Place p = place_of(map, copy_tile);
        const int all = (wave < 2 ? p.m : p.n) * L::TILES, first = all + WT * (wave & 1), four = WT == 4 ? first : all;
#pragma unroll
        for (int i = 0; i < WT; ++i)                         // beyond the last row tile: the last one again
            codes_at[i] = (const char*)mine.codes + (long long)min_of(first + i, mine.tiles - 1) * steps * kMxStepBytes;
        const int base = min_of(four, mine.tiles - 1);
        scales_at = (const char*)mine.scales + (long long)base * steps * kMxScaleBytes;
        scales_off = (uint32_t)(min_of(four + (lane >> 4), mine.tiles - 1) - base) * steps * kMxScaleBytes + 16 * (lane & 15);
    };
    locate();
    uint32_t lane_off = 16 * lane;
    const uint32_t code_slots = lds0 + WT * wave * kHalf, scale_slots = lds0 + L::SCALES + 4 * (WT == 4 ? wave : wave >> 1) * kMxScaleBytes;
    // one of the copies of half a step: kilobyte n % 2 of row tile n / 2; par: parity of the step
    auto copy_codes = [&](int par, auto half_tag, auto n_tag) __attribute__((always_inline)) {
        constexpr int half = decltype(half_tag)::value, n = decltype(n_tag)::value, far = half * kHalf + (n & 1) * 1024;
        copy_1k<far>(codes_at[n >> 1], lane_off, code_slots + par * (2 * L::SLOT), half * L::SLOT + (n >> 1) * kHalf + (n & 1) * 1024);
    };
    auto copy_scales = [&](int par) __attribute__((always_inline)) { copy_lanes(scales_at, scales_off, scale_slots + par * L::SCALE_SLOT); };
    // to the next step; behind the last tile of the result the last one's again, or what follows it, which nobody reads
    auto advance = [&]() __attribute__((always_inline)) {
        const bool more = ++copy_step < steps;
        const int by = more ? 1 : 1 - steps;                 // without a further tile: from the start
        if (!more) {
            copy_step = 0;
            copy_tile += stride;
        }
#pragma unroll
        for (int i = 0; i < WT; ++i) codes_at[i] += (long long)by * kMxStepBytes;
        scales_at += (long long)by * kMxScaleBytes;
        if (!more && copy_tile < end) locate();
    };

    uint4 ca[2][WT], cb[2][WT];
    uint32_t sa[WT], sb[WT], sa_next[WT], sb_next[WT];
    const uint8_t *read_a, *read_b, *read_sa, *read_sb;
    auto read_by = [&](int l) __attribute__((always_inline)) {
        read_a = lds + WT * wm * kHalf + 16 * l;
        read_b = lds + (L::TILES + WT * wn) * kHalf + 16 * l;
        read_sa = lds + L::SCALES + WT * wm * kMxScaleBytes + 4 * l;
        read_sb = lds + L::SCALES + (L::TILES + WT * wn) * kMxScaleBytes + 4 * l;
    };
    read_by(lane);
    // one of the operands of quarter q (0 or 1) of a slot, in the order of their use
    auto read = [&](int set, int slot, int q, int n) __attribute__((always_inline)) {
        const int at_slot = slot * L::SLOT + q * 1024, i = n > WT ? n - WT : 0, j = n > 0 && n <= WT ? n - 1 : 0;
        if (n == 1 || n > WT) ca[set][i] = *reinterpret_cast<const uint4*>(read_a + at_slot + i * kHalf);
        else                  cb[set][j] = *reinterpret_cast<const uint4*>(read_b + at_slot + j * kHalf);
    };
    auto read_scales = [&](int slot, int i) __attribute__((always_inline)) {
        sa_next[i] = *reinterpret_cast<const uint32_t*>(read_sa + slot * L::SCALE_SLOT + i * kMxScaleBytes);
        sb_next[i] = *reinterpret_cast<const uint32_t*>(read_sb + slot * L::SCALE_SLOT + i * kMxScaleBytes);
    };
    v16f acc[WT][WT];
    auto multiply = [&](auto q_tag, int n, bool first) __attribute__((always_inline)) {     // rows 32 (n / WT) .., columns 32 (n % WT) ..
        constexpr int q = decltype(q_tag)::value, set = q & 1;
        const v16f zero = {};
        const int i = n / WT, j = n % WT;
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(cb[set][j]), operand(ca[set][i]), first ? zero : acc[i][j], 4, 4, q,
                                                                    (int)sb[j], q, (int)sa[i]);
    };

    // steps 0 and 1 of the sequence: COPIES + 1 copies a wave for the first half of a step, COPIES for the second
    auto copy_half = [&](int par, auto half_tag) __attribute__((always_inline)) {
        copy_codes(par, half_tag, Count<0>{}); copy_codes(par, half_tag, Count<1>{}); copy_codes(par, half_tag, Count<2>{});
        copy_codes(par, half_tag, Count<3>{});
        if constexpr (WT == 4) {
            copy_codes(par, half_tag, Count<4>{}); copy_codes(par, half_tag, Count<5>{}); copy_codes(par, half_tag, Count<6>{});
            copy_codes(par, half_tag, Count<7>{});
        }
    };
    copy_scales(0);
    copy_half(0, Count<0>{});
    copy_half(0, Count<1>{});
    advance();
    copy_scales(1);
    copy_half(1, Count<0>{});
    copy_half(1, Count<1>{});
    meet<3 * COPIES + 1>();
    int parity = 0;                                          // of the step: its slots are 2 parity and 2 parity + 1
#pragma unroll
    for (int n = 0; n < 2 * WT; ++n) read(0, 0, 0, n);
#pragma unroll
    for (int i = 0; i < WT; ++i) read_scales(0, i);
    const int M = y.all_rows(), N = y.all_cols();
    // ---- a tile's way out: pieces of 32 rows and 64 or 32 columns by way of the wave's own part of the LDS, which gives rows of 128 or 64 bytes.
    // A wave's LDS instructions are carried out in their order, so none of this waits for anything but what it reads.
    constexpr int E = F32 ? 4 : 2, W = 16 / E, JJ = L::ROW / (32 * E), LANES = L::ROW / 16;    // bytes an element, elements of a lane's chunk,
                                                                                             // blocks and chunks of a piece's row
    struct Piece { uint8_t* in; const uint8_t* out; int row; };
    auto piece_of = [&](int l) __attribute__((always_inline)) {
        uint8_t* const piece = lds + L::PIECES + wave * L::PIECE;
        return Piece{piece + (l & 31) * L::PITCH + 4 * (l >> 5) * E, piece + l / LANES * L::PITCH + 16 * (l % LANES), l / LANES};
    };

    // HIDDEN: the sums of the tile before, in bf16: registers 8 (4 i + j) + 2 q, + 1 are columns 8 q + 4 h .. of block (i, j)
    uint32_t sums[HIDDEN ? 128 : 1];
    int done_rows = 0;                                       // rows of it; there is no tile before the first
    uint32_t done_at[2];                                     // where the lane's chunk of each 64 columns lies in its row, of the first rows;
                                                             // all ones, an offset that the store itself drops, outside the matrix
    auto rows_from = [&](int row) __attribute__((always_inline)) {
        return __builtin_amdgcn_make_buffer_rsrc(y.data + row * y.stride_r, 0, 0xFFFFFFF0, 0x00027000);
    };
    __amdgpu_buffer_rsrc_t done = rows_from(0);
    const int stride_r = (int)y.stride_r;
    uint4 chunk[2];
    auto to_piece = [&](const Piece& at, int k, int n) __attribute__((always_inline)) {           // one of the eight writes of piece k
        const int i = k >> 1, j = 2 * (k & 1) + (n >> 2), q = n & 3, r = 8 * (4 * i + j) + 2 * q;
        *reinterpret_cast<uint2*>(at.in + ((n >> 2) * 32 + 8 * q) * 2) = make_uint2(sums[r], sums[r + 1]);
    };
    auto from_piece = [&](const Piece& at, int t) __attribute__((always_inline)) { chunk[t & 1] = *reinterpret_cast<const uint4*>(at.out + 64 / LANES * t * L::PITCH); };
    auto store_chunk = [&](const Piece& at, int k, int t) __attribute__((always_inline)) {        // no branch, which would part the multiplications
        const int down = 32 * (k >> 1) + 8 * t;
        const uint32_t outside = (uint32_t)((done_rows - 1 - down - at.row) >> 31);
        typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
        __builtin_amdgcn_raw_buffer_store_b128(u32x4{chunk[t & 1].x, chunk[t & 1].y, chunk[t & 1].z, chunk[t & 1].w}, done, done_at[k & 1] | outside, down * stride_r, PAST ? 2 : 0);       // 2: past the caches
    };
    // What follows multiplication n of 64 of a tile's first step: piece n / 8 is written, and its four chunks are read and, two
    // multiplications later, stored, two at a time (there are no registers for more)
    auto way_out = [&](const Piece& at, int n) __attribute__((always_inline)) {
        const int k = n >> 3, m = n & 7;
        if (m < 2 && k > 0) store_chunk(at, k - 1, 2 + m);
        if (m == 6 || m == 7) store_chunk(at, k, m - 6);
        if (m < 4) { to_piece(at, k, 2 * m); to_piece(at, k, 2 * m + 1); }
        else from_piece(at, m - 4);
    };
    uint8_t* const bias_out = lds + L::BIAS + wave * L::EDGE * 4;
    const uint32_t bias_slot = lds0 + L::BIAS + wave * L::EDGE * 4;

    for (; tile < end; tile += stride) {
        const int l0 = lane_anew();
        read_by(l0);
        lane_off = 16 * l0;
        const Place p = place_of(map, tile);
        // The order is as written.  A multiplication takes the matrix unit 32 cycles or more and the wave is alone on its SIMD: what else
        // there is to issue, the operands of the next 64 columns and the copies, stands between the multiplications, one at a time.
        auto step = [&](auto first_tag) __attribute__((always_inline)) {
            constexpr bool first = decltype(first_tag)::value, out = HIDDEN && first;
            Piece at_piece;
            if (out) at_piece = piece_of(lane_anew());
#pragma unroll
            for (int i = 0; i < WT; ++i) { sa[i] = sa_next[i]; sb[i] = sb_next[i]; }
            advance();                                       // before all else: behind a branch the multiplications would wait for it
            __builtin_amdgcn_sched_barrier(0);
            auto half = [&](auto h_tag) __attribute__((always_inline)) {
                constexpr int hf = decltype(h_tag)::value;
                const int slot = 2 * parity + hf, next = hf ? 2 * (parity ^ 1) : slot + 1;
#pragma unroll
                for (int n = 0; n < QUARTER; ++n) {
                    multiply(Count<2 * hf>{}, n, first && hf == 0);
                    if (n < 2 * WT) read(1, slot, 1, n);
                    if (out) way_out(at_piece, 32 * hf + n);
                    if (out && hf == 0 && n == 0) {
                        const int c = min_of(p.n * L::EDGE + 4 * lane_anew(), N - 4);
                        copy_lanes((const char*)(bias ? bias : (const float*)b.scales) + (bias ? 4LL * c : 0), bias_slot);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                // The next slot has landed, of two more the copies go on; this one is read.  Behind the copies that are waited for there
                // are the bias and the stores of a first step.
                meet<2 * COPIES + 1 + (out ? (hf ? 23 : 7) : 0)>();
                auto copying = [&](auto n_tag) __attribute__((always_inline)) {
                    constexpr int n = decltype(n_tag)::value;
                    multiply(Count<2 * hf + 1>{}, n, false);
                    if (n < 2 * WT) read(0, next, 0, n);
                    if constexpr (n >= QUARTER - COPIES) copy_codes(parity, h_tag, Count<n - QUARTER + COPIES>{});    // of the step after the next,
                    if (n == QUARTER / 2 - 1 && !hf) copy_scales(parity);                                             // into this slot
                    if (n >= WT && n < 2 * WT && hf) read_scales(parity ^ 1, n - WT);
                    if (out) way_out(at_piece, 32 * hf + 16 + n);
                    __builtin_amdgcn_sched_barrier(0);
                };
                copying(Count<0>{}); copying(Count<1>{}); copying(Count<2>{}); copying(Count<3>{});
                if constexpr (WT == 4) {
                    copying(Count<4>{}); copying(Count<5>{}); copying(Count<6>{}); copying(Count<7>{});
                    copying(Count<8>{}); copying(Count<9>{}); copying(Count<10>{}); copying(Count<11>{});
                    copying(Count<12>{}); copying(Count<13>{}); copying(Count<14>{}); copying(Count<15>{});
                }
            };
            half(Count<0>{});
            half(Count<1>{});
            parity ^= 1;
            if (out) {
#pragma unroll
                for (int t = 2; t < 4; ++t) store_chunk(at_piece, 7, t);
            }
        };
        step(std::true_type{});
        for (int s = 1; s < steps; ++s) step(std::false_type{});

        const int row0 = p.m * L::EDGE + wm * (L::EDGE / 2), col0 = p.n * L::EDGE + wn * (L::EDGE / 2);
        auto biased = [&](int i, int j, int q, float (&v)[4]) __attribute__((always_inline)) {
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = acc[i][j][4 * q + k];
            if (bias) {
                const int c = col0 + 32 * j + 8 * q + 4 * h;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (c + k < N) v[k] += bias[c + k];
            }
        };
        if constexpr (HIDDEN) {
            if (steps == 1) asm volatile("s_waitcnt vmcnt(17)" ::: "memory");        // the bias was copied in this very step
            const int l = lane_anew();
            const uint8_t* const bias_at = bias_out + (wn * 128 + 4 * (l >> 5)) * 4;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float4 read = *reinterpret_cast<const float4*>(bias_at + (32 * j + 8 * q) * 4);
                    const float add[4] = {bias ? read.x : 0.0f, bias ? read.y : 0.0f, bias ? read.z : 0.0f, bias ? read.w : 0.0f};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float v[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) v[k] = acc[i][j][4 * q + k] + add[k];
                        const int r = 8 * (4 * i + j) + 2 * q;
                        sums[r] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{v[0], v[1]}, bf16x2));
                        sums[r + 1] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{v[2], v[3]}, bf16x2));
                    }
                    __builtin_amdgcn_sched_barrier(0);       // the accumulators are read as they are converted
                }
            done = rows_from(row0);
            done_rows = M - row0;
#pragma unroll
            for (int jj = 0; jj < 2; ++jj) {
                const int col = col0 + 64 * jj + 8 * (l & 7);
                done_at[jj] = col < N ? (uint32_t)((l >> 3) * stride_r) + (uint32_t)y.column<2>(col) : 0xFFFFFFFFu;
            }
        } else {
            const Piece at_piece = piece_of(lane);
#pragma unroll
            for (int i = 0; i < WT; ++i)
#pragma unroll
                for (int jj = 0; jj < WT; jj += JJ) {
#pragma unroll
                    for (int j = jj; j < jj + JJ; ++j)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            float v[4];
                            biased(i, j, q, v);
                            uint8_t* const at = at_piece.in + ((j - jj) * 32 + 8 * q) * E;
                            if (F32) *reinterpret_cast<float4*>(at) = make_float4(v[0], v[1], v[2], v[3]);
                            else *reinterpret_cast<uint2*>(at) =
                                     make_uint2(__builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{v[0], v[1]}, bf16x2)),
                                                __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{v[2], v[3]}, bf16x2)));
                        }
#pragma unroll
                    for (int t = 0; t < LANES / 2; ++t) {
                        from_piece(at_piece, t);
                        const int row = row0 + 32 * i + 64 / LANES * t + lane / LANES, col = col0 + 32 * jj + W * (lane % LANES);
                        if (row >= M || col >= N) continue;
                        char* dst = y.row(row) + y.column<E>(col);
                        if (col + W <= N) {
                            __builtin_memcpy(dst, &chunk[t & 1], 16);
                        } else {
                            const uint32_t w[4] = {chunk[t & 1].x, chunk[t & 1].y, chunk[t & 1].z, chunk[t & 1].w};
#pragma unroll
                            for (int k = 0; k < W - 1; ++k)
                                if (col + k < N) {
                                    if (F32) reinterpret_cast<uint32_t*>(dst)[k] = w[k];
                                    else     reinterpret_cast<uint16_t*>(dst)[k] = (uint16_t)(w[k >> 1] >> (16 * (k & 1)));
                                }
                        }
                    }
                }
        }
    }
    if (HIDDEN) {
        const Piece at_piece = piece_of(lane);
#pragma unroll
        for (int n = 0; n < 64; ++n) way_out(at_piece, n);
#pragma unroll
        for (int t = 2; t < 4; ++t) store_chunk(at_piece, 7, t);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // no copy is on its way to LDS that is another workgroup's by then
}

template <int WT>
static int launch_tiles(const void* pa, const void* pb, int K, const float* bias, const fps_view& v, hipStream_t st) {
    const Matrix y(v);
    const Packed a(pa, y.all_rows(), K), b(pb, y.all_cols(), K);
    constexpr int EDGE = 64 * WT;
    TileMap map;
    map.tiles_m = (y.all_rows() + EDGE - 1) / EDGE;
    map.tiles_n = (y.all_cols() + EDGE - 1) / EDGE;
    const long long total = (long long)map.tiles_m * map.tiles_n;
    if (total > 0x0FFFFFFF) { set_error("more tiles than a launch has workgroups for"); return FPS_ERR_UNSUPPORTED; }
    map.total = (int)total;
    map.workgroups = WT == 4 ? 256 : 512;                    // one or two a CU, which stay
    if constexpr (WT == 4) {
        // The stores among the next tile's multiplications are of whole 16-byte chunks, at 32-bit offsets from a tile's first row; a
        // batch whose elements do not follow each other is written between the tiles
        const bool chunks = y.all_cols() % 8 == 0 && (y.stride_h | y.stride_r) % 16 == 0;
        const bool near = y.stride_r < (1 << 22) && 128 * y.stride_r + (y.heads - 1) * y.stride_h + 2LL * y.cols < 0xFFFFFFF0LL;
        // and past the caches, which keep the operands, where the result is more than the Infinity Cache's 256 MB: 75600 x 5120 x 5120 897 -> 887 us,
        // with its quantisation 1061 -> 1037, 32760 x 1536 x 4608 143 -> 138 (173 -> 157); of less, which the cache holds for what reads it next, 8192 x
        // 5120 x 5120 111, 112
        const bool past = 2LL * y.all_rows() * y.all_cols() > (256LL << 20);
        if (v.dt == FPS_OUT_F32)               mx4_large_kernel<4, true, false, false><<<map.workgroups, 256, 0, st>>>(a, b, bias, y, map);
        else if (y.B > 1 || !chunks || !near)  mx4_large_kernel<4, false, false, false><<<map.workgroups, 256, 0, st>>>(a, b, bias, y, map);
        else if (past)                         mx4_large_kernel<4, false, true, true><<<map.workgroups, 256, 0, st>>>(a, b, bias, y, map);
        else                                   mx4_large_kernel<4, false, true, false><<<map.workgroups, 256, 0, st>>>(a, b, bias, y, map);
    } else {
        if (v.dt == FPS_OUT_F32) mx4_large_kernel<2, true, false, false><<<map.workgroups, 256, 0, st>>>(a, b, bias, y, map);
        else                     mx4_large_kernel<2, false, false, false><<<map.workgroups, 256, 0, st>>>(a, b, bias, y, map);
    }
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? FPS_OK : hip_fail(e, "mx4_matmul launch");
}
int launch_mx4_tiles(int edge, const void* a, const void* b, int K, const float* bias, const fps_view& y, hipStream_t st) {
    return edge == 256 ? launch_tiles<4>(a, b, K, bias, y, st) : launch_tiles<2>(a, b, K, bias, y, st);
}

}  // namespace fps
