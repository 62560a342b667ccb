// Matrix products of packed rows (e4m3 codes with a power-of-two scale for
// each row and block of 128 columns), and the gradient of their weights from
// packed activations.
#include "network.h"

#include <algorithm>
#include <type_traits>

namespace fbdt {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

struct Packed {
    const uint8_t *codes;
    int64_t ld;
    const uint8_t *scales;
    int64_t lds;
};

// The bytes of a 16-byte piece of codes that starts `live` columns before the
// row's end: those beyond it read as 0.
__device__ __forceinline__ i32x4 live_codes(i32x4 v, int live) {
    if (live >= 16) return v;
    i32x4 out;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const int have = live - 4 * w;
        const uint32_t mask = have >= 4 ? 0xffffffffu : have <= 0 ? 0u : (1u << (8 * have)) - 1;
        out[w] = v[w] & (int)mask;
    }
    return out;
}

// The bfloat16 values of 8 of a fragment's codes (words 2 q, 2 q + 1) under a scale.
__device__ __forceinline__ bf16x8 unpack_codes(i32x8 f, int q, float scale) {
    bf16x8 v;
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        const bf16x2 p = h % 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[2 * q + h / 2], scale, true)
                               : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[2 * q + h / 2], scale, false);
        v[2 * h] = p[0];
        v[2 * h + 1] = p[1];
    }
    return v;
}

__device__ __forceinline__ float scale_of(int exponent) {
    return __uint_as_float(exponent ? (uint32_t)exponent << 23 : 1u << 22);
}

template <int N>
struct Int {
    static constexpr int value = N;
};

// ---- few rows -------------------------------------------------------------------
// At most 16 rows of a against 16 rows of b per workgroup: what counts is that b
// streams from memory, all of it in flight at once.  A wavefront takes four blocks
// of columns at a time, a dword of scales per row, straight from memory to
// registers (few enough for 5 wavefronts per SIMD), and the wavefronts' sums are
// added in order through LDS.  Sums are in full, also where fast ones are allowed: the 8-bit
// unit's, which cut products off, would take at most a tenth less (one row times 10,240 x
// 2560, weights from memory: 8.8 us, 8.3 by it; 8 rows times 20,480 x 8192 42 and 39).
constexpr int kFewWaves = 8;
constexpr int kFewBlocks = 4;

template <typename O>
__global__ __launch_bounds__(kFewWaves *kWaveLanes) __attribute__((amdgpu_waves_per_eu(5)))
void product_few_kernel(Packed a, Packed b, int m, int n, int k, O *__restrict__ out, int64_t ldo) {
    __shared__ f32x4 sums[kFewWaves][kWaveLanes];
    const int lane = threadIdx.x % kWaveLanes;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWaveLanes);
    const int waves = blockDim.x / kWaveLanes;
    const int r = lane % 16, g = lane / 16;
    const int n0 = blockIdx.x * 16;
    const int arow = std::min(m - 1, r), brow = std::min(n - 1, n0 + r);
    const uint8_t *const pa = a.codes + arow * a.ld + g * 16, *const pb = b.codes + brow * b.ld + g * 16;
    const int steps = (k + kPackBlock - 1) / kPackBlock;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int first = wave * kFewBlocks; first < steps; first += waves * kFewBlocks) {
        i32x8 fb[kFewBlocks], fa[kFewBlocks];
        auto load = [&](const uint8_t *p, int at) {
            const i32x4 *const q = reinterpret_cast<const i32x4 *>(p + (int64_t)at * kPackBlock);
            return __builtin_shufflevector(q[0], q[4], 0, 1, 2, 3, 4, 5, 6, 7);
        };
#pragma unroll
        for (int u = 0; u < kFewBlocks; ++u) fb[u] = load(pb, std::min(first + u, steps - 1));
        const uint32_t eb = *reinterpret_cast<const uint32_t *>(b.scales + brow * b.lds + first);
        const uint32_t ea = *reinterpret_cast<const uint32_t *>(a.scales + arow * a.lds + first);
#pragma unroll
        for (int u = 0; u < kFewBlocks; ++u) fa[u] = load(pa, std::min(first + u, steps - 1));
        auto add = [&](auto U) __attribute__((always_inline)) {
            constexpr int u = decltype(U)::value;
            const int live = k - (first + u) * kPackBlock;   // (a block read again is not added)
            if (live <= 0) return;
            if (live < kPackBlock) {
                auto cut = [&](i32x8 f) {
                    const i32x4 lo = live_codes(__builtin_shufflevector(f, f, 0, 1, 2, 3), live - 16 * g);
                    const i32x4 hi = live_codes(__builtin_shufflevector(f, f, 4, 5, 6, 7), live - 16 * g - 64);
                    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                };
                fa[u] = cut(fa[u]);
                fb[u] = cut(fb[u]);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q)
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                    unpack_codes(fb[u], q, scale_of(eb >> (8 * u) & 255)),
                    unpack_codes(fa[u], q, scale_of(ea >> (8 * u) & 255)), acc, 0, 0, 0);
        };
        add(Int<0>{});
        add(Int<1>{});
        add(Int<2>{});
        add(Int<3>{});
    }
    sums[wave][lane] = acc;
    __syncthreads();
    if (wave > 0) return;
    // lane l holds row l % 16, columns n0 + 4 (l / 16) ..
    for (int w = 1; w < waves; ++w) acc += sums[w][lane];
    if (r < m) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n0 + 4 * g + e < n) out[r * ldo + n0 + 4 * g + e] = (O)acc[e];
    }
}

template <typename O>
hipError_t launch_few(const Packed &a, const Packed &b, int64_t m, int64_t n, int k, O *out,
                      int64_t ldo, hipStream_t s) {
    const int64_t waves = std::min<int64_t>(kFewWaves, ceil_div(ceil_div(k, kPackBlock), kFewBlocks));
    product_few_kernel<O><<<(unsigned)ceil_div(n, 16), (unsigned)(waves * kWaveLanes), 0, s>>>(
        a, b, (int)m, (int)n, k, out, ldo);
    return hipGetLastError();
}

// ---- tiles ----------------------------------------------------------------------
// A workgroup of WM x WN wavefronts computes a tile of the output, FM x FN
// fragments of 16 x 16 per wavefront, in steps of one block of 128 columns: the
// rows of both operands go from memory straight to LDS, one step ahead of the
// matrix instructions that read them.  A workgroup takes tile after tile: a tile's last
// step brings the next one's first rows, which arrive behind the stores of its results.
// (Tiles of 256 x 256 by 8 wavefronts of 128 x 64 each reach 2.8 PFLOP/s at 8192 x 8192 x
// 8192 and 2.45 at 65,536 x 10,240 x 2560; 2.78 and 2.35 by a workgroup per tile; 2.6 and
// 2.35 if a step's transfers are issued through all of it, not in its first half; 2.7
// and 2.3 by a workgroup of 16 wavefronts of 128 x 32 per tile, which has too few
// registers for more.  Matrix units are busy 64% of the time, LDS 25%.  These are fast sums;
// sums in full go through bfloat16 products at half the rate: 1.27 and 1.19 PFLOP/s.)
//
// A row's 128 codes lie in LDS as 8 pieces of 16 bytes; piece c of the row of place r
// among the 16 of its fragment is at position c ^ (r % 8), and lane (r, g) reads
// pieces g and g + 4: a read of 1 KB takes the 4 clocks of LDS's 256 bytes a clock
// (pieces 2 g and 2 g + 1: 8 clocks).  A transfer to LDS writes 16 bytes per lane in
// lane order, 8 rows per wavefront, so the exchange is made on the side of
// memory: lane l fetches piece (l % 8) ^ (r % 8).
__device__ __forceinline__ constexpr int swizzle(int r) { return r & 7; }

// A lane's results of a fragment are 4 consecutive columns; rows of b are dealt to
// fragments so that what it stores at once is 16 bytes and what the 4 lanes of an
// output row store is 64: row r of fragment j is b's row 16 j + r of the
// wavefront's, or for results of 16 bits row 32 (j / 2) + 8 (r / 4) + 4 (j % 2) + r % 4.
template <bool PAIRS>
__device__ __forceinline__ constexpr int b_row(int j, int r) {
    return PAIRS ? j / 2 * 32 + r / 4 * 8 + j % 2 * 4 + r % 4 : 16 * j + r;
}
template <bool PAIRS>
__device__ __forceinline__ constexpr int b_swizzle(int row) {
    return swizzle(PAIRS ? (row >> 3 & 3) * 4 + (row & 3) : row & 15);
}

typedef __attribute__((address_space(3))) void *lds_ptr;

// `bytes` from p on as a buffer that a lane addresses by a 32-bit offset.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void *p, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, (int)bytes, 0x00027000);
}

// 16 bytes per lane from a buffer to LDS at `to` + 16 lane (`to` is the wavefront's).
__device__ __forceinline__ void to_lds16(__amdgpu_buffer_rsrc_t from, uint32_t lane_offset,
                                         uint32_t offset, uint8_t *to) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_ptr)to, 16, (int)lane_offset, (int)offset, 0, 0);
}
__device__ __forceinline__ i32x4 load16(__amdgpu_buffer_rsrc_t from, uint32_t offset) {
    return __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(from, (int)offset, 0, 0));
}
__device__ __forceinline__ void to_lds4(__amdgpu_buffer_rsrc_t from, uint32_t lane_offset,
                                        uint32_t offset, uint8_t *to) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_ptr)to, 4, (int)lane_offset, (int)offset, 0, 0);
}

// The tile of workgroup `id` of a grid of tm x tn: each XCD (workgroups are dealt
// to the 8 XCDs in turn) takes a contiguous range of tiles, so that its L2 holds
// what it reads, in groups of kTileGroup tiles along m.
constexpr int kXcds = 8;
constexpr int kTileGroup = 4;

__device__ __forceinline__ void tile_of(uint32_t id, uint32_t tm, uint32_t tn, uint32_t *im,
                                        uint32_t *in) {
    const uint32_t total = tm * tn, per = total / kXcds, rest = total % kXcds;
    const uint32_t xcd = id % kXcds, q = id / kXcds;
    const uint32_t t = xcd * per + (xcd < rest ? xcd : rest) + q;
    const uint32_t group = t / (kTileGroup * tn);
    const uint32_t first = group * kTileGroup;
    const uint32_t rows = tm - first < kTileGroup ? tm - first : kTileGroup;
    const uint32_t in_group = t - group * kTileGroup * tn;
    *im = first + in_group % rows;
    *in = in_group / rows;
}

template <typename O, bool FAST, int WM, int WN, int FM, int FN, bool HALVES>
__global__ __launch_bounds__(WM *WN *kWaveLanes) void product_tile_kernel(
    Packed a, Packed b, int64_t m, int64_t n, int k, O *__restrict__ out, int64_t ldo, uint32_t tm,
    uint32_t tn, bool once) {
    constexpr int kWaves = WM * WN;
    constexpr int BM = WM * FM * 16, BN = WN * FN * 16;
    constexpr int kLoadsA = BM / 8 / kWaves, kLoadsB = BN / 8 / kWaves;
    constexpr bool kPairs = sizeof(O) == 2;
    static_assert(!kPairs || FN % 2 == 0, "pairs of fragments");
    static_assert(kLoadsA * 8 * kWaves == BM && kLoadsB * 8 * kWaves == BN, "whole loads");
    // one buffer per step parity (arrays of their own: what a step reads cannot be
    // what its transfers write)
    __shared__ __align__(1024) uint8_t codes0[(BM + BN) * kPackBlock];
    __shared__ __align__(1024) uint8_t codes1[(BM + BN) * kPackBlock];
    __shared__ __align__(256) uint8_t scales[2][(BM + BN) * 4];

    const int lane = threadIdx.x % kWaveLanes;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWaveLanes);
    const int steps = (k + kPackBlock - 1) / kPackBlock;

    const int wm = wave % WM * (FM * 16), wn = wave / WM * (FN * 16);
    const int r = lane % 16, g = lane / 16;
    const int arow = wm + r, brow = wn + b_row<kPairs>(0, r);

    // a tile's place and its rows, up to the end of the matrix (what is beyond reads as
    // 0, for results that are not stored)
    struct Tile {
        int64_t m0, n0;
        int live_m, live_n;
    };
    auto tile_at = [&](uint32_t id) __attribute__((always_inline)) {
        uint32_t im, in;
        tile_of(id, tm, tn, &im, &in);
        const int64_t m0 = (int64_t)im * BM, n0 = (int64_t)in * BN;
        return Tile{m0, n0, (int)std::min<int64_t>(BM, m - m0), (int)std::min<int64_t>(BN, n - n0)};
    };
    // what this lane transfers: pieces of rows, kRowsEach rows apart
    constexpr int kRowsEach = kWaves * 8;
    static_assert(kRowsEach % 32 == 0, "rows that are swizzled alike");
    const int own = wave * 8 + lane / 8;
    const uint32_t from_a = own * (uint32_t)a.ld + ((lane % 8) ^ swizzle(own & 15)) * 16;
    const uint32_t from_b = own * (uint32_t)b.ld + ((lane % 8) ^ b_swizzle<kPairs>(own)) * 16;
    constexpr int kScaleLoads = (BM + BN + kWaves * kWaveLanes - 1) / (kWaves * kWaveLanes);

    // rows from `first` on of a tile's `live` ones, as a buffer
    auto rows_from = [&](const uint8_t *p, int64_t ld, int first, int live) __attribute__((always_inline)) {
        return buffer_of(p + first * ld, (uint32_t)std::max(live - first, 0) * (uint32_t)ld);
    };
    // transfer t of the kLoadsB + kLoadsA of a step
    auto fetch = [&](const Tile &tile, int t, int step, uint8_t *codes) __attribute__((always_inline)) {
        if (t < kLoadsB)
            to_lds16(rows_from(b.codes + tile.n0 * b.ld, b.ld, t * kRowsEach, tile.live_n), from_b,
                     step * kPackBlock, codes + BM * kPackBlock + (t * kWaves + wave) * 1024);
        else if (t < kLoadsB + kLoadsA)
            to_lds16(rows_from(a.codes + tile.m0 * a.ld, a.ld, (t - kLoadsB) * kRowsEach, tile.live_m),
                     from_a, step * kPackBlock, codes + ((t - kLoadsB) * kWaves + wave) * 1024);
    };
    auto fetch_scales = [&](const Tile &tile, int step, uint8_t *scales) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < kScaleLoads; ++t) {
            const int first = (t * kWaves + wave) * kWaveLanes;   // 64 rows of a or of b
            if (first >= BM + BN) break;
            const bool of_a = first < BM;
            const uint32_t ld = (uint32_t)(of_a ? a.lds : b.lds);
            to_lds4(of_a ? rows_from(a.scales + tile.m0 * a.lds, a.lds, first, tile.live_m)
                         : rows_from(b.scales + tile.n0 * b.lds, b.lds, first - BM, tile.live_n),
                    lane * ld, step, scales + first * 4);
        }
    };

    f32x4 acc[FM][FN];
    uint32_t ea[FM], eb[FN];

    // (the last step of a width that ends inside a block: codes beyond it read as 0)
    auto read = [&](auto WHOLE, const uint8_t *row, int f, int live) __attribute__((always_inline)) {
        i32x4 lo = *reinterpret_cast<const i32x4 *>(row + (g ^ f) * 16);
        i32x4 hi = *reinterpret_cast<const i32x4 *>(row + ((g + 4) ^ f) * 16);
        if constexpr (!decltype(WHOLE)::value) {
            lo = live_codes(lo, live - 16 * g);
            hi = live_codes(hi, live - 16 * g - 64);
        }
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    // One step; byte s of the scales is its block's.  The next step's transfers are
    // issued among its products: those of the next tile's first step, if there is no
    // other.  (Every step issues them, those that nothing follows once more their own: a
    // branch costs registers that the loop does not have.)
    // They are issued in the first half of a step, to arrive by its end.
    constexpr int kPerFragment = 2 * ((kLoadsA + kLoadsB + FM - 1) / FM);
    auto compute = [&](auto WHOLE, auto S, const uint8_t *codes, int live, const Tile &next_tile,
                       int next_step, uint8_t *next) __attribute__((always_inline)) {
        constexpr int s = decltype(S)::value;
        i32x8 fb[FN];
#pragma unroll
        for (int j = 0; j < FN; ++j)
            fb[j] = read(WHOLE, codes + (BM + brow + b_row<kPairs>(j, 0)) * kPackBlock,
                         b_swizzle<kPairs>(brow + b_row<kPairs>(j, 0)), live);
        i32x8 ahead = read(WHOLE, codes + arow * kPackBlock, swizzle(r), live);
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const i32x8 fa = ahead;   // (the next rows' codes arrive behind these rows' products)
            if (i + 1 < FM) ahead = read(WHOLE, codes + (arow + 16 * (i + 1)) * kPackBlock, swizzle(r), live);
            __builtin_amdgcn_sched_barrier(0);   // (left alone, the compiler reads when it needs)
#pragma unroll
            for (int t = 0; t < kPerFragment; ++t) fetch(next_tile, i * kPerFragment + t, next_step, next);
            if constexpr (FAST) {
                // (cuts a product off 2^-13 below the largest of its 8: the caller's choice, for
                // twice the rate)
#pragma unroll
                for (int j = 0; j < FN; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                        fb[j], fa, acc[i][j], 0, 0, s, (int)eb[j], s, (int)ea[i]);
            } else {
                const float sa = scale_of(ea[i] >> (8 * s) & 255);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const bf16x8 va = unpack_codes(fa, q, sa);
#pragma unroll
                    for (int j = 0; j < FN; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            unpack_codes(fb[j], q, scale_of(eb[j] >> (8 * s) & 255)), va, acc[i][j], 0,
                            0, 0);
                }
            }
        }
    };
    auto read_scales = [&](const uint8_t *scales) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < FM; ++i)
            ea[i] = *reinterpret_cast<const uint32_t *>(scales + (arow + 16 * i) * 4);
#pragma unroll
        for (int j = 0; j < FN; ++j)
            eb[j] = *reinterpret_cast<const uint32_t *>(scales + (BM + brow + b_row<kPairs>(j, 0)) * 4);
    };

    // this step's rows are in LDS, and all wavefronts are done with the last one's
    auto arrive = [&]() __attribute__((always_inline)) {
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
    };
    const int whole = k / kPackBlock;
    constexpr int kEach = kPairs ? 8 : 4;   // consecutive columns that a lane stores
    const uint32_t tiles = tm * tn, stride = gridDim.x;
    Tile tile = tile_at(blockIdx.x);
#pragma unroll
    for (int t = 0; t < kLoadsA + kLoadsB; ++t) fetch(tile, t, 0, codes0);
    fetch_scales(tile, 0, scales[0]);
    // (a wavefront's memory operations complete in order: with no more than the stores of
    // a whole tile under way, which are issued last, the next tile's first rows are there)
    constexpr int kStores = FM * FN * 4 / kEach;
    constexpr int kAllButStores = (kStores & 15) | 7 << 4 | kStores >> 4 << 14;
    static_assert(kStores < 64, "what a wait counts");
    __builtin_amdgcn_s_waitcnt(0);
    for (uint32_t id = blockIdx.x;; id += stride) {
        const bool more = id + stride < tiles;
        const Tile next = tile_at(more ? id + stride : id);
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        // the scales of step `at`, an even one, to the lowest bytes of ea and eb
        auto turn_scales = [&](int at) __attribute__((always_inline)) {
            if (at % 4 == 0) {
                read_scales(scales[at / 4 % 2]);
                if (at + 4 < steps) fetch_scales(tile, at + 4, scales[at / 4 % 2 ^ 1]);
            } else {
#pragma unroll
                for (int i = 0; i < FM; ++i) ea[i] >>= 16;
#pragma unroll
                for (int j = 0; j < FN; ++j) eb[j] >>= 16;
            }
        };
        int at = 0;
        // two steps a round, so that the buffers are constants
        for (; at + 2 <= whole; at += 2) {
            if (at > 0) __builtin_amdgcn_s_waitcnt(0);
            __builtin_amdgcn_s_waitcnt(kAllButStores);
            __syncthreads();
            turn_scales(at);
            compute(Int<1>{}, Int<0>{}, codes0, kPackBlock, tile, std::min(at + 1, steps - 1), codes1);
            arrive();
            const bool last = at + 2 >= steps;
            compute(Int<1>{}, Int<1>{}, codes1, kPackBlock, last ? next : tile, last ? 0 : at + 2, codes0);
        }
        const bool rest = at < steps;
        // an odd whole step, and a width that ends inside a block
        for (bool odd = false; at < steps; ++at, odd = true) {
            arrive();
            if (!odd) {
                turn_scales(at);
            } else {
#pragma unroll
                for (int i = 0; i < FM; ++i) ea[i] >>= 8;
#pragma unroll
                for (int j = 0; j < FN; ++j) eb[j] >>= 8;
            }
            compute(Int<0>{}, Int<0>{}, odd ? codes1 : codes0, std::min(k - at * kPackBlock, kPackBlock),
                    tile, std::min(at + 1, steps - 1), odd ? codes0 : codes1);
        }
        if (more) {
            // the next tile's first rows, if they are not on their way, and scales (all
            // wavefronts have this tile's in registers)
            if (rest) {
                arrive();
#pragma unroll
                for (int t = 0; t < kLoadsA + kLoadsB; ++t) fetch(next, t, 0, codes0);
            }
            fetch_scales(next, 0, scales[0]);
        }
        __builtin_amdgcn_sched_barrier(0);
        // lane l holds rows wm + 16 i + l % 16 and, of fragment j, columns b_row(j, 4 (l / 16)) ..
        // (the compiler does not see that first_row and first_col are the same for every
        // tile: it would keep all places of the results in registers)
        int first_row = arow, first_col = wn + b_row<kPairs>(0, 4 * g);
        asm volatile("" : "+v"(first_row), "+v"(first_col));
        O *const corner = out + tile.m0 * ldo + tile.n0;
        auto values = [&](int i, int j, O (&v)[kEach]) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < kEach; ++e) v[e] = (O)acc[i][j + e / 4][e % 4];
            return corner + (first_row + 16 * i) * ldo + first_col + b_row<kPairs>(j, 0);
        };
        // Rows of 16-bit results that begin inside a dword, as every other one of an odd stride
        // does, would store at half the rate: their lanes' pieces move on by one element, which
        // the lane of the columns behind gives; the first lane stores its first element by
        // itself, the last one 7.  (32,996 x 4287 x 72: 111 us, pieces as they are 164.)
        auto store_at_halves = [&](O *to, int live, const O (&v)[kEach]) __attribute__((always_inline)) {
            if constexpr (HALVES) {
                uint32_t w[5];
                __builtin_memcpy(w, v, 16);
                w[4] = (uint32_t)__shfl((int)w[0], (lane + 16) & 63);
                const bool inside = (reinterpret_cast<uintptr_t>(to) & 2) != 0;
                const int by = inside ? 16 : 0;
                u32x4 raw;
#pragma unroll
                for (int e = 0; e < 4; ++e) raw[e] = __builtin_amdgcn_alignbit(w[e + 1], w[e], by);
                const int skip = inside ? 1 : 0;
                int have = live - skip;
                if (inside && g == 3) have = std::min(have, kEach - 1);
                if (inside && g == 0 && live > 0) to[0] = v[0];
                to += skip;
                if (have >= kEach) {
                    *reinterpret_cast<u32x4_at_2 *>(to) = raw;
                } else if (have > 0) {
                    O t[kEach];
                    __builtin_memcpy(t, &raw, sizeof t);
                    if (have == kEach - 1) {
                        __builtin_memcpy(to, t, 12);
                        to[6] = t[6];
                    } else {
#pragma unroll
                        for (int e = 0; e < kEach - 2; ++e)
                            if (e < have) to[e] = t[e];
                    }
                }
            }
        };
        if (tile.live_m == BM && tile.live_n == BN && !HALVES) {
            // past the cache, which the operands need (1.51 against 1.84 ms for 65,536 x
            // 10,240 x 2560), if the 64 bytes that a row's 4 lanes store are a line's half:
            // 32,996 x 4296 x 72 82 us, past the cache 231
            auto store_all = [&](bool past) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int j = 0; j < FN; j += kEach / 4) {
                        O v[kEach];
                        O *const to = values(i, j, v);
                        u32x4 raw;
                        __builtin_memcpy(&raw, v, sizeof raw);
                        store_piece(to, raw, past);
                    }
            };
            if (once) store_all(true);
            else store_all(false);
        } else {
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; j += kEach / 4) {
                    O v[kEach];
                    O *const to = values(i, j, v);
                    const int live = first_row + 16 * i < tile.live_m
                                         ? tile.live_n - (first_col + b_row<kPairs>(j, 0)) : 0;
                    if constexpr (HALVES) {
                        store_at_halves(to, live, v);
                    } else if (live >= kEach) {
                        u32x4 raw;
                        __builtin_memcpy(&raw, v, sizeof raw);
                        store_piece(to, raw, once);
                    } else {
#pragma unroll
                        for (int e = 0; e < kEach; ++e)
                            if (e < live) to[e] = v[e];
                    }
                }
            __builtin_amdgcn_s_waitcnt(0);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (!more) break;
        tile = next;
    }
}

// A workgroup for each tile, as far as a launch goes.
constexpr int64_t kAllTiles = 1 << 22;

// `groups`: workgroups at most.
template <typename O, bool FAST, int WM, int WN, int FM, int FN>
hipError_t launch_tiles(const Packed &a, const Packed &b, int64_t m, int64_t n, int k, O *out,
                        int64_t ldo, int64_t groups, hipStream_t s) {
    const int64_t tm = ceil_div(m, WM * FM * 16), tn = ceil_div(n, WN * FN * 16);
    constexpr int kThreads = WM * WN * kWaveLanes;
    auto go = [&](auto halves) {
        product_tile_kernel<O, FAST, WM, WN, FM, FN, decltype(halves)::value>
            <<<(unsigned)std::min(tm * tn, groups), kThreads, 0, s>>>(
                a, b, m, n, k, out, ldo, (uint32_t)tm, (uint32_t)tn,
                aligned_to(out, 64) && ldo * sizeof(O) % 64 == 0);
    };
    if constexpr (sizeof(O) == 2) {
        if (!aligned_to(out, 4) || ldo % 2 != 0) go(std::true_type{});
        else go(std::false_type{});
    } else {
        go(std::false_type{});
    }
    return hipGetLastError();
}

// The tile that is done first by these figures, in us, of workgroups per CU at a
// time, start and end of a tile, and a step: 256 x 256: 1, 6.4, 1.42; 128 x 128: 2,
// 2, 0.91 (alone on a CU 3 and 0.55); 64 x 64: 4, 2, 0.65 (alone 0.25, two 0.35).
// Measured, in this order: 4096 x 4096 x 4096 57, 64 and 105 us; 2000 x 2000 x 2000 29,
// 14.6 and 17.3; 3000 x 5000 x 700 34, 26 and 32; 128 x 10,240 x 2560 28, 13.9 and 11.2.
// Few rows take the kernel for them (weights from memory: one row times 10,240 x 2560 8.8 us,
// by tiles with fast sums 18.2; times 1280 x 1280 3.8 and 7.5; times 20,480 x 8192 35 and 55;
// 8 rows times 5120 x 5120 11.8 and 32; 16 rows times 512 x 9000 11.5 and 37).  9 to 16
// rows times many take tiles: 16 times 10,240 x 2560 with weights in cache 8.4, by the other
// 9.7, times 40,000 x 640 6.7 and 12, as the workgroups read more of a than of b (weights
// from memory: 18.2 and 11.4, 9.1 and 13.4).  Sums in full take the 128 x 128 tile where they would take the largest one,
// whose unpacked fragments leave too few registers.
//
// Workgroups that take tile after tile are as many as run at a time: 65,536 x 1280 x 1280
// in 109 us by tiles of 128 x 128 (a workgroup per tile 117), 105 by those of 256 x 256
// (110).  Sums in full and tiles of 64 x 64 take a workgroup per tile (65,536 x 2560 x
// 2560 in full 745 us, in turn 754; 500,000 x 64 x 640 84 and 88).
template <typename O, bool FAST>
hipError_t launch_product(const Packed &a, const Packed &b, int64_t m, int64_t n, int k, O *out,
                          int64_t ldo, int cus, hipStream_t s) {
    const double steps = (double)ceil_div(k, kPackBlock);
    auto tiles = [&](int64_t t) { return ceil_div(m, t) * ceil_div(n, t); };
    const int64_t t256 = tiles(256), t128 = tiles(128), t64 = tiles(64);
    if (m <= 8 || (m <= 16 && t64 <= cus / 4)) return launch_few<O>(a, b, m, n, k, out, ldo, s);
    const double d256 = ceil_div(t256, cus) * (6.4 + 1.42 * steps);
    const double d128 = ceil_div(t128, 2 * cus) * (t128 <= cus ? 3 + 0.55 * steps : 2 + 0.91 * steps);
    const double d64 = ceil_div(t64, 4 * cus) * (2 + steps * (t64 <= cus ? 0.25 : t64 <= 2 * cus ? 0.35 : 0.65));
    if constexpr (FAST) {
        if (d256 <= d128 && d256 <= d64)
            return launch_tiles<O, FAST, 2, 4, 8, 4>(a, b, m, n, k, out, ldo, cus, s);
    }
    if (d128 <= d64) return launch_tiles<O, FAST, 2, 2, 4, 4>(a, b, m, n, k, out, ldo, FAST ? 2 * cus : kAllTiles, s);
    return launch_tiles<O, FAST, 2, 2, 2, 2>(a, b, m, n, k, out, ldo, kAllTiles, s);
}

// ---- gradient of the weights ---------------------------------------------------
// A workgroup of WN x WK wavefronts adds a tile of the gradient (rows: columns of
// dy, columns: those of x) over its share of the rows, kGradRows at a time.  Both
// operands lie in LDS as bfloat16 with the rows of memory as rows, x unpacked on
// the way: a packed value is exact in bfloat16.  The sum runs along the rows, so
// the matrix instructions want 8 rows of one column in a lane: the transposing
// LDS read gives 4 of them, from 4 rows of 16 columns that 16 lanes address.
//
// Piece c (16 bytes, 8 columns) of row r is at position c ^ f(r), so that the
// rows that are read at a time (4 of each 8) lie in different banks.
//
// Rows start at multiples of 16 bytes (others are copied first) and come through
// buffers whose range ends with the share's last row, what is beyond it reads as
// 0: no branch, so loads and stores to LDS go among the matrix instructions of the
// step before.  (65,536 x 2560 x 2560: 750 to 780 us, 1.1 PFLOP/s; with
// the loads before a step's products and the stores after them 989.  Matrix units are
// busy 56% of the time, LDS 42%: each step's first products wait for their fragments.)
constexpr int kGradRows = 64;
constexpr int64_t kAlignedStride = 1 << 22;   // elements: 64 rows in 32-bit offsets

// Rows of n elements at multiples of 8 elements (10,007 x 333: 6 us).
__global__ __launch_bounds__(256) void align_rows_kernel(const __bf16 *__restrict__ dy, int64_t lddy,
                                                         int64_t m, int n, __bf16 *__restrict__ out,
                                                         int64_t ldo) {
    const int64_t per = ldo / kChunk, q = group_number() * 256 + threadIdx.x;
    if (q >= m * per) return;
    const int64_t row = q / per;
    const int c = (int)(q - row * per) * kChunk;
    const RawChunk<__bf16> v = load_raw_once(dy + row * lddy + c, n - c);
    __builtin_memcpy(out + row * ldo + c, &v, sizeof v);
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 *lds_s16x4;

template <int COLUMNS>
__device__ __forceinline__ constexpr int grad_swizzle(int row) {
    return ((row & 3) * 2 | (row >> 3 & 3) * 8) & (COLUMNS / 8 - 1);
}

// Fragments for 32 rows: lane l gets column l % 16 of rows 8 (l / 16) .. + 7.
__device__ __forceinline__ bf16x8 read_columns(const uint8_t *at, int four_rows) {
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)at);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(at + four_rows));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

template <typename O, int WN, int WK, int FN, int FK>
__global__ __launch_bounds__(WN *WK *kWaveLanes) void weight_grad_kernel(
    const __bf16 *__restrict__ dy, int64_t lddy, int64_t m, int n, Packed x, int k,
    O *__restrict__ out, int64_t ldo, int64_t part_stride, uint32_t tn, uint32_t tk,
    int64_t steps_per_part) {
    constexpr int kThreads = WN * WK * kWaveLanes;
    constexpr int BN = WN * FN * 16, BK = WK * FK * 16;
    constexpr int kPiecesY = BN / 8, kPiecesX = BK / 16;          // of a row, 16 bytes of memory each
    constexpr int kLoadsY = kGradRows * kPiecesY / kThreads, kLoadsX = kGradRows * kPiecesX / kThreads;
    constexpr int kRowsY = kThreads / kPiecesY, kRowsX = kThreads / kPiecesX;   // per load
    static_assert(kLoadsY * kRowsY == kGradRows && kLoadsX * kRowsX == kGradRows, "whole loads");
    __shared__ __align__(1024) uint8_t ys[2][kGradRows * BN * 2];
    __shared__ __align__(1024) uint8_t xs[2][kGradRows * BK * 2];

    uint32_t in, ik;
    tile_of(blockIdx.x % (tn * tk), tn, tk, &in, &ik);
    const int64_t part = blockIdx.x / (tn * tk);
    const int n0 = in * BN, k0 = ik * BK;
    const int64_t first = part * steps_per_part * kGradRows;
    const int64_t last = std::min<int64_t>(m, first + steps_per_part * kGradRows);

    // what this thread brings: pieces of one column range of dy and one of x
    const int py = threadIdx.x % kPiecesY, ry = threadIdx.x / kPiecesY;
    const int px = threadIdx.x % kPiecesX, rx = threadIdx.x / kPiecesX;
    i32x4 vy[kLoadsY], vx[kLoadsX];
    uint32_t ex[kLoadsX];
    const uint32_t y_row = (uint32_t)lddy * 2, x_row = (uint32_t)x.ld, e_row = (uint32_t)x.lds;
    const uint32_t y_at = ry * y_row + (n0 + 8 * py) * 2, x_at = rx * x_row + k0 + 16 * px;
    const uint32_t e_at = rx * e_row + (k0 + 16 * px) / kPackBlock;
    auto fetch = [&](int64_t row0) __attribute__((always_inline)) {
        // rows from row0 on: at most kGradRows of them, none from `last` on
        const int64_t rows = std::min<int64_t>(kGradRows, last - row0);
        const uint32_t before = rows > 0 ? (uint32_t)rows - 1 : 0, some = rows > 0;
        const int64_t from = rows > 0 ? row0 : first;
        const __amdgpu_buffer_rsrc_t yb =
            buffer_of(dy + from * lddy, some * (before * y_row + (2 * (uint32_t)n + 3) / 4 * 4));
        const __amdgpu_buffer_rsrc_t xb =
            buffer_of(x.codes + from * x.ld,
                      some * (before * x_row + (uint32_t)((k + kPackBlock - 1) / kPackBlock * kPackBlock)));
        const __amdgpu_buffer_rsrc_t eb =
            buffer_of(x.scales + from * x.lds,
                      some * (before * e_row + (uint32_t)((k + kPackBlock - 1) / kPackBlock)));
#pragma unroll
        for (int t = 0; t < kLoadsY; ++t) vy[t] = load16(yb, y_at + t * kRowsY * y_row);
#pragma unroll
        for (int t = 0; t < kLoadsX; ++t) {
            vx[t] = load16(xb, x_at + t * kRowsX * x_row);
            ex[t] = __builtin_amdgcn_raw_buffer_load_b8(eb, (int)(e_at + t * kRowsX * e_row), 0, 0);
        }
    };
    // piece t of the kLoadsY + kLoadsX that this thread brought, to LDS
    constexpr int kPieces = kLoadsY + kLoadsX;
    auto put = [&](int t, int buffer) __attribute__((always_inline)) {
        if (t < kLoadsY) {
            const int row = ry + t * kRowsY;
            *reinterpret_cast<i32x4 *>(ys[buffer] + row * BN * 2 + (py ^ grad_swizzle<BN>(row)) * 16) =
                vy[t];
        } else if (t < kPieces) {
            const int row = rx + (t - kLoadsY) * kRowsX;
            const i32x4 codes = vx[t - kLoadsY];
            const float scale = scale_of((int)ex[t - kLoadsY]);
            uint8_t *const to = xs[buffer] + row * BK * 2 + ((2 * px) ^ grad_swizzle<BK>(row)) * 16;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                bf16x8 v;
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[2 * h + w], scale, false);
                    const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[2 * h + w], scale, true);
                    v[4 * w] = lo[0];
                    v[4 * w + 1] = lo[1];
                    v[4 * w + 2] = hi[0];
                    v[4 * w + 3] = hi[1];
                }
                *reinterpret_cast<bf16x8 *>(to + 16 * h) = v;
            }
        }
    };

    const int lane = threadIdx.x % kWaveLanes, wave = threadIdx.x / kWaveLanes;
    const int g = lane / 16, j = lane % 16;
    const int wn = wave % WN * (FN * 16), wk = wave / WN * (FK * 16);
    const int row = 8 * g + j / 4;      // of each 32; its 4 columns 4 (j % 4) ..
    int at_y[FN], at_x[FK];
#pragma unroll
    for (int f = 0; f < FN; ++f)
        at_y[f] = row * BN * 2 + (((wn + 16 * f) / 8 + j % 4 / 2) ^ grad_swizzle<BN>(row)) * 16 + j % 2 * 8;
#pragma unroll
    for (int f = 0; f < FK; ++f)
        at_x[f] = row * BK * 2 + (((wk + 16 * f) / 8 + j % 4 / 2) ^ grad_swizzle<BK>(row)) * 16 + j % 2 * 8;
    f32x4 acc[FN][FK];
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
        for (int f = 0; f < FK; ++f) acc[i][f] = f32x4{0.f, 0.f, 0.f, 0.f};

    // One step: the products of what is in `buffer`.  Among them, what was brought for
    // the next step goes to the other buffer, and then the loads for the step after
    // that are issued: neither memory nor LDS is waited for.
    auto compute = [&](int buffer, int64_t row_after) __attribute__((always_inline)) {
        constexpr int kPutEach = (kPieces + FN - 1) / FN;
#pragma unroll
        for (int c = 0; c < kGradRows; c += 32) {
            bf16x8 fx[FK];
#pragma unroll
            for (int f = 0; f < FK; ++f)
                fx[f] = read_columns(xs[buffer] + at_x[f] + c * BK * 2, 4 * BK * 2);
            bf16x8 ahead = read_columns(ys[buffer] + at_y[0] + c * BN * 2, 4 * BN * 2);
#pragma unroll
            for (int i = 0; i < FN; ++i) {
                const bf16x8 fy = ahead;
                if (i + 1 < FN) ahead = read_columns(ys[buffer] + at_y[i + 1] + c * BN * 2, 4 * BN * 2);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int f = 0; f < FK; ++f)
                    acc[i][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fx[f], fy, acc[i][f], 0, 0, 0);
                if (c == 0) {
#pragma unroll
                    for (int t = 0; t < kPutEach; ++t) put(i * kPutEach + t, buffer ^ 1);
                }
            }
            if (c == 0) fetch(row_after);
        }
    };
    if (first < last) {
        fetch(first);
#pragma unroll
        for (int t = 0; t < kPieces; ++t) put(t, 0);
        fetch(first + kGradRows);
        __syncthreads();
        auto step = [&](int buffer, int64_t row0) __attribute__((always_inline)) {
            compute(buffer, row0 + 2 * kGradRows);
            __syncthreads();
        };
        for (int64_t row0 = first; row0 < last; row0 += 2 * kGradRows) {
            step(0, row0);
            if (row0 + kGradRows < last) step(1, row0 + kGradRows);
        }
    }

    // lane l holds row wn + 16 i + l % 16, columns wk + 16 f + 4 (l / 16) ..
    O *const to = out + part * part_stride;
#pragma unroll
    for (int i = 0; i < FN; ++i) {
        const int r = n0 + wn + 16 * i + j;
        if (r >= n) continue;
#pragma unroll
        for (int f = 0; f < FK; ++f) {
            const int c = k0 + wk + 16 * f + 4 * g;
            O v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = (O)acc[i][f][e];
            if (c + 4 <= k) {
                __builtin_memcpy(to + (int64_t)r * ldo + c, v, sizeof v);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (c + e < k) to[(int64_t)r * ldo + c + e] = v[e];
            }
        }
    }
}

// out = the sum of `parts` matrices [n][k], in order (5 of 2560 x 2560: 24 us, 6.4 TB/s).
template <typename O>
__global__ __launch_bounds__(256) void add_parts_kernel(const float *__restrict__ partial, int parts,
                                                        int64_t part_stride, int n, int k,
                                                        O *__restrict__ out, int64_t ldo) {
    const int per = (k + 3) / 4;
    const int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (q >= (int64_t)n * per) return;
    const int64_t row = q / per;
    const int c = (int)(q - row * per) * 4, live = k - c;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    const float *from = partial + row * k + c;
    constexpr int kAhead = 8;
    for (int p = 0; p < parts; p += kAhead, from += kAhead * part_stride) {
        float v[kAhead][4];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[u][e] = 0.f;
            if (p + u < parts) {
                if (live >= 4) {
                    __builtin_memcpy(v[u], from + u * part_stride, sizeof v[u]);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (e < live) v[u][e] = from[u * part_stride + e];
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] += v[u][e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < live) out[row * ldo + c + e] = (O)sum[e];
}

// How the rows are shared out, into `parts` parts per tile: what takes the least
// time by these figures, in us, measured at 64 to 2560 columns and 300 to 65,536
// rows (the plans came out within 15% of the best of 2 x 20).  A step of the
// large tile takes 1.5 and fills a CU; one of the small tile takes 0.8, or 1.15
// where two share a CU.  A workgroup takes 4 to begin and end; parts are written
// and read at about 4 MB per us.
struct GradPlan {
    bool large;            // tiles of 256 x 256, else 128 x 128
    int64_t tn, tk, parts, steps_per_part;
};
constexpr int kPlanCus = 256;          // the plan sizes the workspace without a device

GradPlan plan_weight_grad(int64_t m, int64_t n, int64_t k) {
    GradPlan best = {};
    double least = 0;
    const int64_t steps = std::max<int64_t>(ceil_div(m, kGradRows), 1);
    constexpr int kTries[] = {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 40, 48, 64, 96, 128, 192, 256};
    for (int large = 0; large < 2; ++large) {
        const int64_t tile = large ? 256 : 128, slots = large ? kPlanCus : 2 * kPlanCus;
        const int64_t tn = ceil_div(n, tile), tk = ceil_div(k, tile);
        for (const int64_t tried : kTries) {
            if (tried > steps) break;
            const int64_t per = ceil_div(steps, tried), parts = ceil_div(steps, per);
            const int64_t groups = tn * tk * parts;
            const double step = large ? 1.5 : groups <= kPlanCus ? 0.8 : 1.15;
            double cost = ceil_div(groups, slots) * (4 + per * step);
            if (parts > 1) cost += 3 + 0.05 * parts + 8e-6 / 4 * parts * n * k;
            if (least == 0 || cost < least) {
                least = cost;
                best = {large != 0, tn, tk, parts, per};
            }
        }
    }
    return best;
}

// Bytes of a copy of dy at aligned rows (0: dy's rows are aligned).
int64_t aligned_rows_bytes(const void *dy, int64_t lddy, int64_t m, int64_t n) {
    if (m == 0 || (aligned_to(dy, 16) && (m == 1 || (lddy % kChunk == 0 && lddy <= kAlignedStride)))) return 0;
    return (m * ceil_div(n, kChunk) * kChunk * 2 + 255) / 256 * 256;
}

template <typename O, int WN, int WK, int FN, int FK>
hipError_t launch_weight_grad(const GradPlan &p, const __bf16 *dy, int64_t lddy, int64_t m, int n,
                              const Packed &x, int k, O *out, int64_t ldo, float *work,
                              hipStream_t s) {
    const unsigned grid = (unsigned)(p.tn * p.tk * p.parts);
    constexpr int kThreads = WN * WK * kWaveLanes;
    auto tiles = [&](auto *to, int64_t ld, int64_t part_stride) {
        typedef std::remove_reference_t<decltype(*to)> T;
        weight_grad_kernel<T, WN, WK, FN, FK><<<grid, kThreads, 0, s>>>(
            dy, lddy, m, n, x, k, to, ld, part_stride, (uint32_t)p.tn, (uint32_t)p.tk,
            p.steps_per_part);
        return hipGetLastError();
    };
    if (p.parts == 1) return tiles(out, ldo, 0);
    const int64_t size = (int64_t)n * k;
    hipError_t e = tiles(work, k, size);
    if (e != hipSuccess) return e;
    add_parts_kernel<O><<<(unsigned)ceil_div((int64_t)n * ceil_div(k, 4), 256), 256, 0, s>>>(
        work, (int)p.parts, size, n, k, out, ldo);
    return hipGetLastError();
}

int check_packed(const char *name, const uint8_t *codes, int64_t ld, const uint8_t *scales,
                 int64_t lds, int32_t k) {
    const int64_t blocks = ceil_div(k, kPackBlock);
    if (!codes || !aligned_to(codes, 16))
        return report(FBDT_E_INVAL, "%s: codes must be 16-byte aligned", name);
    // (a tile of 256 rows is addressed by 32-bit offsets)
    if (ld < blocks * kPackBlock || ld % kPackBlock != 0 || ld > 1 << 23)
        return report(FBDT_E_INVAL, "%s: row stride %lld must be a multiple of 128, >= width %d and "
                      "<= 2^23", name, (long long)ld, k);
    if (!scales || !aligned_to(scales, 4))
        return report(FBDT_E_INVAL, "%s: scales must be 4-byte aligned", name);
    if (lds < blocks || lds % 4 != 0 || lds > 1 << 23)
        return report(FBDT_E_INVAL, "%s: scale stride %lld must be a multiple of 4, at most 2^23, and "
                      "hold %lld blocks", name, (long long)lds, (long long)blocks);
    return FBDT_OK;
}

int check_out(void *out, int32_t dtype, int64_t ldo, int64_t n) {
    if (!known_dtype(dtype)) return report(FBDT_E_INVAL, "out: unknown type %d", dtype);
    if (!out || !aligned_to(out, dtype_bytes(dtype)))
        return report(FBDT_E_INVAL, "out must be aligned to its elements");
    if (ldo < n)
        return report(FBDT_E_INVAL, "out: row stride %lld is below the width %lld", (long long)ldo,
                      (long long)n);
    return FBDT_OK;
}

// That a result [rows][width] lies apart from packed rows of width k.
int check_apart_packed(const void *out, int32_t dtype, int64_t rows, int64_t width, int64_t ldo,
                       const char *name, const Packed &p, int64_t packed_rows, int64_t k) {
    const Extent result = {out, rows, width, ldo, dtype_bytes(dtype)};
    const int rc = check_apart("out", result, name, {p.codes, packed_rows, k, p.ld, 1});
    return rc ? rc : check_apart("out", result, name,
                                 {p.scales, packed_rows, ceil_div(k, kPackBlock), p.lds, 1});
}

int check_product(int64_t m, int64_t n, int64_t k) {
    if (m < 0 || m >= (int64_t)1 << 31)
        return report(FBDT_E_INVAL, "m = %lld must be in [0, 2^31)", (long long)m);
    if (n < 1 || n > 1 << 20) return report(FBDT_E_INVAL, "n = %lld must be in [1, 2^20]", (long long)n);
    if (k < 1 || k > 1 << 20) return report(FBDT_E_INVAL, "k = %lld must be in [1, 2^20]", (long long)k);
    if (ceil_div(m, 16) * ceil_div(n, 16) >= (int64_t)1 << 31)
        return report(FBDT_E_INVAL, "m = %lld and n = %lld are too large", (long long)m, (long long)n);
    return FBDT_OK;
}

}  // namespace
}  // namespace fbdt

using namespace fbdt;

extern "C" {

int fbdt_packed_product(const uint8_t *a, int64_t lda, const uint8_t *a_scales, int64_t ldas,
                        int64_t m, const uint8_t *b, int64_t ldb, const uint8_t *b_scales,
                        int64_t ldbs, int32_t n, int32_t k, void *out, int32_t dtype, int64_t ldo,
                        int32_t fast, void *stream) {
    int rc;
    if ((rc = check_product(m, n, k))) return rc;
    if ((rc = check_packed("b", b, ldb, b_scales, ldbs, k))) return rc;
    if (m == 0) return FBDT_OK;
    if ((rc = check_packed("a", a, lda, a_scales, ldas, k))) return rc;
    if ((rc = check_out(out, dtype, ldo, n))) return rc;
    const Packed pa = {a, lda, a_scales, ldas}, pb = {b, ldb, b_scales, ldbs};
    if ((rc = check_apart_packed(out, dtype, m, n, ldo, "a", pa, m, k)) ||
        (rc = check_apart_packed(out, dtype, m, n, ldo, "b", pb, n, k)))
        return rc;
    int cus = 0;
    if ((rc = device_cus(&cus))) return rc;
    NET_TRY(with_dtype(dtype, [&](auto t) {
        typedef decltype(t) O;
        hipStream_t s = static_cast<hipStream_t>(stream);
        O *const o = static_cast<O *>(out);
        return fast ? launch_product<O, true>(pa, pb, m, n, k, o, ldo, cus, s)
                    : launch_product<O, false>(pa, pb, m, n, k, o, ldo, cus, s);
    }));
    return FBDT_OK;
}

int64_t fbdt_packed_weight_grad_work(const void *dy, int64_t lddy, int64_t m, int32_t n, int32_t k) {
    if (check_product(m, n, k)) return -1;
    const GradPlan p = plan_weight_grad(m, n, k);
    return aligned_rows_bytes(dy, lddy, m, n) + (p.parts > 1 ? 4 * p.parts * (int64_t)n * k : 0);
}

int fbdt_packed_weight_grad(const void *dy, int64_t lddy, int64_t m, int32_t n, const uint8_t *x,
                            int64_t ldx, const uint8_t *x_scales, int64_t ldxs, int32_t k, void *out,
                            int32_t dtype, int64_t ldo, void *work, int64_t work_bytes,
                            void *stream) {
    int rc;
    if ((rc = check_product(m, n, k))) return rc;
    if ((rc = check_out(out, dtype, ldo, k))) return rc;
    if (m > 0) {
        if (!dy || !aligned_to(dy, 2)) return report(FBDT_E_INVAL, "dy must be aligned to its elements");
        if (lddy < n)
            return report(FBDT_E_INVAL, "dy: row stride %lld is below the width %d", (long long)lddy, n);
        if ((rc = check_packed("x", x, ldx, x_scales, ldxs, k))) return rc;
    }
    const int64_t need = fbdt_packed_weight_grad_work(dy, lddy, m, n, k);
    if (work_bytes < need || (need > 0 && (!work || !aligned_to(work, 256))))
        return report(FBDT_E_INVAL, "work must hold %lld bytes, 256-byte aligned", (long long)need);
    const Packed px = {x, ldx, x_scales, ldxs};
    if ((rc = check_apart("out", {out, n, k, ldo, dtype_bytes(dtype)}, "dy", {dy, m, n, lddy, 2})) ||
        (rc = check_apart_packed(out, dtype, n, k, ldo, "x", px, m, k)))
        return rc;
    NET_TRY(with_dtype(dtype, [&](auto t) {
        typedef decltype(t) O;
        hipStream_t s = static_cast<hipStream_t>(stream);
        const __bf16 *y = static_cast<const __bf16 *>(dy);
        // (a single row may have any stride: the kernel's offsets are those of whole pieces, so
        // that the rows it has beside this one begin where the buffer's range ends)
        int64_t ldy = m == 1 ? ceil_div(n, kChunk) * kChunk : lddy;
        if (const int64_t bytes = aligned_rows_bytes(dy, lddy, m, n)) {
            __bf16 *const to = static_cast<__bf16 *>(work);
            ldy = ceil_div(n, kChunk) * kChunk;
            const dim3 grid = grid_of(ceil_div(m * (ldy / kChunk), 256), 256);
            align_rows_kernel<<<grid, 256, 0, s>>>(y, lddy, m, n, to, ldy);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            y = to;
            work = static_cast<char *>(work) + bytes;
        }
        float *const w = static_cast<float *>(work);
        const GradPlan p = plan_weight_grad(m, n, k);
        return p.large ? launch_weight_grad<O, 2, 4, 8, 4>(p, y, ldy, m, n, px, k, static_cast<O *>(out),
                                                           ldo, w, s)
                       : launch_weight_grad<O, 2, 2, 4, 4>(p, y, ldy, m, n, px, k, static_cast<O *>(out),
                                                           ldo, w, s);
    }));
    return FBDT_OK;
}

}  // extern "C"
