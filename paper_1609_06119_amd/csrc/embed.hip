// Tokens of binned events, the lookup of their vectors, and the gradient of
// the table by sorted tokens.
#include "network.h"

#include <algorithm>
#include <type_traits>

namespace fbdt {
namespace {

// ---- tokens of binned events ------------------------------------------------
// tokens[i][j] = j B + code[j][i], -1 for a missing value.  The codes are
// feature-major and the tokens event-major: a tile of kTokenEvents events goes
// through LDS, so that both sides move whole cache lines.  Memory bounds it (2M events of
// 40 features: 69 us, 5.8 TB/s; a token per lane at a time 99).
constexpr int kTokenThreads = 256;
constexpr int kTokenEvents = 64;

__global__ __launch_bounds__(kTokenThreads) void event_tokens_kernel(
    const uint8_t *__restrict__ xb, int64_t n, int d, int64_t ldb, int n_bins,
    int32_t *__restrict__ tokens) {
    extern __shared__ uint8_t tile[];   // [d][kTokenEvents]
    const int64_t first = group_number() * kTokenEvents;
    if (first >= n) return;
    const int live = (int)std::min<int64_t>(kTokenEvents, n - first);
    // (rows hold a multiple of 16 codes: a load of 16 that starts before n stays inside)
    for (int q = threadIdx.x; q < d * (kTokenEvents / 16); q += kTokenThreads) {
        const int j = q / (kTokenEvents / 16), i = q % (kTokenEvents / 16) * 16;
        if (i < live)
            *reinterpret_cast<u32x4 *>(tile + j * kTokenEvents + i) =
                *reinterpret_cast<const u32x4 *>(xb + j * ldb + first + i);
    }
    __syncthreads();
    int32_t *const out = tokens + first * d;
    const int count = live * d;
    for (int q = threadIdx.x * 4; q < count; q += kTokenThreads * 4) {
        int i = q / d, j = q - i * d;
        int token[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int code = q + e < count ? tile[j * kTokenEvents + i] : 0;
            token[e] = code < n_bins ? j * n_bins + code : -1;
            if (++j == d) j = 0, ++i;
        }
        if (q + 4 <= count) {
            u32x4 raw;
            __builtin_memcpy(&raw, token, sizeof raw);
            store_piece_once(out + q, raw);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (q + e < count) out[q + e] = token[e];
        }
    }
}

// ---- lookup -----------------------------------------------------------------
// out[i] = scale table[token_i]; a token outside the table gives a row of
// zeros.  A lane moves 16 bytes of a row, 2^log_lanes lanes share one row.  The
// rows written bound it (the table stays in cache): stores that do not stay in
// cache and a single row per lane, which keeps the most wavefronts resident (10M rows of
// 64 bfloat16 values: 195 us, 6.6 TB/s written; 1,000 events of 40 features 3.6).
constexpr int kLookupThreads = 256;

template <typename T, typename I, bool ONCE>
__global__ __launch_bounds__(kLookupThreads) void lookup_kernel(
    const T *__restrict__ table, uint32_t rows, int width, int64_t ldt,
    const I *__restrict__ tokens, int64_t n, float scale, T *__restrict__ out, int64_t ldo,
    int log_lanes) {
    constexpr int kEach = 16 / sizeof(T);
    const int64_t i = (group_number() * kLookupThreads + threadIdx.x) >> log_lanes;
    if (i >= n) return;
    const I token = tokens[i];
    const bool met = token >= 0 && (uint64_t)token < rows;
    const T *const from = table + (met ? (int64_t)token : 0) * ldt;
    T *const to = out + i * ldo;
    for (int c = (threadIdx.x & ((1 << log_lanes) - 1)) * kEach; c < width; c += kEach << log_lanes) {
        T v[kEach];
        if (c + kEach <= width) {
            __builtin_memcpy(v, from + c, sizeof v);
#pragma unroll
            for (int k = 0; k < kEach; ++k) v[k] = met ? (T)((float)v[k] * scale) : (T)0.f;
            u32x4 raw;
            __builtin_memcpy(&raw, v, sizeof raw);
            store_piece(to + c, raw, ONCE);
        } else {
#pragma unroll
            for (int k = 0; k < kEach; ++k)
                if (c + k < width) to[c + k] = met ? (T)((float)from[c + k] * scale) : (T)0.f;
        }
    }
}

// The same for rows that begin inside 16 bytes and lie one after another: a lane moves the
// 16 bytes of the result from a multiple of 16 on, which end one row and begin the next
// where a row ends inside them (no row is shorter than that).  The row is found by the
// width's reciprocal in float64, which may be one off.
template <typename T, typename I>
__global__ __launch_bounds__(kLookupThreads) void lookup_flat_kernel(
    const T *__restrict__ table, uint32_t rows, int width, double per_width, int64_t ldt,
    const I *__restrict__ tokens, int64_t n, float scale, T *__restrict__ out) {
    constexpr int kEach = 16 / sizeof(T);
    const int64_t first = (group_number() * kLookupThreads + threadIdx.x) * kEach;
    const int64_t left = n * width - first;
    if (left <= 0) return;
    int64_t i = (int64_t)((double)first * per_width);
    int64_t c = first - i * width;
    if (c < 0) c += width, --i;
    if (c >= width) c -= width, ++i;
    const int skip = std::max((int)c + kEach - width, 0);   // elements of the next row
    auto row = [&](int64_t at, int from, bool &met) __attribute__((always_inline)) {
        const I token = tokens[at];
        met = token >= 0 && (uint64_t)token < rows;
        unsigned __int128 raw;
        __builtin_memcpy(&raw, table + (met ? (int64_t)token : 0) * ldt + from, sizeof raw);
        return raw;
    };
    bool met, met_next = false;
    unsigned __int128 raw = row(i, (int)c - skip, met) >> (skip * 8 * sizeof(T));
    if (skip > 0 && i + 1 < n) raw |= row(i + 1, 0, met_next) << ((kEach - skip) * 8 * sizeof(T));
    T v[kEach];
    __builtin_memcpy(v, &raw, sizeof v);
#pragma unroll
    for (int k = 0; k < kEach; ++k)
        v[k] = (k < kEach - skip ? met : met_next) ? (T)((float)v[k] * scale) : (T)0.f;
    if (left >= kEach) {
        u32x4 piece;
        __builtin_memcpy(&piece, v, sizeof piece);
        store_piece_once(out + first, piece);
    } else {
#pragma unroll
        for (int k = 0; k < kEach; ++k)
            if (k < left) out[first + k] = v[k];
    }
}

// ---- tokens in order --------------------------------------------------------
// A stable radix sort of (token, position): masked tokens take the key `rows`
// and go last.  A pass counts the digits of each tile, scans the counts of
// each digit over the tiles, and moves every pair to its place: its rank among
// the pairs of its digit in its wavefront (from ballots of the digit's bits)
// after those of the tile's earlier wavefronts, of earlier tiles and of
// smaller digits.  No order depends on timing.  (10M tokens of 13 bits, two passes: counts
// 12 and 11 us, scans 8 each, moves 43 and 35, of which the ranks take most.)
constexpr int kSortThreads = 512;
constexpr int kSortWaves = kSortThreads / kWaveLanes;
constexpr int kSortItems = 8;       // (10M x 64: 404 us in all, 16 420; 1M x 64: 90 and 103)
// few tokens: smaller tiles, up to kFewTiles of them, and no launch to scan their counts
// (20,000 tokens x 64: 44 us in all, sorted as many tokens are 52; 131,072 x 32: 57 and 60;
// 262,144 x 32: 71 and 68; 1M x 64: 135 and 90)
constexpr int kSortFewItems = 4;
constexpr int kFewTiles = 128;
// (wider digits of large sorts would leave room for one workgroup per CU)
constexpr int digit_bits_of(bool few) { return few ? 9 : 8; }
static_assert(1 << digit_bits_of(true) <= kSortThreads, "a thread per digit");

template <typename I>
__device__ __forceinline__ uint32_t key_of(I token, uint32_t rows) {
    return token >= 0 && (uint64_t)token < rows ? (uint32_t)token : rows;
}

// Sorted keys are plain uint32; the first pass reads the caller's tokens.
template <typename I, bool FIRST>
__device__ __forceinline__ uint32_t sort_key(const I *keys, int64_t i, uint32_t rows) {
    if constexpr (FIRST) return key_of(keys[i], rows);
    else return (uint32_t)keys[i];
}

// Zeros in every row of the gradient, 16 bytes per lane, 2^log_lanes lanes per row.
template <typename O>
__device__ __forceinline__ void zero_rows(O *__restrict__ g, int64_t rows, int width, int64_t ldg,
                                          int log_lanes, int64_t thread, int64_t threads) {
    constexpr int kEach = 16 / sizeof(O);
    const bool once = ldg % kEach == 0 || width * sizeof(O) >= 1024;   // (as rows_stored_once)
    for (int64_t r = thread >> log_lanes; r < rows; r += threads >> log_lanes) {
        O *const row = g + r * ldg;
        for (int c = (int)(thread & ((1 << log_lanes) - 1)) * kEach; c < width; c += kEach << log_lanes) {
            if (c + kEach <= width) {
                store_piece(row + c, u32x4{0, 0, 0, 0}, once);
            } else {
                for (int k = c; k < width; ++k) row[k] = (O)0.f;
            }
        }
    }
}

template <typename O>
__global__ __launch_bounds__(256) void zero_rows_kernel(O *__restrict__ g, int64_t rows, int width,
                                                        int64_t ldg, int log_lanes) {
    zero_rows(g, rows, width, ldg, log_lanes, (int64_t)blockIdx.x * 256 + threadIdx.x,
              (int64_t)gridDim.x * 256);
}

// FEW: at most kFewTiles tiles, whose counts lie as [tile][digit] and are summed by the
// workgroups that need them; else as [digit][tile], for digit_scan_kernel.  The first
// pass has more workgroups than tiles: the others write the gradient's zeros.
template <typename I, bool FIRST, bool FEW, typename O>
__global__ __launch_bounds__(kSortThreads) void digit_count_kernel(
    const I *__restrict__ keys, uint32_t n, uint32_t rows, int shift, int bits,
    uint32_t *__restrict__ counts, int tiles, O *__restrict__ g, int width, int64_t ldg,
    int log_lanes) {
    constexpr int kItems = FEW ? kSortFewItems : kSortItems;
    __shared__ uint32_t cnt[1 << digit_bits_of(FEW)];
    if constexpr (FIRST) {
        if ((int)blockIdx.x >= tiles) {
            zero_rows(g, rows, width, ldg, log_lanes,
                      (int64_t)(blockIdx.x - tiles) * kSortThreads + threadIdx.x,
                      (int64_t)(gridDim.x - tiles) * kSortThreads);
            return;
        }
    }
    const int digits = 1 << bits;
    for (int q = threadIdx.x; q < digits; q += kSortThreads) cnt[q] = 0;
    __syncthreads();
    const uint64_t first = (uint64_t)blockIdx.x * (kSortThreads * kItems);
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const uint64_t p = first + i * kSortThreads + threadIdx.x;
        if (p < n) atomicAdd(&cnt[sort_key<I, FIRST>(keys, p, rows) >> shift & (digits - 1)], 1u);
    }
    __syncthreads();
    for (int q = threadIdx.x; q < digits; q += kSortThreads)
        counts[FEW ? (int64_t)blockIdx.x * digits + q : (int64_t)q * tiles + blockIdx.x] = cnt[q];
}

// Exclusive scan over `n` values of a workgroup's threads, and their total.
template <int THREADS>
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t *wave_totals, uint32_t *total) {
    const int lane = threadIdx.x % kWaveLanes, wave = threadIdx.x / kWaveLanes;
    uint32_t inc = v;
#pragma unroll
    for (int s = 1; s < kWaveLanes; s <<= 1) {
        const uint32_t o = __shfl_up(inc, s);
        if (lane >= s) inc += o;
    }
    if (lane == kWaveLanes - 1) wave_totals[wave] = inc;
    __syncthreads();
    uint32_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < THREADS / kWaveLanes; ++w) {
        const uint32_t t = wave_totals[w];
        before += w < wave ? t : 0;
        all += t;
    }
    __syncthreads();
    *total = all;
    return before + inc - v;
}

// One workgroup per digit: counts[digit][tile] -> pairs of the digit in earlier
// tiles; totals[digit] -> all of them.
__global__ __launch_bounds__(256) void digit_scan_kernel(uint32_t *__restrict__ counts, int tiles,
                                                         uint32_t *__restrict__ totals) {
    __shared__ uint32_t wave_totals[4];
    uint32_t *const row = counts + (int64_t)blockIdx.x * tiles;
    uint32_t before = 0;
    for (int t0 = 0; t0 < tiles; t0 += 256) {
        const int t = t0 + threadIdx.x;
        const uint32_t v = t < tiles ? row[t] : 0;
        uint32_t total;
        const uint32_t ex = block_scan<256>(v, wave_totals, &total);
        if (t < tiles) row[t] = before + ex;
        before += total;
    }
    if (threadIdx.x == 0) totals[blockIdx.x] = before;
}

// The lanes that hold the same digit as this one (of the lanes that are live).
__device__ __forceinline__ uint64_t lanes_of_digit(uint32_t digit, int bits, bool live) {
    const uint64_t peers = __ballot(live);
    uint32_t lo = (uint32_t)peers, hi = (uint32_t)(peers >> 32);
    for (int b = 0; b < bits; ++b) {
        const uint32_t other = (digit >> b & 1) - 1;   // all ones where the bit is 0
        const uint64_t m = __ballot(other == 0);
        lo &= (uint32_t)m ^ other;
        hi &= (uint32_t)(m >> 32) ^ other;
    }
    return (uint64_t)hi << 32 | lo;
}

// Rank of this lane's pair among those of its digit that its wavefront has
// ranked, in order; `cnt` counts them per digit.  The lanes of a wavefront run
// in step and its LDS accesses stay in order; the atomics keep the compiler
// from holding a counter in a register.
__device__ __forceinline__ uint32_t rank_in_wave(uint32_t *cnt, uint32_t digit, int bits, bool live) {
    const uint64_t peers = lanes_of_digit(digit, bits, live);
    const int lane = threadIdx.x % kWaveLanes;
    const uint32_t lower = __popcll(peers & ((1ull << lane) - 1));
    uint32_t before = 0;
    if (live)
        before = __hip_atomic_load(&cnt[digit], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (live && lower == 0)
        __hip_atomic_store(&cnt[digit], before + (uint32_t)__popcll(peers), __ATOMIC_RELAXED,
                           __HIP_MEMORY_SCOPE_WORKGROUP);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    return before + lower;
}

// The pairs of a tile are put in order in LDS first, so that neighbouring lanes
// write neighbouring places (10M pairs of 128 digits: 43 us from the tokens, 35 from sorted
// keys; in tiles of twice the size 54, and 110 with every pair written from its register).
template <typename I, bool FIRST, bool FEW>
__global__ __launch_bounds__(kSortThreads) void digit_scatter_kernel(
    const I *__restrict__ keys, const uint32_t *__restrict__ index, uint32_t n, uint32_t rows,
    int shift, int bits, const uint32_t *__restrict__ counts, const uint32_t *__restrict__ totals,
    int tiles, uint32_t *__restrict__ keys_out, uint32_t *__restrict__ index_out) {
    constexpr int kMaxDigits = 1 << digit_bits_of(FEW);
    __shared__ uint32_t cnt[kSortWaves][kMaxDigits];
    __shared__ uint32_t wave_totals[kSortWaves];
    __shared__ uint32_t to_global[kMaxDigits];
    constexpr int kItems = FEW ? kSortFewItems : kSortItems;
    constexpr int kTile = kSortThreads * kItems;
    __shared__ uint32_t keys_tile[kTile], index_tile[kTile];
    const int digits = 1 << bits;
    const int lane = threadIdx.x % kWaveLanes, wave = threadIdx.x / kWaveLanes;
    for (int q = threadIdx.x; q < kSortWaves * kMaxDigits; q += kSortThreads) (&cnt[0][0])[q] = 0;
    const uint64_t tile = (uint64_t)blockIdx.x * kTile;
    const uint64_t first = tile + wave * (kItems * kWaveLanes) + lane;
    uint32_t key[kItems], pos[kItems], rank[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const uint64_t p = first + i * kWaveLanes;
        key[i] = p < n ? sort_key<I, FIRST>(keys, p, rows) : 0u;
        pos[i] = FIRST ? (uint32_t)p : p < n ? index[p] : 0u;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kItems; ++i)
        rank[i] = rank_in_wave(cnt[wave], key[i] >> shift & (digits - 1), bits,
                               first + i * kWaveLanes < n);
    // where the tile's pairs of a digit begin, in order everywhere and in the tile, and
    // in the tile those of each wavefront
    uint32_t total;
    const int dg = threadIdx.x;
    uint32_t everywhere = 0, earlier = 0;   // pairs of the digit, and those of earlier tiles
    if (dg < digits) {
        if constexpr (FEW) {
            constexpr int kAhead = 8;
            for (int t0 = 0; t0 < tiles; t0 += kAhead) {
                uint32_t c[kAhead];
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
                    c[u] = t0 + u < tiles ? counts[(int64_t)(t0 + u) * digits + dg] : 0u;
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    everywhere += c[u];
                    earlier += t0 + u < (int)blockIdx.x ? c[u] : 0u;
                }
            }
        } else {
            everywhere = totals[dg];
            earlier = counts[(int64_t)dg * tiles + blockIdx.x];
        }
    }
    const uint32_t start = block_scan<kSortThreads>(everywhere, wave_totals, &total);
    uint32_t here = 0;
    if (dg < digits) {
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) here += cnt[w][dg];
    }
    uint32_t at = block_scan<kSortThreads>(here, wave_totals, &total);
    if (dg < digits) {
        to_global[dg] = start + earlier - at;
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t c = cnt[w][dg];
            cnt[w][dg] = at;
            at += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kItems; ++i)
        if (first + i * kWaveLanes < n) {
            const uint32_t to = cnt[wave][key[i] >> shift & (digits - 1)] + rank[i];
            keys_tile[to] = key[i];
            index_tile[to] = pos[i];
        }
    __syncthreads();
    const uint32_t live = (uint32_t)std::min<uint64_t>(kTile, n - tile);
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const uint32_t q = i * kSortThreads + threadIdx.x;
        if (q < live) {
            const uint32_t k = keys_tile[q], to = q + to_global[k >> shift & (digits - 1)];
            keys_out[to] = k;
            index_out[to] = index_tile[q];
        }
    }
}

// Up to kSmallSort tokens: workgroup 0 sorts them, all digits in one launch, while
// the others write the gradient's zeros (16,384 tokens of 17 bits beside 268 MB: 52 us).
constexpr int kSmallThreads = 1024;
constexpr int kSmallItems = 16;
constexpr int kSmallWaves = kSmallThreads / kWaveLanes;
constexpr int kSmallSort = kSmallThreads * kSmallItems;
constexpr int kSmallDigitBits = 9;

template <typename I, typename O>
__global__ __launch_bounds__(kSmallThreads) void small_sort_kernel(
    const I *__restrict__ tokens, uint32_t n, uint32_t rows, int all_bits, int digit_bits,
    uint32_t *__restrict__ keys_out, uint32_t *__restrict__ index_out, O *__restrict__ g,
    int width, int64_t ldg, int log_lanes) {
    constexpr int kDigits = 1 << kSmallDigitBits;
    __shared__ uint32_t cnt[kSmallWaves][kDigits];
    __shared__ uint32_t wave_totals[kSmallWaves];
    __shared__ uint32_t keys_tile[kSmallSort];
    __shared__ uint16_t index_tile[kSmallSort];
    if (blockIdx.x > 0) {
        zero_rows(g, rows, width, ldg, log_lanes,
                  (int64_t)(blockIdx.x - 1) * kSmallThreads + threadIdx.x,
                  (int64_t)(gridDim.x - 1) * kSmallThreads);
        return;
    }
    const int lane = threadIdx.x % kWaveLanes, wave = threadIdx.x / kWaveLanes;
    // every wavefront takes as many tokens, in order
    const int items = (int)((n + kSmallThreads - 1) / kSmallThreads);
    const uint32_t first = wave * (items * kWaveLanes) + lane;
    uint32_t key[kSmallItems], pos[kSmallItems], rank[kSmallItems];
#pragma unroll
    for (int i = 0; i < kSmallItems; ++i) {
        pos[i] = first + i * kWaveLanes;
        key[i] = i < items && pos[i] < n ? key_of(tokens[pos[i]], rows) : 0u;
    }
    for (int shift = 0; shift < all_bits; shift += digit_bits) {
        const int bits = std::min(digit_bits, all_bits - shift);
        const int digits = 1 << bits;
        for (int q = threadIdx.x; q < kSmallWaves * kDigits; q += kSmallThreads) (&cnt[0][0])[q] = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kSmallItems; ++i) {
            if (i >= items) break;
            rank[i] = rank_in_wave(cnt[wave], key[i] >> shift & (digits - 1), bits,
                                   first + i * kWaveLanes < n);
        }
        __syncthreads();
        const int dg = threadIdx.x;
        uint32_t here = 0, total;
        if (dg < digits) {
#pragma unroll
            for (int w = 0; w < kSmallWaves; ++w) here += cnt[w][dg];
        }
        uint32_t at = block_scan<kSmallThreads>(here, wave_totals, &total);
        if (dg < digits) {
#pragma unroll
            for (int w = 0; w < kSmallWaves; ++w) {
                const uint32_t c = cnt[w][dg];
                cnt[w][dg] = at;
                at += c;
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kSmallItems; ++i)
            if (i < items && first + i * kWaveLanes < n) {
                const uint32_t to = cnt[wave][key[i] >> shift & (digits - 1)] + rank[i];
                keys_tile[to] = key[i];
                index_tile[to] = (uint16_t)pos[i];
            }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kSmallItems; ++i)
            if (i < items && first + i * kWaveLanes < n) {
                key[i] = keys_tile[first + i * kWaveLanes];
                pos[i] = index_tile[first + i * kWaveLanes];
            }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < kSmallItems; ++i)
        if (i < items && first + i * kWaveLanes < n) {
            keys_out[first + i * kWaveLanes] = key[i];
            index_out[first + i * kWaveLanes] = pos[i];
        }
}

// ---- sums of the rows of each token -------------------------------------------
// The sorted positions are cut into runs; a group of lanes walks a run and adds
// the rows of each token in order, in float32.  A token whose rows lie within
// one run is written to the table's gradient at once.  The others leave one sum
// per run they touch, entries (token, sum) in the same order, which the next
// level adds in the same way; a level of one run writes all.  The order of
// every sum follows from the tokens alone.
constexpr int kWalkThreads = 256;
constexpr int kWalkAhead = 8;                      // rows in flight per group of lanes
constexpr int kEntryRun = 16;                      // entries of a run, all in flight
constexpr int kEntryChunk = 4;                     // columns of an entry per lane
constexpr uint32_t kNoSum = 0x80000000u;           // an entry that holds no sum
constexpr uint32_t kNoKey = 0xffffffffu;
constexpr int kSliceLanes = kWaveLanes;            // a slice of columns: 64 lanes

// The first column of a lane's N.  The last lane of a row begins early enough to have N
// whole columns: some are then two lanes', which add and write the same.
template <int N>
__device__ __forceinline__ int column_of(int lane, int width) {
    const int c = lane * N;
    return c < width && width >= N ? std::min(c, width - N) : c;
}

template <int N, typename O>
__device__ __forceinline__ void store_values(O *p, int live, const float (&v)[N]) {
    if (live >= N) {
        O t[N];
#pragma unroll
        for (int k = 0; k < N; ++k) t[k] = (O)v[k];
        __builtin_memcpy(p, t, sizeof t);
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (k < live) p[k] = (O)v[k];
    }
}

// What a lane knows of the run that it walks: N columns from c on, of which the row has
// `live` (<= 0: the lane only keeps step).
template <int N, typename O>
struct Walk {
    O *grad;                        // of column c
    int64_t ldg;
    int live;
    float scale;
    uint32_t rows;
    uint32_t cur, head_key = kNoKey;
    bool any = false, head_any = false;   // the token has a row with a sum
    bool in_head = true;                  // no token but the run's first yet
    float acc[N] = {}, head[N] = {};

    __device__ __forceinline__ void store(uint32_t key, const float (&sum)[N]) {
        float v[N];
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = sum[k] * scale;
        if (live > 0) store_values(grad + (int64_t)key * ldg, live, v);
    }
    template <typename T>
    __device__ __forceinline__ void add(uint32_t key, const T (&v)[N]) {
        const uint32_t k0 = key & ~kNoSum;
        if (k0 != cur) {
            // (the first token's sum waits: earlier runs may have rows of it)
            if (in_head) {
#pragma unroll
                for (int k = 0; k < N; ++k) head[k] = acc[k];
                head_key = cur;
                head_any = any;
                in_head = false;
            } else if (any) {
                store(cur, acc);
            }
            cur = k0;
            any = false;
#pragma unroll
            for (int k = 0; k < N; ++k) acc[k] = 0.f;
        }
        if (key & kNoSum) return;
        add(v);
    }
    template <typename T>
    __device__ __forceinline__ void add(const T (&v)[N]) {
        any = true;
#pragma unroll
        for (int k = 0; k < N; ++k) acc[k] += (float)v[k];
    }
    // The first and the last token: written, or left to the next level, two entries at
    // up_sums (of column c) and up_keys, which one lane of a run writes (`keeper`).
    __device__ __forceinline__ void finish(uint32_t before, uint32_t after, uint32_t run, int width,
                                           uint32_t *up_keys, float *up_sums, bool keeper) {
        uint32_t left[2];
        auto settle = [&](int slot, uint32_t key, const float (&sum)[N], bool has, bool shared)
                          __attribute__((always_inline)) {
            left[slot] = key | kNoSum;
            if (key >= rows || !has) return;
            if (!shared) {
                store(key, sum);
            } else {
                left[slot] = key;
                if (live > 0) store_values(up_sums + (int64_t)(2 * run + slot) * width, live, sum);
            }
        };
        if (in_head) {
            settle(0, cur, acc, any, before == cur || after == cur);
            left[1] = cur | kNoSum;
        } else {
            settle(0, head_key, head, head_any, before == head_key);
            settle(1, cur, acc, any, after == cur);
        }
        if (keeper) {
            up_keys[2 * (uint64_t)run] = left[0];
            up_keys[2 * (uint64_t)run + 1] = left[1];
        }
    }
};

// The rows of dout, which `index` names in the order of their tokens: they are read once,
// which bounds it (10M rows of 64 bfloat16 values: 250 us, 5.3 TB/s; 16,384 of 1024 20).
template <typename T, typename O>
__global__ __launch_bounds__(kWalkThreads) void walk_rows_kernel(
    const uint32_t *__restrict__ keys, const uint32_t *__restrict__ index, uint32_t n,
    const T *__restrict__ x, int64_t ldx, int width, float scale, uint32_t rows,
    O *__restrict__ grad, int64_t ldg, uint32_t *__restrict__ up_keys, float *__restrict__ up_sums,
    int log_lanes, int run_length) {
    const int lane = threadIdx.x & ((1 << log_lanes) - 1);
    const uint32_t run = (blockIdx.x * (uint32_t)kWalkThreads + threadIdx.x) >> log_lanes;
    const uint64_t begin = (uint64_t)run * run_length;
    if (begin >= n) return;
    const uint32_t a = (uint32_t)begin, b = (uint32_t)std::min<uint64_t>(n, begin + run_length);
    const int c = column_of<kChunk>(blockIdx.y * kSliceLanes + lane, width);
    Walk<kChunk, O> w = {grad + c, ldg, width - c, scale, rows, keys[a]};
    const uint32_t before = a > 0 ? keys[a - 1] : kNoKey, after = b < n ? keys[b] : kNoKey;
    // (the next rows' places are read ahead of their use)
    uint32_t next[kWalkAhead];
    auto places = [&](uint32_t p) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kWalkAhead; ++u) next[u] = index[std::min(p + u, b - 1)];
    };
    places(a);
    uint32_t p = a;
    for (; p + kWalkAhead <= b && w.cur < rows; p += kWalkAhead) {
        RawChunk<T> v[kWalkAhead];
        const uint32_t last = keys[p + kWalkAhead - 1];
#pragma unroll
        for (int u = 0; u < kWalkAhead; ++u) v[u] = load_raw_once(x + (int64_t)next[u] * ldx + c, w.live);
        places(p + kWalkAhead);
        if (last == w.cur) {       // keys ascend: all of these rows are the current token's
#pragma unroll
            for (int u = 0; u < kWalkAhead; ++u) w.add(v[u].v);
            continue;
        }
        uint32_t key[kWalkAhead];
#pragma unroll
        for (int u = 0; u < kWalkAhead; ++u) key[u] = keys[p + u];
#pragma unroll
        for (int u = 0; u < kWalkAhead; ++u) w.add(key[u], v[u].v);
    }
    // (masked tokens are last: from the first of them on, the rest of the run is theirs)
    for (; p < b && w.cur < rows; ++p)
        w.add(keys[p], load_raw_once(x + (int64_t)index[p] * ldx + c, w.live).v);
    w.finish(before, after, run, width, up_keys, up_sums + c,
             up_keys && blockIdx.y == 0 && lane == 0);
}

// Entries of the level before.  A level of a call on few tokens takes as long as its reads,
// one after another, and its instructions: a run's entries are read at once and lie in
// LDS, where a loop finds them by number (16,384 tokens x 1024: 6.4 us a level; read 8 at a
// time 8.8; all 16 in a row of code, 18 KB of it, 7 to 12).
struct EntryStage {
    f32x4 values[kEntryRun][kWalkThreads];
    uint32_t keys[kEntryRun][kWalkThreads];
};

template <typename O>
__device__ __forceinline__ void walk_entries(EntryStage &stage, const uint32_t *keys, uint32_t n,
                                             const float *x, int width, float scale, uint32_t rows,
                                             O *grad, int64_t ldg, uint32_t *up_keys, float *up_sums,
                                             uint32_t run, int c, bool keeper) {
    const uint64_t begin = (uint64_t)run * kEntryRun;
    if (begin >= n) return;
    const uint32_t a = (uint32_t)begin, b = (uint32_t)std::min<uint64_t>(n, begin + kEntryRun);
    const int live = width - c;
    // (beyond the run the last entry again; what an entry without a sum holds is not used)
    uint32_t key[kEntryRun];
    f32x4 v[kEntryRun];
#pragma unroll
    for (int u = 0; u < kEntryRun; ++u) {
        const uint32_t p = std::min(a + u, b - 1);
        key[u] = keys[p];
        const float *from = x + (int64_t)p * width + c;
        if (live >= kEntryChunk) {
            __builtin_memcpy(&v[u], from, sizeof v[u]);
        } else {
#pragma unroll
            for (int k = 0; k < kEntryChunk; ++k) v[u][k] = k < live ? from[k] : 0.f;
        }
    }
    const uint32_t before = a > 0 ? keys[a - 1] & ~kNoSum : kNoKey;
    const uint32_t after = b < n ? keys[b] & ~kNoSum : kNoKey;
    Walk<kEntryChunk, O> w = {grad + c, ldg, live, scale, rows, key[0] & ~kNoSum};
#pragma unroll
    for (int u = 0; u < kEntryRun; ++u) {
        stage.keys[u][threadIdx.x] = key[u];
        stage.values[u][threadIdx.x] = v[u];
    }
    const int count = (int)(b - a);
    f32x4 t = v[0];
    uint32_t k = key[0];
#pragma unroll 1
    for (int u = 1; u <= count; ++u) {
        const int ahead = std::min(u, kEntryRun - 1);
        const f32x4 t_next = stage.values[ahead][threadIdx.x];
        const uint32_t k_next = stage.keys[ahead][threadIdx.x];
        const float e[kEntryChunk] = {t[0], t[1], t[2], t[3]};
        w.add(k, e);
        t = t_next, k = k_next;
    }
    w.finish(before, after, run, width, up_keys, up_sums + c, keeper);
}

template <typename O>
__global__ __launch_bounds__(kWalkThreads) void walk_entries_kernel(
    const uint32_t *__restrict__ keys, uint32_t n, const float *__restrict__ x, int width, float scale,
    uint32_t rows, O *__restrict__ grad, int64_t ldg, uint32_t *__restrict__ up_keys,
    float *__restrict__ up_sums, int log_lanes) {
    __shared__ EntryStage stage;
    const int lane = threadIdx.x & ((1 << log_lanes) - 1);
    const uint32_t run = (blockIdx.x * (uint32_t)kWalkThreads + threadIdx.x) >> log_lanes;
    walk_entries(stage, keys, n, x, width, scale, rows, grad, ldg, up_keys, up_sums, run,
                 column_of<kEntryChunk>(blockIdx.y * kSliceLanes + lane, width),
                 up_keys && blockIdx.y == 0 && lane == 0);
}

// The last levels, from the first that a workgroup per slice of columns can hold at
// once, in one launch, with the levels' keys in LDS (65,536 tokens x 64: 52 us in all, a
// launch for each 54, and fewer launches for the host to make).
constexpr int kTailEntries = kWalkThreads * kEntryRun;
constexpr int kTailLevels = 6;

struct Tail {
    const uint32_t *keys;              // of the first level
    float *sums[kTailLevels];
    uint32_t entries[kTailLevels];
    int levels;
};

template <typename O>
__global__ __launch_bounds__(kWalkThreads) void walk_tail_kernel(Tail t, int width, float scale,
                                                                 uint32_t rows, O *__restrict__ grad,
                                                                 int64_t ldg, int log_lanes) {
    __shared__ EntryStage stage;
    __shared__ uint32_t even_keys[kTailEntries], odd_keys[2 * kTailEntries / kEntryRun];
    for (uint32_t q = threadIdx.x; q < t.entries[0]; q += kWalkThreads) even_keys[q] = t.keys[q];
    __syncthreads();
    const int lane = threadIdx.x & ((1 << log_lanes) - 1);
    const int c = column_of<kEntryChunk>(blockIdx.x * kSliceLanes + lane, width);
#pragma unroll 1
    for (int l = 0; l < t.levels; ++l) {
        const bool up = l + 1 < t.levels;
        const uint32_t runs = (t.entries[l] + kEntryRun - 1) / kEntryRun;
#pragma unroll 1
        for (uint32_t run = threadIdx.x >> log_lanes; run < runs; run += kWalkThreads >> log_lanes)
            walk_entries(stage, l % 2 ? odd_keys : even_keys, t.entries[l], t.sums[l], width, scale, rows,
                         grad, ldg, l % 2 ? even_keys : odd_keys, up ? t.sums[l + 1] : t.sums[l], run, c,
                         up && lane == 0);
        __syncthreads();
    }
}

// Lanes that share a row of `width` elements, `each` per lane at a time: a power of
// two up to a wavefront.
int log_lanes_of(int width, int each) {
    const int chunks = (width + each - 1) / each;
    int l = 0;
    while (l < 6 && (1 << l) < chunks) ++l;
    return l;
}

int64_t round256(int64_t v) { return (v + 255) & ~(int64_t)255; }

// The workspace of a gradient: two lists of (key, position), the digits' counts,
// and the entries of every level of sums.
struct GradPlan {
    bool few;                                      // tiles
    int64_t tiles, bits, passes, digit_bits;
    int64_t keys[2], index[2], counts, totals;     // byte offsets
    int run;                                       // positions of a run
    int levels;                                    // levels that leave entries
    int64_t entries[16], up_keys[16], up_sums[16];
    int64_t bytes;
};

GradPlan plan_grad(int64_t n, int64_t rows, int width) {
    GradPlan p = {};
    p.tiles = ceil_div(n, kSortThreads * kSortFewItems);
    p.few = p.tiles <= kFewTiles;
    if (!p.few) p.tiles = ceil_div(n, kSortThreads * kSortItems);
    p.bits = 1;
    while ((int64_t)1 << p.bits <= rows) ++p.bits;   // keys 0 .. rows
    p.passes = ceil_div(p.bits, digit_bits_of(p.few));
    p.digit_bits = ceil_div(p.bits, p.passes);
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t o = at;
        at += round256(bytes);
        return o;
    };
    for (int k = 0; k < 2; ++k) {
        p.keys[k] = take(4 * n);
        p.index[k] = take(4 * n);
    }
    p.counts = take(4 * ((int64_t)1 << p.digit_bits) * p.tiles);
    p.totals = take(4 << p.digit_bits);
    // Runs of 256 positions, shorter where that leaves too few wavefronts (8 for each of
    // 256 CUs), and of 16 entries: a level has at most a quarter of what is before it.
    // (10M x 64 of 5120 tokens: 418 us in all, with runs of 64 or 512 455 and 428; 3M x 64:
    // runs of 128, 162 us, of 64 or 256 166 and 167; 16,384 x 1024: 16, 94, of 64 100.)
    int first = 256;
    while (first > 8 && ceil_div(n, first) * ceil_div(width, kChunk) < 8 * 256 * kWaveLanes) first /= 2;
    p.run = first;
    for (int64_t m = n, run = first; m > run; run = kEntryRun) {
        const int64_t e = 2 * ceil_div(m, run);
        p.entries[p.levels] = e;
        p.up_keys[p.levels] = take(4 * e);
        p.up_sums[p.levels] = take(4 * e * width);
        ++p.levels;
        m = e;
    }
    p.bytes = at;
    return p;
}

template <bool FEW, typename I, typename O>
hipError_t sort_tokens(const GradPlan &p, const I *tokens, uint32_t n, uint32_t rows, char *work,
                       int *sorted, O *grad, int width, int64_t ldg, int zero_lanes, unsigned zero_groups,
                       hipStream_t s) {
    uint32_t *const counts = reinterpret_cast<uint32_t *>(work + p.counts);
    uint32_t *const totals = reinterpret_cast<uint32_t *>(work + p.totals);
    const int tiles = (int)p.tiles;
    int from = 1;
    for (int pass = 0; pass < p.passes; ++pass) {
        const int shift = pass * (int)p.digit_bits;
        const int bits = std::min((int)p.digit_bits, (int)p.bits - shift);
        const uint32_t *kin = reinterpret_cast<uint32_t *>(work + p.keys[from]);
        const uint32_t *iin = reinterpret_cast<uint32_t *>(work + p.index[from]);
        uint32_t *kout = reinterpret_cast<uint32_t *>(work + p.keys[from ^ 1]);
        uint32_t *iout = reinterpret_cast<uint32_t *>(work + p.index[from ^ 1]);
        if (pass == 0)
            digit_count_kernel<I, true, FEW><<<tiles + zero_groups, kSortThreads, 0, s>>>(
                tokens, n, rows, shift, bits, counts, tiles, grad, width, ldg, zero_lanes);
        else
            digit_count_kernel<uint32_t, false, FEW, float><<<tiles, kSortThreads, 0, s>>>(
                kin, n, rows, shift, bits, counts, tiles, nullptr, 0, 0, 0);
        if (!FEW) digit_scan_kernel<<<1 << bits, 256, 0, s>>>(counts, tiles, totals);
        if (pass == 0)
            digit_scatter_kernel<I, true, FEW><<<tiles, kSortThreads, 0, s>>>(
                tokens, nullptr, n, rows, shift, bits, counts, totals, tiles, kout, iout);
        else
            digit_scatter_kernel<uint32_t, false, FEW><<<tiles, kSortThreads, 0, s>>>(
                kin, iin, n, rows, shift, bits, counts, totals, tiles, kout, iout);
        from ^= 1;
    }
    *sorted = from;
    return hipGetLastError();
}

template <typename T, typename O>
hipError_t table_gradient(const GradPlan &p, const void *tokens, int token_bytes, int64_t n,
                          const T *dout, int64_t ldd, float scale, O *grad, int64_t rows, int width,
                          int64_t ldg, char *work, int cus, hipStream_t s) {
    const int zero_lanes = log_lanes_of(width, 16 / sizeof(O));
    const int64_t zero_threads = rows << zero_lanes;
    hipError_t e = hipSuccess;
    int at = 0;
    // One workgroup sorts few tokens faster than a launch per step (4000: 33 and 38 us in
    // all; 8000: 40 and 40; 16,000: 52 and 43), and up to kSmallSort of them if the
    // zeros beside it take as long (10,000 tokens and 34 MB of zeros, 50 and 49; 67 MB, 50 and
    // 55; 134 MB, 57 and 71; 268 MB, 93 and 104; 16,384 and 67 MB, 61 and 57; 134 MB, 73 and
    // 75; 268 MB, 99 and 111; 537 MB, 157 and 163).
    const bool small = n <= kSmallSort / 2 ||
                       (n <= kSmallSort && rows * width * (int64_t)sizeof(O) >= (int64_t)1 << 27);
    if (n > 0 && small) {
        const unsigned grid =
            1 + (unsigned)std::min<int64_t>(ceil_div(zero_threads, kSmallThreads), 8 * (int64_t)cus);
        auto sort = [&](auto *t) {
            small_sort_kernel<<<grid, kSmallThreads, 0, s>>>(
                t, (uint32_t)n, (uint32_t)rows, (int)p.bits,
                (int)ceil_div(p.bits, ceil_div(p.bits, kSmallDigitBits)),
                reinterpret_cast<uint32_t *>(work + p.keys[0]),
                reinterpret_cast<uint32_t *>(work + p.index[0]), grad, width, ldg, zero_lanes);
            return hipGetLastError();
        };
        e = token_bytes == 8 ? sort(static_cast<const int64_t *>(tokens))
                             : sort(static_cast<const int32_t *>(tokens));
    } else if (n == 0) {
        zero_rows_kernel<O><<<(unsigned)std::min<int64_t>(ceil_div(zero_threads, 256), 32 * (int64_t)cus),
                              256, 0, s>>>(grad, rows, width, ldg, zero_lanes);
        return hipGetLastError();
    } else {
        const unsigned zero_groups =
            (unsigned)std::min<int64_t>(ceil_div(zero_threads, kSortThreads), 16 * (int64_t)cus);
        auto sort = [&](auto *t) {
            return p.few ? sort_tokens<true>(p, t, (uint32_t)n, (uint32_t)rows, work, &at, grad, width, ldg,
                                             zero_lanes, zero_groups, s)
                         : sort_tokens<false>(p, t, (uint32_t)n, (uint32_t)rows, work, &at, grad, width, ldg,
                                              zero_lanes, zero_groups, s);
        };
        e = token_bytes == 8 ? sort(static_cast<const int64_t *>(tokens))
                             : sort(static_cast<const int32_t *>(tokens));
    }
    if (e != hipSuccess) return e;
    auto keys_at = [&](int64_t o) { return reinterpret_cast<uint32_t *>(work + o); };
    auto sums_at = [&](int64_t o) { return reinterpret_cast<float *>(work + o); };
    auto blocks = [&](int64_t runs, int log_lanes, int each) {
        return dim3((unsigned)ceil_div(runs << log_lanes, kWalkThreads),
                    (unsigned)ceil_div(width, kSliceLanes * each));
    };
    const bool more = p.levels > 0;
    int ll = log_lanes_of(width, kChunk);
    walk_rows_kernel<T, O><<<blocks(ceil_div(n, p.run), ll, kChunk), kWalkThreads, 0, s>>>(
        keys_at(p.keys[at]), keys_at(p.index[at]), (uint32_t)n, dout, ldd, width, scale, (uint32_t)rows,
        grad, ldg, more ? keys_at(p.up_keys[0]) : nullptr, more ? sums_at(p.up_sums[0]) : nullptr, ll, p.run);
    ll = log_lanes_of(width, kEntryChunk);
    for (int l = 0; l < p.levels; ++l) {
        if ((e = hipGetLastError()) != hipSuccess) return e;
        const bool up = l + 1 < p.levels;
        if (up && p.entries[l] <= kTailEntries >> ll) {
            Tail t = {keys_at(p.up_keys[l]), {}, {}, p.levels - l};
            for (int k = l; k < p.levels; ++k) {
                t.sums[k - l] = sums_at(p.up_sums[k]);
                t.entries[k - l] = (uint32_t)p.entries[k];
            }
            walk_tail_kernel<O><<<blocks(0, ll, kEntryChunk).y, kWalkThreads, 0, s>>>(
                t, width, scale, (uint32_t)rows, grad, ldg, ll);
            break;
        }
        walk_entries_kernel<O><<<blocks(ceil_div(p.entries[l], kEntryRun), ll, kEntryChunk), kWalkThreads, 0,
                                 s>>>(keys_at(p.up_keys[l]), (uint32_t)p.entries[l], sums_at(p.up_sums[l]),
                                      width, scale, (uint32_t)rows, grad, ldg,
                                      up ? keys_at(p.up_keys[l + 1]) : nullptr,
                                      up ? sums_at(p.up_sums[l + 1]) : nullptr, ll);
    }
    return hipGetLastError();
}

int check_tokens(const void *tokens, int32_t token_bytes, int64_t n) {
    if (token_bytes != 4 && token_bytes != 8)
        return report(FBDT_E_INVAL, "token_bytes = %d must be 4 or 8", token_bytes);
    if (n < 0 || n >= (int64_t)1 << 31)
        return report(FBDT_E_INVAL, "n = %lld must be in [0, 2^31)", (long long)n);
    if (n > 0 && !tokens) return report(FBDT_E_INVAL, "tokens is NULL");
    if (n > 0 && !aligned_to(tokens, token_bytes))
        return report(FBDT_E_INVAL, "tokens must be aligned to its elements");
    return FBDT_OK;
}

int check_matrix(const char *name, const void *p, int32_t dtype, int64_t ld, int32_t width) {
    if (!known_dtype(dtype)) return report(FBDT_E_INVAL, "%s: unknown type %d", name, dtype);
    if (!p) return report(FBDT_E_INVAL, "%s is NULL", name);
    if (!aligned_to(p, dtype_bytes(dtype)))
        return report(FBDT_E_INVAL, "%s must be aligned to its elements", name);
    if (ld < width)
        return report(FBDT_E_INVAL, "%s: row stride %lld is below the width %d", name, (long long)ld,
                      width);
    return FBDT_OK;
}

int check_table(int64_t rows, int32_t width) {
    if (rows < 1 || rows >= (int64_t)1 << 31)
        return report(FBDT_E_INVAL, "rows = %lld must be in [1, 2^31)", (long long)rows);
    if (width < 1 || width > 1 << 20)
        return report(FBDT_E_INVAL, "width = %d must be in [1, 2^20]", width);
    return FBDT_OK;
}

}  // namespace
}  // namespace fbdt

using namespace fbdt;

extern "C" {

int fbdt_event_tokens(const uint8_t *xb, int64_t n, int32_t d, int64_t ldb, int32_t n_bins,
                      int32_t *tokens, void *stream) {
    if (n < 0 || n > (int64_t)1 << 36)
        return report(FBDT_E_INVAL, "n = %lld must be in [0, 2^36]", (long long)n);
    if (d < 1 || d > 255) return report(FBDT_E_INVAL, "d = %d must be in [1, 255]", d);
    if (n_bins < 2 || n_bins > 256)
        return report(FBDT_E_INVAL, "n_bins = %d must be in [2, 256]", n_bins);
    if (ldb < n || ldb % 16 != 0)
        return report(FBDT_E_INVAL, "ldb = %lld must be a multiple of 16 and >= n = %lld",
                      (long long)ldb, (long long)n);
    if (n == 0) return FBDT_OK;
    if (!xb || !aligned_to(xb, 16)) return report(FBDT_E_INVAL, "xb must be 16-byte aligned");
    if (!tokens || !aligned_to(tokens, 4)) return report(FBDT_E_INVAL, "tokens must be 4-byte aligned");
    int rc;
    if ((rc = check_apart("tokens", {tokens, 1, n * d, 0, 4}, "xb", {xb, d, n, ldb, 1}))) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    event_tokens_kernel<<<grid_of(ceil_div(n, kTokenEvents), kTokenThreads), kTokenThreads,
                          d * kTokenEvents, s>>>(
        xb, n, d, ldb, n_bins, tokens);
    NET_TRY(hipGetLastError());
    return FBDT_OK;
}

int fbdt_embed(const void *table, int32_t dtype, int64_t rows, int32_t width, int64_t ldt,
               const void *tokens, int32_t token_bytes, int64_t n, float scale, void *out,
               int64_t ldo, void *stream) {
    int rc;
    if ((rc = check_table(rows, width)) || (rc = check_tokens(tokens, token_bytes, n))) return rc;
    if ((rc = check_matrix("table", table, dtype, ldt, width))) return rc;
    if (n == 0) return FBDT_OK;
    if ((rc = check_matrix("out", out, dtype, ldo, width))) return rc;
    const int64_t size = dtype_bytes(dtype);
    const Extent result = {out, n, width, ldo, size};
    if ((rc = check_apart("out", result, "table", {table, rows, width, ldt, size})) ||
        (rc = check_apart("out", result, "tokens", {tokens, 1, n, 0, token_bytes})))
        return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    NET_TRY(with_dtype(dtype, [&](auto t) {
        typedef decltype(t) T;
        const int ll = log_lanes_of(width, 16 / sizeof(T));
        constexpr int kEach = 16 / sizeof(T);
        // (2.3M rows of 100 values of 16 bits: 117 us, a lane per piece of a row 213)
        const bool flat = ldo == width && width >= kEach && width % kEach != 0 && aligned_to(out, 16);
        const dim3 grid = flat ? grid_of(ceil_div(n * width, kLookupThreads * kEach), kLookupThreads)
                               : grid_of(ceil_div(n, kLookupThreads >> ll), kLookupThreads);
        auto go = [&](auto once, auto *t) {
            typedef std::remove_const_t<std::remove_reference_t<decltype(*t)>> I;
            if (flat)
                lookup_flat_kernel<T, I><<<grid, kLookupThreads, 0, s>>>(
                    static_cast<const T *>(table), (uint32_t)rows, width, 1.0 / width, ldt, t, n, scale,
                    static_cast<T *>(out));
            else lookup_kernel<T, I, decltype(once)::value><<<grid, kLookupThreads, 0, s>>>(
                static_cast<const T *>(table), (uint32_t)rows, width, ldt, t, n, scale,
                static_cast<T *>(out), ldo, ll);
        };
        auto with_tokens = [&](auto once) {
            if (token_bytes == 8) go(once, static_cast<const int64_t *>(tokens));
            else go(once, static_cast<const int32_t *>(tokens));
        };
        if (flat || rows_stored_once(out, ldo * sizeof(T), width * sizeof(T))) with_tokens(std::true_type{});
        else with_tokens(std::false_type{});
        return hipGetLastError();
    }));
    return FBDT_OK;
}

int64_t fbdt_embed_grad_work(int64_t n, int64_t rows, int32_t width) {
    if (n < 0 || n >= (int64_t)1 << 31 || check_table(rows, width)) return -1;
    return plan_grad(n, rows, width).bytes;
}

int fbdt_embed_grad(const void *tokens, int32_t token_bytes, int64_t n, const void *dout,
                    int32_t dtype, int64_t ldd, float scale, void *dtable, int32_t grad_dtype,
                    int64_t rows, int32_t width, int64_t ldg, void *work, int64_t work_bytes,
                    void *stream) {
    int rc;
    if ((rc = check_table(rows, width)) || (rc = check_tokens(tokens, token_bytes, n))) return rc;
    if (n > 0 && (rc = check_matrix("dout", dout, dtype, ldd, width))) return rc;
    if ((rc = check_matrix("dtable", dtable, grad_dtype, ldg, width))) return rc;
    if (!known_dtype(dtype)) return report(FBDT_E_INVAL, "dout: unknown type %d", dtype);
    if (grad_dtype != FBDT_F32 && grad_dtype != dtype)
        return report(FBDT_E_INVAL, "dtable must be float32 or of dout's type");
    const GradPlan p = plan_grad(n, rows, width);
    if (work_bytes < p.bytes || (p.bytes > 0 && (!work || !aligned_to(work, 256))))
        return report(FBDT_E_INVAL, "work must hold %lld bytes, 256-byte aligned",
                      (long long)p.bytes);
    const Extent result = {dtable, rows, width, ldg, dtype_bytes(grad_dtype)};
    if ((rc = check_apart("dtable", result, "dout", {dout, n, width, ldd, dtype_bytes(dtype)})) ||
        (rc = check_apart("dtable", result, "tokens", {tokens, 1, n, 0, token_bytes})))
        return rc;
    int cus = 0;
    if ((rc = device_cus(&cus))) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    char *const w = static_cast<char *>(work);
    NET_TRY(with_dtype(dtype, [&](auto t) {
        typedef decltype(t) T;
        const T *const x = static_cast<const T *>(dout);
        if (grad_dtype == FBDT_F32)
            return table_gradient(p, tokens, token_bytes, n, x, ldd, scale,
                                  static_cast<float *>(dtable), rows, width, ldg, w, cus, s);
        return table_gradient(p, tokens, token_bytes, n, x, ldd, scale, static_cast<T *>(dtable),
                              rows, width, ldg, w, cus, s);
    }));
    return FBDT_OK;
}

}  // extern "C"
