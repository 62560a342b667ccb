// Row operators: root-mean-square norm with the residual's addition and its
// gradient, and rows packed in 8 bits with scales.
#include "network.h"

#include <algorithm>

namespace fbdt {
namespace {

constexpr int kRowThreads = 256;

// Where a norm's rows are and where its results go; null: not there, not asked.
struct NormArgs {
    const void *x, *residual;
    int64_t n, ldx, ldr;
    int width;
    const float *gain;
    float eps;
    void *h, *y;
    int64_t ldh, ldy;
    uint8_t *codes, *scales;
    int64_t ldc, lds;
    float *rstd;
    bool h_once, y_once;
};

// Sum over the LANES lanes of a row (up to 64: of a wavefront; more: the whole
// workgroup, through `part`, of which a call uses the half that `turn` names).
template <int LANES>
__device__ __forceinline__ float row_sum(float v, float (*part)[16], int turn) {
#pragma unroll
    for (int s = 1; s < LANES && s < kWaveLanes; s <<= 1) v += __shfl_xor(v, s);
    if constexpr (LANES > kWaveLanes) {
        if (threadIdx.x % kWaveLanes == 0) part[turn][threadIdx.x / kWaveLanes] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int w = 0; w < LANES / kWaveLanes; ++w) v += part[turn][w];
    }
    return v;
}

// The outputs of one piece of a normed row.
template <typename T>
__device__ __forceinline__ void store_normed(const NormArgs &p, int64_t row, int c, int live,
                                             const float (&y)[kPiece<T>]) {
    if (p.y && live > 0) store_floats(static_cast<T *>(p.y) + row * p.ldy + c, live, y, p.y_once);
    if (p.codes) {
        uint8_t e;
        const Codes<kPiece<T>> q = pack_values(y, &e);
        // codes and scales end with the last block that the width reaches
        if (c < (p.width + kPackBlock - 1) / kPackBlock * kPackBlock) {
            *reinterpret_cast<Codes<kPiece<T>> *>(p.codes + row * p.ldc + c) = q;
            if (c % kPackBlock == 0) p.scales[row * p.lds + c / kPackBlock] = e;
        }
    }
}

// One row per LANES lanes, P pieces of 16 bytes per lane: the row is
// read once and stays in registers as the float32 sum h; the gain stays in registers
// from row to row.  Memory bounds it: float rows are loaded and stored past the
// cache, packed rows are not (65,536 x 2560 bf16, residual, packed result: 186 to 199
// us, 5.9 TB/s; float rows through the cache 290, packed rows past it 212).
template <typename T, int LANES, int P>
__global__ __launch_bounds__(LANES < kRowThreads ? kRowThreads : LANES) void norm_kernel(NormArgs p) {
    __shared__ float part[2][16];
    constexpr int kThreads = LANES < kRowThreads ? kRowThreads : LANES;
    constexpr int kRows = kThreads / LANES;
    constexpr int E = kPiece<T>;
    const int lane = threadIdx.x % LANES;
    float gain[P][E];
#pragma unroll
    for (int r = 0; r < P; ++r) {
        const int c = (lane + r * LANES) * E;
        load_floats(p.gain + c, p.width - c, gain[r]);
    }
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES; row < p.n;
         row += (int64_t)gridDim.x * kRows, turn ^= 1) {
        float h[P][E];
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < P; ++r) {
            const int c = (lane + r * LANES) * E;
            load_floats_once(static_cast<const T *>(p.x) + row * p.ldx + c, p.width - c, h[r]);
        }
        if (p.residual) {
#pragma unroll
            for (int r = 0; r < P; ++r) {
                const int c = (lane + r * LANES) * E;
                float t[E];
                load_floats_once(static_cast<const T *>(p.residual) + row * p.ldr + c, p.width - c, t);
#pragma unroll
                for (int k = 0; k < E; ++k) h[r][k] += t[k];
            }
        }
#pragma unroll
        for (int r = 0; r < P; ++r)
#pragma unroll
            for (int k = 0; k < E; ++k) sum = __builtin_fmaf(h[r][k], h[r][k], sum);
        sum = row_sum<LANES>(sum, part, turn);
        const float rstd = 1.f / __builtin_sqrtf(sum / (float)p.width + p.eps);
        if (p.rstd && lane == 0) p.rstd[row] = rstd;
#pragma unroll
        for (int r = 0; r < P; ++r) {
            const int c = (lane + r * LANES) * E;
            if (p.h && c < p.width)
                store_floats(static_cast<T *>(p.h) + row * p.ldh + c, p.width - c, h[r], p.h_once);
            float y[E];
#pragma unroll
            for (int k = 0; k < E; ++k) y[k] = h[r][k] * rstd * gain[r][k];
            store_normed<T>(p, row, c, p.width - c, y);
        }
    }
}

// Rows too wide for registers: read twice.
template <typename T>
__global__ __launch_bounds__(1024) void norm_wide_kernel(NormArgs p) {
    __shared__ float part[2][16];
    constexpr int E = kPiece<T>;
    int turn = 0;
    // (whole blocks of columns, so that the lanes of a packed block stay together)
    const int span = (p.width + kPackBlock - 1) / kPackBlock * kPackBlock;
    for (int64_t row = blockIdx.x; row < p.n; row += gridDim.x, turn ^= 1) {
        auto sum_of = [&](int c, float (&h)[E]) {
            load_floats_once(static_cast<const T *>(p.x) + row * p.ldx + c, p.width - c, h);
            if (p.residual) {
                float t[E];
                load_floats_once(static_cast<const T *>(p.residual) + row * p.ldr + c, p.width - c, t);
#pragma unroll
                for (int k = 0; k < E; ++k) h[k] += t[k];
            }
        };
        float sum = 0.f;
        for (int c = threadIdx.x * E; c < p.width; c += 1024 * E) {
            float h[E];
            sum_of(c, h);
#pragma unroll
            for (int k = 0; k < E; ++k) sum = __builtin_fmaf(h[k], h[k], sum);
        }
        sum = row_sum<1024>(sum, part, turn);
        const float rstd = 1.f / __builtin_sqrtf(sum / (float)p.width + p.eps);
        if (p.rstd && threadIdx.x == 0) p.rstd[row] = rstd;
        for (int c = threadIdx.x * E; c < span; c += 1024 * E) {
            float h[E], g[E], y[E];
            sum_of(c, h);
            load_floats(p.gain + c, p.width - c, g);
            if (p.h && c < p.width)
                store_floats(static_cast<T *>(p.h) + row * p.ldh + c, p.width - c, h, p.h_once);
#pragma unroll
            for (int k = 0; k < E; ++k) y[k] = h[k] * rstd * g[k];
            store_normed<T>(p, row, c, p.width - c, y);
        }
    }
}

struct NormGradArgs {
    const void *dy, *h, *dh;
    int64_t n, lddy, ldh, lddh;
    int width;
    const float *gain, *rstd;
    void *dx;
    int64_t lddx;
    float *partial;       // [workgroups or row groups][width]: sums of dy xh
    float *coefficient;   // [n], rows too wide for registers: mean(a xh)
    bool once;
};

// One row per LANES lanes as in norm_kernel; each lane adds its columns of the
// gain's gradient over the rows it meets.  (65,536 x 2560 bf16 with dh: 241 us, 5.6
// TB/s, through the cache 374; 20,001 x 1001 float32 with the columns' sums: 66 us, in
// pieces of 32 bytes through the cache 74.)
template <typename T, int LANES, int P>
__global__ __launch_bounds__(LANES < kRowThreads ? kRowThreads : LANES) void norm_grad_kernel(
    NormGradArgs p) {
    constexpr int kThreads = LANES < kRowThreads ? kRowThreads : LANES;
    constexpr int kRows = kThreads / LANES;
    constexpr int E = kPiece<T>;
    __shared__ float part[2][16];
    const int lane = threadIdx.x % LANES;
    float gain[P][E], dgain[P][E];
#pragma unroll
    for (int r = 0; r < P; ++r) {
        const int c = (lane + r * LANES) * E;
        load_floats(p.gain + c, p.width - c, gain[r]);
#pragma unroll
        for (int k = 0; k < E; ++k) dgain[r][k] = 0.f;
    }
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES; row < p.n;
         row += (int64_t)gridDim.x * kRows, turn ^= 1) {
        float xh[P][E], dy[P][E];
        const float rstd = p.rstd[row];
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < P; ++r) {
            const int c = (lane + r * LANES) * E;
            load_floats_once(static_cast<const T *>(p.h) + row * p.ldh + c, p.width - c, xh[r]);
            load_floats_once(static_cast<const T *>(p.dy) + row * p.lddy + c, p.width - c, dy[r]);
        }
#pragma unroll
        for (int r = 0; r < P; ++r)
#pragma unroll
            for (int k = 0; k < E; ++k) {
                xh[r][k] *= rstd;
                dgain[r][k] = __builtin_fmaf(dy[r][k], xh[r][k], dgain[r][k]);
                dy[r][k] *= gain[r][k];
                sum = __builtin_fmaf(dy[r][k], xh[r][k], sum);
            }
        const float mean = row_sum<LANES>(sum, part, turn) / (float)p.width;
#pragma unroll
        for (int r = 0; r < P; ++r) {
            const int c = (lane + r * LANES) * E;
            if (c >= p.width) continue;
            float t[E] = {};
            if (p.dh)
                load_floats_once(static_cast<const T *>(p.dh) + row * p.lddh + c, p.width - c, t);
#pragma unroll
            for (int k = 0; k < E; ++k) t[k] += rstd * (dy[r][k] - xh[r][k] * mean);
            store_floats(static_cast<T *>(p.dx) + row * p.lddx + c, p.width - c, t, p.once);
        }
    }
    // the workgroup's sums: the rows of a wavefront, then its wavefronts (or larger groups)
    // one after another, then a row of partials
    extern __shared__ float sums[];
#pragma unroll
    for (int d = LANES; d < kWaveLanes; d <<= 1)
#pragma unroll
        for (int r = 0; r < P; ++r)
#pragma unroll
            for (int k = 0; k < E; ++k) dgain[r][k] += __shfl_xor(dgain[r][k], d);
    constexpr int kGroup = LANES < kWaveLanes ? kWaveLanes : LANES, kGroups = kThreads / kGroup;
    const int group = threadIdx.x % kGroup < LANES ? (int)threadIdx.x / kGroup : -1;
    if constexpr (kGroups > 1) {
        for (int q = 0; q < kGroups; ++q) {
            __syncthreads();
            if (group == q) {
#pragma unroll
                for (int r = 0; r < P; ++r) {
                    const int c = (lane + r * LANES) * E;
                    if (c < p.width) {
#pragma unroll
                        for (int k = 0; k < E; ++k) {
                            if (q > 0) dgain[r][k] += sums[c + k];
                            if (q < kGroups - 1) sums[c + k] = dgain[r][k];
                        }
                    }
                }
            }
        }
    }
    if (group == kGroups - 1) {
#pragma unroll
        for (int r = 0; r < P; ++r) {
            const int c = (lane + r * LANES) * E;
#pragma unroll
            for (int k = 0; k < E; ++k)
                if (c + k < p.width) p.partial[(int64_t)blockIdx.x * p.width + c + k] = dgain[r][k];
        }
    }
}

// Rows too wide for registers, in two passes: mean(a xh) of each row, then a piece of
// columns per lane over groups of rows.  h and dy are read twice, which bounds it (with dh,
// 3000 x 17,001 f32: 216 us, 3000 x 20,480 241, bf16 158 and 139; the 16,384 columns that
// still fit in registers 149 and 93).
template <typename T>
__global__ __launch_bounds__(1024) void norm_grad_rows_kernel(NormGradArgs p) {
    __shared__ float part[2][16];
    constexpr int E = kPiece<T>;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < p.n; row += gridDim.x, turn ^= 1) {
        const float rstd = p.rstd[row];
        float sum = 0.f;
        for (int c = threadIdx.x * E; c < p.width; c += 1024 * E) {
            float h[E], dy[E], g[E];
            load_floats_once(static_cast<const T *>(p.h) + row * p.ldh + c, p.width - c, h);
            load_floats_once(static_cast<const T *>(p.dy) + row * p.lddy + c, p.width - c, dy);
            load_floats(p.gain + c, p.width - c, g);
#pragma unroll
            for (int k = 0; k < E; ++k)
                sum = __builtin_fmaf(dy[k] * g[k], h[k] * rstd, sum);
        }
        sum = row_sum<1024>(sum, part, turn);
        if (threadIdx.x == 0) p.coefficient[row] = sum / (float)p.width;
    }
}

template <typename T>
__global__ __launch_bounds__(kRowThreads) void norm_grad_columns_kernel(NormGradArgs p, int64_t per) {
    constexpr int E = kPiece<T>;
    const int c = (blockIdx.x * kRowThreads + threadIdx.x) * E;
    if (c >= p.width) return;
    const int live = p.width - c;
    const int64_t first = blockIdx.y * per, last = std::min<int64_t>(p.n, first + per);
    float g[E], dgain[E];
    load_floats(p.gain + c, live, g);
#pragma unroll
    for (int k = 0; k < E; ++k) dgain[k] = 0.f;
    for (int64_t row = first; row < last; ++row) {
        const float rstd = p.rstd[row], mean = p.coefficient[row];
        float h[E], dy[E], t[E] = {};
        load_floats_once(static_cast<const T *>(p.h) + row * p.ldh + c, live, h);
        load_floats_once(static_cast<const T *>(p.dy) + row * p.lddy + c, live, dy);
        if (p.dh) load_floats_once(static_cast<const T *>(p.dh) + row * p.lddh + c, live, t);
#pragma unroll
        for (int k = 0; k < E; ++k) {
            const float xh = h[k] * rstd;
            dgain[k] = __builtin_fmaf(dy[k], xh, dgain[k]);
            t[k] += rstd * (dy[k] * g[k] - xh * mean);
        }
        store_floats(static_cast<T *>(p.dx) + row * p.lddx + c, live, t, p.once);
    }
#pragma unroll
    for (int k = 0; k < E; ++k)
        if (k < live) p.partial[(int64_t)blockIdx.y * p.width + c + k] = dgain[k];
}

// out[c] = sum over `parts` rows of partial, in a fixed order: 32 groups of
// threads add every 32nd row, then the groups' sums are added (1024 x 1001: 4.7 us).
constexpr int kColumnGroups = 32;
constexpr int kColumnWidth = 32;

__global__ __launch_bounds__(kColumnGroups *kColumnWidth) void column_sums_kernel(
    const float *__restrict__ partial, int parts, int width, float *__restrict__ out) {
    __shared__ float sums[kColumnGroups][kColumnWidth];
    const int lane = threadIdx.x % kColumnWidth, g = threadIdx.x / kColumnWidth;
    const int c = blockIdx.x * kColumnWidth + lane;
    float v = 0.f;
    if (c < width) {
#pragma unroll 8
        for (int q = g; q < parts; q += kColumnGroups) v += partial[(int64_t)q * width + c];
    }
    sums[g][lane] = v;
    __syncthreads();
    if (g == 0 && c < width) {
        v = 0.f;
#pragma unroll
        for (int q = 0; q < kColumnGroups; ++q) v += sums[q][lane];
        out[c] = v;
    }
}

// Packed rows of a matrix as it is, a piece per lane.  Memory bounds it (65,536 x 1280
// bfloat16: 50 us, 5.1 TB/s).
template <typename T>
__global__ __launch_bounds__(kRowThreads) void pack_kernel(const T *__restrict__ x, int64_t n,
                                                           int width, int64_t ldx,
                                                           uint8_t *__restrict__ codes, int64_t ldc,
                                                           uint8_t *__restrict__ scales, int64_t lds) {
    constexpr int E = kPiece<T>;
    const int per = (width + kPackBlock - 1) / kPackBlock * (kPackBlock / E);   // pieces of a packed row
    const int64_t total = n * per, step = (int64_t)gridDim.x * kRowThreads;
    // (total and step are multiples of a block's pieces: its lanes stay together)
    for (int64_t q = (int64_t)blockIdx.x * kRowThreads + threadIdx.x; q < total; q += step) {
        const int64_t row = q / per;
        const int c = (int)(q - row * per) * E;
        float v[E];
        load_floats_once(x + row * ldx + c, width - c, v);
        uint8_t e;
        *reinterpret_cast<Codes<E> *>(codes + row * ldc + c) = pack_values(v, &e);
        if (c % kPackBlock == 0) scales[row * lds + c / kPackBlock] = e;
    }
}

// ---- launches -----------------------------------------------------------------
// Rows of up to 32 pieces share a wavefront, rows of up to 4096 elements have one of
// their own (no barrier), up to 8192 elements 256 lanes, up to 16,384 512, up to 32,768
// 1024; wider rows are read twice.
template <typename T, int LANES, int P>
hipError_t norm_of(const NormArgs &p, int cus, hipStream_t s) {
    constexpr int kThreads = LANES < kRowThreads ? kRowThreads : LANES;
    const int64_t groups = ceil_div(p.n, kThreads / LANES);
    const int64_t most = (int64_t)cus * (2048 / kThreads);
    norm_kernel<T, LANES, P><<<(unsigned)std::min(groups, most), kThreads, 0, s>>>(p);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_norm(const NormArgs &p, int cus, hipStream_t s) {
    // Rows of up to half a wavefront's pieces share it (145,827 x 96 bf16, residual: 27 us, a
    // wavefront per row 75).  Packed rows end with a whole block, whose lanes share a row.
    const int block = kPackBlock / kPiece<T>;
    int pieces = (p.width + kPiece<T> - 1) / kPiece<T>;
    if (p.codes) pieces = (pieces + block - 1) / block * block;
    if (pieces <= 8) return norm_of<T, 8, 1>(p, cus, s);
    if (pieces <= 16) return norm_of<T, 16, 1>(p, cus, s);
    if (pieces <= 32) return norm_of<T, 32, 1>(p, cus, s);
    if (pieces <= 64) return norm_of<T, 64, 1>(p, cus, s);
    constexpr int P = kChunk / kPiece<T>;   // pieces of a chunk of 8 elements
    const int chunks = (pieces + P - 1) / P;
    if (chunks <= 64) return norm_of<T, 64, P>(p, cus, s);
    if (chunks <= 128) return norm_of<T, 64, 2 * P>(p, cus, s);
    if (chunks <= 192) return norm_of<T, 64, 3 * P>(p, cus, s);
    if (chunks <= 256) return norm_of<T, 64, 4 * P>(p, cus, s);
    if (chunks <= 320) return norm_of<T, 64, 5 * P>(p, cus, s);
    if (chunks <= 384) return norm_of<T, 64, 6 * P>(p, cus, s);
    if (chunks <= 512) return norm_of<T, 64, 8 * P>(p, cus, s);
    // (lanes for which three or four chunks are enough: 3945 x 9504 bf16, residual, 57 us by 512
    // lanes, by 256 71; 937 x 20,000 f32 57 by 1024 of 3 chunks, of 4 71)
    if (chunks <= 1024) return norm_of<T, 256, 4 * P>(p, cus, s);
    if (chunks <= 1536) return norm_of<T, 512, 3 * P>(p, cus, s);
    if (chunks <= 2048) return norm_of<T, 512, 4 * P>(p, cus, s);
    if (chunks <= 3 * 1024) return norm_of<T, 1024, 3 * P>(p, cus, s);
    // (float rows of four chunks leave a few registers to scratch memory and are still read once:
    // 3000 x 32,768 f32, residual, 297 us, read twice 414; 700 rows 84 and 97, 200 28 and 31;
    // bf16 139 and 216, 34 and 54, 10 and 19)
    if (chunks <= 4096) return norm_of<T, 1024, 4 * P>(p, cus, s);
    norm_wide_kernel<T><<<(unsigned)std::min<int64_t>(p.n, 2 * cus), 1024, 0, s>>>(p);
    return hipGetLastError();
}

// LDS that holds a row of sums in whole chunks.
size_t chunk_bytes(int width) { return (size_t)ceil_div(width, kChunk) * kChunk * sizeof(float); }

// Rows of partials that a gradient leaves, at most.
constexpr int kGradGroups = 1024;
constexpr int kGradRegisterWidth = 16384;

template <typename T, int LANES, int P>
hipError_t norm_grad_of(const NormGradArgs &p, int *parts, hipStream_t s) {
    constexpr int kThreads = LANES < kRowThreads ? kRowThreads : LANES;
    constexpr int kRows = kThreads / LANES;
    // (larger workgroups are fewer at a time: 3945 x 9504 bf16 with dh in 86 us, 512 lanes per
    // row and up to kGradGroups workgroups 116)
    *parts = (int)std::min<int64_t>(ceil_div(p.n, kRows), LANES >= 512 ? kGradGroups / 2 : kGradGroups);
    norm_grad_kernel<T, LANES, P>
        <<<*parts, kThreads, LANES < kThreads ? chunk_bytes(p.width) : 0, s>>>(p);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_norm_grad(const NormGradArgs &p, float *dgain, int cus, hipStream_t s) {
    constexpr int P = kChunk / kPiece<T>;   // pieces of a chunk of 8 elements
    const int pieces = (p.width + kPiece<T> - 1) / kPiece<T>, chunks = (pieces + P - 1) / P;
    int parts = 0;
    hipError_t e = hipSuccess;
    // (narrow rows as in launch_norm: 145,827 x 96 bf16 with dh 32 us, a wavefront per row 86)
    if (p.n == 0) parts = 0;
    else if (pieces <= 8) e = norm_grad_of<T, 8, 1>(p, &parts, s);
    else if (pieces <= 16) e = norm_grad_of<T, 16, 1>(p, &parts, s);
    else if (pieces <= 32) e = norm_grad_of<T, 32, 1>(p, &parts, s);
    else if (pieces <= 64) e = norm_grad_of<T, 64, 1>(p, &parts, s);
    else if (chunks <= 64) e = norm_grad_of<T, 64, P>(p, &parts, s);
    else if (chunks <= 128) e = norm_grad_of<T, 64, 2 * P>(p, &parts, s);
    else if (chunks <= 192) e = norm_grad_of<T, 64, 3 * P>(p, &parts, s);
    else if (chunks <= 256) e = norm_grad_of<T, 64, 4 * P>(p, &parts, s);
    else if (chunks <= 320) e = norm_grad_of<T, 64, 5 * P>(p, &parts, s);
    else if (chunks <= 512) e = norm_grad_of<T, 256, 2 * P>(p, &parts, s);
    else if (chunks <= 1024) e = norm_grad_of<T, 512, 2 * P>(p, &parts, s);
    else if (chunks <= kGradRegisterWidth / kChunk) e = norm_grad_of<T, 1024, 2 * P>(p, &parts, s);
    else {
        norm_grad_rows_kernel<T><<<(unsigned)std::min<int64_t>(p.n, 2 * cus), 1024, 0, s>>>(p);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        const unsigned slices = (unsigned)ceil_div(ceil_div(p.width, kPiece<T>), kRowThreads);
        const int64_t groups = std::min<int64_t>(p.n, ceil_div(8 * cus, slices));
        const int64_t per = ceil_div(p.n, std::min<int64_t>(groups, kGradGroups));
        parts = (int)ceil_div(p.n, per);
        norm_grad_columns_kernel<T><<<dim3(slices, parts), kRowThreads, 0, s>>>(p, per);
        e = hipGetLastError();
    }
    if (e != hipSuccess) return e;
    column_sums_kernel<<<(unsigned)ceil_div(p.width, kColumnWidth), kColumnGroups * kColumnWidth, 0, s>>>(
        p.partial, parts, p.width, dgain);
    return hipGetLastError();
}

int check_rows(const char *name, const void *p, int32_t dtype, int64_t ld, int32_t width) {
    if (!p) return report(FBDT_E_INVAL, "%s is NULL", name);
    if (!aligned_to(p, dtype_bytes(dtype)))
        return report(FBDT_E_INVAL, "%s must be aligned to its elements", name);
    if (ld < width)
        return report(FBDT_E_INVAL, "%s: row stride %lld is below the width %d", name, (long long)ld,
                      width);
    return FBDT_OK;
}

int check_shape(int32_t dtype, int64_t n, int32_t width) {
    if (!known_dtype(dtype)) return report(FBDT_E_INVAL, "unknown type %d", dtype);
    if (n < 0 || n > (int64_t)1 << 36)
        return report(FBDT_E_INVAL, "n = %lld must be in [0, 2^36]", (long long)n);
    if (width < 1 || width > 1 << 20)
        return report(FBDT_E_INVAL, "width = %d must be in [1, 2^20]", width);
    return FBDT_OK;
}

int check_packed_out(const uint8_t *codes, int64_t ldc, const uint8_t *scales, int64_t lds,
                     int32_t width) {
    const int64_t blocks = ceil_div(width, kPackBlock);
    if (!codes || !aligned_to(codes, 16))
        return report(FBDT_E_INVAL, "codes must be 16-byte aligned");
    if (ldc < blocks * kPackBlock || ldc % kPackBlock != 0)
        return report(FBDT_E_INVAL, "codes: row stride %lld must be a multiple of 128 and >= width",
                      (long long)ldc);
    if (!scales || !aligned_to(scales, 4))
        return report(FBDT_E_INVAL, "scales must be 4-byte aligned");
    if (lds < blocks || lds % 4 != 0)
        return report(FBDT_E_INVAL, "scales: row stride %lld must be a multiple of 4 and hold %lld "
                      "blocks", (long long)lds, (long long)blocks);
    return FBDT_OK;
}

}  // namespace
}  // namespace fbdt

using namespace fbdt;

extern "C" {

int fbdt_rms_norm(const void *x, int64_t ldx, const void *residual, int64_t ldr, int32_t dtype,
                  int64_t n, int32_t width, const float *gain, float eps, void *h, int64_t ldh,
                  void *y, int64_t ldy, uint8_t *codes, int64_t ldc, uint8_t *scales, int64_t lds,
                  float *rstd, void *stream) {
    int rc;
    if ((rc = check_shape(dtype, n, width))) return rc;
    if (!(eps > 0.f) || !(eps < __builtin_inff()))
        return report(FBDT_E_INVAL, "eps must be positive and finite");
    if (!gain || !aligned_to(gain, 4)) return report(FBDT_E_INVAL, "gain must be 4-byte aligned");
    if (n == 0) return FBDT_OK;
    if (!y && !codes) return report(FBDT_E_INVAL, "neither y nor codes is given");
    if ((rc = check_rows("x", x, dtype, ldx, width))) return rc;
    if (residual && (rc = check_rows("residual", residual, dtype, ldr, width))) return rc;
    if (h && (rc = check_rows("h", h, dtype, ldh, width))) return rc;
    if (y && (rc = check_rows("y", y, dtype, ldy, width))) return rc;
    if (codes && (rc = check_packed_out(codes, ldc, scales, lds, width))) return rc;
    if (rstd && !aligned_to(rstd, 4)) return report(FBDT_E_INVAL, "rstd must be 4-byte aligned");
    int cus = 0;
    if ((rc = device_cus(&cus))) return rc;
    const int64_t size = dtype_bytes(dtype);
    const NormArgs p = {x, residual, n, ldx, ldr, width, gain, eps, h, y, ldh, ldy, codes, scales,
                        ldc, lds, rstd, rows_stored_once(h, ldh * size, width * size),
                        rows_stored_once(y, ldy * size, width * size)};
    NET_TRY(with_dtype(dtype, [&](auto t) {
        return launch_norm<decltype(t)>(p, cus, static_cast<hipStream_t>(stream));
    }));
    return FBDT_OK;
}

int64_t fbdt_rms_norm_grad_work(int64_t n, int32_t width) {
    if (check_shape(FBDT_F32, n, width)) return -1;
    const int64_t groups = std::min<int64_t>(n, kGradGroups);
    return 4 * groups * width + (width > kGradRegisterWidth ? 4 * n : 0);
}

int fbdt_rms_norm_grad(const void *dy, int64_t lddy, const void *h, int64_t ldh, const void *dh,
                       int64_t lddh, int32_t dtype, int64_t n, int32_t width, const float *gain,
                       const float *rstd, void *dx, int64_t lddx, float *dgain, void *work,
                       int64_t work_bytes, void *stream) {
    int rc;
    if ((rc = check_shape(dtype, n, width))) return rc;
    if (!gain || !aligned_to(gain, 4)) return report(FBDT_E_INVAL, "gain must be 4-byte aligned");
    if (!dgain || !aligned_to(dgain, 4)) return report(FBDT_E_INVAL, "dgain must be 4-byte aligned");
    if (n > 0) {
        if ((rc = check_rows("dy", dy, dtype, lddy, width))) return rc;
        if ((rc = check_rows("h", h, dtype, ldh, width))) return rc;
        if (dh && (rc = check_rows("dh", dh, dtype, lddh, width))) return rc;
        if ((rc = check_rows("dx", dx, dtype, lddx, width))) return rc;
        if (!rstd || !aligned_to(rstd, 4)) return report(FBDT_E_INVAL, "rstd must be 4-byte aligned");
        const int64_t need = fbdt_rms_norm_grad_work(n, width);
        if (!work || !aligned_to(work, 256) || work_bytes < need)
            return report(FBDT_E_INVAL, "work must hold %lld bytes, 256-byte aligned", (long long)need);
    }
    int cus = 0;
    if ((rc = device_cus(&cus))) return rc;
    float *const partial = static_cast<float *>(work);
    NormGradArgs p = {dy, h, dh, n, lddy, ldh, lddh, width, gain, rstd, dx, lddx, partial, nullptr,
                      rows_stored_once(dx, lddx * dtype_bytes(dtype), width * dtype_bytes(dtype))};
    if (n > 0) p.coefficient = partial + std::min<int64_t>(n, kGradGroups) * width;
    NET_TRY(with_dtype(dtype, [&](auto t) {
        return launch_norm_grad<decltype(t)>(p, dgain, cus, static_cast<hipStream_t>(stream));
    }));
    return FBDT_OK;
}

int fbdt_pack(const void *x, int64_t ldx, int32_t dtype, int64_t n, int32_t width, uint8_t *codes,
              int64_t ldc, uint8_t *scales, int64_t lds, void *stream) {
    int rc;
    if ((rc = check_shape(dtype, n, width))) return rc;
    if (n == 0) return FBDT_OK;
    if ((rc = check_rows("x", x, dtype, ldx, width))) return rc;
    if ((rc = check_packed_out(codes, ldc, scales, lds, width))) return rc;
    int cus = 0;
    if ((rc = device_cus(&cus))) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    NET_TRY(with_dtype(dtype, [&](auto t) {
        typedef decltype(t) T;
        const int64_t pieces = n * (ceil_div(width, kPackBlock) * (kPackBlock / kPiece<T>));
        const unsigned grid =
            (unsigned)std::min<int64_t>(ceil_div(pieces, kRowThreads), 16 * (int64_t)cus);
        pack_kernel<T><<<grid, kRowThreads, 0, s>>>(static_cast<const T *>(x), n, width, ldx, codes,
                                                    ldc, scales, lds);
        return hipGetLastError();
    }));
    return FBDT_OK;
}

}  // extern "C"
