// Shared by the network operators (embed.hip, rows.hip, product.hip): what
// they take from the host runtime (capi.hip), element types and packed rows.
// Nothing here is exported from libfbdt.
#pragma once

#include "fbdt.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace fbdt {

// Keeps a message for fbdt_last_error and returns `code`.
int report(int code, const char *fmt, ...) __attribute__((format(printf, 2, 3)));
// Compute units of the current device.
int device_cus(int *cus);

// In an entry of the C ABI.  (Its name stands for the expression, whose text may be a
// whole function and leave the cause no room in the message.)
#define NET_TRY(expr)                                                                        \
    do {                                                                                     \
        const hipError_t e_ = (expr);                                                        \
        if (e_ != hipSuccess)                                                                \
            return report(FBDT_E_DEVICE, "%s failed: %s", __func__, hipGetErrorString(e_));  \
    } while (0)

// A packed row holds e4m3 codes (largest 448) and one power-of-two scale,
// as its biased exponent, for each kPackBlock columns.
constexpr int kPackBlock = 128;
// Elements of a row that a lane adds up at a time.
constexpr int kChunk = 8;
constexpr int kWaveLanes = 64;

inline bool known_dtype(int32_t t) { return t == FBDT_F32 || t == FBDT_BF16 || t == FBDT_F16; }
inline int64_t dtype_bytes(int32_t t) { return t == FBDT_F32 ? 4 : 2; }
inline bool aligned_to(const void *p, uintptr_t a) {
    return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0;
}
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// `rows` rows of `width` elements of `size` bytes, `stride` elements apart.
struct Extent {
    const void *p;
    int64_t rows, width, stride, size;
};

// Whether two matrices share a byte.  Rows of one stride may lie side by side in a wider
// matrix, a single row between the rows of another; rows of two strides that lie among
// each other are taken to meet.
inline bool overlap(const Extent &a, const Extent &b) {
    if (a.rows < 1 || b.rows < 1) return false;
    typedef __int128 wide;
    const wide aw = (wide)a.width * a.size, bw = (wide)b.width * b.size;
    const wide as = (wide)a.stride * a.size, bs = (wide)b.stride * b.size;
    const wide a0 = (wide)reinterpret_cast<uintptr_t>(a.p), b0 = (wide)reinterpret_cast<uintptr_t>(b.p);
    if (a0 + (a.rows - 1) * as + aw <= b0 || b0 + (b.rows - 1) * bs + bw <= a0) return false;
    if (a.rows == 1 && b.rows == 1) return true;
    if (a.rows > 1 && b.rows > 1 && as != bs) return true;
    const wide stride = a.rows > 1 ? as : bs;
    const wide after = ((b0 - a0) % stride + stride) % stride;   // b's columns, from a's on
    return after < aw || after + bw > stride;
}

// Refuses a result that lies on what the call reads.
inline int check_apart(const char *result, const Extent &out, const char *name, const Extent &in) {
    return overlap(out, in) ? report(FBDT_E_INVAL, "%s overlaps %s", result, name) : FBDT_OK;
}

// A launch holds fewer than 2^32 threads along x: `groups` workgroups, in rows along y
// where there are more, and the number of a workgroup among them (of which the last
// row may have more than `groups`).
inline dim3 grid_of(int64_t groups, int threads) {
    const int64_t x = std::min<int64_t>(groups, ((int64_t)1 << 31) / threads);
    return dim3((unsigned)x, (unsigned)ceil_div(groups, x));
}
__device__ __forceinline__ int64_t group_number() {
    return (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
}

// Calls f with a value of the element type that `dtype` names.
template <typename F>
inline hipError_t with_dtype(int32_t dtype, F &&f) {
    if (dtype == FBDT_F32) return f(float{});
    if (dtype == FBDT_BF16) return f(__bf16{});
    return f(_Float16{});
}

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// 16 bytes at p, which is aligned to an element only; `once`: memory that is not
// read or written again soon (it need not stay in cache).
typedef u32x4 u32x4_at_2 __attribute__((aligned(2)));
template <typename T>
__device__ __forceinline__ u32x4 load_piece_once(const T *p) {
    return __builtin_nontemporal_load(reinterpret_cast<const u32x4_at_2 *>(p));
}
template <typename T>
__device__ __forceinline__ void store_piece_once(T *p, u32x4 v) {
    __builtin_nontemporal_store(v, reinterpret_cast<u32x4_at_2 *>(p));
}
template <typename T>
__device__ __forceinline__ void store_piece(T *p, u32x4 v, bool once) {
    // (the empty statements keep the compiler from making one store of both)
    if (once) {
        asm volatile("");
        store_piece_once(p, v);
        asm volatile("");
    } else {
        *reinterpret_cast<u32x4_at_2 *>(p) = v;
    }
}
// Whether the stores of a result's rows, 16 bytes per lane side by side, should pass the
// cache: what they leave of a line goes to memory by itself, so rows that begin inside
// a piece gather in cache unless they are long (a lookup's rows stored one by one, 2.3M of
// 100 bytes: 148 us past the cache, 63 through it; of 96 bytes 36 and 45; 200,000 of
// 2002 bytes 114 and 124).
inline bool rows_stored_once(const void *p, int64_t row_bytes, int64_t width_bytes) {
    return (aligned_to(p, 16) && row_bytes % 16 == 0) || width_bytes >= 1024;
}

// kChunk elements as they are in memory (in half the registers of their float32
// values where T has 16 bits).
template <typename T>
struct RawChunk {
    T v[kChunk];
};

// kChunk elements from p, which is met once; those from `live` on are 0.  Rows may start at
// any element: the loads are as wide as the chunk and aligned to one element only,
// which the hardware takes.
template <typename T>
__device__ __forceinline__ RawChunk<T> load_raw_once(const T *p, int live) {
    RawChunk<T> t;
    if (live >= kChunk) {
        // (a chunk of more than one piece meets its cache lines twice)
        if constexpr (sizeof t == 16) {
            const u32x4 raw = load_piece_once(p);
            __builtin_memcpy(&t, &raw, sizeof t);
        } else {
            __builtin_memcpy(&t, p, sizeof t);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kChunk; ++i) t.v[i] = i < live ? p[i] : (T)0.f;
    }
    return t;
}

// A piece: the elements of T in 16 bytes, as float; those from `live` on are 0 and
// are not stored.
template <typename T>
constexpr int kPiece = 16 / sizeof(T);

template <typename T>
__device__ __forceinline__ void load_floats_once(const T *p, int live, float (&v)[kPiece<T>]) {
    T t[kPiece<T>];
    if (live >= kPiece<T>) {
        const u32x4 raw = load_piece_once(p);
        __builtin_memcpy(t, &raw, sizeof t);
    } else {
#pragma unroll
        for (int i = 0; i < kPiece<T>; ++i) t[i] = i < live ? p[i] : (T)0.f;
    }
#pragma unroll
    for (int i = 0; i < kPiece<T>; ++i) v[i] = (float)t[i];
}

template <typename T>
__device__ __forceinline__ void store_floats(T *p, int live, const float (&v)[kPiece<T>], bool once) {
    T t[kPiece<T>];
#pragma unroll
    for (int i = 0; i < kPiece<T>; ++i) t[i] = (T)v[i];
    if (live >= kPiece<T>) {
        u32x4 raw;
        __builtin_memcpy(&raw, t, sizeof raw);
        store_piece(p, raw, once);
    } else {
#pragma unroll
        for (int i = 0; i < kPiece<T>; ++i)
            if (i < live) p[i] = t[i];
    }
}

// N float32 values that stay in cache; those from `live` on are 0.
template <int N>
__device__ __forceinline__ void load_floats(const float *p, int live, float (&v)[N]) {
    if (live >= N) {
        __builtin_memcpy(v, p, sizeof v);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = i < live ? p[i] : 0.f;
    }
}

// Packs a lane's N values (8 or 4); the 128 / N lanes of its block call together.
// The exponent e is the smallest with amax <= 448 2^e over the block's finite values
// (0 where they are all 0), so that v 2^-e is exact and the conversion, to nearest
// even, is the only rounding.  Infinities and NaN take the code NaN.
template <int N>
struct Codes {
    uint32_t word[N / 4];
};

template <int N>
__device__ __forceinline__ Codes<N> pack_values(const float (&v)[N], uint8_t *exponent) {
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float a = __builtin_fabsf(v[i]);
        amax = a < __builtin_inff() ? __builtin_fmaxf(amax, a) : amax;   // (NaN fails the test)
    }
#pragma unroll
    for (int s = 1; s < kPackBlock / N; s <<= 1) amax = __builtin_fmaxf(amax, __shfl_xor(amax, s));
    // amax = 1.m 2^(E - 127) as a normal number; 448 = 1.75 2^8
    const uint32_t bits = __float_as_uint(amax);
    int biased = (int)(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u);
    biased = biased < 1 ? 1 : biased;
    biased = bits == 0 ? 127 : biased;
    *exponent = (uint8_t)biased;
    const float inv = __uint_as_float((uint32_t)(254 - biased) << 23);   // 2^-e: 7 <= 254 - biased
    float q[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        q[i] = v[i] * inv;
        q[i] = __builtin_fabsf(q[i]) <= 448.f ? q[i] : __builtin_nanf("");
    }
    Codes<N> out;
#pragma unroll
    for (int h = 0; h < N / 4; ++h) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * h], q[4 * h + 1], 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * h + 2], q[4 * h + 3], w, true);
        out.word[h] = (uint32_t)w;
    }
    return out;
}

}  // namespace fbdt
