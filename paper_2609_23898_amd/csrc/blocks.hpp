// The 8-bit block format on the device: power-of-two scales of blocks of 128
// entries, conversions to and from e4m3 and e5m2 codes, and loads and stores
// of neighbouring entries at any alignment of their own type.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "../../include/cerar_train.h"

namespace cerar {

constexpr size_t kBlock = 128;
constexpr size_t round_up(size_t n, size_t m) { return (n + m - 1) / m * m; }
// Row length of the codes, and four-block groups of the scales, of `cols` columns.
constexpr size_t blocks_ld(size_t cols) { return round_up(cols, kBlock); }
constexpr size_t scale_groups(size_t cols) { return (blocks_ld(cols) / kBlock + 3) / 4; }

// Threads of a launch along x: their count has 32 bits.
constexpr uint64_t kMostThreads = 0xFFFFFFFFu;
constexpr unsigned kComputeUnits = 256;              // of the card, which the variants' rules count on

// Byte ranges of a call's buffers, for its overlap checks.
inline bool ranges_meet(const void *a, size_t na, const void *b, size_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return na && nb && x < y + nb && y < x + na;
}

// Bytes from the first entry of a matrix to its last, or false where they pass 2^56, more
// than any address space.
inline bool matrix_bytes(size_t rows, size_t cols, size_t ld, size_t entry, size_t *bytes) {
    constexpr size_t most = (size_t)1 << 56;
    *bytes = 0;
    if (!rows || !cols) return true;
    if (cols > most / entry || (rows > 1 && ld > (most / entry - cols) / (rows - 1))) return false;
    *bytes = ((rows - 1) * ld + cols) * entry;
    return true;
}

namespace {

// Exponent of the largest binade: its largest value is 1.75 * 2^kTop.
template <int F>
constexpr int kTop = F == CERAR_E4M3 ? 8 : 15;

// Magnitude bits of a finite x, 0 of any other: their unsigned maximum is a
// block's largest magnitude.
__device__ inline uint32_t magnitude(float x) {
    const uint32_t u = __float_as_uint(x) & 0x7FFFFFFFu;
    return u < 0x7F800000u ? u : 0u;
}

// Byte of the smallest power of two 2^(byte - 127) with amax <= 1.75 * 2^(top +
// byte - 127), from amax's bits.
__device__ inline uint32_t scale_byte(uint32_t amax, int top) {
    const int b = (int)(amax >> 23) - top + ((amax & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return b > 0 ? (uint32_t)b : 0u;
}
// 2^(127 - byte): a normal number, since a byte is at most 247.
__device__ inline float scale_inverse(uint32_t b) { return __uint_as_float((254u - b) << 23); }
// 2^(byte - 127); byte 0 is below the normal numbers.
__device__ inline float scale_value(uint32_t b) { return __uint_as_float(b ? b << 23 : 0x400000u); }

// Maximum over the 16 lanes of a DPP row.
__device__ inline uint32_t row_max(uint32_t u) {
    u = max(u, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)u, 0x128, 0xF, 0xF, true));   // row_ror:8
    u = max(u, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)u, 0x124, 0xF, 0xF, true));
    u = max(u, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)u, 0x122, 0xF, 0xF, true));
    u = max(u, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)u, 0x121, 0xF, 0xF, true));
    return u;
}

// Maximum over the 32 lanes of either half of a wave.
__device__ inline uint32_t half_max(uint32_t u) {
    u = row_max(u);
    return max(u, (uint32_t)__builtin_amdgcn_ds_swizzle((int)u, 0x401F));    // lane ^ 16
}

typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef float v4f_at4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t v4u_at2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t v2u_at2 __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u_at1 __attribute__((aligned(1)));

// Four values to four codes, to nearest, ties to even.
template <int F>
__device__ inline uint32_t encode4(float a, float b, float c, float d) {
    int w = 0;
    if (F == CERAR_E4M3) {
        w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, w, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    } else {
        w = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, w, false);
        w = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, w, true);
    }
    return (uint32_t)w;
}

// The values of four codes with the scale byte b.
template <int F>
__device__ inline void decode4(uint32_t w, uint32_t b, float (&x)[4]) {
    const float s = scale_value(b);
    v2f lo, hi;
    if (F == CERAR_E4M3) {
        lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
        hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    } else {
        lo = __builtin_amdgcn_cvt_pk_f32_bf8((int)w, false);
        hi = __builtin_amdgcn_cvt_pk_f32_bf8((int)w, true);
    }
    x[0] = lo[0] * s;
    x[1] = lo[1] * s;
    x[2] = hi[0] * s;
    x[3] = hi[1] * s;
}

typedef __bf16 v2b __attribute__((ext_vector_type(2)));

// Two values rounded to bf16, to nearest, ties to even.
__device__ inline uint32_t pack_bf16(float lo, float hi) { return __builtin_bit_cast(uint32_t, v2b{(__bf16)lo, (__bf16)hi}); }

struct Bf16 {
    uint16_t bits;
};
__device__ inline float widen(float x) { return x; }
__device__ inline float widen(Bf16 x) { return __uint_as_float((uint32_t)x.bits << 16); }
__device__ inline void narrow(float x, float *p) { *p = x; }
__device__ inline void narrow(float x, Bf16 *p) { p->bits = (uint16_t)pack_bf16(x, 0.0f); }

// Entries p[0..8), of which the first `left` exist; zeros for the others.
__device__ inline void load8(const float *p, int left, float (&x)[8]) {
    if (left >= 8) {
        const v4f a = *reinterpret_cast<const v4f_at4 *>(p), b = *reinterpret_cast<const v4f_at4 *>(p + 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[j] = a[j];
            x[4 + j] = b[j];
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = j < left ? p[j] : 0.0f;
    }
}
__device__ inline void load8(const Bf16 *p, int left, float (&x)[8]) {
    if (left >= 8) {
        const v4u a = *reinterpret_cast<const v4u_at2 *>(p);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[2 * j] = __uint_as_float(a[j] << 16);
            x[2 * j + 1] = __uint_as_float(a[j] & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = j < left ? widen(p[j]) : 0.0f;
    }
}
__device__ inline void store8(float *p, int left, const float (&x)[8]) {
    if (left >= 8) {
        *reinterpret_cast<v4f_at4 *>(p) = v4f{x[0], x[1], x[2], x[3]};
        *reinterpret_cast<v4f_at4 *>(p + 4) = v4f{x[4], x[5], x[6], x[7]};
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < left) p[j] = x[j];
    }
}
__device__ inline void store8(Bf16 *p, int left, const float (&x)[8]) {
    if (left >= 8) {
        v4u w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = pack_bf16(x[2 * j], x[2 * j + 1]);
        *reinterpret_cast<v4u_at2 *>(p) = w;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < left) narrow(x[j], p + j);
    }
}
// The same for four, with the hint that they are not used again soon: streams that
// pass the caches by (405 million fp32 gradients read at 7.1 TB/s, 6.1 without it; an
// AdamW step over as many 6.1 TB/s, 5.8).
template <class T>
struct Four;                                         // as they are in memory
template <>
struct Four<float> {
    v4f w;
    __device__ __forceinline__ void load(const float *p, int left) {
        if (left >= 4) {
            w = __builtin_nontemporal_load(reinterpret_cast<const v4f_at4 *>(p));
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = j < left ? p[j] : 0.0f;
        }
    }
    __device__ __forceinline__ float operator[](int j) const { return w[j]; }
};
template <>
struct Four<Bf16> {
    v2u w;
    __device__ __forceinline__ void load(const Bf16 *p, int left) {
        if (left >= 4) {
            w = __builtin_nontemporal_load(reinterpret_cast<const v2u_at2 *>(p));
        } else {
            w = v2u{0, 0};
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j < left) w[j / 2] |= (uint32_t)p[j].bits << (j % 2 * 16);
        }
    }
    __device__ __forceinline__ float operator[](int j) const {
        return __uint_as_float(j % 2 ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16);
    }
};
template <class T>
__device__ inline void load4(const T *p, int left, float (&x)[4]) {
    Four<T> f;
    f.load(p, left);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = f[j];
}
__device__ inline uint32_t load4(const uint8_t *p, int left) {
    if (left >= 4) return *reinterpret_cast<const u_at1 *>(p);
    uint32_t w = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < left) w |= (uint32_t)p[j] << (8 * j);
    return w;
}
// (kPast = false: through the caches, where several waves fill a line.)
template <bool kPast = true>
__device__ inline void store4(float *p, int left, const float (&x)[4]) {
    if (left >= 4) {
        const v4f w = {x[0], x[1], x[2], x[3]};
        if (kPast) __builtin_nontemporal_store(w, reinterpret_cast<v4f_at4 *>(p));
        else *reinterpret_cast<v4f_at4 *>(p) = w;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < left) p[j] = x[j];
    }
}
template <bool kPast = true>
__device__ inline void store4(Bf16 *p, int left, const float (&x)[4]) {
    if (left >= 4) {
        const v2u w = {pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
        if (kPast) __builtin_nontemporal_store(w, reinterpret_cast<v2u_at2 *>(p));
        else *reinterpret_cast<v2u_at2 *>(p) = w;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < left) narrow(x[j], p + j);
    }
}
__device__ inline void store4(uint8_t *p, int left, uint32_t w) {
    if (left >= 4) {
        *reinterpret_cast<u_at1 *>(p) = w;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < left) p[j] = (uint8_t)(w >> (8 * j));
    }
}

}  // namespace
}  // namespace cerar
