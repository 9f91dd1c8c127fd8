// Matrices into the 8-bit block format (blocks.hpp), as they are and
// transposed, in one pass.
//
// A workgroup takes a tile of 128 x 128 entries.  A thread holds an 8 x 8 piece
// of it in registers: the largest magnitudes of its 128-entry rows meet over
// one DPP row of 16 lanes, those of its columns over four lanes and then, in
// LDS, over the four waves; so x is read once for both forms.  The transposed
// codes go through LDS, so that a column's 128 bytes leave in one piece.  The bound
// is memory: 12288 x 6144 entries of bf16 take 57 us both ways (5.3 TB/s), 36 by rows
// alone (6.3); 79 and 40 before bf16 entries stayed packed in registers, LDS had the
// places below and tiles that share words of scales one XCD.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "blocks.hpp"
#include "cerar_internal.hpp"

namespace cerar {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = 128;
constexpr int kPitch = kTile + 16;                   // bytes of a column in LDS

struct QuantizeArgs {
    const void *x;
    uint32_t rows, cols;
    size_t ld;
    uint8_t *row_codes, *row_scales, *col_codes, *col_scales;
    uint32_t col_tiles;
};

// Writes the scale byte of (r, block b); the last block also clears the bytes of
// the blocks that fill its group up to four.
__device__ inline void put_scale(uint8_t *scales, size_t rows, size_t r, uint32_t b, uint32_t blocks, uint32_t byte) {
    uint8_t *at = scales + ((b / 4) * rows + r) * 4;
    at[b % 4] = (uint8_t)byte;
    if (b + 1 == blocks)
        for (uint32_t k = b % 4 + 1; k < 4; ++k) at[k] = 0;
}

// Eight neighbouring entries of a row, as they are in memory.
template <class T>
struct Row;
template <>
struct Row<float> {
    float x[8];
    __device__ __forceinline__ void load(const float *p, int left) { load8(p, left, x); }
    __device__ __forceinline__ float operator[](int j) const { return x[j]; }
};
template <>
struct Row<Bf16> {
    v4u w;
    __device__ __forceinline__ void load(const Bf16 *p, int left) {
        if (left >= 8) {
            w = *reinterpret_cast<const v4u_at2 *>(p);
        } else {
            w = v4u{0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < left) w[j / 2] |= (uint32_t)p[j].bits << (j % 2 * 16);
        }
    }
    __device__ __forceinline__ float operator[](int j) const {
        return __uint_as_float(j % 2 ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16);
    }
};

// Place of 8 entries of rows 8 group .. + 7 of column c in LDS: the columns of a wave's
// store, eight apart, then touch all banks.
__device__ inline uint32_t place(uint32_t c, uint32_t group) { return c * kPitch + (group ^ (c / 16 % 8 * 2)) * 8; }

template <class T, int F, bool kWhole>
__global__ __launch_bounds__(kThreads) void k_quantize(QuantizeArgs a) {
    __shared__ uint32_t top[4][kTile];
    __shared__ __align__(16) uint8_t turned[kTile * kPitch];
    // four neighbouring tiles of a row, whose scales share words, to one XCD
    uint32_t id = blockIdx.x;
    if ((id | 31) < gridDim.x) id = (id & ~31u) + id % 8 * 4 + id / 8 % 4;
    const uint32_t tile_r = id / a.col_tiles, tile_c = id % a.col_tiles;
    const uint32_t lane = threadIdx.x % 16, group = threadIdx.x / 16, wave = threadIdx.x / 64;
    const uint32_t r0 = tile_r * kTile + group * 8, c0 = tile_c * kTile + lane * 8;
    Row<T> x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const T *p = static_cast<const T *>(a.x) + (size_t)(r0 + i) * a.ld + c0;
        x[i].load(p, r0 + i < a.rows ? (int)min(a.cols - min(c0, a.cols), 8u) : 0);
    }
    uint32_t col[8], row[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) col[j] = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        row[i] = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t u = magnitude(x[i][j]);
            row[i] = max(row[i], u);
            col[j] = max(col[j], u);
        }
        row[i] = row_max(row[i]);
    }
    if (kWhole) {
        uint32_t t = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) t = max(t, row[i]);
        t = max(t, (uint32_t)__shfl_xor((int)t, 16));
        t = max(t, (uint32_t)__shfl_xor((int)t, 32));
        if (threadIdx.x % 64 == 0) top[wave][0] = t;
        __syncthreads();
        t = max(max(top[0][0], top[1][0]), max(top[2][0], top[3][0]));
#pragma unroll
        for (int j = 0; j < 8; ++j) row[j] = col[j] = t;
    } else if (a.col_codes) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            col[j] = max(col[j], (uint32_t)__shfl_xor((int)col[j], 16));
            col[j] = max(col[j], (uint32_t)__shfl_xor((int)col[j], 32));
            if (threadIdx.x % 64 < 16) top[wave][lane * 8 + j] = col[j];
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t c = lane * 8 + j;
            col[j] = max(max(top[0][c], top[1][c]), max(top[2][c], top[3][c]));
        }
    }
    if (a.row_codes) {
        const size_t ld = (size_t)a.col_tiles * kTile;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t b = scale_byte(row[i], kTop<F>);
            const float s = scale_inverse(b);
            const Row<T> &v = x[i];
            const v2u w = {encode4<F>(v[0] * s, v[1] * s, v[2] * s, v[3] * s),
                           encode4<F>(v[4] * s, v[5] * s, v[6] * s, v[7] * s)};
            if (r0 + i < a.rows) {
                *reinterpret_cast<v2u *>(a.row_codes + (r0 + i) * ld + c0) = w;
                if (lane == 0) put_scale(a.row_scales, a.rows, r0 + i, tile_c, a.col_tiles, b);
            }
        }
    }
    if (!a.col_codes) return;
    const uint32_t row_tiles = (a.rows + kTile - 1) / kTile;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t b = scale_byte(col[j], kTop<F>);
        const float s = scale_inverse(b);
        const v2u w = {encode4<F>(x[0][j] * s, x[1][j] * s, x[2][j] * s, x[3][j] * s),
                       encode4<F>(x[4][j] * s, x[5][j] * s, x[6][j] * s, x[7][j] * s)};
        *reinterpret_cast<v2u *>(turned + place(lane * 8 + j, group)) = w;
        if (group == 0 && c0 + j < a.cols) put_scale(a.col_scales, a.cols, c0 + j, tile_r, row_tiles, b);
    }
    __syncthreads();
    const size_t ld = (size_t)row_tiles * kTile;
#pragma unroll
    for (int k = 0; k < kTile * kTile / 16 / kThreads; ++k) {
        const uint32_t c = (threadIdx.x + k * kThreads) / 8, part = threadIdx.x % 8;
        const uint32_t gc = tile_c * kTile + c;
        if (gc < a.cols)
            *reinterpret_cast<v4u *>(a.col_codes + gc * ld + tile_r * kTile + part * 16) =
                *reinterpret_cast<const v4u *>(turned + place(c, 2 * part));
    }
}

// By rows alone, with a scale for each row and block: a wave takes four blocks of a
// row, whose scales are one word.  45 x 2050 entries take 7 us in tiles, the card
// all but empty, and 3 so.
template <class T, int F>
__global__ __launch_bounds__(kThreads) void k_quantize_rows(QuantizeArgs a) {
    const uint32_t groups = (a.col_tiles + 3) / 4, lane = threadIdx.x % 64;
    const uint64_t item = (uint64_t)blockIdx.x * (kThreads / 64) + threadIdx.x / 64;
    const uint32_t r = (uint32_t)(item / groups), group = (uint32_t)(item % groups);
    if (r >= a.rows) return;
    const uint32_t c = group * 4 * kTile + lane * 8;
    Row<T> x;
    x.load(static_cast<const T *>(a.x) + (size_t)r * a.ld + c, (int)min(a.cols - min(c, a.cols), 8u));
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, magnitude(x[j]));
    const bool exists = c < a.col_tiles * kTile;
    const uint32_t b = exists ? scale_byte(row_max(top), kTop<F>) : 0u;
    const float s = scale_inverse(b);
    if (exists)
        *reinterpret_cast<v2u *>(a.row_codes + (size_t)r * a.col_tiles * kTile + c) =
            v2u{encode4<F>(x[0] * s, x[1] * s, x[2] * s, x[3] * s), encode4<F>(x[4] * s, x[5] * s, x[6] * s, x[7] * s)};
    const uint32_t word = (uint32_t)__builtin_amdgcn_readlane((int)b, 0) | (uint32_t)__builtin_amdgcn_readlane((int)b, 16) << 8 |
                          (uint32_t)__builtin_amdgcn_readlane((int)b, 32) << 16 |
                          (uint32_t)__builtin_amdgcn_readlane((int)b, 48) << 24;
    if (lane == 0) reinterpret_cast<uint32_t *>(a.row_scales)[(size_t)group * a.rows + r] = word;
}

template <class T, int F>
void launch(const QuantizeArgs &a, bool tile, unsigned groups, hipStream_t stream) {
    const uint64_t items = (uint64_t)a.rows * ((a.col_tiles + 3) / 4), waves = kThreads / 64;
    if (!tile && !a.col_codes && items <= kMostThreads / 64) {
        hipLaunchKernelGGL((k_quantize_rows<T, F>), dim3((unsigned)((items + waves - 1) / waves)), dim3(kThreads), 0, stream, a);
        return;
    }
    if (tile) hipLaunchKernelGGL((k_quantize<T, F, true>), dim3(groups), dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL((k_quantize<T, F, false>), dim3(groups), dim3(kThreads), 0, stream, a);
}

}  // namespace

int check_blocks(const cerar_blocks *b, const char *name) {
    if (b->rows >= (size_t)1 << 31 || b->cols >= (size_t)1 << 31)
        return fail(CERAR_E_INVAL, "%s has a size of 2^31 or more", name);
    if ((unsigned)b->format > CERAR_E5M2) return fail(CERAR_E_INVAL, "%s has an unknown format", name);
    if (b->rows && b->cols) {
        if (!b->codes || !b->scales) return fail(CERAR_E_INVAL, "%s has a NULL buffer", name);
        if (reinterpret_cast<uintptr_t>(b->codes) % 16 || reinterpret_cast<uintptr_t>(b->scales) % 4)
            return fail(CERAR_E_INVAL, "%s: codes have to be 16-byte aligned, scales 4-byte", name);
    }
    return CERAR_OK;
}

int quantize(const void *x, cerar_type type, size_t rows, size_t cols, size_t ld, bool tile, cerar_fp8 format,
             const cerar_blocks *by_row, const cerar_blocks *by_col, hipStream_t stream) {
    QuantizeArgs a{x, (uint32_t)rows, (uint32_t)cols, ld, nullptr, nullptr, nullptr, nullptr,
                   (uint32_t)((cols + kTile - 1) / kTile)};
    if (by_row) {
        a.row_codes = static_cast<uint8_t *>(by_row->codes);
        a.row_scales = static_cast<uint8_t *>(by_row->scales);
    }
    if (by_col) {
        a.col_codes = static_cast<uint8_t *>(by_col->codes);
        a.col_scales = static_cast<uint8_t *>(by_col->scales);
    }
    const uint64_t groups = (uint64_t)a.col_tiles * ((rows + kTile - 1) / kTile);
    if (groups == 0) return CERAR_OK;
    if (groups > kMostThreads / kThreads) return fail(CERAR_E_INVAL, "a matrix too large for one launch");
    if (type == CERAR_F32) {
        if (format == CERAR_E4M3) launch<float, CERAR_E4M3>(a, tile, (unsigned)groups, stream);
        else launch<float, CERAR_E5M2>(a, tile, (unsigned)groups, stream);
    } else {
        if (format == CERAR_E4M3) launch<Bf16, CERAR_E4M3>(a, tile, (unsigned)groups, stream);
        else launch<Bf16, CERAR_E5M2>(a, tile, (unsigned)groups, stream);
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? CERAR_OK : fail(CERAR_E_DEVICE, "launch quantize: %s", hipGetErrorString(e));
}

}  // namespace cerar

using namespace cerar;

extern "C" int cerar_quantize_blocks(const void *x, cerar_type type, size_t rows, size_t cols, size_t ld, int tile,
                                     const cerar_blocks *by_row, const cerar_blocks *by_col, cerar_stream stream) {
    clear_error();
    if (!by_row && !by_col) return fail(CERAR_E_INVAL, "no destination");
    if ((unsigned)type > CERAR_BF16) return fail(CERAR_E_INVAL, "unknown type");
    if (rows >= (size_t)1 << 31 || cols >= (size_t)1 << 31) return fail(CERAR_E_INVAL, "x has a size of 2^31 or more");
    if (ld < cols) return fail(CERAR_E_INVAL, "ld=%zu below cols=%zu", ld, cols);
    const size_t entry = type == CERAR_F32 ? 4 : 2;
    size_t bytes;
    if (!matrix_bytes(rows, cols, ld, entry, &bytes)) return fail(CERAR_E_INVAL, "ld=%zu passes the address space", ld);
    if (bytes && !x) return fail(CERAR_E_INVAL, "NULL x");
    if (reinterpret_cast<uintptr_t>(x) % entry) return fail(CERAR_E_INVAL, "x is not aligned to its entries");
    struct Span {
        const void *p;
        size_t n;
    } spans[5] = {{x, bytes}};
    int count = 1;
    for (int k = 0; k < 2; ++k) {
        const cerar_blocks *b = k ? by_col : by_row;
        if (!b) continue;
        const char *name = k ? "by_col" : "by_row";
        const int st = check_blocks(b, name);
        if (st != CERAR_OK) return st;
        if (b->rows != (k ? cols : rows) || b->cols != (k ? rows : cols))
            return fail(CERAR_E_INVAL, "%s is %zu x %zu for x of %zu x %zu", name, b->rows, b->cols, rows, cols);
        spans[count++] = {b->codes, b->rows * blocks_ld(b->cols)};
        spans[count++] = {b->scales, b->rows * scale_groups(b->cols) * 4};
    }
    for (int i = 0; i < count; ++i)
        for (int j = 0; j < i; ++j)
            if (ranges_meet(spans[i].p, spans[i].n, spans[j].p, spans[j].n))
                return fail(CERAR_E_INVAL, "x and the destinations overlap");
    if (by_row && by_col && by_row->format != by_col->format)
        return fail(CERAR_E_INVAL, "by_row and by_col have different formats");
    return quantize(x, type, rows, cols, ld, tile != 0, by_row ? by_row->format : by_col->format, by_row, by_col,
                    reinterpret_cast<hipStream_t>(stream));
}
