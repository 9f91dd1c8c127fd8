// Declarations that the block products' translation units share.
#pragma once

#include <hip/hip_runtime.h>

#include "blocks.hpp"

namespace cerar {

int check_blocks(const cerar_blocks *b, const char *name);
int quantize(const void *x, cerar_type type, size_t rows, size_t cols, size_t ld, bool tile, cerar_fp8 format,
             const cerar_blocks *by_row, const cerar_blocks *by_col, hipStream_t stream);

// Products of few rows (matmul_few.hip): out = A B^T, or out and that, for A in the
// block format with at most kFewRows rows.  Against tiles of 128 x 128 over parts of K,
// fp32 sums, us a call: 64 x 2048 x 512 5.7 and 9.2, 64 x 8192 x 2048 12.5 and 17.0, 64 x 6145 x
// 2050 13.2 and 17.3; 100 x 6145 x 2050 23 and 20.  Long rows of many columns are better off
// in tiles before that: 64 x 2048 x 8192 21.6 and 20.3, 16 x 16384 x 8192 36.1 and 40.6, 32 of them
// 54 and 40, 64 of them 87 and 44.
constexpr size_t kFewRows = 64;

// Whether M x ld activations (ld: K rounded up) are quantised on the way, by each of
// the workgroups of N rows of the weight, or in a launch before.  The launch
// costs 2 to 3 us of a host's call, the way grows with the entries and with workgroups
// that share a compute unit.  Device and call, on the way against before: 1 x 8192 x
// 2048 6.1 and 6.9 against 9.8 us, 16 x 2048 x 512 5.1 and 7.2 against 5.0 and
// 9.5, 32 x 2048 x 512 7.1 and 7.2 against 6.4 and 9.5, 16 x 8192 x 512 9.8 against
// 5.6 and 9.3.
inline bool few_on_the_way(size_t M, size_t N, size_t ld) {
    return N <= 16 * kComputeUnits ? M <= 32 && M * ld <= 12288 : M <= 8 && M * ld <= 8192;
}
int matmul_few(const cerar_blocks &a, const cerar_blocks &b, void *out, cerar_type out_type, size_t ld_out, bool add,
               hipStream_t stream);
int linear_few(const void *x, cerar_type type, size_t M, size_t ld, const cerar_blocks &w, void *out, cerar_type out_type,
               size_t ld_out, hipStream_t stream);

namespace {

typedef __bf16 v8b __attribute__((ext_vector_type(8)));

// Eight codes times a power of two.
template <int F>
__device__ inline v8b widen8(int lo, int hi, float s) {
    v2b p[4];
    if (F == CERAR_E4M3) {
        p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, false);
        p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, true);
        p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, false);
        p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, true);
    } else {
        p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, s, false);
        p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, s, true);
        p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, s, false);
        p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, s, true);
    }
    return v8b{p[0][0], p[0][1], p[1][0], p[1][1], p[2][0], p[2][1], p[3][0], p[3][1]};
}

}  // namespace
}  // namespace cerar
