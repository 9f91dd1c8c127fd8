// Products of few rows in the 8-bit block format: out = A B^T for the tokens that a
// model answers with, one or a few dozen at a time.
//
// The floor is reading B once.  Up to 16 rows of A come within a few microseconds of it
// (8192 x 2048 6.7 us a call, 16384 x 8192 36); with more, widening codes bounds them: 45 x 6145 x
// 2050 takes 12.3 us on the device, its B 1.9.  A workgroup takes 16 rows of B; its waves share out
// the blocks along K and add their results in LDS, in the waves' order.  A lane
// loads 32 bytes of one row of B for a block, four blocks at a time, straight into
// registers: with the loads of all waves in flight before the first product, K is
// as long as one trip to memory.  Codes are widened to bf16 and multiplied by
// v_mfma_f32_16x16x32_bf16, whose sums of a block are exact in fp32 but for their
// rounding; the block's scales are added to the sum's exponent.
//
// Activations are quantised into LDS by the workgroups that multiply with them, while
// their first loads of B are on their way, so that a layer is one launch that
// leaves its workspace alone.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "cerar_internal.hpp"
#include "matmul.hpp"

namespace cerar {
namespace {

constexpr int kAhead = 4;                            // blocks whose loads go out together
constexpr unsigned kMostWaves = 16;

struct FewArgs {
    const uint8_t *a;                                // codes of A, or activations
    const uint32_t *a_scales;
    const uint8_t *b;
    const uint32_t *b_scales;
    uint32_t M, N, K, blocks;
    size_t ld_a, ld_b;                               // of codes in bytes, of activations in entries
    void *out;
    size_t ld_out;
    int bf16, add;
    uint32_t waves;
};

struct Codes32 {
    v4u lo, hi;
    __device__ __forceinline__ void load(const uint8_t *p) {
        lo = reinterpret_cast<const v4u *>(p)[0];
        hi = reinterpret_cast<const v4u *>(p)[1];
    }
    // codes 8 q .. 8 q + 7
    template <int F>
    __device__ __forceinline__ v8b widen(int q) const {
        const v4u &h = q < 2 ? lo : hi;
        return widen8<F>((int)h[q % 2 * 2], (int)h[q % 2 * 2 + 1], 1.0f);
    }
};

// Where A comes from: codes, or activations of type T.
struct FromCodes {};

// The workgroup's activations to codes and scale bytes in LDS, 16 lanes to a block of a
// row: row m's block b at codes + (b M + m) 128, its scale at scales[b M + m].
template <class T>
__device__ __forceinline__ void quantize_rows(const FewArgs &g, uint8_t *codes, uint8_t *scales) {
    const uint32_t lane = threadIdx.x % 16, items = g.M * g.blocks;
    for (uint32_t k = threadIdx.x / 16; k < items; k += blockDim.x / 16) {
        const uint32_t block = k / g.M, m = k % g.M, col = block * (uint32_t)kBlock + lane * 8;
        float x[8];
        load8(reinterpret_cast<const T *>(g.a) + m * g.ld_a + col, (int)min(g.K - min(g.K, col), 8u), x);
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, magnitude(x[j]));
        const uint32_t b = scale_byte(row_max(top), kTop<CERAR_E4M3>);
        const float s = scale_inverse(b);
        *reinterpret_cast<v2u *>(codes + k * kBlock + lane * 8) =
            v2u{encode4<CERAR_E4M3>(x[0] * s, x[1] * s, x[2] * s, x[3] * s),
                encode4<CERAR_E4M3>(x[4] * s, x[5] * s, x[6] * s, x[7] * s)};
        if (lane == 0) scales[k] = (uint8_t)b;
    }
}

// Waves of one workgroup: 16 rows of B, MT times 16 rows of A, wave w the blocks w, w +
// waves, ...  A lane (r, part) holds row r and 32 columns of a block of either operand,
// and of the results row r of A and rows 4 part .. + 3 of B.
template <class S, int FA, int FB, int MT>
__global__ __launch_bounds__(1024) void k_few(FewArgs g) {
    constexpr bool kQuantize = !std::is_same_v<S, FromCodes>;
    extern __shared__ __align__(16) uint8_t lds[];
    v4f *const sums = reinterpret_cast<v4f *>(lds);
    uint8_t *const codes = lds + g.waves * MT * 1024, *const scales = codes + g.M * g.blocks * kBlock;
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, r = lane % 16, part = lane / 16;
    const uint32_t n0 = blockIdx.x * 16;
    const uint8_t *const b = g.b + min(n0 + r, g.N - 1) * g.ld_b + part * 32;
    uint32_t row[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) row[k] = min(n0 + part * 4 + k, g.N - 1);
    v4f total[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) total[t] = v4f{0, 0, 0, 0};
    Codes32 w[kAhead];
    uint32_t word[kAhead][4];
    const auto load = [&](uint32_t first) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const uint32_t block = min(first + u * g.waves, g.blocks - 1);
            w[u].load(b + (size_t)block * kBlock);
#pragma unroll
            for (int k = 0; k < 4; ++k) word[u][k] = g.b_scales[(size_t)(block / 4) * g.N + row[k]];
        }
    };
    if constexpr (kQuantize) {
        if (g.blocks) load(wave);
        quantize_rows<S>(g, codes, scales);
        __syncthreads();
    }
    for (uint32_t first = wave; first < g.blocks; first += kAhead * g.waves) {
        if (!kQuantize || first != wave) load(first);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const uint32_t block = first + u * g.waves;
            if (block >= g.blocks) break;
            v8b wide[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) wide[q] = w[u].widen<FB>(q);
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                const uint32_t m = min(t * 16 + r, g.M - 1);
                Codes32 a;
                int sa;
                if constexpr (kQuantize) {
                    a.load(codes + (block * g.M + m) * kBlock + part * 32);
                    sa = scales[block * g.M + m];
                } else {
                    a.load(g.a + m * g.ld_a + block * kBlock + part * 32);
                    sa = (int)(g.a_scales[(size_t)(block / 4) * g.M + m] >> (block % 4 * 8) & 0xFF);
                }
                v4f s = {0, 0, 0, 0};
#pragma unroll
                for (int q = 0; q < 4; ++q) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide[q], a.template widen<FA>(q), s, 0, 0, 0);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    total[t][k] += ldexpf(s[k], sa + (int)(word[u][k] >> (block % 4 * 8) & 0xFF) - 254);
            }
        }
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) sums[(wave * MT + t) * 64 + lane] = total[t];
    __syncthreads();
    for (uint32_t k = threadIdx.x; k < MT * 64; k += blockDim.x) {
        const uint32_t m = k / 64 * 16 + k % 16, n = n0 + k % 64 / 16 * 4;
        v4f s = sums[k];
        for (uint32_t w = 1; w < g.waves; ++w) s += sums[w * MT * 64 + k];
        if (m >= g.M || n >= g.N) continue;
        const int left = (int)min(g.N - n, 4u);
        float x[4] = {s[0], s[1], s[2], s[3]};
        if (g.bf16) {
            store4<false>(static_cast<Bf16 *>(g.out) + m * g.ld_out + n, left, x);
        } else {
            float *const p = static_cast<float *>(g.out) + m * g.ld_out + n;
            if (g.add) {
                float y[4];
                load4(p, left, y);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] += y[i];
            }
            store4<false>(p, left, x);
        }
    }
}

template <class S, int FA, int FB, int MT>
int start(FewArgs g, hipStream_t stream) {
    // Blocks to a wave.  Of codes one, and four where more than 16 rows share a wave's
    // widened codes of B: 1 x 8192 x 2048 takes 6.3 us, 7.3 with four, and 45 x 6145 x 2050
    // 14.6, 17.1 with one.  Of activations four, so that fewer threads quantise them at
    // once and two workgroups fit a compute unit (6.8 us, 12.3 with one), unless there are
    // fewer workgroups than compute units.
    constexpr bool kCodes = std::is_same_v<S, FromCodes>;
    const unsigned groups = (g.N + 15) / 16, each = kCodes ? (MT == 1 ? 1 : 4) : groups >= kComputeUnits ? 4 : 1;
    g.waves = std::max(1u, std::min((g.blocks + each - 1) / each, kMostWaves));
    if (groups > kMostThreads / (64 * g.waves)) return fail(CERAR_E_INVAL, "a product too large for one launch");
    const size_t lds = g.waves * MT * 1024 + (kCodes ? 0 : (size_t)g.M * g.blocks * (kBlock + 1));
    hipLaunchKernelGGL((k_few<S, FA, FB, MT>), dim3(groups), dim3(64 * g.waves), lds, stream, g);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? CERAR_OK : fail(CERAR_E_DEVICE, "launch product of few rows: %s", hipGetErrorString(e));
}

template <class S, int FA, int FB>
int start_rows(const FewArgs &g, hipStream_t stream) {
    if (g.M <= 16) return start<S, FA, FB, 1>(g, stream);
    if (g.M <= 32) return start<S, FA, FB, 2>(g, stream);
    if constexpr (std::is_same_v<S, FromCodes>) return start<S, FA, FB, 4>(g, stream);
    return fail(CERAR_E_INVAL, "too many rows");
}

template <class S, int FA>
int start_format(const FewArgs &g, cerar_fp8 fb, hipStream_t stream) {
    return fb == CERAR_E4M3 ? start_rows<S, FA, CERAR_E4M3>(g, stream) : start_rows<S, FA, CERAR_E5M2>(g, stream);
}

FewArgs args(const void *a, const void *a_scales, size_t M, size_t ld_a, const cerar_blocks &b, void *out,
             cerar_type out_type, size_t ld_out, bool add) {
    return {static_cast<const uint8_t *>(a), static_cast<const uint32_t *>(a_scales), static_cast<const uint8_t *>(b.codes),
            static_cast<const uint32_t *>(b.scales), (uint32_t)M, (uint32_t)b.rows, (uint32_t)b.cols,
            (uint32_t)(blocks_ld(b.cols) / kBlock), ld_a, blocks_ld(b.cols), out, ld_out, out_type == CERAR_BF16, add, 0};
}

}  // namespace

int matmul_few(const cerar_blocks &a, const cerar_blocks &b, void *out, cerar_type out_type, size_t ld_out, bool add,
               hipStream_t stream) {
    const FewArgs g = args(a.codes, a.scales, a.rows, blocks_ld(a.cols), b, out, out_type, ld_out, add);
    return a.format == CERAR_E4M3 ? start_format<FromCodes, CERAR_E4M3>(g, b.format, stream)
                                  : start_format<FromCodes, CERAR_E5M2>(g, b.format, stream);
}

int linear_few(const void *x, cerar_type type, size_t M, size_t ld, const cerar_blocks &w, void *out, cerar_type out_type,
               size_t ld_out, hipStream_t stream) {
    const FewArgs g = args(x, nullptr, M, ld, w, out, out_type, ld_out, false);
    return type == CERAR_F32 ? start_format<float, CERAR_E4M3>(g, w.format, stream)
                             : start_format<Bf16, CERAR_E4M3>(g, w.format, stream);
}

}  // namespace cerar
