// Products of matrices in the 8-bit block format (blocks.hpp): out = A B^T.
//
// Fast sums go on v_mfma_scale_f32_32x32x64_f8f6f4, which multiplies 32 x 64 codes
// with 64 x 32 and applies a power of two to each operand's row as it goes: the
// blocks' scales cost nothing.  B's rows are the instruction's rows, so that a
// lane's sums are neighbours in a row of out.
//
// That instruction sums eight neighbouring products to 13 bits below the largest
// of them (measured: a term 2^-13 of its neighbour counts, one of 2^-14 does
// not), 1.5e-5 of the result for normally distributed codes.  Fp32 sums go on
// v_mfma_f32_32x32x16_bf16 instead, with codes converted on the way out of LDS:
// half the rate, 1.2e-7 of the result at K = 1000 and 4.8e-7 at 16384.  There an operand's scales are applied
// relative to the largest of its row, r, as 2^(scale - r + 32), and out takes 2^(r_a
// + r_b - 64) at the end, so that neither bf16 nor the sums leave their range: sums
// stay below 2^(16 + 16 + 64 + 31).
//
// Both are bound by the matrix cores.  Tiles of 256 x 256 in four waves of 128 x 128
// keep LDS and the L2 below them: a block of 128 along K takes 2048 cycles of matrix
// instructions, 650 of LDS reads and 1000 of loads.  Measured at M = N = K = 8192: fast
// 418 us (2630 TFLOP/s, the clock then at 1.8 GHz and the matrix cores busy for 74
// percent of its cycles), fp32 sums 852 us (1290 TFLOP/s).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <utility>

#include "cerar_internal.hpp"
#include "matmul.hpp"

namespace cerar {

namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) uint8_t LdsByte;

// f(0), ..., f(N - 1), each inlined by itself: arrays of registers are indexed by
// constants from the start.
template <class F, int... I>
__device__ __forceinline__ void each(F &&f, std::integer_sequence<int, I...>) {
    (f(I), ...);
}
template <int N, class F>
__device__ __forceinline__ void each(F &&f) {
    each(f, std::make_integer_sequence<int, N>{});
}

constexpr int kLift = 32;                            // see above

struct Operand {
    const uint8_t *codes;
    const uint32_t *scales;                          // four blocks of one row
    uint32_t rows;
};

struct MatmulArgs {
    Operand a, b;
    uint32_t blocks;                                 // of 128 along K
    size_t ld;                                       // bytes of a row of codes
    void *out;
    size_t ld_out;
    int bf16, add, past;                             // past: results of whole tiles go past the L2
    uint32_t tiles_m, tiles_n, groups;               // groups: workgroups along x
    uint32_t each;                                   // blocks of one of the parts that K is cut into, or 0
};

// Factor of a block with scale byte s in a row whose largest is r; 0 below 2^-126.
__device__ inline float relative_scale(int s, int r) { return __uint_as_float((uint32_t)max(127 + kLift + s - r, 0) << 23); }

__device__ inline __amdgpu_buffer_rsrc_t buffer(const void *p, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, (int)bytes, 0x20000);
}

// --- tiles of 64 R x 64 R through LDS -----------------------------------------------
//
// Four waves, each R x R tiles of 32 x 32.  Codes come 64 columns at a time
// ("half" a block) straight from memory to LDS, into a ring of four slots.  A
// workgroup goes through its tiles without a pause: the ring runs on into the
// next tile while the last one's results leave.
//
// A slot holds rows of 64 bytes, the 16-byte part p of row r at place p ^ (r / 4
// % 4): sixteen lanes that read the same part of sixteen rows then touch
// all 64 banks.  A wave's load fills 1 KiB in the order of its lanes, so the lanes pick
// the parts.  Rows beyond the matrix, and halves beyond the last tile, lie beyond
// the buffer and read as zeros.
constexpr int kSlots = 4;
constexpr size_t kMostK = (size_t)1 << 23;           // a tile's rows stay below kBeyond bytes
constexpr uint32_t kBeyond = 0x80000000u;            // an offset past every buffer

template <int R>
struct Lds {
    static constexpr int kRows = 64 * R;             // of a tile
    static constexpr int kSlot = kRows * 64;         // one operand's
    static constexpr int kGroup = kRows * 4;         // one operand's scales of four blocks
    static constexpr int kScales = kSlots * 2 * kSlot;
    static constexpr int kTops = kScales + kSlots * 2 * kGroup;      // multiply_f32's
    static constexpr int kEnd = kTops + 2 * kRows * 4;
    // 4 KiB a wave for the results: of their own where tiles follow each other, else in
    // the ring, so that two workgroups fit a compute unit
    static constexpr bool kApart = R == 4;
    static constexpr int kOut = kApart ? kEnd : 0;
    static constexpr int kBytes = kApart ? kEnd + 4 * 4096 : kEnd;
};

// Tile k of the grid's order: each XCD (workgroups go round them) takes a run of
// neighbouring tiles, in bands of eight rows of tiles, so that the 32 that it
// works on at a time share their operands in its L2.
__device__ inline void tile_of(uint32_t id, uint32_t tiles_m, uint32_t tiles_n, uint32_t &m, uint32_t &n) {
    const uint32_t total = tiles_m * tiles_n, xcd = id % 8, each = total / 8, more = total % 8;
    const uint32_t k = xcd * each + min(xcd, more) + id / 8;
    const uint32_t band = k / (8 * tiles_n), height = min(8u, tiles_m - band * 8), in = k - band * 8 * tiles_n;
    m = band * 8 + in % height;
    n = in / height;
}

// The halves that a workgroup multiplies, in order, over all of its tiles.
template <int R>
struct Stream {
    using L = Lds<R>;
    LdsByte *lds;
    __amdgpu_buffer_rsrc_t a, b;
    const uint8_t *sa, *sb;                          // scales of the tile's first rows, from this group of blocks on
    uint32_t rows_a, rows_b, tile, half, halves, wave, lane, at, slot, group;
    __device__ __forceinline__ void init(const MatmulArgs &g, uint8_t *to, uint32_t w, uint32_t l) {
        lds = (LdsByte *)to;
        tile = blockIdx.x, half = 0, halves = 2 * g.blocks, slot = 0, group = 0, wave = w, lane = l;
        const uint32_t row = wave * 16 + lane / 4;
        at = row * (uint32_t)g.ld + ((lane % 4) ^ row / 4 % 4) * 16;
        enter(g);
    }
    __device__ __forceinline__ bool ended(const MatmulArgs &g) const { return tile >= g.tiles_m * g.tiles_n; }
    __device__ __forceinline__ void enter(const MatmulArgs &g) {
        uint32_t tm = 0, tn = 0;
        if (!ended(g)) tile_of(tile, g.tiles_m, g.tiles_n, tm, tn);
        const uint32_t m = tm * L::kRows, n = tn * L::kRows;
        rows_a = min(g.a.rows - m, (uint32_t)L::kRows), rows_b = min(g.b.rows - n, (uint32_t)L::kRows);
        a = buffer(g.a.codes + m * g.ld, rows_a * (uint32_t)g.ld);
        b = buffer(g.b.codes + n * g.ld, rows_b * (uint32_t)g.ld);
        sa = reinterpret_cast<const uint8_t *>(g.a.scales + m);
        sb = reinterpret_cast<const uint8_t *>(g.b.scales + n);
    }
    // rows 64 i .. 64 i + 63 of this half
    __device__ __forceinline__ void load_a(const MatmulArgs &g, int i) const {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(a, lds + slot * 2 * L::kSlot + (i * 4 + wave) * 1024, 16,
                                                 at + ((ended(g) ? kBeyond : half * 64) + i * 64 * (uint32_t)g.ld), 0, 0, 0);
    }
    __device__ __forceinline__ void load_b(const MatmulArgs &g, int i) const {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(b, lds + slot * 2 * L::kSlot + L::kSlot + (i * 4 + wave) * 1024, 16,
                                                 at + ((ended(g) ? kBeyond : half * 64) + i * 64 * (uint32_t)g.ld), 0, 0, 0);
    }
    // the scale bytes of its four blocks, 64 rows a wave, with a group's first half
    __device__ __forceinline__ void load_scales(const MatmulArgs &g) {
        if (half % 8 || ended(g)) return;
        if (wave < R) {
            LdsByte *const to = lds + L::kScales + group * 2 * L::kGroup + wave * 256;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer(sa, rows_a * 4), to, 4, (wave * 64 + lane) * 4, 0, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer(sb, rows_b * 4), to + L::kGroup, 4, (wave * 64 + lane) * 4, 0, 0, 0);
        }
        sa += (size_t)g.a.rows * 4;
        sb += (size_t)g.b.rows * 4;
        group = (group + 1) % kSlots;
    }
    __device__ __forceinline__ void next(const MatmulArgs &g) {
        slot = (slot + 1) % kSlots;
        if (++half == halves) {
            half = 0;
            tile += g.groups;
            enter(g);
        }
    }
};

__device__ inline v8i lds_fragment(const uint8_t *row, uint32_t part, uint32_t key) {
    const v4u lo = *reinterpret_cast<const v4u *>(row + ((2 * part) ^ key) * 16);
    const v4u hi = *reinterpret_cast<const v4u *>(row + ((2 * part + 1) ^ key) * 16);
    return v8i{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
}

// A wave's results to out, 32 rows of 128 bytes at a time (a tile of fp32, two of
// bf16) through its 4 KiB of LDS, so that whole cache lines leave: the 16-byte part
// p of row r lies at place p ^ (r / 2 % 8).  kInside: all of the tile exists.  kPast: the
// stores go past the L2.
template <bool kBf16, bool kInside, bool kPast, int R, class F>
__device__ __forceinline__ void finish_as(const MatmulArgs &g, uint32_t m0, uint32_t n0, uint8_t *lds, uint32_t lane,
                                          const v16f (&acc)[R][R], F &&scaled) {
    constexpr int kSize = kBf16 ? 2 : 4, kPart = 16 / kSize, kTiles = 4 / kSize;
    const uint32_t r = lane % 32, h = lane / 32;
    each<R * R / kTiles>([&](int c) __attribute__((always_inline)) {
        const int i = c / (R / kTiles), j0 = c % (R / kTiles) * kTiles;
        each<kTiles>([&](int jj) __attribute__((always_inline)) {
            v16f s = acc[i][j0 + jj];
            asm volatile("" : "+v"(s));              // one tile's registers at a time
            scaled(i, j0 + jj, s);
            each<4>([&](int a) __attribute__((always_inline)) {
                const uint32_t byte = (jj * 32 + a * 8 + h * 4) * kSize;
                uint8_t *const at = lds + r * 128 + ((byte / 16) ^ (r / 2 % 8)) * 16 + byte % 16;
                if (kBf16)
                    *reinterpret_cast<v2u *>(at) = v2u{pack_bf16(s[4 * a], s[4 * a + 1]), pack_bf16(s[4 * a + 2], s[4 * a + 3])};
                else
                    *reinterpret_cast<v4f *>(at) = v4f{s[4 * a], s[4 * a + 1], s[4 * a + 2], s[4 * a + 3]};
            });
        });
        const uint32_t n = n0 + j0 * 32 + lane % 8 * kPart;
        const int left = (int)(g.b.rows - n);
        each<4>([&](int k) __attribute__((always_inline)) {
            const uint32_t row = k * 8 + lane / 8, m = m0 + i * 32 + row;
            v4u v = *reinterpret_cast<const v4u *>(lds + row * 128 + ((lane % 8) ^ (row / 2 % 8)) * 16);
            uint8_t *const p = static_cast<uint8_t *>(g.out) + ((size_t)m * g.ld_out + n) * kSize;
            if (kInside || (m < g.a.rows && left >= kPart)) {
                if (!kBf16 && g.add)
                    v = __builtin_bit_cast(v4u, __builtin_bit_cast(v4f, v) + *reinterpret_cast<const v4f_at4 *>(p));
                if (kPast) __builtin_nontemporal_store(v, reinterpret_cast<v4u_at2 *>(p));
                else *reinterpret_cast<v4u_at2 *>(p) = v;
            } else if (m < g.a.rows) {
                each<kPart>([&](int e) __attribute__((always_inline)) {
                    if (e >= left) return;
                    if (kBf16) {
                        reinterpret_cast<uint16_t *>(p)[e] = (uint16_t)(v[e / 2 % 4] >> e % 2 * 16);
                    } else {
                        float *const q = reinterpret_cast<float *>(p) + e;
                        *q = __uint_as_float(v[e % 4]) + (g.add ? *q : 0.0f);
                    }
                });
            }
        });
        __builtin_amdgcn_sched_barrier(0);
    });
}

// The results of a wave of the tile whose first row and column are m and n.
template <bool kBf16, int R, class F>
__device__ __forceinline__ void finish(const MatmulArgs &g, uint32_t m, uint32_t n, uint32_t wm, uint32_t wn, uint8_t *lds,
                                       uint32_t lane, const v16f (&acc)[R][R], F &&scaled) {
    if (m + Lds<R>::kRows > g.a.rows || n + Lds<R>::kRows > g.b.rows)
        finish_as<kBf16, false, false>(g, m + wm, n + wn, lds, lane, acc, scaled);
    else if (g.past)
        finish_as<kBf16, true, true>(g, m + wm, n + wn, lds, lane, acc, scaled);
    else
        finish_as<kBf16, true, false>(g, m + wm, n + wn, lds, lane, acc, scaled);
}

// Fast sums: v_mfma_scale_f32_32x32x64_f8f6f4.  While a half is multiplied, the next
// one's fragments are read and the half after the ring's last is fetched, an
// instruction or two between each two matrix instructions.
template <int FA, int FB, bool kBf16, int R>
__device__ __forceinline__ void multiply_fast(const MatmulArgs &g, uint8_t *lds) {
    using L = Lds<R>;
    constexpr int kPending = 2 * 2 * R;              // loads of the two slots after the next
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t r = lane % 32, part = lane / 32, key = r / 4 % 4;
    const uint32_t wm = wave / 2 * 32 * R, wn = wave % 2 * 32 * R;
    Stream<R> f;
    f.init(g, lds, wave, lane);
    const uint8_t *const la = lds + (wm + r) * 64, *const lb = lds + L::kSlot + (wn + r) * 64;
    const uint8_t *const ka = lds + L::kScales + (wm + r) * 4, *const kb = lds + L::kScales + L::kGroup + (wn + r) * 4;
#pragma unroll
    for (int h = 0; h < kSlots; ++h) {
        f.load_scales(g);
        each<R>([&](int i) __attribute__((always_inline)) {
            f.load_a(g, i);
            f.load_b(g, i);
        });
        f.next(g);
    }
    v8i a[2][R], w[2][R];
    uint32_t sa[R], sb[R];
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(3 * 2 * R) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    each<R>([&](int i) __attribute__((always_inline)) {
        a[0][i] = lds_fragment(la + i * 32 * 64, part, key);
        w[0][i] = lds_fragment(lb + i * 32 * 64, part, key);
        sa[i] = *reinterpret_cast<const uint32_t *>(ka + i * 128);
        sb[i] = *reinterpret_cast<const uint32_t *>(kb + i * 128);
    });
    uint32_t there = 0, group = 0;                   // the next half's slot, the next block's group
    for (uint32_t tile = blockIdx.x; tile < g.tiles_m * g.tiles_n; tile += g.groups) {
        v16f acc[R][R] = {};
        uint32_t b = 0;
        do {
            uint32_t ta[R], tb[R];                   // the next block's scales
            each<2>([&](int p) __attribute__((always_inline)) {
                there = (there + 1) % kSlots;
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kPending) : "memory");
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
                f.load_scales(g);
                if (p == 1 && (b % 4 == 3 || b + 1 == g.blocks)) group = (group + 1) % kSlots;
                each<R>([&](int i) __attribute__((always_inline)) {
                    each<R>([&](int j) __attribute__((always_inline)) {
                        __builtin_amdgcn_sched_barrier(0);
                        each<4 / R>([&](int u) __attribute__((always_inline)) {
                            const int k = (i * R + j) * (4 / R) + u;     // of 2 R fragments, then 2 R fetches
                            if (k < 2 * R) {
                                const uint32_t at = there * 2 * L::kSlot + k / 2 * 32 * 64;
                                if (k % 2 == 0) w[1 - p][k / 2] = lds_fragment(lb + at, part, key);
                                else a[1 - p][k / 2] = lds_fragment(la + at, part, key);
                            } else {
                                if (k % 2 == 0) f.load_a(g, k / 2 - R);
                                else f.load_b(g, k / 2 - R);
                            }
                            if (p == 1 && k < R) {
                                ta[k] = *reinterpret_cast<const uint32_t *>(ka + group * 2 * L::kGroup + k * 128);
                                tb[k] = *reinterpret_cast<const uint32_t *>(kb + group * 2 * L::kGroup + k * 128);
                            }
                        });
                        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w[p][j], a[p][i], acc[i][j], FB, FA, 0,
                                                                                    (int)sb[j], 0, (int)sa[i]);
                        asm volatile("" : "+a"(acc[i][j]));   // keeps it here
                    });
                });
                f.next(g);
                __builtin_amdgcn_sched_barrier(0);
            });
            ++b;
            const uint32_t shift = b == g.blocks ? 0 : b % 4 * 8;
            each<R>([&](int i) __attribute__((always_inline)) {
                sa[i] = ta[i] >> shift;
                sb[i] = tb[i] >> shift;
            });
        } while (b < g.blocks);
        uint32_t tm, tn;
        tile_of(tile, g.tiles_m, g.tiles_n, tm, tn);
        const uint32_t m0 = tm * L::kRows, n0 = tn * L::kRows;
        const auto as_is = [](int, int, v16f &) {};
        uint8_t *const mine = lds + L::kOut + wave * 4096;
        if (!L::kApart) __syncthreads();
        finish<kBf16>(g, m0, n0, wm, wn, mine, lane, acc, as_is);
    }
}

// The largest scale byte of each row of a tile, to LDS: row `row` by one thread.
template <int R>
__device__ __forceinline__ void top_scales(const Operand &o, uint32_t row0, uint32_t row, uint32_t blocks, int *to) {
    typedef unsigned short v2s __attribute__((ext_vector_type(2)));
    const uint32_t bytes = min(o.rows - row0, (uint32_t)Lds<R>::kRows) * 4;
    const uint8_t *p = reinterpret_cast<const uint8_t *>(o.scales + row0);
    v2s even = {0, 0}, odd = {0, 0};
#pragma unroll 8
    for (uint32_t k = 0; k < blocks; k += 4, p += (size_t)o.rows * 4) {
        const uint32_t w = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(buffer(p, bytes), row * 4, 0, 0);
        even = __builtin_elementwise_max(even, __builtin_bit_cast(v2s, w & 0x00FF00FFu));
        odd = __builtin_elementwise_max(odd, __builtin_bit_cast(v2s, w >> 8 & 0x00FF00FFu));
    }
    even = __builtin_elementwise_max(even, odd);
    to[row] = max((int)even[0], (int)even[1]);
}

// Fp32 sums: v_mfma_f32_32x32x16_bf16 on widened codes.  A half is four stages of 16
// columns; while one is multiplied, the codes of the next are widened and those of
// the one after it read.
template <int FA, int FB, bool kBf16, int R>
__device__ __forceinline__ void multiply_f32(const MatmulArgs &g, uint8_t *lds) {
    using L = Lds<R>;
    constexpr int kPending = 2 * 2 * R;              // loads of the two slots after the next
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t r = lane % 32, part = lane / 32, key = r / 4 % 4;
    const uint32_t wm = wave / 2 * 32 * R, wn = wave % 2 * 32 * R;
    uint32_t tm, tn;
    tile_of(blockIdx.x, g.tiles_m, g.tiles_n, tm, tn);
    const uint32_t m0 = tm * L::kRows, n0 = tn * L::kRows;
    v16f acc[R][R] = {};
    int ta[R] = {}, tb[R] = {};
    if (g.blocks) {
        Stream<R> f;
        f.init(g, lds, wave, lane);
        // two places of 16 bytes of the lane's rows, and its scales
        const uint8_t *const la = lds + (wm + r) * 64, *const lb = lds + L::kSlot + (wn + r) * 64;
        const uint32_t at0 = ((2 * part) ^ key) * 16, at1 = ((2 * part + 1) ^ key) * 16;
        const uint8_t *const ka = lds + L::kScales + (wm + r) * 4, *const kb = lds + L::kScales + L::kGroup + (wn + r) * 4;
#pragma unroll
        for (int h = 0; h < kSlots; ++h) {
            f.load_scales(g);
            each<R>([&](int i) __attribute__((always_inline)) {
                f.load_a(g, i);
                f.load_b(g, i);
            });
            f.next(g);
        }
        int *const tops = reinterpret_cast<int *>(lds + L::kTops);
        for (uint32_t k = threadIdx.x; k < L::kRows; k += 256) {
            top_scales<R>(g.a, m0, k, g.blocks, tops);
            top_scales<R>(g.b, n0, k, g.blocks, tops + L::kRows);
        }
        v2u raw[2][2 * R];                           // of A's rows, then of B's
        v8b wide[2][2 * R];
        float scale[2 * R], after[2 * R];            // this block's and the next one's
        __syncthreads();
        each<R>([&](int i) __attribute__((always_inline)) {
            ta[i] = tops[wm + i * 32 + r];
            tb[i] = tops[L::kRows + wn + i * 32 + r];
            each<2>([&](int q) __attribute__((always_inline)) {
                raw[q][i] = *reinterpret_cast<const v2u *>(la + i * 2048 + at0 + q * 8);
                raw[q][R + i] = *reinterpret_cast<const v2u *>(lb + i * 2048 + at0 + q * 8);
            });
            scale[i] = relative_scale((int)(*reinterpret_cast<const uint32_t *>(ka + i * 128) & 0xFF), ta[i]);
            scale[R + i] = relative_scale((int)(*reinterpret_cast<const uint32_t *>(kb + i * 128) & 0xFF), tb[i]);
            wide[0][i] = widen8<FA>((int)raw[0][i][0], (int)raw[0][i][1], scale[i]);
            wide[0][R + i] = widen8<FB>((int)raw[0][R + i][0], (int)raw[0][R + i][1], scale[R + i]);
        });
        uint32_t there = 0, group = 0, b = 0;        // the slot and the group of scales that are read from
        do {
            uint32_t word[2 * R];
            each<8>([&](int t) __attribute__((always_inline)) {
                const int q = t % 4;
                if (q == 2) {
                    there = (there + 1) % kSlots;
                    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kPending) : "memory");
                    __builtin_amdgcn_s_barrier();
                    asm volatile("" ::: "memory");
                    f.load_scales(g);
                    if (t == 6 && b % 4 == 3) group = (group + 1) % kSlots;
                }
                each<R>([&](int i) __attribute__((always_inline)) {
                    each<R>([&](int j) __attribute__((always_inline)) {
                        __builtin_amdgcn_sched_barrier(0);
                        each<4 / R>([&](int u) __attribute__((always_inline)) {
                            const int k = (i * R + j) * (4 / R) + u;     // of 2 R codes, then 2 R fetches
                            if (k < 2 * R) {
                                const uint8_t *const row = (k < R ? la : lb) + there * 2 * L::kSlot + k % R * 2048;
                                raw[t % 2][k] = *reinterpret_cast<const v2u *>(row + ((q + 2) % 4 < 2 ? at0 : at1) + q % 2 * 8);
                                if (t == 6)
                                    word[k] = *reinterpret_cast<const uint32_t *>((k < R ? ka : kb) + group * 2 * L::kGroup + k % R * 128);
                            } else if (q == 2) {
                                if (k % 2 == 0) f.load_a(g, k / 2 - R);
                                else f.load_b(g, k / 2 - R);
                            }
                            const int e = k / 2;
                            if (t == 7 && k % 2 == 0)
                                after[e] = relative_scale((int)(word[e] >> ((b + 1) % 4 * 8) & 0xFF), e < R ? ta[e % R] : tb[e % R]);
                            if (k % 2 == 1) {
                                const v2u c = raw[(t + 1) % 2][e];
                                const float s = t == 7 ? after[e] : scale[e];
                                wide[(t + 1) % 2][e] = e < R ? widen8<FA>((int)c[0], (int)c[1], s) : widen8<FB>((int)c[0], (int)c[1], s);
                            }
                        });
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wide[t % 2][R + j], wide[t % 2][i], acc[i][j], 0, 0, 0);
                        asm volatile("" : "+a"(acc[i][j]));   // keeps it here
                    });
                });
                if (q == 2) f.next(g);
                __builtin_amdgcn_sched_barrier(0);
            });
            ++b;
            each<2 * R>([&](int e) __attribute__((always_inline)) { scale[e] = after[e]; });
        } while (b < g.blocks);
    }
    uint8_t *const mine = lds + L::kOut + wave * 4096;
    if (!L::kApart) __syncthreads();
    // 2^(r_a + r_b - 64) of a lane's row and of the 16 rows of B that it has results of
    const auto scaled = [&](int i, int j, v16f &s) __attribute__((always_inline)) {
        each<16>([&](int k) __attribute__((always_inline)) {
            const int t = __shfl(tb[j], k / 4 * 8 + (int)part * 4 + k % 4);
            s[k] = ldexpf(s[k], ta[i] + t - 2 * (127 + kLift));
        });
    };
    finish<kBf16>(g, m0, n0, wm, wn, mine, lane, acc, scaled);
}

template <int FA, int FB, bool kFast, bool kBf16, int R>
__global__ __launch_bounds__(256, Lds<R>::kApart ? 1 : 2) void k_matmul(MatmulArgs g) {
    extern __shared__ __align__(1024) uint8_t lds[];
    if (g.each) {                                    // part blockIdx.y of K, to partial results of its own
        const uint32_t first = blockIdx.y * g.each;
        g.a.codes += (size_t)first * kBlock;
        g.b.codes += (size_t)first * kBlock;
        g.a.scales += (size_t)(first / 4) * g.a.rows;
        g.b.scales += (size_t)(first / 4) * g.b.rows;
        g.out = static_cast<float *>(g.out) + (size_t)blockIdx.y * g.a.rows * g.ld_out;
        g.blocks = min(g.each, g.blocks - first);
    }
    if constexpr (kFast) multiply_fast<FA, FB, kBf16, R>(g, lds);
    else multiply_f32<FA, FB, kBf16, R>(g, lds);
}

// out = the sum of the parts' results (M x N each, one after the other), in their
// order, or out and that.
template <bool kBf16>
__global__ __launch_bounds__(256) void k_join(const float *parts, uint32_t count, size_t M, size_t N, void *out, size_t ld_out,
                                              int add) {
    const size_t per_row = (N + 7) / 8, total = M * per_row;
    for (size_t k = (size_t)blockIdx.x * 256 + threadIdx.x; k < total; k += (size_t)gridDim.x * 256) {
        const size_t m = k / per_row, n = k % per_row * 8;
        const int left = (int)min(N - n, (size_t)8);
        float s[8], x[8];
        load8(parts + m * N + n, left, s);
        for (uint32_t p = 1; p < count; ++p) {
            load8(parts + p * M * N + m * N + n, left, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] += x[i];
        }
        if (kBf16) {
            store8(static_cast<Bf16 *>(out) + m * ld_out + n, left, s);
        } else {
            float *const p = static_cast<float *>(out) + m * ld_out + n;
            if (add) {
                load8(p, left, x);
#pragma unroll
                for (int i = 0; i < 8; ++i) s[i] += x[i];
            }
            store8(p, left, s);
        }
    }
}

// How a product is cut: tiles of 64 R x 64 R, and K into `parts` parts of `each`
// blocks (a multiple of four).
struct Cut {
    int R;
    uint32_t parts, each;
};

// The cut of the least time by what its pieces take: a tile's block 1.4 us on 256
// compute units at R = 4 and 1.0 us at two tiles on each at R = 2 (2.9 and 1.7 with
// fp32 sums), a tile 4 us more for its start and its results, and joining parts 5 us
// and the partial results' bytes at 4 TB/s, written and read.  Measured at M = N =
// 2048, K = 2048: 26.6 us at R = 4, 14.6 at R = 2; at 4096 cubed 58.6 and 83; a
// 1024 x 1024 result over K = 16384 63 us whole at R = 2.
inline Cut cut_of(size_t M, size_t N, size_t blocks, bool fast) {
    Cut best{4, 1, (uint32_t)blocks};
    double least = 1e300;
    for (int R = 2; R <= 4; R += 2) {
        const double tiles = (double)((M + 64 * R - 1) / (64 * R)) * (double)((N + 64 * R - 1) / (64 * R));
        const double block = fast ? (R == 4 ? 1.4 : 1.0) : (R == 4 ? 2.9 : 1.7), places = (R == 4 ? 1 : 2) * kComputeUnits;
        for (size_t parts = 1; parts <= 16; ++parts) {
            const size_t each = parts == 1 ? blocks : round_up((blocks + parts - 1) / parts, 4);
            if (parts > 1 && (parts - 1) * each >= blocks) continue;
            const double rounds = std::ceil(tiles * (double)parts / places);
            const double join = parts == 1 ? 0 : 5 + (double)parts * (double)M * (double)N * 8 / 4e6;
            const double us = rounds * ((double)each * block + 4) + join;
            if (us < least) {
                least = us;
                best = {R, (uint32_t)parts, (uint32_t)each};
            }
        }
    }
    return best;
}

template <int R>
void start(MatmulArgs g, int fa, int fb, bool fast, uint32_t parts, hipStream_t stream) {
    void (*const kernels[2][2][2][2])(MatmulArgs) = {
        {{{k_matmul<0, 0, false, false, R>, k_matmul<0, 0, false, true, R>}, {k_matmul<0, 0, true, false, R>, k_matmul<0, 0, true, true, R>}},
         {{k_matmul<0, 1, false, false, R>, k_matmul<0, 1, false, true, R>}, {k_matmul<0, 1, true, false, R>, k_matmul<0, 1, true, true, R>}}},
        {{{k_matmul<1, 0, false, false, R>, k_matmul<1, 0, false, true, R>}, {k_matmul<1, 0, true, false, R>, k_matmul<1, 0, true, true, R>}},
         {{k_matmul<1, 1, false, false, R>, k_matmul<1, 1, false, true, R>}, {k_matmul<1, 1, true, false, R>, k_matmul<1, 1, true, true, R>}}}};
    g.tiles_m = (g.a.rows + 64 * R - 1) / (64 * R);
    g.tiles_n = (g.b.rows + 64 * R - 1) / (64 * R);
    const uint32_t tiles = g.tiles_m * g.tiles_n;
    // With fast sums a workgroup for each compute unit goes through the tiles; the
    // ring, two blocks long, is then never more than one tile ahead.
    g.groups = fast && Lds<R>::kApart && g.blocks > 1 && parts == 1 ? std::min(tiles, kComputeUnits) : tiles;
    hipLaunchKernelGGL(kernels[fa][fb][fast][g.bf16], dim3(g.groups, parts), dim3(256), Lds<R>::kBytes, stream, g);
}

int matmul(const cerar_blocks &a, const cerar_blocks &b, void *out, cerar_type out_type, size_t ld_out, bool add,
           cerar_sums sums, void *ws, hipStream_t stream) {
    if (a.rows == 0 || b.rows == 0) return CERAR_OK;
    if (a.rows <= kFewRows) return matmul_few(a, b, out, out_type, ld_out, add, stream);
    MatmulArgs g{{static_cast<const uint8_t *>(a.codes), static_cast<const uint32_t *>(a.scales), (uint32_t)a.rows},
                 {static_cast<const uint8_t *>(b.codes), static_cast<const uint32_t *>(b.scales), (uint32_t)b.rows},
                 (uint32_t)(blocks_ld(a.cols) / kBlock), blocks_ld(a.cols), out, ld_out, out_type == CERAR_BF16, add, 0, 0, 0, 0, 0};
    const bool fast = sums == CERAR_SUMS_FAST && g.blocks > 0;    // no blocks: fp32 sums write the zeros
    const Cut cut = cut_of(a.rows, b.rows, g.blocks, fast);
    if ((uint64_t)((a.rows + 127) / 128) * ((b.rows + 127) / 128) > kMostThreads / 256)
        return fail(CERAR_E_INVAL, "a product too large for one launch");
    if (cut.parts > 1) {
        g.out = ws, g.ld_out = b.rows, g.bf16 = 0, g.add = 0, g.each = cut.each;
    }
    // Past the L2 where rows start on its lines, which the stores then fill: 32768 x 8192
    // x 2048 in bf16 472 us, 513 through it.  Rows that share lines, and the tiles at the
    // edge, go through it: 14149 x 5219 x 90 45 us, 115 past it.  A few such tiles lose by
    // it: 100 x 6145 x 2050 16.1 us, 15.1 past it.
    g.past = ((reinterpret_cast<uintptr_t>(g.out) | g.ld_out * (g.bf16 ? 2 : 4)) % 128) == 0;
    if (cut.R == 4) start<4>(g, a.format, b.format, fast, cut.parts, stream);
    else start<2>(g, a.format, b.format, fast, cut.parts, stream);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && cut.parts > 1) {
        const size_t pieces = a.rows * ((b.rows + 7) / 8);
        hipLaunchKernelGGL(out_type == CERAR_BF16 ? k_join<true> : k_join<false>,
                           dim3((unsigned)std::min<size_t>((pieces + 255) / 256, 2048)), dim3(256), 0, stream,
                           static_cast<const float *>(ws), cut.parts, a.rows, b.rows, out, ld_out, (int)add);
        e = hipGetLastError();
    }
    return e == hipSuccess ? CERAR_OK : fail(CERAR_E_DEVICE, "launch matmul: %s", hipGetErrorString(e));
}

// The partial results' part of a call's workspace, for either kind of sums.
size_t parts_bytes(size_t M, size_t N, size_t K) {
    if (M <= kFewRows || !N) return 0;
    const size_t blocks = blocks_ld(K) / kBlock;
    const uint32_t a = cut_of(M, N, blocks, true).parts, b = cut_of(M, N, blocks, false).parts, most = std::max(a, b);
    return most > 1 ? round_up(most * M * N * 4, 16) : 0;
}

struct Span {
    const void *p;
    size_t n;
    const char *name;
};

int check_product(size_t M, size_t N, const cerar_blocks *b, void *out, cerar_type out_type, size_t ld_out, cerar_sums sums,
                  void *ws, size_t ws_bytes, Span (&spans)[6], int used) {
    if ((unsigned)out_type > CERAR_BF16) return fail(CERAR_E_INVAL, "unknown out_type");
    if ((unsigned)sums > CERAR_SUMS_FAST) return fail(CERAR_E_INVAL, "unknown sums");
    if (M >= (size_t)1 << 31) return fail(CERAR_E_INVAL, "a size of 2^31 or more");
    const size_t entry = out_type == CERAR_F32 ? 4 : 2;
    size_t bytes;
    if (!matrix_bytes(M, N, ld_out, entry, &bytes)) return fail(CERAR_E_INVAL, "ld_out=%zu passes the address space", ld_out);
    if (M && N) {
        if (!out) return fail(CERAR_E_INVAL, "NULL out");
        if (ld_out < N) return fail(CERAR_E_INVAL, "ld_out=%zu below N=%zu", ld_out, N);
        if (reinterpret_cast<uintptr_t>(out) % entry) return fail(CERAR_E_INVAL, "out is not aligned to its entries");
        if (ws_bytes && !ws) return fail(CERAR_E_INVAL, "NULL ws, %zu bytes are needed", ws_bytes);
        if (ws_bytes && reinterpret_cast<uintptr_t>(ws) % 16) return fail(CERAR_E_INVAL, "ws is not 16-byte aligned");
    }
    spans[used++] = {b->codes, b->rows * blocks_ld(b->cols), "b"};
    spans[used++] = {b->scales, b->rows * scale_groups(b->cols) * 4, "b"};
    const Span written[2] = {{out, bytes, "out"}, {ws, ws_bytes, "ws"}};
    for (const Span &w : written)
        for (int i = 0; i < used; ++i)
            if (ranges_meet(w.p, w.n, spans[i].p, spans[i].n)) return fail(CERAR_E_INVAL, "%s and %s overlap", w.name, spans[i].name);
    if (ranges_meet(written[0].p, written[0].n, written[1].p, written[1].n)) return fail(CERAR_E_INVAL, "out and ws overlap");
    return CERAR_OK;
}

// The quantised activations' part of a linear call's workspace.
size_t linear_codes(size_t M, size_t K) { return round_up(M * blocks_ld(K), 16); }
size_t linear_scales(size_t M, size_t K) { return round_up(M * scale_groups(K) * 4, 16); }

}  // namespace
}  // namespace cerar

using namespace cerar;

extern "C" int cerar_matmul_workspace_bytes(size_t M, size_t N, size_t K, int linear, size_t *bytes) {
    clear_error();
    if (!bytes) return fail(CERAR_E_INVAL, "NULL argument");
    if ((M | N) >> 31) return fail(CERAR_E_INVAL, "a size of 2^31 or more");
    if (K >= kMostK) return fail(CERAR_E_INVAL, "K=%zu: less than 2^23 is needed", K);
    *bytes = parts_bytes(M, N, K) + (linear ? linear_codes(M, K) + linear_scales(M, K) : 0);
    return CERAR_OK;
}

extern "C" int cerar_matmul_blocks(const cerar_blocks *a, const cerar_blocks *b, void *out, cerar_type out_type,
                                   size_t ld_out, int accumulate, cerar_sums sums, void *ws, cerar_stream stream) {
    clear_error();
    if (!a || !b) return fail(CERAR_E_INVAL, "NULL argument");
    int st = check_blocks(a, "a");
    if (st == CERAR_OK) st = check_blocks(b, "b");
    if (st != CERAR_OK) return st;
    if (a->cols != b->cols) return fail(CERAR_E_INVAL, "a has %zu columns, b %zu", a->cols, b->cols);
    if (accumulate && out_type != CERAR_F32) return fail(CERAR_E_INVAL, "accumulate needs an fp32 out");
    size_t ws_bytes = 0;
    if ((st = cerar_matmul_workspace_bytes(a->rows, b->rows, a->cols, 0, &ws_bytes)) != CERAR_OK) return st;
    Span spans[6] = {{a->codes, a->rows * blocks_ld(a->cols), "a"}, {a->scales, a->rows * scale_groups(a->cols) * 4, "a"}};
    st = check_product(a->rows, b->rows, b, out, out_type, ld_out, sums, ws, ws_bytes, spans, 2);
    if (st != CERAR_OK) return st;
    return matmul(*a, *b, out, out_type, ld_out, accumulate != 0, sums, ws, reinterpret_cast<hipStream_t>(stream));
}

extern "C" int cerar_linear_blocks(const void *x, cerar_type type, size_t M, size_t ld, const cerar_blocks *w, void *out,
                                   cerar_type out_type, size_t ld_out, cerar_sums sums, void *ws,
                                   cerar_stream stream) {
    clear_error();
    if (!w) return fail(CERAR_E_INVAL, "NULL argument");
    int st = check_blocks(w, "w");
    if (st != CERAR_OK) return st;
    const size_t K = w->cols, entry = type == CERAR_F32 ? 4 : 2;
    if ((unsigned)type > CERAR_BF16) return fail(CERAR_E_INVAL, "unknown type");
    if (ld < K) return fail(CERAR_E_INVAL, "ld=%zu below cols=%zu", ld, K);
    size_t x_bytes;
    if (!matrix_bytes(M, K, ld, entry, &x_bytes)) return fail(CERAR_E_INVAL, "ld=%zu passes the address space", ld);
    if (x_bytes && !x) return fail(CERAR_E_INVAL, "NULL x");
    if (reinterpret_cast<uintptr_t>(x) % entry) return fail(CERAR_E_INVAL, "x is not aligned to its entries");
    size_t ws_bytes = 0;
    if ((st = cerar_matmul_workspace_bytes(M, w->rows, K, 1, &ws_bytes)) != CERAR_OK) return st;
    Span spans[6] = {{x, x_bytes, "x"}};
    st = check_product(M, w->rows, w, out, out_type, ld_out, sums, ws, ws_bytes, spans, 1);
    if (st != CERAR_OK || M == 0 || w->rows == 0) return st;
    const hipStream_t hs = reinterpret_cast<hipStream_t>(stream);
    if (few_on_the_way(M, w->rows, blocks_ld(K))) return linear_few(x, type, M, ld, *w, out, out_type, ld_out, hs);
    char *const codes = static_cast<char *>(ws) + parts_bytes(M, w->rows, K);
    const cerar_blocks a{codes, codes + linear_codes(M, K), M, K, CERAR_E4M3};
    st = quantize(x, type, M, K, ld, false, CERAR_E4M3, &a, nullptr, hs);
    return st == CERAR_OK ? matmul(a, *w, out, out_type, ld_out, false, sums, ws, hs) : st;
}
