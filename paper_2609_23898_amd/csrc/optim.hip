// The gradient norm and the AdamW step over all tensors of a model.
//
// Both stream: every entry is read once and every state written once, so the
// bound is memory.  A set's tensors are cut into pieces of a few thousand entries
// on the host; a workgroup looks its piece and the piece's tensor up in tables, so
// that hundreds of tensors of any lengths go in one launch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <limits>
#include <memory>
#include <vector>

#include "blocks.hpp"
#include "cerar_internal.hpp"

namespace cerar {
namespace {

constexpr int kThreads = 256;
constexpr int kPerThread = 4;                        // a block of 128 entries is half a wave
constexpr int kSweep = kThreads * kPerThread;        // entries that a workgroup takes at a time
constexpr unsigned kPieceShift = 3;                   // of a piece's sweeps at most
constexpr int kPlaces = 2048;                        // workgroups that the card holds at a time, about
constexpr int kNormGroups = 2 * kComputeUnits;       // workgroups of the norm at most

struct Piece {
    uint32_t tensor, sweeps;
    uint64_t first;                                  // entry of its tensor, a multiple of the block
};

struct Entry {
    cerar_tensor t;
    uint64_t place;                                  // its first entry's place in the set, a multiple of the block
};

}  // namespace
}  // namespace cerar

struct cerar_tensors {
    int device = 0, state_bits = 0;
    unsigned pieces = 0, shift = 0;                  // a piece has at most 2^shift sweeps
    cerar::Entry *entries = nullptr;
    cerar::Piece *table = nullptr;
    double *partial = nullptr;                       // of the norm's workgroups
};

namespace cerar {
namespace {

int hip_failed(hipError_t e, const char *what) {
    return fail(e == hipErrorOutOfMemory ? CERAR_E_NOMEM : CERAR_E_DEVICE, "%s: %s", what, hipGetErrorString(e));
}

// --- norm ----------------------------------------------------------------------

// How many of the entries from `at` on a tensor of n has, at most a lane's.
__device__ inline int entries_left(uint64_t n, uint64_t at) {
    return n >= at + kPerThread ? kPerThread : n > at ? (int)(n - at) : 0;
}

// Squares of a piece's entries; where all of its sweeps are whole, kFlight loads go
// out together.
template <class G>
__device__ inline double squares(const G *g, uint64_t n, uint64_t at, unsigned sweeps) {
    constexpr unsigned kFlight = 8;
    double s = 0.0;
    unsigned k = 0;
    if (at - threadIdx.x * kPerThread + (uint64_t)sweeps * kSweep <= n) {
        for (; k + kFlight <= sweeps; k += kFlight, at += kFlight * kSweep) {
            float x[kFlight][4];
#pragma unroll
            for (unsigned f = 0; f < kFlight; ++f) load4(g + at + f * kSweep, 4, x[f]);
#pragma unroll
            for (unsigned f = 0; f < kFlight; ++f)
#pragma unroll
                for (int j = 0; j < 4; ++j) s = fma((double)x[f][j], (double)x[f][j], s);
        }
    }
    for (; k < sweeps; ++k, at += kSweep) {
        float x[4];
        load4(g + at, entries_left(n, at), x);
#pragma unroll
        for (int j = 0; j < 4; ++j) s = fma((double)x[j], (double)x[j], s);
    }
    return s;
}

__device__ inline double group_sum(double s, double *lds) {
#pragma unroll
    for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = s;
    __syncthreads();
    s = lds[0] + lds[1] + lds[2] + lds[3];
    __syncthreads();
    return s;
}

// Sum of squares in 64 bits: no finite fp32 gradient overflows it and the result
// rounds once.  Each workgroup's pieces and the order in which their sums are added
// are fixed, so the bits are too.  The sums are added in a launch of their own: a
// count of the workgroups that have arrived, for the last one to add, took 25 ns
// for each of them.
__global__ __launch_bounds__(kThreads) void k_squares(const Entry *entries, const Piece *table, unsigned pieces, double *partial) {
    __shared__ double lds[4];
    double s = 0.0;
    for (unsigned p = blockIdx.x; p < pieces; p += gridDim.x) {
        const Piece w = table[p];
        const Entry &e = entries[w.tensor];
        const uint64_t at = w.first + threadIdx.x * kPerThread;
        if (e.t.grad_type == CERAR_F32) s += squares(static_cast<const float *>(e.t.grad), e.t.n, at, w.sweeps);
        else s += squares(static_cast<const Bf16 *>(e.t.grad), e.t.n, at, w.sweeps);
    }
    s = group_sum(s, lds);
    if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

__global__ __launch_bounds__(kThreads) void k_grad_norm(const double *partial, unsigned count, float grad_scale, float max_norm,
                                                        float *clip) {
    __shared__ double lds[4];
    double s = 0.0;
    for (unsigned k = threadIdx.x; k < count; k += kThreads) s += partial[k];
    s = group_sum(s, lds);
    if (threadIdx.x == 0) {
        const double n = (double)grad_scale * sqrt(s);
        clip[0] = (float)n;
        clip[1] = n > (double)max_norm ? (float)((double)max_norm / n) : 1.0f;
    }
}

// --- AdamW ---------------------------------------------------------------------

constexpr uint64_t kGolden = 0x9E3779B97F4A7C15ull;

// The splitmix64 finaliser (Steele, Lea & Flood, OOPSLA 2014).
__host__ __device__ inline uint64_t mixed(uint64_t z) {
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}

// Codes of magnitudes rounded to a neighbour by chance: r of 2^16 parts are added to
// the bits below the mantissa that stays, and the rest is cut off.  Below the
// smallest normal number the format's spacing is that of its first binade, where
// adding that number puts them.
template <int F>
struct Chance {
    static constexpr int kDrop = F == CERAR_E4M3 ? 20 : 21;                 // bits of an fp32 mantissa that go
    static constexpr uint32_t kFields = F == CERAR_E4M3 ? 120 : 112;        // difference of the exponents' biases
    static constexpr float kLow = F == CERAR_E4M3 ? 0x1p-6f : 0x1p-14f;     // smallest normal number
};

template <int F>
__device__ inline uint32_t any_code(float a, uint32_t r) {
    using C = Chance<F>;
    const bool small = a < C::kLow;
    const uint32_t t = __float_as_uint(small ? a + C::kLow : a) - ((small ? C::kFields + 1 : C::kFields) << 23);
    uint32_t code = (t + (r << (C::kDrop - 16))) >> C::kDrop;
    if (F == CERAR_E5M2) code = __builtin_isfpclass(a, 0x200) ? 0x7Cu : code;    // infinite, where the format has it
    return __builtin_isfpclass(a, F == CERAR_E5M2 ? 0x3 : 0x203) ? 0x7Fu : code;   // NaN
}

// A lane's states, magnitudes in a (fp32 bits) and signs in the top bits of
// sign, with the others of their block, to codes and the block's scale.  Where all
// of a wave's are normal numbers of the format, the scale is an addition to their
// exponents.
template <int F>
__device__ inline void store_codes(uint8_t *codes, uint8_t *scale, int left, const uint32_t (&a)[4], const uint32_t (&sign)[4],
                                   const uint32_t (&r)[4]) {
    using C = Chance<F>;
    uint32_t top = 0, least = 0xFFFFFFFFu, w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        top = max(top, a[j]);
        least = min(least, a[j]);
    }
    uint32_t b = scale_byte(half_max(top), kTop<F>);
    constexpr uint32_t low = C::kFields + 1;                                   // its exponent
    const uint32_t normal = max((low + b - 127u) << 23, 0x800000u);          // low + b - 127 may pass below zero
    if (__all(least >= normal && (int)(low + b - 127u) >= 0 && top < 0x7F800000u)) {
        const uint32_t shift = (127u - b - C::kFields) << 23;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = (a[j] + (r[j] << (C::kDrop - 16)) + shift) >> C::kDrop;
    } else {
        top = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) top = max(top, a[j] < 0x7F800000u ? a[j] : 0u);
        b = scale_byte(half_max(top), kTop<F>);
        const float inv = scale_inverse(b);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float x = __uint_as_float(a[j]) * inv;
            w[j] = any_code<F>(x, r[j]);
            // squares: what has moved stays above zero, also where x is too small for fp32
            if (F == CERAR_E5M2) w[j] = max(w[j], x > 0.0f || a[j] >= 0x800000u ? 1u : 0u);
        }
    }
    uint32_t word = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (F == CERAR_E4M3) w[j] |= sign[j] >> 24 & 0x80u;
        word |= w[j] << (8 * j);
    }
    store4(codes, left, word);
    if (threadIdx.x % 32 == 0 && left > 0) *scale = (uint8_t)b;
}

// Magnitude of an fp64 value as fp32 bits, cut off: what goes lies below the last of
// the 16 places that a code's rounding compares, so the code is that of the fp64
// value.  The conversion rounds subnormal numbers only; from 2^128 on it gives infinity,
// as rounding does for 32-bit states.
__device__ inline uint32_t cut_off(double x) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x) & 0x7FFFFFFFE0000000ull;
    return __float_as_uint((float)__builtin_bit_cast(double, u));
}

// A workgroup's sweep.  The averages are formed in fp64 and rounded once.  sqrt and
// the reciprocal are the hardware's, one unit in the last place each; v below 2^-126
// counts as 0 in the step.  The decay is added to the rest of the step: 1 - decay has no
// more than 24 bits in fp32, an error of one sign at every step (at a decay of 5e-7 4.6
// percent of it, below 3e-8 all).  With kWhole all of its entries exist: no branch is left
// around its loads and stores, which takes 33 million bf16 entries with 8-bit states
// from 97 us to 78.  Fp32 states, which memory alone bounds, keep the branches: 405
// million entries 1.86 ms, 1.93 without.
template <class P, class G, bool kEight, bool kWhole>
__device__ __forceinline__ void adamw_sweep(const Entry &e, uint64_t at, const cerar_adamw_values &h, float gs) {
    const float decay = h.lr * e.t.lr_scale * e.t.weight_decay, size = h.step_size * e.t.lr_scale;
    const double to_m = h.rest1 * (double)gs, to_v = h.rest2 * ((double)gs * (double)gs);
    const int left = kWhole ? kPerThread : entries_left(e.t.n, at);
    float p[4], g[4], m[4], v[4];
    uint32_t am[4], av[4], sm[4];                    // magnitudes and signs of 8-bit states
    load4(static_cast<const G *>(e.t.grad) + at, left, g);
    load4(static_cast<const P *>(e.t.param) + at, left, p);
    if (kEight) {
        const uint64_t b = left > 0 ? at / kBlock : 0;
        decode4<CERAR_E4M3>(load4(static_cast<const uint8_t *>(e.t.m) + at, left), e.t.m_scale[b], m);
        decode4<CERAR_E5M2>(load4(static_cast<const uint8_t *>(e.t.v) + at, left), e.t.v_scale[b], v);
    } else {
        load4(static_cast<const float *>(e.t.m) + at, left, m);
        load4(static_cast<const float *>(e.t.v) + at, left, v);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const double x = (double)g[j];
        const double dm = fma(x, to_m, (double)m[j] * h.beta1), dv = fma(x * x, to_v, (double)v[j] * h.beta2);
        if (kEight) {
            am[j] = cut_off(dm);
            av[j] = cut_off(dv);
            sm[j] = (uint32_t)(__builtin_bit_cast(uint64_t, dm) >> 32);
            m[j] = __uint_as_float(am[j] | (sm[j] & 0x80000000u));
            v[j] = __uint_as_float(av[j]);
        } else {
            m[j] = (float)dm;
            v[j] = (float)dv;
        }
        const float move = size * m[j] * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(v[j]) * h.root2 + h.eps);
        p[j] -= fmaf(decay, p[j], move);
    }
    store4(static_cast<P *>(e.t.param) + at, left, p);
    if (e.t.copy) store4(static_cast<Bf16 *>(e.t.copy) + at, left, p);
    if (kEight) {
        uint32_t rm[4], rv[4];
        const uint64_t pair = h.key + ((e.place + at) / 2 + 1) * kGolden;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint64_t z = mixed(pair + j * kGolden);
            rm[2 * j] = (uint32_t)z & 0xFFFFu;
            rv[2 * j] = (uint32_t)z >> 16;
            rm[2 * j + 1] = (uint32_t)(z >> 32) & 0xFFFFu;
            rv[2 * j + 1] = (uint32_t)(z >> 48);
        }
        store_codes<CERAR_E4M3>(static_cast<uint8_t *>(e.t.m) + at, e.t.m_scale + at / kBlock, left, am, sm, rm);
        store_codes<CERAR_E5M2>(static_cast<uint8_t *>(e.t.v) + at, e.t.v_scale + at / kBlock, left, av, av, rv);
    } else {
        store4(static_cast<float *>(e.t.m) + at, left, m);
        store4(static_cast<float *>(e.t.v) + at, left, v);
    }
}

template <class P, class G, bool kEight>
__device__ inline void adamw(const Entry &e, uint64_t first, const cerar_adamw_values &h, float gs) {
    const uint64_t at = first + threadIdx.x * kPerThread;
    if (kEight && first + kSweep <= e.t.n) adamw_sweep<P, G, kEight, true>(e, at, h, gs);
    else adamw_sweep<P, G, kEight, false>(e, at, h, gs);
}

// A workgroup takes one sweep, of the 2^shift of a piece: neighbouring workgroups then
// work on neighbouring memory and none waits for its own loads twice (405 million
// entries with fp32 states 1.86 ms, 2.20 in whole pieces of eight; 182 million
// with 8-bit ones 525 us, 587 in fours with the next one's loads ahead).
template <bool kEight>
__global__ __launch_bounds__(kThreads) void k_adamw(const Entry *entries, const Piece *table, unsigned shift,
                                                    cerar_adamw_values given, const cerar_adamw_values *kept, const float *clip) {
    const cerar_adamw_values h = kept ? *kept : given;
    float gs = h.grad_scale;
    if (clip) {
        if ((__float_as_uint(clip[0]) & 0x7FFFFFFFu) >= 0x7F800000u) return;
        gs *= clip[1];
    }
    const unsigned part = blockIdx.x & ((1u << shift) - 1);
    const Piece w = table[blockIdx.x >> shift];
    if (part >= w.sweeps) return;
    const uint64_t first = w.first + (uint64_t)part * kSweep;
    const Entry e = entries[w.tensor];               // a copy: stores of bytes would have it read again
    if (e.t.param_type == CERAR_F32) {
        if (e.t.grad_type == CERAR_F32) adamw<float, float, kEight>(e, first, h, gs);
        else adamw<float, Bf16, kEight>(e, first, h, gs);
    } else {
        if (e.t.grad_type == CERAR_F32) adamw<Bf16, float, kEight>(e, first, h, gs);
        else adamw<Bf16, Bf16, kEight>(e, first, h, gs);
    }
}

// --- host ------------------------------------------------------------------------

struct Range {
    uintptr_t first, end;
    bool written;
    int tensor;
    const char *name;
};

int check_tensors(int count, const cerar_tensor *tensors, int state_bits) {
    std::vector<Range> all;
    uint64_t total = 0;
    for (int i = 0; i < count; ++i) {
        const cerar_tensor &t = tensors[i];
        if (t.n > (size_t)1 << 40 || (total += round_up(t.n, kBlock)) > (uint64_t)1 << 40)
            return fail(CERAR_E_INVAL, "more than 2^40 entries");
        if ((unsigned)t.grad_type > CERAR_BF16 || (state_bits && (unsigned)t.param_type > CERAR_BF16))
            return fail(CERAR_E_INVAL, "tensor %d: unknown type", i);
        if (t.n == 0) continue;
        const size_t state = state_bits == 8 ? 1 : 4, blocks = (t.n + kBlock - 1) / kBlock;
        const struct {
            const void *p;
            size_t entry, n;
            bool written, needed;
            const char *name;
        } buffers[] = {{t.grad, (size_t)(t.grad_type == CERAR_BF16 ? 2 : 4), t.n, false, true, "grad"},
                       {t.param, (size_t)(t.param_type == CERAR_BF16 ? 2 : 4), t.n, true, state_bits != 0, "param"},
                       {t.m, state, t.n, true, state_bits != 0, "m"},
                       {t.v, state, t.n, true, state_bits != 0, "v"},
                       {t.m_scale, 1, blocks, true, state_bits == 8, "m_scale"},
                       {t.v_scale, 1, blocks, true, state_bits == 8, "v_scale"},
                       {t.copy, 2, t.n, true, false, "copy"}};
        for (const auto &b : buffers) {
            if (!b.needed && (!b.p || state_bits == 0)) continue;
            if (!b.p) return fail(CERAR_E_INVAL, "tensor %d: %s is NULL", i, b.name);
            if (!b.needed && b.entry == 1) return fail(CERAR_E_INVAL, "tensor %d: %s without 8-bit states", i, b.name);
            const uintptr_t a = reinterpret_cast<uintptr_t>(b.p);
            if (a % b.entry) return fail(CERAR_E_INVAL, "tensor %d: %s is not aligned to its entries", i, b.name);
            all.push_back({a, a + b.entry * b.n, b.written, i, b.name});
        }
        if (state_bits && (!std::isfinite(t.lr_scale) || !std::isfinite(t.weight_decay)))
            return fail(CERAR_E_INVAL, "tensor %d: lr_scale or weight_decay is not finite", i);
    }
    std::sort(all.begin(), all.end(), [](const Range &a, const Range &b) { return a.first < b.first; });
    // the range that reaches furthest so far, of all and of the written ones
    const Range *far = nullptr, *far_written = nullptr;
    for (const Range &r : all) {
        const Range *with = r.written ? far : far_written;
        if (with && with->end > r.first)
            return fail(CERAR_E_INVAL, "tensor %d's %s and tensor %d's %s overlap", with->tensor, with->name, r.tensor, r.name);
        if (!far || r.end > far->end) far = &r;
        if (r.written && (!far_written || r.end > far_written->end)) far_written = &r;
    }
    return CERAR_OK;
}

void release(cerar_tensors *s) {
    int cur = 0;
    const bool have = hipGetDevice(&cur) == hipSuccess;
    if (have) (void)hipSetDevice(s->device);
    (void)hipFree(s->entries);
    (void)hipFree(s->table);
    (void)hipFree(s->partial);
    if (have) (void)hipSetDevice(cur);
    delete s;
}

struct Release {
    void operator()(cerar_tensors *s) const { release(s); }
};

template <class T>
int put(T **dst, const std::vector<T> &src) {
    hipError_t e = hipMalloc((void **)dst, std::max<size_t>(1, src.size()) * sizeof(T));
    if (e != hipSuccess) return hip_failed(e, "hipMalloc (tensor table)");
    if (src.empty()) return CERAR_OK;
    e = hipMemcpy(*dst, src.data(), src.size() * sizeof(T), hipMemcpyHostToDevice);
    return e == hipSuccess ? CERAR_OK : hip_failed(e, "hipMemcpy (tensor table)");
}

int on_its_device(const cerar_tensors *set) {
    int dev = 0;
    const hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return hip_failed(e, "hipGetDevice");
    if (dev != set->device) return fail(CERAR_E_INVAL, "the set is on device %d, the current device is %d", set->device, dev);
    return CERAR_OK;
}

}  // namespace
}  // namespace cerar

using namespace cerar;

extern "C" int cerar_tensors_create(int count, const cerar_tensor *tensors, int state_bits, cerar_tensors **out) {
    clear_error();
    return guarded([&]() -> int {
        if (!tensors || !out) return fail(CERAR_E_INVAL, "NULL argument");
        *out = nullptr;
        if (count < 1 || count > 1 << 20) return fail(CERAR_E_INVAL, "count=%d outside [1, 2^20]", count);
        if (state_bits != 0 && state_bits != 8 && state_bits != 32)
            return fail(CERAR_E_INVAL, "state_bits=%d is none of 0, 8, 32", state_bits);
        int st = check_tensors(count, tensors, state_bits);
        if (st != CERAR_OK) return st;

        uint64_t sweeps = 0;
        for (int i = 0; i < count; ++i) sweeps += (tensors[i].n + kSweep - 1) / kSweep;
        const uint64_t groups = kMostThreads / kThreads;             // that one launch takes
        if (state_bits && sweeps > groups) return fail(CERAR_E_INVAL, "more entries than one launch takes");
        // Pieces of one sweep until that fills the card's places, of up to 2^kPieceShift beyond.
        unsigned shift = 0;
        while (shift < kPieceShift && sweeps >> (shift + 1) >= kPlaces) ++shift;
        const uint64_t most = (uint64_t)1 << shift;
        std::vector<Entry> entries(count);
        std::vector<Piece> table;
        uint64_t place = 0;
        for (int i = 0; i < count; ++i) {
            entries[i] = {tensors[i], place};
            place += round_up(tensors[i].n, kBlock);
            for (uint64_t first = 0; first < tensors[i].n; first += most * kSweep) {
                const uint64_t here = (tensors[i].n - first + kSweep - 1) / kSweep;
                table.push_back({(uint32_t)i, (uint32_t)std::min(most, here), first});
            }
        }
        if (state_bits && (uint64_t)table.size() << shift > groups) return fail(CERAR_E_INVAL, "more entries than one launch takes");

        std::unique_ptr<cerar_tensors, Release> s(new cerar_tensors);
        hipError_t e = hipGetDevice(&s->device);
        if (e != hipSuccess) return hip_failed(e, "hipGetDevice");
        s->state_bits = state_bits;
        s->pieces = (unsigned)table.size();
        s->shift = shift;
        if ((st = put(&s->entries, entries)) != CERAR_OK) return st;
        if ((st = put(&s->table, table)) != CERAR_OK) return st;
        if ((st = put(&s->partial, std::vector<double>(kNormGroups, 0.0))) != CERAR_OK) return st;
        *out = s.release();
        return CERAR_OK;
    });
}

extern "C" void cerar_tensors_destroy(cerar_tensors *set) {
    if (set) release(set);
}

extern "C" int cerar_grad_norm(const cerar_tensors *set, float grad_scale, float max_norm, float *clip,
                               cerar_stream stream) {
    clear_error();
    if (!set || !clip) return fail(CERAR_E_INVAL, "NULL argument");
    if (!(grad_scale > 0.0f) || !std::isfinite(grad_scale)) return fail(CERAR_E_INVAL, "grad_scale=%g", (double)grad_scale);
    if (!(max_norm > 0.0f)) return fail(CERAR_E_INVAL, "max_norm=%g", (double)max_norm);
    const int st = on_its_device(set);
    if (st != CERAR_OK) return st;
    const unsigned groups = std::min<unsigned>(set->pieces, kNormGroups);
    const hipStream_t hs = reinterpret_cast<hipStream_t>(stream);
    hipError_t e = hipSuccess;
    if (groups) {
        hipLaunchKernelGGL(k_squares, dim3(groups), dim3(kThreads), 0, hs, set->entries, set->table, set->pieces, set->partial);
        e = hipGetLastError();
    }
    if (e == hipSuccess) {
        hipLaunchKernelGGL(k_grad_norm, dim3(1), dim3(kThreads), 0, hs, set->partial, groups, grad_scale, max_norm, clip);
        e = hipGetLastError();
    }
    return e == hipSuccess ? CERAR_OK : hip_failed(e, "launch gradient norm");
}

extern "C" int cerar_adamw_pack(const cerar_adamw *h, cerar_adamw_values *v) {
    clear_error();
    if (!h || !v) return fail(CERAR_E_INVAL, "NULL argument");
    if (h->step == 0) return fail(CERAR_E_INVAL, "step=0: the first step is 1");
    if (!(h->beta1 >= 0 && h->beta1 < 1) || !(h->beta2 >= 0 && h->beta2 < 1))
        return fail(CERAR_E_INVAL, "beta1=%g or beta2=%g outside [0, 1)", h->beta1, h->beta2);
    const double t = (double)h->step;
    const cerar_adamw_values w = {h->beta1, 1.0 - h->beta1, h->beta2, 1.0 - h->beta2, mixed(h->seed + (h->step + 1) * kGolden),
          (float)h->lr, (float)h->eps, (float)h->grad_scale, (float)(h->lr / (1.0 - std::pow(h->beta1, t))),
          (float)(1.0 / std::sqrt(1.0 - std::pow(h->beta2, t))), 0.0f};
    // the step divides by eps where v is 0: a normal fp32 number
    if (!(w.eps >= std::numeric_limits<float>::min()) || !std::isfinite(w.eps)) return fail(CERAR_E_INVAL, "eps=%g", h->eps);
    if (!std::isfinite(w.lr) || !std::isfinite(w.grad_scale) || !std::isfinite(w.step_size) || !std::isfinite(w.root2))
        return fail(CERAR_E_INVAL, "lr, grad_scale or the bias corrections leave fp32's range");
    *v = w;
    return CERAR_OK;
}

extern "C" int cerar_adamw_step(const cerar_tensors *set, const cerar_adamw *hyper, const cerar_adamw_values *values,
                                const float *clip, cerar_stream stream) {
    clear_error();
    if (!set) return fail(CERAR_E_INVAL, "NULL argument");
    if (!hyper == !values) return fail(CERAR_E_INVAL, "exactly one of hyper and values is needed");
    if (set->state_bits == 0) return fail(CERAR_E_INVAL, "the set was made for gradients alone");
    cerar_adamw_values given{};
    int st = hyper ? cerar_adamw_pack(hyper, &given) : CERAR_OK;
    if (st == CERAR_OK) st = on_its_device(set);
    if (st != CERAR_OK || set->pieces == 0) return st;
    const auto kernel = set->state_bits == 8 ? k_adamw<true> : k_adamw<false>;
    hipLaunchKernelGGL(kernel, dim3(set->pieces << set->shift), dim3(kThreads), 0, reinterpret_cast<hipStream_t>(stream),
                       set->entries, set->table, set->shift, given, values, clip);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? CERAR_OK : hip_failed(e, "launch AdamW step");
}
