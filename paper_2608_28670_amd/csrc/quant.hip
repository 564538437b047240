// Quantised feature slots: writing a feature as 8- or 4-bit codes and forming
// Eq. 13's weighted sum from such slots, of one feature or of every module site.
//
// The flat feature is cut into groups of 64 consecutive values.  With Q = 127
// (8 bits) or 7 (4 bits), a group holds s = fl32(max|x| / Q) and the codes
// q = rint(x / s), ties to even; the value read back is q s.  The codes are
// exact: the quotient of the real numbers x and s is rounded, not that of an
// approximate reciprocal, so the same feature gives the same codes in any
// arithmetic that follows the definition.
//   A scale below 2^-120 is held as zero, and so is its group (the 4-bit
// forecast works with s / 16, which must not become subnormal).  A group with
// an infinity or a NaN has a NaN scale: it reads back as NaN, so that a bad
// feature cannot pass for a finite one.
//
// A slot is [codes of whole groups | padding to 256 | one fp32 scale per group
// | padding to 256].  8 bits: byte i of a group is value i, two's complement.
// 4 bits: byte b of every 4-byte word holds value b of the word's eight in its
// low half and value b + 4 in its high half, so a mask (after a shift for the
// low halves) leaves each code, times 16, as a signed byte.
#include <cmath>
#include <cstring>

#include "ops.h"

namespace bc {

constexpr int kQThreads = 256;
constexpr float kMinScale = 0x1p-120f;
typedef unsigned int u32x2q __attribute__((ext_vector_type(2)));

// x / s rounded to the nearest integer, ties to even, for |x| <= Q s (1 + eps)
// and a normal s: the rounded product with an approximate 1 / s is off by at most
// one, and the remainder x - q s, which one FMA gives exactly (it is a multiple of
// the smaller of the two's last places and at most s), says so.
__device__ __forceinline__ int code_of(float x, float s, float inv) {
    float q = rintf(x * inv);
    const float r = fmaf(-q, s, x);
    const float r2 = r + r;
    const bool odd = (int)q & 1;
    if (r2 > s || (r2 == s && odd)) q += 1.f;
    else if (r2 < -s || (r2 == -s && odd)) q -= 1.f;
    return (int)q;
}

// The low bytes of four words.
__device__ __forceinline__ uint32_t low_bytes(const uint32_t* u) {
    return __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400u) | __builtin_amdgcn_perm(u[3], u[2], 0x0c0c0400u) << 16;
}

// Eight values per thread, eight threads per group; n (e_in + bits / 8 + 1 / 16)
// bytes, memory bound as long as a code takes few instructions: fma(x, 1 / s, 1.5 *
// 2^23) has the rounded quotient in its low byte.  What that leaves are the ties.
//   bf16: x and max|x| = a have 8-bit mantissas, so Q x / a is half an integer or
// misses every such number by more than 2^-16 of itself ((2k + 1) a' 2^j and 2 Q x'
// are integers), and s is off by 2^-24.  Ties of Q x / a are common then (every wave
// has some), and where s < a / Q (s > a / Q) all of them belong a step further from
// (nearer to) zero: 1 / s grown (shrunk) by 2^-19, which moves nothing else across a
// half, rounds them so.  Where s = a / Q (a group in seven at 4 bits, in 128 at 8) ties
// go to even, the odd one of the two roundings to the other.
//   fp32: a second FMA gives the quotient's distance from the code; the approximate
// 1 / s (1 ulp) moves a quotient of at most 127 by less than 2^-15.9, so only a wave
// with a distance above 0.5 - 2^-15 goes through code_of.  (bf16 waves nearly all do:
// 400 M values into 8 bits 230 us that way, 200 so, 6.1 TB/s; into 4 bits 217 and 174,
// 5.9 TB/s; 4.7 M into 8 bits 6.0 and 4.2.)
//   U eights of a thread are requested together, two for long bf16 features into 4
// bits: 44 M 22.9 us with one, 21.8 with two, 22.9 with four; into 8 bits 25.5, 25.9
// and 27.0, 400 M 200, 211 and 219; 44 M fp32 values written and read 57.4, 58.2, 60.
template <typename T_, int BITS, bool VEC, int U>
__global__ __launch_bounds__(kQThreads) void quantise_kernel(const elem_t<T_>* __restrict__ x, int64_t n,
                                                             uint8_t* __restrict__ codes, float* __restrict__ scales) {
    typedef elem_t<T_> T;
    constexpr float Q = BITS == 8 ? 127.f : 7.f;
    constexpr float kMagic = 12582912.f, kSure = 0.5f - 0x1p-15f, kBias = 0x1p-19f;
    constexpr int CH = sizeof(T) / 2;      // 16-byte chunks of eight values
    const int64_t e0 = ((int64_t)blockIdx.x * (kQThreads * U) + threadIdx.x) * 8;
    u32x4 raw[U][CH];
#pragma unroll
    for (int k = 0; k < U; ++k) {
        const int64_t e = e0 + (int64_t)k * (kQThreads * 8);
        if (VEC && e + 8 <= n) {
#pragma unroll
            for (int c = 0; c < CH; ++c) raw[k][c] = reinterpret_cast<const u32x4*>(x + e)[c];
        }
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
        const int64_t e = e0 + (int64_t)k * (kQThreads * 8);
        if ((e & ~(int64_t)(kQuantGroup - 1)) >= n) return;      // the whole group: its eight threads go together
        float v[8];
        if (VEC && e + 8 <= n) {
            unpack(raw[k][0], v, (const T*)nullptr);
            if constexpr (CH == 2) unpack(raw[k][CH - 1], v + 4, (const T*)nullptr);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = e + i < n ? ld(x + e + i) : 0.f;
        }
        // The largest magnitude as bits: a NaN's are above infinity's.
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
        m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, false));     // lane ^ 1
        m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, false));     // lane ^ 2
        m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x141, 0xF, 0xF, false));    // 7 - lane of eight
        // max / Q, correctly rounded: a faithful quotient, its exact remainder, and one
        // correction with the correctly rounded 1 / Q.
        const float top = __uint_as_float(m), q0 = top * (1.f / Q);
        float s = fmaf(fmaf(-q0, Q, top), 1.f / Q, q0);
        const bool bad = m >= 0x7f800000u;
        if (s < kMinScale) s = 0.f;
        if (bad) s = __uint_as_float(0x7fc00000u);
        const float inv = bad || s == 0.f ? 0.f : __builtin_amdgcn_rcpf(s);
        uint32_t u[8];
        if constexpr (sizeof(T) == 2) {
            const float off = fmaf(s, Q, -top);
            float up = fmaf(inv, kBias, inv), down = fmaf(inv, -kBias, inv);
            if (off > 0.f) up = down;
#pragma unroll
            for (int i = 0; i < 8; ++i) u[i] = __float_as_uint(fmaf(v[i], up, kMagic));
            if (__any(off == 0.f && inv != 0.f)) {
                if (off < 0.f) down = up;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t d = __float_as_uint(fmaf(v[i], down, kMagic));
                    u[i] = d & 1 ? u[i] : d;
                }
            }
        } else {
            float far = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float y = fmaf(v[i], inv, kMagic);
                u[i] = __float_as_uint(y);
                far = fmaxf(far, fabsf(fmaf(v[i], inv, kMagic - y)));
            }
            if (__any(far > kSure)) {
#pragma unroll
                for (int i = 0; i < 8; ++i) u[i] = inv != 0.f ? (uint32_t)code_of(v[i], s, inv) : 0u;
            }
        }
        if constexpr (BITS == 8) {
            *reinterpret_cast<u32x2q*>(codes + e) = u32x2q{low_bytes(u), low_bytes(u + 4)};
        } else {
            *reinterpret_cast<uint32_t*>(codes + e / 2) = (low_bytes(u) & 0x0f0f0f0fu) | (low_bytes(u + 4) << 4 & 0xf0f0f0f0u);
        }
        if ((threadIdx.x & 7) == 0) scales[e / kQuantGroup] = s;
    }
}

struct QuantFcArgs {
    const uint8_t* src[kMaxK];
    float w[kMaxK];
    int64_t scales_at;      // bytes from a slot's start to its scales
    void* out;
    int64_t n;
};

// The codes of eight values, times 16 for 4 bits (their scale is divided by 16 instead).
template <int BITS, bool NT>
__device__ __forceinline__ void decode_eight(const uint8_t* codes, int64_t e, float* f) {
    if constexpr (BITS == 8) {
        const u32x2q* p = reinterpret_cast<const u32x2q*>(codes + e);
        const u32x2q w = NT ? __builtin_nontemporal_load(p) : *p;
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = (float)(int8_t)(w[i >> 2] >> (8 * (i & 3)));
    } else {
        const uint32_t* p = reinterpret_cast<const uint32_t*>(codes + e / 2);
        const uint32_t w = NT ? __builtin_nontemporal_load(p) : *p;
        const uint32_t lo = (w << 4) & 0xf0f0f0f0u, hi = w & 0xf0f0f0f0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[i] = (float)(int8_t)(lo >> (8 * i));
            f[i + 4] = (float)(int8_t)(hi >> (8 * i));
        }
    }
}

template <bool NT, typename V> __device__ __forceinline__ void put(V* p, const V& v) {
    if constexpr (NT) __builtin_nontemporal_store(v, p);
    else *p = v;
}

// sum_j w_j s_j q_j: the weight times the scale is rounded once to fp32, the
// sum is fp32.  Eight values per thread; memory bound, K (bits / 8 + 1 / 16) +
// e_out bytes a value.  Launches that stream past the caches (NT) access codes and
// output non-temporally: three 8-bit nodes of 403 M values 350 -> 312 us (6.7
// TB/s); two units a thread 311, four 358.  Smaller ones 6.1 us without and 6.2 with.
template <int K, typename Tout_, int BITS, bool VEC, bool NT>
__global__ __launch_bounds__(kQThreads) void quant_forecast_kernel(QuantFcArgs a) {
    typedef elem_t<Tout_> Tout;
    const int64_t e = ((int64_t)blockIdx.x * kQThreads + threadIdx.x) * 8;
    if (e >= a.n) return;
    float acc[8];
#pragma unroll
    for (int j = 0; j < K; ++j) {
        const float s = *reinterpret_cast<const float*>(a.src[j] + a.scales_at + (e / kQuantGroup) * 4);
        const float ws = a.w[j] * (BITS == 8 ? s : s * 0.0625f);
        float f[8];
        decode_eight<BITS, NT>(a.src[j], e, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = j == 0 ? ws * f[i] : fmaf(ws, f[i], acc[i]);
    }
    Tout* out = static_cast<Tout*>(a.out) + e;
    if (VEC && e + 8 <= a.n) {
        if constexpr (sizeof(Tout) == 2) {
            bf16x8 o;
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = (bf16)acc[i];
            put<NT>(reinterpret_cast<bf16x8*>(out), o);
        } else {
            put<NT>(reinterpret_cast<f32x4*>(out), f32x4{acc[0], acc[1], acc[2], acc[3]});
            put<NT>(reinterpret_cast<f32x4*>(out + 4), f32x4{acc[4], acc[5], acc[6], acc[7]});
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (e + i < a.n) st(out + i, acc[i]);
}

static int64_t groups_of(int64_t n) { return (n + kQuantGroup - 1) / kQuantGroup; }
static int64_t up256(int64_t v) { return (v + 255) & ~(int64_t)255; }

int64_t quant_scales_at(int64_t n, int bits) { return up256(groups_of(n) * kQuantGroup * bits / 8); }
int64_t quant_slot_bytes(int64_t n, int bits) { return quant_scales_at(n, bits) + up256(groups_of(n) * 4); }

static int check_blocks(int64_t blocks, int64_t n) {
    return blocks > kMaxGrid ? fail(BC_ERR_UNSUPPORTED, "feature of %lld values is too large", (long long)n) : BC_OK;
}

template <typename T, int BITS>
static void run_quantise(const void* x, int64_t n, uint8_t* codes, float* scales, unsigned blocks, hipStream_t s) {
    const T* xt = static_cast<const T*>(x);
    const dim3 b(kQThreads);
    if (reinterpret_cast<uintptr_t>(x) % 16) {
        launch_k(quantise_kernel<tag_t<T>, BITS, false, 1>, dim3(blocks), b, s, xt, n, codes, scales);
        return;
    }
    if constexpr (sizeof(T) == 2 && BITS == 4) {
        if (n >= (int64_t)16 << 20) {      // two eights a thread (see the kernel)
            launch_k(quantise_kernel<tag_t<T>, BITS, true, 2>, dim3((blocks + 1) / 2), b, s, xt, n, codes, scales);
            return;
        }
    }
    launch_k(quantise_kernel<tag_t<T>, BITS, true, 1>, dim3(blocks), b, s, xt, n, codes, scales);
}

int launch_quantise(int in_dt, const void* x, int64_t n, int bits, void* slot, hipStream_t s) {
    if (n <= 0) return BC_OK;
    const int64_t blocks = (groups_of(n) * 8 + kQThreads - 1) / kQThreads;
    const int rc = check_blocks(blocks, n);
    if (rc != BC_OK) return rc;
    uint8_t* codes = static_cast<uint8_t*>(slot);
    float* scales = reinterpret_cast<float*>(codes + quant_scales_at(n, bits));
    prof_begin(PROF_COPY, s, (double)n * (dtype_size(in_dt) + bits / 8.0) + 4.0 * groups_of(n));
    if (in_dt == BC_BF16 && bits == 8) run_quantise<bf16, 8>(x, n, codes, scales, (unsigned)blocks, s);
    else if (in_dt == BC_BF16) run_quantise<bf16, 4>(x, n, codes, scales, (unsigned)blocks, s);
    else if (bits == 8) run_quantise<float, 8>(x, n, codes, scales, (unsigned)blocks, s);
    else run_quantise<float, 4>(x, n, codes, scales, (unsigned)blocks, s);
    prof_end(PROF_COPY, s);
    return check_launch("quantise");
}

template <typename Tout, int BITS, bool VEC, bool NT>
static void run_quant_forecast(const QuantFcArgs& a, int K, unsigned blocks, hipStream_t s) {
    const dim3 g(blocks), b(kQThreads);
    switch (K) {
#define BC_QF_CASE(KK) case KK: launch_k(quant_forecast_kernel<KK, tag_t<Tout>, BITS, VEC, NT>, g, b, s, a); break;
        BC_QF_CASE(1) BC_QF_CASE(2) BC_QF_CASE(3) BC_QF_CASE(4)
        BC_QF_CASE(5) BC_QF_CASE(6) BC_QF_CASE(7) BC_QF_CASE(8)
#undef BC_QF_CASE
        default: break;
    }
}

int launch_quant_forecast(const void* const* slots, const float* w, int K, int64_t n, int bits, void* out, int out_dt,
                          hipStream_t s) {
    if (K < 1 || K > kMaxK) return fail(BC_ERR_INVALID_ARG, "K=%d outside [1, 8]", K);
    if (n <= 0) return BC_OK;
    const int64_t blocks = (n + 8 * kQThreads - 1) / (8 * kQThreads);
    const int rc = check_blocks(blocks, n);
    if (rc != BC_OK) return rc;
    QuantFcArgs a;
    std::memset(&a, 0, sizeof a);
    for (int j = 0; j < K; ++j) {
        a.src[j] = static_cast<const uint8_t*>(slots[j]);
        a.w[j] = w[j];
    }
    a.scales_at = quant_scales_at(n, bits);
    a.out = out;
    a.n = n;
    const bool vec = reinterpret_cast<uintptr_t>(out) % 16 == 0;
    const double bytes = (double)n * (K * bits / 8.0 + dtype_size(out_dt)) + 4.0 * K * groups_of(n);
    prof_begin(PROF_FORECAST, s, bytes);
#define BC_QF_RUN(T, BITS) (!vec ? run_quant_forecast<T, BITS, false, false>(a, K, (unsigned)blocks, s) \
                            : bytes >= 80e6 ? run_quant_forecast<T, BITS, true, true>(a, K, (unsigned)blocks, s) \
                                            : run_quant_forecast<T, BITS, true, false>(a, K, (unsigned)blocks, s))
    if (out_dt == BC_BF16 && bits == 8) BC_QF_RUN(bf16, 8);
    else if (out_dt == BC_BF16) BC_QF_RUN(bf16, 4);
    else if (bits == 8) BC_QF_RUN(float, 8);
    else BC_QF_RUN(float, 4);
#undef BC_QF_RUN
    prof_end(PROF_FORECAST, s);
    return check_launch("quantised forecast");
}

// Blockwise mode's skipped step: x += sum_sites gate (.) sum_j w_j s_j q_j, the
// stream read and written once.  Memory bound: sites K (bits / 8 + 1 / 16) + 8
// bytes a value, and 4 of the gates from L2 for every site and value; a thread
// takes the same eight columns of R rows of one sample, which share them.  42 sites
// of 16 384 x 1152, two 8-bit nodes (1.7 GB): 407 us with R = 1, 364 with 2 (4.6 TB/s),
// 355 with 4; 28 sites of 4096 x 1152, three nodes: 110, 101 and 111.
template <int K, int BITS, int R>
__global__ __launch_bounds__(kQThreads) void blockwise_quant_forecast_kernel(BlockwiseArgs a, int64_t slot_bytes,
                                                                             int64_t scales_at) {
    const int cols = a.D / 8;
    const int64_t t = (int64_t)blockIdx.x * kQThreads + threadIdx.x;
    const int64_t r = t / cols * R;
    if (r >= a.rows) return;
    const int d = (int)(t % cols) * 8;
    const float* mrow = a.mods + (r / a.rows_per_gate) * a.ldm + d;
    const uint8_t* base = static_cast<const uint8_t*>(a.storage);
    const int64_t e = r * a.D + d;
    f32x4 x[R][2];
#pragma unroll
    for (int k = 0; k < R; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) x[k][h] = *reinterpret_cast<const f32x4*>(a.x + e + (int64_t)k * a.D + 4 * h);
#pragma unroll 1
    for (int s = 0; s < a.nsites; ++s) {
        f32x4 g[2] = {{1.f, 1.f, 1.f, 1.f}, {1.f, 1.f, 1.f, 1.f}};
        if (a.goff[s] >= 0) {
            g[0] = *reinterpret_cast<const f32x4*>(mrow + a.goff[s]);
            g[1] = *reinterpret_cast<const f32x4*>(mrow + a.goff[s] + 4);
        }
        float f[R][K][8], ws[R][K];
#pragma unroll
        for (int k = 0; k < R; ++k)
#pragma unroll
            for (int j = 0; j < K; ++j) {
                const uint8_t* slot = base + ((int64_t)s * a.K + a.slot[j]) * slot_bytes;
                const int64_t at = e + (int64_t)k * a.D;
                ws[k][j] = *reinterpret_cast<const float*>(slot + scales_at + (at / kQuantGroup) * 4);
                decode_eight<BITS, false>(slot, at, f[k][j]);
            }
#pragma unroll
        for (int k = 0; k < R; ++k) {
            float acc[8];
#pragma unroll
            for (int j = 0; j < K; ++j) {
                const float w = a.w[j] * (BITS == 8 ? ws[k][j] : ws[k][j] * 0.0625f);
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[i] = j == 0 ? w * f[k][j][i] : fmaf(w, f[k][j][i], acc[i]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) x[k][i >> 2][i & 3] = fmaf(g[i >> 2][i & 3], acc[i], x[k][i >> 2][i & 3]);
        }
    }
#pragma unroll
    for (int k = 0; k < R; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) *reinterpret_cast<f32x4*>(a.x + e + (int64_t)k * a.D + 4 * h) = x[k][h];
}

template <int BITS, int R>
static int run_blockwise(const BlockwiseArgs& a, hipStream_t s) {
    const int64_t slot = quant_slot_bytes(a.numel, BITS), at = quant_scales_at(a.numel, BITS);
    const int64_t blocks = (a.rows / R * (a.D / 8) + kQThreads - 1) / kQThreads;
    const int rc = check_blocks(blocks, a.numel);
    if (rc != BC_OK) return rc;
    const dim3 g((unsigned)blocks);
    switch (a.count) {
#define BC_BQ_CASE(KK) case KK: blockwise_quant_forecast_kernel<KK, BITS, R><<<g, kQThreads, 0, s>>>(a, slot, at); break;
        BC_BQ_CASE(1) BC_BQ_CASE(2) BC_BQ_CASE(3) BC_BQ_CASE(4)
        BC_BQ_CASE(5) BC_BQ_CASE(6) BC_BQ_CASE(7) BC_BQ_CASE(8)
#undef BC_BQ_CASE
        default: break;
    }
    return check_launch("blockwise quantised forecast");
}

int launch_blockwise_quant_forecast(int bits, const BlockwiseArgs& a, hipStream_t s) {
    if (a.D % 8 || a.numel % 8 || a.nsites < 1 || a.nsites > kMaxSites || a.count < 1 || a.count > a.K || a.K > kMaxK ||
        a.ldm % 4 || reinterpret_cast<uintptr_t>(a.storage) % 16 || reinterpret_cast<uintptr_t>(a.x) % 16 ||
        reinterpret_cast<uintptr_t>(a.mods) % 16)
        return fail(BC_ERR_INVALID_ARG, "blockwise forecast: %d sites, count %d of %d", a.nsites, a.count, a.K);
    for (int j = 0; j < a.count; ++j)
        if (a.slot[j] < 0 || a.slot[j] >= a.K) return fail(BC_ERR_INVALID_ARG, "blockwise forecast: slot %d", a.slot[j]);
    for (int q = 0; q < a.nsites; ++q)
        if (a.goff[q] >= 0 && a.goff[q] % 4) return fail(BC_ERR_INVALID_ARG, "blockwise forecast: gate offset %d", a.goff[q]);
    if (a.rows_per_gate % 2 == 0) return bits == 8 ? run_blockwise<8, 2>(a, s) : run_blockwise<4, 2>(a, s);
    return bits == 8 ? run_blockwise<8, 1>(a, s) : run_blockwise<4, 1>(a, s);
}

}  // namespace bc
