// The kernels of score.h's attention, over tensors (KV8 false) or over the 8-bit
// cache (KV8 true).  All of them follow attention.hip's plan: transposed scores S^T
// = K Q^T, so that a lane holds scores of one row; online softmax in log2 units;
// O^T = V^T P^T with the probabilities as they lie.
//
// Tiles of 64 keys that no row of a workgroup sees are never loaded, and masks are
// applied only in tiles that some row sees in part: every 64 tiles, one per lane,
// are classed at once and the ballots walked.
//
// A hidden key's value takes part in the products with a weight of zero, which
// leaves NaN where the value is not finite.  Rather than testing every value, the
// workgroup tests its outputs at the end, and if some are not finite it runs three
// times more (`CAREFUL`): over the infinities and NaN alone, as ones, +inf with NaN
// and -inf with NaN, each key that is seen weighing one, which tells where such a key
// has one, and over the finite values.  (A weight below fp32's least is more than
// nothing all the same: whether it counts must not go by where the keys are cut.)
#pragma once

#include <type_traits>

#include "score.h"

namespace bc {

// A kernel's arguments, read again from memory.  What a tile seldom needs (masks, caps,
// the rows past a sample's end) or the end does is read where it is used: held over the
// key loop, it would take the scalar registers that the loop's own addresses need.
typedef const __attribute__((address_space(4))) ScoreArgs Args;
__device__ __forceinline__ Args* kernel_arguments() { return (Args*)__builtin_amdgcn_kernarg_segment_ptr(); }
__device__ __forceinline__ Args& again(Args* p) {
    asm volatile("" : "+s"(p));
    return *p;
}

// Where the references of a row's softmax start: far below any score, yet finite, so
// that a tile that the row does not see at all (-inf) takes no case of its own.
constexpr float kNoScore = -1e30f;

// A value that all lanes share, in a scalar register.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

template <typename T> __device__ __forceinline__ T* uniform(T* p) {
    const uint64_t x = (uint64_t)p;
    return (T*)((uint64_t)(unsigned)uniform((int)(x >> 32)) << 32 | (unsigned)uniform((int)x));
}

// What a workgroup's rows see; the same in every lane.
struct Seen {
    int n, prefix;                 // keys; of them those that all rows see
    int any_lo, any_hi;            // keys that some row sees (past the prefix)
    int all_lo, all_hi;            // keys that every row sees
    int doc_lo, doc_hi;            // documents of the rows
};
// Tiles still to be visited: [at, hi), and of the present 64 those seen, and those seen by every row.  Their numbers leave out what
// lies between the prefix and the window: from `head` on, tile x is the keys' tile x + gap.
struct Walk {
    int at, hi, head, gap;
    uint64_t some, full;
};

__device__ __forceinline__ int row_lo(Args& a, int p) { return a.window ? p - a.window + 1 : -kMaxPosition * 2; }
__device__ __forceinline__ int row_hi(Args& a, int p) {
    return a.causal ? p : a.window ? p + a.window - 1 : kMaxPosition * 2;
}

// Rows at positions p0..p1 of a sample with n keys.
__device__ __forceinline__ Seen seen_by(Args& a, int b, int n, int p0, int p1) {
    Seen s;
    s.n = n;
    s.prefix = a.prefix ? uniform(min(max(a.prefix[b], 0), n)) : 0;
    s.any_lo = uniform(row_lo(a, p0));
    s.any_hi = uniform(row_hi(a, p1));
    s.all_lo = uniform(row_lo(a, p1));
    s.all_hi = uniform(row_hi(a, p0));
    s.doc_lo = 0;
    s.doc_hi = -1;
    return s;
}

// The tiles of part `part` of `parts`.  (With parts by the keys' own numbers, those of the gap had no work: one query, 4 x 8 heads on
// 65 536 keys, d = 128, a window of 4096 behind a prefix of 4: 113 us, 42 over the cache; 23 and 15 so, 21 and 13 without the prefix.)
__device__ __forceinline__ Walk walk_part(const Seen& s, unsigned part, unsigned parts) {
    const int last = min(max(s.any_hi, s.prefix - 1), s.n - 1);
    const int hi = last < 0 ? 0 : last / kKTile + 1;
    const int lo = min(max(s.any_lo, 0) / kKTile, hi), head = (s.prefix + kKTile - 1) / kKTile;
    Walk w;
    w.head = uniform(head);
    w.gap = uniform(max(lo - head, 0));
    const unsigned len = hi - w.gap;       // at most 2^18, in 256 parts
    w.at = uniform((int)(len * part / parts));
    w.hi = uniform((int)(len * (part + 1) / parts));
    w.some = w.full = 0;
    return w;
}

// The next tile, or -1; `full`: every row sees all of it.
__device__ __forceinline__ int walk_next(const Seen& s, Walk& w, const u32x2* ranges, int lane, bool& full) {
    while (w.some == 0) {
        if (w.at >= w.hi) return -1;
        const int x = min(w.at + lane, w.hi - 1), j = x + (x >= w.head ? w.gap : 0), k0 = j * kKTile, k1 = k0 + kKTile - 1;
        bool some = w.at + lane < w.hi && ((k0 <= s.any_hi && k1 >= s.any_lo) || k0 < s.prefix);
        bool all = k1 < s.n && ((k1 <= s.all_hi && k0 >= s.all_lo) || k1 < s.prefix);
        if (ranges) {
            const u32x2 r = ranges[j];       // (~first if some key has no document, last)
            const int first = (int)r.x < 0 ? ~(int)r.x : (int)r.x, last = (int)r.y;
            some = some && first <= s.doc_hi && last >= s.doc_lo;
            all = all && (int)r.x >= 0 && first == last && s.doc_lo == s.doc_hi && first == s.doc_lo;
        }
        w.some = __ballot(some);
        w.full = __ballot(all);
        w.at += 64;
    }
    const int t = __builtin_ctzll(w.some);
    w.some &= w.some - 1;
    full = (w.full >> t) & 1;
    const int x = w.at - 64 + t;
    return uniform(x + (x >= w.head ? w.gap : 0));
}

// A row's scores of 4 N of its lane's keys, k0 + 16 j + 4 grp + r, from products to log2
// units: the scale, the cap, the distance's share.  PRECISE: fp32.
template <bool PRECISE, int N>
__device__ __forceinline__ void score_map(Args& a, f32x4 (&s)[N], float slope, float p, int k0, int grp) {
    if (a.cap_log2 != 0.f) {
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float x = s[j][r] * a.cap_exp;        // 2 log2(e) z, z the score over the cap
                if constexpr (PRECISE) {
                    s[j][r] = a.cap_log2 * tanhf(x * 0.34657359f);
                } else {
                    float t = __builtin_fmaf(-2.f, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x)), 1.f);
                    if (a.cap_wide) {
                        // z - z^3/3 + 2 z^5/15 - 17 z^7/315, for |z| < 1/4 to 2^-20 of itself
                        const float z = x * 0.34657359f, q = z * z;
                        const float near = z * __builtin_fmaf(q, __builtin_fmaf(q, __builtin_fmaf(q, -17.f / 315.f, 2.f / 15.f), -1.f / 3.f), 1.f);
                        t = fabsf(z) < 0.25f ? near : t;
                    }
                    s[j][r] = a.cap_log2 * t;
                }
            }
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) s[j] *= a.scale_log2;
    }
    if (a.slopes) {
        const float d0 = p - (float)(k0 + 4 * grp);
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) s[j][r] = __builtin_fmaf(-slope, fabsf(d0 - (float)(16 * j + r)), s[j][r]);
    }
}

// -inf for the keys that a row at position p does not see: for its place (by_pos: not if
// every row's place sees the whole tile), for its document (docs: the tile's, if by_doc).
typedef __attribute__((address_space(3))) const int lds_int;
template <int N>
__device__ __forceinline__ void score_mask(Args& a, const Seen& seen, f32x4 (&s)[N], int p, int doc, int k0, int grp, bool by_pos,
                                           bool by_doc, lds_int* docs) {
    typedef int i32x4 __attribute__((ext_vector_type(4)));
    if (by_pos) {
        const int lo = row_lo(a, p), key = k0 + 4 * grp;
        const unsigned from = (unsigned)(key - lo), span = (unsigned)max(min(row_hi(a, p), seen.n - 1) - lo + 1, 0);
        const int all = seen.prefix - key;
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int c = 16 * j + r;
                s[j][r] = ((from + c < span) | (c < all)) ? s[j][r] : -INFINITY;
            }
    }
    if (by_doc) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const i32x4 d = *(__attribute__((address_space(3))) const i32x4*)(docs + 16 * j + 4 * grp);
#pragma unroll
            for (int r = 0; r < 4; ++r) s[j][r] = d[r] == doc ? s[j][r] : -INFINITY;
        }
    }
}

// What a careful run takes for a value: 1 where it is +inf or NaN (POS), -inf or NaN
// (NEG), else 0; or the value where it is finite, else 0.
enum CarefulRun { POS = 0, NEG = 1, FINITE = 2 };
__device__ __forceinline__ float careful(float v, int run) {
    const bool fin = fabsf(v) < INFINITY;
    if (run == FINITE) return fin ? v : 0.f;
    return fin || v == (run == POS ? -INFINITY : INFINITY) ? 0.f : 1.f;
}
__device__ __forceinline__ u32x4 careful(const u32x4& v, int run) {
    const unsigned w[4] = {v.x, v.y, v.z, v.w};
    unsigned o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float lo = careful(__uint_as_float(w[i] << 16), run), hi = careful(__uint_as_float(w[i] & 0xffff0000u), run);
        o[i] = (__float_as_uint(lo) >> 16) | (__float_as_uint(hi) & 0xffff0000u);
    }
    return u32x4{o[0], o[1], o[2], o[3]};
}
// Scores of the runs that look for infinities and NaN: 0 for the keys that are seen.
template <int N> __device__ __forceinline__ void careful_scores(f32x4 (&s)[N], int run) {
    if (run == FINITE) return;
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) s[j][r] = s[j][r] > -INFINITY ? 0.f : -INFINITY;
}
// A run's outputs as a bit each (its N values of a lane; more than 0: some key that is seen has one).
template <int N> __device__ __forceinline__ void careful_bits(const f32x4* o, uint64_t& bits) {
    bits = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) bits |= (uint64_t)(o[i / 4][i % 4] > 0.f) << i;
}
template <int N> __device__ __forceinline__ void careful_join(f32x4* o, uint64_t pos, uint64_t neg) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const bool a = (pos >> i) & 1, b = (neg >> i) & 1;
        const float v = a && b ? __builtin_nanf("") : a ? INFINITY : -INFINITY, f = o[i / 4][i % 4];
        o[i / 4][i % 4] = (a || b) && f == f ? v : f;       // (NaN: of a score)
    }
}

// 16 codes -> bf16 values: 8 bytes each of two operands.
__device__ __forceinline__ void decode16(const u32x4& c, float scale, u32x4& lo, u32x4& hi) {
    const unsigned w[4] = {c.x, c.y, c.z, c.w};
    unsigned o[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        o[2 * i] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, false));
        o[2 * i + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, true));
    }
    lo = u32x4{o[0], o[1], o[2], o[3]};
    hi = u32x4{o[4], o[5], o[6], o[7]};
}
__device__ __forceinline__ void decode4(unsigned c, float scale, float (&f)[4]) {
    const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c, scale, false);
    const auto b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c, scale, true);
    f[0] = a[0]; f[1] = a[1]; f[2] = b[0]; f[3] = b[1];
}

// 4 bytes a lane straight into LDS (see dma16).
__device__ __forceinline__ void dma4(const void* src, const void* lds_base) {
    const unsigned m0 = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)lds_base);
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" : : "v"(src), "s"(m0) : "memory", "m0");
}

// A workgroup's place: its rows, sample, key head and part.
struct Place {
    int b, hk, bh, r0, part, n, count, base;
};
__device__ __forceinline__ Place place_of(Args& a, int rows_wg, bool cache) {
    Place p;
    const int nrt = (a.Tq * a.G + rows_wg - 1) / rows_wg;
    int pid, rt;
    if (a.order || (a.causal && !a.window)) {
        // The longest of every head first: by their documents, or, causal, the last rows.  (A head that came after another
        // would begin with its longest, and end late: 16 heads of 16 384 tokens, causal, d = 64 667 -> 612 us.)
        pid = blockIdx.x;
        p.part = pid % a.parts;
        pid /= a.parts;
        p.bh = pid % (a.B * a.Hk);
        p.b = p.bh / a.Hk;
        rt = pid / (a.B * a.Hk);
        rt = a.order ? a.order[p.b * nrt + rt] : nrt - 1 - rt;
    } else {
        // A head's workgroups, which share its keys, in one L2.
        pid = xcd_contiguous(blockIdx.x, gridDim.x);
        p.part = pid % a.parts;
        pid /= a.parts;
        rt = pid % nrt;
        p.bh = pid / nrt;
        p.b = p.bh / a.Hk;
    }
    p.r0 = rt * rows_wg;
    p.hk = p.bh % a.Hk;
    p.n = a.lens ? __builtin_amdgcn_readfirstlane(min(max(a.lens[p.b], 0), a.Tk)) : a.Tk;
    p.count = a.counts ? __builtin_amdgcn_readfirstlane(min(max(a.counts[p.b], 0), a.Tq)) : a.Tq;
    p.base = cache ? p.n - p.count : a.q_start;
    p.part = uniform(p.part);
    p.r0 = uniform(p.r0);
    p.b = uniform(p.b);
    p.hk = uniform(p.hk);
    p.bh = uniform(p.bh);
    return p;
}

// The documents of the workgroup's rows [r0, r1).
__device__ __forceinline__ void row_documents(Args& a, int b, int r0, int r1, int lane, Seen& s) {
    int lo = 0x7fffffff, hi = -1;
    for (int r = r0 + lane; r < r1; r += 64) {
        const int d = a.q_docs[(int64_t)b * a.Tq + r / a.G];
        if (d >= 0) {
            lo = min(lo, d);
            hi = max(hi, d);
        }
    }
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) {
        lo = min(lo, __shfl_xor(lo, x));
        hi = max(hi, __shfl_xor(hi, x));
    }
    s.doc_lo = __builtin_amdgcn_readfirstlane(lo);
    s.doc_hi = __builtin_amdgcn_readfirstlane(hi);
}

// The rows of a workgroup whose four waves took keys of their own: outputs from `so` ([16][HD + 4] a wave, `stride` apart),
// references and sums from sml, joined (infinities and NaN as they are: times) into the outputs or the part's.  A thread a row
// for the weights, then four columns a thread (16 rows of 32 heads over 4000 keys in fp32: 27.6 us with the weights made anew for
// every column, 22.8 so).
template <typename T, int HD>
__device__ __forceinline__ void join_waves(Args& z, const Place& at, const float* so, int stride, float (*sml)[16][2], int tid) {
    const int rows = z.Tq * z.G, parts = z.parts;
    auto out_row = [&](int r) { return ((int64_t)at.b * z.Tq + r / z.G) * (z.Hk * z.G) + at.hk * z.G + r % z.G; };
    if (tid < rows) {
        float top = kNoScore, sum = 0.f, f[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, sml[w][tid][1] != 0.f ? sml[w][tid][0] : kNoScore);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float lw = sml[w][tid][1];
            f[w] = lw != 0.f ? exp2f(sml[w][tid][0] - top) : 0.f;      // (0: the wave saw no key)
            sum = fmaf(f[w], lw, sum);
        }
        if (parts > 1) {
            float* ml = z.part_ml + (out_row(tid) * parts + at.part) * 2;
            ml[0] = sum != 0.f ? top : -INFINITY;
            ml[1] = sum;
        }
        const float inv = parts > 1 ? 1.f : sum != 0.f ? 1.f / sum : 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) sml[w][tid][0] = sml[w][tid][1] != 0.f ? f[w] * inv : -1.f;
    }
    __syncthreads();
    for (int x = tid; x < rows * (HD / 4); x += 256) {
        const int r = x / (HD / 4), d = 4 * (x - r * (HD / 4));
        auto total = [&](auto keep) __attribute__((always_inline)) {
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float f = sml[w][r][0];       // (-1: the wave saw no key)
                if (!(f < 0.f)) acc += times<decltype(keep)::value>(*reinterpret_cast<const f32x4*>(so + w * stride + r * (HD + 4) + d), f);
            }
            return acc;
        };
        f32x4 acc = total(std::false_type{});
        if (!all_finite(acc)) acc = total(std::true_type{});
        const int64_t row = out_row(r);
        if (parts > 1) {
            *reinterpret_cast<f32x4*>(z.part_o + (row * parts + at.part) * HD + d) = acc;
        } else {
            T y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = (T)acc[e];
            __builtin_memcpy(static_cast<T*>(z.out) + row * HD + d, y, sizeof y);
        }
    }
}

// ---------------------------------------------------------------------------
// fp32: 64 rows a workgroup, four waves of 16; key and value tiles row-major in
// LDS, loaded into registers a tile ahead.  Neither a dot product's nor the
// outputs' order of columns matters to an MFMA, so that lanes take columns that
// lie together: keys 4 (of the last 8 of 72: 2) to a read, values W.  Bound by the
// fp32 MFMAs, a sixteenth of bf16's rate: 16 heads of 4096 tokens, d = 128, 1190 us,
// 116 TFLOP/s; 1410 with one wave a SIMD (280 registers), 1700 so and with a read for
// every value.  Waves without rows that see a tile wait it out.
//   FEW: up to 16 rows in all; each wave takes 16 of a tile's keys for them, and the
// waves meet at the end (16 x 8 heads of one query over 8000 keys, d = 128: 202 us,
// 5.2 TB/s, 262 by 64 rows; 8 x 8 over 2000, d = 64: 21 and 24).
// ---------------------------------------------------------------------------
template <int HD, bool KV8, bool FEW>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(HD >= 72 ? 2 : HD == 64 ? 3 : 4))) void score_f32_kernel(ScoreArgs) {
    Args* args = kernel_arguments();
    Args& a = again(args);
    constexpr int ROWS = FEW ? 16 : 64, NJ = FEW ? 1 : 4;      // rows of a workgroup, 16s of keys of a wave
    constexpr int DV = (HD + 15) / 16 * 16, LD = DV + 4, CPR = HD / 8;
    constexpr int W = HD == 32 ? 2 : 4, WHOLE = HD / (16 * W) * W;     // outputs i < WHOLE: W neighbours a lane
    typedef float piece __attribute__((ext_vector_type(W)));
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    // Column of the dot products' step c, and of output i, element m.
    auto q_col = [](int c, int grp) { return c < HD / 16 * 4 ? c / 4 * 16 + 4 * grp + c % 4 : HD / 16 * 16 + 2 * grp + c % 4; };
    auto o_col = [](int i, int m) { return i < WHOLE ? i / W * 16 * W + W * m + i % W : 16 * i + m; };
    __shared__ __attribute__((aligned(16))) float sK[kKTile][LD];
    __shared__ __attribute__((aligned(16))) float sV[kKTile][LD];
    __shared__ __attribute__((aligned(16))) int sdoc[kKTile];
    __shared__ u32x4 srow[ROWS];              // a row's position, document and slope
    const int tid = threadIdx.x, lane = tid & 63, ql = lane & 15, grp = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Place at = place_of(a, ROWS, KV8);
    const int Hq = a.Hk * a.G;
    const int own_row = (FEW ? 0 : 16 * wave) + ql;
    const int r = at.r0 + own_row, t = r / a.G, head = at.hk * a.G + r - t * a.G;
    bool ok = t < at.count;
    const bool mine = t < a.Tq;
    int doc = 0;
    const int r1 = min(at.r0 + ROWS, at.count * a.G);
    Seen seen = seen_by(a, at.b, at.n, at.base + at.r0 / a.G, at.base + (r1 - 1) / a.G);
    const u32x2* ranges = nullptr;
    if (!KV8 && a.q_docs) {
        row_documents(a, at.b, at.r0, r1, lane, seen);
        doc = ok ? a.q_docs[(int64_t)at.b * a.Tq + t] : -1;
        ok = doc >= 0;
        ranges = a.ranges + (int64_t)at.b * ((a.Tk + kKTile - 1) / kKTile);
    }
    if (grp == 0) {
        const float slope = a.slopes && mine ? a.slopes[head] * 1.44269504f : 0.f;
        srow[own_row] = u32x4{(unsigned)(at.base + t), (unsigned)doc, __float_as_uint(slope), 0u};
    }
    float qf[HD / 4];
    const float* qr = static_cast<const float*>(a.q) + at.b * a.q_batch + (int64_t)t * a.q_row + (int64_t)head * HD;
#pragma unroll
    for (int c = 0; c < HD / 4; ++c) qf[c] = ok ? qr[q_col(c, grp)] : 0.f;
    // Columns past the head (read as rows of V^T that are not stored).
    for (int x = tid; x < kKTile * (LD - HD); x += 256) sV[x / (LD - HD)][HD + x % (LD - HD)] = 0.f;

    constexpr int UNITS = KV8 ? 4 * HD : kKTile * HD / 4, PER = (UNITS + 255) / 256;
    u32x4 rk[PER], rv[PER];
    float ks = 0.f, vs = 0.f;
    int rd = 0;
    auto load = [&](int tile) {
        Args& a = again(args);
        const int64_t ct = (int64_t)at.bh * a.tiles + tile;
        if constexpr (KV8) {
            ks = a.scales[2 * ct];
            vs = a.scales[2 * ct + 1];
        }
#pragma unroll
        for (int x = 0; x < PER; ++x) {
            const int u = tid + 256 * x;
            rk[x] = rv[x] = u32x4{0u, 0u, 0u, 0u};
            if (u >= UNITS) continue;
            if constexpr (KV8) {
                const u32x4* c = reinterpret_cast<const u32x4*>(a.codes + ct * (2 * kKTile * HD));
                rk[x] = c[u];
                rv[x] = c[UNITS + u];
            } else {
                const int row = min(tile * kKTile + u / (HD / 4), at.n - 1), col = at.hk * HD + u % (HD / 4) * 4;
                rk[x] = *reinterpret_cast<const u32x4*>(static_cast<const float*>(a.k) + at.b * a.k_batch + (int64_t)row * a.k_row + col);
                rv[x] = *reinterpret_cast<const u32x4*>(static_cast<const float*>(a.v) + at.b * a.v_batch + (int64_t)row * a.v_row + col);
            }
        }
        if (!KV8 && ranges && tid < kKTile) rd = a.k_docs[(int64_t)at.b * a.Tk + min(tile * kKTile + tid, at.n - 1)];
    };
    auto store = [&]() {
#pragma unroll
        for (int x = 0; x < PER; ++x) {
            const int u = tid + 256 * x;
            if (u >= UNITS) continue;
            if constexpr (KV8) {
                const unsigned wk[4] = {rk[x].x, rk[x].y, rk[x].z, rk[x].w}, wv[4] = {rv[x].x, rv[x].y, rv[x].z, rv[x].w};
                const int l = u & 15, ch = (u >> 4) % CPR, jp = (u >> 4) / CPR;
                const int i = u >> 6, w = min(16, HD - 16 * i), kg = (u & 63) / w, col = 16 * i + (u & 63) % w;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float f[4];
                    decode4(wk[e], ks, f);
                    *reinterpret_cast<f32x4*>(&sK[32 * jp + 16 * (e >> 1) + l][8 * ch + 4 * (e & 1)]) = f32x4{f[0], f[1], f[2], f[3]};
                    decode4(wv[e], vs, f);
#pragma unroll
                    for (int q = 0; q < 4; ++q) sV[32 * (e >> 1) + 16 * (e & 1) + 4 * kg + q][col] = f[q];
                }
            } else {
                const int row = u / (HD / 4), col = u % (HD / 4) * 4;
                *reinterpret_cast<u32x4*>(&sK[row][col]) = rk[x];
                *reinterpret_cast<u32x4*>(&sV[row][col]) = rv[x];
            }
        }
        if (!KV8 && ranges && tid < kKTile) sdoc[tid] = rd;
    };

    // The keys that some row of this wave sees (past the prefix): none if it has no rows.
    const int w0 = at.r0 + (FEW ? 0 : 16 * wave), w1 = min(w0 + 16, r1);
    const int own_lo = uniform(row_lo(a, at.base + w0 / a.G)), own_hi = uniform(w0 < w1 ? row_hi(a, at.base + (w1 - 1) / a.G) : -1);
    const int own_prefix = uniform(w0 < w1 ? seen.prefix : 0);
    const int parts = a.parts;
    f32x4 o[DV / 16];
    float m, l;
    // One tile of keys, from k0 on, for the wave's rows.
    auto compute = [&](auto carefulc, int which, int k0, bool full) __attribute__((always_inline)) {
        constexpr bool CAREFUL = decltype(carefulc)::value;
        f32x4 s[NJ];
#pragma unroll
        for (int j = 0; j < NJ; ++j) s[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < HD / 4; c += 4) {
            f32x4 kf[NJ];
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                const float* at = &sK[16 * (FEW ? wave : j) + ql][q_col(c, grp)];
                if (c < HD / 16 * 4) {
                    kf[j] = *reinterpret_cast<const f32x4*>(at);
                } else {
                    const f32x2 two = *reinterpret_cast<const f32x2*>(at);
                    kf[j] = f32x4{two.x, two.y, 0.f, 0.f};
                }
            }
#pragma unroll
            for (int e = 0; e < 4 && c + e < HD / 4; ++e)
#pragma unroll
                for (int j = 0; j < NJ; ++j) s[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[j][e], qf[c + e], s[j], 0, 0, 0);
        }
        {
            const u32x4 row = srow[own_row];
            const int first = FEW ? 16 * wave : 0;              // of the tile's keys
            score_map<true>(again(args), s, __uint_as_float(row.z), (float)(int)row.x, k0 + first, grp);
            if (!full) score_mask(again(args), seen, s, (int)row.x, (int)row.y, k0 + first, grp, true, !KV8 && ranges, (lds_int*)sdoc + first);
        }
        if constexpr (CAREFUL) careful_scores(s, which);
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < NJ; ++j) top = vmax(top, vmax(vmax(s[j][0], s[j][1]), vmax(s[j][2], s[j][3])));
        const float m_new = vmax(m, group_max(top)), alpha = exp2f(m - m_new);
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                s[j][q] = exp2f(s[j][q] - m_new);
                sum += s[j][q];
            }
        l = l * alpha + group_sum(sum);
        m = m_new;
#pragma unroll
        for (int i = 0; i < DV / 16; ++i) o[i] *= alpha;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float* row = sV[16 * (FEW ? wave : j) + 4 * grp + q];
                float v[DV / 16];
#pragma unroll
                for (int i = 0; i < DV / 16; ++i) {
                    if (i < WHOLE) v[i] = reinterpret_cast<const piece*>(row + o_col(i / W * W, ql))[0][i % W];
                    else v[i] = row[o_col(i, ql)];
                }
#pragma unroll
                for (int i = 0; i < DV / 16; ++i) {
                    if constexpr (CAREFUL) v[i] = careful(v[i], which);
                    o[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[i], s[j][q], o[i], 0, 0, 0);
                }
            }
    };
    auto run = [&](auto carefulc, int which) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < DV / 16; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        m = kNoScore;
        l = 0.f;
        Walk w = walk_part(seen, at.part, parts);
        if (at.r0 >= r1) w.at = w.hi;
        bool full = false, next_full = false;
        int tile = walk_next(seen, w, ranges, lane, full);
        if (tile >= 0) load(tile);
        while (tile >= 0) {
            __syncthreads();
            store();
            __syncthreads();
            const int next = walk_next(seen, w, ranges, lane, next_full), k0 = tile * kKTile;
            if (next >= 0) load(next);
            if ((k0 <= own_hi && k0 + kKTile > own_lo) || k0 < own_prefix) compute(carefulc, which, k0, full);
            tile = next;
            full = next_full;
        }
    };
    run(std::false_type{}, FINITE);
    bool bad = false;
#pragma unroll
    for (int i = 0; i < DV / 16; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) bad = bad || !(fabsf(o[i][e]) < INFINITY);
    if (__syncthreads_or(bad && ok)) {
        uint64_t bits[2];
#pragma unroll 1
        for (int which = POS; which <= FINITE; ++which) {
            run(std::true_type{}, which);
            if (which == POS) careful_bits<DV / 4>(o, bits[0]);
            else if (which == NEG) careful_bits<DV / 4>(o, bits[1]);
        }
        careful_join<DV / 4>(o, bits[0], bits[1]);
    }

    if constexpr (FEW) {
        __syncthreads();        // every wave is done with the tiles
        float* so = &sK[0][0] + (wave * 16 + ql) * (HD + 4);
        float (*sml)[16][2] = reinterpret_cast<float (*)[16][2]>(&sV[0][0]);
#pragma unroll
        for (int i = 0; i < DV / 16; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int col = o_col(i, 4 * grp + e);
                if (i >= WHOLE && col < HD) so[col] = o[i][e];
                if (i < WHOLE && i % W == 0) {
                    piece y;
#pragma unroll
                    for (int w = 0; w < W; ++w) y[w] = o[i + w][e];
                    *reinterpret_cast<piece*>(so + col) = y;
                }
            }
        if (grp == 0) {
            sml[wave][ql][0] = m;
            sml[wave][ql][1] = ok ? l : 0.f;
        }
        __syncthreads();
        join_waves<float, HD>(again(args), at, &sK[0][0], 16 * (HD + 4), sml, tid);
        return;
    }
    if (!mine) return;
    Args& z = again(args);
    const int64_t row = ((int64_t)at.b * z.Tq + t) * Hq + head;
    if (!ok) l = 0.f;
    const bool part = z.parts > 1;
    const int64_t pr = row * z.parts + at.part;
    if (part && grp == 0) {
        z.part_ml[pr * 2] = l != 0.f ? m : -INFINITY;
        z.part_ml[pr * 2 + 1] = l;
    }
    const float inv = part ? 1.f : l != 0.f ? 1.f / l : 0.f;
    float* to = part ? z.part_o + pr * HD : static_cast<float*>(z.out) + row * HD;
#pragma unroll
    for (int i = 0; i < DV / 16; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (!part) o[i][e] = l != 0.f ? o[i][e] * inv : 0.f;
            if (i >= WHOLE && o_col(i, 4 * grp + e) < HD) to[o_col(i, 4 * grp + e)] = o[i][e];
        }
#pragma unroll
    for (int i = 0; i < WHOLE; i += W)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float y[W];
#pragma unroll
            for (int w = 0; w < W; ++w) y[w] = o[i + w][e];
            __builtin_memcpy(to + o_col(i, 4 * grp + e), y, sizeof y);
        }
}

// ---------------------------------------------------------------------------
// bf16: NWV waves of QG groups of 16 rows over a double buffer of key and value
// tiles, one barrier a tile.  Tensors: tiles come straight into LDS, row-major
// (KvLayout), value operands by transposing reads.  Cache: the codes of the tile
// after the next are in registers, those of the next are decoded into LDS in the
// operands' own order as a tile begins, so that every read is 16 bytes at the
// lane's place; a code times its power of two is a bf16 value, so nothing is
// rounded on the way.
//   The probabilities are rounded to bf16 for P V (an fp32 product would take 16
// times the MFMA cycles), and the row sums are those of the rounded ones, from a
// column of ones beside the values.  A row's reference moves when a score exceeds
// it by more than 8 in log2 units.
//   The careful runs are a function of their own, called, not inlined: within the
// kernel they would cost the plain run 30 registers, and d = 128 its spills.
// ---------------------------------------------------------------------------
template <int HD, int QG, int NWV, bool KV8> struct TileShape {
    typedef AttnShape<bf16, HD> S;
    static constexpr int NV = S::DV / 16, NK = S::n32x, RT = 16 * QG * NWV;
    static constexpr int KT = KV8 ? 4 * NK * 512 : kKTile * HD;            // elements of a tile (tensors, values: + slack, read for d >= HD)
    static constexpr int VT = KV8 ? NV * 2 * 512 : kKTile * HD + 32;
    // Tensors whose rows end inside a step of the dot products: the lanes past the end read zeros, KJ apart as the keys' sixteens are.
    static constexpr bool PAST = !KV8 && HD % 32 != 0;
    // A wave's direct-to-LDS loads of a tile and operand; of swizzled rows they are a multiple of 16 rows apart, over which
    // the swizzle repeats: one offset for all.
    static constexpr int NJ = (HD / 8 + NWV - 1) / NWV, NO = KvLayout<HD>::SWZ ? 1 : NJ;
    // Waves of a SIMD: as many as the plain run's registers allow (the careful function would take them all).  The cache's
    // d = 72 at 3 waves keeps 38 registers in memory (16 heads, 1000 x 16 384 tokens: 171 us against 124).
    static constexpr int WAVES = HD == 128 || (KV8 && HD == 72 && QG == 2) ? 2 : QG == 2 || HD == 72 ? 3 : 4;
    // What a workgroup holds in LDS.  row: a row's position, document (-1: it sees nothing) and slope; tiles
    // that need none of them keep no registers for them.
    struct Lds {
        __attribute__((aligned(1024))) bf16 k[2][KT];
        __attribute__((aligned(1024))) bf16 v[2][VT];
        __attribute__((aligned(16))) int doc[KV8 ? 1 : 2][kKTile];
        u32x4 row[RT];
        u32x4 all;                                    // Seen's all_lo, all_hi, prefix and n
        unsigned off[KV8 ? 1 : 2 * NO][64 * NWV];     // tensors: each thread's offsets within a tile of keys, and of values
        __attribute__((aligned(16))) bf16 zero[PAST ? 3 * 16 * HD + 8 : 8];
    };
};

// One pass over the keys (CAREFUL: three); true if an output of this lane is not finite.
template <int HD, int QG, int NWV, bool KV8, bool CAREFUL>
__device__ __forceinline__ bool score_tile_body(Args* args, __attribute__((address_space(3))) typename TileShape<HD, QG, NWV, KV8>::Lds* lds) {
    typedef TileShape<HD, QG, NWV, KV8> TS;
    typedef KvLayout<HD> LY;
    typedef __attribute__((address_space(3))) const char lds_char;
    typedef __attribute__((address_space(3))) const u32x4 lds_u32x4;
    typedef __attribute__((address_space(3))) u32x4 lds_out;
    constexpr int NV = TS::NV, NK = TS::NK, CPR = HD / 8, NT = 64 * NWV, RT = TS::RT, KT = TS::KT, VT = TS::VT;
    constexpr bool PADSUM = HD % 16 != 0;
    Args& a = again(args);
    const int tid = threadIdx.x, lane = tid & 63, ql = lane & 15, grp = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Place at = place_of(a, RT, KV8);
    const int r1 = min(at.r0 + RT, at.count * a.G);
    Seen seen = seen_by(a, at.b, at.n, at.base + at.r0 / a.G, at.base + (r1 - 1) / a.G);
    const u32x2* ranges = nullptr;
    if (!KV8 && a.q_docs) {
        row_documents(a, at.b, at.r0, r1, lane, seen);
        ranges = uniform(a.ranges + (int64_t)at.b * ((a.Tk + kKTile - 1) / kKTile));
    }
    // Operands past the head: the queries' there are zeros, which a key that is not finite would turn into NaN.  In a row-major tile the
    // columns past one key's are the next one's first, which may be hidden: zeros are read in their place (one address for the lanes: 16 heads
    // of 16 384 tokens 1400 us, 1420 with the reads going on).
    if constexpr (KV8) {
        if constexpr (HD % 32 != 0)
            for (int x = tid; x < 2 * KT / 8; x += NT) ((lds_out*)&lds->k[0][0])[x] = u32x4{0u, 0u, 0u, 0u};
        if constexpr (PADSUM)
            for (int x = tid; x < 2 * VT / 8; x += NT) ((lds_out*)&lds->v[0][0])[x] = u32x4{0u, 0u, 0u, 0u};
    } else if (tid < 32) {
#pragma unroll
        for (int nb = 0; nb < 2; ++nb) lds->v[nb][kKTile * HD + tid] = (bf16)0.f;
        if constexpr (TS::PAST) lds->zero[tid / 8 * 16 * HD + tid % 8] = (bf16)0.f;
    }
    for (int x = tid; x < RT; x += NT) {
        const int r = at.r0 + x, t = r / a.G;
        int doc = t < at.count ? 0 : -1;
        if (!KV8 && ranges && doc == 0) doc = a.q_docs[(int64_t)at.b * a.Tq + t];
        const float slope = a.slopes ? a.slopes[at.hk * a.G + r - t * a.G] * 1.44269504f : 0.f;
        lds->row[x] = u32x4{(unsigned)(at.base + t), (unsigned)doc, __float_as_uint(slope), 0u};
    }
    if (!KV8 && tid == 0) lds->all = u32x4{(unsigned)seen.all_lo, (unsigned)seen.all_hi, (unsigned)seen.prefix, (unsigned)seen.n};
    const int myrow = 16 * wave * QG + ql;                          // of the first group
    bf16x8 qf[QG][NK];
#pragma unroll
    for (int g = 0; g < QG; ++g) {
        const int r = at.r0 + myrow + 16 * g, t = r / a.G;
        const bf16* qr = static_cast<const bf16*>(a.q) + at.b * a.q_batch + (int64_t)t * a.q_row + (int64_t)(at.hk * a.G + r - t * a.G) * HD;
#pragma unroll
        for (int c = 0; c < NK; ++c) {
            const int d = 32 * c + 8 * grp;
            qf[g][c] = __builtin_bit_cast(bf16x8, u32x4{0u, 0u, 0u, 0u});
            if (t < at.count && d < HD) qf[g][c] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(qr + d));
        }
    }
    __syncthreads();

    // ---- loading ----
    constexpr int NJ = TS::NJ;
    constexpr int UNITS = 4 * HD, PER = (UNITS + NT - 1) / NT;      // cache: 16-byte units of an operand's tile, of a thread
    u32x4 rk[KV8 ? PER : 1], rv[KV8 ? PER : 1];
    float ks = 0.f, vs = 0.f;
    const char* kb = uniform(static_cast<const char*>(a.k) + 2 * (at.b * a.k_batch + at.hk * HD));
    const char* vb = uniform(static_cast<const char*>(a.v) + 2 * (at.b * a.v_batch + at.hk * HD));
    const int* docs = a.k_docs + (int64_t)at.b * a.Tk;
    // Whole tiles are addressed from uniform rows and lanes' offsets where those fit 32 bits.
    const bool fits = (a.k_row > a.v_row ? a.k_row : a.v_row) < (int64_t)1 << 24;
    const uint32_t k_bytes = 2u * (uint32_t)a.k_row, v_bytes = 2u * (uint32_t)a.v_row;
    // (The offsets stand in LDS: registers for them would be spilled, and 20 instructions a tile make them anew.)
    if constexpr (!KV8) {
#pragma unroll
        for (int q = 0; q < TS::NO; ++q) {
            const uint32_t c = 64 * (wave + NWV * q) + lane, row = c / CPR, col = 16 * LY::slot(row, c % CPR);
            lds->off[q][tid] = row * k_bytes + col;
            lds->off[TS::NO + q][tid] = row * v_bytes + col;
        }
    }
    auto issue = [&](int tile, int buf) __attribute__((always_inline)) {
        if (fits && (tile + 1) * kKTile <= at.n) {
            const char *kt = kb + (uint64_t)k_bytes * (uint32_t)(tile * kKTile), *vt = vb + (uint64_t)v_bytes * (uint32_t)(tile * kKTile);
            const uint32_t lk = (uint32_t)(uintptr_t)&lds->k[buf][0] + 1024u * wave, lv = (uint32_t)(uintptr_t)&lds->v[buf][0] + 1024u * wave;
            uint32_t koff[TS::NO], voff[TS::NO];
#pragma unroll
            for (int q = 0; q < TS::NO; ++q) {
                koff[q] = lds->off[KV8 ? 0 : q][tid];
                voff[q] = lds->off[KV8 ? 0 : TS::NO + q][tid];
            }
#pragma unroll
            for (int q = 0; q < NJ; ++q) {
                if (NJ * NWV != CPR && wave + NWV * q >= CPR) break;
                const uint64_t more = LY::SWZ ? q * (64 * NWV / CPR) : 0;
                dma16s(uniform(kt + more * k_bytes), koff[LY::SWZ ? 0 : q], lk + 1024u * NWV * q);
                dma16s(uniform(vt + more * v_bytes), voff[LY::SWZ ? 0 : q], lv + 1024u * NWV * q);
            }
        } else {
            Args& z = again(args);
#pragma unroll 1
            for (int j = wave; j < CPR; j += NWV) {
                const int c = 64 * j + lane, row = c / CPR, col = at.hk * HD + 8 * LY::slot(row, c % CPR);
                const int64_t key = min(tile * kKTile + row, at.n - 1);      // (rows past the end repeat the last; nothing sees them)
                dma16(static_cast<const bf16*>(z.k) + at.b * z.k_batch + key * z.k_row + col, (const void*)&lds->k[buf][64 * j * 8]);
                dma16(static_cast<const bf16*>(z.v) + at.b * z.v_batch + key * z.v_row + col, (const void*)&lds->v[buf][64 * j * 8]);
            }
        }
        if (ranges && wave == 0) dma4(docs + min(tile * kKTile + lane, at.n - 1), (const void*)&lds->doc[KV8 ? 0 : buf][0]);
    };
    const uint8_t* codes = uniform(a.codes + (int64_t)at.bh * a.tiles * (2 * kKTile * HD));
    const float* scales = uniform(a.scales + (int64_t)at.bh * a.tiles * 2);
    auto fetch = [&](int tile) __attribute__((always_inline)) {
        const u32x4* c = reinterpret_cast<const u32x4*>(codes + (int64_t)tile * (2 * kKTile * HD));
        ks = scales[2 * tile];
        vs = scales[2 * tile + 1];
#pragma unroll
        for (int x = 0; x < PER; ++x) {
            const int u = tid + NT * x;
            if (UNITS % NT == 0 || u < UNITS) {
                rk[x] = c[u];
                rv[x] = c[UNITS + u];
            }
        }
    };
    auto decode = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < PER; ++x) {
            const int u = tid + NT * x;
            if (UNITS % NT != 0 && u >= UNITS) break;
            u32x4 lo, hi;
            const int l = u & 15, ch = (u >> 4) % CPR, jp = (u >> 4) / CPR;
            lds_out* dk = (lds_out*)&lds->k[buf][((2 * jp * NK + (ch >> 2)) * 64 + (ch & 3) * 16 + l) * 8];
            decode16(rk[x], ks, lo, hi);
            dk[0] = lo;
            dk[NK * 64] = hi;
            const int i = u >> 6, w = min(16, HD - 16 * i), kg = (u & 63) / w, cl = (u & 63) % w;
            lds_out* dv = (lds_out*)&lds->v[buf][(i * 128 + kg * 16 + cl) * 8];
            decode16(rv[x], vs, lo, hi);
            dv[0] = lo;
            dv[64] = hi;
        }
    };

    // ---- one tile ----
    uint32_t kofs[NK], vofs[NV];
#pragma unroll
    for (int c = 0; c < NK; ++c) kofs[c] = KV8 ? (uint32_t)(c * 1024 + lane * 16) : 2u * (uint32_t)LY::at(ql, 32 * c + grp * 8);
#pragma unroll
    for (int i = 0; i < NV; ++i) vofs[i] = KV8 ? (uint32_t)(i * 2048 + lane * 16) : 2u * (uint32_t)LY::at(4 * grp + (ql >> 2), 16 * i + 4 * (ql & 3));
    constexpr uint32_t KJ = KV8 ? NK * 1024u : 32u * HD;            // from 16 keys to the next 16
    const bool past = TS::PAST && 32 * (NK - 1) + 8 * grp >= HD;
    if (past) kofs[NK - 1] = (uint32_t)((lds_char*)&lds->zero[0] - (lds_char*)&lds->k[0][0]);
    auto move_keys = [&](int by) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < NK; ++c) kofs[c] += c == NK - 1 && past ? 0 : by;
    };
    f32x4 o[QG][NV], osum[QG];
    float m[QG];
    const int parts = a.parts;
    // What the exponent's one FMA scales: products (plain); of capped scores, c tanh z = c - 2c / (1 + e^2z), the
    // quotients -1 / (1 + e^2z) by 2c, whose constant falls out of the softmax; else finished scores.
    const bool plain = a.cap_log2 == 0.f && !a.slopes, capped = a.cap_log2 != 0.f && !a.slopes && !a.cap_wide;
    const float cap_exp = a.cap_exp, sc = plain ? a.scale_log2 : capped ? 2.f * a.cap_log2 : 1.f;
    auto step = [&](int k0, bool full, int which, int buf) __attribute__((always_inline)) {
        lds_char *Kb = (lds_char*)&lds->k[0][0], *Vb = (lds_char*)&lds->v[0][0];
        f32x4 s[QG][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
#pragma unroll
            for (int c = 0; c < NK; ++c) {
                const bf16x8 kf = __builtin_bit_cast(bf16x8, *(lds_u32x4*)(Kb + kofs[c] + j * KJ));
#pragma unroll
                for (int g = 0; g < QG; ++g)
                    s[g][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[g][c], c == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[g][j], 0, 0, 0);
            }
            if constexpr (CAREFUL) __builtin_amdgcn_sched_barrier(0);
        }
        if (capped) {
#pragma unroll
            for (int g = 0; g < QG; ++g)
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[g][j][r] = __builtin_amdgcn_rcpf(-1.f - __builtin_amdgcn_exp2f(s[g][j][r] * cap_exp));
        } else if (!plain) {
#pragma unroll
            for (int g = 0; g < QG; ++g) {
                const u32x4 row = lds->row[myrow + 16 * g];
                score_map<false>(again(args), s[g], __uint_as_float(row.z), (float)(int)row.x, k0, grp);
            }
        }
        if (!full) {
            // (Documents of ten tiles leave four of ten to be masked for them alone: 16 heads of 16 384 tokens, d = 72, six draws: 143 to
            // 229 us with both masks, 135 to 192 so.)
            bool by_pos = true;
            if (!KV8 && ranges) {
                const u32x4 x = lds->all;
                const int k1 = k0 + kKTile - 1;
                by_pos = uniform(k1 >= (int)x.w || ((k1 > (int)x.y || k0 < (int)x.x) && k1 >= (int)x.z));
            }
#pragma unroll
            for (int g = 0; g < QG; ++g) {
                const u32x4 row = lds->row[myrow + 16 * g];
                score_mask(again(args), seen, s[g], (int)row.x, (int)row.y, k0, grp, by_pos, !KV8 && ranges, (lds_int*)&lds->doc[KV8 ? 0 : buf][0]);
            }
        }
        if constexpr (CAREFUL)
#pragma unroll
            for (int g = 0; g < QG; ++g) careful_scores(s[g], which);
        float top[QG];
        bool move = false;
#pragma unroll
        for (int g = 0; g < QG; ++g) {
            const f32x4* v = s[g];
            const float m1 = vmax(vmax(v[0][0], v[0][1]), v[0][2]), m2 = vmax(vmax(v[0][3], v[1][0]), v[1][1]);
            const float m3 = vmax(vmax(v[1][2], v[1][3]), v[2][0]), m4 = vmax(vmax(v[2][1], v[2][2]), v[2][3]);
            const float m5 = vmax(vmax(v[3][0], v[3][1]), v[3][2]), m6 = vmax(vmax(m1, m2), v[3][3]);
            top[g] = vmax(vmax(vmax(m3, m4), m5), m6);
            move |= (top[g] - m[g]) * sc > 8.f;
        }
        if (__any(move)) {
#pragma unroll
            for (int g = 0; g < QG; ++g) {
                const float m_new = vmax(m[g], group_max(top[g])), alpha = __builtin_amdgcn_exp2f((m[g] - m_new) * sc);
                m[g] = m_new;
                if constexpr (!PADSUM) osum[g] *= alpha;
#pragma unroll
                for (int i = 0; i < NV; ++i) o[g][i] *= alpha;
            }
        }
#pragma unroll
        for (int g = 0; g < QG; ++g) {
            const float mc = m[g] * sc;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) s[g][j][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[g][j][r], sc, -mc));
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            bf16x8 pf[QG];
#pragma unroll
            for (int g = 0; g < QG; ++g)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    pf[g][r] = (bf16)s[g][2 * u][r];
                    pf[g][4 + r] = (bf16)s[g][2 * u + 1][r];
                }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                bf16x8 vf;
                if constexpr (KV8) {
                    vf = __builtin_bit_cast(bf16x8, *(lds_u32x4*)(Vb + vofs[i] + 1024u * u));
                } else {
                    // keys 32u + 4grp + 0..3 and 32u + 16 + 4grp + 0..3 of column 16i + ql
                    lds_char* p = Vb + vofs[i] + 64u * u * HD;
                    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p));
                    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p + 32 * HD)));
                    vf = __builtin_bit_cast(bf16x8, u32x4{lo.x, lo.y, hi.x, hi.y});
                }
                if constexpr (CAREFUL) vf = __builtin_bit_cast(bf16x8, careful(__builtin_bit_cast(u32x4, vf), which));
                if (PADSUM && i == NV - 1 && ql >= HD - 16 * i)
                    vf = __builtin_bit_cast(bf16x8, u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});
#pragma unroll
                for (int g = 0; g < QG; ++g) o[g][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[g], o[g][i], 0, 0, 0);
                if constexpr (CAREFUL) __builtin_amdgcn_sched_barrier(0);      // (few registers: they count for the whole kernel)
            }
            if constexpr (!PADSUM) {
                const bf16x8 ones = __builtin_bit_cast(bf16x8, u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});
#pragma unroll
                for (int g = 0; g < QG; ++g) osum[g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[g], osum[g], 0, 0, 0);
            }
        }
    };
    auto run = [&](int which) __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < QG; ++g) {
            m[g] = kNoScore;
            osum[g] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < NV; ++i) o[g][i] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        Walk w = walk_part(seen, at.part, parts);
        if (at.r0 >= r1) w.at = w.hi;
        bool full = false, full1 = false, full2 = false;
        int t0 = walk_next(seen, w, ranges, lane, full), t1 = -1, t2 = -1;
        if (t0 < 0) return;
        if constexpr (KV8) {
            fetch(t0);
            t1 = walk_next(seen, w, ranges, lane, full1);
            decode(0);
            if (t1 >= 0) fetch(t1);
        } else {
            issue(t0, 0);
        }
        // One body for both buffers: lanes' places move from one to the other and back (two bodies cost the output's
        // registers a copy between them).
        int kmove = 2 * KT, vmove = 2 * VT;
        for (int buf = 0; t0 >= 0; buf ^= 1) {
            if constexpr (KV8) {
                __syncthreads();
                t2 = -1;
                if (t1 >= 0) {
                    decode(buf ^ 1);
                    t2 = walk_next(seen, w, ranges, lane, full2);
                    if (t2 >= 0) fetch(t2);
                }
            } else {
                t1 = walk_next(seen, w, ranges, lane, full1);
                __builtin_amdgcn_s_waitcnt((0 & 15) | (7 << 4) | (15 << 8));   // vmcnt(0): this wave's loads of the tile
                __syncthreads();
                if (t1 >= 0) issue(t1, buf ^ 1);
            }
            step(t0 * kKTile, full, which, buf);
            move_keys(kmove);
#pragma unroll
            for (int i = 0; i < NV; ++i) vofs[i] += vmove;
            kmove = -kmove;
            vmove = -vmove;
            t0 = t1;
            full = full1;
            if constexpr (KV8) {
                t1 = t2;
                full1 = full2;
            }
        }
        if (kmove < 0) {        // back to the first buffer
            move_keys(kmove);
#pragma unroll
            for (int i = 0; i < NV; ++i) vofs[i] += vmove;
        }
    };
    if constexpr (CAREFUL) {
        uint64_t bits[2][QG];
#pragma unroll 1
        for (int which = POS; which <= FINITE; ++which) {
            __syncthreads();        // the run before is done with the tiles
            run(which);
            // (The row sums in the last block are no outputs.)
            const uint64_t outs = 16 * (NV - 1) + 4 * grp < HD ? ~(uint64_t)0 : ((uint64_t)1 << (4 * NV - 4)) - 1;
            uint64_t now[QG];
#pragma unroll
            for (int g = 0; g < QG; ++g) {
                careful_bits<4 * NV>(o[g], now[g]);
                if (which == POS) bits[0][g] = now[g] & outs;
                if (which == NEG) bits[1][g] = now[g] & outs;
            }
        }
#pragma unroll
        for (int g = 0; g < QG; ++g) careful_join<4 * NV>(o[g], bits[0][g], bits[1][g]);
    } else {
        run(FINITE);
    }

    Args& z = again(args);
    bool bad = false;
#pragma unroll
    for (int g = 0; g < QG; ++g) {
        float l = osum[g][0];
        if constexpr (PADSUM) {
            // Lanes 32-63 hold the padding rows of the last block (the row sums), lanes 0-31 take them from l ^ 32.
            const float own = o[g][NV - 1][0], other = __shfl_xor(own, 32);
            l = lane < 32 ? other : own;
        }
        const int r = at.r0 + myrow + 16 * g, t = r / z.G;
        if ((int)lds->row[myrow + 16 * g].y < 0) l = 0.f;
        if (t >= z.Tq) continue;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) bad |= !(fabsf(o[g][i][e]) < INFINITY);
        const int64_t row = ((int64_t)at.b * z.Tq + t) * (z.Hk * z.G) + at.hk * z.G + r - t * z.G;
        if (z.parts > 1) {
            const int64_t pr = row * z.parts + at.part;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (16 * i + 4 * grp < HD) *reinterpret_cast<f32x4*>(z.part_o + pr * HD + 16 * i + 4 * grp) = o[g][i];
            if (grp == 0) {
                z.part_ml[pr * 2] = l != 0.f ? m[g] * sc : -INFINITY;
                z.part_ml[pr * 2 + 1] = l;
            }
            continue;
        }
        const float inv = l != 0.f ? 1.f / l : 0.f;
        bf16* out = static_cast<bf16*>(z.out) + row * HD;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int d = 16 * i + 4 * grp;
            if (d >= HD) continue;
            bf16x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = (bf16)(l != 0.f ? o[g][i][e] * inv : 0.f);
            __builtin_memcpy(out + d, &v, sizeof v);
        }
    }
    return bad;
}

template <int HD, int QG, int NWV, bool KV8>
__device__ __attribute__((noinline)) void score_tile_careful(Args* args,
                                                             __attribute__((address_space(3))) typename TileShape<HD, QG, NWV, KV8>::Lds* lds) {
    score_tile_body<HD, QG, NWV, KV8, true>(uniform(args), lds);
}

template <int HD, int QG, int NWV, bool KV8>
__global__ __launch_bounds__(64 * NWV) __attribute__((amdgpu_waves_per_eu(TileShape<HD, QG, NWV, KV8>::WAVES))) void score_tile_kernel(ScoreArgs) {
    __shared__ typename TileShape<HD, QG, NWV, KV8>::Lds lds;
    auto* at = (__attribute__((address_space(3))) typename TileShape<HD, QG, NWV, KV8>::Lds*)&lds;
    Args* args = kernel_arguments();
    if (__syncthreads_or(score_tile_body<HD, QG, NWV, KV8, false>(args, at))) score_tile_careful<HD, QG, NWV, KV8>(args, at);
}

// ---------------------------------------------------------------------------
// bf16, up to 16 rows of a key head (single tokens): every wave takes a part of the
// keys of its own, with no barrier until the four waves of a workgroup meet in LDS.
// Keys (and from the cache values too) go straight into MFMA operands; a tensor's
// values through the wave's tile in LDS.  Bound by the keys' and values' bytes.
// ---------------------------------------------------------------------------
template <int HD, bool KV8, bool NT>
__global__ __launch_bounds__(256) void score_few_kernel(ScoreArgs) {
    Args* args = kernel_arguments();
    Args& a = again(args);
    typedef AttnShape<bf16, HD> S;
    typedef KvLayout<HD> LY;
    typedef __attribute__((address_space(3))) const char lds_char;
    constexpr int NV = S::DV / 16, NK = S::n32x, CPR = HD / 8;
    constexpr int TILE = kKTile * HD + 32;                // tensors: a wave's value tile + slack; then its outputs, fp32
    __shared__ __attribute__((aligned(1024))) bf16 sv[4][KV8 ? 32 * HD + 128 : TILE];
    __shared__ float sml[4][16][2];
    __shared__ __attribute__((aligned(16))) int sdoc[4][KV8 ? 4 : kKTile];
    const int tid = threadIdx.x, lane = tid & 63, ql = lane & 15, grp = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Place at = place_of(a, 16, KV8);
    const int rows = at.count * a.G;
    const int t = ql / a.G, head = at.hk * a.G + ql - t * a.G;
    bool ok = ql < rows;
    int doc = 0;
    Seen seen = seen_by(a, at.b, at.n, at.base, at.base + (rows - 1) / a.G);
    const u32x2* ranges = nullptr;
    if (!KV8 && a.q_docs) {
        row_documents(a, at.b, 0, rows, lane, seen);
        doc = ok ? a.q_docs[(int64_t)at.b * a.Tq + t] : -1;
        ok = doc >= 0;
        ranges = a.ranges + (int64_t)at.b * ((a.Tk + kKTile - 1) / kKTile);
    }
    const int pos = at.base + t;
    const float slope = a.slopes && ok ? a.slopes[head] * 1.44269504f : 0.f;
    bf16x8 qf[NK];
    const bf16* qr = static_cast<const bf16*>(a.q) + at.b * a.q_batch + (int64_t)t * a.q_row + (int64_t)head * HD;
#pragma unroll
    for (int c = 0; c < NK; ++c) {
        const int d = 32 * c + grp * 8;
        qf[c] = __builtin_bit_cast(bf16x8, u32x4{0u, 0u, 0u, 0u});
        if (ok && d < HD) qf[c] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(qr + d));
    }
    if (!KV8 && lane < 32) sv[wave][kKTile * HD + lane] = (bf16)0.f;
    const bf16* kb = static_cast<const bf16*>(a.k) + at.b * a.k_batch + at.hk * HD;
    const bf16* vb = static_cast<const bf16*>(a.v) + at.b * a.v_batch + at.hk * HD;
    const uint8_t* codes = a.codes + (int64_t)at.bh * a.tiles * (2 * kKTile * HD);
    const float* scales = a.scales + (int64_t)at.bh * a.tiles * 2;
    const int* docs = a.k_docs + (int64_t)at.b * a.Tk;
    const int64_t k_row = a.k_row, v_row = a.v_row;
    lds_char* Vb = (lds_char*)&sv[wave][0];
    const int parts = a.parts;
    f32x4 o[NV];
    float m, l;
    auto run = [&](auto carefulc, int which) __attribute__((always_inline)) {
        constexpr bool CAREFUL = decltype(carefulc)::value;
#pragma unroll
        for (int i = 0; i < NV; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        m = kNoScore;
        l = 0.f;
        Walk w = walk_part(seen, at.part * 4 + wave, parts * 4);
        if (rows == 0) w.at = w.hi;
        bool full = false;
        for (int tile = walk_next(seen, w, ranges, lane, full); tile >= 0; tile = walk_next(seen, w, ranges, lane, full)) {
            const int k0 = tile * kKTile;
            u32x4 kf[4][NK], vc[KV8 ? NV : 1];
            float vs = 0.f;
            if constexpr (KV8) {
                const u32x4* c = reinterpret_cast<const u32x4*>(codes + (int64_t)tile * (2 * kKTile * HD));
                const float ks = scales[2 * tile];
                vs = scales[2 * tile + 1];
                u32x4 kc[2][NK];
#pragma unroll
                for (int jp = 0; jp < 2; ++jp)
#pragma unroll
                    for (int x = 0; x < NK; ++x) {
                        kc[jp][x] = u32x4{0u, 0u, 0u, 0u};
                        const u32x4* from = c + (jp * CPR + 4 * x + grp) * 16 + ql;
                        if (4 * x + grp < CPR) kc[jp][x] = NT ? __builtin_nontemporal_load(from) : *from;
                    }
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int wd = min(16, HD - 16 * i);
                    vc[i] = u32x4{0u, 0u, 0u, 0u};
                    const u32x4* from = c + 4 * HD + i * 64 + grp * wd + ql;
                    if (ql < wd) vc[i] = NT ? __builtin_nontemporal_load(from) : *from;
                }
#pragma unroll
                for (int jp = 0; jp < 2; ++jp)
#pragma unroll
                    for (int x = 0; x < NK; ++x) decode16(kc[jp][x], ks, kf[2 * jp][x], kf[2 * jp + 1][x]);
            } else {
#pragma unroll
                for (int j = 0; j < CPR; ++j) {
                    const int c = 64 * j + lane, row = c / CPR;
                    const bf16* from = vb + (int64_t)min(k0 + row, at.n - 1) * v_row + 8 * LY::slot(row, c % CPR);
                    if constexpr (NT) dma16_nt(from, &sv[wave][64 * j * 8]);
                    else dma16(from, &sv[wave][64 * j * 8]);
                }
                if (ranges) dma4(docs + min(k0 + lane, at.n - 1), &sdoc[wave][0]);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bf16* kr = kb + (int64_t)min(k0 + 16 * j + ql, at.n - 1) * k_row;
#pragma unroll
                    for (int c = 0; c < NK; ++c) {
                        const int d = 32 * c + grp * 8;
                        kf[j][c] = d < HD ? *reinterpret_cast<const u32x4*>(kr + d) : u32x4{0u, 0u, 0u, 0u};
                    }
                }
            }
            f32x4 s[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < NK; ++c)
                    s[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[j][c]), qf[c], s[j], 0, 0, 0);
            }
            score_map<false>(again(args), s, slope, (float)pos, k0, grp);
            if (!KV8) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // the value tile and the documents
            if (!full) score_mask(again(args), seen, s, pos, doc, k0, grp, true, !KV8 && ranges, (lds_int*)sdoc[wave]);
            if constexpr (CAREFUL) careful_scores(s, which);
            float top = -INFINITY;
#pragma unroll
            for (int j = 0; j < 4; ++j) top = vmax(top, vmax(vmax(s[j][0], s[j][1]), vmax(s[j][2], s[j][3])));
            const float m_new = vmax(m, group_max(top)), alpha = __builtin_amdgcn_exp2f(m - m_new);
            m = m_new;
            l *= alpha;
            bf16x8 pf[2];
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const bf16 p = (bf16)__builtin_amdgcn_exp2f(s[j][r] - m);
                    pf[j >> 1][4 * (j & 1) + r] = p;
                    l += (float)p;
                }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                o[i] *= alpha;
                u32x4 vf[2];
                if constexpr (KV8) {
                    decode16(vc[i], vs, vf[0], vf[1]);
                } else {
                    const uint32_t ofs = 2u * (uint32_t)LY::at(4 * grp + (ql >> 2), 16 * i + 4 * (ql & 3));
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        lds_char* p = Vb + ofs + 64u * u * HD;
                        const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p));
                        const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p + 32 * HD)));
                        vf[u] = u32x4{lo.x, lo.y, hi.x, hi.y};
                    }
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    if constexpr (CAREFUL) vf[u] = careful(vf[u], which);
                    o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf[u]), pf[u], o[i], 0, 0, 0);
                }
            }
        }
    };
    run(std::false_type{}, FINITE);
    bool bad = false;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) bad = bad || (ok && 16 * i + 4 * grp + e < HD && !(fabsf(o[i][e]) < INFINITY));
    if (__any(bad)) {
        uint64_t bits[2];
#pragma unroll 1
        for (int which = POS; which <= FINITE; ++which) {
            run(std::true_type{}, which);
            if (which == POS) careful_bits<4 * NV>(o, bits[0]);
            else if (which == NEG) careful_bits<4 * NV>(o, bits[1]);
        }
        careful_join<4 * NV>(o, bits[0], bits[1]);
    }
    l = group_sum(l);
    if (!ok) l = 0.f;
    // The waves meet: outputs [16][HD + 4] fp32 over their value tiles.
    float* so = reinterpret_cast<float*>(&sv[wave][0]);
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (16 * i + 4 * grp < HD) *reinterpret_cast<f32x4*>(so + ql * (HD + 4) + 16 * i + 4 * grp) = o[i];
    if (grp == 0) {
        sml[wave][ql][0] = m;
        sml[wave][ql][1] = l;
    }
    __syncthreads();
    join_waves<bf16, HD>(again(args), at, reinterpret_cast<const float*>(&sv[0][0]), (KV8 ? 32 * HD + 128 : TILE) / 2, sml, tid);
}

// The kernel of a plan; rows a workgroup and the parts are in the plan.
template <bool KV8>
static int launch_score(int dtype, const ScorePlan& p, const ScoreArgs& a, hipStream_t s) {
    const int64_t wgs = (int64_t)a.B * a.Hk * (((int64_t)a.Tq * a.G + p.rows - 1) / p.rows) * p.parts;
    const dim3 g((unsigned)wgs);
#define BC_SCORE(HD)                                                                                          \
    case HD:                                                                                                  \
        if (dtype == BC_F32 && p.rows == 16) launch_k(score_f32_kernel<HD, KV8, true>, g, dim3(256), s, a);   \
        else if (dtype == BC_F32) launch_k(score_f32_kernel<HD, KV8, false>, g, dim3(256), s, a);             \
        else if (p.rows == 16 && a.nt) launch_k(score_few_kernel<HD, KV8, true>, g, dim3(256), s, a);         \
        else if (p.rows == 16) launch_k(score_few_kernel<HD, KV8, false>, g, dim3(256), s, a);                \
        else if (p.rows == 64) launch_k(score_tile_kernel<HD, 1, 4, KV8>, g, dim3(256), s, a);                \
        else launch_k(score_tile_kernel<HD, 2, 4, KV8>, g, dim3(256), s, a);                                  \
        break;
    switch (a.d) {
        BC_SCORE(32) BC_SCORE(64) BC_SCORE(72) BC_SCORE(128)
        default: return fail(BC_ERR_UNSUPPORTED, "head_dim %d (supported: 32, 64, 72, 128)", a.d);
    }
#undef BC_SCORE
    return check_launch(KV8 ? "attention over the cache" : "masked attention");
}

}  // namespace bc
