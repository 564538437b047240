// Rotary positions of queries and keys, for every layout that the models use.
//
// Pair j of an axis with n columns turns by the angle p f_j, p the token's position
// on that axis:  y_a = m (x_a cos - x_b sin),  y_b = m (x_a sin + x_b cos).  The
// angle is formed and reduced to an eighth of a turn in 64 bits (at position 10^6 a
// 32-bit angle is off by 0.06), the sine and cosine of the rest are Taylor sums in 32.
#include <algorithm>
#include <cmath>

#include "ops.h"

namespace bc {

constexpr int kRopeMaxDim = 256;

struct RopeArgs {
    const void *q, *k;
    void *qo, *ko;
    int64_t q_batch, q_row, k_batch, k_row, qo_batch, qo_row, ko_batch, ko_row;
    int B, T, Hq, Hk, d, pairs, axes, items, tokens;    // items: a head's; tokens: a workgroup's
    uint32_t by_token, by_items;                        // 2^32 / (items of a token), / items, rounded up; 0 for one
    const int* pos;
    int64_t pos_batch;
    int64_t start;
    int end[3];                                         // pairs up to the end of each axis
    float amplitude;
    int inverse;
    double turns[kRopeMaxDim / 2];                      // turns per position of each pair
    // An item: VEC columns from `col` on.  dist 0: copied, else columns col + i and
    // col + dist + i are pair + i.
    struct Item {
        int16_t col, dist, pair, pad;
    } item[kRopeMaxDim];
};

// sin and cos of 2 pi r.
__device__ __forceinline__ float2 turn_of(double r) {
    const double n = rint(4.0 * r);
    const float x = (float)((r - 0.25 * n) * 6.283185307179586);      // within pi / 4
    const int quarter = (int)((int64_t)n & 3);
    const float y = x * x;
    const float s = x * fmaf(y, fmaf(y, fmaf(y, fmaf(y, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), 1.f);
    const float c = fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
    const float a = quarter & 1 ? c : s, b = quarter & 1 ? s : c;
    return float2{quarter & 2 ? -a : a, (quarter + 1) & 2 ? -b : b};
}

template <typename T, int VEC> struct RopeVec {
    T v[VEC];
};
// An item, past the caches where it is 16 bytes: the rows are read once.
template <typename T, int VEC, typename V> __device__ __forceinline__ V rope_load(const V* p) {
    if constexpr (sizeof(V) == 16) {
        const u32x4 x = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
        return __builtin_bit_cast(RopeVec<T, VEC>, x);
    } else {
        return *p;
    }
}

// A workgroup takes some tokens.  The first items of its rows are requested, then the
// tokens' sines and cosines, which all heads share, go into LDS, then the items are
// turned.  Bound by the rows' bytes; the angles' 64-bit work lies under the loads:
// 14 310 tokens of 24 + 24 heads of 128 in bf16 (352 MB) 68 us, 5.2 TB/s (58 on the same
// tensors again); 1.26 times that with the rows requested after the angles, 1.13 with the
// inputs kept in the caches.  The outputs stay in them for the attention (past them as
// well: 0.98).
// PAIRS: rows of whole 16-byte items, neighbours paired, whose place is their number;
// else items come from the table.
template <typename T_, int VEC, bool PAIRS>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
    typedef elem_t<T_> T;
    typedef RopeVec<T, VEC> __attribute__((aligned(VEC * sizeof(T)))) V;
    extern __shared__ float2 cs[];                       // [tokens][pairs]
    constexpr int U = PAIRS ? 6 : 3;                     // items of a thread on their way together
    const int tid = threadIdx.x;
    const int64_t t0 = (int64_t)blockIdx.x * a.tokens, all = (int64_t)a.B * a.T;
    const int here = (int)min((int64_t)a.tokens, all - t0);
    const int64_t b0 = t0 / a.T;
    const int first = (int)(t0 - b0 * a.T);              // the workgroup's first token in its sample
    const int per = (a.Hq + a.Hk) * a.items, n = here * per;
    V v0[U], v1[PAIRS ? 1 : U];
    RopeArgs::Item it[U];
    int token[U];
    T* out[U];
    auto request = [&](int x0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int x = min(x0 + 256 * u, n - 1);
            const int tl = a.by_token ? (int)__umulhi((uint32_t)x, a.by_token) : x, y = x - tl * per;
            const int head = a.by_items ? (int)__umulhi((uint32_t)y, a.by_items) : y;
            const int i = y - head * a.items;
            if constexpr (PAIRS) it[u] = {0, (int16_t)(i * VEC / 2 < a.pairs ? -1 : 0), (int16_t)(i * VEC / 2), 0};
            else it[u] = a.item[i];
            int64_t b = b0;
            int t = first + tl;
            while (t >= a.T) {
                t -= a.T;
                ++b;
            }
            const bool key = head >= a.Hq;
            const int col = PAIRS ? (key ? y - a.Hq * a.items : y) * VEC : (key ? head - a.Hq : head) * a.d + it[u].col;
            const T* in = static_cast<const T*>(key ? a.k : a.q) + (b * (key ? a.k_batch : a.q_batch) + t * (key ? a.k_row : a.q_row)) + col;
            out[u] = static_cast<T*>(key ? a.ko : a.qo) + (b * (key ? a.ko_batch : a.qo_batch) + t * (key ? a.ko_row : a.qo_row)) + col;
            token[u] = tl;
            v0[u] = rope_load<T, VEC>(reinterpret_cast<const V*>(in));
            if constexpr (!PAIRS)
                if (it[u].dist > 0) v1[u] = rope_load<T, VEC>(reinterpret_cast<const V*>(in + it[u].dist));
        }
    };
    request(tid);
    for (int x = tid; x < here * a.pairs; x += 256) {
        const int tl = x / a.pairs, j = x - tl * a.pairs;
        int64_t b = b0;
        int t = first + tl;
        while (t >= a.T) {
            t -= a.T;
            ++b;
        }
        const int axis = (j >= a.end[0]) + (j >= a.end[1]);
        const double p = a.pos ? (double)a.pos[b * a.pos_batch + (int64_t)t * a.axes + axis] : (double)(a.start + t);
        const double r = p * a.turns[j];
        float2 v = turn_of(r - rint(r));
        v.x *= a.inverse ? -a.amplitude : a.amplitude;
        v.y *= a.amplitude;
        cs[x] = v;
    }
    __syncthreads();
    for (int x0 = tid; x0 < n;) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (x0 + 256 * u >= n) break;
            const float2* c = cs + token[u] * a.pairs + it[u].pair;
            if (it[u].dist == 0) {
                *reinterpret_cast<V*>(out[u]) = v0[u];
            } else if (PAIRS) {
                V w = v0[u];
#pragma unroll
                for (int e = 0; e < VEC; e += 2) {
                    if (it[u].pair + e / 2 >= a.pairs) break;
                    const float2 z = c[e / 2];
                    const float p = (float)v0[u].v[e], r = (float)v0[u].v[e + (VEC > 1)];
                    w.v[e] = (T)(p * z.y - r * z.x);
                    w.v[e + (VEC > 1)] = (T)(p * z.x + r * z.y);
                }
                *reinterpret_cast<V*>(out[u]) = w;
            } else {
                const V va = v0[u], vb = v1[PAIRS ? 0 : u];
                V w0, w1;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float2 z = c[e];
                    const float p = (float)va.v[e], r = (float)vb.v[e];
                    w0.v[e] = (T)(p * z.y - r * z.x);
                    w1.v[e] = (T)(p * z.x + r * z.y);
                }
                *reinterpret_cast<V*>(out[u]) = w0;
                *reinterpret_cast<V*>(out[u] + it[u].dist) = w1;
            }
        }
        x0 += 256 * U;
        if (x0 < n) request(x0);
    }
}

// One of the call's views: rows of H heads.
struct RopeView {
    const void* p;
    int64_t batch, row;
    int H;
};

// Whether two views share a value.  Views of rows with equal strides, as those into
// one projection's rows are, may lie in each other's gaps.
static bool views_meet(const RopeView& x, const RopeView& y, int B, int T, int d, int e) {
    if (!x.p || !y.p) return false;
    auto bytes = [&](const RopeView& v) { return ((B - 1) * v.batch + (T - 1) * v.row + (int64_t)v.H * d) * e; };
    if (!overlap(x.p, bytes(x), y.p, bytes(y))) return false;
    if (T > 1 && (x.row != y.row || x.row == 0)) return true;
    if (B > 1 && x.batch != y.batch) return true;
    int64_t step = T > 1 ? x.row : x.batch;
    if (B == 1 && T == 1) return true;
    if (B > 1 && T > 1 && x.batch % x.row != 0) return true;
    if (step == 0) return true;
    const int64_t gap = static_cast<const char*>(y.p) - static_cast<const char*>(x.p);
    if (gap % e) return true;
    const int64_t m = ((gap / e) % step + step) % step;         // y's first column in x's rows
    return m < (int64_t)x.H * d || m + (int64_t)y.H * d > step;
}

}  // namespace bc

using namespace bc;

extern "C" {

int bc_rope_frequencies(int n, double theta, int scaling, double factor, int64_t original, double beta_fast, double beta_slow, double* out) {
    clear_error();
    if (!out) return fail(BC_ERR_INVALID_ARG, "NULL pointer");
    if (n < 2 || n % 2 || n > kRopeMaxDim) return fail(BC_ERR_INVALID_ARG, "%d columns: even, 2 to %d", n, kRopeMaxDim);
    if (!(theta > 0.0 && theta < 1e300)) return fail(BC_ERR_INVALID_ARG, "theta %g", theta);
    if (scaling < BC_ROPE_NONE || scaling > BC_ROPE_PARTS) return fail(BC_ERR_INVALID_ARG, "scaling %d", scaling);
    if (scaling != BC_ROPE_NONE && !(factor >= 1.0 && factor <= 1e6)) return fail(BC_ERR_INVALID_ARG, "factor %g outside [1, 1e6]", factor);
    if (scaling == BC_ROPE_PARTS && !(original >= 1 && beta_slow >= 0.0 && beta_fast > beta_slow && beta_fast < 1e12))
        return fail(BC_ERR_INVALID_ARG, "original %lld, beta_fast %g, beta_slow %g", (long long)original, beta_fast, beta_slow);
    if (scaling == BC_ROPE_NTK && n > 2) theta *= std::pow(factor, n / (n - 2.0));
    for (int j = 0; j < n / 2; ++j) {
        double f = std::pow(theta, -2.0 * j / n);
        if (scaling == BC_ROPE_LINEAR) f /= factor;
        if (scaling == BC_ROPE_PARTS) {
            const double turns = (double)original * f / (2.0 * M_PI);
            const double keep = std::min(1.0, std::max(0.0, (turns - beta_slow) / (beta_fast - beta_slow)));
            f *= keep + (1.0 - keep) / factor;
        }
        out[j] = f;
    }
    return BC_OK;
}

int bc_rope(const bc_rope_desc* r, void* stream) {
    clear_error();
    if (!r) return fail(BC_ERR_INVALID_ARG, "NULL pointer");
    if (r->B < 0 || r->T < 0 || r->Hq < 1 || r->Hk < 0 || r->d < 1) return fail(BC_ERR_INVALID_ARG, "rope: %d x %d tokens, %d + %d heads of %d", r->B, r->T, r->Hq, r->Hk, r->d);
    if (r->d > kRopeMaxDim) return fail(BC_ERR_UNSUPPORTED, "head_dim %d above %d", r->d, kRopeMaxDim);
    // (Items of a token are counted by multiplying with a 32-bit inverse: below 2^16.)
    if (((int64_t)r->Hq + r->Hk) * r->d > 65535 || (int64_t)r->B * r->T > ((int64_t)1 << 40))
        return fail(BC_ERR_UNSUPPORTED, "rope: %d x %d tokens of %d + %d heads", r->B, r->T, r->Hq, r->Hk);
    if (r->dtype != BC_F32 && r->dtype != BC_BF16) return fail(BC_ERR_INVALID_ARG, "dtype %d", r->dtype);
    if (r->layout != BC_ROPE_PAIRS && r->layout != BC_ROPE_HALVES) return fail(BC_ERR_INVALID_ARG, "layout %d", r->layout);
    if (r->axes < 1 || r->axes > 3) return fail(BC_ERR_INVALID_ARG, "%d axes: 1 to 3", r->axes);
    if (!r->freqs) return fail(BC_ERR_INVALID_ARG, "freqs is NULL");
    if (!(std::fabs(r->amplitude) <= 1e6f)) return fail(BC_ERR_INVALID_ARG, "amplitude %g", r->amplitude);
    int rot = 0;
    RopeArgs a = {};
    for (int x = 0; x < 3; ++x) {
        const int n = x < r->axes ? r->axis_dim[x] : 0;
        if (x < r->axes && (n < 2 || n % 2 || n > r->d - rot)) return fail(BC_ERR_INVALID_ARG, "axis %d of %d columns (even, together at most %d)", x, n, r->d);
        rot += n;
        a.end[x] = rot / 2;
    }
    if (!r->pos && r->axes > 1) return fail(BC_ERR_INVALID_ARG, "positions are needed for %d axes", r->axes);
    if (r->pos && (reinterpret_cast<uintptr_t>(r->pos) % 4 || !strides_fit(r->B, r->pos_batch, r->T, r->axes)))
        return fail(BC_ERR_INVALID_ARG, "positions: 4-byte aligned, batch stride %lld", (long long)r->pos_batch);
    if (std::llabs(r->start) > ((int64_t)1 << 40)) return fail(BC_ERR_INVALID_ARG, "start %lld", (long long)r->start);
    for (int j = 0; j < rot / 2; ++j) {
        if (!(std::fabs(r->freqs[j]) <= 1e6)) return fail(BC_ERR_INVALID_ARG, "frequency %d is %g", j, r->freqs[j]);
        a.turns[j] = r->freqs[j] / (2.0 * M_PI);
    }
    const bool keys = r->Hk > 0;
    if (r->B == 0 || r->T == 0) return BC_OK;
    const RopeView in[2] = {{r->q, r->q_batch, r->q_row, r->Hq}, {keys ? r->k : nullptr, r->k_batch, r->k_row, r->Hk}};
    const RopeView out[2] = {{r->q_out, r->q_out_batch, r->q_out_row, r->Hq}, {keys ? r->k_out : nullptr, r->k_out_batch, r->k_out_row, r->Hk}};
    const int e = dtype_size(r->dtype);
    for (int x = 0; x < 1 + keys; ++x) {
        if (!in[x].p || !out[x].p) return fail(BC_ERR_INVALID_ARG, "%s is NULL", x ? "k or k_out" : "q or q_out");
        if ((reinterpret_cast<uintptr_t>(in[x].p) | reinterpret_cast<uintptr_t>(out[x].p)) % e) return fail(BC_ERR_INVALID_ARG, "rows must be aligned to their elements");
        for (const RopeView* v : {&in[x], &out[x]})
            if (!strides_fit(r->B, v->batch, r->T, v->row) || v->batch > ((int64_t)1 << 48) || v->row > ((int64_t)1 << 32)) return fail(BC_ERR_INVALID_ARG, "strides %lld, %lld", (long long)v->batch, (long long)v->row);
        if ((r->T > 1 && out[x].row < (int64_t)out[x].H * r->d) || (r->B > 1 && out[x].batch < (r->T - 1) * out[x].row + (int64_t)out[x].H * r->d))
            return fail(BC_ERR_INVALID_ARG, "an output's rows overlap");
    }
    for (int x = 0; x < 1 + keys; ++x)
        for (int y = 0; y < 1 + keys; ++y) {
            const bool same = x == y && in[x].p == out[x].p && (r->T == 1 || in[x].row == out[x].row) && (r->B == 1 || in[x].batch == out[x].batch);
            if ((!same && views_meet(in[x], out[y], r->B, r->T, r->d, e)) || (x < y && views_meet(out[x], out[y], r->B, r->T, r->d, e)))
                return fail(BC_ERR_INVALID_ARG, "an output lies on another operand (in place: the same rows)");
        }
    const int64_t pos_n = r->pos ? ((r->B - 1) * r->pos_batch + (int64_t)r->T * r->axes) * 4 : 0;
    for (int x = 0; x < 1 + keys; ++x)
        if (overlap(out[x].p, ((r->B - 1) * out[x].batch + (r->T - 1) * out[x].row + (int64_t)out[x].H * r->d) * e, r->pos, pos_n))
            return fail(BC_ERR_INVALID_ARG, "an output lies on the positions");
    // Items as large as every row and every piece of a head is a multiple of, up to 16 bytes; neighbours paired: those or one pair
    // (4 x 4000 tokens of 20 + 10 heads of 96 in bf16, halves of 12: 118 us by single columns, 44 by four; of 18 by two 62; pairs 36,
    // of heads of 100 75, of 66 51).
    auto fits = [&](int vec) {
        for (const RopeView* v : {&in[0], &in[1], &out[0], &out[1]})
            if (v->p && (reinterpret_cast<uintptr_t>(v->p) % (vec * e) || (r->B > 1 && v->batch % vec) || (r->T > 1 && v->row % vec))) return false;
        if (r->layout == BC_ROPE_HALVES)
            for (int x = 0; x < r->axes; ++x)
                if (r->axis_dim[x] / 2 % vec) return false;
        return r->d % vec == 0;
    };
    int vec = 16 / e;
    while (vec > 1 && !fits(vec)) vec = r->layout == BC_ROPE_HALVES ? vec / 2 : 1;
    int n = 0, col = 0;
    const bool pairs = r->layout == BC_ROPE_PAIRS && vec > 1;
    if (pairs) {
        n = r->d / vec;      // (their place is their number)
    } else {
        for (int x = 0; x < r->axes; ++x) {
            const int half = r->axis_dim[x] / 2;
            for (int j = 0; j < half; j += vec)
                a.item[n++] = r->layout == BC_ROPE_PAIRS ? RopeArgs::Item{(int16_t)(col + 2 * j), 1, (int16_t)(col / 2 + j), 0}
                                                         : RopeArgs::Item{(int16_t)(col + j), (int16_t)half, (int16_t)(col / 2 + j), 0};
            col += 2 * half;
        }
        for (; col < r->d; col += vec) a.item[n++] = {(int16_t)col, 0, 0, 0};
    }
    a.q = r->q; a.k = r->k; a.qo = r->q_out; a.ko = r->k_out;
    a.q_batch = r->q_batch; a.q_row = r->q_row; a.k_batch = r->k_batch; a.k_row = r->k_row;
    a.qo_batch = r->q_out_batch; a.qo_row = r->q_out_row; a.ko_batch = r->k_out_batch; a.ko_row = r->k_out_row;
    a.B = r->B; a.T = r->T; a.Hq = r->Hq; a.Hk = r->Hk; a.d = r->d;
    a.pairs = rot / 2; a.axes = r->axes; a.items = n;
    a.pos = r->pos; a.pos_batch = r->pos_batch; a.start = r->start;
    a.amplitude = r->amplitude; a.inverse = r->inverse != 0;
    const int64_t per = (int64_t)(r->Hq + r->Hk) * n, all = (int64_t)r->B * r->T;
    // Twelve items a thread, fewer where that leaves CUs idle (14 310 tokens of 24 + 24 heads of 128 in a projection's rows, again
    // and again: 58 us, 65 with six).
    a.tokens = (int)std::max<int64_t>(1, std::min<int64_t>({3072 / per, 16, all / 512}));
    a.by_token = per == 1 ? 0u : (uint32_t)((((uint64_t)1 << 32) + per - 1) / per);
    a.by_items = n == 1 ? 0u : (uint32_t)((((uint64_t)1 << 32) + n - 1) / n);
    const int64_t wgs = (all + a.tokens - 1) / a.tokens;
    if (wgs > kMaxGrid) return fail(BC_ERR_UNSUPPORTED, "rope grid too large");
    hipStream_t s = static_cast<hipStream_t>(stream);
    const dim3 g((unsigned)wgs), block(256);
    const size_t lds = (size_t)a.tokens * a.pairs * sizeof(float2);
#define BC_ROPE(T, V)                                                          \
    case V:                                                                    \
        rope_kernel<T, V, false><<<g, block, lds, s>>>(a);                     \
        break;
    if (pairs) {
        if (r->dtype == BC_BF16) rope_kernel<bf16_tag, 8, true><<<g, block, lds, s>>>(a);
        else rope_kernel<float, 4, true><<<g, block, lds, s>>>(a);
    } else if (r->dtype == BC_BF16) {
        switch (vec) { BC_ROPE(bf16_tag, 8) BC_ROPE(bf16_tag, 4) BC_ROPE(bf16_tag, 2) BC_ROPE(bf16_tag, 1) }
    } else {
        switch (vec) { BC_ROPE(float, 4) BC_ROPE(float, 2) BC_ROPE(float, 1) }
    }
#undef BC_ROPE
    return check_launch("rope");
}

}  // extern "C"
