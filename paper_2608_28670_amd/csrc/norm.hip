// A module's way back into the residual stream in one pass over the rows:
//   z  = P(y)                                the norm after the module
//   x' = a x + gate (.) z                    residual scale, per-sample gate
//   h  = N(x') (1 + scale) + shift           the norm before the next module
// P and N: none, RMSNorm or LayerNorm, with learned weights; statistics fp32,
// two-pass (mean, then squared deviations) from registers.
//
// What bounds it is memory: y and x are read once, x' and h written once, 12
// bytes a value in bf16.  A row lives in the registers of one wave (or, above
// 4096 values and where rows are few, of a workgroup's four), so the statistics of x' need no second read.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "ops.h"

namespace bc {

// Four values of a row, as stored; NT: past the caches.  ANY: at any alignment of
// the elements (the hardware takes it; `any` is the type's form that says so).
template <typename T> struct Raw4 {
    typedef f32x4 v;
    typedef f32x4 any __attribute__((aligned(4)));
};
template <> struct Raw4<bf16> {
    typedef bf16x4 v;
    typedef bf16x4 any __attribute__((aligned(2)));
};
template <bool NT, bool ANY, typename T> __device__ __forceinline__ typename Raw4<T>::v load_row4(const T* p) {
    if constexpr (ANY) return *reinterpret_cast<const typename Raw4<T>::any*>(p);
    const typename Raw4<T>::v* q = reinterpret_cast<const typename Raw4<T>::v*>(p);
    return NT ? __builtin_nontemporal_load(q) : *q;
}
template <bool NT, bool ANY, typename T> __device__ __forceinline__ void store_row4(T* p, const typename Raw4<T>::v& v) {
    typedef std::conditional_t<ANY, typename Raw4<T>::any, typename Raw4<T>::v> v4;
    if constexpr (NT) __builtin_nontemporal_store((v4)v, reinterpret_cast<v4*>(p));
    else *reinterpret_cast<v4*>(p) = v;
}

// V values (4, or 1 without alignment) from p to fp32 and back.
template <int V, typename T> __device__ __forceinline__ void load_v(const T* p, float* v) {
    if constexpr (V == 4) {
        const auto r = load_row4<false, false>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (float)r[e];
    } else {
        v[0] = (float)*p;
    }
}
template <int V, typename T> __device__ __forceinline__ void store_v(T* p, const float* v) {
    if constexpr (V == 4) store_row4<false, false>(p, typename Raw4<T>::v{(T)v[0], (T)v[1], (T)v[2], (T)v[3]});
    else *p = (T)v[0];
}

// W waves per row, lane l of them holding chunks l, l + 64 W, ... of V values.
template <typename T_, int W, int NC, int V>
__global__ __launch_bounds__(256) void norm_residual_kernel(NormArgs a) {
    typedef elem_t<T_> T;
    constexpr int L = 64 * W;
    __shared__ float part[2][4];
    const int tid = threadIdx.x, lane = tid % L;
    const int64_t row = (int64_t)blockIdx.x * (4 / W) + tid / L;
    if (row >= a.rows) return;                      // W == 4: the whole workgroup or none
    const int D = a.D;
    const float width = (float)D;
    int turn = 0;
    auto row_sum = [&](float v) __attribute__((always_inline)) {
        v = wave_sum(v);
        if constexpr (W > 1) {
            // The two halves of `part` take turns: a wave that writes the next sum
            // has passed the barrier behind which the sum before last was read.
            if ((tid & 63) == 0) part[turn][tid >> 6] = v;
            __syncthreads();
            v = (part[turn][0] + part[turn][1]) + (part[turn][2] + part[turn][3]);
            turn ^= 1;
        }
        return v;
    };
    auto each = [&](auto&& f) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const int c = (lane + L * j) * V;
            if (c < D) f(j, c);
        }
    };
    // Norm of the row held in r (chunks past D hold zeros), weight and bias applied.
    auto norm = [&](int kind, const void* wp, const void* bp, float (&r)[NC][V]) __attribute__((always_inline)) {
        float mean = 0.f;
        if (kind == BC_NORM_LAYER) {
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                if constexpr (V == 4) sum += (r[j][0] + r[j][1]) + (r[j][2] + r[j][3]);
                else sum += r[j][0];
            }
            mean = row_sum(sum) / width;
        }
        if (kind != BC_NORM_NONE) {
            float sq = 0.f;
            each([&](int j, int) {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float d = r[j][e] - mean;
                    sq += d * d;
                }
            });
            const float rstd = 1.0f / sqrtf(row_sum(sq) / width + a.eps);
#pragma unroll
            for (int j = 0; j < NC; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) r[j][e] = (r[j][e] - mean) * rstd;
        }
        if (wp) {
            each([&](int j, int c) {
                float w[V], b[V];
                load_v<V>(static_cast<const T*>(wp) + c, w);
#pragma unroll
                for (int e = 0; e < V; ++e) b[e] = 0.f;
                if (bp) load_v<V>(static_cast<const T*>(bp) + c, b);
#pragma unroll
                for (int e = 0; e < V; ++e) r[j][e] = fmaf(r[j][e], w[e], b[e]);
            });
        }
    };

    const int64_t s = row / a.rows_per_sample;
    float z[NC][V], x[NC][V];
#pragma unroll
    for (int j = 0; j < NC; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) z[j][e] = x[j][e] = 0.f;
    each([&](int j, int c) {
        load_v<V>(static_cast<const T*>(a.y) + row * a.ldy + c, z[j]);
        load_v<V>(a.x + row * a.ldx + c, x[j]);
    });
    norm(a.post, a.post_w, a.post_b, z);
    each([&](int j, int c) {
        float g[V];
#pragma unroll
        for (int e = 0; e < V; ++e) g[e] = 1.f;
        if (a.gate) load_v<V>(a.gate + s * a.ld_gate + c, g);
#pragma unroll
        for (int e = 0; e < V; ++e) x[j][e] = fmaf(g[e], z[j][e], a.res_scale * x[j][e]);
        store_v<V>(a.x_out + row * a.ldx + c, x[j]);
    });
    if (!a.h) return;
    norm(a.pre, a.pre_w, a.pre_b, x);
    each([&](int j, int c) {
        if (a.scale) {
            float sh[V], sc[V];
            load_v<V>(a.shift + s * a.ld_mod + c, sh);
            load_v<V>(a.scale + s * a.ld_mod + c, sc);
#pragma unroll
            for (int e = 0; e < V; ++e) x[j][e] = x[j][e] * (1.0f + sc[e]) + sh[e];
        }
        store_v<V>(static_cast<T*>(a.h) + row * a.ldh + c, x[j]);
    });
}

// The same for many rows of a sample: a workgroup takes a row per wave, with the
// vectors that the rows share in LDS (gate, 1 + scale and shift in fp32, the learned
// ones as stored, an absent one as ones or zeros).  Read by every row from L2 instead,
// 16 bytes a value with weights beside the 12 of the rows themselves, they bound the
// launch.  Sums and roundings are those of the kernel above, in its order for a row
// per wave.
//   The vectors are not folded into gate weight, gate bias and so on: an infinite gate
// times an absent bias's 0 is NaN where the formula gives infinity, and a gate times
// a weight may leave fp32's range where gate (n weight) does not.  Folded, four fp32
// vectors instead of 28 (bf16: 20) bytes a column, was about as fast: bf16 16 384 x
// 1152 44 us and 42 so, 14 566 x 3072 100 and 101, 2400 x 2000 13.7 and 13.9, 21 759 x
// 642 40 and 41, 18 000 x 2901 140 and 136; fp32 with weights 8000 x 2944 69 either way,
// 2400 x 4000 37.6 and 39.6, 8192 x 640 18.4 and 20.8.  LEARNED false keeps calls without
// weights free of theirs: 4096 x 1152 11.9 -> 11.4.
//   14 566 x 3072, RMS norms on both sides (537 MB): 173 us by the kernel above, 101 so
// (5.3 TB/s).  Several rows per wave in turn are slower (16 384 x 1152 50 against 45).
// x_out is stored non-temporally, and in launches that stream past the caches (BIG) y
// and x are loaded so, above 1280 values by twice the waves: 119 -> 105 us (rows up to
// 1280 are faster without; 4096 values would spill); 4096 x 1152, whose rows the caches
// hold, 11.6 us as it is, 12.2 as BIG.  The rows' loads go out before the vectors are
// in LDS: 105 -> 100 us; in fp32 BIG launches, whose rows take twice the registers,
// not: 8000 x 2944 68 as it is, 70.5 so.
//   ANY (rows or vectors without 4-value alignment, such as odd widths): the same
// chunks with loads and stores at element alignment, the last 1 to 3 values one to
// a lane: 13 252 x 1367 bf16 52 us where four waves a row with a value a load took
// 115, 4000 x 777 13.6 and 21.3.  x_out is stored non-temporally here too, a gain in
// bf16 (21 759 x 642 47.9 -> 40.0 us) and a small loss in fp32 (8000 x 1999 57 -> 59);
// non-temporal loads by twice the waves lose it again.
constexpr int row_waves(bool big, int nc) { return big && nc > 5 && nc <= 12 ? 16 : 8; }
template <typename T_, int NC, bool BIG, bool ANY, bool LEARNED>
__global__ __launch_bounds__(64 * row_waves(BIG, NC)) void norm_residual_rows_kernel(NormArgs a) {
    typedef elem_t<T_> T;
    constexpr int WAVES = row_waves(BIG, NC);
    __shared__ f32x4 sv[3][64 * NC];                    // gate, 1 + scale, shift
    __shared__ typename Raw4<T>::v lv[LEARNED ? 4 : 1][LEARNED ? 64 * NC : 1];      // weight and bias of P, of N
    const int tid = threadIdx.x, lane = tid & 63;
    // Workgroups of a sample.  (The grid is made for min(rows, rows_per_sample).)
    const int per = (int)((min((int64_t)a.rows_per_sample, a.rows) + WAVES - 1) / WAVES);
    const int64_t s = blockIdx.x / per;
    const int64_t row = s * a.rows_per_sample + (int64_t)(blockIdx.x % per) * WAVES + (tid >> 6);
    const bool there = row < min((s + 1) * a.rows_per_sample, a.rows);
    const int nch = a.D >> 2;
    const int rest = ANY ? a.D & 3 : 0;      // values behind the last chunk: lane l < rest has value 4 nch + l
    // Chunk c of a vector that the rows share, `none` where there is no vector.
    auto vec4 = [&](const auto* p, int c, float none) __attribute__((always_inline)) {
        typedef std::remove_cv_t<std::remove_reference_t<decltype(*p)>> E;
        typename Raw4<E>::v v = {(E)none, (E)none, (E)none, (E)none};
        if (p && ANY && c == nch) {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (e < rest) v[e] = p[4 * c + e];
        } else if (p) {
            v = load_row4<false, ANY>(p + 4 * c);
        }
        return v;
    };
    typename Raw4<T>::v z[NC];      // as stored: a bf16 row takes half the registers
    f32x4 x[NC];
    float zt = 0.f, xt = 0.f;
    const int64_t last = 4 * nch + lane;
    auto take_row = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const int c = lane + 64 * j;
            if (there && c < nch) {
                z[j] = load_row4<BIG, ANY>(static_cast<const T*>(a.y) + row * a.ldy + 4 * c);
                x[j] = load_row4<BIG, ANY>(a.x + row * a.ldx + 4 * c);
            } else {
                z[j] = typename Raw4<T>::v{};
                x[j] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
        }
        if (ANY && there && lane < rest) {
            zt = (float)static_cast<const T*>(a.y)[row * a.ldy + last];
            xt = a.x[row * a.ldx + last];
        }
    };
    constexpr bool EARLY = !(BIG && sizeof(T) == 4);
    if constexpr (EARLY) take_row();
    const float* gate = a.gate ? a.gate + s * a.ld_gate : nullptr;
    const float *shift = a.scale ? a.shift + s * a.ld_mod : nullptr, *scale = a.scale ? a.scale + s * a.ld_mod : nullptr;
    for (int c = tid; c < nch + (rest > 0); c += 64 * WAVES) {
        const f32x4 g = vec4(gate, c, 1.f), sc = vec4(scale, c, 0.f), sh = vec4(shift, c, 0.f);
        if constexpr (LEARNED) {
            const auto w = vec4(static_cast<const T*>(a.post_w), c, 1.f), b = vec4(static_cast<const T*>(a.post_b), c, 0.f);
            const auto pw = vec4(static_cast<const T*>(a.pre_w), c, 1.f), pb = vec4(static_cast<const T*>(a.pre_b), c, 0.f);
            lv[0][c] = w;
            lv[1][c] = b;
            lv[2][c] = pw;
            lv[3][c] = pb;
        }
        sv[0][c] = g;
        sv[1][c] = 1.0f + sc;
        sv[2][c] = sh;
    }
    __syncthreads();
    const float width = (float)a.D;
    // (mean, 1 / std) of the row whose chunk j is r[j], chunks past D zero, and whose rest is t.
    auto stats = [&](int kind, const auto& r, float t, float& mean, float& rstd) __attribute__((always_inline)) {
        mean = 0.f;
        rstd = 1.f;
        if (kind == BC_NORM_LAYER) {
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < NC; ++j) sum += ((float)r[j][0] + (float)r[j][1]) + ((float)r[j][2] + (float)r[j][3]);
            if constexpr (ANY) sum += t;
            mean = wave_sum(sum) / width;
        }
        if (kind != BC_NORM_NONE) {
            float sq = 0.f;
#pragma unroll
            for (int j = 0; j < NC; ++j)
                if (lane + 64 * j < nch) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float d = (float)r[j][e] - mean;
                        sq += d * d;
                    }
                }
            if (ANY && lane < rest) sq += (t - mean) * (t - mean);
            rstd = 1.0f / sqrtf(wave_sum(sq) / width + a.eps);
        }
    };
    if (!there) return;
    if constexpr (!EARLY) take_row();
    float mean, rstd;
    // Chunk c, or the rest, normed: of P (v = 0) or N (v = 2).
    auto normed = [&](const auto& r, int c, int v, float* n) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 4; ++e) n[e] = ((float)r[e] - mean) * rstd;
        if constexpr (LEARNED) {
            const auto w = lv[v][c], b = lv[v + 1][c];
#pragma unroll
            for (int e = 0; e < 4; ++e) n[e] = fmaf(n[e], (float)w[e], (float)b[e]);
        }
    };
    auto normed_rest = [&](float t, int v) __attribute__((always_inline)) {
        const float n = (t - mean) * rstd;
        if constexpr (LEARNED) return fmaf(n, (float)lv[v][nch][lane], (float)lv[v + 1][nch][lane]);
        return n;
    };
    stats(a.post, z, zt, mean, rstd);
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        const int c = lane + 64 * j;
        if (c < nch) {
            const f32x4 g = sv[0][c];
            float n[4];
            normed(z[j], c, 0, n);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[j][e] = fmaf(g[e], n[e], a.res_scale * x[j][e]);
            store_row4<true, ANY>(a.x_out + row * a.ldx + 4 * c, x[j]);
        }
    }
    if (ANY && lane < rest) {
        xt = fmaf(sv[0][nch][lane], normed_rest(zt, 0), a.res_scale * xt);
        a.x_out[row * a.ldx + last] = xt;
    }
    if (!a.h) return;
    stats(a.pre, x, xt, mean, rstd);
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        const int c = lane + 64 * j;
        if (c < nch) {
            const f32x4 sc = sv[1][c], sh = sv[2][c];
            float n[4];
            normed(x[j], c, 2, n);
            typename Raw4<T>::v o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = (T)fmaf(n[e], sc[e], sh[e]);
            store_row4<false, ANY>(static_cast<T*>(a.h) + row * a.ldh + 4 * c, o);
        }
    }
    if (ANY && lane < rest)
        static_cast<T*>(a.h)[row * a.ldh + last] = (T)fmaf(normed_rest(xt, 2), sv[1][nch][lane], sv[2][nch][lane]);
}

template <typename T, bool BIG, bool ANY>
static int run_norm_rows(const NormArgs& a, int nc, hipStream_t s) {
    const int64_t samples = (a.rows + a.rows_per_sample - 1) / a.rows_per_sample;
    const int waves = row_waves(BIG, nc);
    const int per = (int)std::min<int64_t>(a.rows_per_sample, a.rows);
    const dim3 g((unsigned)(samples * ((per + waves - 1) / waves))), b(64 * waves);
#define BC_NR(NC) (a.post_w || a.pre_w ? launch_k(norm_residual_rows_kernel<tag_t<T>, NC, BIG, ANY, true>, g, b, s, a) \
                                       : launch_k(norm_residual_rows_kernel<tag_t<T>, NC, BIG, ANY, false>, g, b, s, a))
    if (nc <= 1) BC_NR(1);
    else if (nc <= 2) BC_NR(2);
    else if (nc <= 5) BC_NR(5);
    else if (nc <= 8) BC_NR(8);
    else if (nc <= 12) BC_NR(12);
    else BC_NR(16);
#undef BC_NR
    return check_launch("norm_residual");
}

template <typename T>
static int run_norm_residual(const NormArgs& a, bool vec, hipStream_t s) {
    const dim3 b(256);
    const dim3 wave_rows((unsigned)((a.rows + 3) / 4)), rows((unsigned)a.rows);
    const int nc = ((a.D + 3) / 4 + 63) / 64;
#define BC_NR(W, NC, V, G) launch_k(norm_residual_kernel<tag_t<T>, W, NC, V>, G, b, s, a)
    // Up to one round of workgroups: a row's four waves, whose loads and sums are
    // shorter chains.  63 rows of 2960 11.1 us by rows of a sample and 6.3 so, 16 of
    // 4096 12.4 and 6.7, one of 1152 4.85 and 4.0; 1024 of 640, 1152, 2560 and 4096 5.5,
    // 7.3, 14.3, 16.1 and 5.0, 7.2, 11.7, 14.5 (in samples of four 5.7, 7.8, 14.2, 16.4
    // and 6.2, 8.9, 13.1, 18.1); 2048 6.4, 8.4, 15.9, 21.4 and 7.6, 11.0, 16.0, 24.
    if (vec && nc <= 16 && a.rows <= 1024 && !a.wave_rows) {
        if (nc <= 4) BC_NR(4, 1, 4, rows);
        else if (nc <= 8) BC_NR(4, 2, 4, rows);
        else BC_NR(4, 4, 4, rows);
        return check_launch("norm_residual");
    }
    // Rows by rows of a sample, except where hardly any share one: 4096 rows of
    // 1152 in samples of 1, 2 and 4 take 33, 25 and 15.0 us so and 23, 18 and 14.7 us
    // below, 8192 x 2048 in fours 49 and 66; few rows 5.0 and 6.1 whatever they share.
    // Without alignment 4096 of 1151 in samples of 1, 2, 4 and 8: 77, 42, 23 and 16 us
    // against 42, 32, 30 and 30; 400 rows in samples of 1 9.2 and 10.4.
    if (nc <= 16 && (a.rows_per_sample >= 4 || a.rows < 512)) {
        if (!vec) return run_norm_rows<T, false, true>(a, nc, s);
        // The caches' reach: 57 MB 11.4 us as a small launch and 12.2 as a big one, 98 MB 44.2 and 39.0.
        const double bytes = (double)a.rows * a.D * (sizeof(T) * (a.h ? 2 : 1) + 8);
        return bytes >= 80e6 && a.rows_per_sample >= 16 ? run_norm_rows<T, true, false>(a, nc, s)
                                                        : run_norm_rows<T, false, false>(a, nc, s);
    }
    if (!vec) {
        if (a.D <= 8 * 256) BC_NR(4, 8, 1, rows);
        else BC_NR(4, 64, 1, rows);
    } else if (nc <= 1) BC_NR(1, 1, 4, wave_rows);
    else if (nc <= 2) BC_NR(1, 2, 4, wave_rows);
    else if (nc <= 5) BC_NR(1, 5, 4, wave_rows);
    else if (nc <= 8) BC_NR(1, 8, 4, wave_rows);
    else if (nc <= 12) BC_NR(1, 12, 4, wave_rows);
    else if (nc <= 16) BC_NR(1, 16, 4, wave_rows);
    else BC_NR(4, 16, 4, rows);
#undef BC_NR
    return check_launch("norm_residual");
}

int launch_norm_residual(int dt, const NormArgs& a, hipStream_t s) {
    if (a.rows <= 0) return BC_OK;
    const uintptr_t el = reinterpret_cast<uintptr_t>(a.y) | reinterpret_cast<uintptr_t>(a.h) |
                         reinterpret_cast<uintptr_t>(a.post_w) | reinterpret_cast<uintptr_t>(a.post_b) |
                         reinterpret_cast<uintptr_t>(a.pre_w) | reinterpret_cast<uintptr_t>(a.pre_b);
    const uintptr_t f4 = reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.x_out) |
                         reinterpret_cast<uintptr_t>(a.gate) | reinterpret_cast<uintptr_t>(a.shift) |
                         reinterpret_cast<uintptr_t>(a.scale);
    const bool vec = (a.D | a.ldy | a.ldx | a.ldh | a.ld_gate | a.ld_mod) % 4 == 0 &&
                     el % (4 * dtype_size(dt)) == 0 && f4 % 16 == 0;
    prof_begin(PROF_LAYERNORM, s, (double)a.rows * a.D * (dtype_size(dt) * (a.h ? 2 : 1) + 8));
    const int rc = dt == BC_BF16 ? run_norm_residual<bf16>(a, vec, s) : run_norm_residual<float>(a, vec, s);
    prof_end(PROF_LAYERNORM, s);
    return rc;
}

}  // namespace bc

using namespace bc;

extern "C" int bc_norm_gate_residual(const bc_norm_desc* dp, void* stream) {
    clear_error();
    if (!dp) return fail(BC_ERR_INVALID_ARG, "NULL pointer");
    const bc_norm_desc& d = *dp;
    if (d.dtype != BC_F32 && d.dtype != BC_BF16) return fail(BC_ERR_INVALID_ARG, "dtype %d", d.dtype);
    if (d.rows < 0 || d.D < 1 || d.rows_per_sample < 1)
        return fail(BC_ERR_INVALID_ARG, "rows %lld, D %d, rows per sample %d", (long long)d.rows, d.D, d.rows_per_sample);
    if (d.D > kMaxNormWidth) return fail(BC_ERR_UNSUPPORTED, "D=%d > %d", d.D, kMaxNormWidth);
    const bool some = d.rows > 0;      // (without rows every row operand may be NULL, as an empty tensor's address is)
    if (some && (!d.y || !d.x || !d.x_out)) return fail(BC_ERR_INVALID_ARG, "NULL pointer");
    for (int i = 0; i < 2; ++i) {
        const int kind = i ? d.pre : d.post;
        const void *w = i ? d.pre_w : d.post_w, *b = i ? d.pre_b : d.post_b;
        if (kind < BC_NORM_NONE || kind > BC_NORM_LAYER) return fail(BC_ERR_INVALID_ARG, "norm kind %d", kind);
        if ((kind == BC_NORM_NONE && w) || (kind != BC_NORM_LAYER && b) || (b && !w))
            return fail(BC_ERR_INVALID_ARG, "a weight needs a norm, a bias a LayerNorm with a weight");
    }
    if (some && !d.scale != !d.shift) return fail(BC_ERR_INVALID_ARG, "shift and scale go together");
    if (some && !d.h && (d.pre != BC_NORM_NONE || d.scale)) return fail(BC_ERR_INVALID_ARG, "a norm before the next module needs h");
    if (!(d.eps > 0.f) || !std::isfinite(d.eps) || !std::isfinite(d.res_scale))
        return fail(BC_ERR_INVALID_ARG, "eps %g, residual scale %g", d.eps, d.res_scale);
    const int64_t most = (int64_t)1 << 36;
    if (d.ldy < d.D || d.ldx < d.D || (d.h && d.ldh < d.D) || (d.gate && d.ld_gate < d.D) || (d.scale && d.ld_mod < d.D) ||
        d.ldy > most || d.ldx > most || d.ldh > most || d.ld_gate > most || d.ld_mod > most)
        return fail(BC_ERR_INVALID_ARG, "a row stride is smaller than D=%d or too large", d.D);
    if (!some) return BC_OK;
    if (d.rows > kMaxGrid) return fail(BC_ERR_UNSUPPORTED, "%lld rows", (long long)d.rows);
    // A row is read whole before any of it is written, so the outputs may lie
    // on their own inputs exactly; other overlaps would race between rows.
    const int64_t esz = dtype_size(d.dtype);
    const int64_t ny = ((d.rows - 1) * d.ldy + d.D) * esz, nh = ((d.rows - 1) * d.ldh + d.D) * esz,
                  nx = ((d.rows - 1) * d.ldx + d.D) * 4;
    if ((d.x_out != d.x && overlap(d.x, nx, d.x_out, nx)) || overlap(d.y, ny, d.x_out, nx) || overlap(d.h, nh, d.x_out, nx) ||
        overlap(d.h, nh, d.x, nx) || (overlap(d.y, ny, d.h, nh) && !(d.y == d.h && d.ldy == d.ldh)))
        return fail(BC_ERR_INVALID_ARG, "x_out may be x and h may be y (same stride); no other overlap");
    const int64_t samples = (d.rows + d.rows_per_sample - 1) / d.rows_per_sample, nd = d.D * esz;
    const struct { const void* p; int64_t bytes, align; } vectors[] = {
        {d.post_w, nd, esz}, {d.post_b, nd, esz}, {d.pre_w, nd, esz}, {d.pre_b, nd, esz}, {d.y, 0, esz}, {d.h, 0, esz},
        {d.x, 0, 4}, {d.x_out, 0, 4}, {d.gate, ((samples - 1) * d.ld_gate + d.D) * 4, 4},
        {d.shift, ((samples - 1) * d.ld_mod + d.D) * 4, 4}, {d.scale, ((samples - 1) * d.ld_mod + d.D) * 4, 4}};
    for (const auto& v : vectors) {
        if (reinterpret_cast<uintptr_t>(v.p) % v.align) return fail(BC_ERR_INVALID_ARG, "a pointer is not aligned to its elements");
        if (v.bytes && (overlap(v.p, v.bytes, d.x_out, nx) || overlap(v.p, v.bytes, d.h, nh)))
            return fail(BC_ERR_INVALID_ARG, "an output overlaps a weight, gate, shift or scale");
    }
    NormArgs a = {};
    a.rows = d.rows; a.D = d.D; a.rows_per_sample = d.rows_per_sample;
    a.y = d.y; a.ldy = d.ldy;
    a.post = d.post; a.post_w = d.post_w; a.post_b = d.post_b;
    a.gate = d.gate; a.ld_gate = d.gate ? d.ld_gate : 0;
    a.res_scale = d.res_scale;
    a.x = d.x; a.x_out = d.x_out; a.ldx = d.ldx;
    a.pre = d.pre; a.pre_w = d.pre_w; a.pre_b = d.pre_b;
    a.shift = d.shift; a.scale = d.scale; a.ld_mod = d.scale ? d.ld_mod : 0;
    a.h = d.h; a.ldh = d.h ? d.ldh : 0;
    a.eps = d.eps;
    return launch_norm_residual(d.dtype, a, static_cast<hipStream_t>(stream));
}
