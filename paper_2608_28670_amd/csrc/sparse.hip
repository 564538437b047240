// Attention over selected key blocks: the score that selects them, and the
// entry points (the attention itself is attention.hip's, over a list of tiles).
//
// For every sample and head, block i of 128 queries scores block j of 64 keys
// by the product of their means, mean(q_i) . mean(k_j), and keeps the `keep`
// best.  Means and products are held in 64 bits: which of two nearly equal
// blocks is taken then hangs on the values and not on a rounding (sums of at
// most 128 bf16 values are exact), and the arithmetic is 0.1 % of what the
// attention over the blocks takes.
#include <cmath>

#include "attention.h"

namespace bc {

struct SelectArgs {
    const void *q, *k;
    const int* lens;
    int B, H, Tq, Tk, d, keep, keep_last;
    int nqb, nkb;
    double *qm, *km;        // means: [B][query blocks][H d], [B][key blocks][H d]
    int* blocks;
};

__device__ __forceinline__ int select_keys(const SelectArgs& a, int b) {
    return a.lens ? min(max(a.lens[b], 0), a.Tk) : a.Tk;
}

// Means of the blocks.  A workgroup takes 32 chunks of 8 columns of one block's
// rows, eight threads per chunk each an eighth of the rows (16 bytes a load,
// 512 consecutive bytes per row), which meet in LDS in a fixed order.  Rows
// past the end are not read; a block without rows has zero means.
template <typename T_>
__global__ __launch_bounds__(256) void block_mean_kernel(SelectArgs a) {
    typedef elem_t<T_> T;
    __shared__ double red[8][32][9];
    const int tid = threadIdx.x, ch = tid & 31, part = tid >> 5;
    const int chunks = a.H * a.d / 8, per = (chunks + 31) / 32;
    const int piece = blockIdx.x % per;
    int64_t blk = blockIdx.x / per;                     // sample-major; a sample's query blocks, then its key blocks
    const int b = (int)(blk / (a.nqb + a.nkb));
    int i = (int)(blk % (a.nqb + a.nkb));
    const bool keys = i >= a.nqb;
    if (keys) i -= a.nqb;
    const int rows = keys ? kSparseK : kSparseQ, T_all = keys ? a.Tk : a.Tq;
    const int n = min(rows, (keys ? select_keys(a, b) : a.Tq) - i * rows);
    const int c = piece * 32 + ch;
    const int64_t ld_row = (int64_t)a.H * a.d;
    double sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (c < chunks) {
        const T* p = static_cast<const T*>(keys ? a.k : a.q) + ((int64_t)b * T_all + (int64_t)i * rows) * ld_row + c * 8;
#pragma unroll 8
        for (int r = part; r < n; r += 8) {
            float v[8];
            if constexpr (sizeof(T) == 2) {
                unpack(*reinterpret_cast<const u32x4*>(p + r * ld_row), v, (const bf16*)nullptr);
            } else {
                unpack(*reinterpret_cast<const u32x4*>(p + r * ld_row), v, (const float*)nullptr);
                unpack(*reinterpret_cast<const u32x4*>(p + r * ld_row + 4), v + 4, (const float*)nullptr);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += (double)v[e];
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) red[part][ch][e] = sum[e];
    __syncthreads();
    const int oc = tid >> 3, e = tid & 7;
    if (piece * 32 + oc >= chunks) return;
    double t = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) t += red[w][oc][e];
    double* out = (keys ? a.km + ((int64_t)b * a.nkb + i) * ld_row : a.qm + ((int64_t)b * a.nqb + i) * ld_row);
    out[piece * 256 + tid] = n > 0 ? t / (double)n : 0.0;
}

// The order of scores as unsigned integers: -0 as +0, a NaN below every number;
// 0 is kept for blocks that are not there.
__device__ __forceinline__ uint64_t score_key(double s) {
    if (s != s) return 1;
    const uint64_t u = (uint64_t)__double_as_longlong(s + 0.0);
    return u >> 63 ? ~u : u | ((uint64_t)1 << 63);
}

// Scores of R query blocks per wave against every key block (lane l holds the
// key blocks l, l + 64, ..., NR of them), then the keep-th largest key by
// bisection over its bits, with ballots, and the list in ascending order.
// Key blocks' means pass through LDS 64 at a time for the four waves; a row of
// D + 2 doubles keeps the 16-byte reads of neighbouring lanes on other banks.
template <int D, int NR, int R>
__global__ __launch_bounds__(256) void score_select_kernel(SelectArgs a) {
    constexpr int LD = D + 2;
    __shared__ __attribute__((aligned(16))) double sk[64 * LD];
    typedef double d2 __attribute__((ext_vector_type(2)));
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int groups = (a.nqb + 4 * R - 1) / (4 * R);
    const int bh = blockIdx.x / groups, b = bh / a.H, h = bh % a.H;
    const int i0 = (blockIdx.x % groups) * 4 * R + wave * R;
    const int64_t ld_row = (int64_t)a.H * D;
    const int valid = (select_keys(a, b) + kSparseK - 1) / kSparseK;      // key blocks that there are
    const double* km = a.km + (int64_t)b * a.nkb * ld_row + h * D;
    const double* qm[R];
#pragma unroll
    for (int r = 0; r < R; ++r) qm[r] = a.qm + ((int64_t)b * a.nqb + min(i0 + r, a.nqb - 1)) * ld_row + h * D;
    uint64_t key[R][NR];
#pragma unroll
    for (int t = 0; t < NR; ++t) {
        if (64 * t < valid) {
            __syncthreads();
            for (int x = tid; x < 64 * (D / 2); x += 256) {
                const int row = x / (D / 2), col = 2 * (x % (D / 2));
                const int j = min(64 * t + row, valid - 1);
                *reinterpret_cast<d2*>(&sk[row * LD + col]) = *reinterpret_cast<const d2*>(km + j * ld_row + col);
            }
            __syncthreads();
            double acc[R];
#pragma unroll
            for (int r = 0; r < R; ++r) acc[r] = 0.0;
#pragma unroll 4
            for (int c = 0; c < D; c += 2) {
                const d2 kv = *reinterpret_cast<const d2*>(&sk[lane * LD + c]);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    acc[r] = fma(qm[r][c], kv[0], acc[r]);
                    acc[r] = fma(qm[r][c + 1], kv[1], acc[r]);
                }
            }
            const int j = 64 * t + lane;
#pragma unroll
            for (int r = 0; r < R; ++r)
                key[r][t] = j >= valid ? 0 : j >= valid - a.keep_last ? ~(uint64_t)0 : score_key(acc[r]);
        } else {
#pragma unroll
            for (int r = 0; r < R; ++r) key[r][t] = 0;
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (i0 + r >= a.nqb) break;
        int* out = a.blocks + ((int64_t)bh * a.nqb + i0 + r) * a.keep;
        auto count_from = [&](uint64_t least) __attribute__((always_inline)) {
            int n = 0;
#pragma unroll
            for (int t = 0; t < NR; ++t) n += __popcll(__ballot(key[r][t] >= least));
            return n;
        };
        // The largest T with at least `keep` keys >= T (1, every block there is, if there are fewer).
        uint64_t T = 1;
        if (valid > a.keep) {
            T = 0;
            for (int bit = 63; bit >= 0; --bit) {
                const uint64_t cand = T | ((uint64_t)1 << bit);
                const int n = count_from(cand);
                if (n >= a.keep) T = cand;
                if (n == a.keep) break;
            }
        }
        const int above = T == ~(uint64_t)0 ? 0 : count_from(T + 1);
        const uint64_t before = ((uint64_t)1 << lane) - 1;
        int ties = min(a.keep, valid) - above, at = 0, tied = 0;      // keys equal to T that are still wanted
#pragma unroll
        for (int t = 0; t < NR; ++t) {
            const uint64_t eq = __ballot(key[r][t] == T);
            const bool sel = key[r][t] > T || (key[r][t] == T && tied + __popcll(eq & before) < ties);
            const uint64_t sm = __ballot(sel);
            if (sel) out[at + __popcll(sm & before)] = 64 * t + lane;
            at += __popcll(sm);
            tied += __popcll(eq);
        }
        for (int x = at + lane; x < a.keep; x += 64) out[x] = -1;
    }
}

template <int D>
static void run_score_select(const SelectArgs& a, hipStream_t s) {
    const int nr = (a.nkb + 63) / 64;
    auto go = [&](auto kernel, int rows) {
        const int64_t wgs = (int64_t)a.B * a.H * ((a.nqb + rows - 1) / rows);
        launch_k(kernel, dim3((unsigned)wgs), dim3(256), s, a);
    };
    if (nr <= 2) go(score_select_kernel<D, 2, 4>, 16);
    else if (nr <= 4) go(score_select_kernel<D, 4, 4>, 16);
    else if (nr <= 16) go(score_select_kernel<D, 16, 2>, 8);
    else go(score_select_kernel<D, 64, 1>, 4);
}

static size_t select_ws(int B, int H, int Tq, int Tk, int d) {
    const size_t blocks = (size_t)((Tq + kSparseQ - 1) / kSparseQ) + (size_t)((Tk + kSparseK - 1) / kSparseK);
    return (size_t)B * H * d * blocks * sizeof(double);
}

// Shape checks that both calls share.
static int check_shape(int B, int H, int Tq, int Tk, int d, int keep, int dtype) {
    if (B < 1 || H < 1 || Tq < 1 || Tk < 1 || d < 1 || keep < 1) return fail(BC_ERR_INVALID_ARG, "empty attention");
    if (dtype != BC_F32 && dtype != BC_BF16) return fail(BC_ERR_INVALID_ARG, "dtype %d", dtype);
    if (!attention_supported(d) || (dtype == BC_F32 && d > 64))
        return fail(BC_ERR_UNSUPPORTED, "head_dim %d (supported: 32, 64, 72, 128; fp32: 32, 64)", d);
    if (Tk > kSparseMaxBlocks * kSparseK)
        return fail(BC_ERR_UNSUPPORTED, "%d keys: at most %d", Tk, kSparseMaxBlocks * kSparseK);
    if (Tq > (1 << 30) || (int64_t)B * H > (1 << 24) || (int64_t)H * d > (1 << 24) || keep > kSparseMaxBlocks)
        return fail(BC_ERR_UNSUPPORTED, "attention over blocks: %d x %d x %d, keep %d", B, H, Tq, keep);
    return BC_OK;
}

static bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

}  // namespace bc

using namespace bc;

extern "C" {

int bc_attention_select_workspace_size(int B, int H, int Tq, int Tk, int d, int keep, int dtype, size_t* bytes) {
    clear_error();
    if (!bytes) return fail(BC_ERR_INVALID_ARG, "NULL pointer");
    const int rc = check_shape(B, H, Tq, Tk, d, keep, dtype);
    if (rc != BC_OK) return rc;
    *bytes = select_ws(B, H, Tq, Tk, d);
    return BC_OK;
}

int bc_attention_select(int B, int H, int Tq, int Tk, int d, const void* q, const void* k, const int32_t* lens, int keep,
                        int keep_last, int32_t* blocks, int dtype, void* ws, size_t ws_bytes, void* stream) {
    clear_error();
    if (!q || !k || !blocks || !ws) return fail(BC_ERR_INVALID_ARG, "NULL pointer");
    int rc = check_shape(B, H, Tq, Tk, d, keep, dtype);
    if (rc != BC_OK) return rc;
    if (keep_last < 0 || keep_last > keep) return fail(BC_ERR_INVALID_ARG, "keep_last=%d outside [0, keep=%d]", keep_last, keep);
    if (!aligned16(q) || !aligned16(k) || reinterpret_cast<uintptr_t>(ws) % 256)
        return fail(BC_ERR_INVALID_ARG, "q and k must be 16-byte, the workspace 256-byte aligned");
    if (ws_bytes < select_ws(B, H, Tq, Tk, d))
        return fail(BC_ERR_INVALID_ARG, "workspace %zu < %zu bytes", ws_bytes, select_ws(B, H, Tq, Tk, d));
    SelectArgs a;
    a.q = q; a.k = k; a.lens = lens;
    a.B = B; a.H = H; a.Tq = Tq; a.Tk = Tk; a.d = d; a.keep = keep; a.keep_last = keep_last;
    a.nqb = (Tq + kSparseQ - 1) / kSparseQ;
    a.nkb = (Tk + kSparseK - 1) / kSparseK;
    a.qm = static_cast<double*>(ws);
    a.km = a.qm + (int64_t)B * a.nqb * H * d;
    a.blocks = blocks;
    const int64_t means = (int64_t)B * (a.nqb + a.nkb) * ((H * d / 8 + 31) / 32), rows = (int64_t)B * H * a.nqb;
    if (means > 0x7fffffff || rows > 0x7fffffff) return fail(BC_ERR_UNSUPPORTED, "block selection grid too large");
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (dtype == BC_BF16) launch_k(block_mean_kernel<bf16_tag>, dim3((unsigned)means), dim3(256), s, a);
    else launch_k(block_mean_kernel<float>, dim3((unsigned)means), dim3(256), s, a);
    rc = check_launch("block means");
    if (rc != BC_OK) return rc;
    switch (d) {
        case 32: run_score_select<32>(a, s); break;
        case 64: run_score_select<64>(a, s); break;
        case 72: run_score_select<72>(a, s); break;
        default: run_score_select<128>(a, s); break;
    }
    return check_launch("block selection");
}

int bc_attention_sparse_workspace_size(int B, int H, int Tq, int Tk, int d, int keep, int dtype, size_t* bytes) {
    clear_error();
    if (!bytes) return fail(BC_ERR_INVALID_ARG, "NULL pointer");
    const int rc = check_shape(B, H, Tq, Tk, d, keep, dtype);
    if (rc != BC_OK) return rc;
    *bytes = 0;
    return BC_OK;
}

int bc_attention_sparse(int B, int H, int Tq, int Tk, int d, const void* q, const void* k, const void* v,
                        const int32_t* lens, const int32_t* blocks, int keep, void* out, int prescaled, int dtype, void* ws,
                        size_t ws_bytes, void* stream) {
    clear_error();
    (void)ws; (void)ws_bytes;
    if (!q || !k || !v || !blocks || !out) return fail(BC_ERR_INVALID_ARG, "NULL pointer");
    const int rc = check_shape(B, H, Tq, Tk, d, keep, dtype);
    if (rc != BC_OK) return rc;
    if (prescaled && dtype != BC_BF16) return fail(BC_ERR_UNSUPPORTED, "pre-scaled queries are bf16 only");
    if (!aligned16(q) || !aligned16(k) || !aligned16(v)) return fail(BC_ERR_INVALID_ARG, "q, k and v must be 16-byte aligned");
    AttnArgs a = {};
    a.q_scaled = prescaled ? 1 : 0;
    a.q0 = a.q1 = q; a.Tq0 = Tq; a.ldq = (int64_t)H * d;
    a.k0 = a.k1 = k; a.Tk0 = Tk; a.ldk = (int64_t)H * d;
    a.v0 = a.v1 = v; a.ldv = (int64_t)H * d;
    a.o0 = a.o1 = out; a.ldo = (int64_t)H * d;
    a.B = B; a.H = H; a.d = d;
    a.blocks = blocks; a.keep = keep; a.lens = lens;
    return launch_sparse_attention(dtype, a, static_cast<hipStream_t>(stream));
}

}  // extern "C"
