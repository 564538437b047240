// Attention over tensors with capped scores, distance biases and masks (score.h):
// documents of key tiles, how a call is laid out, the entry point.
#include <algorithm>
#include <cmath>

#include "score_kernels.h"

namespace bc {

// The documents of every tile of 64 keys of a sample (the lowest, complemented if
// some key has none; the highest), keys without a document left aside, then those of
// every 64 queries; a wave a tile.
__global__ __launch_bounds__(256) void document_ranges_kernel(const int* k_docs, const int* q_docs, const int* lens, int B, int Tk, int Tq,
                                                              u32x2* out) {
    const int kt = (Tk + 63) / 64, qt = (Tq + 63) / 64;
    int64_t x = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (x >= (int64_t)B * (kt + qt)) return;
    out += x;
    const bool query = x >= (int64_t)B * kt;
    if (query) x -= (int64_t)B * kt;
    const int tiles = query ? qt : kt, T = query ? Tq : Tk;
    const int b = (int)(x / tiles), lane = threadIdx.x & 63, t = (int)(x % tiles) * 64 + lane;
    const int n = lens && !query ? min(max(lens[b], 0), T) : T;
    const int d = t < n ? (query ? q_docs : k_docs)[(int64_t)b * T + t] : -1;
    int lo = d >= 0 ? d : 0x7fffffff, hi = d >= 0 ? d : -1;
    const bool none = __any(t < n && d < 0);
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        lo = min(lo, __shfl_xor(lo, s));
        hi = max(hi, __shfl_xor(hi, s));
    }
    if (lane == 0) *out = u32x2{(unsigned)(none ? ~lo : lo), (unsigned)hi};
}

// The row tiles of a sample in the order of how many key tiles share a document with
// them, the most first; a workgroup a sample (256 key tiles, 128 of rows: 14.5 us with a thread a row tile).  Where a call makes
// more than one round of workgroups, long documents that start late would end it alone
// (16 heads of 16 384 tokens, 24 documents, d = 72, six draws: 164 to 274 us in the order of the rows, 135 to 192 so).
constexpr int kOrderRows = 1024, kOrderKeys = 4096;
__global__ __launch_bounds__(kOrderRows) void row_order_kernel(const u32x2* ranges, int B, int Tk, int Tq, int G, int rows, int row_tiles, int* order) {
    __shared__ u32x2 keys[kOrderKeys];
    __shared__ u32x2 rows_docs[kOrderRows];
    __shared__ int count[kOrderRows];
    const int b = blockIdx.x, tid = threadIdx.x, kt = (Tk + 63) / 64, qt = (Tq + 63) / 64;
    const u32x2* qr = ranges + (int64_t)B * kt + (int64_t)b * qt;
    for (int x = tid; x < kt; x += kOrderRows) keys[x] = ranges[(int64_t)b * kt + x];
    int lo = 0x7fffffff, hi = -1;
    if (tid < row_tiles)
        for (int t = tid * rows / G / 64; t <= min(((tid + 1) * rows - 1) / G / 64, qt - 1); ++t) {
            const int first = (int)qr[t].x;
            lo = min(lo, first < 0 ? ~first : first);
            hi = max(hi, (int)qr[t].y);
        }
    __syncthreads();
    // `per` threads a row tile count its keys, and then the rows before it, between them.
    int per = 1;
    while (2 * per * row_tiles <= kOrderRows && per < 64) per *= 2;
    const int sub = tid & (per - 1);
    if (tid < row_tiles) rows_docs[tid] = u32x2{(unsigned)lo, (unsigned)hi};
    __syncthreads();
    const int row = min(tid / per, row_tiles - 1);
    lo = (int)rows_docs[row].x;
    hi = (int)rows_docs[row].y;
    int n = 0;
    for (int x = sub; x < kt; x += per) {
        const int first = (int)keys[x].x;
        n += (first < 0 ? ~first : first) <= hi && (int)keys[x].y >= lo;
    }
    for (int s = 1; s < per; s <<= 1) n += __shfl_xor(n, s);
    if (sub == 0) count[row] = n;
    __syncthreads();
    int rank = 0;
    for (int x = sub; x < row_tiles; x += per) rank += count[x] > n || (count[x] == n && x < row);
    for (int s = 1; s < per; s <<= 1) rank += __shfl_xor(rank, s);
    if (sub == 0 && tid / per < row_tiles) order[(int64_t)b * row_tiles + rank] = row;
}

// Single tokens in bf16: a tile of keys per wave, up to 512 workgroups.
//   The other kernels: as many parts as cost least.  A part's tiles take as long as
// its CU needs for all its workgroups, `busy` us a tile of each, or as one workgroup needs
// by itself, `alone`; parts add the outputs' way through memory and the join's launch.
// 24 heads of 1590 queries over 14 310 keys, d = 128 (312 workgroups of 224 tiles): 408 us
// in one part, 313 in four; fp32, 12 heads of 777 queries: 46 us in one, 38 in three; 64 of
// one query over 2000 keys, d = 64, 21 us in eight parts, 26 in 32.
ScorePlan score_plan(int dtype, int B, int Hk, int64_t rows, int Tk, int d) {
    const bool f32 = dtype != BC_BF16;
    ScorePlan p;
    p.rows = rows <= 16 ? 16 : f32 || rows <= 64 ? 64 : 128;
    const int64_t wgs = (int64_t)B * Hk * ((rows + p.rows - 1) / p.rows), tiles = (Tk + kKTile - 1) / kKTile, most = 64;
    if (p.rows == 16 && !f32) {
        p.parts = (int)std::max<int64_t>(1, std::min<int64_t>({512 / wgs, (tiles + 3) / 4, most}));
        return p;
    }
    const double busy = f32 && p.rows == 16 ? 0.4 + d / 64.0 : (f32 ? 4.0 : p.rows == 64 ? 0.6 : 1.0) * d / 128.0;
    const double alone = f32 ? (p.rows == 16 ? 1.5 + d / 128.0 : 2.0 + d / 32.0) : (p.rows == 64 ? 1.0 : 1.5) * (0.4 + 0.6 * d / 128.0);
    const double part = 8.0 * B * Hk * rows * d / 5e6;
    double best = 0.0;
    p.parts = 1;
    for (int64_t n = 1; n <= std::min(most, tiles); ++n) {
        const int64_t rounds = (wgs * n + 255) / 256;
        const double cost = (double)((tiles + n - 1) / n) * std::max(rounds * busy, alone) + (n > 1 ? 5.0 + n * part : 0.0);
        if (n == 1 || cost < best) {
            best = cost;
            p.parts = (int)n;
        }
        if (rounds > 16) break;
    }
    return p;
}

size_t score_part_bytes(const ScorePlan& p, int B, int Hq, int Tq, int d) {
    return p.parts < 2 ? 0 : (size_t)B * Tq * Hq * p.parts * (d + 2) * sizeof(float);
}

int score_shape(int B, int Hq, int Hk, int Tq, int Tk, int d, int dtype) {
    if (B < 1 || Hq < 1 || Hk < 1 || Tq < 1 || Tk < 1 || d < 1) return fail(BC_ERR_INVALID_ARG, "empty attention");
    if (Hq % Hk) return fail(BC_ERR_INVALID_ARG, "%d query heads over %d key heads", Hq, Hk);
    if (dtype != BC_F32 && dtype != BC_BF16) return fail(BC_ERR_INVALID_ARG, "dtype %d", dtype);
    if (!attention_supported(d)) return fail(BC_ERR_UNSUPPORTED, "head_dim %d (supported: 32, 64, 72, 128)", d);
    if (Tq > kMaxPosition || Tk > kMaxPosition)
        return fail(BC_ERR_UNSUPPORTED, "attention of %d queries over %d keys: at most %d", Tq, Tk, kMaxPosition);
    if ((int64_t)B * Hq > (1 << 20) || (int64_t)Hq * d > (1 << 24) || (int64_t)Tq * Hq > (1 << 30) || (int64_t)B * Tk > 0x7fffffff)
        return fail(BC_ERR_UNSUPPORTED, "attention: %d x %d heads of %d queries over %d keys", B, Hq, Tq, Tk);
    return BC_OK;
}

int score_options(const bc_score_opts* o, int d, ScoreArgs* a) {
    const bc_score_opts none = {};
    if (!o) o = &none;
    const double scale = o->scale == 0.0 ? 1.0 / std::sqrt((double)d) : o->scale;
    if (!(scale >= 1e-6 && scale <= 1e5)) return fail(BC_ERR_INVALID_ARG, "scale %g outside [1e-6, 1e5]", scale);
    if (o->cap != 0.0 && !(o->cap >= 1e-3 && o->cap <= 1e6)) return fail(BC_ERR_INVALID_ARG, "cap %g: 0 or in [1e-3, 1e6]", o->cap);
    if (o->window < 0 || o->window > kMaxPosition) return fail(BC_ERR_INVALID_ARG, "window %d outside [0, %d]", o->window, kMaxPosition);
    if (reinterpret_cast<uintptr_t>(o->slopes) % 4 || reinterpret_cast<uintptr_t>(o->prefix) % 4)
        return fail(BC_ERR_INVALID_ARG, "slopes and prefix must be 4-byte aligned");
    const double log2e = 1.4426950408889634;
    a->scale_log2 = (float)(scale * log2e);
    a->cap_log2 = (float)(o->cap * log2e);
    a->cap_exp = o->cap != 0.0 ? (float)(2.0 * log2e * scale / o->cap) : 0.f;
    a->cap_wide = o->cap > kCapNear;
    a->slopes = o->slopes;
    a->causal = o->causal != 0;
    a->window = o->window;
    a->prefix = o->prefix;
    return BC_OK;
}

int score_operand(const char* name, const void* p, int64_t batch, int64_t row, int B, int64_t T, int64_t width, int dtype, Span* s) {
    const int e = dtype_size(dtype);
    if (!p) return fail(BC_ERR_INVALID_ARG, "%s is NULL", name);
    if (!strides_fit(B, batch, T, row) || batch > ((int64_t)1 << 48) || row > ((int64_t)1 << 32))
        return fail(BC_ERR_INVALID_ARG, "%s: strides %lld, %lld", name, (long long)batch, (long long)row);
    if (reinterpret_cast<uintptr_t>(p) % 16 || (B > 1 && batch * e % 16) || (T > 1 && row * e % 16))
        return fail(BC_ERR_INVALID_ARG, "%s: rows must be 16-byte aligned", name);
    *s = {p, ((B - 1) * batch + (T - 1) * row + width) * e};
    return BC_OK;
}

int score_apart(const Span* written, int nw, const Span* read, int nr) {
    for (int i = 0; i < nw; ++i) {
        for (int j = 0; j < nr; ++j)
            if (overlap(written[i].p, written[i].n, read[j].p, read[j].n))
                return fail(BC_ERR_INVALID_ARG, "the output and the workspace must not overlap another operand");
        for (int j = 0; j < i; ++j)
            if (overlap(written[i].p, written[i].n, written[j].p, written[j].n))
                return fail(BC_ERR_INVALID_ARG, "the output and the workspace must not overlap");
    }
    return BC_OK;
}

int score_grid(const ScorePlan& p, const ScoreArgs& a) {
    const int64_t wgs = (int64_t)a.B * a.Hk * (((int64_t)a.Tq * a.G + p.rows - 1) / p.rows) * p.parts;
    const int64_t rows = (int64_t)a.B * a.Tq * a.Hk * a.G;
    if (wgs > kMaxGrid || (p.parts > 1 && rows * (a.d / 4) > kMaxGrid * 256)) return fail(BC_ERR_UNSUPPORTED, "attention grid too large");
    return BC_OK;
}

int score_join(int dtype, const ScoreArgs& a, hipStream_t s) {
    AttnArgs j = {};
    j.B = a.B; j.H = a.Hk * a.G; j.Tq0 = a.Tq; j.d = a.d;
    j.o0 = a.out;
    j.parts = a.parts; j.part_o = a.part_o; j.part_ml = a.part_ml;
    return launch_attention_join(dtype, j, true, s);
}

// The documents' part of the workspace: ranges of keys and queries, and the order of the rows where there is one.
static size_t range_bytes(int B, int Tk, int Tq) { return ((size_t)B * ((Tk + 63) / 64 + (Tq + 63) / 64) * sizeof(u32x2) + 255) / 256 * 256; }
static bool ordered(const ScorePlan& p, int B, int Hk, int64_t rows, int Tk) {
    const int64_t n = (rows + p.rows - 1) / p.rows;
    return n * B * Hk > 512 && n <= kOrderRows && Tk <= 64 * kOrderKeys;
}
static size_t document_bytes(const ScorePlan& p, int B, int Hk, int64_t rows, int Tk, int Tq) {
    return range_bytes(B, Tk, Tq) + (ordered(p, B, Hk, rows, Tk) ? ((size_t)B * ((rows + p.rows - 1) / p.rows) * sizeof(int) + 255) / 256 * 256 : 0);
}

}  // namespace bc

using namespace bc;

extern "C" {

int bc_attention_masked_workspace_size(int B, int Hq, int Hk, int Tq, int Tk, int d, int dtype, size_t* bytes) {
    clear_error();
    if (!bytes) return fail(BC_ERR_INVALID_ARG, "NULL pointer");
    const int rc = score_shape(B, Hq, Hk, Tq, Tk, d, dtype);
    if (rc != BC_OK) return rc;
    const int64_t rows = (int64_t)Tq * (Hq / Hk);
    const ScorePlan plan = score_plan(dtype, B, Hk, rows, Tk, d);
    *bytes = document_bytes(plan, B, Hk, rows, Tk, Tq) + score_part_bytes(plan, B, Hq, Tq, d);
    return BC_OK;
}

int bc_attention_masked(const bc_masked_desc* d, void* ws, size_t ws_bytes, void* stream) {
    clear_error();
    if (!d) return fail(BC_ERR_INVALID_ARG, "NULL pointer");
    int rc = score_shape(d->B, d->Hq, d->Hk, d->Tq, d->Tk, d->d, d->dtype);
    if (rc != BC_OK) return rc;
    ScoreArgs a = {};
    Span out[2], in[8];
    int nr = 3;
    const int64_t wk = (int64_t)d->Hk * d->d;
    if ((rc = score_operand("q", d->q, d->q_batch, d->q_row, d->B, d->Tq, (int64_t)d->Hq * d->d, d->dtype, &in[0])) != BC_OK ||
        (rc = score_operand("k", d->k, d->k_batch, d->k_row, d->B, d->Tk, wk, d->dtype, &in[1])) != BC_OK ||
        (rc = score_operand("v", d->v, d->v_batch, d->v_row, d->B, d->Tk, wk, d->dtype, &in[2])) != BC_OK ||
        (rc = score_options(&d->opts, d->d, &a)) != BC_OK)
        return rc;
    if (!d->out || reinterpret_cast<uintptr_t>(d->out) % dtype_size(d->dtype)) return fail(BC_ERR_INVALID_ARG, "out: NULL or not aligned to its elements");
    if (!d->q_docs != !d->k_docs) return fail(BC_ERR_INVALID_ARG, "documents of the queries and of the keys: both or neither");
    if ((reinterpret_cast<uintptr_t>(d->lens) | reinterpret_cast<uintptr_t>(d->q_docs) | reinterpret_cast<uintptr_t>(d->k_docs)) % 4)
        return fail(BC_ERR_INVALID_ARG, "lens and documents must be 4-byte aligned");
    if (d->q_start < -kMaxPosition || d->q_start > kMaxPosition - d->Tq)
        return fail(BC_ERR_INVALID_ARG, "q_start %lld: positions within 2^24", (long long)d->q_start);
    a.q = d->q; a.k = d->k; a.v = d->v; a.out = d->out;
    a.q_batch = d->q_batch; a.q_row = d->q_row; a.k_batch = d->k_batch; a.k_row = d->k_row; a.v_batch = d->v_batch; a.v_row = d->v_row;
    a.B = d->B; a.Hk = d->Hk; a.G = d->Hq / d->Hk; a.Tq = d->Tq; a.Tk = d->Tk; a.d = d->d;
    a.lens = d->lens; a.q_docs = d->q_docs; a.k_docs = d->k_docs;
    a.q_start = (int)d->q_start;
    const ScorePlan plan = score_plan(d->dtype, d->B, d->Hk, (int64_t)d->Tq * a.G, d->Tk, d->d);
    a.parts = plan.parts;
    a.nt = plan.rows == 16 && 2.0 * d->B * wk * d->Tk * dtype_size(d->dtype) >= 80e6;
    if ((rc = score_grid(plan, a)) != BC_OK) return rc;
    const int64_t rows = (int64_t)d->Tq * a.G;
    const size_t ranges = d->q_docs ? document_bytes(plan, d->B, d->Hk, rows, d->Tk, d->Tq) : 0, parts = score_part_bytes(plan, d->B, d->Hq, d->Tq, d->d);
    out[0] = {d->out, (int64_t)d->B * d->Tq * d->Hq * d->d * dtype_size(d->dtype)};
    out[1] = {ws, (int64_t)(ranges + parts)};
    in[nr++] = {d->lens, (int64_t)d->B * 4};
    in[nr++] = {d->q_docs, (int64_t)d->B * d->Tq * 4};
    in[nr++] = {d->k_docs, (int64_t)d->B * d->Tk * 4};
    in[nr++] = {a.slopes, (int64_t)d->Hq * 4};
    in[nr++] = {a.prefix, (int64_t)d->B * 4};
    if (ranges + parts) {
        if (!ws || reinterpret_cast<uintptr_t>(ws) % 256) return fail(BC_ERR_INVALID_ARG, "a 256-byte aligned workspace is needed");
        if (ws_bytes < ranges + parts) return fail(BC_ERR_INVALID_ARG, "workspace %zu < %zu bytes", ws_bytes, ranges + parts);
    }
    if ((rc = score_apart(out, ranges + parts ? 2 : 1, in, nr)) != BC_OK) return rc;
    if (parts) {
        a.part_o = reinterpret_cast<float*>(static_cast<char*>(ws) + ranges);
        a.part_ml = a.part_o + (int64_t)d->B * d->Tq * d->Hq * a.parts * d->d;
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    prof_begin(PROF_ATTENTION, s, 4.0 * d->B * d->Hq * (double)d->Tq * d->Tk * d->d);
    if (ranges) {
        const int64_t tiles = (int64_t)d->B * ((d->Tk + 63) / 64 + (d->Tq + 63) / 64);
        a.ranges = static_cast<const u32x2*>(ws);
        launch_k(document_ranges_kernel, dim3((unsigned)((tiles + 3) / 4)), dim3(256), s, d->k_docs, d->q_docs, d->lens, d->B, d->Tk, d->Tq,
                 static_cast<u32x2*>(ws));
        rc = check_launch("document ranges");
        if (rc == BC_OK && ordered(plan, d->B, d->Hk, rows, d->Tk)) {
            int* order = reinterpret_cast<int*>(static_cast<char*>(ws) + range_bytes(d->B, d->Tk, d->Tq));
            a.order = order;
            launch_k(row_order_kernel, dim3((unsigned)d->B), dim3(kOrderRows), s, a.ranges, d->B, d->Tk, d->Tq, a.G, plan.rows,
                     (int)((rows + plan.rows - 1) / plan.rows), order);
            rc = check_launch("row order");
        }
    }
    if (rc == BC_OK) rc = launch_score<false>(d->dtype, plan, a, s);
    if (rc == BC_OK && plan.parts > 1) rc = score_join(d->dtype, a, s);
    prof_end(PROF_ATTENTION, s);
    return rc;
}

}  // extern "C"
