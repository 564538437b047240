// Attention over selected key blocks: the score that selects them, and the
// entry points (the attention itself is attention.hip's, over a list of tiles).
//
// For every sample and head, block i of 128 queries scores block j of 64 keys
// by the product of their means, mean(q_i) . mean(k_j), and keeps the `keep`
// best.  Means and products are held in 64 bits: a score is off by at most about
// (d + 130) 2^-53 of the magnitudes summed, so that only blocks whose scores agree to
// that may change places; equal blocks have equal scores, which go to the lowest
// index.  The arithmetic is 0.1 % of what the attention over the blocks takes.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "attention_tile.h"

namespace bc {

struct SelectArgs {
    const void *q, *k;
    const int* lens;
    int B, H, Tq, Tk, d, keep, keep_last;
    int nqb, nkb;
    double *qm, *km;        // means of the query and of the key blocks, [B][H][mean_at]
    int* blocks;
};

// Where a head's mean of column c of block i stands: 16 blocks' pieces of eight
// columns side by side, so that a wave of the scores loads 1024 consecutive bytes.
__host__ __device__ __forceinline__ int64_t mean_at(int i, int c, int d) {
    return ((int64_t)(i >> 4) * (d >> 3) + (c >> 3)) * 128 + (i & 15) * 8 + (c & 7);
}
// Values of a head's means, whole groups of 16 blocks.
__host__ __device__ __forceinline__ int64_t mean_size(int blocks, int d) { return (int64_t)((blocks + 15) / 16) * 16 * d; }

__device__ __forceinline__ int select_keys(const SelectArgs& a, int b) {
    return a.lens ? min(max(a.lens[b], 0), a.Tk) : a.Tk;
}

// Means of the blocks: memory bound, q and k once.  A workgroup takes 32 chunks
// of 8 columns of one block's rows, eight threads per chunk each an eighth of the
// rows (16 bytes a load, 512 consecutive bytes per row), which meet in LDS in a
// fixed order.  14 566 x 3072 queries and keys (179 MB): 34 us, 5.3 TB/s (8 or 16
// loads on their way instead of 4: 1 us more; non-temporal ones 3 us less there, but
// 4 more on 61 MB, which the caches hold, as they do for the attention that reads
// the tensors next).  Rows past the end are not read; a block without rows has zero
// means.
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
#pragma unroll 4
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
    const int col = piece * 256 + tid, h = col / a.d;
    double* out = keys ? a.km + (b * a.H + h) * mean_size(a.nkb, a.d) : a.qm + (b * a.H + h) * mean_size(a.nqb, a.d);
    out[mean_at(i, col - h * a.d, a.d)] = n > 0 ? t / (double)n : 0.0;
}

// The order of scores as unsigned integers: -0 as +0, a NaN below every number;
// 0 is kept for blocks that are not there.
__device__ __forceinline__ uint64_t score_key(double s) {
    if (s != s) return 1;
    const uint64_t u = (uint64_t)__double_as_longlong(s + 0.0);
    return u >> 63 ? ~u : u | ((uint64_t)1 << 63);
}

// The list of one row of keys, key[t] of lane l being that of block 64 t + l: the
// keep-th largest by bisection over the bits, with ballots, then the blocks above
// it and as many equal to it, the lowest first, as are still wanted.
template <int NR>
__device__ __forceinline__ void write_list(const uint64_t (&key)[NR], int valid, int keep, int lane, int* out) {
    auto count_from = [&](uint64_t least) __attribute__((always_inline)) {
        int n = 0;
#pragma unroll
        for (int t = 0; t < NR; ++t) n += __popcll(__ballot(key[t] >= least));
        return n;
    };
    uint64_t T = 1;      // every block that is there, if they are no more than `keep`
    if (valid > keep) {
        // The upper 32 bits by themselves: half the work a bit, and mostly enough.
        uint32_t top = 0;
        int n = 0;
        for (int bit = 31; bit >= 0 && n != keep; --bit) {
            const uint32_t cand = top | (1u << bit);
            n = 0;
#pragma unroll
            for (int t = 0; t < NR; ++t) n += __popcll(__ballot((uint32_t)(key[t] >> 32) >= cand));
            if (n >= keep) top = cand;
        }
        T = (uint64_t)top << 32;
        for (int bit = 31; bit >= 0 && n != keep; --bit) {
            const uint64_t cand = T | ((uint64_t)1 << bit);
            n = count_from(cand);
            if (n >= keep) T = cand;
        }
    }
    const int above = T == ~(uint64_t)0 ? 0 : count_from(T + 1);
    const uint64_t before = ((uint64_t)1 << lane) - 1;
    const int wanted = min(keep, valid) - above;
    int at = 0, tied = 0;
#pragma unroll
    for (int t = 0; t < NR; ++t) {
        const uint64_t eq = __ballot(key[t] == T);
        const bool sel = key[t] > T || (key[t] == T && tied + __popcll(eq & before) < wanted);
        const uint64_t sm = __ballot(sel);
        if (sel) out[at + __popcll(sm & before)] = 64 * t + lane;
        at += __popcll(sm);
        tied += __popcll(eq);
    }
    for (int x = at + lane; x < keep; x += 64) out[x] = -1;
}

// Scores of 16 query blocks against every key block on fp64 MFMAs, a tile of 16
// key blocks a wave at a time, into LDS as keys; then a wave per query block writes
// its list.  The query means come once into LDS, the key means straight from
// memory: a lane's 16 bytes are two of its row's values, which two MFMAs take, so k
// runs permuted alike in both.  24 heads of 114 x 228 blocks, d = 128, with the
// means' 35 us: 87 us with a query block per wave, key blocks through LDS and vector
// FMAs; 55.6 with a block's means one row, so that a load takes 64 bytes of each of
// 16 rows; 50.6 laid out as in mean_at; 48.5 with the query means in LDS (4 of them
// the lists; 192 workgroups in one round: the chain of one, loads, 32 MFMAs of four
// waves a SIMD, bisection, is the time).  625 x 625 blocks 190 -> 149 us.
template <int D, int NR>
__global__ __launch_bounds__(1024) void score_select_kernel(SelectArgs a) {
    typedef double d2 __attribute__((ext_vector_type(2)));
    typedef double d4 __attribute__((ext_vector_type(4)));
    __shared__ uint64_t sk[16][64 * NR];
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, grp = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int groups = (a.nqb + 15) / 16;
    const int pid = xcd_contiguous(blockIdx.x, gridDim.x);      // a head's workgroups share its means in one L2
    const int bh = pid / groups, b = bh / a.H;
    const int i0 = (pid % groups) * 16;
    const int valid = (select_keys(a, b) + kSparseK - 1) / kSparseK;      // key blocks that there are
    // (Blocks past the last one take part with what the workspace holds; no list has them.)
    const d2* qm = reinterpret_cast<const d2*>(a.qm + bh * mean_size(a.nqb, D) + mean_at(i0, 0, D));
    __shared__ d2 sq[8 * D];
    if (tid < 8 * D) sq[tid] = qm[tid];
    __syncthreads();
    for (int j0 = 16 * wave; j0 < valid; j0 += 256) {
        const d2* km = reinterpret_cast<const d2*>(a.km + bh * mean_size(a.nkb, D) + mean_at(j0 + l16, 2 * grp, D));
        d4 acc = {0.0, 0.0, 0.0, 0.0};
#pragma unroll 8
        for (int c = 0; c < D / 8; ++c) {
            const d2 qv = sq[64 * c + 4 * l16 + grp], kv = km[64 * c];
            acc = __builtin_amdgcn_mfma_f64_16x16x4f64(qv[0], kv[0], acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f64_16x16x4f64(qv[1], kv[1], acc, 0, 0, 0);
        }
        // Register r of lane l: query block 4 r + l / 16, key block l % 16.
        const int j = j0 + l16;
#pragma unroll
        for (int r = 0; r < 4; ++r)
            sk[4 * r + grp][j] = j >= valid ? 0 : j >= valid - a.keep_last ? ~(uint64_t)0 : score_key(acc[r]);
    }
    __syncthreads();
    if (i0 + wave >= a.nqb) return;
    uint64_t key[NR];
#pragma unroll
    for (int t = 0; t < NR; ++t) key[t] = 64 * t + lane < valid ? sk[wave][64 * t + lane] : 0;
    write_list<NR>(key, valid, a.keep, lane, a.blocks + ((int64_t)bh * a.nqb + i0 + wave) * a.keep);
}

// Above 1024 key blocks, whose keys LDS does not hold for 16 rows: a query block
// per wave, lane l the key blocks l, l + 64, ... in registers, their means through
// LDS 64 at a time for the four waves (a row of D + 2 doubles keeps the 16-byte
// reads of neighbouring lanes on other banks).  2 heads of 782 x 1563 blocks, d =
// 128: 187 us with the means.
template <int D>
__global__ __launch_bounds__(256) void score_select_long_kernel(SelectArgs a) {
    constexpr int LD = D + 2, NR = kSparseMaxBlocks / 64;
    __shared__ __attribute__((aligned(16))) double sk[64 * LD];
    typedef double d2 __attribute__((ext_vector_type(2)));
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int groups = (a.nqb + 3) / 4;
    const int pid = xcd_contiguous(blockIdx.x, gridDim.x);
    const int bh = pid / groups, b = bh / a.H;
    const int i = (pid % groups) * 4 + wave;
    const int valid = (select_keys(a, b) + kSparseK - 1) / kSparseK;
    const double* km = a.km + bh * mean_size(a.nkb, D);
    const double* qm = a.qm + bh * mean_size(a.nqb, D);
    const int iq = min(i, a.nqb - 1);
    uint64_t key[NR];
#pragma unroll
    for (int t = 0; t < NR; ++t) {
        key[t] = 0;
        if (64 * t < valid) {
            __syncthreads();
            // In the order they stand: groups of 16 blocks, of the last tile those that there are.
            const int n = min(4, (valid + 15) / 16 - 4 * t) * 8 * D;
            for (int x = tid; x < n; x += 256) {
                const int row = 16 * (x / (8 * D)) + (x % 64) / 4, col = x % (8 * D) / 64 * 8 + 2 * (x % 4);
                *reinterpret_cast<d2*>(&sk[row * LD + col]) = reinterpret_cast<const d2*>(km + mean_at(64 * t, 0, D))[x];
            }
            __syncthreads();
            double acc = 0.0;
#pragma unroll 4
            for (int c = 0; c < D; c += 2) {
                const d2 kv = *reinterpret_cast<const d2*>(&sk[lane * LD + c]);
                const double* qv = qm + mean_at(iq, c, D);
                acc = fma(qv[0], kv[0], acc);
                acc = fma(qv[1], kv[1], acc);
            }
            const int j = 64 * t + lane;
            key[t] = j >= valid ? 0 : j >= valid - a.keep_last ? ~(uint64_t)0 : score_key(acc);
        }
    }
    if (i < a.nqb) write_list<NR>(key, valid, a.keep, lane, a.blocks + ((int64_t)bh * a.nqb + i) * a.keep);
}

template <int D>
static void run_score_select(const SelectArgs& a, hipStream_t s) {
    const int nr = (a.nkb + 63) / 64;
    const dim3 g((unsigned)((int64_t)a.B * a.H * ((a.nqb + 15) / 16))), block(1024);
    if (nr <= 1) launch_k(score_select_kernel<D, 1>, g, block, s, a);
    else if (nr <= 4) launch_k(score_select_kernel<D, 4>, g, block, s, a);
    else if (nr <= 16) launch_k(score_select_kernel<D, 16>, g, block, s, a);
    else launch_k(score_select_long_kernel<D>, dim3((unsigned)((int64_t)a.B * a.H * ((a.nqb + 3) / 4))), dim3(256), s, a);
}

// ---------------------------------------------------------------------------
// Up to 16 queries per head (single tokens): bf16, one MFMA tile of queries.
// Such a call is a chain of latencies (the list, its keys, the join) over few
// bytes, so each wave takes key blocks of its own, with no barrier until its
// workgroup's four waves meet in LDS: keys go straight into MFMA operands,
// values through the wave's LDS tile, both requested at once.  The code is kept
// short: these launches run each line once or twice, and one-wave tiles of the
// streaming kernel took 7 us a step.
//   The probabilities are rounded to bf16 (by 2^-8 of themselves at most) because P V
// is then an MFMA on the values as they lie: in fp32 it would take 16 times the MFMA
// cycles and a conversion of every value, for an error that over a row's keys comes
// to about the output's own rounding.  The row sums are those of the rounded ones, so
// that a row's weights add up to one.
//   NT: launches whose lists stream past the caches fetch the values so: 4 x 16
// heads of 256 blocks, d = 128 (537 MB) 111 -> 103 us (5.2 TB/s), 134 MB 37 -> 34;
// 33 MB 13.5 either way, 4 MB 7.7 and 8.5.  The keys as well: no better.
// ---------------------------------------------------------------------------
template <int HD, bool QS, bool NT>
__global__ __launch_bounds__(256) void sparse_few_kernel(AttnArgs a) {
    typedef AttnShape<bf16, HD> S;
    typedef KvLayout<HD> LY;
    typedef __attribute__((address_space(3))) const char lds_char;
    constexpr int TILE = kKTile * HD + 32;                // + slack, read for operand rows d >= HD
    __shared__ __attribute__((aligned(1024))) bf16 sV[4][TILE];
    __shared__ float sml[4][16][2];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int pid = xcd_contiguous(blockIdx.x, gridDim.x);
    const int part = pid % a.parts, bh = pid / a.parts;
    const int b = bh / a.H, h = bh % a.H;
    const int Tq = a.Tq0, ql = lane & 15, grp = lane >> 4;
    const int Tk = __builtin_amdgcn_readfirstlane(sparse_keys(a, b));
    const int* list = a.blocks + (int64_t)bh * a.keep;
    bf16x8 qf[S::n32x];
#pragma unroll
    for (int c = 0; c < S::n32x; ++c) {
        const int d = 32 * c + grp * 8;
        qf[c] = __builtin_bit_cast(bf16x8, u32x4{0u, 0u, 0u, 0u});
        if (ql < Tq && d < HD)
            qf[c] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(static_cast<const bf16*>(a.q0) + ((int64_t)b * Tq + ql) * a.ldq + h * HD + d));
    }
    if (lane < 32) sV[wave][kKTile * HD + lane] = (bf16)0.f;
    const bf16* kb = static_cast<const bf16*>(a.k0) + (int64_t)b * a.Tk0 * a.ldk + h * HD;
    const bf16* vb = static_cast<const bf16*>(a.v0) + (int64_t)b * a.Tk0 * a.ldv + h * HD;
    const float sc = QS ? 1.f : a.scale_log2;
    const int n = sparse_list_length(list, a.keep, (Tk + kKTile - 1) / kKTile, lane);
    f32x4 o[S::DV / 16];
#pragma unroll
    for (int i = 0; i < S::DV / 16; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    lds_char* Vb = (lds_char*)&sV[wave][0];
#pragma unroll 1
    for (int t = part * 4 + wave; t < n; t += 4 * a.parts) {
        const int k0 = __builtin_amdgcn_readfirstlane(list[t]) * kKTile;
        // Rows past the sample's last key repeat it; their scores are masked, and their
        // values zeroed before they are read (a masked infinity would be NaN).
#pragma unroll
        for (int j = 0; j < LY::CPR; ++j) {
            const int c = 64 * j + lane, row = c / LY::CPR, slot = c % LY::CPR;
            const bf16* from = vb + (int64_t)min(k0 + row, Tk - 1) * a.ldv + 8 * LY::slot(row, slot);
            if constexpr (NT) dma16_nt(from, &sV[wave][64 * j * 8]);
            else dma16(from, &sV[wave][64 * j * 8]);
        }
        u32x4 kf[4][S::n32x];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bf16* kr = kb + (int64_t)min(k0 + 16 * j + ql, Tk - 1) * a.ldk;
#pragma unroll
            for (int c = 0; c < S::n32x; ++c) {
                const int d = 32 * c + grp * 8;
                kf[j][c] = d < HD ? *reinterpret_cast<const u32x4*>(kr + d) : u32x4{0u, 0u, 0u, 0u};
            }
        }
        f32x4 s[4];
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            s[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < S::n32x; ++c)
                s[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[j][c]), qf[c], s[j], 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s[j][r] = k0 + 16 * j + 4 * grp + r < Tk ? s[j][r] * sc : -INFINITY;
                top = vmax(top, s[j][r]);
            }
        }
        const float m_new = vmax(m, group_max(top));
        const float alpha = __builtin_amdgcn_exp2f(m - m_new);
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
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // the value tile
        if (k0 + kKTile > Tk)
            for (int x = lane; x < (k0 + kKTile - Tk) * LY::CPR; x += 64)
                *reinterpret_cast<u32x4*>(&sV[wave][(Tk - k0) * HD + 8 * x]) = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int i = 0; i < S::DV / 16; ++i) {
            o[i] *= alpha;
            const uint32_t at = 2u * (uint32_t)LY::at(4 * grp + (ql >> 2), 16 * i + 4 * (ql & 3));
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                // keys 32u + 4grp + 0..3 and 32u + 16 + 4grp + 0..3 of column 16i + ql
                lds_char* p = Vb + at + 64u * u * HD;
                const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p));
                const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p + 32 * HD)));
                o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, u32x4{lo.x, lo.y, hi.x, hi.y}), pf[u], o[i], 0, 0, 0);
            }
        }
    }
    l = group_sum(l);
    // The waves meet: outputs [16][HD] fp32 over their value tiles.
    float* so = reinterpret_cast<float*>(&sV[wave][0]);
#pragma unroll
    for (int i = 0; i < S::DV / 16; ++i)
        if (16 * i + 4 * grp < HD && ql < Tq) *reinterpret_cast<f32x4*>(so + ql * HD + 16 * i + 4 * grp) = o[i];
    if (grp == 0) {
        sml[wave][ql][0] = m;
        sml[wave][ql][1] = l;
    }
    __syncthreads();
    for (int x = tid; x < Tq * HD; x += 256) {
        const int q = x / HD, d = x - q * HD;
        float top = sml[0][q][0];
#pragma unroll
        for (int w = 1; w < 4; ++w) top = fmaxf(top, sml[w][q][0]);
        float acc = 0.f, sum = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = sml[w][q][1] != 0.f ? exp2f(sml[w][q][0] - top) : 0.f;      // (0: the wave had no block)
            acc = fmaf(f, f != 0.f ? reinterpret_cast<const float*>(&sV[w][0])[x] : 0.f, acc);
            sum = fmaf(f, sml[w][q][1], sum);
        }
        const int64_t row = ((int64_t)b * Tq + q) * a.H + h;
        if (a.parts > 1) {
            a.part_o[(row * a.parts + part) * HD + d] = acc;
            if (d == 0) {
                a.part_ml[(row * a.parts + part) * 2] = top;
                a.part_ml[(row * a.parts + part) * 2 + 1] = sum;
            }
        } else {
            static_cast<bf16*>(a.o0)[((int64_t)b * Tq + q) * a.ldo + h * HD + d] = (bf16)(sum != 0.f ? acc / sum : 0.f);
        }
    }
}

// Joins the parts of a query's list: sum_p 2^(m_p - M) o_p over sum_p 2^(m_p - M)
// l_p, M the largest m_p.  A workgroup per query and head: 256 / (d / 4) parts at
// a time, four columns a thread, then over the parts in LDS in a fixed order.
// KEEP (launch_attention_join): where a sum is not finite, it is made anew from outputs of which those
// that are not finite stay what they are.
constexpr int kMaxParts = 64;
template <typename T_, int HD, bool KEEP>
__global__ __launch_bounds__(256) void sparse_join_kernel(AttnArgs a) {
    typedef elem_t<T_> T;
    constexpr int C = HD / 4, SLOTS = 256 / C, TURNS = (kMaxParts + SLOTS - 1) / SLOTS;
    __shared__ f32x4 red[SLOTS][C];
    const int tid = threadIdx.x, lane = tid & 63, col = tid % C, slot = tid / C;
    const int64_t row = blockIdx.x;                       // (b Tq + q) H + h
    const float* po = a.part_o + row * a.parts * HD + col * 4;
    const float* ml = a.part_ml + row * a.parts * 2;
    f32x4 v[TURNS];
    float mp[TURNS];
#pragma unroll
    for (int u = 0; u < TURNS; ++u) {
        const int p = slot + SLOTS * u;
        const bool there = slot < SLOTS && p < a.parts && ml[2 * p + 1] != 0.f;      // a part without blocks wrote no outputs
        mp[u] = there ? ml[2 * p] : -INFINITY;
        v[u] = there ? *reinterpret_cast<const f32x4*>(po + (int64_t)p * HD) : f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const float m = lane < a.parts ? ml[2 * lane] : -INFINITY, l = lane < a.parts ? ml[2 * lane + 1] : 0.f;
    float top = m;
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) top = fmaxf(top, __shfl_xor(top, x));
    const float sum = wave_sum(l != 0.f ? exp2f(m - top) * l : 0.f);
    auto total = [&](auto keep) __attribute__((always_inline)) {
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < TURNS; ++u) acc += times<decltype(keep)::value>(v[u], top == -INFINITY ? 0.f : exp2f(mp[u] - top));
        return acc;
    };
    f32x4 acc = total(std::false_type{});
    if (KEEP && !all_finite(acc)) acc = total(std::true_type{});
    if (slot < SLOTS) red[slot][col] = acc;
    __syncthreads();
    if (tid >= C) return;
    acc = red[0][tid];
#pragma unroll
    for (int x = 1; x < SLOTS; ++x) acc += red[x][tid];
    const float inv = sum != 0.f ? 1.f / sum : 0.f;
    T* out = static_cast<T*>(a.o0) + row * HD + tid * 4;
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] = (T)(acc[e] * inv);
}

// The same for many rows: a thread takes four columns of a row over its few parts.
template <typename T_, int HD, bool KEEP>
__global__ __launch_bounds__(256) void sparse_join_rows_kernel(AttnArgs a, int64_t rows) {
    typedef elem_t<T_> T;
    constexpr int C = HD / 4, U = 4;
    const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t row = x / C;
    if (row >= rows) return;
    const float* po = a.part_o + row * a.parts * HD + (x - row * C) * 4;
    const float* ml = a.part_ml + row * a.parts * 2;
    float top, sum;
    f32x4 acc;
    auto total = [&](auto keep) __attribute__((always_inline)) {
        top = -INFINITY;
        sum = 0.f;
        acc = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int p0 = 0; p0 < a.parts; p0 += U) {
            f32x4 v[U];
            float m[U], l[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int p = p0 + u;
                m[u] = p < a.parts ? ml[2 * p] : -INFINITY;
                l[u] = p < a.parts ? ml[2 * p + 1] : 0.f;
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
                v[u] = l[u] != 0.f ? *reinterpret_cast<const f32x4*>(po + (int64_t)(p0 + u) * HD) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (l[u] == 0.f) continue;      // a part without blocks wrote no outputs
                const float next = fmaxf(top, m[u]), down = exp2f(top - next), f = exp2f(m[u] - next);
                sum = fmaf(f, l[u], sum * down);
                acc = times<decltype(keep)::value>(acc, down) + times<decltype(keep)::value>(v[u], f);
                top = next;
            }
        }
    };
    total(std::false_type{});
    if (KEEP && !all_finite(acc)) total(std::true_type{});
    const float inv = sum != 0.f ? 1.f / sum : 0.f;
    T* out = static_cast<T*>(a.o0) + x * 4;
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] = (T)(acc[e] * inv);
}

// How a call is laid out: queries of a workgroup, and the parts that each list is
// cut into where its workgroups alone would leave CUs idle.
//   Single tokens: a block per wave, up to 512 workgroups (16 heads x 128 blocks,
// d = 64, 13.9 us; 16 x 256 at 16 queries, d = 128, 38 us, 44 with up to 1024).
//   Tiles of 64 or 128 queries: parts for at most a workgroup per CU, of two blocks
// at least, where a list is six blocks shorter for it (the join is a launch, 4-5
// us): 24 heads of 40 queries over 64 blocks 61 us in one part, 18.8 so, 22 with
// two workgroups per CU; 4 x 2 workgroups of 16 blocks 16.8 and 10.4; 192
// workgroups of 17 blocks 29.2 in one part, 36.8 in two, 99 of 9 blocks 18.7 and 20.4.
//   fp32, whose block takes a workgroup about 4 us: down to a block a part, two
// workgroups per CU, where a list is two blocks shorter.  2 heads of one query over
// 60 blocks 232 us in one part, 11.8 so, 14.9 with two blocks a part; 16 x 5
// workgroups of 24 blocks 61, 25 so, 28 with one workgroup per CU; 32 x 8 of 30 123,
// 105, 125.
struct SparsePlan {
    int tile, parts;
};
static SparsePlan sparse_plan(int dtype, int B, int H, int Tq, int Tk, int keep) {
    const int tile = dtype != BC_BF16 ? 64 : Tq <= 16 ? 16 : Tq <= 64 ? 64 : kSparseQ;
    const int64_t wgs = (int64_t)B * H * ((Tq + tile - 1) / tile);
    const int64_t blocks = std::min(keep, (Tk + kSparseK - 1) / kSparseK);     // of a list
    if (tile == 16) return {tile, (int)std::max<int64_t>(1, std::min<int64_t>({512 / wgs, (blocks + 3) / 4, kMaxParts}))};
    const bool f32 = dtype != BC_BF16;
    const int64_t parts = std::max<int64_t>(1, std::min<int64_t>({(f32 ? 512 : 256) / wgs, f32 ? blocks : blocks / 2, kMaxParts}));
    return {tile, blocks - blocks / parts >= (f32 ? 2 : 6) ? (int)parts : 1};
}
static size_t part_bytes(const SparsePlan& p, int B, int H, int Tq, int d) {
    return p.parts < 2 ? 0 : (size_t)B * Tq * H * p.parts * (d + 2) * sizeof(float);
}

template <typename T, int HD, bool KEEP>
static int run_sparse_join(const AttnArgs& a, hipStream_t s) {
    const int64_t rows = (int64_t)a.B * a.H * a.Tq0;
    // Rows: 528 of 16 parts 12.8 us the call either way, 3135 of 4 parts 16.3 and 13.4; 16 of 32 13.9 and 18.8.
    if (rows < 512) launch_k(sparse_join_kernel<tag_t<T>, HD, KEEP>, dim3((unsigned)rows), dim3(256), s, a);
    else launch_k(sparse_join_rows_kernel<tag_t<T>, HD, KEEP>, dim3((unsigned)((rows * (HD / 4) + 255) / 256)), dim3(256), s, a, rows);
    return check_launch("sparse join");
}

template <typename T, int HD>
static int run_join(const AttnArgs& a, bool keep, hipStream_t s) {
    return keep ? run_sparse_join<T, HD, true>(a, s) : run_sparse_join<T, HD, false>(a, s);
}

int launch_attention_join(int dtype, const AttnArgs& a, bool keep, hipStream_t s) {
    switch (a.d) {
        case 32: return dtype == BC_F32 ? run_join<float, 32>(a, keep, s) : run_join<bf16, 32>(a, keep, s);
        case 64: return dtype == BC_F32 ? run_join<float, 64>(a, keep, s) : run_join<bf16, 64>(a, keep, s);
        case 72: return dtype == BC_F32 ? run_join<float, 72>(a, keep, s) : run_join<bf16, 72>(a, keep, s);
        default: return dtype == BC_F32 ? run_join<float, 128>(a, keep, s) : run_join<bf16, 128>(a, keep, s);
    }
}

template <int HD>
static int run_sparse(const SparsePlan& p, const AttnArgs& a, hipStream_t s) {
    int rc;
    if (p.tile == 16) {
        const dim3 g((unsigned)(a.B * a.H * a.parts));
        const bool nt = 4.0 * a.B * a.H * HD * std::min((double)a.keep * kSparseK, (double)a.Tk0) >= 80e6;
        if (a.q_scaled && nt) launch_k(sparse_few_kernel<HD, true, true>, g, dim3(256), s, a);
        else if (a.q_scaled) launch_k(sparse_few_kernel<HD, true, false>, g, dim3(256), s, a);
        else if (nt) launch_k(sparse_few_kernel<HD, false, true>, g, dim3(256), s, a);
        else launch_k(sparse_few_kernel<HD, false, false>, g, dim3(256), s, a);
        rc = check_launch("sparse attention");
    } else {
        rc = launch_sparse_tiles(BC_BF16, a, p.tile, s);
    }
    return rc != BC_OK || p.parts == 1 ? rc : run_sparse_join<bf16, HD, false>(a, s);
}

static int launch_sparse_attention(int dtype, const SparsePlan& p, const AttnArgs& a, hipStream_t s) {
    if (dtype == BC_F32) {
        const int rc = launch_sparse_tiles(dtype, a, p.tile, s);
        return rc != BC_OK || p.parts == 1 ? rc : launch_attention_join(dtype, a, false, s);
    }
    switch (a.d) {
        case 32: return run_sparse<32>(p, a, s);
        case 64: return run_sparse<64>(p, a, s);
        case 72: return run_sparse<72>(p, a, s);
        default: return run_sparse<128>(p, a, s);
    }
}

static size_t select_ws(int B, int H, int Tq, int Tk, int d) {
    return (size_t)B * H * (mean_size((Tq + kSparseQ - 1) / kSparseQ, d) + mean_size((Tk + kSparseK - 1) / kSparseK, d)) * sizeof(double);
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

static bool aligned(const void* p, int n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

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
    if (!aligned(lens, 4) || !aligned(blocks, 4)) return fail(BC_ERR_INVALID_ARG, "lens and blocks must be 4-byte aligned");
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(ws, 256))
        return fail(BC_ERR_INVALID_ARG, "q and k must be 16-byte, the workspace 256-byte aligned");
    const size_t need = select_ws(B, H, Tq, Tk, d);
    if (ws_bytes < need) return fail(BC_ERR_INVALID_ARG, "workspace %zu < %zu bytes", ws_bytes, need);
    SelectArgs a;
    a.q = q; a.k = k; a.lens = lens;
    a.B = B; a.H = H; a.Tq = Tq; a.Tk = Tk; a.d = d; a.keep = keep; a.keep_last = keep_last;
    a.nqb = (Tq + kSparseQ - 1) / kSparseQ;
    a.nkb = (Tk + kSparseK - 1) / kSparseK;
    a.qm = static_cast<double*>(ws);
    a.km = a.qm + B * H * mean_size(a.nqb, d);
    a.blocks = blocks;
    const int64_t means = (int64_t)B * (a.nqb + a.nkb) * ((H * d / 8 + 31) / 32), rows = (int64_t)B * H * a.nqb;
    // (The scores take workgroups of 1024 threads for 16 query blocks.)
    if (means > kMaxGrid || rows > kMaxGrid || (int64_t)B * H * ((a.nqb + 15) / 16) > kMaxGrid / 4) return fail(BC_ERR_UNSUPPORTED, "block selection grid too large");
    const int64_t nb = rows * keep * 4, e = dtype_size(dtype);
    const int64_t nq = (int64_t)B * Tq * H * d * e, nk = (int64_t)B * Tk * H * d * e, nw = (int64_t)need;
    if (overlap(blocks, nb, q, nq) || overlap(blocks, nb, k, nk) || overlap(blocks, nb, ws, nw) || overlap(blocks, nb, lens, (int64_t)B * 4) ||
        overlap(ws, nw, q, nq) || overlap(ws, nw, k, nk) || overlap(ws, nw, lens, (int64_t)B * 4))
        return fail(BC_ERR_INVALID_ARG, "blocks and the workspace must not overlap another operand");
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
    *bytes = part_bytes(sparse_plan(dtype, B, H, Tq, Tk, keep), B, H, Tq, d);
    return BC_OK;
}

int bc_attention_sparse(int B, int H, int Tq, int Tk, int d, const void* q, const void* k, const void* v,
                        const int32_t* lens, const int32_t* blocks, int keep, void* out, int prescaled, int dtype, void* ws,
                        size_t ws_bytes, void* stream) {
    clear_error();
    if (!q || !k || !v || !blocks || !out) return fail(BC_ERR_INVALID_ARG, "NULL pointer");
    const int rc = check_shape(B, H, Tq, Tk, d, keep, dtype);
    if (rc != BC_OK) return rc;
    if (prescaled && dtype != BC_BF16) return fail(BC_ERR_UNSUPPORTED, "pre-scaled queries are bf16 only");
    if (!aligned(lens, 4) || !aligned(blocks, 4) || !aligned(out, dtype_size(dtype)))
        return fail(BC_ERR_INVALID_ARG, "lens, blocks and out must be aligned to their elements");
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16)) return fail(BC_ERR_INVALID_ARG, "q, k and v must be 16-byte aligned");
    AttnArgs a = {};
    a.q_scaled = prescaled ? 1 : 0;
    a.q0 = a.q1 = q; a.Tq0 = Tq; a.ldq = (int64_t)H * d;
    a.k0 = a.k1 = k; a.Tk0 = Tk; a.ldk = (int64_t)H * d;
    a.v0 = a.v1 = v; a.ldv = (int64_t)H * d;
    a.o0 = a.o1 = out; a.ldo = (int64_t)H * d;
    a.B = B; a.H = H; a.d = d;
    a.blocks = blocks; a.keep = keep; a.lens = lens;
    a.scale_log2 = prescaled ? 1.0f : attn_q_scale(d);
    const SparsePlan plan = sparse_plan(dtype, B, H, Tq, Tk, keep);
    a.parts = plan.parts;
    const int64_t nwg = (int64_t)B * H * ((Tq + plan.tile - 1) / plan.tile) * plan.parts, rows = (int64_t)B * H * Tq;
    if (nwg > kMaxGrid || (plan.parts > 1 && rows * (d / 4) > kMaxGrid * 256))
        return fail(BC_ERR_UNSUPPORTED, "attention over blocks: grid too large");
    const int64_t no = rows * d * dtype_size(dtype), nk = (int64_t)B * Tk * H * d * dtype_size(dtype);
    const size_t need = part_bytes(plan, B, H, Tq, d);
    const int64_t nb = (int64_t)B * H * ((Tq + kSparseQ - 1) / kSparseQ) * keep * 4, nl = (int64_t)B * 4, nw = (int64_t)need;
    if (overlap(out, no, q, no) || overlap(out, no, k, nk) || overlap(out, no, v, nk) || overlap(out, no, blocks, nb) || overlap(out, no, lens, nl) ||
        (need && (overlap(ws, nw, out, no) || overlap(ws, nw, q, no) || overlap(ws, nw, k, nk) || overlap(ws, nw, v, nk) ||
                  overlap(ws, nw, blocks, nb) || overlap(ws, nw, lens, nl))))
        return fail(BC_ERR_INVALID_ARG, "the output and the workspace must not overlap another operand");
    if (need) {
        if (!ws || reinterpret_cast<uintptr_t>(ws) % 256) return fail(BC_ERR_INVALID_ARG, "a 256-byte aligned workspace is needed");
        if (ws_bytes < need) return fail(BC_ERR_INVALID_ARG, "workspace %zu < %zu bytes", ws_bytes, need);
        a.part_o = static_cast<float*>(ws);
        a.part_ml = a.part_o + (int64_t)B * Tq * H * a.parts * d;
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    prof_begin(PROF_ATTENTION, s, 4.0 * B * H * Tq * std::min((double)keep * kSparseK, (double)Tk) * d);
    const int ran = launch_sparse_attention(dtype, plan, a, s);
    prof_end(PROF_ATTENTION, s);
    return ran;
}

}  // extern "C"
