// The key-value cache in 8 bits: pushing tokens, reading them back, attention over it.
//
// A cache holds [B][H][tiles] tiles of 64 tokens.  A tile's keys and its values have
// a power of two each as scale, s = the least one from 2^-100 up with max|x| <= 448 s,
// and codes x / s in e4m3 (four significant bits from 2^-6 up, multiples of 2^-9 below,
// to nearest, ties to even).  A power of two divides exactly: the codes are those of
// the definition in any arithmetic, a code times its scale is a bf16 value, and a scale
// that grows with later tokens moves the codes that stand without rounding them again,
// but for those that fall below 2^-6.  What is not finite is held as NaN.
//
// Codes stand in the order in which the attention's matrix instructions take them, in
// units of 16 bytes:
//   keys:   unit (jp CPR + c) 16 + l, jp = 0, 1, c < CPR = d / 8, l < 16: columns 8c..8c+7
//           of key 32 jp + l, then of key 32 jp + 16 + l;
//   values: unit 64 i + g w + l of column 16 i + l (w = 16, or 8 in the last group where
//           d % 16 = 8), g < 4: keys 4 g + 0..3 of each of the tile's four sixteens.
// [codes, tile after tile: keys, values][scales, two a tile], 2 + 1 / 8 d bytes a token and column pair.
#include <algorithm>

#include "score_kernels.h"

namespace bc {

struct PushArgs {
    const void *k, *v;
    int64_t k_batch, k_row, v_batch, v_row;
    int B, H, T, capacity, tiles, most;         // most: tiles that a sample's tokens may touch
    const int *lens, *counts;
    uint8_t* codes;
    float* scales;
};

constexpr float kMinKvScale = 0x1p-100f;

__device__ __forceinline__ float finite_abs(float x) {
    const float y = fabsf(x);
    return y < INFINITY ? y : 0.f;
}
// The least power of two from 2^-100 up that holds `top`: 448 is 1.75 * 2^8.
__device__ __forceinline__ float kv_scale(float top) {
    const int e = (int)((__float_as_uint(top) + 0x1fffffu) >> 23) - 8;
    return __uint_as_float((unsigned)max(e, 27) << 23);
}
// Codes of four values (times the scale's inverse).
__device__ __forceinline__ unsigned encode4(const float (&x)[4], float inv) {
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = fabsf(x[i]) < INFINITY ? x[i] * inv : __builtin_nanf("");
    unsigned c = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], c, true);
}
// Codes at a scale 1 / down times as large.
__device__ __forceinline__ unsigned rescale4(unsigned c, float down) {
    float f[4];
    decode4(c, 1.f, f);
    return encode4(f, down);
}

// A workgroup a tile: the new tokens' keys and values into registers, their largest
// magnitudes, the scales, the codes.  A tile's first token starts its scale afresh and
// clears the tokens behind; a tile that holds tokens already keeps at least its scale,
// and a larger one moves their codes.
//   Bound by the bytes of the tokens.  A whole tile's codes meet in LDS and leave 16
// consecutive bytes a lane (14 310 tokens of 24 x 128 columns, 264 MB: 101 us with a store
// for every 8 codes of a key and 4 of a column, each lane's 128 or 256 bytes from the next).
// Unit u stands at u ^ (u / 16 mod 16), which spreads the units that a wave writes over the banks.
// The tokens are read once and pass by the caches (49 us, 55 without).
template <typename T_, int HD>
__global__ __launch_bounds__(256) void kv_push_kernel(PushArgs a) {
    typedef elem_t<T_> T;
    constexpr int CPR = HD / 8, KPER = (64 * CPR + 255) / 256, VPER = (16 * CPR + 255) / 256, W = sizeof(T) / 2;
    __shared__ float red[2][4];
    __shared__ u32x4 tile_codes[8 * HD];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int h = blockIdx.x % a.H, i = blockIdx.x / a.H % a.most, b = blockIdx.x / a.H / a.most;
    const int n = min(max(a.lens[b], 0), a.capacity), count = a.counts ? min(max(a.counts[b], 0), a.T) : a.T;
    const int first = n - count, tile = max(first, 0) / 64 + i, t0 = tile * 64;
    if (t0 >= n || count == 0) return;
    const int r0 = max(first - t0, 0), r1 = min(n - t0, 64);         // the tile's rows that are written
    const int64_t ct = ((int64_t)b * a.H + h) * a.tiles + tile;
    uint8_t* ck = a.codes + ct * (128 * HD);
    uint8_t* cv = ck + 64 * HD;
    const T* kb = static_cast<const T*>(a.k) + b * a.k_batch + (int64_t)(t0 - first) * a.k_row + h * HD;
    const T* vb = static_cast<const T*>(a.v) + b * a.v_batch + (int64_t)(t0 - first) * a.v_row + h * HD;
    u32x4 xk[KPER][W], xv[VPER][4][W];
    float top[2] = {0.f, 0.f};
    auto widen = [&](const u32x4 (&x)[W], float (&f)[8]) {
#pragma unroll
        for (int w = 0; w < W; ++w) unpack(x[w], f + 8 / W * w, (const T*)nullptr);
    };
#pragma unroll
    for (int x = 0; x < KPER; ++x) {
        const int u = tid + 256 * x, row = u / CPR, ch = u % CPR;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            xk[x][w] = u32x4{0u, 0u, 0u, 0u};
            if (row >= r0 && row < r1) xk[x][w] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(kb + row * a.k_row + 8 * ch) + w);
        }
    }
#pragma unroll
    for (int x = 0; x < VPER; ++x) {
        const int u = tid + 256 * x, rows = u / CPR * 4, ch = u % CPR;
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int w = 0; w < W; ++w) {
                xv[x][q][w] = u32x4{0u, 0u, 0u, 0u};
                if (rows + q >= r0 && rows + q < r1) xv[x][q][w] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(vb + (rows + q) * a.v_row + 8 * ch) + w);
            }
    }
    float f[8];
#pragma unroll
    for (int x = 0; x < KPER; ++x) {
        widen(xk[x], f);
#pragma unroll
        for (int e = 0; e < 8; ++e) top[0] = fmaxf(top[0], finite_abs(f[e]));
    }
#pragma unroll
    for (int x = 0; x < VPER; ++x)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            widen(xv[x][q], f);
#pragma unroll
            for (int e = 0; e < 8; ++e) top[1] = fmaxf(top[1], finite_abs(f[e]));
        }
#pragma unroll
    for (int z = 0; z < 2; ++z) {
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) top[z] = fmaxf(top[z], __shfl_xor(top[z], s));
        if (lane == 0) red[z][wave] = top[z];
    }
    __syncthreads();
    float scale[2], down[2];
#pragma unroll
    for (int z = 0; z < 2; ++z) {
        scale[z] = kv_scale(fmaxf(fmaxf(red[z][0], red[z][1]), fmaxf(red[z][2], red[z][3])));
        down[z] = 1.f;
        if (r0 > 0) {
            const float old = a.scales[2 * ct + z];
            const unsigned ob = __float_as_uint(old);
            // (Anything else than a scale: nothing was pushed there; what it held means nothing.)
            if ((ob & 0x807fffffu) == 0u && old >= kMinKvScale && old <= 0x1p120f) {
                scale[z] = fmaxf(scale[z], old);
                down[z] = old / scale[z];
            }
        }
    }
    __syncthreads();       // every wave has read the old scales
    if (tid < 2) a.scales[2 * ct + tid] = scale[tid];
    const float ik = 1.f / scale[0], iv = 1.f / scale[1];
    if (r0 == 0) {
        auto place = [](int unit, int byte) { return (unit ^ ((unit >> 4) & 15)) * 16 + byte; };
        char* codes = reinterpret_cast<char*>(tile_codes);
#pragma unroll
        for (int x = 0; x < KPER; ++x) {
            const int u = tid + 256 * x, row = u / CPR, ch = u % CPR;
            if (64 * CPR % 256 != 0 && row >= 64) break;
            widen(xk[x], f);
            const float lo[4] = {f[0], f[1], f[2], f[3]}, hi[4] = {f[4], f[5], f[6], f[7]};
            *reinterpret_cast<u32x2*>(codes + place(((row >> 5) * CPR + ch) * 16 + (row & 15), 8 * ((row >> 4) & 1))) = u32x2{encode4(lo, ik), encode4(hi, ik)};
        }
#pragma unroll
        for (int x = 0; x < VPER; ++x) {
            const int u = tid + 256 * x, rows = u / CPR * 4, ch = u % CPR;
            if (16 * CPR % 256 != 0 && rows >= 64) break;
            float fq[4][8];
#pragma unroll
            for (int q = 0; q < 4; ++q) widen(xv[x][q], fq[q]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int col = 8 * ch + e, ci = col >> 4, w = min(16, HD - 16 * ci);
                const float y[4] = {fq[0][e], fq[1][e], fq[2][e], fq[3][e]};
                *reinterpret_cast<unsigned*>(codes + place(4 * HD + 64 * ci + ((rows >> 2) & 3) * w + (col & 15), 4 * (rows >> 4))) = encode4(y, iv);
            }
        }
        __syncthreads();
        for (int u = tid; u < 8 * HD; u += 256) reinterpret_cast<u32x4*>(ck)[u] = tile_codes[u ^ ((u >> 4) & 15)];
        return;
    }
    // A tile that holds tokens: the new rows' bytes, and where a scale has grown the held ones' too.
#pragma unroll
    for (int x = 0; x < KPER; ++x) {
        const int u = tid + 256 * x, row = u / CPR, ch = u % CPR;
        if (64 * CPR % 256 != 0 && row >= 64) break;
        u32x2* to = reinterpret_cast<u32x2*>(ck + (((row >> 5) * CPR + ch) * 16 + (row & 15)) * 16 + 8 * ((row >> 4) & 1));
        if (row >= r0 && row < r1) {
            widen(xk[x], f);
            const float lo[4] = {f[0], f[1], f[2], f[3]}, hi[4] = {f[4], f[5], f[6], f[7]};
            *to = u32x2{encode4(lo, ik), encode4(hi, ik)};
        } else if (row < r0 && down[0] != 1.f) {
            const u32x2 c = *to;
            *to = u32x2{rescale4(c.x, down[0]), rescale4(c.y, down[0])};
        }
    }
#pragma unroll
    for (int x = 0; x < VPER; ++x) {
        const int u = tid + 256 * x, rows = u / CPR * 4, ch = u % CPR;
        if (16 * CPR % 256 != 0 && rows >= 64) break;
        const bool some = rows < r1 && rows + 4 > r0, held = rows < r0;
        if (!some && !(held && down[1] != 1.f)) continue;
        float fq[4][8];
#pragma unroll
        for (int q = 0; q < 4; ++q) widen(xv[x][q], fq[q]);
        unsigned fresh = 0u, kept = 0u;              // bytes of the word that are new, and that are held
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (rows + q >= r0 && rows + q < r1) fresh |= 0xffu << (8 * q);
            if (rows + q < r0) kept |= 0xffu << (8 * q);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int col = 8 * ch + e, ci = col >> 4, w = min(16, HD - 16 * ci);
            unsigned* to = reinterpret_cast<unsigned*>(cv + (64 * ci + ((rows >> 2) & 3) * w + (col & 15)) * 16 + 4 * (rows >> 4));
            const float y[4] = {fq[0][e], fq[1][e], fq[2][e], fq[3][e]};
            unsigned c = encode4(y, iv) & fresh;
            if (fresh != 0xffffffffu) {
                const unsigned old = *to;
                c |= (down[1] != 1.f ? rescale4(old, down[1]) : old) & kept;
                c |= old & ~(fresh | kept);
            }
            *to = c;
        }
    }
}

struct ReadArgs {
    int B, H, first, n, capacity, tiles, most;
    const int* lens;
    const uint8_t* codes;
    const float* scales;
    void *k, *v;              // [B, n, H, d]
};

// Tokens first..first + n - 1 as values, zeros behind a sample's last; a workgroup a
// tile, whose codes come through LDS, swizzled as in the push (14 310 tokens of 24 x 128
// columns: 40 us, 51 with the codes read where they lie).  Bound by the outputs' bytes,
// which pass by the caches (8 samples of 8 x 128 columns, 1000 tokens: 7.4 us against 9.7).
template <typename T_, int HD>
__global__ __launch_bounds__(256) void kv_read_kernel(ReadArgs a) {
    typedef elem_t<T_> T;
    typedef unsigned int loose __attribute__((ext_vector_type(4), aligned(2)));     // the outputs are aligned to their elements
    constexpr int CPR = HD / 8;
    __shared__ u32x4 tile_codes[8 * HD];
    const int tid = threadIdx.x;
    const int h = blockIdx.x % a.H, i = blockIdx.x / a.H % a.most, b = blockIdx.x / a.H / a.most;
    const int tile = a.first / 64 + i, t0 = tile * 64;
    const int n = min(max(a.lens[b], 0), a.capacity);
    const int64_t ct = ((int64_t)b * a.H + h) * a.tiles + tile;
    const u32x4* codes = reinterpret_cast<const u32x4*>(a.codes + ct * (128 * HD));
    const bool some = t0 < n;
    const float ks = some ? a.scales[2 * ct] : 0.f, vs = some ? a.scales[2 * ct + 1] : 0.f;
    if (some)
        for (int u = tid; u < 8 * HD; u += 256) tile_codes[u ^ ((u >> 4) & 15)] = codes[u];
    __syncthreads();
    auto at = [&](int unit, int byte) { return reinterpret_cast<const char*>(tile_codes) + (unit ^ ((unit >> 4) & 15)) * 16 + byte; };
    auto put = [&](void* to, int row, int col, const float (&f)[8]) {
        const int t = t0 + row - a.first;
        if (t < 0 || t >= a.n) return;
        T* o = static_cast<T*>(to) + (((int64_t)b * a.n + t) * a.H + h) * HD + col;
        T v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (T)(t0 + row < n ? f[e] : 0.f);
        loose p[sizeof v / 16];
        __builtin_memcpy(p, v, sizeof v);
#pragma unroll
        for (unsigned w = 0; w < sizeof v / 16; ++w) __builtin_nontemporal_store(p[w], reinterpret_cast<loose*>(o) + w);
    };
    for (int u = tid; u < 64 * CPR; u += 256) {
        const int row = u / CPR, ch = u % CPR;
        float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (some) {
            const u32x2 c = *reinterpret_cast<const u32x2*>(at(((row >> 5) * CPR + ch) * 16 + (row & 15), 8 * ((row >> 4) & 1)));
            float lo[4], hi[4];
            decode4(c.x, ks, lo);
            decode4(c.y, ks, hi);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                f[e] = lo[e];
                f[4 + e] = hi[e];
            }
        }
        put(a.k, row, 8 * ch, f);
    }
    for (int u = tid; u < 16 * CPR; u += 256) {
        const int rows = u / CPR * 4, ch = u % CPR;
        float f[4][8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int col = 8 * ch + e, ci = col >> 4, w = min(16, HD - 16 * ci);
            float x[4] = {0.f, 0.f, 0.f, 0.f};
            if (some) decode4(*reinterpret_cast<const unsigned*>(at(4 * HD + 64 * ci + ((rows >> 2) & 3) * w + (col & 15), 4 * (rows >> 4))), vs, x);
#pragma unroll
            for (int q = 0; q < 4; ++q) f[q][e] = x[q];
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) put(a.v, rows + q, 8 * ch, f[q]);
    }
}

static int64_t cache_tiles(int capacity) { return (capacity + 63) / 64; }
static int64_t code_bytes(const bc_kv_cache& c) { return (int64_t)c.B * c.H * cache_tiles(c.capacity) * 128 * c.d; }
static int64_t cache_bytes(const bc_kv_cache& c) { return code_bytes(c) + (int64_t)c.B * c.H * cache_tiles(c.capacity) * 8; }

static int check_cache(const bc_kv_cache* c, bool storage) {
    if (!c) return fail(BC_ERR_INVALID_ARG, "NULL pointer");
    if (c->B < 1 || c->H < 1 || c->capacity < 1 || c->d < 1) return fail(BC_ERR_INVALID_ARG, "empty cache");
    if (!attention_supported(c->d)) return fail(BC_ERR_UNSUPPORTED, "head_dim %d (supported: 32, 64, 72, 128)", c->d);
    if (c->capacity > kMaxPosition - 64 || (int64_t)c->B * c->H > (1 << 20) || (int64_t)c->H * c->d > (1 << 24) ||
        (int64_t)c->B * c->capacity > 0x7fffffff)
        return fail(BC_ERR_UNSUPPORTED, "cache of %d x %d heads, %d tokens", c->B, c->H, c->capacity);
    if (storage && (!c->storage || reinterpret_cast<uintptr_t>(c->storage) % 256))
        return fail(BC_ERR_INVALID_ARG, "the cache's storage must be 256-byte aligned");
    return BC_OK;
}

#define BC_KV_CASE(KERNEL, HD)                                                                      \
    case HD:                                                                                        \
        if (dtype == BC_BF16) launch_k(KERNEL<bf16_tag, HD>, grid, dim3(256), s, a);                \
        else launch_k(KERNEL<float, HD>, grid, dim3(256), s, a);                                    \
        break;

}  // namespace bc

using namespace bc;

extern "C" {

int bc_kv_cache_size(int B, int H, int d, int capacity, size_t* bytes) {
    clear_error();
    if (!bytes) return fail(BC_ERR_INVALID_ARG, "NULL pointer");
    const bc_kv_cache c = {B, H, d, capacity, nullptr};
    const int rc = check_cache(&c, false);
    if (rc != BC_OK) return rc;
    *bytes = (size_t)cache_bytes(c);
    return BC_OK;
}

int bc_kv_push(const bc_kv_cache* c, int T, const void* k, int64_t k_batch, int64_t k_row, const void* v, int64_t v_batch, int64_t v_row,
               const int32_t* lens, const int32_t* counts, int dtype, void* stream) {
    clear_error();
    int rc = check_cache(c, true);
    if (rc != BC_OK) return rc;
    if (T < 1 || T > kMaxPosition) return fail(BC_ERR_INVALID_ARG, "%d tokens", T);
    if (dtype != BC_F32 && dtype != BC_BF16) return fail(BC_ERR_INVALID_ARG, "dtype %d", dtype);
    if (!lens || (reinterpret_cast<uintptr_t>(lens) | reinterpret_cast<uintptr_t>(counts)) % 4)
        return fail(BC_ERR_INVALID_ARG, "lens (needed) and counts must be 4-byte aligned");
    Span in[4], out[1] = {{c->storage, cache_bytes(*c)}};
    if ((rc = score_operand("k", k, k_batch, k_row, c->B, T, (int64_t)c->H * c->d, dtype, &in[0])) != BC_OK ||
        (rc = score_operand("v", v, v_batch, v_row, c->B, T, (int64_t)c->H * c->d, dtype, &in[1])) != BC_OK)
        return rc;
    in[2] = {lens, (int64_t)c->B * 4};
    in[3] = {counts, (int64_t)c->B * 4};
    if ((rc = score_apart(out, 1, in, 4)) != BC_OK) return rc;
    PushArgs a = {};
    a.k = k; a.v = v; a.k_batch = k_batch; a.k_row = k_row; a.v_batch = v_batch; a.v_row = v_row;
    a.B = c->B; a.H = c->H; a.T = T; a.capacity = c->capacity; a.tiles = (int)cache_tiles(c->capacity);
    a.most = (int)std::min<int64_t>(a.tiles, ((int64_t)T + 62) / 64 + 1);
    a.lens = lens; a.counts = counts;
    a.codes = static_cast<uint8_t*>(c->storage);
    a.scales = reinterpret_cast<float*>(a.codes + code_bytes(*c));
    const int64_t wgs = (int64_t)c->B * c->H * a.most;
    if (wgs > kMaxGrid) return fail(BC_ERR_UNSUPPORTED, "push grid too large");
    const dim3 grid((unsigned)wgs);
    hipStream_t s = static_cast<hipStream_t>(stream);
    prof_begin(PROF_COPY, s, 2.0 * c->B * c->H * (double)T * c->d * (dtype_size(dtype) + 1));
    switch (c->d) {
        BC_KV_CASE(kv_push_kernel, 32) BC_KV_CASE(kv_push_kernel, 64) BC_KV_CASE(kv_push_kernel, 72) BC_KV_CASE(kv_push_kernel, 128)
    }
    prof_end(PROF_COPY, s);
    return check_launch("push into the cache");
}

int bc_kv_read(const bc_kv_cache* c, int first, int n, const int32_t* lens, void* k_out, void* v_out, int dtype, void* stream) {
    clear_error();
    int rc = check_cache(c, true);
    if (rc != BC_OK) return rc;
    if (dtype != BC_F32 && dtype != BC_BF16) return fail(BC_ERR_INVALID_ARG, "dtype %d", dtype);
    if (first < 0 || n < 1 || first > c->capacity - n) return fail(BC_ERR_INVALID_ARG, "tokens %d + %d of %d", first, n, c->capacity);
    const int e = dtype_size(dtype);
    if (!k_out || !v_out || (reinterpret_cast<uintptr_t>(k_out) | reinterpret_cast<uintptr_t>(v_out)) % e)
        return fail(BC_ERR_INVALID_ARG, "outputs: NULL or not aligned to their elements");
    if (!lens || reinterpret_cast<uintptr_t>(lens) % 4) return fail(BC_ERR_INVALID_ARG, "lens: NULL or not 4-byte aligned");
    const int64_t bytes = (int64_t)c->B * n * c->H * c->d * e;
    const Span out[2] = {{k_out, bytes}, {v_out, bytes}}, in[2] = {{c->storage, cache_bytes(*c)}, {lens, (int64_t)c->B * 4}};
    if ((rc = score_apart(out, 2, in, 2)) != BC_OK) return rc;
    ReadArgs a = {};
    a.B = c->B; a.H = c->H; a.first = first; a.n = n; a.capacity = c->capacity; a.tiles = (int)cache_tiles(c->capacity);
    a.most = (first + n - 1) / 64 - first / 64 + 1;
    a.lens = lens;
    a.codes = static_cast<const uint8_t*>(c->storage);
    a.scales = reinterpret_cast<const float*>(a.codes + code_bytes(*c));
    a.k = k_out; a.v = v_out;
    const int64_t wgs = (int64_t)c->B * c->H * a.most;
    if (wgs > kMaxGrid) return fail(BC_ERR_UNSUPPORTED, "read grid too large");
    const dim3 grid((unsigned)wgs);
    hipStream_t s = static_cast<hipStream_t>(stream);
    prof_begin(PROF_COPY, s, (double)bytes * 2.0 * (e + 1) / e);
    switch (c->d) {
        BC_KV_CASE(kv_read_kernel, 32) BC_KV_CASE(kv_read_kernel, 64) BC_KV_CASE(kv_read_kernel, 72) BC_KV_CASE(kv_read_kernel, 128)
    }
    prof_end(PROF_COPY, s);
    return check_launch("read of the cache");
}

int bc_kv_attention_workspace_size(const bc_kv_cache* c, int Hq, int Tq, int dtype, size_t* bytes) {
    clear_error();
    if (!bytes) return fail(BC_ERR_INVALID_ARG, "NULL pointer");
    int rc = check_cache(c, false);
    if (rc == BC_OK) rc = score_shape(c->B, Hq, c->H, Tq, c->capacity, c->d, dtype);
    if (rc != BC_OK) return rc;
    *bytes = score_part_bytes(score_plan(dtype, c->B, c->H, (int64_t)Tq * (Hq / c->H), c->capacity, c->d), c->B, Hq, Tq, c->d);
    return BC_OK;
}

int bc_kv_attention(const bc_kv_cache* c, int Hq, int Tq, const void* q, int64_t q_batch, int64_t q_row, const int32_t* lens,
                    const int32_t* counts, const bc_score_opts* opts, void* out, int dtype, void* ws, size_t ws_bytes, void* stream) {
    clear_error();
    int rc = check_cache(c, true);
    if (rc == BC_OK) rc = score_shape(c->B, Hq, c->H, Tq, c->capacity, c->d, dtype);
    if (rc != BC_OK) return rc;
    ScoreArgs a = {};
    Span in[6], to[2];
    if ((rc = score_operand("q", q, q_batch, q_row, c->B, Tq, (int64_t)Hq * c->d, dtype, &in[0])) != BC_OK ||
        (rc = score_options(opts, c->d, &a)) != BC_OK)
        return rc;
    if (!out || reinterpret_cast<uintptr_t>(out) % dtype_size(dtype)) return fail(BC_ERR_INVALID_ARG, "out: NULL or not aligned to its elements");
    if (!lens || (reinterpret_cast<uintptr_t>(lens) | reinterpret_cast<uintptr_t>(counts)) % 4)
        return fail(BC_ERR_INVALID_ARG, "lens (needed) and counts must be 4-byte aligned");
    a.q = q; a.q_batch = q_batch; a.q_row = q_row; a.out = out;
    a.B = c->B; a.Hk = c->H; a.G = Hq / c->H; a.Tq = Tq; a.Tk = c->capacity; a.d = c->d;
    a.lens = lens; a.counts = counts;
    a.tiles = (int)cache_tiles(c->capacity);
    a.codes = static_cast<const uint8_t*>(c->storage);
    a.scales = reinterpret_cast<const float*>(a.codes + code_bytes(*c));
    const ScorePlan plan = score_plan(dtype, c->B, c->H, (int64_t)Tq * a.G, c->capacity, c->d);
    a.parts = plan.parts;
    a.nt = plan.rows == 16 && code_bytes(*c) >= 80e6;
    if ((rc = score_grid(plan, a)) != BC_OK) return rc;
    const size_t need = score_part_bytes(plan, c->B, Hq, Tq, c->d);
    if (need) {
        if (!ws || reinterpret_cast<uintptr_t>(ws) % 256) return fail(BC_ERR_INVALID_ARG, "a 256-byte aligned workspace is needed");
        if (ws_bytes < need) return fail(BC_ERR_INVALID_ARG, "workspace %zu < %zu bytes", ws_bytes, need);
        a.part_o = static_cast<float*>(ws);
        a.part_ml = a.part_o + (int64_t)c->B * Tq * Hq * a.parts * c->d;
    }
    to[0] = {out, (int64_t)c->B * Tq * Hq * c->d * dtype_size(dtype)};
    to[1] = {ws, (int64_t)need};
    in[1] = {c->storage, cache_bytes(*c)};
    in[2] = {lens, (int64_t)c->B * 4};
    in[3] = {counts, (int64_t)c->B * 4};
    in[4] = {a.slopes, (int64_t)Hq * 4};
    in[5] = {a.prefix, (int64_t)c->B * 4};
    if ((rc = score_apart(to, need ? 2 : 1, in, 6)) != BC_OK) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    prof_begin(PROF_ATTENTION, s, 4.0 * c->B * Hq * (double)Tq * c->capacity * c->d);
    rc = launch_score<true>(dtype, plan, a, s);
    if (rc == BC_OK && plan.parts > 1) rc = score_join(dtype, a, s);
    prof_end(PROF_ATTENTION, s);
    return rc;
}

}  // extern "C"
