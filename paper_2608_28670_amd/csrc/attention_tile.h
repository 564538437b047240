// Pieces that the attention kernels share: operand shapes, the LDS layout of a
// key or value tile, reductions over a query's lanes, lists of key blocks.
#pragma once

#include "attention.h"

namespace bc {

constexpr int kKTile = 64;   // keys per step

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

template <typename T, int HD> struct AttnShape {
    // K dimension of Q K^T: bf16 uses 32-wide MFMA steps, the last one padded
    // with zero Q columns (a 16-wide 16x16x16 tail step was dropped: in one
    // schedule its accumulator was read back before the MFMA had written
    // it); fp32 uses 4-wide steps.
    static constexpr int n32x = sizeof(T) == 2 ? (HD + 31) / 32 : 0;   // 32-wide steps
    static constexpr int DK = sizeof(T) == 2 ? 32 * n32x : HD;
    static constexpr int DV = (HD + 15) / 16 * 16;           // rows of O^T
    static constexpr int EPC = 16 / (int)sizeof(T);          // elements per 16-byte chunk
    static constexpr int CPR = HD / EPC;                     // chunks per head row
    static constexpr int KPAD = EPC;                         // LDS row padding (elements)
};

// A key or value tile in LDS: row-major, head_dim contiguous; rows of 128 or
// 256 bytes are XOR-swizzled by 16-byte chunk.
template <int HD> struct KvLayout {
    static constexpr int CPR = HD / 8;                       // 16-byte chunks per row
    static constexpr int RPB = (HD * 2) >= 256 ? 1 : 256 / (HD * 2);   // rows per 256 bytes
    static constexpr bool SWZ = (CPR & (CPR - 1)) == 0;      // power-of-two rows are swizzled
    __device__ static int slot(int row, int chunk) { return SWZ ? chunk ^ ((row / RPB) % CPR) : chunk; }
    // element offset of (row, column d) in a tile
    __device__ static int at(int row, int d) { return row * HD + slot(row, d >> 3) * 8 + (d & 7); }
};

// Reductions over the four lanes l, l ^ 16, l ^ 32, l ^ 48 that hold one
// query's scores: with both operands equal, v_permlane16_swap returns the
// value of lane l in one result and of lane l ^ 16 in the other (likewise
// v_permlane32_swap for l ^ 32), so no LDS round trip is needed.
// Maximum without the NaN-quieting canonicalisation that fmaxf's IEEE
// semantics add per operand (gfx950 has a native three-input form); scores
// are finite or -inf.
__device__ __forceinline__ float vmax(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float group_max(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = vmax(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return vmax(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float group_sum(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

static_assert(kKTile == kSparseK, "a key tile is a key block");

// A sample's keys: lens[b], held to [0, Tk]; without lens all Tk.
__device__ __forceinline__ int sparse_keys(const AttnArgs& a, int b) {
    return a.lens ? min(max(a.lens[b], 0), a.Tk0) : a.Tk0;
}
// Entries of a list before its end (see attention.h); the same in every lane.
__device__ __forceinline__ int sparse_list_length(const int* list, int keep, int nkb, int lane) {
    for (int base = 0; base < keep; base += 256) {      // the loads of four rounds go out together
        int v[4], before[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int i = base + 64 * u + lane;
            v[u] = i < keep ? list[i] : -1;
            before[u] = i > 0 && i < keep ? list[i - 1] : -1;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const uint64_t bad = ~__ballot(v[u] > before[u] && v[u] >= 0 && v[u] < nkb);
            if (bad) return base + 64 * u + __builtin_ctzll(bad);
        }
    }
    return keep;
}
// A list's entries through the scalar cache (a vector load would have to be
// waited for among the direct-to-LDS loads).
typedef const __attribute__((address_space(4))) int const_int;

}  // namespace bc
