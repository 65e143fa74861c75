// Shared by the attention kernels of crossattn.hip (forward) and
// crossattn_backward.hip: arguments, tiles in LDS and matrix fragments.
//
// Everything is built from 32 x 32 products whose operands are held as
// "fragments" of 16 reduction indices: lane l holds 8 values of row (A) or
// column (B) l % 32, the half hi = l / 32 the second eight.  One
// v_mfma_f32_32x32x16_bf16 consumes a bf16 fragment pair, eight
// v_mfma_f32_32x32x2_f32 an fp32 pair (any pairing of reduction indices with
// steps is right as long as A and B agree: step e takes value e of each half).
// The result's layout does not depend on the type: column l % 32, register
// 4 a + e holds row 8 a + 4 hi + e.
//
// A tile is KC rows (keys, or queries in the key-owned backward) of DP
// channels, row-major.  The row that stands for product row 8 a + 4 h + e of
// the b-th 32-row product is (KC / 2) h + 16 b + 4 a + e, so that a lane's KC / 2
// results belong to consecutive rows: their bias values are contiguous, and
// the eight that feed one step of the next product are as well.
#pragma once

#include "common.h"
#include "kernels.h"

#include <type_traits>

namespace trimul {

__device__ __forceinline__ float xor32(float v) { return __shfl_xor(v, 32); }

// ds_read_b64_tr_b16: in each 16-lane group g, lane 16 g + 4 a + b receives
// element b of the 8-byte chunks addressed by lanes 16 g + a, + 4, + 8, + 12.
typedef short v4i16_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint2 lds_tr4(const void* p) {
    typedef __attribute__((address_space(3))) v4i16_t lds_v4i16_t;
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_t*)(p)));
}

template <typename T> struct Frag;
template <> struct Frag<bf16_t> {
    uint4 u;
    __device__ __forceinline__ void zero() { u = make_uint4(0, 0, 0, 0); }
    // sum of the products of the two fragments' own values
    static __device__ __forceinline__ float dot(const Frag& x, const Frag& y) {
        const uint32_t a[4] = {x.u.x, x.u.y, x.u.z, x.u.w}, b[4] = {y.u.x, y.u.y, y.u.z, y.u.w};
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s = __builtin_fmaf(__uint_as_float(a[i] << 16), __uint_as_float(b[i] << 16), s);
            s = __builtin_fmaf(__uint_as_float(a[i] & 0xffff0000u), __uint_as_float(b[i] & 0xffff0000u), s);
        }
        return s;
    }
};
template <> struct Frag<float> {
    float v[8];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.f;
    }
    static __device__ __forceinline__ float dot(const Frag& x, const Frag& y) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s = __builtin_fmaf(x.v[i], y.v[i], s);
        return s;
    }
};

__device__ __forceinline__ f32x16_t mma(const Frag<bf16_t>& a, const Frag<bf16_t>& b, f32x16_t c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a.u), __builtin_bit_cast(bf16x8_t, b.u),
                                                   c, 0, 0, 0);
}
__device__ __forceinline__ f32x16_t mma(const Frag<float>& a, const Frag<float>& b, f32x16_t c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[e], b.v[e], c, 0, 0, 0);
    return c;
}

// Registers 8 t .. 8 t + 7 of a result as the fragment of the next product
// (rounded to nearest for bf16).
__device__ __forceinline__ void take8(const f32x16_t& s, int t, Frag<bf16_t>& f) {
    f.u = make_uint4(pack_bf16x2(s[8 * t], s[8 * t + 1]), pack_bf16x2(s[8 * t + 2], s[8 * t + 3]),
                     pack_bf16x2(s[8 * t + 4], s[8 * t + 5]), pack_bf16x2(s[8 * t + 6], s[8 * t + 7]));
}
__device__ __forceinline__ void take8(const f32x16_t& s, int t, Frag<float>& f) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f.v[e] = s[8 * t + e];
}

// A fragment of one token's channels straight from memory: values 16 s2 + 8 hi
// .. + 7 of a row of d channels (zero past d).
__device__ __forceinline__ void load_row(const bf16_t* row, int s2, int hi, int d, Frag<bf16_t>& f) {
    const int c = 16 * s2 + 8 * hi;
    f.u = *reinterpret_cast<const uint4*>(row + (c < d ? c : 0));
    if (c >= d) f.zero();
}
__device__ __forceinline__ void load_row(const float* row, int s2, int hi, int d, Frag<float>& f) {
    const int c = 16 * s2 + 8 * hi;
    const float4* p = reinterpret_cast<const float4*>(row + (c < d ? c : 0));
    const float4 x = p[0], y = p[1];
    const float v[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) f.v[e] = c < d ? v[e] : 0.f;
}

template <typename T, int DP, int KC>
struct Tile {
    static constexpr int kRowBytes = DP * (int)sizeof(T);
    static constexpr int kPieces = kRowBytes / 16;             // 16-byte pieces of a row
    static constexpr int kPer = 16 / (int)sizeof(T);           // values of a piece
    static constexpr int kBytes = KC * kRowBytes;

    // Byte offset of a piece.  Pieces are XOR-swizzled so that both kinds of
    // read are free of bank conflicts: the 16 rows (4 consecutive ones at four
    // distances) whose same piece a row read takes at a time, and the 64-byte
    // spans of four consecutive rows of a transposing read.
    static __device__ __forceinline__ uint32_t off(int row, int piece) {
        const int g = ((row >> 2) & 1) | (row >= KC / 2 ? 2 : 0);
        const int z = kPieces >= 16 ? (row & 3) << 2 : kPieces == 8 ? ((row >> 1) & 1) << 2 : 0;
        return (uint32_t)(row * kRowBytes + ((piece ^ z ^ g) << 4));
    }
    // The row of this lane's product row (A operand) in the b-th product.
    static __device__ __forceinline__ int row_of(int lane, int b) {
        const int l = lane & 31;
        return (KC / 2) * ((l >> 2) & 1) + 16 * b + 4 * (l >> 3) + (l & 3);
    }
    // A operand: rows of the b-th product, channels 16 s2 ..
    static __device__ __forceinline__ void rows(const char* t, int lane, int b, int s2, Frag<bf16_t>& f) {
        f.u = *reinterpret_cast<const uint4*>(t + off(row_of(lane, b), 2 * s2 + (lane >> 5)));
    }
    static __device__ __forceinline__ void rows(const char* t, int lane, int b, int s2, Frag<float>& f) {
        const int r = row_of(lane, b), p = 4 * s2 + 2 * (lane >> 5);
        const float4 x = *reinterpret_cast<const float4*>(t + off(r, p));
        const float4 y = *reinterpret_cast<const float4*>(t + off(r, p + 1));
        const float v[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) f.v[e] = v[e];
    }
    // A operand, transposed: channels 32 db + lane % 32, reduction over the tile rows that
    // registers 8 t .. of the b-th product stand for.
    static __device__ __forceinline__ void cols(const char* t, int lane, int b, int tt, int db, Frag<bf16_t>& f) {
        const int r = (KC / 2) * (lane >> 5) + 16 * b + 8 * tt + ((lane >> 2) & 3);
        const int p = 4 * db + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1), s = (lane & 1) * 8;
        const uint2 x = lds_tr4(t + off(r, p) + s), y = lds_tr4(t + off(r + 4, p) + s);
        f.u = make_uint4(x.x, x.y, y.x, y.y);
    }
    static __device__ __forceinline__ void cols(const char* t, int lane, int b, int tt, int db, Frag<float>& f) {
        const int r = (KC / 2) * (lane >> 5) + 16 * b + 8 * tt, c = 32 * db + (lane & 31);
#pragma unroll
        for (int e = 0; e < 8; ++e) f.v[e] = *reinterpret_cast<const float*>(t + off(r + e, c >> 2) + (c & 3) * 4);
    }
};

// The part of a tile that one of NT threads brings in: pieces t + NT i.  Rows
// past the last one and pieces past d channels repeat valid ones (the first
// are masked by the caller, the second meet zeros of the other operand or
// give channels that are not written).
template <typename T, int DP, int KC, int NT>
struct Part {
    using TL = Tile<T, DP, KC>;
    static constexpr int kN = KC * TL::kPieces / NT;
    static_assert(KC * TL::kPieces % NT == 0, "whole pieces per thread");
    uint4 p[kN];

    static __device__ __forceinline__ int row(int t, int i) { return (t + i * NT) / TL::kPieces; }
    // rows r0 + row of a [n][stride] tensor, n > r0
    __device__ __forceinline__ void load(const T* base, int64_t stride, int r0, int n, int d, int t) {
        const T* first = base + (int64_t)r0 * stride;
        const int last = n - 1 - r0;
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const int piece = (t + i * NT) % TL::kPieces;
            const int r = min(row(t, i), last), c = piece * TL::kPer < d ? piece * TL::kPer : 0;
            p[i] = *reinterpret_cast<const uint4*>(first + (uint32_t)(r * (int)stride + c));
        }
    }
    // present: bit r of the chunk's row r; rows without theirs become zero
    __device__ __forceinline__ void stage(char* tile, int t, bool some_absent, uint64_t present) const {
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const int r = row(t, i);
            uint4 x = p[i];
            if (some_absent && !((present >> r) & 1)) x = make_uint4(0, 0, 0, 0);
            *reinterpret_cast<uint4*>(tile + TL::off(r, (t + i * NT) % TL::kPieces)) = x;
        }
    }
};

// Bits of the keys [k0, k0 + KC) that are in range and present, the same in every lane of the wave.
struct KeyByte {
    uint32_t m;
    __device__ __forceinline__ void load(const uint8_t* mask, int k0, int nk, int lane) {
        m = mask ? mask[min(k0 + lane, nk - 1)] : 1u;
    }
    __device__ __forceinline__ uint64_t bits(int k0, int kend, int lane) const {
        return __ballot(k0 + lane < kend && m != 0);
    }
};

constexpr float kLog2e = 1.4426950408889634f;

// exp(x - M) as exp2 of one FMA (x log2 e - M log2 e) rounds M log2 e once, by at
// most half a step of it; below this magnitude that is of the size of the
// rounding of x itself, which fp32 scores carry anyway.  Beyond it (biases of
// -1e9 or of the type's lowest value all along a row) the difference is taken
// first: one more operation a score, and exact.
constexpr float kFmaMax = 1024.f;

// Four consecutive values of a row as floats.
__device__ __forceinline__ float4 bf4(uint32_t lo, uint32_t hi) {
    return make_float4(__uint_as_float(lo << 16), __uint_as_float(lo & 0xffff0000u), __uint_as_float(hi << 16),
                       __uint_as_float(hi & 0xffff0000u));
}

// The bias of one lane's KC / 2 consecutive keys of its query.
template <typename T, int KC>
struct BiasRow {
    static constexpr int kPer = 16 / (int)sizeof(T), kN = KC / 2 / kPer;
    uint4 p[kN];
    // row: the query's bias; keys k .. ; pieces that start past the last key repeat the row's first
    __device__ __forceinline__ void load(const T* row, int k, int nk) {
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const int c = k + i * kPer;
            p[i] = *reinterpret_cast<const uint4*>(row + (c < nk ? c : 0));
        }
    }
    // values 16 b + 4 a .. + 3
    __device__ __forceinline__ float4 get(int b, int a) const {
        if constexpr (sizeof(T) == 2) {
            const uint4 x = p[2 * b + (a >> 1)];
            return a & 1 ? bf4(x.z, x.w) : bf4(x.x, x.y);
        } else {
            return __builtin_bit_cast(float4, p[4 * b + a]);
        }
    }
};

}  // namespace trimul
