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

// x where bit i of `bits` is set, else -inf: a sign-extended bit and a bitwise select.
__device__ __forceinline__ float present_or_inf(float x, uint32_t bits, int i) {
    const uint32_t m = (uint32_t)((int32_t)(bits << (31 - i)) >> 31);
    return __uint_as_float((__float_as_uint(x) & m) | (0xff800000u & ~m));
}

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

// The values of a fragment to memory (16-byte aligned), the first n of them.
__device__ __forceinline__ void store8(bf16_t* p, const Frag<bf16_t>& f, int n) {
    if (n >= 8) {
        *reinterpret_cast<uint4*>(p) = f.u;
    } else {
        const uint32_t w[4] = {f.u.x, f.u.y, f.u.z, f.u.w};
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n) p[e] = (bf16_t)(w[e >> 1] >> (16 * (e & 1)));
    }
}
__device__ __forceinline__ void store8(float* p, const Frag<float>& f, int n) {
    if (n >= 8) {
        reinterpret_cast<float4*>(p)[0] = make_float4(f.v[0], f.v[1], f.v[2], f.v[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(f.v[4], f.v[5], f.v[6], f.v[7]);
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n) p[e] = f.v[e];
    }
}

// A fragment of one token's channels straight from memory: values 16 s2 + 8 hi
// .. + 7 of a row of d channels (zero past d).
__device__ __forceinline__ void load_row(const bf16_t* row, int s2, int hi, int d, Frag<bf16_t>& f) {
    const int c = 16 * s2 + 8 * hi;
    const uint4 x = *reinterpret_cast<const uint4*>(row + (c < d ? c : 0));
    const uint32_t m = c < d ? ~0u : 0u;   // (an `if` here becomes a branch around the load, and a wait for each)
    f.u = make_uint4(x.x & m, x.y & m, x.z & m, x.w & m);
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
    // spans of four consecutive rows of a transposing read.  The swizzle looks
    // at bits 0 to 2 of the row and at its half of the tile alone, so that a
    // lane's offsets differ between products by constants added to the row and
    // constants XORed to the piece.
    static __host__ __device__ constexpr int twist(int row, int half) {
        return (((row >> 2) & 1) | (half << 1)) ^
               (kPieces >= 16 ? (row & 3) << 2 : kPieces == 8 ? ((row >> 1) & 1) << 2 : 0);
    }
    static __device__ __forceinline__ uint32_t off(int row, int piece) {
        return (uint32_t)(row * kRowBytes + ((piece ^ twist(row, row >= KC / 2 ? 1 : 0)) << 4));
    }

    uint32_t ar, ac;   // this lane's first row read and transposing read
    __device__ __forceinline__ void init(int lane) {
        const int l = lane & 31, hi = lane >> 5;
        // product row l of the b-th product: tile row (KC / 2) ((l / 4) % 2) + 16 b + 4 (l / 8) + l % 4
        ar = off((KC / 2) * ((l >> 2) & 1) + 4 * (l >> 3) + (l & 3), (sizeof(T) == 2 ? 1 : 2) * hi);
        if constexpr (sizeof(T) == 2)
            ac = off((KC / 2) * hi + ((lane >> 2) & 3), 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1)) + (lane & 1) * 8;
        else
            ac = off((KC / 2) * hi, l >> 2) + (l & 3) * 4;
    }
    // A operand: rows of the b-th product, channels 16 s2 ..
    __device__ __forceinline__ void rows(const char* t, int b, int s2, Frag<bf16_t>& f) const {
        f.u = *reinterpret_cast<const uint4*>(t + (ar ^ (s2 << 5)) + b * 16 * kRowBytes);
    }
    __device__ __forceinline__ void rows(const char* t, int b, int s2, Frag<float>& f) const {
        const float4 x = *reinterpret_cast<const float4*>(t + (ar ^ (s2 << 6)) + b * 16 * kRowBytes);
        const float4 y = *reinterpret_cast<const float4*>(t + (ar ^ (s2 << 6) ^ 16) + b * 16 * kRowBytes);
        const float v[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) f.v[e] = v[e];
    }
    // One row's channels 16 s2 + 8 hi .. (rows in their own order)
    static __device__ __forceinline__ void row(const char* t, int r, int hi, int s2, Frag<bf16_t>& f) {
        f.u = *reinterpret_cast<const uint4*>(t + off(r, 2 * s2 + hi));
    }
    static __device__ __forceinline__ void row(const char* t, int r, int hi, int s2, Frag<float>& f) {
        const float4 x = *reinterpret_cast<const float4*>(t + off(r, 4 * s2 + 2 * hi));
        const float4 y = *reinterpret_cast<const float4*>(t + off(r, 4 * s2 + 2 * hi + 1));
        const float v[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) f.v[e] = v[e];
    }
    // A operand, transposed: channels 32 db + lane % 32, reduction over the tile rows that
    // registers 8 tt .. of the b-th product stand for.
    __device__ __forceinline__ void cols(const char* t, int b, int tt, int db, Frag<bf16_t>& f) const {
        const char* p = t + (16 * b + 8 * tt) * kRowBytes;
        const uint2 x = lds_tr4(p + (ac ^ (db << 6))), y = lds_tr4(p + 4 * kRowBytes + (ac ^ (db << 6) ^ 16));
        f.u = make_uint4(x.x, x.y, y.x, y.y);
    }
    __device__ __forceinline__ void cols(const char* t, int b, int tt, int db, Frag<float>& f) const {
        const char* p = t + (16 * b + 8 * tt) * kRowBytes;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            f.v[e] = *reinterpret_cast<const float*>(p + e * kRowBytes + (ac ^ (db << 7) ^ (twist(e, 0) << 4)));
    }
};

// The part of a tile that one of NT threads brings in: pieces t + NT i of its
// rows, through a buffer descriptor of the rows that exist (scalar registers:
// the base moves from chunk to chunk, a thread's offsets stay).  Rows past the
// last one and pieces past d channels read zero.
template <typename T, int DP, int KC, int NT>
struct Part {
    using TL = Tile<T, DP, KC>;
    static constexpr int kAll = KC * TL::kPieces, kN = (kAll + NT - 1) / NT;
    static_assert(kAll % NT == 0 || kAll < NT, "whole pieces per thread");
    uint32_t off[kN];
    uint4 p[kN];

    static __device__ __forceinline__ int row(int t, int i) { return (t + i * NT) / TL::kPieces; }
    static __device__ __forceinline__ int piece(int t, int i) { return (t + i * NT) % TL::kPieces; }
    static __device__ __forceinline__ bool mine(int t) { return kAll >= NT || t < kAll; }
    __device__ __forceinline__ void init(int64_t stride, int d, int t) {
#pragma unroll
        for (int i = 0; i < kN; ++i)
            off[i] = mine(t) && piece(t, i) * TL::kPer < d
                         ? (uint32_t)row(t, i) * (uint32_t)(stride * (int)sizeof(T)) + 16 * piece(t, i)
                         : 0xfffffff0u;
    }
    // rows r0 .. of n rows at base; no row left: nothing is read
    __device__ __forceinline__ void load(const T* base, int64_t stride, int r0, int n, int d) {
        const int rows = min(n - r0, KC);
        const auto r = make_rsrc(base + (int64_t)r0 * stride,
                                 rows > 0 ? (uint32_t)((rows - 1) * (uint32_t)stride + d) * (uint32_t)sizeof(T) : 0u);
#pragma unroll
        for (int i = 0; i < kN; ++i) p[i] = buf_load16(r, off[i]);
    }
    // present: bit r of the chunk's row r; rows without theirs become zero
    __device__ __forceinline__ void stage(char* tile, int t, bool some_absent, uint64_t present) const {
        if (!mine(t)) return;
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const int r = row(t, i);
            uint4 x = p[i];
            if (some_absent && !((present >> r) & 1)) x = make_uint4(0, 0, 0, 0);
            *reinterpret_cast<uint4*>(tile + TL::off(r, piece(t, i))) = x;
        }
    }
};

// Work-groups go to the eight XCDs in turn; this order gives each XCD consecutive
// ones, which read the same keys (or queries), so that its L2 serves the repeats.
// (32 bits: a grid is below 2^24, and the divisions that take the number apart
// are four times as long in 64.)
__device__ __forceinline__ uint32_t xcd_block() {
    const uint32_t n = gridDim.x, x = blockIdx.x & 7, i = blockIdx.x >> 3;
    return x * (n >> 3) + min(x, n & 7) + i;
}

// Wave-private LDS: a wave's LDS operations run in order, only the compiler has to be kept from moving them.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The four waves' results of the same 32 columns added up: wave w gets channels 8 ND w .. + 8 ND - 1 (as registers
// 4 j + e, j < ND: channel 8 (ND w + j) + 4 hi + e).  buf: 4 * ND * 16 * 64 floats that no wave uses any more.
template <int ND>
__device__ __forceinline__ void add_waves(f32x16_t (&o)[ND], float* buf, int w, int lane) {
#pragma unroll
    for (int i = 0; i < ND; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) buf[(w * ND * 16 + 16 * i + r) * 64 + lane] = o[i][r];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < ND; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float x = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) x += buf[(i * ND * 16 + 4 * (w * ND + j) + e) * 64 + lane];
            o[j / 4][4 * (j % 4) + e] = x;
        }
}

// Bits of the keys [k0, k0 + KC) that are in range and present, the same in every lane of the wave.
struct KeyByte {
    uint32_t m;
    // (loads without branches: the compiler then knows how many are in flight)
    __device__ __forceinline__ void load(const uint8_t* mask, int k0, int nk, int lane) {
        m = __builtin_amdgcn_raw_buffer_load_b8(make_rsrc(mask, mask ? (uint32_t)nk : 0u), k0 + lane, 0, 0);
    }
    __device__ __forceinline__ uint64_t bits(const uint8_t* mask, int k0, int kend, int lane) const {
        return __ballot(k0 + lane < kend && (m != 0 || mask == nullptr));
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

template <typename T>
__device__ __forceinline__ void store4(T* p, float a, float b, float c, float d) {
    if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d);
    else *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(a, b), pack_bf16x2(c, d));
}

// Channel groups g0 .. of a result (registers 4 j + e: channel 8 (g0 + j) + 4 hi + e), scaled, to a row of d channels.
template <int ND, typename T>
__device__ __forceinline__ void store_row(T* row, const f32x16_t (&o)[ND], int groups, int g0, int hi, int d, float scale) {
#pragma unroll
    for (int j = 0; j < 4 * ND; ++j) {
        const int c = 8 * (g0 + j) + 4 * hi;
        if (j < groups && c < d)
            store4(row + c, o[j / 4][4 * (j % 4)] * scale, o[j / 4][4 * (j % 4) + 1] * scale,
                   o[j / 4][4 * (j % 4) + 2] * scale, o[j / 4][4 * (j % 4) + 3] * scale);
    }
}

// What rounding the same values to bf16 takes from them, rounded to bf16 itself.
__device__ __forceinline__ float rounded_off(float x) { return x - bf2f(f2bf(x)); }
template <int ND>
__device__ __forceinline__ void store_rest(bf16_t* row, const f32x16_t (&o)[ND], int groups, int g0, int hi, int d, float scale) {
#pragma unroll
    for (int j = 0; j < 4 * ND; ++j) {
        const int c = 8 * (g0 + j) + 4 * hi;
        if (j < groups && c < d)
            store4(row + c, rounded_off(o[j / 4][4 * (j % 4)] * scale), rounded_off(o[j / 4][4 * (j % 4) + 1] * scale),
                   rounded_off(o[j / 4][4 * (j % 4) + 2] * scale), rounded_off(o[j / 4][4 * (j % 4) + 3] * scale));
    }
}

// The bias of one lane's KC / 2 consecutive keys of its query, through a
// descriptor of the rows of its wave's 32 columns: from the first one's to the
// end of the last one's keys (rounded up to 8: nothing behind that is read; a
// piece past the keys of another row reads whatever follows it).
template <typename T, int KC>
struct BiasRow {
    static constexpr int kPer = 16 / (int)sizeof(T), kN = KC / 2 / kPer;
    const T* first;      // uniform
    uint32_t span, off;  // bytes; off: this lane's row, first key of its half
    uint4 p[kN];
    // columns c0 .. c1 (uniform) of key head hk, this lane's query and head
    __device__ __forceinline__ void init(const CrossArgs& a, int64_t b, int hk, int c0, int c1, int qi, int h, int hi) {
        const int q0 = c0 / a.group, q1 = c1 / a.group;
        first = (const T*)a.bias.data + b * a.bias.batch + (int64_t)(hk * a.group) * a.bias.head + (int64_t)q0 * a.bias.row;
        span = (uint32_t)((q1 - q0) * a.bias.row + (a.group - 1) * a.bias.head + ((a.nk + 7) & ~7)) * (uint32_t)sizeof(T);
        off = (uint32_t)((qi - q0) * a.bias.row + (h - hk * a.group) * a.bias.head + (KC / 2) * hi) * (uint32_t)sizeof(T);
    }
    // queries q0 .. q1 (uniform) of one head, this lane's query
    __device__ __forceinline__ void init(const CrossArgs& a, int64_t b, int h, int q0, int q1, int qi, int hi) {
        first = (const T*)a.bias.data + b * a.bias.batch + (int64_t)h * a.bias.head + (int64_t)q0 * a.bias.row;
        span = (uint32_t)((q1 - q0) * a.bias.row + ((a.nk + 7) & ~7)) * (uint32_t)sizeof(T);
        off = (uint32_t)((qi - q0) * a.bias.row + (KC / 2) * hi) * (uint32_t)sizeof(T);
    }
    __device__ __forceinline__ void load(int k0, int nk) {
        const auto r = make_rsrc(first + k0, k0 < nk ? span - (uint32_t)k0 * (uint32_t)sizeof(T) : 0u);
#pragma unroll
        for (int i = 0; i < kN; ++i) p[i] = buf_load16(r, off + 16 * i);
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
