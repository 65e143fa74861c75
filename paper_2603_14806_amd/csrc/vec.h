// Loads and stores of several consecutive values of a tensor as floats (gfx950).
#pragma once

#include "common.h"

namespace trimul {

// V consecutive values (1, 4 or 8; of floats also 2) as floats, and back.
template <typename T, int V> struct Vec {
    float f[V];
    __device__ __forceinline__ void load(const T* p) {
        if constexpr (V == 1) {
            f[0] = Store<T>::ld(p);
        } else if constexpr (V == 2 && sizeof(T) == 4) {
            const float2 x = *reinterpret_cast<const float2*>(p);
            f[0] = x.x; f[1] = x.y;
        } else if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < V / 4; ++i) {
                const float4 x = reinterpret_cast<const float4*>(p)[i];
                f[4 * i] = x.x; f[4 * i + 1] = x.y; f[4 * i + 2] = x.z; f[4 * i + 3] = x.w;
            }
        } else {
            uint32_t w[V / 2];
            if constexpr (V == 8) {
                const uint4 x = *reinterpret_cast<const uint4*>(p);
                w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
            } else {
                const uint2 x = *reinterpret_cast<const uint2*>(p);
                w[0] = x.x; w[1] = x.y;
            }
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                f[2 * i] = __uint_as_float(w[i] << 16);
                f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        }
    }
    __device__ __forceinline__ void store(T* p) const {
        if constexpr (V == 1) {
            Store<T>::st(p, f[0]);
        } else if constexpr (V == 2 && sizeof(T) == 4) {
            *reinterpret_cast<float2*>(p) = make_float2(f[0], f[1]);
        } else if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < V / 4; ++i)
                reinterpret_cast<float4*>(p)[i] = make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
        } else if constexpr (V == 8) {
            *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]),
                                                      pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
        } else {
            *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]));
        }
    }
};

// The same values as they lie in memory.  Where loads are to be under way together, these are what is loaded: a
// conversion beside a load, in a branch, waits for it there.
template <typename T, int V> struct Words {
    static constexpr int kWords = V * sizeof(T) < 4 ? 1 : V * (int)sizeof(T) / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0;
    }
    __device__ __forceinline__ void load(const T* p) {
        if constexpr (V * sizeof(T) == 2) w[0] = *reinterpret_cast<const uint16_t*>(p);
        else if constexpr (kWords == 1) w[0] = *reinterpret_cast<const uint32_t*>(p);
        else if constexpr (kWords == 2) {
            const uint2 x = *reinterpret_cast<const uint2*>(p);
            w[0] = x.x; w[1] = x.y;
        } else {
#pragma unroll
            for (int i = 0; i < kWords / 4; ++i) {
                const uint4 x = reinterpret_cast<const uint4*>(p)[i];
                w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w;
            }
        }
    }
    // The first n of them, one by one (the first stands in for what is not there, and is 0 in its place; with n = 0 it
    // has to be readable all the same).
    __device__ __forceinline__ void load_some(const T* p, int n) {
        T x[V];
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = p[i < n ? i : 0];
        clear();
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if constexpr (sizeof(T) == 4) w[i] = i < n ? __float_as_uint(x[i]) : 0u;
            else w[i / 2] |= i < n ? (uint32_t)x[i] << (16 * (i & 1)) : 0u;
        }
    }
    __device__ __forceinline__ Vec<T, V> values() const {
        Vec<T, V> v;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if constexpr (sizeof(T) == 4) v.f[i] = __uint_as_float(w[i]);
            else v.f[i] = __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        }
        return v;
    }
};

// Eight values of which the first n exist; wide: p is 16-byte aligned.
template <typename T>
__device__ __forceinline__ void store_some(const Vec<T, 8>& v, T* p, int n, bool wide) {
    if (wide && n >= 8) {
        v.store(p);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) Store<T>::st(p + i, v.f[i]);
    }
}

}  // namespace trimul
