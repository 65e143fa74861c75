// Activations to 8 bits with a power of two for each group, and back (include/checkpoint8.h).
//
// A lane takes eight consecutive values, G lanes (the next power of two) a group; the maximum over them is a few DPP
// steps.  Bound by memory: 1024 x 1024 x 128 bf16 in groups of 32 takes 85 us to pack and 60 to unpack (0.41 GB each, 4.7 and
// 6.7 TB/s, the second partly from the last-level cache); 333 x 30 floats 4.3 and 5.8 us, a launch.
#include <type_traits>

#include "codes8.h"
#include "kernels.h"
#include "vec.h"

namespace trimul {
namespace {

// Where a lane's eight values are.
struct Place {
    int64_t x, code, power;
    int n;      // how many of them exist (<= 0: none)
};

// Lane `lane` of group `slot`; FLAT: all rows are one.
template <bool FLAT>
__device__ __forceinline__ Place place(const CheckpointArgs& a, int64_t slot, int lane) {
    if (slot >= a.slots) return Place{0, 0, 0, 0};
    int64_t row = 0, g = slot;
    if constexpr (!FLAT) {
        if (a.slots >> 32 == 0) {
            row = (uint32_t)slot / (uint32_t)a.groups;
        } else {
            row = slot / a.groups;
        }
        g = slot - row * a.groups;
    }
    const int64_t at = g * a.group + 8 * lane;
    const int64_t left = min((int64_t)(a.group - 8 * lane), a.n - at);
    return Place{row * a.ld + at, row * a.n + at, slot, (int)min(left, (int64_t)8)};
}

constexpr int kCheckpointUnroll = 4;      // groups of a lane, their loads under way together

template <typename T, int G, bool FLAT>
__global__ __launch_bounds__(256) void k_checkpoint_pack(const CheckpointArgs a, const T* x, int8_t* codes, uint8_t* powers) {
    constexpr int kSlots = 256 / G;
    const int lane = threadIdx.x % G;
    const int64_t first = (int64_t)blockIdx.x * (kSlots * kCheckpointUnroll) + threadIdx.x / G;
    Place p[kCheckpointUnroll];
    Words<T, 8> w[kCheckpointUnroll];
#pragma unroll
    for (int u = 0; u < kCheckpointUnroll; ++u) {
        p[u] = place<FLAT>(a, first + u * kSlots, lane);
        w[u].clear();
        if (a.wide && p[u].n >= 8) w[u].load(x + p[u].x);
        else if (p[u].n > 0) w[u].load_some(x + p[u].x, p[u].n);
    }
    Vec<T, 8> v[kCheckpointUnroll];
#pragma unroll
    for (int u = 0; u < kCheckpointUnroll; ++u) {
        v[u] = w[u].values();
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[u].f[i]) & 0x7fffffffu);
        top = umax_lanes<G>(top);
        const uint32_t byte = power_byte(top);
        const float inverse = power_inverse(byte);
        if (power_cut(top))
#pragma unroll
            for (int i = 0; i < 8; ++i) v[u].f[i] = fminf(fmaxf(v[u].f[i], -kTopValue), kTopValue);
        const uint32_t lo = codes4(v[u].f[0], v[u].f[1], v[u].f[2], v[u].f[3], inverse);
        const uint32_t hi = codes4(v[u].f[4], v[u].f[5], v[u].f[6], v[u].f[7], inverse);
        int8_t* to = codes + p[u].code;
        if (a.wide && p[u].n >= 8) {
            *reinterpret_cast<uint2*>(to) = make_uint2(lo, hi);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < p[u].n) to[i] = (int8_t)((i < 4 ? lo : hi) >> (8 * (i & 3)));
        }
        if (lane == 0 && p[u].n > 0) powers[p[u].power] = (uint8_t)byte;
    }
}

template <typename T, int G, bool FLAT>
__global__ __launch_bounds__(256) void k_checkpoint_unpack(const CheckpointArgs a, const int8_t* codes, const uint8_t* powers, T* out) {
    constexpr int kSlots = 256 / G;
    const int lane = threadIdx.x % G;
    const int64_t first = (int64_t)blockIdx.x * (kSlots * kCheckpointUnroll) + threadIdx.x / G;
    Place p[kCheckpointUnroll];
    uint2 w[kCheckpointUnroll];
    uint32_t byte[kCheckpointUnroll];
#pragma unroll
    for (int u = 0; u < kCheckpointUnroll; ++u) {
        p[u] = place<FLAT>(a, first + u * kSlots, lane);
        w[u] = make_uint2(0, 0);
        byte[u] = p[u].n > 0 ? powers[p[u].power] : 0;
        const int8_t* from = codes + p[u].code;
        if (a.wide && p[u].n >= 8) {
            w[u] = *reinterpret_cast<const uint2*>(from);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t b = i < p[u].n ? (uint32_t)(uint8_t)from[i] << (8 * (i & 3)) : 0u;
                if (i < 4) w[u].x |= b;
                else w[u].y |= b;
            }
        }
    }
#pragma unroll
    for (int u = 0; u < kCheckpointUnroll; ++u) {
        const float scale = power_value(byte[u]);
        Vec<T, 8> v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v.f[i] = code_value(i < 4 ? w[u].x : w[u].y, i & 3) * scale;
        store_some(v, out + p[u].x, p[u].n, a.wide);
    }
}

// Lanes of a group: the next power of two.
int group_lanes(int group) {
    int g = 1;
    while (8 * g < group) g *= 2;
    return g;
}

template <typename F>
hipError_t by_lanes(int lanes, F f) {
    switch (lanes) {
        case 1: return f(std::integral_constant<int, 1>{});
        case 2: return f(std::integral_constant<int, 2>{});
        case 4: return f(std::integral_constant<int, 4>{});
        case 8: return f(std::integral_constant<int, 8>{});
        case 16: return f(std::integral_constant<int, 16>{});
        default: return f(std::integral_constant<int, 32>{});
    }
}

// Fills in a: rows that follow each other without a gap and hold whole groups are one long row.
bool flatten(CheckpointArgs& a) {
    const bool flat = a.rows == 1 || (a.ld == a.n && a.n % a.group == 0);
    if (flat) {
        a.n *= a.rows;
        a.rows = 1;
    }
    a.groups = (a.n + a.group - 1) / a.group;
    a.slots = a.rows * a.groups;
    return flat;
}

template <typename T, bool FLAT>
hipError_t launch(bool pack, const CheckpointArgs& a, const void* from, const uint8_t* powers, void* to, hipStream_t s) {
    const int lanes = group_lanes(a.group);
    const int64_t per = 256 / lanes * kCheckpointUnroll;
    const dim3 grid((unsigned)((a.slots + per - 1) / per)), block(256);
    return by_lanes(lanes, [&](auto g) {
        constexpr int G = decltype(g)::value;
        if (pack) hipLaunchKernelGGL((k_checkpoint_pack<T, G, FLAT>), grid, block, 0, s, a, (const T*)from, (int8_t*)to, const_cast<uint8_t*>(powers));
        else hipLaunchKernelGGL((k_checkpoint_unpack<T, G, FLAT>), grid, block, 0, s, a, (const int8_t*)from, powers, (T*)to);
        return hipGetLastError();
    });
}

}  // namespace

int64_t checkpoint8_work_groups(CheckpointArgs a) {
    flatten(a);
    const int64_t per = 256 / group_lanes(a.group) * kCheckpointUnroll;
    return (a.slots + per - 1) / per;
}

hipError_t launch_checkpoint8(int dtype, bool pack, CheckpointArgs a, const void* from, const uint8_t* powers, void* to, hipStream_t s) {
    const bool flat = flatten(a);
    const void* x = pack ? from : to;
    const void* codes = pack ? to : from;
    a.wide = (reinterpret_cast<uintptr_t>(x) & 15) == 0 && (reinterpret_cast<uintptr_t>(codes) & 7) == 0 && (a.rows == 1 || (a.n % 8 == 0 && a.ld % 8 == 0));
    if (dtype == 1) return flat ? launch<bf16_t, true>(pack, a, from, powers, to, s) : launch<bf16_t, false>(pack, a, from, powers, to, s);
    return flat ? launch<float, true>(pack, a, from, powers, to, s) : launch<float, false>(pack, a, from, powers, to, s);
}

}  // namespace trimul
