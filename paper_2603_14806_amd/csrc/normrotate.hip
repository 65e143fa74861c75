// Norms of queries and keys by head with the position rotation, and their gradients (include/norm_rotate.h).
//
// A lane takes eight values of a row: four pairs that are turned together (halves: four values from each half), so that a
// rotation needs no other lane.  G lanes (the next power of two of d / 8) are a row, and sum over it by DPP.  The angles
// belong to the token: a wave turns all heads of its tokens, queries and keys, and where the entries of the batch share
// their positions those of several entries, with one sine and cosine a pair.
#include <algorithm>

#include "codes8.h"
#include "common.h"
#include "kernels.h"
#include "vec.h"

namespace trimul {
namespace {

constexpr double kInvTwoPi = 0.15915494309189533577;

// cos and sin of p f, f in turns: the angle in quarter turns is reduced in 64 bits, where far positions keep their
// fraction, and what is left is at most half a quarter turn either way.
__device__ __forceinline__ void turn(int p, double f, float& c, float& s) {
    const double t = 4.0 * ((double)p * f), q = rint(t);
    float a, b;
    sincospif(0.5f * (float)(t - q), &b, &a);
    const int k = (int)(q - 4.0 * floor(q * 0.25));            // quarter turns, 0..3
    c = k == 0 ? a : k == 1 ? -b : k == 2 ? -a : b;
    s = k == 0 ? b : k == 1 ? a : k == 2 ? -b : -a;
}

// A lane's eight values: f[0..3] and f[4..7] are the two halves of its places lo and hi (HALVES), or eight in a row.
template <typename T, bool HALVES>
__device__ __forceinline__ void load8(float (&f)[8], const T* p, int lo, int hi) {
    if constexpr (HALVES) {
        Vec<T, 4> a, b;
        a.load(p + lo);
        b.load(p + hi);
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[i] = a.f[i]; f[4 + i] = b.f[i]; }
    } else {
        Vec<T, 8> a;
        a.load(p + lo);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = a.f[i];
    }
}
template <typename T, bool HALVES>
__device__ __forceinline__ void store8(const float (&f)[8], T* p, int lo, int hi) {
    if constexpr (HALVES) {
        Vec<T, 4> a, b;
#pragma unroll
        for (int i = 0; i < 4; ++i) { a.f[i] = f[i]; b.f[i] = f[4 + i]; }
        a.store(p + lo);
        b.store(p + hi);
    } else {
        Vec<T, 8> a;
#pragma unroll
        for (int i = 0; i < 8; ++i) a.f[i] = f[i];
        a.store(p + lo);
    }
}

// Pair m of a lane is (f[m], f[4 + m]) of halves, (f[2 m], f[2 m + 1]) of neighbours; back: by the negative angle.
template <bool HALVES, bool BACK>
__device__ __forceinline__ void rotate8(float (&f)[8], const float (&c)[4], const float (&s)[4]) {
#pragma unroll
    for (int m = 0; m < 4; ++m) {
        constexpr float sign = BACK ? -1.f : 1.f;
        float& a = f[HALVES ? m : 2 * m];
        float& b = f[HALVES ? 4 + m : 2 * m + 1];
        const float ya = a * c[m] - sign * (b * s[m]), yb = sign * (a * s[m]) + b * c[m];
        a = ya;
        b = yb;
    }
}

// A wave's place in an item: which lanes are where.
struct Lane {
    int l, lo, hi;          // eighth of the row, and where its values are
    int head, token;        // slots
    bool live;              // the row has an eighth l
};

template <int G, bool HALVES>
__device__ __forceinline__ Lane lane_of(const NormArgs& a) {
    const int lane = threadIdx.x % 64, slot = lane / G;
    Lane x;
    x.l = lane % G;
    x.live = 8 * x.l < a.d;
    x.head = slot & (a.head_slots - 1);
    x.token = slot / a.head_slots;
    const bool turned = HALVES && 8 * x.l < a.rot;
    x.lo = turned ? 4 * x.l : 8 * x.l;
    x.hi = turned ? a.rot / 2 + 4 * x.l : 8 * x.l + 4;
    return x;
}

// Eight of a side's weights, in the lane's places.
template <bool HALVES>
__device__ __forceinline__ void weights8(float (&f)[8], const void* w, bool bf16, const Lane& x, float none) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = none;
    if (!w || !x.live) return;
    if (bf16) load8<bf16_t, HALVES>(f, static_cast<const bf16_t*>(w), x.lo, x.hi);
    else load8<float, HALVES>(f, static_cast<const float*>(w), x.lo, x.hi);
}

// u (in the place of x) and r of a row.
template <int G>
__device__ __forceinline__ float normalise8(float (&f)[8], const NormArgs& a, bool live) {
    if (a.layer) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += f[i];
        const float mean = sum_lanes<G>(sum) * a.inv_d;
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = live ? f[i] - mean : 0.f;
    }
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(f[i], f[i], sum);
    const float r = rsqrtf(sum_lanes<G>(sum) * a.inv_d + a.eps);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] *= r;
    return r;
}

// The angles of a token's pairs in this lane.
__device__ __forceinline__ void angles(const NormArgs& a, const Lane& x, const double (&f)[4], int64_t entry, int64_t token, float (&c)[4], float (&s)[4]) {
    const bool turned = 8 * x.l < a.rot && token < a.n;
    const int p = turned ? a.positions[entry * a.positions_batch + token] : 0;
#pragma unroll
    for (int m = 0; m < 4; ++m) turn(p, f[m], c[m], s[m]);
}

__device__ __forceinline__ void frequencies(const NormArgs& a, const Lane& x, double (&f)[4]) {
#pragma unroll
    for (int m = 0; m < 4; ++m) f[m] = 8 * x.l < a.rot ? a.freqs[4 * x.l + m] * kInvTwoPi : 0.0;
}

// A wave's items: token tile and chunk of entries, `waves` items apart.
struct Item {
    int64_t tile, chunk;
    __device__ __forceinline__ Item(const NormArgs& a, int64_t wave) : tile(wave % a.tiles), chunk(wave / a.tiles) {}
    __device__ __forceinline__ void next(const NormArgs& a) {
        tile += a.step_tile;
        chunk += a.step_chunk;
        if (tile >= a.tiles) {
            tile -= a.tiles;
            ++chunk;
        }
    }
};

// A row's place: head step i of an item's entries.
struct Row {
    int64_t entry;
    int head;
    bool live;
};

template <typename T, int G, bool HALVES>
__global__ __launch_bounds__(256) void k_norm_rotate(const NormArgs a) {
    constexpr int U = 4;
    const Lane x = lane_of<G, HALVES>(a);
    const int tokens = 64 / G / a.head_slots;
    double f[4];
    frequencies(a, x, f);
    const int64_t wave = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
    for (Item item(a, wave); item.chunk < a.chunks; item.next(a)) {
        const int64_t token = item.tile * tokens + x.token, b0 = item.chunk * a.chunk;
        const int entries = (int)min(a.chunk, a.batch - b0);
        float c[4], s[4];
        angles(a, x, f, b0, token, c, s);
#pragma unroll 1
        for (int side = 0; side < 2; ++side) {
            const NormSide& q = a.side[side];
            if (q.heads == 0) continue;
            float gain[8], shift[8];
            weights8<HALVES>(gain, q.gain, a.weight_bf16, x, 1.f);
            weights8<HALVES>(shift, q.shift, a.weight_bf16, x, 0.f);
            const int rows = entries * q.steps;
            int entry = 0, step = 0;
            for (int i = 0; i < rows; i += U) {
                float v[U][8];
                Row row[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    row[u] = Row{b0 + entry, step * a.head_slots + x.head, false};
                    row[u].live = i + u < rows && x.live && token < a.n && row[u].head < q.heads;
                    if (++step == q.steps) {
                        step = 0;
                        ++entry;
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[u][e] = 0.f;
                    if (row[u].live) load8<T, HALVES>(v[u], static_cast<const T*>(q.x.data) + row[u].entry * q.x.batch + token * q.x.token + row[u].head * q.x.head, x.lo, x.hi);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (i + u >= rows) break;
                    if (q.codes) {
                        uint32_t top = 0;
#pragma unroll
                        for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[u][e]) & 0x7fffffffu);
                        top = umax_lanes<G>(top);
                        const uint32_t byte = power_byte(top);
                        const float inverse = power_inverse(byte);
                        float w[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) w[e] = power_cut(top) ? fminf(fmaxf(v[u][e], -kTopValue), kTopValue) : v[u][e];
                        const uint32_t lo = codes4(w[0], w[1], w[2], w[3], inverse), hi = codes4(w[4], w[5], w[6], w[7], inverse);
                        if (row[u].live) {
                            const int64_t at = (row[u].entry * a.n + token) * q.heads + row[u].head;
                            int8_t* to = q.codes + at * a.d;
                            if constexpr (HALVES) {
                                *reinterpret_cast<uint32_t*>(to + x.lo) = lo;
                                *reinterpret_cast<uint32_t*>(to + x.hi) = hi;
                            } else {
                                *reinterpret_cast<uint2*>(to + x.lo) = make_uint2(lo, hi);
                            }
                            if (x.l == 0) q.powers[at] = (uint8_t)byte;
                        }
                    }
                    normalise8<G>(v[u], a, x.live);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[u][e] = __builtin_fmaf(v[u][e], gain[e], shift[e]);
                    rotate8<HALVES, false>(v[u], c, s);
                    if (row[u].live) store8<T, HALVES>(v[u], static_cast<T*>(q.y.data) + row[u].entry * q.y.batch + token * q.y.token + row[u].head * q.y.head, x.lo, x.hi);
                }
            }
        }
    }
}

template <typename T, int G, bool HALVES>
__global__ __launch_bounds__(256) void k_norm_rotate_backward(const NormArgs a) {
    constexpr int U = 2;
    __shared__ float sums[4][4][256];                       // by wave: dgain and dshift of the queries, and of the keys
    const Lane x = lane_of<G, HALVES>(a);
    const int tokens = 64 / G / a.head_slots, w = threadIdx.x / 64;
    double f[4];
    frequencies(a, x, f);
    float total[2][2][8];
#pragma unroll
    for (int i = 0; i < 32; ++i) total[i / 16][i / 8 % 2][i % 8] = 0.f;
    const int64_t wave = (int64_t)blockIdx.x * 4 + w;
    for (Item item(a, wave); item.chunk < a.chunks; item.next(a)) {
        const int64_t token = item.tile * tokens + x.token, b0 = item.chunk * a.chunk;
        const int entries = (int)min(a.chunk, a.batch - b0);
        float c[4], s[4];
        angles(a, x, f, b0, token, c, s);
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            const NormSide& q = a.side[side];
            if (q.heads == 0) continue;
            float gain[8];
            weights8<HALVES>(gain, q.gain, a.weight_bf16, x, 1.f);
            const int rows = entries * q.steps;
            int entry = 0, step = 0;
            for (int i = 0; i < rows; i += U) {
                float v[U][8], g[U][8];
                Row row[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    row[u] = Row{b0 + entry, step * a.head_slots + x.head, false};
                    row[u].live = i + u < rows && x.live && token < a.n && row[u].head < q.heads;
                    if (++step == q.steps) {
                        step = 0;
                        ++entry;
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[u][e] = g[u][e] = 0.f;
                    if (!row[u].live) continue;
                    if (q.x.data) {
                        load8<T, HALVES>(v[u], static_cast<const T*>(q.x.data) + row[u].entry * q.x.batch + token * q.x.token + row[u].head * q.x.head, x.lo, x.hi);
                    } else {
                        const int64_t at = (row[u].entry * a.n + token) * q.heads + row[u].head;
                        const int8_t* from = q.codes + at * a.d;
                        const float scale = power_value(q.powers[at]);
                        const uint32_t lo = *reinterpret_cast<const uint32_t*>(from + x.lo), hi = *reinterpret_cast<const uint32_t*>(from + x.hi);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            v[u][e] = code_value(lo, e) * scale;
                            v[u][4 + e] = code_value(hi, e) * scale;
                        }
                    }
                    load8<T, HALVES>(g[u], static_cast<const T*>(q.y.data) + row[u].entry * q.y.batch + token * q.y.token + row[u].head * q.y.head, x.lo, x.hi);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (i + u >= rows) break;
                    const float r = normalise8<G>(v[u], a, x.live);
                    rotate8<HALVES, true>(g[u], c, s);
                    float mean = 0.f, along = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        total[side][0][e] = __builtin_fmaf(g[u][e], v[u][e], total[side][0][e]);
                        total[side][1][e] += g[u][e];
                        g[u][e] *= gain[e];
                        mean += g[u][e];
                        along = __builtin_fmaf(g[u][e], v[u][e], along);
                    }
                    along = sum_lanes<G>(along) * a.inv_d;
                    mean = a.layer ? sum_lanes<G>(mean) * a.inv_d : 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) g[u][e] = r * (g[u][e] - __builtin_fmaf(v[u][e], along, mean));
                    if (row[u].live) store8<T, HALVES>(g[u], static_cast<T*>(q.dx.data) + row[u].entry * q.dx.batch + token * q.dx.token + row[u].head * q.dx.head, x.lo, x.hi);
                }
            }
        }
    }
    // over the rows of the wave, then over the waves
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float t = total[k / 2][k % 2][e];
#pragma unroll
            for (int m = G; m < 64; m *= 2) t += __shfl_xor(t, m);
            if (threadIdx.x % 64 < G && x.live) sums[w][k][(e < 4 ? x.lo : x.hi - 4) + e] = t;
        }
    __syncthreads();
    for (int i = threadIdx.x; i < 4 * a.d; i += 256) {
        const int k = i / a.d, e = i - k * a.d;
        const float t = sums[0][k][e] + sums[1][k][e] + (sums[2][k][e] + sums[3][k][e]);
        if (gridDim.x == 1) {
            float* to = k % 2 ? a.side[k / 2].dshift : a.side[k / 2].dgain;
            if (to) to[e] = t;
        } else {
            a.part[(int64_t)blockIdx.x * 4 * a.d + i] = t;
        }
    }
}

// The weights' gradients from the work-groups' sums: a lane for each value, a wave for every 16th work-group.
__global__ __launch_bounds__(1024) void k_norm_rotate_join(const NormArgs a, int groups) {
    __shared__ double sums[16][64];
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, i = blockIdx.x * 64 + lane;
    const int k = i / a.d, e = i - k * a.d;
    float* to = k < 4 ? (k % 2 ? a.side[k / 2].dshift : a.side[k / 2].dgain) : nullptr;
    double sum = 0;
    if (to)
#pragma unroll 8
        for (int g = wave; g < groups; g += 16) sum += a.part[(int64_t)g * 4 * a.d + i];
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave || !to) return;
    for (int w = 1; w < 16; ++w) sum += sums[w][lane];
    to[e] = (float)sum;
}

__global__ __launch_bounds__(256) void k_norm_rotate_zero(const NormArgs a) {
    for (int i = threadIdx.x; i < 4 * a.d; i += 256) {
        const int k = i / a.d;
        float* to = k % 2 ? a.side[k / 2].dshift : a.side[k / 2].dgain;
        if (to) to[i - k * a.d] = 0.f;
    }
}

int pow2_from(int n, int most) {
    int p = 1;
    while (p < most && p < n) p *= 2;
    return p;
}

// Work-groups, and in a how the tokens, heads and entries lie on the waves.
int64_t plan(NormArgs& a, bool backward) {
    const int lanes = pow2_from(a.d / 8, 32), slots = 64 / lanes;
    a.head_slots = pow2_from(std::max(a.side[0].heads, a.side[1].heads), slots);
    for (NormSide& q : a.side) q.steps = (q.heads + a.head_slots - 1) / a.head_slots;
    const int tokens = slots / a.head_slots;
    a.tiles = (a.n + tokens - 1) / tokens;
    const int64_t most = 4096;                                   // waves: 16 for each compute unit
    a.chunk = a.positions_batch == 0 || a.rot == 0 ? std::max<int64_t>(1, std::min(a.batch, a.batch * a.tiles / (2 * most))) : 1;
    a.chunks = (a.batch + a.chunk - 1) / a.chunk;
    a.items = a.tiles * a.chunks;
    const int64_t groups = std::min((a.items + 3) / 4, backward ? most / 4 : int64_t(1) << 20);
    a.waves = groups * 4;
    a.step_chunk = a.waves / a.tiles;
    a.step_tile = a.waves % a.tiles;
    return groups;
}

}  // namespace

int64_t norm_rotate_groups(NormArgs a, bool backward) { return plan(a, backward); }

hipError_t launch_norm_rotate(int dtype, bool adjacent, bool backward, NormArgs a, hipStream_t s) {
    if (a.batch == 0 || a.n == 0) {
        if (!backward) return hipSuccess;
        hipLaunchKernelGGL(k_norm_rotate_zero, dim3(1), dim3(256), 0, s, a);
        return hipGetLastError();
    }
    const int64_t groups = plan(a, backward);
    a.inv_d = 1.f / (float)a.d;
    auto go = [&](auto zero, auto lanes, auto halves) {
        using T = decltype(zero);
        constexpr int G = decltype(lanes)::value;
        constexpr bool H = decltype(halves)::value;
        if (backward) hipLaunchKernelGGL((k_norm_rotate_backward<T, G, H>), dim3((unsigned)groups), dim3(256), 0, s, a);
        else hipLaunchKernelGGL((k_norm_rotate<T, G, H>), dim3((unsigned)groups), dim3(256), 0, s, a);
        return hipGetLastError();
    };
    auto by_lanes = [&](auto zero, auto halves) {
        switch (pow2_from(a.d / 8, 32)) {
            case 1: return go(zero, std::integral_constant<int, 1>{}, halves);
            case 2: return go(zero, std::integral_constant<int, 2>{}, halves);
            case 4: return go(zero, std::integral_constant<int, 4>{}, halves);
            case 8: return go(zero, std::integral_constant<int, 8>{}, halves);
            case 16: return go(zero, std::integral_constant<int, 16>{}, halves);
            default: return go(zero, std::integral_constant<int, 32>{}, halves);
        }
    };
    const bool halves = !adjacent && a.rot > 0;
    const hipError_t e = dtype == 1 ? halves ? by_lanes(bf16_t{}, std::true_type{}) : by_lanes(bf16_t{}, std::false_type{})
                                    : halves ? by_lanes(float{}, std::true_type{}) : by_lanes(float{}, std::false_type{});
    if (e != hipSuccess || !backward || groups == 1) return e;
    hipLaunchKernelGGL(k_norm_rotate_join, dim3((unsigned)((4 * a.d + 63) / 64)), dim3(1024), 0, s, a, (int)groups);
    return hipGetLastError();
}

}  // namespace trimul
