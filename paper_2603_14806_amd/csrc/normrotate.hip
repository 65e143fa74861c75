// Norms of queries and keys by head with the position rotation, and their gradients (include/norm_rotate.h).
//
// A lane takes eight values of a row: four pairs that are turned together (halves: four values from each half), so that a
// rotation needs no other lane.  G lanes (the next power of two of d / 8) are a row, and sum over it by DPP.  The angles
// belong to the token: a wave turns all heads of its tokens, of the queries or of the keys, and where the entries of the
// batch share their positions those of several entries, with one sine and cosine a pair.
//
// What bounds it (kernel times, bf16): memory, and next to it the vector units, busy for 61 to 67% of the cycles with 140 to 160
// instructions for a wave's rows in the forward, 240 in the backward and with codes.  2 x 6000 tokens, 16 + 16 heads of 128, rms: 40 us (0.20 GB, 4.9
// TB/s; a 1 GiB copy reaches 5.1).  384 x 384 tokens, 4 + 4 heads of 32, layer: 36.5 us (0.15 GB, 4.1 TB/s; neighbouring
// pairs 34.4: half rows of 32 bytes are two accesses to each line) and backward 52 (0.23 GB, 4.3 TB/s).  4 x 2048 tokens with positions of
// their own, 16 + 4 heads of 128, to and from 8 bits: 28 and 33 us (0.11 GB each, 3.8 and 3.2 TB/s: an item has the rows of a
// token alone, and waits for its position and its rows once each).  4 single tokens: 4.2 us, a chain of two loads; 8192 with
// positions of their own 33 us (42 MB), since token slots of a wave are of one entry and stay empty (15 with one position for all).
// fp32: 2 x 6000 tokens 81 and 121 us (0.39 and 0.59 GB, 4.9 TB/s), 384 x 384 tokens 64 and 111 us (4.7 and 4.1 TB/s), 4 x 2048
// to and from 8 bits 46 and 48 us (0.19 GB, 4.1 and 3.9 TB/s).
#include <algorithm>
#include <type_traits>

#include "codes8.h"
#include "common.h"
#include "kernels.h"

// Products and sums are joined where the source says so and nowhere else: a row has the same bits whichever of the kernels
// below, and whichever place in its loop, it comes to.
#pragma clang fp contract(off)

namespace trimul {
namespace {

constexpr double kTwoOverPi = 0.63661977236758134308;

// cos and sin of p f, f in quarter turns.  The angle is reduced in 64 bits, where far positions keep their fraction:
// adding 1.5 2^52 rounds it to whole quarters (their number in the low bits), and at most half a quarter r is left
// either way.  There sin(pi / 2 r) = r S(r^2) and cos(pi / 2 r) = 1 + r^2 C(r^2) with cubics S and C through the
// Chebyshev points of [0, 1/4] (3.2e-9 and 1.9e-10 off; with float32's own rounding 1.5 2^-24 and 1.0 2^-24).
// (A library call for both made the forward of 2 x 6000 tokens, 16 + 16 heads of 128, bf16, 46.2 us that is 42.3 with this.)
__device__ __forceinline__ void turn(int p, double f, float& c, float& s) {
    constexpr double kWhole = 6755399441055744.0;
    const double t = (double)p * f, m = t + kWhole;
    const float r = (float)(t - (m - kWhole)), x = r * r;
    const uint32_t k = (uint32_t)__double2loint(m);
    const float b = r * __builtin_fmaf(__builtin_fmaf(__builtin_fmaf(-4.602149212632179e-3f, x, 7.968021764769763e-2f), x, -0.6459634776648043f), x, 1.5707963219532355f);
    const float a = __builtin_fmaf(__builtin_fmaf(__builtin_fmaf(__builtin_fmaf(9.067398957297847e-4f, x, -2.086152834093593e-2f), x, 0.253669410356929f), x, -1.2337005493742117f), x, 1.f);
    const bool odd = k & 1;
    c = __uint_as_float(__float_as_uint(odd ? b : a) ^ ((k + 1) << 30 & 0x80000000u));
    s = __uint_as_float(__float_as_uint(odd ? a : b) ^ (k << 30 & 0x80000000u));
}

// A lane's eight values as they lie in memory: four from each of two places (HALVES), or eight in a row.
template <typename T, bool HALVES> struct Raw {
    static constexpr int kWords = sizeof(T) == 4 ? 8 : 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0;
    }
    __device__ __forceinline__ void load(const T* p, int lo, int hi) {
        if constexpr (sizeof(T) == 4) {
            put(0, *reinterpret_cast<const uint4*>(p + lo));
            put(4, *reinterpret_cast<const uint4*>(p + (HALVES ? hi : lo + 4)));
        } else if constexpr (HALVES) {
            const uint2 a = *reinterpret_cast<const uint2*>(p + lo), b = *reinterpret_cast<const uint2*>(p + hi);
            w[0] = a.x; w[1] = a.y; w[2] = b.x; w[3] = b.y;
        } else {
            put(0, *reinterpret_cast<const uint4*>(p + lo));
        }
    }
    __device__ __forceinline__ void values(float (&f)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            f[i] = sizeof(T) == 4 ? __uint_as_float(w[i % kWords]) : __uint_as_float(i & 1 ? w[i / 2 % kWords] & 0xffff0000u : w[i / 2 % kWords] << 16);
    }
    static __device__ __forceinline__ void store(const float (&f)[8], T* p, int lo, int hi) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float4*>(p + lo) = make_float4(f[0], f[1], f[2], f[3]);
            *reinterpret_cast<float4*>(p + (HALVES ? hi : lo + 4)) = make_float4(f[4], f[5], f[6], f[7]);
        } else if constexpr (HALVES) {
            *reinterpret_cast<uint2*>(p + lo) = make_uint2(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]));
            *reinterpret_cast<uint2*>(p + hi) = make_uint2(pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
        } else {
            *reinterpret_cast<uint4*>(p + lo) = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
        }
    }
private:
    __device__ __forceinline__ void put(int i, uint4 x) { w[i % kWords] = x.x; w[(i + 1) % kWords] = x.y; w[(i + 2) % kWords] = x.z; w[(i + 3) % kWords] = x.w; }
};

// Pair m of a lane is (f[m], f[4 + m]) of halves, (f[2 m], f[2 m + 1]) of neighbours; back: by the negative angle.
template <bool HALVES, bool BACK>
__device__ __forceinline__ void rotate8(float (&f)[8], const float (&c)[4], const float (&s)[4]) {
#pragma unroll
    for (int m = 0; m < 4; ++m) {
        const float sine = BACK ? -s[m] : s[m];
        float& a = f[HALVES ? m : 2 * m];
        float& b = f[HALVES ? 4 + m : 2 * m + 1];
        const float ya = __builtin_fmaf(a, c[m], -(b * sine)), yb = __builtin_fmaf(b, c[m], a * sine);
        a = ya;
        b = yb;
    }
}

// What a lane of a wave has of every item.
struct Lane {
    int l, lo, hi;          // eighth of the row, and where its values are
    int head, token;        // slots
    bool live;              // the row has an eighth l (another lane reads the first one again, and counts for nothing)
};

template <int G, bool HALVES>
__device__ __forceinline__ Lane lane_of(const NormArgs& a, const NormSide& q) {
    const int lane = threadIdx.x % 64, slot = lane / G;
    Lane x;
    x.l = lane % G;
    x.live = 8 * x.l < a.d;
    x.head = slot & (q.slots - 1);
    x.token = slot / q.slots;
    const int l = x.live ? x.l : 0;
    const bool turned = HALVES && 8 * l < a.rot;
    x.lo = turned ? 4 * l : 8 * l;
    x.hi = turned ? a.rot / 2 + 4 * l : 8 * l + 4;
    return x;
}

// Eight of a side's weights, in the lane's places.
template <bool HALVES>
__device__ __forceinline__ void weights8(float (&f)[8], const void* w, bool bf16, const Lane& x, float none) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = none;
    if (!w) return;
    if (bf16) {
        Raw<bf16_t, HALVES> r;
        r.load(static_cast<const bf16_t*>(w), x.lo, x.hi);
        r.values(f);
    } else {
        Raw<float, HALVES> r;
        r.load(static_cast<const float*>(w), x.lo, x.hi);
        r.values(f);
    }
}

// u (in the place of x) and r of a row.
template <int G, bool LAYER>
__device__ __forceinline__ float normalise8(float (&f)[8], const NormArgs& a, bool live) {
    if constexpr (LAYER) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += f[i];
        const float total = sum_lanes<G>(sum);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = __builtin_fmaf(-total, a.inv_d, f[i]);
        if (a.ragged)
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = live ? f[i] : 0.f;
    }
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(f[i], f[i], sum);
    const float r = rsqrtf(__builtin_fmaf(sum_lanes<G>(sum), a.inv_d, a.eps));
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] *= r;
    return r;
}

// A wave's items: token tile and chunk of entries, as many items apart as there are waves on its side.
struct Item {
    int64_t tile, chunk;
    __device__ __forceinline__ Item(const NormArgs& a, const NormSide& q, bool keys) {
        const int64_t wave = (int64_t)(blockIdx.x - (keys ? a.side[0].groups : 0)) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        tile = wave % q.tiles;
        chunk = wave / q.tiles;
    }
    __device__ __forceinline__ void next(const NormSide& q) {
        tile += q.step_tile;
        chunk += q.step_chunk;
        if (tile >= q.tiles) {
            tile -= q.tiles;
            ++chunk;
        }
    }
};

// Where an item's rows are.
struct Place {
    int64_t token0, token, entry;      // the tile's first token, the lane's, the first entry
    int rows;
    __device__ __forceinline__ Place(const NormArgs& a, const NormSide& q, const Item& item, const Lane& x, int tokens)
        : token0(item.tile * tokens), token(token0 + x.token), entry(item.chunk * q.chunk), rows((int)min(q.chunk, a.batch - entry) * q.steps) {}
};

// The rows of a side in an item, one after the other: head steps of an entry, then the next entry.
struct Rows {
    int64_t entry;
    int step;
    __device__ __forceinline__ void next(int steps) {
        if (++step == steps) {
            step = 0;
            ++entry;
        }
    }
    // of a tensor: the part of a row's place that is the same for the wave, and the lane's own part
    __device__ __forceinline__ int64_t of(const NormSide& q, const CrossTensor& t, int64_t token0) const {
        return entry * t.batch + token0 * t.token + (int64_t)(step * q.slots) * t.head;
    }
    static __device__ __forceinline__ int64_t own(const CrossTensor& t, const Lane& x) { return x.token * t.token + x.head * t.head; }
    // the same of the row's number in contiguous codes and powers
    __device__ __forceinline__ int64_t number(const NormArgs& a, const NormSide& q, int64_t token0) const {
        return (entry * a.n + token0) * q.heads + step * q.slots;
    }
    static __device__ __forceinline__ int own_number(const NormSide& q, const Lane& x) { return x.token * q.heads + x.head; }
};

// The angles' part of an item: the position is asked for early, the sines follow when the rows are on their way.
struct Angles {
    double f[4];
    int p;                  // the position that was asked for last
    __device__ __forceinline__ Angles(const NormArgs& a, const Lane& x) : p(0) {
        const bool turned = x.live && 8 * x.l < a.rot;
#pragma unroll
        for (int m = 0; m < 4; ++m) f[m] = turned ? a.freqs[4 * x.l + m] * kTwoOverPi : 0.0;
    }
    __device__ __forceinline__ void ask(const NormArgs& a, const Place& at) {
        if (a.rot && at.token < a.n) p = a.positions[at.entry * a.positions_batch + at.token];
    }
    __device__ __forceinline__ void get(const NormArgs& a, float (&c)[4], float (&s)[4]) const {
        if (a.rot == 0) return;
#pragma unroll
        for (int m = 0; m < 4; ++m) turn(p, f[m], c[m], s[m]);
    }
};

// Four rows are in flight while four are worked on, side by side (single ones at the end).  The rows of the next item are
// not asked for ahead: that takes 130 registers, and 12 waves a compute unit or spills (53 and 43.6 us for the 40 above).
template <typename T, int G, bool HALVES, bool LAYER, bool HOLD>
__global__ __launch_bounds__(256, sizeof(T) == 2 && !HOLD ? 4 : 3) void k_norm_rotate(const NormArgs a) {
    constexpr int U = 4;
    const bool keys = blockIdx.x >= a.side[0].groups;
    const NormSide& q = a.side[keys];
    const Lane x = lane_of<G, HALVES>(a, q);
    const int tokens = 64 / G / q.slots;
    Angles angles(a, x);
    float gain[8], shift[8];
    weights8<HALVES>(gain, q.gain, a.weight_bf16, x, 1.f);
    weights8<HALVES>(shift, q.shift, a.weight_bf16, x, 0.f);
    const int64_t own_x = Rows::own(q.x, x), own_y = Rows::own(q.y, x);
    const int own_number = Rows::own_number(q, x);
    Raw<T, HALVES> raw[U];
    auto load = [&](const Place& at, Rows& row, int left) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            raw[u].clear();
            if (u < left && at.token < a.n && row.step * q.slots + x.head < q.heads)
                raw[u].load(static_cast<const T*>(q.x.data) + row.of(q, q.x, at.token0) + own_x, x.lo, x.hi);
            row.next(q.steps);
        }
    };
    for (Item item(a, q, keys); item.chunk < q.chunks; item.next(q)) {
        const Place here(a, q, item, x, tokens);
        const int64_t token0 = here.token0, token = here.token;
        angles.ask(a, here);
        Rows ahead{here.entry, 0}, row{here.entry, 0};
        load(here, ahead, here.rows);
        float c[4] = {1.f, 1.f, 1.f, 1.f}, s[4] = {0.f, 0.f, 0.f, 0.f};
        angles.get(a, c, s);
        auto work = [&](auto count, const Raw<T, HALVES>* now) {
            constexpr int N = decltype(count)::value;
            float v[N][8];
            bool live[N];
            Rows at[N];
#pragma unroll
            for (int u = 0; u < N; ++u) {
                at[u] = row;
                live[u] = token < a.n && row.step * q.slots + x.head < q.heads && x.live;
                row.next(q.steps);
                now[u].values(v[u]);
                if (a.ragged)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[u][e] = x.live ? v[u][e] : 0.f;
            }
            if (HOLD && q.codes) {
#pragma unroll
                for (int u = 0; u < N; ++u) {
                    uint32_t top = 0;
#pragma unroll
                    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[u][e]) & 0x7fffffffu);
                    top = umax_lanes<G>(top);
                    const uint32_t byte = power_byte(top);
                    const float inverse = power_inverse(byte);
                    uint32_t lo, hi;
                    if (power_cut(top)) {
                        float w[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) w[e] = fminf(fmaxf(v[u][e], -kTopValue), kTopValue);
                        lo = codes4(w[0], w[1], w[2], w[3], inverse);
                        hi = codes4(w[4], w[5], w[6], w[7], inverse);
                    } else {
                        lo = codes4(v[u][0], v[u][1], v[u][2], v[u][3], inverse);
                        hi = codes4(v[u][4], v[u][5], v[u][6], v[u][7], inverse);
                    }
                    if (!live[u]) continue;
                    const int64_t number = at[u].number(a, q, token0);
                    int8_t* to = q.codes + number * a.d + own_number * a.d;
                    if constexpr (HALVES) {
                        *reinterpret_cast<uint32_t*>(to + x.lo) = lo;
                        *reinterpret_cast<uint32_t*>(to + x.hi) = hi;
                    } else {
                        *reinterpret_cast<uint2*>(to + x.lo) = make_uint2(lo, hi);
                    }
                    if (x.l == 0) (q.powers + number)[own_number] = (uint8_t)byte;
                }
            }
#pragma unroll
            for (int u = 0; u < N; ++u) {
                normalise8<G, LAYER>(v[u], a, x.live);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[u][e] = __builtin_fmaf(v[u][e], gain[e], shift[e]);
                rotate8<HALVES, false>(v[u], c, s);
            }
#pragma unroll
            for (int u = 0; u < N; ++u)
                if (live[u]) Raw<T, HALVES>::store(v[u], static_cast<T*>(q.y.data) + at[u].of(q, q.y, token0) + own_y, x.lo, x.hi);
        };
        for (int i = 0; i < here.rows; i += U) {
            Raw<T, HALVES> now[U];
#pragma unroll
            for (int u = 0; u < U; ++u) now[u] = raw[u];
            if (i + U < here.rows) load(here, ahead, here.rows - i - U);
            if (i + U <= here.rows) {
                work(std::integral_constant<int, U>{}, now);
            } else {
#pragma unroll
                for (int u = 0; u < U - 1; ++u)
                    if (i + u < here.rows) work(std::integral_constant<int, 1>{}, now + u);
            }
        }
    }
}

// A lane's eight inputs of the backward: values, or codes and their power.
template <typename T, bool HALVES, bool HELD> struct Input {
    Raw<T, HALVES> raw;
    __device__ __forceinline__ void clear() { raw.clear(); }
    __device__ __forceinline__ void values(float (&f)[8]) const { raw.values(f); }
};
template <typename T, bool HALVES> struct Input<T, HALVES, true> {
    uint32_t lo, hi, byte;
    __device__ __forceinline__ void clear() { lo = hi = byte = 0; }
    __device__ __forceinline__ void values(float (&f)[8]) const {
        const float scale = power_value(byte);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f[e] = code_value(lo, e) * scale;
            f[4 + e] = code_value(hi, e) * scale;
        }
    }
};

template <typename T, int G, bool HALVES, bool LAYER, bool HELD>
__global__ __launch_bounds__(256) void k_norm_rotate_backward(const NormArgs a) {
    constexpr int U = 2;
    __shared__ float sums[4][2][256];                       // by wave: dgain and dshift
    const bool keys = blockIdx.x >= a.side[0].groups;
    const NormSide& q = a.side[keys];
    const Lane x = lane_of<G, HALVES>(a, q);
    const int tokens = 64 / G / q.slots, w = threadIdx.x / 64;
    Angles angles(a, x);
    float total[2][8], gain[8];
    weights8<HALVES>(gain, q.gain, a.weight_bf16, x, 1.f);
#pragma unroll
    for (int e = 0; e < 8; ++e) total[0][e] = total[1][e] = 0.f;
    const int64_t own_x = Rows::own(q.x, x), own_y = Rows::own(q.y, x), own_dx = Rows::own(q.dx, x);
    const int own_number = Rows::own_number(q, x);
    Input<T, HALVES, HELD> in[U];
    Raw<T, HALVES> dy[U];
    auto load = [&](const Place& at, Rows& row, int left) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            in[u].clear();
            dy[u].clear();
            if (u < left && at.token < a.n && row.step * q.slots + x.head < q.heads) {
                if constexpr (HELD) {
                    const int64_t number = row.number(a, q, at.token0);
                    const int8_t* from = q.codes + number * a.d + own_number * a.d;
                    if constexpr (HALVES) {
                        in[u].lo = *reinterpret_cast<const uint32_t*>(from + x.lo);
                        in[u].hi = *reinterpret_cast<const uint32_t*>(from + x.hi);
                    } else {
                        const uint2 both = *reinterpret_cast<const uint2*>(from + x.lo);
                        in[u].lo = both.x;
                        in[u].hi = both.y;
                    }
                    in[u].byte = (q.powers + number)[own_number];
                } else {
                    in[u].raw.load(static_cast<const T*>(q.x.data) + row.of(q, q.x, at.token0) + own_x, x.lo, x.hi);
                }
                dy[u].load(static_cast<const T*>(q.y.data) + row.of(q, q.y, at.token0) + own_y, x.lo, x.hi);
            }
            row.next(q.steps);
        }
    };
    for (Item item(a, q, keys); item.chunk < q.chunks; item.next(q)) {
        const Place here(a, q, item, x, tokens);
        const int64_t token0 = here.token0, token = here.token;
        angles.ask(a, here);
        Rows ahead{here.entry, 0}, row{here.entry, 0};
        load(here, ahead, here.rows);
        float c[4] = {1.f, 1.f, 1.f, 1.f}, s[4] = {0.f, 0.f, 0.f, 0.f};
        angles.get(a, c, s);
        auto work = [&](auto count, const Input<T, HALVES, HELD>* in_now, const Raw<T, HALVES>* dy_now) {
            constexpr int N = decltype(count)::value;
            float v[N][8], g[N][8];
#pragma unroll
            for (int u = 0; u < N; ++u) {
                in_now[u].values(v[u]);
                dy_now[u].values(g[u]);
                if (a.ragged)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        v[u][e] = x.live ? v[u][e] : 0.f;
                        g[u][e] = x.live ? g[u][e] : 0.f;
                    }
            }
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const float r = normalise8<G, LAYER>(v[u], a, x.live);
                rotate8<HALVES, true>(g[u], c, s);
                float along = 0.f, mean = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    total[1][e] += g[u][e];
                    total[0][e] = __builtin_fmaf(g[u][e], v[u][e], total[0][e]);
                    g[u][e] *= gain[e];
                    along = __builtin_fmaf(g[u][e], v[u][e], along);
                    if constexpr (LAYER) mean += g[u][e];
                }
                along = sum_lanes<G>(along) * (a.inv_d * r);
                if constexpr (LAYER) mean = sum_lanes<G>(mean) * (a.inv_d * r);
#pragma unroll
                for (int e = 0; e < 8; ++e) g[u][e] = __builtin_fmaf(g[u][e], r, -__builtin_fmaf(v[u][e], along, mean));
            }
#pragma unroll
            for (int u = 0; u < N; ++u) {
                if (token < a.n && row.step * q.slots + x.head < q.heads && x.live)
                    Raw<T, HALVES>::store(g[u], static_cast<T*>(q.dx.data) + row.of(q, q.dx, token0) + own_dx, x.lo, x.hi);
                row.next(q.steps);
            }
        };
        for (int i = 0; i < here.rows; i += U) {
            Input<T, HALVES, HELD> in_now[U];
            Raw<T, HALVES> dy_now[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                in_now[u] = in[u];
                dy_now[u] = dy[u];
            }
            if (i + U < here.rows) load(here, ahead, here.rows - i - U);
            if (i + U <= here.rows) work(std::integral_constant<int, U>{}, in_now, dy_now);
            else work(std::integral_constant<int, 1>{}, in_now, dy_now);
        }
    }
    // over the rows of the wave, then over the waves
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float t = total[k][e];
#pragma unroll
            for (int m = G; m < 64; m *= 2) t += __shfl_xor(t, m);
            if (threadIdx.x % 64 < G && x.live) sums[w][k][(e < 4 ? x.lo : x.hi - 4) + e] = t;
        }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * a.d; i += 256) {
        const int k = i / a.d, e = i - k * a.d;
        const float t = sums[0][k][e] + sums[1][k][e] + (sums[2][k][e] + sums[3][k][e]);
        if (q.groups == 1) {
            float* to = k ? q.dshift : q.dgain;
            if (to) to[e] = t;
        } else {
            a.part[(int64_t)blockIdx.x * 2 * a.d + i] = t;
        }
    }
}

// The weights' gradients from the work-groups' sums: a lane for each value, a wave for every 16th work-group.
__global__ __launch_bounds__(1024) void k_norm_rotate_join(const NormArgs a) {
    __shared__ double sums[16][64];
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, i = blockIdx.x * 64 + lane;
    const int side = i / (2 * a.d), k = i / a.d % 2, e = i % a.d;
    float* to = side < 2 ? (k ? a.side[side].dshift : a.side[side].dgain) : nullptr;
    double sum = 0;
    if (to) {
        const float* part = a.part + ((int64_t)(side ? a.side[0].groups : 0) * 2 + k) * a.d + e;
        const int groups = a.side[side].groups;
        if (groups == 1) to = nullptr;                      // (it has written its own)
#pragma unroll 8
        for (int g = wave; g < groups; g += 16) sum += part[(int64_t)g * 2 * a.d];
    }
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

// Lanes of a row: the next power of two of d / 8, and 4 for 8 and 16 channels too (heads that narrow are not worth kernels
// of their own).
int lanes_of(int d) { return d <= 32 ? 4 : pow2_from(d / 8, 32); }

int64_t up(int64_t n, int64_t d) { return (n + d - 1) / d; }

// Work-groups, and in a how the tokens, heads and entries lie on the waves.  A work-group has the queries or the keys.
int64_t plan(NormArgs& a, int dtype, bool backward) {
    const int rows = 64 / lanes_of(a.d);                        // of a wave at once
    const bool shared = a.positions_batch == 0 || a.rot == 0;
    const bool few = a.batch * a.n * (a.side[0].heads + a.side[1].heads) < 4096 * (int64_t)rows;
    int64_t work[2], total = 0;
    for (int i = 0; i < 2; ++i) {
        NormSide& q = a.side[i];
        // An item should have several rows for its angles, which take as long as one, and a second group of rows to ask
        // for: several entries, or, where each has its own positions, fewer heads at once (of 128 bytes at least) and up to
        // eight head steps (four: 30.8 us in place of 28.2 for the forward to 8 bits above).  Not where the rows are too few
        // to fill the waves: there steps are latency (4 single tokens of 16 + 4 heads of 64: eight steps 7.5 us, two 4.2).
        const int least = shared || few ? rows : pow2_from((int)up(128, a.d * (dtype == 1 ? 2 : 4)), rows);
        q.slots = pow2_from(shared || few ? q.heads : std::max((int)up(q.heads, 8), std::min(least, q.heads)), rows);
        q.steps = (int)up(q.heads, q.slots);
        q.tiles = up(a.n, rows / q.slots);
        work[i] = a.batch * q.tiles * q.steps;
        total += work[i];
    }
    // Waves that go round: 16 for each compute unit, 12 in the backward, as many as its registers let be there at once.  (The
    // forward in fp32 or with codes has 12 there at once too, and takes its last quarter in a second round: 2 x 6000 tokens,
    // 16 + 16 heads of 128, fp32 81 us where 12 take 72, bf16 to 8 bits 70 and 58.5.)  A forward whose entries have their own
    // positions has short items, and a wave for each.
    const int64_t waves = 256 * (backward ? 12 : 16);
    for (int i = 0; i < 2; ++i) {
        NormSide& q = a.side[i];
        q.chunk = shared && q.heads ? std::min(a.batch, up(std::max<int64_t>(4, total / (8 * waves)), q.steps)) : 1;
        q.chunks = up(a.batch, q.chunk);
        const int64_t groups = up(q.tiles * q.chunks, 4);
        q.groups = q.heads ? (int)std::min(groups, backward || shared ? std::max<int64_t>(1, waves / 4 * work[i] / total) : int64_t(1) << 22) : 0;
        if (q.heads) {
            q.step_chunk = 4 * (int64_t)q.groups / q.tiles;
            q.step_tile = 4 * (int64_t)q.groups % q.tiles;
        }
    }
    return (int64_t)a.side[0].groups + a.side[1].groups;
}

}  // namespace

int64_t norm_rotate_backward_groups(NormArgs a, int dtype) { return plan(a, dtype, true); }

hipError_t launch_norm_rotate(int dtype, bool adjacent, bool backward, NormArgs a, hipStream_t s) {
    if (a.batch == 0 || a.n == 0) {
        if (!backward) return hipSuccess;
        hipLaunchKernelGGL(k_norm_rotate_zero, dim3(1), dim3(256), 0, s, a);
        return hipGetLastError();
    }
    const int64_t groups = plan(a, dtype, backward);
    a.inv_d = 1.f / (float)a.d;
    a.ragged = 8 * lanes_of(a.d) != a.d;
    const bool held = backward && !a.side[a.side[0].heads ? 0 : 1].x.data;
    const bool hold = a.side[0].codes || a.side[1].codes;
    auto go = [&](auto zero, auto lanes, auto halves, auto layer) {
        using T = decltype(zero);
        constexpr int G = decltype(lanes)::value;
        constexpr bool H = decltype(halves)::value, L = decltype(layer)::value;
        const dim3 grid((unsigned)groups), block(256);
        if (backward) {
            if (held) hipLaunchKernelGGL((k_norm_rotate_backward<T, G, H, L, true>), grid, block, 0, s, a);
            else hipLaunchKernelGGL((k_norm_rotate_backward<T, G, H, L, false>), grid, block, 0, s, a);
        } else {
            if (hold) hipLaunchKernelGGL((k_norm_rotate<T, G, H, L, true>), grid, block, 0, s, a);
            else hipLaunchKernelGGL((k_norm_rotate<T, G, H, L, false>), grid, block, 0, s, a);
        }
        return hipGetLastError();
    };
    auto by_lanes = [&](auto zero, auto halves) {
        auto by_norm = [&](auto lanes) { return a.layer ? go(zero, lanes, halves, std::true_type{}) : go(zero, lanes, halves, std::false_type{}); };
        switch (lanes_of(a.d)) {
            case 4: return by_norm(std::integral_constant<int, 4>{});
            case 8: return by_norm(std::integral_constant<int, 8>{});
            case 16: return by_norm(std::integral_constant<int, 16>{});
            default: return by_norm(std::integral_constant<int, 32>{});
        }
    };
    const bool halves = !adjacent && a.rot > 0;
    const hipError_t e = dtype == 1 ? halves ? by_lanes(bf16_t{}, std::true_type{}) : by_lanes(bf16_t{}, std::false_type{})
                                    : halves ? by_lanes(float{}, std::true_type{}) : by_lanes(float{}, std::false_type{});
    if (e != hipSuccess || !backward || (a.side[0].groups < 2 && a.side[1].groups < 2)) return e;
    hipLaunchKernelGGL(k_norm_rotate_join, dim3((unsigned)((4 * a.d + 63) / 64)), dim3(1024), 0, s, a);
    return hipGetLastError();
}

}  // namespace trimul
