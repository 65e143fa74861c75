// Relative position bias by buckets and the gradient of its table (include/relative_bias.h).
//
// Both forms of the forward are a look-up in LDS beside a stream of stores (and of the base's loads).  The gradient is
// a sum by bucket: every lane adds into a column of LDS of its own, so that no two lanes meet, the order of the
// sums is fixed, and no two lanes of a wave share a bank.  They read, add and write: LDS's own float additions take about
// 200 cycles of a compute unit for a wave's 64 (169 us for the gradient of 1300 x 1300 x 16 that takes 39 now).
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "kernels.h"
#include "vec.h"

namespace trimul {
namespace {

// The place of distance p_k - p_q in the look-up table, [0, 2 reach].
__device__ __forceinline__ int distance_index(int pk, int pq, int reach) {
    return min(max(__builtin_elementwise_sub_sat(pk, pq), -reach), reach) + reach;
}

// Work-groups go to the eight XCDs in turn; this gives each XCD neighbouring ones, so that lines which two of them share
// (rows that are no multiple of 128 bytes) meet in one L2.
__device__ __forceinline__ int64_t by_xcd(uint32_t group, uint32_t groups) {
    const uint32_t per = groups / 8, rest = groups % 8, x = group % 8, i = group / 8;
    return (int64_t)x * per + min(x, rest) + i;
}

// Lanes take eight neighbouring keys each, usually at eight neighbouring distances: with one place left free after
// every eight, the lanes of a wave read different banks.
__device__ __forceinline__ int skewed(int i) { return i + (i >> 3); }

__device__ __forceinline__ float table_value(const RelativeArgs& a, int row, int col) {
    const int64_t at = (int64_t)row * a.heads + col;
    return a.table_bf16 ? bf2f(static_cast<const bf16_t*>(a.table)[at]) : static_cast<const float*>(a.table)[at];
}

__device__ __forceinline__ int bucket_of(const RelativeArgs& a, int index) { return min((int)a.lut[index], a.buckets - 1); }

// val[h * stride + skewed(i)]: what head h0 + h (h < nh of HB) adds at distance index i, and behind the last index what it
// adds in another segment.  Look-ups that depend on each other, so several of them are under way at once.
template <int HB>
__device__ __forceinline__ void values_by_distance(const RelativeArgs& a, float* val, int h0, int nh, int entries, int stride, int threads) {
    constexpr int U = 4;
    for (int e0 = threadIdx.x; e0 < entries * HB; e0 += U * threads) {
        int row[U];
        float x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = min((e0 + u * threads) / HB, entries - 1);
            row[u] = i == entries - 1 ? a.buckets - 1 : bucket_of(a, i);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = table_value(a, row[u], h0 + min((e0 + u * threads) % HB, nh - 1));
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int e = e0 + u * threads;
            if (e < entries * HB) val[e % HB * stride + skewed(e / HB)] = x[u];
        }
    }
}

__device__ __forceinline__ void lut_to_lds(const RelativeArgs& a, uint8_t* lut, int threads) {
    for (int e = threadIdx.x; e <= 2 * a.reach; e += threads) lut[e] = (uint8_t)bucket_of(a, e);
}
__device__ __forceinline__ void zero_lds(float* p, int n, int threads) {      // n a multiple of 4
    for (int e = 4 * threadIdx.x; e < n; e += 4 * threads) *reinterpret_cast<float4*>(p + e) = make_float4(0.f, 0.f, 0.f, 0.f);
}

// Eight integers of which the first n exist (the last stands for the rest); wide: p is 16-byte aligned.
__device__ __forceinline__ void eight(const int32_t* p, int n, bool wide, int (&v)[8]) {
    if (wide && n >= 8) {
        const int4 x = reinterpret_cast<const int4*>(p)[0], y = reinterpret_cast<const int4*>(p)[1];
        v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
        v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = p[min(i, n - 1)];
    }
}

// A lane's eight keys: the first of them, and how many exist (0: the lane is past the end, and is given the first keys to
// look at).  whole: every lane of the wave has eight or none, which a vector load can take.
struct KeyPlace {
    int64_t j;
    int n;
    bool whole;
    __device__ __forceinline__ KeyPlace(const RelativeArgs& a, int64_t chunk) {
        const int64_t left = a.nk - 8 * chunk;
        j = left > 0 ? 8 * chunk : 0;
        n = left >= 8 ? 8 : left > 0 ? (int)left : 0;
        whole = a.wide && a.nk >= 8 && __ballot(n > 0 && n < 8) == 0;
    }
};

// Eight neighbouring keys (n of them exist, the last stands for the rest): positions, segments, and whether all have one
// distance index to a query.  The index does not fall as the position rises, so the first and the last decide.
template <bool SEG> struct Keys {
    int pos[8], seg[8], least, most;
    bool alike;       // one segment
    __device__ __forceinline__ Keys(const RelativeArgs& a, int64_t b, int64_t j, int n) {
        eight(a.pos_k + b * a.pos_k_batch + j, n, a.wide_keys, pos);
        if constexpr (SEG) eight(a.seg_k + b * a.seg_k_batch + j, n, a.wide_keys, seg);
        least = most = pos[0];
        alike = true;
#pragma unroll
        for (int i = 1; i < 8; ++i) {
            least = min(least, pos[i]);
            most = max(most, pos[i]);
            if constexpr (SEG) alike = alike && seg[i] == seg[0];
        }
    }
    // The index that all eight have, other where the segments differ; -1 if there is none.
    __device__ __forceinline__ int common(int pq, int sq, int reach, int other) const {
        const int i = distance_index(least, pq, reach);
        if constexpr (SEG) {
            bool any = seg[0] == sq;
            if (!alike)
#pragma unroll
                for (int e = 1; e < 8; ++e) any = any || seg[e] == sq;
            if (!any) return other;
            if (!alike) return -1;
        }
        return i == distance_index(most, pq, reach) ? i : -1;
    }
    __device__ __forceinline__ int index(int i, int pq, int sq, int reach, int other) const {
        return SEG && seg[i] != sq ? other : distance_index(pos[i], pq, reach);
    }
};

// ---------------------------------------------------------------- bias [batch][heads][nq][nk]

// A work-group: HB heads, a.tx threads along the keys (eight each), 256 / a.tx rows at a time, a.loop times.  Where all
// lanes of a wave have keys of one distance index each, as away from the diagonal, a head is one look-up.
// Bound by memory, and by each work-group's start (table and positions into LDS: about 5 us at a reach of 32, and with the reach
// more of it: 8 x 1786 x 523, 3 heads, bf16, 19 us at 128 and 27 at 1000, 45 MB).  16 heads, bf16: 1300 x 1300 18 us (54 MB
// written, 3.0 TB/s), 2048 x 3000 46 us (0.20 GB, 4.3 TB/s), the same with a base 101 us (0.39 GB, 3.9 TB/s); fp32: 36 us (3.0 TB/s),
// 122 us (0.39 GB, 3.2 TB/s) and 224 us (0.79 GB, 3.5 TB/s).
template <typename T, bool SEG, bool BASE, int HB>
__global__ __launch_bounds__(256) void k_relative_bias(const RelativeArgs a) {
    extern __shared__ float val[];
    int64_t at = by_xcd(blockIdx.x, gridDim.x);
    const int cb = (int)(at % a.cblocks);
    at /= a.cblocks;
    const int rb = (int)(at % a.rblocks);
    at /= a.rblocks;
    const int hg = (int)(at % a.hblocks);
    const int64_t b = at / a.hblocks;
    const int h0 = hg * HB, nh = min(HB, a.heads - h0);
    const int other = 2 * a.reach + 1, stride = skewed(other + 1) + 1;
    values_by_distance<HB>(a, val, h0, nh, other + 1, stride, 256);
    const int tx = threadIdx.x & (a.tx - 1), ty = threadIdx.x / a.tx, rows = 256 / a.tx;
    const KeyPlace at_keys(a, (int64_t)cb * a.tx + tx);
    const int64_t j = at_keys.j;
    const int n = at_keys.n;
    const bool whole = at_keys.whole;
    const Keys<SEG> keys(a, b, j, max(n, 1));
    __syncthreads();
    const T* base = static_cast<const T*>(a.base.data) + b * a.base.batch + h0 * a.base.head + j;
    T* out = static_cast<T*>(a.out.data) + b * a.out.batch + h0 * a.out.head + j;
    const int64_t r0 = (int64_t)rb * rows * a.loop, r1 = min(r0 + (int64_t)rows * a.loop, a.nq);
    constexpr int N = HB < 4 ? HB : 4;                  // heads at once
    for (int64_t r = r0 + ty; r < r1; r += rows) {
        const int pq = a.pos_q[b * a.pos_q_batch + r], sq = SEG ? a.seg_q[b * a.seg_q_batch + r] : 0;
        const T* from = base + r * a.base.row;
        T* to = out + r * a.out.row;
        const int common = keys.common(pq, sq, a.reach, other);
        int idx[8];
        const bool one = __ballot(common < 0) == 0;
        idx[0] = skewed(common);
        if (!one)
#pragma unroll
            for (int i = 0; i < 8; ++i) idx[i] = skewed(keys.index(i, pq, sq, a.reach, other));
        for (int h = 0; h < nh; h += N) {
            Vec<T, 8> v[N];
            if constexpr (BASE) {
                Words<T, 8> w[N];
                if (whole)
#pragma unroll
                    for (int u = 0; u < N; ++u) w[u].load(from + min(h + u, nh - 1) * a.base.head);
                else
#pragma unroll
                    for (int u = 0; u < N; ++u) w[u].load_some(from + min(h + u, nh - 1) * a.base.head, n);
#pragma unroll
                for (int u = 0; u < N; ++u) v[u] = w[u].values();
            }
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const float* t = val + min(h + u, nh - 1) * stride;
                if (one) {
                    const float x = t[idx[0]];
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[u].f[i] = BASE ? v[u].f[i] + x : x;
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[u].f[i] = BASE ? v[u].f[i] + t[idx[i]] : t[idx[i]];
                }
            }
#pragma unroll
            for (int u = 0; u < N; ++u)
                if (h + u < nh) store_some(v[u], to + (h + u) * a.out.head, n, a.wide);
        }
    }
}

// A work-group: one head of a.loop entries, the rows of one split; a wave: a.span times the keys of its lanes.  A lane has
// a column of LDS for itself, a place for each bucket and one for what is not to be kept.
//   Away from the diagonal a lane's eight keys have one distance index: their sum stays in a register while its bucket
//   does not change.  Near it a lane's buckets usually rise or fall: equal neighbours are added up, and the eight
//   places, all different then, are read, added to and written together.  Otherwise one after the other.
// Bound by waiting: seven to twelve waves a compute unit, as LDS holds their columns, with one set of loads ahead each.  bf16, 16
// heads, 66 buckets: 1300 x 1300 32 us in one chain, 39 in five (54 MB, 1.7 and 1.4 TB/s); 32 buckets, 2048 x 3000 73 us (2.7 TB/s);
// 1500 windows of 32 x 128, 4 heads, 38 us (a work-group for each entry: 63, and 14 for their sums in place of 5).
template <typename T, bool SEG>
__global__ __launch_bounds__(256) void k_relative_bias_backward(const RelativeArgs a) {
    extern __shared__ float val[];
    constexpr int U = 4;
    const int columns = (a.buckets + 1) * 64;
    uint8_t* lut = reinterpret_cast<uint8_t*>(val + (size_t)a.waves * columns);
    int64_t at = by_xcd(blockIdx.x, gridDim.x);
    const int group = (int)(at % a.cblocks);
    at /= a.cblocks;
    const int split = (int)(at % a.splits);
    at /= a.splits;
    const int h = (int)(at % a.heads);
    const int64_t part_of_batch = at / a.heads, b1 = min((part_of_batch + 1) * a.loop, a.batch);
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, threads = a.waves * 64;
    const int other = 2 * a.reach + 1;                   // (its place in lut holds the last bucket)
    lut_to_lds(a, lut, threads);
    if (threadIdx.x == 0) lut[other] = (uint8_t)(a.buckets - 1);
    zero_lds(val, a.waves * columns, threads);
    __syncthreads();
    float* acc = val + wave * columns + lane;
    const int tx = lane & (a.tx - 1), ty = lane / a.tx, rows = 64 / a.tx;
    const int64_t per = (a.nq + a.splits - 1) / a.splits, r0 = split * per, r1 = min(r0 + per, a.nq);
    int cur = a.buckets;                                 // the bucket of `sum` (at first: none)
    float sum = 0.f;
    for (int64_t b = part_of_batch * a.loop; b < b1; ++b) {
        const T* from = static_cast<const T*>(a.out.data) + b * a.out.batch + h * a.out.head;
        const int32_t* pos_q = a.pos_q + b * a.pos_q_batch;
        const int32_t* seg_q = SEG ? a.seg_q + b * a.seg_q_batch : nullptr;
        for (int k = 0; k < a.span; ++k) {
            const int64_t c = ((int64_t)group * a.waves + wave) * a.span + k;
            if (c * a.tx * 8 >= a.nk) break;
            const KeyPlace at_keys(a, c * a.tx + tx);
            const int64_t j = at_keys.j;
            const int n = at_keys.n;
            const Keys<SEG> keys(a, b, j, max(n, 1));
            Words<T, 8> ahead[U];
            int pq_ahead[U], sq_ahead[U];
            auto load = [&](int64_t first) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int64_t r = min(first + ty + u * rows, r1 - 1);
                    if (at_keys.whole) ahead[u].load(from + r * a.out.row + j);
                    else ahead[u].load_some(from + r * a.out.row + j, n);
                    pq_ahead[u] = pos_q[r];
                    sq_ahead[u] = SEG ? seg_q[r] : 0;
                }
            };
            if (r0 < r1) load(r0);
            for (int64_t first = r0; first < r1; first += U * rows) {
                Vec<T, 8> v[U];
                int pq[U], sq[U], common[U];
                const bool some = __ballot(n == 0) != 0 || first + U * rows > r1;       // lanes or rows that count for nothing
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    v[u] = ahead[u].values();
                    if (some)
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[u].f[i] = n > 0 && first + ty + u * rows < r1 ? v[u].f[i] : 0.f;
                    pq[u] = pq_ahead[u];
                    sq[u] = sq_ahead[u];
                }
                if (first + U * rows < r1) load(first + U * rows);
#pragma unroll
                for (int u = 0; u < U; ++u) common[u] = keys.common(pq[u], sq[u], a.reach, other);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const float* f = v[u].f;
                    if (__ballot(common[u] < 0) == 0) {
                        const int t = lut[common[u]];
                        const float x = ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
                        if (__ballot(t != cur) == 0) {
                            sum += x;
                        } else {
                            acc[cur * 64] += sum;
                            cur = t;
                            sum = x;
                        }
                        continue;
                    }
                    int t[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) t[i] = lut[keys.index(i, pq[u], sq[u], a.reach, other)];
                    bool rises = true, falls = true;
#pragma unroll
                    for (int i = 1; i < 8; ++i) {
                        rises = rises && t[i] >= t[i - 1];
                        falls = falls && t[i] <= t[i - 1];
                    }
                    if (__ballot(!(rises || falls)) == 0) {
                        float x[8], old[8];
                        int to[8];
                        x[0] = f[0];
#pragma unroll
                        for (int i = 1; i < 8; ++i) x[i] = t[i] == t[i - 1] ? x[i - 1] + f[i] : f[i];
#pragma unroll
                        for (int i = 0; i < 8; ++i) to[i] = (i < 7 && t[i] == t[(i + 1) & 7] ? a.buckets : t[i]) * 64;
#pragma unroll
                        for (int i = 0; i < 8; ++i) old[i] = acc[to[i]];
#pragma unroll
                        for (int i = 0; i < 8; ++i) acc[to[i]] = old[i] + x[i];
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i) acc[t[i] * 64] += f[i];
                    }
                }
            }
        }
    }
    acc[cur * 64] += sum;
    __syncthreads();
    // a bucket's columns: eight lanes, each eight columns of every wave, in an order that keeps the banks apart
    for (int e = threadIdx.x; e < (a.buckets + 7) / 8 * 64; e += threads) {
        const int t = e / 8, part = e % 8;
        double sum = 0;
        if (t < a.buckets)
            for (int w = 0; w < a.waves; ++w)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += val[w * columns + t * 64 + part * 8 + ((i + t) & 7)];
#pragma unroll
        for (int m = 1; m < 8; m *= 2) sum += __shfl_xor(sum, m);
        if (t < a.buckets && part == 0) {
            if (a.loop >= a.batch && a.splits * a.cblocks == 1) a.dtable[(int64_t)t * a.heads + h] = (float)sum;
            else a.part[(((part_of_batch * a.splits + split) * a.cblocks + group) * a.heads + h) * a.buckets + t] = (float)sum;
        }
    }
}

// dtable from `slots` partial tables [heads][buckets]: a lane for each value, a wave for every 16th slot.
__global__ __launch_bounds__(1024) void k_relative_join(const RelativeArgs a, int64_t slots) {
    __shared__ double sums[16][64];
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, n = a.heads * a.buckets;
    const int e = blockIdx.x * 64 + lane;
    double sum = 0;
    if (e < n)
#pragma unroll 8
        for (int64_t s = wave; s < slots; s += 16) sum += a.part[s * n + e];
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && e < n) {
        for (int w = 1; w < 16; ++w) sum += sums[w][lane];
        const int h = e / a.buckets, t = e - h * a.buckets;
        a.dtable[(int64_t)t * a.heads + h] = (float)sum;
    }
}

__global__ __launch_bounds__(256) void k_relative_zero(float* p, int64_t n) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < n) p[i] = 0.f;
}

// ---------------------------------------------------------------- pair [nq][nk][channels]

// Bound by memory: 2048 x 2048 x 128 bf16 with a base 435 us (2.1 GB, 4.9 TB/s), 500 x 700 x 128 fp32 84 us (4.2 TB/s).
// A work-group: channels [cb * a.cwidth, + a.cwidth) of 4 * 256 / a.tx columns and a.loop rows; a.tx lanes take a pair.
template <typename T, int V, bool SEG, bool BASE>
__global__ __launch_bounds__(256) void k_relative_pair(const RelativeArgs a) {
    extern __shared__ float val[];
    const int width = a.tx * V;                                         // floats of a bucket in LDS
    uint8_t* lut = reinterpret_cast<uint8_t*>(val + (size_t)a.buckets * width);
    int64_t at = blockIdx.x;
    const int jb = (int)(at % a.cblocks);
    at /= a.cblocks;
    const int cb = (int)(at % a.hblocks);
    const int64_t rb = at / a.hblocks;
    const int c0 = cb * a.cwidth, nc = min(a.cwidth, a.heads - c0);
#pragma unroll 8
    for (int e = threadIdx.x; e < a.buckets * width; e += 256) {
        const int t = e / width, c = e & (width - 1);                   // (width is a power of two)
        val[e] = table_value(a, t, c0 + min(c, nc - 1));
    }
    lut_to_lds(a, lut, 256);
    __syncthreads();
    const int lane = threadIdx.x & (a.tx - 1), pair = threadIdx.x / a.tx, pairs = 256 / a.tx;
    if (lane * V >= nc) return;
    const int64_t j0 = (int64_t)jb * 4 * pairs + pair;
    int pk[4], sk[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int64_t j = j0 + u * pairs;
        pk[u] = j < a.nk ? a.pos_k[j] : 0;
        sk[u] = SEG && j < a.nk ? a.seg_k[j] : 0;
    }
    const int64_t r0 = rb * a.loop, r1 = min(r0 + a.loop, a.nq);
    const T* base = static_cast<const T*>(a.base.data) + c0 + lane * V;
    T* out = static_cast<T*>(a.out.data) + c0 + lane * V;
    for (int64_t r = r0; r < r1; ++r) {
        const int pq = a.pos_q[r], sq = SEG ? a.seg_q[r] : 0;
        Words<T, V> x[4];
        if constexpr (BASE)
#pragma unroll
            for (int u = 0; u < 4; ++u) x[u].load(base + r * a.base.row + min(j0 + u * pairs, a.nk - 1) * a.heads);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t j = j0 + u * pairs;
            int t = lut[distance_index(pk[u], pq, a.reach)];
            if constexpr (SEG) t = sk[u] == sq ? t : a.buckets - 1;
            Vec<float, V> w;
            w.load(val + t * width + lane * V);
            Vec<T, V> v;
            if constexpr (BASE) v = x[u].values();
#pragma unroll
            for (int i = 0; i < V; ++i) v.f[i] = BASE ? v.f[i] + w.f[i] : w.f[i];
            if (j < a.nk) v.store(out + r * a.out.row + j * a.heads);
        }
    }
}

// Sums by bucket over a tile of pairs.  A wave takes one pair at a time (a lane for V of its channels), so the bucket is
// one for the wave: the sum stays in registers while it does not change, and goes to the wave's own table in LDS
// when it does.  32 pairs are on their way while 32 are added; where their buckets rise or fall, as near the diagonal,
// equal neighbours are added up and the places, all different then, are read, added to and written together.
// Bound by waiting and issue: 66 buckets of 128 channels leave LDS for four waves a compute unit, one a SIMD.  1000 x 1000 bf16
// 90 us in five chains, 93 in one (0.26 GB, 2.8 TB/s; 9 buckets, 16 waves, 83), 500 x 700 fp32 63 us (0.18 GB, 2.8 TB/s).
template <typename T, int V, bool SEG>
__global__ __launch_bounds__(256) void k_relative_pair_backward(const RelativeArgs a) {
    extern __shared__ float val[];
    constexpr int kAhead = 32;
    const int table = a.buckets * 64 * V, own = table + 64 * V;      // (and a place for what is not to be kept)
    uint32_t* touched = reinterpret_cast<uint32_t*>(val + (size_t)a.waves * own);
    uint8_t* lut = reinterpret_cast<uint8_t*>(touched + 8);
    int64_t at = blockIdx.x;
    const int cb = (int)(at % a.hblocks);
    at /= a.hblocks;
    const int64_t tile = at;
    const int64_t r0 = tile / a.cblocks * a.loop, j0 = tile % a.cblocks * a.span;
    const int64_t r1 = min(r0 + a.loop, a.nq), j1 = min(j0 + a.span, a.nk);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, threads = a.waves * 64;
    const int c0 = cb * 64 * V + lane * V;
    const bool live = c0 < a.heads;                    // (V = 2 only where the channels are even)
    const int per_row = (int)((j1 - j0 + kAhead - 1) / kAhead), steps = (int)(r1 - r0) * per_row;
    const T* from = static_cast<const T*>(a.out.data) + (live ? c0 : 0);
    Words<T, V> ahead[kAhead];
    int index = 0;                                     // of pair (lane % kAhead) of the pairs ahead; beyond reach: other segment
    auto load = [&](int g) {
        const int64_t r = r0 + g / per_row, j = j0 + (int64_t)(g % per_row) * kAhead;
        const T* pair = from + r * a.out.row + j * a.heads;
        if (j + kAhead <= j1) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) ahead[u].load(pair + (int64_t)u * a.heads);
        } else {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) ahead[u].load(pair + min((int64_t)u, j1 - 1 - j) * a.heads);
        }
        const int64_t mine = min(j + (lane & (kAhead - 1)), j1 - 1);
        index = distance_index(a.pos_k[mine], a.pos_q[r], a.reach);
        if constexpr (SEG) index = a.seg_k[mine] == a.seg_q[r] ? index : 2 * a.reach + 1;
    };
    if (wave < steps) load(wave);
    lut_to_lds(a, lut, threads);
    if (threadIdx.x == 0) lut[2 * a.reach + 1] = (uint8_t)(a.buckets - 1);
    zero_lds(val, a.waves * own, threads);
    if (threadIdx.x < 8) touched[threadIdx.x] = 0;
    __syncthreads();
    float* acc = val + (size_t)wave * own + lane * V;
    float sum[V];
#pragma unroll
    for (int i = 0; i < V; ++i) sum[i] = 0.f;
    // `sum` belongs to bucket cur; what left the registers before it is on its way to bucket late: the old value has been
    // asked for, and is added to when the next one leaves.
    int cur = -1, late = -1;
    Vec<float, V> old;
    float due[V];
    auto settle = [&]() {
        if (late < 0) return;
#pragma unroll
        for (int i = 0; i < V; ++i) old.f[i] += due[i];
        old.store(acc + late * 64 * V);
        late = -1;
    };
    auto turn_to = [&](int t) {
        if (t == cur) return;
        settle();
        if (cur >= 0) {
            old.load(acc + cur * 64 * V);
#pragma unroll
            for (int i = 0; i < V; ++i) due[i] = sum[i];
            late = cur;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) sum[i] = 0.f;
        cur = t;
    };
    for (int g = wave; g < steps; g += a.waves) {
        const int left = (int)min((int64_t)kAhead, j1 - j0 - (int64_t)(g % per_row) * kAhead);
        Vec<T, V> v[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) v[u] = ahead[u].values();
        const int t = lut[index], first = __builtin_amdgcn_readfirstlane(t);
        if (g + a.waves < steps) load(g + a.waves);
        if (lane < left) atomicOr(touched + t / 32, 1u << (t & 31));
        const int before = __shfl_up(t, 1);
        const uint64_t inner = 0xfffffffe;                         // lanes 1..31
        if (left == kAhead && __ballot(t != first) == 0) {         // one bucket for all of them: a tree
            turn_to(first);
#pragma unroll
            for (int i = 0; i < V; ++i) {
#pragma unroll
                for (int level = 0; level < 5; ++level)
#pragma unroll
                    for (int u = 0; u < 16 >> level; ++u) v[u].f[i] += v[u + (16 >> level)].f[i];
                sum[i] += v[0].f[i];
            }
        } else if (left == kAhead && ((__ballot(t >= before) & inner) == inner || (__ballot(t <= before) & inner) == inner)) {
            turn_to(-1);
            settle();
#pragma unroll
            for (int u0 = 0; u0 < kAhead; u0 += 16) {
                Vec<float, V> x[16];
                int to[16];
#pragma unroll
                for (int u = 0; u < 16; ++u) {
                    const int here = __builtin_amdgcn_readlane(t, u0 + u);
                    const bool last = u == 15 || here != __builtin_amdgcn_readlane(t, (u0 + u + 1) & 31);
                    to[u] = (last ? here : a.buckets) * 64 * V;
                    x[u].load(acc + to[u]);
                    if (!last)
#pragma unroll
                        for (int i = 0; i < V; ++i) v[(u0 + u + 1) & 31].f[i] += v[u0 + u].f[i];
                }
#pragma unroll
                for (int u = 0; u < 16; ++u) {
#pragma unroll
                    for (int i = 0; i < V; ++i) x[u].f[i] += v[u0 + u].f[i];
                    x[u].store(acc + to[u]);
                }
            }
        } else {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (u < left) {
                    turn_to(__builtin_amdgcn_readlane(t, u));
#pragma unroll
                    for (int i = 0; i < V; ++i) sum[i] += v[u].f[i];
                }
            }
        }
    }
    turn_to(-1);
    settle();
    __syncthreads();
    const int64_t slot = tile * a.hblocks + cb;
    float* part = a.part + slot * table;
#pragma unroll 4
    for (int e = threadIdx.x; e < table; e += threads) {
        const int t = e / (64 * V);
        if (!(touched[t / 32] >> (t & 31) & 1)) continue;
        float s = 0.f;
        for (int w = 0; w < a.waves; ++w) s += val[(size_t)w * own + e];
        part[e] = s;
    }
    if (threadIdx.x < 8) a.masks[slot * 8 + threadIdx.x] = touched[threadIdx.x];
}

// dtable from the tiles' sums: a work-group for a bucket and 64 V channels, a wave for every 16th tile.
template <int V>
__global__ __launch_bounds__(1024) void k_relative_pair_join(const RelativeArgs a, int64_t tiles) {
    __shared__ double sums[16][64 * V];
    const int cb = blockIdx.x % a.hblocks, t = blockIdx.x / a.hblocks;
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, table = a.buckets * 64 * V;
    double sum[V];
#pragma unroll
    for (int i = 0; i < V; ++i) sum[i] = 0;
    for (int64_t first = wave; first < tiles; first += 16 * 64) {
        const int64_t mine = first + 16 * lane;
        const bool set = mine < tiles && (a.masks[(mine * a.hblocks + cb) * 8 + t / 32] >> (t & 31) & 1);
        uint64_t left = __ballot(set);
        while (left) {                                 // four tiles at a time
            float x[4][V];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int k = left ? __ffsll((unsigned long long)left) - 1 : 0;
                const float* part = a.part + ((first + 16 * k) * a.hblocks + cb) * table + (t * 64 + lane) * V;
#pragma unroll
                for (int i = 0; i < V; ++i) x[u][i] = left ? part[i] : 0.f;
                left &= left - 1;
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int i = 0; i < V; ++i) sum[i] += x[u][i];
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) sums[wave][lane * V + i] = sum[i];
    __syncthreads();
    for (int e = threadIdx.x; e < 64 * V; e += 1024) {
        double s = 0;
        for (int w = 0; w < 16; ++w) s += sums[w][e];
        const int c = cb * 64 * V + e;
        if (c < a.heads) a.dtable[(int64_t)t * a.heads + c] = (float)s;
    }
}

int pow2_from(int64_t n, int most) {
    int p = 1;
    while (p < most && p < n) p *= 2;
    return p;
}

int64_t up(int64_t n, int64_t d) { return (n + d - 1) / d; }

bool strides_wide(const CrossBias& t, int64_t batch, int64_t heads, int64_t nq) {
    return !t.data || ((reinterpret_cast<uintptr_t>(t.data) & 15) == 0 && (batch == 1 || t.batch % 8 == 0) && (heads == 1 || t.head % 8 == 0) && (nq == 1 || t.row % 8 == 0));
}

bool keys_wide(const RelativeArgs& a) {
    return ((reinterpret_cast<uintptr_t>(a.pos_k) | reinterpret_cast<uintptr_t>(a.seg_k)) & 15) == 0 && ((a.pos_k_batch | a.seg_k_batch) & 3) == 0;
}

size_t lut_bytes(int reach) { return ((size_t)2 * reach + 2 + 15) & ~size_t(15); }

template <typename K>
hipError_t with_lds(K kernel, size_t lds) {
    return lds <= 65536 ? hipSuccess : hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
}

}  // namespace

namespace {
size_t bias_backward_lds(const RelativeArgs& a) { return (size_t)a.waves * (a.buckets + 1) * 256 + lut_bytes(a.reach); }
size_t values_bytes(const RelativeArgs& a) {            // of one head: values_by_distance
    const size_t entries = 2 * (size_t)a.reach + 2;
    return (entries + entries / 8 + 1) * 4;
}
}  // namespace

constexpr int kBaseHeads = 2;      // the most heads at once with a base

int64_t relative_bias_plan(RelativeArgs& a) {
    a.tx = pow2_from(up(a.nk, 8), 16);
    const int rows = 256 / a.tx;
    // Heads at once: without a base eight share an index, with one, two: each head is two streams, and heads are often as far
    // apart as memory channels repeat.  Measured with 16 heads, without a base by two, four and eight at once: bf16, 1300 x
    // 1300 18.6, 17.7 and 17.7 us, 2048 x 3000 51, 44 and 46; fp32 36.3, 36.9 and 36.3, and 111, 126 and 122, where the
    // streams meet as with a base.  With one by one, two and four, 2048 x 3000: bf16 110, 101 and 114 us, fp32 245, 224 and 225.
    a.hb = pow2_from(a.heads, a.base.data ? kBaseHeads : 8);
    while (a.hb > 1 && a.hb * values_bytes(a) > 40960) a.hb /= 2;
    a.cblocks = (int)up(a.nk, 8 * a.tx);
    auto groups = [&]() { return a.batch * up(a.heads, a.hb) * a.cblocks * up(a.nq, rows); };
    while (a.hb > 1 && groups() < 512) a.hb /= 2;
    a.loop = std::min<int64_t>(64, up(groups(), a.base.data ? 1024 : 512));   // (1024 and 512 work-groups, which begin by filling LDS)
    a.hblocks = (int)up(a.heads, a.hb);
    a.rblocks = up(a.nq, rows * a.loop);
    return a.batch * a.hblocks * a.cblocks * a.rblocks;
}

hipError_t launch_relative_bias(int dtype, RelativeArgs a, hipStream_t s) {
    const int64_t groups = relative_bias_plan(a);
    a.wide_keys = keys_wide(a);
    a.wide = strides_wide(a.base, a.batch, a.heads, a.nq) && strides_wide(a.out, a.batch, a.heads, a.nq);
    const size_t lds = values_bytes(a) * a.hb;
    const dim3 grid((unsigned)groups), block(256);
    const bool seg = a.seg_q, base = a.base.data;
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, block, lds, s, a);
        return hipGetLastError();
    };
    auto pick = [&](auto zero, auto heads) {
        using T = decltype(zero);
        constexpr int HB = decltype(heads)::value;
        if constexpr (HB <= kBaseHeads)
            if (base) return seg ? go(k_relative_bias<T, true, true, HB>) : go(k_relative_bias<T, false, true, HB>);
        return seg ? go(k_relative_bias<T, true, false, HB>) : go(k_relative_bias<T, false, false, HB>);
    };
    auto by_heads = [&](auto zero) {
        switch (a.hb) {
            case 1: return pick(zero, std::integral_constant<int, 1>{});
            case 2: return pick(zero, std::integral_constant<int, 2>{});
            case 4: return pick(zero, std::integral_constant<int, 4>{});
            default: return pick(zero, std::integral_constant<int, 8>{});
        }
    };
    return dtype == 1 ? by_heads(bf16_t{}) : by_heads(float{});
}

// Work-groups, and in a how rows and keys lie on their waves: two (one where their columns would outgrow 64 KB).  As many
// as are at once on the compute units, by LDS and at most six on each (registers); rows are split where the keys are too
// few for that, 128 to a wave at least.
int64_t relative_bias_backward_plan(RelativeArgs& a) {
    a.tx = pow2_from(up(a.nk, 8), 8);
    a.waves = a.buckets <= 127 ? 2 : 1;
    const int64_t batch = std::max<int64_t>(1, a.batch), heads = batch * a.heads, keys = std::max<int64_t>(1, up(a.nk, 8 * a.tx));
    const int64_t most = 256 * std::max<int64_t>(1, std::min<int64_t>(6, 163840 / (int64_t)bias_backward_lds(a)));
    a.splits = (int)std::max<int64_t>(1, std::min(most / (heads * up(keys, a.waves)), up(a.nq, 128)));
    a.span = std::max<int64_t>(1, std::min(up(keys, a.waves), up(heads * keys * a.splits, most * a.waves)));
    a.cblocks = (int)up(keys, a.span * a.waves);
    a.loop = std::max<int64_t>(1, std::min(batch, heads * a.cblocks / most));     // small entries, many of them: several to each
    return up(batch, a.loop) * a.heads * a.splits * a.cblocks;
}
namespace {
int64_t bias_slots(const RelativeArgs& a) { return up(a.batch, a.loop) * a.splits * a.cblocks; }
}  // namespace
size_t relative_bias_part_floats(RelativeArgs a) {
    relative_bias_backward_plan(a);
    return bias_slots(a) <= 1 ? 0 : (size_t)bias_slots(a) * a.heads * a.buckets;
}

hipError_t launch_relative_bias_backward(int dtype, RelativeArgs a, hipStream_t s) {
    const int64_t groups = relative_bias_backward_plan(a), n = (int64_t)a.heads * a.buckets;
    if (a.batch == 0 || a.nq == 0 || a.nk == 0) {
        hipLaunchKernelGGL(k_relative_zero, dim3((unsigned)up(n, 256)), dim3(256), 0, s, a.dtable, n);
        return hipGetLastError();
    }
    a.wide_keys = keys_wide(a);
    a.wide = strides_wide(a.out, a.batch, a.heads, a.nq);
    const size_t lds = bias_backward_lds(a);
    const dim3 grid((unsigned)groups), block(a.waves * 64);
    auto go = [&](auto kernel) {
        if (hipError_t e = with_lds(kernel, lds); e != hipSuccess) return e;
        hipLaunchKernelGGL(kernel, grid, block, lds, s, a);
        return hipGetLastError();
    };
    const hipError_t e = dtype == 1 ? a.seg_q ? go(k_relative_bias_backward<bf16_t, true>) : go(k_relative_bias_backward<bf16_t, false>)
                                    : a.seg_q ? go(k_relative_bias_backward<float, true>) : go(k_relative_bias_backward<float, false>);
    if (e != hipSuccess || bias_slots(a) == 1) return e;
    hipLaunchKernelGGL(k_relative_join, dim3((unsigned)up(n, 64)), dim3(1024), 0, s, a, bias_slots(a));
    return hipGetLastError();
}

namespace {
// The largest vector that channels, row strides and pointers allow.
int pair_vector(const RelativeArgs& a) {
    const uintptr_t ptr = reinterpret_cast<uintptr_t>(a.base.data) | reinterpret_cast<uintptr_t>(a.out.data);
    const int64_t bits = a.heads | (a.nq > 1 ? a.out.row | (a.base.data ? a.base.row : 0) : 0);
    return ptr & 15 ? 1 : bits % 8 == 0 ? 8 : bits % 4 == 0 ? 4 : 1;
}
}  // namespace

int64_t relative_pair_plan(RelativeArgs& a, int vector) {
    const int most = vector == 8 ? 16 : vector == 4 ? 32 : 64;          // lanes of a pair: up to 128 channels (64 by single values)
    a.tx = pow2_from(up(a.heads, vector), most);
    a.cwidth = a.tx * vector;
    a.hblocks = (int)up(a.heads, a.cwidth);
    a.cblocks = (int)up(a.nk, 4 * (256 / a.tx));
    const int64_t groups = (int64_t)a.hblocks * a.cblocks * a.nq;
    a.loop = std::min<int64_t>(64, up(groups, 1024));
    a.rblocks = up(a.nq, a.loop);
    return (int64_t)a.hblocks * a.cblocks * a.rblocks;
}
int64_t relative_pair_groups(RelativeArgs a) { return relative_pair_plan(a, pair_vector(a)); }

hipError_t launch_relative_pair(int dtype, RelativeArgs a, hipStream_t s) {
    const int v = pair_vector(a);
    const int64_t groups = relative_pair_plan(a, v);
    const size_t lds = (size_t)a.buckets * a.tx * v * 4 + lut_bytes(a.reach);
    const dim3 grid((unsigned)groups), block(256);
    auto go = [&](auto kernel) {
        if (hipError_t e = with_lds(kernel, lds); e != hipSuccess) return e;
        hipLaunchKernelGGL(kernel, grid, block, lds, s, a);
        return hipGetLastError();
    };
    const bool seg = a.seg_q, base = a.base.data;
    auto pick = [&](auto zero, auto vec) {
        using T = decltype(zero);
        constexpr int V = decltype(vec)::value;
        return seg ? base ? go(k_relative_pair<T, V, true, true>) : go(k_relative_pair<T, V, true, false>)
                   : base ? go(k_relative_pair<T, V, false, true>) : go(k_relative_pair<T, V, false, false>);
    };
    using V8 = std::integral_constant<int, 8>;
    using V4 = std::integral_constant<int, 4>;
    using V1 = std::integral_constant<int, 1>;
    if (dtype == 1) return v == 8 ? pick(bf16_t{}, V8{}) : v == 4 ? pick(bf16_t{}, V4{}) : pick(bf16_t{}, V1{});
    return v == 8 ? pick(float{}, V8{}) : v == 4 ? pick(float{}, V4{}) : pick(float{}, V1{});
}

namespace {
// V channels a lane: 2 where channels, rows and pointer allow it.
int pair_backward_vector(const RelativeArgs& a, int dtype) {
    const int64_t bits = a.heads | (a.nq > 1 ? a.out.row : 0);
    return bits % 2 == 0 && reinterpret_cast<uintptr_t>(a.out.data) % (dtype == 1 ? 4 : 8) == 0 ? 2 : 1;
}
}  // namespace

namespace {
size_t pair_backward_lds(const RelativeArgs& a, int vector) { return (size_t)a.waves * (a.buckets + 1) * 256 * vector + 32 + lut_bytes(a.reach); }
}  // namespace

// Tiles, as many as LDS lets the compute units have at once (one each for 66 buckets; one more than fit would take a
// second round): whole rows, so that each has its share of the diagonal and reads long pieces (1000 x 1000 x 128 bf16:
// 90 us in five chains, 93 in one; tiles of 64 columns 138 and 112; 500 x 700 x 128 fp32 63 and 78), and parts of a row where
// there are fewer rows than tiles.
int64_t relative_pair_backward_plan(RelativeArgs& a, int vector) {
    a.hblocks = (int)up(a.heads, 64 * vector);
    a.waves = std::min(4, std::max(1, 143360 / ((a.buckets + 1) * 256 * vector)));
    const int64_t at_once = 256 * std::min<int64_t>(4, std::max<int64_t>(1, 163840 / (int64_t)pair_backward_lds(a, vector)));
    const int64_t tiles = std::max<int64_t>(1, at_once / a.hblocks);
    a.loop = up(a.nq, std::min(a.nq, tiles));
    a.rblocks = up(a.nq, a.loop);
    a.span = up(a.nk, std::max<int64_t>(1, std::min(up(a.nk, 64), tiles / a.rblocks)));
    a.cblocks = (int)up(a.nk, a.span);
    return a.cblocks * a.rblocks;
}
// Floats of the partial sums: for V = 2 and V = 1, whichever is more (the vector follows from the pointer).
size_t relative_pair_part_floats(RelativeArgs a) {
    size_t most = 0;
    for (int v : {1, 2}) {
        const int64_t tiles = relative_pair_backward_plan(a, v);
        most = std::max(most, (size_t)tiles * a.hblocks * ((size_t)a.buckets * 64 * v + 8));
    }
    return most;
}

hipError_t launch_relative_pair_backward(int dtype, RelativeArgs a, hipStream_t s) {
    const int64_t n = (int64_t)a.heads * a.buckets;
    if (a.nq == 0 || a.nk == 0) {
        hipLaunchKernelGGL(k_relative_zero, dim3((unsigned)up(n, 256)), dim3(256), 0, s, a.dtable, n);
        return hipGetLastError();
    }
    const int v = pair_backward_vector(a, dtype);
    const int64_t tiles = relative_pair_backward_plan(a, v);
    a.masks = reinterpret_cast<uint32_t*>(a.part + (size_t)tiles * a.hblocks * a.buckets * 64 * v);
    const size_t lds = pair_backward_lds(a, v);
    const dim3 grid((unsigned)(tiles * a.hblocks)), block(a.waves * 64);
    auto go = [&](auto kernel) {
        if (hipError_t e = with_lds(kernel, lds); e != hipSuccess) return e;
        hipLaunchKernelGGL(kernel, grid, block, lds, s, a);
        return hipGetLastError();
    };
    auto pick = [&](auto zero) {
        using T = decltype(zero);
        return v == 2 ? a.seg_q ? go(k_relative_pair_backward<T, 2, true>) : go(k_relative_pair_backward<T, 2, false>)
                      : a.seg_q ? go(k_relative_pair_backward<T, 1, true>) : go(k_relative_pair_backward<T, 1, false>);
    };
    const hipError_t e = dtype == 1 ? pick(bf16_t{}) : pick(float{});
    if (e != hipSuccess) return e;
    const dim3 join((unsigned)(a.buckets * a.hblocks));
    if (v == 2) hipLaunchKernelGGL(k_relative_pair_join<2>, join, dim3(1024), 0, s, a, tiles);
    else hipLaunchKernelGGL(k_relative_pair_join<1>, join, dim3(1024), 0, s, a, tiles);
    return hipGetLastError();
}

}  // namespace trimul
